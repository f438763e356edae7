// Pages and slots of a serving step, from request lengths on the device: the
// free pages are a stack, a request's needs follow from its lengths, and two
// prefix sums over the requests (token rows, pages) place everything.
//
//   need_b  = (ceil((s_b + n_b) / 64) - ceil(s_b / 64)) * Hkv
//   row_b   = sum_{i<b} n_i            (the request's first token row)
//   taken_b = sum_{i<=b} need_i        (granted while taken_b <= free pages)
//   page of needed (block, head) x of request b = free_pages[count - 1 - (taken_b - need_b + x)]
//
// Every workgroup makes the sums itself, kSlotThreads requests at a time, and
// writes the token rows of its own range, so one launch does it and no
// workgroup waits for another.  What bounds a call is latency: the lengths, the
// sums, and the ids that hang on them, one after the other.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kSlotThreads = 1024;
constexpr int kSlotWaves = kSlotThreads / kWave;
constexpr int kSlotGroups = 256;
constexpr int kReleaseGroups = 64;
constexpr int kAloneRounds = 4;   // of one workgroup's threads, where it works alone

// The value of a lane before this one in 64-bit halves (0 where there is none).
template <int CTRL, int ROWS>
__device__ __forceinline__ long long dpp64(long long v) {
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return (long long)(((unsigned long long)(unsigned)hi << 32) | lo);
}
__device__ __forceinline__ long long wave_inclusive_sum(long long v) {
  v += dpp64<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8: within 16 lanes
  v += dpp64<0x112, 0xf>(v);
  v += dpp64<0x114, 0xf>(v);
  v += dpp64<0x118, 0xf>(v);
  v += dpp64<0x142, 0xa>(v);   // lane 15 to the next 16, lane 47 to the last
  v += dpp64<0x143, 0xc>(v);   // lane 31 to the upper half
  return v;
}

// Inclusive sums over the workgroup's threads of two values, and their totals.
struct Sums {
  long long a, b;
};
__device__ __forceinline__ Sums block_inclusive_sums(Sums v, Sums* part, Sums* all) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  v.a = wave_inclusive_sum(v.a);
  v.b = wave_inclusive_sum(v.b);
  if (lane == kWave - 1) part[wv] = v;
  __syncthreads();
  // the waves' totals: lane l of every 16 holds wave l's
  const Sums p = part[lane & (kSlotWaves - 1)];
  Sums s = p;
  s.a += dpp64<0x111, 0xf>(s.a), s.b += dpp64<0x111, 0xf>(s.b);
  s.a += dpp64<0x112, 0xf>(s.a), s.b += dpp64<0x112, 0xf>(s.b);
  s.a += dpp64<0x114, 0xf>(s.a), s.b += dpp64<0x114, 0xf>(s.b);
  s.a += dpp64<0x118, 0xf>(s.a), s.b += dpp64<0x118, 0xf>(s.b);
  auto of_lane = [](long long x, int l) {
    const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)x, l);
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32) | lo);
  };
  const int w = __builtin_amdgcn_readfirstlane(wv);
  v.a += of_lane(s.a - p.a, w), v.b += of_lane(s.b - p.b, w);
  *all = {of_lane(s.a, kSlotWaves - 1), of_lane(s.b, kSlotWaves - 1)};
  return v;
}
static_assert(kSlotWaves == 16, "one row of 16 lanes sums the waves");

__device__ __forceinline__ long long blocks_of(long long tokens) {
  return (tokens + kPage - 1) / kPage;
}

// Last index i in [0, n) with start[i] <= x (start ascending, start[0] <= x).
__device__ __forceinline__ int last_at_most(const long long* start, int n, long long x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct SlotArgs {
  SlotLaunch l;
  int B, Hkv, max_kv_blocks, num_pages;
  int rows_at_once;   // token rows that a workgroup's threads write together
  int rows_per_wg;    // a multiple of it
  int what;           // kRows, kState: what this launch writes
};
constexpr int kRows = 1;    // token rows and page-table entries, or the free list
constexpr int kState = 2;   // everything by request

__global__ __launch_bounds__(kSlotThreads) void assign_slots_kernel(const SlotArgs a) {
  __shared__ Sums s_part[kSlotWaves];
  __shared__ long long s_row[kSlotThreads];     // first token row of a request
  __shared__ long long s_taken[kSlotThreads];   // pages taken before it
  __shared__ int s_old[kSlotThreads];           // its cached tokens, -1: refused
  __shared__ long long s_given;
  const SlotLaunch& l = a.l;
  const int tid = threadIdx.x, H = a.Hkv;
  const bool first = blockIdx.x == 0 && (a.what & kState);
  const long long T = l.num_tokens;
  long long lo = (long long)blockIdx.x * a.rows_per_wg;
  long long hi = a.what & kRows ? lo + a.rows_per_wg : lo;
  lo = lo < T ? lo : T;
  hi = hi < T ? hi : T;
  // this thread's row among those written together, and its first head
  const int r0 = a.rows_at_once > 1 ? tid / H : 0, h0 = a.rows_at_once > 1 ? tid - r0 * H : tid;
  const bool writes = r0 < a.rows_at_once;
  int count = l.free_count[0];
  count = count < 0 ? 0 : (count > l.free_capacity ? l.free_capacity : count);
  if (tid == 0) s_given = 0;
  if (first && tid == 0) l.token_indptr[0] = 0;

  long long row0 = 0, taken0 = 0;   // sums before this round's requests
  for (int b0 = 0; b0 < a.B; b0 += kSlotThreads) {
    const int b = b0 + tid;
    long long old = 0, add = 0;
    if (b < a.B) old = l.seq_len[b], add = l.step[b];
    const long long rows = add > 0 ? add : 0;
    bool fits = old >= 0 && add >= 0 && old + add <= (long long)a.max_kv_blocks * kPage;
    // what a request past the last row needs may be summed: all that follow
    // it and need pages are past the last row too
    const long long need = fits ? (blocks_of(old + add) - blocks_of(old)) * H : 0;
    Sums all;
    const Sums s = block_inclusive_sums({rows, need}, s_part, &all);
    const long long end = row0 + s.a, taken = taken0 + s.b;
    fits = fits && end <= T && (need == 0 || taken <= count);
    s_row[tid] = end - rows;
    s_taken[tid] = taken - need;
    s_old[tid] = fits ? (int)old : -1;
    if (first && b < a.B) {
      l.token_indptr[b + 1] = (int)(end < T ? end : T);
      l.granted[b] = fits ? (int)add : 0;
      l.seq_len_out[b] = (int)(old + (fits ? add : 0));
      if (fits && need > 0)
        atomicAdd(reinterpret_cast<unsigned long long*>(&s_given), (unsigned long long)need);
    }
    __syncthreads();
    const int n_here = a.B - b0 < kSlotThreads ? a.B - b0 : kSlotThreads;
    const long long row1 = row0 + all.a;
    const long long from = lo > row0 ? lo : row0, to = hi < row1 ? hi : row1;
    for (long long t = from + r0; writes && t < to; t += a.rows_at_once) {
      const int i = last_at_most(s_row, n_here, t);
      const int had = s_old[i];
      const int pos = had >= 0 ? (int)(had + (t - s_row[i])) : 0;
      const int j = pos / kPage, fresh = j - (int)blocks_of(had);
      for (int h = h0; h < H; h += kSlotThreads) {
        long long slot = -1;
        if (had >= 0) {
          int32_t* entry = l.page_table + ((long long)(b0 + i) * H + h) * a.max_kv_blocks + j;
          int page;
          if (fresh >= 0) {
            page = l.free_pages[count - 1 - (s_taken[i] + (long long)fresh * H + h)];
            if (pos % kPage == 0) *entry = page;
          } else {
            page = *entry;
          }
          if (page >= 0 && page < a.num_pages) slot = (long long)page * kPage + pos % kPage;
        }
        l.slot_map[t * H + h] = slot;
        if (h == 0) l.positions[t] = pos;
      }
    }
    row0 = row1;
    taken0 += all.b;
    if (!first && row0 >= hi) break;
    __syncthreads();
  }
  // padding rows behind the last request
  const long long pad = lo > row0 ? lo : row0;
  for (long long t = pad + r0; writes && t < hi; t += a.rows_at_once)
    for (int h = h0; h < H; h += kSlotThreads) {
      l.slot_map[t * H + h] = -1;
      if (h == 0) l.positions[t] = 0;
    }
  if (first && tid == 0) l.free_count_out[0] = count - (int)s_given;
}

__global__ __launch_bounds__(kSlotThreads) void release_pages_kernel(const SlotArgs a) {
  __shared__ Sums s_part[kSlotWaves];
  __shared__ long long s_start[kSlotThreads];   // pages released before the request
  __shared__ int s_kept[kSlotThreads];          // 1: does not fit
  __shared__ long long s_given;
  const SlotLaunch& l = a.l;
  const int tid = threadIdx.x, H = a.Hkv;
  const bool first = blockIdx.x == 0 && (a.what & kState);
  int count = l.free_count[0];
  count = count < 0 ? 0 : (count > l.free_capacity ? l.free_capacity : count);
  if (tid == 0) s_given = 0;
  long long sum0 = 0;
  for (int b0 = 0; b0 < a.B; b0 += kSlotThreads) {
    const int b = b0 + tid;
    int old = 0;
    bool ends = false;
    if (b < a.B) old = l.seq_len[b], ends = l.step[b] != 0;
    ends = ends && old >= 0 && old <= a.max_kv_blocks * kPage;
    const long long need = ends ? blocks_of(old) * H : 0;
    Sums all;
    const long long after = sum0 + block_inclusive_sums({need, 0}, s_part, &all).a;
    const bool fits = need == 0 || count + after <= l.free_capacity;
    s_start[tid] = after - need;
    s_kept[tid] = !fits;
    if (first && b < a.B) {
      l.seq_len_out[b] = ends && fits ? 0 : old;
      if (fits && need > 0)
        atomicAdd(reinterpret_cast<unsigned long long*>(&s_given), (unsigned long long)need);
    }
    __syncthreads();
    const int n_here = a.B - b0 < kSlotThreads ? a.B - b0 : kSlotThreads;
    const long long end = sum0 + all.a, stop = a.what & kRows ? end : sum0;
    for (long long x = sum0 + (long long)blockIdx.x * kSlotThreads + tid; x < stop;
         x += (long long)gridDim.x * kSlotThreads) {
      const int i = last_at_most(s_start, n_here, x);
      if (s_kept[i]) continue;
      const int u = (int)(x - s_start[i]), j = u / H, h = u - j * H;
      l.free_pages[count + x] = l.page_table[((long long)(b0 + i) * H + h) * a.max_kv_blocks + j];
    }
    sum0 = end;
    __syncthreads();
  }
  if (first && tid == 0) l.free_count_out[0] = count + (int)s_given;
}

}  // namespace

// As many workgroups as write their rows in one go (8256 rows of 8 heads: 71 us with
// one, 4.7 with 65).  In place, no workgroup may write a length that another has yet
// to read: one does it all where it has little to write (256 rows of 8 heads: 5.4
// us, and 4.8 out of place), else a second launch writes what is known by request.
hipError_t launch_assign_slots(const CacheDims& d, const SlotLaunch& l, hipStream_t st) {
  SlotArgs a{l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, 0, 0, kRows | kState};
  a.rows_at_once = d.Hkv < kSlotThreads ? kSlotThreads / d.Hkv : 1;
  const bool in_place = l.seq_len_out == l.seq_len || l.free_count_out == l.free_count;
  const long long rounds = ((long long)l.num_tokens + a.rows_at_once - 1) / a.rows_at_once;
  const bool alone = in_place && rounds <= kAloneRounds;
  // at most kSlotGroups, so that few workgroups repeat the sums
  const long long each = alone ? rounds : (rounds + kSlotGroups - 1) / kSlotGroups;
  const long long per_wg = (each > 0 ? each : 1) * a.rows_at_once;
  a.rows_per_wg = (int)(per_wg < INT32_MAX ? per_wg : INT32_MAX);
  const int grid = alone || rounds == 0 ? 1 : (int)((rounds + each - 1) / each);
  if (in_place && !alone) a.what = kRows;
  assign_slots_kernel<<<grid, kSlotThreads, 0, st>>>(a);
  if (a.what != kRows) return hipGetLastError();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.what = kState;
  assign_slots_kernel<<<1, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

// 64 requests of 512 blocks and 8 heads: 213 us with one workgroup, 17.9 with 16, 8.0
// with 64; 9 of 256 requests of 40 blocks: 5.6, 3.8 and 3.8.  In place as above.
hipError_t launch_release_pages(const CacheDims& d, const SlotLaunch& l, hipStream_t st) {
  SlotArgs a{l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, 0, 0, kRows | kState};
  const bool in_place = l.seq_len_out == l.seq_len || l.free_count_out == l.free_count;
  const bool alone = (long long)d.B * d.Hkv * d.max_kv_blocks <= kAloneRounds * kSlotThreads;
  if (in_place && !alone) a.what = kRows;
  release_pages_kernel<<<alone ? 1 : kReleaseGroups, kSlotThreads, 0, st>>>(a);
  if (a.what != kRows) return hipGetLastError();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.what = kState;
  release_pages_kernel<<<1, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
