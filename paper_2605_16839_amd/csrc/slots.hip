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
// workgroup waits for another.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kSlotThreads = 256;
constexpr int kSlotWaves = kSlotThreads / kWave;

// Inclusive sums over the workgroup's threads of two values.
struct Sums {
  long long a, b;
};
__device__ __forceinline__ Sums block_inclusive_sums(Sums v, Sums* part) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long ta = __shfl_up(v.a, o, kWave), tb = __shfl_up(v.b, o, kWave);
    if (lane >= o) v.a += ta, v.b += tb;
  }
  __syncthreads();   // the previous use of part
  if (lane == kWave - 1) part[wv] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSlotWaves; ++w)
    if (w < wv) v.a += part[w].a, v.b += part[w].b;
  return v;
}

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
  int B, Hkv, max_kv_blocks, num_pages, rows_per_wg;
};

__global__ __launch_bounds__(kSlotThreads) void assign_slots_kernel(const SlotArgs a) {
  __shared__ Sums s_part[kSlotWaves];
  __shared__ long long s_row[kSlotThreads];     // first token row of a request
  __shared__ long long s_taken[kSlotThreads];   // pages taken before it
  __shared__ int s_old[kSlotThreads];           // its cached tokens, -1: refused
  __shared__ Sums s_end;                        // both sums after the last request of the round
  __shared__ long long s_given;
  const SlotLaunch& l = a.l;
  const int tid = threadIdx.x, H = a.Hkv;
  const bool first = blockIdx.x == 0;
  const long long T = l.num_tokens;
  long long lo = (long long)blockIdx.x * a.rows_per_wg;
  long long hi = lo + a.rows_per_wg;
  lo = lo < T ? lo : T;
  hi = hi < T ? hi : T;
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
    // the rows are summed first: a request past the last row needs no pages
    const Sums r = block_inclusive_sums({rows, 0}, s_part);
    fits = fits && row0 + r.a <= T;
    const long long need = fits ? (blocks_of(old + add) - blocks_of(old)) * H : 0;
    const Sums n = block_inclusive_sums({need, 0}, s_part);
    const long long taken = taken0 + n.a;
    fits = fits && (need == 0 || taken <= count);
    s_row[tid] = row0 + r.a - rows;
    s_taken[tid] = taken - need;
    s_old[tid] = fits ? (int)old : -1;
    if (tid == kSlotThreads - 1) s_end = {row0 + r.a, taken};
    if (first && b < a.B) {
      const long long end = row0 + r.a;
      l.token_indptr[b + 1] = (int)(end < T ? end : T);
      l.granted[b] = fits ? (int)add : 0;
      l.seq_len_out[b] = (int)(old + (fits ? add : 0));
      if (fits && need > 0)
        atomicAdd(reinterpret_cast<unsigned long long*>(&s_given), (unsigned long long)need);
    }
    __syncthreads();
    const int n_here = a.B - b0 < kSlotThreads ? a.B - b0 : kSlotThreads;
    const long long from = lo > row0 ? lo : row0, to = hi < s_end.a ? hi : s_end.a;
    for (long long x = from * H + tid; x < to * H; x += kSlotThreads) {
      const long long t = x / H;
      const int h = (int)(x - t * H);
      const int i = last_at_most(s_row, n_here, t);
      const int had = s_old[i];
      long long slot = -1;
      int pos = 0;
      if (had >= 0) {
        pos = (int)(had + (t - s_row[i]));
        const int j = pos / kPage, fresh = j - (int)blocks_of(had);
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
      l.slot_map[x] = slot;
      if (h == 0) l.positions[t] = pos;
    }
    row0 = s_end.a;
    taken0 = s_end.b;
    __syncthreads();
    if (!first && row0 >= hi) break;
  }
  // padding rows behind the last request
  const long long pad = lo > row0 ? lo : row0;
  for (long long x = pad * H + tid; x < hi * H; x += kSlotThreads) {
    l.slot_map[x] = -1;
    if (x % H == 0) l.positions[x / H] = 0;
  }
  if (first && tid == 0) l.free_count_out[0] = count - (int)s_given;
}

__global__ __launch_bounds__(kSlotThreads) void release_pages_kernel(const SlotArgs a) {
  __shared__ Sums s_part[kSlotWaves];
  __shared__ long long s_start[kSlotThreads];   // pages released before the request
  __shared__ int s_kept[kSlotThreads];          // 1: does not fit
  __shared__ long long s_end, s_given;
  const SlotLaunch& l = a.l;
  const int tid = threadIdx.x, H = a.Hkv;
  const bool first = blockIdx.x == 0;
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
    const Sums s = block_inclusive_sums({need, 0}, s_part);
    const long long after = sum0 + s.a;
    const bool fits = need == 0 || count + after <= l.free_capacity;
    s_start[tid] = after - need;
    s_kept[tid] = !fits;
    if (tid == kSlotThreads - 1) s_end = after;
    if (first && b < a.B) {
      l.seq_len_out[b] = ends && fits ? 0 : old;
      if (fits && need > 0)
        atomicAdd(reinterpret_cast<unsigned long long*>(&s_given), (unsigned long long)need);
    }
    __syncthreads();
    const int n_here = a.B - b0 < kSlotThreads ? a.B - b0 : kSlotThreads;
    const long long end = s_end;
    for (long long x = sum0 + (long long)blockIdx.x * kSlotThreads + tid; x < end;
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

hipError_t launch_assign_slots(const CacheDims& d, const SlotLaunch& l, hipStream_t st) {
  SlotArgs a{l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, l.num_tokens};
  assign_slots_kernel<<<1, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_release_pages(const CacheDims& d, const SlotLaunch& l, hipStream_t st) {
  SlotArgs a{l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, 0};
  release_pages_kernel<<<1, kSlotThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
