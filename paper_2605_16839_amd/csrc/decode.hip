// Attention of one new token per request over its paged cache: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// in one pass over the keys with the running maximum m and sum.
//
// What bounds it: every K and V page is read once and used for the few query
// heads of its KV head, 2 flops per byte and head, so HBM does; with little to read,
// the latency of length, page id, page and joined pieces, one after the other.  96
// requests of 4K to 32K tokens (32/8 heads, D = 128, 5.6 GB): 825 us, 6.8 TB/s,
// where a bare reader of such pages in such shares takes 810.  Everything below serves an even
// stream of page loads:
//   * the requests' lengths are on the GPU only and may be as different as they
//     like, so the pages of all (request, KV head) rows are laid end to end and
//     cut in equal shares, one per workgroup and within it one per wave; every
//     wave finds its share from a prefix sum over the lengths;
//   * a wave has its own rows and pages: it asks for a whole page, 16 loads of
//     1 KB (D = 128), takes it through its 8 KB of LDS half by half, and asks for
//     the next, K, V, K, .., while it computes: 128 KB of a CU are on their way.
//     Across a row's end too: the next row's ids are there before;
//   * S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_16x16x32_bf16, the heads of
//     the KV head being the 16 columns (more than 16 heads: tiles of 16 that read the
//     pages each).  key_of gives a lane 8 consecutive keys of each 32-key step,
//     as the P^T fragment wants them; token-major V is read from LDS transposed;
//   * weights count with 16 bits: bf16(p), and the part of p that it loses as a second
//     bf16 (p - bf16(p)).  Up to 8 heads leave half of the columns free: they hold
//     the same heads again, and carry the second part at no cost.  With 9 to 16 heads it takes
//     a second MFMA on the same V fragment, into sums of its own (454 MB for 16 heads, D =
//     128: 88.7 us, 85.1 without; transposed V 85.2 and 84.8);
//   * a row that lies inside one wave's share is written at once; pieces of
//     a workgroup's waves are joined in its LDS, and rows that several workgroups
//     share by the last of them (join_row), or by a second launch where few rows may
//     be in many pieces (decode_join_kernel).  Pieces are taken in page order, so
//     the result does not depend on who is last.
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kWaves = 8;                   // per workgroup
constexpr int kThreads = kWaves * kWave;
constexpr int kGroups = 256;                // one workgroup per CU
constexpr int kFewRows = 8;                 // so many rows at most are joined by a launch of its own
constexpr int kManyPieces = 64;             // .. and if a row may have more than so many pages
constexpr int kShortRow = 4;                // pages
constexpr int kTileHeads = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeArgs {
  DecodeLaunch l;
  int B, Hq, Hkv, G, HT, items, per_item, max_kv_blocks, num_pages;
  float scale_log2;
  // pieces that a workgroup leaves to others: [0] of the row that its share
  // starts in the middle of, [1] of the row that goes on after its share
  float* part_o;                    // [kGroups][2][16][D]
  float* part_ml;                   // [kGroups][2][16][2]: maximum (log2 units) and sum
  unsigned long long* arrived;      // [kGroups]: pieces there are of the row that starts in a share
  unsigned long long piece;         // what a piece counts, see last_of
  bool join_later;                  // decode_join_kernel joins the rows
};

template <typename T>
__device__ __forceinline__ T uniform(T v) {
  static_assert(sizeof(T) == 4, "");
  return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}
__device__ __forceinline__ long long uniform64(long long v) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((int)(unsigned)v);
  const int hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (long long)(((unsigned long long)(unsigned)hi << 32) | lo);
}

__device__ __forceinline__ float max2(float a, float b) {
  return __builtin_elementwise_maximum(a, b);   // a NaN stays
}
// Over the 4 lane groups that hold the same column.
__device__ __forceinline__ float groups_max(float x) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(max2(__uint_as_float(r[0]), __uint_as_float(r[1])));
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The value of the lane 8 columns on.
__device__ __forceinline__ float other_half(float x) {
  return __uint_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128 /* row_ror:8 */, 0xf, 0xf, true));
}

// 2^x, and the maxima in log2 units: exp2 of -inf is 0.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Pages of a workgroup's share at least.  A CU draws some 30 GB/s, so few pages go to
// many: 2 to each for 1024 tokens of 8 KV heads take 10.2 us, 4 take 11.8 and 8 14.5 (1
// takes 9.8, but 16K tokens of one KV head then 16.1 instead of 12.4: pieces to join).
// One page each where 128 or fewer are there: 700 tokens of one KV head take 8.4 us, 9.0
// with two.  Rows of up to kShortRow pages on average stay whole, as a join costs
// more than their other pages: 128 tokens of 8 KV heads take 7.9 us so, 9.7 with a page
// each; rows of 8 pages take 11.1 whole, 9.8 cut.
__device__ __forceinline__ int least_pages(const DecodeArgs& a, long long total) {
  if (total >= kGroups * kShortRow) return 1;   // every share has more
  const int pages = (int)total;
  const long long rows = (long long)a.items * a.per_item;
  if (pages <= rows) return 1;
  if (pages <= rows * kShortRow) return (pages + (int)rows - 1) / (int)rows;
  return pages <= kGroups / 2 ? 1 : 2;
}

// First page of share w when `total` pages are dealt, and the share of page u.
__device__ __forceinline__ long long share_start(long long total, int least, int w) {
  if (total >= (long long)kGroups * least) return (total * w) / kGroups;
  const long long s = (long long)w * least;
  return s < total ? s : total;
}
// Below kGroups also for a page that is none of `total` (lengths changed under the kernel).
__device__ __forceinline__ int share_of(long long total, int least, long long u) {
  int w;
  if (total < (long long)kGroups * least) {
    w = (int)u / least;
  } else {
    w = (int)((float)u / (float)total * kGroups);   // off by one at most
    if (w > 0 && share_start(total, least, w) > u) --w;
    else if (share_start(total, least, w + 1) <= u) ++w;
  }
  return w < 0 ? 0 : (w < kGroups - 1 ? w : kGroups - 1);
}

// Sum over the lanes up to this one.
__device__ __forceinline__ unsigned lanes_sum(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);   // across rows of 16
  v += __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
  return v;
}

// Pages of an item: a request's blocks (every KV head and head tile reads as
// many), or a table row's entries.  Bounds that no table has count as none.
__device__ __forceinline__ int request_len(const DecodeArgs& a, int b) {
  const int len = a.l.kv_len[b], most = a.max_kv_blocks * kPage;
  return len < 0 ? 0 : (len < most ? len : most);
}
__device__ __forceinline__ int item_pages(const DecodeArgs& a, int i) {
  if (!a.l.kv_indptr) return blocks_for(request_len(a, i));
  const int at = a.l.kv_indptr[i], end = a.l.kv_indptr[i + 1];
  const long long cap = (long long)a.items * a.max_kv_blocks;
  const long long n = (long long)end - at;
  return at < 0 || n < 0 || n > a.max_kv_blocks || end > cap ? 0 : (int)n;
}

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// Key that row r of 16-key tile kt of a page stands for: lane group g, which the
// 16x16 result gives rows 4g .. 4g+3, then holds keys 32p + 8g .. 32p + 8g + 7
// of the 32-key step p (tiles 2p, 2p + 1).
constexpr int key_of(int kt, int r) {
  return 32 * (kt >> 1) + 8 * (r >> 2) + 4 * (kt & 1) + (r & 3);
}
// Half a page in LDS: 32 keys of K or token-major V (rows of D), D / 2 rows of a
// transposed V page (64 keys each).  16-byte chunk where chunk c of row r lies, so
// that operand reads meet no bank twice:
//   K: 16 lanes read 16 bytes each, of rows that differ in bits 0, 1, 3 and 4;
//   token-major V: 32 lanes of a transpose read cover rows {0..3, 8..11} (+
//     multiples) x 32 bytes, so bits 0, 1 and 3 pick the 32-byte pair;
//   transposed V: 16 lanes read 16 bytes each, of 16 rows in a row.
// Where rows are 128 bytes, two share the 256 bytes of all banks, by bit 0.
enum Half { kHalfK, kHalfV, kHalfVT };
template <int D, Half H>
__device__ __forceinline__ int swizzle(int r, int c) {
  if (H == kHalfVT) return c ^ ((r >> 1) & 7);
  if (H == kHalfK)
    return D == 128 ? (c ^ ((r & 3) | (((r >> 3) & 3) << 2)))
                    : (c ^ (((r >> 1) & 1) | (((r >> 3) & 3) << 1)));
  return D == 128 ? (c ^ (((r & 3) | (((r >> 3) & 1) << 2)) << 1))
                  : (c ^ ((((r >> 1) & 1) | (((r >> 3) & 1) << 1)) << 1));
}

// What workgroups hand to each other goes past the XCD's L2, which the others do
// not see, as agent-scope atomic accesses of 8 bytes: fences would write back and
// invalidate the whole L2 under the workgroups that still stream (one 128K
// request: 139 us with them).
__device__ __forceinline__ void put2(float* p, float x, float y) {
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p),
                     (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
  const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p),
                                                 __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}

// Counts a piece of a row in; true for the last of n.  A counter is 0 between launches,
// and each piece adds `piece`, a number of this launch with 1 in the low 16 bits: k pieces
// are k * piece, which no number of pieces of another launch is (replays of one graph share
// theirs).  A workspace may hold
// anything at first, the counts of an earlier launch too whose pieces never came together:
// who finds a value that is no count of this launch makes it one, with a swap that only
// one of those who find it can win, and counts in if it is another.
constexpr unsigned long long kLaunchTop = 0xa7ull << 40;   // above the 40 bits of a launch's number
__device__ __forceinline__ bool last_of(unsigned long long* counter, unsigned long long piece, int n) {
  const unsigned long long others = (unsigned long long)(n - 1) * piece;   // while the add is on its way
  auto counts = [&](unsigned long long v) { return (int)(v & 0xffff) < n && v == (v & 0xffff) * piece; };
  unsigned long long was =
      __hip_atomic_fetch_add(counter, piece, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  while (__builtin_expect(was != others && !counts(was), 0)) {
    unsigned long long now = __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!counts(now)) {
      if (__hip_atomic_compare_exchange_strong(counter, &now, piece, __ATOMIC_RELAXED,
                                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
        was = 0;
    } else {
      was = __hip_atomic_fetch_add(counter, piece, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (was != others) return false;
  __hip_atomic_store(counter, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// Joins the row whose first piece is workgroup w0's and whose last is w1's.
struct JoinSpace {   // in LDS
  float4 sums[kThreads];
  float weight[kGroups][kTileHeads];
  float part[2][kWaves][kTileHeads];
};
template <int D>
__device__ __forceinline__ void join_row(const DecodeArgs& a, int w0, int w1, long long row, int heads,
                                         JoinSpace& s) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, col = tid & 15;
  auto slot_of = [&](int e) { return 2 * e + (e == w0 ? 1 : 0); };
  const int pieces = w1 - w0 + 1;
  // a thread takes one head's maximum and sum of every 32nd piece, and one of the
  // n float4 of every lots-th piece
  constexpr int kEach = (kGroups * kTileHeads + kThreads - 1) / kThreads;
  float2 ml[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int e = (kThreads / kTileHeads) * k + tid / kTileHeads;
    ml[k] = make_float2(-INFINITY, 0.f);
    if (e < pieces) ml[k] = get2(a.part_ml + 2 * (slot_of(w0 + e) * kTileHeads + col));
  }
  const int n = heads * (D / 4), lots = kThreads / n, lot = tid / n, at = tid - lot * n;
  auto piece = [&](int e) {
    const float* const from = a.part_o + (long long)slot_of(w0 + e) * (kTileHeads * D) + 4 * at;
    const float2 x = get2(from), y = get2(from + 2);
    return make_float4(x.x, x.y, y.x, y.y);
  };
  constexpr int kAhead = 8;
  float4 x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int e = lot + lots * k;
    x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (lot < lots && e < pieces) x[k] = piece(e);
  }
  float top = ml[0].x;
#pragma unroll
  for (int k = 1; k < kEach; ++k) top = max2(top, ml[k].x);
  top = groups_max(top);
  if (lane < kTileHeads) s.part[0][wv][col] = top;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kWaves; ++v) top = max2(top, s.part[0][v][col]);
  const float base = top == -INFINITY ? 0.f : top;
  float all = 0.f;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int e = (kThreads / kTileHeads) * k + tid / kTileHeads;
    const float c = fast_exp2(ml[k].x - base);
    if (e < pieces) s.weight[e][col] = c;
    all += c * ml[k].y;
  }
  all = groups_sum(all);
  if (lane < kTileHeads) s.part[1][wv][col] = all;
  __syncthreads();
  if (tid < heads && a.l.lse) {
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) sum += s.part[1][v][col];
    a.l.lse[row + col] = sum > 0.f ? (top + __log2f(sum)) * kLn2 : -INFINITY;
  }
  const int head = at / (D / 4);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](int e, const float4& y) {
    const float c = s.weight[e][head];
    acc.x += c * y.x, acc.y += c * y.y, acc.z += c * y.z, acc.w += c * y.w;
  };
  if (lot < lots) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (lot + lots * k < pieces) add(lot + lots * k, x[k]);
#pragma unroll 8
    for (int e = lot + lots * kAhead; e < pieces; e += lots) add(e, piece(e));
    s.sums[tid] = acc;
  }
  __syncthreads();
  if (tid >= n) return;
  for (int e = 1; e < lots; ++e) {
    const float4 y = s.sums[e * n + tid];
    acc.x += y.x, acc.y += y.y, acc.z += y.z, acc.w += y.w;
  }
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) sum += s.part[1][v][head];
  const float inv = sum == 0.f ? 0.f : 1.f / sum;   // sum is NaN after a score of NaN or +inf
  reinterpret_cast<u32x2*>(a.l.out + row * D)[tid] =
      u32x2{pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)};
}

// A row's pages in a wave's share: pages p .. p + cnt - 1 of its n.
struct Part {
  int item, sub, n, p, cnt;
  int row, heads;        // first output head (b * Hq + head), heads
  int nkb, last_keys;    // the request's blocks, keys of the last
  const int32_t* table;  // the page ids of its KV head
  const int32_t* list;   // its table row's entries, nullptr: every block
  long long item_start;  // the item's first page
};

// VT: transposed V pages.  DUP: at most 8 heads per tile, whose weights' second parts
// are in the upper columns.
template <int D, bool VT, bool DUP>
__global__ __launch_bounds__(kThreads, 2) void decode_kernel(const DecodeArgs a) {
  constexpr int NX = D / 16, NK = D / 32;      // d tiles, k-steps of a score
  constexpr int NL = D / 8;                    // 16-byte loads of a page, per lane
  constexpr int kFrag = NX * 64;               // float4 of a fragment
  constexpr int kStage = 32 * D * 2;           // bytes of half a V page
  static_assert(kFrag * 16 >= kStage, "");
  __shared__ __align__(16) float4 s_frag[kWaves][2][kFrag];   // [1] is the V stage until the end
  __shared__ float2 s_ml[kWaves][2][kTileHeads];
  __shared__ int4 s_meta[kWaves][2];   // row, heads, 1 starts | 2 ends | 4 valid
  __shared__ long long s_row[kWaves][2][2];   // the piece's row's first and last page
  static_assert(sizeof(s_frag) >= sizeof(JoinSpace), "");
  const DecodeLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int w = blockIdx.x;

  // ---- this wave's share ---------------------------------------------------
  // Sums of the items' pages, `per` of them to a lane; every wave makes them by
  // itself, in registers, which is quicker than to wait for the others.
  const int per = (a.items + kWave - 1) / kWave;
  unsigned mine = 0;
  int my_len = 0;   // of the request, where a lane has one and no tables are given
  if (per == 1 && !l.kv_indptr) {
    if (lane < a.items) my_len = request_len(a, lane);
    mine = blocks_for(my_len);
  } else {
    for (int i = lane * per; i < (lane + 1) * per; ++i)
      if (i < a.items) mine += item_pages(a, i);
  }
  const unsigned incl = lanes_sum(mine);
  const long long total = (long long)(unsigned)__builtin_amdgcn_readlane((int)incl, 63) * a.per_item;
  auto pages_of = [&](int i) -> int {
    return per == 1 ? __builtin_amdgcn_readlane((int)mine, i) : uniform(item_pages(a, i));
  };
  const int least = least_pages(a, total);
  const long long u0 = share_start(total, least, w), nu = share_start(total, least, w + 1) - u0;
  const long long my0 = u0 + nu * wv / kWaves, my1 = u0 + nu * (wv + 1) / kWaves;
  if (lane < 2) s_meta[wv][lane].z = 0;

  // ---- its pages, row by row ------------------------------------------------
  int rem = (int)(my1 - my0);
  int item = 0, sub = 0, n = 0, p = 0;
  long long item_start = 0;   // first page of the item
  if (rem > 0) {
    // the item with excl <= my0 / per_item < incl
    unsigned at = (unsigned)((double)my0 / (double)a.per_item);
    if ((long long)at * a.per_item > my0) --at;
    else if ((long long)(at + 1) * a.per_item <= my0) ++at;
    const int found = __builtin_ctzll(__ballot(incl - mine <= at && at < incl));
    unsigned start = __builtin_amdgcn_readlane((int)(incl - mine), found);
    item = found * per;
    n = pages_of(item);
    if (per > 1) {   // among the lane's items, 64 at a time
      for (int i = item;; i += kWave) {
        const unsigned here = i + lane < a.items ? item_pages(a, i + lane) : 0;
        const unsigned sums = start + lanes_sum(here);
        const unsigned long long hit = __ballot(sums - here <= at && at < sums);
        if (hit) {
          const int k = __builtin_ctzll(hit);
          item = i + k;
          n = __builtin_amdgcn_readlane((int)here, k);
          start = __builtin_amdgcn_readlane((int)(sums - here), k);
          break;
        }
        start = __builtin_amdgcn_readlane((int)sums, 63);
        if (i + kWave >= a.items) {   // only if the lengths changed under the kernel
          rem = 0;
          break;
        }
      }
    }
    item_start = (long long)start * a.per_item;
    const unsigned off = (unsigned)(my0 - item_start);
    if (n > 0) {
      sub = (int)(off / (unsigned)n);
      sub = sub < a.per_item ? sub : a.per_item - 1;
      p = (int)(off % (unsigned)n);
    } else {
      rem = 0;   // as above
    }
  }
  auto part_of = [&](int item, int sub, int n, int p, int left, long long item_start) {
    Part t;
    t.item = item, t.sub = sub, t.n = n, t.p = p, t.item_start = item_start;
    t.cnt = left < n - p ? left : n - p;
    int b, g, ht;
    if (l.kv_indptr) b = item / a.G, g = item - b * a.G, ht = sub;
    else b = item, g = sub / a.HT, ht = sub - g * a.HT;
    const int kvh = (int)((long long)g * l.group_size / (a.Hq / a.Hkv));
    t.row = b * a.Hq + g * l.group_size + ht * kTileHeads;
    t.heads = l.group_size - ht * kTileHeads;
    t.heads = t.heads < kTileHeads ? t.heads : kTileHeads;
    const int len = per == 1 && !l.kv_indptr ? __builtin_amdgcn_readlane(my_len, item)
                                             : uniform(request_len(a, b));
    t.nkb = blocks_for(len);
    t.last_keys = len - (t.nkb - 1) * kPage;
    t.table = l.page_table + ((long long)b * a.Hkv + kvh) * a.max_kv_blocks;
    t.list = l.kv_indptr ? l.kv_indices + uniform(l.kv_indptr[item]) : nullptr;
    return t;
  };
  // the row after t in a share with `left` more pages
  auto part_after = [&](const Part& t, int left) {
    int item = t.item, sub = t.sub + 1, n = t.n;
    long long item_start = t.item_start;
    if (sub == a.per_item) {
      sub = 0;
      item_start += (long long)n * a.per_item;
      if (per == 1) {
        do n = ++item < a.items ? pages_of(item) : -1; while (n == 0);
      } else {   // 64 at a time: 1000 idle requests would be as many loads one after the other
        n = -1;
        for (int i = item + 1; n < 0 && i < a.items; i += kWave) {
          const int here = i + lane < a.items ? item_pages(a, i + lane) : 0;
          const unsigned long long hit = __ballot(here > 0);
          if (!hit) continue;
          const int k = __builtin_ctzll(hit);
          item = i + k;
          n = __builtin_amdgcn_readlane(here, k);
        }
      }
      if (n < 0) item = t.item, n = 1;   // only if the lengths changed under the kernel
    }
    return part_of(item, sub, n, 0, left, item_start);
  };
  // ids of 64 of its pages from `at` on, one per lane: -1 where there is no page
  // to read, the sign bit set at the request's last block (num_pages < 2^31)
  auto fetch_ids = [&](const Part& t, int at) {
    int id = -1;
    if (at + lane < t.cnt) {
      const int j = t.list ? t.list[t.p + at + lane] : t.p + at + lane;
      if (j >= 0 && j < t.nkb) {
        const int page = t.table[j];
        if (page >= 0 && page < a.num_pages) id = j == t.nkb - 1 ? page | INT32_MIN : page;
      }
    }
    return id;
  };
  char* const stage = reinterpret_cast<char*>(&s_frag[wv][1][0]);

  // The waves keep step, a barrier each page, with the next page already on its
  // way: left alone, some are served first throughout, and end 30 us of 80 before
  // the others, with too little in flight for the rest (52 ragged requests: 112.4 us
  // without, 109.7 with).  All take as many barriers as the longest share has pages.
  int step = 0;
  const int steps = (int)((nu + kWaves - 1) / kWaves);
  Part cur = {}, nxt = {};
  int ids = -1, next_ids = -1, nxt_ids = -1;
  if (rem > 0) {
    cur = part_of(item, sub, n, p, rem, item_start);
    ids = fetch_ids(cur, 0);
  }
  // the ids of all waves are asked for before any wave's pages: behind the
  // pages of 8 waves they come some 10 us later
  __syncthreads();
  if (rem > 0) {
    rem -= cur.cnt;
    bf16x8 q[NK];
    auto load_q = [&](const Part& t) {
      const int head = DUP ? (col & 7) : col;
      const uint16_t* src = l.q + ((long long)t.row + head) * D + 8 * grp;
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        u32x4 x = {0, 0, 0, 0};
        if (head < t.heads) x = *reinterpret_cast<const u32x4*>(src + 32 * s);
        q[s] = __builtin_bit_cast(bf16x8, x);
      }
    };
    // A page on its way: whole rows, 1 KB a load, lines that no one keeps.  One page
    // of a wave at a time, K(i), V(i), K(i + 1), ..: a bare reader of 537 MB takes 80 us
    // so, 103 with K(i + 1) asked for while V(i) is on its way, and 91 with
    // ordinary loads; 16 rows x 64 bytes a load (fragments straight to
    // registers) took this kernel 991 us of 5.6 GB instead of 834.
    u32x4 x[NL];
    auto load = [&](const uint16_t* pool, int id) {
      // a page that is not there: page 0 is read in its place and counts for nothing
      const uint16_t* page = pool + (long long)(id == -1 ? 0 : id & INT32_MAX) * (kPage * D);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < NL; ++y)
        x[y] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(page + 512 * y + 8 * lane));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto to_stage = [&](auto kind, int half) {
      constexpr Half H = decltype(kind)::value;
      constexpr int RL = H == kHalfVT ? kPage : D;   // elements of a row
#pragma unroll
      for (int y = 0; y < NL / 2; ++y) {
        const int e = 512 * y + 8 * lane, r = e / RL, c = (e % RL) / 8;
        *reinterpret_cast<u32x4*>(stage + r * RL * 2 + 16 * swizzle<D, H>(r, c)) = x[half * (NL / 2) + y];
      }
      __builtin_amdgcn_wave_barrier();
    };
    constexpr int NR = DUP ? 0 : NX;   // d tiles of the weights' second parts
    f32x4 o[NX], rest[NR > 0 ? NR : 1];
    // m is carried scaled and rounded, as the weights take it off: while the maximum
    // stays, its factor is 1 exactly.  Scaled anew for every page it would be fused into the
    // difference and leave the product's rounding there, on all earlier pages, every time
    // (512 pages to a wave, largest scores of 180 in each: lse 2.6e-3 off, 5e-6 so).
    float m, sum;
    auto clear = [&] {
#pragma unroll
      for (int x = 0; x < NX; ++x) o[x] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NR; ++x) rest[x] = {0.f, 0.f, 0.f, 0.f};
      m = -INFINITY, sum = 0.f;
    };
    clear();

    int id = __builtin_amdgcn_readlane(ids, 0);
    load_q(cur);
    load(l.k_pool, id);
    if (rem > 0) {
      nxt = part_after(cur, rem);
      nxt_ids = fetch_ids(nxt, 0);
    }
    for (int i = 0;;) {
      // the next page, of this row or of the next
      const bool row_done = i + 1 == cur.cnt, go = !row_done || rem > 0;
      if ((i & 63) == 0) next_ids = fetch_ids(cur, i + 64);
      if ((i & 63) == 63) ids = next_ids;
      const int id2 = row_done ? __builtin_amdgcn_readlane(nxt_ids, 0)
                               : __builtin_amdgcn_readlane(ids, (i + 1) & 63);
      f32x4 s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) s[t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        to_stage(std::integral_constant<Half, kHalfK>{}, h);
        if (h == 1) load(l.v_pool, id);
        const int r0 = 8 * (col >> 2) + (col & 3);
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const u32x4 f = *reinterpret_cast<const u32x4*>(
                stage + (r0 + 4 * t) * D * 2 + 16 * swizzle<D, kHalfK>(r0, 4 * c + grp));
            s[2 * h + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), q[c],
                                                                   s[2 * h + t], 0, 0, 0);
          }
        __builtin_amdgcn_wave_barrier();
      }
      if (id < 0) {   // the last page, or one that is not there
        const int keys = id == -1 ? 0 : cur.last_keys;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key_of(t, 0) + 8 * grp + e >= keys) s[t][e] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max2(top, s[t][e]);
      const float mn = max2(m, groups_max(top) * a.scale_log2);
      const float base = mn == -INFINITY ? 0.f : mn;
      const float alpha = fast_exp2(m - base);
      m = mn;
      float part = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][e] = fast_exp2(__builtin_fmaf(s[t][e], a.scale_log2, -base));
          part += s[t][e];
        }
      sum = __builtin_fmaf(sum, alpha, part);
      bf16x8 pt[2], pr[2];
      const float keep = DUP && col >= 8 ? 1.f : 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[2 * c + (e >> 2)][e & 3];
          // weights to 16 bits, in two parts
          const __bf16 hi = (__bf16)x;
          pt[c][e] = DUP ? (__bf16)__builtin_fmaf(-keep, (float)hi, x) : hi;
          if constexpr (!DUP) pr[c][e] = (__bf16)(x - (float)hi);
        }
#pragma unroll
      for (int x = 0; x < NX; ++x) o[x] *= alpha;
#pragma unroll
      for (int x = 0; x < NR; ++x) rest[x] *= alpha;
      if (id < 0) {
        const int keys = id == -1 ? 0 : cur.last_keys;
        // weights of 0 do not undo a NaN in V
#pragma unroll
        for (int y = 0; y < NL; ++y) {
          if constexpr (VT) {
            const int first = 8 * (lane & 7);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (first + 2 * e >= keys) x[y][e] = 0;
              else if (first + 2 * e + 1 >= keys) x[y][e] &= 0xffffu;
            }
          } else {
            if ((512 * y + 8 * lane) / D >= keys) x[y] = {0, 0, 0, 0};
          }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        to_stage(std::integral_constant<Half, VT ? kHalfVT : kHalfV>{}, h);
        if (h == 1 && go) {
          if (row_done) load_q(nxt);
          load(l.k_pool, id2);
        }
        if (h == 1) {   // see `steps`
          __builtin_amdgcn_s_barrier();
          ++step;
        }
        // d tile t of the result, 32-key step c
        auto add_v = [&](const u32x4& f, int t, int c) {
          o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pt[c], o[t], 0, 0, 0);
          if constexpr (!DUP)
            rest[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pr[c], rest[t], 0, 0, 0);
        };
        if constexpr (VT) {
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int y = 0; y < NX / 2; ++y) {
              const u32x4 f = *reinterpret_cast<const u32x4*>(
                  stage + (16 * y + col) * kPage * 2 + 16 * swizzle<D, kHalfVT>(col, 4 * c + grp));
              add_v(f, h * (NX / 2) + y, c);
            }
        } else {
          const int r0 = 8 * grp + (col >> 2);
#pragma unroll
          for (int y = 0; y < NX; ++y) {
            const int d = 16 * y + 4 * (col & 3);
            const char* src = stage + r0 * D * 2 + 16 * swizzle<D, kHalfV>(r0, d >> 3) + 2 * (d & 7);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src);
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 4 * D * 2));
            const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
            const u32x4 f = {l2[0], l2[1], h2[0], h2[1]};
            add_v(f, y, h);
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
      id = id2;
      ++i;
      if (!row_done) continue;

      // ---- the row's end, or the share's
      sum = groups_sum(sum);
      // an infinity of v reaches the second parts with any sign, or none (inf * 0)
      float far = 0.f;
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) far = max2(far, __builtin_fabsf(o[x][e]));
      const bool finite = __ballot(!(far < INFINITY)) == 0;
      if (__builtin_expect(!finite, 0)) {   // out of the way: code is cold at a row's end
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float second = DUP ? other_half(o[x][e]) : rest[NR > 0 ? x : 0][e];
            o[x][e] += __builtin_isfinite(o[x][e]) ? second : 0.f;
          }
      } else {
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x][e] += DUP ? other_half(o[x][e]) : rest[NR > 0 ? x : 0][e];
      }
      const bool starts = cur.p == 0, ends = cur.p + cur.cnt == cur.n;
      if (starts && ends) {
        if (col < cur.heads) {
          const long long row = (long long)cur.row + col;
          const float inv = sum == 0.f ? 0.f : 1.f / sum;   // sum is NaN after a score of NaN or +inf
#pragma unroll
          for (int x = 0; x < NX; ++x)
            *reinterpret_cast<u32x2*>(l.out + row * D + 16 * x + 4 * grp) =
                u32x2{pack_bf16x2(o[x][0] * inv, o[x][1] * inv), pack_bf16x2(o[x][2] * inv, o[x][3] * inv)};
          if (l.lse && grp == 0) l.lse[row] = sum > 0.f ? (m + __log2f(sum)) * kLn2 : -INFINITY;
        }
      } else {
        const int f = starts ? 1 : 0;   // [1] is the wave's last: its stage is free
#pragma unroll
        for (int x = 0; x < NX; ++x)
          s_frag[wv][f][64 * x + lane] = make_float4(o[x][0], o[x][1], o[x][2], o[x][3]);
        if (grp == 0) s_ml[wv][f][col] = make_float2(m, sum);
        if (lane == 0) {
          s_meta[wv][f] = make_int4(cur.row, cur.heads, (starts ? 1 : 0) | (ends ? 2 : 0) | 4, 0);
          s_row[wv][f][0] = cur.item_start + (long long)cur.sub * cur.n;
          s_row[wv][f][1] = cur.item_start + (long long)(cur.sub + 1) * cur.n - 1;
        }
      }
      if (!go) break;
      clear();
      cur = nxt;
      ids = nxt_ids;
      i = 0;
      rem -= cur.cnt;
      if (rem > 0) {
        nxt = part_after(cur, rem);
        nxt_ids = fetch_ids(nxt, 0);
      }
    }
  }
  for (; step < steps; ++step) __builtin_amdgcn_s_barrier();
  __syncthreads();

  // ---- the waves' pieces, row by row -----------------------------------------
  // In page order they are piece 2 v + f of wave v; one that does not start a row
  // goes on with the row of the piece before it, so a row has one of a wave at most.
  // Rows that other workgroups share: [0] the one before the share, [1] behind it.
  int left_w0[2] = {-1, -1}, left_w1[2] = {0, 0}, left_heads[2] = {0, 0}, left_row[2] = {0, 0};
  int4 meta = make_int4(0, 0, 0, 0);
  if (lane < 2 * kWaves) meta = s_meta[lane >> 1][lane & 1];
  const unsigned valid = (unsigned)__ballot((meta.z & 4) != 0);
  const unsigned starting = (unsigned)__ballot((meta.z & 5) == 5);
  const unsigned ending = (unsigned)__ballot((meta.z & 6) == 6);
  const unsigned firsts = starting | (valid & (0u - valid));   // the first piece of every row
  const int rows = __builtin_popcount(firsts);
  // few rows: several waves to a row, each some of the d tiles
  const int per_row = rows >= kWaves ? 1 : kWaves / (rows > 0 ? rows : 1);
  unsigned ahead = firsts;   // without the rows before the one at hand
  for (int r = 0, at_row = wv / per_row; r < rows; ++r, ahead &= ahead - 1) {
    const int f = __builtin_ctz(ahead);
    const unsigned next = ahead & (ahead - 1);
    const unsigned set = valid & ~((1u << f) - 1) & (next ? (next & (0u - next)) - 1 : ~0u);
    const int last = 31 - __builtin_clz(set);
    const int flags = ((starting >> f) & 1) | (((ending >> last) & 1) << 1);
    const int row = __builtin_amdgcn_readlane(meta.x, f), heads = __builtin_amdgcn_readlane(meta.y, f);
    if (flags != 3) {
      const int side = flags & 1;
      const int w0 = share_of(total, least, uniform64(s_row[f >> 1][f & 1][0]));
      const int w1 = share_of(total, least, uniform64(s_row[f >> 1][f & 1][1]));
      if (side) left_w0[1] = w0, left_w1[1] = w1, left_heads[1] = heads, left_row[1] = row;
      else left_w0[0] = w0, left_w1[0] = w1, left_heads[0] = heads, left_row[0] = row;
    }
    if (r != at_row) continue;
    at_row += kWaves / per_row;
    // pieces one after the other, in order, the d tiles of a piece together
    const int x0 = wv % per_row;
    float top = -INFINITY, all = 0.f;
    float4 acc[NX];
#pragma unroll
    for (int k = 0; k < NX; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (unsigned rest = set; rest; rest &= rest - 1) {
      const int at = __builtin_ctz(rest);
      const float2 ml = s_ml[at >> 1][at & 1][col];
      const float4* const o = &s_frag[at >> 1][at & 1][64 * x0 + lane];
      const float mn = max2(top, ml.x), base = mn == -INFINITY ? 0.f : mn;
      const float c0 = fast_exp2(top - base), c1 = fast_exp2(ml.x - base);
      all = all * c0 + ml.y * c1;
      top = mn;
#pragma unroll
      for (int k = 0; k < NX; ++k) {
        if (x0 + k * per_row >= NX) break;
        const float4 y = o[64 * k * per_row];
        acc[k].x = acc[k].x * c0 + y.x * c1, acc[k].y = acc[k].y * c0 + y.y * c1;
        acc[k].z = acc[k].z * c0 + y.z * c1, acc[k].w = acc[k].w * c0 + y.w * c1;
      }
    }
    const float inv = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
    for (int k = 0; k < NX; ++k) {
      const int x = x0 + k * per_row, d = 16 * x + 4 * grp;
      if (x >= NX) break;
      if (col >= heads) {
        // no such head
      } else if (flags == 3) {
        *reinterpret_cast<u32x2*>(l.out + ((long long)row + col) * D + d) =
            u32x2{pack_bf16x2(acc[k].x * inv, acc[k].y * inv), pack_bf16x2(acc[k].z * inv, acc[k].w * inv)};
        if (l.lse && x == 0 && grp == 0)
          l.lse[row + col] = all > 0.f ? (top + __log2f(all)) * kLn2 : -INFINITY;
      } else {
        const int slot = 2 * w + (flags & 1);
        float* const to = a.part_o + ((long long)slot * kTileHeads + col) * D + d;
        put2(to, acc[k].x, acc[k].y);
        put2(to + 2, acc[k].z, acc[k].w);
        if (x == 0 && grp == 0) put2(a.part_ml + 2 * (slot * kTileHeads + col), top, all);
      }
    }
  }
  if (!a.join_later && (left_w0[0] >= 0 || left_w0[1] >= 0)) {
    // a piece counts once every wave's stores of it are done
    __shared__ int s_last[2];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid < 2) {
      const int w0 = tid ? left_w0[1] : left_w0[0], w1 = tid ? left_w1[1] : left_w1[0];
      s_last[tid] = w0 >= 0 && last_of(a.arrived + w0, a.piece, w1 - w0 + 1);
    }
    JoinSpace& space = *reinterpret_cast<JoinSpace*>(&s_frag[0][0][0]);
    __syncthreads();
#pragma nounroll
    for (int side = 0; side < 2; ++side)   // one copy of the code: it is cold when it is needed
      if (s_last[side]) {
        join_row<D>(a, side ? left_w0[1] : left_w0[0], side ? left_w1[1] : left_w1[0],
                    side ? left_row[1] : left_row[0], side ? left_heads[1] : left_heads[0], space);
        __syncthreads();   // its LDS
      }
  }

  // ---- requests and rows without a page -----------------------------------
  for (int i = w; i < a.items; i += kGroups) {
    if (pages_of(i) > 0) continue;
    const int nh = a.Hq / (l.kv_indptr ? a.G : 1);
    const long long row = l.kv_indptr ? (long long)(i / a.G) * a.Hq + (long long)(i % a.G) * nh
                                      : (long long)i * a.Hq;
    for (int x = tid; x < nh * (D / 8); x += kThreads)
      reinterpret_cast<u32x4*>(l.out + row * D)[x] = u32x4{0, 0, 0, 0};
    if (l.lse)
      for (int x = tid; x < nh; x += kThreads) l.lse[row + x] = -INFINITY;
  }
}

// The rows that several workgroups share, where there are few rows: one row may
// then be in 256 pieces, too many bytes for one workgroup (a 128K request of one KV
// head: 36 us with join_row, 24 with this).  A workgroup takes 16 dimensions
// of a row; its threads take a float4 of a head, of every lots-th piece.
template <int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const DecodeArgs a) {
  __shared__ float4 s_o[kThreads];
  __shared__ float2 s_ml[kThreads];
  const int tid = threadIdx.x;
  const int item = blockIdx.x / a.per_item, sub = blockIdx.x % a.per_item, x = blockIdx.y;
  long long start = 0, total = 0;
  int n = 0;
  for (int i = 0; i < a.items; ++i) {   // kFewRows at most
    const int pages = item_pages(a, i);
    if (i == item) n = pages;
    if (i < item) start += (long long)pages * a.per_item;
    total += (long long)pages * a.per_item;
  }
  if (n == 0) return;
  start += (long long)sub * n;
  const int least = least_pages(a, total);
  const int w0 = share_of(total, least, start), w1 = share_of(total, least, start + n - 1);
  if (w0 == w1) return;
  int b, g, ht;
  if (a.l.kv_indptr) b = item / a.G, g = item - b * a.G, ht = sub;
  else b = item, g = sub / a.HT, ht = sub - g * a.HT;
  const long long row = (long long)b * a.Hq + g * a.l.group_size + ht * kTileHeads;
  int heads = a.l.group_size - ht * kTileHeads;
  heads = heads < kTileHeads ? heads : kTileHeads;
  const int per = 4 * heads, lots = kThreads / per, lot = tid / per;
  const int head = (tid - lot * per) >> 2, d = 16 * x + 4 * (tid & 3);
  float top = -INFINITY, all = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, const float4& o) {
    const float mn = max2(top, ml.x), base = mn == -INFINITY ? 0.f : mn;
    const float c0 = fast_exp2(top - base), c1 = fast_exp2(ml.x - base);
    all = all * c0 + ml.y * c1;
    acc.x = acc.x * c0 + o.x * c1, acc.y = acc.y * c0 + o.y * c1;
    acc.z = acc.z * c0 + o.z * c1, acc.w = acc.w * c0 + o.w * c1;
    top = mn;
  };
  if (lot < lots)
#pragma unroll 8
    for (int e = w0 + lot; e <= w1; e += lots) {
      const int at = (2 * e + (e == w0 ? 1 : 0)) * kTileHeads + head;
      add(reinterpret_cast<const float2*>(a.part_ml)[at],
          *reinterpret_cast<const float4*>(a.part_o + (long long)at * D + d));
    }
  // halves: lot i takes lot i + half's
  for (int n_lots = lots; n_lots > 1;) {
    const int half = (n_lots + 1) / 2;
    __syncthreads();
    if (lot >= half && lot < n_lots) s_o[tid] = acc, s_ml[tid] = make_float2(top, all);
    __syncthreads();
    if (lot + half < n_lots) add(s_ml[tid + half * per], s_o[tid + half * per]);
    n_lots = half;
  }
  if (lot > 0) return;
  const float inv = all == 0.f ? 0.f : 1.f / all;
  *reinterpret_cast<u32x2*>(a.l.out + (row + head) * D + d) =
      u32x2{pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)};
  if (a.l.lse && x == 0 && (tid & 3) == 0)
    a.l.lse[row + head] = all > 0.f ? (top + __log2f(all)) * kLn2 : -INFINITY;
}

template <int D, bool VT>
hipError_t launch(const DecodeArgs& a, hipStream_t st) {
  if (a.l.group_size <= 8) decode_kernel<D, VT, true><<<kGroups, kThreads, 0, st>>>(a);
  else decode_kernel<D, VT, false><<<kGroups, kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.join_later) return e;
  decode_join_kernel<D><<<dim3(a.items * a.per_item, D / 16), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t decode_ws_bytes(const CacheDims& d) {
  return (size_t)kGroups * (2 * kTileHeads * (d.D * sizeof(float) + sizeof(float2)) +
                           sizeof(unsigned long long));
}

hipError_t launch_decode(const CacheDims& d, const DecodeLaunch& l, hipStream_t st) {
  DecodeArgs a;
  a.l = l;
  a.B = d.B;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.G = d.Hq / l.group_size;
  a.HT = (l.group_size + kTileHeads - 1) / kTileHeads;
  a.items = l.kv_indptr ? d.B * a.G : d.B;
  a.per_item = l.kv_indptr ? a.HT : a.G * a.HT;
  a.max_kv_blocks = d.max_kv_blocks;
  a.num_pages = d.num_pages;
  a.scale_log2 = l.sm_scale * kLog2e;
  a.part_o = static_cast<float*>(l.ws);
  a.part_ml = a.part_o + (size_t)kGroups * 2 * kTileHeads * d.D;
  a.arrived = reinterpret_cast<unsigned long long*>(a.part_ml + (size_t)kGroups * 2 * kTileHeads * 2);
  static std::atomic<unsigned long long> launches{0};
  a.piece = (kLaunchTop | (launches.fetch_add(1, std::memory_order_relaxed) & 0xff'ffff'ffffull)) << 16 | 1;
  // a row of at most 64 pieces (32 and fewer as a rule) is joined in the launch, whatever the rows
  a.join_later = (long long)a.items * a.per_item <= kFewRows && a.max_kv_blocks > kManyPieces;
  const bool vt = d.v_layout != 0;
  if (d.D == 64) return vt ? launch<64, true>(a, st) : launch<64, false>(a, st);
  return vt ? launch<128, true>(a, st) : launch<128, false>(a, st);
}

}  // namespace ca
