// Attention of one new token per request where requests share prefixes: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// in one pass over the keys with the running maximum m and sum, the share's whole pages
// (through its first member's row) once for all members, the others for their request.
//
// The work is a stream of pages.  A set is a share with two members or more (its whole
// pages; rows: the queries of all members) or a request (the pages behind; rows: its own
// queries), an item a set's KV head and tile of 256 rows.  The pages of all items are laid
// end to end and cut in equal shares, one per workgroup, which every workgroup finds from the
// lengths on the GPU; pieces of an item that several workgroups have are joined by a
// second launch, with the prefix's and the request's parts of every row.
#include <type_traits>

#include "common.hpp"
#include "pages.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kGroups = 256;                  // one workgroup per CU
constexpr int kTile = kPrefixRows;            // query rows of an item
constexpr int kSets = kPrefixShares + kPrefixRequests;
constexpr int kQueue = 128;                   // pages that are looked up together
constexpr int kLoaders = 6;                   // waves kLoaders and on ask for K and V pages
constexpr int kJoinThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PrefixArgs {
  PrefixLaunch l;
  int B, Hq, Hkv, G, tiles;        // G heads on a KV head, in `tiles` tiles
  int max_kv_blocks, num_pages, slot_rows;
  float scale_log2;
  // items that lie in one workgroup's share: [0] of shares, [1] of requests, by query row
  float* whole_o;                  // [2][B * Hq][D], not normalised
  float* whole_ml;                 // [2][B * Hq][2]: maximum (log2 units) and sum
  // pieces: [0] of the item that a workgroup's share starts inside of, [1] of the one that goes on after it
  float* part_o;                   // [kGroups][2][slot_rows][D]
  float* part_ml;                  // [kGroups][2][slot_rows][2]
  int4* plan;                      // [B][2]: see Where
};

// Where the join finds a request's parts.
struct Where {
  int own_start, own_pages;        // first page of its own items in the stream, pages of one
  int share_start, share_pages;    // of its share's
  int rank, share_tiles, total;    // its place among the members; pages of all items
};

// Pages of the stream before workgroup w's share, and the share of page u.  Every workgroup before one that
// has pages has some, so a row's pieces are in workgroups side by side.
__device__ __forceinline__ int share_start(int total, int w) {
  if (total >= kGroups) return (int)((long long)total * w / kGroups);
  return w < total ? w : total;
}
__device__ __forceinline__ int share_of(int total, int u) {
  long long w = u;
  if (total >= kGroups) w = ((long long)(u + 1) * kGroups - 1) / total;
  return w < 0 ? 0 : (w < kGroups ? (int)w : kGroups - 1);
}

__device__ __forceinline__ int request_len(const PrefixArgs& a, int b) {
  const int len = a.l.kv_len[b], most = a.max_kv_blocks * kPage;
  return len < 0 ? 0 : (len < most ? len : most);
}
__device__ __forceinline__ int share_blocks(const PrefixArgs& a, int s) {
  const int n = a.l.share_len[s] / kPage;
  return n < 0 ? 0 : (n < a.max_kv_blocks ? n : a.max_kv_blocks);
}
// The share that request b of len tokens is a member of, -1: none.
__device__ __forceinline__ int share_of_request(const PrefixArgs& a, int b, int len) {
  if (a.l.num_shares == 0) return -1;
  const int s = a.l.share[b];
  if (s < 0 || s >= a.l.num_shares) return -1;
  const int blocks = share_blocks(a, s);
  return blocks > 0 && len >= blocks * kPage ? s : -1;
}

// s_waitcnt's operand: at most n vector memory operations are left.
constexpr int vm_count(int n) { return (n & 15) | (n >> 4) << 14 | 7 << 4 | 15 << 8; }

struct Entry {      // a page of the stream
  int page, set, sub;   // sub: KV head and tile of the item
  int keys;             // its keys that count, 0: no page; kFirst, kLast: of its item
};
constexpr int kFirst = 128, kLast = 256;

template <int D>
struct Shared {
  static constexpr int kPageBytes = kPage * D * 2;
  static constexpr int kRing = 131072 / (2 * kPageBytes);   // pages that are there or on their way
  char pages[kRing][2][kPageBytes];    // K and V
  float2 merge_ml[4][2][16];
  int start[kSets + 1];                // pages of the stream before a set
  uint16_t count[kPrefixShares], first[kPrefixShares];   // members of a share, and the first
  Entry queue[kQueue];
  uint16_t member[kTile + 2];          // requests of the tile at hand, in order
  int part[kWaves];
};

typedef __attribute__((address_space(3))) void lds_void;

// The compiler neither makes x earlier nor reads it later than here.
template <typename T>
__device__ __forceinline__ void made_here(T& x) {
  asm volatile("" : "+v"(x));
}

// A barrier for what waves write to LDS themselves: __syncthreads would wait for all pages on their way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One wave's loads of a page straight to LDS, 1 KB each, lane l to bytes 16 l of it, from where the swizzle
// puts them; what lies `bytes` or more into the page reads as 0.
template <int D, Half H>
__device__ __forceinline__ void page_to_lds(const uint16_t* from, int bytes, char* to, int lane) {
  constexpr int RL = H == kHalfVT ? kPage : D;   // elements of a row
  // a row's swizzle is the XOR of its bits', so those of a load's first row come in by one XOR
  int at = 2 * (8 * lane / RL * RL) + 16 * swizzle<D, H>(8 * lane / RL, 8 * lane % RL / 8);
  made_here(at);   // not kept for every load over the loop
#pragma unroll
  for (int y = 0; y < D / 8; ++y) {
    const int source = (at ^ (16 * swizzle<D, H>(512 * y / RL, 0))) + 1024 * y;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(from), 0, bytes, 0x00020000),
        (lds_void*)(to + 1024 * y), 16, source, 0, 0, 2 /* nt */);
  }
}

template <int D, bool VT>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(const PrefixArgs a) {
  constexpr int NX = D / 16, NK = D / 32;   // d tiles, k-steps of a score
  constexpr int NL = D / 8;                 // loads of a K or V page, 1 KB each
  constexpr int R = Shared<D>::kRing;
  constexpr Half HV = VT ? kHalfVT : kHalfV;
  __shared__ __align__(16) Shared<D> s;
  const PrefixLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63, w = blockIdx.x;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int S = l.num_shares, sets = S + a.B;

  // ---- the stream, from the lengths -------------------------------------------
  int* const count = reinterpret_cast<int*>(&s.pages[0][0][0]);   // no page is there yet
  int* const first = count + kPrefixShares;
  for (int i = tid; i < S; i += kThreads) count[i] = 0, first[i] = a.B;
  __syncthreads();
  if (S > 0)
    for (int b = tid; b < a.B; b += kThreads) {
      const int share = share_of_request(a, b, request_len(a, b));
      if (share >= 0) atomicAdd(&count[share], 1), atomicMin(&first[share], b);
    }
  __syncthreads();
  for (int i = tid; i < S; i += kThreads) s.count[i] = (uint16_t)count[i], s.first[i] = (uint16_t)first[i];
  __syncthreads();
  auto share_tiles = [&](int share) {
    const long long rows = (long long)s.count[share] * a.G;
    return (int)((rows + kTile - 1) / kTile);
  };
  // pages of one item of a set
  auto item_pages = [&](int set) {
    if (set < S) return s.count[set] > 1 ? share_blocks(a, set) : 0;
    const int b = set - S, len = request_len(a, b), share = share_of_request(a, b, len);
    return blocks_for(len) - (share >= 0 && s.count[share] > 1 ? share_blocks(a, share) : 0);
  };
  const int per = (sets + kThreads - 1) / kThreads;
  {
    int mine = 0;
    for (int i = tid * per; i < (tid + 1) * per && i < sets; ++i) {
      const int n = item_pages(i) * a.Hkv * (i < S ? share_tiles(i) : a.tiles);
      s.start[i] = n;
      mine += n;
    }
    int before = wave_inclusive_scan(mine);
    if (lane == kWave - 1) s.part[wv] = before;
    __syncthreads();
    before -= mine;
    for (int v = 0; v < wv; ++v) before += s.part[v];
    for (int i = tid * per; i < (tid + 1) * per && i < sets; ++i) {
      const int n = s.start[i];
      s.start[i] = before;
      before += n;
    }
    if (tid == kThreads - 1) s.start[sets] = before;
    __syncthreads();
  }
  const int total = s.start[sets];
  const int u0 = share_start(total, w), u1 = share_start(total, w + 1);

  // ---- where the join finds the requests' parts: some requests each -------------
  for (int b = w * kWaves + wv; b < a.B; b += kGroups * kWaves) {
    const int share = share_of_request(a, b, request_len(a, b));
    const bool shared = share >= 0 && s.count[share] > 1;
    int rank = 0;
    for (int i0 = 0; shared && i0 < b; i0 += kWave) {
      const int i = i0 + lane;
      rank += __popcll(__ballot(i < b && share_of_request(a, i, request_len(a, i)) == share));
    }
    if (lane == 0) {
      a.plan[2 * b] = make_int4(s.start[S + b], item_pages(S + b), shared ? s.start[share] : 0,
                                shared ? item_pages(share) : 0);
      a.plan[2 * b + 1] = make_int4(rank, shared ? share_tiles(share) : 1, total, 0);
    }
  }

  // ---- the pages of this share, some looked up at a time ------------------------
  // page u of the stream
  auto look_up = [&](int u) {
    int lo = 0, hi = sets;   // the last set that starts at u or before: it has pages
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s.start[mid] <= u) lo = mid;
      else hi = mid;
    }
    const int off = u - s.start[lo], n = item_pages(lo);
    Entry e = {-1, lo, 0, 0};
    int row, block, tiles;
    if (n <= 0) return e;   // only if the lengths changed under the kernel
    e.sub = off / n;
    const int p = off - e.sub * n;
    if (lo < S) {
      row = s.first[lo], block = p, tiles = share_tiles(lo);
      e.keys = kPage;
    } else {
      row = lo - S, tiles = a.tiles;
      const int len = request_len(a, row);
      block = blocks_for(len) - n + p;
      e.keys = len - block * kPage < kPage ? len - block * kPage : kPage;
    }
    const int kvh = e.sub / (tiles > 0 ? tiles : 1);
    if (row < a.B && kvh < a.Hkv && block >= 0 && block < a.max_kv_blocks)
      e.page = l.page_table[((long long)row * a.Hkv + kvh) * a.max_kv_blocks + block];
    if (e.page < 0 || e.page >= a.num_pages || e.keys < 0) e.page = -1, e.keys = 0;
    e.keys |= (p == 0 ? kFirst : 0) | (p == n - 1 ? kLast : 0);
    return e;
  };
  // Two waves ask for the pages, one for K and one for V, straight to LDS: the others never wait
  // for memory but at an item's ends, and those two only for pages.  A page that is not there, or past
  // the end, is a buffer of no bytes, which reads as 0; so do the rows behind the last key.
  auto load = [&](int i, int n) __attribute__((always_inline)) {
    const bool value = wv == kLoaders + 1;
    int page = -1, keys = 0;
    if (i < n) page = uniform(s.queue[i].page), keys = uniform(s.queue[i].keys) & 127;
    const uint16_t* const from = (value ? l.v_pool : l.k_pool) + (long long)(page < 0 ? 0 : page) * (kPage * D);
    const int bytes = page < 0 ? 0 : (VT && value ? kPage : keys) * D * 2;
    char* const to = s.pages[i % R][value ? 1 : 0];
    if (value) page_to_lds<D, HV>(from, bytes, to, lane);
    else page_to_lds<D, kHalfK>(from, bytes, to, lane);
  };

  // ---- the item at hand ----------------------------------------------------------
  // Up to 128 rows: 4 groups of 32 rows, each two waves with half of a page's keys; more: 8
  // groups, a wave each with all keys.
  int set = -1, sub = 0, rows = 0;
  bool starts = false, whole = false, active = false;
  int rg = 0, kh = 0;
  int row_of[2];               // of the lane's column: b * Hq + head, -1: none
  bf16x8 q[2][NK];
  f32x4 o[NX][2];
  float m[2], sum[2];

  auto begin = [&](const Entry& e) __attribute__((always_inline)) {
    set = e.set, sub = e.sub, starts = (e.keys & kFirst) != 0;
    const bool share = set < S;
    const int count = share ? s.count[set] : 1, tiles = share ? share_tiles(set) : a.tiles;
    const int kvh = sub / tiles, tile = sub - kvh * tiles, first = tile * kTile / a.G;
    if (share) {   // the members whose queries are in the tile, in order
      int n = 0;
      lds_barrier();
      for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        const bool in = b < a.B && share_of_request(a, b, request_len(a, b)) == set;
        const unsigned long long hits = __ballot(in);
        if (lane == 0) s.part[wv] = __popcll(hits);
        lds_barrier();
        int at = n - first + lanes_below(hits);
        for (int v = 0; v < kWaves; ++v) {
          if (v < wv) at += s.part[v];
          n += s.part[v];
        }
        if (in && at >= 0 && at < kTile + 2) s.member[at] = (uint16_t)b;
        lds_barrier();
      }
    }
    rows = count * a.G - tile * kTile;
    rows = rows < kTile ? rows : kTile;
    whole = rows > kTile / 2;
    rg = whole ? wv : wv >> 1, kh = whole ? 0 : wv & 1;
    active = 32 * rg < rows;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = 32 * rg + 16 * c + col;
      row_of[c] = -1;
      if (r < rows) {
        const int at = tile * kTile + r, i = at / a.G, head = at - i * a.G;
        const int b = share ? s.member[i - first] : set - S;
        if (b < a.B) row_of[c] = b * a.Hq + kvh * a.G + head;
      }
#pragma unroll
      for (int t = 0; t < NK; ++t) {
        u32x4 x = {0, 0, 0, 0};
        if (row_of[c] >= 0) x = *reinterpret_cast<const u32x4*>(l.q + (long long)row_of[c] * D + 32 * t + 8 * grp);
        q[c][t] = __builtin_bit_cast(bf16x8, x);
      }
      m[c] = -INFINITY, sum[c] = 0.f;
#pragma unroll
      for (int x = 0; x < NX; ++x) o[x][c] = {0.f, 0.f, 0.f, 0.f};
    }
    // waited for here: with every page they would be, and for all pages on their way then
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int t = 0; t < NK; ++t) made_here(q[c][t]);
  };

  // Scores, weights and sums of NP key steps (32 keys each) of the page in LDS, from step p0 on.
  auto attend = [&](auto steps, int p0, int buf, int keys) __attribute__((always_inline)) {
    constexpr int NP = decltype(steps)::value;
    const char* const kp = s.pages[buf][0];
    const char* const vp = s.pages[buf][1];
    f32x4 x[2 * NP][2];
#pragma unroll
    for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) x[t][c] = {0.f, 0.f, 0.f, 0.f};
    const int r0 = 8 * (col >> 2) + (col & 3) + 32 * p0;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t) {
        const u32x4 f = *reinterpret_cast<const u32x4*>(
            kp + (r0 + 32 * (t >> 1) + 4 * (t & 1)) * D * 2 + 16 * swizzle<D, kHalfK>(r0, 4 * ks + grp));
#pragma unroll
        for (int c = 0; c < 2; ++c)
          x[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), q[c][ks], x[t][c], 0, 0, 0);
      }
    if (keys < kPage) {
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (32 * p0 + key_of(t, 0) + 8 * grp + e >= keys) x[t][0][e] = x[t][1][e] = -INFINITY;
    }
    bool moved = false;
    float alpha[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float top = x[0][c][0];
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max2(top, x[t][c][e]);
      const float mn = max2(m[c], groups_max(top) * a.scale_log2);
      const float base = mn == -INFINITY ? 0.f : mn;
      alpha[c] = fast_exp2(m[c] - base);
      moved = moved || !(alpha[c] == 1.f);
      m[c] = mn;
      float part = 0.f;
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[t][c][e] = fast_exp2(__builtin_fmaf(x[t][c][e], a.scale_log2, -base));
          part += x[t][c][e];
        }
      sum[c] = __builtin_fmaf(sum[c], alpha[c], part);
    }
    if (__ballot(moved) != 0) {
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int c = 0; c < 2; ++c) o[y][c] *= alpha[c];
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      // weights to 16 bits, in two parts: the upper half of p's bits, and what that leaves, which is never
      // negative, and never 0 so that an infinity of v stays one
      u32x4 hi[2], lo[2];
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[2 * p + (e >> 1)][c][2 * (e & 1)], v = x[2 * p + (e >> 1)][c][2 * (e & 1) + 1];
          const uint32_t ub = __float_as_uint(u), vb = __float_as_uint(v);
          hi[c][e] = __builtin_amdgcn_perm(vb, ub, 0x07060302);
          constexpr float kLeast = 0x1p-126f;
          lo[c][e] = pack_bf16x2(fmaxf(u - __uint_as_float(ub & 0xffff0000u), kLeast),
                                 fmaxf(v - __uint_as_float(vb & 0xffff0000u), kLeast));
        }
#pragma unroll
      for (int y = 0; y < NX; ++y) {
        u32x4 f;
        if constexpr (VT) {
          f = *reinterpret_cast<const u32x4*>(vp + (16 * y + col) * kPage * 2 +
                                              16 * swizzle<D, kHalfVT>(col, 4 * (p0 + p) + grp));
        } else {
          const int v0 = 8 * grp + (col >> 2), d = 16 * y + 4 * (col & 3);
          const char* const src = vp + (v0 + 32 * (p0 + p)) * D * 2 + 16 * swizzle<D, kHalfV>(v0, d >> 3) + 2 * (d & 7);
          const u32x2 a2 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src));
          const u32x2 b2 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 4 * D * 2)));
          f = u32x4{a2[0], a2[1], b2[0], b2[1]};
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          o[y][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, hi[c]), o[y][c], 0, 0, 0);
          o[y][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, lo[c]), o[y][c], 0, 0, 0);
        }
      }
    }
  };

  // The piece's sums: the two halves of the keys together, then to where the join looks.
  auto finish = [&](bool ends, int buf) __attribute__((always_inline)) {
    float4* const merge = reinterpret_cast<float4*>(s.pages[buf][0]) + rg * (NX * kWave);   // the page is done with
#pragma unroll
    for (int c = 0; c < 2; ++c) sum[c] = groups_sum(sum[c]);
    if (!whole) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        lds_barrier();
        if (active && kh == 1) {
#pragma unroll
          for (int y = 0; y < NX; ++y)
            merge[64 * y + lane] = make_float4(o[y][c][0], o[y][c][1], o[y][c][2], o[y][c][3]);
          if (grp == 0) s.merge_ml[rg][c][col] = make_float2(m[c], sum[c]);
        }
        lds_barrier();
        if (active && kh == 0) {
          const float2 ml = s.merge_ml[rg][c][col];
          const float mn = max2(m[c], ml.x), base = mn == -INFINITY ? 0.f : mn;
          const float c0 = fast_exp2(m[c] - base), c1 = fast_exp2(ml.x - base);
          m[c] = mn;
          sum[c] = sum[c] * c0 + ml.y * c1;
#pragma unroll
          for (int y = 0; y < NX; ++y) {
            const float4 z = merge[64 * y + lane];
            o[y][c][0] = o[y][c][0] * c0 + z.x * c1, o[y][c][1] = o[y][c][1] * c0 + z.y * c1;
            o[y][c][2] = o[y][c][2] * c0 + z.z * c1, o[y][c][3] = o[y][c][3] * c0 + z.w * c1;
          }
        }
      }
    }
    if (!active || kh != 0) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (row_of[c] < 0) continue;
      float *to, *ml;
      if (starts && ends) {
        const long long row = (set < S ? 0 : (long long)a.B * a.Hq) + row_of[c];
        to = a.whole_o + row * D, ml = a.whole_ml + 2 * row;
      } else {
        const long long row = (long long)(2 * w + (starts ? 1 : 0)) * a.slot_rows + 32 * rg + 16 * c + col;
        to = a.part_o + row * D, ml = a.part_ml + 2 * row;
      }
#pragma unroll
      for (int y = 0; y < NX; ++y) *reinterpret_cast<f32x4*>(to + 16 * y + 4 * grp) = o[y][c];
      if (grp == 0) *reinterpret_cast<float2*>(ml) = make_float2(m[c], sum[c]);
    }
  };

  for (int base = u0; base < u1; base += kQueue) {
    const int n = u1 - base < kQueue ? u1 - base : kQueue;
    lds_barrier();
    if (tid < n) s.queue[tid] = look_up(base + tid);
    lds_barrier();   // the last pages of the queue before are done with, too
    if (wv >= kLoaders)
      for (int i = 0; i < R - 1; ++i) load(i, n);
    for (int i = 0; i < n; ++i) {
      Entry e = s.queue[i];
      e.page = uniform(e.page), e.set = uniform(e.set), e.sub = uniform(e.sub), e.keys = uniform(e.keys);
      const int keys = e.keys & 127, buf = i % R;
      // all but the pages after this one are there; then everyone is done with the one before
      if (wv >= kLoaders) __builtin_amdgcn_s_waitcnt(vm_count((R - 2) * NL));
      lds_barrier();
      if (wv >= kLoaders) load(i + R - 1, n);
      if (VT && keys < kPage) {   // weights of 0 do not undo a NaN in V: columns behind the last key
        for (int at = 8 * tid; at < kPage * D; at += 8 * kThreads) {
          const int r = at / kPage, first = at % kPage;
          if (first + 8 <= keys) continue;
          u32x4* const x = reinterpret_cast<u32x4*>(s.pages[buf][1] + r * kPage * 2 + 16 * swizzle<D, kHalfVT>(r, first / 8));
          u32x4 y = *x;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            if (first + 2 * z >= keys) y[z] = 0;
            else if (first + 2 * z + 1 >= keys) y[z] &= 0xffffu;
          }
          *x = y;
        }
        lds_barrier();
      }
      if ((e.keys & kFirst) || base + i == u0) begin(e);
      if (active) {
        if (whole) attend(std::integral_constant<int, 2>{}, 0, buf, keys);
        else attend(std::integral_constant<int, 1>{}, kh, buf, keys);
      }
      if ((e.keys & kLast) || base + i == u1 - 1) finish((e.keys & kLast) != 0, buf);
    }
  }
}

// A query row's parts: of its share's items and of its own, each whole or in the pieces of several
// workgroups.  A thread takes 4 dimensions of every lots-th piece.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void prefix_join_kernel(const PrefixArgs a) {
  constexpr int kEach = D / 4, kLots = kJoinThreads / kEach;
  __shared__ float4 s_o[kJoinThreads];
  __shared__ float2 s_ml[kLots];
  const int tid = threadIdx.x, lot = tid / kEach, d = 4 * (tid % kEach);
  const int b = blockIdx.x / a.Hq, h = blockIdx.x - b * a.Hq, kvh = h / a.G, head = h - kvh * a.G;
  const int4 p0 = a.plan[2 * b], p1 = a.plan[2 * b + 1];
  const Where at = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z};
  const long long out_row = (long long)b * a.Hq + h;
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
  // parts of the item of n pages from start on, whose row r is this one
  auto parts = [&](int kind, int start, int n, int r) {
    if (n <= 0) return;
    const int w0 = share_of(at.total, start), w1 = share_of(at.total, start + n - 1);
    if (w0 == w1) {
      if (lot != (kind == 0 ? 0 : kLots - 1)) return;
      const long long row = (kind ? (long long)a.B * a.Hq : 0) + out_row;
      add(*reinterpret_cast<const float2*>(a.whole_ml + 2 * row),
          *reinterpret_cast<const float4*>(a.whole_o + row * D + d));
      return;
    }
#pragma unroll 4
    for (int w = w0 + lot; w <= w1; w += kLots) {
      const long long row = (long long)(2 * w + (w == w0 ? 1 : 0)) * a.slot_rows + r;
      add(*reinterpret_cast<const float2*>(a.part_ml + 2 * row),
          *reinterpret_cast<const float4*>(a.part_o + row * D + d));
    }
  };
  const int share_row = at.rank * a.G + head;
  parts(0, at.share_start + (kvh * at.share_tiles + share_row / kTile) * at.share_pages, at.share_pages, share_row % kTile);
  parts(1, at.own_start + (kvh * a.tiles + head / kTile) * at.own_pages, at.own_pages, head % kTile);
  s_o[tid] = acc;
  if (d == 0) s_ml[lot] = make_float2(top, all);
  __syncthreads();
  if (lot > 0) return;
#pragma unroll
  for (int i = 1; i < kLots; ++i) add(s_ml[i], s_o[i * kEach + tid]);
  const float inv = all == 0.f ? 0.f : 1.f / all;   // all is NaN after a score of NaN or +inf
  *reinterpret_cast<u32x2*>(a.l.out + out_row * D + d) =
      u32x2{pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)};
  if (a.l.lse && tid == 0) a.l.lse[out_row] = all > 0.f ? (top + __log2f(all)) * kLn2 : -INFINITY;
}

// Rows of a tile at most.
int slot_rows_of(const CacheDims& d) {
  const long long rows = (long long)d.B * (d.Hq / d.Hkv);
  return rows < kTile ? (int)rows : kTile;
}

template <int D, bool VT>
hipError_t launch(const PrefixArgs& a, hipStream_t st) {
  prefix_kernel<D, VT><<<kGroups, kThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  prefix_join_kernel<D><<<a.B * a.Hq, kJoinThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t prefix_ws_bytes(const CacheDims& d) {
  const size_t rows = 2 * (size_t)d.B * d.Hq + 2 * (size_t)kGroups * slot_rows_of(d);
  return rows * (d.D + 2) * sizeof(float) + 2 * (size_t)d.B * sizeof(int4);
}

hipError_t launch_prefix(const CacheDims& d, const PrefixLaunch& l, hipStream_t st) {
  PrefixArgs a;
  a.l = l;
  a.B = d.B;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.G = d.Hq / d.Hkv;
  a.tiles = (a.G + kTile - 1) / kTile;
  a.max_kv_blocks = d.max_kv_blocks;
  a.num_pages = d.num_pages;
  a.slot_rows = slot_rows_of(d);
  a.scale_log2 = l.sm_scale * kLog2e;
  const size_t whole = 2 * (size_t)d.B * d.Hq, parts = 2 * (size_t)kGroups * a.slot_rows;
  a.plan = static_cast<int4*>(l.ws);
  a.whole_o = reinterpret_cast<float*>(a.plan + 2 * (size_t)d.B);
  a.part_o = a.whole_o + whole * d.D;
  a.whole_ml = a.part_o + parts * d.D;
  a.part_ml = a.whole_ml + 2 * whole;
  const bool vt = d.v_layout != 0;
  if (d.D == 64) return vt ? launch<64, true>(a, st) : launch<64, false>(a, st);
  return vt ? launch<128, true>(a, st) : launch<128, false>(a, st);
}

}  // namespace ca
