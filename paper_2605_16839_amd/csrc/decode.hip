// Attention of one new token per request over its paged cache: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// in one pass over the keys with the running maximum m and sum.
//
// What bounds it: every K and V page is read once and used for the few query
// heads of its KV head, 2 flops per byte and head, so HBM does.  Everything
// below serves an even, deep stream of page loads:
//   * the requests' lengths are on the GPU only and may be as different as they
//     like, so the pages of all (request, KV head) rows are laid end to end and
//     cut in equal shares, one per workgroup and within it one per wave; every
//     workgroup finds its share from a prefix sum over the lengths;
//   * a wave is on its own until its share ends: it loads K and V pages to
//     registers (32 KB of them in flight per wave, 256 KB per CU), and no
//     barrier or other wave is waited for;
//   * S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_16x16x32_bf16, the heads of
//     the KV head being the 16 columns.  K fragments are the registers as loaded
//     (key_of gives a lane 8 consecutive keys of each 32-key step, as the P^T
//     fragment wants them), transposed V pages too; token-major V goes through
//     8 KB of LDS per wave for the transpose read;
//   * up to 8 heads leave half of the columns free: they hold the same heads
//     again, and carry the part of the weights that bf16 loses (p - bf16(p)),
//     so the weights count with 16 bits at no cost;
//   * a row that lies inside one wave's share is written at once; pieces of
//     a workgroup's waves are joined in its LDS, and rows that several workgroups
//     share by a second launch (decode_join_kernel).
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kWaves = 8;                   // per workgroup
constexpr int kThreads = kWaves * kWave;
constexpr int kGroups = 256;                // one workgroup per CU
constexpr int kMinPages = 4;                // of a workgroup's share
constexpr int kTileHeads = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Share {   // what decode_join_kernel has to know about a workgroup's share
  long long row_end;   // end (in pages) of the row that goes on after the share, 0: none
  long long total;     // pages of all rows
  int out_row;         // that row's first output head (b * Hq + head)
  int heads;
};

struct DecodeArgs {
  DecodeLaunch l;
  int B, Hq, Hkv, G, HT, items, per_item, max_kv_blocks, num_pages;
  float scale_log2;
  float4* part_o;    // [kGroups][2][D / 16][64]: O^T fragments as the registers lie
  float2* part_ml;   // [kGroups][2][16]: maximum (log2 units) and sum
  Share* shares;     // [kGroups]
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

// First page of share w when `total` pages are dealt.
__device__ __forceinline__ long long share_start(long long total, int w) {
  if (total >= (long long)kGroups * kMinPages) return (total * w) / kGroups;
  const long long s = (long long)w * kMinPages;
  return s < total ? s : total;
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
// 16-byte chunk where chunk c of row r of a token-major V tile lies: 32 lanes of
// a transpose read cover keys {0..3, 8..11} (+ multiples) x 32 bytes, so bits 0, 1
// and 3 of the key pick the 32-byte pair (64-element rows: bit 0 picks the half
// of the 256-byte bank window).
template <int D>
__device__ __forceinline__ int v_swz(int r, int c) {
  return D == 128 ? (c ^ (((r & 3) | (((r >> 3) & 1) << 2)) << 1))
                  : (c ^ ((((r >> 1) & 1) | (((r >> 3) & 1) << 1)) << 1));
}

// VT: transposed V pages.  DUP: at most 8 heads per tile, see above.
template <int D, bool VT, bool DUP>
__global__ __launch_bounds__(kThreads, 2) void decode_kernel(const DecodeArgs a) {
  constexpr int NX = D / 16, NK = D / 32;      // d tiles, k-steps of a score
  constexpr int NL = D / 8;                    // 16-byte loads of a page, per lane
  constexpr int kFrag = NX * 64;               // float4 of a fragment
  constexpr int kStage = 32 * D * 2;           // bytes of half a V page
  static_assert(kFrag * 16 >= kStage, "");
  __shared__ __align__(16) float4 s_frag[kWaves][2][kFrag];   // [1] is the V stage until the end
  __shared__ float2 s_ml[kWaves][2][kTileHeads];
  __shared__ int4 s_meta[kWaves][2];   // item, sub, 1 starts | 2 ends, 1 valid
  __shared__ long long s_sum[kWaves], s_base[kWaves];
  __shared__ int s_item[kWaves];
  const DecodeLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int w = blockIdx.x;

  // ---- shares: prefix sums of the items' pages --------------------------
  const int per = (a.items + kThreads - 1) / kThreads;
  const int i0 = tid * per < a.items ? tid * per : a.items;
  const int i1 = i0 + per < a.items ? i0 + per : a.items;
  long long mine = 0;
  for (int i = i0; i < i1; ++i) mine += item_pages(a, i);
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const long long t = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += t;
  }
  if (lane == 63) s_sum[wv] = incl;
  if (lane < 2) s_meta[wv][lane].w = 0;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    if (v < wv) before += s_sum[v];
    total += s_sum[v];
  }
  total = uniform64(total) * a.per_item;
  const long long u0 = share_start(total, w), u1 = share_start(total, w + 1), nu = u1 - u0;
  {
    long long at = (before + incl - mine) * a.per_item;
    const long long end = (before + incl) * a.per_item;
    if (end > u0 && at < u1) {
      for (int i = i0; i < i1; ++i) {
        const long long next = per == 1 ? end : at + (long long)item_pages(a, i) * a.per_item;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          const long long s = u0 + nu * v / kWaves;
          if (s >= at && s < next) s_item[v] = i, s_base[v] = at;
        }
        at = next;
      }
    }
  }
  __syncthreads();
  const long long my0 = u0 + nu * wv / kWaves, my1 = u0 + nu * (wv + 1) / kWaves;

  // ---- this wave's pages, row by row --------------------------------------
  int rem = (int)(my1 - my0);   // at most B * Hq * 16384 / 2048
  int item = 0, sub = 0, n = 0, p = 0;
  if (rem > 0) {
    item = uniform(s_item[wv]);
    const unsigned off = (unsigned)(my0 - uniform64(s_base[wv]));
    n = uniform(item_pages(a, item));
    sub = (int)(off / (unsigned)n);
    p = (int)(off - (unsigned)sub * (unsigned)n);
  }
  // element offsets of the lane's loads in a page
  const uint32_t k_off = (uint32_t)((8 * (col >> 2) + (col & 3)) * D + 8 * grp);
  const uint32_t v_off = VT ? (uint32_t)(col * kPage + 8 * grp) : (uint32_t)(lane * 8);
  char* const stage = reinterpret_cast<char*>(&s_frag[wv][1][0]);

  while (rem > 0) {
    const int cnt = rem < n - p ? rem : n - p;
    const bool starts = p == 0, ends = p + cnt == n;
    int b, g, ht;
    if (l.kv_indptr) b = item / a.G, g = item - b * a.G, ht = sub;
    else b = item, g = sub / a.HT, ht = sub - g * a.HT;
    const int kvh = (int)((long long)g * l.group_size / (a.Hq / a.Hkv));
    const int h0 = g * l.group_size + ht * kTileHeads;
    int heads = l.group_size - ht * kTileHeads;
    heads = heads < kTileHeads ? heads : kTileHeads;
    const int len = uniform(request_len(a, b)), nkb = blocks_for(len);
    const int32_t* const table = l.page_table + ((long long)b * a.Hkv + kvh) * a.max_kv_blocks;
    const int32_t* const list = l.kv_indptr ? l.kv_indices + l.kv_indptr[item] : nullptr;

    // ids of 64 pages at a time, one per lane; keys: how many of a page count
    int ids, keys_of, next_ids = 0, next_keys = 0;
    auto fetch_ids = [&](int at, int& id, int& keys) {
      id = 0, keys = 0;
      if (at + lane < cnt) {
        const int j = list ? list[p + at + lane] : p + at + lane;
        if (j >= 0 && j < nkb) {
          const int page = table[j];
          if (page >= 0 && page < a.num_pages) {
            id = page;
            keys = len - j * kPage < kPage ? len - j * kPage : kPage;
          }
        }
      }
    };
    fetch_ids(0, ids, keys_of);

    bf16x8 q[NK];
    {
      const int head = DUP ? (col & 7) : col;
      const uint16_t* src = l.q + ((long long)b * a.Hq + h0 + head) * D + 8 * grp;
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        u32x4 x = {0, 0, 0, 0};
        if (head < heads) x = *reinterpret_cast<const u32x4*>(src + 32 * s);
        q[s] = __builtin_bit_cast(bf16x8, x);
      }
    }
    u32x4 k[4][NK], v[NL];
    auto load_k = [&](int id) {
      const uint16_t* page = l.k_pool + (long long)id * (kPage * D);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int s = 0; s < NK; ++s)
          k[t][s] = *reinterpret_cast<const u32x4*>(page + k_off + key_of(t, 0) * D + 32 * s);
    };
    auto load_v = [&](int id) {
      const uint16_t* page = l.v_pool + (long long)id * (kPage * D);
#pragma unroll
      for (int m = 0; m < NL; ++m)   // VT: d tile m / 2, 32-key step m % 2
        v[m] = *reinterpret_cast<const u32x4*>(
            page + v_off + (VT ? 16 * kPage * (m >> 1) + 32 * (m & 1) : 512 * m));
    };
    f32x4 o[NX];
#pragma unroll
    for (int x = 0; x < NX; ++x) o[x] = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, sum = 0.f;   // m: of q.k, before the scale

    int id = __builtin_amdgcn_readlane(ids, 0), keys = __builtin_amdgcn_readlane(keys_of, 0);
    load_k(id);
    load_v(id);
    for (int i = 0; i < cnt; ++i) {
      if ((i & 63) == 0) fetch_ids(i + 64, next_ids, next_keys);
      int id2 = 0, keys2 = 0;
      if ((i & 63) == 63) ids = next_ids, keys_of = next_keys;
      id2 = __builtin_amdgcn_readlane(ids, (i + 1) & 63);
      keys2 = __builtin_amdgcn_readlane(keys_of, (i + 1) & 63);
      f32x4 s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) s[t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NK; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][c]), q[c],
                                                         s[t], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < cnt) load_k(id2);
      __builtin_amdgcn_sched_barrier(0);
      if (keys < kPage) {   // the last page, or one that is not there
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key_of(t, 0) + 8 * grp + e >= keys) s[t][e] = -INFINITY;
        // weights of 0 do not undo a NaN in V
#pragma unroll
        for (int x = 0; x < NL; ++x) {
          if constexpr (VT) {
            const int first = 32 * (x & 1) + 8 * grp;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (first + 2 * e >= keys) v[x][e] = 0;
              else if (first + 2 * e + 1 >= keys) v[x][e] &= 0xffffu;
            }
          } else {
            if ((512 * x + 8 * lane) / D >= keys) v[x] = {0, 0, 0, 0};
          }
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max2(top, s[t][e]);
      const float mn = max2(m, groups_max(top));
      const float base = mn == -INFINITY ? 0.f : mn * a.scale_log2;
      const float alpha = fast_exp2(m * a.scale_log2 - base);
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
      bf16x8 pt[2];
      const float keep = DUP && col >= 8 ? 1.f : 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[2 * c + (e >> 2)][e & 3];
          // weights to bf16: to 8 bits, or with the upper columns to 16
          const __bf16 hi = (__bf16)x;
          pt[c][e] = DUP ? (__bf16)__builtin_fmaf(-keep, (float)hi, x) : hi;
        }
#pragma unroll
      for (int x = 0; x < NX; ++x) o[x] *= alpha;
      if constexpr (VT) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int x = 0; x < NX; ++x)
            o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, v[2 * x + c]), pt[c], o[x], 0, 0, 0);
      } else {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int y = 0; y < NL / 2; ++y) {
            const int e = 512 * y + 8 * lane, r = e / D, ch = (e % D) / 8;
            *reinterpret_cast<u32x4*>(stage + r * D * 2 + 16 * v_swz<D>(r, ch)) = v[c * (NL / 2) + y];
          }
          __builtin_amdgcn_wave_barrier();
          const int r0 = 8 * grp + (col >> 2);
#pragma unroll
          for (int x = 0; x < NX; ++x) {
            const int d = 16 * x + 4 * (col & 3);
            const char* src = stage + r0 * D * 2 + 16 * v_swz<D>(r0, d >> 3) + 2 * (d & 7);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src);
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 4 * D * 2));
            const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
            const u32x4 f = {l2[0], l2[1], h2[0], h2[1]};
            o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pt[c],
                                                           o[x], 0, 0, 0);
          }
          __builtin_amdgcn_wave_barrier();
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < cnt) load_v(id2);
      keys = keys2;
    }

    sum = groups_sum(sum);
    if constexpr (DUP)
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] += other_half(o[x][e]);
    const float ml = m * a.scale_log2;
    if (starts && ends) {
      if (col < heads) {
        const long long row = (long long)b * a.Hq + h0 + col;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // sum is NaN after a score of NaN or +inf
#pragma unroll
        for (int x = 0; x < NX; ++x)
          *reinterpret_cast<u32x2*>(l.out + row * D + 16 * x + 4 * grp) =
              u32x2{pack_bf16x2(o[x][0] * inv, o[x][1] * inv), pack_bf16x2(o[x][2] * inv, o[x][3] * inv)};
        if (l.lse && grp == 0) l.lse[row] = sum > 0.f ? (ml + __log2f(sum)) * kLn2 : -INFINITY;
      }
    } else {
      const int f = starts ? 1 : 0;   // [1] is the wave's last: its stage is free
#pragma unroll
      for (int x = 0; x < NX; ++x)
        s_frag[wv][f][64 * x + lane] = make_float4(o[x][0], o[x][1], o[x][2], o[x][3]);
      if (grp == 0) s_ml[wv][f][col] = make_float2(ml, sum);
      if (lane == 0) s_meta[wv][f] = make_int4(item, sub, (starts ? 1 : 0) | (ends ? 2 : 0), 1);
    }
    rem -= cnt;
    p = 0;
    if (rem > 0 && ++sub == a.per_item) {
      sub = 0;
      do n = ++item < a.items ? uniform(item_pages(a, item)) : -1; while (n == 0);
      if (n < 0) break;   // only if the lengths changed under the kernel
    }
  }
  __syncthreads();

  // ---- the waves' pieces, row by row -----------------------------------------
  long long row_end = 0;
  int next_row = 0, next_heads = 0;
  for (int f = 0; f < 2 * kWaves;) {
    const int4 meta = s_meta[f >> 1][f & 1];
    if (!meta.w) {
      ++f;
      continue;
    }
    int last = f, flags = meta.z;
    for (int e = f + 1; e < 2 * kWaves; ++e) {
      const int4 other = s_meta[e >> 1][e & 1];
      if (!other.w) continue;
      if (other.x != meta.x || other.y != meta.y) break;
      last = e;
      flags |= other.z & 2;
    }
    int b, g, ht;
    if (l.kv_indptr) b = meta.x / a.G, g = meta.x - b * a.G, ht = meta.y;
    else b = meta.x, g = meta.y / a.HT, ht = meta.y - g * a.HT;
    const int h0 = g * l.group_size + ht * kTileHeads;
    int heads = l.group_size - ht * kTileHeads;
    heads = heads < kTileHeads ? heads : kTileHeads;
    const long long row = (long long)b * a.Hq + h0 + col;
    if (wv < NX) {
      float top = -INFINITY, all = 0.f;
      for (int e = f; e <= last; ++e)
        if (s_meta[e >> 1][e & 1].w) top = max2(top, s_ml[e >> 1][e & 1][col].x);
      const float base = top == -INFINITY ? 0.f : top;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int e = f; e <= last; ++e) {
        if (!s_meta[e >> 1][e & 1].w) continue;
        const float2 ml = s_ml[e >> 1][e & 1][col];
        const float4 x = s_frag[e >> 1][e & 1][64 * wv + lane];
        const float c = fast_exp2(ml.x - base);
        all += c * ml.y;
        acc.x += c * x.x, acc.y += c * x.y, acc.z += c * x.z, acc.w += c * x.w;
      }
      if (flags == 3) {
        if (col < heads) {
          const float inv = all == 0.f ? 0.f : 1.f / all;
          *reinterpret_cast<u32x2*>(l.out + row * D + 16 * wv + 4 * grp) =
              u32x2{pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)};
          if (l.lse && wv == 0 && grp == 0)
            l.lse[row] = all > 0.f ? (top + __log2f(all)) * kLn2 : -INFINITY;
        }
      } else {   // [1]: the row starts here and goes on; [0]: it started before
        const int slot = 2 * w + (flags & 1);
        a.part_o[(long long)slot * kFrag + 64 * wv + lane] = acc;
        if (wv == 0 && grp == 0) a.part_ml[slot * kTileHeads + col] = make_float2(top, all);
      }
    }
    if (flags == 1 && tid == 0) {
      // where the row ends: its item's first page, and the rows of the item before it
      const int v = last >> 1;
      const int pages = item_pages(a, meta.x);
      long long base = s_base[v];
      // s_base is of the item that wave v starts in; walk to the piece's
      for (int i = s_item[v]; i < meta.x; ++i) base += (long long)item_pages(a, i) * a.per_item;
      row_end = base + (long long)(meta.y + 1) * pages;
      next_row = (int)((long long)b * a.Hq + h0);
      next_heads = heads;
    }
    f = last + 1;
  }
  if (tid == 0) a.shares[w] = Share{row_end, total, next_row, next_heads};

  // ---- requests and rows without a page -----------------------------------
  for (int i = w; i < a.items; i += kGroups) {
    if (item_pages(a, i) > 0) continue;
    const int nh = a.Hq / (l.kv_indptr ? a.G : 1);
    const long long row = l.kv_indptr ? (long long)(i / a.G) * a.Hq + (long long)(i % a.G) * nh
                                      : (long long)i * a.Hq;
    for (int x = tid; x < nh * (D / 8); x += kThreads)
      reinterpret_cast<u32x4*>(l.out + row * D)[x] = u32x4{0, 0, 0, 0};
    if (l.lse)
      for (int x = tid; x < nh; x += kThreads) l.lse[row + x] = -INFINITY;
  }
}

// Rows that several workgroups share: workgroup (w, x) joins d tile x of the
// row that starts in share w and goes on after it; its waves take the pieces in
// turn, and are joined in LDS.
template <int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const DecodeArgs a) {
  constexpr int kFrag = D / 16 * 64;
  __shared__ float4 s_o[kWaves][64];
  __shared__ float2 s_ml[kWaves][kTileHeads];
  const int w = blockIdx.x, x = blockIdx.y;
  const Share s = a.shares[w];
  if (s.row_end == 0) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
  float top = -INFINITY, all = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, float4 o) {
    const float mn = max2(top, ml.x), base = mn == -INFINITY ? 0.f : mn;
    const float c0 = fast_exp2(top - base), c1 = fast_exp2(ml.x - base);
    all = all * c0 + ml.y * c1;
    acc.x = acc.x * c0 + o.x * c1, acc.y = acc.y * c0 + o.y * c1;
    acc.z = acc.z * c0 + o.z * c1, acc.w = acc.w * c0 + o.w * c1;
    top = mn;
  };
  for (int e = w + wv; e < kGroups && (e == w || share_start(s.total, e) < s.row_end); e += kWaves) {
    const int slot = 2 * e + (e == w ? 1 : 0);
    add(a.part_ml[slot * kTileHeads + col], a.part_o[(long long)slot * kFrag + 64 * x + lane]);
  }
  s_o[wv][lane] = acc;
  if (grp == 0) s_ml[wv][col] = make_float2(top, all);
  __syncthreads();
  if (wv > 0) return;
  for (int e = 1; e < kWaves; ++e) add(s_ml[e][col], s_o[e][lane]);
  if (col >= s.heads) return;
  const long long row = (long long)s.out_row + col;
  const float inv = all == 0.f ? 0.f : 1.f / all;
  *reinterpret_cast<u32x2*>(a.l.out + row * D + 16 * x + 4 * grp) =
      u32x2{pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)};
  if (a.l.lse && x == 0 && grp == 0)
    a.l.lse[row] = all > 0.f ? (top + __log2f(all)) * kLn2 : -INFINITY;
}

template <int D, bool VT>
hipError_t launch(const DecodeArgs& a, hipStream_t st) {
  if (a.l.group_size <= 8) decode_kernel<D, VT, true><<<kGroups, kThreads, 0, st>>>(a);
  else decode_kernel<D, VT, false><<<kGroups, kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  decode_join_kernel<D><<<dim3(kGroups, D / 16), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t decode_ws_bytes(const CacheDims& d, int) {
  return (size_t)kGroups * (2 * kTileHeads * (d.D * sizeof(float) + sizeof(float2)) + sizeof(Share));
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
  a.part_o = static_cast<float4*>(l.ws);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)kGroups * 2 * kTileHeads * d.D / 4);
  a.shares = reinterpret_cast<Share*>(a.part_ml + (size_t)kGroups * 2 * kTileHeads);
  const bool vt = d.v_layout != 0;
  if (d.D == 64) return vt ? launch<64, true>(a, st) : launch<64, false>(a, st);
  return vt ? launch<128, true>(a, st) : launch<128, false>(a, st);
}

}  // namespace ca
