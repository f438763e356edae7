// Rotary positions and the cache write of a serving step, in one pass.
//
// Pair i of every head turns by angle_i = position[axis(i)] * inv_freq[i].  In
// fp32 the product of a far position loses its place in the turn (2^17 rad has
// steps of 2^-7), so the turn angle / 2 pi is formed in double, its whole part
// dropped there, and only the rest (at most half a turn) goes to fp32, where
// cosine and sine are taken and the pair is rotated; the result is rounded once.
//
// What bounds it: every element is read and written once, so HBM does, and the
// latency of positions, turns and rows one after the other with few tokens.  8192
// tokens of 32/8 heads, D = 128: 36 us, 5.6 TB/s (a large copy reaches 5.2 here).
// Transposed V pages want 64 tokens of a dimension side by side: tiles of 64 tokens
// are turned over in LDS and leave in runs of 8 slots (4353 tokens: 38 us with
// 2-byte stores, 20 with tiles).
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kMinTileTokens = 512;
constexpr double kTurnsPerRadian = 0.15915494309189533576888;

struct AppendArgs {
  AppendLaunch l;
  int Hq, Hkv, D;
  long long num_slots;
  bool v_transposed;
  int v_tiles;
};

__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[2 * e] = bf16_lo(w[e]), x[2 * e + 1] = bf16_hi(w[e]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  *reinterpret_cast<u32x4*>(p) = w;
}

// 64 tokens of a KV head's values into transposed pages.  A run is 8 tokens whose
// slots follow one another from a multiple of 8 on: 16 bytes of a page row.
constexpr int kTileTokens = 64;
constexpr int kTileDims = 64;
struct Tile {
  uint32_t v[kTileTokens][kTileDims / 2 + 1];   // + 1: 8 tokens on is 8 banks on
  long long slot[kTileTokens];
  int runs, alone;                  // how many there are, and
  uint8_t run[kTileTokens / 8];     // the first token of each run,
  uint8_t lone[kTileTokens];        // the tokens that are in none
};
__device__ __forceinline__ void transposed_tile(const AppendArgs& a, int tile, Tile& s) {
  const AppendLaunch& l = a.l;
  const int tid = threadIdx.x, slices = a.D / kTileDims;
  const int slice = tile % slices, head = tile / slices % a.Hkv;
  const long long t0 = (long long)(tile / slices / a.Hkv) * kTileTokens;
  const int n = l.num_tokens - t0 < kTileTokens ? (int)(l.num_tokens - t0) : kTileTokens;
  if (tid < kWave) {   // one wave: lane i has token i
    long long slot = -1;
    if (tid < n) slot = l.slot_map[(t0 + tid) * a.Hkv + head];
    if (slot < 0 || slot >= a.num_slots) slot = -1;
    s.slot[tid] = slot;
    // follows: the next token has the next slot
    const long long next = __shfl_down(slot, 1, kWave);   // of every lane, so before any condition
    const unsigned long long follows = __ballot(slot >= 0 && next == slot + 1);
    const bool starts = slot >= 0 && slot % 8 == 0 && tid <= kTileTokens - 8 &&
                        ((follows >> tid) & 0x7f) == 0x7f;
    const unsigned long long runs = __ballot(starts);
    unsigned long long in = runs;   // runs do not overlap: they start 8 slots apart
    in |= in << 1, in |= in << 2, in |= in << 4;
    const unsigned long long alone = __ballot(slot >= 0) & ~in;
    const unsigned long long before = (1ull << tid) - 1;
    if (starts) s.run[__popcll(runs & before)] = tid;
    if ((alone >> tid) & 1) s.lone[__popcll(alone & before)] = tid;
    if (tid == 0) s.runs = __popcll(runs), s.alone = __popcll(alone);
  }
  const uint16_t* const src = l.v + t0 * l.v_stride + (long long)head * a.D + slice * kTileDims;
#pragma unroll
  for (int w = tid; w < kTileTokens * (kTileDims / 8); w += kAppendThreads) {
    const int i = w / (kTileDims / 8), c = w % (kTileDims / 8);
    if (i < n) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + i * l.v_stride + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) s.v[i][4 * c + e] = x[e];
    }
  }
  __syncthreads();
  auto row = [&](long long slot, int d) {   // element of dimension d of the slice
    return l.v_pool + (slot / kPage) * (kPage * a.D) + (long long)(slice * kTileDims + d) * kPage + slot % kPage;
  };
  // two dimensions of a run: neighbouring threads take neighbouring runs
  for (int w = tid; w < 8 * (kTileDims / 2); w += kAppendThreads) {
    const int r = w % 8, p = w / 8;
    if (r >= s.runs) continue;
    const int i0 = s.run[r];
    u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = s.v[i0 + 2 * e][p], y = s.v[i0 + 2 * e + 1][p];
      lo[e] = (x & 0xffffu) | (y << 16);
      hi[e] = (x >> 16) | (y & 0xffff0000u);
    }
    *reinterpret_cast<u32x4*>(row(s.slot[i0], 2 * p)) = lo;
    *reinterpret_cast<u32x4*>(row(s.slot[i0], 2 * p + 1)) = hi;
  }
  for (int w = tid; w < s.alone * (kTileDims / 2); w += kAppendThreads) {
    const int i = s.lone[w / (kTileDims / 2)], p = w % (kTileDims / 2);
    const uint32_t x = s.v[i][p];
    uint16_t* const to = row(s.slot[i], 2 * p);
    to[0] = (uint16_t)x;
    to[kPage] = (uint16_t)(x >> 16);
  }
}

// The first v_tiles workgroups take tiles of values, the others a token each.
__global__ __launch_bounds__(kAppendThreads) void rotary_append_kernel(const AppendArgs a) {
  __shared__ union {
    Tile tile;
    struct {
      float cos[kMaxPairs], sin[kMaxPairs];
    } turn;
  } s;
  if ((int)blockIdx.x < a.v_tiles) {
    transposed_tile(a, blockIdx.x, s.tile);
    return;
  }
  float* const s_cos = s.turn.cos;
  float* const s_sin = s.turn.sin;
  const AppendLaunch& l = a.l;
  const int tid = threadIdx.x, D = a.D, half = l.rot_dim / 2;
  const long long t = (int)blockIdx.x - a.v_tiles;
  if (tid < half) {
    const int axis = (int)(l.pair_axis[tid >> 5] >> (2 * (tid & 31))) & 3;
    const int pos = l.positions[(long long)axis * l.num_tokens + t];
    const double turns = (double)pos * ((double)l.inv_freq[tid] * kTurnsPerRadian);
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    s_cos[tid] = cs;
    s_sin[tid] = sn;
  }
  __syncthreads();

  // queries and keys: a work item is 8 pairs of a head (16 elements), or 16
  // elements past rot_dim
  const int per_head = D / 16, turned = half / 8;
  for (int w = tid; w < (a.Hq + a.Hkv) * per_head; w += kAppendThreads) {
    const int head = w / per_head, c = w - head * per_head;
    const bool key = head >= a.Hq;
    const uint16_t* src = key ? l.k + t * l.k_stride + (long long)(head - a.Hq) * D
                              : l.q + t * l.q_stride + (long long)head * D;
    uint16_t* dst;
    if (key) {
      const long long slot = l.slot_map[t * a.Hkv + head - a.Hq];
      if (slot < 0 || slot >= a.num_slots) continue;
      dst = l.k_pool + slot * D;
    } else {
      dst = l.q_out + (t * a.Hq + head) * D;
    }
    int o0, o1;
    if (c < turned && !l.interleaved) o0 = 8 * c, o1 = half + 8 * c;
    else o0 = 16 * c, o1 = 16 * c + 8;   // 8 pairs side by side, or 16 elements left alone
    float x[8], y[8];
    load8(src + o0, x);
    load8(src + o1, y);
    if (c < turned) {
      if (l.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float c0 = s_cos[8 * c + e], s0 = s_sin[8 * c + e];
          const float c1 = s_cos[8 * c + 4 + e], s1 = s_sin[8 * c + 4 + e];
          const float p = x[2 * e], q = x[2 * e + 1], r = y[2 * e], u = y[2 * e + 1];
          x[2 * e] = p * c0 - q * s0, x[2 * e + 1] = q * c0 + p * s0;
          y[2 * e] = r * c1 - u * s1, y[2 * e + 1] = u * c1 + r * s1;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float cs = s_cos[8 * c + e], sn = s_sin[8 * c + e];
          const float p = x[e], q = y[e];
          x[e] = p * cs - q * sn, y[e] = q * cs + p * sn;
        }
      }
    }
    store8(dst + o0, x);
    store8(dst + o1, y);
  }

  // values
  if (a.v_tiles > 0) return;
  const int chunks = D / 8;
  for (int w = tid; w < a.Hkv * chunks; w += kAppendThreads) {
    const int head = w / chunks, c = w - head * chunks;
    const long long slot = l.slot_map[t * a.Hkv + head];
    if (slot < 0 || slot >= a.num_slots) continue;
    const uint16_t* src = l.v + t * l.v_stride + (long long)head * D + 8 * c;
    const u32x4 x = *reinterpret_cast<const u32x4*>(src);
    if (a.v_transposed) {
      uint16_t* dst = l.v_pool + (slot / kPage) * kPage * D + (long long)(8 * c) * kPage + slot % kPage;
#pragma unroll
      for (int e = 0; e < 8; ++e) dst[e * kPage] = (uint16_t)(x[e / 2] >> (16 * (e & 1)));
    } else {
      *reinterpret_cast<u32x4*>(l.v_pool + slot * D + 8 * c) = x;
    }
  }
}

}  // namespace

hipError_t launch_rotary_append(const CacheDims& d, const AppendLaunch& l, hipStream_t st) {
  if (l.num_tokens == 0) return hipSuccess;
  AppendArgs a{l, d.Hq, d.Hkv, d.D, (long long)d.num_pages * kPage, d.v_layout != 0, 0};
  // Tiles pay where tokens lie in runs, which the host does not know; by their number a
  // prompt's chunk and a decode step's tokens, which lie in a page each, are told apart.
  // 32/8 heads, D = 128, without tiles and with: 512 tokens of a prompt 8.1 and 4.7 us, 2048
  // 18.7 and 10.7, 512 requests of 4 tokens 33.7 and 16.5; 512 single tokens 10.7 and 11.2, 2048
  // of them 35.6 and 34.9 (4/1 heads 4.3 and 5.5, 7.5 and 8.3).  Below, 256 of a prompt 5.9
  // and 4.1, and 64 single tokens, an ordinary step, 4.9 and 5.5.
  const long long tiles = (long long)(l.num_tokens + kTileTokens - 1) / kTileTokens * d.Hkv * (d.D / kTileDims);
  if (a.v_transposed && l.num_tokens >= kMinTileTokens && tiles <= 1 << 22) a.v_tiles = (int)tiles;
  rotary_append_kernel<<<a.v_tiles + l.num_tokens, kAppendThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
