// Rotary positions and the cache write of a serving step, in one pass.
//
// Pair i of every head turns by angle_i = position[axis(i)] * inv_freq[i].  In
// fp32 the product of a far position loses its place in the turn (2^17 rad has
// steps of 2^-7), so the turn angle / 2 pi is formed in double, its whole part
// dropped there, and only the rest (at most half a turn) goes to fp32, where
// cosine and sine are taken and the pair is rotated; the result is rounded once.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kAppendThreads = 256;
constexpr double kTurnsPerRadian = 0.15915494309189533576888;

struct AppendArgs {
  AppendLaunch l;
  int Hq, Hkv, D;
  long long num_slots;
  bool v_transposed;
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

// One workgroup per token.
__global__ __launch_bounds__(kAppendThreads) void rotary_append_kernel(const AppendArgs a) {
  __shared__ float s_cos[kMaxPairs], s_sin[kMaxPairs];
  const AppendLaunch& l = a.l;
  const int tid = threadIdx.x, D = a.D, half = l.rot_dim / 2;
  const long long t = blockIdx.x;
  if (tid < half) {
    const int axis = (int)(l.pair_axis[tid >> 5] >> (2 * (tid & 31))) & 3;
    const int pos = l.positions[(long long)axis * l.num_tokens + t];
    const double turns = (double)pos * ((double)l.inv_freq[tid] * kTurnsPerRadian);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    s_cos[tid] = c;
    s_sin[tid] = s;
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
  AppendArgs a{l, d.Hq, d.Hkv, d.D, (long long)d.num_pages * kPage, d.v_layout != 0};
  rotary_append_kernel<<<l.num_tokens, kAppendThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
