// Attention of one new token per request over its paged cache: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// in one pass over the keys with the running maximum m and sum.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kDecodeThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeArgs {
  DecodeLaunch l;
  int B, Hq, Hkv, G, max_kv_blocks, num_pages;
  bool v_transposed;
  float scale_log2;
};

// One workgroup per (request, query head); a wave takes every fourth page, a
// lane one key of it for the scores and D / 64 dimensions for the sum.
template <int D>
__global__ __launch_bounds__(kDecodeThreads) void decode_kernel(const DecodeArgs a) {
  constexpr int NW = kDecodeThreads / kWave, DL = D / kWave;
  __shared__ float s_q[D], s_p[NW][kPage], s_o[NW][D], s_m[NW], s_l[NW];
  const DecodeLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
  const int kvh = h / (a.Hq / a.Hkv);
  if (tid < D) s_q[tid] = bf16_bits_to_float(l.q[(long long)blockIdx.x * D + tid]) * a.scale_log2;
  __syncthreads();
  int len = l.kv_len[b];
  len = len < 0 ? 0 : (len > a.max_kv_blocks * kPage ? a.max_kv_blocks * kPage : len);
  const int nkb = blocks_for(len);
  int n = nkb;
  long long at = 0;
  if (l.kv_indptr) {
    const long long r = (long long)b * a.G + h / l.group_size;
    const long long cap = (long long)a.B * a.G * a.max_kv_blocks;
    at = l.kv_indptr[r];
    n = l.kv_indptr[r + 1] - (int)at;
    if (at < 0 || n < 0 || n > a.max_kv_blocks || at + n > cap) n = 0;
  }
  float m = -INFINITY, sum = 0.f, o[DL] = {};
  for (int i = wv; i < n; i += NW) {
    const int j = l.kv_indptr ? l.kv_indices[at + i] : i;
    if (j < 0 || j >= nkb) continue;
    const int page = l.page_table[((long long)b * a.Hkv + kvh) * a.max_kv_blocks + j];
    if (page < 0 || page >= a.num_pages) continue;
    const int keys = len - j * kPage < kPage ? len - j * kPage : kPage;
    float x = -INFINITY;
    if (lane < keys) {
      const uint16_t* k = l.k_pool + ((long long)page * kPage + lane) * D;
      x = 0.f;
      for (int d = 0; d < D; ++d) x += s_q[d] * bf16_bits_to_float(k[d]);
    }
    float top = x;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
      const float y = __shfl_xor(top, s, kWave);
      top = __builtin_elementwise_maximum(top, y);   // a NaN stays
    }
    const float mn = __builtin_elementwise_maximum(m, top);
    const float base = mn == -INFINITY ? 0.f : mn;
    const float p = exp2f(x - base), alpha = exp2f(m - base);
    sum = sum * alpha + wave_sum(p);
    m = mn;
    s_p[wv][lane] = p;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < DL; ++e) o[e] *= alpha;
    for (int r = 0; r < keys; ++r)
#pragma unroll
      for (int e = 0; e < DL; ++e) {
        const int d = e * kWave + lane;
        const uint16_t v = a.v_transposed ? l.v_pool[((long long)page * D + d) * kPage + r]
                                          : l.v_pool[((long long)page * kPage + r) * D + d];
        o[e] += s_p[wv][r] * bf16_bits_to_float(v);
      }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int e = 0; e < DL; ++e) s_o[wv][e * kWave + lane] = o[e];
  if (lane == 0) s_m[wv] = m, s_l[wv] = sum;
  __syncthreads();
  if (tid < D) {
    float top = s_m[0], all = 0.f, acc = 0.f;
    for (int w = 1; w < NW; ++w) top = __builtin_elementwise_maximum(top, s_m[w]);
    const float base = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < NW; ++w) {
      const float f = exp2f(s_m[w] - base);
      all += f * s_l[w];
      acc += f * s_o[w][tid];
    }
    // a score of NaN or +inf: all is NaN
    const float y = all == 0.f ? 0.f : acc / all;
    l.out[(long long)blockIdx.x * D + tid] = float_to_bf16_bits(y);
    if (l.lse && tid == 0)
      l.lse[blockIdx.x] = all > 0.f ? (top + log2f(all)) * kLn2 : -INFINITY;
  }
}

}  // namespace

size_t decode_ws_bytes(const CacheDims&, int) { return 0; }

hipError_t launch_decode(const CacheDims& d, const DecodeLaunch& l, hipStream_t st) {
  DecodeArgs a{l, d.B, d.Hq, d.Hkv, d.Hq / l.group_size, d.max_kv_blocks, d.num_pages,
               d.v_layout != 0, l.sm_scale * kLog2e};
  const int grid = d.B * d.Hq;
  if (d.D == 64) decode_kernel<64><<<grid, kDecodeThreads, 0, st>>>(a);
  else decode_kernel<128><<<grid, kDecodeThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
