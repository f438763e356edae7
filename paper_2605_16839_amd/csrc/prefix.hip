// Attention of one new token per request where requests share prefixes: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// over the share's whole pages (through its first member's row) and the request's own.
//
// One workgroup to a (request, head), vector arithmetic: 256 keys at a time.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PrefixArgs {
  PrefixLaunch l;
  int B, Hq, Hkv, D, max_kv_blocks, num_pages;
  bool vt;
};

__global__ __launch_bounds__(kThreads) void prefix_kernel(const PrefixArgs a) {
  __shared__ float s_q[128], s_p[kThreads], s_red[kThreads], s_o[kThreads];
  __shared__ int s_first;
  const PrefixLaunch& l = a.l;
  const int tid = threadIdx.x, b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, D = a.D;
  const int kvh = h / (a.Hq / a.Hkv), most = a.max_kv_blocks * kPage;
  auto len_of = [&](int i) {
    const int n = l.kv_len[i];
    return n < 0 ? 0 : (n < most ? n : most);
  };
  const int len = len_of(b);
  int skip = 0, share = -1;
  if (l.num_shares > 0) share = l.share[b];
  if (share >= 0 && share < l.num_shares) {
    skip = l.share_len[share] / kPage;
    skip = skip < 0 ? 0 : (skip < a.max_kv_blocks ? skip : a.max_kv_blocks);
    if (len < skip * kPage) skip = 0;
  }
  if (tid == 0) s_first = b;
  if (tid < D) s_q[tid] = bf16_bits_to_float(l.q[((long long)b * a.Hq + h) * D + tid]);
  __syncthreads();
  if (skip > 0)
    for (int i = tid; i < b; i += kThreads)
      if (l.share[i] == share && len_of(i) >= skip * kPage) atomicMin(&s_first, i);
  __syncthreads();
  const int first = s_first;
  const int dim = tid % D, part = tid / D, parts = kThreads / D;
  float m = -INFINITY, sum = 0.f, acc = 0.f;
  auto page_of = [&](int j) {
    const int row = j < skip ? first : b;
    const int page = l.page_table[((long long)row * a.Hkv + kvh) * a.max_kv_blocks + j];
    return page >= 0 && page < a.num_pages ? page : -1;
  };
  for (int k0 = 0; k0 < len; k0 += kThreads) {
    const int key = k0 + tid, page = key < len ? page_of(key / kPage) : -1;
    float x = -INFINITY;
    if (page >= 0) {
      const uint16_t* k = l.k_pool + ((long long)page * kPage + key % kPage) * D;
      x = 0.f;
      for (int d = 0; d < D; d += 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(k + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) x += s_q[d + 2 * e] * bf16_lo(w[e]) + s_q[d + 2 * e + 1] * bf16_hi(w[e]);
      }
      x *= l.sm_scale * kLog2e;
    }
    s_red[tid] = x;
    __syncthreads();
    for (int o = kThreads / 2; o > 0; o >>= 1) {
      if (tid < o) s_red[tid] = __builtin_elementwise_maximum(s_red[tid], s_red[tid + o]);
      __syncthreads();
    }
    const float mn = __builtin_elementwise_maximum(m, s_red[0]), base = mn == -INFINITY ? 0.f : mn;
    const float alpha = exp2f(m - base), p = exp2f(x - base);
    m = mn;
    s_p[tid] = p;
    __syncthreads();
    s_red[tid] = p;
    __syncthreads();
    for (int o = kThreads / 2; o > 0; o >>= 1) {
      if (tid < o) s_red[tid] += s_red[tid + o];
      __syncthreads();
    }
    sum = sum * alpha + s_red[0];
    acc *= alpha;
    const int n = len - k0 < kThreads ? len - k0 : kThreads;
    for (int i = part; i < n; i += parts) {
      const int pg = page_of((k0 + i) / kPage);
      if (pg < 0) continue;
      const long long at = (long long)pg * kPage * D;
      const int r = (k0 + i) % kPage;
      acc += s_p[i] * bf16_bits_to_float(l.v_pool[at + (a.vt ? dim * kPage + r : r * D + dim)]);
    }
    __syncthreads();
  }
  s_o[tid] = acc;
  __syncthreads();
  if (tid < D) {
    for (int i = 1; i < parts; ++i) acc += s_o[tid + i * D];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    l.out[((long long)b * a.Hq + h) * D + tid] = float_to_bf16_bits(acc * inv);
  }
  if (tid == 0 && l.lse)
    l.lse[(long long)b * a.Hq + h] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

}  // namespace

size_t prefix_ws_bytes(const CacheDims&) { return 16; }

hipError_t launch_prefix(const CacheDims& d, const PrefixLaunch& l, hipStream_t st) {
  const PrefixArgs a = {l, d.B, d.Hq, d.Hkv, d.D, d.max_kv_blocks, d.num_pages, d.v_layout != 0};
  prefix_kernel<<<d.B * d.Hq, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
