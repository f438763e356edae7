// Internal launcher interface of the serving step (slots, rotary append, decode
// attention) between the C ABI (api.hip) and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ca {

// Validated ca_cache.
struct CacheDims {
  int B, Hq, Hkv, D, max_kv_blocks, num_pages, v_layout;
};

struct SlotLaunch {
  const int32_t* step;       // new_len (assign) or the release flags
  const int32_t* seq_len;
  int32_t* page_table;
  int32_t* free_pages;       // read by assign, written by release
  const int32_t* free_count;
  int64_t* slot_map;
  int32_t* positions;
  int32_t* token_indptr;
  int32_t* granted;
  int32_t* seq_len_out;
  int32_t* free_count_out;
  int free_capacity, num_tokens;
};
hipError_t launch_assign_slots(const CacheDims& d, const SlotLaunch& a, hipStream_t st);
hipError_t launch_release_pages(const CacheDims& d, const SlotLaunch& a, hipStream_t st);

constexpr int kMaxPairs = 64;   // rot_dim / 2 <= 64

struct AppendLaunch {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  long long q_stride, k_stride, v_stride;
  const int32_t* positions;
  const int64_t* slot_map;
  const float* inv_freq;
  uint16_t* q_out;
  uint16_t* k_pool;
  uint16_t* v_pool;
  int num_tokens, rot_dim, num_axes;
  bool interleaved;
  uint64_t pair_axis[2];   // 2 bits per pair
};
hipError_t launch_rotary_append(const CacheDims& d, const AppendLaunch& a, hipStream_t st);

struct DecodeLaunch {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* page_table;
  const int32_t* kv_len;
  const int32_t* kv_indptr;    // nullptr: every block
  const int32_t* kv_indices;
  uint16_t* out;
  float* lse;
  void* ws;
  int group_size;
  float sm_scale;
};
size_t decode_ws_bytes(const CacheDims& d);
hipError_t launch_decode(const CacheDims& d, const DecodeLaunch& a, hipStream_t st);

}  // namespace ca
