// Internal launcher interface of the serving step (slots, rotary append, decode
// attention, requests that share pages) between the C ABI (api.hip) and the kernels.
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
  // norms of the heads (norm): nullptr weights leave a side as it is
  const void* q_weight;
  const void* k_weight;
  bool norm, weight_fp32;
  float weight_offset, eps;
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

constexpr int kForkRequests = (1 << 24) - 1;   // at most: a launch has fewer than 2^32 threads, 256 for a request

struct ForkLaunch {
  const int32_t* parent;
  const int32_t* keep_len;     // nullptr: all tokens
  const int32_t* seq_len;
  const int32_t* page_table;
  const int32_t* page_shares;
  const int32_t* free_pages;
  const int32_t* free_count;
  uint16_t* k_pool;
  uint16_t* v_pool;
  int32_t* seq_len_out;
  int32_t* page_table_out;
  int32_t* page_shares_out;
  int32_t* free_pages_out;
  int32_t* free_count_out;
  void* ws;
  int free_capacity;
};
size_t fork_ws_bytes(const CacheDims& d);
hipError_t launch_fork(const CacheDims& d, const ForkLaunch& a, hipStream_t st);

struct CompactLaunch {
  const int32_t* seq_len;
  const int32_t* page_table;
  const int32_t* page_shares;  // nullptr: none
  const int32_t* free_pages;
  const int32_t* free_count;
  uint16_t* k_pool;
  uint16_t* v_pool;
  int32_t* new_page;
  int32_t* page_table_out;
  int32_t* page_shares_out;
  int32_t* free_pages_out;
  int32_t* free_count_out;
  void* ws;
  int free_capacity;
};
size_t compact_ws_bytes(const CacheDims& d);
hipError_t launch_compact(const CacheDims& d, const CompactLaunch& a, hipStream_t st);

constexpr int kPrefixRequests = 2048;   // at most
constexpr int kPrefixShares = 512;
constexpr int kPrefixRows = 256;        // query rows of a tile

struct PrefixLaunch {
  const uint16_t* q;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* page_table;
  const int32_t* kv_len;
  const int32_t* share;
  const int32_t* share_len;
  uint16_t* out;
  float* lse;
  void* ws;
  int num_shares;
  float sm_scale;
};
size_t prefix_ws_bytes(const CacheDims& d);
hipError_t launch_prefix(const CacheDims& d, const PrefixLaunch& a, hipStream_t st);

}  // namespace ca
