// Requests that share pages: forks, and the pages that no one holds any more; a
// pool's pages moved together.
//
// Fork.  Request b goes on from row r = parent[b] as it was, with n of its tokens:
//   full_b = n / 64 whole pages are r's own ids; a part-filled last page is r's too for one of r's forks
//   at most, else a free page and a copy;
//   page_shares += (new holds of the page) - (old ones), over the rows that change; below 0: free.
// Three launches, since each needs all of the one before: the plan (one workgroup: who takes a page
// over, who gets free ones, by prefix sums in the requests' order), the new rows, counts and
// copies (workgroups by row: row r's workgroup also sums what its pages gain and lose
// by all of its forks, so a page takes one atomic of each row and not one of each fork), then the pages
// that have become free, in the order of their ids, and what is written in place.
//
// Compaction.  With U pages in use, the i-th used id from U on moves to the i-th free id
// below U; both ranks are prefix sums over the ids.  Small pools: FreeMap.
//
// What bounds them: latency, launch by launch; with many pages to copy HBM, read and write.  A prompt of
// 32741 tokens (8 KV heads of 128) for 64 requests: 15.7 us a call, of which plan 4.3 (one workgroup, its
// barriers), rows 7.4 (four loads that wait for each other, then 504 pages copied), free 3.1; in place 2 us more
// (rows are written twice), 16 prompts of 4 beams 17.0 and 5 more.  Compaction of a pool of 81K pages, half of them in use
// and 20K of those moved, 285 us, of which the moves 268: 1.33 GB at 5 TB/s; in place the same, a small pool
// 2 us more for its second launch.
#include "common.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kRowThreads = 256;
constexpr int kChunks = 256;       // of the page ids
constexpr int kMarks = 1024;       // entries of the free list that a workgroup takes together
constexpr int kLdsPages = 16384;   // a pool of so many is compacted by way of LDS
constexpr int kLdsRequests = 4096; // so many requests' marks lie in LDS

struct Plan {
  int src;      // the row it goes on from, -1: none
  int now, old; // tokens after and before
  int fresh;    // the first of its free pages counted from the list's end, -1: none
};

struct ForkArgs {
  ForkLaunch l;
  int B, Hkv, max_kv_blocks, num_pages, page_elems, chunk;
  bool in_place;          // the page table
  Plan* plan;             // [B]
  int2* mark;             // [B], where B > kLdsRequests
  int* chunk_freed;       // [kChunks]: pages of a chunk that no one holds any more
  int* used;              // [2]: free pages there were, and were taken
  int32_t* stage;         // [B, Hkv, max_kv_blocks]: rows that change, in place
};

__device__ __forceinline__ int length_of(int len, int max_kv_blocks) {
  return len < 0 || len > max_kv_blocks * kPage ? 0 : len;
}
__device__ __forceinline__ int free_count_of(const int32_t* count, int capacity) {
  const int n = count[0];
  return n < 0 ? 0 : (n < capacity ? n : capacity);
}
__device__ __forceinline__ bool changes(const Plan& p, int b) { return p.src != b || p.now != p.old; }

// Past the L1, which does not see the atomics.
__device__ __forceinline__ int now_at(const int* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Inclusive sum over the workgroup's threads, and its total.
__device__ __forceinline__ int block_sum(int v, int* part, int* all) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, waves = blockDim.x / kWave;
  v = wave_inclusive_scan(v);
  __syncthreads();   // of an earlier call's parts
  if (lane == kWave - 1) part[wv] = v;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < waves; ++w) {
    if (w < wv) before += part[w];
    total += part[w];
  }
  *all = total;
  return before + v;
}

// Workgroup 0 makes the plan, the others copy the counts where they are not in place.
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(const ForkArgs a) {
  __shared__ int2 s_mark[kLdsRequests];   // of a parent: most whole pages of a fork; who of those
  __shared__ int s_part[kPlanThreads / kWave];   // that end in a part-filled page takes it over
  const ForkLaunch& l = a.l;
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {
    for (long long p = (long long)(blockIdx.x - 1) * kPlanThreads + tid; p < a.num_pages;
         p += (long long)(gridDim.x - 1) * kPlanThreads)
      l.page_shares_out[p] = l.page_shares[p];
    return;
  }
  int2* const mark = a.B <= kLdsRequests ? s_mark : a.mark;
  for (int i = tid; i < kChunks; i += kPlanThreads) a.chunk_freed[i] = 0;
  for (int b = tid; b < a.B; b += kPlanThreads) {
    __hip_atomic_store(&mark[b].x, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&mark[b].y, INT32_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    Plan p = {l.parent[b], 0, length_of(l.seq_len[b], a.max_kv_blocks), -1};
    if (p.src < 0 || p.src >= a.B) p.src = -1;
    if (p.src >= 0) {
      p.now = length_of(l.seq_len[p.src], a.max_kv_blocks);
      if (l.keep_len) {
        const int keep = l.keep_len[b] > 0 ? l.keep_len[b] : 0;
        p.now = p.now < keep ? p.now : keep;
      }
      atomicMax(&mark[p.src].x, p.now / kPage);
    }
    a.plan[b] = p;
  }
  __syncthreads();
  // -1 for the parent itself, so that it comes before all others
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Plan p = a.plan[b];
    if (p.src >= 0 && p.now % kPage != 0 && p.now / kPage == now_at(&mark[p.src].x))
      atomicMin(&mark[p.src].y, p.src == b ? -1 : b);
  }
  __syncthreads();
  const int count = free_count_of(l.free_count, l.free_capacity);
  long long need0 = 0;
  int used = 0;   // in the thread whose request is the last that is served
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    Plan p = {-1, 0, 0, -1};
    bool copy = false;
    if (b < a.B) {
      p = a.plan[b];
      if (p.src >= 0 && p.now % kPage != 0 && changes(p, b)) {
        const int j = p.now / kPage;
        copy = now_at(&mark[p.src].x) > j || now_at(&mark[p.src].y) != (p.src == b ? -1 : b);
        const int32_t* at = l.page_table + (long long)p.src * a.Hkv * a.max_kv_blocks + j;
        for (int h = 0; !copy && h < a.Hkv; ++h) {
          const int page = at[(long long)h * a.max_kv_blocks];
          copy = page >= 0 && page < a.num_pages && l.page_shares[page] > 0;
        }
      }
    }
    int copies;
    const long long upto = need0 + (long long)block_sum(copy ? 1 : 0, s_part, &copies) * a.Hkv;
    if (copy && upto <= count) {
      p.fresh = (int)(upto - a.Hkv);
      used = (int)upto;
    } else if (copy) {
      p.now -= p.now % kPage;
    }
    if (b < a.B) a.plan[b] = p, l.seq_len_out[b] = p.now;
    need0 += (long long)copies * a.Hkv;
  }
  // the most that any thread has seen served
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const int other = __shfl_xor(used, o, kWave);
    used = used > other ? used : other;
  }
  __syncthreads();
  if ((tid & 63) == 0) s_part[tid >> 6] = used;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kPlanThreads / kWave; ++w) used = used > s_part[w] ? used : s_part[w];
    a.used[0] = count;
    a.used[1] = used;
  }
}

// A whole page of both pools, to another place: all loads before the first store, so that they wait together.
// The pages differ; thread: of kRowThreads.
__device__ __forceinline__ void copy_pages(uint16_t* k_pool, uint16_t* v_pool, int from, int to, int page_elems,
                                           int thread) {
  constexpr int N = kPage * 128 / 8 / kRowThreads;   // loads of a thread for a page of the largest heads
  const long long src = (long long)from * page_elems, dst = (long long)to * page_elems;
  u32x4 k[N], v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = 8 * (kRowThreads * i + thread);
    if (at >= page_elems) continue;
    k[i] = *reinterpret_cast<const u32x4*>(k_pool + src + at);
    v[i] = *reinterpret_cast<const u32x4*>(v_pool + src + at);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = 8 * (kRowThreads * i + thread);
    if (at >= page_elems) continue;
    *reinterpret_cast<u32x4*>(k_pool + dst + at) = k[i];
    *reinterpret_cast<u32x4*>(v_pool + dst + at) = v[i];
  }
}

// What the row's pages gain and lose by its forks.
__device__ __forceinline__ void fork_counts(const ForkArgs& a, int r, const Plan& me, int h0, int hs) {
  __shared__ int s_holds[1024];   // pages that each of the row's forks shares with it
  __shared__ int s_forks;
  const ForkLaunch& l = a.l;
  const int tid = threadIdx.x, old_blocks = blocks_for(me.old);
  for (int b0 = 0; b0 < a.B && old_blocks > 0; b0 += 1024) {
    __syncthreads();
    if (tid == 0) s_forks = 0;
    __syncthreads();
    for (int b = b0 + tid; b < a.B && b < b0 + 1024; b += kRowThreads) {
      const Plan p = a.plan[b];
      if (p.src == r && changes(p, b)) {
        const int n = p.fresh >= 0 ? p.now / kPage : blocks_for(p.now);
        if (n > 0) s_holds[atomicAdd(&s_forks, 1)] = n;   // in any order: they are counted
      }
    }
    __syncthreads();
    const int forks = s_forks, lost = b0 == 0 && changes(me, r) ? 1 : 0;
    if (forks == 0 && lost == 0) continue;
    for (int h = h0; h < a.Hkv; h += hs)
      for (int j = tid; j < old_blocks; j += kRowThreads) {
        const int page = l.page_table[((long long)r * a.Hkv + h) * a.max_kv_blocks + j];
        int gain = -lost;
#pragma unroll 8
        for (int i = 0; i < forks; ++i) gain += s_holds[i] > j ? 1 : 0;
        if (gain == 0 || page < 0 || page >= a.num_pages) continue;
        const int was = atomicAdd(l.page_shares_out + page, gain);
        const int freed = (was + gain < 0 ? 1 : 0) - (was < 0 ? 1 : 0);
        if (freed != 0) atomicAdd(a.chunk_freed + page / a.chunk, freed);
      }
  }
}

// A request's new entries, and the copy of its last page.
__device__ __forceinline__ void fork_entries(const ForkArgs& a, int r, const Plan& me, int h0, int hs) {
  const ForkLaunch& l = a.l;
  if (me.src < 0 || (a.in_place && !changes(me, r))) return;
  const int tid = threadIdx.x, blocks = blocks_for(me.now), count = a.used[0];
  int32_t* const to = a.in_place ? a.stage : l.page_table_out;
  for (int h = h0; h < a.Hkv; h += hs) {
    const long long mine = ((long long)r * a.Hkv + h) * a.max_kv_blocks;
    const int32_t* const old = l.page_table + ((long long)me.src * a.Hkv + h) * a.max_kv_blocks;
    int fresh = -1;
    if (me.fresh >= 0) {
      fresh = l.free_pages[count - 1 - (me.fresh + h)];
      const int from = old[blocks - 1];
      if (from >= 0 && from < a.num_pages && fresh >= 0 && fresh < a.num_pages && from != fresh)
        copy_pages(l.k_pool, l.v_pool, from, fresh, a.page_elems, tid);
    }
    for (int j = tid; j < blocks; j += kRowThreads)
      to[mine + j] = me.fresh >= 0 && j == blocks - 1 ? fresh : old[j];
  }
}

// blockIdx.x: the row, as a parent (blockIdx.z 0) or as a request (1); blockIdx.y: some of the KV heads.
__global__ __launch_bounds__(kRowThreads) void fork_rows_kernel(const ForkArgs a) {
  const Plan me = a.plan[blockIdx.x];
  if (blockIdx.z == 0) fork_counts(a, blockIdx.x, me, blockIdx.y, gridDim.y);
  else fork_entries(a, blockIdx.x, me, blockIdx.y, gridDim.y);
}

// Workgroup i: the pages of chunk i that have become free, its part of the free
// list, and of the rows that were made apart.
__global__ __launch_bounds__(kRowThreads) void fork_free_kernel(const ForkArgs a) {
  __shared__ int s_part[kRowThreads / kWave];
  const ForkLaunch& l = a.l;
  const int tid = threadIdx.x, c = blockIdx.x;
  const int left = a.used[0] - a.used[1];
  int all, mine;
  block_sum(tid < c ? a.chunk_freed[tid] : 0, s_part, &mine);
  block_sum(a.chunk_freed[tid], s_part, &all);
  int at = left + mine;
  const long long first = (long long)c * a.chunk;
  const long long last = first + a.chunk < a.num_pages ? first + a.chunk : a.num_pages;
  if (a.chunk_freed[c] > 0)
    for (long long p0 = first; p0 < last; p0 += kRowThreads) {
      const long long p = p0 + tid;
      const bool gone = p < last && l.page_shares_out[p] < 0;
      int n;
      const int place = at + block_sum(gone ? 1 : 0, s_part, &n) - 1;
      if (gone) {
        l.page_shares_out[p] = 0;
        // (below 0 where a count was below 0 before: such a page may be listed and not counted)
        if (place >= 0 && place < l.free_capacity) l.free_pages_out[place] = (int)p;
      }
      at += n;
    }
  if (l.free_pages_out != l.free_pages)
    for (long long i = (long long)c * kRowThreads + tid; i < left; i += kChunks * kRowThreads)
      l.free_pages_out[i] = l.free_pages[i];
  if (a.in_place)
    for (long long row = c; row < (long long)a.B * a.Hkv; row += kChunks) {
      const int b = (int)(row / a.Hkv);
      const Plan p = a.plan[b];
      if (!changes(p, b)) continue;
      const long long from = row * a.max_kv_blocks;
      for (int j = tid; j < blocks_for(p.now); j += kRowThreads)
        l.page_table_out[from + j] = a.stage[from + j];
    }
  if (c == 0 && tid == 0) {
    const long long n = (long long)left + all;
    l.free_count_out[0] = (int)(n < 0 ? 0 : (n < l.free_capacity ? n : l.free_capacity));
  }
}

// ---------------------------------------------------------------------------
struct CompactArgs {
  CompactLaunch l;
  int B, Hkv, max_kv_blocks, num_pages, page_elems, chunk;
  bool apart;        // the free list and its count after the call are not those before it
  int* free;         // [num_pages]: 1 for a free page
  int* from;         // [num_pages / 2 + 1]: the pages that move, ascending, and
  int* to;           // where they go
  int* chunk_free;   // [kChunks]
  int* count;        // [2]: pages in use, pages that move
};

__global__ __launch_bounds__(kRowThreads) void compact_clear_kernel(const CompactArgs a) {
  const long long i0 = (long long)blockIdx.x * kRowThreads + threadIdx.x;
  for (long long i = i0; i < a.num_pages; i += (long long)gridDim.x * kRowThreads) a.free[i] = 0;
  if (i0 < kChunks) a.chunk_free[i0] = 0;
}

// Counts of the chunks by way of LDS: with an atomic on a chunk's counter for every page, 41K free pages took
// 29 us, most of it in line for the counters; so 5.
__global__ __launch_bounds__(kRowThreads) void compact_mark_kernel(const CompactArgs a) {
  __shared__ int s_count[kChunks];
  const int n = free_count_of(a.l.free_count, a.l.free_capacity), tid = threadIdx.x;
  constexpr int N = kMarks / kRowThreads;
  s_count[tid] = 0;
  __syncthreads();
  for (long long i0 = (long long)blockIdx.x * kMarks; i0 < n; i0 += (long long)gridDim.x * kMarks) {
    int p[N], was[N];
#pragma unroll
    for (int y = 0; y < N; ++y) {
      const long long i = i0 + kRowThreads * y + tid;
      p[y] = i < n ? a.l.free_pages[i] : -1;
    }
#pragma unroll
    for (int y = 0; y < N; ++y) was[y] = p[y] >= 0 && p[y] < a.num_pages ? atomicExch(a.free + p[y], 1) : 1;
#pragma unroll
    for (int y = 0; y < N; ++y)
      if (was[y] == 0) atomicAdd(&s_count[p[y] / a.chunk], 1);
  }
  __syncthreads();
  if (s_count[tid] > 0) atomicAdd(a.chunk_free + tid, s_count[tid]);
}

// Workgroup i: the ranks in chunk i.
__global__ __launch_bounds__(kRowThreads) void compact_rank_kernel(const CompactArgs a) {
  __shared__ int s_part[kRowThreads / kWave];
  const int tid = threadIdx.x, c = blockIdx.x;
  int total, before, before_u;
  block_sum(a.chunk_free[tid], s_part, &total);
  block_sum(tid < c ? a.chunk_free[tid] : 0, s_part, &before);
  const int U = a.num_pages - total;   // the ids below it will be in use
  // free ids below U: whole chunks, and those of the chunk that U is in
  const int cu = U / a.chunk;
  block_sum(tid < cu ? a.chunk_free[tid] : 0, s_part, &before_u);
  int part = 0, there;
  for (long long p = (long long)cu * a.chunk + tid; p < U; p += kRowThreads) part += a.free[p] == 1 ? 1 : 0;
  block_sum(part, s_part, &there);
  const int moves = before_u + there;
  if (c == 0 && tid == 0) a.count[0] = U, a.count[1] = moves;
  const long long first = (long long)c * a.chunk;
  const long long last = first + a.chunk < a.num_pages ? first + a.chunk : a.num_pages;
  int at = before;
  for (long long p0 = first; p0 < last; p0 += kRowThreads) {
    const long long p = p0 + tid;
    const bool free = p < last && a.free[p] == 1;
    int n;
    const int upto = at + block_sum(free ? 1 : 0, s_part, &n);   // free ids up to p
    if (p < last) {
      if (free && p < U) a.to[upto - 1] = (int)p;
      if (!free && p >= U) a.from[(p - upto) - (U - moves)] = (int)p;
    }
    at += n;
  }
}

__global__ __launch_bounds__(kRowThreads) void compact_move_kernel(const CompactArgs a) {
  const CompactLaunch& l = a.l;
  const int tid = threadIdx.x, U = a.count[0], moves = a.count[1];
  const long long all = (long long)gridDim.x * kRowThreads, me = (long long)blockIdx.x * kRowThreads + tid;
  // the place of a page: the moved ones are found in `from`, which ascends
  auto place = [&](int p) {
    if (a.free[p] == 1) return -1;
    if (p < U) return p;
    int lo = 0, hi = moves;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.from[mid] <= p) lo = mid;
      else hi = mid;
    }
    return a.to[lo];
  };
  for (long long i = me; i < a.num_pages; i += all) {
    const int p = (int)i, at = place(p);
    l.new_page[p] = at;
    if (l.page_shares) {
      if (at >= 0) {
        const int n = l.page_shares[p];
        l.page_shares_out[at] = n;
      }
      if (p >= U) l.page_shares_out[p] = 0;
    }
    if (p >= U) l.free_pages_out[a.num_pages - 1 - p] = p;
  }
  const long long rows = (long long)a.B * a.Hkv;
  for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
    const int blocks = blocks_for(length_of(l.seq_len[row / a.Hkv], a.max_kv_blocks));
    for (int j = tid; j < blocks; j += kRowThreads) {
      const int p = l.page_table[row * a.max_kv_blocks + j];
      l.page_table_out[row * a.max_kv_blocks + j] = p >= 0 && p < a.num_pages ? place(p) : p;
    }
  }
  for (int i = blockIdx.x; i < moves; i += gridDim.x)
    copy_pages(l.k_pool, l.v_pool, a.from[i], a.to[i], a.page_elems, tid);
  if (me == 0) l.free_count_out[0] = a.num_pages - U;
}

// Pools of up to kLdsPages pages: every workgroup makes a map of the free ids in LDS, and takes its share
// of everything; neither marks nor ranks go by way of memory, and one launch does what four do else, two in
// place.  us so and with four, pages of 64 dimensions, half of them free: 300 pages 7.6 and 12.5, 4000 12.0 and
// 20.4, 16384 25.7 and 34.3, 65536 (twice the workgroups) 137 and 128; nearly all free: 16384 12.4 and 16.8,
// 65536 40 and 22, since every workgroup reads the whole free list.
struct FreeMap {
  uint32_t bits[kLdsPages / 32 + 1];   // 1: a free page
  int before[kLdsPages / 32 + 1];      // free ids before a word
  int words;

  __device__ __forceinline__ bool free(int p) const { return (bits[p >> 5] >> (p & 31) & 1) != 0; }
  __device__ __forceinline__ int free_below(int p) const {
    return before[p >> 5] + __popc(bits[p >> 5] & ((1u << (p & 31)) - 1));
  }
  // the r-th id (from 0) that is free, or used; there is one
  __device__ __forceinline__ int nth(int r, bool used) const {
    int lo = 0, hi = words;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((used ? 32 * mid - before[mid] : before[mid]) <= r) lo = mid;
      else hi = mid;
    }
    uint32_t left = used ? ~bits[lo] : bits[lo];
    for (int i = used ? 32 * lo - before[lo] : before[lo]; i < r; ++i) left &= left - 1;
    return 32 * lo + __ffs(left) - 1;
  }
};

__device__ __forceinline__ void write_free_list(const CompactLaunch& l, int num_pages, int U, long long me, long long all) {
  for (long long i = U + me; i < num_pages; i += all) l.free_pages_out[num_pages - 1 - i] = (int)i;
  if (me == 0) l.free_count_out[0] = num_pages - U;
}

__global__ __launch_bounds__(kPlanThreads) void compact_lds_kernel(const CompactArgs a) {
  __shared__ FreeMap s_map;
  __shared__ int s_part[kPlanThreads / kWave];
  __shared__ int s_from[kPlanThreads], s_to[kPlanThreads];   // of the moves at hand
  const CompactLaunch& l = a.l;
  const int tid = threadIdx.x, words = (a.num_pages + 31) / 32;
  const long long all = (long long)gridDim.x * kPlanThreads, me = (long long)blockIdx.x * kPlanThreads + tid;
  if (tid == 0) s_map.words = words;
  if (tid <= words) s_map.bits[tid] = 0;
  __syncthreads();
  const int n = free_count_of(l.free_count, l.free_capacity);
#pragma unroll 4
  for (int i = tid; i < n; i += kPlanThreads) {
    const int p = l.free_pages[i];
    if (p >= 0 && p < a.num_pages) atomicOr(&s_map.bits[p >> 5], 1u << (p & 31));
  }
  __syncthreads();
  static_assert(kLdsPages / 32 < kPlanThreads, "a thread for every word, and one behind");
  const int mine = tid <= words ? __popc(s_map.bits[tid]) : 0;
  int total;
  const int upto = block_sum(mine, s_part, &total);
  if (tid <= words) s_map.before[tid] = upto - mine;
  __syncthreads();
  const int U = a.num_pages - total, moves = s_map.free_below(U);
  auto place = [&](int p) {
    if (s_map.free(p)) return -1;
    return p < U ? p : s_map.nth(p - s_map.free_below(p) - (U - moves), false);
  };
  for (long long i = me; i < a.num_pages; i += all) {
    const int p = (int)i, at = place(p);
    l.new_page[p] = at;
    if (l.page_shares) {
      if (at >= 0) {
        const int holds = l.page_shares[p];
        l.page_shares_out[at] = holds;
      }
      if (p >= U) l.page_shares_out[p] = 0;
    }
  }
  const long long rows = (long long)a.B * a.Hkv;
  for (long long row = (long long)blockIdx.x * (kPlanThreads / kWave) + (tid >> 6); row < rows;
       row += (long long)gridDim.x * (kPlanThreads / kWave)) {
    const int blocks = blocks_for(length_of(l.seq_len[row / a.Hkv], a.max_kv_blocks));
    for (int j = tid & 63; j < blocks; j += kWave) {
      const int p = l.page_table[row * a.max_kv_blocks + j];
      l.page_table_out[row * a.max_kv_blocks + j] = p >= 0 && p < a.num_pages ? place(p) : p;
    }
  }
  if (a.apart) write_free_list(l, a.num_pages, U, me, all);   // else others may still read it
  else if (me == 0) a.count[0] = U;
  // move i: the i-th id in use from U on to the i-th free one
  const int first = (int)((long long)moves * blockIdx.x / gridDim.x);
  const int last = (int)((long long)moves * (blockIdx.x + 1) / gridDim.x);
  for (int i0 = first; i0 < last; i0 += kPlanThreads) {
    const int some = last - i0 < kPlanThreads ? last - i0 : kPlanThreads;
    __syncthreads();
    if (tid < some) s_from[tid] = s_map.nth(U - moves + i0 + tid, true), s_to[tid] = s_map.nth(i0 + tid, false);
    __syncthreads();
    for (int i = tid / kRowThreads; i < some; i += kPlanThreads / kRowThreads)
      copy_pages(l.k_pool, l.v_pool, s_from[i], s_to[i], a.page_elems, tid % kRowThreads);
  }
}

__global__ __launch_bounds__(kRowThreads) void compact_list_kernel(const CompactArgs a) {
  write_free_list(a.l, a.num_pages, a.count[0], (long long)blockIdx.x * kRowThreads + threadIdx.x,
                  (long long)gridDim.x * kRowThreads);
}

int chunk_of(int num_pages) {   // ids of a chunk: whole rounds of a workgroup's threads
  const int each = num_pages / kChunks + 1;
  return (each + kRowThreads - 1) / kRowThreads * kRowThreads;
}
size_t aligned16(size_t n) { return (n + 15) / 16 * 16; }
static_assert(kChunks == kRowThreads, "a thread for every chunk");
static_assert((long long)kForkRequests * kRowThreads <= UINT32_MAX, "workgroups of fork_rows_kernel");

}  // namespace

size_t fork_ws_bytes(const CacheDims& d) {
  const size_t table = (size_t)d.B * d.Hkv * d.max_kv_blocks;
  return (size_t)d.B * (sizeof(Plan) + sizeof(int2)) + 16 + kChunks * sizeof(int) + 16 +
         table * sizeof(int32_t);
}

hipError_t launch_fork(const CacheDims& d, const ForkLaunch& l, hipStream_t st) {
  ForkArgs a = {l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, kPage * d.D, chunk_of(d.num_pages),
                l.page_table_out == l.page_table};
  char* at = static_cast<char*>(l.ws);
  a.plan = reinterpret_cast<Plan*>(at);
  at += (size_t)d.B * sizeof(Plan);
  a.used = reinterpret_cast<int*>(at);
  at += 16;
  a.chunk_freed = reinterpret_cast<int*>(at);
  at += kChunks * sizeof(int);
  a.mark = reinterpret_cast<int2*>(at);
  at += aligned16((size_t)d.B * sizeof(int2));
  a.stage = reinterpret_cast<int32_t*>(at);
  const bool counts = l.page_shares_out != l.page_shares;
  const int copiers = (d.num_pages + kPlanThreads - 1) / kPlanThreads;
  fork_plan_kernel<<<1 + (counts ? (copiers < 255 ? copiers : 255) : 0), kPlanThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int heads = d.B >= 512 ? 1 : 512 / d.B;
  fork_rows_kernel<<<dim3(d.B, heads < d.Hkv ? heads : d.Hkv, 2), kRowThreads, 0, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  fork_free_kernel<<<kChunks, kRowThreads, 0, st>>>(a);
  return hipGetLastError();
}

size_t compact_ws_bytes(const CacheDims& d) {
  return ((size_t)d.num_pages + 2 * ((size_t)d.num_pages / 2 + 1) + kChunks + 4) * sizeof(int);
}

hipError_t launch_compact(const CacheDims& d, const CompactLaunch& l, hipStream_t st) {
  CompactArgs a = {l, d.B, d.Hkv, d.max_kv_blocks, d.num_pages, kPage * d.D, chunk_of(d.num_pages),
                   l.free_pages_out != l.free_pages && l.free_count_out != l.free_count};
  a.free = static_cast<int*>(l.ws);
  a.from = a.free + d.num_pages;
  a.to = a.from + (d.num_pages / 2 + 1);
  a.chunk_free = a.to + (d.num_pages / 2 + 1);
  a.count = a.chunk_free + kChunks;
  const int each = (d.num_pages + kRowThreads - 1) / kRowThreads, grid = each < 1024 ? each : 1024;
  if (d.num_pages <= kLdsPages) {
    const int wanted = d.num_pages / 16 + 1;   // half of the pages move at most, four at a time
    compact_lds_kernel<<<wanted < 256 ? wanted : 256, kPlanThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.apart) return e;
    compact_list_kernel<<<grid, kRowThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  compact_clear_kernel<<<grid, kRowThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int marks = (d.num_pages + kMarks - 1) / kMarks;   // a grid-stride loop, and no free list is much longer
  compact_mark_kernel<<<marks < 1024 ? marks : 1024, kRowThreads, 0, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  compact_rank_kernel<<<kChunks, kRowThreads, 0, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  compact_move_kernel<<<2048, kRowThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ca
