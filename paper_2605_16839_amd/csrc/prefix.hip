// Attention of one new token per request where requests share prefixes: per query head
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),  x_j = sm_scale q.k_j,
// in one pass over the keys with the running maximum m and sum, the share's whole pages
// (through its first member's row) once for all members, the others for their request.
//
// The work is a stream of pages.  A set is a share with two members or more (its whole
// pages; rows: the queries of all members) or a request (the pages behind; rows: its own
// queries), an item a set's KV head and tile of at most 256 rows.  The pages of all items are laid
// end to end and cut in shares of equal cost, one per workgroup, which every workgroup finds from
// the lengths on the GPU; pieces of an item that several workgroups have are joined by a
// second launch, with the prefix's and the request's parts of every row.
//
// S^T = K Q^T and O^T += V^T P^T are v_mfma_f32_16x16x32_bf16, as in the decode attention, but a page
// is read from LDS by all waves, for 16 or 32 rows each.
//
// What bounds it (32 and 8 heads of 128): behind one prefix of 126976 tokens, 128 requests with up to 4096
// of their own take 490 us from graphs (488 to 497; 540 in the first launches after a pause), 547 TFLOP/s.  No
// unit is full: of a SIMD's cycles MFMA has 39%, the other VALU instructions 46% (an exponential two turns), LDS
// 16%; waves wait 30% of their time for a barrier or for loads, and 30% for their turn.  A wave makes a page's weights before its
// first MFMA of V, and all meet at a barrier every page, so the two kinds of work mostly come one after
// the other.  Left to the compiler's order, scores half a page ahead of their weights took 3% more, half of the
// waves half a page behind the others the same; row sums by MFMA 6% more.
// Own pages and short prefixes are bound by memory: 96 requests, 6 prefixes of 1500 to 16000 tokens,
// up to 6000 of their own, 163 us, 4.6 TB/s.  The smallest calls, 14.5 us, are two launches, the plan and the walk
// from lengths to pages.  Where few requests share little, ca_decode_attention is faster: 8.8 us for 3 requests
// behind 700 tokens; 8 requests (8 KV heads of 128) break even at 3000 shared tokens, 64 at 1200.
#include <type_traits>

#pragma clang diagnostic ignored "-Winline-asm"   // page_to_lds names m0, which is reserved, as what it changes

#include "common.hpp"
#include "pages.hpp"
#include "serving.hpp"

namespace ca {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kGroups = 256;                  // one workgroup per CU
constexpr int kTile = kPrefixRows;            // query rows of an item at most
constexpr int kSets = kPrefixShares + kPrefixRequests;
constexpr int kQueue = 128;                   // pages that are looked up together
constexpr int kPairRows = 8;                  // rows of a request's item that a pair of waves takes
constexpr int kPairs = 3;                     // of those; the other two waves ask for pages then
constexpr int kCost = 4;                      // of a page that memory bounds, see page_cost
// From so many pages on they count by their cost.  Of 22 calls of 4 to 128 requests, with 32 kGroups 64 requests
// behind 16000 tokens (8 KV heads) take 120 us instead of 83 and five calls 6 to 8% more; with kGroups 64 behind 2000
// (2 KV heads) take 29 instead of 35; the others are within 4%.
constexpr int kManyPages = 4 * kGroups;
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 1 << 23;            // of a launch: one has fewer than 2^32 threads
constexpr float kSlack = 8.f;                 // log2 of the largest weight
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
  int4* plan;                      // [B][3]: see Where
};

// Where the join finds a request's parts.
struct Where {
  int own_start, own_pages, own_cost;         // of its own items: the first page's place, pages of an item, cost of one
  int share_start, share_pages, share_cost;   // of its share's
  int share_tiles, tile_rows, rank;           // its share's tiles, rows of one, its place among the members
  int total;                                  // cost of all items
};

// Rows of each of a set's tiles: as even as groups of 32 allow.
__device__ __forceinline__ int tiles_of(long long rows) { return (int)((rows + kTile - 1) / kTile); }
__device__ __forceinline__ int rows_of_tile(long long rows) {
  const int tiles = tiles_of(rows);
  return tiles < 2 ? kTile : (int)(((rows + tiles - 1) / tiles + 31) / 32 * 32);
}
// What a page costs with so many rows to a tile, in units of which a page of up to 32 rows, that memory
// bounds, has kCost.  Measured of a page of 128 dimensions: 1.2 us (8 rows), 1.5 (56), 2.2 (128), 3.4 (256),
// or 4, 5, 7.3 and 11.3.  Against costs of 4, 4, 6 and 7: the 96 requests above 165 us and 189, the 128 488 and 493, 16
// behind a document (128 rows) 57.6 and 57.0, shares of 128 rows beside as many own pages 141 and 147, with four times the own pages
// 241 and 268.  128 rows have 5 and not 7 for calls of little else: with 7 the document takes 61.2, but the two others
// 135 and 218, and the 96 requests 153.  Pages of 64 dimensions have the same costs: 196 us and 214 with many own
// pages, 410 and 372 for the 128.
__device__ __forceinline__ int page_cost(long long rows) {
  const long long all = rows < kTile ? rows : rows_of_tile(rows);
  return all <= 32 ? kCost : all <= 128 ? 5 : (all <= 192 ? 9 : 11);
}

// Where workgroup w's share begins on the line of costs, and the share of the page that begins at u.
// Every workgroup before one that has pages has some, so a row's pieces are in workgroups side
// by side: a share is longer than a page's cost, or pages count 1.
__device__ __forceinline__ int share_start(int total, int w) {
  if (total >= kGroups) return (int)((long long)total * w / kGroups);
  return w < total ? w : total;
}
__device__ __forceinline__ int share_of(int total, int u) {
  long long w = u;
  if (total >= kGroups) w = ((long long)(u + 1) * kGroups - 1) / total;
  return w < 0 ? 0 : (w < kGroups ? (int)w : kGroups - 1);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int request_len(const PrefixArgs& a, int b) {
  const int len = a.l.kv_len[b], most = a.max_kv_blocks * kPage;
  return len < 0 ? 0 : (len < most ? len : most);
}
__device__ __forceinline__ int share_blocks(const PrefixArgs& a, int s) {
  const int n = a.l.share_len[s] / kPage;
  return n < 0 ? 0 : (n < a.max_kv_blocks ? n : a.max_kv_blocks);
}
struct Entry {          // a page of the stream
  int page, set, sub;   // sub: KV head and tile of the item
  int keys;             // its keys that count, 0: no page; kFirst, kLast: of its item; kStop: of the share
};
constexpr int kFirst = 128, kLast = 256, kStop = 512;

template <int D>
struct Shared {
  static constexpr int kPageBytes = kPage * D * 2;
  static constexpr int kRing = 131072 / (2 * kPageBytes);   // pages that are there or on their way
  char pages[kRing][2][kPageBytes];    // K and V
  float pair_o[2][kPairRows * D];      // sums of a pair's second half of keys, of this item and the one before
  float2 pair_ml[2][kPairRows];
  float2 merge_ml[4][2][16];
  Entry queue[kQueue + kRing];
  int start[kSets + 1];                // cost of the sets before a set
  uint16_t blocks[kPrefixShares];      // whole pages of a share's prefix
  uint16_t count[kPrefixShares], first[kPrefixShares];   // its members, and the first
  uint16_t share[kPrefixRequests];     // the share that a request is a member of, kNoShare
  uint16_t member[kTile + 2];          // requests of the tile at hand, in order
  int part[kWaves];
  int pages_all, kinds, run_end;
};
constexpr int kNoShare = 0xffff;

// The compiler neither makes x earlier nor reads it later than here.
template <typename T>
__device__ __forceinline__ void made_here(T& x) {
  asm volatile("" : "+v"(x));
}

// The lane, made here.
__device__ __forceinline__ int lane_here() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// A barrier for what waves write to LDS themselves: __syncthreads would wait for all pages on their way.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// At most n of the wave's memory operations are left, for an n that is no less than one of these.
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void vm_left(int n) {
  if (n >= 48) vm_wait<48>();
  else if (n >= 40) vm_wait<40>();
  else if (n >= 32) vm_wait<32>();
  else if (n >= 16) vm_wait<16>();
  else if (n >= 11) vm_wait<11>();
  else if (n >= 6) vm_wait<6>();
  else if (n >= 3) vm_wait<3>();
  else vm_wait<0>();
}

// Loads first .. first + count - 1 of a page, 1 KB each, straight to LDS: lane l to bytes 16 l of it, from where
// the swizzle puts them; what lies `bytes` or more into the page reads as 0.  In assembly, because the compiler
// makes every transposing read of LDS wait for all copies that it knows of; nothing comes back to registers,
// and vm_left counts them.
template <int D, Half H>
__device__ __forceinline__ void page_to_lds(const uint16_t* from, int bytes, char* to, int first, int count) {
  constexpr int RL = H == kHalfVT ? kPage : D;   // elements of a row
  u32x4 page;
  const uint64_t at = reinterpret_cast<uint64_t>(from);
  page[0] = uniform((uint32_t)at), page[1] = uniform((uint32_t)(at >> 32) & 0xffffu);
  page[2] = uniform((uint32_t)bytes), page[3] = 0x00020000;   // raw buffer
  const int lane = lane_here();   // addresses are not kept over the loop
  // a row's swizzle is the XOR of its bits', so those of a load's first row come in by one XOR
  const int mine = 2 * (8 * lane / RL * RL) + 16 * swizzle<D, H>(8 * lane / RL, 8 * lane % RL / 8);
  const uint32_t lds = uniform((uint32_t)(uintptr_t)(lds_void*)to);
  for (int y = first; y < first + count; ++y) {
    const int source = (mine ^ (16 * swizzle<D, H>(512 * y / RL, 0))) + 1024 * y;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                 :: "s"(lds + 1024 * y), "v"(source), "s"(page) : "m0", "memory");
  }
}

// The sets, and the line of their pages' costs, when a workgroup has found them.
template <int D>
struct Line {
  const PrefixArgs& a;
  Shared<D>& s;
  const int S;
  bool weighted;   // pages count by their cost

  // the share whose pages a request does without, -1: none
  __device__ __forceinline__ int shared(int b) const {
    const int share = s.share[b];
    return share != kNoShare && s.count[share] > 1 ? share : -1;
  }
  __device__ __forceinline__ long long rows(int set) const { return (set < S ? s.count[set] : 1) * (long long)a.G; }
  // pages of one item of a set, items
  __device__ __forceinline__ int pages(int set) const {
    if (set < S) return s.count[set] > 1 ? s.blocks[set] : 0;
    const int b = set - S, share = shared(b);
    const int n = blocks_for(request_len(a, b)) - (share >= 0 ? s.blocks[share] : 0);
    return n > 0 ? n : 0;   // it is below 0 only if the lengths changed under the kernel
  }
  __device__ __forceinline__ int items(int set) const { return a.Hkv * (set < S ? tiles_of(rows(set)) : a.tiles); }
  __device__ __forceinline__ int cost(int set) const { return weighted ? page_cost(rows(set)) : 1; }
  // whether a wave has all keys of a page for its 32 rows: more rows than four groups of 32; else two waves share one
  __device__ __forceinline__ bool all_keys(int set) const {
    const long long all = rows(set);
    return (all < kTile ? all : rows_of_tile(all)) > kTile / 2;
  }
  // the last set that starts at u or before: it has pages
  __device__ __forceinline__ int set_at(int u) const {
    int lo = 0, hi = S + a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s.start[mid] <= u) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// How a workgroup takes the pages of a run of items.
enum Mode {
  kAllKeys,    // more than 128 rows: a wave has all keys of a page for 32 rows
  kHalfKeys,   // up to 128 rows: half of them, so two waves to 32 rows
  kPair        // a request's item of up to 8 rows: two waves with half of the keys each.  Pairs take turns, so that
};             // one begins and one ends an item while another computes.

// The pages from `from` to `to` on the line, all of items of one kind.
template <int D, bool VT, Mode MODE>
__device__ __forceinline__ void run_pages(const Line<D>& line, int from, int to) {
  constexpr int NX = D / 16, NK = D / 32;   // d tiles, k-steps of a score
  constexpr int NL = D / 8, NW = NL / kWaves;   // loads of a K or V page, 1 KB each; of one wave
  constexpr int R = Shared<D>::kRing;
  constexpr Half HV = VT ? kHalfVT : kHalfV;
  const PrefixArgs& a = line.a;
  Shared<D>& s = line.s;
  const PrefixLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63, w = blockIdx.x, S = line.S;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  // the page that begins at u on the line of costs, if one does (its set is -1 otherwise)
  auto look_up = [&](int u, int to) {
    const int lo = line.set_at(u), cost = line.cost(lo), off = u - s.start[lo];
    const int each = line.items(lo), all = (s.start[lo + 1] - s.start[lo]) / cost;
    const int at = off / cost, n = each > 0 ? all / each : 0;
    Entry e = {-1, lo, 0, 0};
    if (n <= 0 || at * cost != off) {
      e.set = -1;
      return e;
    }
    e.sub = at / n;
    const int p = at - e.sub * n, tiles = each / a.Hkv, kvh = e.sub / tiles;
    int row = lo - S, block = p;
    e.keys = kPage;
    if (lo < S) {
      row = s.first[lo];
    } else {
      const int len = request_len(a, row);
      block = blocks_for(len) - n + p;
      e.keys = len - block * kPage < kPage ? len - block * kPage : kPage;
    }
    if (row < a.B && kvh < a.Hkv && block >= 0 && block < a.max_kv_blocks)
      e.page = l.page_table[((long long)row * a.Hkv + kvh) * a.max_kv_blocks + block];
    if (e.page < 0 || e.page >= a.num_pages || e.keys < 0) e.page = -1, e.keys = 0;
    e.keys |= (p == 0 ? kFirst : 0) | (p == n - 1 ? kLast : 0) | (u + cost >= to ? kStop : 0);
    return e;
  };
  // A page's K or V to its place in the ring: all of it, or this wave's part.  A page that is not there is a buffer
  // of no bytes, which reads as 0; so do the rows behind the last key.  Returns how many loads the wave made.
  auto load = [&](const Entry& e, bool there, int place, bool value, int from, int loads) __attribute__((always_inline)) {
    if (!there) return 0;
    const int page = uniform(e.page), keys = uniform(e.keys) & 127;
    const uint16_t* const at = (value ? l.v_pool : l.k_pool) + (long long)(page < 0 ? 0 : page) * (kPage * D);
    const int bytes = page < 0 ? 0 : (VT && value ? kPage : keys) * D * 2;
    char* const to = s.pages[place % R][value ? 1 : 0];
    if (value) page_to_lds<D, HV>(at, bytes, to, from, loads);
    else page_to_lds<D, kHalfK>(at, bytes, to, from, loads);
    return loads;
  };

  // ---- the item at hand ----------------------------------------------------------
  // Up to 128 rows: 4 groups of 32 rows, each two waves with half of a page's keys; more: 8 groups, a wave
  // each with all keys.
  int set = -1, sub = 0, rows = 0;
  bool starts = false, active = false;
  int rg = 0, kh = 0;
  int row_of[2];               // of the lane's column: b * Hq + head, -1: none
  bf16x8 q[2][NK];
  f32x4 o[NX][2], x[4][2];     // x: scores, then weights
  float m[2], sum[2];

  auto load_q = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      u32x4 y = {0, 0, 0, 0};
      if (row_of[c] >= 0) y = *reinterpret_cast<const u32x4*>(l.q + (long long)row_of[c] * D + 32 * t + 8 * grp);
      q[c][t] = __builtin_bit_cast(bf16x8, y);
    }
    m[c] = -INFINITY, sum[c] = 0.f;
#pragma unroll
    for (int y = 0; y < NX; ++y) o[y][c] = {0.f, 0.f, 0.f, 0.f};
  };
  auto begin_pair = [&](const Entry& e) __attribute__((always_inline)) {
    set = e.set, sub = e.sub, starts = (e.keys & kFirst) != 0;
    row_of[0] = col < a.G ? (set - S) * a.Hq + sub * a.G + col : -1;
    row_of[1] = -1;
    load_q(0);
    // waited for here: with every page they would be, and for all pages on their way then
#pragma unroll
    for (int t = 0; t < NK; ++t) made_here(q[0][t]);
  };
  auto begin = [&](const Entry& e) __attribute__((always_inline)) {
    set = e.set, sub = e.sub, starts = (e.keys & kFirst) != 0;
    const bool share = set < S;
    const long long every = line.rows(set);
    const int tile_rows = rows_of_tile(every), tiles = tiles_of(every);
    const int kvh = sub / tiles, tile = sub - kvh * tiles, first = tile * tile_rows / a.G;
    if (share) {   // the members whose queries are in the tile, in order
      int n = 0;
      lds_barrier();
      for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        const bool in = b < a.B && s.share[b] == set;
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
    rows = (int)(every - (long long)tile * tile_rows);
    rows = rows < tile_rows ? rows : tile_rows;
    rg = MODE == kAllKeys ? wv : wv >> 1, kh = MODE == kAllKeys ? 0 : wv & 1;
    active = uniform(32 * rg < rows ? 1 : 0) != 0;   // a branch of the whole wave
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = 32 * rg + 16 * c + col;
      row_of[c] = -1;
      if (r < rows) {
        const int at = tile * tile_rows + r, i = at / a.G, head = at - i * a.G;
        const int b = share ? s.member[i - first] : set - S;
        if (b < a.B) row_of[c] = b * a.Hq + kvh * a.G + head;
      }
      load_q(c);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int t = 0; t < NK; ++t) made_here(q[c][t]);
  };

  // All operand fragments of a part are asked for before its first MFMA: the compiler would ask for two or
  // three at a time and wait for LDS with each.  Addresses are made here: kept over the loop they would be
  // spilled, and read back behind all pages on their way.  A swizzle is an XOR, so a fragment's chunk
  // comes in by one.
  auto read_k = [&](auto steps, u32x4 (&f)[2 * decltype(steps)::value][NK], int p0, int buf) __attribute__((always_inline)) {
    constexpr int NP = decltype(steps)::value;
    const int me = lane_here(), r0 = 8 * ((me & 15) >> 2) + (me & 3);
    const int from = (r0 + 32 * p0) * D * 2 + 16 * swizzle<D, kHalfK>(r0, me >> 4);
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
        f[t][ks] = *reinterpret_cast<const u32x4*>(s.pages[buf][0] + (from ^ (64 * ks)) + (32 * (t >> 1) + 4 * (t & 1)) * D * 2);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto read_v = [&](u32x4 (&f)[NX], int p, int buf) __attribute__((always_inline)) {
    const char* const vp = s.pages[buf][1];
    const int me = lane_here(), c16 = me & 15, v0 = 8 * (me >> 4) + (c16 >> 2), d0 = 4 * (me & 3);
    const int from = VT ? c16 * kPage * 2 + 16 * swizzle<D, kHalfVT>(c16, 4 * p + (me >> 4))
                        : (v0 + 32 * p) * D * 2 + 16 * swizzle<D, kHalfV>(v0, d0 >> 3) + 2 * (d0 & 7);
#pragma unroll
    for (int y = 0; y < NX; ++y) {
      if constexpr (VT) {
        f[y] = *reinterpret_cast<const u32x4*>(vp + from + 16 * y * kPage * 2);
      } else {
        const char* const src = vp + (from ^ (32 * y));
        const u32x2 a2 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)src));
        const u32x2 b2 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 4 * D * 2)));
        f[y] = u32x4{a2[0], a2[1], b2[0], b2[1]};
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // Scores of NP key steps (32 keys each) from step p0 on, for NC column tiles.
  auto score = [&](auto steps, auto columns, int p0, int buf, int keys) __attribute__((always_inline)) {
    constexpr int NP = decltype(steps)::value, NC = decltype(columns)::value;
    u32x4 f[2 * NP][NK];
    read_k(steps, f, p0, buf);
#pragma unroll
    for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
      for (int c = 0; c < NC; ++c) x[t][c] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          x[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[t][ks]), q[c][ks], x[t][c], 0, 0, 0);
    if (keys < kPage) {
      const int left = keys - 32 * p0 - 8 * (lane_here() >> 4);
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < NC; ++c) x[t][c][e] = key_of(t, 0) + e >= left ? -INFINITY : x[t][c][e];
    }
  };
  // Weights.  m, what they are relative to (log2 units), moves only when a score passes it by more than kSlack: most
  // pages rescale nothing.  It is carried scaled and rounded, as the weights take it off.
  auto weigh = [&](auto steps, auto columns) __attribute__((always_inline)) {
    constexpr int NP = decltype(steps)::value, NC = decltype(columns)::value;
    float top[NC];
    bool moves = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      top[c] = x[0][c][0];
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t) {
        top[c] = max2(max2(top[c], x[t][c][0]), x[t][c][1]);
        top[c] = max2(max2(top[c], x[t][c][2]), x[t][c][3]);
      }
      moves = moves || !(top[c] * a.scale_log2 <= m[c] + kSlack);   // a NaN moves it too
    }
    if (__ballot(moves) != 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float mn = max2(m[c], groups_max(top[c]) * a.scale_log2);
        const float alpha = fast_exp2(m[c] - (mn == -INFINITY ? 0.f : mn));
        m[c] = mn;
        sum[c] *= alpha;
#pragma unroll
        for (int y = 0; y < NX; ++y) o[y][c] *= alpha;
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float base = m[c] == -INFINITY ? 0.f : m[c];
      float part = 0.f;
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[t][c][e] = fast_exp2(__builtin_fmaf(x[t][c][e], a.scale_log2, -base));
          part += x[t][c][e];
        }
      sum[c] += part;
    }
  };
  // O^T += V^T P^T of the weights in x.
  auto add_v = [&](auto steps, auto columns, int p0, int buf) __attribute__((always_inline)) {
    constexpr int NP = decltype(steps)::value, NC = decltype(columns)::value;
    u32x4 f[NP][NX];
    read_v(f[0], p0, buf);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      // weights to 16 bits, in two parts: the upper half of p's bits, and what that leaves, which is never
      // negative.  The second part of a weight that is not 0 is made no less than 2^-126, so that an infinity of v stays
      // one; a weight of 0 has none, and adds nothing however large v is.
      u32x4 hi[NC], lo[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[2 * p + (e >> 1)][c][2 * (e & 1)], v = x[2 * p + (e >> 1)][c][2 * (e & 1) + 1];
          const uint32_t ub = __float_as_uint(u), vb = __float_as_uint(v);
          const uint32_t first = __builtin_amdgcn_perm(vb, ub, 0x07060302);
          hi[c][e] = first;   // (__builtin_bit_cast of hi[c][e] itself would take hi[c][0])
          const f32x2 rest = {u - __uint_as_float(ub & 0xffff0000u), v - __uint_as_float(vb & 0xffff0000u)};
          // (bf16 that are not negative compare as integers)
          const u16x2 least = __builtin_elementwise_min(__builtin_bit_cast(u16x2, first), u16x2{0x80, 0x80});
          lo[c][e] = __builtin_bit_cast(
              uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, __builtin_convertvector(rest, bf16x2)), least));
        }
      if (p + 1 < NP) read_v(f[p + 1 < NP ? p + 1 : 0], p0 + p + 1, buf);
#pragma unroll
      for (int y = 0; y < NX; ++y) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
          o[y][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[p][y]), __builtin_bit_cast(bf16x8, hi[c]), o[y][c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < NC; ++c)
          o[y][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[p][y]), __builtin_bit_cast(bf16x8, lo[c]), o[y][c], 0, 0, 0);
      }
    }
  };
  constexpr std::integral_constant<int, 1> k1{};
  constexpr std::integral_constant<int, 2> k2{};

  // To where the join looks.
  auto store = [&](bool ends, int c, int r) __attribute__((always_inline)) {
    if (row_of[c] < 0) return;
    float *to, *ml;
    if (starts && ends) {
      const long long row = (set < S ? 0 : (long long)a.B * a.Hq) + row_of[c];
      to = a.whole_o + row * D, ml = a.whole_ml + 2 * row;
    } else {
      const long long row = (long long)(2 * w + (starts ? 1 : 0)) * a.slot_rows + r;
      to = a.part_o + row * D, ml = a.part_ml + 2 * row;
    }
#pragma unroll
    for (int y = 0; y < NX; ++y) *reinterpret_cast<f32x4*>(to + 16 * y + 4 * grp) = o[y][c];
    if (grp == 0) *reinterpret_cast<float2*>(ml) = make_float2(m[c], sum[c]);
  };
  // The second half of the keys' sums come to the first's.
  auto join = [&](int c, float2 ml, auto part) __attribute__((always_inline)) {
    const float mn = max2(m[c], ml.x), base = mn == -INFINITY ? 0.f : mn;
    const float c0 = fast_exp2(m[c] - base), c1 = fast_exp2(ml.x - base);
    m[c] = mn;
    sum[c] = sum[c] * c0 + ml.y * c1;
#pragma unroll
    for (int y = 0; y < NX; ++y) {
      const float4 z = part(y);
      o[y][c][0] = o[y][c][0] * c0 + z.x * c1, o[y][c][1] = o[y][c][1] * c0 + z.y * c1;
      o[y][c][2] = o[y][c][2] * c0 + z.z * c1, o[y][c][3] = o[y][c][3] * c0 + z.w * c1;
    }
  };
  auto finish = [&](bool ends, int buf) __attribute__((always_inline)) {
    float4* const merge = reinterpret_cast<float4*>(s.pages[buf][0]) + rg * (NX * kWave);   // the page is done with
#pragma unroll
    for (int c = 0; c < 2; ++c) sum[c] = groups_sum(sum[c]);
    if constexpr (MODE == kHalfKeys) {
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
        if (active && kh == 0)
          join(c, s.merge_ml[rg][c][col], [&](int y) { return merge[64 * y + lane]; });
      }
    }
    if (!active || kh != 0) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) store(ends, c, 32 * rg + 16 * c + col);
  };
  // The pages from `from` to `to` on the line of costs, page by page: step(e, next, buf, first, more) for page e in
  // place buf of the ring, the first of them or not.  Pairs: the last two waves ask for all pages, one for
  // K and one for V, so the others never wait for pages on their way when they wait for queries.
  auto stream = [&](auto ahead, auto step) __attribute__((always_inline)) {
    int ring = 0;   // the place of the queue's first page
    bool first = true;
    for (int base = from; base < to;) {
      // the next pages: a thread looks at one place of the line, those where a page begins are kept, in order
      lds_barrier();   // the queue's last readers
      int n = 0;
      {
        const int span = line.weighted ? kThreads : kQueue;
        Entry e = {-1, -1, 0, 0};
        if (tid < span && tid < to - base) e = look_up(base + tid, to);
        const unsigned long long hits = __ballot(e.set >= 0);
        if (lane == 0) s.part[wv] = __popcll(hits);
        lds_barrier();
        int at = lanes_below(hits);
        for (int v = 0; v < kWaves; ++v) {
          if (v < wv) at += s.part[v];
          n += s.part[v];
        }
        if (e.set >= 0) s.queue[at] = e;
        base = span < to - base ? base + span : to;
        lds_barrier();
      }
      // the loads of each of the steps before: K of the page R - 1 on, V of the page R - 2 on
      int made_k[R - 2], made_v[R - 2];
      auto ask = [&](int i, const Entry& ek, const Entry& ev) __attribute__((always_inline)) {
        const bool is_k = i + R - 1 < n, is_v = i + R - 2 >= 0 && i + R - 2 < n;
        int k = 0, v = 0;
        if constexpr (MODE == kPair) {
          if (wv == kWaves - 1) v = load(ev, is_v, ring + i + R - 2, true, 0, NL);
          else if (wv == kWaves - 2) k = load(ek, is_k, ring + i + R - 1, false, 0, NL);
        } else {
          v = load(ev, is_v, ring + i + R - 2, true, NW * wv, NW);
          k = load(ek, is_k, ring + i + R - 1, false, NW * wv, NW);
        }
#pragma unroll
        for (int j = R - 3; j > 0; --j) made_k[j] = made_k[j - 1], made_v[j] = made_v[j - 1];
        made_k[0] = k, made_v[0] = v;
      };
#pragma unroll
      for (int j = 0; j < R - 2; ++j) made_k[j] = made_v[j] = 0;
#pragma unroll 1
      for (int j = 1 - R; j < 0; ++j) ask(j, s.queue[j + R - 1], s.queue[j + R - 2 < 0 ? 0 : j + R - 2]);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        // (what is past the queue's end is read, and not used)
        Entry e = s.queue[i];
        const Entry ek = s.queue[i + R - 1], ev = s.queue[i + R - 2];
        e.page = uniform(e.page), e.set = uniform(e.set), e.sub = uniform(e.sub), e.keys = uniform(e.keys);
        const int keys = e.keys & 127, buf = (ring + i) % R;
        if (first) ahead(e);   // while the first pages are on their way
        // K and V of this page are there; then everyone is done with the V of the page before the last
        int n_left = made_k[R - 3];
#pragma unroll
        for (int j = 0; j < R - 3; ++j) n_left += made_k[j] + made_v[j];
        vm_left(n_left);
        lds_barrier();
        auto more = [&]() __attribute__((always_inline)) { ask(i, ek, ev); };
        if (VT && keys < kPage) {   // weights of 0 do not undo a NaN in V: columns behind the last key
          for (int at = 8 * tid; at < kPage * D; at += 8 * kThreads) {
            const int r = at / kPage, key = at % kPage;
            if (key + 8 <= keys) continue;
            u32x4* const y = reinterpret_cast<u32x4*>(s.pages[buf][1] + r * kPage * 2 + 16 * swizzle<D, kHalfVT>(r, key / 8));
            u32x4 z = *y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (key + 2 * j >= keys) z[j] = 0;
              else if (key + 2 * j + 1 >= keys) z[j] &= 0xffffu;
            }
            *y = z;
          }
          lds_barrier();
        }
        Entry next = {-1, -1, 0, 0};
        if (MODE == kPair && i + 1 < n) {
          next = s.queue[i + 1];
          next.set = uniform(next.set), next.sub = uniform(next.sub), next.keys = uniform(next.keys);
        }
        step(e, next, buf, first, more);
        first = false;
      }
      ring = (ring + n) % R;
    }
    lds_barrier();
  };

  if constexpr (MODE != kPair) {
    constexpr std::integral_constant<int, MODE == kAllKeys ? 2 : 1> steps{};
    stream(begin,
           [&](const Entry& e, const Entry&, int buf, bool first, auto more) __attribute__((always_inline)) {
      if ((e.keys & kFirst) && !first) begin(e);
      if (active) {
        score(steps, k2, kh, buf, e.keys & 127);
        more();   // asked for while the weights are made
        weigh(steps, k2);
        add_v(steps, k2, kh, buf);
      } else {
        more();
      }
      if (e.keys & (kLast | kStop)) finish((e.keys & kLast) != 0, buf);
    });
  } else {
    int turn = -1, left = 0;                  // the pairs' items so far, less 1; the turn whose sums wait
    bool waits = false, waits_ends = false;   // this wave has an item to end
    auto end_pair = [&]() __attribute__((always_inline)) {
      waits = false;
      if (col >= a.G) return;
      join(0, s.pair_ml[left & 1][col], [&](int y) {
        return *reinterpret_cast<const float4*>(&s.pair_o[left & 1][((4 * y + grp) * kPairRows + col) * 4]);
      });
      store(waits_ends, 0, col);
    };
    stream([](const Entry&) {},
           [&](const Entry& e, const Entry& next, int buf, bool first, auto more) __attribute__((always_inline)) {
      more();
      if (waits) end_pair();
      if (first || (e.keys & kFirst)) ++turn;
      if (wv >> 1 == turn % kPairs) {
        if (set != e.set || sub != e.sub) begin_pair(e);   // if not ahead of its turn
        score(k1, k1, wv & 1, buf, e.keys & 127);
        weigh(k1, k1);
        add_v(k1, k1, wv & 1, buf);
        if (e.keys & (kLast | kStop)) {   // the second wave leaves its sums, the first takes them a barrier later
          sum[0] = groups_sum(sum[0]);
          left = turn;
          waits = (wv & 1) == 0, waits_ends = (e.keys & kLast) != 0;
          if (!waits && col < a.G) {
#pragma unroll
            for (int y = 0; y < NX; ++y)
              *reinterpret_cast<f32x4*>(&s.pair_o[turn & 1][((4 * y + grp) * kPairRows + col) * 4]) = o[y][0];
            if (grp == 0) s.pair_ml[turn & 1][col] = make_float2(m[0], sum[0]);
          }
        }
      } else if (wv >> 1 == (turn + 1) % kPairs && (next.keys & kFirst)) {
        begin_pair(next);
      }
    });
    if (waits) end_pair();
  }
}

template <int D, bool VT>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(const PrefixArgs a) {
  __shared__ __align__(16) Shared<D> s;
  const PrefixLaunch& l = a.l;
  const int tid = threadIdx.x, lane = tid & 63, w = blockIdx.x;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int S = l.num_shares, sets = S + a.B;

  // ---- the stream, from the lengths -------------------------------------------
  int* const count = reinterpret_cast<int*>(&s.pages[0][0][0]);   // no page is there yet
  int* const first = count + kPrefixShares;
  for (int i = tid; i < S; i += kThreads) count[i] = 0, first[i] = a.B, s.blocks[i] = (uint16_t)share_blocks(a, i);
  if (tid == 0) s.pages_all = 0, s.kinds = 0;
  __syncthreads();
  for (int b = tid; b < a.B; b += kThreads) {
    const int len = request_len(a, b);
    int share = S > 0 ? l.share[b] : -1;
    if (share >= 0 && share < S && s.blocks[share] > 0 && len >= s.blocks[share] * kPage)
      atomicAdd(&count[share], 1), atomicMin(&first[share], b);
    else
      share = kNoShare;
    s.share[b] = (uint16_t)share;
  }
  __syncthreads();
  for (int i = tid; i < S; i += kThreads) s.count[i] = (uint16_t)count[i], s.first[i] = (uint16_t)first[i];
  __syncthreads();
  Line<D> line = {a, s, S, false};
  const int per = (sets + kThreads - 1) / kThreads;
  int total;
  {
    int pages = 0;
    double cost = 0.;
    for (int i = tid * per; i < (tid + 1) * per && i < sets; ++i) {
      const int n = line.pages(i) * line.items(i);
      s.start[i] = n;
      pages += n, cost += (double)n * page_cost(line.rows(i));
      if (n > 0 && (i < S || a.G > kPairRows)) atomicOr(&s.kinds, line.all_keys(i) ? 2 : 1);
    }
    // by cost only where shares are long, and the line of costs is not
    if (pages > 0) atomicAdd(&s.pages_all, pages);
    const int few = __syncthreads_and(cost < 2147483647. / kThreads);
    line.weighted = few && s.pages_all >= kManyPages;
    const int mine = line.weighted ? (int)cost : pages;
    int before = wave_inclusive_scan(mine);
    if (lane == kWave - 1) s.part[wv] = before;
    __syncthreads();
    before -= mine;
    for (int v = 0; v < wv; ++v) before += s.part[v];
    for (int i = tid * per; i < (tid + 1) * per && i < sets; ++i) {
      const int n = s.start[i] * line.cost(i);
      s.start[i] = before;
      before += n;
    }
    if (tid == kThreads - 1) s.start[sets] = before;
    __syncthreads();
    total = s.start[sets];
  }
  const int u0 = share_start(total, w), u1 = share_start(total, w + 1);

  // ---- where the join finds the requests' parts: some requests each -------------
  for (int b = (kGroups - 1 - w) * kWaves + wv; b < a.B; b += kGroups * kWaves) {   // the last have least to do
    const int share = line.shared(b);
    int rank = 0;
    for (int i0 = 0; share >= 0 && i0 < b; i0 += kWave) {
      const int i = i0 + lane;
      rank += __popcll(__ballot(i < b && s.share[i] == share));
    }
    if (lane == 0) {
      const long long rows = share >= 0 ? line.rows(share) : 1;
      a.plan[3 * b] = make_int4(s.start[S + b], line.pages(S + b), line.cost(S + b), share >= 0 ? s.start[share] : 0);
      a.plan[3 * b + 1] = make_int4(share >= 0 ? line.pages(share) : 0, share >= 0 ? line.cost(share) : 1, tiles_of(rows),
                                    rows_of_tile(rows));
      a.plan[3 * b + 2] = make_int4(rank, total, 0, 0);
    }
  }

  // ---- its pages: shares and requests of many heads in runs of one kind, then the pairs' ------
  const int split = a.G <= kPairRows ? s.start[S] : total;
  for (int u = u0, end = u1 < split ? u1 : split; u < end;) {
    const int set = line.set_at(u);
    const bool all_keys = uniform(line.all_keys(set) ? 1 : 0);
    int to = end;
    if (s.kinds == 3) {   // up to the first set of the other kind
      lds_barrier();
      if (tid == 0) s.run_end = end;
      lds_barrier();
      for (int i = set + 1 + tid; i < sets; i += kThreads)
        if (s.start[i] < s.start[i + 1] && s.start[i] < end && line.all_keys(i) != all_keys) atomicMin(&s.run_end, s.start[i]);
      lds_barrier();
      to = s.run_end;
    }
    to = uniform(to);
    if (all_keys) run_pages<D, VT, kAllKeys>(line, u, to);
    else run_pages<D, VT, kHalfKeys>(line, u, to);
    u = to;
  }
  run_pages<D, VT, kPair>(line, u0 > split ? u0 : split, u1);
}

// A query row's parts: of its share's items and of its own, each whole or in the pieces of several
// workgroups.  A thread takes 4 dimensions of every lots-th piece.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void prefix_join_kernel(const PrefixArgs a, int first) {
  constexpr int kEach = D / 4, kLots = kJoinThreads / kEach;
  __shared__ float4 s_o[kJoinThreads];
  __shared__ float2 s_ml[kLots];
  const int tid = threadIdx.x, lot = tid / kEach, d = 4 * (tid % kEach);
  const int at_row = first + blockIdx.x, b = at_row / a.Hq, h = at_row - b * a.Hq, kvh = h / a.G, head = h - kvh * a.G;
  const int4 p0 = a.plan[3 * b], p1 = a.plan[3 * b + 1], p2 = a.plan[3 * b + 2];
  const Where at = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w, p2.x, p2.y};
  const long long out_row = at_row;
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
  auto parts = [&](int kind, int start, int n, int cost, int r) {
    if (n <= 0) return;
    const int w0 = share_of(at.total, start), w1 = share_of(at.total, start + (n - 1) * cost);
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
  const long long share_row = (long long)at.rank * a.G + head;
  const int tile = (int)(share_row / at.tile_rows), own_rows = rows_of_tile(a.G), own_tile = head / own_rows;
  parts(0, at.share_start + (kvh * at.share_tiles + tile) * at.share_pages * at.share_cost, at.share_pages, at.share_cost,
        (int)(share_row - (long long)tile * at.tile_rows));
  parts(1, at.own_start + (kvh * a.tiles + own_tile) * at.own_pages * at.own_cost, at.own_pages, at.own_cost,
        head - own_tile * own_rows);
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
  hipError_t e = hipGetLastError();
  const int rows = a.B * a.Hq;   // below 2^28
  for (int first = 0; e == hipSuccess && first < rows; first += kJoinRows) {
    const int n = rows - first < kJoinRows ? rows - first : kJoinRows;
    prefix_join_kernel<D><<<n, kJoinThreads, 0, st>>>(a, first);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t prefix_ws_bytes(const CacheDims& d) {
  const size_t rows = 2 * (size_t)d.B * d.Hq + 2 * (size_t)kGroups * slot_rows_of(d);
  return rows * (d.D + 2) * sizeof(float) + 3 * (size_t)d.B * sizeof(int4);
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
  a.whole_o = reinterpret_cast<float*>(a.plan + 3 * (size_t)d.B);
  a.part_o = a.whole_o + whole * d.D;
  a.whole_ml = a.part_o + parts * d.D;
  a.part_ml = a.whole_ml + 2 * whole;
  const bool vt = d.v_layout != 0;
  if (d.D == 64) return vt ? launch<64, true>(a, st) : launch<64, false>(a, st);
  return vt ? launch<128, true>(a, st) : launch<128, false>(a, st);
}

}  // namespace ca
