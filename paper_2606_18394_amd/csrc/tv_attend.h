// What the attention kernels share on the device: arguments, the split of a batch into
// work items, memory access with explicit waits, the steps of one key tile and the
// merge of chunk partials.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tv_plan.h"
#include "tv_walk.h"

namespace tv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

struct AttnArgs {
  const __bf16* q;
  const __bf16* kc;
  const __bf16* vc;
  const __bf16* kt;
  const __bf16* vt;
  const int32_t* parent;
  const int32_t* kv_len;
  __bf16* out;
  f32x4* ws_o;
  float2* ws_ml;
  unsigned int* arrived;  // per row block: chunks that have stored partials
  int* tree_bad;          // per row block: invalid parent array seen
  int B, N, Hq, Hkv, Lmax, G, M, nRB, S, chunk, nwork;
  int fused;   // split-KV merge inside the main kernel (else a second kernel)
  int slots, min_chunk;  // even split (tv_plan.h): chunks per (KV head, row block), else 0
  float rslots, rslack;  // 1 / slots, 1 / (slots - B)
  int spread;  // work order of several sequences (tv_plan.h, work_item)
  float c;  // scale * log2(e): scores live in base-2 exponent units
  const int32_t* block_table;  // paged cache: [B, max_blocks], else NULL
  int block_shift, max_blocks, num_blocks;
  int tail;    // tree-tail layout: node i's K/V are cache row kv_len + i
  int cgroup;  // sequences sharing one cache (sequence b reads cache b / cgroup)
};

// The kernel's arguments, fetched (again) from where this is called on: what only
// the epilogue needs then holds no scalar registers during the tile loop, whose
// own would otherwise be spilled to vector lanes and read back at every tile.
typedef const __attribute__((address_space(4))) AttnArgs LateArgs;
__device__ __forceinline__ const LateArgs* late_args() {
  const LateArgs* p = (const LateArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

// Context rows of sequence b: its kv_len clamped to what the cache holds (in
// the tree-tail layout behind room for the tree); a NULL kv_len means full.
__device__ __forceinline__ int context_rows(const AttnArgs& a, int b) {
  const int cap = a.tail ? a.Lmax - a.N : a.Lmax;
  const int kvl = a.kv_len ? a.kv_len[b] : cap;
  return kvl < 0 ? 0 : (kvl > cap ? cap : kvl);
}
// The same from a kv_len asked for earlier (any value for a NULL one).
__device__ __forceinline__ int context_rows_of(const AttnArgs& a, int asked) {
  const int cap = a.tail ? a.Lmax - a.N : a.Lmax;
  return a.kv_len && asked < cap ? max(asked, 0) : cap;
}

// The key tiles a row block attends over, behind kvl context rows and up to
// node i_hi.  Separate tree K/V: nct cache tiles (rows < kvl) then the tree
// tiles of nodes 0..i_hi.  Tree-tail layout: the tree rows follow the context
// in the cache and one run of nct = T tiles covers rows 0 .. kvl + i_hi.
struct Segment {
  int nct, T;
};
__device__ __forceinline__ Segment segment(const AttnArgs& a, int kvl, int i_hi) {
  if (a.tail) {
    const int t = (kvl + i_hi + kKeyTile) / kKeyTile;
    return Segment{t, t};
  }
  const int nct = (kvl + kKeyTile - 1) / kKeyTile;
  return Segment{nct, nct + i_hi / kKeyTile + 1};
}

// Longest-first order of a ragged batch (spread = 2).  XCD x serves one KV
// head and lane x / Hkv of L = 8 / Hkv lanes of chunks; pair p of the lane
// is sequence p / (S / L) and its (p % (S / L))-th chunk in that lane, as in
// work_item.  Each pair gets the distinct key (tile count << 16 | 0xFFFF - p)
// (longest first, lower pair index on ties), and the workgroup takes the
// pair whose key is the (i+1)-th largest, i its own pair index: with one
// pair per lane by counting larger keys over lane exchanges, else by
// bisection on the key value with wave-wide counts (each lane holds up to
// kRankPerLane pairs).  Every workgroup finds the same order, so this
// permutes the pairs: every work item is still covered once.
constexpr int kRankPerLane = 16;  // == kMaxRankPairs / 64 in tv_plan.h

__device__ __forceinline__ void longest_first(const AttnArgs& a, int bid, WorkItem& it) {
  const int lane = threadIdx.x & 63;
  const int L = kXcds / a.Hkv, per_b = a.S / L, npairs = a.B * per_b;  // L: a power of two
  const int x = bid % kXcds, target = (bid / kXcds) / a.nRB, ln = x / a.Hkv;
  const int nk = (npairs + 63) / 64;  // pair slots in use per lane
  // pair p's sequence (p < 2^10: the reciprocal is exact enough), and its chunk
  const float rper = __builtin_amdgcn_rcpf((float)per_b);
  auto seq = [&](int p) { return (int)(((float)p + 0.5f) * rper); };
  auto chunk_of = [&](int p, int b) { return ((ln - b) & (L - 1)) + L * (p - b * per_b); };
  int key[kRankPerLane];
  // all lengths are requested before any is used
#pragma unroll
  for (int k = 0; k < kRankPerLane; ++k)
    key[k] = k < nk ? context_rows(a, seq(min(lane + 64 * k, npairs - 1))) : -1;
#pragma unroll
  for (int k = 0; k < kRankPerLane; ++k) {
    const int p = lane + 64 * k;
    if (k < nk) {
      const int tiles = (key[k] + kKeyTile - 1) / kKeyTile + (a.N - 1) / kKeyTile + 1;
      const int work = max(0, min(a.chunk, tiles - chunk_of(p, seq(p)) * a.chunk));  // < 2^14 (plan)
      key[k] = p < npairs ? (work << 16) | (0xFFFF - p) : -1;
    }
  }
  int p;
  if (nk == 1) {
    // one pair per lane: every lane counts the larger keys by lane exchanges
    int rank = 0;
    for (int q = 0; q < 64; ++q) rank += __shfl(key[0], q) > key[0];
    const unsigned long long hit = __ballot(lane < npairs && rank == target);
    p = __builtin_amdgcn_readfirstlane(hit ? (int)__builtin_ctzll(hit) : 0);
  } else {
    // the largest v with at least target + 1 keys >= v is the wanted key (unused
    // slots count for none; four at a time, since a branch over each costs more
    // than it skips)
    int lo = 0, hi = 1 << 30;
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1);
      int c = 0;
#pragma unroll
      for (int k4 = 0; k4 < kRankPerLane; k4 += 4) {
        if (k4 >= nk) break;
#pragma unroll
        for (int k = k4; k < k4 + 4; ++k) c += __popcll(__ballot(key[k] >= mid));
      }
      if (c >= target + 1) lo = mid;
      else hi = mid;
    }
    p = 0xFFFF - (lo & 0xFFFF);
  }
  it.b = seq(p);
  it.s = chunk_of(p, it.b);
}

// ceil(x / c) for 0 <= x < 2^20, 1 <= c < 2^20, rc = 1 / c to one ulp: the
// quotient's distance to the next whole number below, at least 1 / (2 c), is
// above the errors of the reciprocal and the product (together 1.5 * 2^-23 of a
// quotient of at most (x + c) / c)
__device__ __forceinline__ int ceil_div(int x, int c, float rc) {
  return (int)(((float)(x + c) - 0.5f) * rc);
}

// Even split of the batch (a.slots > 0): one chunk size for all sequences, the
// smallest for which they need at most a.slots chunks together.  Every wave
// finds it alike from the kv_lens, and with it the sequence b and the chunk s of
// it that a work item is (s < 0: past the work), the number `first` of that
// sequence's first chunk and its context rows kvl.  All of it comes before a
// workgroup's first load of keys, so it is kept short: a whole division is some
// 40 instructions and another look at kv_len a round trip to the cache, so the
// quotients are taken with reciprocals (the host's where the divisor is its) and
// kvl comes out of the lane that holds it.  (With whole divisions, a scan over the
// LDS crossbar and kv_len read twice: 33 nodes x 16 sequences of 300 to 4096 rows
// 54.7 us, now 53.6; 2 x 24 nodes over 4360 rows 18.5, now 17.7; 37 x 4 nodes over
// 271 rows 13.7, now 13.1; 64 nodes over 4096 rows 20.0, now 19.9.)
struct EvenItem {
  int chunk, b, s, first, kvl;
};

// One sequence: the item's number is the chunk's.
template <bool kAsked>
__device__ __forceinline__ EvenItem even_one(const AttnArgs& a, int item, int asked) {
  const int kvl = kAsked ? context_rows_of(a, asked) : context_rows(a, 0);
  const int t = segment(a, kvl, a.N - 1).T;
  const int chunk = max(a.min_chunk, ceil_div(t, a.slots, a.rslots));
  return EvenItem{chunk, 0, item * chunk < t ? item : -1, 0, kvl};
}

// Several, P consecutive ones per lane (all slots are computed, those past the
// batch hold no tiles: a branch over each costs more than it skips).  The tiles
// are those of the last row block: a chunk's row blocks read the same keys.  With
// item < 0 it is sequence b that is looked up (its s is then of no use).
template <int P>
__device__ __forceinline__ EvenItem even_lanes(const AttnArgs& a, int item, int b) {
  const int b0 = P * (threadIdx.x & 63);
  int kvl[P], t[P], n[P], sum = 0, most = 0;
#pragma unroll
  for (int k = 0; k < P; ++k) kvl[k] = context_rows(a, min(b0 + k, a.B - 1));
#pragma unroll
  for (int k = 0; k < P; ++k) {
    t[k] = b0 + k < a.B ? segment(a, kvl[k], a.N - 1).T : 0;
    sum += t[k];
    most = max(most, t[k]);
  }
  const float total = (float)wave_sum(sum);
  const int longest = (int)wave_max_u32((unsigned)most);
  // Chunks of less than total / slots tiles are too many, those of total /
  // (slots - B) few enough (the sum of ceil(t / c) is below total / c + B); the
  // margins cover the rounding.
  int lo = max(a.min_chunk - 1, (int)(total * a.rslots * 0.999999f) - 1);
  int hi = max(min(longest, (int)(total * a.rslack * 1.000001f) + 1), lo + 1);
  auto chunks = [&](int c) {
    const float rc = __builtin_amdgcn_rcpf((float)c);
    int s = 0;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      n[k] = ceil_div(t[k], c, rc);
      s += n[k];
    }
    return s;
  };
  while (hi - lo > 1) {
    const int mid = lo + ((hi - lo) >> 1);
    if (wave_sum(chunks(mid)) <= a.slots) hi = mid;
    else lo = mid;
  }
  const int upto = wave_scan(chunks(hi));
  int first = upto;
#pragma unroll
  for (int k = 0; k < P; ++k) first -= n[k];
  // the last sequence that starts at or before the item: its lane, then its
  // place there (every sequence has a chunk, so places past the batch start with
  // the lane after them)
  const int owner = item < 0 ? b / P : __popcll(__ballot(b0 < a.B && first <= item)) - 1;
  int place = 0, kv = kvl[0], end = first + n[0];
#pragma unroll
  for (int k = 1; k < P; ++k) {
    const bool next = item < 0 ? b % P >= k : end <= item && b0 + k < a.B;
    place = next ? k : place;
    kv = next ? kvl[k] : kv;
    first = next ? end : first;
    end += n[k];
  }
  first = __builtin_amdgcn_readlane(first, owner);
  return EvenItem{hi, P * owner + __builtin_amdgcn_readlane(place, owner),
                  item < __builtin_amdgcn_readlane(upto, 63) ? item - first : -1, first,
                  __builtin_amdgcn_readlane(kv, owner)};
}

// Work item `item` of the batch, or (item < 0) what concerns sequence b; asked: the
// first sequence's kv_len where kAsked, else of no use.
template <bool kAsked>
__device__ __forceinline__ EvenItem even_split(const AttnArgs& a, int item, int b, int asked) {
  static_assert(kEvenSequences == 16 * 64, "sequences per lane");
  if (a.B == 1) return even_one<kAsked>(a, item, asked);
  if (a.B <= 64) return even_lanes<1>(a, item, b);
  return a.B <= 256 ? even_lanes<4>(a, item, b) : even_lanes<16>(a, item, b);
}

// Four output values, or four NaN when the sequence's tree is invalid (the
// NaN is written as a bit pattern: the kernels assume no NaN arithmetic).
__device__ __forceinline__ void store_out4(__bf16* p, const f32x4& acc, float inv, bool nan) {
  const bf16x4 v = {(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
                    (__bf16)(acc[3] * inv)};
  i16x4 bits = __builtin_bit_cast(i16x4, v);
  if (nan) bits = i16x4{0x7FC0, 0x7FC0, 0x7FC0, 0x7FC0};
  *reinterpret_cast<i16x4*>(p) = bits;
}

// Split-KV partials cross workgroups (and XCDs) through device-scope
// accesses: the sc1 bit makes a store complete only once it is visible at
// device scope and a load read at that level, which is how the compiler
// lowers relaxed agent-scope atomic loads and stores; these are their
// 8- and 16-byte forms.  Publishing then needs only vmcnt(0) before the
// arrival counter, where a release fence would write back the whole L2,
// and the merging workgroup needs no L2 invalidate (which would evict the
// keys that other workgroups are still reading).
__device__ __forceinline__ void store_dev(f32x4* p, f32x4 v) {
  asm volatile("global_store_dwordx4 %0, %1, off sc1" ::"v"(p), "v"(v) : "memory");
}
__device__ __forceinline__ void store_dev(float2* p, float2 v) {
  asm volatile("global_store_dwordx2 %0, %1, off sc1" ::"v"(p), "v"(v) : "memory");
}
__device__ __forceinline__ f32x4 load_dev(const f32x4* p) {
  f32x4 v;
  asm volatile("global_load_dwordx4 %0, %1, off sc1" : "=v"(v) : "v"(p) : "memory");
  return v;
}
__device__ __forceinline__ float2 load_dev(const float2* p) {
  float2 v;
  asm volatile("global_load_dwordx2 %0, %1, off sc1" : "=v"(v) : "v"(p) : "memory");
  return v;
}
// Plain 16- and 4-byte loads issued as inline assembly, for the prologue:
// the compiler does not track them, so it inserts no wait of its own that
// would also drain the tile DMAs issued after them.  Loads return in issue
// order, so an explicit vmcnt that leaves exactly the younger DMAs
// outstanding covers them; `loaded` then ties each value to that wait.
__device__ __forceinline__ bf16x8 load_b128(const __bf16* p) {
  bf16x8 v;
  asm volatile("global_load_dwordx4 %0, %1, off" : "=v"(v) : "v"(p) : "memory");
  return v;
}
__device__ __forceinline__ int load_i32(const int32_t* p) {
  int v;
  asm volatile("global_load_dword %0, %1, off" : "=v"(v) : "v"(p) : "memory");
  return v;
}
// Waits for every outstanding vector memory access; `loaded` values of
// load_dev are tied to the wait so no use is scheduled before it.
__device__ __forceinline__ void wait_all_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
template <class T>
__device__ __forceinline__ void loaded(T& v) {
  asm volatile("" : "+v"(v));
}

__device__ __forceinline__ float wave_max_across_groups(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

// 16 bytes per lane from global memory straight into LDS: lane i reads
// sbase + voff (sbase wave-uniform, voff a per-lane byte offset) and its
// bytes land at lds_addr + 16 * i (lds_addr wave-uniform).  Issued as inline
// assembly so the compiler does not serialise every later LDS read behind
// it; completion is awaited with explicit vmcnt waits.
__device__ __forceinline__ void dma16(const void* sbase, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(sbase)
               : "memory");
}

// A wave-uniform pointer the compiler cannot prove uniform, moved to SGPRs
// (the DMA's base address operand must be scalar).
__device__ __forceinline__ const char* uniform_ptr(const char* p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const char*)(((uint64_t)hi << 32) | lo);
}

// s_waitcnt vmcnt(n) with the other counters left alone (gfx9 encoding).
template <int n>
__device__ __forceinline__ void wait_vm() {
  static_assert(n >= 0 && n < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// s_waitcnt vmcnt(n) for a wave-uniform n in 0..63 (the prologue's waits:
// queries and DMAs still in flight); anything else waits for everything.
__device__ __forceinline__ void wait_vm_any(int n) {
  switch (n) {
#define TV_WAIT_CASE(k) \
  case k:               \
    wait_vm<k>();       \
    break;
#define TV_WAIT_CASES8(k)                                                                    \
  TV_WAIT_CASE(k) TV_WAIT_CASE(k + 1) TV_WAIT_CASE(k + 2) TV_WAIT_CASE(k + 3) TV_WAIT_CASE(k + 4) \
      TV_WAIT_CASE(k + 5) TV_WAIT_CASE(k + 6) TV_WAIT_CASE(k + 7)
    TV_WAIT_CASES8(0) TV_WAIT_CASES8(8) TV_WAIT_CASES8(16) TV_WAIT_CASES8(24)
    TV_WAIT_CASES8(32) TV_WAIT_CASES8(40) TV_WAIT_CASES8(48) TV_WAIT_CASES8(56)
#undef TV_WAIT_CASES8
#undef TV_WAIT_CASE
    default: wait_vm<0>(); break;
  }
}

// s_waitcnt vmcnt(PW * min(n, T)): at most n tiles of PW DMAs in flight
template <int PW, int T>
__device__ __forceinline__ void wait_tiles(int n) {
  if constexpr (T == 0) {
    wait_vm<0>();
  } else {
    if (n >= T) wait_vm<T * PW>();
    else wait_tiles<PW, T - 1>(n);
  }
}

// Layout of one 32-key tile in LDS: row-major, D bf16 per row, 16-byte
// chunks XOR-swizzled by the row.  With reads served 256 bytes at a time
// (64 banks; 16 lanes of a ds_read_b128, 32 of a ds_read_b64_tr_b16) the
// swizzle is free of bank conflicts: 16 rows at one logical chunk (the K
// operand reads) land in 16 bank groups, and the transposing V reads (rows
// 8k..8k+7, two adjacent chunks) cover every bank once.  The hardware
// serves the K reads 128 bytes at a time (8 lanes), where rows r and r + 4
// collide: the K reads are 2-way, a third of the LDS-active cycles, as the
// bank-conflict counter shows.  A swizzle free of conflicts at both widths
// (((r & 3) << 1) | ((r >> 2) & 1) | (((r >> 2) ^ (r >> 3)) & 1) << 3 for
// D = 128) removed them and a third of the LDS-active cycles but not a
// cycle of the kernel (about 1% slower), so this one stays.
template <int D>
struct TileLayout {
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kCPR = D / 8;               // 16-byte chunks per row
  static constexpr int kBytes = kKeyTile * kRowBytes;
  static constexpr int kDma = kBytes / 1024;       // 1 KB DMA instructions per tile
  static constexpr int kRowsPerDma = 64 / kCPR;
  __device__ static __forceinline__ int swz(int r) {
    return D == 128 ? (((r & 7) << 1) | ((r >> 3) & 1))
                    : ((((r >> 1) & 3) << 1) | ((r >> 3) & 1));
  }
  __device__ static __forceinline__ int off(int r, int chunk) {
    return r * kRowBytes + ((chunk ^ swz(r)) << 4);
  }
};

// Where a wave's K/V rows come from: the cache of one (sequence, KV head)
// pair, then its tree K/V.  The cache is either padded (row t at kcache +
// t * row_bytes) or paged (row t in pool block btab[t >> shift], whose rows
// are 2^shift apart from kcache + block * 2^shift * row_bytes; a 32-key
// tile never straddles blocks since blocks hold a power of two >= 32 rows).
// Block numbers are clamped into the pool.  Pointers are byte pointers.
struct TreeSrc {
  const char* kcache;
  const char* vcache;
  const char* ktree;
  const char* vtree;
  const int32_t* btab;  // this sequence's block table row, or NULL
  int shift, nblk;      // log2(block size), blocks in the pool
  int row_bytes;  // bytes between consecutive keys
  int rows;       // valid cache rows (the tree's too in the tree-tail layout)
  int nct;        // cache tiles
  int i_hi;       // last tree node the row block can see
};

// Issue this lane's DMA instructions for tile t into the stage at kdst (K
// tile, then V tile).  The scalar base is the tile's first row; rows past
// the valid range are clamped onto a valid row (the mask gives them zero
// weight, the clamp keeps reads in range).  dma_off is the per-lane byte
// offset of its chunk within a full tile.
template <int D, int PW, bool kPaged>
__device__ __forceinline__ void issue_tile(const TreeSrc& src, const uint32_t (&dma_off)[PW],
                                           int wr, int lane, int t, uint32_t kdst) {
  using TL = TileLayout<D>;
  const bool cache = t < src.nct;
  const int first = cache ? t * kKeyTile : (t - src.nct) * kKeyTile;
  const char* kb;
  const char* vb;
  if constexpr (kPaged) {
    size_t tofs = (size_t)first * src.row_bytes;
    if (cache) {
      // A scalar load through the constant address space (the table is
      // read-only here and the tile index wave-uniform): a vector load
      // would make the compiler wait for every DMA in flight.
      typedef const __attribute__((address_space(4))) int32_t ctab_t;
      int blk = ((ctab_t*)src.btab)[__builtin_amdgcn_readfirstlane(first >> src.shift)];
      blk = blk < 0 ? 0 : (blk >= src.nblk ? src.nblk - 1 : blk);
      tofs = (((size_t)blk << src.shift) + (first & ((1 << src.shift) - 1))) * src.row_bytes;
    }
    kb = uniform_ptr((cache ? src.kcache : src.ktree) + tofs);
    vb = uniform_ptr((cache ? src.vcache : src.vtree) + tofs);
  } else {
    kb = (cache ? src.kcache : src.ktree) + (size_t)first * src.row_bytes;
    vb = (cache ? src.vcache : src.vtree) + (size_t)first * src.row_bytes;
  }
  if (cache && (t + 1) * kKeyTile <= src.rows) {
#pragma unroll
    for (int k = 0; k < PW; ++k) {
      const int q = wr * PW + k;
      const bool isv = q >= TL::kDma;
      dma16(isv ? vb : kb, dma_off[k], kdst + (isv ? TL::kBytes : 0) + (q % TL::kDma) * 1024);
    }
    return;
  }
  const int last = cache ? src.rows - 1 : src.i_hi;  // >= first for every existing tile
#pragma unroll
  for (int k = 0; k < PW; ++k) {
    const int q = wr * PW + k;
    const bool isv = q >= TL::kDma;
    const int r = (q % TL::kDma) * TL::kRowsPerDma + lane / TL::kCPR;
    const int row = min(first + r, last) - first;
    const uint32_t off = (uint32_t)(row * src.row_bytes + ((lane % TL::kCPR) ^ TL::swz(r)) * 16);
    dma16(isv ? vb : kb, off, kdst + (isv ? TL::kBytes : 0) + (q % TL::kDma) * 1024);
  }
}

// Where a tile's scores need masking: the cache tail and the tree tiles.
struct MaskInfo {
  int t, nct, kvl, ntt, tail;
  const uint32_t* anc;
};

constexpr float kSlack = 8.f;  // log2 units a row's reference may lag its maximum

// Steps of one 32-key tile for a wave's 32 rows (two 16-row tiles nt).
//
// The compiler must not move instructions across this point: it would sink
// the LDS reads to just before their uses (fewer registers) and chain the
// score products, and the tile then waits for every LDS and matrix latency in
// turn.
__device__ __forceinline__ void pin_order() { __builtin_amdgcn_sched_barrier(0); }

// The tile's V^T operand from transposing LDS reads: lane (g4, l16) receives
// V[key 4*g4 + j (+16)][16*dt + l16], the key order of P^T.
template <int D>
__device__ __forceinline__ void read_values(const unsigned char* vt_lds, i16x4 (&vf)[D / 16][2],
                                            int g4, int l16) {
  using TL = TileLayout<D>;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const int rr = 4 * g4 + (l16 >> 2);
    const int chunk = 2 * dt + ((l16 & 3) >> 1);
    const int inb = 8 * (l16 & 1);
    vf[dt][0] =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt_lds + TL::off(rr, chunk) + inb));
    vf[dt][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_i16x4*)(vt_lds + TL::off(rr + 16, chunk) + inb));
  }
}

// scores: S^T = K Q^T on the matrix cores; lane (g4, l16) holds
//   S^T[key 16*tt + 4*g4 + j][row 16*nt + l16].
template <int D, int NT>
__device__ __forceinline__ void tile_scores(const bf16x8 (&kf)[2][D / 32], const bf16x8 (&qf)[NT][D / 32],
                                            f32x4 (&sc)[2][NT]) {
  constexpr int NC = D / 32;
#pragma unroll
  for (int cc = 0; cc < NC; ++cc) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        sc[tt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[tt][cc], qf[nt][cc],
                                                             cc == 0 ? zero : sc[tt][nt], 0, 0, 0);
      }
    pin_order();
  }
}

// The first n keys of a tile (n < 0: none, n > 32: all) as a visibility word.
__device__ __forceinline__ uint32_t first_keys(int n) {
  n = n < 0 ? 0 : (n > kKeyTile ? kKeyTile : n);
  return (uint32_t)((1ull << n) - 1ull);
}

// The visible keys of tile mk.t for this lane's row of every 16-row tile, one
// bit per key: cache keys below kv_len, and tree keys of the row's
// ancestor-or-self set (one 32-bit word of its bitmask per tile).
template <int NT>
__device__ __forceinline__ void tile_bits(const MaskInfo& mk, const int (&node_rel)[NT],
                                          uint32_t (&bits)[NT]) {
  if (mk.tail) {
    // Tree-tail layout: key k of the tile is node s + k (s < 0: a context
    // row).  Its visibility bits are a 32-bit window of the row's ancestor
    // bitmask, words w0 and w0 + 1, with all-ones standing in for context
    // rows (word -1) and zeros past the last word.
    const int s = mk.t * kKeyTile - mk.kvl;  // > -kKeyTile in the masked tiles
    const int w0 = s >> 5, sh = s & 31;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint32_t* wp = mk.anc + node_rel[nt] * mk.ntt;
      const uint32_t lo = w0 < 0 ? 0xFFFFFFFFu : wp[w0];
      const uint32_t hi = w0 + 1 < mk.ntt ? wp[w0 + 1] : 0u;
      bits[nt] = (uint32_t)((((uint64_t)hi << 32) | lo) >> sh);
    }
  } else if (mk.t < mk.nct) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) bits[nt] = first_keys(mk.kvl - mk.t * kKeyTile);
  } else {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) bits[nt] = mk.anc[node_rel[nt] * mk.ntt + mk.t - mk.nct];
  }
}

// mask: -inf for the keys a row does not see.
template <int NT>
__device__ __forceinline__ void tile_mask(f32x4 (&sc)[2][NT], const uint32_t (&bits)[NT], int g4) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!((bits[nt] >> (16 * tt + 4 * g4 + j)) & 1u)) sc[tt][nt][j] = -INFINITY;
}

// reference: online softmax in base 2 with a lazily moved reference.  A
//   row's reference m (log2 units) only moves when one of its scores
//   exceeds it by more than kSlack, so weights stay below 2^kSlack (far
//   inside the fp32 and bf16 ranges) and rescaling is rare.  Each lane
//   compares its raw scores with thr = (m + kSlack) / c; only a moving tile
//   pays for exact row maxima, and rows that move rescale O and l.
template <int DT, int NT>
__device__ __forceinline__ void tile_reference(const f32x4 (&sc)[2][NT], float (&m)[NT],
                                               float (&thr)[NT], f32x4 (&o)[DT][NT],
                                               f32x4 (&lacc)[NT], float c, float inv_c) {
  float mx[NT];
  bool move = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float v = fmaxf(fmaxf(sc[0][nt][0], sc[0][nt][1]), sc[0][nt][2]);
    v = fmaxf(fmaxf(v, sc[0][nt][3]), sc[1][nt][0]);
    v = fmaxf(fmaxf(v, sc[1][nt][1]), sc[1][nt][2]);
    v = fmaxf(v, sc[1][nt][3]);
    mx[nt] = v;
    move |= v > thr[nt];
  }
  if (__any(move)) {
    // rare: a row that has not moved keeps its scale; its m may still be -inf
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mx[nt] = wave_max_across_groups(mx[nt]) * c;
      const bool moved = mx[nt] > m[nt] + kSlack;
      const float alpha = moved ? __builtin_amdgcn_exp2f(m[nt] - mx[nt]) : 1.f;
      m[nt] = moved ? mx[nt] : m[nt];
      thr[nt] = (m[nt] + kSlack) * inv_c;
      lacc[nt] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][nt] *= alpha;
    }
  }
}

// weights: the bf16 P^T operand, exactly as it lies in the accumulators.
//   Each is rounded once, by half a step (2^-8 of it) at most, because the
//   matrix cores multiply fp32 at a sixteenth of the bf16 rate; the row sum
//   is taken of the same rounded weights, so what is left is an average of
//   roundings (outputs over the 8-bit cache are off by 0.0019 to 0.0023 of
//   their norm; the output's own rounding to bf16 alone gives 0.0016).
template <int NT>
__device__ __forceinline__ void tile_weights(const f32x4 (&sc)[2][NT], const float (&m)[NT], float c,
                                             bf16x8 (&pf)[NT]) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float mref = fmaxf(m[nt], -3.0e38f);  // rows with nothing visible yet: weights 0
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        pf[nt][4 * tt + j] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sc[tt][nt][j], c, -mref));
  }
}

// values: row sums ones^T P^T into lacc (same rounded weights as the
//   numerator) and O^T += V^T P^T.
template <int D, int NT>
__device__ __forceinline__ void tile_values(const i16x4 (&vf)[D / 16][2], const bf16x8 (&pf)[NT],
                                            const bf16x8& ones, f32x4 (&o)[D / 16][NT],
                                            f32x4 (&lacc)[NT]) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    lacc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[nt], lacc[nt], 0, 0, 0);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const bf16x4 lo = __builtin_bit_cast(bf16x4, vf[dt][0]), hi = __builtin_bit_cast(bf16x4, vf[dt][1]);
    const bf16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      o[dt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[nt], o[dt][nt], 0, 0, 0);
  }
}

// The whole tile in order (the loop form without lookahead).
template <int D, int NT, bool kMasked>
__device__ __forceinline__ void attend_tile(const unsigned char* kt_lds, const bf16x8 (&qf)[NT][D / 32],
                                            f32x4 (&o)[D / 16][NT], f32x4 (&lacc)[NT],
                                            float (&m)[NT], float (&thr)[NT], const bf16x8& ones,
                                            float c, float inv_c, const uint32_t (&bits)[NT],
                                            int g4, int l16) {
  using TL = TileLayout<D>;
  constexpr int NC = D / 32;
  // All of the tile's LDS reads go out first, K before V.
  bf16x8 kf[2][NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
      kf[tt][cc] = *reinterpret_cast<const bf16x8*>(kt_lds + TL::off(16 * tt + l16, 4 * cc + g4));
  i16x4 vf[D / 16][2];
  pin_order();
  f32x4 sc[2][NT];
  // The score products run at raised wave priority: the SIMD's other wave
  // is then mostly in its softmax (vector work) while these matrix
  // instructions issue back to back (measured 5-8% faster on matrix-bound
  // shapes than equal priority or raising it for the value products too).
  __builtin_amdgcn_s_setprio(1);
  tile_scores<D, NT>(kf, qf, sc);
  __builtin_amdgcn_s_setprio(0);
  read_values<D>(kt_lds + TL::kBytes, vf, g4, l16);
  pin_order();
  if (kMasked) tile_mask<NT>(sc, bits, g4);
  tile_reference<D / 16, NT>(sc, m, thr, o, lacc, c, inv_c);
  bf16x8 pf[NT];
  tile_weights<NT>(sc, m, c, pf);
  pin_order();
  tile_values<D, NT>(vf, pf, ones, o, lacc);
}

// Merge of the chunk partials of one row block, run by the workgroup whose
// chunk arrived last: out = sum_s e_s O_s / sum_s e_s l_s, e_s = 2^(m_s - m*),
// folded in online over s in batches of loads.  Wave w takes one 16-row
// tile and every WPN-th 16-column tile of it (or several row tiles when the
// block has more row tiles than the workgroup has waves), so each lane
// reads its rows' (m, l) once.
template <int D, int RB, int kWaves>
__device__ __forceinline__ void merge_chunks(const LateArgs* a, size_t part0, int nval, int b,
                                             int g, int r0, bool bad, int wave, int lane) {
  constexpr int DT = D / 16, NTG = RB / 16;
  constexpr bool kSplitCols = kWaves >= NTG;
  constexpr int WPN = kSplitCols ? kWaves / NTG : 1;  // waves per row tile
  constexpr int NPW = kSplitCols ? 1 : NTG / kWaves;  // row tiles per wave
  constexpr int DPW = DT / WPN;                       // column tiles per wave
  constexpr int UB = 32 / DPW;                        // chunks per batch of loads
  // every wave gets whole column tiles of one row tile, or whole row tiles
  static_assert(kSplitCols ? (kWaves % NTG == 0 && DT % WPN == 0) : (NTG % kWaves == 0),
                "merge split");
  const int g4 = lane >> 4, l16 = lane & 15;
#pragma unroll
  for (int k = 0; k < NPW; ++k) {
    const int ntg = kSplitCols ? wave % NTG : wave + k * kWaves;
    if (r0 + ntg * 16 >= a->M) continue;  // no rows
    const int dt0 = kSplitCols ? wave / NTG : 0;
    const int row = ntg * 16 + l16;
    float m = -INFINITY, l = 0.f;
    f32x4 acc[DPW];
#pragma unroll
    for (int j = 0; j < DPW; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < nval; s0 += UB) {
      float2 ml[UB];
      f32x4 ov[UB][DPW];
#pragma unroll
      for (int u = 0; u < UB; ++u)
        if (s0 + u < nval) {
          const size_t ps = part0 + s0 + u;
          ml[u] = load_dev(&a->ws_ml[ps * RB + row]);
#pragma unroll
          for (int j = 0; j < DPW; ++j)
            ov[u][j] = load_dev(&a->ws_o[(ps * DT * NTG + (dt0 + j * WPN) * NTG + ntg) * 64 + lane]);
        }
      wait_all_vm();
#pragma unroll
      for (int u = 0; u < UB; ++u)
        if (s0 + u < nval) {
          loaded(ml[u]);
#pragma unroll
          for (int j = 0; j < DPW; ++j) loaded(ov[u][j]);
        }
#pragma unroll
      for (int u = 0; u < UB; ++u)
        if (s0 + u < nval && ml[u].x != -INFINITY) {
          const float mn = fmaxf(m, ml[u].x);
          const float ea = __builtin_amdgcn_exp2f(m - mn);  // 0 while m = -inf
          const float eb = __builtin_amdgcn_exp2f(ml[u].x - mn);
          l = l * ea + eb * ml[u].y;
#pragma unroll
          for (int j = 0; j < DPW; ++j) acc[j] = acc[j] * ea + eb * ov[u][j];
          m = mn;
        }
    }
    const int r = r0 + row;
    if (r < a->M) {
      const int node = r / a->G, h = g * a->G + r % a->G;
      __bf16* op = a->out + ((size_t)(b * a->N + node) * a->Hq + h) * D + 4 * g4;
      const float inv = 1.f / l;
#pragma unroll
      for (int j = 0; j < DPW; ++j) store_out4(op + 16 * (dt0 + j * WPN), acc[j], inv, bad);
    }
  }
}

}  // namespace tv
