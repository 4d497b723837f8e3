// Tree-verification attention over a paged cache in 8 bits, for CDNA4 (gfx950).
//
// What tv_attention.hip computes, softmax(q_v K^T * scale + M_v) V over a sequence's
// cached prefix and its tree, with the prefix's K and V held as e4m3 codes and an
// exponent byte e per group of 32 positions, page and head: a code stands for
// code * 2^(e - 127).  The tree's own K and V are bf16.  Its work decomposition is that
// of tv_attention.hip too: 32-key tiles in chunks of one size for the whole batch, a
// workgroup per chunk and block of 16 * NT * WR rows, WR x WK waves, an LDS ring per key
// group, chunk partials merged by the last workgroup or by a second kernel.
//
// Layout.  A page holds its heads one after the other, [num_blocks, Hkv, block_size, D],
// so a group, which is a key tile, is 32 * D contiguous bytes.  Pages that hold all heads
// of a position together gave rows of 128 bytes every Hkv * 128: read by workgroups that
// keep a head to an XCD they came in at 4.2 TB/s, groups at 6.0 (1 GiB).
//
// Codes stay codes in the ring, half the bytes and half the LDS reads of bf16, and become
// bf16 exactly on their way to the matrix cores: v_cvt_scalef32_pk_bf16_fp8 takes the
// exponent along and runs at the rate of an fma, 64 of them per tile and wave at D = 128.
// From there on a tile is one of the bf16 cache's.
//
// A unit of the ring is 64 * D bytes: a cache tile (codes of K, then of V) is one, a tree
// tile, whose K and V are bf16, two.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>
#include <type_traits>

#include "tv_attend.h"
#include "tv_plan_fp8.h"

namespace tv {

struct Fp8Args : AttnArgs {
  const uint8_t* ke;  // exponents of K and V, [num_blocks, Hkv, block_size / 32]
  const uint8_t* ve;
};

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef const __attribute__((address_space(3))) i32x4 lds_i32x4;

// A tile's codes in LDS: rows of D bytes, 16-byte chunks XOR-swizzled by the row.  K is
// read 16 bytes a lane, 16 rows at one chunk; V by ds_read_b64_tr_b8, whose 16 lanes
// take a column each of 8 rows of 16 codes, every pair of lanes naming its own row: rows
// 4 g4 .. + 4 and 16 + 4 g4 .. + 4, the key order of P^T.  At 64 banks both are free of
// conflicts.
template <int D>
struct CodeLayout {
  static constexpr int kCPR = D / 16;  // 16-byte chunks per row
  static constexpr int kBytes = kKeyTile * D;
  static constexpr int kRowsPerDma = 64 / kCPR;
  static constexpr int kDma = kBytes / 1024;
  __device__ static __forceinline__ int swz(int r) {
    return D == 128 ? (((r >> 1) & 7) ^ ((r >> 4) << 2)) : (((r >> 2) & 3) ^ ((r >> 4) << 1));
  }
  __device__ static __forceinline__ int off(int r, int chunk) {
    return r * D + ((chunk ^ swz(r)) << 4);
  }
  // swz(r) ^ swz(r + 16), as a byte offset: a lane's other addresses are its first one
  // with such bits flipped
  static constexpr uint32_t kFlip = D == 128 ? 64 : 32;
  // the same for the first rows of DMAs 0 and j of a tile
  __device__ static constexpr uint32_t dma_flip(int j) {
    return D == 128 ? ((j ^ (j >> 1)) & 1 ? 64 : 0) : (j & 1 ? 32 : 0);
  }
};

// First of the eight head dims that lane group g4 takes in score product cc.  16 bytes of
// codes are two products' worth, so products 2 p and 2 p + 1 share the 16 dims from
// 64 p + 16 g4 on; queries and the tree's keys follow that order.
__device__ __forceinline__ int head_dim(int cc, int g4) {
  return 64 * (cc >> 1) + 16 * g4 + 8 * (cc & 1);
}

// Four codes as bf16.
__device__ __forceinline__ i32x2 from_codes(int w, float scale) {
  return i32x2{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
}

// An exponent byte, loaded like the prologue's parents and queries.
__device__ __forceinline__ int load_u8(const uint8_t* p) {
  int v;
  asm volatile("global_load_ubyte %0, %1, off" : "=v"(v) : "v"(p) : "memory");
  return v;
}

// dma16 of what is read once: it does not stay in the caches.
__device__ __forceinline__ void dma16_once(const void* sbase, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(sbase)
               : "memory");
}

// The scheduler's order inside the region up to the next pin_order(): n times `mfma`
// matrix instructions, then `valu` vector ones.
template <int n, int mfma, int valu>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int k = 0; k < n; ++k) {
    __builtin_amdgcn_sched_group_barrier(0x8, mfma, 0);
    __builtin_amdgcn_sched_group_barrier(0x2, valu, 0);
  }
}

// A tile's codes in a wave's registers, as the products take them.
template <int D>
struct Codes {
  i32x4 k[2][D / 64];
  i32x2 v[D / 16];
};
// (The tile begins at a multiple of 128 bytes.)
template <int D>
__device__ __forceinline__ void read_keys(uint32_t lds, Codes<D>& t, int g4, int l16) {
  using CL = CodeLayout<D>;
  const uint32_t k0 = lds + CL::off(l16, g4);
#pragma unroll
  for (int p = 0; p < D / 64; ++p)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
      t.k[tt][p] = *((lds_i32x4*)(k0 ^ (64 * p) ^ (CL::kFlip * tt)) + tt * D);
}
template <int D>
__device__ __forceinline__ void read_values(uint32_t lds, Codes<D>& t, int g4, int l16) {
  using CL = CodeLayout<D>;
  const int r = l16 >> 1, row = 4 * g4 + r + (r < 4 ? 0 : 12);
  const uint32_t v0 = lds + CL::off(row, 0) + 8 * (l16 & 1);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
    t.v[dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(v0 ^ (16 * dt)) + CL::kBytes / 8);
}

// One 32-key tile of codes for a wave's rows, with the scales of K and V.  The
// conversions go between the products before theirs: a product keeps the matrix core
// busy for 16 cycles and issues in 4.  The values are read behind the scores unless they
// are there already (kHeld).
template <int D, int NT, bool kMasked, bool kHeld>
__device__ __forceinline__ void attend_codes(Codes<D>& t, uint32_t lds, float kscale, float vscale,
                                             const bf16x8 (&qf)[NT][D / 32], f32x4 (&o)[D / 16][NT],
                                             f32x4 (&lacc)[NT], float (&m)[NT], float (&thr)[NT],
                                             const bf16x8& ones, float c, float inv_c,
                                             const uint32_t (&bits)[NT], int g4, int l16) {
  constexpr int NP = D / 64, DT = D / 16;
  pin_order();
  f32x4 sc[2][NT];
  __builtin_amdgcn_s_setprio(1);
  bf16x8 kf[2][2 * NP];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const i32x2 lo = from_codes(t.k[tt][p][2 * h], kscale);
        const i32x2 hi = from_codes(t.k[tt][p][2 * h + 1], kscale);
        kf[tt][2 * p + h] = __builtin_bit_cast(bf16x8, i32x4{lo[0], lo[1], hi[0], hi[1]});
      }
#pragma unroll
  for (int cc = 0; cc < 2 * NP; ++cc)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        sc[tt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[tt][cc], qf[nt][cc],
                                                             cc == 0 ? zero : sc[tt][nt], 0, 0, 0);
      }
  __builtin_amdgcn_sched_group_barrier(0x2, 8, 0);
  interleave<(2 * NP - 1) * 2 * NT, 1, 4 / NT>();
  pin_order();
  __builtin_amdgcn_s_setprio(0);
  if (!kHeld) read_values<D>(lds, t, g4, l16);
  pin_order();
  if (kMasked) tile_mask<NT>(sc, bits, g4);
  tile_reference<DT, NT>(sc, m, thr, o, lacc, c, inv_c);
  bf16x8 pf[NT];
  tile_weights<NT>(sc, m, c, pf);
  pin_order();
  i16x4 vf[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int h = 0; h < 2; ++h) vf[dt][h] = __builtin_bit_cast(i16x4, from_codes(t.v[dt][h], vscale));
  tile_values<D, NT>(vf, pf, ones, o, lacc);
  interleave<DT, NT, 4>();
  pin_order();
}

// One 32-key tile of the tree.
template <int D, int NT>
__device__ __forceinline__ void attend_tree(const unsigned char* k_lds, const unsigned char* v_lds,
                                            const bf16x8 (&qf)[NT][D / 32], f32x4 (&o)[D / 16][NT],
                                            f32x4 (&lacc)[NT], float (&m)[NT], float (&thr)[NT],
                                            const bf16x8& ones, float c, float inv_c,
                                            const uint32_t (&bits)[NT], int g4, int l16) {
  using TL = TileLayout<D>;
  constexpr int NC = D / 32, DT = D / 16;
  bf16x8 kf[2][NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc)
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
      kf[tt][cc] = *reinterpret_cast<const bf16x8*>(k_lds +
                                                    TL::off(16 * tt + l16, head_dim(cc, g4) / 8));
  f32x4 sc[2][NT];
  tile_scores<D, NT>(kf, qf, sc);
  tile_mask<NT>(sc, bits, g4);
  tile_reference<DT, NT>(sc, m, thr, o, lacc, c, inv_c);
  bf16x8 pf[NT];
  tile_weights<NT>(sc, m, c, pf);
  pin_order();
  i16x4 vf[DT][2];
  tv::read_values<D>(v_lds, vf, g4, l16);
  tile_values<D, NT>(vf, pf, ones, o, lacc);
}

// WR row groups x WK key groups of one wave64 each.  A wave owns 16 * NT rows of its row
// group; the WR waves of a key group share a ring of NU units and walk that group's
// tiles (every WK-th of the chunk) in lock step.
template <int D, int WR, int WK, int NT, int NU>
__global__ __launch_bounds__(64 * WR * WK) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_fp8(Fp8Args a) {
  using TL = TileLayout<D>;
  using CL = CodeLayout<D>;
  constexpr int kThreads = 64 * WR * WK, kWaves = WR * WK;
  constexpr int kRows = 16 * NT, RB = kRows * WR, NTG = NT * WR;
  constexpr bool kAlone = WR == 1;  // a wave with a ring of its own
  constexpr int NC = D / 32, DT = D / 16;
  constexpr int UNIT = 64 * D;
  constexpr int kDma = UNIT / 1024;                 // 1 KB DMA instructions per unit,
  constexpr int PU = kDma >= WR ? kDma / WR : 1;    // and per wave of it (wr < kDma / PU)
  static_assert(UNIT == TL::kBytes && kDma == 2 * CL::kDma && PU * NU + 8 < 48, "a unit");
  static_assert(NU >= 2, "a tree tile is two units");
  extern __shared__ __attribute__((aligned(128))) unsigned char smem[];

  // The work item: one of the even split, which goes by the kv_lens, or (unsplit) one that
  // is known at once, with the sequence's length still on its way.
  WorkItem it{};
  int chunk = a.chunk, kvl = 0, asked = 0, part0 = 0;  // part0: the row block's first chunk partial
  const bool split = a.slots > 0;
  if (split) {
    const int item = even_item(blockIdx.x, a.slots, a.nRB, a.Hkv, it);
    if (item < 0) return;
    const EvenItem ev = even_split<false>(a, item, 0, 0);
    if (ev.s < 0) return;
    it.b = ev.b;
    it.s = ev.s;
    chunk = ev.chunk;
    kvl = ev.kvl;
    part0 = (it.g * a.nRB + it.rb) * a.slots + ev.first;
  } else {
    // (a contiguous run of items per XCD, so whole sequences: of 64 sequences of 512 to
    // 8192 rows the XCD with the most has 1.1 to 1.5 times the mean)
    if (!work_item(gridDim.x, a.nwork, a.S, a.nRB, 0, a.B, a.Hkv, blockIdx.x, it)) return;
    if (a.kv_len) asked = a.kv_len[it.b];
  }
  const int s = it.s, rb = it.rb, g = it.g, b = it.b;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int g4 = lane >> 4, l16 = lane & 15;
  const int r0 = rb * RB;
  const int rows = min(RB, a.M - r0);
  const int i_lo = r0 / a.G, i_hi = (r0 + rows - 1) / a.G;
  const int ntt = i_hi / kKeyTile + 1;  // words of a node's ancestor bitmask
  const int t0 = s * chunk;

  // All that does not hang on the length is asked for before it is there: parents (of up
  // to 32 nodes every wave has its own, else the workgroup shares them), queries, and
  // the places of the first tiles.  One round trip to memory less: a single token over
  // 200 rows 6.7 -> 6.0 us.
  const bool small = a.N <= 32;
  constexpr int kParPerThread = (kMaxNodes + kThreads - 1) / kThreads;
  constexpr int NQ = NT * NC;  // query loads per lane
  int pv[kParPerThread];
  const int32_t* pr = a.parent ? a.parent + (size_t)b * a.N : (const int32_t*)a.q;  // NULL: a chain
  int own_parent = load_i32(pr + (a.parent && lane < a.N ? lane : 0));
  if (!small) {
    // indices clamped rather than branched on, so the loads stay in flight
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) {
      const int i = tid + kThreads * k;
      pv[k] = load_i32(pr + (!a.parent ? 0 : i < a.N ? i : a.N - 1));
    }
  }
  // ---- queries: B operand of S^T = K Q^T
  const int wrow0 = r0 + kRows * wr;
  bf16x8 qf[NT][NC];
  bool qok[NT];
  int node_of[NT];  // this lane's row's, of the last row past it
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = wrow0 + nt * 16 + l16;
    const int in = min(r, a.M - 1);
    qok[nt] = r < a.M;
    node_of[nt] = in / a.G;
    const int h = g * a.G + in % a.G;
    const __bf16* qp = a.q + ((size_t)(b * a.N + node_of[nt]) * a.Hq + h) * D + head_dim(0, g4);
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) qf[nt][cc] = load_b128(qp + head_dim(cc, 0));
  }
  // Tile i0 + lane's place in the pools, in groups (of tiles past the cache's, or the
  // capacity, somewhere in the pool).  Block numbers are clamped into the pool.
  auto group_of = [&](int i0) {
    const int first = min((t0 + wk + WK * (i0 + lane)) * kKeyTile, a.Lmax - kKeyTile);
    const int blk = a.block_table[(size_t)b * a.max_blocks + (first >> a.block_shift)];
    const int page = min(max(blk, 0), a.num_blocks - 1), per = a.block_shift - 5;
    return ((page * a.Hkv + g) << per) + ((first >> 5) & ((1 << per) - 1));
  };
  int group = 0;  // of tiles 64 j + lane, j that of the tile issued last
  if (a.Lmax > 0) group = group_of(0);
  // exponents of tiles 64 j + lane, j that of the tile attended to (without a cache
  // anything that may be read: the loads are counted below)
  int kexp = load_u8(a.Lmax > 0 ? a.ke + group : (const uint8_t*)a.q);
  int vexp = load_u8(a.Lmax > 0 ? a.ve + group : (const uint8_t*)a.q);

  if (!split) kvl = context_rows_of(a, asked);
  const Segment sg = segment(a, kvl, i_hi);
  const int nct = sg.nct, T = sg.T;
  const int t1 = min(T, t0 + chunk);
  if (t0 >= t1) return;  // empty chunk: the merge reads only chunks with tiles
  const bool has_tree = t1 > nct;

  const uint32_t ring = (uint32_t)(uintptr_t)smem + wk * NU * UNIT;
  const unsigned char* ring_ptr = smem + wk * NU * UNIT;
  uint32_t* anc = reinterpret_cast<uint32_t*>(smem + WK * NU * UNIT);  // behind the rings
  int32_t* par = reinterpret_cast<int32_t*>(anc + (RB / a.G + 2) * ntt);
  __shared__ unsigned long long brk[kMaxNodes / 64];

  // The key group's tiles are t0 + wk + WK * i, n_mine of them, the first n_c the cache's.
  // All waves take n_iter steps, so that the steps' barriers line up.
  const int n_iter = (t1 - t0 + WK - 1) / WK;
  const int n_mine = t0 + wk < t1 ? (t1 - t0 - wk + WK - 1) / WK : 0;
  const int n_c = max(0, (min(t1, nct) - t0 - wk + WK - 1) / WK);
  const int n_units = 2 * n_mine - n_c;

  const size_t krow = (size_t)a.Hkv * D;  // the tree's: elements between consecutive nodes
  const size_t tree0 = ((size_t)b * a.N * a.Hkv + g) * D;
  const char* ktree = (const char*)(a.kt + tree0);
  const char* vtree = (const char*)(a.vt + tree0);

  // Moves unit u into its place of the ring.  DMA q of it fetches rows q * kRowsPerDma ..
  // of K or V, a lane one row's chunk that the swizzle places at the lane's; rows past the
  // valid ones are clamped onto one (the mask gives them no weight, and what lies there
  // may be no number).
  const bool mover = wr * PU < kDma;
  const uint32_t code_off = CL::off(lane / CL::kCPR, lane % CL::kCPR);
  auto issue_codes = [&](int u, uint32_t dst, auto read_once) __attribute__((always_inline)) {
    const size_t at = (size_t)__builtin_amdgcn_readlane(group, u & 63) * CL::kBytes;
    const int valid = kvl - (t0 + wk + WK * u) * kKeyTile;
#pragma unroll
    for (int k = 0; k < PU; ++k) {
      const int q = wr * PU + k, j = q % CL::kDma;
      const char* base = (q >= CL::kDma ? (const char*)a.vc : (const char*)a.kc) + at;
      uint32_t off = (code_off ^ CL::dma_flip(j)) + j * 1024;
      if (valid < kKeyTile) off -= D * max(0, j * CL::kRowsPerDma + lane / CL::kCPR - (valid - 1));
      if constexpr (read_once.value) dma16_once(base, off, dst + q * 1024);
      else dma16(base, off, dst + q * 1024);
    }
  };
  // A tile that only one row block reads does not stay in the caches: single tokens of 64
  // sequences of 512 to 8192 rows 114 us, else 131; two trees of 16 nodes over 131072 rows
  // 114, else 118; over 1200 drawn shapes of up to 32 rows 4% less time.  With more row
  // blocks the others' reads would miss (four tokens of five sequences, two row blocks: 68
  // -> 76 us); four waves that share a ring have them.  (Pages that several sequences share
  // are read by each of them: tokens of 64 sequences of 8192 rows 174 us, with eight at a
  // time on the same pages 104; ordinary loads were not tried there.)
  const bool once = WR <= 2 && a.nRB == 1;
  auto issue_unit = [&](int u) __attribute__((always_inline)) {
    const uint32_t dst = ring + (u % NU) * UNIT;
    if (u < n_c) {
      if (once) issue_codes(u, dst, std::true_type{});
      else issue_codes(u, dst, std::false_type{});
    } else {
      const int first = (t0 + wk + WK * (n_c + ((u - n_c) >> 1)) - nct) * kKeyTile;
      const char* base = ((u - n_c) & 1 ? vtree : ktree) + (size_t)first * krow * 2;
#pragma unroll
      for (int k = 0; k < PU; ++k) {
        const int q = wr * PU + k;
        const int r = q * TL::kRowsPerDma + lane / TL::kCPR;
        const int row = min(first + r, i_hi) - first;
        dma16(base, (uint32_t)(row * (int)krow * 2 + ((lane % TL::kCPR) ^ TL::swz(r)) * 16),
              dst + q * 1024);
      }
    }
  };
  int issued = min(NU, n_units);
  const int in_flight = mover ? issued * PU : 0;  // the prologue's DMAs
  if (mover)
    for (int u = 0; u < issued; ++u) issue_unit(u);

  // ---- tree structure: which nodes are a node's ancestors or itself, as bits
  int invalid = 0;
  // of this lane's rows: the nodes relative to i_lo, in small trees what they see of it
  int node_rel[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) node_rel[nt] = node_of[nt] - i_lo;
  // the parents are done once at most queries, exponents and DMAs are in flight
  wait_vm_any(NQ + 2 + in_flight);
  loaded(own_parent);
  if (has_tree && small) {
    // node `lane`: twice as far up with every step
    const int p = a.parent ? own_parent : lane - 1;
    const bool in = lane < a.N;
    invalid = __any(in && (lane == 0 ? p != -1 : p < 0 || p >= lane));
    uint32_t up = in ? 1u << lane : 0u;
    int to = in && lane > 0 && !invalid ? p : lane;
    for (int far = 1; far < a.N; far *= 2) {
      up |= __shfl(up, to);
      to = __shfl(to, to);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) node_rel[nt] = __shfl((int)up, node_of[nt]);
  }
  if (!small) {
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) loaded(pv[k]);
  }
  if (has_tree && !small) {
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) {
      const int i = tid + kThreads * k;
      const int p = a.parent ? pv[k] : i - 1;
      const bool in = i < a.N;
      if (in) par[i] = p;
      invalid |= in && ((i == 0) ? (p != -1) : (p < 0 || p >= i));
      // nodes whose parent is not the node before them
      const unsigned long long breaks = __ballot(in && p != i - 1);
      if (lane == 0 && in) brk[i >> 6] = breaks;
    }
    invalid = __syncthreads_or(invalid);
    // Up from node to node; after some steps, which end what drafts are usually like, a
    // run of nodes that follow their parents at a time (of a chain 64: step by step a
    // chain of 269 nodes took 30 us; 86 nodes of depth 12 by runs alone 1 us more).
    const int nodes = i_hi - i_lo + 1;
    for (int t = tid; t < nodes; t += kThreads) {
      uint32_t* wd = anc + t * ntt;
      for (int k = 0; k < ntt; ++k) wd[k] = 0u;
      int u = i_lo + t;
      for (int steps = 0; steps < 16 && u > 0; ++steps) {
        wd[u >> 5] |= 1u << (u & 31);
        const int p = par[u];
        u = p >= 0 && p < u ? p : -1;  // invalid tree: the output becomes NaN
      }
      while (u >= 0) {
        const int base = u & ~63;
        const unsigned long long m = brk[u >> 6] & (~0ull >> (63 - (u & 63)));
        const int top = m ? base + 63 - __clzll((long long)m) : base;  // the run's first node
        const unsigned long long run = (~0ull >> (63 - (u - top))) << (top & 63);
        wd[base >> 5] |= (uint32_t)run;
        if ((base >> 5) + 1 < ntt) wd[(base >> 5) + 1] |= (uint32_t)(run >> 32);
        if (top == 0) break;
        const int p = m ? par[top] : top - 1;
        if (p < 0 || p >= top) break;  // invalid tree: the output becomes NaN
        u = p;
      }
    }
    __syncthreads();
  }

  // queries and exponents are done once at most the DMAs are in flight
  wait_vm_any(in_flight);
  loaded(kexp);
  loaded(vexp);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) {
      loaded(qf[nt][cc]);
      if (!qok[nt]) qf[nt][cc] = bf16x8{};
    }

  // O^T accumulators, and the row sums of the rounded weights as ones^T P^T
  f32x4 o[DT][NT], lacc[NT];
  float m[NT], thr[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = thr[nt] = -INFINITY;
    lacc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8 ones = {(__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f,
                 (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f};
  asm volatile("" : "+v"(ones));  // keep it in registers, not rebuilt every tile
  const float inv_c = 1.f / a.c;

  const bool busy = wrow0 < a.M;  // else only the tiles are moved
  uint32_t bits[NT] = {};
  int head = 0;  // units taken so far
  // Fills the places of the units before `head` again.  Their LDS reads must be done by
  // then: behind a shared ring's barrier they are, and a wave alone waits for its own
  // (that their values were used earlier does not order the reads before the DMAs).
  auto refill = [&]() {
    if (kAlone) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    while (issued < n_units && issued < head + NU) {
      if (issued < n_c && (issued & 63) == 0) {
        group = group_of(issued);
        loaded(group);
      }
      if (mover) issue_unit(issued);
      ++issued;
    }
  };
  // Waits for the units before `next`, which are there once at most the later ones' DMAs
  // are in flight.  In a shared ring the barrier makes the whole group's visible, and the
  // units that were taken before it are done with: their places are filled again.
  auto arrive = [&](int next) {
    if (next > head && mover) wait_tiles<PU, NU>(issued - next);
    if (!kAlone) {
      __syncthreads();
      refill();
    }
    head = next;
  };
  auto exponents = [&](int i) {  // of tile i and the ones after it, every 64 tiles
    if (i > 0 && i < n_c && (i & 63) == 0) {
      const int at = group_of(i);
      kexp = a.ke[at];
      vexp = a.ve[at];
      loaded(kexp);
      loaded(vexp);
    }
  };
  // A wave alone frees a cache tile's place as soon as it holds the codes.
  Codes<D> codes;
  auto take = [&](uint32_t unit, int hg4, int hl16) {
    read_keys<D>(unit, codes, hg4, hl16);
    if (kAlone) {
      read_values<D>(unit, codes, hg4, hl16);
      refill();
    }
  };
  auto scale_of = [&](int exps, int i) {
    return __int_as_float(__builtin_amdgcn_readlane(exps, i & 63) << 23);
  };
  // Full cache tiles first, without masking.  Waves that share a ring meet once for half
  // of it, not at every tile: between two meetings they drift apart, so that one's matrix
  // work falls on the other's vector work.
  constexpr int kMeet = kAlone ? 1 : NU / 2;
  static_assert(64 % kMeet == 0, "exponents are looked up where waves meet");
  auto full_tiles = [&](int k) {  // of key group k
    return max(0, (min(t1, kvl / kKeyTile) - t0 - k + WK - 1) / WK);
  };
  const int n_full = full_tiles(wk);
  const int n_meet = kAlone ? n_full : (full_tiles(0) + kMeet - 1) / kMeet;  // the same for all groups
  int i = 0;
  for (int k = 0; k < n_meet; ++k) {
    const int end = min(n_full, (k + 1) * kMeet);
    arrive(max(end, head));
    exponents(i);
    for (; i < end && busy; ++i) {
      const uint32_t unit = ring + (i % NU) * UNIT;
      take(unit, g4, l16);
      attend_codes<D, NT, false, kAlone>(codes, unit, scale_of(kexp, i), scale_of(vexp, i), qf, o, lacc, m,
                                         thr, ones, a.c, inv_c, bits, g4, l16);
    }
  }
  // Then the cache's tail and the tree, tile by tile (as many steps for all groups).
  const int n_rest = kAlone ? n_mine - n_full : n_iter - full_tiles(WK - 1);
  for (int k = 0; k < n_rest; ++k) {
    i = n_full + k;
    const int at = (head % NU) * UNIT, at_v = ((head + 1) % NU) * UNIT;
    arrive(head + (i < n_mine ? (i < n_c ? 1 : 2) : 0));
    exponents(i);
    if (i >= n_mine || !busy) continue;
    // (opaque lane numbers: the addresses of these few tiles' reads are not kept through
    // the loop above)
    int hg4 = g4, hl16 = l16;
    asm volatile("" : "+v"(hg4), "+v"(hl16));
    if (i < n_c || !small) {
      tile_bits<NT>(MaskInfo{t0 + wk + WK * i, nct, kvl, ntt, 0, anc}, node_rel, bits);
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) bits[nt] = (uint32_t)node_rel[nt];
    }
    if (i < n_c) {
      take(ring + at, hg4, hl16);
      attend_codes<D, NT, true, kAlone>(codes, ring + at, scale_of(kexp, i), scale_of(vexp, i), qf, o, lacc,
                                        m, thr, ones, a.c, inv_c, bits, hg4, hl16);
    } else {
      attend_tree<D, NT>(ring_ptr + at, ring_ptr + at_v, qf, o, lacc, m, thr, ones, a.c, inv_c, bits, hg4,
                         hl16);
      if (kAlone) refill();
    }
  }

  const LateArgs* z = late_args();
  float lsum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) lsum[nt] = lacc[nt][0];
  // A row block that is one chunk writes its output here, else its partial; fragments
  // wholly past the last row are neither stored nor read by the merges.
  const int nval = (T + chunk - 1) / chunk;
  const bool whole = z->S == 1 || nval == 1;
  const size_t grp = (size_t)(b * z->Hkv + g) * z->nRB + rb;  // row block id
  auto rows_at = [&](int ntg) { return r0 + ntg * 16 < z->M; };
  auto emit = [&](int dt, int ntg, const f32x4& acc, float mstar, float l) {
    if (whole) {
      const int r = r0 + ntg * 16 + l16;
      if (r >= z->M) return;
      const int node = r / z->G, h = g * z->G + r % z->G;
      store_out4(z->out + ((size_t)(b * z->N + node) * z->Hq + h) * D + 16 * dt + 4 * g4, acc, 1.f / l,
                 invalid != 0);
      return;
    }
    f32x4* po = &z->ws_o[((size_t)(part0 + s) * DT * NTG + dt * NTG + ntg) * 64 + lane];
    float2* pml = &z->ws_ml[(size_t)(part0 + s) * RB + ntg * 16 + l16];
    if (z->fused) {  // read by another workgroup of this kernel
      store_dev(po, acc);
      if (dt == 0 && g4 == 0) store_dev(pml, make_float2(mstar, l));
    } else {         // read by the merge kernel
      *po = acc;
      if (dt == 0 && g4 == 0) *pml = make_float2(mstar, l);
    }
  };
  if (WK == 1) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int ntg = wr * NT + nt;
      if (!rows_at(ntg)) break;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) emit(dt, ntg, o[dt][nt], m[nt], lsum[nt]);
    }
  } else {
    // ---- merge the WK key groups of each row group (same rows, disjoint keys)
    __syncthreads();  // rings and tree tables are dead from here on
    f32x4* obuf = reinterpret_cast<f32x4*>(smem);
    float2* mlbuf = reinterpret_cast<float2*>(smem + (size_t)kWaves * kRows * D * 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) obuf[((wave * DT + dt) * NT + nt) * 64 + lane] = o[dt][nt];
    if (g4 == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        mlbuf[wave * kRows + nt * 16 + l16] = make_float2(m[nt], lsum[nt]);
    }
    __syncthreads();
    for (int f = wk; f < DT * NT; f += WK) {
      const int dt = f / NT, nt = f % NT;
      if (!rows_at(wr * NT + nt)) continue;
      const int rw = nt * 16 + l16;  // row within the wave's 32
      float mw[WK], mstar = -INFINITY;
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        mw[k] = mlbuf[(k * WR + wr) * kRows + rw].x;
        mstar = fmaxf(mstar, mw[k]);
      }
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float e = mw[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[k] - mstar);
        l += e * mlbuf[(k * WR + wr) * kRows + rw].y;
        acc += e * obuf[(((k * WR + wr) * DT + dt) * NT + nt) * 64 + lane];
      }
      emit(dt, wr * NT + nt, acc, mstar, l);
    }
  }
  if (whole || !z->fused) return;

  // ---- fused split-KV merge, as in attn_main: the chunk that arrives last merges
  __shared__ int s_last;
  if (has_tree && tid == 0)  // every row block has a chunk with tree tiles
    __hip_atomic_store(z->tree_bad + grp, invalid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  wait_all_vm();
  __syncthreads();
  if (tid == 0) {
    const unsigned int before =
        __hip_atomic_fetch_add(z->arrived + grp, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before + 1 == (unsigned int)nval;
    if (last) __hip_atomic_store(z->arrived + grp, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = last;
  }
  __syncthreads();
  if (!s_last) return;
  const bool bad = __hip_atomic_load(z->tree_bad + grp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0;
  constexpr int kMerge = kWaves < NTG * DT ? kWaves : NTG * DT;  // a wave per fragment at most
  if (wave < kMerge) merge_chunks<D, RB, kMerge>(z, part0, nval, b, g, r0, bad, wave, lane);
}

// Second kernel of the plans whose merge is too much for one workgroup:
// out = sum_s e_s O_s / sum_s e_s l_s with e_s = 2^(m_s - m*).  A workgroup per 16 x 16
// fragment, whose four waves take the row block's chunks in turn and are joined in LDS
// (two trees of 16 nodes over 131072 rows, 64 chunks each: 114.4 us, with a wave per
// fragment 119.7).
// What can be asked for before the number of chunks is known is asked for at once, as in
// attn_combine (slots past the chunks lie inside the workspace).
template <int D, int RB>
__global__ __launch_bounds__(256) void combine_fp8(Fp8Args a) {
  constexpr int NTG = RB / 16, DT = D / 16, U = 8, W = 4;
  constexpr int kParPerThread = kMaxNodes / 256;
  __shared__ f32x4 accs[W][64];
  __shared__ float2 mls[W][16];
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int f = blockIdx.x % (DT * NTG), blk = blockIdx.x / (DT * NTG);
  const int rb = blk % a.nRB, g = blk / a.nRB % a.Hkv, b = blk / a.nRB / a.Hkv;
  const int dt = f / NTG, ntg = f % NTG;
  const int row = ntg * 16 + l16, r = rb * RB + row;
  if (rb * RB + ntg * 16 >= a.M) return;  // no rows: nothing was stored
  int pv[kParPerThread];
#pragma unroll
  for (int k = 0; k < kParPerThread; ++k) {
    const int i = threadIdx.x + 256 * k;
    pv[k] = i >= a.N ? 0 : (a.parent ? a.parent[(size_t)b * a.N + i] : i - 1);
  }
  const int i_hi = (min(rb * RB + RB, a.M) - 1) / a.G;
  EvenItem ev{a.chunk, b, 0, 0, 0};
  if (a.B > 1) ev = even_split<false>(a, -1, b, 0);
  const size_t base = (size_t)(g * a.nRB + rb) * a.slots + ev.first;  // the first chunk partial
  const int nslot = a.slots - ev.first;
  float2 ml[U];
  f32x4 ov[U];
  auto ask = [&](int s0, int end) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + W * u;
      if (s < end) {
        ml[u] = a.ws_ml[(base + s) * RB + row];
        ov[u] = a.ws_o[((base + s) * DT * NTG + dt * NTG + ntg) * 64 + lane];
      }
    }
  };
  ask(wave, nslot);
  if (a.B == 1) ev = even_one<false>(a, 0, 0);
  const int nval = (segment(a, ev.kvl, i_hi).T + ev.chunk - 1) / ev.chunk;
  if (nval == 1) return;  // written by its only chunk
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = wave; s0 < nval; s0 += W * U) {
    if (s0 >= W * U) ask(s0, nval);
    float mb = m;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + W * u < nval) mb = fmaxf(mb, ml[u].x);
    if (mb != -INFINITY) {  // else every chunk so far saw no key: nothing to add
      const float ea = __builtin_amdgcn_exp2f(m - mb);  // 0 while m = -inf
      l *= ea;
      acc *= ea;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s0 + W * u < nval && ml[u].x != -INFINITY) {
          const float e = __builtin_amdgcn_exp2f(ml[u].x - mb);
          l += e * ml[u].y;
          acc += e * ov[u];
        }
      m = mb;
    }
  }
  int bad = 0;
#pragma unroll
  for (int k = 0; k < kParPerThread; ++k) {
    const int i = threadIdx.x + 256 * k;
    if (i < a.N) bad |= (i == 0) ? (pv[k] != -1) : (pv[k] < 0 || pv[k] >= i);
  }
  accs[wave][lane] = acc;
  if (g4 == 0) mls[wave][l16] = make_float2(m, l);
  bad = __syncthreads_or(bad);
  if (wave > 0 || r >= a.M) return;
  float mstar = -INFINITY;
#pragma unroll
  for (int w = 0; w < W; ++w) mstar = fmaxf(mstar, mls[w][l16].x);
  l = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float mw = mls[w][l16].x;
    const float e = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mstar);
    l += e * mls[w][l16].y;
    acc += e * accs[w][lane];
  }
  const int node = r / a.G, h = g * a.G + r % a.G;
  store_out4(a.out + ((size_t)(b * a.N + node) * a.Hq + h) * D + 16 * dt + 4 * g4, acc, 1.f / l, bad != 0);
}

template <int D, int ARR>
static hipError_t launch_fp8_t(const Fp8Args& a, const AttnPlan& p, hipStream_t st) {
  constexpr ArrangementFp8 ar = kArrangementsFp8[ARR];
  constexpr auto kernel = &attn_fp8<D, ar.WR, ar.WK, ar.NT, D == 128 ? ar.NU128 : ar.NU64>;
  // the kernel's LDS limit on each device, raised only when a call needs more
  constexpr int kDevices = 64;
  static std::atomic<int> limit[kDevices];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kDevices) return hipErrorInvalidDevice;
  if (limit[dev].load(std::memory_order_acquire) < (int)p.lds_bytes) {
    static std::mutex raising;
    std::lock_guard<std::mutex> hold(raising);
    if (limit[dev].load(std::memory_order_relaxed) < (int)p.lds_bytes) {
      e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)p.lds_bytes);
      if (e != hipSuccess) return e;
      limit[dev].store((int)p.lds_bytes, std::memory_order_release);
    }
  }
  hipLaunchKernelGGL(kernel, dim3(p.slots > 0 ? p.even_grid : p.grid), dim3(p.threads), p.lds_bytes, st,
                     a);
  e = hipGetLastError();
  if (e != hipSuccess || p.S == 1 || p.fused) return e;
  constexpr int RB = 16 * ar.NT * ar.WR;
  const int frags = a.B * a.Hkv * a.nRB * (D / 16) * (RB / 16);
  hipLaunchKernelGGL((combine_fp8<D, RB>), dim3(frags), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int D, int K = 0>
static hipError_t launch_fp8_d(const Fp8Args& a, const AttnPlan& p, hipStream_t st) {
  if constexpr (K < kNumArrangementsFp8)
    return p.arr == K ? launch_fp8_t<D, K>(a, p, st) : launch_fp8_d<D, K + 1>(a, p, st);
  else
    return hipErrorInvalidValue;
}

hipError_t launch_attention_fp8(const void* q, const void* kp, const void* vp, const uint8_t* ke,
                                const uint8_t* ve, const int32_t* block_table, int block_shift,
                                int max_blocks, int num_blocks, const void* kt, const void* vt,
                                const int32_t* parent, const int32_t* kv_len, void* out, int B, int N,
                                int Hq, int Hkv, int D, int Lmax, float scale, void* ws,
                                const AttnPlan& p, hipStream_t st) {
  Fp8Args a{};
  a.q = (const __bf16*)q;
  a.kc = (const __bf16*)kp;  // (bytes: codes)
  a.vc = (const __bf16*)vp;
  a.ke = ke;
  a.ve = ve;
  a.block_table = block_table;
  a.block_shift = block_shift;
  a.max_blocks = max_blocks;
  a.num_blocks = num_blocks;
  a.kt = (const __bf16*)kt;
  a.vt = (const __bf16*)vt;
  a.parent = parent;
  a.kv_len = kv_len;
  a.out = (__bf16*)out;
  a.arrived = (unsigned int*)ws;
  a.tree_bad = (int*)ws + kSyncGroups;
  a.ws_o = (f32x4*)((char*)ws + p.ws_sync_bytes);
  a.ws_ml = (float2*)((char*)ws + p.ws_sync_bytes + p.ws_o_bytes);
  a.B = B;
  a.N = N;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.Lmax = Lmax;
  a.G = p.G;
  a.M = p.M;
  a.nRB = p.nRB;
  a.S = p.S;
  a.chunk = p.chunk;
  a.nwork = p.nwork;
  a.fused = p.fused;
  a.slots = p.slots;
  a.min_chunk = p.min_chunk;
  a.rslots = p.slots > 0 ? 1.f / (float)p.slots : 0.f;
  a.rslack = p.slots > B ? 1.f / (float)(p.slots - B) : 1.f;
  a.cgroup = 1;
  a.c = scale * 1.4426950408889634f;
  return D == 128 ? launch_fp8_d<128>(a, p, st) : launch_fp8_d<64>(a, p, st);
}

}  // namespace tv
