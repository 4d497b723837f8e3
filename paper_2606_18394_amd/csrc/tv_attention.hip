// Tree-verification attention for CDNA4 (gfx950).
//
// Computes, for every draft-tree node v of every sequence and every query
// head, softmax(q_v K^T * scale + M_v) V over the sequence's cached prefix
// and the tree nodes, where the tree-causal mask M_v keeps only v's
// ancestors and v itself (Sec. 2.2, tree-causal mask and masked attention
// equations).  The ancestor relation is rebuilt inside each workgroup as a
// bitmask in LDS from the parent array; no dense mask ever exists (App. E).
//
// Work decomposition.  Rows of one (sequence b, KV head g) pair are the N*G
// (node, head-in-group) pairs, row r = node * G + head.  Keys are cut into
// 32-key tiles: ceil(kv_len/32) cache tiles, then the tree tiles up to the
// last node of the row block (a node never sees a later node because
// parents precede children).  The tiles are cut into contiguous chunks
// (split-KV) of one size for the whole batch, found on the device from the
// kv_lens (even_split), so that a capacity far above the lengths or a ragged
// batch still gives chunks of like size; a sequence of one chunk is written
// straight to the output.  A workgroup takes one block of 32*WR rows and
// one chunk with WR x WK wave64s: WR row groups of 32 rows, and WK key
// groups that share out the chunk's tiles, each streaming its tiles through
// an LDS ring of NS stages; key groups merge their softmax states in LDS at
// the end.  The host plan (tv_plan.h) picks WR, WK, NS and S per shape so
// that every CU holds 8 waves (two per SIMD).  The prologue requests the
// parents, the queries and every ring stage before it uses any of them;
// with several key groups on a full grid, key group 0 alone loads the
// queries and hands them to the others through LDS.
//
// Per tile.  K and V move HBM -> LDS with global_load_lds_dwordx4 (no
// register staging), rows XOR-swizzled in 16-byte chunks so the transposing
// V reads are free of bank conflicts and the K reads at most two-way (see
// TileLayout).  A wave computes S^T = K Q^T with
// v_mfma_f32_16x16x32_bf16 (keys on the M side, its 32 rows on the N side),
// runs an fp32 base-2 online softmax on the accumulators with a lazily moved
// reference maximum, and accumulates O^T += V^T P^T: P^T comes straight from
// the S^T accumulators (the 32 keys are ordered so the B operand needs no
// data movement) and V^T from ds_read_b64_tr_b16 transposing reads.
//
// Split-KV merge (sequences of several chunks).  Every chunk stores its (max,
// sum, O) partial.  The chunk that finishes last merges its row block inside
// this kernel (arrival counters in the workspace) when the plan prices that
// below a second kernel that merges all row blocks.
//
// The training mask of many small blocks has a kernel of its own (attn_packed).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "tv_attend.h"

namespace tv {

// A workgroup of WR x WK wave64s: WR row groups x WK key groups.  A wave owns 32 rows of its row group; the WR
// waves of a key group share one LDS ring and walk that group's tiles (every
// WK-th tile of the chunk) in lock step; WK > 1 groups merge their partial
// softmax states in LDS at the end.
template <int D, int WR, int WK, int NS, bool kPaged, bool kShareQ>
__global__ __launch_bounds__(64 * WR * WK) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_main(AttnArgs a) {
  using TL = TileLayout<D>;
  constexpr int kThreads = 64 * WR * WK;
  constexpr int kWaves = WR * WK;
  constexpr int RB = kRowsPerWave * WR; // rows per workgroup
  constexpr int NT = kRowsPerWave / 16; // 16-row tiles per wave
  constexpr int NTG = RB / 16;          // 16-row tiles per workgroup
  constexpr int NC = D / 32;            // 32-wide head-dim chunks (QK^T)
  constexpr int DT = D / 16;            // 16-wide head-dim tiles (PV)
  constexpr int STAGE = 2 * TL::kBytes; // K tile + V tile
  constexpr int PW = 2 * TL::kDma / WR; // DMAs per wave per tile
  static_assert(PW >= 1 && PW * WR == 2 * TL::kDma, "DMA split");
  static_assert(NS >= 1, "ring does not fit");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  WorkItem it{};
  int chunk = a.chunk, kvl, part0;  // part0: the row block's first chunk partial
  // One sequence's length is on its way while the work item is found (64 nodes over
  // 4096 rows 18.04 -> 17.80 us).  Not with one key group, whose plans have long
  // chunks: there 512 nodes over 8192 rows took 148.3 us so, and 147.7 without.
  int asked = 0;
  if constexpr (WK > 1) {
    if (a.kv_len) asked = a.kv_len[0];
    asm volatile("" ::: "memory");
  }
  if (a.slots > 0) {
    const int item = even_item(blockIdx.x, a.slots, a.nRB, a.Hkv, it);
    if (item < 0) return;
    const EvenItem ev = even_split<(WK > 1)>(a, item, 0, asked);
    if (ev.s < 0) return;
    it.b = ev.b;
    it.s = ev.s;
    chunk = ev.chunk;
    kvl = ev.kvl;
    part0 = (it.g * a.nRB + it.rb) * a.slots + ev.first;
  } else {
    if (!work_item(gridDim.x, a.nwork, a.S, a.nRB, a.spread, a.B, a.Hkv, blockIdx.x, it)) return;
    if (a.spread == 2) longest_first(a, blockIdx.x, it);
    kvl = context_rows(a, it.b);
    part0 = ((it.b * a.Hkv + it.g) * a.nRB + it.rb) * a.S;
  }
  const int s = it.s, rb = it.rb, g = it.g, b = it.b;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int g4 = lane >> 4, l16 = lane & 15;

  const int r0 = rb * RB;
  const int rows = min(RB, a.M - r0);
  const int i_lo = r0 / a.G, i_hi = (r0 + rows - 1) / a.G;
  const Segment sg = segment(a, kvl, i_hi);
  const int nct = sg.nct, T = sg.T;
  const int ntt = i_hi / kKeyTile + 1;  // words of a node's ancestor bitmask
  const int t0 = s * chunk;
  const int t1 = min(T, t0 + chunk);
  if (t0 >= t1) return;  // empty chunk: the merge reads only chunks with tiles
  const bool has_tree = a.tail ? t1 * kKeyTile > kvl : t1 > nct;

  constexpr int RING = WK * NS * STAGE;
  const uint32_t ring = (uint32_t)(uintptr_t)smem + wk * NS * STAGE;
  const unsigned char* ring_ptr = smem + wk * NS * STAGE;
  // the block's queries (kShareQ) follow the rings, then the tree tables
  static_assert(!kShareQ || (WK > 1 && WR > 1), "queries are shared between key groups");
  constexpr bool qshare = kShareQ;
  const bool qload = !qshare || wk == 0;  // this wave loads its queries from memory
  unsigned char* qlds = smem + RING;
  uint32_t* anc = reinterpret_cast<uint32_t*>(smem + RING + (qshare ? RB * D * 2 : 0));
  const int anc_nodes = RB / a.G + 2;
  int32_t* par = reinterpret_cast<int32_t*>(anc + anc_nodes * ntt);
  int* flag = par + a.N;

  const size_t krow = (size_t)a.Hkv * D;  // elements between consecutive keys
  const size_t cache0 = kPaged ? 0 : (size_t)(b / a.cgroup) * a.Lmax * krow;  // paged: pool
  const __bf16* kcache = a.kc + cache0 + (size_t)g * D;
  const __bf16* vcache = a.vc + cache0 + (size_t)g * D;
  const size_t tree0 = (size_t)b * a.N * krow + (size_t)g * D;  // unused with a tree tail
  const __bf16* ktree = a.tail ? kcache : a.kt + tree0;
  const __bf16* vtree = a.tail ? vcache : a.vt + tree0;

  // This lane's share of the DMA instructions of one tile: instruction q
  // (q < kDma: K, else V) covers tile rows j*kRowsPerDma.. (j = q % kDma);
  // lane i fetches row j*kRowsPerDma + i/kCPR at the logical chunk that the
  // swizzle places at physical chunk i % kCPR.  dma_off is that byte offset
  // from the first row of a full tile.
  uint32_t dma_off[PW];
#pragma unroll
  for (int k = 0; k < PW; ++k) {
    const int q = wr * PW + k;
    const int r = (q % TL::kDma) * TL::kRowsPerDma + lane / TL::kCPR;
    dma_off[k] = (uint32_t)(r * (int)krow * 2 + ((lane % TL::kCPR) ^ TL::swz(r)) * 16);
  }
  const TreeSrc src{(const char*)kcache,
                    (const char*)vcache,
                    (const char*)ktree,
                    (const char*)vtree,
                    kPaged ? a.block_table + (size_t)b * a.max_blocks : nullptr,
                    a.block_shift,
                    a.num_blocks,
                    (int)krow * 2,
                    a.tail ? kvl + i_hi + 1 : kvl,
                    nct,
                    i_hi};

  // iteration i handles tile t0 + wk + WK*i of this wave's key group; all
  // waves run n_iter iterations so the per-iteration barriers line up
  const int n_iter = t1 > t0 ? (t1 - t0 + WK - 1) / WK : 0;
  const int n_mine = t0 + wk < t1 ? (t1 - t0 - wk + WK - 1) / WK : 0;  // valid tiles

  // Issue order: parents, queries, then the first tiles' DMAs, all before
  // any of them is used.  When the WR waves of a key group share its ring
  // (WR > 1) the prologue fills every stage: the ring's own refills come
  // after a workgroup barrier, and the first of them would otherwise wait
  // for the first tile's round trip.  A single-wave key group refills
  // before its waits and keeps one stage for that.  (Measured on the
  // Qwen3-8B-shaped 64-node, 4096-row call, together with the shared
  // queries below: 20.6 -> 19.6 us.)
  constexpr int kParPerThread = (kMaxNodes + kThreads - 1) / kThreads;
  constexpr int NQ = NT * NC;  // query loads per lane
  constexpr int kPro = WR > 1 ? NS : NS - 1;
  const int npro = min(kPro, n_mine);  // tiles the prologue issues
  int pv[kParPerThread];
  if (has_tree) {
    // indices clamped rather than branched on, so the loads stay in flight
    const int32_t* pr = a.parent + (size_t)b * a.N;
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) {
      const int i = tid + kThreads * k;
      pv[k] = a.parent ? load_i32(pr + (i < a.N ? i : a.N - 1)) : i - 1;  // NULL: a chain
    }
  }

  // ---- queries: B operand of S^T = K Q^T, lane holds Q[row l16][8*g4 .. +8]
  const int wrow0 = r0 + kRowsPerWave * wr;
  bf16x8 qf[NT][NC];
  bool qok[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = wrow0 + nt * 16 + l16;
    const bool ok = r < a.M;
    qok[nt] = ok;
    const int node = ok ? r / a.G : 0;
    const int h = g * a.G + (ok ? r % a.G : 0);
    const __bf16* qp = a.q + ((size_t)(b * a.N + node) * a.Hq + h) * D + 8 * g4;
    if (qload) {
#pragma unroll
      for (int c = 0; c < NC; ++c) qf[nt][c] = load_b128(qp + 32 * c);
    }
  }

#pragma unroll
  for (int i = 0; i < kPro; ++i)
    if (i < n_mine) issue_tile<D, PW, kPaged>(src, dma_off, wr, lane, t0 + wk + WK * i, ring + i * STAGE);

  // ---- tree structure: ancestor-or-self bitmask of this block's nodes
  if (has_tree) {
    // the parents are done once at most the queries and the DMAs are in flight
    wait_vm_any((qload ? NQ : 0) + npro * PW);
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) loaded(pv[k]);
    int bad = 0;
#pragma unroll
    for (int k = 0; k < kParPerThread; ++k) {
      const int i = tid + kThreads * k;
      if (i >= a.N) break;
      const int p = pv[k];
      par[i] = p;
      bad |= (i == 0) ? (p != -1) : (p < 0 || p >= i);
    }
    bad = __syncthreads_or(bad);
    const int nodes = i_hi - i_lo + 1;
    for (int t = tid; t < nodes; t += kThreads) {
      uint32_t* wd = anc + t * ntt;
      for (int k = 0; k < ntt; ++k) wd[k] = 0u;
      int u = i_lo + t;
      for (;;) {
        wd[u >> 5] |= 1u << (u & 31);
        if (u == 0) break;
        const int p = par[u];
        if (p < 0 || p >= u) break;  // invalid tree: the output becomes NaN
        u = p;
      }
    }
    if (tid == 0) *flag = bad;
    __syncthreads();
  }

  // the queries are done once at most the DMAs are in flight; rows past the
  // block's last row get zero queries.  Shared queries sit in LDS in the
  // tile layout, one 32-row tile per row group, read like the K operand.
  if (qload) {
    wait_vm_any(npro * PW);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        loaded(qf[nt][c]);
        if (!qok[nt]) qf[nt][c] = bf16x8{};
      }
  }
  // (the other key groups read them after the first ring step's barrier)
  unsigned char* qt = qlds + wr * TL::kBytes;
  if (qshare && wk == 0) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        *reinterpret_cast<bf16x8*>(qt + TL::off(16 * nt + l16, 4 * c + g4)) = qf[nt][c];
  }

  // O^T accumulators, and l: row sums of the bf16 weights, accumulated on
  // the matrix cores as ones^T P^T so numerator and denominator see the same
  // rounded weights (all 4 entries of lacc[nt] hold the lane's row sum)
  f32x4 o[DT][NT], lacc[NT];
  float m[NT];
  const bf16x8 ones = {(__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f,
                       (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    lacc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // node of this lane's row in each 16-row tile, relative to i_lo
  int node_rel[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = wrow0 + nt * 16 + l16;
    node_rel[nt] = (r < a.M ? r : a.M - 1) / a.G - i_lo;
  }

  float thr[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) thr[nt] = -INFINITY;  // m = -inf: any visible score moves
  const float inv_c = 1.f / a.c;
  bf16x8 ones_v = ones;
  asm volatile("" : "+v"(ones_v));  // keep it in registers, not rebuilt every tile
  // Ring step of iteration i: wait for this key group's tile i and refill
  // the ring.  With WR > 1 the prologue issued tiles 0..NS-1 and step j >= 1
  // issues tile j+NS-1, so my DMAs of tile i are done once at most
  // min(later tiles, NS-1 at step 0, NS-2 after) tiles' DMAs are
  // outstanding; the barrier makes the whole group's visible and guarantees
  // the slot of tile i-1 is no longer read.
  auto ring_step = [&](int i) {
    const bool mine = i < n_mine;
    if (WR > 1) {
      if (mine) {
        if (i == 0) wait_tiles<PW, NS - 1>(n_mine - 1);
        else wait_tiles<PW, NS - 2>(n_mine - 1 - i);
      }
      __syncthreads();
      if (i >= 1 && i + NS - 1 < n_mine)
        issue_tile<D, PW, kPaged>(src, dma_off, wr, lane, t0 + wk + WK * (i + NS - 1),
                          ring + ((i + NS - 1) % NS) * STAGE);
    } else {
      // a wave by itself: its LDS reads of tile i-1, whose stage the DMAs take
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (i + NS - 1 < n_mine)
        issue_tile<D, PW, kPaged>(src, dma_off, wr, lane, t0 + wk + WK * (i + NS - 1),
                          ring + ((i + NS - 1) % NS) * STAGE);
      if (mine) wait_tiles<PW, NS - 1>(n_mine - 1 - i);
    }
  };
  // Full cache tiles first, without masking; the tiles that need a mask
  // (the cache tail, then the tree tiles) all come after them.  Shared
  // queries are read behind the first step's workgroup barrier: every
  // workgroup here has n_iter >= 1, so this loop always runs step 0.
  auto shared_queries = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        qf[nt][c] = *reinterpret_cast<const bf16x8*>(qt + TL::off(16 * nt + l16, 4 * c + g4));
  };
  // a wave whose rows all lie past the last one only moves tiles
  const bool busy = wrow0 < a.M;
  uint32_t bits[NT] = {};
  int i = 0;
  for (; i < n_iter; ++i) {
    ring_step(i);
    if (i == 0 && qshare && wk != 0) shared_queries();
    const int t = t0 + wk + WK * i;
    if (i >= n_mine || t >= nct || (t + 1) * kKeyTile > kvl) break;
    if (!busy) continue;
    attend_tile<D, NT, false>(ring_ptr + (i % NS) * STAGE, qf, o, lacc, m, thr, ones_v, a.c, inv_c,
                              bits, g4, l16);
  }
  for (bool stepped = true; i < n_iter; ++i, stepped = false) {
    if (!stepped) ring_step(i);
    if (i >= n_mine || !busy) continue;
    const int t = t0 + wk + WK * i;
    tile_bits<NT>(MaskInfo{t, nct, kvl, ntt, a.tail, anc}, node_rel, bits);
    attend_tile<D, NT, true>(ring_ptr + (i % NS) * STAGE, qf, o, lacc, m, thr, ones_v, a.c, inv_c,
                             bits, g4, l16);
  }

  const LateArgs* z = late_args();
  float lsum[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) lsum[nt] = lacc[nt][0];
  const int invalid = has_tree ? *flag : 0;
  // Only chunks that hold tiles take part in a merge, nval of them; a row
  // block that is one chunk needs none and writes its output here.
  const int nval = (T + chunk - 1) / chunk;
  const bool whole = z->S == 1 || nval == 1;
  const int bg = b * z->Hkv + g;
  const size_t grp = (size_t)bg * z->nRB + rb;  // row block id

  // Final values of 16x16 fragments (dt, ntg) of this workgroup's rows: either
  // the normalised bf16 output (single chunk) or the chunk partial.  Fragments
  // wholly past the last row are neither stored here nor read by the merges,
  // which the plan's cost counts on (2 x 3 nodes, 32 heads on 8, 1361 rows: 19.0
  // -> 16.9 us; 64 x 2 nodes 55.5 -> 50.8; 16 x 33 nodes 53.0 -> 51.2).
  auto rows_at = [&](int ntg) { return r0 + ntg * 16 < z->M; };
  auto emit_out = [&](int dt, int ntg, const f32x4& acc, float l) {
    const int r = r0 + ntg * 16 + l16;
    if (r < z->M) {
      const int node = r / z->G, h = g * z->G + r % z->G;
      store_out4(z->out + ((size_t)(b * z->N + node) * z->Hq + h) * D + 16 * dt + 4 * g4, acc,
                 1.f / l, invalid != 0);
    }
  };
  auto emit_part = [&](bool dev, int dt, int ntg, const f32x4& acc, float mstar, float l) {
    f32x4* po = &z->ws_o[((size_t)(part0 + s) * DT * NTG + dt * NTG + ntg) * 64 + lane];
    float2* pml = &z->ws_ml[(size_t)(part0 + s) * RB + ntg * 16 + l16];
    if (dev) {  // read by another workgroup of this kernel
      store_dev(po, acc);
      if (dt == 0 && g4 == 0) store_dev(pml, make_float2(mstar, l));
    } else {    // read by the merge kernel
      *po = acc;
      if (dt == 0 && g4 == 0) *pml = make_float2(mstar, l);
    }
  };

  if (WK == 1) {
    // The kind of store is settled once per row tile, not at every fragment.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int ntg = wr * NT + nt;
      if (!rows_at(ntg)) break;
      if (whole) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) emit_out(dt, ntg, o[dt][nt], lsum[nt]);
      } else if (z->fused) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) emit_part(true, dt, ntg, o[dt][nt], m[nt], lsum[nt]);
      } else {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) emit_part(false, dt, ntg, o[dt][nt], m[nt], lsum[nt]);
      }
    }
  } else {
    // ---- merge the WK key groups of each row group (same rows, disjoint keys)
    __syncthreads();  // rings and tree tables are dead from here on
    f32x4* obuf = reinterpret_cast<f32x4*>(smem);
    float2* mlbuf = reinterpret_cast<float2*>(smem + (size_t)kWaves * kRowsPerWave * D * 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) obuf[((wave * DT + dt) * NT + nt) * 64 + lane] = o[dt][nt];
    if (g4 == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        mlbuf[wave * kRowsPerWave + nt * 16 + l16] = make_float2(m[nt], lsum[nt]);
    }
    __syncthreads();
    for (int f = wk; f < DT * NT; f += WK) {
      const int dt = f / NT, nt = f % NT;
      if (!rows_at(wr * NT + nt)) continue;
      const int rw = nt * 16 + l16;  // row within the wave's 32
      float mw[WK], mstar = -INFINITY;
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        mw[k] = mlbuf[(k * WR + wr) * kRowsPerWave + rw].x;
        mstar = fmaxf(mstar, mw[k]);
      }
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float e = mw[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[k] - mstar);
        l += e * mlbuf[(k * WR + wr) * kRowsPerWave + rw].y;
        acc += e * obuf[(((k * WR + wr) * DT + dt) * NT + nt) * 64 + lane];
      }
      if (whole) emit_out(dt, wr * NT + nt, acc, l);
      else if (z->fused) emit_part(true, dt, wr * NT + nt, acc, mstar, l);
      else emit_part(false, dt, wr * NT + nt, acc, mstar, l);
    }
  }
  if (whole || !z->fused) return;

  // ---- fused split-KV merge: the chunk that arrives last merges its row
  // block.  Every workgroup publishes its partial (device-scope stores,
  // completed before the count), then counts itself in; the one that
  // completes the count merges and resets the counter for the next call.
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
  merge_chunks<D, RB, kWaves>(z, part0, nval, b, g, r0, bad, wave, lane);
}

// Training mask, several blocks to a workgroup.  The A blocks of an example read
// the same context up to their anchors.  With one block per workgroup a block of
// S * G <= 64 rows leaves a workgroup of four waves half empty, or (two waves)
// moves every tile through LDS for its few rows only, and what bounds it is the
// tiles' way into LDS.  So nb blocks with neighbouring anchors (pack_order sorts
// them, largest first) share a workgroup of 128 rows: row R belongs to block
// R / M of the pack.  The workgroup streams the context up to its largest anchor,
// then every block's own keys; a wave skips the tiles none of its rows sees, and
// a row's visible keys are counted per row (key < anchor in the context, key <=
// position in its own block).  A ring of four tiles (64 KB) lets two workgroups
// share a CU.  Now bound by the matrix products and the softmax between them.
// Measured (8 KV heads, D = 128 unless said, random anchors): one example of 512
// blocks of 16, G = 4, 4096 positions: 350 -> 292 us; 2 x 200 blocks of 8, G = 4,
// 2048: 185 -> 91; 3 x 223 blocks of 32, G = 1, 390: 183 -> 74; 3 x 300 of 16,
// G = 2, D = 64, 1000: 258 -> 87; pack_order 5-7 us of each.  When it is taken:
// tv_plan.h, pack_plan.
struct PackArgs {
  const __bf16* q;
  const __bf16* kc;
  const __bf16* vc;
  const __bf16* kt;
  const __bf16* vt;
  const int32_t* anchors;
  const int32_t* order;  // [B, A]: the example's blocks, largest anchor first
  __bf16* out;
  int B, A, S, Hq, Hkv, L, G, M, nb, packs;
  float c;
};

// Place of each of an example's blocks by anchor: kPackRank blocks per workgroup,
// every workgroup with all keys in LDS, four lanes per block on a quarter of them
// each, four at a time.
__global__ __launch_bounds__(4 * kPackRank) void pack_order(const int32_t* anchors, int32_t* order,
                                                            int A) {
  __shared__ __attribute__((aligned(16))) int key[kPackMaxBlocks];
  const int per = (A + kPackRank - 1) / kPackRank, b = blockIdx.x / per, A16 = (A + 15) & ~15;
  for (int i = threadIdx.x; i < A16; i += 4 * kPackRank)
    key[i] = i < A ? anchors[(size_t)b * A + i] : INT32_MIN;
  __syncthreads();
  const int i = (int)(blockIdx.x % per) * kPackRank + (int)(threadIdx.x >> 2);
  const int v = i < A ? key[i] : 0;
  int rank = 0;
  for (int j = 4 * (int)(threadIdx.x & 3); j < A16; j += 16) {
    const int4 k = *(const int4*)(key + j);
    rank += k.x > v || (k.x == v && j < i);
    rank += k.y > v || (k.y == v && j + 1 < i);
    rank += k.z > v || (k.z == v && j + 2 < i);
    rank += k.w > v || (k.w == v && j + 3 < i);
  }
  rank += __shfl_xor(rank, 1);
  rank += __shfl_xor(rank, 2);
  if (i < A && (threadIdx.x & 3) == 0) order[(size_t)b * A + rank] = i;
}

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_packed(PackArgs a) {
  using TL = TileLayout<D>;
  constexpr int WR = kPackRows / kRowsPerWave, NS = 4;
  constexpr int NT = kRowsPerWave / 16, NC = D / 32, DT = D / 16;
  constexpr int STAGE = 2 * TL::kBytes, PW = 2 * TL::kDma / WR, NQ = NT * NC;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15;
  const int wr = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  // KV heads in turn, then examples; the packs of the largest anchors come first.
  // Workgroups go to the XCDs in turn too, so an XCD reads the context of Hkv /
  // gcd(8, Hkv) heads: one with 8 of them, all where their number is odd.
  const int g = (int)blockIdx.x % a.Hkv, u = (int)blockIdx.x / a.Hkv;
  const int b = u % a.B, p = u / a.B;
  if (p >= a.packs) return;

  // the pack's blocks, one per lane
  const int nv = min(a.nb, a.A - p * a.nb);
  const int mine = lane < nv ? a.order[(size_t)b * a.A + p * a.nb + lane] : 0;
  int anchor = lane < nv ? a.anchors[(size_t)b * a.A + mine] : 0;
  anchor = anchor < 0 ? 0 : (anchor > a.L ? a.L : anchor);
  const int ntt = (a.S - 1) / kKeyTile + 1;

  // this lane's rows
  int blk[NT], node[NT];
  size_t orow[NT];
  bool ok[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int R = kRowsPerWave * wr + 16 * nt + l16, rr = R % a.M;
    blk[nt] = R / a.M;
    ok[nt] = blk[nt] < nv;
    node[nt] = rr / a.G;
    const int src = ok[nt] ? blk[nt] : 0;
    orow[nt] = (((size_t)b * a.A + __shfl(mine, src)) * a.S + node[nt]) * a.Hq + g * a.G + rr % a.G;
  }
  const int blk_lo = kRowsPerWave * wr / a.M, blk_hi = (kRowsPerWave * (wr + 1) - 1) / a.M;

  const size_t krow = (size_t)a.Hkv * D;
  const size_t cache0 = (size_t)b * a.L * krow + (size_t)g * D;
  uint32_t dma_off[PW];
#pragma unroll
  for (int k = 0; k < PW; ++k) {
    const int r = ((wr * PW + k) % TL::kDma) * TL::kRowsPerDma + lane / TL::kCPR;
    dma_off[k] = (uint32_t)(r * (int)krow * 2 + ((lane % TL::kCPR) ^ TL::swz(r)) * 16);
  }
  const char* kctx = uniform_ptr((const char*)(a.kc + cache0));
  const char* vctx = uniform_ptr((const char*)(a.vc + cache0));

  bf16x8 qf[NT][NC];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) {
      const bf16x8 v =
          *reinterpret_cast<const bf16x8*>(a.q + orow[nt] * D + 8 * g4 + 32 * cc);
      qf[nt][cc] = ok[nt] ? v : bf16x8{};
    }
  // (the queries are in before the first tiles go out: the compiler's wait for
  // them would otherwise drain the tiles too)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int cc = 0; cc < NC; ++cc) asm volatile("" : "+v"(qf[nt][cc]));
  // one pass over all blocks, or one per block (below)
  for (int j0 = 0, j1 = nv;;) {
    // the pass's tiles: the context up to its blocks' largest anchor, then their own
    const bool in = lane >= j0 && lane < j1;
    const int longest = (int)wave_max_u32(in ? (unsigned)anchor : 0u);
    const int nct = (longest + kKeyTile - 1) / kKeyTile, T = nct + (j1 - j0) * ntt;
    // its rows, and the smallest and largest of the wave's anchors
    bool on[NT];
    int kvl[NT], lo = a.L, hi = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      on[nt] = ok[nt] && blk[nt] >= j0 && blk[nt] < j1;
      kvl[nt] = __shfl(anchor, blk[nt] & 63);
      if (!on[nt]) kvl[nt] = 0;
      else lo = min(lo, kvl[nt]);
      hi = max(hi, kvl[nt]);
    }
    lo = a.L - (int)wave_max_u32((unsigned)(a.L - lo));
    hi = (int)wave_max_u32((unsigned)hi);
    if (hi == 0) lo = 0;  // no context, or no rows
    // tile t: of the context, or of block j0 + (t - nct) / ntt's own keys
    auto issue = [&](int t) {
      TreeSrc src{kctx, vctx, kctx, vctx, nullptr, 0, 0, (int)krow * 2, longest, nct, a.S - 1};
      if (t >= nct) {
        const int j = j0 + (t - nct) / ntt;
        const size_t own =
            ((size_t)b * a.A + __builtin_amdgcn_readlane(mine, j)) * a.S * krow + (size_t)g * D;
        src.ktree = uniform_ptr((const char*)(a.kt + own));
        src.vtree = uniform_ptr((const char*)(a.vt + own));
        src.nct = nct + (j - j0) * ntt;
      }
      issue_tile<D, PW, false>(src, dma_off, wr, lane, t, (uint32_t)(uintptr_t)smem + (t % NS) * STAGE);
    };

#pragma unroll
    for (int t = 0; t < NS; ++t)
      if (t < T) issue(t);

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
    asm volatile("" : "+v"(ones));
    const float inv_c = 1.f / a.c;
    uint32_t bits[NT] = {};
    auto ring_step = [&](int t) {
      if (t == 0) wait_tiles<PW, NS - 1>(T - 1);
      else wait_tiles<PW, NS - 2>(T - 1 - t);
      __syncthreads();
      if (t >= 1 && t + NS - 1 < T) issue(t + NS - 1);
    };
    int t = 0;
    for (; t < T; ++t) {  // context tiles that all of the wave's rows see whole
      ring_step(t);
      if (t >= nct || (t + 1) * kKeyTile > lo) break;
      attend_tile<D, NT, false>(smem + (t % NS) * STAGE, qf, o, lacc, m, thr, ones, a.c, inv_c, bits,
                                g4, l16);
    }
    for (bool stepped = true; t < T; ++t, stepped = false) {
      if (!stepped) ring_step(t);
      const int j = t < nct ? 0 : j0 + (t - nct) / ntt;
      if (t < nct ? t * kKeyTile >= hi : (j < blk_lo || j > blk_hi)) continue;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        bits[nt] = t < nct ? first_keys(kvl[nt] - t * kKeyTile)
                           : (blk[nt] == j ? first_keys(node[nt] + 1 - (t - nct) % ntt * kKeyTile) : 0u);
      attend_tile<D, NT, true>(smem + (t % NS) * STAGE, qf, o, lacc, m, thr, ones, a.c, inv_c, bits, g4,
                               l16);
    }
    // Non-finite outputs: a value that is an infinity or NaN reaches, times a
    // weight of zero, rows of the pack that do not see its key.  Then every block
    // is done again by itself.
    if (j0 == 0 && j1 == nv && nv > 1) {
      bool bad = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w = __float_as_uint(o[dt][nt][e]);
            asm("" : "+v"(w));  // (no assumption that it is a number)
            bad |= on[nt] && (w & 0x7f800000u) == 0x7f800000u;
          }
      if (__syncthreads_or(bad)) {
        j1 = 1;
        continue;
      }
      j1 = nv + 1;  // done after the store
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (!on[nt]) continue;
      const float inv = 1.f / lacc[nt][0];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        store_out4(a.out + orow[nt] * D + 16 * dt + 4 * g4, o[dt][nt], inv, false);
    }
    if (j1 >= nv) return;
    __syncthreads();  // the ring is free
    j0 = j1++;
  }
}

// Second kernel of the split-KV plans whose merge is too large for one
// workgroup: out = sum_s e_s O_s / sum_s e_s l_s with e_s = 2^(m_s - m*),
// folded in online over batches of U chunks.  Only chunks that hold tiles
// of this row block were written.  One wave per 16x16 fragment.  The
// parents (for the tree check), kv_len and the first batch of partials are
// all requested before any is used, so a merge of up to U chunks waits for
// one round of memory latency: the first batch reads the slots of the
// first min(S, U) chunks whether or not they were written by this call
// (they lie inside the workspace), and only the nval chunks that hold
// tiles, known once kv_len arrives, are folded in.
template <int D, int RB>
__global__ __launch_bounds__(256) void attn_combine(AttnArgs a) {
  constexpr int NTG = RB / 16, DT = D / 16, U = 16;
  constexpr int kParPerThread = kMaxNodes / 256;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g4 = lane >> 4, l16 = lane & 15;
  const int F = blockIdx.x * 4 + wave;  // fragment id; all 4 of a block share (b,g,rb)
  const int per_blk = DT * NTG;
  const int blk = F / per_blk, f = F % per_blk;
  const int rb = blk % a.nRB, bg = blk / a.nRB;
  const int b = bg / a.Hkv, g = bg % a.Hkv;
  int pv[kParPerThread];
#pragma unroll
  for (int k = 0; k < kParPerThread; ++k) {
    const int i = threadIdx.x + 256 * k;
    pv[k] = i >= a.N ? 0 : (a.parent ? a.parent[(size_t)b * a.N + i] : i - 1);
  }
  const int dt = f / NTG, ntg = f % NTG;
  const int row = ntg * 16 + l16, r = rb * RB + row;
  // chunks of this row block that hold tiles (the same count the main
  // kernel derives from kv_len and the block's last node)
  const int i_hi = (min(rb * RB + RB, a.M) - 1) / a.G;
  // the first chunk partial, and the partials from there on
  EvenItem ev{a.chunk, b, 0, 0, 0};
  size_t base = (size_t)(bg * a.nRB + rb) * a.S;
  int nslot = a.S;
  if (a.slots > 0) {
    if (a.B > 1) ev = even_split<false>(a, -1, b, 0);
    base = (size_t)(g * a.nRB + rb) * a.slots + ev.first;
    nslot = a.slots - ev.first;
  }
  float2 ml0[U];
  f32x4 ov0[U];
  const bool any = rb * RB + ntg * 16 < a.M;  // else no rows: nothing was stored
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u < nslot && any) {
      ml0[u] = a.ws_ml[(base + u) * RB + row];
      ov0[u] = a.ws_o[((base + u) * DT * NTG + dt * NTG + ntg) * 64 + lane];
    }
  if (a.slots == 0) ev.kvl = context_rows(a, b);
  else if (a.B == 1) ev = even_one<false>(a, 0, 0);
  const int T = segment(a, ev.kvl, i_hi).T;
  int nval = (T + ev.chunk - 1) / ev.chunk;
  if (nval == 1) return;  // written by its only chunk
  if (!any) nval = 0;
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < nval; s0 += U) {
    float2 ml[U];
    f32x4 ov[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u < nval) {
        if (s0 == 0) {
          ml[u] = ml0[u];
          ov[u] = ov0[u];
        } else {
          ml[u] = a.ws_ml[(base + s0 + u) * RB + row];
          ov[u] = a.ws_o[((base + s0 + u) * DT * NTG + dt * NTG + ntg) * 64 + lane];
        }
      }
    float mb = m;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u < nval) mb = fmaxf(mb, ml[u].x);
    if (mb != -INFINITY) {  // else every chunk so far saw no key: nothing to add
      const float ea = __builtin_amdgcn_exp2f(m - mb);  // 0 while m = -inf
      l *= ea;
      acc *= ea;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s0 + u < nval && ml[u].x != -INFINITY) {
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
  bad = __syncthreads_or(bad);
  if (r >= a.M) return;
  const int node = r / a.G, h = g * a.G + r % a.G;
  store_out4(a.out + ((size_t)(b * a.N + node) * a.Hq + h) * D + 16 * dt + 4 * g4, acc, 1.f / l,
             bad != 0);
}

template <int D, int WR, int WK, int NS, bool kPaged, bool kShareQ>
static hipError_t launch_main(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
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
      e = hipFuncSetAttribute((const void*)attn_main<D, WR, WK, NS, kPaged, kShareQ>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds_bytes);
      if (e != hipSuccess) return e;
      limit[dev].store((int)p.lds_bytes, std::memory_order_release);
    }
  }
  hipLaunchKernelGGL((attn_main<D, WR, WK, NS, kPaged, kShareQ>),
                     dim3(p.slots > 0 ? p.even_grid : p.grid), dim3(64 * WR * WK),
                     p.lds_bytes, st, a);
  return hipGetLastError();
}

template <int D, int ARR, bool kPaged>
static hipError_t launch_attn_t(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  constexpr Arrangement ar = kArrangements[ARR];
  constexpr int NS = arr_stages(ar, D);
  if constexpr (NS == 0) {
    return hipErrorInvalidValue;  // never planned: the ring does not fit
  } else {
    // query sharing is a separate instantiation, so the kernels without it
    // carry none of its code or scalar registers
    hipError_t e;
    if constexpr (ar.WK > 1 && ar.WR > 1)
      e = p.qshare ? launch_main<D, ar.WR, ar.WK, NS, kPaged, true>(a, p, st)
                   : launch_main<D, ar.WR, ar.WK, NS, kPaged, false>(a, p, st);
    else
      e = launch_main<D, ar.WR, ar.WK, NS, kPaged, false>(a, p, st);
    if (e != hipSuccess || p.S == 1 || p.fused) return e;
    constexpr int RB = kRowsPerWave * ar.WR;
    const int frags = a.B * a.Hkv * p.nRB * (D / 16) * (RB / 16);
    hipLaunchKernelGGL((attn_combine<D, RB>), dim3(frags / 4), dim3(256), 0, st, a);
    return hipGetLastError();
  }
}

template <int D, int K = 0>
static hipError_t launch_attn_d(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  if constexpr (K < kNumArrangements) {
    if (p.arr == K)
      return a.block_table ? launch_attn_t<D, K, true>(a, p, st)
                           : launch_attn_t<D, K, false>(a, p, st);
    return launch_attn_d<D, K + 1>(a, p, st);
  } else {
    return hipErrorInvalidValue;
  }
}

hipError_t launch_attention(const void* q, const void* kc, const void* vc, const void* kt,
                            const void* vt, const int32_t* parent, const int32_t* kv_len,
                            void* out, int B, int N, int Hq, int Hkv, int D, int Lmax,
                            float scale, void* ws, const AttnPlan& p, hipStream_t st,
                            const int32_t* block_table, int block_shift, int max_blocks,
                            int num_blocks, int cgroup) {
  AttnArgs a;
  a.tail = kt == nullptr;
  a.cgroup = cgroup;
  a.block_table = block_table;
  a.block_shift = block_shift;
  a.max_blocks = max_blocks;
  a.num_blocks = num_blocks;
  a.q = (const __bf16*)q;
  a.kc = (const __bf16*)kc;
  a.vc = (const __bf16*)vc;
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
  a.spread = p.spread;
  a.slots = p.slots;
  a.min_chunk = p.min_chunk;
  a.rslots = p.slots > 0 ? 1.f / (float)p.slots : 0.f;
  a.rslack = p.slots > B ? 1.f / (float)(p.slots - B) : 1.f;
  a.c = scale * 1.4426950408889634f;
  return D == 128 ? launch_attn_d<128>(a, p, st) : launch_attn_d<64>(a, p, st);
}

template <int D>
static hipError_t launch_packed_d(const PackArgs& a, hipStream_t st) {
  constexpr int lds = 4 * 2 * TileLayout<D>::kBytes;  // at most 64 KB: no limit to raise
  static_assert(lds <= 64 * 1024, "the ring");
  const dim3 grid(kXcds * cdiv((long long)a.B * a.packs * a.Hkv, kXcds));
  hipLaunchKernelGGL(attn_packed<D>, grid, dim3(256), lds, st, a);
  return hipGetLastError();
}

hipError_t launch_packed(const void* q, const void* kc, const void* vc, const void* kt, const void* vt,
                         const int32_t* anchors, void* out, int B, int A, int S, int Hq, int Hkv, int D,
                         int L, float scale, void* ws, const PackPlan& p, hipStream_t st) {
  int32_t* order = (int32_t*)((char*)ws + kSyncBytes);
  hipLaunchKernelGGL(pack_order, dim3(B * cdiv(A, kPackRank)), dim3(4 * kPackRank), 0, st, anchors,
                     order, A);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  PackArgs a{(const __bf16*)q, (const __bf16*)kc, (const __bf16*)vc, (const __bf16*)kt,
             (const __bf16*)vt, anchors, order, (__bf16*)out, B, A, S, Hq, Hkv, L, Hq / Hkv,
             S * (Hq / Hkv), p.nb, p.packs, scale * 1.4426950408889634f};
  return D == 128 ? launch_packed_d<128>(a, st) : launch_packed_d<64>(a, st);
}

}  // namespace tv
