// Host-side launch planning of the attention over the 8-bit paged cache.  Pure C++
// (no HIP), like tv_plan.h whose work decomposition it uses.
#pragma once
#include "tv_plan.h"

namespace tv {

// WR x WK waves of 16 * NT rows each; units of a key group's ring (8 KB at D = 128, 4 KB
// at D = 64).  A CU holds 8 waves.
struct ArrangementFp8 {
  int WR, WK, NT, NU128, NU64;
};
constexpr ArrangementFp8 kArrangementsFp8[] = {
    {1, 8, 1, 2, 4}, {1, 4, 1, 2, 4}, {1, 8, 2, 2, 4}, {1, 4, 2, 2, 4}, {2, 4, 2, 4, 8}, {2, 2, 2, 4, 8},
    {4, 1, 2, 8, 16},
};
constexpr int kNumArrangementsFp8 = sizeof(kArrangementsFp8) / sizeof(kArrangementsFp8[0]);

// Dynamic LDS: the rings, then the tree tables; the key-group merge reuses it.
inline size_t attn_fp8_lds_bytes(const ArrangementFp8& ar, int D, int G, int N) {
  const int RB = 16 * ar.NT * ar.WR, waves = ar.WR * ar.WK;
  const size_t ring = (size_t)ar.WK * (D == 128 ? ar.NU128 : ar.NU64) * 64 * D;
  const size_t tree = (size_t)(RB / G + 2) * cdiv(N, 32) * 4 + (size_t)N * 4 + 16;
  const size_t merge = ar.WK == 1 ? 0 : (size_t)waves * 16 * ar.NT * (D * 4 + 8);
  return ring + tree > merge ? ring + tree : merge;
}
constexpr size_t kFp8StaticLds = 1024;  // what the kernel has beside it, rounded up

inline AttnPlan attn_plan_fp8_arr(int B, int N, int Hq, int Hkv, int D, int Lmax, int arr, long long want) {
  const ArrangementFp8& ar = kArrangementsFp8[arr];
  AttnPlan p{};
  p.arr = arr;
  p.WR = ar.WR;
  p.WK = ar.WK;
  p.NS = D == 128 ? ar.NU128 : ar.NU64;
  p.threads = 64 * ar.WR * ar.WK;
  p.G = Hq / Hkv;
  p.wg_per_cu = kWavesPerCU / (ar.WR * ar.WK);
  p.M = N * p.G;
  p.RB = 16 * ar.NT * ar.WR;
  p.nRB = cdiv(p.M, p.RB);
  p.lds_bytes = attn_fp8_lds_bytes(ar, D, p.G, N);
  const int tiles = cdiv(Lmax, kKeyTile) + cdiv(N, kKeyTile);
  const long long base = (long long)B * Hkv * p.nRB;
  const int min_chunk = 2 * ar.WK;
  const long long max_s = tiles / min_chunk > 1 ? tiles / min_chunk : 1;
  long long S = (want + B - 1) / B;
  if (S > max_s) S = max_s;
  if (S < 1 || base > kSyncGroups || B > kEvenSequences || tiles >= kEvenTiles) S = 1;
  p.chunk = cdiv(tiles, S);
  p.S = cdiv(tiles, p.chunk);
  p.nwork = (int)(base * p.S);
  p.grid = cdiv(p.nwork, kXcds) * kXcds;
  if (p.S > 1) {
    p.slots = (int)(want < (long long)B * p.S ? want : (long long)B * p.S);
    p.min_chunk = min_chunk;
    p.even_grid = kXcds * p.nRB * cdiv((long long)p.slots * Hkv, kXcds);
    const int DT = D / 16, NTG = p.RB / 16;
    p.ws_sync_bytes = kSyncBytes;
    p.ws_o_bytes = (size_t)B * Hkv * p.nRB * p.S * DT * NTG * 64 * 16;
    p.ws_ml_bytes = (size_t)B * Hkv * p.nRB * p.S * p.RB * 8;
  }
  p.ws_bytes = p.ws_sync_bytes + p.ws_o_bytes + p.ws_ml_bytes;
  return p;
}

inline bool attn_plan_fp8_fits(const AttnPlan& p) {
  return (p.lds_bytes + kFp8StaticLds) * p.wg_per_cu <= kMaxLds;
}

// Relative time of a plan, roughly in microseconds, like attn_plan_cost (tv_plan.h):
// tiles take their turns, a chunk's at one time per tile and key group (alone, or the
// CU's share of 8 waves at work); then the fixed costs, HBM (also what the CUs at work
// can ask for), the tree and the partials.  The constants are fitted together to 294
// shapes drawn over the ranges of 1 to 64 sequences, 1 to 512 nodes, up to 131072 rows
// and the heads above, each in all arrangements and up to 14 splits and merges, those of
// the merge by a second kernel to 6000 times of both merges.  The plan picked is 2.3%
// slower than the fastest on average on 1800 shapes that the fit has not seen (row blocks
// as large as the tree fills, split to fill the GPU once: 18%).  As a time the cost is
// rougher than that: all but the merge's constants were fitted before tiles that are read
// once passed the caches by (single tokens of 64 sequences: cost 133, time 104 to 112;
// two trees of 16 nodes over 131072 rows: 84, 115), and trees of more than 512 nodes were
// not among the shapes.
constexpr double kFp8Fill = 0.703;  // mean length of several sequences over the capacity
constexpr double kFp8Full[] = {1.04, 0, 1.598, 1.582, 1.414, 1.202, 0.911};  // 8 waves at work
static_assert(sizeof(kFp8Full) / sizeof(kFp8Full[0]) == kNumArrangementsFp8, "one per arrangement");

inline double attn_plan_fp8_cost(AttnPlan& p, int B, int Hkv, int D, int Lmax, int N) {
  const ArrangementFp8& ar = kArrangementsFp8[p.arr];
  const int ct = cdiv(Lmax, kKeyTile), nt = cdiv(N, kKeyTile);
  const double longest = ct + nt, mean = B == 1 ? longest : kFp8Fill * ct + nt;
  double chunk = longest, items = B;
  if (p.slots > 0) {
    const double slack = p.slots - 0.687 * B;
    chunk = B == 1 ? (double)cdiv((long long)longest, p.slots)
                   : B * mean / (slack > 0.3 * B + 0.1 ? slack : 0.3 * B + 0.1);
    if (chunk < p.min_chunk) chunk = p.min_chunk;
    if (chunk > longest) chunk = longest;
    items = B == 1 ? longest / chunk : B * mean / chunk + 0.5 * B;
    if (B == 1 && items > (int)items) items = (int)items + 1;
    if (B > 1 && items > p.slots) items = p.slots;
  }
  const double wgs = items * Hkv * p.nRB, room = 256.0 * p.wg_per_cu;
  double per_cu = wgs / 256.0;
  per_cu = per_cu < 1.0 ? 1.0 : (per_cu > p.wg_per_cu ? p.wg_per_cu : per_cu);
  const double row_tiles = (double)cdiv(p.M, 16 * ar.NT) / p.nRB;
  const double waves = per_cu * p.WK * (row_tiles < p.WR ? row_tiles : p.WR);
  double tile = ar.NT == 1 ? 0.98 : 1.102;
  if (kFp8Full[p.arr] * waves / 8.0 > tile) tile = kFp8Full[p.arr] * waves / 8.0;
  if (D == 64) tile *= 0.669;
  const int steps = (int)(chunk / p.WK) + (chunk / p.WK > (int)(chunk / p.WK));
  double t = steps * tile;
  const long long per_xcd = (long long)cdiv((long long)(items * Hkv + 0.999), kXcds) * p.nRB;
  const long long rounds = p.slots > 0 ? cdiv(per_xcd, 32LL * p.wg_per_cu)
                                       : cdiv((long long)(wgs + 0.999), (long long)room);
  if (rounds > 1) {
    const double queue = B * mean * Hkv * p.nRB / room / p.WK * tile + 0.677 * t, turns = rounds * t;
    const double least = queue < turns ? queue : turns;
    if (least > t) t = least;
  }
  const double asked = (wgs < 256 ? wgs : 256) * 42.0e3;
  const double hbm = B * mean * kKeyTile * Hkv * D * 2.0 / (asked < 6.0e6 ? asked : 6.0e6);
  t = t > hbm ? t : hbm;
  t += 5.8 + 5.86 * (rounds - 1) + 0.645 * nt;
  const double chunks = p.slots > 0 ? cdiv((long long)longest, (long long)(chunk + 0.999)) : 1;
  if (chunks > 1) {
    // the partials, and whichever merge takes less time (of a row block by its last
    // workgroup, a few waves of it; or a kernel that spreads all over the GPU)
    const int NTG = p.RB / 16, waves_wg = p.WR * p.WK, rows = cdiv(p.M < p.RB ? p.M : p.RB, 16);
    const int active = waves_wg >= NTG ? waves_wg / NTG * rows : (rows < waves_wg ? rows : waves_wg);
    const double block = rows * 16.0 * D * 4.0, all = wgs / p.nRB * cdiv(p.M, 16) * 16.0 * D * 4.0;
    const double fused = 2.63 + chunks * block / (active * 15.4e3 < 86.7e3 ? active * 15.4e3 : 86.7e3);
    const double frags = (double)B * Hkv * cdiv(p.M, 16) * (D / 16);
    const double second = 2.87 + all / 2.49e6 + 0.00306 * frags;
    p.fused = fused <= second;
    t += (p.fused ? fused : second) + all / 5.0e6;
  }
  return t;
}

inline AttnPlan attn_plan_fp8(int B, int N, int Hq, int Hkv, int D, int Lmax) {
  AttnPlan best{};
  double best_cost = 0;
  bool have = false;
  for (int k = 0; k < kNumArrangementsFp8; ++k) {
    const AttnPlan one = attn_plan_fp8_arr(B, N, Hq, Hkv, D, Lmax, k, B);
    // what leaves most of a row block empty, or wants a CU to itself (long tree tables),
    // only where there is nothing else: the last one always runs
    const bool last = k == kNumArrangementsFp8 - 1;
    if (one.RB > 16 && one.RB >= 4 * one.M && !(last && !have)) continue;
    if (!attn_plan_fp8_fits(one) && !(last && !have)) continue;
    // one chunk per sequence, or a quarter, half, once, twice or four times what fills the GPU
    const long long fill = 256LL * one.wg_per_cu / one.nRB / Hkv;
    const long long cand[6] = {B, fill / 4, fill / 2, fill, 2 * fill, 4 * fill};
    for (int c = 0; c < 6; ++c) {
      if (c > 0 && cand[c] <= B) continue;
      AttnPlan p = c == 0 ? one : attn_plan_fp8_arr(B, N, Hq, Hkv, D, Lmax, k, cand[c]);
      const double t = attn_plan_fp8_cost(p, B, Hkv, D, Lmax, N);
      if (!have || t < best_cost) {
        best = p;
        best_cost = t;
        have = true;
      }
    }
  }
  return best;
}

}  // namespace tv
