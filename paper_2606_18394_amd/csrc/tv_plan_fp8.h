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
  p.fused = p.S > 1 && (size_t)p.S * p.RB * D * 4 <= (size_t)1024 * p.threads;
  return p;
}

inline bool attn_plan_fp8_fits(const AttnPlan& p) {
  return (p.lds_bytes + kFp8StaticLds) * p.wg_per_cu <= kMaxLds;
}

inline AttnPlan attn_plan_fp8(int B, int N, int Hq, int Hkv, int D, int Lmax) {
  const int M = N * (Hq / Hkv);
  int arr = M <= 16 ? 0 : (M <= 32 ? 2 : (M <= 64 ? 4 : 6));
  AttnPlan one = attn_plan_fp8_arr(B, N, Hq, Hkv, D, Lmax, arr, B);
  const long long fill = 256LL * one.wg_per_cu / one.nRB / Hkv;
  return fill > B ? attn_plan_fp8_arr(B, N, Hq, Hkv, D, Lmax, arr, fill) : one;
}

}  // namespace tv
