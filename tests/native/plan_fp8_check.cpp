// Plans of the attention over the 8-bit cache: every one launches (LDS, sync words, sizes),
// its workspace covers every chunk partial that the even split can give, and the search
// always finds one.  Prints the number of shapes looked at.
#include <cstdio>
#include <cstdlib>

#include "tv_plan_fp8.h"

using namespace tv;

static int failures = 0, shapes = 0;

static void check(int B, int N, int Hq, int Hkv, int D, int Lmax) {
  const AttnPlan p = attn_plan_fp8(B, N, Hq, Hkv, D, Lmax);
  const ArrangementFp8& ar = kArrangementsFp8[p.arr];
  const int G = Hq / Hkv, tiles = cdiv(Lmax, kKeyTile) + cdiv(N, kKeyTile);
  bool ok = p.G == G && p.M == N * G && p.RB == 16 * ar.NT * ar.WR && p.nRB == cdiv(p.M, p.RB);
  ok = ok && p.threads == 64 * ar.WR * ar.WK && p.wg_per_cu * ar.WR * ar.WK == kWavesPerCU;
  ok = ok && p.lds_bytes + kFp8StaticLds <= kMaxLds;
  // rings, tree tables and the key groups' merge lie inside the LDS asked for
  const size_t ring = (size_t)ar.WK * (D == 128 ? ar.NU128 : ar.NU64) * 64 * D;
  ok = ok && p.lds_bytes >= ring + ((size_t)(p.RB / G + 2) * cdiv(N, 32) + N) * 4;
  if (ar.WK > 1) ok = ok && p.lds_bytes >= (size_t)ar.WR * ar.WK * 16 * ar.NT * (D * 4 + 8);
  ok = ok && p.chunk >= 1 && p.S >= 1 && (long long)p.chunk * p.S >= tiles;
  const long long base = (long long)B * Hkv * p.nRB;
  if (p.S > 1) {
    ok = ok && base <= kSyncGroups && B <= kEvenSequences && tiles < kEvenTiles;
    ok = ok && p.slots > B && p.slots <= (long long)B * p.S && p.min_chunk == 2 * ar.WK;
    // partial `part0 + s` of a (KV head, row block): below slots for each of them
    const size_t partials = (size_t)p.slots * Hkv * p.nRB;
    ok = ok && p.ws_sync_bytes == kSyncBytes && p.ws_o_bytes >= partials * p.RB * D * 4;
    ok = ok && p.ws_ml_bytes >= partials * p.RB * 8;
    ok = ok && p.ws_bytes == p.ws_sync_bytes + p.ws_o_bytes + p.ws_ml_bytes;
    // every (chunk, head) pair has its workgroups
    WorkItem it{};
    long long seen = 0;
    if (p.even_grid <= 1 << 14)
      for (int bid = 0; bid < p.even_grid; ++bid) {
        const int item = even_item(bid, p.slots, p.nRB, Hkv, it);
        seen += item >= 0 && item < p.slots && it.g < Hkv && it.rb < p.nRB;
      }
    ok = ok && (p.even_grid > 1 << 14 || seen == (long long)p.slots * Hkv * p.nRB);
  } else {
    ok = ok && p.slots == 0 && p.ws_bytes == 0 && p.grid >= base;
  }
  ++shapes;
  if (!ok) {
    ++failures;
    printf("bad plan: B %d N %d Hq %d Hkv %d D %d Lmax %d (arrangement %d, S %d, slots %d)\n", B, N, Hq,
           Hkv, D, Lmax, p.arr, p.S, p.slots);
  }
}

int main(int argc, char**) {
  if (argc > 1) {  // the way that each shape of the input takes: D, arrangement, merge (-1: unsplit)
    int B, N, Hq, Hkv, D, L;
    while (scanf("%d %d %d %d %d %d", &B, &N, &Hq, &Hkv, &D, &L) == 6) {
      const AttnPlan p = attn_plan_fp8(B, N, Hq, Hkv, D, L);
      printf("%d %d %d\n", D, p.arr, p.S == 1 ? -1 : p.fused);
    }
    return 0;
  }
  const int Bs[] = {1, 2, 3, 7, 16, 64, 65, 256, 1024, 1025, 4096}, Ns[] = {1, 2, 5, 16, 31, 32, 33, 64, 100, 512, 2048};
  const int Ls[] = {0, 32, 96, 1024, 5024, 32768, 131072, 1 << 20, 1 << 26};
  const int heads[][2] = {{1, 1}, {4, 2}, {8, 8}, {32, 4}, {32, 8}, {64, 8}, {24, 8}, {16, 1}, {7, 7}, {40, 10}};
  for (int B : Bs)
    for (int N : Ns)
      for (int L : Ls)
        for (const auto& h : heads)
          for (int D = 64; D <= 128; D += 64)
            if ((long long)B * N * h[0] <= 1ll << 31 && (long long)B * L <= 1ll << 31) check(B, N, h[0], h[1], D, L);
  srand(1);
  for (int k = 0; k < 20000; ++k) {
    const int Hkv = 1 + rand() % 12, G = 1 + rand() % 12;
    check(1 + rand() % 70, 1 + rand() % (k % 2 ? 40 : 2048), Hkv * G, Hkv, k % 3 ? 128 : 64, 32 * (rand() % 5000));
  }
  printf("%d shapes\n", shapes);
  return failures != 0;
}
