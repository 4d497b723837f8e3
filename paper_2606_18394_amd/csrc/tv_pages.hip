// Whose page is whose, for CDNA4 (gfx950): pages of a paged cache are handed out, shared
// between sequences, given back and drawn together, and their contents copied.
//
// State is what the caches use anyway plus a count: block_table [B, max_blocks] (a row's
// pages come first, -1 behind them), kv_len [B] and ref_count [num_blocks], how many rows
// name a page (0: free).  A new page is always the free one of the lowest number, so the
// outcome depends on nothing but the arguments, and no list of free pages has to be kept:
// finding them is one pass over ref_count, 4 bytes a page.  What many workgroups count at
// once (pages shared or given back) are whole numbers, whose order of adding does not show.
//
// The deciding is latency, the copying HBM: a page is copied in pieces of 16 KB, a
// workgroup each, of any pools whose first axis is the page.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tv_pages.h"
#include "tv_walk.h"

namespace tv {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kDecide = 1024;  // threads of a deciding workgroup

// Sum of x over the workgroup's (kDecide) threads before this one, and over all of them.
__device__ __forceinline__ int block_scan(int x, int& total) {
  constexpr int kWaves = kDecide / 64;
  __shared__ __attribute__((aligned(16))) int sums[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_scan(x);
  __syncthreads();  // the sums of a call before this one are read
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int n = sums[w];
    before += w < wave ? n : 0;
    total += n;
  }
  return before + upto - x;
}

// Which of a thread's kRun pages from `first` on are free, as a bit mask.
constexpr int kRun = 8;
__device__ __forceinline__ unsigned free_mask(const int32_t* ref, int num_blocks, long long first) {
  unsigned free = 0;
  if (first >= 0 && first + kRun <= num_blocks) {
    const int4 lo = *(const int4*)(ref + first), hi = *(const int4*)(ref + first + 4);
    free = (lo.x <= 0) | (lo.y <= 0) << 1 | (lo.z <= 0) << 2 | (lo.w <= 0) << 3 | (hi.x <= 0) << 4 |
           (hi.y <= 0) << 5 | (hi.z <= 0) << 6 | (hi.w <= 0) << 7;
  } else {
    for (int k = 0; k < kRun; ++k)
      if (first + k >= 0 && first + k < num_blocks && ref[first + k] <= 0) free |= 1u << k;
  }
  return free;
}

// The first page of the workgroup's first pass over ref_count, whose runs begin at
// multiples of 16 bytes wherever it begins; a pass takes kDecide * kRun pages.
__device__ __forceinline__ long long pass_start(const int32_t* ref) {
  return -(long long)((uintptr_t)ref / 4 % 4);
}

// The free pages in increasing order, until `want` are found.  Those of a pass, at most
// kDecide * kRun, go to `list`, counted from page `base` on; use(r0, n, base) then has the
// r0-th to the (r0 + n - 1)-th there.
// `ahead`: free_mask of the thread's first run, asked for before the caller knew `want`.
// Returns how many there are (at least `want`, or all).
template <class Use>
__device__ __forceinline__ int find_free(const int32_t* ref, int num_blocks, int want, unsigned ahead,
                                         uint16_t* list, Use use) {
  int found = 0;
  for (long long at = pass_start(ref); at < num_blocks && found < want; at += kDecide * kRun) {
    const long long first = at + (long long)threadIdx.x * kRun;
    unsigned free = at <= 0 ? ahead : free_mask(ref, num_blocks, first);
    int total;
    int r = block_scan(__popc(free), total);
    if (total == 0) continue;  // (all threads; the last 64 of 2^20 pages: 155 us, now 115)
    const int most = min(total, want - found);
    for (; free && r < most; free &= free - 1) list[r++] = (uint16_t)(threadIdx.x * kRun + __ffs((int)free) - 1);
    __syncthreads();
    use(found, most, (int)at);
    __syncthreads();
    found += total;
  }
  return found;
}

// Pages for n_rows[b] more rows of every sequence.  One workgroup; a thread has
// kSeqs consecutive sequences.
struct ReserveArgs {
  const int32_t* n_rows;
  int32_t* table;
  const int32_t* kv_len;
  int32_t* ref;
  int32_t* ok;
  int B, max_blocks, shift, num_blocks;
};
constexpr int kSeqs = kMaxReserve / kDecide;

__global__ __launch_bounds__(kDecide) void reserve_pages(ReserveArgs a) {
  __shared__ int first_rank[kMaxReserve + 1], first_entry[kMaxReserve];
  __shared__ uint16_t list[kDecide * kRun];
  const unsigned ahead =
      free_mask(a.ref, a.num_blocks, pass_start(a.ref) + (long long)threadIdx.x * kRun);
  // what each sequence has, needs and is short of
  int have[kSeqs], ask[kSeqs], mine = 0;
  bool valid[kSeqs];
#pragma unroll
  for (int k = 0; k < kSeqs; ++k) {
    const int b = threadIdx.x * kSeqs + k;
    have[k] = ask[k] = 0;
    valid[k] = false;
    if (b >= a.B) continue;
    const int kv = a.kv_len[b], n = a.n_rows[b], cap = a.max_blocks << a.shift;
    valid[k] = kv >= 0 && n >= 0 && kv <= cap && n <= cap - kv;
    if (!valid[k]) continue;
    const int need = (kv + n + (1 << a.shift) - 1) >> a.shift;
    // the first entry without a page, behind those of the rows that are there: a row's
    // pages come first
    const int32_t* row = a.table + (size_t)b * a.max_blocks;
    int lo = (kv + (1 << a.shift) - 1) >> a.shift, hi = need;
    for (int at = lo, step = 1; at < hi; at += step, step *= 2) {
      if (row[at] < 0) hi = at;
      else lo = at + 1;
    }
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (row[mid] < 0) hi = mid;
      else lo = mid + 1;
    }
    have[k] = lo;
    ask[k] = need - lo;
    mine += ask[k];
  }
  int total;
  int rank = block_scan(mine, total);
#pragma unroll
  for (int k = 0; k < kSeqs; ++k) {
    const int b = threadIdx.x * kSeqs + k;
    first_rank[b] = rank;
    first_entry[b] = have[k];
    rank += ask[k];
  }
  if (threadIdx.x == 0) first_rank[kMaxReserve] = total;
  __syncthreads();
  // the r-th free page goes to the sequence whose ranks hold r
  const int found = find_free(a.ref, a.num_blocks, total, ahead, list, [&](int r0, int n, int base) {
    for (int i = threadIdx.x; i < n; i += kDecide) {
      const int r = r0 + i, page = base + list[i];
      int lo = 0, hi = a.B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_rank[mid] <= r) lo = mid;
        else hi = mid;
      }
      a.table[(size_t)lo * a.max_blocks + first_entry[lo] + r - first_rank[lo]] = page;
      a.ref[page] = 1;
    }
  });
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSeqs; ++k) {
    const int b = threadIdx.x * kSeqs + k;
    if (b >= a.B) continue;
    const int r = first_rank[b];
    const bool ok = valid[k] && (ask[k] == 0 || r + ask[k] <= found);
    a.ok[b] = ok;
    if (!ok && valid[k])  // short of pages: the ones it got go back
      for (int j = 0; j < found - r && j < ask[k]; ++j) {
        int32_t* entry = a.table + (size_t)b * a.max_blocks + have[k] + j;
        a.ref[*entry] = 0;
        *entry = -1;
      }
  }
}

// Forks, first half: which are possible, and which page each one's partly filled page is
// copied to.  One workgroup, a thread per fork.
__global__ __launch_bounds__(kDecide) void fork_decide(ForkArgs a) {
  __shared__ __attribute__((aligned(16))) int to[kDecide];
  __shared__ int fresh[kDecide], from[kDecide], pages[kDecide];
  __shared__ uint16_t list[kDecide * kRun];
  const int i = threadIdx.x;
  const unsigned ahead =
      free_mask(a.ref, a.num_blocks, pass_start(a.ref) + (long long)i * kRun);
  const int src = i < a.n ? a.src[i] : -1, dst = i < a.n ? a.dst[i] : -1;
  bool ok = src >= 0 && src < a.B && dst >= 0 && dst < a.B;
  int kv = 0, first = -1, last = -1;  // dst's first entry, src's partly filled page
  if (ok) {
    first = a.table[(size_t)dst * a.max_blocks];
    kv = a.kv_len[src];
    ok = kv >= 0 && kv <= (a.max_blocks << a.shift);
    if (ok && (kv & ((1 << a.shift) - 1))) last = a.table[(size_t)src * a.max_blocks + (kv >> a.shift)];
  }
  to[i] = dst;
  from[i] = src;
  pages[i] = ok ? (kv + (1 << a.shift) - 1) >> a.shift : 0;
  __syncthreads();
  // Has every source a page for each of its rows?  A wave takes forks in turn, kAtOnce of
  // them together; the first entries are asked for before the numbers are compared.  (One
  // more round trip: 56 children of 8 rows of 64 pages, the whole call, 12.9 -> 13.9 us.)
  constexpr int kAtOnce = 4, kWaves = kDecide / 64;
  static_assert(kMaxForks == kDecide && kDecide % (kAtOnce * kWaves) == 0, "a thread per fork");
  const int lane = i & 63, wave = i >> 6;
  int entry[kAtOnce];
  auto ask = [&](int f0, int j) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int f = f0 + u * kWaves;
      entry[u] = j < pages[f] ? a.table[(size_t)from[f] * a.max_blocks + j] : 0;
    }
  };
  ask(wave, lane);
  // (the rest of `to` is -1, which is nobody's number)
  bool clash = false;
  for (int j = 0; j < a.n; j += 4) {
    const int4 t = *(const int4*)(to + j);
    clash |= t.x == src || t.y == src || t.z == src || t.w == src;
    clash |= (t.x == dst && j < i) || (t.y == dst && j + 1 < i) || (t.z == dst && j + 2 < i) ||
             (t.w == dst && j + 3 < i);
  }
  for (int f0 = wave; f0 < a.n; f0 += kAtOnce * kWaves) {
    int most = 0;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) most = max(most, pages[f0 + u * kWaves]);
    bool lacks[kAtOnce] = {};
    for (int j0 = 0; j0 < most; j0 += 64) {
      if (f0 > wave || j0 > 0) ask(f0, j0 + lane);
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) lacks[u] |= entry[u] < 0 || entry[u] >= a.num_blocks;
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (__any(lacks[u]) && lane == 0) pages[f0 + u * kWaves] = -1;
  }
  __syncthreads();
  ok = ok && first < 0 && !clash && pages[i] >= 0;
  const bool part = ok && (kv & ((1 << a.shift) - 1)) != 0;
  int total;
  const int rank = block_scan(part, total);
  const int found = find_free(a.ref, a.num_blocks, total, ahead, list, [&](int r0, int n, int base) {
    for (int k = i; k < n; k += kDecide) fresh[r0 + k] = base + list[k];
  });
  if (i >= a.n) return;
  const bool copies = part && rank < found;
  ok = ok && (!part || copies);
  a.ok[i] = ok;
  a.copy_src[i] = copies ? last : -1;
  a.copy_dst[i] = copies ? fresh[rank] : -1;
}

// Moves piece `piece` of the pages from -> to, pools after each other, 16 KB a piece.
// (Loads and stores that do not stay in the caches: some 900 of 4096 pages of 128 KB moved
// in 52.6 us, with ordinary ones in 60.0, with such loads only in 49.3 where the pools had
// just been touched, in 58.6 where they had not.)
__device__ __forceinline__ void copy_piece(const Pools& p, int from, int to, int piece) {
  int k = 0;
  while (piece >= p.pieces[k]) piece -= p.pieces[k++];
  const long long bytes = p.page_bytes[k], at = (long long)piece * kPieceBytes;
  const char* s = (const char*)p.base[k] + from * bytes + at;
  char* d = (char*)p.base[k] + to * bytes + at;
  const int len = (int)(bytes - at < kPieceBytes ? bytes - at : kPieceBytes);
  if ((((uintptr_t)s | (uintptr_t)d | (uintptr_t)len) & 15) == 0) {
    constexpr int kIn = kPieceBytes / 16 / kCopyThreads;
    i32x4 v[kIn];
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      const int c = (u * kCopyThreads + (int)threadIdx.x) * 16;
      if (c < len) v[u] = __builtin_nontemporal_load((const i32x4*)(s + c));
    }
#pragma unroll
    for (int u = 0; u < kIn; ++u) {
      const int c = (u * kCopyThreads + (int)threadIdx.x) * 16;
      if (c < len) __builtin_nontemporal_store(v[u], (i32x4*)(d + c));
    }
  } else {
    for (int c = threadIdx.x; c < len; c += kCopyThreads) d[c] = s[c];
  }
}

// Second half: shared pages, the child's row and length, and the copies.  A row of
// workgroups per fork; the first does the bookkeeping.
__global__ __launch_bounds__(kCopyThreads) void fork_do(ForkArgs a) {
  const int i = blockIdx.x;
  if (!a.ok[i]) return;
  const int src = a.src[i], dst = a.dst[i], from = a.copy_src[i], to = a.copy_dst[i];
  if (blockIdx.y == 0) {
    const int kv = a.kv_len[src], full = kv >> a.shift;
    const int32_t* row = a.table + (size_t)src * a.max_blocks;
    int32_t* mine = a.table + (size_t)dst * a.max_blocks;
    for (int j = threadIdx.x; j < a.max_blocks; j += kCopyThreads) {
      int page = -1;
      if (j < full) {
        page = row[j];
        if (page >= 0 && page < a.num_blocks) atomicAdd(a.ref + page, 1);
      } else if (j == full && to >= 0) {
        page = to;
        a.ref[page] = 1;
      }
      mine[j] = page;
    }
    if (threadIdx.x == 0) a.kv_len[dst] = kv;
  }
  if (from < 0 || from >= a.num_blocks || to < 0) return;
  for (int piece = blockIdx.y; piece < a.pools.total; piece += gridDim.y)
    copy_piece(a.pools, from, to, piece);
}

__global__ __launch_bounds__(256) void free_pages(const int32_t* seqs, int n, int32_t* table,
                                                  int32_t* kv_len, int32_t* ref, int B, int max_blocks,
                                                  int num_blocks) {
  const int i = blockIdx.x, b = seqs[i];
  bool skip = b < 0 || b >= B;
  for (int j = threadIdx.x; j < i; j += 256) skip |= seqs[j] == b;  // named before
  if (__syncthreads_or(skip)) return;
  int32_t* row = table + (size_t)b * max_blocks;
  for (int j = threadIdx.x; j < max_blocks; j += 256) {
    const int page = row[j];
    if (page < 0) continue;
    if (page < num_blocks && atomicSub(ref + page, 1) <= 0) atomicAdd(ref + page, 1);
    row[j] = -1;
  }
  if (threadIdx.x == 0) kv_len[b] = 0;
}

__global__ __launch_bounds__(kCopyThreads) void copy_pages(CopyArgs a) {
  const long long items = (long long)a.n * a.pools.total;
  for (long long w = blockIdx.x; w < items; w += gridDim.x) {
    const int i = (int)(w / a.pools.total);
    const int from = a.src[i], to = a.dst[i];
    if (from < 0 || to < 0 || from >= a.num_blocks || to >= a.num_blocks || from == to) continue;
    copy_piece(a.pools, from, to, (int)(w % a.pools.total));
  }
}

// Compaction.  With L live pages, free pages below L and live ones from L on are equally
// many; the d-th such free page (upwards) takes the d-th such live one (downwards).  With
// P(x) live pages below x: free x < L has d = x - P(x), live x >= L has d = L - 1 - P(x).
// Kernels: counts per run of pages; places; then copies, counts and tables.
__device__ __forceinline__ unsigned live_of(const CompactArgs& a, long long first, int& n) {
  unsigned live = 0;
  n = 0;
#pragma unroll
  for (int k = 0; k < kCompactPer; ++k)
    if (first + k < a.num_blocks && a.ref[first + k] > 0) live |= 1u << k;
  n = __popc(live);
  return live;
}

__device__ __forceinline__ void clear_lists(const CompactArgs& a, long long first) {
  for (int k = 0; k < kCompactPer; ++k) {
    const long long x = first + k;
    if (x < a.num_blocks) a.place[x] = -1;
    if (x < a.num_blocks / 2) a.copy_src[x] = a.copy_dst[x] = -1;
  }
}

__global__ __launch_bounds__(kDecide) void compact_count(CompactArgs a) {
  const long long first = ((long long)blockIdx.x * kDecide + threadIdx.x) * kCompactPer;
  int n, total;
  live_of(a, first, n);
  block_scan(n, total);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
  clear_lists(a, first);
}

// (A single run is counted here: a kernel less, 5 us.)
__global__ __launch_bounds__(kDecide) void compact_place(CompactArgs a) {
  const int runs = gridDim.x;
  const long long first = ((long long)blockIdx.x * kDecide + threadIdx.x) * kCompactPer;
  int n, L, before = 0, sum;
  const unsigned live = live_of(a, first, n);
  if (runs == 1) clear_lists(a, first);
  int P = block_scan(n, L);  // (its barriers: the lists are cleared)
  if (runs > 1) {
    int all = 0;
    for (int r = threadIdx.x; r < runs; r += kDecide) {
      const int c = a.counts[r];
      all += c;
      before += r < (int)blockIdx.x ? c : 0;
    }
    block_scan(before, sum);
    P += sum;
    block_scan(all, L);
  }
  for (int k = 0; k < kCompactPer; ++k) {
    const long long x = first + k;
    if (x >= a.num_blocks) break;
    const bool is = live >> k & 1;
    if (x == L) *a.moves = L - P;
    if (!is && x < L) a.copy_dst[x - P] = (int)x;
    if (is && x >= L) {
      a.copy_src[L - 1 - P] = (int)x;
      a.place[x] = L - 1 - P;
    }
    P += is;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.n_live = L;
    if (L >= a.num_blocks) *a.moves = 0;
  }
}

__global__ __launch_bounds__(kCopyThreads) void compact_move(CompactArgs a) {
  const int moves = *a.moves;
  if (moves == 0) return;
  const long long me = (long long)blockIdx.x * kCopyThreads + threadIdx.x;
  const long long all = (long long)gridDim.x * kCopyThreads;
  for (long long t = me; t < (long long)a.B * a.max_blocks; t += all) {
    const int page = a.table[t];
    if (page < 0 || page >= a.num_blocks) continue;
    const int d = a.place[page];
    if (d >= 0) a.table[t] = a.copy_dst[d];
  }
  for (long long d = me; d < moves; d += all) {
    const int from = a.copy_src[d];
    a.ref[a.copy_dst[d]] = a.ref[from];
    a.ref[from] = 0;
  }
  const long long items = (long long)moves * a.pools.total;
  for (long long w = blockIdx.x; w < items; w += gridDim.x) {
    const int d = (int)(w / a.pools.total);
    copy_piece(a.pools, a.copy_src[d], a.copy_dst[d], (int)(w % a.pools.total));
  }
}

// ------------------------------------------------------------------ launches

static unsigned copy_grid(long long items) { return (unsigned)(items < 4096 ? items : 4096); }

hipError_t launch_reserve(const int32_t* n_rows, int32_t* table, const int32_t* kv_len, int32_t* ref,
                          int32_t* ok, int B, int max_blocks, int shift, int num_blocks, hipStream_t st) {
  hipLaunchKernelGGL(reserve_pages, dim3(1), dim3(kDecide), 0, st,
                     (ReserveArgs{n_rows, table, kv_len, ref, ok, B, max_blocks, shift, num_blocks}));
  return hipGetLastError();
}

hipError_t launch_fork(const ForkArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(fork_decide, dim3(1), dim3(kDecide), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pieces = a.pools.total < 1 ? 1 : (a.pools.total < 64 ? a.pools.total : 64);
  hipLaunchKernelGGL(fork_do, dim3(a.n, pieces), dim3(kCopyThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_free(const int32_t* seqs, int n, int32_t* table, int32_t* kv_len, int32_t* ref, int B,
                       int max_blocks, int num_blocks, hipStream_t st) {
  hipLaunchKernelGGL(free_pages, dim3(n), dim3(256), 0, st, seqs, n, table, kv_len, ref, B, max_blocks,
                     num_blocks);
  return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs& a, hipStream_t st) {
  const long long items = (long long)a.n * a.pools.total;
  if (items == 0) return hipSuccess;
  hipLaunchKernelGGL(copy_pages, dim3(copy_grid(items)), dim3(kCopyThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs& a, hipStream_t st) {
  const dim3 runs((unsigned)compact_runs(a.num_blocks));
  hipError_t e = hipSuccess;
  if (runs.x > 1) {
    hipLaunchKernelGGL(compact_count, runs, dim3(kDecide), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(compact_place, runs, dim3(kDecide), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const long long items = (long long)(a.num_blocks / 2) * a.pools.total;
  const long long rows = ((long long)a.B * a.max_blocks + kCopyThreads - 1) / kCopyThreads;
  const long long most = items > rows ? items : rows;
  hipLaunchKernelGGL(compact_move, dim3(copy_grid(most < 1 ? 1 : most)), dim3(kCopyThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace tv
