// Arguments of the page kernels (tv_pages.hip), filled in by the entry points.
#pragma once
#include <stdint.h>

namespace tv {

constexpr int kMaxPools = 64;            // == TV_MAX_POOLS
constexpr int kMaxForks = 1024;          // == TV_MAX_FORKS
constexpr int kMaxReserve = 4096;        // == TV_MAX_RESERVE
constexpr int kPieceBytes = 16384, kCopyThreads = 256;
constexpr int kCompactPer = 4;           // pages a thread of the compaction counts
constexpr int kCompactRun = 1024 * kCompactPer;

// Pools whose first axis is the page; a page of pool k is page_bytes[k] bytes, copied in
// pieces[k] pieces, total in all.
struct Pools {
  void* base[kMaxPools];
  long long page_bytes[kMaxPools];
  int pieces[kMaxPools];
  int n, total;
};

struct ForkArgs {
  const int32_t* src;
  const int32_t* dst;
  int32_t* table;
  int32_t* kv_len;
  int32_t* ref;
  int32_t* ok;
  int32_t* copy_src;
  int32_t* copy_dst;
  int n, B, max_blocks, shift, num_blocks;
  Pools pools;
};

struct CopyArgs {
  const int32_t* src;
  const int32_t* dst;
  int n, num_blocks;
  Pools pools;
};

struct CompactArgs {
  int32_t* table;
  int32_t* ref;
  int32_t* n_live;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* place;   // workspace: [num_blocks] a moved page's place in the lists, -1
  int32_t* counts;  // [runs] live pages of a run
  int32_t* moves;   // [1]
  int B, max_blocks, num_blocks;
  Pools pools;
};

inline int compact_runs(int num_blocks) { return (num_blocks + kCompactRun - 1) / kCompactRun; }

}  // namespace tv
