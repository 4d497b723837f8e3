// The writers of the paged cache in 8 bits, for CDNA4 (gfx950): rows of new keys and
// values, or the accepted path's of a draft tree, become e4m3 codes behind a sequence's
// kv_len rows, and kv_len grows.
//
// Per sequence, group of 32 positions that gets rows, head, and K or V:
//   a   the largest size among the group's new values that are finite numbers (the others
//       become codes that are no numbers, and cost their group nothing else)
//   e   the least byte of [16, 247] with a <= 448 * 2^(e - 127); if the group holds older
//       rows of the sequence, at least its byte so far
//   new codes: the nearest to x * 2^(127 - e), 240 at most where e is 247; older codes: the
//   nearest to what they stand for at the new exponent, so unchanged unless it grew
// Powers of two make every step but the one rounding exact, and older codes lose nothing
// but what falls below the smallest code.
//
// One wave per unit (group, K or V, head): rows come in 16 bytes a lane, the largest size
// is a maximum over bf16 bit patterns, and the wave keeps its values in registers until
// the exponent is known.  Bound by HBM where there are rows enough (6 bytes per element
// pair of K and V), by latency below.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tv_plan.h"
#include "tv_walk.h"

namespace tv {

constexpr int kGroup = 32, kExpMin = 16, kExpMax = 247;
constexpr int kInfBits = 0x7F80;  // bf16 sizes from here on are no finite numbers

struct WriteArgs {
  const __bf16* x[2];  // K's and V's rows, [B, T, Hkv, D]
  uint8_t* pool[2];    // [num_blocks, Hkv, block_size, D]
  uint8_t* exps[2];    // [num_blocks, Hkv, block_size / 32]
  const int32_t* n_new;  // rows of each sequence, NULL: T
  const int32_t* path;   // commit: [B, P], the rows' places in x; else NULL
  const int32_t* block_table;
  int32_t* kv_len;
  int shift, max_blocks, num_blocks;
  int B, T, P, Hkv, groups;  // groups: most that P rows touch
};

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// What sequence b gets: n rows, 0 where it is left as it is; but that it has a page for
// all of them is known only once `lacking` is looked at, in any lane.
struct Rows {
  int n, page;   // page: of this lane's, the sequence's entry `lane` behind the first one's
  bool lacking;
};
__device__ __forceinline__ Rows rows_of(const WriteArgs& a, int b, int kv) {
  Rows r{0, -1, false};
  const int n = a.n_new ? a.n_new[b] : a.P, lane = threadIdx.x & 63;
  const int cap = a.max_blocks << a.shift;
  if (n < 1 || n > a.P || kv < 0 || kv > cap - n) return r;
  const int first = kv >> a.shift, last = (kv + n - 1) >> a.shift;
  const int32_t* row = a.block_table + (size_t)b * a.max_blocks;
  if (first + lane <= last) {
    r.page = row[first + lane];
    r.lacking = r.page < 0 || r.page >= a.num_blocks;
  }
  for (int j = first + lane + 64; j <= last; j += 64) r.lacking |= row[j] < 0 || row[j] >= a.num_blocks;
  if (a.path) {
    bool bad = false;
    for (int j = lane; j < n; j += 64) {
      const int node = a.path[(size_t)b * a.P + j];
      bad |= node < 0 || node >= a.T;
    }
    if (__any(bad)) return r;
  }
  r.n = n;
  return r;
}

__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// Two bf16 numbers of a word, scaled, as codes in the low or high half of `into`.
template <bool kHigh>
__device__ __forceinline__ int two_codes(int w, float scale, int into) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(__int_as_float(w << 16) * scale,
                                         __int_as_float(w & 0xFFFF0000) * scale, into, kHigh);
}

// At the largest exponent code 0x78 would stand for 2^128, which neither bf16 nor fp32
// holds (the largest numbers, scaled, are below 256 and may round to it): such codes
// become 0x77, 240.
__device__ __forceinline__ int limited(int w) {
  const int ones = w >> 3 & w >> 4 & w >> 5 & w >> 6, rest = w | w >> 1 | w >> 2;
  return w - (ones & ~rest & 0x01010101);
}

// Four codes at another exponent.
__device__ __forceinline__ int rescaled(int w, float scale) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  const int half = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * scale, lo[1] * scale, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * scale, hi[1] * scale, half, true);
}

// Unit (group gi of those that get rows, head h, K or V) of sequence b with its new rows
// from kv on.  kMany: loads and stores that do not stay in the caches (four prompts, 125 MB in
// all: 39 us, now 33).
template <int D, bool kMany>
__device__ __forceinline__ void write_unit(const WriteArgs& a, int b, int kv, const Rows& rows, int gi, int h,
                                           int isv) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kLoads = kGroup / kRows;
  const int lane = threadIdx.x & 63, l = lane % kLanes;
  const int first = ((kv >> 5) + gi) * kGroup, n = rows.n;  // the group's first position
  if (first >= kv + n) return;
  i32x4 v[kLoads];
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int j = first + k * kRows + lane / kLanes - kv;  // new row
    v[k] = i32x4{0, 0, 0, 0};
    if (j >= 0 && j < n) {
      const int row = a.path ? a.path[(size_t)b * a.P + j] : j;
      const i32x4* x = (const i32x4*)(a.x[isv] + (((size_t)b * a.T + row) * a.Hkv + h) * D + 8 * l);
      v[k] = kMany ? __builtin_nontemporal_load(x) : *x;
    }
  }
  // the rows are on their way: is there a page for each, and which is this group's
  if (__any(rows.lacking)) return;
  const int at = (first >> a.shift) - (kv >> a.shift);
  const int blk = at < 64 ? __builtin_amdgcn_readlane(rows.page, at)
                          : a.block_table[(size_t)b * a.max_blocks + (first >> a.shift)];
  const int per = a.shift - 5;
  const size_t group = (((size_t)blk * a.Hkv + h) << per) + ((first >> 5) & ((1 << per) - 1));
  const bool older = first < kv;
  const int was = older ? a.exps[isv][group] : 0;
  // the largest of the bit patterns + margin, as signed numbers, less margin (sizes: 0x7FFF
  // twice, opaque so that what a second look needs is not kept from the first)
  auto largest = [&](uint16_t margin) {
    int sizes = 0x7FFF7FFF;
    asm volatile("" : "+s"(sizes));
    i16x2 most = {0, 0};
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        most = __builtin_elementwise_max(
            most, __builtin_bit_cast(i16x2, __builtin_bit_cast(u16x2, v[k][w] & sizes) + margin));
    return max(0, (int)wave_max_u32(most[0] > most[1] ? most[0] : most[1]) - margin);
  };
  int a_bits = largest(0);
  if (a_bits >= kInfBits) a_bits = largest(0x8000 - kInfBits);  // which those are negative with
  // 448 = 1.75 * 2^8: the exponent 8 below the value's, one more above 1.75
  int e = (a_bits >> 7) - 8 + ((a_bits & 127) > 96);
  e = e < kExpMin ? kExpMin : (e > kExpMax ? kExpMax : e);
  e = e < was ? was : e;
  const float scale = power_of_two(127 - e);
  uint8_t* out = a.pool[isv] + group * (kGroup * D) + 8 * l;
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int r = k * kRows + lane / kLanes, j = first + r - kv;
    if (j >= 0 && j < n) {
      i32x2 c;
#pragma unroll
      for (int w = 0; w < 2; ++w)
        c[w] = two_codes<true>(v[k][2 * w + 1], scale, two_codes<false>(v[k][2 * w], scale, 0));
      if (e == kExpMax) c = i32x2{limited(c[0]), limited(c[1])};
      if (kMany) __builtin_nontemporal_store(c, (i32x2*)(out + r * D));
      else *(i32x2*)(out + r * D) = c;
    } else if (older && j < 0 && e > was) {
      const float down = power_of_two(was - e < -126 ? -126 : was - e);
      i32x2 c = *(const i32x2*)(out + r * D);
      c[0] = rescaled(c[0], down);
      c[1] = rescaled(c[1], down);
      *(i32x2*)(out + r * D) = c;
    }
  }
  if (lane == 0 && e != was) a.exps[isv][group] = (uint8_t)e;
}

// Few groups per sequence: a workgroup per sequence, its waves take the units in turn.
template <int D>
__global__ __launch_bounds__(1024) void write_sequence(WriteArgs a) {
  const int b = blockIdx.x, waves = blockDim.x / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv = a.kv_len[b];
  const Rows rows = rows_of(a, b, kv);
  const int units = rows.n > 0 ? a.groups * 2 * a.Hkv : 0;
  for (int u = wave; u < units; u += waves) {
    const int h = u % a.Hkv, r = u / a.Hkv;
    write_unit<D, false>(a, b, kv, rows, r >> 1, h, r & 1);
  }
  const bool lacking = __any(rows.lacking);
  __syncthreads();  // every wave has read kv_len
  if (threadIdx.x == 0 && rows.n > 0 && !lacking) a.kv_len[b] = kv + rows.n;
}

// Many: a wave per unit, and kv_len grows in a second kernel.
template <int D>
__global__ __launch_bounds__(256) void write_groups(WriteArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long u = (long long)blockIdx.x * 4 + wave;
  const int h = (int)(u % a.Hkv), isv = (int)(u / a.Hkv % 2);
  const long long r = u / (2 * a.Hkv);
  const int gi = (int)(r % a.groups);
  const long long b = r / a.groups;
  if (b >= a.B) return;
  const int kv = a.kv_len[b];
  const Rows rows = rows_of(a, (int)b, kv);
  if (rows.n > 0) write_unit<D, true>(a, (int)b, kv, rows, gi, h, isv);
}

__global__ __launch_bounds__(64) void grow_lengths(WriteArgs a) {
  const int b = blockIdx.x, kv = a.kv_len[b];
  const Rows rows = rows_of(a, b, kv);
  const bool lacking = __any(rows.lacking);
  if (threadIdx.x == 0 && rows.n > 0 && !lacking) a.kv_len[b] = kv + rows.n;
}

// x: K's and V's rows [B, T, Hkv, D]; P: rows at most that a sequence gets.
hipError_t launch_write_fp8(const void* k, const void* v, const int32_t* n_new, const int32_t* path,
                            void* k_pool, void* v_pool, uint8_t* k_exp, uint8_t* v_exp,
                            const int32_t* block_table, int shift, int max_blocks, int num_blocks,
                            int32_t* kv_len, int B, int T, int P, int Hkv, int D, hipStream_t st) {
  const int cap = max_blocks << shift, most = P < cap ? P : cap;
  WriteArgs a{{(const __bf16*)k, (const __bf16*)v}, {(uint8_t*)k_pool, (uint8_t*)v_pool}, {k_exp, v_exp},
              n_new, path, block_table, kv_len, shift, max_blocks, num_blocks, B, T, P, Hkv,
              (most + 30) / kGroup + 1};
  const long long units = 2LL * Hkv * a.groups;
  if (units <= 64) {
    const dim3 threads(64 * (unsigned)(units < 16 ? units : 16));
    if (D == 128) hipLaunchKernelGGL(write_sequence<128>, dim3(B), threads, 0, st, a);
    else hipLaunchKernelGGL(write_sequence<64>, dim3(B), threads, 0, st, a);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((units * B + 3) / 4));
  if (D == 128) hipLaunchKernelGGL(write_groups<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(write_groups<64>, grid, dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grow_lengths, dim3(B), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace tv
