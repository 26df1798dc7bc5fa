// What the kernels of the paged cache's attention share: parameters, codes to fp16, and the line of work that is cut into runs.
#pragma once

#include <cuda_fp16.h>
#include <math_constants.h>

#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace skv {

constexpr int kAttMaxRuns = 592;       // thread blocks of a call: four on each of 148 SMs
constexpr int kAttPartRows = 2 * kAttMaxRuns * 32;   // rows of partial results: two parts of a run, up to 32 columns each (or 128 of a quarter of the runs)
constexpr int kHdrUnitsDone = 16;      // words 16, 17 of the status block: units of a call that runs a block for each
constexpr float kAttLazy = 8.f;        // how far a score may exceed the running reference, in powers of two
constexpr float kAttPScale = 128.f;    // p <= 2^8 times this stays inside fp16

struct AttendParams {
  Pool pool;
  Table table;
  View q, out;
  int hn, n_rows, cols;      // query heads per KV head, new rows, columns in all
  int groups;                // column groups of a (layer, seq, KV head): its units
  int units_per;             // heads * groups
  int per_shift;             // log2 of the blocks of a page
  float scale;               // softmax scale * log2(e)
  int whole_units;           // 1: every run is one unit, nothing is left to join
  int part_cols;             // columns of a part
  float* part;               // [2 * runs][part_cols][d]: O of the parts of units that several runs share
  float2* stat;              // [2 * runs][part_cols]: their m and sum
  int2* lead;                // [runs] the unit that a run is the first to continue and its number of parts; unit -1: none, -2: a wait gave up
  uint32_t* hdr;             // status block of the workspace
  long long wait_cycles;     // bound of a wait
  int withhold;              // for tests: the block that does not ask for its first keys; -1: none
};

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// N = 2 or 4 neighbouring elements
template <int N>
__device__ __forceinline__ void load_elements(const float* p, float (&x)[N]) {
  if constexpr (N == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else {
    const float2 v = *reinterpret_cast<const float2*>(p);
    x[0] = v.x; x[1] = v.y;
  }
}
template <int N>
__device__ __forceinline__ void load_elements(const __nv_bfloat16* p, float (&x)[N]) {
  uint32_t w[N / 2];
  if constexpr (N == 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// two of the four codes in w (bytes 0, 1 with HI = 0; 2, 3 with HI = 1) as two fp16 numbers
template <int FMT, int HI>
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t w) {
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    // w holds code + 128: 1024 + that is an fp16 number whose low byte it is
    const uint32_t x = __byte_perm(w, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 off = __half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&x), off);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    uint32_t v;
    if constexpr (HI) asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(v) : "r"(w));
    else asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(v) : "r"(w));
    return v;
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t prepare_codes(uint32_t w) { return FMT == SPINDLEKV_PAGED_INT8 ? w ^ 0x80808080u : w; }
// E4M3 codes of slots behind the last token may be its NaN patterns, whose product with a weight of 0 is not 0: a bit less, and
// they are numbers
__device__ __forceinline__ uint32_t without_nan(uint32_t w) { return w ^ ((((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u); }

// The line: unit (ls, head, group) takes SETUP places, which stand for looking up its pages, reading its queries and joining its
// warps, and then one for every TOKENS tokens; all units of a (layer, seq) lie side by side.  Without the first places a run with the
// ends of two or three units in it finishes last.
template <int TOKENS, int SETUP>
__device__ __forceinline__ int places_of(const AttendParams& p, int ls) {
  const int len = unit_len(p.table, p.pool, ls);
  return len ? (len + TOKENS - 1) / TOKENS + SETUP : 0;
}

// prefix[ls]: places of a unit of every (layer, seq) before; returns all of them.  All threads of the block
template <int TOKENS, int SETUP>
__device__ __forceinline__ int line_prefix(const AttendParams& p, int* prefix, int* warp_sums) {
  const int n_ls = p.table.n_layers * p.table.n_seqs, lane = threadIdx.x & 31;
  int total = 0;
  if (n_ls <= 32) {      // every warp for itself, the same values
    const int n = lane < n_ls ? places_of<TOKENS, SETUP>(p, lane) : 0;
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int below = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += below;
    }
    if (lane < n_ls) prefix[lane] = upto - n;
    total = __shfl_sync(0xffffffffu, upto, 31);
    if (lane == 0) prefix[n_ls] = total;
    __syncwarp();
  } else {
    for (int base = 0; base < n_ls; base += (int)blockDim.x) {
      const int ls = base + (int)threadIdx.x;
      const int n = ls < n_ls ? places_of<TOKENS, SETUP>(p, ls) : 0;
      int sum;
      const int at = block_exclusive_scan(n, warp_sums, sum);
      if (ls < n_ls) prefix[ls] = total + at;
      total += sum;
    }
    if (threadIdx.x == 0) prefix[n_ls] = total;
    __syncthreads();
  }
  return total;
}

// Run i has the places from all * i / runs (rounded down) on; runs without any are the last ones
struct Runs {
  int runs, share, left;
  float per_runs, runs_per_place;
  __device__ __forceinline__ Runs(int all, int blocks) {
    runs = min(blocks, max(all, 1));
    share = all / runs;
    left = all - share * runs;
    per_runs = 1.f / (float)runs;
    runs_per_place = (float)runs / (float)max(all, 1);
  }
  // left * i < 2^20 and runs < 2^10: the product is off by less than half of 1 / runs, so the quotient is exact
  __device__ __forceinline__ int start(int i) const { return share * i + (int)(((float)(left * i) + 0.5f) * per_runs); }
  __device__ __forceinline__ int of(int place) const {
    int i = (int)((float)place * runs_per_place);
    while (start(i) > place) --i;
    while (start(i + 1) <= place) ++i;
    return i;
  }
};

// the (layer, seq) that holds a place
__device__ __forceinline__ int unit_at(const AttendParams& p, const int* prefix, int place) {
  int lo = 0, hi = p.table.n_layers * p.table.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] * p.units_per <= place) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// sequences without tokens give zeros
template <typename T, int D>
__device__ __forceinline__ void zero_empty(const AttendParams& p, const int* prefix) {
  const int n_ls = p.table.n_layers * p.table.n_seqs;
  for (int e = blockIdx.x; e < n_ls; e += gridDim.x)
    if (prefix[e + 1] == prefix[e]) {
      const int layer = e / p.table.n_seqs, seq = e - layer * p.table.n_seqs, per_head = p.n_rows * D;
      T* dst = reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + (int64_t)layer * p.out.sl + (int64_t)seq * p.out.ss;
      for (int i = threadIdx.x; i < p.pool.heads * p.hn * per_head; i += (int)blockDim.x) {
        const int h = i / per_head, r = (i - h * per_head) / D, d = i % D;
        dst[(int64_t)h * p.out.sh + (int64_t)r * p.out.st + d] = T(0.f);
      }
    }
}

// attention of 17 to 128 bf16 columns of 128 elements on the tensor cores' own memory; false: not this call
bool paged_attend_tiles(AttendParams& p, int format, int max_len, cudaStream_t st, int* runs, spindlekv_status* status);

// codes [page][row][d] -> 3-D map (d, row, page), box d x box_rows, swizzled as wide as a row
bool make_code_map(CUtensorMap* map, const void* codes, int head_dim, int rows, int n_pages, int box_rows);

}  // namespace skv
