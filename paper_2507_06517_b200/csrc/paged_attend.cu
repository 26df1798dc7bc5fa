// Attention of the newest tokens over the 8-bit paged cache.
//
// Bound: every cached byte has to come from memory once (2 d bytes per token and KV head, plus 8/16 bytes of scales), so all
// query heads of a KV head, and all new rows, are served by one pass over its codes.
//
// Mathematics.  The tensor cores multiply fp16 by fp16 into fp32.  Codes are exact in fp16, and so are the numbers
// of E4M3.  Queries enter scaled by a power of two per row: bf16 queries are exact in one fp16 piece (elements below
// 2^-29 of the row's largest fade out), fp32 queries in two pieces (22 bits).  S^T = K Q^T, then p = 2^(S s_k c - m) with a running
// reference m per query that moves only when a score exceeds it by 8 (p stays below 2^8), O^T += s_v (V^T P^T) with P in one fp16
// piece for bf16 (2^-12 relative, below the output's rounding) or two for fp32; the scale s_v of a block is applied to the product of
// that block in fp32, so blocks of very different scale do not disturb one another.  m, the sum of p and O are fp32.
//
// Layout.  A warp takes one block of 16 tokens at a time: K is the 16 x d operand of m16n8k16, the queries are its 8 columns.  Which
// token or element a lane's fragment registers stand for is free as long as both operands agree, so codes go from memory straight into
// the registers that need them, 16 bytes per lane, without shared memory: a lane's 16 bytes of a K row are four k-steps; for V it reads
// the same 16 bytes of four tokens and transposes bytes between registers.  The next block's loads are in flight while this one is
// computed.  P changes layout by an 8x8 transposition inside the warp.
//
// Split.  All blocks of all (layer, sequence, head) units form one line, cut into equal runs, one per resident thread block;
// the eight warps of a thread block deal a run's blocks among themselves.  Every run thus has the same work however
// uneven the lengths are.  A unit that lies inside one run is finished there; of the others each run leaves (m, sum, O), which a second
// kernel joins in the order of the runs.
#include <algorithm>

#include <cuda_fp16.h>
#include <math_constants.h>

#include "paged.cuh"

namespace skv {

constexpr int kAttThreads = 256;
constexpr int kAttWarps = kAttThreads / 32;
constexpr int kAttMaxRuns = 592;       // thread blocks of a call: four on each of 148 SMs
constexpr int kAttMaxCols = 32;        // (query head, row) columns of a unit
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
  float* part;               // [2 * kAttMaxRuns][kAttMaxCols][d]: O of the parts of units that several runs share
  float2* stat;              // [2 * kAttMaxRuns][kAttMaxCols]: their m and sum
  int32_t* lead;             // [runs] the unit that a run begins in the middle of, or -1
};

__device__ __forceinline__ uint4 load_code16(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_code8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint2 b) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
// the same from zero
__device__ __forceinline__ void mma16816_first(float (&d)[4], const uint32_t (&a)[4], uint2 b) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "f"(0.f));
}
// 2^x, to two units in the last place of fp32; results below the smallest normal number are 0
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

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

// the line of blocks: unit (ls, head, group) has blocks_of(ls) of them, all units of a (layer, seq) side by side
__device__ __forceinline__ int blocks_of(const AttendParams& p, int ls) { return (unit_len(p.table, p.pool, ls) + kPagedBlock - 1) / kPagedBlock; }

template <typename T, int FMT, int D, int NT>
__global__ void __launch_bounds__(kAttThreads, NT == 4 ? 1 : 2) paged_attend_kernel(AttendParams p) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;      // fp16 pieces of a query and of a weight
  constexpr int KS = D / 16;                      // k-steps of a score, and m-tiles of an output
  constexpr int KH = D / 64;                      // 16-byte pieces of a K row per lane
  constexpr int VW = D / 32;                      // words of a V row per lane
  constexpr int COLS = 8 * NT;
  constexpr int OP = D + 4;                       // row pitch of the partial outputs in shared memory
  constexpr float kVFactor = 1.f / kAttPScale;
  extern __shared__ uint4 smem_raw[];
  // prefix sums over the (layer, seq) pairs; then the queries' fragments, per-column factors, the warps' results
  const int n_ls = p.table.n_layers * p.table.n_seqs;
  float* so = reinterpret_cast<float*>(smem_raw);                       // [kAttWarps][COLS][OP]
  uint2* sq = reinterpret_cast<uint2*>(so + kAttWarps * COLS * OP);     // [NP][NT][KS][32]
  float* sfac = reinterpret_cast<float*>(sq + NP * NT * KS * 32);       // [COLS] score factor
  float* sm_m = sfac + COLS;                                            // [kAttWarps][COLS]
  float* sm_l = sm_m + kAttWarps * COLS;                                // [kAttWarps][COLS]
  int* warp_sums = reinterpret_cast<int*>(sm_l + kAttWarps * COLS);     // [33]
  int* prefix = warp_sums + 36;                                         // [n_ls + 1]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;   // g, c: the fragments' rows and columns

  // blocks of a (layer, seq) per unit, summed
  int total = 0;
  for (int base = 0; base < n_ls; base += kAttThreads) {
    const int ls = base + tid;
    const int n = ls < n_ls ? blocks_of(p, ls) : 0;
    int sum;
    const int at = block_exclusive_scan(n, warp_sums, sum);
    if (ls < n_ls) prefix[ls] = total + at;
    total += sum;
  }
  if (tid == 0) prefix[n_ls] = total;
  __syncthreads();
  const long long all = (long long)total * p.units_per;
  const long long per_run = (all + gridDim.x - 1) / gridDim.x;      // runs without blocks are the last ones
  long long at = per_run * blockIdx.x;
  const long long stop = min(at + per_run, all);
  // sequences without tokens give zeros
  for (int e = blockIdx.x; e < n_ls; e += gridDim.x)
    if (prefix[e + 1] == prefix[e]) {
      const int layer = e / p.table.n_seqs, seq = e - layer * p.table.n_seqs, per_head = p.n_rows * D;
      T* dst = reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + (int64_t)layer * p.out.sl + (int64_t)seq * p.out.ss;
      for (int i = tid; i < p.pool.heads * p.hn * per_head; i += kAttThreads) {
        const int h = i / per_head, r = (i - h * per_head) / D, d = i % D;
        dst[(int64_t)h * p.out.sh + (int64_t)r * p.out.st + d] = T(0.f);
      }
    }
  if (at >= stop) {
    if (tid == 0) p.lead[blockIdx.x] = -1;
    return;
  }
  int ls;
  {   // the (layer, seq) that holds block `at`
    int lo = 0, hi = n_ls - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((long long)prefix[mid] * p.units_per <= at) lo = mid; else hi = mid - 1;
    }
    ls = lo;
  }
  while (at < stop) {
    while (prefix[ls + 1] == prefix[ls] || (long long)prefix[ls + 1] * p.units_per <= at) ++ls;
    const int nb = prefix[ls + 1] - prefix[ls];
    const long long inside = at - (long long)prefix[ls] * p.units_per;
    const int uh = (int)(inside / nb), b0 = (int)(inside - (long long)uh * nb);       // (head, group), first block
    const int b1 = (int)min((long long)nb, b0 + (stop - at));
    const int head = uh / p.groups, group = uh - head * p.groups;
    if (tid == 0 && at == per_run * blockIdx.x) p.lead[blockIdx.x] = b0 > 0 ? ls * p.units_per + uh : -1;
    const int layer = ls / p.table.n_seqs, seq = ls - layer * p.table.n_seqs;
    const int len = unit_len(p.table, p.pool, ls);
    const int col0 = group * COLS, ncols = min(COLS, p.cols - col0);
    // ---- queries -> fragments: warp w takes columns w, w + 8, ... ----
    for (int col = warp; col < COLS; col += kAttWarps) {
      float x[D / 32];
      float amax = 0.f;
      if (col < ncols) {
        const int gi = (col0 + col) / p.n_rows, r = (col0 + col) - gi * p.n_rows;
        const T* row = reinterpret_cast<const T*>(p.q.ptr) + (int64_t)layer * p.q.sl + (int64_t)seq * p.q.ss +
                       (int64_t)(head * p.hn + gi) * p.q.sh + (int64_t)r * p.q.st;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = to_f32(row[lane * (D / 32) + i]);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) amax = fmaxf(amax, fabsf(x[i]));
      } else {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = 0.f;
      }
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      // power of two that brings the largest element into [2^14, 2^15); an infinite or NaN row goes through as it is
      int e = 0;
      if (amax > 0.f && amax < CUDART_INF_F) e = min(max(14 - ilogbf(amax), -126), 126);
      const float up = __int_as_float((127 + e) << 23);
      const float down = __int_as_float((127 - e) << 23);
      if (lane == 0) sfac[col] = p.scale * down;
      // element d sits in k-step (d / 64) * 4 + (d % 16) / 4 of the lanes with (d % 64) / 16 as their place in the quad
      constexpr int E = D / 32;          // this lane's elements: 4 or 2 neighbours
      const int d0 = lane * E;
      const int ks = (d0 / 64) * 4 + (d0 % 16) / 4, owner = (col & 7) * 4 + (d0 % 64) / 16;
#pragma unroll
      for (int pc = 0; pc < NP; ++pc) {
        uint32_t h[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const float a = x[2 * i] * (pc ? 1.f : up), b = x[2 * i + 1] * (pc ? 1.f : up);
          h[i] = pack_half2(a, b);
          const float2 got = unpack_half2(h[i]);
          x[2 * i] = a - got.x;
          x[2 * i + 1] = b - got.y;
        }
        uint2* slot = sq + ((pc * NT + (col >> 3)) * KS + ks) * 32 + owner;
        if constexpr (E == 4) *slot = make_uint2(h[0], h[1]);
        else reinterpret_cast<uint32_t*>(slot)[(d0 % 4) / 2] = h[0];
      }
    }
    __syncthreads();
    float fac[NT][2];
    int lim[NT][2];                     // tokens that a column sees
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int col = 8 * t + 2 * c + i;
        fac[t][i] = sfac[col];
        lim[t][i] = col < ncols ? len - p.n_rows + 1 + (col0 + col) % p.n_rows : 0;
      }
    float o[KS][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = -CUDART_INF_F;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[k][t][i] = 0.f;
    }
    const int32_t* row = p.table.pages + (int64_t)ls * p.table.max_pages;
    const int sh = p.per_shift;
    // block b of the sequence -> its place in the pool, or -1
    auto place = [&](int page, int b) -> int64_t {
      return page >= 0 && page < p.pool.n_pages ? (((int64_t)page * p.pool.heads + head) << sh) + (b & ((1 << sh) - 1)) : -1;
    };
    uint4 kr[2][KH];
    uint32_t vr[4][VW];
    float ks_c = 0.f, vs_c = 0.f;
    const int koff = g * D + c * 16, voff = 2 * c * D + g * (D / 8);
    auto load_k = [&](int64_t at_block) {
      if (at_block < 0) return;
      const uint8_t* src = p.pool.kc + at_block * (kPagedBlock * D) + koff;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int h = 0; h < KH; ++h) kr[r][h] = load_code16(src + r * 8 * D + h * 64);
      ks_c = __ldg(p.pool.ks + at_block);
    };
    auto load_v = [&](int64_t at_block) {
      if (at_block < 0) return;
      const uint8_t* src = p.pool.vc + at_block * (kPagedBlock * D) + voff;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t* s = src + ((r & 1) + (r >> 1) * 8) * D;
        if constexpr (VW == 4) {
          const uint4 v = load_code16(s);
          vr[r][0] = v.x; vr[r][1] = v.y; vr[r][2] = v.z; vr[r][3] = v.w;
        } else {
          const uint2 v = load_code8(s);
          vr[r][0] = v.x; vr[r][1] = v.y;
        }
      }
      vs_c = __ldg(p.pool.vs + at_block);
    };
    int b = b0 + warp;
    int64_t cur = -1, nxt = -1;
    if (b < b1) {
      cur = place(__ldg(row + (b >> sh)), b);
      load_k(cur);
      load_v(cur);
    }
    int page_n = b + kAttWarps < b1 ? __ldg(row + ((b + kAttWarps) >> sh)) : -1;
    for (; b < b1; b += kAttWarps) {
      const int bn = b + kAttWarps;
      nxt = bn < b1 ? place(page_n, bn) : -1;
      page_n = bn + kAttWarps < b1 ? __ldg(row + ((bn + kAttWarps) >> sh)) : -1;
      // ---- scores ----
      float sc[NT][4];
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint4& r0 = kr[0][k / 4];
        const uint4& r1 = kr[1][k / 4];
        const uint32_t w0 = prepare_codes<FMT>((k & 3) == 0 ? r0.x : (k & 3) == 1 ? r0.y : (k & 3) == 2 ? r0.z : r0.w);
        const uint32_t w1 = prepare_codes<FMT>((k & 3) == 0 ? r1.x : (k & 3) == 1 ? r1.y : (k & 3) == 2 ? r1.z : r1.w);
        const uint32_t a[4] = {codes_to_half2<FMT, 0>(w0), codes_to_half2<FMT, 0>(w1), codes_to_half2<FMT, 1>(w0), codes_to_half2<FMT, 1>(w1)};
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int pc = 0; pc < NP; ++pc) {
            const uint2 b = sq[((pc * NT + t) * KS + k) * 32 + lane];
            if (k == 0 && pc == 0) mma16816_first(sc[t], a, b);
            else mma16816(sc[t], a, b);
          }
      }
      const float ks_b = ks_c;
      load_k(nxt);
      // ---- softmax weights ----
      const int t0 = b * kPagedBlock;
      const bool masked = cur < 0 || t0 + kPagedBlock > len - p.n_rows + 1;
      bool rise = false;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[t][i] *= ks_b * fac[t][i & 1];
        if (masked) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (cur < 0 || t0 + g + (i >> 1) * 8 >= lim[t][i & 1]) sc[t][i] = -CUDART_INF_F;
        }
        rise |= fmaxf(sc[t][0], sc[t][2]) > m[t][0] + kAttLazy || fmaxf(sc[t][1], sc[t][3]) > m[t][1] + kAttLazy;
      }
      if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = fmaxf(sc[t][i], sc[t][i + 2]);
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            x = fmaxf(x, m[t][i]);
            const float f = x == m[t][i] ? 1.f : pow2(m[t][i] - x);
            m[t][i] = x;
            l[t][i] *= f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              o[k][t][i] *= f;
              o[k][t][i + 2] *= f;
            }
          }
      }
      uint2 pf[NT][NP];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ref = m[t][i & 1] == -CUDART_INF_F ? 0.f : m[t][i & 1];
          w[i] = pow2(sc[t][i] - ref);
        }
        l[t][0] += w[0] + w[2];
        l[t][1] += w[1] + w[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] *= kAttPScale;
#pragma unroll
        for (int pc = 0; pc < NP; ++pc) {
          const uint32_t h0 = pack_half2(w[0], w[1]), h1 = pack_half2(w[2], w[3]);
          pf[t][pc] = make_uint2(transpose8x8(h0), transpose8x8(h1));
          if (pc + 1 < NP) {
            const float2 g0 = unpack_half2(h0), g1 = unpack_half2(h1);
            w[0] -= g0.x; w[1] -= g0.y; w[2] -= g1.x; w[3] -= g1.y;
          }
        }
      }
      // ---- values ----
      const float sv = (cur < 0 ? 0.f : vs_c) * kVFactor;
      float svc[NT][2];      // a column that sees nothing of the block takes nothing from it, not even a NaN
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) svc[t][i] = masked && t0 >= lim[t][i] ? 0.f : sv;
#pragma unroll
      for (int q = 0; q < VW; ++q) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = prepare_codes<FMT>(vr[r][q]);
          if (FMT == SPINDLEKV_PAGED_E4M3 && masked) w[r] = without_nan(w[r]);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          // elements 4 q + 2 x and + 1 of the lane's piece: tokens 2c, 2c+1 in one word, 2c+8, 2c+9 in the other
          const uint32_t lo = __byte_perm(w[0], w[1], x ? 0x7362 : 0x5140), hi = __byte_perm(w[2], w[3], x ? 0x7362 : 0x5140);
          const uint32_t a[4] = {codes_to_half2<FMT, 0>(lo), codes_to_half2<FMT, 1>(lo), codes_to_half2<FMT, 0>(hi), codes_to_half2<FMT, 1>(hi)};
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float acc[4];
            mma16816_first(acc, a, pf[t][0]);
            if constexpr (NP == 2) mma16816(acc, a, pf[t][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[2 * q + x][t][i] = fmaf(svc[t][i & 1], acc[i], o[2 * q + x][t][i]);
          }
        }
      }
      load_v(nxt);
      cur = nxt;
    }
    // ---- the warps' results meet ----
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d <= 16; d <<= 1) l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], d);
        if (g == 0) {
          sm_m[warp * COLS + 8 * t + 2 * c + i] = m[t][i];
          sm_l[warp * COLS + 8 * t + 2 * c + i] = l[t][i];
        }
      }
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)   // elements d, d + 1 of column 2c + i
          *reinterpret_cast<float2*>(so + (warp * COLS + 8 * t + 2 * c + i) * OP + g * (D / 8) + 2 * k) = make_float2(o[k][t][i], o[k][t][i + 2]);
    __syncthreads();
    const bool whole = b0 == 0 && b1 == nb;
    // what is left for the join: a unit that began in an earlier run is this run's first, one that begins here and goes on its last
    const int64_t slot = (int64_t)(2 * blockIdx.x + (b0 == 0 ? 1 : 0)) * kAttMaxCols;
    for (int i = tid; i < ncols * (D / 4); i += kAttThreads) {
      const int col = i / (D / 4), d = (i - col * (D / 4)) * 4;
      float top = -CUDART_INF_F;
#pragma unroll
      for (int w = 0; w < kAttWarps; ++w) top = fmaxf(top, sm_m[w * COLS + col]);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float den = 0.f;
#pragma unroll
      for (int w = 0; w < kAttWarps; ++w) {
        const float mw = sm_m[w * COLS + col];
        const float f = mw == top ? 1.f : pow2(mw - top);
        const float4 v = *reinterpret_cast<const float4*>(so + (w * COLS + col) * OP + d);
        sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y); sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
        den = fmaf(f, sm_l[w * COLS + col], den);
      }
      if (whole) {
        const int gi = (col0 + col) / p.n_rows, r = (col0 + col) - gi * p.n_rows;
        T* dst = reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + (int64_t)layer * p.out.sl + (int64_t)seq * p.out.ss +
                 (int64_t)(head * p.hn + gi) * p.out.sh + (int64_t)r * p.out.st + d;
        const bool none = den == 0.f;
        const float v[4] = {none ? 0.f : sum.x / den, none ? 0.f : sum.y / den, none ? 0.f : sum.z / den, none ? 0.f : sum.w / den};
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), e = __floats2bfloat162_rn(v[2], v[3]);
          *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&e));
        }
      } else {
        *reinterpret_cast<float4*>(p.part + (slot + col) * D + d) = sum;
        if (d == 0) p.stat[slot + col] = make_float2(top, den);
      }
    }
    __syncthreads();          // the shared memory is free for the next segment
    at += b1 - b0;
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Joins the parts of a unit: block (j, x) takes four columns of the unit that run j is the first to continue.  Four warps to a
// column, each with every fourth run; the order of the sums is the order of the runs.
constexpr int kJoinThreads = 512;

template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(AttendParams p, int cols_per_unit) {
  constexpr int E = D / 32;
  __shared__ float so[4][4][D];
  __shared__ float sden[4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int run = blockIdx.x, unit = p.lead[run];
  if (unit < 0 || (run > 0 && p.lead[run - 1] == unit)) return;
  int n = 1;                                 // parts: the run before, which the unit begins in, and those that continue it
  for (int r = run; r < (int)gridDim.x; r += kJoinThreads) n += __syncthreads_count(r + (int)threadIdx.x < (int)gridDim.x && p.lead[r + threadIdx.x] == unit);
  const int ls = unit / p.units_per, uh = unit - ls * p.units_per, head = uh / p.groups, group = uh - head * p.groups;
  const int layer = ls / p.table.n_seqs, seq = ls - layer * p.table.n_seqs;
  const int col0 = group * cols_per_unit, ncols = min(cols_per_unit, p.cols - col0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, which = warp & 3, turn = warp >> 2;
  const int col = blockIdx.y * 4 + which;
  const bool mine = col < ncols;
  auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * (run - 1) + 1 : 2 * (run - 1 + i)) * kAttMaxCols + col; };
  float num[E];
#pragma unroll
  for (int e = 0; e < E; ++e) num[e] = 0.f;
  if (mine) {
    float top = -CUDART_INF_F;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, p.stat[slot(i)].x);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float den = 0.f;
    for (int i0 = 0; i0 < n; i0 += 32) {
      float f = 0.f;
      if (i0 + lane < n) {
        const float2 st = p.stat[slot(i0 + lane)];
        f = st.x == top ? 1.f : pow2(st.x - top);
        den = fmaf(f, st.y, den);
      }
      const int last = min(32, n - i0);
#pragma unroll 4
      for (int k = turn; k < last; k += 4) {
        const float w = __shfl_sync(0xffffffffu, f, k);
        const float* src = p.part + slot(i0 + k) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 v = *reinterpret_cast<const float2*>(src + e);
          num[e] = fmaf(w, v.x, num[e]);
          num[e + 1] = fmaf(w, v.y, num[e + 1]);
        }
      }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
    if (turn == 0 && lane == 0) sden[which] = den;
#pragma unroll
    for (int e = 0; e < E; ++e) so[turn][which][lane * E + e] = num[e];
  }
  __syncthreads();
  if (!mine || turn) return;
  const int gi = (col0 + col) / p.n_rows, r = (col0 + col) - gi * p.n_rows;
  T* dst = reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + (int64_t)layer * p.out.sl + (int64_t)seq * p.out.ss +
           (int64_t)(head * p.hn + gi) * p.out.sh + (int64_t)r * p.out.st;
  const float den = sden[which];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = e * 32 + lane;
    const float sum = so[0][which][d] + so[1][which][d] + so[2][which][d] + so[3][which][d];
    dst[d] = T(den == 0.f ? 0.f : sum / den);
  }
}

// thread blocks that the device holds at once, by kernel
template <typename K>
static int resident_blocks(K kernel, size_t smem, int (&cache)[kMaxDevices], int dev) {
  if (!cache[dev]) {
    int sms = 0, per = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) return 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kAttThreads, smem) != cudaSuccess) return 0;
    cache[dev] = std::max(sms * per, 1);
  }
  return cache[dev];
}

static int column_tiles(int cols) { return cols <= 8 ? 1 : cols <= 16 ? 2 : 4; }

constexpr size_t kPartRows = (size_t)2 * kAttMaxRuns * kAttMaxCols;

size_t paged_workspace_bytes(const spindlekv_page_pool& pool) {
  return kHeaderBytes + kPartRows * (pool.head_dim * sizeof(float) + sizeof(float2)) + kAttMaxRuns * sizeof(int32_t);
}

template <typename T, int FMT, int D, int NT>
static spindlekv_status launch_attend(AttendParams& p, int max_len, cudaStream_t st) {
  static int resident[kMaxDevices] = {};
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  constexpr int NP = sizeof(T) == 4 ? 2 : 1, COLS = 8 * NT;
  const int n_ls = p.table.n_layers * p.table.n_seqs;
  auto kernel = paged_attend_kernel<T, FMT, D, NT>;
  const size_t fixed = (size_t)kAttWarps * COLS * (D + 4) * 4 + (size_t)NP * NT * (D / 16) * 32 * 8 + (size_t)COLS * 4 * (1 + 2 * kAttWarps) + 36 * 4;
  const size_t smem = align_up(fixed + (size_t)(n_ls + 1) * 4, 16);
  // the prefix sums of a usual batch do not change how many blocks fit; with those of thousands of sequences fewer may, and
  // the rest simply follow
  const int slots = resident_blocks(kernel, align_up(fixed + 1024, 16), resident, dev);
  if (slots <= 0) return SPINDLEKV_CUDA;
  // a run of fewer blocks than there are warps leaves warps idle
  const int64_t line = (int64_t)n_ls * p.units_per * ceil_div((int)std::min<int64_t>(max_len, (int64_t)p.table.max_pages * p.pool.ps), kPagedBlock);
  const int runs = (int)std::min<int64_t>(std::min(slots, kAttMaxRuns), std::max<int64_t>((line + kAttWarps - 1) / kAttWarps, 1));
  {
    LaunchScope ls(KC_PAGED_ATTEND, st);
    kernel<<<runs, kAttThreads, smem, st>>>(p);
  }
  if (cudaGetLastError() != cudaSuccess) return SPINDLEKV_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(runs, ceil_div(std::min(COLS, p.cols), 4));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_PAGED_ATTEND, st);
  return cudaLaunchKernelEx(&cfg, paged_join_kernel<T, D>, p, COLS) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

template <typename T, int FMT, int D>
static spindlekv_status launch_columns(AttendParams& p, int max_len, cudaStream_t st) {
  const int nt = column_tiles(p.cols);
  p.groups = ceil_div(p.cols, 8 * nt);
  p.units_per = p.pool.heads * p.groups;
  if (nt == 1) return launch_attend<T, FMT, D, 1>(p, max_len, st);
  if (nt == 2) return launch_attend<T, FMT, D, 2>(p, max_len, st);
  return launch_attend<T, FMT, D, 4>(p, max_len, st);
}

template <typename T>
static spindlekv_status launch_format(AttendParams& p, int format, int max_len, cudaStream_t st) {
  if (format == SPINDLEKV_PAGED_INT8)
    return p.pool.d == 64 ? launch_columns<T, SPINDLEKV_PAGED_INT8, 64>(p, max_len, st) : launch_columns<T, SPINDLEKV_PAGED_INT8, 128>(p, max_len, st);
  return p.pool.d == 64 ? launch_columns<T, SPINDLEKV_PAGED_E4M3, 64>(p, max_len, st) : launch_columns<T, SPINDLEKV_PAGED_E4M3, 128>(p, max_len, st);
}

spindlekv_status paged_attend_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, int n_q_heads, int n_rows, int max_len,
                                   float scale, const spindlekv_tensor& q, const spindlekv_tensor& out, void* ws, size_t ws_bytes,
                                   cudaStream_t st) {
  if (ws_bytes < paged_workspace_bytes(pool)) return SPINDLEKV_WORKSPACE_TOO_SMALL;
  AttendParams p;
  p.pool = make_pool(pool);
  p.table = make_table(table);
  p.q = make_view(q);
  p.out = make_view(out);
  p.per_shift = pool.page_size == 16 ? 0 : pool.page_size == 32 ? 1 : pool.page_size == 64 ? 2 : 3;
  p.hn = n_q_heads / pool.n_kv_heads;
  p.n_rows = n_rows;
  p.cols = p.hn * n_rows;
  p.scale = (scale == 0.f ? 1.f / sqrtf((float)pool.head_dim) : scale) * 1.44269504088896340736f;
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kHeaderBytes);
  p.stat = reinterpret_cast<float2*>(p.part + kPartRows * pool.head_dim);
  p.lead = reinterpret_cast<int32_t*>(p.stat + kPartRows);
  return q.dtype == SPINDLEKV_BF16 ? launch_format<__nv_bfloat16>(p, pool.format, max_len, st) : launch_format<float>(p, pool.format, max_len, st);
}

}  // namespace skv
