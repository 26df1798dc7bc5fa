// Rows -> codes of the 8-bit paged cache, one scale per block of 16 tokens and head.
//
// One warp per (layer, sequence, KV head, block, K or V).  A lane holds 8 neighbouring elements of every (D/8)th ... row of
// the block, so that a block's rows are in registers once: the largest magnitude is an integer maximum of the magnitudes'
// bits (a NaN is larger than an infinity, an infinity larger than any number, so either shows), one warp reduction gives the
// scale, and the codes leave from the same registers.  A block that begins with earlier tokens takes the larger of both scales; only if
// that grows are the earlier codes read and rounded again.
//
// int8: code = nearest integer to x / s, ties to even, on the exact quotient.  q0 = rint(x * (1/s)) is off by one at most;
// r = x - q0 s is exact in fp32 (one fused multiply-add: |r| <= s, and both x and q0 s are multiples of a unit within 24 bits of
// s), so comparing |r| with s/2 settles the rest without a division per element.
// E4M3: s is a power of two, x / s exact, the conversion instruction rounds once.
#include <algorithm>

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "paged.cuh"

namespace skv {

struct AppendParams {
  Pool pool;
  Table table;
  View K, V;
  const int32_t* start;
  const int32_t* idx;
  int idx_len, idx_seq;
  int max_new, n_rows, n_blocks;
  long long n_items;
};

template <int FMT>
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  if (amax_bits == 0) return 0.f;
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    return fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 127.f), 1.17549435e-38f);
  } else {
    // amax = 1.m 2^(e-127): least k with 1.m 2^(e-127) <= 1.75 2^(8+k)
    const int e = (int)(amax_bits >> 23);
    const int k = max(e - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), -126);
    return __uint_as_float((uint32_t)(k + 127) << 23);
  }
}

// inv: 1 / s (exact for E4M3)
__device__ __forceinline__ int round_int8(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), half = 0.5f * s;
  const float up = r > 0.f ? 1.f : -1.f;
  const bool odd = ((int)q & 1) != 0;
  if (fabsf(r) > half || (fabsf(r) == half && odd)) q += up;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

template <int FMT>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float s, float inv) {
  uint32_t w[2] = {0u, 0u};
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(round_int8(x[i], s, inv) & 0xFF) << (8 * (i & 3));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      w[i >> 1] |= two << (16 * (i & 1));
    }
  }
  return make_uint2(w[0], w[1]);
}

// codes at scale `was` -> codes at the larger scale `s`
template <int FMT>
__device__ __forceinline__ uint2 recode8(uint2 c, float was, float s) {
  const uint32_t in[2] = {c.x, c.y};
  uint32_t w[2] = {0u, 0u};
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    // code * was has up to 31 bits: in double, where the product is exact and the quotient's rounding cannot reach a tie
    // that the exact quotient does not have
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int v = (int)(int8_t)(in[i >> 2] >> (8 * (i & 3)));
      const int q = (int)rint((double)v * (double)was / (double)s);
      w[i >> 2] |= (uint32_t)(q & 0xFF) << (8 * (i & 3));
    }
  } else {
    const float f = __fdiv_rn(was, s);   // a power of two; what falls below the smallest fp32 number falls below E4M3's too
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(in[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
      const float2 v = __half22float2(__half2(h));
      const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(v.x * f, v.y * f), __NV_SATFINITE, __NV_E4M3);
      w[i >> 1] |= two << (16 * (i & 1));
    }
  }
  return make_uint2(w[0], w[1]);
}

// 8 elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint32_t amax() const {   // bits of the largest magnitude, as fp32
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(m & 0xFFFF0000u, m << 16);
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <> struct Raw8<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const uint4*>(p));
    b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint32_t amax() const {
    const uint32_t k = 0x7FFFFFFFu;
    return max(max(max(a.x & k, a.y & k), max(a.z & k, a.w & k)), max(max(b.x & k, b.y & k), max(b.z & k, b.w & k)));
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  }
};

constexpr int kAppendThreads = 256;

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(AppendParams p) {
  constexpr int LPR = D / 8;            // lanes of a row
  constexpr int RPI = 32 / LPR;         // rows side by side in a warp
  constexpr int NI = kPagedBlock / RPI;
  const long long item = (long long)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
  if (item >= p.n_items) return;
  const int lane = threadIdx.x & 31;
  const bool is_v = (item & 1) != 0;
  long long rest = item >> 1;
  const int rel = (int)(rest % p.n_blocks);
  rest /= p.n_blocks;
  const int head = (int)(rest % p.pool.heads);
  const int u = (int)(rest / p.pool.heads);
  const int layer = u / p.table.n_seqs, s = u - layer * p.table.n_seqs;
  const int start = p.start[u];
  if (start < 0) return;
  const int end = (int)min((long long)unit_len(p.table, p.pool, u), (long long)start + p.max_new);
  const int blk = start / kPagedBlock + rel;
  const int t0 = blk * kPagedBlock;
  if (t0 >= end || start >= end) return;
  const int page = p.table.pages[(int64_t)u * p.table.max_pages + t0 / p.pool.ps];
  if (page < 0 || page >= p.pool.n_pages) return;
  const int per = p.pool.per_page();
  const int64_t slab = ((int64_t)page * p.pool.heads + head) * per + blk % per;   // index of the block
  uint8_t* codes = (is_v ? p.pool.vc : p.pool.kc) + slab * (kPagedBlock * D);
  float* scale = (is_v ? p.pool.vs : p.pool.ks) + slab;
  const View& src = is_v ? p.V : p.K;
  const T* rows = reinterpret_cast<const T*>(src.ptr) + (int64_t)layer * src.sl + (int64_t)s * src.ss + (int64_t)head * src.sh;
  const int first = max(start - t0, 0), last = min(end - t0, kPagedBlock);   // new slots of the block: [first, last)
  // row of this lane's slot (lanes 0..15), handed to the lanes that load it
  int my_row = -1;
  if (lane >= first && lane < last) {
    const int i = t0 + lane - start;
    my_row = i;
    if (p.idx) my_row = p.idx[((int64_t)layer * p.pool.heads + head) * p.idx_len + (int64_t)s * p.idx_seq + i];
    if (my_row < 0 || my_row >= p.n_rows) my_row = -1;
  }
  const int sub = lane / LPR, col = (lane % LPR) * 8;
  Raw8<T> x[NI];
  uint32_t amax = 0;
  const float was = first > 0 ? *scale : 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = __shfl_sync(0xffffffffu, my_row, i * RPI + sub);
    if (row >= 0) x[i].load(rows + (int64_t)row * src.st + col);
    else x[i].zero();
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) amax = max(amax, x[i].amax());
  amax = __reduce_max_sync(0xffffffffu, amax);
  const bool poisoned = amax >= 0x7F800000u || !(was < __uint_as_float(0x7F800000u));
  const float sc = poisoned ? __uint_as_float(0x7FC00000u) : fmaxf(was, scale_of<FMT>(amax));
  __syncwarp();                          // every lane has read the old scale
  if (lane == 0) *scale = sc;
  const bool empty = poisoned || sc == 0.f;
  const float inv = empty ? 0.f : __fdiv_rn(1.f, sc);
  if (first > 0 && sc != was) {   // earlier tokens of the block move to the larger scale (NaN: to codes of zero)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + sub;
      if (slot < first) {
        uint2* at = reinterpret_cast<uint2*>(codes + slot * D + col);
        *at = empty ? make_uint2(0, 0) : recode8<FMT>(*at, was, sc);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int slot = i * RPI + sub;
    if (slot >= first && slot < last) {
      float f[8];
      x[i].floats(f);
      *reinterpret_cast<uint2*>(codes + slot * D + col) = empty ? make_uint2(0, 0) : encode8<FMT>(f, sc, inv);
    }
  }
}

template <typename T, int FMT>
static void launch_append(const AppendParams& p, cudaStream_t st) {
  const unsigned grid = (unsigned)((p.n_items + kAppendThreads / 32 - 1) / (kAppendThreads / 32));
  LaunchScope ls(KC_PAGED_APPEND, st);
  if (p.pool.d == 64) paged_append_kernel<T, FMT, 64><<<grid, kAppendThreads, 0, st>>>(p);
  else paged_append_kernel<T, FMT, 128><<<grid, kAppendThreads, 0, st>>>(p);
}

spindlekv_status paged_append_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, const int32_t* start, int max_new,
                                   const spindlekv_tensor& K, const spindlekv_tensor& V, int n_rows, const int32_t* idx, int idx_len,
                                   int idx_seq, cudaStream_t st) {
  AppendParams p;
  p.pool = make_pool(pool);
  p.table = make_table(table);
  p.K = make_view(K);
  p.V = make_view(V);
  p.start = start;
  p.idx = idx;
  p.idx_len = idx_len;
  p.idx_seq = idx_seq;
  // no sequence can take more than its table row holds
  p.max_new = (int)std::min<int64_t>(max_new, (int64_t)table.max_pages * pool.page_size);
  p.n_rows = n_rows;
  p.n_blocks = (int)(((int64_t)p.max_new + kPagedBlock - 2) / kPagedBlock) + 1;   // a run that begins inside a block touches one more
  p.n_items = 2ll * table.n_layers * table.n_seqs * pool.n_kv_heads * p.n_blocks;
  if (p.n_items / (kAppendThreads / 32) >= 0x7FFFFFFFll) return SPINDLEKV_UNSUPPORTED;
  const bool bf = K.dtype == SPINDLEKV_BF16, i8 = pool.format == SPINDLEKV_PAGED_INT8;
  if (bf && i8) launch_append<__nv_bfloat16, SPINDLEKV_PAGED_INT8>(p, st);
  else if (bf) launch_append<__nv_bfloat16, SPINDLEKV_PAGED_E4M3>(p, st);
  else if (i8) launch_append<float, SPINDLEKV_PAGED_INT8>(p, st);
  else launch_append<float, SPINDLEKV_PAGED_E4M3>(p, st);
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
