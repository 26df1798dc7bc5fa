// Rows -> codes of the 8-bit paged cache, one scale per block of 16 tokens and head.
//
// One warp per (layer, sequence, KV head, block, K or V).  A lane holds 8 neighbouring elements of every second row of the block (d = 128;
// of every fourth for d = 64), so that a block's rows are in registers once: the largest magnitude (in which a NaN or an infinity shows), one warp
// reduction of its bits, the scale, and the codes leave from the same registers.  A block that begins with earlier tokens takes the larger of both scales; only if
// that grows are the earlier codes read and rounded again.
//
// int8: code = nearest integer to x / s, ties to even, on the exact quotient.  q0 = rint(x * (1/s)) is off by one at most;
// r = x - q0 s is exact in fp32 (one fused multiply-add: |r| <= s, and both x and q0 s are multiples of a unit within 24 bits of
// s), so comparing |r| with s/2 settles the rest without a division per element.  Rounding is the addition of 1.5 2^23, whose sum's low
// byte is the code; only a warp in which some |r| reaches s/2 (one in fifty) takes the second look.
// E4M3: s is a power of two, x / s exact, the conversion instruction rounds once.
//
// Bound by memory: 4 layers x 4 prompts of 6000 fp32 rows on average, 8 heads, 177 us (1.0 GB, 5.7 TB/s, 88% of a copy's rate); 16 layers x
// 1000 bf16 rows picked by a list 22.6 us (69%; 18.0 when the 67 MB of rows still lie in L2): list entry, then row, then the end of the warp.  One
// token for each of 96 sequences 3.8 us on the device, which is launch and latency; a call from Python takes 14, the host's.
#include <algorithm>

#include "paged_rounding.cuh"

namespace skv {

struct PagedAppendParams {
  Pool pool;
  Table table;
  View K, V;
  const int32_t* start;
  const int32_t* idx;
  int idx_len, idx_seq;
  int max_new, n_rows, n_blocks;
  int per_shift, page_shift;   // log2 of the blocks and of the tokens of a page
  unsigned n_items;
};

// 8 elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  using Max = __nv_bfloat162;
  __device__ __forceinline__ static Max none() { return __floats2bfloat162_rn(0.f, 0.f); }
  __device__ __forceinline__ static uint32_t bits(Max m) {     // of the fp32 magnitude; a NaN is above all numbers
    const float2 f = __bfloat1622float2(m);
    return max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu);
  }
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  // the largest magnitude, two at a time; NaN if there is one
  __device__ __forceinline__ static __nv_bfloat162 pair(uint32_t w) { return __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w)); }
  __device__ __forceinline__ void amax(__nv_bfloat162& m) const {
    m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(pair(v.x), pair(v.y)), __hmax2_nan(pair(v.z), pair(v.w))));
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
  using Max = float2;
  __device__ __forceinline__ static Max none() { return make_float2(0.f, 0.f); }
  __device__ __forceinline__ static uint32_t bits(Max m) { return m.y == 0.f ? __float_as_uint(m.x) : 0x7FC00000u; }
  uint4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const uint4*>(p));
    b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
  // .x: the largest magnitude; .y: 0, or NaN if there is a NaN or an infinity
  __device__ __forceinline__ void amax(float2& m) const {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m.x = fmaxf(m.x, fabsf(__uint_as_float(w[i])));
      m.y = fmaf(__uint_as_float(w[i]), 0.f, m.y);
    }
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  }
};

constexpr int kAppendThreads = 256;

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(PagedAppendParams p) {
  constexpr int LPR = D / 8;            // lanes of a row
  constexpr int RPI = 32 / LPR;         // rows side by side in a warp
  constexpr int NI = kPagedBlock / RPI;
  const unsigned item = blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);   // of this unit: (head, block, K or V)
  if (item >= p.n_items) return;
  const int lane = threadIdx.x & 31;
  const bool is_v = (item & 1) != 0;
  const int head = (int)((item >> 1) / (unsigned)p.n_blocks), rel = (int)(item >> 1) - head * p.n_blocks, u = blockIdx.y;
  const int layer = u / p.table.n_seqs, s = u - layer * p.table.n_seqs;
  const int start = p.start[u];
  if (start < 0) return;
  const int end = (int)min((long long)unit_len(p.table, p.pool, u), (long long)start + p.max_new);
  const int blk = start / kPagedBlock + rel;
  const int t0 = blk * kPagedBlock;
  if (t0 >= end || start >= end) return;
  const int page = p.table.pages[(int64_t)u * p.table.max_pages + (t0 >> p.page_shift)];
  if (page < 0 || page >= p.pool.n_pages) return;
  const int64_t slab = (((int64_t)page * p.pool.heads + head) << p.per_shift) + (blk & ((1 << p.per_shift) - 1));   // index of the block
  uint8_t* codes = (is_v ? p.pool.vc : p.pool.kc) + slab * (kPagedBlock * D);
  float* scale = (is_v ? p.pool.vs : p.pool.ks) + slab;
  const View src = is_v ? p.V : p.K;
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
  typename Raw8<T>::Max most = Raw8<T>::none();
  const float was = first > 0 ? *scale : 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = __shfl_sync(0xffffffffu, my_row, i * RPI + sub);
    if (row >= 0) x[i].load(rows + (int64_t)row * src.st + col);
    else x[i].zero();
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) x[i].amax(most);
  const uint32_t amax = __reduce_max_sync(0xffffffffu, Raw8<T>::bits(most));
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
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int slot = i * RPI + sub;
    if (slot >= first && slot < last) {
      float f[8];
      x[i].floats(f);
      *reinterpret_cast<uint2*>(codes + slot * D + col) = empty ? make_uint2(0, 0) : encode8<FMT>(f, sc, inv, worst);
    }
  }
  if (FMT == SPINDLEKV_PAGED_INT8 && !empty && worst >= 0.5f * sc) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + sub;
      if (slot >= first && slot < last) {
        float f[8];
        x[i].floats(f);
        *reinterpret_cast<uint2*>(codes + slot * D + col) = encode8_exactly(f, sc, inv);
      }
    }
  }
}

template <typename T, int FMT>
static void launch_append(const PagedAppendParams& p, cudaStream_t st) {
  const dim3 grid((p.n_items + kAppendThreads / 32 - 1) / (kAppendThreads / 32), p.table.n_layers * p.table.n_seqs);   // at most 8192 units
  LaunchScope ls(KC_PAGED_APPEND, st);
  if (p.pool.d == 64) paged_append_kernel<T, FMT, 64><<<grid, kAppendThreads, 0, st>>>(p);
  else paged_append_kernel<T, FMT, 128><<<grid, kAppendThreads, 0, st>>>(p);
}

spindlekv_status paged_append_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, const int32_t* start, int max_new,
                                   const spindlekv_tensor& K, const spindlekv_tensor& V, int n_rows, const int32_t* idx, int idx_len,
                                   int idx_seq, cudaStream_t st) {
  PagedAppendParams p;
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
  const int64_t items = 2ll * pool.n_kv_heads * p.n_blocks;
  if (items > 0x7FFFFFFF) return SPINDLEKV_UNSUPPORTED;
  p.n_items = (unsigned)items;
  p.page_shift = pool.page_size == 16 ? 4 : pool.page_size == 32 ? 5 : pool.page_size == 64 ? 6 : 7;
  p.per_shift = p.page_shift - 4;
  const bool bf = K.dtype == SPINDLEKV_BF16, i8 = pool.format == SPINDLEKV_PAGED_INT8;
  if (bf && i8) launch_append<__nv_bfloat16, SPINDLEKV_PAGED_INT8>(p, st);
  else if (bf) launch_append<__nv_bfloat16, SPINDLEKV_PAGED_E4M3>(p, st);
  else if (i8) launch_append<float, SPINDLEKV_PAGED_INT8>(p, st);
  else launch_append<float, SPINDLEKV_PAGED_E4M3>(p, st);
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
