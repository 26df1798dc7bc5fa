// Rows -> codes of the 8-bit paged cache with the position's rotation on the way, and rotated queries beside them.
//
// Elements i and i + d/2 of a row at position t become  x_i c - x_(i+d/2) s  and  x_(i+d/2) c + x_i s  with the table's cosine and sine of (t, i): four
// products, a difference and a sum, each rounded to fp32 by itself, then the row's own type, as if the rotated row had been stored; codes are those of
// that row.  So the result is the same, bit for bit, as rotating first and appending then, without the rotated rows' way through memory.
//
// A lane holds four neighbouring elements of either half of a row, so that a pair never leaves its lane; 16 lanes (d = 128) or 8 (d = 64) make a row.
// Keys and values: a warp per (layer, sequence, KV head, block of 16 tokens, K or V), as in the append without rotation.  The warps of a thread block
// are the heads of the same tokens, whose table rows (512 bytes each, twice a bf16 row) then come from the first-level cache, into shared memory.  Queries: a warp takes 16
// tokens of eight heads and keeps a token's cosines and sines for all of them.
//
// Large calls are bound by memory and, at 28 % of the warps an SM can have, by its latency: 22615 bf16 tokens of 8 KV heads and 32 query heads, keys and queries
// given out, 120 us (556 MB, 4.6 TB/s, 71 % of the copy rate; one row at a time and table rows through registers 345); 16 layers x 8 x 1000 fp32 rows by list
// 52 us (3.2 TB/s; the row, its position's turn, the block's maximum and the codes follow one another).  One token of 96 sequences is latency: 6 us.
#include <algorithm>

#include "paged_rounding.cuh"

namespace skv {

struct RotateParams {
  Pool pool;
  Table table;
  View K, V, K_out, Q, Q_out;
  const int32_t *start, *idx, *first_pos;
  const float2* rope;        // [positions][d / 2]
  int positions;
  int idx_len, idx_seq, max_new, n_rows, n_blocks, q_heads, q_groups, q_chunks;
  int per_shift, page_shift;
  unsigned n_kv, n_items;    // warps of a unit: for keys and values, and in all
};

constexpr int kRotateThreads = 256, kRotateHeads = 8;      // query heads of a warp

// Four elements of either half of a row, as they lie in memory (plain loads: the rotated rows may take the rows' place)
template <typename T> struct Pairs;
template <> struct Pairs<float> {
  using Max = float2;        // the largest magnitude; and 0, or NaN if there is a NaN or an infinity
  __device__ __forceinline__ static Max none() { return make_float2(0.f, 0.f); }
  __device__ __forceinline__ static uint32_t bits(Max m) { return m.y == 0.f ? __float_as_uint(m.x) : 0x7FC00000u; }
  __device__ __forceinline__ void amax(Max& m) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m.x = fmaxf(m.x, fabsf(x[i]));
      m.y = fmaf(x[i], 0.f, m.y);
    }
  }
  float x[8];
  __device__ __forceinline__ void load(const float* p, int half) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + half);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void store(float* p, int half) const {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + half) = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
  }
  __device__ __forceinline__ void floats(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
  }
  __device__ __forceinline__ void set(const float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i];
  }
};
template <> struct Pairs<__nv_bfloat16> {
  using Max = __nv_bfloat162;          // the largest magnitudes, two at a time; NaN if there is one
  __device__ __forceinline__ static Max none() { return __floats2bfloat162_rn(0.f, 0.f); }
  __device__ __forceinline__ static uint32_t bits(Max m) {     // of the fp32 magnitude; a NaN is above all numbers
    const float2 f = __bfloat1622float2(m);
    return max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu);
  }
  __device__ __forceinline__ static __nv_bfloat162 two(uint32_t w) { return __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w)); }
  __device__ __forceinline__ void amax(Max& m) const { m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(two(w[0]), two(w[1])), __hmax2_nan(two(w[2]), two(w[3])))); }
  uint32_t w[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int half) {
    const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + half);
    w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p, int half) const {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(p + half) = make_uint2(w[2], w[3]);
  }
  __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0u; }
  __device__ __forceinline__ void floats(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = __uint_as_float(w[i] << 16);
      y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
};

// cosines and sines of four pairs at a position; NaN outside the table
__device__ __forceinline__ void load_turn(const RotateParams& p, long long pos, int col, int half, float2 (&t)[4]) {
  if (pos >= 0 && pos < p.positions) {
    const float4* at = reinterpret_cast<const float4*>(p.rope + pos * half + col);
    const float4 a = __ldg(at), b = __ldg(at + 1);
    t[0] = make_float2(a.x, a.y); t[1] = make_float2(a.z, a.w);
    t[2] = make_float2(b.x, b.y); t[3] = make_float2(b.z, b.w);
  } else {
    const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = make_float2(nan, nan);
  }
}
template <typename T>
__device__ __forceinline__ void turn(Pairs<T>& row, const float2 (&t)[4]) {
  float x[8];
  row.floats(x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[i], b = x[i + 4];
    x[i] = __fsub_rn(__fmul_rn(a, t[i].x), __fmul_rn(b, t[i].y));
    x[i + 4] = __fadd_rn(__fmul_rn(b, t[i].x), __fmul_rn(a, t[i].y));
  }
  row.set(x);
}

template <typename T, int D>
__device__ __forceinline__ void rotate_queries(const RotateParams& p, int layer, int s, unsigned item, long long first, int n_new) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, NI = kPagedBlock / RPI, HALF = D / 2;
  const int lane = threadIdx.x & 31, sub = lane / LPR, col = (lane % LPR) * 4;
  const int chunk = (int)(item / (unsigned)p.q_groups), group = (int)(item - (unsigned)chunk * p.q_groups);
  const int r0 = chunk * kPagedBlock, h0 = group * kRotateHeads, heads = min(kRotateHeads, p.q_heads - h0);
  if (r0 >= n_new) return;
  const T* from = reinterpret_cast<const T*>(p.Q.ptr) + (int64_t)layer * p.Q.sl + (int64_t)s * p.Q.ss + (int64_t)h0 * p.Q.sh + col;
  T* to = reinterpret_cast<T*>(const_cast<void*>(p.Q_out.ptr)) + (int64_t)layer * p.Q_out.sl + (int64_t)s * p.Q_out.ss + (int64_t)h0 * p.Q_out.sh + col;
#pragma unroll 1
  for (int i = 0; i < NI; ++i) {
    const int r = r0 + i * RPI + sub;
    if (r0 + i * RPI >= n_new) break;
    if (r >= n_new) continue;
    float2 t[4];
    load_turn(p, first + r, col, HALF, t);
    Pairs<T> x[kRotateHeads];
#pragma unroll
    for (int h = 0; h < kRotateHeads; ++h)
      if (h < heads) x[h].load(from + (int64_t)h * p.Q.sh + (int64_t)r * p.Q.st, HALF);
#pragma unroll
    for (int h = 0; h < kRotateHeads; ++h)
      if (h < heads) {
        turn(x[h], t);
        x[h].store(to + (int64_t)h * p.Q_out.sh + (int64_t)r * p.Q_out.st, HALF);
      }
  }
}

template <typename T> constexpr int kRotateBlocks = sizeof(T) == 2 ? 3 : 2;      // of an SM

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kRotateThreads, kRotateBlocks<T>) paged_append_rotated_kernel(const __grid_constant__ RotateParams p) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, NI = kPagedBlock / RPI, HALF = D / 2;
  __shared__ float2 shared_turns[kRotateThreads / 64 * kPagedBlock * HALF];      // keys are the even items
  const unsigned item = blockIdx.x * (kRotateThreads / 32) + (threadIdx.x >> 5);
  if (item >= p.n_items) return;
  const int lane = threadIdx.x & 31, u = blockIdx.y;
  const int layer = u / p.table.n_seqs, s = u - layer * p.table.n_seqs;
  const int start = p.start[u], from = p.first_pos ? p.first_pos[u] : p.idx ? 0 : start;      // (the lengths are asked for before the first is looked at)
  const int len = unit_len(p.table, p.pool, u);
  // A list's entries too, for a cache that begins here, which is what a list mostly fills (otherwise they are asked for again)
  const int rel = (int)(item / (2u * p.pool.heads)), rest = (int)(item - (unsigned)rel * 2u * p.pool.heads), head = rest >> 1;
  const int32_t* list = p.idx ? p.idx + ((int64_t)layer * p.pool.heads + head) * p.idx_len + (int64_t)s * p.idx_seq : nullptr;
  int listed = -1;
  if (p.idx && lane < kPagedBlock && rel * kPagedBlock + lane < p.max_new) listed = list[rel * kPagedBlock + lane];
  if (start < 0) return;
  const int end = (int)min((long long)len, (long long)start + p.max_new);
  if (start >= end) return;
  if (item >= p.n_kv) return rotate_queries<T, D>(p, layer, s, item - p.n_kv, from, min(end - start, p.n_rows));
  const bool is_v = (rest & 1) != 0;
  const int blk = start / kPagedBlock + rel, t0 = blk * kPagedBlock;
  if (t0 >= end) return;
  const int page = p.table.pages[(int64_t)u * p.table.max_pages + (t0 >> p.page_shift)];
  const bool in_pool = page >= 0 && page < p.pool.n_pages;
  const bool keeps = !is_v && p.K_out.ptr;
  const int64_t slab = (((int64_t)(in_pool ? page : 0) * p.pool.heads + head) << p.per_shift) + (blk & ((1 << p.per_shift) - 1));
  const int sub = lane / LPR, col = (lane % LPR) * 4;
  uint8_t* codes = (is_v ? p.pool.vc : p.pool.kc) + slab * (kPagedBlock * D) + col;
  float* scale = (is_v ? p.pool.vs : p.pool.ks) + slab;
  const View src = is_v ? p.V : p.K;
  const T* rows = reinterpret_cast<const T*>(src.ptr) + (int64_t)layer * src.sl + (int64_t)s * src.ss + (int64_t)head * src.sh + col;
  const int first = max(start - t0, 0), last = min(end - t0, kPagedBlock);       // new slots of the block: [first, last)
  int my_row = -1;
  if (lane >= first && lane < last) {
    const int i = t0 + lane - start;
    my_row = i;
    if (p.idx) my_row = start == 0 ? listed : list[i];
    if (my_row < 0 || my_row >= p.n_rows) my_row = -1;
  }
  // The rows' cosines and sines come into shared memory while the rows are on their way (into registers, two rows ahead: 79 us in place of 67 for keys,
  // their rotated rows and values of 22615 bf16 tokens)
  float2* turns = shared_turns + (threadIdx.x >> 6) * (kPagedBlock * HALF);      // of this warp, a key's: every second one
  int my_pos = -1;
  if (!is_v) {
    const long long at = (long long)from + my_row;
    if (my_row >= 0 && at >= 0 && at < p.positions) my_pos = (int)at;
#pragma unroll
    for (int c = 0; c < kPagedBlock * HALF / 64; ++c) {                          // 32 lanes x 16 bytes
      const int e = c * 64 + lane * 2, pos = __shfl_sync(0xffffffffu, my_pos, e / HALF);
      if (pos >= 0)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(turns + e)), "l"(p.rope + (int64_t)pos * HALF + e % HALF) : "memory");
    }
  }
  Pairs<T> x[NI];
  typename Pairs<T>::Max most = Pairs<T>::none();
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = __shfl_sync(0xffffffffu, my_row, i * RPI + sub);
    if (row >= 0) {
      x[i].load(rows + (int64_t)row * src.st, HALF);
    } else {
      x[i].zero();
    }
  }
  const float was = first > 0 && in_pool ? *scale : 0.f;       // (behind the rows, which need no page)
  if (!is_v) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + sub, row = __shfl_sync(0xffffffffu, my_row, slot), pos = __shfl_sync(0xffffffffu, my_pos, slot);
      if (row >= 0) {
        float2 t[4];
        const float4 a = *reinterpret_cast<const float4*>(turns + slot * HALF + col), b = *reinterpret_cast<const float4*>(turns + slot * HALF + col + 2);
        const float nan = __uint_as_float(0x7FC00000u);                          // outside the table
        t[0] = pos >= 0 ? make_float2(a.x, a.y) : make_float2(nan, nan);
        t[1] = pos >= 0 ? make_float2(a.z, a.w) : make_float2(nan, nan);
        t[2] = pos >= 0 ? make_float2(b.x, b.y) : make_float2(nan, nan);
        t[3] = pos >= 0 ? make_float2(b.z, b.w) : make_float2(nan, nan);
        turn(x[i], t);
        if (keeps)
          x[i].store(reinterpret_cast<T*>(const_cast<void*>(p.K_out.ptr)) + (int64_t)layer * p.K_out.sl + (int64_t)s * p.K_out.ss + (int64_t)head * p.K_out.sh +
                         (int64_t)row * p.K_out.st + col, HALF);
      }
    }
  }
  if (!in_pool) return;
#pragma unroll
  for (int i = 0; i < NI; ++i) x[i].amax(most);
  const uint32_t amax = __reduce_max_sync(0xffffffffu, Pairs<T>::bits(most));
  const bool poisoned = amax >= 0x7F800000u || !(was < __uint_as_float(0x7F800000u));
  const float sc = poisoned ? __uint_as_float(0x7FC00000u) : fmaxf(was, scale_of<FMT>(amax));
  __syncwarp();                              // every lane has read the old scale
  if (lane == 0) *scale = sc;
  const bool empty = poisoned || sc == 0.f;
  const float inv = empty ? 0.f : __fdiv_rn(1.f, sc);
  auto put = [&](int slot, uint2 c) {
    *reinterpret_cast<uint32_t*>(codes + slot * D) = c.x;
    *reinterpret_cast<uint32_t*>(codes + slot * D + HALF) = c.y;
  };
  if (first > 0 && sc != was) {              // earlier tokens of the block move to the larger scale (NaN: to codes of zero)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + sub;
      if (slot < first) {
        const uint2 old = make_uint2(*reinterpret_cast<const uint32_t*>(codes + slot * D), *reinterpret_cast<const uint32_t*>(codes + slot * D + HALF));
        put(slot, empty ? make_uint2(0, 0) : recode8<FMT>(old, was, sc));
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
      put(slot, empty ? make_uint2(0, 0) : encode8<FMT>(f, sc, inv, worst));
    }
  }
  if (FMT == SPINDLEKV_PAGED_INT8 && !empty && worst >= 0.5f * sc) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int slot = i * RPI + sub;
      if (slot >= first && slot < last) {
        float f[8];
        x[i].floats(f);
        put(slot, encode8_exactly(f, sc, inv));
      }
    }
  }
}

template <typename T, int FMT>
static void launch_rotated(const RotateParams& p, cudaStream_t st) {
  const dim3 grid((p.n_items + kRotateThreads / 32 - 1) / (kRotateThreads / 32), p.table.n_layers * p.table.n_seqs);
  LaunchScope ls(KC_PAGED_APPEND, st);
  if (p.pool.d == 64) paged_append_rotated_kernel<T, FMT, 64><<<grid, kRotateThreads, 0, st>>>(p);
  else paged_append_rotated_kernel<T, FMT, 128><<<grid, kRotateThreads, 0, st>>>(p);
}

spindlekv_status paged_append_rotated_impl(const spindlekv_page_pool& pool, const spindlekv_page_table& table, const int32_t* start, int max_new,
                                           const spindlekv_tensor& K, const spindlekv_tensor& V, int n_rows, const int32_t* idx, int idx_len, int idx_seq,
                                           const void* rope, int positions, const int32_t* first_pos, const spindlekv_tensor& K_out, int n_q_heads,
                                           const spindlekv_tensor& Q, const spindlekv_tensor& Q_out, cudaStream_t st) {
  RotateParams p;
  p.pool = make_pool(pool);
  p.table = make_table(table);
  p.K = make_view(K);
  p.V = make_view(V);
  p.K_out = make_view(K_out);
  p.Q = make_view(Q);
  p.Q_out = make_view(Q_out);
  p.start = start;
  p.idx = idx;
  p.first_pos = first_pos;
  p.rope = static_cast<const float2*>(rope);
  p.positions = positions;
  p.idx_len = idx_len;
  p.idx_seq = idx_seq;
  p.max_new = (int)std::min<int64_t>(max_new, (int64_t)table.max_pages * pool.page_size);      // no sequence can take more than its table row holds
  p.n_rows = n_rows;
  p.n_blocks = (int)(((int64_t)p.max_new + kPagedBlock - 2) / kPagedBlock) + 1;
  p.q_heads = n_q_heads;
  p.q_groups = ceil_div(n_q_heads, kRotateHeads);
  p.q_chunks = ceil_div(std::min(p.max_new, n_rows), kPagedBlock);
  const int64_t kv = 2ll * pool.n_kv_heads * p.n_blocks, items = kv + (int64_t)p.q_groups * p.q_chunks;
  if (items > 0x7FFFFFFF) return SPINDLEKV_UNSUPPORTED;
  p.n_kv = (unsigned)kv;
  p.n_items = (unsigned)items;
  p.page_shift = pool.page_size == 16 ? 4 : pool.page_size == 32 ? 5 : pool.page_size == 64 ? 6 : 7;
  p.per_shift = p.page_shift - 4;
  const bool bf = K.dtype == SPINDLEKV_BF16, i8 = pool.format == SPINDLEKV_PAGED_INT8;
  if (bf && i8) launch_rotated<__nv_bfloat16, SPINDLEKV_PAGED_INT8>(p, st);
  else if (bf) launch_rotated<__nv_bfloat16, SPINDLEKV_PAGED_E4M3>(p, st);
  else if (i8) launch_rotated<float, SPINDLEKV_PAGED_INT8>(p, st);
  else launch_rotated<float, SPINDLEKV_PAGED_E4M3>(p, st);
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
