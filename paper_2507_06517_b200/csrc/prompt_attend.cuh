// What the kernels of the prompt's attention share: parameters, lengths, the list of work items, the join of split keys.
#pragma once

#include <math.h>
#include <math_constants.h>

#include <type_traits>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace skv {

constexpr int kPromptRows = 128;          // rows of a tile: (position, query head of the group), heads next to one another
constexpr int kPromptMaxItems = 4096;     // items of a block, at most: one bit each for those that are done again
constexpr int kPromptHdrDone = 16;        // words 16, 17 of the status block: blocks that have arrived
constexpr float kPromptLazy = 8.f;        // how far a score may exceed the running reference, in powers of two

struct PromptParams {
  Batch keys, rows;
  View q, k, v, out;         // (q, k, v as the caller has them)
  int heads, hn;             // KV heads, query heads of each
  int pt;                    // positions of a row tile: 128 / hn, rounded down
  int per_item;              // positions of an item
  int max_blocks;            // items of the longest sequence, a head and a split
  int splits;                // parts that the keys of an item are cut into
  float scale;               // softmax scale * log2(e)
  float* lse;                // [layer][query head][T], or null
  float* part;               // [splits][layer][T][query head][d] and
  float2* stat;              // [splits][layer][T][query head]: O, reference and sum of a part
  float* kept;               // bf16: sums of long keys (keep_sums), kPromptKept<d> numbers for each block
  uint32_t* hdr;
  long long wait_cycles;
  int withhold;              // for tests: the block that does not ask for its first keys; -1: none
};

// rows of (layer, seq): the first one's number in a packed tensor (0 in a padded one) and how many there are, never outside the tensor
struct Span { int base, len; };
__device__ __forceinline__ Span span_of(const Batch& b, int layer, int s) {
  if (b.cu) {
    const int base = min(max(b.cu[s], 0), b.total_len);
    return {base, max(0, min(min(b.cu[s + 1], b.total_len) - base, b.max_len))};
  }
  return {0, b.ll ? max(0, min(b.ll[layer * b.n_seqs + s], b.max_len)) : b.max_len};
}
// keys that row i of n_r sees among n_k
__device__ __forceinline__ int seen_by(int i, int n_r, int n_k) { return max(0, n_k - n_r + i + 1); }

// One item: `per_item` positions of a (layer, seq) and KV head, and a part of the keys that they see.
struct PromptItem {
  int ls, head, blk, split;   // ls -1: no more of them
  int n_r, n_k, base_r, base_k;
  int careful, number, pad[2];
};

// Items in falling order of their block's number, which is nearly that of their work: all sequences' last positions first.  A warp finds item
// `i` by the number of blocks with a number of b or more, which falls with b.  What the item before it showed (its number's share of the items, and the
// sequences ahead of it) is kept, so that a call with many sequences does not count them for every item (32 layers x 32 sequences of 50 to 200 tokens,
// 32 / 8 heads: 0.82 ms in place of 2.9).
struct PromptList {
  Span rows, keys;            // of (layer, seq) lane, where there are up to 32
  int n_ls, all;
  int blk, from, to;          // items' numbers [from, to) are those of block number blk
  int group, before;          // the 32 (layer, seq) that held the last item, and how many of these blocks lie ahead of them
  __device__ __forceinline__ static Span span_at(const Batch& b, int ls) {
    const int layer = ls / b.n_seqs;
    return span_of(b, layer, ls - layer * b.n_seqs);
  }
  __device__ __forceinline__ int blocks_of(const PromptParams& p, int ls) const {       // with up to 32: of this lane's
    if (n_ls <= 32) return (rows.len + p.per_item - 1) / p.per_item;
    return ls < n_ls ? (span_at(p.rows, ls).len + p.per_item - 1) / p.per_item : 0;
  }
  __device__ __forceinline__ int count(const PromptParams& p, int b) const {            // blocks with the number b or a larger one
    int n = 0;
#pragma unroll 4
    for (int ls = threadIdx.x & 31; ls < (n_ls + 31) / 32 * 32; ls += 32) n += max(blocks_of(p, ls) - b, 0);
    return __reduce_add_sync(0xffffffffu, n);
  }
  __device__ __forceinline__ PromptList(const PromptParams& p) {
    const int lane = threadIdx.x & 31;
    n_ls = p.rows.n_layers * p.rows.n_seqs;
    rows = keys = {0, 0};
    if (n_ls <= 32 && lane < n_ls) {
      rows = span_at(p.rows, lane);
      keys = span_at(p.keys, lane);
    }
    all = count(p, 0);
    blk = from = to = group = before = 0;
  }
  // The block's k-th item, or one with ls = -1; every other round goes backwards, so that no block gets the longest of all rounds
  __device__ __forceinline__ PromptItem item(const PromptParams& p, int k) {
    const int lane = threadIdx.x & 31;
    PromptItem it = {};
    it.ls = -1;
    const long long i = (long long)k * gridDim.x + ((k & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    const int per = p.heads * p.splits;
    if (i >= (long long)all * per) return it;
    const int q = i <= 0x7FFFFFFF ? (int)i / per : (int)(i / per), inner = (int)(i - (long long)q * per);
    if (q < from || q >= to) {
      int lo = 0, hi = p.max_blocks - 1;                   // the largest b with more than q blocks of that number or more
      from = 0;
      to = all;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1, c = count(p, mid);
        if (c > q) { lo = mid; to = c; }
        else { hi = mid - 1; from = c; }
      }
      blk = lo;
      group = before = 0;
    }
    if (q - from < before) group = before = 0;
    int rank = q - from - before, found = -1;
    for (; group < n_ls; group += 32) {
      uint32_t has = __ballot_sync(0xffffffffu, blocks_of(p, group + lane) > blk);
      if (rank >= __popc(has)) {
        rank -= __popc(has);
        before += __popc(has);
        continue;
      }
      while (rank-- > 0) has &= has - 1;
      found = group + __ffs(has) - 1;
      break;
    }
    if (found < 0) return it;
    it.ls = found;
    it.blk = blk;
    it.head = inner / p.splits;
    it.split = inner - it.head * p.splits;
    if (n_ls <= 32) {
      it.n_r = __shfl_sync(0xffffffffu, rows.len, found);
      it.n_k = __shfl_sync(0xffffffffu, keys.len, found);
      it.base_r = __shfl_sync(0xffffffffu, rows.base, found);
      it.base_k = __shfl_sync(0xffffffffu, keys.base, found);
    } else {
      const Span r = span_at(p.rows, found), n = span_at(p.keys, found);
      it.n_r = r.len;
      it.n_k = n.len;
      it.base_r = r.base;
      it.base_k = n.base;
    }
    it.number = k;
    return it;
  }
};

// Tiles of KT keys that an item's row tiles have: [first, first + count[w]) for row tile w, of which the last ones, from `even[w]` of them on, hide keys
// from some row
template <int NT, int KT>
struct PromptTiles {
  int first, count[NT], even[NT], most;
  __device__ __forceinline__ PromptTiles(const PromptParams& p, const PromptItem& it) {
    int n[NT], all = 0;
#pragma unroll
    for (int w = 0; w < NT; ++w) {
      const int from = it.blk * p.per_item + w * p.pt, last = min(from + p.pt, it.n_r) - 1;
      n[w] = last >= from ? (seen_by(last, it.n_r, it.n_k) + KT - 1) / KT : 0;
      even[w] = last >= from ? seen_by(from, it.n_r, it.n_k) / KT : 0;
      all = max(all, n[w]);
    }
    first = (int)((long long)all * it.split / p.splits);
    const int end = (int)((long long)all * (it.split + 1) / p.splits);
    most = 0;
#pragma unroll
    for (int w = 0; w < NT; ++w) {
      count[w] = max(0, min(end, n[w]) - first);
      even[w] = max(0, min(min(end, even[w]) - first, count[w]));
      most = max(most, count[w]);
    }
  }
};

// element of (layer, seq, query head, position) of a tensor of rows
__device__ __forceinline__ int64_t row_offset(const View& v, const Batch& b, int layer, int s, int base, int head, int pos) {
  return (int64_t)layer * v.sl + (b.cu ? 0 : (int64_t)s * v.ss) + (int64_t)head * v.sh + (int64_t)(base + pos) * v.st;
}
// (layer, T column, query head) as one number, and its place in lse
__device__ __forceinline__ int column_of(const PromptParams& p, int s, int base, int pos) { return p.rows.cu ? base + pos : s * p.rows.max_len + pos; }
__device__ __forceinline__ int64_t row_number(const PromptParams& p, int layer, int s, int base, int head, int pos) {
  return ((int64_t)layer * p.rows.total_len + column_of(p, s, base, pos)) * (p.heads * p.hn) + head;
}
__device__ __forceinline__ void put_lse(const PromptParams& p, int layer, int col, int head, float m, float l) {
  if (p.lse) p.lse[((int64_t)layer * (p.heads * p.hn) + head) * p.rows.total_len + col] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * 0.69314718055994530942f;
}

// The status word.  Blocks are counted as they begin, which nobody waits for; the last one writes OK.  A block that fails says so to the last one to begin,
// or, if that has been, in the status word itself: the word is written before the count starts again from zero.
__device__ __forceinline__ void prompt_begins(const PromptParams& p) {        // one thread
  unsigned long long* word = reinterpret_cast<unsigned long long*>(p.hdr + kPromptHdrDone);
  const unsigned long long was = count_arrival<24>(word);
  if ((int)(was & 0xFFFFu) + 1 != (int)gridDim.x) return;
  // (a failure that comes in now changes the word, and is seen)
  for (unsigned long long now = was + 1;;) {
    *reinterpret_cast<volatile uint32_t*>(p.hdr + kHdrStatus) = now >> 16 & 1u ? SPINDLEKV_TIMEOUT : SPINDLEKV_OK;
    __threadfence();
    const unsigned long long seen = atomicCAS(word, now, kNoArrivals<24>);
    if (seen == now) return;
    now = seen;
  }
}
__device__ __forceinline__ void prompt_failed(const PromptParams& p) {        // one thread, after its block has been counted
  unsigned long long* word = reinterpret_cast<unsigned long long*>(p.hdr + kPromptHdrDone);
  for (unsigned long long now = *reinterpret_cast<volatile unsigned long long*>(word); now >> 24 == kNoArrivals<24> >> 24 && (now & 0xFFFFu);) {
    const unsigned long long seen = atomicCAS(word, now, now | 1ull << 16);
    if (seen == now) return;
    now = seen;
  }
  __threadfence();
  *reinterpret_cast<volatile uint32_t*>(p.hdr + kHdrStatus) = SPINDLEKV_TIMEOUT;
}

// a x b + c of two numbers at a time
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  unsigned long long x, y, z, r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
  asm("mov.b64 %0, {%1, %2};" : "=l"(z) : "f"(c.x), "f"(c.y));
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  float2 o;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
  return o;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  unsigned long long x, y, r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  float2 o;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
  return o;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The largest of three (a NaN only if all are: the weights show it)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// NP x 16 bytes of a warp's 32 rows, a row in each lane, to memory: through shared memory, so that a store covers whole pieces of few rows.
// `row`: where a lane's row lies behind `base`, in bytes; negative: nowhere
template <int NP>
__device__ __forceinline__ void put_rows(uint8_t* stage, const uint4 (&piece)[NP], uint8_t* base, int64_t row) {
  constexpr int kRows = 32 / NP;         // of a store
  const int lane = threadIdx.x & 31;
  // (rows that share banks take different places for a piece)
  auto place = [](int r, int i) { return r * (NP * 16) + ((i ^ (NP == 8 ? r : r >> 1) & (NP - 1)) << 4); };
#pragma unroll
  for (int i = 0; i < NP; ++i) *reinterpret_cast<uint4*>(stage + place(lane, i)) = piece[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int r = i * kRows + lane / NP;
    const int64_t at = __shfl_sync(0xffffffffu, row, r);
    const uint4 x = *reinterpret_cast<const uint4*>(stage + place(r, lane % NP));
    if (at >= 0) *reinterpret_cast<uint4*>(base + at + (lane % NP) * 16) = x;
  }
  __syncwarp();
}

// What a row's tiles that hide keys from some row give to the elements [c0, c1) of O in tensor memory (`o_tmem`: this warp's lanes), key by key: the keys
// [from, to) of a row, none for to <= from.  `begins`: O holds nothing yet.  Rare, and so a function of its own that costs the others no registers
template <typename T, int D>
__device__ __noinline__ void add_by_hand(const PromptParams& p, const PromptItem& it, uint32_t o_tmem, int c0, int c1, bool begins, int head, int pos, int from, int to, float ref) {
  const int layer = it.ls / p.rows.n_seqs, seq = it.ls - layer * p.rows.n_seqs;
  const T* q = reinterpret_cast<const T*>(p.q.ptr) + row_offset(p.q, p.rows, layer, seq, it.base_r, head, pos);
#pragma unroll 1
  for (int c = c0; c < c1; c += 32) {
    uint32_t o[32];
    __syncwarp();
    ptx::tmem_ld_32x32_sync(o_tmem + c, o);
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = begins ? 0.f : __uint_as_float(o[i]);
#pragma unroll 1
    for (int j = from; j < to; ++j) {
      const T* k = reinterpret_cast<const T*>(p.k.ptr) + row_offset(p.k, p.keys, layer, seq, it.base_k, it.head, j);
      const T* v = reinterpret_cast<const T*>(p.v.ptr) + row_offset(p.v, p.keys, layer, seq, it.base_k, it.head, j) + c;
      float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int d = 0; d < D; d += 8) {
        float a[8], b[8];
        load8(q + d, a);
        load8(k + d, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = fmaf(a[i], b[i], s[i]);
      }
      const float w = pow2(fmaf(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])), p.scale, -ref));
#pragma unroll
      for (int d = 0; d < 32; d += 8) {
        float b[8];
        load8(v + d, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[d + i] = fmaf(w, b[i], x[d + i]);
      }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(x[i]);
    ptx::tmem_st_32x32(o_tmem + c, o);
  }
  ptx::tmem_st_wait();
}

// Joins the parts of a row: a warp for each (layer, column, query head).  Latency bounds it: parts one after the other took 6 us more a call (18 parts).
template <typename T, int D>
__global__ void __launch_bounds__(256) prompt_join_kernel(const __grid_constant__ PromptParams p) {
  constexpr int E = D / 32;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int hq = p.heads * p.hn, lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)p.rows.n_layers * p.rows.total_len * hq, number = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (number >= rows) return;
  const int64_t lt = number / hq;
  const int head = (int)(number - lt * hq), layer = (int)(lt / p.rows.total_len), col = (int)(lt - (int64_t)layer * p.rows.total_len);
  int seq, pos;
  if (p.rows.cu) {                       // the sequence that holds the column
    int lo = 0, hi = p.rows.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.rows.cu[mid + 1] > col) hi = mid; else lo = mid + 1;
    }
    seq = lo;
  } else {
    seq = col / p.rows.max_len;
  }
  const Span r = span_of(p.rows, layer, seq);
  pos = p.rows.cu ? col - r.base : col - seq * p.rows.max_len;
  if (pos < 0 || pos >= r.len) return;
  // Eight parts at a time, asked for ahead of what weighs them (a part without keys has the sum 0 and may hold anything)
  constexpr int kAhead = 8;
  using Piece = std::conditional_t<E == 4, float4, float2>;
  const float* mine = p.part + number * D + lane * E;
  Piece x[kAhead];
  auto ask = [&](int z) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = *reinterpret_cast<const Piece*>(mine + (int64_t)min(z + i, p.splits - 1) * rows * D);
  };
  ask(0);
  float top = -CUDART_INF_F, den = 0.f, num[E];
#pragma unroll
  for (int e = 0; e < E; ++e) num[e] = 0.f;
  for (int z0 = 0; z0 < p.splits; z0 += 32) {
    const float2 st = z0 + lane < p.splits ? p.stat[(int64_t)(z0 + lane) * rows + number] : make_float2(-CUDART_INF_F, 0.f);
    float high = fmaxf(top, st.x);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
    const float was = top == high ? 1.f : pow2(top - high);
    top = high;
    const float f = st.y == 0.f ? -0.f : st.x == top ? 1.f : pow2(st.x - top);      // -0: not this part at all
    float d = f * st.y;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    den = fmaf(den, was, d);
#pragma unroll
    for (int e = 0; e < E; ++e) num[e] *= was;
    for (int z = z0; z < min(z0 + 32, p.splits); z += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const float w = __shfl_sync(0xffffffffu, f, z + i - z0);
        const float* y = reinterpret_cast<const float*>(&x[i]);
#pragma unroll
        for (int e = 0; e < E; ++e) num[e] = __float_as_uint(w) == 0x80000000u ? num[e] : fmaf(w, y[e], num[e]);
      }
      ask(z + kAhead);
    }
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  T* dst = reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + row_offset(p.out, p.rows, layer, seq, r.base, head, pos) + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = T(num[e] * inv);
  if (lane == 0) put_lse(p, layer, col, head, top, den);
}

// ---- host ----------------------------------------------------------------------------------------

// Launches a kernel that waits by itself for the one before it on the stream
template <typename K, typename... A>
spindlekv_status launch_after(K kernel, int64_t blocks, int threads, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_PROMPT, st);
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

// behind the attention itself: joins the parts, if there are any
template <typename T, int D>
spindlekv_status launch_prompt_join(const PromptParams& p, cudaStream_t st) {
  if (p.splits == 1) return SPINDLEKV_OK;
  const int64_t rows = (int64_t)p.rows.n_layers * p.rows.total_len * p.heads * p.hn;
  return launch_after(prompt_join_kernel<T, D>, (rows + 7) / 8, 256, 0, st, p);
}

bool make_rows_map_bf16(CUtensorMap* map, const spindlekv_tensor& t, const spindlekv_batch& b, int n_heads, int head_dim, int box_heads, int box_rows);
bool make_tensor_map_bf16(CUtensorMap* map, const spindlekv_tensor& t, const spindlekv_batch& b, int n_heads, int head_dim, int box_rows);

// fp32: bytes of the pieces, and the call with `pieces` to put them into
size_t prompt_pieces_bytes(const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int n_kv_heads, int head_dim);
spindlekv_status prompt_attend_f32(const PromptParams& p, const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int head_dim, void* pieces,
                                   int64_t blocks, cudaStream_t st);

// few rows: parts of the keys, 0 where a call does not go that way; and the call
int prompt_few_rows(const spindlekv_batch& keys, const spindlekv_batch& rows, int heads, int hn, int head_dim, int dtype);
spindlekv_status prompt_attend_few(const PromptParams& p, const spindlekv_batch& keys, int max_rows, int head_dim, const spindlekv_tensor& k, const spindlekv_tensor& v,
                                   cudaStream_t st);

}  // namespace skv
