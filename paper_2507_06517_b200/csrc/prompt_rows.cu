// Attention of a prompt's last rows in fp32, few of them: on CUDA cores, each key and value read once for up to eight (row, query head) columns.
//
//     O_i = sum_j p_ij V_j / sum_j p_ij,  p_ij = 2^(c q_i.k_j - m_i)
//
// Memory bounds it: two products a key, column and element, where a tile of matrix instructions would have 128 rows to fill, and fp32 would have
// to be taken apart for them.  A warp takes eight keys at a time, which copies of its own bring into its slots of shared memory.  A lane has four elements
// of a row (d = 64: of one of two rows): it multiplies them for eight keys and four columns, and a warp's 32 sums meet lane by lane in 31 exchanges, after
// which each lane holds the score of one key and column, forms its weight and gives it back to all for the second product.  Scores, weights, sums and
// O are fp32.  The reference m moves only when a score exceeds it by 2^8.
//
// A value that a column does not see is passed over (its weight is -0), so that it may be anything.
#include <algorithm>
#include <type_traits>

#include "args.cuh"
#include "prompt_attend.cuh"

namespace skv {

constexpr int kFewKeys = 8;               // of a step
constexpr int kFewPart = 2048;            // keys of a block, at most: a warp then adds up 256
template <int D, int C>
struct FewSmem {
  static constexpr int kWarps = 8, kSlots = 3;
  static constexpr int kHalf = kFewKeys * D * 4, kSlot = 2 * kHalf;      // keys, values
  static constexpr int bytes = kWarps * kSlots * kSlot;
  static_assert(kSlots * kSlot >= C * D * 4, "a warp's result takes the place of its slots");
};

// a row from global memory, or several that lie behind one another
__device__ __forceinline__ void copy_rows(void* to, const void* from, uint64_t* bar, uint32_t bytes) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(to)), "l"(from), "r"(bytes),
               "r"(ptx::smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }

template <int D, int C>
__global__ void __launch_bounds__(FewSmem<D, C>::kWarps * 32) prompt_rows_kernel(const __grid_constant__ PromptParams p, const int chunks) {
  using S = FewSmem<D, C>;
  constexpr int W = S::kWarps, SLOTS = S::kSlots, L = D / 4, R = 32 / L, N = kFewKeys / R, G = C / 4;      // lanes of a row, rows side by side, loads of a step, fours of columns
  static_assert(N * 4 == L, "a score for each lane");
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[W * SLOTS];
  __shared__ int abort_flag[2];
  __shared__ float2 stats[W][C];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, e0 = lane % L * 4;
  if (tid < W * SLOTS) ptx::mbar_init(full + tid, 1);
  if (tid < 2) abort_flag[tid] = 0;
  if (tid == 0) ptx::fence_barrier_init();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) prompt_begins(p);
  __syncthreads();

  int unit = (int)(blockIdx.x / p.splits);
  const int split = (int)blockIdx.x - unit * p.splits;
  const int chunk = unit % chunks;
  unit /= chunks;
  const int ls = unit / p.heads, kv_head = unit - ls * p.heads;
  const int layer = ls / p.rows.n_seqs, seq = ls - layer * p.rows.n_seqs;
  const Span rows = span_of(p.rows, layer, seq), keys = span_of(p.keys, layer, seq);
  const int columns = min(C, rows.len * p.hn - chunk * C);                // columns are (position, query head), heads next to one another
  if (columns <= 0) return;
  // Keys that a lane's columns see, and those that the first and the last column see
  auto sees = [&](int c) { return c < columns ? seen_by((chunk * C + c) / p.hn, rows.len, keys.len) : 0; };
  int limit[G];
#pragma unroll
  for (int g = 0; g < G; ++g) limit[g] = sees(g * 4 + (lane & 3));
  const int all_see = sees(0), n = sees(columns - 1);
  const int steps = (n + kFewKeys - 1) / kFewKeys, begin = (int)((long long)steps * split / p.splits) + warp, end = (int)((long long)steps * (split + 1) / p.splits);
  const int mine = max(0, (end - begin + W - 1) / W);
  const float* kp = reinterpret_cast<const float*>(p.k.ptr) + row_offset(p.k, p.keys, layer, seq, keys.base, kv_head, 0);
  const float* vp = reinterpret_cast<const float*>(p.v.ptr) + row_offset(p.v, p.keys, layer, seq, keys.base, kv_head, 0);
  uint8_t* slots = ring + warp * SLOTS * S::kSlot;
  uint64_t* bars = full + warp * SLOTS;
  const bool joined = p.k.st == D && p.v.st == D;                         // rows lie behind one another
  const int withheld = (int)blockIdx.x == p.withhold && warp == 0 ? 0 : -1;
  auto ask = [&](int i) {
    if (i >= mine || i == withheld) return;
    const int key = (begin + i * W) * kFewKeys, count = min(kFewKeys, n - key);
    uint8_t* to = slots + i % SLOTS * S::kSlot;
    uint64_t* bar = bars + i % SLOTS;
    if (lane == 0) ptx::mbar_expect_tx(bar, 2 * count * D * 4);
    __syncwarp();
    if (joined) {
      if (lane < 2) copy_rows(to + lane * S::kHalf, (lane ? vp : kp) + (int64_t)key * D, bar, count * D * 4);
    } else if ((lane & 7) < count && lane < 16) {
      const int r = lane & 7;
      copy_rows(to + (lane >> 3) * S::kHalf + r * D * 4, lane < 8 ? kp + (int64_t)(key + r) * p.k.st : vp + (int64_t)(key + r) * p.v.st, bar, D * 4);
    }
  };
  for (int i = 0; i < SLOTS - 1; ++i) ask(i);
  int asked = min(mine, SLOTS - 1);

  float4 q[C], o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int cc = chunk * C + c, pos = cc / p.hn;
    q[c] = o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < columns) {
      q[c] = load4(reinterpret_cast<const float*>(p.q.ptr) + row_offset(p.q, p.rows, layer, seq, rows.base, kv_head * p.hn + cc - pos * p.hn, pos) + e0);
      q[c].x *= p.scale; q[c].y *= p.scale; q[c].z *= p.scale; q[c].w *= p.scale;
    }
  }
  float m[G], l[G];
#pragma unroll
  for (int g = 0; g < G; ++g) { m[g] = -CUDART_INF_F; l[g] = 0.f; }
  bool ok = true;
  int i = 0;
  for (; i < mine; ++i) {
    __syncwarp();                                                          // the slot that is asked for again was read by all lanes
    ask(i + SLOTS - 1);
    asked = min(mine, i + SLOTS);
    ok = __all_sync(0xffffffffu, ptx::mbar_wait(bars + i % SLOTS, (i / SLOTS) & 1, abort_flag, p.wait_cycles));
    if (!ok) break;
    const int key = (begin + i * W) * kFewKeys;
    const float* ks = reinterpret_cast<const float*>(slots + i % SLOTS * S::kSlot) + (lane / L) * D + e0;
    const float* vs = ks + S::kHalf / 4;
    const bool hides = key + kFewKeys > all_see;
    float w[G];
    {
      float4 k[N];
#pragma unroll
      for (int r = 0; r < N; ++r) k[r] = load4(ks + r * R * D);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float x[L];
#pragma unroll
        for (int r = 0; r < N; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float4 a = q[g * 4 + c];
            x[r * 4 + c] = fmaf(a.w, k[r].w, fmaf(a.z, k[r].z, fmaf(a.y, k[r].y, a.x * k[r].x)));
          }
        // sums of L lanes: each exchange halves what a lane holds, and lane i ends with number i % L: key i / 4 * R + its own of R, column i % 4
#pragma unroll
        for (int h = L / 2; h >= 1; h >>= 1)
#pragma unroll
          for (int e = 0; e < h; ++e) {
            const float away = lane & h ? x[e] : x[e + h], stays = lane & h ? x[e + h] : x[e];
            x[e] = stays + __shfl_xor_sync(0xffffffffu, away, h);
          }
        w[g] = x[0];
      }
    }
    const int this_key = key + (lane % L >> 2) * R + lane / L;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const bool seen = !hides || this_key < limit[g];
      const float s = seen ? w[g] : -CUDART_INF_F;
      if (__any_sync(0xffffffffu, s > m[g] + kPromptLazy)) {
        float high = fmaxf(s, m[g]);
#pragma unroll
        for (int h = 4; h < 32; h <<= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, h));
        const float f = high == m[g] ? 1.f : pow2(m[g] - high);
        m[g] = high;
        l[g] *= f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float fc = __shfl_sync(0xffffffffu, f, c);
          float4& a = o[g * 4 + c];
          a.x *= fc; a.y *= fc; a.z *= fc; a.w *= fc;
        }
      }
      w[g] = seen ? pow2(s - (m[g] == -CUDART_INF_F ? 0.f : m[g])) : -0.f;
      l[g] += w[g];
    }
    float4 v[N];
#pragma unroll
    for (int r = 0; r < N; ++r) v[r] = load4(vs + r * R * D);
    auto add = [&](auto some_hidden) {
#pragma unroll
      for (int r = 0; r < N; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float wc = __shfl_sync(0xffffffffu, w[c / 4], (lane & ~(L - 1)) | r * 4 | (c & 3));
          if (decltype(some_hidden)::value && __float_as_uint(wc) == 0x80000000u) continue;
          o[c].x = fmaf(wc, v[r].x, o[c].x);
          o[c].y = fmaf(wc, v[r].y, o[c].y);
          o[c].z = fmaf(wc, v[r].z, o[c].z);
          o[c].w = fmaf(wc, v[r].w, o[c].w);
        }
    };
    if (hides) add(std::true_type()); else add(std::false_type());
  }
  if (!ok) {
    // the copies that are still on their way come in before the block goes
    __syncwarp();
    for (; i < asked; ++i)
      if (i != withheld) ptx::mbar_wait(bars + i % SLOTS, (i / SLOTS) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
  }
  // ---- the warps' results, joined ----
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int h = 4; h < 32; h <<= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], h);
    if (lane < 4) stats[warp][g * 4 + lane] = make_float2(m[g], l[g]);
  }
  __syncwarp();
  float* result = reinterpret_cast<float*>(slots);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (R == 2) {
      o[c].x += __shfl_xor_sync(0xffffffffu, o[c].x, 16);
      o[c].y += __shfl_xor_sync(0xffffffffu, o[c].y, 16);
      o[c].z += __shfl_xor_sync(0xffffffffu, o[c].z, 16);
      o[c].w += __shfl_xor_sync(0xffffffffu, o[c].w, 16);
    }
    if (lane < L) store4(result + c * D + e0, o[c]);
  }
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(abort_flag)) {
    if (tid == 0) prompt_failed(p);
    return;
  }
  for (int x = tid; x < C * L; x += W * 32) {
    const int c = x / L, e = x % L * 4;
    if (c >= columns) break;
    float top = -CUDART_INF_F, sum = 0.f;
#pragma unroll
    for (int y = 0; y < W; ++y) top = fmaxf(top, stats[y][c].x);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const float2 st = stats[y][c];
      const float f = st.y == 0.f ? 0.f : st.x == top ? 1.f : pow2(st.x - top);
      const float4 b = load4(reinterpret_cast<const float*>(ring + y * SLOTS * S::kSlot) + c * D + e);
      sum = fmaf(f, st.y, sum);
      a.x = fmaf(f, b.x, a.x);
      a.y = fmaf(f, b.y, a.y);
      a.z = fmaf(f, b.z, a.z);
      a.w = fmaf(f, b.w, a.w);
    }
    const int cc = chunk * C + c, pos = cc / p.hn, head = kv_head * p.hn + cc - pos * p.hn;
    if (p.splits > 1) {
      const int64_t number = row_number(p, layer, seq, rows.base, head, pos) + (int64_t)split * p.rows.n_layers * p.rows.total_len * (p.heads * p.hn);
      store4(p.part + number * D + e, a);
      if (e == 0) p.stat[number] = make_float2(top, sum);
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      store4(reinterpret_cast<float*>(const_cast<void*>(p.out.ptr)) + row_offset(p.out, p.rows, layer, seq, rows.base, head, pos) + e,
             make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
      if (e == 0) put_lse(p, layer, column_of(p, seq, rows.base, pos), head, top, sum);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------

// Columns of a thread block
static int few_columns(int columns) { return columns <= 4 ? 4 : 8; }

// Parts of the keys for calls that come here, 0 for those that do not.  fp32 with up to 24 columns: 4 x 16384 keys, 32 / 8 heads, d = 128, 4 / 16 columns
// 94 / 234 us here and 397 / 406 by matrix instructions, which take the keys apart first; one sequence with 32 columns 120 and 130.  bf16 stays with those:
// 63 and 58 us at 4 columns, 237 and 59 at 16.
int prompt_few_rows(const spindlekv_batch& keys, const spindlekv_batch& rows, int heads, int hn, int head_dim, int dtype) {
  const int64_t columns = (int64_t)rows.max_len * hn;
  if (dtype != SPINDLEKV_F32 || columns > 24) return 0;
  const int c = few_columns((int)columns);
  const int64_t units = (int64_t)rows.n_layers * rows.n_seqs * heads * ((columns + c - 1) / c), wave = 148 * (head_dim == 64 ? 2 : 1);
  // one wave of blocks; several where a block's part would be long, which also evens out sequences of different lengths
  const int64_t splits = std::max<int64_t>((keys.max_len + kFewPart - 1) / kFewPart, std::min<int64_t>(wave / units, keys.max_len / 64));
  return splits * units <= 65535 ? (int)splits : 0;
}

template <int D, int C>
static spindlekv_status launch_few(const PromptParams& p, int64_t blocks, int chunks, cudaStream_t st) {
  using S = FewSmem<D, C>;
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    if (cudaFuncSetAttribute(prompt_rows_kernel<D, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::bytes) != cudaSuccess) return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  const spindlekv_status s = launch_after(prompt_rows_kernel<D, C>, blocks, S::kWarps * 32, S::bytes, st, p, chunks);
  return s == SPINDLEKV_OK ? launch_prompt_join<float, D>(p, st) : s;
}

spindlekv_status prompt_attend_few(const PromptParams& p, int max_rows, int head_dim, cudaStream_t st) {
  const int columns = max_rows * p.hn, c = few_columns(columns), chunks = (columns + c - 1) / c;
  const int64_t blocks = (int64_t)p.rows.n_layers * p.rows.n_seqs * p.heads * chunks * p.splits;
  if (head_dim == 64) return c == 4 ? launch_few<64, 4>(p, blocks, chunks, st) : launch_few<64, 8>(p, blocks, chunks, st);
  return c == 4 ? launch_few<128, 4>(p, blocks, chunks, st) : launch_few<128, 8>(p, blocks, chunks, st);
}

}  // namespace skv
