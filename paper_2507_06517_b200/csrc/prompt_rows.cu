// Attention of a prompt's last rows, few of them: each key and value is read once for up to sixteen (row, query head) columns.
//
//     O_i = sum_j p_ij V_j / sum_j p_ij,  p_ij = 2^(c q_i.k_j - m_i)
//
// Memory bounds it, and what there is of products does not fill the 128 rows of a tile of the tensor cores, nor pays for fp32 to be taken apart for them.
// The keys of a (layer, sequence, KV head) are cut into parts for thread blocks, and these into steps of 8 (fp32) or 16 (bf16) keys that its warps take in
// turn; each warp has slots of its own, two or more steps ahead, so that no warp waits for another until the results are joined.
//
// fp32: a lane has four elements of a row (d = 64: of one of two rows); it multiplies them for eight keys and four columns, and a warp's 32 sums meet lane
// by lane in 31 exchanges, after which each lane holds the score of one key and column, forms its weight and gives it back to all for the second product.
// bf16: warp-wide matrix instructions with the keys as their 16 rows, S^T = K Q^T and O^T += V^T P^T, so that eight columns are a whole instruction.
//
// Scores, weights, sums and O are fp32; bf16 weights are rounded to bf16 where they meet the values, which costs what the result's own rounding does.
// The reference m moves only when a score exceeds it by 2^8.  A value that a column does not see is passed over, so that it may be anything: by its weight
// of -0 in fp32; in bf16 steps that hide keys from some column look whether all of their values are finite, and multiply by hand if they are not.
//
// 4 x 16384 keys, 32 query heads over 8, d = 128, one row: bf16 48 us (5.6 TB/s, issue slots 24 % busy), fp32 87 us (6.1 TB/s, 47 %); one sequence of them
// 15 and 29 us, of 2000 keys 9 and 10, where the launch, the lengths, the first copies and the join follow one another.
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
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 x) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w)); }

// What a thread block does: a part of the keys for some columns of a KV head
struct FewUnit {
  int layer, seq, kv_head, split, first, columns;      // columns [first, first + columns), (position, query head) with heads next to one another
  Span rows, keys;
  int all_see, n;                                      // keys that the first of them sees, and the last
  int begin, mine;                                     // this warp's first step and how many it has, `warps` apart
  __device__ __forceinline__ FewUnit(const PromptParams& p, int chunks, int most, int keys_of_step, int warps) {
    int unit = (int)(blockIdx.x / p.splits);
    split = (int)blockIdx.x - unit * p.splits;
    const int chunk = unit % chunks;
    unit /= chunks;
    const int ls = unit / p.heads;
    kv_head = unit - ls * p.heads;
    layer = ls / p.rows.n_seqs;
    seq = ls - layer * p.rows.n_seqs;
    rows = span_of(p.rows, layer, seq);
    keys = span_of(p.keys, layer, seq);
    first = chunk * most;
    columns = min(most, rows.len * p.hn - first);
    all_see = sees(p, 0);
    n = columns > 0 ? sees(p, columns - 1) : 0;
    const int steps = (n + keys_of_step - 1) / keys_of_step, end = (int)((long long)steps * (split + 1) / p.splits);
    begin = (int)((long long)steps * split / p.splits) + (threadIdx.x >> 5);
    mine = max(0, (end - begin + warps - 1) / warps);
  }
  __device__ __forceinline__ int sees(const PromptParams& p, int c) const { return c < columns ? seen_by((first + c) / p.hn, rows.len, keys.len) : 0; }
};

// The warps' results (`ring`: O of each, `apart` bytes from one another; stats: reference and sum) as the block's: its part, or rows of out
template <typename T, int D, int C, int W>
__device__ __forceinline__ void join_warps(const PromptParams& p, const FewUnit& u, const uint8_t* ring, int apart, const float2 (&stats)[W][C]) {
  for (int x = threadIdx.x; x < C * (D / 4); x += W * 32) {
    const int c = x / (D / 4), e = x % (D / 4) * 4;
    if (c >= u.columns) break;
    float top = -CUDART_INF_F, sum = 0.f;
#pragma unroll
    for (int y = 0; y < W; ++y) top = fmaxf(top, stats[y][c].x);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const float2 st = stats[y][c];
      const float f = st.y == 0.f ? 0.f : st.x == top ? 1.f : pow2(st.x - top);
      const float4 b = load4(reinterpret_cast<const float*>(ring + y * apart) + c * D + e);
      sum = fmaf(f, st.y, sum);
      a.x = fmaf(f, b.x, a.x);
      a.y = fmaf(f, b.y, a.y);
      a.z = fmaf(f, b.z, a.z);
      a.w = fmaf(f, b.w, a.w);
    }
    const int cc = u.first + c, pos = cc / p.hn, head = u.kv_head * p.hn + cc - pos * p.hn;
    if (p.splits > 1) {
      const int64_t number = row_number(p, u.layer, u.seq, u.rows.base, head, pos) + (int64_t)u.split * p.rows.n_layers * p.rows.total_len * (p.heads * p.hn);
      store4(p.part + number * D + e, a);
      if (e == 0) p.stat[number] = make_float2(top, sum);
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      store4(reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + row_offset(p.out, p.rows, u.layer, u.seq, u.rows.base, head, pos) + e,
             make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
      if (e == 0) put_lse(p, u.layer, column_of(p, u.seq, u.rows.base, pos), head, top, sum);
    }
  }
}

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
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const FewUnit u(p, chunks, C, kFewKeys, W);
  const bool counts = tid == W * 32 - 1;                // (one thread whose warp has asked for its keys by then)
  if (u.columns <= 0) {
    if (counts) prompt_begins(p);
    return;
  }
  int limit[G];
#pragma unroll
  for (int g = 0; g < G; ++g) limit[g] = u.sees(p, g * 4 + (lane & 3));
  const float* kp = reinterpret_cast<const float*>(p.k.ptr) + row_offset(p.k, p.keys, u.layer, u.seq, u.keys.base, u.kv_head, 0);
  const float* vp = reinterpret_cast<const float*>(p.v.ptr) + row_offset(p.v, p.keys, u.layer, u.seq, u.keys.base, u.kv_head, 0);
  uint8_t* slots = ring + warp * SLOTS * S::kSlot;
  uint64_t* bars = full + warp * SLOTS;
  const bool joined = p.k.st == D && p.v.st == D;                         // rows lie behind one another
  const int withheld = (int)blockIdx.x == p.withhold && warp == 0 ? 0 : -1;
  auto ask = [&](int i) {
    if (i >= u.mine || i == withheld) return;
    const int key = (u.begin + i * W) * kFewKeys, count = min(kFewKeys, u.n - key);
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
  int asked = min(u.mine, SLOTS - 1);
  if (counts) prompt_begins(p);
  __syncwarp();

  float4 q[C], o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int cc = u.first + c, pos = cc / p.hn;
    q[c] = o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < u.columns) {
      q[c] = load4(reinterpret_cast<const float*>(p.q.ptr) + row_offset(p.q, p.rows, u.layer, u.seq, u.rows.base, u.kv_head * p.hn + cc - pos * p.hn, pos) + e0);
      q[c].x *= p.scale; q[c].y *= p.scale; q[c].z *= p.scale; q[c].w *= p.scale;
    }
  }
  float m[G], l[G];
#pragma unroll
  for (int g = 0; g < G; ++g) { m[g] = -CUDART_INF_F; l[g] = 0.f; }
  bool ok = true;
  int i = 0;
  for (; i < u.mine; ++i) {
    __syncwarp();                                                          // the slot that is asked for again was read by all lanes
    ask(i + SLOTS - 1);
    asked = min(u.mine, i + SLOTS);
    ok = __all_sync(0xffffffffu, ptx::mbar_wait(bars + i % SLOTS, (i / SLOTS) & 1, abort_flag, p.wait_cycles));
    if (!ok) break;
    const int key = (u.begin + i * W) * kFewKeys;
    const float* ks = reinterpret_cast<const float*>(slots + i % SLOTS * S::kSlot) + (lane / L) * D + e0;
    const float* vs = ks + S::kHalf / 4;
    const bool hides = key + kFewKeys > u.all_see;
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
  join_warps<float, D, C, W>(p, u, ring, SLOTS * S::kSlot, stats);
}

// ---- bf16 ----------------------------------------------------------------------------------------

constexpr int kFewKeysBf16 = 16;
template <int D, int NT>                  // NT: eights of columns
struct FewSmemBf16 {
  static constexpr int kWarps = 8, kSlots = 3;
  static constexpr int kHalf = kFewKeysBf16 * 128, kTile = D / 64 * kHalf, kSlot = 2 * kTile;      // 64 elements of 16 rows; keys; keys and values
  static constexpr int bytes = 1024 + kWarps * kSlots * kSlot;
};

__device__ __forceinline__ void matrix_rows(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void matrix_columns(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ bool all_finite(uint4 x) {
  auto odd = [](uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; };
  return !(odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w));
}

// Fragments, with r = lane / 4 and t = lane % 4: S^T has keys r and r + 8 and columns 2 t, 2 t + 1 (of eight); O^T elements 16 i + r and + 8, the same columns.
template <int D, int NT>
__global__ void __launch_bounds__(FewSmemBf16<D, NT>::kWarps * 32) prompt_rows_bf16_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                                                       const __grid_constant__ PromptParams p, const int chunks) {
  using S = FewSmemBf16<D, NT>;
  using T = __nv_bfloat16;
  constexpr int W = S::kWarps, SLOTS = S::kSlots, C = NT * 8, KS = kFewKeysBf16;
  static_assert(SLOTS * S::kSlot >= C * D * 4, "a warp's result takes the place of its slots");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t full[W * SLOTS];
  __shared__ int abort_flag[2];
  __shared__ float2 stats[W][C];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, t = lane & 3;
  if (tid < W * SLOTS) ptx::mbar_init(full + tid, 1);
  if (tid < 2) abort_flag[tid] = 0;
  if (tid == 0) {
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&kmap);
    ptx::prefetch_tensormap(&vmap);
  }
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const FewUnit u(p, chunks, C, KS, W);
  const bool counts = tid == W * 32 - 1;                // (one thread whose warp has asked for its keys by then)
  if (u.columns <= 0) {
    if (counts) prompt_begins(p);
    return;
  }
  uint8_t* slots = ring + warp * SLOTS * S::kSlot;
  uint64_t* bars = full + warp * SLOTS;
  const int withheld = (int)blockIdx.x == p.withhold && warp == 0 ? 0 : -1;
  auto ask = [&](int i) {
    if (i >= u.mine || i == withheld || lane != 0) return;
    uint8_t* to = slots + i % SLOTS * S::kSlot;
    uint64_t* bar = bars + i % SLOTS;
    const int row = u.keys.base + (u.begin + i * W) * KS, seq = p.keys.cu ? 0 : u.seq;
    ptx::mbar_expect_tx(bar, S::kSlot);
#pragma unroll
    for (int h = 0; h < D / 64; ++h) ptx::tma_load_5d(to + h * S::kHalf, &kmap, bar, h * 64, row, u.kv_head, seq, u.layer);
#pragma unroll
    for (int h = 0; h < D / 64; ++h) ptx::tma_load_5d(to + S::kTile + h * S::kHalf, &vmap, bar, h * 64, row, u.kv_head, seq, u.layer);
  };
  for (int i = 0; i < SLOTS - 1; ++i) ask(i);
  int asked = min(u.mine, SLOTS - 1);
  if (counts) prompt_begins(p);
  __syncwarp();

  uint32_t q[NT][D / 16][2];
  int limit[NT][2];
#pragma unroll
  for (int g = 0; g < NT; ++g) {
    const int c = g * 8 + r, cc = u.first + c, pos = cc / p.hn;
    const T* from = reinterpret_cast<const T*>(p.q.ptr) + (c < u.columns ? row_offset(p.q, p.rows, u.layer, u.seq, u.rows.base, u.kv_head * p.hn + cc - pos * p.hn, pos) : 0) + 2 * t;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) q[g][k][h] = c < u.columns ? *reinterpret_cast<const uint32_t*>(from + k * 16 + h * 8) : 0u;
    limit[g][0] = u.sees(p, g * 8 + 2 * t);
    limit[g][1] = u.sees(p, g * 8 + 2 * t + 1);
  }
  float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int g = 0; g < NT; ++g) {
    m[g][0] = m[g][1] = -CUDART_INF_F;
    l[g][0] = l[g][1] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[g][k][e] = 0.f;
  }
  // byte of (row, 16 bytes number `piece`) of a tile whose rows of 128 bytes are swizzled
  auto place = [](int row, int piece) { return (piece >> 3) * S::kHalf + row * 128 + (((piece ^ row) & 7) << 4); };
  bool ok = true;
  int i = 0;
  for (; i < u.mine; ++i) {
    __syncwarp();                                                          // the slot that is asked for again was read by all lanes
    ask(i + SLOTS - 1);
    asked = min(u.mine, i + SLOTS);
    ok = __all_sync(0xffffffffu, ptx::mbar_wait(bars + i % SLOTS, (i / SLOTS) & 1, abort_flag, p.wait_cycles));
    if (!ok) break;
    const int key = (u.begin + i * W) * KS;
    const uint8_t* ks = slots + i % SLOTS * S::kSlot;
    const uint32_t ka = ptx::smem_u32(ks), va = ka + S::kTile;
    const bool hides = key + KS > u.all_see;
    float x[NT][4];
#pragma unroll
    for (int g = 0; g < NT; ++g) x[g][0] = x[g][1] = x[g][2] = x[g][3] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      matrix_rows(ka + place(lane & 15, k * 2 + (lane >> 4)), a);
#pragma unroll
      for (int g = 0; g < NT; ++g) multiply(x[g], a, q[g][k][0], q[g][k][1]);
    }
    uint32_t b[NT][2];
#pragma unroll
    for (int g = 0; g < NT; ++g) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[g][e] *= p.scale;
        if (hides && key + r + (e >> 1) * 8 >= limit[g][e & 1]) x[g][e] = -CUDART_INF_F;
      }
      float high[2] = {fmaxf(x[g][0], x[g][2]), fmaxf(x[g][1], x[g][3])};
      if (__any_sync(0xffffffffu, high[0] > m[g][0] + kPromptLazy || high[1] > m[g][1] + kPromptLazy)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int h = 4; h < 32; h <<= 1) high[e] = fmaxf(high[e], __shfl_xor_sync(0xffffffffu, high[e], h));
          const float now = fmaxf(m[g][e], high[e]), f = now == m[g][e] ? 1.f : pow2(m[g][e] - now);
          m[g][e] = now;
          l[g][e] *= f;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            o[g][k][e] *= f;
            o[g][k][e + 2] *= f;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) x[g][e] = pow2(x[g][e] - (m[g][e & 1] == -CUDART_INF_F ? 0.f : m[g][e & 1]));
      l[g][0] += x[g][0] + x[g][2];
      l[g][1] += x[g][1] + x[g][3];
      b[g][0] = transposed(pack_bf16(x[g][0], x[g][1]));
      b[g][1] = transposed(pack_bf16(x[g][2], x[g][3]));
    }
    bool by_hand = false;
    if (hides) {
      bool fine = true;
#pragma unroll
      for (int y = 0; y < S::kTile / 512; ++y) fine = all_finite(*reinterpret_cast<const uint4*>(ks + S::kTile + (y * 32 + lane) * 16)) && fine;
      by_hand = !__all_sync(0xffffffffu, fine);
    }
    if (!by_hand) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t a[4];
        matrix_columns(va + place((lane & 7) + (lane >> 4) * 8, k * 2 + (lane >> 3 & 1)), a);
#pragma unroll
        for (int g = 0; g < NT; ++g) multiply(o[g][k], a, b[g][0], b[g][1]);
      }
    } else {
#pragma unroll 1
      for (int y = 0; y < KS; ++y) {
#pragma unroll
        for (int g = 0; g < NT; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float w = __bfloat162float(T(__shfl_sync(0xffffffffu, y < 8 ? x[g][e] : x[g][e + 2], (y & 7) * 4 + t)));
            if (key + y >= limit[g][e]) continue;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                o[g][k][e + 2 * h] = fmaf(w, __bfloat162float(*reinterpret_cast<const T*>(ks + S::kTile + place(y, k * 2 + h) + r * 2)), o[g][k][e + 2 * h]);
          }
      }
    }
  }
  if (!ok) {
    // the copies that are still on their way come in before the block goes
    __syncwarp();
    for (; i < asked; ++i)
      if (i != withheld) ptx::mbar_wait(bars + i % SLOTS, (i / SLOTS) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
  }
  __syncwarp();
  float* result = reinterpret_cast<float*>(slots);
#pragma unroll
  for (int g = 0; g < NT; ++g)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int h = 4; h < 32; h <<= 1) l[g][e] += __shfl_xor_sync(0xffffffffu, l[g][e], h);
      const int c = g * 8 + 2 * t + e;
      if (r == 0) stats[warp][c] = make_float2(m[g][e], l[g][e]);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        result[c * D + k * 16 + r] = o[g][k][e];
        result[c * D + k * 16 + r + 8] = o[g][k][e + 2];
      }
    }
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(abort_flag)) {
    if (tid == 0) prompt_failed(p);
    return;
  }
  join_warps<T, D, C, W>(p, u, ring, SLOTS * S::kSlot, stats);
}

// ---- host ----------------------------------------------------------------------------------------

// Columns of a KV head's rows that come here.  Both ways measured (32 / 8 heads, d = 128; here / by whole tiles):
//   bf16, 16384 keys, 4 / 16 / 32 columns 15 / 20 / 25 us and 23 / 25 / 27; 4 x 16384, 4 / 16 columns 48 / 54 and 56 / 58; 32 sequences of 200 to 4000 keys,
//   4 columns 51 and 100.  More than 16 columns would be two thread blocks that read the same keys.
//   fp32, 16384 keys, 4 / 16 / 32 columns 29 / 58 / 121 us and 118 / 120 / 122; 4 x 16384, 4 / 16 columns 87 / 227 and 406 / 407.
// d = 64: bf16, 16384 keys, 4 / 16 / 32 columns 17 / 20 / 23 and 25 / 27 / 28, 8 x 4096 17 / 21 / 28 and 33 / 35 / 36; fp32, 4 / 16 / 24 / 32 columns 23 / 41 / 53 / 66 and 70 to 73, 8 x 4096
// 33 / 71 / 102 / 125 and 122.  2000 keys of two KV heads: bf16, 4 / 16 columns 13 / 16 and 19; fp32 15 / 18 and 32.  One KV head of one sequence is where tiles do better in bf16, having few
// parts to join (16384 keys, 4 / 16 columns: d = 128 20 / 26 and 20, d = 64 26 / 28 and 19); fp32 22 / 24 and 39, 27 / 26 and 30.
constexpr int kFewMostBf16 = 16, kFewMostF32 = 24;
// Columns of a thread block
static int few_columns(int columns, int dtype) { return dtype == SPINDLEKV_F32 ? (columns <= 4 ? 4 : 8) : columns <= 8 ? 8 : 16; }

// Parts of the keys for calls that come here, 0 for those that do not
int prompt_few_rows(const spindlekv_batch& keys, const spindlekv_batch& rows, int heads, int hn, int head_dim, int dtype) {
  const int64_t columns = (int64_t)rows.max_len * hn;
  if (columns > (dtype == SPINDLEKV_F32 ? kFewMostF32 : kFewMostBf16)) return 0;
  const int c = few_columns((int)columns, dtype);
  const int64_t units = (int64_t)rows.n_layers * rows.n_seqs * heads * ((columns + c - 1) / c), wave = 148 * (head_dim == 64 ? 2 : 1);
  // one wave of blocks; several where a block's part would be long, which also evens out sequences of different lengths
  const int64_t splits = std::max<int64_t>((keys.max_len + kFewPart - 1) / kFewPart, std::min<int64_t>(wave / units, keys.max_len / 64));
  return splits * units <= 65535 ? (int)splits : 0;
}

// A kernel of this file and what joins its parts
template <typename T, int D, typename S, typename K, typename... A>
static spindlekv_status launch_few(K kernel, const PromptParams& p, int max_rows, int most, cudaStream_t st, const A&... maps) {
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::bytes) != cudaSuccess) return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  const int chunks = ceil_div(max_rows * p.hn, most);
  const int64_t blocks = (int64_t)p.rows.n_layers * p.rows.n_seqs * p.heads * chunks * p.splits;
  const spindlekv_status s = launch_after(kernel, blocks, S::kWarps * 32, S::bytes, st, maps..., p, chunks);
  return s == SPINDLEKV_OK ? launch_prompt_join<T, D>(p, st) : s;
}

template <int D>
static spindlekv_status launch_few(const PromptParams& p, const spindlekv_batch& keys, int max_rows, const spindlekv_tensor& k, const spindlekv_tensor& v, cudaStream_t st) {
  const int most = few_columns(max_rows * p.hn, k.dtype);
  if (k.dtype == SPINDLEKV_F32)
    return most == 4 ? launch_few<float, D, FewSmem<D, 4>>(prompt_rows_kernel<D, 4>, p, max_rows, most, st)
                     : launch_few<float, D, FewSmem<D, 8>>(prompt_rows_kernel<D, 8>, p, max_rows, most, st);
  CUtensorMap kmap, vmap;
  if (!make_tensor_map_bf16(&kmap, k, keys, p.heads, D, kFewKeysBf16) || !make_tensor_map_bf16(&vmap, v, keys, p.heads, D, kFewKeysBf16)) return SPINDLEKV_UNSUPPORTED;
  return most == 8 ? launch_few<__nv_bfloat16, D, FewSmemBf16<D, 1>>(prompt_rows_bf16_kernel<D, 1>, p, max_rows, most, st, kmap, vmap)
                   : launch_few<__nv_bfloat16, D, FewSmemBf16<D, 2>>(prompt_rows_bf16_kernel<D, 2>, p, max_rows, most, st, kmap, vmap);
}

spindlekv_status prompt_attend_few(const PromptParams& p, const spindlekv_batch& keys, int max_rows, int head_dim, const spindlekv_tensor& k, const spindlekv_tensor& v,
                                   cudaStream_t st) {
  return head_dim == 64 ? launch_few<64>(p, keys, max_rows, k, v, st) : launch_few<128>(p, keys, max_rows, k, v, st);
}

}  // namespace skv
