// Attention of the newest tokens over the 8-bit paged cache.
//
// Bound: every cached byte has to come from memory once (2 d bytes per token and KV head, plus 8/16 bytes of scales), so all
// query heads of a KV head, and all new rows, are served by one pass over its codes.
//
// Mathematics.  The tensor cores multiply fp16 by fp16 into fp32.  Codes are exact in fp16, and so are the numbers
// of E4M3.  Queries enter scaled by a power of two per row: bf16 queries are exact in one fp16 piece (elements below
// 2^-29 of the row's largest fade out), fp32 queries in two pieces (22 bits).  S^T = K Q^T, then p = 2^(S s_k c - m) with a running
// reference m per query that moves only when a score exceeds it by 8 (p stays below 2^8), O^T += s_v (V^T P^T) with P in one fp16
// piece for bf16 (2^-12 relative, below the output's rounding) or two for fp32.  s_v, relative to a power of two above all scales so far,
// joins the weights before they are rounded where that is safe and is else applied to the block's product in fp32, so blocks of very
// different scale do not disturb one another.  m, the sum of p and O are fp32.
//
// Layout.  A warp takes one block of 16 tokens at a time: K is the 16 x d operand of m16n8k16, the queries are its 8 columns.  Which
// token or element a lane's fragment registers stand for is free as long as both operands agree: a lane's 16 bytes of a K row are four
// k-steps, and for V it takes the same 16 bytes of four tokens and transposes bytes between registers.  Two blocks are computed
// side by side.  They arrive by TMA, in their warp's own slots (the next keys as soon as these are read, the next values likewise), in swizzled rows and
// with the tokens assigned so that no two lanes meet in a bank; nothing but the warp waits for them.  P changes layout by an 8x8
// transposition inside the warp.
//
// Split.  All blocks of all (layer, sequence, head) units form one line, cut into equal runs, one per resident thread block;
// the eight warps of a thread block deal a run's blocks among themselves.  Every run thus has the same work however
// uneven the lengths are.  A unit that lies inside one run is finished there; of the others each run leaves (m, sum, O), which a second
// kernel joins in the order of the runs.
//
// Measured (device time): 16384 tokens, 8 KV heads, 32 query heads 15.0 us, of which the loop is 5 at the copy rate and the rest set-up
// (4.5), join (4) and launch; 8 sequences of 2048 to 16384, 13000 on average (213 MB), 46.6 us (4.6 TB/s); 4 x 16384 tokens with 4 to 8 columns per KV
// head 34 to 36 us (4.0 TB/s), 16 columns 41 to 44, with fp32 queries 37 to 54; 32 columns of fp32 queries 88 (E4M3) and 92 (int8) (two column tiles
// and more have the SM to themselves, eight warps: latency), 128 columns 281 and 297 (four passes).  More than 16 bf16 columns of 128 elements take
// paged_attend_tiles.cu.
#include <algorithm>

#include "paged_attend.cuh"

namespace skv {

constexpr int kAttThreads = 256;
constexpr int kAttWarps = kAttThreads / 32;
constexpr int kAttCols = 32;            // columns of a part, at most
constexpr int kSetUp = 6;              // places of a unit's beginning and end, in pairs of blocks
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
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float2 unpack_half2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// the same, offset int8 codes as subnormal numbers
template <int HI>
__device__ __forceinline__ uint32_t offset_to_half2(uint32_t w) { return __byte_perm(w, 0u, HI ? 0x4342 : 0x4140); }
template <int D, int NT>
__host__ __device__ constexpr size_t ring_bytes() {   // the warps' results take the ring's place when a segment ends
  const size_t ring = (size_t)kAttWarps * 4 * kPagedBlock * D, results = (size_t)kAttWarps * 8 * NT * (D + 4) * 4;
  return ring > results ? ring : results;
}

// The token of a block that fragment row i (and i + 8, eight tokens on) stands for.  With it the lanes that read shared memory
// together find their 16 bytes of the swizzled rows (128 bytes for d = 128, 64 for d = 64) in different banks, for K and for V.
template <int D>
__device__ __forceinline__ int token_of(int i) { return ((D == 128 ? 0x37156240 : 0x65742130) >> (4 * i)) & 7; }

template <typename T, int FMT, int D, int NT>
__global__ void __launch_bounds__(kAttThreads, NT >= 2 ? 1 : 2) paged_attend_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                                  const __grid_constant__ CUtensorMap vmap, AttendParams p) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;      // fp16 pieces of a query and of a weight
  constexpr int KS = D / 16;                      // k-steps of a score, and m-tiles of an output
  constexpr int KH = D / 64;                      // 16-byte pieces of a K row per lane
  constexpr int VW = D / 32;                      // words of a V row per lane
  constexpr int COLS = 8 * NT;
  // int8 keys under one query piece enter as (code + 128) 2^-24, a subnormal fp16 number, which saves a subtraction per two of them;
  // the scores lose 128 times the query's sum.  The accumulator's roundings are then relative to sum |q_i| (|code_i| + 128) in place of
  // sum |q_i code_i|: three times as much where codes fill their range, a hundred times where one outlier channel has set the block's
  // scale and the other codes are small.  Against sum |q_i| times the block's largest key that is 2^-19 at most, below what bf16 results show
  // for scores up to some hundreds; too much for fp32 queries
  constexpr bool kOffset = FMT == SPINDLEKV_PAGED_INT8 && NP == 1 && NT == 1;
  constexpr int OP = D + 4;                       // row pitch of the partial outputs in shared memory
  constexpr int kHalf = kPagedBlock * D;          // bytes of a block's K, or V
  constexpr int kSlot = 2 * kHalf;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  // prefix sums over the (layer, seq) pairs; then the queries' fragments, per-column factors, the warps' results
  const int n_ls = p.table.n_layers * p.table.n_seqs;
  float* so = reinterpret_cast<float*>(smem);                            // [kAttWarps][COLS][OP], over the ring
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + ring_bytes<D, NT>());    // [kAttWarps][2]
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + kAttWarps * 2);   // a wait gave up; and one for the waits after that
  uint2* sq = reinterpret_cast<uint2*>(bars + kAttWarps * 2 + 2);             // [NP][NT][KS][32]
  float* sfac = reinterpret_cast<float*>(sq + NP * NT * KS * 32);       // [COLS] factor of a score, NaN for an infinite query
  float* scorr = sfac + COLS;                                           // [COLS] and what the codes' offset adds to the product before
  float* sm_m = scorr + COLS;                                            // [kAttWarps][COLS]
  float* sm_l = sm_m + kAttWarps * COLS;                                // [kAttWarps][COLS]
  int* warp_sums = reinterpret_cast<int*>(sm_l + kAttWarps * COLS);     // [33]
  int* prefix = warp_sums + 36;                                         // [n_ls + 1]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;   // g, c: the fragments' rows and columns

  if (lane == 0) {       // each warp its own
    ptx::mbar_init(bars + warp * 2, 1);
    ptx::mbar_init(bars + warp * 2 + 1, 1);
    ptx::fence_barrier_init();
    if (warp == 0) {
      abort_flag[0] = abort_flag[1] = 0;
      ptx::prefetch_tensormap(&kmap);
      ptx::prefetch_tensormap(&vmap);
    }
  }
  // up to here nothing was read or written that an earlier kernel of the stream knows of
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  uint8_t* ring = smem + warp * 2 * kSlot;   // K of a pair, V of a pair
  uint64_t* full = bars + warp * 2;          // the keys, the values have arrived
  uint32_t phase = 0;
  const int total = line_prefix<2 * kPagedBlock, kSetUp>(p, prefix, warp_sums);
  const Runs cut(total * p.units_per, (int)gridDim.x);
  int at, stop;
  if (p.whole_units) {
    const int e = blockIdx.x / p.units_per, u = blockIdx.x - e * p.units_per, places = prefix[e + 1] - prefix[e];
    at = prefix[e] * p.units_per + u * places;
    stop = at + places;
  } else {
    at = cut.start(blockIdx.x);
    stop = (int)blockIdx.x < cut.runs ? cut.start(blockIdx.x + 1) : at;
  }
  // With a block per unit there is no join to write the status word: the last block does, when it is known whether one has given up.  (The last
  // warp asks, which has the least to do with a unit's result.)
  auto settle = [&](bool gave_up) {
    if (!p.whole_units || tid != kAttThreads - 32) return;
    const int end = last_to_arrive(reinterpret_cast<unsigned long long*>(p.hdr + kHdrUnitsDone), (int)gridDim.x, gave_up);
    if (end) p.hdr[kHdrStatus] = end == 1 ? SPINDLEKV_OK : SPINDLEKV_TIMEOUT;
  };
  if (!p.whole_units && tid == 0) p.lead[blockIdx.x] = make_int2(-1, 0);
  zero_empty<T, D>(p, prefix);
  if (at >= stop) {
    settle(false);
    return;
  }
  int ls = unit_at(p, prefix, at);
  while (at < stop) {
    while (prefix[ls + 1] == prefix[ls] || prefix[ls + 1] * p.units_per <= at) ++ls;
    const int places = prefix[ls + 1] - prefix[ls], nb = places - kSetUp;
    const int inside = at - prefix[ls] * p.units_per;
    const int uh = inside / places, v0 = inside - uh * places;            // (head, group), and how far into it
    const int v1 = min(places, v0 + (stop - at));
    const int b0 = max(v0 - kSetUp, 0), b1 = max(v1 - kSetUp, 0);         // first pair, and the one behind the last
    const int begin = at - v0;
    at += v1 - v0;
    if (b0 == b1) continue;
    const int head = p.groups == 1 ? uh : uh / p.groups, group = uh - head * p.groups;
    if (tid == 0 && b0 > 0 && !p.whole_units) {
      // a unit's parts: of the run with its first pair, of the next one (which leads the join), and on to the one with its last
      const int first = cut.of(begin + kSetUp);
      if (first == (int)blockIdx.x - 1) p.lead[blockIdx.x] = make_int2(ls * p.units_per + uh, cut.of(begin + places - 1) - first + 1);
    }
    const int layer = ls / p.table.n_seqs, seq = ls - layer * p.table.n_seqs;
    const int len = unit_len(p.table, p.pool, ls);
    const int col0 = group * COLS, ncols = min(COLS, p.cols - col0);
    // this warp's queries: columns w, w + 8, ...  Asked for before the keys, behind which they would have to wait
    constexpr int E = D / 32;          // a lane's elements
    float xq[NT][E];
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      const int col = warp + y * kAttWarps;
#pragma unroll
      for (int i = 0; i < E; ++i) xq[y][i] = 0.f;
      if (col < ncols) {
        const int gi = p.n_rows == 1 ? col0 + col : (col0 + col) / p.n_rows, r = (col0 + col) - gi * p.n_rows;
        load_elements<E>(reinterpret_cast<const T*>(p.q.ptr) + (int64_t)layer * p.q.sl + (int64_t)seq * p.q.ss +
                             (int64_t)(head * p.hn + gi) * p.q.sh + (int64_t)r * p.q.st + lane * E,
                         xq[y]);
      }
    }
    const int32_t* row = p.table.pages + (int64_t)ls * p.table.max_pages;
    const int sh = p.per_shift;
    int koff[KH], voff[2];              // where this lane's bytes of a K row and of the V rows of two tokens lie in a stage
    {
      const int r = token_of<D>(g);
#pragma unroll
      for (int h = 0; h < KH; ++h) koff[h] = r * D + (D == 128 ? (c + 4 * h) ^ r : c ^ (r >> 1)) * 16;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = token_of<D>(2 * c + i);
        voff[i] = kSlot + t * D + (D == 128 ? (g ^ t) * 16 : ((g >> 1) ^ (t >> 1)) * 16 + (g & 1) * 8);
      }
    }
    // this warp's pairs are b0 + warp + 8 n.  Lane i knows the pages and the scales of the i-th of 32 at a time; the next 32 are
    // looked up while these are computed
    const int n_it = b0 + warp < b1 ? (b1 - b0 - warp + kAttWarps - 1) / kAttWarps : 0;
    auto block_of = [&](int n, int x) { return 2 * (b0 + warp + n * kAttWarps) + x; };
    auto look_up = [&](int n, int x) {          // a page outside the pool, and a block behind the last token: -1
      const int blk = block_of(n, x);
      const int page = n < n_it && blk * kPagedBlock < len ? __ldg(row + (blk >> sh)) : -1;
      return page < p.pool.n_pages ? page : -1;
    };
    auto scales_of = [&](int n, int x, int page) {
      if (page < 0) return make_float2(-1.f, 0.f);
      const int64_t at_block = (((int64_t)page * p.pool.heads + head) << sh) + (block_of(n, x) & ((1 << sh) - 1));
      return make_float2(__ldg(p.pool.ks + at_block), __ldg(p.pool.vs + at_block));
    };
    int page[2], page_next[2];
    float2 scales[2], scales_next[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      page[x] = look_up(lane, x);
      page_next[x] = -1;
      scales_next[x] = make_float2(-1.f, 0.f);
    }
    // K or V of pair n on its way: the lane that knows its pages sends for it
    auto fetch = [&](int n, bool next, int v) {
      if (lane == (n & 31)) {
        const int pg[2] = {next ? page_next[0] : page[0], next ? page_next[1] : page[1]};
        uint64_t* bar = full + v;
        const int blocks = (pg[0] >= 0) + (pg[1] >= 0);
        if (blocks) ptx::mbar_expect_tx(bar, blocks * kHalf);
        else ptx::mbar_arrive(bar);
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (pg[x] >= 0)
            ptx::tma_load_3d(ring + v * kSlot + x * kHalf, v ? &vmap : &kmap, bar, 0, head * p.pool.ps + (block_of(n, x) & ((1 << sh) - 1)) * kPagedBlock, pg[x]);
      }
    };
    if (n_it > 0) {
      if ((int)blockIdx.x != p.withhold) fetch(0, false, 0);
      fetch(0, false, 1);
    }
    int owed = 0;                       // copies that a wait which gave up has left: 1 the keys', 2 the values', 4 the next keys'
#pragma unroll
    for (int x = 0; x < 2; ++x) scales[x] = scales_of(lane, x, page[x]);
    // ---- queries -> fragments ----
#pragma unroll
    for (int y = 0; y < NT; ++y) {
      const int col = warp + y * kAttWarps;
      float (&x)[E] = xq[y];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      // power of two that brings the largest element into [2^14, 2^15); an infinite or NaN row goes through as it is
      int e = 0;
      if (amax > 0.f && amax < CUDART_INF_F) e = min(max(14 - ilogbf(amax), -126), 126);
      const float up = __int_as_float((127 + e) << 23);
      const float down = __int_as_float((127 - e) << 23);
      // element d sits in k-step (d / 64) * 4 + (d % 16) / 4 of the lanes with (d % 64) / 16 as their place in the quad
      const int d0 = lane * E;
      const int ks = (d0 / 64) * 4 + (d0 % 16) / 4, owner = (col & 7) * 4 + (d0 % 64) / 16;
      float sum = 0.f;
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
          sum += got.x + got.y;
        }
        uint2* to = sq + ((pc * NT + (col >> 3)) * KS + ks) * 32 + owner;
        if constexpr (E == 4) *to = make_uint2(h[0], h[1]);
        else reinterpret_cast<uint32_t*>(to)[(d0 % 4) / 2] = h[0];
      }
      if constexpr (kOffset) {
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      }
      if (lane == 0) {
        sfac[col] = amax < CUDART_INF_F ? p.scale * down : CUDART_NAN_F;
        scorr[col] = kOffset ? sum * 128.f : 0.f;
      }
    }
    __syncthreads();
    float fac[NT][2], corr[NT][2];
    int lim[NT][2];                     // tokens that a column sees
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int col = 8 * t + 2 * c + i;
        fac[t][i] = sfac[col];
        corr[t][i] = scorr[col];
        lim[t][i] = col < ncols ? len - p.n_rows + 1 + (p.n_rows == 1 ? 0 : (col0 + col) % p.n_rows) : 0;
      }
    float o[KS][NT][4], m[NT][2], l[NT][2];
    float vinv = 0x1p126f;              // O is in units of 1 / vinv, a power of two that no scale so far exceeds
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = -CUDART_INF_F;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[k][t][i] = 0.f;
    }
    for (int n = 0; n < n_it; ++n) {
      if ((n & 31) == 0 && n) {
#pragma unroll
        for (int x = 0; x < 2; ++x) { page[x] = page_next[x]; scales[x] = scales_next[x]; }
      }
      if ((n & 31) == 8) {
#pragma unroll
        for (int x = 0; x < 2; ++x) page_next[x] = look_up((n & ~31) + 32 + lane, x);
      }
      if ((n & 31) == 20) {
#pragma unroll
        for (int x = 0; x < 2; ++x) scales_next[x] = scales_of((n & ~31) + 32 + lane, x, page_next[x]);
      }
      float ks_b[2], vs_b[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        ks_b[x] = __shfl_sync(0xffffffffu, scales[x].x, n & 31);
        vs_b[x] = __shfl_sync(0xffffffffu, scales[x].y, n & 31);
      }
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(full, phase, abort_flag, p.wait_cycles))) {      // the warp gives up as one
        owed = 3;
        break;
      }
      // ---- scores of both blocks ----
      float sc[2][NT][4];
#pragma unroll
      for (int h = 0; h < KH; ++h) {
        uint4 kr[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 2; ++r) kr[x][r] = *reinterpret_cast<const uint4*>(ring + koff[h] + x * kHalf + r * 8 * D);
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4) {
          const int k = 4 * h + k4;
          uint32_t a[2][4];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint4 &r0 = kr[x][0], &r1 = kr[x][1];
            const uint32_t w0 = prepare_codes<FMT>(k4 == 0 ? r0.x : k4 == 1 ? r0.y : k4 == 2 ? r0.z : r0.w);
            const uint32_t w1 = prepare_codes<FMT>(k4 == 0 ? r1.x : k4 == 1 ? r1.y : k4 == 2 ? r1.z : r1.w);
            a[x][0] = kOffset ? offset_to_half2<0>(w0) : codes_to_half2<FMT, 0>(w0);
            a[x][1] = kOffset ? offset_to_half2<0>(w1) : codes_to_half2<FMT, 0>(w1);
            a[x][2] = kOffset ? offset_to_half2<1>(w0) : codes_to_half2<FMT, 1>(w0);
            a[x][3] = kOffset ? offset_to_half2<1>(w1) : codes_to_half2<FMT, 1>(w1);
          }
#pragma unroll
          for (int pc = 0; pc < NP; ++pc)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint2 qf = sq[((pc * NT + t) * KS + k) * 32 + lane];
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                if (k == 0 && pc == 0) mma16816_first(sc[x][t], a[x], qf);
                else mma16816(sc[x][t], a[x], qf);
              }
            }
        }
      }
      __syncwarp();                     // every lane has read the keys
      const bool more = n + 1 < n_it, crosses = (n & 31) == 31;
      if (more) fetch(n + 1, crosses, 0);
      // ---- softmax weights ----
      const int t0 = block_of(n, 0) * kPagedBlock;
      const bool masked = ks_b[0] == -1.f || ks_b[1] == -1.f || t0 + 2 * kPagedBlock > len - p.n_rows + 1;
      float high[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) sc[x][t][i] = (kOffset ? fmaf(sc[x][t][i], 16777216.f, -corr[t][i & 1]) : sc[x][t][i]) * (ks_b[x] * fac[t][i & 1]);
      }
      if (masked) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (ks_b[x] == -1.f || t0 + x * kPagedBlock + token_of<D>(g) + (i >> 1) * 8 >= lim[t][i & 1]) sc[x][t][i] = -CUDART_INF_F;
      }
      bool rise = false;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          high[t][i] = fmaxf(fmaxf(sc[0][t][i], sc[0][t][i + 2]), fmaxf(sc[1][t][i], sc[1][t][i + 2]));
          rise |= high[t][i] > m[t][i] + kAttLazy;
        }
      if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = high[t][i];
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
      float ref[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) ref[t][i] = m[t][i] == -CUDART_INF_F ? 0.f : m[t][i];
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(full + 1, phase, abort_flag, p.wait_cycles))) {
        owed = more ? 6 : 2;
        break;
      }
      phase ^= 1;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // a block's scale counts relative to the largest so far (in fp32 itself, large values would overflow before they are divided by
        // the weights' sum).  One piece: it joins the weights, unless it is much smaller (the weights would run out of fp16's range) or
        // the block is masked; then, and for two pieces always, it is applied to the block's product
        float ratio = vs_b[x] * vinv;                // exact
        if (ratio > 1.f) {                           // (not for a NaN)
          const uint32_t to = min((__float_as_uint(vs_b[x]) & 0x7F800000u) + 0x00800000u, 0x7E800000u);   // the next power of two
          const float now = __uint_as_float(0x7F000000u - to), f = now * __uint_as_float(0x7F000000u - __float_as_uint(vinv));
          vinv = now;
          ratio = vs_b[x] * vinv;
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[k][t][i] *= f;
        }
        const bool joined = NP == 1 && !masked && ratio >= 0.00390625f;
        const float wfac = joined ? ratio * kAttPScale : kAttPScale;
        uint2 pf[NT][NP];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pow2(sc[x][t][i] - ref[t][i & 1]);
          l[t][0] += w[0] + w[2];
          l[t][1] += w[1] + w[3];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] *= wfac;
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
        uint32_t vr[4][VW];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint8_t* src = ring + voff[r & 1] + x * kHalf + (r >> 1) * 8 * D;
          if constexpr (VW == 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(src);
            vr[r][0] = v.x; vr[r][1] = v.y; vr[r][2] = v.z; vr[r][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(src);
            vr[r][0] = v.x; vr[r][1] = v.y;
          }
        }
        if (FMT == SPINDLEKV_PAGED_E4M3 && masked) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int q = 0; q < VW; ++q) vr[r][q] = without_nan(vr[r][q]);
        }
        // elements 4 q + 2 y and + 1 of the lane's piece: tokens of columns 2c, 2c+1 in one word, 2c+8, 2c+9 in the other
        auto operand = [&](int q, int y, uint32_t (&a)[4]) {
          uint32_t w[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) w[r] = prepare_codes<FMT>(vr[r][q]);
          const uint32_t lo = __byte_perm(w[0], w[1], y ? 0x7362 : 0x5140), hi = __byte_perm(w[2], w[3], y ? 0x7362 : 0x5140);
          a[0] = codes_to_half2<FMT, 0>(lo);
          a[1] = codes_to_half2<FMT, 1>(lo);
          a[2] = codes_to_half2<FMT, 0>(hi);
          a[3] = codes_to_half2<FMT, 1>(hi);
        };
        if (joined) {
#pragma unroll
          for (int q = 0; q < VW; ++q)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t a[4];
              operand(q, y, a);
#pragma unroll
              for (int t = 0; t < NT; ++t) mma16816(o[2 * q + y][t], a, pf[t][0]);
            }
        } else {
          float svc[NT][2];      // a column that sees nothing of the block takes nothing from it, not even a NaN
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) svc[t][i] = masked && t0 + x * kPagedBlock >= lim[t][i] ? 0.f : ratio;
#pragma unroll
          for (int q = 0; q < VW; ++q)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t a[4];
              operand(q, y, a);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                float acc[4];
                mma16816_first(acc, a, pf[t][0]);
                if constexpr (NP == 2) mma16816(acc, a, pf[t][1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[2 * q + y][t][i] = fmaf(svc[t][i & 1], acc[i], o[2 * q + y][t][i]);
              }
            }
        }
      }
      __syncwarp();                     // and the values
      if (more) fetch(n + 1, crosses, 1);
    }
    // ---- the warps' results meet, where the ring was ----
    __syncthreads();
    if (*abort_flag) {
      // give up, but not before what is still on its way has arrived (within the default bound)
      if (owed & 1) ptx::mbar_wait(full, phase, abort_flag + 1, kDefaultMbarWaitCycles);
      if (owed & 2) ptx::mbar_wait(full + 1, phase, abort_flag + 1, kDefaultMbarWaitCycles);
      if (owed & 4) ptx::mbar_wait(full, phase ^ 1, abort_flag + 1, kDefaultMbarWaitCycles);
      if (!p.whole_units && tid == 0) p.lead[blockIdx.x] = make_int2(-2, 0);
      settle(true);
      return;
    }
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
    const float unit = __uint_as_float(0x7F000000u - __float_as_uint(vinv)) / kAttPScale;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)   // elements d, d + 1 of column 2c + i
          *reinterpret_cast<float2*>(so + (warp * COLS + 8 * t + 2 * c + i) * OP + g * (D / 8) + 2 * k) = make_float2(o[k][t][i] * unit, o[k][t][i + 2] * unit);
    __syncthreads();
    settle(false);
    const bool whole = b0 == 0 && b1 == nb;
    // what is left for the join: a unit that began in an earlier run is this run's first, one that begins here and goes on its last
    const int64_t place = (int64_t)(2 * blockIdx.x + (b0 == 0 ? 1 : 0)) * p.part_cols;
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
        *reinterpret_cast<float4*>(p.part + (place + col) * D + d) = sum;
        if (d == 0) p.stat[place + col] = make_float2(top, den);
      }
    }
    ptx::fence_proxy_async();
    __syncthreads();          // the shared memory is free for the next segment's copies
  }
}

// Joins the parts of a unit: block (j, x) takes 16 / TURNS columns of the unit that run j is the first to continue.  TURNS warps to a
// column, each with every TURNS-th run; the order of the sums is the order of the runs.  Four for few columns, whose units are cut into many
// parts; one for more than 16, of which there are many and in few parts.
constexpr int kJoinThreads = 512;

template <typename T, int D, int TURNS>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(AttendParams p, int cols_per_unit) {
  constexpr int E = D / 32, COLS = kJoinThreads / 32 / TURNS, PASS = 16 * TURNS, ST = (PASS + 31) / 32;
  __shared__ float so[TURNS][COLS][D];
  __shared__ float sden[COLS];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    bool gave_up = false;
    for (int r = threadIdx.x; r < (int)gridDim.x; r += kJoinThreads) gave_up |= p.lead[r].x == -2;
    gave_up = __syncthreads_or(gave_up);
    if (threadIdx.x == 0) p.hdr[kHdrStatus] = gave_up ? SPINDLEKV_TIMEOUT : SPINDLEKV_OK;
  }
  const int run = blockIdx.x;
  const int2 lead = p.lead[run];
  const int unit = lead.x, n = lead.y;       // parts: of the run before, in which the unit begins, of this one, and so on
  if (unit < 0) return;
  const int ls = unit / p.units_per, uh = unit - ls * p.units_per, head = uh / p.groups, group = uh - head * p.groups;
  const int layer = ls / p.table.n_seqs, seq = ls - layer * p.table.n_seqs;
  const int col0 = group * cols_per_unit, ncols = min(cols_per_unit, p.cols - col0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, which = warp % COLS, turn = warp / COLS;
  const int col = blockIdx.y * COLS + which;
  const bool mine = col < ncols;
  auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * (run - 1) + 1 : 2 * (run - 1 + i)) * p.part_cols + col; };
  if (mine) {
    float num[E], den = 0.f, top = -CUDART_INF_F;
#pragma unroll
    for (int e = 0; e < E; ++e) num[e] = 0.f;
    // PASS parts at a time, 16 to a warp, all of them asked for at once; the weights are formed meanwhile
    for (int i0 = 0; i0 < n; i0 += PASS) {
      float v[16][E];
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (i0 + TURNS * k + turn < n) load_elements<E>(p.part + slot(i0 + TURNS * k + turn) * D + lane * E, v[k]);
      float2 st[ST];
#pragma unroll
      for (int h = 0; h < ST; ++h) st[h] = 32 * h + lane < PASS && i0 + 32 * h + lane < n ? p.stat[slot(i0 + 32 * h + lane)] : make_float2(-CUDART_INF_F, 0.f);
      float high = top;
#pragma unroll
      for (int h = 0; h < ST; ++h) high = fmaxf(high, st[h].x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
      const float old = top == high ? 1.f : pow2(top - high);
      top = high;
      den *= old;
#pragma unroll
      for (int e = 0; e < E; ++e) num[e] *= old;
      float f[ST];
#pragma unroll
      for (int h = 0; h < ST; ++h) {
        f[h] = st[h].x == top ? 1.f : pow2(st[h].x - top);
        den = fmaf(f[h], st[h].y, den);
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float w = __shfl_sync(0xffffffffu, f[TURNS * k / 32], (TURNS * k + turn) & 31);
        if (i0 + TURNS * k + turn < n) {
#pragma unroll
          for (int e = 0; e < E; ++e) num[e] = fmaf(w, v[k][e], num[e]);
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
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) sum += so[i][which][d];
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


size_t paged_workspace_bytes(const spindlekv_page_pool& pool) {
  return kHeaderBytes + kAttPartRows * (pool.head_dim * sizeof(float) + sizeof(float2)) + kAttMaxRuns * sizeof(int2);
}

template <typename T, int D>
static spindlekv_status launch_join(const AttendParams& p, int runs, int cols_per_unit, cudaStream_t st) {
  const int cols = std::min(cols_per_unit, p.cols), per_block = cols <= 16 ? 4 : 16;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(runs, ceil_div(cols, per_block));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_PAGED_ATTEND, st);
  return cudaLaunchKernelEx(&cfg, per_block == 4 ? paged_join_kernel<T, D, 4> : paged_join_kernel<T, D, 1>, p, cols_per_unit) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

template <typename T, int FMT, int D, int NT>
static spindlekv_status launch_attend(AttendParams& p, const CUtensorMap& kmap, const CUtensorMap& vmap, int max_len, cudaStream_t st) {
  static int resident[kMaxDevices] = {};
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  constexpr int NP = sizeof(T) == 4 ? 2 : 1, COLS = 8 * NT;
  const int n_ls = p.table.n_layers * p.table.n_seqs;
  auto kernel = paged_attend_kernel<T, FMT, D, NT>;
  const size_t fixed = 1024 + ring_bytes<D, NT>() + (size_t)kAttWarps * 16 + 16 + (size_t)NP * NT * (D / 16) * 32 * 8 + (size_t)COLS * 4 * (2 + 2 * kAttWarps) + 36 * 4;
  const size_t smem = align_up(fixed + (size_t)(n_ls + 1) * 4, 16);
  // the prefix sums of a usual batch do not change how many blocks fit; with those of thousands of sequences fewer may, and
  // the rest simply follow
  const int slots = resident_blocks(kernel, align_up(fixed + 1024, 16), resident, dev);
  if (slots <= 0) return SPINDLEKV_CUDA;
  // a run of fewer pairs than there are warps leaves warps idle
  const int64_t capacity = (int64_t)p.table.max_pages * p.pool.ps;
  const int64_t line = (int64_t)n_ls * p.units_per * ceil_div((int)std::min<int64_t>(max_len, capacity), 2 * kPagedBlock);   // pairs
  if ((int64_t)n_ls * p.units_per * ((capacity + 2 * kPagedBlock - 1) / (2 * kPagedBlock) + kSetUp) > 0x7FFFFFFF) return SPINDLEKV_UNSUPPORTED;
  // Short units (two pairs per warp at most) gain nothing from being split: a block for each, and no second kernel (190 tokens, two KV
  // heads: 5.4 us in place of 6.0).  Whatever the lengths turn out to be, both ways serve them
  const int64_t units = (int64_t)n_ls * p.units_per;
  p.whole_units = line <= units * 2 * kAttWarps && units <= 0xFFFF;
  const int runs = p.whole_units ? (int)units : (int)std::min<int64_t>(std::min(slots, kAttMaxRuns), std::max<int64_t>((line + kAttWarps - 1) / kAttWarps, 1));
  // both kernels may be made ready while the one before them on the stream still runs; they wait for it before they touch memory
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(runs);
  cfg.blockDim = dim3(kAttThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  {
    LaunchScope ls(KC_PAGED_ATTEND, st);
    if (cudaLaunchKernelEx(&cfg, kernel, kmap, vmap, p) != cudaSuccess) return SPINDLEKV_CUDA;
  }
  if (p.whole_units) return SPINDLEKV_OK;
  return launch_join<T, D>(p, runs, COLS, st);
}

template <typename T, int FMT, int D>
static spindlekv_status launch_columns(AttendParams& p, int max_len, cudaStream_t st) {
  if constexpr (sizeof(T) == 2 && D == 128) {
    int runs = 0;
    spindlekv_status status = SPINDLEKV_OK;
    if (paged_attend_tiles(p, FMT, max_len, st, &runs, &status)) return status == SPINDLEKV_OK ? launch_join<T, D>(p, runs, p.part_cols, st) : status;
  }
  CUtensorMap kmap, vmap;
  const int rows = p.pool.heads * p.pool.ps;
  if (!make_code_map(&kmap, p.pool.kc, D, rows, p.pool.n_pages, kPagedBlock) || !make_code_map(&vmap, p.pool.vc, D, rows, p.pool.n_pages, kPagedBlock))
    return SPINDLEKV_CUDA;
  p.part_cols = kAttCols;
  const int nt = column_tiles(p.cols);
  p.groups = ceil_div(p.cols, 8 * nt);
  p.units_per = p.pool.heads * p.groups;
  if (nt == 1) return launch_attend<T, FMT, D, 1>(p, kmap, vmap, max_len, st);
  if (nt == 2) return launch_attend<T, FMT, D, 2>(p, kmap, vmap, max_len, st);
  return launch_attend<T, FMT, D, 4>(p, kmap, vmap, max_len, st);
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
  p.hdr = static_cast<uint32_t*>(ws);
  const Tuning tune = current_tuning();
  p.wait_cycles = tune.mbar_wait_cycles;
  p.withhold = tune.paged_withhold;
  p.stat = reinterpret_cast<float2*>(p.part + kAttPartRows * pool.head_dim);
  p.lead = reinterpret_cast<int2*>(p.stat + kAttPartRows);
  return q.dtype == SPINDLEKV_BF16 ? launch_format<__nv_bfloat16>(p, pool.format, max_len, st) : launch_format<float>(p, pool.format, max_len, st);
}

}  // namespace skv
