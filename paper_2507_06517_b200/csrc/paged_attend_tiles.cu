// Attention of many new rows over the 8-bit paged cache: 17 to 128 (query head, row) columns per KV head, bf16, d = 128.
//
// Bound: the cached bytes once, as for few columns; but there the codes are widened to fp16 in registers for every eight warps' worth of
// columns, and from two column tiles on that and the exponentials leave the memory idle.  Here a tile of 128 tokens is widened once, into
// shared memory, for all columns, and the 5th-generation tensor cores multiply it out of there:
//     S^T [tokens x columns] = K Q^T          A = K  [tokens][d]    (d contiguous)       B = Q [columns][d]
//     O^T [d x columns]     += V^T P          A = V  [tokens][d]    (read transposed)    B = P [tokens][columns] (read transposed)
// so that K, V and P are stored the way they arise, token by token, and both products have 128 rows whatever the number of columns.
// The numbers are those of the kernel for few columns: codes exact in fp16, queries scaled by a power of two (exact), p <= 2^8 by a
// running reference that moves when a score exceeds it by 8, block scales of V joined with the weights (relative to a power of two above
// all scales so far) before their one rounding to fp16; m, the sums and O are fp32.  Where a scale is less than 2^-8 of that power, the
// weights would run out of fp16's range, for a value perhaps that has no weight or that a row does not even see.  Such a tile's values
// are multiplied in groups of blocks of like scales (a block is a K step of the product), each relative to a power of two of its own and into
// an accumulator of its own, which the weights' warps add to O in fp32.
//
// Roles (one block per SM).  One warp asks for the codes (TMA, a page at a time, a ring of K and V tiles); four widen them; two issue
// the products, one each, the keys' two tiles ahead of the values'; sixteen turn scores into weights: a thread has a token and a quarter of
// the columns, so that only what happens rarely, a new reference, needs the other tokens.  A tile's scores are read before the weights of
// the tile before are given away, because such a read waits for the products that are under way.
//
// Split.  The line of all units' tiles is cut into equal runs, one per SM, and the parts of a unit are joined as for few columns.
//
// Measured (4 sequences x 16384 tokens, 8 KV heads, int8; beside it the kernel for few columns, which reads the codes once per 32 columns): 32
// columns 49 us (64), 64 columns 73 (101), 128 columns 124 (179); 6 x 26000 tokens, 32 columns 97 us (117), i.e. 3.4 TB/s.  Bound by the
// weights' warps: of 2000 cycles per tile at 32 columns (memory would allow 1450) they wait for 500; issue slots are 50% busy, the products
// take 45 cycles per instruction (360 of 8 steps), widening 600 per tile of codes.  A unit's beginning and end are 7 us, its first tile among them.
// The way out for uneven tiles costs the others registers (48.2, 71, 118.5 without it); with a block of 2^40 in front of every sequence, against which
// all later tiles are uneven (one group each), 75, 100 and 145 us, with four sizes in turn (four groups) 140, 177 and 237.
// Tried: fewer and wider warps for the weights (eight: 60 us at 32 columns), two groups of them that take turns at the tiles (73), two tiles at a
// time (53, as one at a time then), eight widening warps (50), one thread issuing both products (65), a box of 16 tokens per copy (180 cycles per
// copy instruction).
#include <algorithm>

#include "paged_attend.cuh"

namespace skv {

constexpr int kTile = 128;             // tokens
constexpr int kTileSetUp = 6;          // places of a unit's beginning and end, which take 7 us (2: 54 us for 4 x 16384 tokens and 32 columns, 4: 52.6, 6: 51.8)
constexpr int kSoftWarps = 16, kWidenWarps = 4, kAskWarp = kSoftWarps, kScoreWarp = kAskWarp + 1, kValueWarp = kScoreWarp + 1, kWidenFirst = kValueWarp + 1;
constexpr int kTilesThreads = 32 * (kWidenFirst + kWidenWarps);
constexpr float kTileEven = 0.00390625f;   // smallest scale, in units of the power of two above the largest, that joins the weights
constexpr int kRawBytes = kTile * 128, kWideBytes = 2 * kRawBytes;

__device__ __forceinline__ void warps_meet(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ bool warps_any(int id, int threads, bool x) {
  uint32_t y;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(y) : "r"((uint32_t)x), "r"(id), "r"(threads) : "memory");
  return y != 0;
}
// Eight values per lane -> each of the eight reduced over the warp's lanes; lane i gets the one of number reduced_by(i).  Half of the values
// change hands at each of the first three steps: 9 shuffles in place of 40.
__device__ __forceinline__ int reduced_by(int lane) { return (lane >> 2 & 4) | (lane >> 2 & 2) | (lane >> 2 & 1); }
template <typename Op>
__device__ __forceinline__ float reduce_eight(const float* v, int lane, Op op) {
  float a[4], b[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = op(lane & 16 ? v[i + 4] : v[i], __shfl_xor_sync(0xffffffffu, lane & 16 ? v[i] : v[i + 4], 16));
#pragma unroll
  for (int i = 0; i < 2; ++i) b[i] = op(lane & 8 ? a[i + 2] : a[i], __shfl_xor_sync(0xffffffffu, lane & 8 ? a[i] : a[i + 2], 8));
  float c = op(lane & 4 ? b[1] : b[0], __shfl_xor_sync(0xffffffffu, lane & 4 ? b[0] : b[1], 4));
  c = op(c, __shfl_xor_sync(0xffffffffu, c, 2));
  return op(c, __shfl_xor_sync(0xffffffffu, c, 1));
}

template <int N>
struct TilesSmem {
  static constexpr int kK = 2, kV = N == 32 ? 2 : 1;                        // tiles of keys and of values in fp16, 32 KB each
  static constexpr int kRaw = N == 128 ? 3 : 4;                             // tiles of codes, 16 KB each
  static constexpr int kP = N == 128 ? 1 : 2;                               // buffers of weights; 32 columns each share rows of 64
  static constexpr size_t wide = 0, raw = wide + (kK + kV) * kWideBytes, q = raw + kRaw * kRawBytes, p = q + N * 256;
  static constexpr size_t bars = p + (N == 32 ? 1 : kP * N / 64) * kRawBytes;
  static constexpr int kBars = 2 * kRaw + 2 * kK + 2 * kV + 2 + 2 + 2 + 2 + 5;
  static constexpr size_t words = bars + kBars * 8;                         // abort flags, TMEM address, flags of the raw slots, bound of a wait
  static constexpr size_t groups = (words + 16 * 4 + 15) / 16 * 16;         // [8]
  static constexpr size_t counts = groups + 8 * 8;                          // [kSoftWarps] groups that a warp has read
  static constexpr size_t fm = counts + kSoftWarps * 4;                     // [N] score factor and reference, read two at a time
  static constexpr size_t change = fm + N * 8;                              // [N] factor of what is summed, difference of the references
  static constexpr size_t top = change + N * 8;                             // [N] running maximum
  static constexpr size_t lim = top + N * 4;                                // [N] tokens that a column sees
  static constexpr size_t high = lim + N * 4;                               // [kSoftWarps][32]
  static constexpr size_t sums = high + kSoftWarps * 32 * 4;                // [kSoftWarps][columns of a warp]
  static constexpr size_t scan = sums + 4 * N * 4;                          // [36]
  static constexpr size_t prefix = scan + 36 * 4;                           // [n_ls + 1]
  static constexpr size_t bytes(int n_ls) { return 1024 + prefix + (size_t)(n_ls + 1) * 4; }
};

static_assert(TilesSmem<32>::fm % 16 == 0 && TilesSmem<64>::fm % 16 == 0 && TilesSmem<128>::fm % 16 == 0 && TilesSmem<32>::bars % 1024 == 0 &&
              TilesSmem<64>::bars % 1024 == 0 && TilesSmem<128>::bars % 1024 == 0, "alignment of what is read in 16 bytes, and of the tiles");

// ---- uneven tiles (rare; the loop over the others is to have its registers to itself) ----
// Lanes hold the V scales of the 32 blocks of four tiles.  A scale that is a number, or 0: zeros alone, NaN, no page
__device__ __forceinline__ float number(float scale) { return scale > 0.f && scale < CUDART_INF_F ? scale : 0.f; }
// the next power of two, and 1 / a power of two
__device__ __forceinline__ float power_above(float x) { return __uint_as_float(min((__float_as_uint(x) & 0x7F800000u) + 0x00800000u, 0x7E800000u)); }
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float(0x7F000000u - __float_as_uint(x)); }
// The blocks among `left` that belong together: those within kTileEven of the power of two above the largest scale, and those without a number for
// one, which any power serves
__device__ __forceinline__ uint32_t next_group(float v, uint32_t left, float& power) {
  power = power_above(__uint_as_float(__reduce_max_sync(0xffffffffu, left >> (threadIdx.x & 31) & 1 ? __float_as_uint(v) : 0u)));
  return left & __ballot_sync(0xffffffffu, v == 0.f || v * inverse_power(power) >= kTileEven);
}
// 1 / the power of two of a block's group where its tile is uneven (`lows`: the blocks that are far below the tile's reference), `even` elsewhere; the
// first thread of all writes the groups down, from tile `tile` on
__device__ __noinline__ float group_blocks(float scale, uint32_t lows, float even, int tile, volatile uint64_t* table) {
  const int lane = threadIdx.x & 31;
  const float v = number(scale);
  float mine = even;
  for (int j = 0; j < 4; ++j) {
    uint32_t left = lows >> (8 * j) & 0xFFu ? 0xFFu << (8 * j) : 0u;
    uint64_t groups = 0;
    for (int at = 0; left; at += 8) {
      float power;
      const uint32_t members = next_group(v, left, power);
      if (members >> lane & 1) mine = inverse_power(power);
      groups |= (uint64_t)(members >> (8 * j)) << at;
      left &= ~members;
    }
    if (groups && threadIdx.x == 0) table[(tile + j) & 7] = groups;      // (entries that were cleared when their tiles were done)
  }
  return mine;
}
// Adds the groups' products to O, one after the other as they are done.  (What it needs it finds in shared memory: arguments would be kept in registers
// by the loop that hardly ever comes here: 50.2 and 74.4 us with 32 and 64 columns in place of 49.5 and 72.7.)
template <int N>
__device__ __forceinline__ void add_groups(uint8_t* smem, float scale, float ref, int first, bool begins) {
  using S = TilesSmem<N>;
  constexpr int NC = N * 4 / kSoftWarps;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::words);
  const long long wait_cycles = *reinterpret_cast<const long long*>(smem + S::words + 32);
  uint64_t *done = reinterpret_cast<uint64_t*>(smem + S::bars) + S::kBars - 2, *read = done + 1;
  int* number_done = reinterpret_cast<int*>(smem + S::counts) + warp;
  const uint32_t to = reinterpret_cast<const uint32_t*>(smem + S::words)[2] + 2 * N + (warp >> 2) * NC + ((uint32_t)((warp & 3) * 32) << 16), from = to + N;
  const float v = number(scale);
  for (uint32_t left = 0xFFu << first; left; begins = false) {
    float power;
    left &= ~next_group(v, left, power);
    const int turn = *number_done;
    __syncwarp();
    if (lane == 0) *number_done = turn + 1;
    ptx::mbar_wait(done, turn & 1, abort_flag, wait_cycles);
    __syncwarp();
    ptx::tc_fence_after();
    const float rel = power * inverse_power(ref);  // at most 1
#pragma unroll 1
    for (int c0 = 0; c0 < NC; c0 += 8) {
      uint32_t x[8], o[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
      ptx::tmem_ld_32x8_sync(from + c0, x);
      if (!begins) ptx::tmem_ld_32x8_sync(to + c0, o);
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c] = __float_as_uint(fmaf(__uint_as_float(x[c]), rel, __uint_as_float(o[c])));
      ptx::tmem_st_32x8_sync(to + c0, o);
    }
    ptx::tc_fence_before();
    __syncwarp();
    if (left && lane == 0) ptx::mbar_arrive(read);
  }
}

template <int FMT, int N>
__global__ void __launch_bounds__(kTilesThreads, 1) paged_attend_tiles_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                              const __grid_constant__ CUtensorMap vmap, AttendParams p) {
  using S = TilesSmem<N>;
  using T = __nv_bfloat16;
  constexpr int D = 128, NC = N * 4 / kSoftWarps, CW = 8, AHEAD = N < 128, RAW = S::kRaw, PB = S::kP;
  constexpr int kPNext = N == 32 ? 64 : N / 64 * kRawBytes;                 // bytes from one buffer of weights to the other
  constexpr uint32_t kTmemCols = 4 * N;                                     // two score buffers, O, and a group's product
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* raw_full = reinterpret_cast<uint64_t*>(smem + S::bars);
  uint64_t *raw_empty = raw_full + RAW, *k_full = raw_empty + RAW, *k_empty = k_full + S::kK, *v_full = k_empty + S::kK, *v_empty = v_full + S::kV;
  uint64_t *s_full = v_empty + S::kV, *s_empty = s_full + 2, *p_full = s_empty + 2, *pv_done = p_full + 2, *q_full = pv_done + 2, *o_free = q_full + 1, *drained = o_free + 1,
           *group_done = drained + 1, *group_read = group_done + 1;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::words);   // a wait gave up; and one for the waits after that
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::words) + 2;
  volatile int* n_asked = reinterpret_cast<volatile int*>(smem + S::words) + 3;
  volatile int* holes = reinterpret_cast<volatile int*>(smem + S::words) + 4;    // [kRaw] blocks of the tile are missing
  // [8] groups of the uneven ones among the last tiles: byte i holds the blocks of the i-th, 0 behind the last; 0 for an even tile
  volatile uint64_t* groups = reinterpret_cast<volatile uint64_t*>(smem + S::groups);
  float2* fm = reinterpret_cast<float2*>(smem + S::fm);
  float2* change = reinterpret_cast<float2*>(smem + S::change);
  float* top = reinterpret_cast<float*>(smem + S::top);
  int* lim = reinterpret_cast<int*>(smem + S::lim);
  float* high = reinterpret_cast<float*>(smem + S::high);
  float* sums = reinterpret_cast<float*>(smem + S::sums);
  int* prefix = reinterpret_cast<int*>(smem + S::prefix);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < RAW; ++i) { ptx::mbar_init(raw_full + i, 1); ptx::mbar_init(raw_empty + i, kWidenWarps); }
    for (int i = 0; i < S::kK; ++i) { ptx::mbar_init(k_full + i, kWidenWarps); ptx::mbar_init(k_empty + i, 1); }
    for (int i = 0; i < S::kV; ++i) { ptx::mbar_init(v_full + i, kWidenWarps); ptx::mbar_init(v_empty + i, 1); }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(s_full + i, 1);
      ptx::mbar_init(s_empty + i, kSoftWarps);
      ptx::mbar_init(p_full + i, kSoftWarps);
      ptx::mbar_init(pv_done + i, 1);
    }
    ptx::mbar_init(q_full, kSoftWarps);
    ptx::mbar_init(o_free, kSoftWarps);
    ptx::mbar_init(drained, 2);
    ptx::mbar_init(group_done, 1);
    ptx::mbar_init(group_read, kSoftWarps);
    ptx::fence_barrier_init();
    abort_flag[0] = abort_flag[1] = 0;
    *n_asked = 0;
    for (int i = 0; i < 8; ++i) groups[i] = 0;
    for (int i = 0; i < kSoftWarps; ++i) reinterpret_cast<int*>(smem + S::counts)[i] = 0;
    *reinterpret_cast<long long*>(smem + S::words + 32) = p.wait_cycles;
    ptx::prefetch_tensormap(&kmap);
    ptx::prefetch_tensormap(&vmap);
  }
  // up to here nothing was read or written that an earlier kernel of the stream knows of
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int total = line_prefix<kTile, kTileSetUp>(p, prefix, reinterpret_cast<int*>(smem + S::scan));
  const Runs cut(total * p.units_per, (int)gridDim.x);
  const int first_place = cut.start(blockIdx.x), stop = (int)blockIdx.x < cut.runs ? cut.start(blockIdx.x + 1) : first_place;
  if (tid == 0) p.lead[blockIdx.x] = make_int2(-1, 0);
  __syncthreads();                       // the prefix sums of all warps agree; the barriers are set up
  zero_empty<T, D>(p, prefix);
  if (first_place >= stop) return;
  const int first_ls = unit_at(p, prefix, first_place);
  if (warp == kScoreWarp) {
    ptx::tmem_alloc(tmem_slot, kTmemCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before();
  }
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot, tmem_o = tmem + 2 * N, tmem_group = tmem + 3 * N;

  // every role walks the same segments: tiles [b0, b1) of the nb of unit (ls, head), whose places begin at `begin`
  struct Segment { int ls, head, b0, b1, nb, begin, places; };
  auto segments = [&](auto&& body) {
    int at = first_place, ls = first_ls;
    while (at < stop) {
      while (prefix[ls + 1] == prefix[ls] || prefix[ls + 1] * p.units_per <= at) ++ls;
      Segment g;
      g.ls = ls;
      g.places = prefix[ls + 1] - prefix[ls];
      g.nb = g.places - kTileSetUp;
      const int inside = at - prefix[ls] * p.units_per;
      g.head = inside / g.places;
      const int v0 = inside - g.head * g.places, v1 = min(g.places, v0 + (stop - at));
      g.b0 = max(v0 - kTileSetUp, 0);
      g.b1 = max(v1 - kTileSetUp, 0);
      g.begin = at - v0;
      at += v1 - v0;
      if (g.b0 < g.b1) body(g);
    }
  };
  const int sh = p.per_shift;
  // page of a block, -1 behind the last token.  (Whether it is a page of the pool is asked where it is used: here it has just been asked for.)
  auto page_of = [&](const Segment& g, int blk, int len) {
    return blk < g.b1 * (kTile / kPagedBlock) && blk * kPagedBlock < len ? __ldg(p.table.pages + (int64_t)g.ls * p.table.max_pages + (blk >> sh)) : -1;
  };
  auto in_pool = [&](int page) { return page >= 0 && page < p.pool.n_pages; };

  if (warp == kAskWarp) {
    // ---- the codes, a page or a tile's part of it at a time: lane i asks for a tile's i-th page.  Everywhere the keys are two tiles ahead of the values ----
    const int per = 8 >> sh, group = 4 << sh;      // pages of a tile, tiles of 32 pages
    int item = 0;
    bool ok = true;
    segments([&](const Segment& g) {
      const int len = unit_len(p.table, p.pool, g.ls), n_it = g.b1 - g.b0;
      const int32_t* row = p.table.pages + (int64_t)g.ls * p.table.max_pages;
      auto look_up = [&](int n) {                  // this lane's of the 32 pages from tile n on
        const int at = (g.b0 + n) * per + lane;
        return at < g.b1 * per && at * p.pool.ps < len ? __ldg(row + at) : -1;
      };
      int page[2] = {look_up(0), -1}, page_next = -1;      // the keys', and the values'
      for (int i = 0; i < n_it + 2 && ok; ++i) {
        const int turn = i & (group - 1);
        if (turn == 0 && i) page[0] = page_next;
        if (turn == 1) page_next = look_up(i - 1 + group);
        if (turn == 2) page[1] = page[0];
        for (int v = 0; v < 2; ++v) {
          const int n = i - 2 * v;
          if (n < 0 || n >= n_it) continue;
          const int mine = __shfl_sync(0xffffffffu, page[v], (n & (group - 1)) * per + (lane & (per - 1)));
          const int there = __popc(__ballot_sync(0xffffffffu, lane < per && in_pool(mine)));
          const int slot = item % RAW;
          ok = ok && __all_sync(0xffffffffu, ptx::mbar_wait(raw_empty + slot, ((item / RAW) & 1) ^ 1, abort_flag, p.wait_cycles));
          if (!ok) break;
          const bool ask = item || (int)blockIdx.x != p.withhold;
          if (lane == 0) {
            holes[slot] = there < per;
            *n_asked = item + 1;
            if (ask && there) ptx::mbar_expect_tx(raw_full + slot, there * p.pool.ps * D);
            else if (ask) ptx::mbar_arrive(raw_full + slot);
          }
          __syncwarp();
          if (ask && lane < per && in_pool(mine))
            ptx::tma_load_3d(smem + S::raw + slot * kRawBytes + lane * p.pool.ps * D, v ? &vmap : &kmap, raw_full + slot, 0, g.head * p.pool.ps, mine);
          ++item;
        }
      }
    });
  } else if (warp >= kWidenFirst) {
    // ---- codes -> fp16, in rows of 64 elements (two halves of d), 16-byte pieces swizzled as the products expect them.  Eight lanes take four
    // neighbouring pieces of the rows r and r ^ 5, which swizzling puts into different banks on both sides ----
    // this lane's row of eight, its first of four rows eight apart; piece: of the lower half of a row of codes, in bytes
    const int r = (lane >> 3) ^ ((lane >> 2) & 1) * 5, first_row = (warp - kWidenFirst) * (kTile / kWidenWarps) * 128 + r * 128, xor_r = r << 4, piece = (lane & 3) << 4;
    int item = 0, done[2] = {0, 0};
    segments([&](const Segment& g) {
      const int len = unit_len(p.table, p.pool, g.ls);
      for (int i = g.b0; i < g.b1 + 2; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int n = i - 2 * v;
          if (n < g.b0 || n >= g.b1) continue;
          const int rs = item % RAW, slots = v ? S::kV : S::kK, ws = done[v] % slots, round = done[v] / slots;
          uint64_t *full = (v ? v_full : k_full) + ws, *empty = (v ? v_empty : k_empty) + ws;
          bool ok = ptx::mbar_wait(raw_full + rs, (item / RAW) & 1, abort_flag, p.wait_cycles);
          ok = ptx::mbar_wait(empty, (round & 1) ^ 1, abort_flag, p.wait_cycles) && ok;
          if (__all_sync(0xffffffffu, ok)) {
            const bool clean = FMT == SPINDLEKV_PAGED_E4M3 && v && (holes[rs] || (n + 1) * kTile > len);
            const uint8_t* from = smem + S::raw + rs * kRawBytes + first_row;
            uint8_t* to = smem + S::wide + (ws + (v ? S::kK : 0)) * kWideBytes + first_row;
            constexpr int kPieces = 32 / kWidenWarps;
            uint4 raw[kPieces];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) raw[j] = *reinterpret_cast<const uint4*>(from + (j >> 1) * 1024 + ((piece ^ ((j & 1) << 6)) ^ xor_r));
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
              const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
              uint32_t h[8];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t y = prepare_codes<FMT>(clean ? without_nan(w[k]) : w[k]);
                h[2 * k] = codes_to_half2<FMT, 0>(y);
                h[2 * k + 1] = codes_to_half2<FMT, 1>(y);
              }
              uint8_t* row = to + (j & 1) * kRawBytes + (j >> 1) * 1024;
              *reinterpret_cast<uint4*>(row + ((2 * piece) ^ xor_r)) = make_uint4(h[0], h[1], h[2], h[3]);
              *reinterpret_cast<uint4*>(row + ((2 * piece + 16) ^ xor_r)) = make_uint4(h[4], h[5], h[6], h[7]);
            }
            ptx::fence_proxy_async();
          }
          __syncwarp();
          if (lane == 0) {
            ptx::mbar_arrive(raw_empty + rs);
            ptx::mbar_arrive(full);
          }
          ++item;
          ++done[v];
        }
    });
  } else if (warp == kScoreWarp) {
    // ---- the scores' products; addresses of descriptors count in 16 bytes ----
    constexpr uint32_t idesc = ptx::idesc_f16_f32(kTile, N, false, false);
    const uint32_t issues = ptx::elect_one();
    const uint64_t sk = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::wide)), sq = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::q));
    int n = 0, seg = 0;
    bool ok = true;
    segments([&](const Segment& g) {
      ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(q_full, seg & 1, abort_flag, p.wait_cycles));      // the warp gives up as one
      for (int i = g.b0; i < g.b1 && ok; ++i) {
        const int slot = n % S::kK, sb = n & 1;
        ok = ptx::mbar_wait(k_full + slot, (n / S::kK) & 1, abort_flag, p.wait_cycles);
        ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(s_empty + sb, ((n >> 1) & 1) ^ 1, abort_flag, p.wait_cycles));
        if (!ok) break;
        ptx::tc_fence_after();
        const uint64_t a = sk + slot * (kWideBytes >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          ptx::umma_f16_elected(tmem + sb * N, a + (((k >> 2) * kRawBytes + (k & 3) * 32) >> 4), sq + (((k >> 2) * (N * 128) + (k & 3) * 32) >> 4), idesc, k ? 1u : 0u, issues);
        if (issues) {
          ptx::umma_commit(s_full + sb);
          ptx::umma_commit(k_empty + slot);
        }
        __syncwarp();
        ++n;
      }
      ++seg;
    });
    if (issues) ptx::umma_commit(drained);
    __syncwarp();
  } else if (warp == kValueWarp) {
    // ---- the values' products ----
    constexpr uint32_t idesc = ptx::idesc_f16_f32(D, N, true, true);
    const uint32_t issues = ptx::elect_one();
    const uint64_t sv = ptx::smem_desc_sw128_mn(ptx::smem_u32(smem + S::wide) + S::kK * kWideBytes, kRawBytes), sp = ptx::smem_desc_sw128_mn(ptx::smem_u32(smem + S::p), kRawBytes);
    int n = 0, seg = 0, read = 0;
    bool ok = true;
    segments([&](const Segment& g) {
      ok = __all_sync(0xffffffffu, ok && (seg == 0 || ptx::mbar_wait(o_free, (seg - 1) & 1, abort_flag, p.wait_cycles)));
      for (int i = g.b0; i < g.b1 && ok; ++i) {
        const int slot = n % S::kV, pb = n & 1;
        ok = ptx::mbar_wait(v_full + slot, (n / S::kV) & 1, abort_flag, p.wait_cycles);
        ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(p_full + pb, (n >> 1) & 1, abort_flag, p.wait_cycles));
        if (!ok) break;
        ptx::tc_fence_after();
        const uint64_t a = sv + slot * (kWideBytes >> 4), b = sp + ((PB == 2 ? pb : 0) * kPNext >> 4);
        uint64_t left = groups[n & 7];
        if (__all_sync(0xffffffffu, left == 0)) {          // (a vote, so that the warp is seen to stay together)
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k) ptx::umma_f16_elected(tmem_o, a + (k * 2048 >> 4), b + (k * 2048 >> 4), idesc, i == g.b0 && k == 0 ? 0u : 1u, issues);
        }
        while (left) {
          const uint32_t blocks = (uint32_t)left & 0xFFu;
          left >>= 8;
#pragma unroll 1
          for (int k = 0; k < kTile / 16; ++k)
            if (blocks >> k & 1) ptx::umma_f16_elected(tmem_group, a + (k * 2048 >> 4), b + (k * 2048 >> 4), idesc, blocks & ((1u << k) - 1u) ? 1u : 0u, issues);
          if (issues) ptx::umma_commit(group_done);
          __syncwarp();
          if (left) {                    // (behind the last group the next tile's weights say that it has been read)
            ok = __all_sync(0xffffffffu, ptx::mbar_wait(group_read, read++ & 1, abort_flag, p.wait_cycles));
            if (!ok) break;
            ptx::tc_fence_after();
          }
        }
        if (!ok) break;
        if (issues) {
          ptx::umma_commit(pv_done + pb);
          ptx::umma_commit(v_empty + slot);
        }
        __syncwarp();
        ++n;
      }
      ++seg;
    });
    if (issues) ptx::umma_commit(drained);
    __syncwarp();
  } else {
    // ---- scores -> weights.  A thread has token (or, of O, element) `mine` and columns wg * NC .. ----
    const int wg = warp >> 2, quad = warp & 3, mine = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    int tile = 0;
    bool ok = true;
    segments([&](const Segment& g) {
      const int layer = g.ls / p.table.n_seqs, seq = g.ls - layer * p.table.n_seqs;
      const int len = unit_len(p.table, p.pool, g.ls), n_it = g.b1 - g.b0;
      if (tid == 0 && g.b0 > 0) {
        // a unit's parts: of the run with its first tile, of the next one (which leads the join), and on to the one with its last
        const int first = cut.of(g.begin + kTileSetUp);
        if (first == (int)blockIdx.x - 1) p.lead[blockIdx.x] = make_int2(g.ls * p.units_per + g.head, cut.of(g.begin + g.places - 1) - first + 1);
      }
      auto scales_of = [&](int blk, int page) {
        if (!in_pool(page)) return make_float2(-1.f, 0.f);
        const int64_t at = (((int64_t)page * p.pool.heads + g.head) << sh) + (blk & ((1 << sh) - 1));
        return make_float2(__ldg(p.pool.ks + at), __ldg(p.pool.vs + at));
      };
      const int blk0 = g.b0 * 8 + lane;            // this lane knows the scales of a block of four tiles, and looks up the next four's
      int page_next = page_of(g, blk0, len);
      // queries: a warp takes columns warp, warp + 16, ..., two at a time; a lane four elements
#pragma unroll 1
      for (int first = warp; first < N; first += 2 * kSoftWarps) {
        float x[2][4];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int col = first + y * kSoftWarps, gi = col / p.n_rows, r = col - gi * p.n_rows;
          x[y][0] = x[y][1] = x[y][2] = x[y][3] = 0.f;
          if (col < p.cols)
            load_elements<4>(reinterpret_cast<const T*>(p.q.ptr) + (int64_t)layer * p.q.sl + (int64_t)seq * p.q.ss +
                                 (int64_t)(g.head * p.hn + gi) * p.q.sh + (int64_t)r * p.q.st + lane * 4, x[y]);
        }
        if (first == warp) warps_meet(1 + kSoftWarps / 4, kSoftWarps * 32);      // nobody reads the columns' numbers of the segment before any more
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int col = first + y * kSoftWarps;
          float amax = fmaxf(fmaxf(fabsf(x[y][0]), fabsf(x[y][1])), fmaxf(fabsf(x[y][2]), fabsf(x[y][3])));
#pragma unroll
          for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
          // power of two that brings the largest element into [2^14, 2^15)
          int e = 0;
          if (amax > 0.f && amax < CUDART_INF_F) e = min(max(14 - ilogbf(amax), -126), 126);
          const float up = __int_as_float((127 + e) << 23), down = __int_as_float((127 - e) << 23);
          const int piece = (lane & 15) >> 1;
          *reinterpret_cast<uint2*>(smem + S::q + (lane >> 4) * (N * 128) + col * 128 + ((piece ^ (col & 7)) << 4) + (lane & 1) * 8) =
              make_uint2(pack_half2(x[y][0] * up, x[y][1] * up), pack_half2(x[y][2] * up, x[y][3] * up));
          if (lane == 0) {
            fm[col] = make_float2(amax < CUDART_INF_F ? p.scale * down : CUDART_NAN_F, 0.f);
            top[col] = -CUDART_INF_F;
            lim[col] = col < p.cols ? len - p.n_rows + 1 + col % p.n_rows : 0;
          }
        }
      }
      ptx::fence_proxy_async();
      warps_meet(1 + kSoftWarps / 4, kSoftWarps * 32);
      if (lane == 0) ptx::mbar_arrive(q_full);
      float2 sc = make_float2(0.f, 0.f), sc_next = scales_of(blk0, page_next);
      float power = 0.f, factor = 0.f;
      uint32_t missing = 0, lows = 0;              // blocks without a page, and with a scale far below their tile's unit
      bool unset = true;                           // no token so far: the references say nothing yet
      float l[NC], vref = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) l[c] = 0.f;
      // scores of the next tile: read before this tile's weights are given away, since loads wait for the products that are under way.  (With 128
      // columns there are no registers for that.)
      uint32_t s[AHEAD ? NC : CW];
      auto read_scores = [&](int t) {
        ok = ptx::mbar_wait(s_full + (t & 1), (t >> 1) & 1, abort_flag, p.wait_cycles) && ok;
        __syncwarp();
        ptx::tc_fence_after();
#pragma unroll
        for (int c = 0; c < (AHEAD ? NC : 0); c += 8) ptx::tmem_ld_32x8(tmem + (t & 1) * N + wg * NC + c + lanes, s + c);
        if (!AHEAD) return;
        ptx::tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+r"(s[AHEAD ? c : 0]));    // no use of them before the wait
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(s_empty + (t & 1));
      };
      if (AHEAD) read_scores(tile);
      for (int n = 0; n < n_it; ++n, ++tile) {
        if ((n & 3) == 0) {
          sc = sc_next;
          missing = __ballot_sync(0xffffffffu, sc.x == -1.f);
          // O is in units of a power of two above every scale so far: this lane's block's tile's, and the weights' factor
          float most = fmaxf(sc.y, 0.f);
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
#pragma unroll
          for (int o = 8; o < 32; o <<= 1) {
            const float before = __shfl_up_sync(0xffffffffu, most, o);
            if (lane >= o) most = fmaxf(most, before);
          }
          power = most > vref ? power_above(most) : vref;
          float inv = inverse_power(power);
          lows = __ballot_sync(0xffffffffu, number(sc.y) > 0.f && sc.y * inv < kTileEven);
          if (lows) inv = group_blocks(sc.y, lows, inv, tile, groups);
          factor = sc.y * inv * kAttPScale;
          page_next = page_of(g, blk0 + 8 * (n + 4), len);
        }
        if ((n & 3) == 1) sc_next = scales_of(blk0 + 8 * (n + 3), page_next);
        const int block = (n & 3) * 8 + quad * 2 + (lane >> 4);
        const float ks = __shfl_sync(0xffffffffu, sc.x, block), wfac = __shfl_sync(0xffffffffu, factor, block), vnow = __shfl_sync(0xffffffffu, power, block);
        const int t0 = (g.b0 + n) * kTile, t = t0 + mine;
        const uint32_t absent = missing >> ((n & 3) * 8) & 0xFFu;     // blocks of the tile without a page
        const bool masked = absent || t0 + kTile > len - p.n_rows + 1;
        const bool grows = vnow > vref;
        const float vf = vref * inverse_power(vnow);
        vref = vnow;
        auto wait_values = [&](int t) {            // the values' product of tile t is done
          if (t >= 0) ok = ptx::mbar_wait(pv_done + (t & 1), (t >> 1) & 1, abort_flag, p.wait_cycles) && ok;
        };
#pragma unroll
        for (int ch = 0; ch < NC / CW; ++ch) {
          const int col0 = wg * NC + ch * CW;
          float x[CW];
          {
            if (!AHEAD) {
              if (ch == 0) read_scores(tile);
              __syncwarp();
              ptx::tmem_ld_32x8(tmem + (tile & 1) * N + col0 + lanes, s);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < CW; ++c) asm volatile("" : "+r"(s[c]));
              if (ch == NC / CW - 1) {
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(s_empty + (tile & 1));
              }
            }
            float most[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int c = 0; c < CW; c += 2) {
              const float4 f = *reinterpret_cast<const float4*>(fm + col0 + c);
              x[c] = fmaf(__uint_as_float(s[(AHEAD ? ch * CW : 0) + c]), ks * f.x, -f.y);
              x[c + 1] = fmaf(__uint_as_float(s[(AHEAD ? ch * CW : 0) + c + 1]), ks * f.z, -f.w);
            }
            if (masked) {
#pragma unroll
              for (int c = 0; c < CW; ++c)
                if (ks == -1.f || t >= lim[col0 + c]) x[c] = -CUDART_INF_F;
            }
#pragma unroll
            for (int c = 0; c < CW; ++c) most[c & 3] = fmaxf(most[c & 3], x[c]);
            if (warps_any(1 + wg, 128, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) > kAttLazy || grows || unset)) {
              // ---- new references for these columns: their largest score; what is summed so far moves along ----
              wait_values(tile - 1);
              __syncwarp();
              ptx::tc_fence_after();
              const float highest = reduce_eight(x, lane, [](float a, float b) { return fmaxf(a, b); });
              if ((lane & 3) == 0) high[warp * 32 + reduced_by(lane)] = highest;
              warps_meet(1 + wg, 128);
              if (quad == 0 && lane < CW) {
                const float* hs = high + wg * 128 + lane;
                const float was = top[col0 + lane], ref = fm[col0 + lane].y;
                const float now = fmaxf(was, fmaxf(fmaxf(hs[0], hs[32]), fmaxf(hs[64], hs[96])) + ref);
                const float to = now == -CUDART_INF_F ? 0.f : now;
                top[col0 + lane] = now;
                fm[col0 + lane].y = to;
                change[col0 + lane] = make_float2(was == now ? 1.f : was == -CUDART_INF_F ? 0.f : pow2(was - now), ref - to);
              }
              warps_meet(1 + wg, 128);
#pragma unroll
              for (int c = 0; c < CW; ++c) {
                const float2 f = change[col0 + c];
                l[ch * CW + c] *= f.x;
                x[c] += f.y;
              }
              if (n > 0) {
                uint32_t o[CW];
                ptx::tmem_ld_32x8_sync(tmem_o + col0 + lanes, o);
#pragma unroll
                for (int c = 0; c < CW; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * (change[col0 + c].x * vf));
                ptx::tmem_st_32x8_sync(tmem_o + col0 + lanes, o);
              }
            }
          }
          if (ch == 0) wait_values(tile - PB);     // and so has it read this buffer of weights
          uint32_t h[CW / 2];
#pragma unroll
          for (int c = 0; c < CW; c += 2) {
            const float a = pow2(x[c]), b = pow2(x[c + 1]);
            l[ch * CW + c] += a;
            l[ch * CW + c + 1] += b;
            h[c / 2] = pack_half2(a * wfac, b * wfac);
          }
          if (masked) {                            // a column that does not see the token takes nothing from it, not even a NaN
#pragma unroll
            for (int c = 0; c < CW; c += 2)
              h[c / 2] &= (x[c] == -CUDART_INF_F ? 0u : 0xFFFFu) | (x[c + 1] == -CUDART_INF_F ? 0u : 0xFFFF0000u);
          }
          uint8_t* row = smem + S::p + (PB == 2 && N > 32 ? (tile & 1) * kPNext : 0) + (col0 >> 6) * kRawBytes + mine * 128;
          const int piece = ((col0 & 63) >> 3) + (N == 32 ? (tile & 1) * 4 : 0);
#pragma unroll
          for (int c = 0; c < CW; c += 8)
            *reinterpret_cast<uint4*>(row + (((piece + c / 8) ^ (mine & 7)) << 4)) = make_uint4(h[c / 2], h[c / 2 + 1], h[c / 2 + 2], h[c / 2 + 3]);
        }
        unset = unset && absent == 0xFFu;
        ptx::fence_proxy_async();
        if (lows >> ((n & 3) * 8) & 0xFFu) {
          // (the next tile's scores are read afterwards: their registers are what the additions need)
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full + (tile & 1));
          add_groups<N>(smem, sc.y, vref, (n & 3) * 8, n == 0);
          if (tid == 0) groups[tile & 7] = 0;              // (read before the first product)
          if (AHEAD && n + 1 < n_it) read_scores(tile + 1);
        } else {
          if (AHEAD && n + 1 < n_it) read_scores(tile + 1);
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full + (tile & 1));
        }
      }
      // ---- the segment's result ----
      ok = ptx::mbar_wait(pv_done + ((tile - 1) & 1), ((tile - 1) >> 1) & 1, abort_flag, p.wait_cycles) && ok;
      __syncwarp();
      ptx::tc_fence_after();
#pragma unroll
      for (int c = 0; c < NC; c += 8) {
        const float sum = reduce_eight(l + c, lane, [](float a, float b) { return a + b; });
        if ((lane & 3) == 0) sums[warp * NC + c + reduced_by(lane)] = sum;
      }
      warps_meet(1 + wg, 128);
      if (quad == 0 && lane < NC) {
        float* of = sums + warp * NC + lane;
        of[0] = of[0] + of[NC] + of[2 * NC] + of[3 * NC];
      }
      warps_meet(1 + wg, 128);
      const bool whole = g.b0 == 0 && g.b1 == g.nb, write = ok && !*abort_flag;
      const int64_t place = (int64_t)(2 * blockIdx.x + (g.b0 == 0 ? 1 : 0)) * N;
      const float unit = vref / kAttPScale;
      const float* den_of = sums + wg * 4 * NC;
#pragma unroll 1
      for (int c0 = 0; c0 < NC; c0 += CW) {
        uint32_t o[CW];
        __syncwarp();
        ptx::tmem_ld_32x8_sync(tmem_o + wg * NC + c0 + lanes, o);
#pragma unroll
        for (int c = 0; c < CW; ++c) {
          const int col = wg * NC + c0 + c;
          if (col < p.cols && write) {
            const float v = __uint_as_float(o[c]) * unit;
            if (whole) {
              const int gi = col / p.n_rows, r = col - gi * p.n_rows;
              const float den = den_of[c0 + c];
              (reinterpret_cast<T*>(const_cast<void*>(p.out.ptr)) + (int64_t)layer * p.out.sl + (int64_t)seq * p.out.ss +
               (int64_t)(g.head * p.hn + gi) * p.out.sh + (int64_t)r * p.out.st)[mine] = T(den == 0.f ? 0.f : v / den);
            } else {
              p.part[(place + col) * D + mine] = v;
            }
          }
        }
      }
      if (!whole && write && mine < NC && wg * NC + mine < p.cols) p.stat[place + wg * NC + mine] = make_float2(top[wg * NC + mine], den_of[mine]);
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(o_free);
    });
  }
  __syncthreads();
  // all products are done, and with them their arrivals, before the block goes; after a wait that gave up so are the codes that were still on
  // their way (within the default bound)
  if (tid == kScoreWarp * 32) ptx::mbar_wait(drained, 0, abort_flag + 1, kDefaultMbarWaitCycles);
  if (tid == 0 && *abort_flag) {
    for (int item = max(*n_asked - RAW, 0); item < *n_asked; ++item)
      ptx::mbar_wait(raw_full + item % RAW, (item / RAW) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
    p.lead[blockIdx.x] = make_int2(-2, 0);
  }
  __syncthreads();
  if (warp == kScoreWarp) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, kTmemCols);
  }
}

template <int FMT, int N>
static spindlekv_status launch_tiles(AttendParams& p, const CUtensorMap& kmap, const CUtensorMap& vmap, int64_t tiles, cudaStream_t st, int* runs) {
  static int resident[kMaxDevices] = {};
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  auto kernel = paged_attend_tiles_kernel<FMT, N>;
  if (!resident[dev]) {
    int sms = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess) return SPINDLEKV_CUDA;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return SPINDLEKV_CUDA;
    resident[dev] = sms;
  }
  p.part_cols = N;
  *runs = (int)std::min<int64_t>(std::min(resident[dev], kAttPartRows / (2 * N)), std::max<int64_t>(tiles, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(*runs);
  cfg.blockDim = dim3(kTilesThreads);
  cfg.dynamicSmemBytes = TilesSmem<N>::bytes(p.table.n_layers * p.table.n_seqs);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_PAGED_ATTEND, st);
  return cudaLaunchKernelEx(&cfg, kernel, kmap, vmap, p) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

bool paged_attend_tiles(AttendParams& p, int format, int max_len, cudaStream_t st, int* runs, spindlekv_status* status) {
  const int n_ls = p.table.n_layers * p.table.n_seqs, n = p.cols <= 32 ? 32 : p.cols <= 64 ? 64 : 128;
  const int64_t capacity = (int64_t)p.table.max_pages * p.pool.ps;
  const size_t smem = n == 32 ? TilesSmem<32>::bytes(n_ls) : n == 64 ? TilesSmem<64>::bytes(n_ls) : TilesSmem<128>::bytes(n_ls);
  if (p.cols <= 16 || p.cols > 128 || smem > 227 * 1024) return false;   // (16 columns, 4 x 16384 tokens: 44 us in the other kernel, 51 here)
  const int64_t units = (int64_t)n_ls * p.pool.heads, tiles = units * ((std::min<int64_t>(max_len, capacity) + kTile - 1) / kTile);
  // Short units, if the other kernel has a block for each at once (4 sequences of 350 tokens, 8 KV heads: 15.7 us there with 32 columns, 16.1 with
  // 64, 16.2 with 128; here 15.3, 22.2, 35.0.  32 sequences: 31, 60, 108 there; here 30, 45, 72)
  if (max_len <= 4 * kTile && units * ceil_div(p.cols, 32) <= 148) return false;
  // many columns over few tiles, which do not make up for the longer beginning and end (128 columns, one sequence of 1200 tokens: 27 us there, 31
  // here; of 5000: 36 and 37; two of 5000: 48 and 43)
  if (p.cols > 64 && tiles < 200) return false;
  p.groups = 1;
  p.units_per = p.pool.heads;
  if ((int64_t)n_ls * p.units_per * ((capacity + kTile - 1) / kTile + kTileSetUp) > 0x7FFFFFFF) return false;
  p.whole_units = 0;
  CUtensorMap kmap, vmap;
  const int rows = p.pool.heads * p.pool.ps;
  if (!make_code_map(&kmap, p.pool.kc, 128, rows, p.pool.n_pages, p.pool.ps) || !make_code_map(&vmap, p.pool.vc, 128, rows, p.pool.n_pages, p.pool.ps)) {
    *status = SPINDLEKV_CUDA;
    return true;
  }
  const bool i8 = format == SPINDLEKV_PAGED_INT8;
  if (n == 32) *status = i8 ? launch_tiles<SPINDLEKV_PAGED_INT8, 32>(p, kmap, vmap, tiles, st, runs) : launch_tiles<SPINDLEKV_PAGED_E4M3, 32>(p, kmap, vmap, tiles, st, runs);
  else if (n == 64) *status = i8 ? launch_tiles<SPINDLEKV_PAGED_INT8, 64>(p, kmap, vmap, tiles, st, runs) : launch_tiles<SPINDLEKV_PAGED_E4M3, 64>(p, kmap, vmap, tiles, st, runs);
  else *status = i8 ? launch_tiles<SPINDLEKV_PAGED_INT8, 128>(p, kmap, vmap, tiles, st, runs) : launch_tiles<SPINDLEKV_PAGED_E4M3, 128>(p, kmap, vmap, tiles, st, runs);
  return true;
}

}  // namespace skv
