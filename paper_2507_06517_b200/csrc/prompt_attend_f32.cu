// Causal attention of a prompt's rows, fp32, on the bf16 tensor cores.
//
// An fp32 number is the sum of three numbers of 8 bits each, x = x1 + x2 + x3, cut off rather than rounded, so that nothing runs out of range and
// the sum is exact (splitting in the manner of Dekker).  Of the nine products of two such sums the six with the largest factors are formed,
//     x y = x1 y1 + (x1 y2 + x2 y1) + (x2 y2 + x1 y3 + x3 y1) + ... ,
// in rising order into one fp32 accumulator; what is left out is below 2^-24 of |x y| each.  Six products at the bf16 rate are a sixth of it: half a
// tf32 pair's three products would cost the same and keep 22 bits.
//
// A first kernel writes the pieces of q, k and v, three planes each, as bf16 tensors that TMA can read.  Then as
// for bf16, with one row tile of 128 (position, head) rows and 64 keys at a time: their pieces fill the shared memory.  The scores of the next keys are
// multiplied while this one's weights are formed: two buffers of scores and of weights in tensor memory.
//     tensor memory: S [2][64 columns], P [2][3 pieces][32 columns], O [d columns]
// The accumulator cuts off what it adds, always towards zero; over the products of thousands of keys that would be 2^-17 of the result (8.6e-6 at 4000
// tokens).  So O holds one tile at a time, whose largest product comes last, and a warpgroup of its own adds the tiles up in its registers, rounding as
// usual (7e-7).  An infinite value is its first piece, and a weight may have a piece of 0: rows that see one get NaN here, where calls of few rows give the infinity.
// Bound by the products: 6 x (128 x 64 x d) x 2 for 64 keys, 3840 cycles at d = 128 where N = 64 has no full rate (the tensor pipe is 69 % busy at 4096 tokens);
// short sequences by the pieces' way into shared memory, 96 KB of rows and 96 KB for 64 keys.  32 query heads over 8, d = 128: 512 tokens 38 us, 2048 191,
// 4096 640 to 690 (200 to 210 TFLOP/s, 1.2 PFLOP/s of products), of which the pieces are 42.
#include <algorithm>

#include "args.cuh"
#include "prompt_attend.cuh"

namespace skv {

// warps 0-3: scores to weights, 4-7: sums of the tiles
constexpr int kExactThreads = 320, kExactAsk = 8, kExactIssue = 9, kExactKeys = 64;
constexpr int kExactFactors = 4;          // tiles whose factors of what is summed are kept: one that is read, and those that may be ahead of it
constexpr int kExactSlots = 4;            // of the list of items
constexpr int kPieces = 3;

template <int D>
struct ExactSmem {
  static constexpr int kQHalf = kPromptRows * 128, kQPiece = D / 64 * kQHalf;
  static constexpr int kHalf = kExactKeys * 128, kPiece = D / 64 * kHalf, kSlot = kPieces * kPiece;
  static constexpr int kRing = D == 128 ? 1 : 2;                             // slots of keys, and of values
  static constexpr int q = 0, k = kPieces * kQPiece, v = k + kRing * kSlot, stage = v + kRing * kSlot, factors = stage + 4 * 4096, stats = factors + kExactFactors * kPromptRows * 4,
                       bars = stats + kPromptRows * 8;
  static constexpr int kBars = 4 * kRing + 2 + 2 + 1 + 2 + 1 + 2 + 2 * kExactSlots + 1;
  static constexpr int words = bars + kBars * 8;
  static constexpr int items = (words + 32 + 15) / 16 * 16;
  static constexpr int redo = items + kExactSlots * (int)sizeof(PromptItem);
  static constexpr int bytes = 1024 + redo + kPromptMaxItems / 8;
};
static_assert(ExactSmem<128>::bytes <= 227 * 1024 && ExactSmem<64>::bytes > 114 * 1024, "shared memory: one block per SM, which takes all tensor memory");

// x -> three bf16 numbers (upper halves of words) whose sum it is; a NaN or an infinity is the first of them
__device__ __forceinline__ void pieces_of(float x, uint32_t& a, uint32_t& b, uint32_t& c) {
  a = __float_as_uint(x) & 0xFFFF0000u;
  const float r = x - __uint_as_float(a);
  b = __float_as_uint(r) & 0xFFFF0000u;
  c = __float_as_uint(r - __uint_as_float(b)) & 0xFFFF0000u;
}
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __byte_perm(lo, hi, 0x7632); }

struct SplitSource {
  View from;                 // fp32 [layer][seq][head][token][d]
  Batch batch;
  __nv_bfloat16* to;         // [piece][layer][seq] of (head, token) or (token, head), d
  int heads, by_token;       // by_token: the heads of a token lie side by side
  int behind;                // tokens behind the last one that get zeros
};
struct SplitParams { SplitSource t[3]; };
// Memory bounds it (4 bytes in, 6 out for each element); a thread takes four times 8 elements, in the pieces' order, and asks for all of them at once
constexpr int kSplitTurns = 4;

template <int D>
__global__ void __launch_bounds__(256) prompt_pieces_kernel(const __grid_constant__ SplitParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const SplitSource& t = p.t[blockIdx.z];
  const Batch& b = t.batch;
  const int seqs = b.cu ? 1 : b.n_seqs, tokens = b.cu ? b.total_len : b.max_len, ls = blockIdx.y;
  const unsigned items = (unsigned)tokens * t.heads * (D / 8), first = blockIdx.x * (kSplitTurns * 256) + threadIdx.x;
  if (ls >= seqs * b.n_layers) return;
  const int layer = ls / seqs, seq = ls - layer * seqs;
  const int from = b.cu ? max(b.cu[0], 0) : 0, end = b.cu ? min(b.cu[b.n_seqs], b.total_len) : span_of(b, layer, seq).len;
  const int64_t plane = (int64_t)b.n_layers * seqs * items * 8;
  const float* src = reinterpret_cast<const float*>(t.from.ptr) + (int64_t)layer * t.from.sl + (b.cu ? 0 : (int64_t)seq * t.from.ss);
  __nv_bfloat16* dst = t.to + (int64_t)ls * items * 8;
  float x[kSplitTurns][8];
  bool writes[kSplitTurns];
#pragma unroll
  for (int k = 0; k < kSplitTurns; ++k) {
    const unsigned i = first + k * 256, row = i / (D / 8), major = row / (unsigned)(t.by_token ? t.heads : tokens), minor = row - major * (unsigned)(t.by_token ? t.heads : tokens);
    const int token = t.by_token ? major : minor, head = t.by_token ? minor : major;
    writes[k] = i < items && token >= from && token < end + t.behind;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[k][u] = 0.f;
    if (writes[k] && token < end) load8(src + (int64_t)head * t.from.sh + (int64_t)token * t.from.st + i % (D / 8) * 8, x[k]);
  }
#pragma unroll
  for (int k = 0; k < kSplitTurns; ++k) {
    const unsigned i = first + k * 256;
    if (!writes[k]) continue;
    uint32_t w[kPieces][4];
#pragma unroll
    for (int u = 0; u < 8; u += 2) {
      uint32_t y[2][kPieces];
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const float z = x[k][u + v];
        pieces_of(z, y[v][0], y[v][1], y[v][2]);
        if (!(fabsf(z) < CUDART_INF_F)) {
          y[v][0] = z != z ? 0x7FC00000u : __float_as_uint(z);
          y[v][1] = y[v][2] = 0u;
        }
      }
#pragma unroll
      for (int c = 0; c < kPieces; ++c) w[c][u / 2] = upper_halves(y[0][c], y[1][c]);
    }
#pragma unroll
    for (int c = 0; c < kPieces; ++c) *reinterpret_cast<uint4*>(dst + c * plane + (int64_t)i * 8) = make_uint4(w[c][0], w[c][1], w[c][2], w[c][3]);
  }
}

template <int D>
__global__ void __launch_bounds__(kExactThreads, 1) prompt_attend_f32_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                                             const __grid_constant__ CUtensorMap vmap, const __grid_constant__ PromptParams p) {
  using S = ExactSmem<D>;
  using T = float;
  constexpr int KT = kExactKeys, RING = S::kRing, SLOTS = kExactSlots;
  constexpr int kProducts = 6, kFirst[kProducts] = {2, 0, 1, 1, 0, 0}, kSecond[kProducts] = {0, 2, 1, 0, 1, 0};      // pieces, in rising order
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + S::bars);
  uint64_t *k_empty = k_full + RING, *v_full = k_empty + RING, *v_empty = v_full + RING, *q_full = v_empty + RING, *q_empty = q_full + 1, *s_full = q_empty + 1,
           *pv_done = s_full + 2, *p_full = pv_done + 1, *o_read = p_full + 2, *l_full = o_read + 1, *l_empty = l_full + 1, *item_full = l_empty + 1, *item_empty = item_full + SLOTS,
           *drained = item_empty + SLOTS;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::words);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::words) + 2;
  volatile int* any_redo = reinterpret_cast<volatile int*>(smem + S::words) + 3;
  volatile int* asked = reinterpret_cast<volatile int*>(smem + S::words) + 4;    // keys, rows, values
  PromptItem* items = reinterpret_cast<PromptItem*>(smem + S::items);
  uint32_t* redo = reinterpret_cast<uint32_t*>(smem + S::redo);
  float* factors = reinterpret_cast<float*>(smem + S::factors);
  float2* stats = reinterpret_cast<float2*>(smem + S::stats);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < RING; ++i) {
      ptx::mbar_init(k_full + i, 1);
      ptx::mbar_init(k_empty + i, 1);
      ptx::mbar_init(v_full + i, 1);
      ptx::mbar_init(v_empty + i, 1);
    }
    ptx::mbar_init(q_full, 1);
    ptx::mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(s_full + i, 1);
      ptx::mbar_init(p_full + i, 4);          // (two: a warp may be done with the next tile's weights before another is with this one's)
    }
    ptx::mbar_init(pv_done, 1);
    ptx::mbar_init(o_read, 4);
    ptx::mbar_init(l_full, 4);
    ptx::mbar_init(l_empty, 4);
    for (int i = 0; i < SLOTS; ++i) { ptx::mbar_init(item_full + i, 1); ptx::mbar_init(item_empty + i, 9); }
    ptx::mbar_init(drained, 1);
    ptx::fence_barrier_init();
    abort_flag[0] = abort_flag[1] = 0;
    *any_redo = 0;
    asked[0] = asked[1] = asked[2] = 0;
    ptx::prefetch_tensormap(&qmap);
    ptx::prefetch_tensormap(&kmap);
    ptx::prefetch_tensormap(&vmap);
  }
  for (int i = tid; i < kPromptMaxItems / 32; i += kExactThreads) redo[i] = 0;
  // rows that no copy fills (hn does not divide 128) hold zeros
  for (int i = p.pt * p.hn * 8 + tid; i < kPromptRows * 8; i += kExactThreads)
    for (int h = 0; h < kPieces * D / 64; ++h) *reinterpret_cast<uint4*>(smem + S::q + h * S::kQHalf + i * 16) = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  if (warp == kExactIssue) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
    ptx::tc_fence_before();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0), tmem_p = tmem + 128, tmem_o = tmem + 384;

  auto wait = [&](uint64_t* bar, int phase) { return ptx::mbar_wait(bar, phase & 1, abort_flag, p.wait_cycles); };
  int item_no = 0;
  auto next_item = [&](PromptItem& it, bool& ok) {
    const int slot = item_no % SLOTS;
    ok = __all_sync(0xffffffffu, wait(item_full + slot, item_no / SLOTS));
    if (!ok) return false;
    it = items[slot];
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(item_empty + slot);
    ++item_no;
    return it.ls >= 0;
  };
  auto again = [&]() {
    __syncthreads();
    return __syncthreads_and(*any_redo && !*abort_flag) != 0;
  };
  bool ok = true;
  int n_kv = 0, n_q = 0;                  // tiles of keys (and of values) and row tiles so far
  if (warp == kExactAsk) {
    PromptList list(p);
    for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      for (int k = 0; ok; ++k) {
        while (pass && k < kPromptMaxItems && !(redo[k >> 5] >> (k & 31) & 1u)) ++k;
        PromptItem it = {};
        it.ls = -1;
        if (k < kPromptMaxItems) it = list.item(p, k);
        it.careful = pass;
        const int slot = item_no % SLOTS;
        ok = __all_sync(0xffffffffu, wait(item_empty + slot, item_no / SLOTS + 1));
        if (!ok) break;
        if (lane == 0) {
          items[slot] = it;
          ptx::mbar_arrive(item_full + slot);
        }
        __syncwarp();
        ++item_no;
        if (it.ls < 0) break;
        const PromptTiles<1, KT> tiles(p, it);
        if (tiles.most == 0) continue;
        const int layer = it.ls / p.rows.n_seqs, seq = it.ls - layer * p.rows.n_seqs;
        ok = __all_sync(0xffffffffu, wait(q_empty, n_q + 1));
        if (!ok) break;
        if (lane == 0) {
          ptx::mbar_expect_tx(q_full, kPieces * (D / 64) * p.pt * p.hn * 128);
          for (int h = 0; h < kPieces * (D / 64); ++h)
            ptx::tma_load_5d(smem + S::q + h * S::kQHalf, &qmap, q_full, h % (D / 64) * 64, it.head * p.hn, it.base_r + it.blk * p.per_item, p.rows.cu ? 0 : seq,
                             h / (D / 64) * p.rows.n_layers + layer);
          asked[1] = n_q + 1;
        }
        __syncwarp();
        ++n_q;
        auto ask = [&](int v, int tile) {
          const int n = n_kv + tile, at = n % RING;
          uint64_t *full = (v ? v_full : k_full) + at, *empty = (v ? v_empty : k_empty) + at;
          ok = __all_sync(0xffffffffu, ok && wait(empty, n / RING + 1));
          if (!ok) return;
          if (lane == 0) {
            if (v || n || (int)blockIdx.x != p.withhold) {
              ptx::mbar_expect_tx(full, S::kSlot);
              for (int h = 0; h < kPieces * (D / 64); ++h)
                ptx::tma_load_5d(smem + (v ? S::v : S::k) + at * S::kSlot + h * S::kHalf, v ? &vmap : &kmap, full, h % (D / 64) * 64,
                                 it.base_k + (tiles.first + tile) * KT, it.head, p.keys.cu ? 0 : seq, h / (D / 64) * p.keys.n_layers + layer);
            }
            asked[v ? 2 : 0] = n + 1;
          }
          __syncwarp();
        };
        // in the order in which the products let go of the slots: keys are two tiles ahead of the values
        ask(0, 0);
        ask(1, 0);
        if (tiles.most > 1) ask(0, 1);
        for (int t = 1; t < tiles.most && ok; ++t) {
          if (t + 1 < tiles.most) ask(0, t + 1);
          ask(1, t);
        }
        n_kv += tiles.most;
      }
    }
  } else if (warp == kExactIssue) {
    constexpr uint32_t idesc_s = ptx::idesc_bf16_f32(128, KT), idesc_o = ptx::idesc_bf16_f32(128, D) | (1u << 16);
    const uint32_t issues = ptx::elect_one();
    const uint64_t dq = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::q)), dk = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::k)),
                   dv = ptx::smem_desc_sw128_mn(ptx::smem_u32(smem + S::v), S::kHalf);
    for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      PromptItem it;
      while (ok && next_item(it, ok)) {
        int most, even;
        {
          const PromptTiles<1, KT> tiles(p, it);
          most = __shfl_sync(0xffffffffu, tiles.most, 0);
          even = __shfl_sync(0xffffffffu, it.careful ? tiles.even[0] : tiles.most, 0);      // tiles whose values are multiplied here
        }
        if (most == 0) continue;
        auto release = [&](uint64_t* bar) {
          if (issues) ptx::umma_commit(bar);
          __syncwarp();
        };
        auto scores = [&](int n) {            // of tile number n, all items' counted
          const int at = n % RING;
          ok = __all_sync(0xffffffffu, wait(k_full + at, n / RING));
          if (!ok) return;
          ptx::tc_fence_after();
#pragma unroll
          for (int x = 0; x < kProducts; ++x)
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              ptx::umma_f16_elected(tmem + (n & 1) * KT, dq + ((kFirst[x] * S::kQPiece + (k >> 2) * S::kQHalf + (k & 3) * 32) >> 4),
                                    dk + ((at * S::kSlot + kSecond[x] * S::kPiece + (k >> 2) * S::kHalf + (k & 3) * 32) >> 4), idesc_s, x || k ? 1u : 0u, issues);
          release(s_full + (n & 1));
          release(k_empty + at);
        };
        ok = __all_sync(0xffffffffu, wait(q_full, n_q++));
        if (!ok) break;
        scores(n_kv);
        if (most == 1) release(q_empty);
        for (int j = 0; j < most && ok; ++j, ++n_kv) {
          if (j + 1 < most) {
            scores(n_kv + 1);
            if (j + 2 == most) release(q_empty);
          }
          const int at = n_kv % RING;
          ok = wait(v_full + at, n_kv / RING) && ok;
          ok = wait(o_read, n_kv + 1) && ok;               // the tile before has been read
          ok = __all_sync(0xffffffffu, wait(p_full + (n_kv & 1), n_kv >> 1) && ok);
          if (!ok) break;
          ptx::tc_fence_after();
          if (j < even) {
#pragma unroll
            for (int x = 0; x < kProducts; ++x)
#pragma unroll
              for (int k = 0; k < KT / 16; ++k)
                ptx::umma_bf16_ts_elected(tmem_o, tmem_p + (n_kv & 1) * 96 + kFirst[x] * 32 + k * 8, dv + ((at * S::kSlot + kSecond[x] * S::kPiece + k * 2048) >> 4), idesc_o,
                                          x == 0 && k == 0 ? 0u : 1u, issues);
          }
          release(v_empty + at);
          release(pv_done);
        }
      }
    }
  } else if (warp < 4) {
    // ---- scores -> weights: a thread has a row ----
    const int row = warp * 32 + lane;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    int n_items = 0;
    for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      PromptItem it;
      while (ok && next_item(it, ok)) {
        const PromptTiles<1, KT> tiles(p, it);
        const int within = row / p.hn, pos = it.blk * p.per_item + within;
        const bool there = within < p.pt && pos < it.n_r;
        const int n = tiles.count[0], sees = there ? seen_by(pos, it.n_r, it.n_k) : 0x7FFFFFFF;
        float m = -CUDART_INF_F, l = 0.f;
        for (int j = 0; j < n; ++j, ++n_kv) {
          ok = wait(s_full + (n_kv & 1), n_kv >> 1) && ok;
          __syncwarp();
          ptx::tc_fence_after();
          uint32_t s[KT];
          ptx::tmem_ld_32x64_sync(tmem + (n_kv & 1) * KT + lanes, s);
          if (j >= tiles.even[0]) {
            const int left = sees - (tiles.first + j) * KT;
#pragma unroll
            for (int c = 0; c < KT; ++c)
              if (c >= left) s[c] = 0xFF800000u;
          }
          float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
          for (int c = 0; c < KT; ++c) top[c & 3] = fmaxf(top[c & 3], __uint_as_float(s[c]));
          const float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale;
          float f = 1.f;                       // of what is summed so far
          if (j == 0) {
            m = high;
          } else if (high > m + kPromptLazy) {
            f = pow2(m - high);
            m = high;
            l *= f;
          }
          factors[(n_kv % kExactFactors) * kPromptRows + row] = f;
          const float ref = m == -CUDART_INF_F ? 0.f : m;
          float sum[2] = {0.f, 0.f};
          const uint32_t tp = tmem_p + (n_kv & 1) * 96 + lanes;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t h[kPieces][16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              uint32_t a[2][kPieces];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const float x = pow2(fmaf(__uint_as_float(s[c * 32 + i + u]), p.scale, -ref));
                sum[u] += x;
                pieces_of(x, a[u][0], a[u][1], a[u][2]);
              }
#pragma unroll
              for (int y = 0; y < kPieces; ++y) h[y][i >> 1] = upper_halves(a[0][y], a[1][y]);
            }
#pragma unroll
            for (int y = 0; y < kPieces; ++y) ptx::tmem_st_32x16(tp + y * 32 + c * 16, h[y]);
          }
          l += sum[0] + sum[1];
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full + (n_kv & 1));
        }
        ok = wait(l_empty, n_items++ + 1) && ok;
        stats[row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(l_full);
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else {
    // ---- the tiles' products are summed, and the result leaves: a thread has a row ----
    const int row = (warp - 4) * 32 + lane;
    const uint32_t to = tmem_o + ((uint32_t)((warp - 4) * 32) << 16);
    if (tid == 4 * 32) prompt_begins(p);
    __syncwarp();
    int n_items = 0;
    float o[D];
    auto read = [&](auto&& each) {
#pragma unroll
      for (int c = 0; c < D; c += 16) {
        uint32_t x[16];
        ptx::tmem_ld_32x16_sync(to + c, x);
#pragma unroll
        for (int i = 0; i < 16; ++i) each(c + i, __uint_as_float(x[i]));
      }
    };
    for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      PromptItem it;
      while (ok && next_item(it, ok)) {
        const PromptTiles<1, KT> tiles(p, it);
        const int layer = it.ls / p.rows.n_seqs, seq = it.ls - layer * p.rows.n_seqs;
        const int within = row / p.hn, head = it.head * p.hn + row - within * p.hn, pos = it.blk * p.per_item + within;
        const bool there = within < p.pt && pos < it.n_r, by_hand = it.careful && tiles.count[0] > tiles.even[0];
        const int n = tiles.count[0];
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] = 0.f;
        for (int j = 0; j < n; ++j, ++n_kv) {
          ok = wait(pv_done, n_kv) && ok;
          __syncwarp();
          ptx::tc_fence_after();
          const float f = factors[(n_kv % kExactFactors) * kPromptRows + row];
          if (!by_hand || j < tiles.even[0]) {
            read([&](int i, float x) { o[i] = fmaf(o[i], f, x); });
          } else {
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] *= f;
          }
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0 && !(by_hand && j + 1 == n)) ptx::mbar_arrive(o_read);
        }
        ok = wait(l_full, n_items++) && ok;
        const float m = stats[row].x, l = stats[row].y;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(l_empty);
        if (by_hand) {                         // by way of the tensor memory, which is this item's until its last tile counts as read
#pragma unroll
          for (int c = 0; c < D; c += 16) {
            uint32_t x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(o[c + i]);
            ptx::tmem_st_32x16(to + c, x);
          }
          ptx::tmem_st_wait();
          const int sees = there ? seen_by(pos, it.n_r, it.n_k) : 0;
          add_by_hand<T, D>(p, it, to, 0, D, false, head, there ? pos : 0, (tiles.first + tiles.even[0]) * KT, min(sees, (tiles.first + n) * KT), m == -CUDART_INF_F ? 0.f : m);
          __syncwarp();
          read([&](int i, float x) { o[i] = x; });
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(o_read);
        }
        const bool write = there && ok && !*abort_flag;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t number = row_number(p, layer, seq, it.base_r, head, pos);
        const int64_t parts = (int64_t)it.split * p.rows.n_layers * p.rows.total_len * (p.heads * p.hn);
        const int64_t at = !write ? -1 : (p.splits > 1 ? (parts + number) * D : row_offset(p.out, p.rows, layer, seq, it.base_r, head, pos)) * 4;
        uint8_t* base = reinterpret_cast<uint8_t*>(p.splits > 1 ? p.part : const_cast<void*>(p.out.ptr));
        const float f = p.splits > 1 ? 1.f : inv;
        bool odd = false;
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint4 h[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float* x = o + c + 4 * e;
            odd |= x[0] != x[0] || x[1] != x[1] || x[2] != x[2] || x[3] != x[3];
            h[e] = make_uint4(__float_as_uint(x[0] * f), __float_as_uint(x[1] * f), __float_as_uint(x[2] * f), __float_as_uint(x[3] * f));
          }
          put_rows(smem + S::stage + (warp - 4) * 4096, h, base + c * 4, at);
        }
        if (write) {
          if (p.splits > 1) p.stat[parts + number] = make_float2(m, l);
          else put_lse(p, layer, column_of(p, seq, it.base_r, pos), head, m, l);
          if (odd && !it.careful && l == l) {
            atomicOr(redo + (it.number >> 5), 1u << (it.number & 31));
            *any_redo = 1;
          }
        }
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  }
  __syncthreads();                        // nobody reads the tensor memory any more
  if (warp == kExactIssue) {
    if (ptx::elect_one()) ptx::umma_commit(drained);
    __syncwarp();
    // as in the bf16 kernel: nothing is under way any more when the block goes
    ptx::mbar_wait(drained, 0, abort_flag + 1, kDefaultMbarWaitCycles);
    __syncwarp();
    if (lane == 0 && *abort_flag) {
      const int held = (int)blockIdx.x == p.withhold ? 1 : 0;
      for (int i = max(asked[0] - RING, held); i < asked[0]; ++i) ptx::mbar_wait(k_full + i % RING, (i / RING) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
      for (int i = max(asked[2] - RING, 0); i < asked[2]; ++i) ptx::mbar_wait(v_full + i % RING, (i / RING) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
      if (asked[1] > 0) ptx::mbar_wait(q_full, (asked[1] - 1) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
    }
    __syncwarp();
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  if (tid == 0 && *abort_flag) prompt_failed(p);
}

// ---- host ----------------------------------------------------------------------------------------

static size_t rows_of(const spindlekv_batch& b) { return (size_t)b.n_layers * b.total_len; }

size_t prompt_pieces_bytes(const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int n_kv_heads, int head_dim) {
  const size_t row = kPieces * 2 * (size_t)head_dim;      // (a multiple of 128, which suits the copies' 16 bytes)
  return row * (rows_of(rows) * n_q_heads + 2 * rows_of(keys) * n_kv_heads);
}

template <int D>
static spindlekv_status launch_exact(const PromptParams& p, const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, void* pieces, int64_t blocks,
                                     cudaStream_t st) {
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    if (cudaFuncSetAttribute(prompt_attend_f32_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, ExactSmem<D>::bytes) != cudaSuccess) return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  __nv_bfloat16* to = static_cast<__nv_bfloat16*>(pieces);
  const size_t nq = rows_of(rows) * n_q_heads * D * kPieces, nk = rows_of(keys) * p.heads * D * kPieces;
  SplitParams sp;
  // What lies behind a sequence's last row may be anything where rows and scores are concerned, which nobody reads or which are replaced; values are multiplied by
  // weights of 0 up to the end of their tile
  sp.t[0] = {p.q, p.rows, to, n_q_heads, 1, 0};
  sp.t[1] = {p.k, p.keys, to + nq, p.heads, 0, 0};
  sp.t[2] = {p.v, p.keys, to + nq + nk, p.heads, 0, kExactKeys};
  int64_t blocks_of = 0, units = 0;
  for (const SplitSource& t : sp.t) {
    const int64_t seqs = t.batch.cu ? 1 : t.batch.n_seqs, tokens = t.batch.cu ? t.batch.total_len : t.batch.max_len, items = tokens * t.heads * (D / 8);
    if (items > 0xFFFF0000ll) return SPINDLEKV_UNSUPPORTED;      // more pieces than there is memory
    blocks_of = std::max(blocks_of, (items + kSplitTurns * 256 - 1) / (kSplitTurns * 256));
    units = std::max(units, seqs * t.batch.n_layers);
  }
  // the planes as tensors: three times as many layers
  spindlekv_batch kb = keys, rb = rows;
  kb.n_layers *= kPieces;
  rb.n_layers *= kPieces;
  auto tensor = [](void* ptr, const spindlekv_batch& b, int heads, bool by_token) {
    const int64_t tokens = b.cu_seqlens ? b.total_len : b.max_len, seq = tokens * heads * D;
    return spindlekv_tensor{ptr, SPINDLEKV_BF16, b.cu_seqlens ? seq : seq * b.n_seqs, seq, by_token ? D : tokens * D, by_token ? (int64_t)heads * D : D};
  };
  CUtensorMap qmap, kmap, vmap;
  if (!make_rows_map_bf16(&qmap, tensor(to, rb, n_q_heads, true), rb, n_q_heads, D, p.hn, p.pt) ||
      !make_tensor_map_bf16(&kmap, tensor(to + nq, kb, p.heads, false), kb, p.heads, D, kExactKeys) ||
      !make_tensor_map_bf16(&vmap, tensor(to + nq + nk, kb, p.heads, false), kb, p.heads, D, kExactKeys))
    return SPINDLEKV_UNSUPPORTED;
  {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks_of, (unsigned)units, 3);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    LaunchScope ls(KC_PROMPT, st);
    if (cudaLaunchKernelEx(&cfg, prompt_pieces_kernel<D>, sp) != cudaSuccess) return SPINDLEKV_CUDA;
  }
  const spindlekv_status s = launch_after(prompt_attend_f32_kernel<D>, blocks, kExactThreads, ExactSmem<D>::bytes, st, qmap, kmap, vmap, p);
  return s == SPINDLEKV_OK ? launch_prompt_join<float, D>(p, st) : s;
}

spindlekv_status prompt_attend_f32(const PromptParams& p, const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int head_dim, void* pieces,
                                   int64_t blocks, cudaStream_t st) {
  return head_dim == 64 ? launch_exact<64>(p, keys, rows, n_q_heads, pieces, blocks, st) : launch_exact<128>(p, keys, rows, n_q_heads, pieces, blocks, st);
}

}  // namespace skv
