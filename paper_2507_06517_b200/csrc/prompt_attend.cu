// Causal attention of a prompt's rows over its keys and values, bf16, grouped heads.
//
// Row i of n_r over n_k keys sees the first n_k - n_r + i + 1 of them:  O_i = sum_j p_ij V_j / sum_j p_ij,  p_ij = 2^(c q_i.k_j - m_i).
//
// A tile of 128 rows holds 128 / hn positions of all hn query heads of a KV head, so that keys and values are read once for the group and the
// triangle that is computed for nothing shrinks with the positions of a tile; a block has two tiles and walks 128 keys at a time:
//     S_w [128 rows x 128 keys] = Q_w K^T      both operands in shared memory, d contiguous
//     O_w [128 rows x d]       += P_w V        P_w in tensor memory, where S_w was; V read transposed
// Tensor memory: S_0, S_1, O_0, O_1.
//
// Roles: two warpgroups turn scores into weights, a thread for each row of their tile; one warp asks for Q, K and V (TMA); one issues the
// products.  While one tile's weights are formed the products of the other run.  The reference m of a row moves only when a score exceeds
// it by 2^8 (then O is multiplied by the row's thread: the products that wrote it are done when the scores that follow them are).
// Sums and references are fp32 (sums of very long keys are taken out of tensor memory: keep_sums); the weights enter the second product in bf16, where values are, to half a step of 2^-8: as much as the result's
// own rounding, and independent from key to key.
//
// Values that a row does not see are multiplied by 0, which does nothing unless they are NaN or infinite.  A result that is NaN though its sum
// is not says so, and its item is done again, with the tiles that hide keys from some row multiplied by hand.
//
// Bound by products and exponentials alike (d = 128: 2048 cycles of either for a step of two tiles, both pipes 68 % busy at 8192 tokens; d = 64: half the
// products, exponentials 75 % busy) and by the chain of a step from scores over their maximum (415 cycles) and weights (1350) to the second product.
// 32 query heads over 8, d = 128: 512 tokens 15 us, 2048 38, 4096 111 to 121 (1240 to 1140 TFLOP/s), 16384 1.55 to 1.75 ms
// (1420 to 1260), replayed; one call after another with inputs in rotation, at the power limit's lower clocks, 135 us and 1.82 ms (1020 and 1210).
// Not kept: 64 keys a step (4096 tokens 189 us where this took 131), two threads a row (163), exponentials in part by a polynomial (112 to 136 for 111).
#include <algorithm>

#include "args.cuh"
#include "prompt_attend.cuh"

namespace skv {

// Three warpgroups of 168 registers a thread; the two with rows take 208 and leave the third 88 (2 x 208 + 88 = 3 x 168).
constexpr int kPromptThreads = 384, kAskRole = 8, kIssueRole = 9;
constexpr int kPromptItemSlots = 4;
constexpr int kPart = 96;                 // keys of a tile whose weights the second product starts with

template <int D>
struct PromptSmem {
  static constexpr int kTile = kPromptRows * D * 2;                // bytes of a tile of rows, keys or values
  static constexpr int kHalf = kPromptRows * 128;                  // of its 64 elements side by side
  static constexpr int kRing = D == 128 ? 4 : 6;
  static constexpr int q = 0, ring = 2 * kTile, stage = ring + kRing * kTile, bars = stage + 8 * 4096;      // stage: 4 KB for each warp with rows
  static constexpr int kBars = 2 * kRing + 2 + 2 * 5 + 2 * kPromptItemSlots + 1;
  static constexpr int words = bars + kBars * 8;                   // abort flags [2], TMEM address, redo at all, [4] copies that were asked for
  static constexpr int items = (words + 32 + 15) / 16 * 16;
  static constexpr int redo = items + kPromptItemSlots * (int)sizeof(PromptItem);
  static constexpr int bytes = 1024 + redo + kPromptMaxItems / 8;
};
static_assert(PromptSmem<128>::bytes <= 227 * 1024, "shared memory");

// The accumulator in tensor memory cuts off what it adds, towards zero: with values of one sign results come out smaller by 7e-5 over 16384 keys, 3.6e-4 over 65536, 1.7e-3
// over 262144 (half a step of bf16 is 2e-3).  So after every 128 tiles a row's thread adds what is there to a sum of its own in memory, rounding as usual, and the products begin
// anew.  It does so between a tile's scores and its weights, where it may touch O anyway: the products that wrote it are done when the scores that follow them are.  Of a
// warp: [element / 4][lane] 16 bytes, so that lanes lie next to one another, and behind them the reference that the sums go by.  7e-5 is then left at any length, and the longest
// calls take 2 to 3 % more (2000 rows, 32 / 8 heads, d = 128: behind 40000 keys 980 -> 1000 us, 131072 3.25 -> 3.35 ms); others have a kernel without it, which the loop's changed registers would
// cost 3 % too (4096 tokens 121 -> 125).
constexpr int kPromptKeep = 128;          // tiles
template <int D> constexpr int kPromptKept = (D + 1) * 256;      // numbers for the 256 rows of a block

template <int D>
__device__ __noinline__ void keep_sums(float* kept, uint32_t o_tmem, bool first, float m) {
  const int lane = threadIdx.x & 31;
  float4* sums = reinterpret_cast<float4*>(kept) + lane;
  float* ref = kept + D * 32 + lane;
  const float was = first ? m : *ref, f = was == m ? 1.f : pow2(was - m);
  *ref = m;
#pragma unroll 1
  for (int c = 0; c < D; c += 64) {
    float4 y[16];                         // (asked for together)
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = first ? make_float4(0.f, 0.f, 0.f, 0.f) : sums[(c / 4 + i) * 32];
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
      uint32_t o[32];
      __syncwarp();
      ptx::tmem_ld_32x32_sync(o_tmem + c + h, o);
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const float4 z = y[(h + i) / 4];
        sums[(c + h + i) / 4 * 32] = make_float4(fmaf(z.x, f, __uint_as_float(o[i])), fmaf(z.y, f, __uint_as_float(o[i + 1])), fmaf(z.z, f, __uint_as_float(o[i + 2])),
                                                 fmaf(z.w, f, __uint_as_float(o[i + 3])));
      }
    }
  }
  __syncwarp();
}

// LONG: keys that are longer than this in some part
template <int D, bool LONG>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_attend_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                                          const __grid_constant__ CUtensorMap vmap, const __grid_constant__ PromptParams p) {
  using S = PromptSmem<D>;
  using T = __nv_bfloat16;
  constexpr int KT = 128, RING = S::kRing, SLOTS = kPromptItemSlots;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem + S::bars);
  uint64_t *kv_empty = kv_full + RING, *q_full = kv_empty + RING, *q_empty = q_full + 1, *s_full = q_empty + 1, *p_full = s_full + 2, *o_full = p_full + 2,
           *o_empty = o_full + 2, *p_part = o_empty + 2, *item_full = p_part + 2, *item_empty = item_full + SLOTS, *drained = item_empty + SLOTS;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + S::words);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::words) + 2;
  volatile int* any_redo = reinterpret_cast<volatile int*>(smem + S::words) + 3;
  volatile int* asked = reinterpret_cast<volatile int*>(smem + S::words) + 4;    // keys or values, rows
  PromptItem* items = reinterpret_cast<PromptItem*>(smem + S::items);
  uint32_t* redo = reinterpret_cast<uint32_t*>(smem + S::redo);
  // (broadcasts, here and where products are issued, say that a value is the whole warp's: descriptors are then formed where the products take them from)
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < RING; ++i) { ptx::mbar_init(kv_full + i, 1); ptx::mbar_init(kv_empty + i, 1); }
    ptx::mbar_init(q_full, 1);
    ptx::mbar_init(q_empty, 1);
    for (int w = 0; w < 2; ++w) {
      ptx::mbar_init(s_full + w, 1);
      ptx::mbar_init(p_part + w, 4);
      ptx::mbar_init(p_full + w, 4);
      ptx::mbar_init(o_full + w, 1);
      ptx::mbar_init(o_empty + w, 4);
    }
    for (int i = 0; i < SLOTS; ++i) { ptx::mbar_init(item_full + i, 1); ptx::mbar_init(item_empty + i, 9); }
    ptx::mbar_init(drained, 1);
    ptx::fence_barrier_init();
    abort_flag[0] = abort_flag[1] = 0;
    *any_redo = 0;
    asked[0] = asked[1] = 0;
    ptx::prefetch_tensormap(&qmap);
    ptx::prefetch_tensormap(&kmap);
    ptx::prefetch_tensormap(&vmap);
  }
  for (int i = tid; i < kPromptMaxItems / 32; i += kPromptThreads) redo[i] = 0;
  // rows that no copy fills (hn does not divide 128) hold zeros
  for (int i = p.pt * p.hn * 8 + tid; i < kPromptRows * 8; i += kPromptThreads)
    for (int h = 0; h < 2 * D / 64; ++h) *reinterpret_cast<uint4*>(smem + S::q + h * S::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  if (warp == kIssueRole) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
    ptx::tc_fence_before();
  }
  // up to here nothing was read or written that an earlier kernel of the stream knows of
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0), tmem_o = tmem + 256;

  auto wait = [&](uint64_t* bar, int phase) { return ptx::mbar_wait(bar, phase & 1, abort_flag, p.wait_cycles); };
  int item_no = 0;                        // items so far, both passes' and the ends of passes
  // what the other roles do with an item; false: the pass is over
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
  bool ok = true;
  int n_kv = 0, n_q = 0;                  // ring slots and row tiles so far (asking and issuing role)
  // All roles meet at the end of a pass; the second one is for items that have to be done again.  One answer for all
  auto again = [&]() {
    __syncthreads();
    return __syncthreads_and(*any_redo && !*abort_flag) != 0;
  };
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    int n_s = 0, n_o = 0;                 // scores and results so far
    for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      const int w = warp >> 2, row = (warp & 3) * 32 + lane;
      uint8_t* stage = smem + S::stage + warp * 4096;
      float* kept = LONG ? p.kept + ((int64_t)blockIdx.x * 8 + warp) * (kPromptKept<D> / 8) : nullptr;
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ts = tmem + w * 128 + lanes, to = tmem_o + w * D + lanes;
      while (ok) {
        // The item stays in its slot until its result is written: registers are short here
        const int slot = item_no % SLOTS;
        ok = __all_sync(0xffffffffu, wait(item_full + slot, item_no / SLOTS));
        if (!ok) break;
        const PromptItem* held = items + slot;
        ++item_no;
        if (held->ls < 0) {
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(item_empty + slot);
          break;
        }
        int n, first, even, sees;
        bool careful;
        {
          const PromptItem it = *held;
          const PromptTiles<2, KT> tiles(p, it);
          const int within = row / p.hn, pos = it.blk * p.per_item + w * p.pt + within;
          n = w ? tiles.count[1] : tiles.count[0];
          even = w ? tiles.even[1] : tiles.even[0];
          first = tiles.first;
          careful = it.careful != 0;
          sees = within < p.pt && pos < it.n_r ? seen_by(pos, it.n_r, it.n_k) : 0x7FFFFFFF;
        }
        float m = -CUDART_INF_F, l = 0.f;
        for (int j0 = 0; j0 < (LONG ? n : 1); j0 += kPromptKeep) {
        if (LONG && j0 > 0 && (!careful || j0 - kPromptKeep < even)) {
          ok = wait(s_full + w, n_s) && ok;
          __syncwarp();
          ptx::tc_fence_after();
          keep_sums<D>(kept, to, j0 == kPromptKeep, m);
        }
        for (int j = LONG ? j0 : 0, end = LONG ? min(n, j0 + kPromptKeep) : n; j < end; ++j) {
          ok = wait(s_full + w, n_s++) && ok;
          __syncwarp();
          ptx::tc_fence_after();
          uint32_t s[128];
          ptx::tmem_ld_32x128_sync(ts, s);
          if (j >= even) {
            const int left = sees - (first + j) * KT;
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c >= left) s[c] = 0xFF800000u;
          }
          float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
          for (int c = 0; c < 128; c += 2) top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
          const float high = max3(max3(top[0], top[1], top[2]), top[3], top[3]) * p.scale;
          if (j == 0) {
            m = high;
          } else if (__any_sync(0xffffffffu, high > m + kPromptLazy)) {
            const float now = fmaxf(m, high), f = now == m ? 1.f : pow2(m - now);
            m = now;
            l *= f;
            if (!careful || even > 0) {
#pragma unroll 1
              for (int c = 0; c < D; c += 8) {
                uint32_t o[8];
                ptx::tmem_ld_32x8_sync(to + c, o);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                ptx::tmem_st_32x8_sync(to + c, o);
              }
            }
          }
          const float ref = m == -CUDART_INF_F ? 0.f : m;
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t h[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float2 x = fma_pair(make_float2(__uint_as_float(s[c * 32 + i]), __uint_as_float(s[c * 32 + i + 1])), make_float2(p.scale, p.scale), make_float2(-ref, -ref));
              x.x = pow2(x.x);
              x.y = pow2(x.y);
              sum[(i >> 1) & 1] = add_pair(sum[(i >> 1) & 1], x);
              h[i >> 1] = pack_bf16(x.x, x.y);
            }
            ptx::tmem_st_32x16(ts + c * 16, h);
            if (c == kPart / 32 - 1) {
              ptx::tmem_st_wait();
              ptx::tc_fence_before();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(p_part + w);
            }
          }
          l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
          ptx::tmem_st_wait();
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(p_full + w);
        }
        }
        // ---- the item's result ----
        const PromptItem it = *held;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(item_empty + slot);
        const int layer = it.ls / p.rows.n_seqs, seq = it.ls - layer * p.rows.n_seqs;
        const int within = row / p.hn, head = it.head * p.hn + row - within * p.hn, pos = it.blk * p.per_item + w * p.pt + within;
        const bool there = sees != 0x7FFFFFFF;
        if (n > 0) ok = wait(o_full + w, n_o++) && ok;
        __syncwarp();
        ptx::tc_fence_after();
        if (careful && n > even)
          add_by_hand<T, D>(p, it, to, 0, D, even <= (LONG ? (n - 1) / kPromptKeep * kPromptKeep : 0), head, there ? pos : 0, (first + even) * KT, there ? min(sees, (first + n) * KT) : 0, m == -CUDART_INF_F ? 0.f : m);
        const bool write = there && ok && !*abort_flag;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t number = row_number(p, layer, seq, it.base_r, head, pos), parts = (int64_t)it.split * p.rows.n_layers * p.rows.total_len * (p.heads * p.hn);
        const int64_t at = !write ? -1 : p.splits > 1 ? (parts + number) * D * 4 : row_offset(p.out, p.rows, layer, seq, it.base_r, head, pos) * 2;
        uint8_t* base = reinterpret_cast<uint8_t*>(p.splits > 1 ? p.part : const_cast<void*>(p.out.ptr));
        bool odd = false;
        const bool keeps = LONG && n > kPromptKeep && (!careful || even > 0);
        float f_kept = 0.f;
        if (keeps) {
          const float was = kept[D * 32 + lane];
          f_kept = was == m ? 1.f : pow2(was - m);
        }
#pragma unroll 1
        for (int c = 0; c < D; c += 64) {
          float x[64];
#pragma unroll
          for (int i = 0; i < 64; i += 32) {
            uint32_t o[32];
            if (n > 0) {
              __syncwarp();
              ptx::tmem_ld_32x32_sync(to + c + i, o);
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) x[i + e] = n > 0 ? __uint_as_float(o[e]) : 0.f;
          }
          if (keeps) {
            const float4* sums = reinterpret_cast<const float4*>(kept) + c / 4 * 32 + lane;
#pragma unroll
            for (int e = 0; e < 64; e += 4) {
              const float4 y = sums[e / 4 * 32];
              x[e] = fmaf(y.x, f_kept, x[e]);
              x[e + 1] = fmaf(y.y, f_kept, x[e + 1]);
              x[e + 2] = fmaf(y.z, f_kept, x[e + 2]);
              x[e + 3] = fmaf(y.w, f_kept, x[e + 3]);
            }
          }
#pragma unroll
          for (int e = 0; e < 64; ++e) odd |= x[e] != x[e];
          uint4 h[8];
          if (p.splits > 1) {
#pragma unroll
            for (int i = 0; i < 64; i += 32) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                h[e] = make_uint4(__float_as_uint(x[i + 4 * e]), __float_as_uint(x[i + 4 * e + 1]), __float_as_uint(x[i + 4 * e + 2]), __float_as_uint(x[i + 4 * e + 3]));
              put_rows(stage, h, base + (c + i) * 4, at);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              h[e] = make_uint4(pack_bf16(x[8 * e] * inv, x[8 * e + 1] * inv), pack_bf16(x[8 * e + 2] * inv, x[8 * e + 3] * inv),
                                pack_bf16(x[8 * e + 4] * inv, x[8 * e + 5] * inv), pack_bf16(x[8 * e + 6] * inv, x[8 * e + 7] * inv));
            put_rows(stage, h, base + c * 2, at);
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (n > 0 && lane == 0) ptx::mbar_arrive(o_empty + w);
        if (write) {
          if (p.splits > 1) p.stat[parts + number] = make_float2(m, l);
          else put_lse(p, layer, column_of(p, seq, it.base_r, pos), head, m, l);
          // (only what is hidden from a row can make its result NaN where its sum is a number; what it sees does so again)
          if (odd && !it.careful && l == l) {
            atomicOr(redo + (it.number >> 5), 1u << (it.number & 31));
            *any_redo = 1;
          }
        }
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kAskRole) {
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
        const PromptTiles<2, KT> tiles(p, it);
        if (tiles.most == 0) continue;
        const int layer = it.ls / p.rows.n_seqs, seq = it.ls - layer * p.rows.n_seqs;
        ok = __all_sync(0xffffffffu, wait(q_empty, n_q + 1));
        if (!ok) break;
        if (lane == 0) {
          const int box = p.pt * p.hn * 128;
          ptx::mbar_expect_tx(q_full, ((tiles.count[0] > 0) + (tiles.count[1] > 0)) * (D / 64) * box);
#pragma unroll
          for (int w = 0; w < 2; ++w)
            if (tiles.count[w] > 0)
              for (int h = 0; h < D / 64; ++h)
                ptx::tma_load_5d(smem + S::q + w * S::kTile + h * S::kHalf, &qmap, q_full, h * 64, it.head * p.hn, it.base_r + it.blk * p.per_item + w * p.pt,
                                 p.rows.cu ? 0 : seq, layer);
          asked[1] = n_q + 1;
        }
        __syncwarp();
        ++n_q;
        for (int i = 0; i < 2 * tiles.most; ++i) {         // K and V in turn
          const int at = n_kv % RING;
          ok = __all_sync(0xffffffffu, wait(kv_empty + at, n_kv / RING + 1));
          if (!ok) break;
          if (lane == 0) {
            if (n_kv || (int)blockIdx.x != p.withhold) {
              ptx::mbar_expect_tx(kv_full + at, S::kTile);
              for (int h = 0; h < D / 64; ++h)
                ptx::tma_load_5d(smem + S::ring + at * S::kTile + h * S::kHalf, i & 1 ? &vmap : &kmap, kv_full + at, h * 64, it.base_k + (tiles.first + (i >> 1)) * KT, it.head,
                                 p.keys.cu ? 0 : seq, layer);
            }
            asked[0] = n_kv + 1;
          }
          __syncwarp();
          ++n_kv;
        }
      }
      }
    } else if (warp == kIssueRole) {
      int n_s[2] = {0, 0}, n_o[2] = {0, 0};      // scores and results so far, by tile
      for (int pass = 0; pass == 0 || (pass == 1 && again()); ++pass) {
      constexpr uint32_t idesc_s = ptx::idesc_bf16_f32(128, KT), idesc_o = ptx::idesc_bf16_f32(128, D) | (1u << 16);
      const uint32_t issues = ptx::elect_one();
      const uint64_t dq = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::q)), dk = ptx::smem_desc_sw128(ptx::smem_u32(smem + S::ring)),
                     dv = ptx::smem_desc_sw128_mn(ptx::smem_u32(smem + S::ring), S::kHalf);
      PromptItem it;
      while (ok && next_item(it, ok)) {
        int most, count[2], even[2];
        {
          const PromptTiles<2, KT> tiles(p, it);
          auto all = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
          most = all(tiles.most);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            count[w] = all(tiles.count[w]);
            even[w] = all(it.careful ? tiles.even[w] : tiles.count[w]);      // tiles whose values are multiplied here
          }
        }
        if (most == 0) continue;
        auto scores = [&](int w, int at) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t step = ((k >> 2) * S::kHalf + (k & 3) * 32) >> 4;
            ptx::umma_f16_elected(tmem + w * 128, dq + (w * S::kTile >> 4) + step, dk + (at * S::kTile >> 4) + step, idesc_s, k ? 1u : 0u, issues);
          }
          if (issues) ptx::umma_commit(s_full + w);
          __syncwarp();
        };
        auto release = [&](uint64_t* bar) {
          if (issues) ptx::umma_commit(bar);
          __syncwarp();
        };
        ok = wait(q_full, n_q++);
        int at = n_kv % RING;
        ok = __all_sync(0xffffffffu, wait(kv_full + at, n_kv / RING) && ok);
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (count[w] > 0) scores(w, at);
        release(kv_empty + at);
        ++n_kv;
        if (most == 1) release(q_empty);
        for (int j = 0; j < most && ok; ++j) {
          const int av = n_kv % RING, ak = (n_kv + 1) % RING;
          const bool more = j + 1 < most;
          ok = wait(kv_full + av, n_kv / RING);
          if (more) ok = wait(kv_full + ak, (n_kv + 1) / RING) && ok;
          ok = __all_sync(0xffffffffu, ok);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (j >= count[w] || !ok) continue;
            if (j == 0) ok = wait(o_empty + w, n_o[w]++ + 1);
            auto values = [&](int k0, int k1) {      // of 16 keys each
              ptx::tc_fence_after();
              if (j >= even[w]) return;
#pragma unroll
              for (int k = k0; k < k1; ++k)
                ptx::umma_bf16_ts_elected(tmem_o + w * D, tmem + w * 128 + k * 8, dv + (av * S::kTile >> 4) + (k * 2048 >> 4), idesc_o, (LONG ? j % kPromptKeep : j) == 0 && k == 0 ? 0u : 1u, issues);
            };
            ok = __all_sync(0xffffffffu, wait(p_part + w, n_s[w]) && ok);
            if (ok) values(0, kPart / 16);
            ok = __all_sync(0xffffffffu, wait(p_full + w, n_s[w]++) && ok);
            if (!ok) continue;
            values(kPart / 16, KT / 16);
            if (j + 1 < count[w]) scores(w, ak);
            else release(o_full + w);
          }
          if (!ok) break;
          release(kv_empty + av);
          if (more) release(kv_empty + ak);
          if (j + 2 == most) release(q_empty);
          n_kv += more ? 2 : 1;
        }
      }
      }
    } else {
      if (tid == kPromptThreads - 1) prompt_begins(p);
      again();
    }
  }
  __syncthreads();                        // nobody reads the tensor memory any more
  if (warp == kIssueRole) {
    if (ptx::elect_one()) ptx::umma_commit(drained);
    __syncwarp();
    // all products are done, and with them their arrivals, before the block goes; after a wait that gave up so are the copies that were still on
    // their way (within the default bound)
    ptx::mbar_wait(drained, 0, abort_flag + 1, kDefaultMbarWaitCycles);
    __syncwarp();
    if (lane == 0 && *abort_flag) {
      const int held = (int)blockIdx.x == p.withhold ? 1 : 0;        // (a copy that was never asked for)
      for (int i = max(asked[0] - RING, held); i < asked[0]; ++i) ptx::mbar_wait(kv_full + i % RING, (i / RING) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
      if (asked[1] > 0) ptx::mbar_wait(q_full, (asked[1] - 1) & 1, abort_flag + 1, kDefaultMbarWaitCycles);
    }
    __syncwarp();
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  if (tid == 0 && *abort_flag) prompt_failed(p);
}

// ---- host ----------------------------------------------------------------------------------------

bool sim_tc_available();

constexpr int kPromptSms = 148;
// the most items of a call, by what the host knows
static int64_t prompt_items(const spindlekv_batch& rows, int heads, int per_item) {
  const int64_t blocks = rows.cu_seqlens ? (int64_t)rows.total_len / per_item + rows.n_seqs : (int64_t)rows.n_seqs * ((rows.max_len + per_item - 1) / per_item);
  return blocks * rows.n_layers * heads;
}
// Parts that the keys are cut into: as many as bring the items to one for each SM, of two tiles of keys at least, where that saves more than the parts' way
// through memory and the kernel that joins them cost (128 keys take 1.4 us, in fp32 twice that; the join 3.5 us and its bytes; a whole prompt of 512, 32 / 8 heads, in two
// parts 22 us, in one 15; one row of 2000 keys in seven parts 16 us, in three 18, in one 28)
static int prompt_splits(const spindlekv_batch& keys, const spindlekv_batch& rows, int heads, int per_item, int row_bytes, int dtype) {
  const int64_t items = prompt_items(rows, heads, per_item);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kPromptSms / items, keys.max_len / 256));
  const double saved = (dtype == SPINDLEKV_BF16 ? 1.4 : 2.8) * (keys.max_len / 128.) * (1. - 1. / most), bytes = 2. * most * rows.n_layers * rows.total_len * row_bytes;
  return saved > 3.5 + bytes / 4e6 ? (int)most : 1;
}
static int prompt_per_item(int hn, int dtype) { return (dtype == SPINDLEKV_BF16 ? 2 : 1) * (kPromptRows / hn); }
// One block per SM; more only where a block's list of items would not do
static int64_t prompt_blocks(int64_t items) { return std::min(items, std::max<int64_t>(kPromptSms, (items + kPromptMaxItems - 1) / kPromptMaxItems)); }
// bf16: bytes for the sums of keys that are longer, in a part, than the products sum up by themselves
static size_t prompt_kept_bytes(const spindlekv_batch& keys, int64_t blocks, int splits, int head_dim) {
  if (ceil_div(ceil_div(keys.max_len, 128), splits) <= kPromptKeep) return 0;
  return (size_t)blocks * (head_dim == 64 ? kPromptKept<64> : kPromptKept<128>) * sizeof(float);
}

size_t prompt_workspace_bytes(const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int n_kv_heads, int head_dim, int dtype) {
  const int few = prompt_few_rows(keys, rows, n_kv_heads, n_q_heads / n_kv_heads, head_dim, dtype);
  const int splits = few ? few : prompt_splits(keys, rows, n_kv_heads, prompt_per_item(n_q_heads / n_kv_heads, dtype), n_q_heads * head_dim * 4, dtype);
  const size_t numbers = (size_t)rows.n_layers * rows.total_len * n_q_heads;
  const size_t parts = kHeaderBytes + (splits > 1 ? align_up(splits * numbers * (head_dim * sizeof(float) + sizeof(float2)), 256) : 0);
  if (few) return parts;
  if (dtype == SPINDLEKV_F32) return parts + prompt_pieces_bytes(keys, rows, n_q_heads, n_kv_heads, head_dim);
  const int64_t items = prompt_items(rows, n_kv_heads, prompt_per_item(n_q_heads / n_kv_heads, dtype)) * splits;
  return parts + prompt_kept_bytes(keys, prompt_blocks(items), splits, head_dim);
}

template <int D, bool LONG>
static spindlekv_status launch_prompt(const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap, const PromptParams& p, int64_t blocks, cudaStream_t st) {
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    if (cudaFuncSetAttribute(prompt_attend_kernel<D, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, PromptSmem<D>::bytes) != cudaSuccess) return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  const spindlekv_status s = launch_after(prompt_attend_kernel<D, LONG>, blocks, kPromptThreads, PromptSmem<D>::bytes, st, qmap, kmap, vmap, p);
  return s == SPINDLEKV_OK ? launch_prompt_join<__nv_bfloat16, D>(p, st) : s;
}

spindlekv_status prompt_attend_impl(const spindlekv_batch& keys, const spindlekv_batch& rows, int n_q_heads, int n_kv_heads, int head_dim, float scale,
                                    const spindlekv_tensor& q, const spindlekv_tensor& k, const spindlekv_tensor& v, const spindlekv_tensor& out, float* lse, void* ws,
                                    size_t ws_bytes, cudaStream_t st) {
  if (ws_bytes < prompt_workspace_bytes(keys, rows, n_q_heads, n_kv_heads, head_dim, q.dtype)) return SPINDLEKV_WORKSPACE_TOO_SMALL;
  if (!sim_tc_available()) return SPINDLEKV_UNSUPPORTED;
  PromptParams p;
  p.keys = make_batch(keys);
  p.rows = make_batch(rows);
  p.q = make_view(q);
  p.k = make_view(k);
  p.v = make_view(v);
  p.out = make_view(out);
  p.heads = n_kv_heads;
  p.hn = n_q_heads / n_kv_heads;
  p.pt = kPromptRows / p.hn;
  p.per_item = prompt_per_item(p.hn, q.dtype);
  p.max_blocks = ceil_div(rows.max_len, p.per_item);
  const int few = prompt_few_rows(keys, rows, n_kv_heads, p.hn, head_dim, q.dtype);
  p.splits = few ? few : prompt_splits(keys, rows, n_kv_heads, p.per_item, n_q_heads * head_dim * 4, q.dtype);
  p.scale = (scale == 0.f ? 1.f / sqrtf((float)head_dim) : scale) * 1.44269504088896340736f;
  p.lse = lse;
  const size_t numbers = (size_t)rows.n_layers * rows.total_len * n_q_heads;
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kHeaderBytes);
  p.stat = reinterpret_cast<float2*>(p.part + p.splits * numbers * head_dim);
  p.kept = nullptr;
  p.hdr = static_cast<uint32_t*>(ws);
  const Tuning tune = current_tuning();
  p.wait_cycles = tune.mbar_wait_cycles;
  p.withhold = tune.paged_withhold;
  if (few) return prompt_attend_few(p, keys, rows.max_len, head_dim, k, v, st);
  const int64_t blocks = prompt_blocks(prompt_items(rows, n_kv_heads, p.per_item) * p.splits);
  if (blocks > 65535) return SPINDLEKV_UNSUPPORTED;
  uint8_t* behind = static_cast<uint8_t*>(ws) + kHeaderBytes + (p.splits > 1 ? align_up(p.splits * numbers * (head_dim * sizeof(float) + sizeof(float2)), 256) : 0);
  if (q.dtype == SPINDLEKV_F32) return prompt_attend_f32(p, keys, rows, n_q_heads, head_dim, behind, blocks, st);
  if (prompt_kept_bytes(keys, blocks, p.splits, head_dim)) p.kept = reinterpret_cast<float*>(behind);
  CUtensorMap qmap, kmap, vmap;
  if (!make_rows_map_bf16(&qmap, q, rows, n_q_heads, head_dim, p.hn, p.pt) || !make_tensor_map_bf16(&kmap, k, keys, n_kv_heads, head_dim, 128) ||
      !make_tensor_map_bf16(&vmap, v, keys, n_kv_heads, head_dim, 128))
    return SPINDLEKV_UNSUPPORTED;
  if (head_dim == 64) return p.kept ? launch_prompt<64, true>(qmap, kmap, vmap, p, blocks, st) : launch_prompt<64, false>(qmap, kmap, vmap, p, blocks, st);
  return p.kept ? launch_prompt<128, true>(qmap, kmap, vmap, p, blocks, st) : launch_prompt<128, false>(qmap, kmap, vmap, p, blocks, st);
}

}  // namespace skv
