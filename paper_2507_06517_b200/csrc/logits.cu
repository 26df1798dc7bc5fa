// Logits ahead of a selection: penalties for repeated tokens, biases, and a mask of allowed tokens.
//
// For token t of a row with n_t occurrences in what has been generated, and s_t whether it occurs in that or in the prompt,
//     z = s_t ? (x > 0 ? x / repetition : x * repetition) : x
//     z = n_t > 0 ? z - (frequency * n_t + presence) : z
//     z = z + every bias of t, in the order of the list
//     z = allowed_t ? z : -infinity
// all in fp32, each operation rounded by itself, and once more to the logits' type.
//
// A thread block takes a slice of a row: it counts the history's tokens that fall into the slice in shared memory (whole numbers, so that no order
// shows), marks the biased ones, and then streams the slice, where a word of counts tells the few tokens that change from the many that do not.
//
// 128 x 128256 in fp32: without rules 21 us (6.3 TB/s), masks 22.5, 64 biases a row 34, histories of 16384 tokens 51, all of them 62.  Bound by the additions in
// shared memory (every slice looks through its row's whole history: eight slices, and four lanes of a warp find a token of theirs) and by the turns for the
// tokens that change.  Smaller slices look through it more often (8192: 85 us), larger ones leave one block an SM (68).  Small calls are latency:
// 4 x 32000 in bf16 6 us.
#include <algorithm>

#include <math_constants.h>

#include "common.cuh"

namespace skv {

struct LogitsParams {
  const void* in;
  void* out;
  int64_t in_stride, out_stride;
  spindlekv_logit_rules r;
  int vocab, slice;
};

constexpr int kLogitsThreads = 512, kLogitsMaxSlice = 16384, kLogitsFewBiases = 64;
constexpr uint32_t kBiased = 1u << 31, kInPrompt = 1u << 30, kCountBits = kInPrompt - 1;

// penalties of a token that the history has
__device__ __forceinline__ float penalised(float x, uint32_t word, float rep, float presence, float frequency) {
  if ((word & ~kBiased) == 0u) return x;
  float z = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
  const uint32_t n = word & kCountBits;
  if (n) z = __fsub_rn(z, __fadd_rn(__fmul_rn(frequency, (float)n), presence));
  return z;
}

// Few biases (64 at most): a biased token looks through the whole list, in shared memory.  MANY: they are added ahead of the streaming, 512 of the list at a time: those of this
// slice are put next to one another, in order; the first one of a token forms the token's number and adds it and those behind it, and the number takes the place of the count.
// Work then grows with the list, and not with its square.  Looked through / added ahead, without histories: 128 x 128256 in fp32, 32, 64, 128, 512 biases 26 / 31, 31 / 33, 48 / 35,
// 263 / 43 us, in bf16 18 / 20, 23 / 21, 38 / 23, 200 / 30; 4 x 32000 in bf16, 64, 128 biases 5.4 / 5.6, 9.4 / 6.1; 2 x 131072 in fp32, a bias for every token 18 / 0.38 ms.
template <typename T, bool MANY>
__global__ void __launch_bounds__(kLogitsThreads, 2) logits_adjust_kernel(const __grid_constant__ LogitsParams p) {
  constexpr int E = 16 / sizeof(T), V = kLogitsMaxSlice / E / kLogitsThreads;        // elements of 16 bytes; a thread's pieces of 16 bytes
  extern __shared__ uint4 shared[];
  uint32_t* words = reinterpret_cast<uint32_t*>(shared);
  __shared__ uint32_t mask[kLogitsMaxSlice / 32 + 1];
  __shared__ int32_t bias_token[MANY ? kLogitsThreads : kLogitsFewBiases];
  __shared__ float bias_value[MANY ? kLogitsThreads : kLogitsFewBiases];
  __shared__ uint32_t formed[MANY ? kLogitsMaxSlice / 32 + 1 : 1];       // tokens whose word is their number
  __shared__ int found[MANY ? kLogitsThreads / 32 : 1];
  const int row = blockIdx.y, lo = blockIdx.x * p.slice, hi = min(lo + p.slice, p.vocab), tid = threadIdx.x;
  const T* in = reinterpret_cast<const T*>(p.in) + (int64_t)row * p.in_stride;
  T* out = reinterpret_cast<T*>(p.out) + (int64_t)row * p.out_stride;
  // 16 bytes at a time where both rows lie alike, the elements before and behind one by one.  They are asked for first, and come while the history is counted
  const int off = (int)(reinterpret_cast<uintptr_t>(in + lo) % 16 / sizeof(T));
  const bool alike = reinterpret_cast<uintptr_t>(in + lo) % 16 == reinterpret_cast<uintptr_t>(out + lo) % 16;
  const int first = alike ? min(hi, lo + (off ? E - off : 0)) : hi, vectors = (hi - first) / E, last = first + vectors * E;
  // Everything small is asked for before the logits, so that nothing waits behind them: the row's numbers, a bias and a word of the mask for each thread, and
  // the history's first 8192 tokens, 16 bytes at a time from where they begin
  const bool counts = p.r.history || p.r.n_bias > 0, masked = p.r.allowed != nullptr;
  float rep = 1.f, presence = 0.f, frequency = 0.f;
  int n = 0, prompt = 0;
  const int32_t* h = p.r.history + (int64_t)row * p.r.history_stride;
  const int head = (int)((16 - reinterpret_cast<uintptr_t>(h) % 16) % 16 / 4), most = (p.r.max_history - head) / 4;
  const int4* h4 = reinterpret_cast<const int4*>(h + head);
  int4 said[4];
  auto ask = [&](int q0) {
#pragma unroll
    for (int a = 0; a < 4; ++a) said[a] = q0 + a * kLogitsThreads < most ? __ldg(h4 + q0 + a * kLogitsThreads) : make_int4(-1, -1, -1, -1);
  };
  if (p.r.history) {
    n = p.r.history_lens ? __ldg(p.r.history_lens + row) : p.r.max_history;
    if (p.r.n_prompt) prompt = __ldg(p.r.n_prompt + row);
    if (p.r.repetition) rep = __ldg(p.r.repetition + row);
    if (p.r.presence) presence = __ldg(p.r.presence + row);
    if (p.r.frequency) frequency = __ldg(p.r.frequency + row);
    ask(tid);
  }
  const int32_t* tok = p.r.bias_token + (int64_t)row * p.r.n_bias;
  const float* val = p.r.bias_value + (int64_t)row * p.r.n_bias;
  const uint32_t* allowed = p.r.allowed + (int64_t)row * p.r.allowed_stride + lo / 32;
  static_assert(kLogitsFewBiases <= kLogitsThreads && kLogitsMaxSlice / 32 <= kLogitsThreads, "one for each thread");
  const int my_bias = tid < p.r.n_bias ? __ldg(tok + tid) : -1;
  const float my_value = tid < p.r.n_bias ? __ldg(val + tid) : 0.f;
  const uint32_t my_mask = masked && tid < (hi - lo + 31) / 32 ? __ldg(allowed + tid) : 0u;
  uint4 raw[V];
#pragma unroll
  for (int a = 0; a < V; ++a) {
    const int v = tid + a * kLogitsThreads;
    raw[a] = v < vectors ? *reinterpret_cast<const uint4*>(in + first + v * E) : make_uint4(0u, 0u, 0u, 0u);
  }
  if (masked && tid < kLogitsMaxSlice / 32) mask[tid] = my_mask;
  if (counts) {
    for (int i = tid; i < (hi - lo + 3) / 4; i += kLogitsThreads) shared[i] = make_uint4(0u, 0u, 0u, 0u);
    if (MANY && tid < kLogitsMaxSlice / 32) formed[tid] = 0u;
    __syncthreads();
    if (p.r.history) {
      n = min(max(n, 0), p.r.max_history);
      const uint32_t size = hi - lo;
      auto count = [&](int i, int t) {
        const uint32_t at = (uint32_t)(t - lo);
        if (at >= size || i >= n) return;
        if (i >= prompt) atomicAdd(words + at, 1u);
        else atomicOr(words + at, kInPrompt);
      };
      if (tid < min(head, n)) count(tid, __ldg(h + tid));
      for (int i = max(head, head + 4 * most) + tid; i < n; i += kLogitsThreads) count(i, __ldg(h + i));      // what is left of the row behind its last whole 16 bytes
      const int quads = min(n > head ? (n - head + 3) / 4 : 0, most);                                         // (the last one may reach beyond n, but not beyond the row)
#pragma unroll 1
      for (int q0 = tid; q0 < quads; q0 += 4 * kLogitsThreads) {
        if (q0 != tid) ask(q0);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int i = head + 4 * (q0 + a * kLogitsThreads);
          count(i, said[a].x);
          count(i + 1, said[a].y);
          count(i + 2, said[a].z);
          count(i + 3, said[a].w);
        }
      }
    }
    if constexpr (!MANY) {
      if (tid < kLogitsFewBiases) {
        bias_token[tid] = my_bias;
        bias_value[tid] = my_value;
      }
      if (my_bias >= lo && my_bias < hi) atomicOr(words + (my_bias - lo), kBiased);
    } else {
      int t = my_bias;
      float b = my_value;
      for (long long at = tid; at - tid < p.r.n_bias; at += kLogitsThreads) {
        const bool here = t >= lo && t < hi;
        const uint32_t lanes = __ballot_sync(0xffffffffu, here);
        if (tid % 32 == 0) found[tid / 32] = __popc(lanes);
        __syncthreads();                       // (the first time the history has been counted, too)
        int place = __popc(lanes & ((1u << tid % 32) - 1u)), all = 0;
#pragma unroll
        for (int w = 0; w < kLogitsThreads / 32; ++w) {
          place += w < tid / 32 ? found[w] : 0;
          all += found[w];
        }
        if (here) {
          bias_token[place] = t;
          bias_value[place] = b;
        }
        const bool more = at + kLogitsThreads < p.r.n_bias;      // the next ones are asked for
        t = more ? __ldg(tok + at + kLogitsThreads) : -1;
        b = more ? __ldg(val + at + kLogitsThreads) : 0.f;
        __syncthreads();
        if (tid < all) {
          const int mine = bias_token[tid], i = mine - lo;
          bool first_one = true;
          for (int j = 0; j < tid && first_one; ++j) first_one = bias_token[j] != mine;
          if (first_one) {
            float z = formed[i >> 5] >> (i & 31) & 1u ? __uint_as_float(words[i]) : penalised(to_f32(in[mine]), words[i], rep, presence, frequency);
            for (int j = tid; j < all; ++j)
              if (bias_token[j] == mine) z = __fadd_rn(z, bias_value[j]);
            words[i] = __float_as_uint(z);
            atomicOr(formed + (i >> 5), 1u << (i & 31));
          }
        }
        __syncthreads();
      }
    }
  }
  if (counts || masked) __syncthreads();
  auto is_allowed = [&](int t) { return !masked || (mask[(t - lo) >> 5] >> ((t - lo) & 31) & 1u); };
  auto by_rules = [&](int t, float x, uint32_t word) {
    float z;
    if (MANY && (formed[(t - lo) >> 5] >> ((t - lo) & 31) & 1u)) {
      z = __uint_as_float(word);
    } else {
      z = penalised(x, word, rep, presence, frequency);
      if (!MANY && (word & kBiased)) {
#pragma unroll 4
        for (int j = 0; j < p.r.n_bias; ++j)
          if (bias_token[j] == t) z = __fadd_rn(z, bias_value[j]);
      }
    }
    out[t] = T(is_allowed(t) ? z : -CUDART_INF_F);
  };
  for (int t = lo + tid; t < first; t += kLogitsThreads) by_rules(t, to_f32(in[t]), counts ? words[t - lo] : 0u);
  for (int t = last + tid; t < hi; t += kLogitsThreads) by_rules(t, to_f32(in[t]), counts ? words[t - lo] : 0u);
  const bool even = (first - lo) % 4 == 0;
#pragma unroll
  for (int a = 0; a < V; ++a) {
    const int v = tid + a * kLogitsThreads, t = first + v * E, i = t - lo;
    if (v >= vectors) break;
    uint32_t bits = ~0u;
    if (masked) bits = __funnelshift_r(mask[i >> 5], mask[(i >> 5) + 1], i & 31);      // (the word behind the slice's last is there, and its bits are not used)
    const uint32_t r4[4] = {raw[a].x, raw[a].y, raw[a].z, raw[a].w};
    uint32_t o4[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4) o4[e] = bits >> e & 1u ? r4[e] : 0xFF800000u;
      else o4[e] = (bits >> (2 * e) & 1u ? r4[e] & 0xFFFFu : 0xFF80u) | (bits >> (2 * e + 1) & 1u ? r4[e] & 0xFFFF0000u : 0xFF800000u);
    }
    *reinterpret_cast<uint4*>(out + t) = make_uint4(o4[0], o4[1], o4[2], o4[3]);
    if (!counts) continue;
    // Tokens that the history has or a bias names are few, but nearly every warp meets some: a lane goes from one of its own to the next, so that the warp
    // takes as many turns as its lanes have at most (all elements in turn: 62 us in place of 49, collected in a queue and worked off by 32: 65)
    uint32_t met = 0u;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const uint32_t* from = words + i + e;
      uint4 w;
      if (even) w = *reinterpret_cast<const uint4*>(from);
      else w = make_uint4(from[0], from[1], from[2], from[3]);
      met |= ((w.x ? 1u : 0u) | (w.y ? 2u : 0u) | (w.z ? 4u : 0u) | (w.w ? 8u : 0u)) << e;
    }
    if (MANY) met |= __funnelshift_r(formed[i >> 5], formed[(i >> 5) + 1], i & 31) & ((1u << E) - 1u);      // (a number may be zero)
    for (; met; met &= met - 1u) {
      const int e = __ffs(met) - 1, k = sizeof(T) == 4 ? e : e >> 1;
      const uint32_t r = k < 2 ? (k == 0 ? r4[0] : r4[1]) : (k == 2 ? r4[2] : r4[3]);
      by_rules(t + e, __uint_as_float(sizeof(T) == 4 ? r : e & 1 ? r & 0xFFFF0000u : r << 16), words[i + e]);
    }
  }
}

spindlekv_status logits_adjust_impl(int n_rows, int vocab, const void* logits, int dtype, int64_t row_stride, const spindlekv_logit_rules& rules, void* out,
                                    int64_t out_stride, cudaStream_t st) {
  LogitsParams p;
  p.in = logits;
  p.out = out;
  p.in_stride = row_stride;
  p.out_stride = out_stride;
  p.r = rules;
  p.vocab = vocab;
  // Slices of whole mask words, as many as fill the SMs once with two blocks each (37 x 50257 bf16, histories of 2500: twice as many slices 12.7 us, these
  // 10.1; masks alone 5.8 and 4.4; 100 x 50000 fp32, masks alone, where the largest slices are more than fill them, 7.2 and 8.0)
  const bool counts = rules.history || rules.n_bias > 0;
  const int64_t wanted = std::max<int64_t>(1, 2 * 148 / n_rows);
  const int64_t slice = std::min<int64_t>(kLogitsMaxSlice, std::max<int64_t>(2048, (vocab + wanted - 1) / wanted));
  p.slice = (int)((slice + 1023) / 1024 * 1024);
  const size_t smem = counts ? (size_t)std::min(p.slice, (vocab + 3) / 4 * 4) * 4 : 0;
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    for (auto kernel : {logits_adjust_kernel<float, false>, logits_adjust_kernel<float, true>, logits_adjust_kernel<__nv_bfloat16, false>, logits_adjust_kernel<__nv_bfloat16, true>})
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLogitsMaxSlice * 4) != cudaSuccess) return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  const dim3 grid((vocab + p.slice - 1) / p.slice, n_rows);
  LaunchScope ls(KC_LOGITS, st);
  const bool many = rules.n_bias > kLogitsFewBiases;
  if (dtype == SPINDLEKV_BF16) (many ? logits_adjust_kernel<__nv_bfloat16, true> : logits_adjust_kernel<__nv_bfloat16, false>)<<<grid, kLogitsThreads, smem, st>>>(p);
  else (many ? logits_adjust_kernel<float, true> : logits_adjust_kernel<float, false>)<<<grid, kLogitsThreads, smem, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
