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

constexpr int kLogitsThreads = 512, kLogitsMaxSlice = 16384;
constexpr uint32_t kBiased = 1u << 31, kInPrompt = 1u << 30, kCountBits = kInPrompt - 1;

template <typename T>
__device__ __forceinline__ float adjusted(const LogitsParams& p, int row, int t, float x, uint32_t word, bool allowed, float rep, float presence, float frequency) {
  if (!allowed) return -CUDART_INF_F;
  if (word == 0u) return x;
  float z = x;
  if (word & ~kBiased) z = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
  const uint32_t n = word & kCountBits;
  if (n) z = __fsub_rn(z, __fadd_rn(__fmul_rn(frequency, (float)n), presence));
  if (word & kBiased) {
    const int32_t* tok = p.r.bias_token + (int64_t)row * p.r.n_bias;
    for (int i = 0; i < p.r.n_bias; ++i)
      if (__ldg(tok + i) == t) z = __fadd_rn(z, __ldg(p.r.bias_value + (int64_t)row * p.r.n_bias + i));
  }
  return z;
}

template <typename T>
__global__ void __launch_bounds__(kLogitsThreads) logits_adjust_kernel(const __grid_constant__ LogitsParams p) {
  constexpr int E = 16 / sizeof(T);        // elements of 16 bytes
  extern __shared__ uint32_t words[];
  const int row = blockIdx.y, lo = blockIdx.x * p.slice, hi = min(lo + p.slice, p.vocab), tid = threadIdx.x;
  const T* in = reinterpret_cast<const T*>(p.in) + (int64_t)row * p.in_stride;
  T* out = reinterpret_cast<T*>(p.out) + (int64_t)row * p.out_stride;
  const uint32_t* allowed = p.r.allowed ? p.r.allowed + (int64_t)row * p.r.allowed_stride : nullptr;
  float rep = 1.f, presence = 0.f, frequency = 0.f;
  const bool counts = p.r.history || p.r.n_bias > 0;
  if (counts) {
    for (int i = tid; i < hi - lo; i += kLogitsThreads) words[i] = 0u;
    __syncthreads();
    if (p.r.history) {
      if (p.r.repetition) rep = __ldg(p.r.repetition + row);
      if (p.r.presence) presence = __ldg(p.r.presence + row);
      if (p.r.frequency) frequency = __ldg(p.r.frequency + row);
      const int32_t* h = p.r.history + (int64_t)row * p.r.history_stride;
      const int n = p.r.history_lens ? min(max(__ldg(p.r.history_lens + row), 0), p.r.max_history) : p.r.max_history;
      const int prompt = p.r.n_prompt ? __ldg(p.r.n_prompt + row) : 0;
#pragma unroll 8
      for (int i = tid; i < n; i += kLogitsThreads) {
        const int t = __ldg(h + i);
        if (t >= lo && t < hi) {
          if (i >= prompt) atomicAdd(words + (t - lo), 1u);
          else atomicOr(words + (t - lo), kInPrompt);
        }
      }
    }
    for (int i = tid; i < p.r.n_bias; i += kLogitsThreads) {
      const int t = __ldg(p.r.bias_token + (int64_t)row * p.r.n_bias + i);
      if (t >= lo && t < hi) atomicOr(words + (t - lo), kBiased);
    }
    __syncthreads();
  }
  auto one = [&](int t) {
    const bool ok = !allowed || (__ldg(allowed + (t >> 5)) >> (t & 31) & 1u);
    out[t] = T(adjusted<T>(p, row, t, to_f32(in[t]), counts ? words[t - lo] : 0u, ok, rep, presence, frequency));
  };
  // 16 bytes at a time where both rows lie alike; the elements before and behind one by one
  const int off = (int)(reinterpret_cast<uintptr_t>(in + lo) % 16 / sizeof(T));
  const bool alike = reinterpret_cast<uintptr_t>(in + lo) % 16 == reinterpret_cast<uintptr_t>(out + lo) % 16;
  const int first = alike ? min(hi, lo + (off ? E - off : 0)) : hi, vectors = (hi - first) / E, last = first + vectors * E;
  for (int t = lo + tid; t < first; t += kLogitsThreads) one(t);
  for (int t = last + tid; t < hi; t += kLogitsThreads) one(t);
#pragma unroll 4
  for (int v = tid; v < vectors; v += kLogitsThreads) {
    const int t = first + v * E;
    const uint4 raw = *reinterpret_cast<const uint4*>(in + t);
    uint32_t bits = ~0u;
    if (allowed) {
      const int w = t >> 5, s = t & 31;
      bits = __ldg(allowed + w) >> s;
      if (s > 32 - E) bits |= __ldg(allowed + w + 1) << (32 - s);
    }
    float x[E];
    uint32_t word[E], any = 0u;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      word[e] = counts ? words[t - lo + e] : 0u;
      any |= word[e];
    }
    const uint32_t r4[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t o4[4];
    if (any == 0u) {
      // nothing but the mask
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o4[e] = bits >> e & 1u ? r4[e] : 0xFF800000u;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o4[e] = (bits >> (2 * e) & 1u ? r4[e] & 0xFFFFu : 0xFF80u) | (bits >> (2 * e + 1) & 1u ? r4[e] & 0xFFFF0000u : 0xFF800000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(r4[e]);
        else x[e] = __uint_as_float(e & 1 ? r4[e / 2] & 0xFFFF0000u : r4[e / 2] << 16);
        x[e] = adjusted<T>(p, row, t + e, x[e], word[e], bits >> e & 1u, rep, presence, frequency);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
          o4[e] = __float_as_uint(x[e]);
        } else {
          const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
          o4[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
      }
    }
    *reinterpret_cast<uint4*>(out + t) = make_uint4(o4[0], o4[1], o4[2], o4[3]);
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
  // slices of whole mask words, as many as give every SM a few blocks
  const int64_t wanted = std::max<int64_t>(1, 4 * 148 / n_rows);
  const int64_t slice = std::min<int64_t>(kLogitsMaxSlice, std::max<int64_t>(2048, (vocab + wanted - 1) / wanted));
  p.slice = (int)((slice + 1023) / 1024 * 1024);
  const size_t smem = rules.history || rules.n_bias > 0 ? (size_t)std::min(p.slice, vocab) * 4 : 0;
  static PerDeviceOnce once;
  const int dev = PerDeviceOnce::current();
  if (dev < 0) return SPINDLEKV_CUDA;
  if (!once.done[dev]) {
    if (cudaFuncSetAttribute(logits_adjust_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLogitsMaxSlice * 4) != cudaSuccess ||
        cudaFuncSetAttribute(logits_adjust_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLogitsMaxSlice * 4) != cudaSuccess)
      return SPINDLEKV_CUDA;
    once.done[dev] = true;
  }
  const dim3 grid((vocab + p.slice - 1) / p.slice, n_rows);
  LaunchScope ls(KC_LOGITS, st);
  if (dtype == SPINDLEKV_BF16) logits_adjust_kernel<__nv_bfloat16><<<grid, kLogitsThreads, smem, st>>>(p);
  else logits_adjust_kernel<float><<<grid, kLogitsThreads, smem, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
