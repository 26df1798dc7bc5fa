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
// shows), marks the biased ones, which it does one by one, and then streams the slice, where a word of counts tells the few tokens that change from the many that do not.
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

// penalties of a token that the history has
__device__ __forceinline__ float penalised(float x, uint32_t word, float rep, float presence, float frequency) {
  if ((word & ~kBiased) == 0u) return x;
  float z = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
  const uint32_t n = word & kCountBits;
  if (n) z = __fsub_rn(z, __fadd_rn(__fmul_rn(frequency, (float)n), presence));
  return z;
}

template <typename T>
__global__ void __launch_bounds__(kLogitsThreads, 2) logits_adjust_kernel(const __grid_constant__ LogitsParams p) {
  constexpr int E = 16 / sizeof(T), V = kLogitsMaxSlice / E / kLogitsThreads;        // elements of 16 bytes; a thread's pieces of 16 bytes
  extern __shared__ uint4 shared[];
  uint32_t* words = reinterpret_cast<uint32_t*>(shared);
  __shared__ uint32_t mask[kLogitsMaxSlice / 32 + 1];
  const int row = blockIdx.y, lo = blockIdx.x * p.slice, hi = min(lo + p.slice, p.vocab), tid = threadIdx.x;
  const T* in = reinterpret_cast<const T*>(p.in) + (int64_t)row * p.in_stride;
  T* out = reinterpret_cast<T*>(p.out) + (int64_t)row * p.out_stride;
  // 16 bytes at a time where both rows lie alike, the elements before and behind one by one.  They are asked for first, and come while the history is counted
  const int off = (int)(reinterpret_cast<uintptr_t>(in + lo) % 16 / sizeof(T));
  const bool alike = reinterpret_cast<uintptr_t>(in + lo) % 16 == reinterpret_cast<uintptr_t>(out + lo) % 16;
  const int first = alike ? min(hi, lo + (off ? E - off : 0)) : hi, vectors = (hi - first) / E, last = first + vectors * E;
  uint4 raw[V];
#pragma unroll
  for (int a = 0; a < V; ++a) {
    const int v = tid + a * kLogitsThreads;
    raw[a] = v < vectors ? *reinterpret_cast<const uint4*>(in + first + v * E) : make_uint4(0u, 0u, 0u, 0u);
  }
  const bool counts = p.r.history || p.r.n_bias > 0, masked = p.r.allowed != nullptr;
  const uint32_t* allowed = p.r.allowed + (int64_t)row * p.r.allowed_stride + lo / 32;
  if (masked)
    for (int i = tid; i < (hi - lo + 31) / 32; i += kLogitsThreads) mask[i] = __ldg(allowed + i);
  float rep = 1.f, presence = 0.f, frequency = 0.f;
  if (counts) {
    for (int i = tid; i < (hi - lo + 3) / 4; i += kLogitsThreads) shared[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    if (p.r.history) {
      if (p.r.repetition) rep = __ldg(p.r.repetition + row);
      if (p.r.presence) presence = __ldg(p.r.presence + row);
      if (p.r.frequency) frequency = __ldg(p.r.frequency + row);
      const int32_t* h = p.r.history + (int64_t)row * p.r.history_stride;
      const int n = p.r.history_lens ? min(max(__ldg(p.r.history_lens + row), 0), p.r.max_history) : p.r.max_history;
      const int prompt = p.r.n_prompt ? __ldg(p.r.n_prompt + row) : 0;
      auto count = [&](int i, int t) {
        if (t < lo || t >= hi) return;
        if (i >= prompt) atomicAdd(words + (t - lo), 1u);
        else atomicOr(words + (t - lo), kInPrompt);
      };
      // 16 bytes at a time from where they begin, and four of those asked for together (one by one: 80 us in place of 53 for 128 rows of up to 16384 tokens)
      const int head = min(n, (int)((16 - reinterpret_cast<uintptr_t>(h) % 16) % 16 / 4)), quads = (n - head) / 4;
      const int4* h4 = reinterpret_cast<const int4*>(h + head);
      if (tid < head) count(tid, __ldg(h + tid));
      for (int i = head + 4 * quads + tid; i < n; i += kLogitsThreads) count(i, __ldg(h + i));
#pragma unroll 1
      for (int q0 = tid; q0 < quads; q0 += 4 * kLogitsThreads) {
        int4 t[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) t[a] = q0 + a * kLogitsThreads < quads ? __ldg(h4 + q0 + a * kLogitsThreads) : make_int4(-1, -1, -1, -1);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int i = head + 4 * (q0 + a * kLogitsThreads);
          count(i, t[a].x);
          count(i + 1, t[a].y);
          count(i + 2, t[a].z);
          count(i + 3, t[a].w);
        }
      }
    }
    for (int i = tid; i < p.r.n_bias; i += kLogitsThreads) {
      const int t = __ldg(p.r.bias_token + (int64_t)row * p.r.n_bias + i);
      if (t >= lo && t < hi) atomicOr(words + (t - lo), kBiased);
    }
  }
  if (counts || masked) __syncthreads();
  auto is_allowed = [&](int t) { return !masked || (mask[(t - lo) >> 5] >> ((t - lo) & 31) & 1u); };
  auto one = [&](int t) {
    const uint32_t word = counts ? words[t - lo] : 0u;
    if (word & kBiased) return;
    out[t] = T(is_allowed(t) ? penalised(to_f32(in[t]), word, rep, presence, frequency) : -CUDART_INF_F);
  };
  for (int t = lo + tid; t < first; t += kLogitsThreads) one(t);
  for (int t = last + tid; t < hi; t += kLogitsThreads) one(t);
  const bool even = (first - lo) % 4 == 0;
#pragma unroll
  for (int a = 0; a < V; ++a) {
    const int v = tid + a * kLogitsThreads, t = first + v * E, i = t - lo;
    if (v >= vectors) break;
    uint32_t word[E], any = 0u, bits = ~0u;
    if (masked) bits = __funnelshift_r(mask[i >> 5], mask[(i >> 5) + 1], i & 31);      // (the word behind the slice's last is there, and its bits are not used)
    if (counts) {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const uint32_t* from = words + i + e;
        if (even) {
          const uint4 w = *reinterpret_cast<const uint4*>(from);
          word[e] = w.x; word[e + 1] = w.y; word[e + 2] = w.z; word[e + 3] = w.w;
        } else {
          word[e] = from[0]; word[e + 1] = from[1]; word[e + 2] = from[2]; word[e + 3] = from[3];
        }
        any |= word[e] | word[e + 1] | word[e + 2] | word[e + 3];
      }
    }
    const uint32_t r4[4] = {raw[a].x, raw[a].y, raw[a].z, raw[a].w};
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
      float x[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(r4[e]);
        else x[e] = __uint_as_float(e & 1 ? r4[e / 2] & 0xFFFF0000u : r4[e / 2] << 16);
        x[e] = bits >> e & 1u ? penalised(x[e], word[e], rep, presence, frequency) : -CUDART_INF_F;
      }
      if (any & kBiased) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!(word[e] & kBiased)) out[t + e] = T(x[e]);
        continue;
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
  // A biased token is the warp's alone that has its first bias: the others have passed it over.  The lanes look through the list together
  const int warp = tid >> 5, lane = tid & 31;
  for (int i = warp; i < p.r.n_bias; i += kLogitsThreads / 32) {
    const int32_t* tok = p.r.bias_token + (int64_t)row * p.r.n_bias;
    const float* val = p.r.bias_value + (int64_t)row * p.r.n_bias;
    const int t = __ldg(tok + i);
    if (t < lo || t >= hi) continue;
    float z = penalised(to_f32(in[t]), words[t - lo], rep, presence, frequency);
    bool mine = true;
    for (int j0 = 0; j0 < p.r.n_bias && mine; j0 += 32) {
      const bool same = j0 + lane < p.r.n_bias && __ldg(tok + j0 + lane) == t;
      const float v = same ? __ldg(val + j0 + lane) : 0.f;
      for (uint32_t left = __ballot_sync(0xffffffffu, same); left; left &= left - 1) {
        const int k = __ffs(left) - 1;
        mine = mine && j0 + k >= i;
        z = __fadd_rn(z, __shfl_sync(0xffffffffu, v, k));
      }
    }
    __syncwarp();
    if (mine && lane == 0) out[t] = T(is_allowed(t) ? z : -CUDART_INF_F);
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
  const size_t smem = rules.history || rules.n_bias > 0 ? (size_t)std::min(p.slice, (vocab + 3) / 4 * 4) * 4 : 0;
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
