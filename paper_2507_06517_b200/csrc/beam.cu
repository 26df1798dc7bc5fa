// Beam search's selection: the n_out best of n_beams x vocab continuations of every sequence.
//
// Bound by reading the logits once.  First kernel, one block per slice of a row: the slice is in registers after one pass of wide
// loads; its maximum and exp-sum go to the workspace, and so do its n_out largest logits.  Those are found without sorting: the
// block's threads form 64 groups of four, and the n_out-th largest of the groups' maxima is a bound that only n_out groups reach, so at
// most n_out times a group's elements remain (a dozen or two, mostly), whatever the values are; they are ranked by counting.  Keys are
// (value, index) with the lower index above, so no two are equal and ties need no care.  Within a row the order of logits is the order of totals.
// Second kernel, one block per sequence: log-sum-exp of the beams from the slices' pieces (added in double), totals in double, and the
// same selection over the slices' lists, 2048 entries at a time beside the best so far.
#include <algorithm>

#include <math_constants.h>

#include "common.cuh"

namespace skv {

constexpr int kBeamThreads = 256;
constexpr int kBeamMaxOut = 32;
constexpr int kBeamPer = 8;            // entries per thread and step of the second kernel
constexpr int kBeamGroups = 64;        // groups of threads whose maxima give the bound; at least kBeamMaxOut
constexpr int kBeamGroup = kBeamThreads / kBeamGroups;
static_assert(kBeamGroups >= kBeamMaxOut && kBeamGroup == 4, "the bound is the n_out-th of the groups' maxima; a group is a quad of lanes");

struct BeamParams {
  int n_seqs, n_beams, vocab, k, slices;
  const void* logits;
  int64_t row_stride;
  const float* score;
  const uint8_t* finished;
  int eos;
  float* out_score;
  int32_t *out_parent, *out_token;
  float2* stat;        // [rows][slices] maximum and exp-sum
  int2* cand;          // [rows][slices][k] (logit bits, token), best first; token -1: none
};

// 2^x, to two units in the last place of fp32; results below the smallest normal number are 0
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// a key whose unsigned order is the order of the value, then of falling index; never 0
__device__ __forceinline__ unsigned long long key_of(float x, int i) {
  const uint32_t b = __float_as_uint(x + 0.f);               // -0 and 0 are one value
  const uint32_t u = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((unsigned long long)u << 32) | (uint32_t)~i;
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ uint32_t key_value_bits(unsigned long long k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return (u & 0x80000000u) ? u & 0x7FFFFFFFu : ~u;
}

// a row that takes part: not finished, and with a finite score
__device__ __forceinline__ bool row_runs(const BeamParams& p, int row) {
  if (p.finished && p.finished[row]) return false;
  return fabsf(p.score[row]) < CUDART_INF_F;
}

template <typename T, int EPT, bool VEC>
__global__ void __launch_bounds__(kBeamThreads) beam_slice_kernel(BeamParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ __align__(16) unsigned long long tops[kBeamGroups];
  __shared__ unsigned long long found[kBeamMaxOut * kBeamGroup * EPT];
  __shared__ unsigned long long bound;
  __shared__ float red[2 * (kBeamThreads / 32)];
  __shared__ int n_found;
  const int row = blockIdx.y, slice = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (!row_runs(p, row)) return;
  if (tid == 0) { n_found = 0; bound = 1; }
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1;          // elements per load
  const T* x = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int s0 = slice * (kBeamThreads * EPT);
  float v[EPT];
  auto index = [&](int i) { return s0 + ((i / W) * kBeamThreads + tid) * W + i % W; };
#pragma unroll
  for (int j = 0; j < EPT / W; ++j) {
    const int at = index(j * W);
    if constexpr (VEC) {
      // whole pieces: the row is 16-byte aligned; the last piece may be short
      if (at + W <= p.vocab) {
        const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(x + at));
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[j * W + i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[j * W + 2 * i] = __uint_as_float(w[i] << 16);
            v[j * W + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[j * W + i] = at + i < p.vocab ? to_f32(x[at + i]) : -CUDART_INF_F;
      }
    } else {
      v[j] = at < p.vocab ? to_f32(x[at]) : -CUDART_INF_F;
    }
  }
  // ---- maximum and its lowest place (a thread's indices rise with i) ----
  float mx = -CUDART_INF_F;
#pragma unroll
  for (int i = 0; i < EPT; ++i) mx = fmaxf(mx, v[i]);
  unsigned long long top = 0;
  if (mx > -CUDART_INF_F) {
    int first = 0;
#pragma unroll
    for (int i = EPT - 1; i >= 0; --i) first = v[i] == mx ? i : first;
    top = key_of(mx, s0 + ((first / W) * kBeamThreads + tid) * W + first % W);
  } else {          // nothing but -infinity (or NaN), some of it perhaps behind the row's end
#pragma unroll
    for (int i = EPT - 1; i >= 0; --i)
      if (v[i] == mx && index(i) < p.vocab) top = key_of(mx, index(i));
  }
  float all = mx;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
  unsigned long long quad = top;
#pragma unroll
  for (int o = 1; o < kBeamGroup; o <<= 1) quad = max(quad, __shfl_xor_sync(0xffffffffu, quad, o));
  if (tid % kBeamGroup == 0) tops[tid / kBeamGroup] = quad;
  if (lane == 0) red[warp] = all;
  __syncthreads();
  // ---- exp-sum (a NaN anywhere must show in it); beside it the n_out-th largest of the groups' maxima ----
  all = red[0];
#pragma unroll
  for (int w = 1; w < kBeamThreads / 32; ++w) all = fmaxf(all, red[w]);
  float sum = 0.f;
  const float ref = all == -CUDART_INF_F ? 0.f : all;
#pragma unroll
  for (int i = 0; i < EPT; ++i) sum += pow2((v[i] - ref) * 1.44269504f);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) red[kBeamThreads / 32 + warp] = sum;
  if (tid < kBeamGroups) {
    const unsigned long long own = tops[tid];
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < kBeamGroups; i += 2) {
      const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(tops + i);
      rank += (q.x > own) + (q.y > own);
    }
    if (rank == p.k - 1 && own) bound = own;
  }
  __syncthreads();
  if (tid == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kBeamThreads / 32; ++w) s += red[kBeamThreads / 32 + w];
    p.stat[(int64_t)row * p.slices + slice] = make_float2(all, s);
  }
  const unsigned long long least = bound;
  if (top >= least) {
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int at = index(i);
      const unsigned long long q = key_of(v[i], at);
      if (at < p.vocab && q >= least) found[atomicAdd(&n_found, 1)] = q;
    }
  }
  __syncthreads();
  const int n = n_found;
  int2* out = p.cand + ((int64_t)row * p.slices + slice) * p.k;
  for (int i = tid; i < n; i += kBeamThreads) {
    const unsigned long long q = found[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += found[j] > q;
    if (r < p.k) out[r] = make_int2((int)key_value_bits(q), key_index(q));
  }
  for (int i = n + tid; i < p.k; i += kBeamThreads) out[i] = make_int2(0, -1);
}

struct Entry {                 // larger: the better one
  unsigned long long value;    // ordered bits of the total
  uint32_t index;              // ~(beam * vocab + token); 0 with value 0: none
};
__device__ __forceinline__ bool better(const Entry& a, const Entry& b) { return a.value > b.value || (a.value == b.value && a.index > b.index); }
__device__ __forceinline__ Entry make_entry(double total, int flat) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(total + 0.0);
  return Entry{(b >> 63) ? ~b : b | 0x8000000000000000ull, (uint32_t)~flat};
}

__global__ void __launch_bounds__(kBeamThreads) beam_join_kernel(BeamParams p) {
  __shared__ Entry tops[kBeamGroups];
  __shared__ Entry found[kBeamMaxOut * kBeamGroup * (kBeamPer + 1)];
  __shared__ Entry best[kBeamMaxOut];
  __shared__ Entry bound;
  __shared__ double base[64];
  __shared__ int kind[64];       // 0: takes part, 1: finished, 2: offers its tokens at -infinity
  __shared__ int n_found;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_beam = p.slices * p.k, entries = p.n_beams * per_beam;
  const int2* cand = p.cand + (int64_t)seq * entries;
  int2 raw[kBeamPer];            // the first step's entries are on their way while the log-sum-exps are formed
#pragma unroll
  for (int i = 0; i < kBeamPer; ++i) {
    const int e = i * kBeamThreads + tid;
    raw[i] = e < entries ? cand[e] : make_int2(0, -1);
  }
  for (int w = warp; w < p.n_beams; w += kBeamThreads / 32) {
    const int row = seq * p.n_beams + w;
    const float sc = p.score[row];
    const bool done = p.finished && p.finished[row];
    if (!(fabsf(sc) < CUDART_INF_F)) {
      if (lane == 0) kind[w] = 2;
    } else if (done) {
      if (lane == 0) { kind[w] = 1; base[w] = sc; }
    } else {
      const float2* st = p.stat + (int64_t)row * p.slices;
      float mx = -CUDART_INF_F;
      for (int i = lane; i < p.slices; i += 32) mx = fmaxf(mx, st[i].x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      double sum = 0.0;
      for (int i = lane; i < p.slices; i += 32) {
        const float2 s = st[i];   // a slice of -infinity alone has the sum 0, or NaN
        sum += s.x == -CUDART_INF_F ? s.y : s.y * expf(s.x - mx);
      }
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) {
        const double lse = (double)mx + log(sum);
        const bool fine = lse > -CUDART_INF && lse < CUDART_INF;
        kind[w] = fine ? 0 : 2;
        base[w] = (double)sc - lse;
      }
    }
  }
  for (int i = tid; i < p.k; i += kBeamThreads) best[i] = Entry{0, 0};
  __syncthreads();
  const int offered = min(p.k, p.vocab);      // entries of a beam that does not take part
  for (int e0 = 0; e0 < entries; e0 += kBeamThreads * kBeamPer) {
    if (tid == 0) { n_found = 0; bound = Entry{0, 1}; }
    Entry mine[kBeamPer + 1];
    Entry top{0, 0};
#pragma unroll
    for (int i = 0; i < kBeamPer; ++i) {
      mine[i] = Entry{0, 0};
      const int e = e0 + i * kBeamThreads + tid;
      if (e < entries) {
        const int w = e / per_beam, at = e - w * per_beam;
        if (kind[w] == 0) {
          const int2 c = e0 ? cand[e] : raw[i];
          if (c.y >= 0) mine[i] = make_entry(base[w] + (double)__int_as_float(c.x), w * p.vocab + c.y);
        } else if (at < offered) {
          int token = at;
          double total = -CUDART_INF;
          if (kind[w] == 1) {                 // the end token first, then the others in order
            token = at == 0 ? p.eos : at <= p.eos ? at - 1 : at;
            if (at == 0) total = base[w];
          }
          mine[i] = make_entry(total, w * p.vocab + token);
        }
      }
      if (better(mine[i], top)) top = mine[i];
    }
    mine[kBeamPer] = tid < p.k ? best[tid] : Entry{0, 0};
    if (better(mine[kBeamPer], top)) top = mine[kBeamPer];
    Entry quad = top;
#pragma unroll
    for (int o = 1; o < kBeamGroup; o <<= 1) {
      const Entry other{__shfl_xor_sync(0xffffffffu, quad.value, o), __shfl_xor_sync(0xffffffffu, quad.index, o)};
      if (better(other, quad)) quad = other;
    }
    if (tid % kBeamGroup == 0) tops[tid / kBeamGroup] = quad;
    __syncthreads();
    if (tid < kBeamGroups) {
      const Entry own = tops[tid];
      int rank = 0;
#pragma unroll 8
      for (int i = 0; i < kBeamGroups; ++i) rank += better(tops[i], own);
      if (rank == p.k - 1 && own.value) bound = own;
    }
    __syncthreads();
    const Entry least = bound;
#pragma unroll
    for (int i = 0; i <= kBeamPer; ++i)
      if (mine[i].value && !better(least, mine[i])) found[atomicAdd(&n_found, 1)] = mine[i];
    __syncthreads();
    const int n = n_found;
    for (int i = tid; i < n; i += kBeamThreads) {
      const Entry q = found[i];
      int r = 0;
      for (int j = 0; j < n; ++j) r += better(found[j], q);
      if (r < p.k) best[r] = q;
    }
    __syncthreads();
  }
  for (int i = tid; i < p.k; i += kBeamThreads) {
    const Entry q = best[i];
    const int flat = (int)~q.index, w = flat / p.vocab;
    const unsigned long long b = (q.value >> 63) ? q.value & 0x7FFFFFFFFFFFFFFFull : ~q.value;
    const int64_t at = (int64_t)seq * p.k + i;
    p.out_score[at] = (float)__longlong_as_double((long long)b);
    p.out_parent[at] = seq * p.n_beams + w;
    p.out_token[at] = flat - w * p.vocab;
  }
}

// Elements per thread of a slice: 32 keep the lists that the second kernel reads short; 8 give a call of few rows four times the
// blocks.  The border is one block per SM.
static int beam_per_thread(int64_t rows, int vocab) { return rows * ceil_div(vocab, kBeamThreads * 32) >= 148 ? 32 : 8; }

size_t beam_workspace_bytes(int n_seqs, int n_beams, int vocab, int k) {
  const size_t rows = (size_t)n_seqs * n_beams, slices = (size_t)ceil_div(vocab, kBeamThreads * beam_per_thread((int64_t)rows, vocab));
  return kHeaderBytes + align_up(rows * slices * sizeof(float2), 256) + align_up(rows * slices * k * sizeof(int2), 256);
}

template <typename T, int EPT>
static void launch_slices(const BeamParams& p, bool vec, cudaStream_t st) {
  const dim3 grid(p.slices, p.n_seqs * p.n_beams);
  LaunchScope ls(KC_BEAM, st);
  if (vec) beam_slice_kernel<T, EPT, true><<<grid, kBeamThreads, 0, st>>>(p);
  else beam_slice_kernel<T, EPT, false><<<grid, kBeamThreads, 0, st>>>(p);
}

spindlekv_status beam_select_impl(int n_seqs, int n_beams, int vocab, int k, const void* logits, int dtype, int64_t row_stride,
                                  const float* score, const uint8_t* finished, int eos, float* out_score, int32_t* out_parent,
                                  int32_t* out_token, void* ws, size_t ws_bytes, cudaStream_t st) {
  if (ws_bytes < beam_workspace_bytes(n_seqs, n_beams, vocab, k)) return SPINDLEKV_WORKSPACE_TOO_SMALL;
  const int64_t rows = (int64_t)n_seqs * n_beams;
  if (rows > 65535) return SPINDLEKV_UNSUPPORTED;
  const int per = beam_per_thread(rows, vocab);
  BeamParams p{n_seqs, n_beams, vocab, k, ceil_div(vocab, kBeamThreads * per), logits, row_stride, score, finished, eos,
               out_score, out_parent, out_token, nullptr, nullptr};
  uint8_t* at = static_cast<uint8_t*>(ws) + kHeaderBytes;
  p.stat = reinterpret_cast<float2*>(at);
  p.cand = reinterpret_cast<int2*>(at + align_up((size_t)rows * p.slices * sizeof(float2), 256));
  const int size = dtype == SPINDLEKV_BF16 ? 2 : 4;
  const bool vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && row_stride * size % 16 == 0;
  if (dtype == SPINDLEKV_BF16) {
    if (per == 32) launch_slices<__nv_bfloat16, 32>(p, vec, st);
    else launch_slices<__nv_bfloat16, 8>(p, vec, st);
  } else {
    if (per == 32) launch_slices<float, 32>(p, vec, st);
    else launch_slices<float, 8>(p, vec, st);
  }
  if (cudaGetLastError() != cudaSuccess) return SPINDLEKV_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_seqs);
  cfg.blockDim = dim3(kBeamThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LaunchScope ls(KC_BEAM, st);
  return cudaLaunchKernelEx(&cfg, beam_join_kernel, p) == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
