// Beam search's selection: the n_out best of n_beams x vocab continuations of every sequence.
//
// Bound by reading the logits once.  One block walks a slice of a row, tile by tile (8192 logits, 32 per thread in registers after one
// pass of wide loads).  Every thread keeps a running maximum and exp-sum of its own; the slice's go to the workspace, and so do its
// n_out largest logits.  Those are found without sorting: in the first tile the block's threads form 64 groups of four, and the
// n_out-th largest of the groups' maxima is a bound that n_out logits reach and, mostly, a dozen or two in all; in later tiles only what
// exceeds the bound counts (an equal logit has a higher index than n_out others).  The candidates, keys of value and index with the lower
// index above, are ranked by counting.  Where many logits equal the bound (rows that are masked for the most part) the lowest of them are
// read off in order; where a later tile exceeds the bound too often it makes a new one as the first did.  Within a row the order of
// logits is the order of totals.
// The last block of a sequence to arrive joins its slices: log-sum-exp of the beams from the slices' pieces (added in double), totals in
// double, and the same selection over the slices' lists, 2048 entries at a time beside the best so far.  (A second kernel for that cost
// 2 us more, and 3 us on the host.)
// Measured: 4 beams x 32000 bf16 logits 8.7 us (slices 3.5, join 4.5: latency); 128 rows x 128256 fp32 27.2 us (23.9 when the 66 MB of logits
// still lie in L2), a tile 1.9 to 2.5, of which the exponentials are 1: load, exponentials and block barriers follow one another, issue slots 22%
// busy.  More and smaller slices repeat the search for a bound and take 25 to 28 (in L2).
#include <algorithm>

#include <math_constants.h>

#include "common.cuh"

namespace skv {

constexpr int kBeamThreads = 256;
constexpr int kBeamMaxOut = 32;
constexpr int kBeamPer = 8;            // entries per thread and step of the join
constexpr int kBeamGroups = 64;        // groups of threads whose maxima give the bound; at least kBeamMaxOut
constexpr int kBeamGroup = kBeamThreads / kBeamGroups;
static_assert(kBeamGroups >= kBeamMaxOut && kBeamGroup == 4, "the bound is the n_out-th of the groups' maxima; a group is a quad of lanes, and four threads rank one");

struct BeamParams {
  int n_seqs, n_beams, vocab, k, slices;
  int tiles;           // of a slice
  const void* logits;
  int64_t row_stride;
  const float* score;
  const uint8_t* finished;
  int eos;
  float* out_score;
  int32_t *out_parent, *out_token;
  float2* stat;        // [rows][slices] maximum and exp-sum
  int2* cand;          // [rows][slices][k] (logit bits, token), best first; token -1: none
  unsigned long long* arrived;   // [n_seqs]
};
constexpr int kBeamKeep = 256;         // candidates of a slice beyond which only the n_out best are kept
constexpr int kBeamTies = 512;         // candidates of a tile beyond which those equal to the bound are read off in order
constexpr float kLog2e = 1.44269504f;

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

struct Entry {                 // larger: the better one
  unsigned long long value;    // ordered bits of the total
  uint32_t index;              // ~(beam * vocab + token); 0 with value 0: none
};
__device__ __forceinline__ bool better(const Entry& a, const Entry& b) {   // without branches: the loops over it are unrolled
  return (a.value > b.value) | ((a.value == b.value) & (a.index > b.index));
}
__device__ __forceinline__ Entry make_entry(double total, int flat) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(total + 0.0);
  return Entry{(b >> 63) ? ~b : b | 0x8000000000000000ull, (uint32_t)~flat};
}

struct JoinScratch {           // shared memory of the join, where the slice's candidates were
  Entry tops[kBeamGroups];
  Entry found[kBeamMaxOut * kBeamGroup * (kBeamPer + 1)];
  Entry best[kBeamMaxOut];
  Entry bound;
  double base[64];
  int kind[64];                // 0: takes part, 1: finished, 2: offers its tokens at -infinity
  int n_found;
};
__device__ __noinline__ void beam_join(const BeamParams& p, int seq, JoinScratch& sm);

template <typename T, int EPT, bool VEC>
__global__ void __launch_bounds__(kBeamThreads, 4) beam_kernel(const __grid_constant__ BeamParams p) {
  __shared__ __align__(16) float tops[kBeamGroups];
  // what a compaction leaves or a tile adds at most: fewer than n_out groups exceed a bound
  constexpr int kFound = kBeamKeep + kBeamMaxOut * kBeamGroup * EPT + 2 * kBeamTies;
  __shared__ __align__(16) unsigned char scratch[kFound * 8 > sizeof(JoinScratch) ? kFound * 8 : sizeof(JoinScratch)];
  unsigned long long* found = reinterpret_cast<unsigned long long*>(scratch);
  __shared__ float bound, red[2 * (kBeamThreads / 32)];
  __shared__ int n_found, last;
  const int row = blockIdx.y, slice = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the block's results are written: the last block of the sequence joins them
  auto arrive = [&]() {
    __threadfence();
    __syncthreads();
    const int seq = row / p.n_beams;
    if (tid == 0) last = last_to_arrive(p.arrived + seq, p.n_beams * p.slices);
    __syncthreads();
    if (last) {
      __threadfence();
      beam_join(p, seq, *reinterpret_cast<JoinScratch*>(scratch));
    }
  };
  if (!row_runs(p, row)) {
    arrive();
    return;
  }
  if (tid == 0) { n_found = 0; bound = -CUDART_INF_F; }
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1;          // elements per load
  constexpr int kTile = kBeamThreads * EPT;
  const T* x = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  float m = -CUDART_INF_F, sum = 0.f;                       // of this thread's logits
  const int begin = slice * p.tiles * kTile, end = min(begin + p.tiles * kTile, p.vocab);
  for (int s0 = begin; s0 < end; s0 += kTile) {
    float v[EPT];
    auto index = [&](int i) { return s0 + ((i / W) * kBeamThreads + tid) * W + i % W; };   // rises with i
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
    float mx = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < EPT; ++i) mx = fmaxf(mx, v[i]);
    // exp-sum relative to the thread's maximum (a NaN must show in it).  The difference first: a product of the type's lowest value
    // overflows, and a row of nothing else is a uniform one
    {
      const float high = fmaxf(m, mx), ref = high == -CUDART_INF_F ? 0.f : high;
      sum *= m == high ? 1.f : pow2((m - ref) * kLog2e);
      m = high;
#pragma unroll
      for (int i = 0; i < EPT; ++i) sum += pow2((v[i] - ref) * kLog2e);
    }
    // hits of this tile: what exceeds `least`, or what equals it.  What stands behind the row's end, at -infinity, is none
    auto push = [&](float least, bool equal) {
      uint32_t hits = 0;
#pragma unroll
      for (int i = 0; i < EPT; ++i) hits |= (equal ? v[i] == least : v[i] > least) ? 1u << i : 0u;
      for (; hits; hits &= hits - 1) {
        const int at = index(__ffs(hits) - 1);
        if (at >= p.vocab) continue;
        const int slot = atomicAdd(&n_found, 1);
        if (slot < kFound) found[slot] = key_of(to_f32(x[at]), at);      // read once more: the place is not known before
      }
    };
    const int before = s0 == begin ? 0 : n_found;           // (nobody adds to it before the next barrier)
    bool anew = s0 == begin;
    if (!anew) {
      __syncthreads();                                      // everybody knows `before`
      if (mx > bound) push(bound, false);
      __syncthreads();
      anew = n_found > before + kBeamTies;
    }
    if (anew) {
      // ---- a bound from this tile: the n_out-th largest of the groups' maxima (equal ones by their number) ----
      float quad = mx;
#pragma unroll
      for (int o = 1; o < kBeamGroup; o <<= 1) quad = fmaxf(quad, __shfl_xor_sync(0xffffffffu, quad, o));
      if (tid % kBeamGroup == 0) tops[tid / kBeamGroup] = quad;
      __syncthreads();
      {   // four threads to a group, each against a quarter of the groups
        const int mine = tid / 4, from = tid % 4 * (kBeamGroups / 4);
        const float own = tops[mine];
        int rank = 0;
#pragma unroll
        for (int i = from; i < from + kBeamGroups / 4; i += 4) {
          const float4 q = *reinterpret_cast<const float4*>(tops + i);
          rank += ((q.x > own) | ((q.x == own) & (i < mine))) + ((q.y > own) | ((q.y == own) & (i + 1 < mine))) +
                  ((q.z > own) | ((q.z == own) & (i + 2 < mine))) + ((q.w > own) | ((q.w == own) & (i + 3 < mine)));
        }
        rank += __shfl_xor_sync(0xffffffffu, rank, 1);
        rank += __shfl_xor_sync(0xffffffffu, rank, 2);
        if (rank == p.k - 1 && tid % 4 == 0) {
          n_found = before;
          bound = fmaxf(bound, own);                        // (a lower one would not have been exceeded so often)
        }
      }
      __syncthreads();
      const float least = bound;
      if (mx >= least) {                                    // most warps have some: straight from the registers
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
          if (v[i] >= least && index(i) < p.vocab) {
            const int slot = atomicAdd(&n_found, 1);
            if (slot < kFound) found[slot] = key_of(v[i], index(i));
          }
        }
      }
      __syncthreads();
      int above = before;
      bool ties = n_found > before + kBeamTies;             // rarely: so many that those equal to it have to be counted apart
      if (ties) {
        __syncthreads();
        if (tid == 0) n_found = before;
        __syncthreads();
        if (mx > least) push(least, false);
        __syncthreads();
        above = n_found;
        __syncthreads();
        if (mx >= least) push(least, true);
        __syncthreads();
        ties = n_found > above + kBeamTies;
      }
      if (ties) {
        // too many equal it: the lowest n_out of them, in order
        __syncthreads();
        if (warp == 0) {
          int got = 0;
          const int stop = min(s0 + kTile, p.vocab);
          for (int at = s0 + lane; __any_sync(0xffffffffu, at < stop) && got < p.k; at += 32) {
            const bool tie = at < stop && to_f32(x[at]) == least;
            const uint32_t votes = __ballot_sync(0xffffffffu, tie);
            if (tie) found[above + got + __popc(votes & ((1u << lane) - 1u))] = key_of(least, at);
            got += __popc(votes);
          }
          if (lane == 0) n_found = above + got;
        }
        __syncthreads();
      }
    }
    if (n_found > kBeamKeep) {
      // ---- only the n_out best stay; the last of them is the bound ----
      const int n = n_found;
      constexpr int kMine = (kFound + kBeamThreads - 1) / kBeamThreads;
      uint32_t rank_of[kMine];
      unsigned long long mine[kMine];
#pragma unroll 1
      for (int c = 0; c < kMine; ++c) {
        const int at = c * kBeamThreads + tid;
        mine[c] = at < n ? found[at] : 0;
        uint32_t r = 0;
        if (at < n) {
#pragma unroll 4
          for (int j = 0; j < n; ++j) r += found[j] > mine[c];
        }
        rank_of[c] = r;
      }
      __syncthreads();
#pragma unroll 1
      for (int c = 0; c < kMine; ++c) {
        if (mine[c] && rank_of[c] < (uint32_t)p.k) {
          found[rank_of[c]] = mine[c];
          if (rank_of[c] == (uint32_t)p.k - 1) bound = __uint_as_float(key_value_bits(mine[c]));
        }
      }
      if (tid == 0) n_found = min(n, p.k);
      __syncthreads();
    }
  }
  // ---- the slice's maximum and exp-sum ----
  float all = m;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
  if (lane == 0) red[warp] = all;
  __syncthreads();
  all = red[0];
#pragma unroll
  for (int w = 1; w < kBeamThreads / 32; ++w) all = fmaxf(all, red[w]);
  sum *= m == all ? 1.f : pow2((m - (all == -CUDART_INF_F ? 0.f : all)) * kLog2e);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) red[kBeamThreads / 32 + warp] = sum;
  // ---- its best candidates ----
  const int n = n_found;
  int2* out = p.cand + ((int64_t)row * p.slices + slice) * p.k;
  for (int i = tid; i < n; i += kBeamThreads) {
    const unsigned long long q = found[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += found[j] > q;
    if (r < p.k) out[r] = make_int2((int)key_value_bits(q), key_index(q));
  }
  for (int i = n + tid; i < p.k; i += kBeamThreads) out[i] = make_int2(0, -1);
  __syncthreads();
  if (tid == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kBeamThreads / 32; ++w) s += red[kBeamThreads / 32 + w];
    p.stat[(int64_t)row * p.slices + slice] = make_float2(all, s);
  }
  arrive();
}

// All threads of the block.  (A function of its own, so that its registers do not count against the slices' loop.)
__device__ __noinline__ void beam_join(const BeamParams& p, int seq, JoinScratch& sm) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_beam = p.slices * p.k, entries = p.n_beams * per_beam;
  const int2* cand = p.cand + (int64_t)seq * entries;
  int2 raw[kBeamPer];            // the first step's entries are on their way while the log-sum-exps are formed
#pragma unroll
  for (int i = 0; i < kBeamPer; ++i) {
    const int e = i * kBeamThreads + tid;
    raw[i] = e < entries ? __ldcg(cand + e) : make_int2(0, -1);
  }
  for (int w = warp; w < p.n_beams; w += kBeamThreads / 32) {
    const int row = seq * p.n_beams + w;
    const float sc = p.score[row];
    const bool done = p.finished && p.finished[row];
    const float2* st = p.stat + (int64_t)row * p.slices;
    const float2 mine = lane < p.slices ? __ldcg(st + lane) : make_float2(-CUDART_INF_F, 0.f);   // (of a row that runs)
    if (!(fabsf(sc) < CUDART_INF_F)) {
      if (lane == 0) sm.kind[w] = 2;
    } else if (done) {
      if (lane == 0) { sm.kind[w] = 1; sm.base[w] = sc; }
    } else {
      float mx = mine.x;
      for (int i = lane + 32; i < p.slices; i += 32) mx = fmaxf(mx, __ldcg(st + i).x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      // a slice of -infinity alone has the sum 0, or NaN
      auto part = [&](float2 s) { return (double)(s.x == -CUDART_INF_F ? s.y : s.y * expf(s.x - mx)); };
      double sum = part(mine);
      for (int i = lane + 32; i < p.slices; i += 32) sum += part(__ldcg(st + i));
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) {
        const double lse = (double)mx + log(sum);
        const bool fine = lse > -CUDART_INF && lse < CUDART_INF;
        sm.kind[w] = fine ? 0 : 2;
        sm.base[w] = (double)sc - lse;
      }
    }
  }
  for (int i = tid; i < p.k; i += kBeamThreads) sm.best[i] = Entry{0, 0};
  __syncthreads();
  const int offered = min(p.k, p.vocab);      // entries of a beam that does not take part
  const float per_entry = 1.f / (float)per_beam;
  for (int e0 = 0; e0 < entries; e0 += kBeamThreads * kBeamPer) {
    if (tid == 0) { sm.n_found = 0; sm.bound = Entry{0, 1}; }
    Entry mine[kBeamPer + 1];
    Entry top{0, 0};
#pragma unroll
    for (int i = 0; i < kBeamPer; ++i) {
      mine[i] = Entry{0, 0};
      const int e = e0 + i * kBeamThreads + tid;
      if (e < entries) {
        int w = (int)((float)e * per_entry), at = e - w * per_beam;   // a quotient that may be one off
        if (at < 0) { --w; at += per_beam; }
        if (at >= per_beam) { ++w; at -= per_beam; }
        if (sm.kind[w] == 0) {
          const int2 c = e0 ? __ldcg(cand + e) : raw[i];
          if (c.y >= 0) mine[i] = make_entry(sm.base[w] + (double)__int_as_float(c.x), w * p.vocab + c.y);
        } else if (at < offered) {
          int token = at;
          double total = -CUDART_INF;
          if (sm.kind[w] == 1) {                 // the end token first, then the others in order
            token = at == 0 ? p.eos : at <= p.eos ? at - 1 : at;
            if (at == 0) total = sm.base[w];
          }
          mine[i] = make_entry(total, w * p.vocab + token);
        }
      }
      if (better(mine[i], top)) top = mine[i];
    }
    mine[kBeamPer] = tid < p.k ? sm.best[tid] : Entry{0, 0};
    if (better(mine[kBeamPer], top)) top = mine[kBeamPer];
    Entry quad = top;
#pragma unroll
    for (int o = 1; o < kBeamGroup; o <<= 1) {
      const Entry other{__shfl_xor_sync(0xffffffffu, quad.value, o), __shfl_xor_sync(0xffffffffu, quad.index, o)};
      if (better(other, quad)) quad = other;
    }
    if (tid % kBeamGroup == 0) sm.tops[tid / kBeamGroup] = quad;
    __syncthreads();
    {   // four threads to a group, each against a quarter of the groups
      const Entry own = sm.tops[tid / 4];
      int rank = 0;
#pragma unroll
      for (int i = 0; i < kBeamGroups / 4; ++i) rank += better(sm.tops[i * 4 + tid % 4], own);
      rank += __shfl_xor_sync(0xffffffffu, rank, 1);
      rank += __shfl_xor_sync(0xffffffffu, rank, 2);
      if (rank == p.k - 1 && own.value) sm.bound = own;
    }
    __syncthreads();
    const Entry least = sm.bound;
#pragma unroll
    for (int i = 0; i <= kBeamPer; ++i)
      if (mine[i].value && !better(least, mine[i])) sm.found[atomicAdd(&sm.n_found, 1)] = mine[i];
    __syncthreads();
    const int n = sm.n_found;
    for (int i = tid; i < n; i += kBeamThreads) {
      const Entry q = sm.found[i];
      int r = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) r += better(sm.found[j], q);
      if (r < p.k) sm.best[r] = q;
    }
    __syncthreads();
  }
  for (int i = tid; i < p.k; i += kBeamThreads) {
    const Entry q = sm.best[i];
    const int flat = (int)~q.index, w = flat / p.vocab;
    const unsigned long long b = (q.value >> 63) ? q.value & 0x7FFFFFFFFFFFFFFFull : ~q.value;
    const int64_t at = (int64_t)seq * p.k + i;
    p.out_score[at] = (float)__longlong_as_double((long long)b);
    p.out_parent[at] = seq * p.n_beams + w;
    p.out_token[at] = flat - w * p.vocab;
  }
}

// How a row is cut.  Tiles of 32 logits per thread, as many to a block as keep all blocks on the device at once (four to an SM); where
// that leaves SMs without a block, tiles of 8 per thread and one to a block.
struct BeamCut { int per_thread, tiles, slices; };
static BeamCut beam_cut(int64_t rows, int vocab) {
  const int tiles = ceil_div(vocab, kBeamThreads * 32);
  if (rows * tiles < 148) return BeamCut{8, 1, ceil_div(vocab, kBeamThreads * 8)};
  const int blocks = (int)std::max<int64_t>(1, 592 / rows), per = ceil_div(tiles, blocks);
  return BeamCut{32, per, ceil_div(tiles, per)};
}

size_t beam_workspace_bytes(int n_seqs, int n_beams, int vocab, int k) {
  const size_t rows = (size_t)n_seqs * n_beams, slices = (size_t)beam_cut((int64_t)rows, vocab).slices;
  return kHeaderBytes + align_up(rows * slices * sizeof(float2), 256) + align_up(rows * slices * k * sizeof(int2), 256) + align_up((size_t)n_seqs * 8, 256);
}

template <typename T, int EPT>
static void launch_slices(const BeamParams& p, bool vec, cudaStream_t st) {
  const dim3 grid(p.slices, p.n_seqs * p.n_beams);
  LaunchScope ls(KC_BEAM, st);
  if (vec) beam_kernel<T, EPT, true><<<grid, kBeamThreads, 0, st>>>(p);
  else beam_kernel<T, EPT, false><<<grid, kBeamThreads, 0, st>>>(p);
}

spindlekv_status beam_select_impl(int n_seqs, int n_beams, int vocab, int k, const void* logits, int dtype, int64_t row_stride,
                                  const float* score, const uint8_t* finished, int eos, float* out_score, int32_t* out_parent,
                                  int32_t* out_token, void* ws, size_t ws_bytes, cudaStream_t st) {
  if (ws_bytes < beam_workspace_bytes(n_seqs, n_beams, vocab, k)) return SPINDLEKV_WORKSPACE_TOO_SMALL;
  const int64_t rows = (int64_t)n_seqs * n_beams;
  if (rows > 65535) return SPINDLEKV_UNSUPPORTED;
  const BeamCut cut = beam_cut(rows, vocab);
  BeamParams p{n_seqs, n_beams, vocab, k, cut.slices, cut.tiles, logits, row_stride, score, finished, eos,
               out_score, out_parent, out_token, nullptr, nullptr, nullptr};
  uint8_t* at = static_cast<uint8_t*>(ws) + kHeaderBytes;
  p.stat = reinterpret_cast<float2*>(at);
  p.cand = reinterpret_cast<int2*>(at + align_up((size_t)rows * p.slices * sizeof(float2), 256));
  p.arrived = reinterpret_cast<unsigned long long*>(at + align_up((size_t)rows * p.slices * sizeof(float2), 256) +
                                                    align_up((size_t)rows * p.slices * k * sizeof(int2), 256));
  if ((int64_t)n_beams * p.slices > 0xFFFF) return SPINDLEKV_UNSUPPORTED;   // the count has 16 bits
  const int size = dtype == SPINDLEKV_BF16 ? 2 : 4;
  const bool vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && row_stride * size % 16 == 0;
  if (dtype == SPINDLEKV_BF16) {
    if (cut.per_thread == 32) launch_slices<__nv_bfloat16, 32>(p, vec, st);
    else launch_slices<__nv_bfloat16, 8>(p, vec, st);
  } else {
    if (cut.per_thread == 32) launch_slices<float, 32>(p, vec, st);
    else launch_slices<float, 8>(p, vec, st);
  }
  return cudaGetLastError() == cudaSuccess ? SPINDLEKV_OK : SPINDLEKV_CUDA;
}

}  // namespace skv
