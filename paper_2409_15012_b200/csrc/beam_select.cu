// Beam selection: log-softmax over each beam's logits and the best n_out continuations of every
// group of beams.
//
// A candidate (beam, token) scores  score_beam + x - lse_beam,  lse = log sum exp(x) over the
// beam's finite logits.  Within a beam the order is that of the logits, so one pass over the
// logits gives both the sum and the beam's best n_out, and only those meet the other beams:
//   * beam_scan_kernel: one CTA per (beam, chunk of the vocabulary) reads its logits once, keeps
//     a running (maximum, sum) per thread and the chunk's best n_out in shared memory;
//   * beam_merge_kernel: one CTA per group forms lse in double precision, scores the chunks'
//     lists and picks the group's best.
// The scan is bound by HBM (the logits are read once).
//
// Selection without sorting: a tile gives every thread 32 logits.  The n-th largest of the 256
// threads' maxima is a lower bound T of the tile's n-th largest logit, and only n threads have a
// maximum >= T, so at most 32 n logits reach T -- usually barely more than n.  They are ranked
// by counting, together with the list so far.  Once the list is full, a later tile only matters
// if it holds a logit above the list's last one (an equal one has a higher index and loses),
// which one barrier vote tells.  Keys are (logit, ~index), so no two are equal and ties go to the
// lowest index whatever the order of the atomics.
#include <cuda_bf16.h>

#include <type_traits>

#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 32;                       // logits of a tile held by one thread
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Order-preserving image of a finite float; both zeros give the same one.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t make_key(float x, uint32_t index) {
  return ((uint64_t)ordered(x) << 32) | (uint32_t)~index;
}

// Ranks m distinct keys by counting and writes the best n in descending order to `best`;
// returns how many there are.  All threads of the block call it; `keys` and `best` do not overlap.
template <typename Key, typename Greater>
__device__ __forceinline__ int keep_best(const Key* keys, int m, Key* best, int n, Greater greater) {
  for (int i = threadIdx.x; i < m; i += kThreads) {
    const Key k = keys[i];
    int rank = 0;
    for (int j = 0; j < m; ++j) rank += greater(keys[j], k);
    if (rank < n) best[rank] = k;
  }
  __syncthreads();
  return m < n ? m : n;
}

// T: float or __nv_bfloat16
template <typename T>
__global__ void __launch_bounds__(kThreads) beam_scan_kernel(const __grid_constant__ BeamParams p) {
  constexpr int kVec = 16 / (int)sizeof(T);          // logits per 16-byte granule
  constexpr int kVecs = kPerThread / kVec;
  const int row = blockIdx.y, n = p.n_out;
  if (p.finished != nullptr && p.finished[row]) return;   // its logits are not read
  extern __shared__ __align__(16) unsigned char smem[];
  uint64_t* list = reinterpret_cast<uint64_t*>(smem);          // [n] best so far, descending
  uint64_t* tops = list + n;                                    // [kThreads] thread maxima of a tile
  uint64_t* pool = tops + kThreads;                             // [n + 32 n] list and candidates to rank
  __shared__ uint64_t s_floor;
  __shared__ int s_count;
  __shared__ float s_red[2][kThreads / 32];

  // granules of 16 aligned bytes; the row starts `lead` logits into granule 0
  const T* x0 = static_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int lead = (int)((reinterpret_cast<uintptr_t>(x0) & 15) / sizeof(T));
  const T* base = x0 - lead;
  const int granules = (lead + p.vocab + kVec - 1) / kVec;
  const int g0 = blockIdx.x * p.chunk_granules;
  const int g1 = min(granules, g0 + p.chunk_granules);

  float ref = -INFINITY, sum = 0.f;   // largest of this thread's logits, sum of e^(x - ref)
  int have = 0;                       // entries in `list`
  float last = -INFINITY;             // its n-th logit once it is full
  for (int gt = g0; gt < g1; gt += kThreads * kVecs) {
    float x[kPerThread];
    int4 raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int g = gt + v * kThreads + (int)threadIdx.x;
      const int first = g * kVec - lead;      // index of the granule's first logit
      raw[v] = make_int4(0, 0, 0, 0);
      if (g < g1 && first >= 0 && first + kVec <= p.vocab) raw[v] = __ldcs(reinterpret_cast<const int4*>(base) + g);
    }
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int g = gt + v * kThreads + (int)threadIdx.x;
      const int first = g * kVec - lead;
      const int w[4] = {raw[v].x, raw[v].y, raw[v].z, raw[v].w};
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (std::is_same_v<T, float>) x[v * kVec + e] = __int_as_float(w[e]);
        else x[v * kVec + e] = __uint_as_float(e & 1 ? (uint32_t)w[e >> 1] & 0xffff0000u : (uint32_t)w[e >> 1] << 16);
      }
      if (!(g < g1 && first >= 0 && first + kVec <= p.vocab)) {   // past the chunk, or an edge granule: one by one
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          x[v * kVec + e] = -INFINITY;
          if (g < g1 && first + e >= 0 && first + e < p.vocab) x[v * kVec + e] = (float)x0[first + e];
        }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
      x[e] = fabsf(x[e]) < 0x1p126f ? x[e] : -INFINITY;   // only finite logits count (their differences are finite too)
      top = fmaxf(top, x[e]);
    }
    if (top > -INFINITY) {
      // (x - ref is formed before the factor log2(e): x log2(e) - ref log2(e) in one step would carry
      // the rounding of the second product into every term, which is not small for large logits)
      if (top > ref) {
        sum *= ex2((ref - top) * kLog2e);   // (2^-inf = 0 for the first tile)
        ref = top;
      }
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < kPerThread; e += 2) {
        s0 += ex2((x[e] - ref) * kLog2e);
        s1 += ex2((x[e + 1] - ref) * kLog2e);
      }
      sum += s0 + s1;
    }
    // ---- the chunk's best ----
    const bool in = top > last;
    const int n_in = __syncthreads_count(in);
    if (n_in == 0) continue;
    if (threadIdx.x == 0) { s_floor = 0; s_count = have; }
    auto index_of = [&](int e) { return (uint32_t)((gt + (e / kVec) * kThreads + (int)threadIdx.x) * kVec + e % kVec - lead); };
    uint64_t top_key = 0;
    if (in) {
#pragma unroll
      for (int e = kPerThread - 1; e >= 0; --e)
        if (x[e] == top) top_key = make_key(top, index_of(e));   // the lowest index of the maximum
    }
    tops[threadIdx.x] = top_key;
    for (int i = threadIdx.x; i < have; i += kThreads) pool[i] = list[i];
    __syncthreads();
    if (n_in > n && in) {   // the n-th largest maximum
      int rank = 0;
      for (int j = 0; j < kThreads; ++j) rank += tops[j] > top_key;
      if (rank == n - 1) s_floor = top_key;
    }
    __syncthreads();
    const uint64_t floor_key = s_floor;
    if (in && top_key >= floor_key) {
#pragma unroll
      for (int e = 0; e < kPerThread; ++e) {
        if (x[e] > last) {
          const uint64_t key = make_key(x[e], index_of(e));
          if (key >= floor_key) pool[atomicAdd(&s_count, 1)] = key;
        }
      }
    }
    __syncthreads();
    have = keep_best(pool, s_count, list, n, [](uint64_t a, uint64_t b) { return a > b; });
    if (have == n) last = unordered((uint32_t)(list[n - 1] >> 32));
    __syncthreads();   // (the counters and pools are free again)
  }
  // ---- results of the chunk ----
  const int64_t part = (int64_t)row * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < n; i += kThreads) p.part_keys[part * n + i] = i < have ? list[i] : 0;
  float m = ref;
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sh));
  if ((threadIdx.x & 31) == 0) s_red[0][threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, s_red[0][w]);
  float s = ref > -INFINITY ? sum * ex2((ref - m) * kLog2e) : 0.f;
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) s += __shfl_xor_sync(0xffffffffu, s, sh);
  if ((threadIdx.x & 31) == 0) s_red[1][threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) s += s_red[1][w];
    p.part_sums[part] = make_float2(m, s);
  }
}

struct Scored {
  double score;
  int32_t flat;      // beam * vocab + token
  int32_t pad;
};

__global__ void __launch_bounds__(kThreads) beam_merge_kernel(const __grid_constant__ BeamParams p) {
  const int group = blockIdx.x, n = p.n_out, nb = p.n_beams, nc = p.n_chunks;
  extern __shared__ __align__(16) unsigned char smem[];
  Scored* list = reinterpret_cast<Scored*>(smem);                 // [n]
  Scored* pool = list + n;                                         // [n + kThreads]
  double* lse = reinterpret_cast<double*>(pool + n + kThreads);    // [nb]
  __shared__ int s_count;
  auto greater = [](const Scored& a, const Scored& b) { return a.score > b.score || (a.score == b.score && a.flat < b.flat); };

  // lse in double from the chunks' fp32 sums
  for (int b = threadIdx.x; b < nb; b += kThreads) {
    const float2* ps = p.part_sums + (int64_t)(group * nb + b) * nc;
    const bool skip = p.finished != nullptr && p.finished[group * nb + b];
    float m = -INFINITY;
    for (int c = 0; c < nc && !skip; ++c) m = fmaxf(m, ps[c].x);
    double s = 0.0;
    for (int c = 0; c < nc && !skip; ++c)
      if (ps[c].x > -INFINITY) s += (double)ps[c].y * exp((double)ps[c].x - (double)m);
    lse[b] = (double)m + log(s);
  }
  __syncthreads();

  // The chunks' lists are sorted: walk them rank by rank and stop at a rank that adds nothing.
  int have = 0;
  Scored worst = {-INFINITY, 0, 0};
  const int lists = nb * nc;
  bool more = true;
  for (int r = 0; r < n && more; ++r) {
    more = false;
    for (int l0 = 0; l0 < lists; l0 += kThreads) {
      const int l = l0 + (int)threadIdx.x;
      Scored cand = {-INFINITY, 0, 0};
      bool in = false;
      if (l < lists) {
        const int b = l / nc, c = l - b * nc, row = group * nb + b;
        const float start = p.scores[row];
        if (fabsf(start) < INFINITY) {
          if (p.finished != nullptr && p.finished[row]) {
            in = r == 0 && c == 0;
            cand.score = (double)start;
            cand.flat = b * p.vocab + p.eos;
          } else {
            const uint64_t key = p.part_keys[((int64_t)row * nc + c) * n + r];
            in = key != 0;
            cand.score = (double)unordered((uint32_t)(key >> 32)) - lse[b] + (double)start;
            cand.flat = b * p.vocab + (int32_t)(uint32_t)~(uint32_t)key;
          }
          in = in && (have < n || greater(cand, worst));
        }
      }
      if (threadIdx.x == 0) s_count = have;
      for (int i = threadIdx.x; i < have; i += kThreads) pool[i] = list[i];
      const int n_in = __syncthreads_count(in);
      if (n_in == 0) continue;
      more = true;
      if (in) pool[atomicAdd(&s_count, 1)] = cand;
      __syncthreads();
      have = keep_best(pool, s_count, list, n, greater);
      if (have == n) worst = list[n - 1];
      __syncthreads();
    }
  }
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int64_t o = (int64_t)group * n + i;
    p.out_scores[o] = i < have ? (float)list[i].score : -INFINITY;
    p.out_beams[o] = i < have ? list[i].flat / p.vocab : -1;
    p.out_tokens[o] = i < have ? list[i].flat % p.vocab : -1;
  }
}

}  // namespace

// Logits a chunk should hold: enough chunks to give every SM several CTAs, and no more, since
// each chunk hands the merge a list; whole multiples of 2048 so that few lanes idle.
int beam_chunks(int rows, int vocab, int elem_bytes, int sm_count, int* chunk_granules) {
  const int vec = 16 / elem_bytes;
  const int64_t granules = ((int64_t)vocab + vec - 1) / vec + 1;   // + 1: a row may start inside a granule
  const int64_t want = ((int64_t)4 * sm_count + rows - 1) / rows;
  int64_t len = (granules + want - 1) / want;
  len = (len + kThreads - 1) / kThreads * kThreads;
  *chunk_granules = (int)len;
  return (int)((granules + len - 1) / len);
}

cudaError_t launch_beam_scan(const BeamParams& p, int elem_bytes, cudaStream_t st) {
  const size_t smem = (size_t)(34 * p.n_out + kThreads) * sizeof(uint64_t);
  const dim3 grid(p.n_chunks, p.n_groups * p.n_beams);
  if (elem_bytes == 2) beam_scan_kernel<__nv_bfloat16><<<grid, kThreads, smem, st>>>(p);
  else beam_scan_kernel<float><<<grid, kThreads, smem, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_beam_merge(const BeamParams& p, cudaStream_t st) {
  const size_t smem = (size_t)(2 * p.n_out + kThreads) * sizeof(Scored) + (size_t)p.n_beams * sizeof(double);
  beam_merge_kernel<<<p.n_groups, kThreads, smem, st>>>(p);
  return cudaGetLastError();
}

}  // namespace mixattn
