// Beam selection: log-softmax over each beam's logits and the best n_out continuations of every
// group of beams.
//
// A candidate (beam, token) scores  score_beam + x - lse_beam,  lse = log sum exp(x) over the
// beam's finite logits.  Within a beam the order is that of the logits, so one pass over the
// logits gives both the sum and the beam's best n_out, and only those meet the other beams:
//   * one CTA per (beam, chunk of the vocabulary) reads its logits once, keeps a running (maximum,
//     sum) per thread and the chunk's best n_out in shared memory;
//   * the last CTA of a group to finish (a ticket counter) forms lse in double precision, scores the
//     chunks' lists and picks the group's best.  (A second kernel for this cost 3 us of launch and
//     set-up on the smallest calls.)
// The scan is bound by HBM (the logits are read once): tiles of 16 KB stream into
// shared memory with bulk async copies, two stages per CTA, four CTAs per SM.
//
// The scan is one pass with packed fp32 pairs: per logit about half an instruction each for the
// subtraction of the reference, the factor log2(e), the sum and the maximum, one for unpacking
// bf16 and one exponential.  The reference a thread subtracts is within 2 of the largest logit it
// has seen, so that the terms that matter have small exponents: the subtraction and the product
// round in proportion to them (a reference that may lag by 60 costs 2^-18 of the sum; by 2, and with
// the moves' factors kept to full precision, the logarithm of the sum is right to 2^-20).  A tile
// that holds an infinity or a NaN, which the plain code below would let into the sum, is noticed
// from its maximum and sum and is done over.
//
// Selection without sorting: a thread's logits matter only if they are above the list's n-th
// entry `last`.  The few that are wait in shared memory, and now and then the list
// and what waits are ranked by counting; a tile costs one barrier vote on whether to.  The first
// tile has no `last` yet: it takes the smallest of n or more groups' maxima, which at least n
// logits reach.  Should a tile find no room (sorted or equal logits), the
// threads' maxima are ranked: the n-th largest of them is reached by at least n logits of n
// threads, at most a tile's share (16 or 32) each.  Keys are (logit, ~index), so no two are equal
// and ties go to the lowest index whatever the order of the atomics.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "f32x2.cuh"
#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                             // 16-byte loads of a tile per thread
constexpr int kScanCtas = 4;                         // CTAs of the scan per SM
constexpr int kStages = 2;                           // tiles in shared memory
constexpr int kTileBytes = kThreads * kVecs * 16;
constexpr int kPending = 512;                        // candidates of a chunk waiting to be ranked
constexpr long long kWaitLimitCycles = 4000000000ll; // about two seconds of SM clock
constexpr float kMaxLead = 2.f;                      // of a logit over the reference: see below
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eRest = 1.9259629911e-8f;       // log2(e) - kLog2e

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// e^(a - b) for a <= b, with what the difference and the factor log2(e) round off kept in the exponent.
__device__ __forceinline__ float exp_of_lag(float a, float b) {
  const float d = a - b;
  if (!(d > -100.f)) return 0.f;                     // (below fp32's normal numbers; a = -inf among them)
  const float b2 = a - d, a2 = d + b2, rest = (a - a2) + (b2 - b);
  const float p = d * kLog2e;
  const float r = fmaf(d, kLog2e, -p) + fmaf(d, kLog2eRest, rest * kLog2e);
  const float t = ex2(p);
  return fmaf(t, r * 0.6931472f, t);
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
// returns how many there are.  A few keys are compared by 2, 4 or 8 lanes each.  All threads of
// the block call it; `keys` and `best` do not overlap.
template <typename Key, typename Greater>
__device__ __forceinline__ int keep_best(const Key* keys, int m, Key* best, int n, Greater greater) {
  const int share = m <= 32 ? 8 : m <= 64 ? 4 : m <= 128 ? 2 : 1;
  const int part = (int)threadIdx.x & (share - 1);
  const int step = kThreads / share;
  for (int i0 = 0; i0 < m; i0 += step) {
    const int i = i0 + (int)threadIdx.x / share;
    int rank = 0;
    Key k{};
    if (i < m) {
      k = keys[i];
      int j = part;
      for (; j + 7 * share < m; j += 8 * share) {   // (eight loads in flight)
        Key o[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = keys[j + u * share];
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += greater(o[u], k);
      }
      for (; j < m; j += share) rank += greater(keys[j], k);
    }
    for (int sh = 1; sh < share; sh <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, sh);
    if (i < m && part == 0 && rank < n) best[rank] = k;
  }
  __syncthreads();
  return m < n ? m : n;
}

__device__ __forceinline__ float fmax3(float a, float b, float c) {   // one instruction; NaN operands are ignored
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Logit e of a 16-byte granule.
template <typename T>
__device__ __forceinline__ float logit_of(const int4& raw, int e) {
  const int w[4] = {raw.x, raw.y, raw.z, raw.w};
  if constexpr (std::is_same_v<T, float>) return __int_as_float(w[e]);
  else return __uint_as_float(e & 1 ? (uint32_t)w[e >> 1] & 0xffff0000u : (uint32_t)w[e >> 1] << 16);
}
// The same made -inf (bf16: 0xff80).
template <typename T>
__device__ __forceinline__ void drop_logit(int4& raw, int e) {
  int* w = &raw.x;
  if constexpr (std::is_same_v<T, float>) w[e] = (int)0xff800000u;
  else w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffff) | (int)0xff800000u : (w[e >> 1] & (int)0xffff0000u) | 0xff80;
}
// Largest logit of a granule; NaN are ignored.
template <typename T>
__device__ __forceinline__ float granule_max(const int4& raw) {
  if constexpr (std::is_same_v<T, float>) {
    return fmax3(fmaxf(__int_as_float(raw.x), __int_as_float(raw.y)), __int_as_float(raw.z), __int_as_float(raw.w));
  } else {
    auto as2 = [](int w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 m = __hmax2(__hmax2(as2(raw.x), as2(raw.y)), __hmax2(as2(raw.z), as2(raw.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
}
// One bit per logit of granule v of a thread's tile that is above `floor` (for bf16, two logits
// per comparison: the word's low one at bit w, its high one at bit 16 + w, w = 4 v + word).
template <typename T>
__device__ __forceinline__ uint32_t granule_above(const int4& raw, float floor, int v) {
  const int w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t mask = 0;
  if constexpr (std::is_same_v<T, float>) {
#pragma unroll
    for (int e = 0; e < 4; ++e) mask |= __int_as_float(w[e]) > floor ? 1u << (4 * v + e) : 0u;
  } else {
    const __nv_bfloat162 f = __float2bfloat162_rn(floor);   // (exact: floors are bf16 numbers)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      mask |= __hgt2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[e]), f) & (0x00010001u << (4 * v + e));
  }
  return mask;
}
// Place of a mask bit: granule and logit within it.
template <typename T>
__device__ __forceinline__ void place_of(int bit, int* v, int* e) {
  if constexpr (std::is_same_v<T, float>) {
    *v = bit >> 2;
    *e = bit & 3;
  } else {
    *v = (bit & 15) >> 2;
    *e = 2 * (bit & 3) + (bit >> 4);
  }
}
// The set bit with the lowest logit index.
template <typename T>
__device__ __forceinline__ int first_bit(uint32_t mask) {
  if constexpr (std::is_same_v<T, float>) return __ffs(mask) - 1;
  const int w = __ffs((mask | mask >> 16) & 0xffffu) - 1;
  return mask >> w & 1u ? w : w + 16;
}
// The number just below x (x finite) in T's own steps, as a float.
template <typename T>
__device__ __forceinline__ float below(float x) {
  constexpr uint32_t step = std::is_same_v<T, float> ? 1u : 0x10000u;
  return __uint_as_float(x == 0.f ? 0x80000000u + step : x > 0.f ? __float_as_uint(x) - step : __float_as_uint(x) + step);
}
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {   // bounded
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > kWaitLimitCycles) return false;
  return true;
}

// A scored continuation; the score as an order-preserving integer, because ranking compares a lot.
struct Scored {
  uint64_t score;
  int32_t flat;      // beam * vocab + token
  int32_t pad;
};
__device__ __forceinline__ Scored scored(double x, int32_t flat) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return Scored{b >> 63 ? ~b : b | 0x8000000000000000ull, flat, 0};
}
__device__ __forceinline__ double score_of(const Scored& s) {
  return __longlong_as_double((long long)(s.score >> 63 ? s.score & 0x7fffffffffffffffull : ~s.score));
}

constexpr int kMergePool = 512;

// The lists are sorted, so bounds come from one entry of each: with r such that the lists hold
// n entries up to rank r, the k-th largest of their entries of rank r, k = ceil(n / (r + 1)), is
// reached by at least k (r + 1) >= n candidates.  What reaches it is collected and ranked.
__device__ __forceinline__ void merge_group(const BeamParams& p, int group, unsigned char* smem) {
  const int n = p.n_out, nb = p.n_beams, nc = p.n_chunks;
  Scored* list = reinterpret_cast<Scored*>(smem);                 // [n]
  Scored* pool = list + n;                                         // [n + kMergePool]
  double* offset = reinterpret_cast<double*>(pool + n + kMergePool);   // [nb] log of a beam's sum of e^(x - most)
  float* most = reinterpret_cast<float*>(offset + nb);             // [nb] its reference
  float* start = most + nb;                                        // [nb] its score; NaN: no continuation
  uint8_t* done = reinterpret_cast<uint8_t*>(start + nb);          // [nb]
  __shared__ int s_count;
  __shared__ Scored s_floor;
  auto greater = [](const Scored& a, const Scored& b) { return (bool)((a.score > b.score) | ((a.score == b.score) & (a.flat < b.flat))); };   // (no branches)
  const int lists = nb * nc, lane = (int)threadIdx.x & 31;
  const int64_t total = (int64_t)lists * n;
  const uint64_t* keys = p.part_keys + (int64_t)group * total;
  const float2* sums = p.part_sums + (int64_t)group * lists;
  // bounds from rank r0 of the k best lists (see above)
  const int r0 = (n + lists - 1) / lists - 1, k = (n + r0) / (r0 + 1);

  // What the other CTAs left is a trip to L2 away: everything most groups need is asked for at once.
  // (Entries of finished beams are zeros, their sums empty; neither is used.)
  constexpr int kEarly = 4;
  uint64_t early[kEarly], head = 0;
  float2 part = make_float2(-INFINITY, 0.f);
#pragma unroll
  for (int i = 0; i < kEarly; ++i) {
    const int64_t at = (int)threadIdx.x + i * kThreads;
    early[i] = at < total ? __ldcg(keys + at) : 0;
  }
  if ((int)threadIdx.x < lists) head = __ldcg(keys + (int64_t)threadIdx.x * n + r0);
  const int b0 = (int)threadIdx.x >> 5;   // a warp per beam
  if (b0 < nb && lane < nc) part = __ldcg(sums + b0 * nc + lane);
  for (int b = threadIdx.x; b < nb; b += kThreads) {
    const float s = p.scores[group * nb + b];
    start[b] = fabsf(s) < INFINITY ? s : __int_as_float(0x7fc00000);
    done[b] = p.finished != nullptr && p.finished[group * nb + b] != 0;
  }
  if (threadIdx.x == 0) { s_count = 0; s_floor = Scored{0, 0x7fffffff, 0}; }
  __syncthreads();
  // lse in double from the chunks' fp32 sums
  for (int b = b0; b < nb; b += kThreads / 32) {
    if (done[b]) continue;
    if (b != b0) part = lane < nc ? __ldcg(sums + b * nc + lane) : make_float2(-INFINITY, 0.f);
    float m = part.x;
    for (int c = lane + 32; c < nc; c += 32) m = fmaxf(m, __ldcg(sums + b * nc + c).x);
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sh));
    auto share = [&](const float2& x) {   // (most beams have their maximum in one chunk or are one)
      return x.x == m ? (double)x.y : x.x > -INFINITY ? (double)x.y * exp((double)x.x - (double)m) : 0.0;
    };
    double s = share(part);
    for (int c = lane + 32; c < nc; c += 32) s += share(__ldcg(sums + b * nc + c));
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) s += __shfl_xor_sync(0xffffffffu, s, sh);
    if (lane == 0) { offset[b] = log(s); most[b] = m; }
  }
  __syncthreads();

  // entry r of list l, whose key is `key`
  auto candidate = [&](int l, int r, uint64_t key, Scored* out) {
    const int b = l / nc, c = l - b * nc;
    const float s = start[b];
    if (!(fabsf(s) < INFINITY)) return false;
    if (done[b]) {   // one continuation
      *out = scored((double)s, b * p.vocab + p.eos);
      return r == 0 && c == 0;
    }
    // (in this order: next to a reference of 1e38 the logarithm would be lost)
    *out = scored((double)unordered((uint32_t)(key >> 32)) - (double)most[b] - offset[b] + (double)s,
                  b * p.vocab + (int32_t)(uint32_t)~(uint32_t)key);
    return key != 0;
  };
  int have = 0;
  if (lists <= kThreads) {   // (more lists: everything is looked at)
    Scored x;
    const bool in = (int)threadIdx.x < lists && candidate((int)threadIdx.x, r0, head, &x);
    if (in) pool[atomicAdd(&s_count, 1)] = x;
    have = __syncthreads_count(in);
    if (have >= k) {
      keep_best(pool, have, list, k, greater);
      if (threadIdx.x == 0) s_floor = list[k - 1];
    }
    if (threadIdx.x == 0) s_count = 0;
    have = 0;
    __syncthreads();
  }
  Scored floor = s_floor;
  for (int i = 0; (int64_t)i * kThreads < total; ++i) {
    const int64_t at = (int)threadIdx.x + (int64_t)i * kThreads;
    Scored x;
    bool in = false;
    if (at < total) {
      uint64_t key = 0;
#pragma unroll
      for (int j = 0; j < kEarly; ++j)
        if (i == j) key = early[j];
      if (i >= kEarly) key = __ldcg(keys + at);
      in = candidate((int)(at / n), (int)(at % n), key, &x) && !greater(floor, x);
    }
    const int n_in = __syncthreads_count(in);
    if (n_in == 0) continue;
    if (have + n_in > n + kMergePool) {   // (uniform) a full pool shrinks to its best n, which raise the bound
      have = keep_best(pool, have, list, n, greater);
      for (int j = threadIdx.x; j < have; j += kThreads) pool[j] = list[j];
      if (threadIdx.x == 0) s_count = have;
      if (have == n) floor = list[n - 1];
      __syncthreads();
    }
    if (in) pool[atomicAdd(&s_count, 1)] = x;
    have += n_in;
  }
  __syncthreads();
  have = keep_best(pool, have, list, n, greater);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int64_t o = (int64_t)group * n + i;
    p.out_scores[o] = i < have ? (float)score_of(list[i]) : -INFINITY;
    p.out_beams[o] = i < have ? list[i].flat / p.vocab : -1;
    p.out_tokens[o] = i < have ? list[i].flat % p.vocab : -1;
  }
}

// T: float or __nv_bfloat16
template <typename T>
__global__ void __launch_bounds__(kThreads, kScanCtas) beam_select_kernel(const __grid_constant__ BeamParams p) {
  constexpr int kVec = 16 / (int)sizeof(T);          // logits per 16-byte granule
  constexpr int kTileGranules = kThreads * kVecs;
  const int row = blockIdx.y, n = p.n_out;
  const bool finished = p.finished != nullptr && p.finished[row] != 0;   // its logits are not read
  extern __shared__ __align__(128) unsigned char smem[];       // [kStages] tiles, then:
  uint64_t* list = reinterpret_cast<uint64_t*>(smem + kStages * kTileBytes);   // [n] the best so far, descending
  uint64_t* scratch = list + n;                                 // [n + max(kPending, n * logits of a thread)]: see below
  __shared__ uint64_t s_tops[kThreads];
  __shared__ uint64_t s_bar[kStages];
  __shared__ uint64_t s_floor;
  __shared__ int s_count, s_valid;   // pending candidates; of those, the first that found no room
  __shared__ float s_refs[kThreads / 32];
  __shared__ double s_sums[kThreads / 32];
  uint64_t* pending = scratch + n;                              // candidates wait behind n places for the list

  // granules of 16 aligned bytes; the row starts `lead` logits into granule 0
  const T* x0 = static_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int lead = (int)((reinterpret_cast<uintptr_t>(x0) & 15) / sizeof(T));
  const char* base = reinterpret_cast<const char*>(x0 - lead);
  const int granules = (int)(((int64_t)lead + p.vocab + kVec - 1) / kVec);
  const int g0 = blockIdx.x * p.chunk_granules;
  const int g1 = min(granules, g0 + p.chunk_granules);
  // Whole granules [gw0, gw1) are copied; the row's first and last one may be partial and are read one by one.
  const int gw0 = max(g0, lead > 0 ? 1 : 0), gw1 = min(g1, (int)(((int64_t)lead + p.vocab) / kVec));
  const int n_tiles = finished ? 0 : (g1 - g0 + kTileGranules - 1) / kTileGranules;   // (not positive: nothing of the row in this chunk)
  auto issue = [&](int k) {   // thread 0: tile k into its stage
    const int a = max(gw0, g0 + k * kTileGranules), b = min(gw1, g0 + (k + 1) * kTileGranules);
    const uint32_t bar = smem_u32(&s_bar[k % kStages]);
    const uint32_t bytes = b > a ? (uint32_t)(b - a) * 16u : 0u;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
    if (bytes > 0)
      asm volatile(
          "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
          ::"r"(smem_u32(smem + (k % kStages) * kTileBytes) + (uint32_t)(a - g0 - k * kTileGranules) * 16u),
            "l"(base + (int64_t)a * 16), "r"(bytes), "r"(bar)
          : "memory");
  };
  if (threadIdx.x == 0) {
    s_count = 0;
    s_valid = kPending;
    for (int i = 0; i < kStages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&s_bar[i])));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int k = 0; k < min(n_tiles, kStages); ++k) issue(k);
  }
  __syncthreads();

  float ref = -INFINITY, sum = 0.f, rest = 0.f;   // sum + rest = sum of e^(x - ref) over this thread's logits
  float last = -INFINITY;             // logits up to this one are out
  bool full = false;                  // `last` is the n-th best so far (else the first tile is still to come)
  int have = 0;                       // entries in the list
  int waited = n_tiles;               // the tile whose wait ran out
  for (int k = 0; k < n_tiles; ++k) {
    const int gt = g0 + k * kTileGranules;
    unsigned char* tile_at = smem + (k % kStages) * kTileBytes;
    if (k < waited && !mbar_wait(smem_u32(&s_bar[k % kStages]), (k / kStages) & 1)) {
      waited = k;   // the status word tells that the results are invalid; no further copy or wait in this loop
      atomicExch(p.status, kDevWaitTimeout);
    }
    int4 raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) raw[v] = reinterpret_cast<const int4*>(tile_at)[v * kThreads + threadIdx.x];
    if (gt < gw0 || gt + kTileGranules > gw1) {   // the tile holds an end of the row or of the chunk
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int g = gt + v * kThreads + (int)threadIdx.x;
        if (g >= gw0 && g < gw1) continue;
        T edge[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const int64_t i = (int64_t)g * kVec + e - lead;
          edge[e] = g < g1 && i >= 0 && i < p.vocab ? x0[i] : (T)-INFINITY;
        }
        T* to = reinterpret_cast<T*>(tile_at + (size_t)(v * kThreads + threadIdx.x) * 16);
#pragma unroll
        for (int e = 0; e < kVec; ++e) to[e] = edge[e];   // (candidates are looked up there)
        raw[v] = *reinterpret_cast<const int4*>(to);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before a later copy into this stage
    }
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) top = fmaxf(top, granule_max<T>(raw[v]));
    auto add_tile = [&]() {
      const f32x2 minus = pack2(-ref, -ref), log2e = pack2(kLog2e, kLog2e);
      f32x2 s0 = pack2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
#pragma unroll
        for (int e = 0; e < kVec; e += 4) {
          const float2 a = unpack2(mul2(add2(pack2(logit_of<T>(raw[v], e), logit_of<T>(raw[v], e + 1)), minus), log2e));
          const float2 b = unpack2(mul2(add2(pack2(logit_of<T>(raw[v], e + 2), logit_of<T>(raw[v], e + 3)), minus), log2e));
          s0 = add2(s0, pack2(ex2(a.x), ex2(a.y)));
          s1 = add2(s1, pack2(ex2(b.x), ex2(b.y)));
        }
      const float2 s = unpack2(add2(s0, s1));
      return s.x + s.y;
    };
    auto follow = [&]() {   // the reference moves up to the tile's maximum
      if (top > ref + kMaxLead) {
        const float f = exp_of_lag(ref, top);
        sum *= f;
        rest *= f;
        ref = top;
      }
    };
    float tile = 0.f;
    bool over = !(top < INFINITY);                   // an infinity
    if (!over) {
      follow();
      if (ref > -INFINITY) tile = add_tile();        // (else: nothing but -inf and NaN so far)
      over = !(tile < INFINITY);                     // a NaN
    }
    if (over) {
      // only finite logits count: the others become -inf
      top = -INFINITY;
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float x = logit_of<T>(raw[v], e);
          if (fabsf(x) < INFINITY) top = fmaxf(top, x);
          else drop_logit<T>(raw[v], e);
        }
      follow();
      tile = ref > -INFINITY ? add_tile() : 0.f;
    }
    {   // sum + rest += tile; what the addition rounds off goes to rest
      const float s = sum + tile, t2 = s - sum, s2 = s - t2;
      rest += (sum - s2) + (tile - t2);
      sum = s;
    }

    // ---- the chunk's best ----
    float floor_x = last;                            // logits above it are candidates
    if (!full) {
      // first tile: maxima of at least n groups of threads.  A group takes its threads from all
      // warps (every other one if n > 32), so that a short tile leaves none empty.
      float* tops = reinterpret_cast<float*>(s_tops);
      const int lane = (int)threadIdx.x & 31;
      tops[threadIdx.x] = top;
      __syncthreads();
      float m = -INFINITY, odd = -INFINITY;
#pragma unroll
      for (int w = 0; w < kThreads / 32; w += 2) {
        m = fmaxf(m, tops[w * 32 + lane]);
        odd = fmaxf(odd, tops[w * 32 + 32 + lane]);
      }
      m = n > 32 ? fminf(m, odd) : fmaxf(m, odd);                      // 2 x 32 or 32 groups ...
      if (n <= 16) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));   // ... 16 ...
      if (n <= 8) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));    // ... or 8
#pragma unroll
      for (int sh = 1; sh < 32; sh <<= 1) m = fminf(m, __shfl_xor_sync(0xffffffffu, m, sh));
      if (m > -INFINITY) floor_x = below<T>(m);      // (a group without a logit: all are in)
    }
    auto above = [&]() {   // the logits of this thread's tile above floor_x
      uint32_t mask = 0;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) mask |= granule_above<T>(raw[v], floor_x, v);
      return mask;
    };
    auto key_of = [&](int bit) {   // (the value from shared memory: no register is indexed by a variable)
      int v, e;
      place_of<T>(bit, &v, &e);
      const int i = (v * kThreads + (int)threadIdx.x) * kVec + e;
      return make_key((float)reinterpret_cast<const T*>(tile_at)[i], (uint32_t)(gt * kVec - lead + i));
    };
    const auto greater = [](uint64_t a, uint64_t b) { return a > b; };
    uint32_t mask = 0;
    if (__any_sync(0xffffffffu, top > floor_x)) mask = above();
    bool failed = false, crowded = false;
    if (mask != 0) {
      const int c = __popc(mask);
      int at = atomicAdd(&s_count, c);
      if (at + c <= kPending) {
        crowded = at + c > 2 * n + 16;               // rank now and then: the higher `last`, the fewer candidates
        for (; mask != 0; mask &= mask - 1) pending[at++] = key_of(__ffs(mask) - 1);
      } else {
        failed = true;
        atomicMin(&s_valid, at);
      }
    }
    if (__syncthreads_or(failed || crowded) || !full || k + 1 == n_tiles) {
      const bool any_failed = __syncthreads_or(failed);
      const int m = min(s_count, s_valid);
      // the list goes right in front of the pending keys
      uint64_t* keys = pending - have;
      for (int i = threadIdx.x; i < have; i += kThreads) keys[i] = list[i];
      __syncthreads();
      have = keep_best(keys, have + m, list, n, greater);
      if (have == n) {
        last = unordered((uint32_t)(list[n - 1] >> 32));
        full = true;
      }
      if (any_failed) {
        // sorted or equal logits: rank the maxima of the threads that found no room
        // (an equal logit of this tile may still have a lower index than one that found room)
        const uint64_t beat = full ? list[n - 1] : 0;
        if (full) floor_x = fmaxf(floor_x, below<T>(last));
        uint64_t top_key = 0;
        if (failed && top > floor_x) {
          const float f = floor_x;
          floor_x = below<T>(top);
          top_key = key_of(first_bit<T>(above()));   // its lowest index
          floor_x = f;
          if (top_key <= beat) top_key = 0;
        }
        s_tops[threadIdx.x] = top_key;
        if (threadIdx.x == 0) { s_floor = 0; s_count = have; }
        for (int i = threadIdx.x; i < have; i += kThreads) scratch[i] = list[i];
        __syncthreads();
        if (top_key != 0) {
          int rank = 0;
          for (int j = 0; j < kThreads; ++j) rank += s_tops[j] > top_key;
          if (rank == n - 1) s_floor = top_key;
        }
        __syncthreads();
        const uint64_t floor_key = s_floor > beat ? s_floor : beat + 1;
        if (top_key >= floor_key) {
          floor_x = fmaxf(floor_x, below<T>(unordered((uint32_t)(floor_key >> 32))));
          for (mask = above(); mask != 0; mask &= mask - 1) {
            const uint64_t key = key_of(__ffs(mask) - 1);
            if (key >= floor_key) scratch[atomicAdd(&s_count, 1)] = key;
          }
        }
        __syncthreads();
        have = keep_best(scratch, s_count, list, n, greater);
        if (have == n) {
          last = unordered((uint32_t)(list[n - 1] >> 32));
          full = true;
        }
      }
      __syncthreads();
      if (threadIdx.x == 0) { s_count = 0; s_valid = kPending; }
      __syncthreads();
    }
    if (threadIdx.x == 0 && k + kStages < waited) issue(k + kStages);   // (every thread is done with the stage)
  }
  if (threadIdx.x == 0)   // after a wait that ran out: copies may still be on their way into this block's memory
    for (int k = waited; k < min(n_tiles, waited + kStages); ++k)
      mbar_wait(smem_u32(&s_bar[k % kStages]), (k / kStages) & 1);
  // ---- results of the chunk ----
  const int64_t part = (int64_t)row * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < n; i += kThreads) p.part_keys[part * n + i] = i < have ? list[i] : 0;
  float m = ref;
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sh));
  if ((threadIdx.x & 31) == 0) s_refs[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, s_refs[w]);
  double s = ref > -INFINITY ? (double)exp_of_lag(ref, m) * ((double)sum + (double)rest) : 0.0;
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) s += __shfl_xor_sync(0xffffffffu, s, sh);
  if ((threadIdx.x & 31) == 0) s_sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < kThreads / 32; ++w) s += s_sums[w];
    p.part_sums[part] = make_float2(m, (float)s);
  }
  // ---- the last CTA of the group merges its lists ----
  __threadfence();
  __syncthreads();
  const int group = row / p.n_beams;
  if (threadIdx.x == 0) {
    const int32_t before = atomicAdd(&p.tickets[group], 1);
    s_count = before == p.n_beams * (int)gridDim.x - 1;
    if (s_count) p.tickets[group] = 0;   // (as the next call wants it)
  }
  __syncthreads();
  if (!s_count) return;
  __threadfence();
  merge_group(p, group, smem);
}

}  // namespace

// How the rows are cut.  A chunk's first tile fills the list and its last one ranks it, which
// costs about as much as streaming two more tiles, so chunks should be long; but the grid should
// fill whole waves of CTAs.  The best product of the two shares wins.
int beam_chunks(int rows, int vocab, int elem_bytes, int sm_count, int* chunk_granules) {
  const int vec = 16 / elem_bytes;
  const int64_t granules = ((int64_t)vocab + vec - 1) / vec + 1;   // + 1: a row may start inside a granule
  const int64_t slots = (int64_t)kScanCtas * sm_count;
  int64_t best_len = granules;
  double best = 0.0;
  const int64_t most = std::max<int64_t>(std::min<int64_t>((granules + kThreads - 1) / kThreads, std::max<int64_t>(slots / rows, 16)), 1);
  for (int64_t nc = 1; nc <= most; ++nc) {
    int64_t len = (granules + nc - 1) / nc;
    len = (len + kThreads - 1) / kThreads * kThreads;    // whole loads of the block, so that few lanes idle
    const int64_t chunks = (granules + len - 1) / len, ctas = chunks * rows;
    const int64_t waves = (ctas + slots - 1) / slots;
    // time of a wave in tiles, with the overhead, times the waves (less than one wave counts as one)
    const double tiles = (double)len / (kThreads * kVecs) + 2.0;
    const double speed = 1.0 / (tiles * (double)waves);
    if (speed > best * 1.0001) {
      best = speed;
      best_len = len;
    }
  }
  *chunk_granules = (int)best_len;
  return (int)((granules + best_len - 1) / best_len);
}

cudaError_t prepare_beam_select() {
  constexpr auto kAttr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(beam_select_kernel<__nv_bfloat16>, kAttr, 56 * 1024);
  return e == cudaSuccess ? cudaFuncSetAttribute(beam_select_kernel<float>, kAttr, 56 * 1024) : e;
}

cudaError_t launch_beam_select(const BeamParams& p, int elem_bytes, cudaStream_t st) {
  const int keys = 2 * p.n_out + std::max(kPending, p.n_out * kVecs * 16 / elem_bytes);
  const size_t smem = (size_t)kStages * kTileBytes + (size_t)keys * sizeof(uint64_t);
  static_assert((2 * MIXATTN_MAX_BEAM_OUT + kMergePool) * sizeof(Scored) + MIXATTN_MAX_BEAMS * 17 <= kStages * kTileBytes,
                "the merge works where the tiles were");
  const dim3 grid(p.n_chunks, p.n_groups * p.n_beams);
  if (elem_bytes == 2) beam_select_kernel<__nv_bfloat16><<<grid, kThreads, smem, st>>>(p);
  else beam_select_kernel<float><<<grid, kThreads, smem, st>>>(p);
  return cudaGetLastError();
}

}  // namespace mixattn
