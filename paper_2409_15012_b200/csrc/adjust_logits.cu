// Penalties for repeated tokens, biases and grammar masks on logits (mixattn_adjust_logits).
//
// What stands between a model's logits and the selection of the next token, per row:
//     a = seen ? (x > 0 ? x / repetition : x * repetition) : x
//     b = a - frequency * c - (c > 0 ? presence : 0)
//     y = (b + bias) / temperature,   -inf where the mask forbids
// Bound by memory: the logits are read and written once.  What a row has seen is a short list of tokens, what the
// logits need is a count per token of the vocabulary: a cluster of CTAs takes a row, each CTA a
// part of the vocabulary with one word per token in its shared memory; each scans its share of the list
// and adds to the word of the CTA that owns the token, through distributed shared memory.  So the list is read once,
// nothing per token of the vocabulary is ever in global memory, and whole-number sums make the result
// independent of their order.  Then each CTA streams its part of the row.
#include <cuda_bf16.h>

#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPart = 24576;   // tokens per CTA: 96 KB of words, two CTAs per SM
// a token's word: times it was generated | occurs in the prompt | 1 + its place in the list of biases
constexpr uint32_t kCountMask = (1u << 20) - 1, kPromptBit = 1u << 20;
constexpr int kBiasShift = 21;
static_assert(MIXATTN_MAX_RULE_TOKENS <= (int)kCountMask && MIXATTN_MAX_RULE_BIASES < (1 << (32 - kBiasShift)), "fields");

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t map_to_cta(uint32_t local, int cta) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(cta));
  return remote;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct Row {                 // one row's rules
  float repetition, frequency, presence, scale;   // scale: bf16 outputs multiply by 1 / temperature
  const float* bias;
};

// one logit; w = its word
template <bool kDivide>
__device__ __forceinline__ float adjusted(float x, uint32_t w, const Row& r) {
  if (w != 0) {
    const uint32_t c = w & kCountMask;
    if (w & (kCountMask | kPromptBit)) x = x > 0.f ? x / r.repetition : x * r.repetition;
    if (c) x -= r.frequency * (float)c + r.presence;
    if (w >> kBiasShift) x += r.bias[(w >> kBiasShift) - 1];
  }
  // (an fp32 result is rounded once per step of the formula; a bf16 one loses nothing by the
  // reciprocal's extra 2^-24)
  return kDivide ? x / r.scale : x * r.scale;
}

template <typename TO>
__device__ __forceinline__ TO rounded(float x) {
  if constexpr (sizeof(TO) == 2) return __float2bfloat16_rn(x);
  else return x;
}
__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(__nv_bfloat16 x) { return __bfloat162float(x); }

// bits [at, at + 8) of a mask of `words` words; at >= 0
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* mask, int at, int words) {
  const int w = at >> 5;
  const uint32_t lo = __ldg(mask + w), hi = (at & 31) > 24 && w + 1 < words ? __ldg(mask + w + 1) : 0u;
  return __funnelshift_r(lo, hi, at & 31);
}

template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Vec { T v[N]; };

// kTable: some token may have a word (a list of tokens or of biases is there)
template <typename TI, typename TO, bool kTable>
__global__ void __launch_bounds__(kThreads) adjust_logits_kernel(const __grid_constant__ AdjustParams p, const int cluster) {
  extern __shared__ __align__(16) uint32_t words[];
  constexpr int kVec = 16 / sizeof(TI);           // logits per 16-byte load
  constexpr bool kDivide = sizeof(TO) == 4;
  const mixattn_logit_rules& ru = p.rules;
  const int rank = blockIdx.x % cluster;
  const int64_t row = blockIdx.x / cluster;
  const int first = (blockIdx.y * cluster + rank) * p.part;       // this CTA's tokens [first, last)
  const int last = min(p.vocab, first + p.part);
  asm volatile("griddepcontrol.wait;" ::: "memory");              // (a no-op after an ordinary launch)

  Row r;
  r.repetition = ru.repetition ? ru.repetition[row] : 1.f;
  r.frequency = ru.frequency ? ru.frequency[row] : 0.f;
  r.presence = ru.presence ? ru.presence[row] : 0.f;
  const float temperature = ru.temperature ? ru.temperature[row] : 1.f;
  r.scale = kDivide ? temperature : 1.f / temperature;
  r.bias = ru.bias_values + row * ru.n_bias;

  if constexpr (kTable) {
    for (int i = threadIdx.x; i < p.part / 4; i += kThreads) reinterpret_cast<uint4*>(words)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    // the last of several biases for one token counts
    for (int i = threadIdx.x; i < ru.n_bias; i += kThreads) {
      const int t = ru.bias_tokens[row * ru.n_bias + i];
      if (t >= first && t < last) atomicMax(words + (t - first), (uint32_t)(i + 1) << kBiasShift);
    }
    int n = 0, prompt = 0;
    if (ru.tokens) {
      n = ru.n_tokens ? min(max(ru.n_tokens[row], 0), ru.max_tokens) : ru.max_tokens;
      prompt = ru.n_prompt ? min(max(ru.n_prompt[row], 0), n) : 0;
    }
    if (cluster > 1) cluster_sync();   // every CTA's words are cleared and carry their biases
    else __syncthreads();
    const int lo = blockIdx.y * cluster * p.part;                                                // the cluster's tokens
    const int hi = (int)min((int64_t)p.vocab, (int64_t)lo + (int64_t)cluster * p.part);
    const int32_t* list = ru.tokens + row * ru.token_stride;
    const uint32_t own = smem_u32(words);
    for (int i = rank * kThreads + threadIdx.x; i < n; i += cluster * kThreads) {
      const int t = list[i];
      if (t < lo || t >= hi) continue;   // (another launch row's part, or no token at all)
      const int cta = (t - lo) / p.part;
      const uint32_t at = own + 4 * (t - lo - cta * p.part), to = cluster > 1 ? map_to_cta(at, cta) : at;
      if (i < prompt) asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(to), "r"(kPromptBit) : "memory");
      else asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(to), "r"(1u) : "memory");
    }
    if (cluster > 1) cluster_sync();   // (and nobody leaves while others still add to its words)
    else __syncthreads();
  }
  if (first >= last) return;

  const uint32_t* mask = nullptr;
  const int mask_words = (p.vocab + 31) / 32;
  if (ru.allowed) {
    const int64_t which = ru.allowed_rows ? ru.allowed_rows[row] : row;
    if (which >= 0 && which < ru.n_allowed) mask = ru.allowed + which * ru.allowed_stride;
  }
  const TI* in = reinterpret_cast<const TI*>(p.logits) + row * p.row_stride;
  TO* out = reinterpret_cast<TO*>(p.out) + row * p.out_stride;
  auto one = [&](int t) {
    const uint32_t w = kTable ? words[t - first] : 0u;
    const bool ok = mask == nullptr || (__ldg(mask + (t >> 5)) >> (t & 31) & 1u);
    if (!ok) out[t] = rounded<TO>(-INFINITY);
    else if (!(p.in_place && w == 0 && temperature == 1.f)) out[t] = rounded<TO>(adjusted<kDivide>(widened(in[t]), w, r));
  };
  // 16-byte accesses from the first token on at which both rows are aligned (rows of an odd
  // vocabulary start anywhere); single ones where there is none
  int head = 0;
  while (head < kVec && ((((size_t)(in + first + head)) | ((size_t)(out + first + head))) & 15)) ++head;
  const int body = head < kVec ? max(0, (last - first - head) / kVec) : 0;
  const int v0 = first + min(head, last - first);
  if (body == 0) {
    for (int t = first + threadIdx.x; t < last; t += kThreads) one(t);
    return;
  }
  if ((int)threadIdx.x < v0 - first) one(first + threadIdx.x);
  for (int t = v0 + body * kVec + threadIdx.x; t < last; t += kThreads) one(t);

  const bool skip = p.in_place && temperature == 1.f;   // a token without a word stays as it is
  constexpr int kUnroll = 4;
  for (int b0 = threadIdx.x; b0 < body; b0 += kUnroll * kThreads) {
    Vec<TI, kVec> x[kUnroll];
    uint32_t w[kUnroll][kVec], allow[kUnroll];
    bool touch[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int b = b0 + u * kThreads;
      touch[u] = b < body;
      if (!touch[u]) continue;
      const int t = v0 + b * kVec;
      uint32_t any = 0;
      if constexpr (kTable) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) any |= w[u][i] = words[t - first + i];
      }
      allow[u] = mask ? mask_bits(mask, t, mask_words) & ((1u << kVec) - 1) : (1u << kVec) - 1;
      if (skip && any == 0 && allow[u] == (1u << kVec) - 1) { touch[u] = false; continue; }
      if (allow[u] != 0) x[u] = *reinterpret_cast<const Vec<TI, kVec>*>(in + t);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!touch[u]) continue;
      const int t = v0 + (b0 + u * kThreads) * kVec;
      Vec<TO, kVec> y;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        float f = -INFINITY;
        if (allow[u] >> i & 1u) f = adjusted<kDivide>(widened(x[u].v[i]), kTable ? w[u][i] : 0u, r);
        y.v[i] = rounded<TO>(f);
      }
      *reinterpret_cast<Vec<TO, kVec>*>(out + t) = y;
    }
  }
}

template <typename TI, typename TO>
cudaError_t prepare() {
  return cudaFuncSetAttribute(adjust_logits_kernel<TI, TO, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxPart * 4);
}

template <typename TI, typename TO>
cudaError_t launch(const AdjustParams& p, int cluster, int spans, cudaStream_t st) {
  const bool table = p.rules.tokens != nullptr || p.rules.n_bias > 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_rows * cluster, spans);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = table ? p.part * 4 : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return table ? cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, true>, p, cluster)
               : cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, false>, p, cluster);
}

}  // namespace

cudaError_t prepare_adjust_logits() {
  cudaError_t e = prepare<float, float>();
  if (e == cudaSuccess) e = prepare<__nv_bfloat16, __nv_bfloat16>();
  return e == cudaSuccess ? prepare<__nv_bfloat16, float>() : e;
}

cudaError_t launch_adjust_logits(const AdjustParams& pp, int in_dtype, int out_dtype, int sm_count, cudaStream_t st) {
  AdjustParams p = pp;
  // CTAs per row: enough for the vocabulary at kMaxPart tokens each, and up to eight where rows are few
  int cluster = 1;
  while (cluster < 8 && ((int64_t)cluster * kMaxPart < p.vocab || (p.n_rows * cluster < 2 * sm_count && p.vocab > cluster * 2048)))
    cluster *= 2;
  const int64_t per = ((int64_t)p.vocab + cluster - 1) / cluster;
  p.part = (int)((per < kMaxPart ? per : kMaxPart) + 31) / 32 * 32;
  const int spans = (int)(((int64_t)p.vocab + (int64_t)cluster * p.part - 1) / ((int64_t)cluster * p.part));
  if (spans > 65535) return cudaErrorInvalidValue;
  if (in_dtype == MIXATTN_F32) return launch<float, float>(p, cluster, spans, st);
  return out_dtype == MIXATTN_BF16 ? launch<__nv_bfloat16, __nv_bfloat16>(p, cluster, spans, st)
                                   : launch<__nv_bfloat16, float>(p, cluster, spans, st);
}

}  // namespace mixattn
