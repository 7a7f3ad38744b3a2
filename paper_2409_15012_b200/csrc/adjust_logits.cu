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
// independent of their order.  A CTA's part of the row is small enough to be asked for at the very start, 16 bytes
// by 16 into registers, and is on its way while the words are cleared and the list is read; then it is
// adjusted and written.
#include <cuda_bf16.h>

#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kLongList = 32768;
constexpr int kPer = 8;           // 16-byte pieces of the row per thread: 16384 bf16 or 8192 fp32 logits per CTA
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
  float repetition, inv_repetition, frequency, presence, scale;   // scale: 1 / temperature
  const float* bias;
};

// one logit, w = its word, without the division by the temperature.  (Quotients as products with a reciprocal: one more rounding of 2^-24,
// at a fifth of the instructions.)
__device__ __forceinline__ float adjusted(float x, uint32_t w, const Row& r) {
  const uint32_t c = w & kCountMask;
  if (w & (kCountMask | kPromptBit)) x *= x > 0.f ? r.inv_repetition : r.repetition;
  if (c) x -= fmaf(r.frequency, (float)c, r.presence);
  if (w >> kBiasShift) x += r.bias[(w >> kBiasShift) - 1];
  return x;
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
__global__ void __launch_bounds__(kThreads, 3)
adjust_logits_kernel(const __grid_constant__ AdjustParams p, const int cluster, const int spans) {
  extern __shared__ __align__(16) uint32_t words[];
  constexpr int kVec = 16 / sizeof(TI);           // logits per 16-byte load
  constexpr uint32_t kAll = (1u << kVec) - 1;
  const mixattn_logit_rules& ru = p.rules;
  const int rank = blockIdx.x % cluster, at_span = blockIdx.x / cluster;
  const int64_t row = at_span / spans;
  const int span = at_span % spans;
  const int first = (span * cluster + rank) * p.part;             // this CTA's tokens [first, last)
  const int last = min(p.vocab, first + p.part);
  asm volatile("griddepcontrol.wait;" ::: "memory");              // (a no-op after an ordinary launch)

  Row r;
  r.repetition = ru.repetition ? ru.repetition[row] : 1.f;
  r.inv_repetition = 1.f / r.repetition;
  r.frequency = ru.frequency ? ru.frequency[row] : 0.f;
  r.presence = ru.presence ? ru.presence[row] : 0.f;
  const float temperature = ru.temperature ? ru.temperature[row] : 1.f;
  r.scale = fminf(1.f / temperature, 3.4028235e38f);              // (finite: 0 stays 0)
  r.bias = ru.bias_values + row * ru.n_bias;
  const uint32_t* mask = nullptr;
  const int mask_words = (p.vocab + 31) / 32;
  if (ru.allowed) {
    const int64_t which = ru.allowed_rows ? ru.allowed_rows[row] : row;
    if (which >= 0 && which < ru.n_allowed) mask = ru.allowed + which * ru.allowed_stride;
  }
  const TI* in = reinterpret_cast<const TI*>(p.logits) + row * p.row_stride;
  TO* out = reinterpret_cast<TO*>(p.out) + row * p.out_stride;
  const bool skip = p.in_place && temperature == 1.f;             // a token without a word stays as it is

  // 16-byte accesses from the first token on at which both rows are aligned (rows of an odd vocabulary start
  // anywhere; parts are whole 16-byte pieces, so the answer is the same in all of them); single ones where there is none
  int head = 0;
  while (head < kVec && ((((size_t)(in + head)) | ((size_t)(out + head))) & 15)) ++head;
  const bool pieces = head < kVec;
  if (!pieces) head = 0;
  const int v0 = min(first + head, max(last, first));
  const int body = pieces ? max(0, last - v0) / kVec : 0;
  const int pad = (kVec - head) % kVec;                           // the words of a piece are 16-byte aligned
  Vec<TI, kVec> x[kPer];
  uint32_t allow[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int b = threadIdx.x + u * kThreads;
    allow[u] = kAll;
    if (b < body) {
      if (mask) allow[u] = mask_bits(mask, v0 + b * kVec, mask_words) & kAll;
      if (!skip && allow[u] != 0) x[u] = *reinterpret_cast<const Vec<TI, kVec>*>(in + v0 + b * kVec);
    }
  }

  if constexpr (kTable) {
    for (int i = threadIdx.x; i < (p.part + kVec) / 4; i += kThreads) reinterpret_cast<uint4*>(words)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    // the last of several biases for one token counts
    for (int i = threadIdx.x; i < ru.n_bias; i += kThreads) {
      const int t = ru.bias_tokens[row * ru.n_bias + i];
      if (t >= first && t < last) atomicMax(words + (t - first + pad), (uint32_t)(i + 1) << kBiasShift);
    }
    int n = 0, prompt = 0;
    if (ru.tokens) {
      n = ru.n_tokens ? min(max(ru.n_tokens[row], 0), ru.max_tokens) : ru.max_tokens;
      prompt = ru.n_prompt ? min(max(ru.n_prompt[row], 0), n) : 0;
    }
    if (cluster > 1) cluster_sync();   // every CTA's words are cleared and carry their biases
    else __syncthreads();
    const int lo = span * cluster * p.part;                                                      // the cluster's tokens
    const int hi = (int)min((int64_t)p.vocab, (int64_t)lo + (int64_t)cluster * p.part);
    const int32_t* list = ru.tokens + row * ru.token_stride;
    constexpr int kBatch = 8;          // entries in flight per thread
    const int step = cluster * kThreads;
    for (int i0 = rank * kThreads + threadIdx.x; i0 < n; i0 += kBatch * step) {
      int t[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) t[j] = i0 + j * step < n ? list[i0 + j * step] : -1;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (t[j] < lo || t[j] >= hi) continue;   // (another cluster's, or no token at all)
        const bool read = i0 + j * step < prompt;
        if (cluster == 1) {
          uint32_t* at = words + (t[j] - lo + pad);
          if (read) atomicOr(at, kPromptBit);
          else atomicAdd(at, 1u);
        } else {
          const int cta = (t[j] - lo) / p.part;
          const uint32_t to = map_to_cta(smem_u32(words) + 4 * (t[j] - lo - cta * p.part + pad), cta);
          if (read) asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(to), "r"(kPromptBit) : "memory");
          else asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(to), "r"(1u) : "memory");
        }
      }
    }
    if (cluster > 1) cluster_sync();   // (and nobody leaves while others still add to its words)
    else __syncthreads();
  }
  if (first >= last) return;

  auto one = [&](int t) {
    const uint32_t w = kTable ? words[t - first + pad] : 0u;
    const bool ok = mask == nullptr || (__ldg(mask + (t >> 5)) >> (t & 31) & 1u);
    if (!ok) out[t] = rounded<TO>(-INFINITY);
    else if (!skip || w != 0) out[t] = rounded<TO>(adjusted(widened(in[t]), w, r) * r.scale);
  };
  if (!pieces) {
    for (int t = first + threadIdx.x; t < last; t += kThreads) one(t);
    return;
  }
  if ((int)threadIdx.x < v0 - first) one(first + threadIdx.x);
  for (int t = v0 + body * kVec + threadIdx.x; t < last; t += kThreads) one(t);
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int b = threadIdx.x + u * kThreads;
    if (b >= body) break;
    const int t = v0 + b * kVec;
    uint32_t w[kVec], any = 0;
    if constexpr (kTable) {
#pragma unroll
      for (int i = 0; i < kVec; i += 4) {
        const uint4 q = *reinterpret_cast<const uint4*>(words + (t - first + pad) + i);
        w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
        any |= q.x | q.y | q.z | q.w;
      }
    }
    if (skip) {
      if (any == 0 && allow[u] == kAll) continue;
      if (allow[u] != 0) x[u] = *reinterpret_cast<const Vec<TI, kVec>*>(in + t);
    }
    Vec<TO, kVec> y;
    float f[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) f[i] = widened(x[u].v[i]);
    if (any != 0) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (w[i] != 0) f[i] = adjusted(f[i], w[i], r);
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      f[i] *= r.scale;
      if (!(allow[u] >> i & 1u)) f[i] = -INFINITY;
      y.v[i] = rounded<TO>(f[i]);
    }
    *reinterpret_cast<Vec<TO, kVec>*>(out + t) = y;
  }
}

// tokens per CTA at most
template <typename TI>
constexpr int max_part() { return kThreads * kPer * (16 / (int)sizeof(TI)); }
template <typename TI>
constexpr int table_bytes(int part) { return (part + 16 / (int)sizeof(TI)) * 4; }

template <typename TI, typename TO>
cudaError_t prepare() {
  return cudaFuncSetAttribute(adjust_logits_kernel<TI, TO, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, table_bytes<TI>(max_part<TI>()));
}

template <typename TI, typename TO>
cudaError_t launch(AdjustParams& p, int sm_count, cudaStream_t st) {
  const bool table = p.rules.tokens != nullptr || p.rules.n_bias > 0;
  // CTAs per row: enough for the vocabulary, more (up to eight) where rows are few
  int64_t parts = ((int64_t)p.vocab + max_part<TI>() - 1) / max_part<TI>();
  while (parts < 8 && p.n_rows * parts < 2 * sm_count && p.vocab > parts * 2048) parts *= 2;
  // A list of usual length is read by every CTA of the row for itself; only a long one is worth a cluster's two
  // barriers and remote sums (512 rows x 131072: WAS
  const int cluster = p.rules.tokens != nullptr && p.rules.max_tokens > kLongList && parts > 1 ? 8 : 1;
  parts = (parts + cluster - 1) / cluster * cluster;
  p.part = (int)((((int64_t)p.vocab + parts - 1) / parts + 31) / 32 * 32);
  const int spans = (int)(parts / cluster);
  if (p.n_rows * parts > INT32_MAX) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.n_rows * parts));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = table ? table_bytes<TI>(p.part) : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return table ? cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, true>, p, cluster, spans)
               : cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, false>, p, cluster, spans);
}

}  // namespace

cudaError_t prepare_adjust_logits() {
  cudaError_t e = prepare<float, float>();
  if (e == cudaSuccess) e = prepare<__nv_bfloat16, __nv_bfloat16>();
  return e == cudaSuccess ? prepare<__nv_bfloat16, float>() : e;
}

cudaError_t launch_adjust_logits(const AdjustParams& pp, int in_dtype, int out_dtype, int sm_count, cudaStream_t st) {
  AdjustParams p = pp;
  if (in_dtype == MIXATTN_F32) return launch<float, float>(p, sm_count, st);
  return out_dtype == MIXATTN_BF16 ? launch<__nv_bfloat16, __nv_bfloat16>(p, sm_count, st) : launch<__nv_bfloat16, float>(p, sm_count, st);
}

}  // namespace mixattn
