// Penalties for repeated tokens, biases and grammar masks on logits (mixattn_adjust_logits).
//
// What stands between a model's logits and the choice of the next token, per row:
//     a = seen ? (x > 0 ? x / repetition : x * repetition) : x
//     b = a - frequency * c - (c > 0 ? presence : 0)
//     y = (b + bias) / temperature,   -inf where the mask forbids
// Bound by memory: the logits are read and written once.  What a row has seen is a short list of tokens, what the
// logits need is a count per token of the vocabulary.  A CTA takes parts of rows (up to 12288 bf16 or 6144
// fp32 logits): it asks for the part's logits, 16 bytes by 16 into registers, reads the row's list meanwhile and
// adds up, in one word per token of the part in shared memory, what is said about the token (whole-number
// sums: the result does not depend on their order), then adjusts and writes, and clears the words that were not
// zero for its next part.  512 rows x 131072 bf16 with lists of 100 to 9000 tokens: 93 us.  On the way: a cluster of CTAs per
// row that shared one reading of the list, through distributed shared memory, 317 against 312; the tokens of the list
// taken out of the words one by one beside the stream, 286, by warps of their own, 258, or put adjusted in the
// words' place by a second reading of the list, 171; quotients instead of products with a reciprocal, 278.
#include <cuda_bf16.h>

#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 6;           // 16-byte pieces per thread
constexpr int kCtasPerSm = 4;     // (the words: 48 KB; with 8 pieces per thread and three CTAs 15 us more, with 4 and four 22)
// a token's word: times it was generated | occurs in the prompt | 1 + its place in the list of biases
constexpr uint32_t kCountMask = (1u << 20) - 1, kPromptBit = 1u << 20;
constexpr int kBiasShift = 21;
static_assert(MIXATTN_MAX_RULE_TOKENS <= (int)kCountMask && MIXATTN_MAX_RULE_BIASES < (1 << (32 - kBiasShift)), "fields");

// What a row divides by, as a factor.  bf16 results take the product with the reciprocal, one more rounding of 2^-24
// beside their 2^-8.  fp32 results take the reciprocal in two terms, cut off and not rounded in the first, so that the
// second is positive (for an infinity): x hi + x lo, rounded once, is the quotient within half a step (1 + 2^-21).
// (fp32 rows with lists of 2000 tokens, 512 x 131072: 114 us with products, 121 so, 126 corrected by the quotient's residual,
// 154 with divisions; penalties alone in place 120, 136.)  Divisors at the ends of fp32's range, whose reciprocal is none or an inexact one, are left to the
// division itself: their rows go one logit at a time.  (0 is no divisor; it multiplies by fp32's largest number, so that
// a logit of 0 does not turn into a NaN.)
__device__ __forceinline__ bool ordinary(float by) { return (by >= 0x1p-120f && by <= 0x1p60f) || by == 0.f; }
__device__ __forceinline__ float cut_off_reciprocal(float x) { return __frcp_rz(x); }
template <bool kExact>
struct Inverse {
  float hi, lo;
  Inverse() = default;
  __device__ __forceinline__ explicit Inverse(float by) : hi(fminf(kExact ? cut_off_reciprocal(by) : 1.f / by, 3.4028235e38f)), lo(0.f) {
    if (kExact) lo = by == 0.f ? 0x1p-149f : fmaxf(fmaf(-by, hi, 1.f) / by, 0x1p-149f);
  }
  __device__ __forceinline__ float times(float x) const { return kExact ? fmaf(x, hi, x * lo) : x * hi; }
};

template <bool kExact>
struct Row {                      // one row's rules
  float repetition, frequency, presence;
  Inverse<kExact> inv_repetition;
  const float* bias;
};

// A logit whose token's word is w, but for the temperature.
template <bool kExact>
__device__ __forceinline__ float adjusted(float x, uint32_t w, const Row<kExact>& r, bool divide = false) {
  const uint32_t c = w & kCountMask;
  if (w & (kCountMask | kPromptBit)) {
    const bool up = x > 0.f;
    if constexpr (kExact) {
      if (divide) x = up ? x / r.repetition : x * r.repetition;
      else x = fmaf(x, up ? r.inv_repetition.hi : r.repetition, up ? x * r.inv_repetition.lo : -0.f);   // (adding -0 changes nothing)
    }
    else x = up && divide ? x / r.repetition : x * (up ? r.inv_repetition.hi : r.repetition);
  }
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

// bits [at, at + 8) of a mask of `words` words, of which lo is the one with bit `at`; at >= 0
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* mask, uint32_t lo, int at, int words) {
  const int w = at >> 5;
  const uint32_t hi = (at & 31) > 24 && w + 1 < words ? __ldg(mask + w + 1) : 0u;
  return __funnelshift_r(lo, hi, at & 31);
}

// f(tokens, index of the first) for the entries of a list, eight at a time per thread; -1 where there is none
template <typename F>
__device__ __forceinline__ void for_each_8(const int32_t* list, int n, F f) {
  const int tid = threadIdx.x;
  const int lead = min((int)(-(intptr_t)((size_t)list >> 2) & 3), n), quads = (n - lead) / 4, tail = lead + 4 * quads;
  const int4* at = reinterpret_cast<const int4*>(list + lead);
  for (int q = 2 * tid; q < quads; q += 2 * kThreads) {
    const int4 a = at[q], b = q + 1 < quads ? at[q + 1] : make_int4(-1, -1, -1, -1);
    const int t[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    f(t, lead + 4 * q);
  }
  if (tid < 2) {   // in front of the first 16-byte boundary, behind the last
    const int first = tid ? tail : 0, end = tid ? n : lead;
    int t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = first + j < end ? list[first + j] : -1;
    f(t, first);
  }
}

// What a part of a row has to do with.
template <typename TI, typename TO>
struct Part {
  static constexpr int kVec = 16 / sizeof(TI);    // logits per 16-byte load
  int64_t row;
  int first, last;                                // tokens [first, last)
  const TI* in;
  TO* out;
  const uint32_t* mask;
  int v0, body;                                   // first token and number of whole pieces
  bool pieces;
  float temperature;
  __device__ __forceinline__ Part(const AdjustParams& p, int64_t item, int parts) {
    const mixattn_logit_rules& ru = p.rules;
    row = item / parts;
    first = (int)(item - row * parts) * p.part;
    last = min(p.vocab, first + p.part);
    in = reinterpret_cast<const TI*>(p.logits) + row * p.row_stride;
    out = reinterpret_cast<TO*>(p.out) + row * p.out_stride;
    temperature = ru.temperature ? ru.temperature[row] : 1.f;
    mask = nullptr;
    if (ru.allowed) {
      const int64_t which = ru.allowed_rows ? ru.allowed_rows[row] : row;
      if (which >= 0 && which < ru.n_allowed) mask = ru.allowed + which * ru.allowed_stride;
    }
    // 16-byte accesses from the first token on at which both rows are aligned (rows of an odd vocabulary
    // start anywhere); single ones where there is none
    const int head_in = (int)(-(intptr_t)((size_t)(in + first) / sizeof(TI)) & (kVec - 1));
    pieces = ((size_t)(out + first + head_in) & 15) == 0;
    v0 = pieces ? min(first + head_in, last) : last;
    body = max(0, last - v0) / kVec;
  }
  __device__ __forceinline__ bool allowed(int t) const { return mask == nullptr || (__ldg(mask + (t >> 5)) >> (t & 31) & 1u); }
};

// kTable: some token may have a word (a list of tokens or of biases is there).  parts: CTAs' worth of work per row
template <typename TI, typename TO, bool kTable>
__global__ void __launch_bounds__(kThreads, kTable ? kCtasPerSm : 4)
adjust_logits_kernel(const __grid_constant__ AdjustParams p, const int parts) {
  using P = Part<TI, TO>;
  constexpr bool kExact = sizeof(TO) == 4;
  constexpr int kVec = P::kVec;
  constexpr uint32_t kAll = (1u << kVec) - 1;
  extern __shared__ __align__(16) uint32_t words[];
  const mixattn_logit_rules& ru = p.rules;
  const int tid = threadIdx.x;
  const int64_t items = (int64_t)p.n_rows * parts;
  if constexpr (kTable)
    for (int i = tid; i < (p.part + 2 * kVec) / 4; i += kThreads) reinterpret_cast<uint4*>(words)[i] = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("griddepcontrol.wait;" ::: "memory");                  // (a no-op after an ordinary launch)
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const P a(p, item, parts);
    const bool still = p.in_place && a.temperature == 1.f;            // a token that no rule names stays as it is
    const Inverse<kExact> cooled(a.temperature);
    const uint4* src = reinterpret_cast<const uint4*>(a.in + a.v0);
    uint4 x[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (tid + u * kThreads < a.body && !still) x[u] = src[tid + u * kThreads];
    uint32_t* word = words;                                           // of token a.first; those of a piece are 16-byte aligned
    Row<kExact> r;
    if constexpr (kTable) {
      word += a.pieces ? (kVec - (a.v0 - a.first) % kVec) % kVec : 0;
      int n = 0, prompt = 0;
      if (ru.tokens) {
        n = ru.n_tokens ? min(max(ru.n_tokens[a.row], 0), ru.max_tokens) : ru.max_tokens;
        prompt = ru.n_prompt ? min(max(ru.n_prompt[a.row], 0), n) : 0;
      }
      r.repetition = ru.repetition ? ru.repetition[a.row] : 1.f;
      r.inv_repetition = Inverse<kExact>(r.repetition);
      r.frequency = ru.frequency ? ru.frequency[a.row] : 0.f;
      r.presence = ru.presence ? ru.presence[a.row] : 0.f;
      r.bias = ru.bias_values + a.row * ru.n_bias;
      const unsigned span = a.last > a.first ? a.last - a.first : 0;
      __syncthreads();                                                // the words are zero
      if (ru.n_bias > 0) {
        // the last of several biases for one token counts: the largest place, while nothing else is in the words
        for (int i = tid; i < ru.n_bias; i += kThreads) {
          const unsigned at = (unsigned)(ru.bias_tokens[a.row * ru.n_bias + i] - a.first);
          if (at < span) atomicMax(word + at, (uint32_t)(i + 1) << kBiasShift);
        }
        __syncthreads();
      }
      for_each_8(ru.tokens + a.row * ru.token_stride, n, [&](const int (&t)[8], int i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unsigned at = (unsigned)(t[j] - a.first);             // (another part's, or no token at all)
          if (t[j] < 0 || at >= span) continue;
          if (i + j < prompt) atomicOr(word + at, kPromptBit);
          else atomicAdd(word + at, 1u);
        }
      });
      __syncthreads();
    }
    bool divide = !ordinary(a.temperature);
    if constexpr (kTable) divide = divide || !ordinary(r.repetition);
    uint32_t lo[kPer];                                                // the pieces' mask words, all under way at once (one after the other: 102 us)
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (a.mask && tid + u * kThreads < a.body) lo[u] = __ldg(a.mask + ((a.v0 + (tid + u * kThreads) * kVec) >> 5));
    auto one = [&](int t) {
      uint32_t w = 0u;
      if constexpr (kTable) {
        w = word[t - a.first];
        word[t - a.first] = 0u;
      }
      if (!a.allowed(t)) {
        a.out[t] = rounded<TO>(-INFINITY);
      } else if (!still || w != 0u) {
        float f = widened(a.in[t]);
        if (kTable && w != 0u) f = adjusted<kExact>(f, w, r, divide);
        a.out[t] = rounded<TO>(divide ? f / a.temperature : cooled.times(f));
      }
    };
    if (!a.pieces || divide) {
      for (int t = a.first + tid; t < a.last; t += kThreads) one(t);
      continue;
    }
    if (tid < a.v0 - a.first) one(a.first + tid);
    for (int t = a.v0 + a.body * kVec + tid; t < a.last; t += kThreads) one(t);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int b = tid + u * kThreads, t = a.v0 + b * kVec;
      if (b >= a.body) break;
      const uint32_t allow = a.mask ? mask_bits(a.mask, lo[u], t, (p.vocab + 31) / 32) & kAll : kAll;
      uint32_t w[kVec], any = 0u;
      if constexpr (kTable) {
        uint4* at = reinterpret_cast<uint4*>(word + (t - a.first));
#pragma unroll
        for (int i = 0; i < kVec / 4; ++i) {
          const uint4 q = at[i];
          w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
          any |= q.x | q.y | q.z | q.w;
        }
        if (any != 0u)
#pragma unroll
          for (int i = 0; i < kVec / 4; ++i) at[i] = make_uint4(0u, 0u, 0u, 0u);
      }
      if (still) {
        if (any == 0u && allow == kAll) continue;
        x[u] = src[b];
      }
      const uint32_t v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      float f[kVec];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kVec == 8) {
          f[2 * i] = __uint_as_float(v[i] << 16);
          f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        } else {
          f[i] = __uint_as_float(v[i]);
        }
      }
      if (kTable && any != 0u) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (w[i] != 0u) f[i] = adjusted<kExact>(f[i], w[i], r);
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) f[i] = cooled.times(f[i]);
      if (allow != kAll) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (!(allow >> i & 1u)) f[i] = -INFINITY;
      }
      uint4* to = reinterpret_cast<uint4*>(a.out + t);
      if constexpr (sizeof(TO) == 2) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
          y[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *to = make_uint4(y[0], y[1], y[2], y[3]);
      } else {
#pragma unroll
        for (int i = 0; i < kVec / 4; ++i)
          to[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3]));
      }
    }
  }
}

// tokens per part at most, and the words of a part
template <typename TI>
constexpr int max_part() { return kThreads * kPer * (16 / (int)sizeof(TI)); }
template <typename TI>
constexpr int table_bytes(int part) { return (part + 2 * (16 / (int)sizeof(TI))) * 4; }

template <typename TI, typename TO>
cudaError_t prepare() {
  return cudaFuncSetAttribute(adjust_logits_kernel<TI, TO, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, table_bytes<TI>(max_part<TI>()));
}

template <typename TI, typename TO>
cudaError_t launch(AdjustParams& p, int sm_count, cudaStream_t st) {
  const bool table = p.rules.tokens != nullptr || p.rules.n_bias > 0;
  // parts per row: as few as registers and shared memory allow, more (down to 2048 tokens each) where rows are few
  int64_t parts = ((int64_t)p.vocab + max_part<TI>() - 1) / max_part<TI>();
  while (p.n_rows * parts < 2 * sm_count && p.vocab > parts * 2048) parts *= 2;
  p.part = (int)((((int64_t)p.vocab + parts - 1) / parts + 31) / 32 * 32);
  const int64_t items = p.n_rows * parts;
  if (parts > INT32_MAX) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  const int64_t slots = (int64_t)sm_count * (table ? kCtasPerSm : 4);
  cfg.gridDim = dim3((unsigned)(items < slots ? items : slots));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = table ? table_bytes<TI>(p.part) : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return table ? cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, true>, p, (int)parts)
               : cudaLaunchKernelEx(&cfg, adjust_logits_kernel<TI, TO, false>, p, (int)parts);
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
