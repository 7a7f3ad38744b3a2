// Prompt attention on CUDA cores with exact fp32 arithmetic (fp32 or bf16 tensors).
//
// Paper, Section 3 with the causal order of Section 1: query i attends to keys j <= i
// (standard layer) or i - window < j <= i (sliding window).  This is the fp32-mode
// prefill and the fallback for shapes the tensor-core kernel does not take.  A sequence's
// queries may sit behind `prefix` keys that earlier calls cached: query row r then has
// position prefix + r among the sequence's prefix + S key rows.
// Flash-attention tiling (32 queries x 32 keys per step, online softmax in base 2); key
// tiles outside the band are skipped.
#include <cuda_bf16.h>

#include <type_traits>

#include "internal.h"
#include "score_shape.cuh"

namespace mixattn {

namespace {

constexpr int kBM = 32, kBN = 32, kThreads = 128;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_out(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

struct Plain {};   // plain scores: no further parameters

// SH: Plain, or ScoreShape for a layer whose scores are capped and / or biased by distance
template <typename T, int D, typename SH>
__global__ void __launch_bounds__(kThreads)
prefill_simple_kernel(const __grid_constant__ PrefillParams p, const __grid_constant__ SH shape) {
  constexpr int kRow = D + 4;          // row pitch: 16-byte aligned, and eight rows apart fall on different banks
  extern __shared__ __align__(16) float sm[];
  float* Qs = sm;                      // [kBM][kRow]
  float* Ks = Qs + kBM * kRow;         // [kBN][kRow]
  float* Vs = Ks + kBN * kRow;         // [kBN][D]
  float* Ps = Vs + kBN * D;            // [kBM][kBN + 4]

  const int b = blockIdx.z, h = blockIdx.y;
  const int S = p.row0[b + 1] - p.row0[b];
  const int i0 = blockIdx.x * kBM;
  if (i0 >= S) return;
  const int g = h / (p.n_q_heads / p.n_kv_heads);
  const int64_t base = p.row0[b], kbase = p.krow0[b];
  const int P = p.prefix[b];            // key rows before the first query
  const T* q = reinterpret_cast<const T*>(p.q);
  const T* k = reinterpret_cast<const T*>(p.k);
  const T* v = reinterpret_cast<const T*>(p.v);
  const int tid = threadIdx.x, r = tid >> 2, c = tid & 3;

  for (int e = tid; e < kBM * D; e += kThreads) {
    const int rr = e / D, d = e - rr * D;
    Qs[rr * kRow + d] = i0 + rr < S ? to_f32(q[((base + i0 + rr) * p.n_q_heads + h) * D + d]) : 0.f;
  }
  float o[D / 4];
#pragma unroll
  for (int e = 0; e < D / 4; ++e) o[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int i = P + i0 + r;  // this thread's query position
  const bool row_ok = i0 + r < S;

  const int n_keys = P + S;
  const int i_last = P + min(S, i0 + kBM) - 1;
  int j_lo = 0;
  if (p.window > 0) j_lo = max(0, P + i0 - p.window + 1) / kBN * kBN;
  // this thread loads channel ld of every kThreads / D-th row of a tile
  constexpr int kStep = kThreads / D, kPer = kBN / kStep;
  const int ld = tid % D, lj = tid / D;
  const int64_t pitch = (int64_t)p.n_kv_heads * D;
  const T* kp = k + (kbase + lj) * pitch + g * D + ld;
  const T* vp = v + (kbase + lj) * pitch + g * D + ld;
  for (int j0 = j_lo; j0 <= i_last; j0 += kBN) {
    __syncthreads();
#pragma unroll 8
    for (int e = 0; e < kPer; ++e) {
      const int jj = lj + e * kStep;
      const bool in = j0 + jj < n_keys;
      const int64_t at = (int64_t)(j0 + e * kStep) * pitch;
      Ks[jj * kRow + ld] = in ? to_f32(kp[at]) : 0.f;
      Vs[jj * D + ld] = in ? to_f32(vp[at]) : 0.f;
    }
    __syncthreads();
    // (the eight sums of a thread advance together, four channels per load; each adds its channels in order)
    float s[kBN / 4];
    float mx = -INFINITY;
#pragma unroll
    for (int jj = 0; jj < kBN / 4; ++jj) s[jj] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      const float4 a = *reinterpret_cast<const float4*>(Qs + r * kRow + d);
#pragma unroll
      for (int jj = 0; jj < kBN / 4; ++jj) {
        const float4 b = *reinterpret_cast<const float4*>(Ks + (c + 4 * jj) * kRow + d);
        s[jj] = fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, s[jj]))));
      }
    }
#pragma unroll
    for (int jj = 0; jj < kBN / 4; ++jj) {
      const int j = j0 + c + 4 * jj;
      const float acc = s[jj];
      const bool seen = j <= i && row_ok && (p.window == 0 || i - j < p.window);
      if constexpr (std::is_same_v<SH, ScoreShape>)
        s[jj] = seen ? shaped_score_exact(acc, shape, shape.biased ? -shape.slope[h] * (float)(i - j) : 0.f) : -INFINITY;
      else
        s[jj] = seen ? acc * p.scale_log2e : -INFINITY;
      mx = fmaxf(mx, s[jj]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float mn = fmaxf(m, mx);
    // a row that has seen no key yet keeps m = -inf: its weights are 0, not NaN
    const float a = mn == -INFINITY ? 1.f : exp2f(m - mn);
    float sum = 0.f;
#pragma unroll
    for (int jj = 0; jj < kBN / 4; ++jj) {
      const float pe = mn == -INFINITY ? 0.f : exp2f(s[jj] - mn);
      Ps[r * (kBN + 4) + c + 4 * jj] = pe;
      sum += pe;
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    l = l * a + sum;
    m = mn;
    __syncwarp();
#pragma unroll
    for (int e = 0; e < D / 4; ++e) o[e] *= a;
    // this thread's channels: groups of four, c, c + 4, c + 8, ...
    for (int jj = 0; jj < kBN; ++jj) {
      const float pe = Ps[r * (kBN + 4) + jj];
#pragma unroll
      for (int e = 0; e < D / 4; e += 4) {
        const float4 x = *reinterpret_cast<const float4*>(Vs + jj * D + 4 * c + 4 * e);
        o[e] = fmaf(pe, x.x, o[e]);
        o[e + 1] = fmaf(pe, x.y, o[e + 1]);
        o[e + 2] = fmaf(pe, x.z, o[e + 2]);
        o[e + 3] = fmaf(pe, x.w, o[e + 3]);
      }
    }
  }
  if (row_ok) {
    T* out = reinterpret_cast<T*>(p.out) + ((base + i0 + r) * p.n_q_heads + h) * D;
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < D / 4; ++e) store_out(out + 4 * c + 16 * (e / 4) + e % 4, o[e] * inv);
  }
}

template <typename T, int D, typename SH>
cudaError_t launch(const PrefillParams& p, const SH& shape, int max_len, cudaStream_t st) {
  const size_t smem = (size_t)((kBM + kBN) * (D + 4) + kBN * D + kBM * (kBN + 4)) * 4;
  cudaError_t e = cudaFuncSetAttribute(prefill_simple_kernel<T, D, SH>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  dim3 grid((max_len + kBM - 1) / kBM, p.n_q_heads, p.n_seqs);
  prefill_simple_kernel<T, D, SH><<<grid, kThreads, smem, st>>>(p, shape);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const PrefillParams& p, int max_len, cudaStream_t st) {
  return p.shape != nullptr ? launch<T, D, ScoreShape>(p, *p.shape, max_len, st)
                            : launch<T, D, Plain>(p, Plain{}, max_len, st);
}

}  // namespace

cudaError_t launch_prefill_simple(const PrefillParams& p, int dtype, int max_len, cudaStream_t st) {
  if (p.n_seqs <= 0 || max_len <= 0) return cudaSuccess;
  if (dtype == MIXATTN_BF16)
    return p.head_dim == 128 ? launch<__nv_bfloat16, 128>(p, max_len, st)
                             : launch<__nv_bfloat16, 64>(p, max_len, st);
  return p.head_dim == 128 ? launch<float, 128>(p, max_len, st) : launch<float, 64>(p, max_len, st);
}

}  // namespace mixattn
