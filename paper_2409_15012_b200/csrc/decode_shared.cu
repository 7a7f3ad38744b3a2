// Decode attention over a tree of shared prefixes: the form for fp32 caches, in exact fp32 arithmetic, and the merge
// of the partial results.  (bf16 and quantised caches: decode_shared_tc.cu.)
//
// Section 5.4's kind of workload has many requests behind the same instruction, and generation with
// several hypotheses many behind the same prompt: their caches share pages, which a decode that goes
// sequence by sequence reads once per sequence.  Here a node of the tree (a range of keys and the sequences that
// have it in common) is read once for the query heads of all of its sequences: they are the rows of
// one flash-attention pass, out = sum_j p_j v_j with p_j = e^(b_j - m), running maximum m and sum l
// per row.  A sequence's result is the merge of the passes along its path from the root,
//     out = sum_c o_c 2^(m_c - M) / sum_c l_c 2^(m_c - M),   M = max_c m_c.
// How the work is cut is described with SharedDecodeParams (internal.h).
#include <cuda_bf16.h>

#include "internal.h"
#include "score_shape.cuh"

namespace mixattn {

namespace {

// ---------------------------------------------------------------- fp32 caches
// 32 rows x 32 keys per step on the CUDA cores; eight threads per row.
constexpr int kRows = 32, kKeys = 32, kThreads = 256, kPerRow = kThreads / kRows;
constexpr int kPad = 4;   // floats between rows: eight rows' 16-byte words fall into different banks

template <int D>
constexpr int simple_smem() { return (2 * kRows * (D + kPad) + kKeys * D + kRows * (kKeys + 1)) * 4; }

template <int D>
__global__ void __launch_bounds__(kThreads) decode_shared_kernel(const __grid_constant__ SharedDecodeParams p) {
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;                              // [kRows][D + kPad]
  float* sk = sq + kRows * (D + kPad);         // [kKeys][D + kPad]
  float* sv = sk + kKeys * (D + kPad);         // [kKeys][D]
  float* sp = sv + kKeys * D;                  // [kRows][kKeys + 1]
  const int tid = threadIdx.x, r = tid / kPerRow, sub = tid % kPerRow;
  const KvGeom& ge = p.geom;
  ShareWalk w = share_begin(p, blockIdx.x);
  ShareSegment s;
  while (share_next(p, blockIdx.x, w, s)) {
    const ShareNode& nd = p.node[s.node];
    const int32_t* tbl = p.table + (int64_t)nd.slot * p.table_stride;
    __syncthreads();   // the previous segment's reads
    for (int e = tid; e < kRows * (D / 4); e += kThreads) {
      const int row = e / (D / 4), c = e - row * (D / 4);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < s.rows) {
        const int R = s.row_first + row;
        const int64_t at = ((int64_t)p.order[s.s0 + R / p.group] * p.n_q_heads + s.g * p.group + R % p.group) * D + 4 * c;
        x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + at);
      }
      *reinterpret_cast<float4*>(sq + row * (D + kPad) + 4 * c) = x;
    }
    const int R = s.row_first + min(r, s.rows - 1);
    const int newest = p.newest[s.s0 + R / p.group];
    const float slope = p.shaped && p.shape.biased ? p.shape.slope[s.g * p.group + R % p.group] : 0.f;
    float m = -INFINITY, l = 0.f, o[D / kPerRow];
#pragma unroll
    for (int j = 0; j < D / kPerRow; ++j) o[j] = 0.f;
    for (int t = s.t0; t < s.t1; t += kKeys) {
      __syncthreads();
      for (int e = tid; e < 2 * kKeys * (D / 4); e += kThreads) {
        const int which = e / (kKeys * (D / 4)), f = e - which * kKeys * (D / 4), key = f / (D / 4), c = f - key * (D / 4);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);   // (what lies behind the last key is not read)
        if (t + key < s.t1)
          x = *reinterpret_cast<const float4*>(p.pool + kv_chunk_offset(ge, tbl[(t + key) / kPage], s.g, which, (t + key) % kPage, c));
        *reinterpret_cast<float4*>(which ? sv + key * D + 4 * c : sk + key * (D + kPad) + 4 * c) = x;
      }
      __syncthreads();
      float x[kKeys / kPerRow];   // keys sub, sub + 8, ...
#pragma unroll
      for (int j = 0; j < kKeys / kPerRow; ++j) x[j] = 0.f;
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        const float4 q = *reinterpret_cast<const float4*>(sq + r * (D + kPad) + c);
#pragma unroll
        for (int j = 0; j < kKeys / kPerRow; ++j) {
          const float4 k = *reinterpret_cast<const float4*>(sk + (sub + kPerRow * j) * (D + kPad) + c);
          x[j] = fmaf(q.w, k.w, fmaf(q.z, k.z, fmaf(q.y, k.y, fmaf(q.x, k.x, x[j]))));
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < kKeys / kPerRow; ++j) {
        const int key = t + sub + kPerRow * j;
        const float y = p.shaped ? shaped_score_exact(x[j], p.shape, -slope * (float)(newest - key)) : x[j] * p.scale_log2e;
        x[j] = key < s.t1 ? y : -INFINITY;
        mx = fmaxf(mx, x[j]);
      }
#pragma unroll
      for (int sh = 1; sh < kPerRow; sh <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
      const float mn = fmaxf(m, mx), a = exp2f(m - mn);   // (the step's first key is there, so mn is finite)
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < kKeys / kPerRow; ++j) {
        x[j] = exp2f(x[j] - mn);
        sum += x[j];
        sp[r * (kKeys + 1) + sub + kPerRow * j] = x[j];
      }
#pragma unroll
      for (int sh = 1; sh < kPerRow; sh <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
      m = mn;
      l = l * a + sum;
      __syncwarp();   // (a row's eight threads are in one warp)
#pragma unroll
      for (int j = 0; j < D / kPerRow; ++j) o[j] *= a;
#pragma unroll 4
      for (int key = 0; key < kKeys; ++key) {
        const float pe = sp[r * (kKeys + 1) + key];
#pragma unroll
        for (int j = 0; j < D / kPerRow; ++j) o[j] = fmaf(pe, sv[key * D + sub + kPerRow * j], o[j]);
      }
      __syncwarp();
    }
    if (r < s.rows) {
      float* to = p.part_o + (int64_t)s.seg_row * D;
#pragma unroll
      for (int j = 0; j < D / kPerRow; ++j) {
        const int d = sub + kPerRow * j;
        to[(d / 4) * s.rows * 4 + r * 4 + d % 4] = o[j];
      }
      if (sub == 0) p.part_ml[s.seg_row + r] = make_float2(m, l);
    }
  }
}

// ---------------------------------------------------------------- merge
// kLanes threads per four channels of an output row take turns over the partial results of the row's path,
// four loads in flight each, and join in shared memory: a row behind a long prefix has some twenty segments,
// and one after the other their latencies were the whole kernel (20 us of 8 sequences' 79).  As many lanes
// as keep the grid within one wave.  The partials
// of a segment lie [D / 4][rows][4], so that the tensor-core kernel, which has a row per thread, writes whole lines.
constexpr int kMergeThreads = 256;

struct Partial {
  float M, L;
  float4 o;
};
__device__ __forceinline__ void join(Partial& a, float m, float l, float4 o) {
  const float mn = fmaxf(a.M, m);
  const float s0 = mn == -INFINITY ? 1.f : exp2f(a.M - mn), s1 = mn == -INFINITY ? 0.f : exp2f(m - mn);
  a.M = mn;
  a.L = a.L * s0 + l * s1;
  a.o.x = a.o.x * s0 + o.x * s1;
  a.o.y = a.o.y * s0 + o.y * s1;
  a.o.z = a.o.z * s0 + o.z * s1;
  a.o.w = a.o.w * s0 + o.w * s1;
}

template <typename T, int kLanes>
__global__ void __launch_bounds__(kMergeThreads, 4) merge_shared_kernel(const __grid_constant__ SharedDecodeParams p) {
  __shared__ Partial sm[kMergeThreads];
  const int D = p.geom.head_dim, per_row = D / 4;
  const int per_block = kMergeThreads / kLanes;                  // (row, channels) pairs per block
  const int kl = threadIdx.x / per_block, local = threadIdx.x % per_block;
  // the heads of a group next to each other (they are neighbouring rows of a segment), then the channels
  const int e = blockIdx.x * per_block + local, g = e / (p.group * per_row), c4 = (e - g * p.group * per_row) / p.group;
  const int hh = e % p.group, h = g * p.group + hh;
  const int i = blockIdx.y;
  const bool there = h < p.n_q_heads;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (a no-op after an ordinary launch)
  Partial acc{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  if (there) {
    int turn = kl;   // this thread's next segment, counted from the node's first
    for (int v = p.leaf[i]; v >= 0; v = p.node[v].parent) {
      const ShareNode& nd = p.node[v];
      int n, step, row;       // segments, rows between them, first row
      int64_t at;             // of the channels, in floats
      const float* po = p.part_o;
      const float2* pm = p.part_ml;
      int64_t o_step;
      if (nd.max_segs < 0) {
        n = -nd.max_segs;
        step = p.n_q_heads;
        row = nd.row0 * p.n_q_heads + h;
        at = (int64_t)row * D + 4 * c4;
        o_step = (int64_t)step * D;
        po = p.split_o;
        pm = p.split_ml;
      } else {
        const int tiles = (nd.t1 - nd.t0 + p.tile_keys - 1) / p.tile_keys;
        const int all = nd.ns * p.group, chunks = (all + p.row_chunk - 1) / p.row_chunk;
        const int R = (i - nd.s0) * p.group + hh, rc = R / p.row_chunk, rows = min(p.row_chunk, all - rc * p.row_chunk);
        const int a = nd.unit0 + (g * chunks + rc) * nd.item_len + p.item_units;
        n = (a + tiles - 1) / p.quota - a / p.quota + 1;
        const int row0 = nd.row0 + (g * all + rc * p.row_chunk) * nd.max_segs, r = R - rc * p.row_chunk;
        step = rows;
        row = row0 + r;
        at = (int64_t)row0 * D + ((int64_t)c4 * rows + r) * 4;
        o_step = (int64_t)rows * D;
      }
      int k = turn;
      for (; k < n; k += 4 * kLanes) {
        float2 ml[4];
        float4 o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kj = k + j * kLanes;
          ml[j] = make_float2(-INFINITY, 0.f);
          o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (kj < n) {
            ml[j] = pm[row + kj * step];
            o[j] = *reinterpret_cast<const float4*>(po + at + kj * o_step);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) join(acc, ml[j].x, ml[j].y, o[j]);
      }
      turn = ((turn - n) % kLanes + kLanes) % kLanes;   // the lanes go on where the others stopped
    }
    if (kl > 0) sm[threadIdx.x] = acc;
  }
  __syncthreads();
  if (kl > 0 || !there) return;
#pragma unroll
  for (int j = 1; j < kLanes; ++j) {
    const Partial& x = sm[j * per_block + local];
    join(acc, x.M, x.L, x.o);
  }
  const float inv = 1.f / acc.L;
  const int64_t at = ((int64_t)p.order[i] * p.n_q_heads + h) * D + 4 * c4;
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.o.x * inv, acc.o.y * inv), hi = __floats2bfloat162_rn(acc.o.z * inv, acc.o.w * inv);
    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  } else {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + at) = make_float4(acc.o.x * inv, acc.o.y * inv, acc.o.z * inv, acc.o.w * inv);
  }
}

}  // namespace

cudaError_t prepare_decode_shared() {
  constexpr auto kAttr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(decode_shared_kernel<128>, kAttr, simple_smem<128>());
  return e == cudaSuccess ? cudaFuncSetAttribute(decode_shared_kernel<64>, kAttr, simple_smem<64>()) : e;
}

cudaError_t launch_decode_shared(const SharedDecodeParams& p, cudaStream_t st) {
  if (p.row_chunk > kRows) return cudaErrorInvalidValue;
  if (p.geom.head_dim == 128) decode_shared_kernel<128><<<p.n_ctas, kThreads, simple_smem<128>(), st>>>(p);
  else decode_shared_kernel<64><<<p.n_ctas, kThreads, simple_smem<64>(), st>>>(p);
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch_merge(const SharedDecodeParams& p, int sm_count, cudaStream_t st) {
  const int64_t n = (int64_t)p.n_q_heads * (p.geom.head_dim / 4), room = (int64_t)sm_count * 4 * kMergeThreads;
  int lanes = 8;
  while (lanes > 1 && n * p.n_seqs * lanes > room) lanes /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((n * lanes + kMergeThreads - 1) / kMergeThreads), p.n_seqs);
  cfg.blockDim = dim3(kMergeThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (lanes == 8) return cudaLaunchKernelEx(&cfg, merge_shared_kernel<T, 8>, p);
  if (lanes == 4) return cudaLaunchKernelEx(&cfg, merge_shared_kernel<T, 4>, p);
  if (lanes == 2) return cudaLaunchKernelEx(&cfg, merge_shared_kernel<T, 2>, p);
  return cudaLaunchKernelEx(&cfg, merge_shared_kernel<T, 1>, p);
}

cudaError_t launch_merge_shared(const SharedDecodeParams& p, int dtype, int sm_count, cudaStream_t st) {
  return dtype == MIXATTN_BF16 ? launch_merge<__nv_bfloat16>(p, sm_count, st) : launch_merge<float>(p, sm_count, st);
}

}  // namespace mixattn
