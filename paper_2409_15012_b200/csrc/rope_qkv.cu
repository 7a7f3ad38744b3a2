// Rotary embedding of a projection's rows on their way into a cache (mixattn_rope_qkv).
//
// Section 3 of the paper rotates queries and keys (RoFormer's embedding): channel pair (x, y) of a head
// vector at position t turns by t f_p,
//     x' = x cos - y sin,   y' = x sin + y cos,
// pairs (2p, 2p + 1) or (p, p + n/2).  Bound by memory: every row is read and written once, 16 bytes per access.
// A thread keeps one place of the head vectors of one token, two 16-byte chunks that hold whole
// pairs, and goes over the heads: the sines it needs stay in registers.  A block's sines are
// formed once, in shared memory: the angle in double precision (positions reach 10^5 and beyond, the first pairs turn
// by a radian per position), reduced by whole turns, sine and cosine in fp32.  The product of position and
// frequency reaches 2 10^15, where a double's step is 1/4: its rounding error and 2 pi's are carried along, which leaves
// the reduced angle good to 2^-49 everywhere.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;

template <typename T>
struct Chunk {                        // 16 bytes as fp32
  static constexpr int N = 16 / sizeof(T);
  float f[N];
};
__device__ __forceinline__ void widen(Chunk<__nv_bfloat16>& c, uint4 w) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c.f[2 * i] = __uint_as_float(v[i] << 16);
    c.f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(Chunk<float>& c, uint4 w) {
  c.f[0] = __uint_as_float(w.x); c.f[1] = __uint_as_float(w.y); c.f[2] = __uint_as_float(w.z); c.f[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ uint4 bits_of(const Chunk<__nv_bfloat16>& c) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(c.f[2 * i], c.f[2 * i + 1]);
    v[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint4 bits_of(const Chunk<float>& c) {
  return make_uint4(__float_as_uint(c.f[0]), __float_as_uint(c.f[1]), __float_as_uint(c.f[2]), __float_as_uint(c.f[3]));
}

// Stores a quantised head vector (format and rounding: append.cu).  Its kLanes lanes hold chunks c0
// and c1 (bf16 bits) each.
template <int kLanes>
__device__ __forceinline__ void store_fp8(const RopeParams& p, int64_t page, int slot, int g, int which, int c0, int c1,
                                          uint4 b0, uint4 b1, bool leader) {
  const KvGeom& ge = p.geom;
  const uint32_t w[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
  const uint32_t lanes = kLanes == 32 ? 0xffffffffu : ((1u << kLanes) - 1) << (threadIdx.x & 31 & ~(kLanes - 1));
#pragma unroll
  for (int sh = kLanes / 2; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor_sync(lanes, top, sh, kLanes));
  const int ef = (__float_as_int(top) >> 23) & 0xff;
  int X = ef == 0 ? -127 : ef - 127 - 8;
  X = max(-127, min(127, X));
  const float inv = __int_as_float((127 - X) << 23);   // 2^-X, exact
  uint32_t code[4] = {0, 0, 0, 0};                     // chunk c0: 0, 1; chunk c1: 2, 3
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = make_float2(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
    code[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3) << (16 * (i & 1));
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int c = half ? c1 : c0;
    const uint2 v = make_uint2(code[2 * half], code[2 * half + 1]);
    if (which == 0) {
      *reinterpret_cast<uint2*>(p.pool + kv_chunk_offset(ge, page, g, 0, slot, c >> 1) + (c & 1) * 8) = v;
    } else {   // transposed: this token's byte of each channel row
      unsigned char* to = reinterpret_cast<unsigned char*>(p.pool) + kv_fp8_v_offset(ge, page, g, c * 8, slot);
#pragma unroll
      for (int i = 0; i < 8; ++i) to[i * kPage] = (unsigned char)((i < 4 ? v.x >> (8 * i) : v.y >> (8 * (i - 4))) & 0xffu);
    }
  }
  if (leader) *reinterpret_cast<unsigned char*>(p.pool + kv_exp_offset(ge, page, g, which, slot)) = (unsigned char)(X + 127);
}

// kTokens tokens of a sequence per block.  kFp8: what is stored is quantised
template <typename T, int D, int kTokens, bool kFp8>
__global__ void __launch_bounds__(kThreads, 4) rope_qkv_kernel(const __grid_constant__ RopeParams p) {
  constexpr int E = Chunk<T>::N;             // channels per chunk
  constexpr int kLanes = D / E / 2;          // threads per head vector, two chunks each
  constexpr int kGroups = kThreads / (kLanes * kTokens);   // heads in flight per token
  static_assert(kGroups >= 1, "threads");
  __shared__ float2 turn[kTokens][kMaxRotary / 2];   // (cos, sin) times the scale
  const RopeEntry& en = p.e[blockIdx.y];
  const KvGeom& ge = p.geom;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (a no-op after an ordinary launch)
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.pool != nullptr && en.tbl_idx >= 0) p.table[en.tbl_idx] = en.page_hint;
  const int tok0 = blockIdx.x * kTokens;
  if (tok0 >= en.n_new) return;
  const int n_tok = min(kTokens, en.n_new - tok0), pairs = p.rotary / 2;
  const int lane = threadIdx.x % kLanes, t = threadIdx.x / kLanes % kTokens, grp = threadIdx.x / (kLanes * kTokens);
  // this thread's two chunks: a pair of halves, or neighbours
  const int turned = p.rotary / E;           // chunks that turn (even: rotary is a multiple of 16)
  const bool rotates = lane < turned / 2, split = p.halves && rotates;
  const int c0 = split ? lane : 2 * lane, c1 = split ? lane + turned / 2 : 2 * lane + 1;
  const int64_t row = (int64_t)en.row0 + tok0 + t;
  const int nq = p.q != nullptr ? p.n_q_heads : 0, nk = p.k != nullptr ? ge.n_kv_heads : 0, nv = p.v != nullptr ? ge.n_kv_heads : 0;
  const int heads = t < n_tok ? nq + nk + nv : 0;
  auto source = [&](int h) {
    const char* src = h < nq ? p.q + row * p.q_stride : h < nq + nk ? p.k + row * p.k_stride : p.v + row * p.v_stride;
    return src + (int64_t)(h < nq ? h : h < nq + nk ? h - nq : h - nq - nk) * ge.row_bytes;
  };
  // A row is asked for one head before it is needed, the first one before the sines are formed; more rows under way
  // take registers, and with them blocks, away (8192 rows: none ahead 54 us, one 40, two 46 with two or three blocks per SM).
  uint4 ahead[2];
  auto fetch = [&](int h) {
    if (h >= heads) return;
    const char* src = source(h);
    ahead[0] = __ldcs(reinterpret_cast<const uint4*>(src + c0 * 16));   // (read once)
    ahead[1] = __ldcs(reinterpret_cast<const uint4*>(src + c1 * 16));
  };
  fetch(grp);
  for (int i = threadIdx.x; i < n_tok * pairs; i += kThreads) {
    const int x = i / pairs, pr = i - x * pairs;
    const double at = en.pos0 + tok0 + x, f = p.freq[pr], far = at * f, turns = rint(far * 0.15915494309189533577);
    // at f = far + what its rounding lost; 2 pi in two terms: the first difference is exact to 2^-51
    const double a = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, far)) + fma(at, f, -far);
    float sn, cs;
    sincosf((float)a, &sn, &cs);
    turn[x][pr] = make_float2(cs * p.scale, sn * p.scale);
  }
  __syncthreads();
  float cs[E], sn[E];
  if (rotates) {
#pragma unroll
    for (int i = 0; i < E; ++i) {            // halves: channels c0 E + i and c1 E + i; else (2 i, 2 i + 1) of the two chunks' 2 E
      const float2 w = turn[t][lane * E + i];
      cs[i] = w.x;
      sn[i] = w.y;
    }
  }
  int64_t page = 0;
  int slot = 0;
  bool keep = p.pool != nullptr && t < n_tok;
  if (keep) {
    // a ring only keeps the last `window` tokens of the call
    keep = !(p.is_ring && en.n_new > p.window && tok0 + t < en.n_new - p.window);
    const int pos = en.start_pos + tok0 + t;
    if (p.is_ring) {
      const int rs = pos % p.window;
      page = (int64_t)en.seq * p.ring_pages + rs / kPage;
      slot = rs % kPage;
    } else {
      page = en.page_hint >= 0 ? en.page_hint : p.table[(int64_t)en.seq * p.table_stride + pos / kPage];
      slot = pos % kPage;
    }
  }
  for (int h = grp; h < heads; h += kGroups) {   // (whole head vectors: the lanes that shuffle stay together)
    uint4 b0 = ahead[0], b1 = ahead[1];
    fetch(h + kGroups);
    const int which = h < nq ? 0 : h < nq + nk ? 1 : 2, hh = which == 0 ? h : which == 1 ? h - nq : h - nq - nk;
    if (rotates && which != 2) {
      Chunk<T> a, b;
      widen(a, b0);
      widen(b, b1);
      if (split) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float x = a.f[i], y = b.f[i];
          a.f[i] = x * cs[i] - y * sn[i];
          b.f[i] = x * sn[i] + y * cs[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          float& fx = i < E / 2 ? a.f[2 * i] : b.f[2 * i - E];
          float& fy = i < E / 2 ? a.f[2 * i + 1] : b.f[2 * i - E + 1];
          const float x = fx, y = fy;
          fx = x * cs[i] - y * sn[i];
          fy = x * sn[i] + y * cs[i];
        }
      }
      b0 = bits_of(a);
      b1 = bits_of(b);
    }
    char* out = which == 0 ? p.q_out : which == 1 ? p.k_out : p.v_out;
    if (out != nullptr) {
      out += (row * (which == 0 ? p.n_q_heads : ge.n_kv_heads) + hh) * ge.row_bytes;
      *reinterpret_cast<uint4*>(out + c0 * 16) = b0;
      *reinterpret_cast<uint4*>(out + c1 * 16) = b1;
    }
    if (which != 0 && keep) {
      if constexpr (kFp8) {
        store_fp8<kLanes>(p, page, slot, hh, which - 1, c0, c1, b0, b1, lane == 0);
        continue;
      }
      *reinterpret_cast<uint4*>(p.pool + kv_chunk_offset(ge, page, hh, which - 1, slot, c0)) = b0;
      *reinterpret_cast<uint4*>(p.pool + kv_chunk_offset(ge, page, hh, which - 1, slot, c1)) = b1;
    }
  }
}

template <typename T, int D, int kTokens, bool kFp8 = false>
cudaError_t launch(const RopeParams& p, int max_n_new, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((max_n_new + kTokens - 1) / kTokens, p.n_entries);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rope_qkv_kernel<T, D, kTokens, kFp8>, p);
}

}  // namespace

cudaError_t launch_rope_qkv(const RopeParams& p, int max_n_new, cudaStream_t st) {
  if (p.n_entries <= 0) return cudaSuccess;
  if (max_n_new < 1) max_n_new = 1;
  // a token or two per sequence: a block's threads share one token's heads
  const bool step = max_n_new <= 2, wide = p.geom.head_dim == 128;
  if (p.geom.fp8 && p.pool != nullptr)   // (head_dim 128)
    return step ? launch<__nv_bfloat16, 128, 1, true>(p, max_n_new, st) : launch<__nv_bfloat16, 128, 4, true>(p, max_n_new, st);
  if (p.geom.elem_bytes == 2) {
    if (step) return wide ? launch<__nv_bfloat16, 128, 1>(p, max_n_new, st) : launch<__nv_bfloat16, 64, 1>(p, max_n_new, st);
    return wide ? launch<__nv_bfloat16, 128, 4>(p, max_n_new, st) : launch<__nv_bfloat16, 64, 4>(p, max_n_new, st);
  }
  if (step) return wide ? launch<float, 128, 1>(p, max_n_new, st) : launch<float, 64, 1>(p, max_n_new, st);
  return wide ? launch<float, 128, 4>(p, max_n_new, st) : launch<float, 64, 4>(p, max_n_new, st);
}

}  // namespace mixattn
