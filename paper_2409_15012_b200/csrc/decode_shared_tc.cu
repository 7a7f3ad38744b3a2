// Decode over a tree of shared prefixes on the 5th-generation tensor cores (tcgen05 + TMEM), bf16 and quantised caches.
//
// The pieces of the tree, their items and segments are described with SharedDecodeParams
// (internal.h), the mathematics in decode_shared.cu.  Here the rows of an item, the query heads that
// read the same keys (up to 128: sequences x heads of a KV head), are the M dimension of the
// products, so that a page of the cache is read from HBM once for all of them; more rows are chunks of their own, which
// read the keys again, from L2 (their CTAs walk side by side).  What bounds a segment: a tile of 128 keys and head_dim 128
// is 64 KB, 2800 cycles of an SM's share of HBM, and costs each chunk 1536 cycles of products and about as many of
// exponentials.  So one chunk follows the stream, and with two the products come first (64 sequences of 4 heads behind
// 32k: tensor pipe 66 % busy, DRAM at 25 %).  The keys that only one sequence has do not come here: a row that stands
// alone would cost a tile of products like 128 (plan_own_keys, api.cu).
//
//   warps 0, 3 page producers for K and for V: ids from the block table, 2 KB tensor copies (16 tokens x
//              64 channels) into a ring of 128-key stages each.  A warp needs about 100 cycles per
//              copy: with one warp for both, its 32 copies per tile were the limit (3200 cycles)
//   warp 1     issues S = Q K^T into one of two S buffers, a stream's half at a time
//   warp 2     P V of both streams, P in two bf16 terms (value and rounding residual: 16 bits, as
//              the other decode kernels hold them) from tensor memory
//   warps 4-7, 8-11  the softmax of stream 0 and 1, a row per thread
//   warps 12-15  rows of Q into shared memory for the next segment, then the results of this one
//
// Operands straight from the pages.  A page block holds 16 rows of K and 16 of V whose 16-byte
// chunks are stored permuted by (token & 7), inside 128 bytes the image of a 128-byte-swizzled operand; a
// copy of one 64-channel half of a page's K lays down 16 such rows, and eight pages one after the other
// are the [128 keys x 64 channels] block that a matrix descriptor names.  Stream h takes the keys of pages 4 h .. 4 h + 3 of
// every tile: two independent flash-attention passes with their own reference, sum and accumulator, merged at
// the end.  K and V have rings of their own because a tile's K is done with when its scores are, a softmax and a
// product earlier than its V: with both in one ring of three stages, the loads of the tile after next came
// too late (2400 cycles a tile where neither HBM nor products limit, with any number of products).
//
// Quantised caches (kFp8; format in internal.h).  A page block is one untiled copy of 4128 bytes into a ring of
// 64-key stages, and the warps of Q and of the results turn its codes into fp16 operands between those duties (one
// conversion per pair, exact; Q is taken to fp16 as in the other decode kernel): K rows as above, V, which is
// stored transposed, with its keys contiguous.  A K row's exponent multiplies its scores.  A V row's exponent X
// is added to its base-2 score: the weight 2^(s + X - n) is what multiplies the row's codes, and with
// n the row's reference for s + X, its fp16 rounding (2^-12 of it, or 2^-25 of the largest) is
// relative to what the keys contribute, however their magnitudes differ.  The sum of the softmax takes the
// weights times 2^-X in fp32, so reference, sum and accumulator are as ever.  X is taken as -60 at least: the sum's
// terms stay below 2^75, and a key whose values hardly count keeps its weight in the sum beside exponents of up to
// 14 (the weight is flushed 126 below the reference).  What a lower X, or a vector of zeros, lacks then is taken off its
// codes while they are converted (rare): values below 2^-51 in steps of 2^-84.  (V as bf16, the weight in two terms:
// 2500 cycles a tile for the conversion alone.)  K has one operand buffer (its scores come early), V
// two, so that a stage is free again as soon as it is converted.
//
// TMEM: S0, S1, O_0, O_1 = 4 x 128 columns.  All mbarrier waits are bounded; on time-out a status
// word is raised and every role leaves its loop.
#include <cuda_fp16.h>

#include <type_traits>

#include "f32x2.cuh"
#include "internal.h"
#include "score_shape.cuh"
#include "tc_ops.cuh"

namespace mixattn {

namespace {

constexpr int kThreads = 512;
constexpr int kRows = 128, kTile = 128;          // rows of an item, keys per tile
constexpr int kTilePages = kTile / kPage;
constexpr int kPiece = 2048;                     // 64 channels of one page's K or V
constexpr int kHalf = kTilePages * kPiece;       // 64 channels of a tile's K or V
constexpr int kQHalf = kRows * 128;              // 64 channels of Q
constexpr uint32_t kColS = 0, kColO = 256;

enum {
  B_QF = 0, B_QE = 1,        // Q there / consumed by the segment's score products
  B_SF = 2, B_SR = 6,        // + 2 stream + buffer: the stream's half of an S buffer: scores there / P in it consumed
  B_PF = 10,                 // + 2 stream + buffer: P written
  B_OF = 14,                 // per stream: the segment's last P V done
  B_XC = 16, B_OR = 17,      // references and sums published / results read
  B_KF = 18                  // K stages full, then free, V stages full, then free
};

template <int D, bool kFp8>
struct Layout {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kHalf;              // K or V of a tile as operand
  // native: rings of operand tiles for K and V.  Quantised: a ring of raw stages (64 keys, K and V), one
  // operand buffer for K and two for V; what a tile's exponents come to, four tiles deep
  static constexpr int kStages = kFp8 ? 5 : D == 128 ? 3 : 6;
  static constexpr int kKBufs = kFp8 ? 1 : kStages, kVBufs = kFp8 ? 2 : kStages;
  static constexpr int kRawBlk = 2 * kPage * D + 2 * kPage, kRawStage = 4 * kRawBlk;
  static constexpr int kKE = B_KF + kKBufs, kVF = kKE + kKBufs, kVE = kVF + kVBufs, kRF = kVE + kVBufs;
  static constexpr int kRE = kRF + (kFp8 ? kStages : 0), kXF = kRE + (kFp8 ? kStages : 0), kBars = kXF + (kFp8 ? 4 : 0);
  static constexpr int kSmQ = 0;
  static constexpr int kSmK = kHalves * kQHalf;
  static constexpr int kSmV = kSmK + kKBufs * kTileBytes;
  static constexpr int kSmRaw = kSmV + kVBufs * kTileBytes;
  static constexpr int kSmX = kSmRaw + (kFp8 ? kStages * kRawStage : 0);
  static constexpr int kSmBar = kSmX + (kFp8 ? 4 * 3 * kTile * 4 : 0);
  static constexpr int kSmXchg = kSmBar + (kBars * 8 + 16 + 255) / 256 * 256;
  static constexpr int kBytes = kSmXchg + 2 * kRows * 8 + 768;   // + slack to align a 256-byte aligned base to 1024
  static_assert(kBytes <= 227 * 1024, "shared memory");
  static_assert(!kFp8 || D == 128, "quantised caches have 128 channels");
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// four E4M3 codes -> fp16 pairs (bytes 0, 1 and bytes 2, 3), exact
__device__ __forceinline__ void codes_to_f16(uint32_t x, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(x));
}
// Lowest exponent of a V row that its weight and the row's sum take in (see the top): byte of 2^-60.
constexpr uint32_t kLowByte = 127 - 60;
// two fp16 elements times what the exponents in the two low bytes of e have below that, 2^(byte - kLowByte) (0 for byte 0)
__device__ __forceinline__ uint32_t times_rest(uint32_t x, uint32_t e) {
  const float a = __int_as_float((127 + min((int)(e & 0xffu) - (int)kLowByte, 0)) << 23);
  const float b = __int_as_float((127 + min((int)(e >> 8 & 0xffu) - (int)kLowByte, 0)) << 23);
  const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&x), __floats2half2_rn(a, b));
  return *reinterpret_cast<const uint32_t*>(&y);
}
// One channel of a tile's V, converted already, times what its keys' exponents have below 2^-60.  Rare, and out of line: the
// conversion is inlined in three places (tree of two levels, quantised: 39.9 us without this, 39.1 so, 40.4 inlined, 48.5
// with a test per page in the conversion's loop).
template <int D, int kRawBlk>
__device__ __noinline__ void take_rest(unsigned char* v, const unsigned char* raw0, const unsigned char* raw1, int n, int keys) {
#pragma unroll 1
  for (int x = 0; 16 * x < keys; ++x) {
    const uint4 e = *reinterpret_cast<const uint4*>((x < 4 ? raw0 : raw1) + (x & 3) * kRawBlk + 2 * kPage * D + kPage);
    unsigned char* row = v + (x >> 2) * (128 * 128) + n * 128;
    uint4* lo = reinterpret_cast<uint4*>(row + (((2 * x & 7) ^ (n & 7)) << 4));
    uint4* hi = reinterpret_cast<uint4*>(row + (((2 * x & 7) + 1 ^ (n & 7)) << 4));
    *lo = make_uint4(times_rest(lo->x, e.x), times_rest(lo->y, e.x >> 16), times_rest(lo->z, e.y), times_rest(lo->w, e.y >> 16));
    *hi = make_uint4(times_rest(hi->x, e.z), times_rest(hi->y, e.z >> 16), times_rest(hi->z, e.w), times_rest(hi->w, e.w >> 16));
  }
}
__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t x) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(__uint_as_float(x & 0xffff0000u)), "f"(__uint_as_float(x << 16)));
  return d;
}

// kShape: scores capped (1), biased (2), both (3)
template <int D, int kShape, bool kFp8>
__global__ void __launch_bounds__(kThreads, 1)
decode_shared_tc_kernel(const __grid_constant__ CUtensorMap pages, const __grid_constant__ SharedDecodeParams p) {
  using L = Layout<D, kFp8>;
  constexpr int kStages = L::kStages;
  // A score this far (base 2) above its row's reference moves it; 64 weights that do not lead that far
  // add up to no more than kMaxSum (fp16 weights have to stay below 65504 themselves).
  constexpr float kMaxLead = kFp8 ? 9.f : 32.f, kMaxSum = kFp8 ? 0x1p15f : 0x1p38f;
  // A segment's j-th tile (of n) and its first key.  With a distance bias, which lifts the scores towards the query,
  // the newest tile comes first: from the oldest on, a steep head would move its reference at every tile
  // (32 sequences of 64k, quantised cache: 124 -> 105 us).
  auto tiles_of = [](const ShareSegment& q) { return (q.t1 - q.t0 + kTile - 1) / kTile; };
  auto tile_key = [](const ShareSegment& q, int j, int n) { return q.t0 + ((kShape & 2) ? n - 1 - j : j) * kTile; };
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = base + L::kSmBar;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gbase + L::kSmBar + L::kBars * 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gbase + L::kSmBar + L::kBars * 8 + 8);
#define BAR(i) (bar0 + 8u * (i))
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(BAR(B_QF), 4);
    mbar_init(BAR(B_QE), 1);
    for (int s = 0; s < L::kKBufs; ++s) {
      mbar_init(BAR(B_KF + s), kFp8 ? 4 : 1);   // by the four converting warps
      mbar_init(BAR(L::kKE + s), 1);
    }
    for (int s = 0; s < L::kVBufs; ++s) {
      mbar_init(BAR(L::kVF + s), kFp8 ? 4 : 1);
      mbar_init(BAR(L::kVE + s), 1);
    }
    if constexpr (kFp8) {
      for (int s = 0; s < kStages; ++s) {
        mbar_init(BAR(L::kRF + s), 1);
        mbar_init(BAR(L::kRE + s), 4);
      }
      for (int s = 0; s < 4; ++s) mbar_init(BAR(L::kXF + s), 4);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(BAR(B_SF + s), 1);
      mbar_init(BAR(B_SR + s), 1);
      mbar_init(BAR(B_PF + s), 4);
    }
    mbar_init(BAR(B_OF + 0), 1);
    mbar_init(BAR(B_OF + 1), 1);
    mbar_init(BAR(B_XC), 8);
    mbar_init(BAR(B_OR), 4);
    abort_flag[0] = 0;   // any role gave up
    abort_flag[1] = 0;   // never set: the producer's last wait runs to its own limit
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // Every role walks the same segments with the same counters: G tiles, it segments so far.
  ShareWalk walk = share_begin(p, blockIdx.x);
  // The kernels ahead in the stream are done; only then may the next one start: the split pass of the
  // sequences' own keys does not wait for this kernel before it begins.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  ShareSegment s;
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (kFp8 && warp == 0) {
      // ------------------------------ page producer, quantised ------------------------------
      bool ok = true;
      int H = 0;   // stages of four pages so far
      while (ok && share_next(p, blockIdx.x, walk, s)) {
        const int32_t* tbl = p.table + (int64_t)p.node[s.node].slot * p.table_stride;
        const int page_hi = (s.t1 + kPage - 1) / kPage, n_tiles = tiles_of(s);
        // a tile's ids are fetched while the one before is on its way
        auto ids_of = [&](int j) {
          const int pg = tile_key(s, j, n_tiles) / kPage + (lane & (kTilePages - 1));
          return j < n_tiles && pg < page_hi ? tbl[pg] : 0;
        };
        int ids = ids_of(0);
        for (int j = 0; ok && j < n_tiles; ++j) {
          const int ids_next = ids_of(j + 1), pages_here = min(kTilePages, page_hi - tile_key(s, j, n_tiles) / kPage);
          for (int pg = 0; pg < pages_here; pg += 4, ++H) {
          const int st = H % kStages, turn = H / kStages, n_pg = min(4, pages_here - pg);
          const int id = __shfl_sync(0xffffffffu, ids, pg + (lane & 3));
          if (turn > 0) {
            int w = 1;
            if (lane == 0) w = mbar_wait(BAR(L::kRE + st), (turn - 1) & 1, abort_flag);
            if (!__shfl_sync(0xffffffffu, w, 0)) { ok = false; break; }
          }
          if (lane == 0) mbar_expect_tx(BAR(L::kRF + st), n_pg * L::kRawBlk);
          __syncwarp();
          if (lane < n_pg)
            bulk_load(base + L::kSmRaw + st * L::kRawStage + lane * L::kRawBlk,
                      p.pool + (int64_t)id * p.geom.page_bytes + (int64_t)s.g * L::kRawBlk, L::kRawBlk, BAR(L::kRF + st));
          }
          ids = ids_next;
        }
      }
      if (!ok && lane == 0) {
        atomicExch(p.status, kDevWaitTimeout);
        for (int back = 1; back <= kStages && H - back >= 0; ++back)
          mbar_wait(BAR(L::kRF + (H - back) % kStages), ((H - back) / kStages) & 1, abort_flag + 1);
      }
    } else if (!kFp8 && (warp == 0 || warp == 3)) {
      // ------------------------------ page producers ------------------------------
      const int v = warp == 3;   // K or V
      const int full = v ? L::kVF : B_KF, free = v ? L::kVE : L::kKE;
      const uint32_t ring = base + (v ? L::kSmV : L::kSmK);
      bool ok = true;
      int G = 0;
      if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&pages) : "memory");
      while (ok && share_next(p, blockIdx.x, walk, s)) {
        const int32_t* tbl = p.table + (int64_t)p.node[s.node].slot * p.table_stride;
        const int page_hi = (s.t1 + kPage - 1) / kPage, n_tiles = tiles_of(s), j = lane & (kTilePages - 1), h = lane / kTilePages;
        // a tile's ids are fetched while the one before is on its way
        auto id_of = [&](int x) {
          const int pg = tile_key(s, x, n_tiles) / kPage + j;
          return x < n_tiles && pg < page_hi ? tbl[pg] : 0;
        };
        int id_next = id_of(0);
        for (int x = 0; x < n_tiles; ++x, ++G) {
          const int id = id_next;
          id_next = id_of(x + 1);
          const int st = G % kStages, turn = G / kStages, n_pg = min(kTilePages, page_hi - tile_key(s, x, n_tiles) / kPage);
          if (turn > 0) {   // lane 0 waits; the verdict is made warp-uniform
            int w = 1;
            if (lane == 0) w = mbar_wait(BAR(free + st), (turn - 1) & 1, abort_flag);
            if (!__shfl_sync(0xffffffffu, w, 0)) { ok = false; break; }
          }
          if (lane == 0) mbar_expect_tx(BAR(full + st), n_pg * L::kHalves * kPiece);
          __syncwarp();
          if (h < L::kHalves && j < n_pg)
            tma_load_4d(ring + st * L::kTileBytes + h * kHalf + j * kPiece, &pages, 64 * h, 0, v,
                        id * p.geom.n_kv_heads + s.g, BAR(full + st));
        }
      }
      if (!ok && lane == 0) {   // leave only after the copies already issued have landed (bounded)
        atomicExch(p.status, kDevWaitTimeout);
        for (int back = 1; back <= kStages && G - back >= 0; ++back)
          mbar_wait(BAR(full + (G - back) % kStages), ((G - back) / kStages) & 1, abort_flag + 1);
      }
    } else if (warp == 1) {
      // ------------------------------ score products ------------------------------
      constexpr uint32_t kIdesc = kFp8 ? idesc_f16(0, 64) : idesc_bf16(0, 64);
      const uint64_t qdesc = smem_desc(base + L::kSmQ, 16, 1024);
      bool ok = true;
      int G = 0;
      for (int it = 0; ok && share_next(p, blockIdx.x, walk, s); ++it) {
        ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_QF), it & 1, abort_flag));
        const int n_tiles = tiles_of(s);
        for (int j = 0; j < n_tiles && ok; ++j, ++G) {
          const int sb = G & 1, st = G % L::kKBufs;
          ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_KF + st), (G / L::kKBufs) & 1, abort_flag));
#pragma unroll
          for (int g = 0; g < 2; ++g) {   // a stream's half waits for its own P V alone
            if (ok && G >= 2) ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_SR + 2 * g + sb), ((G >> 1) - 1) & 1, abort_flag));
            if (!ok) break;
            tc_fence_after();
            const uint64_t kdesc = smem_desc(base + L::kSmK + st * L::kTileBytes + g * 64 * 128, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              umma_bf16_warp(tmem + kColS + sb * 128 + g * 64, qdesc + (uint64_t)((ks >> 2) * (kQHalf >> 4) + (ks & 3) * 2),
                             kdesc + (uint64_t)((ks >> 2) * (kHalf >> 4) + (ks & 3) * 2), kIdesc, ks > 0);
            umma_commit_warp(BAR(B_SF + 2 * g + sb));
          }
          if (!ok) break;
          umma_commit_warp(BAR(L::kKE + st));
        }
        if (ok) umma_commit_warp(BAR(B_QE));
      }
      if (!ok && lane == 0) atomicExch(p.status, kDevWaitTimeout);
    } else if (warp == 2) {
      // ------------------------------ P V ------------------------------
      constexpr uint32_t kIdesc = kFp8 ? idesc_f16(0, D) : idesc_bf16(1, D);   // V with its keys contiguous, or its channels
      constexpr int kTerms = kFp8 ? 4 : 8;                        // four steps of the weights, four of their residuals
      constexpr int kGStep = kFp8 ? 128 * 128 : 64 * 128;         // a stream's keys behind the other's
      constexpr int kStep = kFp8 ? 32 : kPiece;                   // 16 keys
      bool ok = true;
      int G = 0;
      for (int it = 0; ok && share_next(p, blockIdx.x, walk, s); ++it) {
        // the segment's first P V overwrites the accumulators
        if (it >= 1) ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_OR), (it - 1) & 1, abort_flag));
        const int n_tiles = tiles_of(s);
        for (int j = 0; j < n_tiles && ok; ++j, ++G) {
          const int sb = G & 1, st = G % L::kVBufs;
          ok = __all_sync(0xffffffffu, mbar_wait(BAR(L::kVF + st), (G / L::kVBufs) & 1, abort_flag));
          if (!ok) break;
          // A stream's steps of 16 keys are pages; the segment's last tile may hold fewer (one at least is taken: the
          // accumulator is read), and rows that are no keys (behind the last one, or of a page that was not
          // loaded), whose weight of zero an infinity or a NaN would survive, are cleared meanwhile.
          const int left = s.t1 - tile_key(s, j, n_tiles);
          if (!kFp8 && left < kTile) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const int steps = min(max((left - 64 * g + 15) >> 4, 1), 4), first = min(max(left - 64 * g, 0), 16 * steps);
              unsigned char* v = gbase + L::kSmV + st * L::kTileBytes + g * 64 * 128;
              for (int x = lane; x < (16 * steps - first) * (D / 8); x += 32) {   // 16-byte chunks
                const int row = first + x / (D / 8), c = x % (D / 8);
                *reinterpret_cast<uint4*>(v + (c >> 3) * kHalf + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the products read through the async proxy
            __syncwarp();
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait(BAR(B_PF + 2 * g + sb), (G >> 1) & 1, abort_flag));
            if (!ok) break;
            tc_fence_after();
            const uint64_t vdesc = smem_desc(base + L::kSmV + st * L::kTileBytes + g * kGStep, kFp8 ? 16 : kHalf, 1024);
            const uint32_t o = tmem + kColO + g * 128, pcol = tmem + kColS + sb * 128 + g * 64;
            if (left - 64 * g >= 64) {
              umma_bf16_ts_warp(o, pcol, vdesc, kIdesc, j > 0);
#pragma unroll
              for (int x = 1; x < kTerms; ++x)
                umma_bf16_ts_warp(o, pcol + 8 * x, vdesc + (uint64_t)((x & 3) * (kStep >> 4)), kIdesc, 1u);
            } else {
              const int steps = max((left - 64 * g + 15) >> 4, 1);
#pragma unroll 1
              for (int x = 0; x < kTerms; ++x)
                if ((x & 3) < steps)
                  umma_bf16_ts_warp(o, pcol + 8 * x, vdesc + (uint64_t)((x & 3) * (kStep >> 4)), kIdesc, j > 0 || x > 0);
            }
            if (j == n_tiles - 1) umma_commit_warp(BAR(B_OF + g));
            umma_commit_warp(BAR(B_SR + 2 * g + sb));
            if (g == 1) umma_commit_warp(BAR(L::kVE + st));
          }
        }
      }
      if (!ok && lane == 0) atomicExch(p.status, kDevWaitTimeout);
    }
  } else if (warp >= 12) {
    // ------------------------------ Q in, results out ------------------------------
    const int qd = warp & 3, r = qd * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(qd * 32) << 16);
    const float2* xchg = reinterpret_cast<const float2*>(gbase + L::kSmXchg);
    auto put_q = [&](const ShareSegment& q, int it) {   // this thread's row of Q, rows behind the last as zeros
      uint4 x[D / 8];
#pragma unroll
      for (int c = 0; c < D / 8; ++c) x[c] = make_uint4(0u, 0u, 0u, 0u);
      if (r < q.rows) {
        const int R = q.row_first + r;
        const uint4* src = reinterpret_cast<const uint4*>(
            reinterpret_cast<const __nv_bfloat16*>(p.q) +
            ((int64_t)p.order[q.s0 + R / p.group] * p.n_q_heads + q.g * p.group + R % p.group) * D);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) x[c] = src[c];
      }
      if constexpr (kFp8) {   // the score products run on fp16
#pragma unroll
        for (int c = 0; c < D / 8; ++c)
          x[c] = make_uint4(bf16x2_to_f16x2(x[c].x), bf16x2_to_f16x2(x[c].y), bf16x2_to_f16x2(x[c].z), bf16x2_to_f16x2(x[c].w));
      }
      if (it >= 1 && !__all_sync(0xffffffffu, mbar_wait(BAR(B_QE), (it - 1) & 1, abort_flag))) return false;
      unsigned char* to = gbase + L::kSmQ + r * 128;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4*>(to + (c >> 3) * kQHalf + (((c & 7) ^ (r & 7)) << 4)) = x[c];
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_QF));
      return true;
    };
    // Quantised: a tile's codes into operands; every thread of the four warps takes 8 chunks of 16 codes of K and of V.
    auto convert = [&](const ShareSegment& q, int t, int G, int H) {
      const int n = threadIdx.x - 12 * 32, left = q.t1 - t, stages = left > 64 ? 2 : 1;
      const unsigned char* raw[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        raw[x] = gbase + L::kSmRaw + (H + x) % kStages * L::kRawStage;
        if (x < stages && !__all_sync(0xffffffffu, mbar_wait(BAR(L::kRF + (H + x) % kStages), ((H + x) / kStages) & 1, abort_flag))) return false;
      }
      if (G >= 1 && !__all_sync(0xffffffffu, mbar_wait(BAR(L::kKE), (G - 1) & 1, abort_flag))) return false;
      // (All of a thread's loads come before its stores, which the compiler could not pass: taken one by one, each
      // chunk waited for its own load, 2800 cycles a tile for K and V together.)
      uint4 w[8];
      // K: chunk c of key's row is 16 channels
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int key = x * 16 + (n >> 3), c = n & 7, tok = key & 15;
        w[x] = make_uint4(0u, 0u, 0u, 0u);
        if (key < left)   // (the others are masked later)
          w[x] = *reinterpret_cast<const uint4*>(raw[x >> 2] + (x & 3) * L::kRawBlk + tok * D + ((c ^ fp8_k_swizzle(tok)) << 4));
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int key = x * 16 + (n >> 3), c = n & 7, at = (c & 3) * 2;
        uint4 lo, hi;
        codes_to_f16(w[x].x, lo.x, lo.y);
        codes_to_f16(w[x].y, lo.z, lo.w);
        codes_to_f16(w[x].z, hi.x, hi.y);
        codes_to_f16(w[x].w, hi.z, hi.w);
        unsigned char* to = gbase + L::kSmK + (c >> 2) * kHalf + key * 128;
        *reinterpret_cast<uint4*>(to + ((at ^ (key & 7)) << 4)) = lo;
        *reinterpret_cast<uint4*>(to + (((at + 1) ^ (key & 7)) << 4)) = hi;
      }
      {   // the exponents: factor of the scores, summand of the weight's, factor of the sum's
        float* f = reinterpret_cast<float*>(gbase + L::kSmX) + (G & 3) * 3 * kTile;
        const float fold = kShape == 0 ? p.scale_log2e : kShape == 2 ? p.shape.pre : 1.f;
        const unsigned char* xs = raw[n >> 6] + ((n >> 4) & 3) * L::kRawBlk + 2 * kPage * D + (n & 15);
        float fk = 0.f, xv = 0.f, gv = 0.f;   // (keys that are not there are masked)
        if (n < left) {
          fk = __int_as_float((int)xs[0] << 23) * fold;           // 2^(byte - 127); byte 0 reads as zeros
          const int e = max((int)xs[kPage], (int)kLowByte) - 127;      // (what is missing below is in the codes)
          xv = (float)e;
          gv = __int_as_float((127 - e) << 23);
        }
        f[n] = fk;
        f[kTile + n] = xv;
        f[2 * kTile + n] = gv;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(BAR(B_KF));
        mbar_arrive(BAR(L::kXF + (G & 3)));
      }
      // some V exponent of the tile below kLowByte (looked at four keys per lane)
      bool low = false;
      if (4 * lane < left) {
        const uint32_t x4 = *reinterpret_cast<const uint32_t*>(raw[lane >> 4] + ((lane >> 2) & 3) * L::kRawBlk + 2 * kPage * D + kPage + 4 * (lane & 3));
        low = ((x4 - 0x01010101u * kLowByte) & ~x4 & 0x80808080u) != 0u;
      }
      low = __any_sync(0xffffffffu, low);
      if (G >= 2 && !__all_sync(0xffffffffu, mbar_wait(BAR(L::kVE + (G & 1)), ((G >> 1) - 1) & 1, abort_flag))) return false;
      // V: a channel's 16 keys of a page; rows are channels, 64 keys of a stream each
      if (left >= kTile) {
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x] = *reinterpret_cast<const uint4*>(raw[x >> 2] + (x & 3) * L::kRawBlk + kPage * D + n * kPage);
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int there = left - 16 * x;   // keys of this page; what lies behind the last key may be any code, a NaN too
          auto keep = [&](uint32_t v, int first) {
            const int m = there - first;
            return m >= 4 ? v : m <= 0 ? 0u : v & ((1u << (8 * m)) - 1u);
          };
          w[x] = make_uint4(0u, 0u, 0u, 0u);
          if (there > 0) {
            w[x] = *reinterpret_cast<const uint4*>(raw[x >> 2] + (x & 3) * L::kRawBlk + kPage * D + n * kPage);
            w[x] = make_uint4(keep(w[x].x, 0), keep(w[x].y, 4), keep(w[x].z, 8), keep(w[x].w, 12));
          }
        }
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        uint4 lo, hi;
        codes_to_f16(w[x].x, lo.x, lo.y);
        codes_to_f16(w[x].y, lo.z, lo.w);
        codes_to_f16(w[x].z, hi.x, hi.y);
        codes_to_f16(w[x].w, hi.z, hi.w);
        unsigned char* to = gbase + L::kSmV + (G & 1) * L::kTileBytes + (x >> 2) * (128 * 128) + n * 128;
        const int at = (x & 3) * 2;
        *reinterpret_cast<uint4*>(to + ((at ^ (n & 7)) << 4)) = lo;
        *reinterpret_cast<uint4*>(to + (((at + 1) ^ (n & 7)) << 4)) = hi;
      }
      if (low) take_rest<D, L::kRawBlk>(gbase + L::kSmV + (G & 1) * L::kTileBytes, raw[0], raw[1], n, min(left, kTile));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(BAR(L::kVF + (G & 1)));
        for (int x = 0; x < stages; ++x) mbar_arrive(BAR(L::kRE + (H + x) % kStages));
      }
      return true;
    };
    int G = 0, H = 0;   // quantised: tiles and raw stages so far
    auto convert_tiles = [&](const ShareSegment& q, int from, int to) {
      bool fine = true;
      const int n_tiles = tiles_of(q);
      for (int j = from; fine && j < min(to, n_tiles); ++j, ++G) {
        const int t = tile_key(q, j, n_tiles);
        fine = convert(q, t, G, H);
        H += q.t1 - t > 64 ? 2 : 1;
      }
      return fine;
    };
    bool more = share_next(p, blockIdx.x, walk, s), ok = true;
    if (more) ok = put_q(s, 0);
    if (kFp8 && more && ok) ok = convert_tiles(s, 0, 1);
    for (int it = 0; ok && more; ++it) {
      const ShareSegment now = s;
      if (kFp8 && !convert_tiles(now, 1, INT32_MAX)) { ok = false; break; }
      more = share_next(p, blockIdx.x, walk, s);
      // (the next segment's first tile before this one's results: its scores can start under them)
      if (more) ok = put_q(s, it + 1) && (!kFp8 || convert_tiles(s, 0, 1));
      if (!ok) break;
      ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_XC), it & 1, abort_flag));
      if (!ok) break;
      const float2 lo = xchg[r], hi = xchg[kRows + r];
      ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_OF + 0), it & 1, abort_flag) && mbar_wait(BAR(B_OF + 1), it & 1, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const float m = fmaxf(lo.x, hi.x);   // (finite: stream 0 has the segment's first key)
      const float e_lo = ex2_approx(lo.x - m), e_hi = ex2_approx(hi.x - m);
      float* to = p.part_o + (int64_t)now.seg_row * D + r * 4;
      const bool mine = r < now.rows;
      if (qd * 32 < now.rows) {            // (warps without a row have nothing to read)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t a[32], b[32];
          tmem_ld32(lane_base + kColO + c * 32, a);
          tmem_ld32(lane_base + kColO + 128 + c * 32, b);
          tmem_wait_ld_pin(a, b);
          if (mine) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float4 o;
              // (a stream without a key has a weight of zero and an accumulator of zeros)
              o.x = __uint_as_float(a[e]) * e_lo + __uint_as_float(b[e]) * e_hi;
              o.y = __uint_as_float(a[e + 1]) * e_lo + __uint_as_float(b[e + 1]) * e_hi;
              o.z = __uint_as_float(a[e + 2]) * e_lo + __uint_as_float(b[e + 2]) * e_hi;
              o.w = __uint_as_float(a[e + 3]) * e_lo + __uint_as_float(b[e + 3]) * e_hi;
              *reinterpret_cast<float4*>(to + (int64_t)(c * 8 + e / 4) * now.rows * 4) = o;
            }
          }
        }
        if (mine) p.part_ml[now.seg_row + r] = make_float2(m, lo.y * e_lo + hi.y * e_hi);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_OR));
    }
    if (!ok && lane == 0) atomicExch(p.status, kDevWaitTimeout);
  } else {
    // ------------------------------ softmax ------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    const int g = (warp - 4) >> 2, qd = warp & 3, r = qd * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(qd * 32) << 16);
    const uint32_t o_addr = lane_base + kColO + g * 128;
    float2* xchg = reinterpret_cast<float2*>(gbase + L::kSmXchg);
    bool ok = true;
    int G = 0;
    for (int it = 0; ok && share_next(p, blockIdx.x, walk, s); ++it) {
      const bool idle = qd * 32 >= s.rows;    // none of this warp's rows exists
      float m_ref = -INFINITY, l = 0.f;
      float slope = 0.f;
      int newest = 0;
      if constexpr (kShape & 2) {
        const int R = s.row_first + min(r, s.rows - 1);
        slope = p.shape.slope[s.g * p.group + R % p.group];
        newest = p.newest[s.s0 + R / p.group];
      }
      const int n_tiles = tiles_of(s);
      for (int j = 0; j < n_tiles; ++j, ++G) {
        const int t = tile_key(s, j, n_tiles);
        const int sb = G & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(BAR(B_SF + 2 * g + sb), (G >> 1) & 1, abort_flag))) { ok = false; break; }
        if (!idle) {
          tc_fence_after();
          const uint32_t s_addr = lane_base + kColS + sb * 128 + g * 64;
          uint32_t sv[64];
          auto& s0 = *reinterpret_cast<uint32_t(*)[32]>(&sv[0]);
          auto& s1 = *reinterpret_cast<uint32_t(*)[32]>(&sv[32]);
          tmem_ld32(s_addr, s0);
          tmem_ld32(s_addr + 32, s1);
          tmem_wait_ld_pin(s0, s1);
          const float* factor = reinterpret_cast<const float*>(gbase + L::kSmX) + (G & 3) * 3 * kTile + 64 * g;   // kFp8
          const float first = (kShape & 2) ? -slope * (float)(newest - t - 64 * g) : 0.f;   // bias of column 0
          auto scale_keys = [&]() {   // products of codes -> products, or (no cap) what the weights are taken of
#pragma unroll
            for (int e = 0; e < 64; e += 4) {
              const float4 f = *reinterpret_cast<const float4*>(factor + e);
              float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
              if constexpr (!(kShape & 1)) x = *reinterpret_cast<const float4*>(factor + kTile + e);
              if constexpr (kShape == 2) {
                x.x += fmaf(slope, (float)e, first);
                x.y += fmaf(slope, (float)(e + 1), first);
                x.z += fmaf(slope, (float)(e + 2), first);
                x.w += fmaf(slope, (float)(e + 3), first);
              }
              sv[e] = __float_as_uint(fmaf(__uint_as_float(sv[e]), f.x, x.x));
              sv[e + 1] = __float_as_uint(fmaf(__uint_as_float(sv[e + 1]), f.y, x.y));
              sv[e + 2] = __float_as_uint(fmaf(__uint_as_float(sv[e + 2]), f.z, x.z));
              sv[e + 3] = __float_as_uint(fmaf(__uint_as_float(sv[e + 3]), f.w, x.w));
            }
          };
          if constexpr (kFp8) {
            if (!__all_sync(0xffffffffu, mbar_wait(BAR(L::kXF + (G & 3)), (G >> 2) & 1, abort_flag))) { ok = false; break; }
            scale_keys();
          }
          // Columns behind the last key hold products with whatever lies there (a page's old rows, an earlier tile).  Their
          // scores are masked below, but until then they must not have a say in which form of the cap all keys take.
          if constexpr ((kShape & 1) && !kFp8) {
            if (t + kTile > s.t1) {
              const int left = s.t1 - t - 64 * g;
#pragma unroll
              for (int e = 0; e < 64; ++e)
                if (e >= left) sv[e] = 0u;
            }
          }
          if constexpr (kShape != 0 && !(kFp8 && kShape == 2)) {   // raw products -> shaped base-2 scores
            float top = 0.f;   // largest square of a product
#pragma unroll
            for (int e = 0; e < 64; e += 2) {
              const f32x2 raw = pack2(__uint_as_float(sv[e]), __uint_as_float(sv[e + 1]));
              const f32x2 off = pack2(fmaf(slope, (float)e, first), fmaf(slope, (float)(e + 1), first));
              f32x2 x;
              if constexpr (kShape & 1) {   // a cubic in the product's square, good to half the cap (score_shape.cuh)
                const f32x2 u = mul2(raw, raw);
                f32x2 q = fma2(pack2(p.shape.near[3], p.shape.near[3]), u, pack2(p.shape.near[2], p.shape.near[2]));
                q = fma2(q, u, pack2(p.shape.near[1], p.shape.near[1]));
                q = fma2(q, u, pack2(p.shape.near[0], p.shape.near[0]));
                const float2 uu = unpack2(u);
                top = fmax3(top, uu.x, uu.y);
                x = (kShape & 2) ? fma2(q, raw, off) : mul2(q, raw);
              } else {
                x = fma2(raw, pack2(p.shape.pre, p.shape.pre), off);
              }
              const float2 y = unpack2(x);
              sv[e] = __float_as_uint(y.x);
              sv[e + 1] = __float_as_uint(y.y);
            }
            if constexpr (kShape & 1) {
              if (__any_sync(0xffffffffu, !(top <= p.shape.near_sq))) {   // beyond it: again from the raw products
                tmem_ld32(s_addr, s0);
                tmem_ld32(s_addr + 32, s1);
                tmem_wait_ld_pin(s0, s1);
                if constexpr (kFp8) scale_keys();
#pragma unroll
                for (int e = 0; e < 64; ++e) {
                  const float x = __uint_as_float(sv[e]) * p.shape.pre, o = (kShape & 2) ? fmaf(slope, (float)e, first) : 0.f;
                  const float a = tanh_poly(x), b = tanh_exp(x);
                  sv[e] = __float_as_uint(fmaf(fabsf(x) <= 1.f ? a : b, p.shape.post, o));
                }
              }
            }
          }
          if constexpr (kFp8 && (kShape & 1)) {
#pragma unroll
            for (int e = 0; e < 64; e += 2) {
              const float2 x = *reinterpret_cast<const float2*>(factor + kTile + e);
              sv[e] = __float_as_uint(__uint_as_float(sv[e]) + x.x);
              sv[e + 1] = __float_as_uint(__uint_as_float(sv[e + 1]) + x.y);
            }
          }
          const float scale = kShape || kFp8 ? 1.f : p.scale_log2e;
          if (t + kTile > s.t1) {
            const int left = s.t1 - t - 64 * g;
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (e >= left) sv[e] = 0xff800000u;
          }
          // A row's reference is the maximum of the first tile in which it has a key and only moves when a later score leads it
          // by more than 2^kMaxLead, which shows in the sum of the tile's weights: so the exponentials
          // wait for no maximum, and none is computed.
          auto tile_max = [&]() {
            float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
            for (int e = 0; e < 64; e += 4) {
              mx0 = fmax3(mx0, __uint_as_float(sv[e]), __uint_as_float(sv[e + 1]));
              mx1 = fmax3(mx1, __uint_as_float(sv[e + 2]), __uint_as_float(sv[e + 3]));
            }
            return fmaxf(mx0, mx1) * scale;
          };
          if (__any_sync(0xffffffffu, m_ref == -INFINITY)) {
            const float mt = tile_max();
            if (m_ref == -INFINITY) m_ref = mt;
          }
          float sum, part;   // of the weights, and what they add to the row's sum
          // P: values over the first 32 of the stream's columns, residuals over the others (the scores are
          // all in registers by now); in two halves, which keeps the registers within the launch's 128
          auto weights = [&]() {
            const float neg = m_ref == -INFINITY ? 0.f : -m_ref;   // (a stream without a key: weights 0, no NaN)
            f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0, part0 = sum0;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t pk[16], pl[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const int e = 32 * half + i;
                const float a = ex2_approx(fmaf(__uint_as_float(sv[e]), scale, neg));
                const float b = ex2_approx(fmaf(__uint_as_float(sv[e + 1]), scale, neg));
                if (i & 2) sum1 = add2(sum1, pack2(a, b));
                else sum0 = add2(sum0, pack2(a, b));
                if constexpr (kFp8) {
                  const float2 f = *reinterpret_cast<const float2*>(factor + 2 * kTile + e);
                  part0 = fma2(pack2(a, b), pack2(f.x, f.y), part0);
                  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(pk[i >> 1]) : "f"(b), "f"(a));
                } else {
                  split_bf16(a, b, pk[i >> 1], pl[i >> 1]);
                }
              }
              tmem_st16(s_addr + 16 * half, pk);
              if constexpr (!kFp8) tmem_st16(s_addr + 32 + 16 * half, pl);
            }
            float2 x = unpack2(add2(sum0, sum1));
            part = sum = x.x + x.y;
            if constexpr (kFp8) {
              x = unpack2(part0);
              part = x.x + x.y;
            }
          };
          weights();
          if (__any_sync(0xffffffffu, !(sum <= kMaxSum))) {
            // rare (an overflow gives infinity or NaN, which fail the comparison too): move the reference of
            // the leading rows and rescale what they have accumulated, once this stream's previous P V has landed
            const float mt = tile_max();
            const bool far = mt > m_ref + kMaxLead;
            const float alpha = far ? ex2_approx(m_ref - mt) : 1.f;
            if (j > 0) {
              if (!__all_sync(0xffffffffu, mbar_wait(BAR(B_SR + 2 * g + (sb ^ 1)), ((G - 1) >> 1) & 1, abort_flag))) { ok = false; break; }
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                uint32_t ov[32];
                tmem_ld32(o_addr + c * 32, ov);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
                tmem_st32(o_addr + c * 32, ov);
              }
            }
            l *= alpha;
            if (far) m_ref = mt;
            weights();
          }
          l += part;
          tmem_wait_st();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(B_PF + 2 * g + sb));
      }
      if (!ok) break;
      if (it >= 1) ok = __all_sync(0xffffffffu, mbar_wait(BAR(B_OR), (it - 1) & 1, abort_flag));   // the slot is free
      if (!ok) break;
      xchg[g * kRows + r] = make_float2(m_ref, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(B_XC));
    }
    if (!ok && lane == 0) atomicExch(p.status, kDevWaitTimeout);
  }
  // common exit: everyone is past its last TMEM access
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
#undef BAR
}

// Paged storage of one owner layer, native bf16 format, as [page and head][K | V][16 tokens][channels];
// box = 64 channels of 16 tokens of K or V.  The stored chunks are permuted already, so the copy does not swizzle.
bool make_page_map(CUtensorMap* map, const void* pool, const KvGeom& ge, int64_t pages) {
  EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[4] = {(cuuint64_t)ge.head_dim, (cuuint64_t)kPage, 2, (cuuint64_t)(pages * ge.n_kv_heads)};
  cuuint64_t strides[3] = {(cuuint64_t)ge.row_bytes, (cuuint64_t)kPage * ge.row_bytes, (cuuint64_t)ge.blk_bytes};
  cuuint32_t box[4] = {64, (cuuint32_t)kPage, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int kShape, bool kFp8>
cudaError_t launch(const SharedDecodeParams& p, const CUtensorMap& map, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Layout<D, kFp8>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, decode_shared_tc_kernel<D, kShape, kFp8>, map, p);
}
template <int D, bool kFp8>
cudaError_t launch_shape(const SharedDecodeParams& p, const CUtensorMap& map, cudaStream_t st) {
  const int shape = !p.shaped ? 0 : (p.shape.post > 0.f ? 1 : 0) | (p.shape.biased ? 2 : 0);
  if (shape == 0) return launch<D, 0, kFp8>(p, map, st);
  if (shape == 1) return launch<D, 1, kFp8>(p, map, st);
  return shape == 2 ? launch<D, 2, kFp8>(p, map, st) : launch<D, 3, kFp8>(p, map, st);
}

template <int D, bool kFp8>
cudaError_t prepare() {
  constexpr auto kAttr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  constexpr int kBytes = Layout<D, kFp8>::kBytes;
  cudaError_t e = cudaFuncSetAttribute(decode_shared_tc_kernel<D, 0, kFp8>, kAttr, kBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(decode_shared_tc_kernel<D, 1, kFp8>, kAttr, kBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(decode_shared_tc_kernel<D, 2, kFp8>, kAttr, kBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(decode_shared_tc_kernel<D, 3, kFp8>, kAttr, kBytes);
  return e;
}

}  // namespace

bool shared_tc_supported(const KvGeom& ge) { return ge.elem_bytes == 2 && (ge.fp8 || encode_fn() != nullptr); }

void shared_tc_tiles(SharedDecodeParams* p) {
  p->tile_keys = kTile;
  p->row_chunk = kRows;
  p->item_units = 1;
}

cudaError_t prepare_decode_shared_tc() {
  cudaError_t e = prepare<128, false>();
  if (e == cudaSuccess) e = prepare<64, false>();
  return e == cudaSuccess ? prepare<128, true>() : e;
}

cudaError_t launch_decode_shared_tc(const SharedDecodeParams& p, cudaStream_t st) {
  if (p.tile_keys != kTile || p.row_chunk != kRows) return cudaErrorInvalidValue;
  CUtensorMap map = {};
  if (p.geom.fp8) return p.geom.head_dim == 128 ? launch_shape<128, true>(p, map, st) : cudaErrorInvalidValue;
  if (!make_page_map(&map, p.pool, p.geom, p.n_pages)) return cudaErrorInvalidValue;
  return p.geom.head_dim == 128 ? launch_shape<128, false>(p, map, st) : launch_shape<64, false>(p, map, st);
}

}  // namespace mixattn
