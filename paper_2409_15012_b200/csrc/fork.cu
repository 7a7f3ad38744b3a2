// Forking of cached sequences and reading a cache back as plain tensors.
//
// Paper, Section 3: the caches a layer stack keeps are a paged pool per standard owner and a ring
// per sliding-window owner.  A copy of a sequence shares the pages no append writes to any more
// (host bookkeeping, cache_manager.hpp); what is left to move are the partly filled page of each
// paged pool, the rings and the sequence's row of the block table.  Both kernels are HBM-bound
// copies with 16-byte accesses.
#include "internal.h"

namespace mixattn {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 8;                            // 16-byte loads in flight per thread
constexpr int kReadVecs = 2;                          // (32 copies of 4103 tokens, 32 query / 8 KV heads of 128 bf16: 1: 172 us, 2: 161, 4: 162, 8: 197)
constexpr int kBlock16 = kThreads * kUnroll;          // 16-byte units per block: 32 KB

template <typename Params>
__global__ void __launch_bounds__(kThreads) fork_copy_kernel(const __grid_constant__ Params p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // a read that follows may get ready
  const int y = blockIdx.y;
  if (y < p.n_segs) {
    const CopySeg& s = p.seg[y];
    const uint32_t u0 = blockIdx.x * (uint32_t)kBlock16 + threadIdx.x;
    if (u0 - threadIdx.x >= s.n16) return;
    const int4* src = reinterpret_cast<const int4*>(p.arena + s.src);
    int4* dst = reinterpret_cast<int4*>(p.arena + s.dst);
    int4 v[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (u0 + i * kThreads < s.n16) v[i] = src[u0 + i * kThreads];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (u0 + i * kThreads < s.n16) dst[u0 + i * kThreads] = v[i];
    return;
  }
  if (blockIdx.x > 0) return;
  const TableRow& r = p.row[y - p.n_segs];
  const int32_t* src = p.table + (int64_t)r.src_slot * p.table_stride;
  int32_t* dst = p.table + (int64_t)r.dst_slot * p.table_stride;
  for (int b = r.copy0 + (int)threadIdx.x; b < r.copy0 + r.n_copy; b += kThreads) dst[b] = src[b];
  if ((int)threadIdx.x < r.n_set) dst[r.set0 + threadIdx.x] = r.page[threadIdx.x];
}

// The head vectors of the rows in the order they are written are dealt out to the blocks, kReadVecs
// per group of threads that copies one (a thread per 16 bytes): a block writes one contiguous
// stretch of K and one of V, with all its loads in flight at once.  (Reading a page that several
// copies share once for all of them, in one block, was slower, 195 us against 184 for the fork and
// the read back of the case below: the rows written bound it, not the pages read.)
__global__ void __launch_bounds__(kThreads, 8) read_kv_kernel(const __grid_constant__ GatherParams p) {
  // (launched while the kernel ahead in the stream still runs; nothing is read before that one is done)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const GatherEntry& e = p.e[blockIdx.y];
  const KvGeom& ge = p.geom;
  const int chunks = ge.row_bytes / 16;                // 8, 16 or 32
  const int chunk = (int)threadIdx.x % chunks, groups = kThreads / chunks;
  const int64_t vecs = (int64_t)e.n_prefix * ge.n_kv_heads;
  const int64_t v0 = (int64_t)blockIdx.x * groups * kReadVecs + (int)threadIdx.x / chunks;
  const int32_t* tbl = p.table + (int64_t)e.seq * p.table_stride;
  int4 a[kReadVecs], b[kReadVecs];
#pragma unroll
  for (int i = 0; i < kReadVecs; ++i) {
    const int64_t x = v0 + i * groups;
    if (x >= vecs) break;
    const int t = (int)(x / ge.n_kv_heads), g = (int)(x - (int64_t)t * ge.n_kv_heads), pos = e.pos0 + t;
    int64_t page;
    int slot;
    if (p.is_ring) {
      const int rs = pos % p.window;
      page = (int64_t)e.seq * p.ring_pages + rs / kPage;
      slot = rs % kPage;
    } else {
      page = tbl[pos / kPage];
      slot = pos % kPage;
    }
    const char* k = p.pool + kv_chunk_offset(ge, page, g, 0, slot, chunk);
    a[i] = *reinterpret_cast<const int4*>(k);
    b[i] = *reinterpret_cast<const int4*>(k + (int64_t)kPage * ge.st_row_bytes);
  }
#pragma unroll
  for (int i = 0; i < kReadVecs; ++i) {
    const int64_t x = v0 + i * groups;
    if (x >= vecs) break;
    const int64_t out = ((int64_t)e.dst_row0 * ge.n_kv_heads + x) * ge.row_bytes + chunk * 16;
    __stcs(reinterpret_cast<int4*>(static_cast<char*>(p.k_out) + out), a[i]);   // (not read again here: shared pages and rings are)
    __stcs(reinterpret_cast<int4*>(static_cast<char*>(p.v_out) + out), b[i]);
  }
}

}  // namespace

cudaError_t launch_fork_copy(const ForkParams& p, cudaStream_t st) {
  if (p.n_segs + p.n_rows <= 0) return cudaSuccess;
  uint32_t longest = 0;
  for (int i = 0; i < p.n_segs; ++i) longest = p.seg[i].n16 > longest ? p.seg[i].n16 : longest;
  unsigned bx = (longest + kBlock16 - 1) / kBlock16;
  if (bx < 1) bx = 1;
  const dim3 grid(bx, p.n_segs + p.n_rows);
  if (p.n_segs > SmallForkParams::kMaxSegs || p.n_rows > SmallForkParams::kMaxRows) {
    fork_copy_kernel<<<grid, kThreads, 0, st>>>(p);
    return cudaGetLastError();
  }
  SmallForkParams s;
  s.arena = p.arena;
  s.table = p.table;
  s.table_stride = p.table_stride;
  s.n_segs = p.n_segs;
  s.n_rows = p.n_rows;
  for (int i = 0; i < p.n_segs; ++i) s.seg[i] = p.seg[i];
  for (int i = 0; i < p.n_rows; ++i) s.row[i] = p.row[i];
  fork_copy_kernel<<<grid, kThreads, 0, st>>>(s);
  return cudaGetLastError();
}

cudaError_t launch_read_kv(const GatherParams& p, int max_rows, cudaStream_t st) {
  if (p.geom.fp8) return launch_gather(p, max_rows, st);   // dequantises
  if (p.n_entries <= 0 || max_rows <= 0) return cudaSuccess;
  const int64_t per_block = (int64_t)kThreads / (p.geom.row_bytes / 16) * kReadVecs;
  const int64_t blocks = ((int64_t)max_rows * p.geom.n_kv_heads + per_block - 1) / per_block;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, p.n_entries);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, read_kv_kernel, p);
}

}  // namespace mixattn
