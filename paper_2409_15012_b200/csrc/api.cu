// The C ABI (include/mixattn.h): argument validation, host bookkeeping, arena carving and
// kernel launches.  Everything that can fail is checked on the host before any launch.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <new>
#include <utility>
#include <vector>

#include "cache_manager.hpp"
#include "internal.h"
#include "share_plan.hpp"

using namespace mixattn;

namespace {

constexpr size_t kAlign = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSplitTokens = 4096;    // automatic split length of long caches (keys)
constexpr int kFewItems = 8;          // items per SM below which a shaped launch takes shorter splits
constexpr int kMinSplitTokens = 1024; // single-wave splitting never makes splits shorter than this
constexpr double kL2FitsShare = 0.55;  // a re-read ring up to this share of the L2 is cached whole
constexpr double kL2KeepShare = 0.45;  // of a larger one, this share of the L2 is kept

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct ArenaPlan {
  std::vector<size_t> owner_off;  // per owner slot
  std::vector<size_t> owner_bytes;
  size_t table_off = 0, table_bytes = 0;
  size_t status_off = 0, ticket_off = 0;
  size_t chunk_k_off = 0, chunk_v_off = 0;   // [chunk_scratch_tokens, Hkv, D] each
  // the split-KV workspace, at the end of the arena: partial results of split_bytes, and what a shared decode lacks beside them
  size_t part_o_off = 0, part_ml_off = 0, split_bytes = 0;
  size_t cache_bytes = 0, least = 0, total = 0;   // least: without the latter
};

// Shared decode on the tensor cores (bf16 and quantised caches) divides the workspace: the split pass of the own keys
// has kOwnChunks slots of a row per query head, the rest is for the tensor-core kernel: at most a segment of 128 rows
// per CTA, and where items end another.  With 32 query heads of 128 that is the workspace of the ordinary decode; fewer
// heads need up to 10.4 MB on top to use every SM (12 of 128: 6.7).
constexpr int kOwnExtraChunks = 384, kOwnChunks = kMaxCallSeqs + kOwnExtraChunks;
constexpr int kSharedCtas = 160;   // (148 SMs)
int64_t shared_rows(int n_q_heads) { return kSharedCtas * 128 + 2 * (int64_t)kMaxCallSeqs * n_q_heads; }

size_t rows_bytes(int64_t rows, int head_dim) {
  return align_up((size_t)rows * head_dim * sizeof(float)) + align_up((size_t)rows * sizeof(float2));
}

// Rows (at most shared_rows) that fit a workspace of `bytes` behind the own keys' slots.
int64_t shared_rows_that_fit(size_t bytes, int n_q_heads, int head_dim) {
  const size_t own = rows_bytes((int64_t)kOwnChunks * n_q_heads, head_dim);
  if (bytes <= own) return 0;
  int64_t rows = std::min<int64_t>((bytes - own) / (head_dim * sizeof(float) + sizeof(float2)), shared_rows(n_q_heads));
  while (rows > 0 && own + rows_bytes(rows, head_dim) > bytes) --rows;
  return rows;
}

int ring_pages_of(int window) { return (window + kPage - 1) / kPage; }

ArenaPlan plan_arena(const CacheManager& cm, const mixattn_config& cfg) {
  ArenaPlan pl;
  KvGeom ge = make_geom(cfg.n_kv_heads, cfg.head_dim, cfg.dtype, cfg.kv_format);
  size_t off = 0;
  for (int o : cm.owners()) {
    const LayerInfo& li = cm.layer(o);
    size_t bytes = li.kind == MIXATTN_FULL
                       ? (size_t)cfg.n_pages * ge.page_bytes
                       : (size_t)cfg.max_seqs * ring_pages_of(li.window) * ge.page_bytes;
    pl.owner_off.push_back(off);
    pl.owner_bytes.push_back(bytes);
    pl.cache_bytes += bytes;
    off += align_up(bytes);
  }
  pl.table_off = off;
  pl.table_bytes = (size_t)cm.max_seqs() * cm.max_blocks() * sizeof(int32_t);
  off += align_up(pl.table_bytes);
  pl.status_off = off;
  off += kAlign;
  pl.ticket_off = off;
  off += align_up(kBeamTickets * sizeof(int32_t));
  if (cfg.chunk_scratch_tokens > 0) {
    const size_t bytes = align_up((size_t)cfg.chunk_scratch_tokens * ge.n_kv_heads * ge.row_bytes);
    pl.chunk_k_off = off;
    off += bytes;
    pl.chunk_v_off = off;
    off += bytes;
  }
  const int64_t split_rows = (int64_t)kWsChunks * cfg.n_q_heads;
  pl.part_o_off = off;
  pl.part_ml_off = off + align_up((size_t)split_rows * cfg.head_dim * sizeof(float));
  pl.split_bytes = rows_bytes(split_rows, cfg.head_dim);
  pl.least = pl.total = off + pl.split_bytes;
  if (cm.n_full_owners() > 0 && cfg.dtype == MIXATTN_BF16)
    pl.total = std::max(pl.total, off + rows_bytes((int64_t)kOwnChunks * cfg.n_q_heads, cfg.head_dim) +
                                      rows_bytes(shared_rows(cfg.n_q_heads), cfg.head_dim));
  return pl;
}

// mixattn_set_layer_scores of one layer
struct LayerScores {
  float softcap = 0.f;
  std::vector<float> slopes;   // per query head; empty = no bias
  bool plain() const { return softcap == 0.f && slopes.empty(); }
};

struct ProfileRecord {
  int cls;
  cudaEvent_t start, stop;
};

}  // namespace

struct mixattn_ctx {
  CacheManager cm;
  mixattn_config cfg;  // layers / free_order pointers are not kept
  KvGeom geom;
  ArenaPlan plan;
  char* arena = nullptr;
  bool host_only = true;
  int device = -1;
  int sm_count = 148;
  int64_t l2_bytes = 0;
  float scale = 0.f;
  std::vector<LayerScores> scores;   // per layer
  int32_t split_tokens = 0;
  int64_t launches = 0;
  bool profiling = false;
  std::vector<ProfileRecord> records;
  std::vector<cudaEvent_t> event_pool;
  bool sticky_cuda_error = false;
  // Chunk calls of layers that share a cache gather the same rows: what the scratch holds is
  // remembered so that, when the caller has enabled it, the copy runs once per run of such calls.
  bool chunk_reuse = false;
  // Chunk calls of sliding-window layers whose window is a whole number of key tiles read the
  // cached keys in place from the ring (no copy); off = every chunk call copies.
  bool chunk_ring_direct = true;
  int64_t shared_room = 0;       // rows of a shared decode's partial results that the arena holds
  bool prefix_sharing = false;   // decode calls go the way of mixattn_decode_shared
  int64_t share_min_bytes = -1;  // what such a call has to save; < 0 = automatic
  uint64_t cache_epoch = 0;   // bumped by every call that changes a cache
  struct GatherKey {
    bool valid = false;
    int owner = -1;
    uint64_t epoch = 0;
    const void* k = nullptr;
    const void* v = nullptr;
    cudaStream_t st = nullptr;
    std::vector<int32_t> ids, lens;
  } scratch_holds;

  char* owner_storage(int layer) const { return arena + plan.owner_off[cm.layer(layer).owner_slot]; }
  int32_t* dev_table() const { return reinterpret_cast<int32_t*>(arena + plan.table_off); }
  int32_t* dev_status() const { return reinterpret_cast<int32_t*>(arena + plan.status_off); }
};

namespace {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    target = dev;
  }
  ~DeviceGuard() {
    if (ok && prev >= 0 && prev != target) cudaSetDevice(prev);
  }
  int target = -1;
};

cudaEvent_t take_event(mixattn_ctx* c) {
  if (!c->event_pool.empty()) {
    cudaEvent_t e = c->event_pool.back();
    c->event_pool.pop_back();
    return e;
  }
  cudaEvent_t e = nullptr;
  cudaEventCreate(&e);
  return e;
}

// Brackets one launch with events when profiling is on.
template <typename F>
cudaError_t launch_recorded(mixattn_ctx* c, int cls, cudaStream_t st, F&& f) {
  ProfileRecord rec{cls, nullptr, nullptr};
  if (c->profiling) {
    rec.start = take_event(c);
    rec.stop = take_event(c);
    if (rec.start) cudaEventRecord(rec.start, st);
  }
  cudaError_t e = f();
  if (c->profiling) {
    if (rec.stop) cudaEventRecord(rec.stop, st);
    c->records.push_back(rec);
  }
  if (e == cudaSuccess) ++c->launches;
  else c->sticky_cuda_error = true;
  return e;
}

int validate_config(const mixattn_config* cfg, CacheManager* cm, bool allocate = true) {
  if (cfg == nullptr) return MIXATTN_ERR_INVALID_ARG;
  int rc = cm->init(*cfg, allocate);
  if (rc != MIXATTN_OK) return rc;
  if (cfg->softmax_scale < 0.f || !isfinite(cfg->softmax_scale)) return MIXATTN_ERR_INVALID_ARG;
  if (cm->n_full_owners() > 0 && cfg->n_pages < 1) return MIXATTN_ERR_INVALID_ARG;
  if (cfg->chunk_scratch_tokens < 0) return MIXATTN_ERR_INVALID_ARG;
  if (cfg->kv_format != MIXATTN_KV_NATIVE && cfg->kv_format != MIXATTN_KV_FP8_E4M3) return MIXATTN_ERR_INVALID_ARG;
  if (cfg->kv_format == MIXATTN_KV_FP8_E4M3 && (cfg->dtype != MIXATTN_BF16 || cfg->head_dim != 128))
    return MIXATTN_ERR_UNSUPPORTED;
  return MIXATTN_OK;
}

// Block-table entries of a bulk append: they travel in kernel parameters (no host copy that would
// wait for the stream or depend on pageable memory) and are set by a small kernel ahead of the one
// that stores the tokens, which reads the table.
int enqueue_grants(mixattn_ctx* c, const std::vector<PageGrant>& grants, cudaStream_t st) {
  const int stride = c->cm.max_blocks();
  TableSetParams tp;
  tp.table = c->dev_table();
  for (size_t a = 0; a < grants.size(); a += kTableSetMax) {
    const size_t n = grants.size() - a < (size_t)kTableSetMax ? grants.size() - a : (size_t)kTableSetMax;
    for (size_t i = 0; i < n; ++i) {
      tp.idx[i] = c->cm.slot(grants[a + i].seq) * stride + grants[a + i].block;
      tp.page[i] = grants[a + i].page;
    }
    tp.n = (int32_t)n;
    cudaError_t e = launch_recorded(c, MIXATTN_K_APPEND, st, [&] { return launch_table_set(tp, st); });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

// Enqueues the device side of an append the host bookkeeping has already applied.
int enqueue_append(mixattn_ctx* c, int layer, int n_seqs, const int32_t* seq_ids,
                   const int32_t* n_new, const std::vector<int32_t>& start_pos,
                   const std::vector<PageGrant>& grants, const void* k, const void* v,
                   cudaStream_t st, double rope_log2_theta = 0.0) {
  const LayerInfo& li = c->cm.layer(layer);
  const bool ring = li.kind == MIXATTN_SLIDING;
  bool single = true;
  for (int i = 0; i < n_seqs; ++i) single = single && (n_new == nullptr || n_new[i] == 1);
  const int stride = c->cm.max_blocks();
  if (!ring && !single && !grants.empty()) {
    const int rc = enqueue_grants(c, grants, st);
    if (rc != MIXATTN_OK) return rc;
  }
  AppendParams p;
  p.k = k;
  p.v = v;
  p.pool = c->owner_storage(layer);
  p.table = c->dev_table();
  p.table_stride = stride;
  p.is_ring = ring;
  p.window = ring ? li.window : 0;
  p.ring_pages = ring ? ring_pages_of(li.window) : 0;
  p.geom = c->geom;
  p.rope_log2_theta = rope_log2_theta;
  int row = 0;
  size_t gi = 0;
  for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
    const int nb = n_seqs - i0 < kMaxCallSeqs ? n_seqs - i0 : kMaxCallSeqs;
    int max_new = 0;
    for (int j = 0; j < nb; ++j) {
      const int i = i0 + j;
      AppendEntry& e = p.e[j];
      e.seq = c->cm.slot(seq_ids[i]);
      e.start_pos = start_pos[i];
      e.n_new = n_new ? n_new[i] : 1;
      e.src_row0 = row;
      e.page_hint = -1;
      e.tbl_idx = -1;
      if (!ring && single) {
        e.page_hint = c->cm.table_row(seq_ids[i])[e.start_pos / kPage];
        // grants are in call order: at most one per sequence in single-token mode
        if (gi < grants.size() && grants[gi].seq == seq_ids[i]) {
          e.tbl_idx = e.seq * stride + grants[gi].block;
          ++gi;
        }
      }
      row += e.n_new;
      if (e.n_new > max_new) max_new = e.n_new;
    }
    p.n_entries = nb;
    if (max_new == 0) {
      bool any_tbl = false;
      for (int j = 0; j < nb; ++j) any_tbl = any_tbl || p.e[j].tbl_idx >= 0;
      if (!any_tbl) continue;
    }
    cudaError_t e = launch_recorded(c, MIXATTN_K_APPEND, st, [&] { return launch_append(p, max_new, st); });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

}  // namespace

extern "C" {

int mixattn_arena_bytes(const mixattn_config* cfg, size_t* out_bytes) {
  if (out_bytes == nullptr) return MIXATTN_ERR_INVALID_ARG;
  CacheManager cm;
  int rc = validate_config(cfg, &cm, false);
  if (rc != MIXATTN_OK) return rc;
  *out_bytes = plan_arena(cm, *cfg).total;
  return MIXATTN_OK;
}

int mixattn_cache_bytes(const mixattn_config* cfg, size_t* out_bytes) {
  if (out_bytes == nullptr) return MIXATTN_ERR_INVALID_ARG;
  CacheManager cm;
  int rc = validate_config(cfg, &cm, false);
  if (rc != MIXATTN_OK) return rc;
  *out_bytes = plan_arena(cm, *cfg).cache_bytes;
  return MIXATTN_OK;
}

int mixattn_create(const mixattn_config* cfg, mixattn_ctx** out) {
  if (out == nullptr) return MIXATTN_ERR_INVALID_ARG;
  *out = nullptr;
  mixattn_ctx* c = new (std::nothrow) mixattn_ctx();
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  int rc = validate_config(cfg, &c->cm);
  if (rc != MIXATTN_OK) { delete c; return rc; }
  c->cfg = *cfg;
  c->cfg.layers = nullptr;
  c->cfg.free_order = nullptr;
  c->geom = make_geom(cfg->n_kv_heads, cfg->head_dim, cfg->dtype, cfg->kv_format);
  c->plan = plan_arena(c->cm, *cfg);
  c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / sqrtf((float)cfg->head_dim);
  c->scores.resize(cfg->n_layers);
  c->host_only = cfg->device < 0;
  c->device = cfg->device;
  if (!c->host_only) {
    if (cfg->arena == nullptr || cfg->arena_bytes < c->plan.least ||
        (reinterpret_cast<uintptr_t>(cfg->arena) % kAlign) != 0) {
      delete c;
      return MIXATTN_ERR_INVALID_ARG;
    }
    c->arena = static_cast<char*>(cfg->arena);
    const size_t arena_bytes = std::min(cfg->arena_bytes, c->plan.total);
    c->shared_room = shared_rows_that_fit(arena_bytes - c->plan.part_o_off, cfg->n_q_heads, cfg->head_dim);
    DeviceGuard g(c->device);
    int sms = 0, l2 = 0;   // (single attributes: filling the whole property block takes milliseconds)
    if (!g.ok || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, c->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&l2, cudaDevAttrL2CacheSize, c->device) != cudaSuccess) {
      delete c;
      return MIXATTN_ERR_CUDA;
    }
    c->sm_count = sms;
    c->l2_bytes = l2;
    if (prepare_decode_bf16() != cudaSuccess || prepare_prefill_tc() != cudaSuccess ||
        prepare_beam_select() != cudaSuccess || prepare_decode_shared() != cudaSuccess ||
        prepare_decode_shared_tc() != cudaSuccess ||
        prepare_adjust_logits() != cudaSuccess) { delete c; return MIXATTN_ERR_CUDA; }
    if (cudaMemsetAsync(c->arena, 0, arena_bytes, 0) != cudaSuccess ||
        cudaStreamSynchronize(0) != cudaSuccess) {
      delete c;
      return MIXATTN_ERR_CUDA;
    }
  }
  *out = c;
  return MIXATTN_OK;
}

int mixattn_destroy(mixattn_ctx* c) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  if (!c->host_only) {
    DeviceGuard g(c->device);
    for (auto& r : c->records) {
      if (r.start) cudaEventDestroy(r.start);
      if (r.stop) cudaEventDestroy(r.stop);
    }
    for (auto e : c->event_pool) cudaEventDestroy(e);
  }
  delete c;
  return MIXATTN_OK;
}

int mixattn_seq_reset(mixattn_ctx* c, int32_t seq) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  c->cm.seq_reset(seq);
  ++c->cache_epoch;
  return MIXATTN_OK;
}

// Device side of the copies a fork made (see CacheManager::apply_fork).
static int enqueue_fork(mixattn_ctx* c, const ForkPlan& plan, cudaStream_t st) {
  ForkParams p;
  p.arena = c->arena;
  p.table = c->dev_table();
  p.table_stride = c->cm.max_blocks();
  p.n_segs = p.n_rows = 0;
  auto flush = [&]() {
    if (p.n_segs + p.n_rows == 0) return cudaSuccess;
    cudaError_t e = launch_recorded(c, MIXATTN_K_FORK, st, [&] { return launch_fork_copy(p, st); });
    p.n_segs = p.n_rows = 0;
    return e;
  };
  auto add_seg = [&](size_t src, size_t dst, int64_t bytes) {
    cudaError_t e = p.n_segs == ForkParams::kMaxSegs ? flush() : cudaSuccess;
    p.seg[p.n_segs++] = CopySeg{(int64_t)src, (int64_t)dst, (uint32_t)(bytes / 16)};
    return e;
  };
  const int64_t page_bytes = c->geom.page_bytes;
  // a segment's length is counted in 32 bits of 16-byte units; rings longer than that are cut
  const int64_t max_bytes = (int64_t)1 << 34;
  for (const ForkCopy& f : plan.copies) {
    const int32_t* src_pages = plan.src_pages.data() + f.tail0;
    const int32_t* dst_pages = plan.dst_pages.data() + f.tail0;
    for (size_t o = 0; o < c->cm.owners().size(); ++o) {
      const LayerInfo& li = c->cm.layer(c->cm.owners()[o]);
      const size_t pool = c->plan.owner_off[o];
      if (li.kind == MIXATTN_FULL) {
        for (int b = 0; b < f.n_tail; ++b)
          if (add_seg(pool + (size_t)src_pages[b] * page_bytes, pool + (size_t)dst_pages[b] * page_bytes, page_bytes) != cudaSuccess)
            return MIXATTN_ERR_CUDA;
        continue;
      }
      const int32_t n = c->cm.slot_len((int)o, f.dst_slot), valid = n < li.window ? n : li.window;
      const size_t ring = (size_t)ring_pages_of(li.window) * page_bytes;
      const int64_t bytes = (int64_t)ring_pages_of(valid) * page_bytes;
      for (int64_t a = 0; a < bytes; a += max_bytes)
        if (add_seg(pool + f.src_slot * ring + a, pool + f.dst_slot * ring + a, std::min(max_bytes, bytes - a)) != cudaSuccess)
          return MIXATTN_ERR_CUDA;
    }
    int32_t done = 0;
    bool first = f.n_shared > f.same;
    while (first || done < f.n_tail) {
      if (p.n_rows == ForkParams::kMaxRows && flush() != cudaSuccess) return MIXATTN_ERR_CUDA;
      TableRow& r = p.row[p.n_rows++];
      r.src_slot = f.src_slot;
      r.dst_slot = f.dst_slot;
      r.copy0 = f.same;
      r.n_copy = first ? f.n_shared - f.same : 0;
      r.set0 = f.n_shared + done;
      r.n_set = std::min(f.n_tail - done, kRowPages);
      for (int i = 0; i < r.n_set; ++i) r.page[i] = dst_pages[done + i];
      done += r.n_set;
      first = false;
    }
  }
  return flush() == cudaSuccess ? MIXATTN_OK : MIXATTN_ERR_CUDA;
}

int mixattn_fork_seqs(mixattn_ctx* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  bool moved = false;
  try {
    int rc = c->cm.check_fork(n, src, dst);
    if (rc != MIXATTN_OK) return rc;
    if (!c->host_only && c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
    ForkPlan plan;
    moved = true;
    rc = c->cm.apply_fork(n, src, dst, &plan);
    if (rc != MIXATTN_OK) return rc;
    ++c->cache_epoch;
    if (c->host_only || plan.copies.empty()) return MIXATTN_OK;
    DeviceGuard g(c->device);
    if (!g.ok) {
      c->sticky_cuda_error = true;   // the bookkeeping has moved
      return MIXATTN_ERR_CUDA;
    }
    return enqueue_fork(c, plan, static_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {   // no host memory: the bookkeeping may have moved, so the context is done
    if (moved) c->sticky_cuda_error = true;
    return MIXATTN_ERR_CUDA;
  }
}

int mixattn_read_kv(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, const int32_t* first_pos,
                    const int32_t* n_tokens, void* k, void* v, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0 || (n_seqs > 0 && seq_ids == nullptr))
    return MIXATTN_ERR_INVALID_ARG;
  const LayerInfo& li = c->cm.layer(layer);
  const bool ring = li.kind == MIXATTN_SLIDING;
  // range of sequence i: [first, first + n) inside the stored tokens
  auto range = [&](int i, int32_t* first, int32_t* n) {
    const int32_t end = c->cm.len(layer, seq_ids[i]), oldest = end - c->cm.n_attended(layer, seq_ids[i]);
    *first = first_pos ? first_pos[i] : oldest;
    *n = n_tokens ? n_tokens[i] : end - *first;
    return *first >= oldest && *n >= 0 && *first <= end && *n <= end - *first;
  };
  int64_t total = 0;
  for (int i = 0; i < n_seqs; ++i) {
    int32_t first, n;
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
    if (!range(i, &first, &n)) return MIXATTN_ERR_INVALID_ARG;
    total += n;
  }
  if (total > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (total == 0) return MIXATTN_OK;
  if (k == nullptr || v == nullptr || ((((size_t)k) | ((size_t)v)) & 15)) return MIXATTN_ERR_INVALID_ARG;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  GatherParams p;
  p.k_chunk = p.v_chunk = nullptr;
  p.k_out = k;
  p.v_out = v;
  p.pool = c->owner_storage(layer);
  p.table = c->dev_table();
  p.table_stride = c->cm.max_blocks();
  p.is_ring = ring;
  p.window = ring ? li.window : 0;
  p.ring_pages = ring ? ring_pages_of(li.window) : 0;
  p.geom = c->geom;
  int32_t row = 0;
  for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
    int longest = 0;
    p.n_entries = std::min(n_seqs - i0, kMaxCallSeqs);
    for (int j = 0; j < p.n_entries; ++j) {
      GatherEntry& e = p.e[j];
      range(i0 + j, &e.pos0, &e.n_prefix);
      e.seq = c->cm.slot(seq_ids[i0 + j]);
      e.n_chunk = e.src_row0 = 0;
      e.dst_row0 = row;
      row += e.n_prefix;
      longest = std::max(longest, e.n_prefix);
    }
    if (longest == 0) continue;
    if (launch_recorded(c, MIXATTN_K_READ, st, [&] { return launch_read_kv(p, longest, st); }) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

int mixattn_beam_select(mixattn_ctx* c, int32_t n_groups, int32_t n_beams, int32_t vocab, int32_t logits_dtype,
                        const void* logits, int64_t row_stride, const float* scores, const uint8_t* finished,
                        int32_t eos_token, int32_t n_out, float* out_scores, int32_t* out_beams,
                        int32_t* out_tokens, void* stream) {
  if (c == nullptr || n_groups < 0 || n_beams < 1 || n_beams > MIXATTN_MAX_BEAMS || vocab < 1 || n_out < 1 ||
      n_out > MIXATTN_MAX_BEAM_OUT || (logits_dtype != MIXATTN_F32 && logits_dtype != MIXATTN_BF16) ||
      row_stride < vocab)
    return MIXATTN_ERR_INVALID_ARG;
  if (vocab > MIXATTN_MAX_VOCAB || (int64_t)n_beams * vocab > INT32_MAX || (int64_t)n_groups * n_beams > INT32_MAX)
    return MIXATTN_ERR_INVALID_ARG;
  if (row_stride > INT64_MAX / 8 / std::max<int64_t>((int64_t)n_groups * n_beams, 1)) return MIXATTN_ERR_INVALID_ARG;   // byte offsets in 64 bits
  if (finished != nullptr && (eos_token < 0 || eos_token >= vocab)) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_groups == 0) return MIXATTN_OK;
  const int elem = logits_dtype == MIXATTN_BF16 ? 2 : 4;
  if (logits == nullptr || scores == nullptr || out_scores == nullptr || out_beams == nullptr || out_tokens == nullptr ||
      (size_t)logits % elem != 0)
    return MIXATTN_ERR_INVALID_ARG;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  BeamParams p;
  p.status = c->dev_status();
  p.tickets = reinterpret_cast<int32_t*>(c->arena + c->plan.ticket_off);
  p.row_stride = row_stride;
  p.n_beams = n_beams;
  p.vocab = vocab;
  p.n_out = n_out;
  p.eos = eos_token;
  // the chunks' results live in the split-KV workspace; groups that do not fit it together run
  // one batch after the other
  const size_t room = c->plan.split_bytes;
  const size_t per_chunk = sizeof(float2) + (size_t)n_out * sizeof(uint64_t);
  const int64_t rows = (int64_t)n_groups * n_beams;
  p.n_chunks = beam_chunks((int)rows, vocab, elem, c->sm_count, &p.chunk_granules);
  if ((size_t)n_beams * p.n_chunks * per_chunk > room) {   // one group must fit: fewer chunks (the workspace holds MIXATTN_MAX_BEAMS rows of one)
    const int64_t fit = (int64_t)(room / (n_beams * per_chunk));
    const int64_t granules = (int64_t)p.n_chunks * p.chunk_granules;
    p.chunk_granules = (int)((granules + fit - 1) / fit);
    p.n_chunks = (int)((granules + p.chunk_granules - 1) / p.chunk_granules);
  }
  const size_t per_group = (size_t)n_beams * p.n_chunks * per_chunk;
  int64_t batch = (int64_t)(room / per_group);
  batch = std::min<int64_t>(std::min<int64_t>(batch, 65535 / n_beams), kBeamTickets);
  char* ws = c->arena + c->plan.part_o_off;
  for (int64_t g0 = 0; g0 < n_groups; g0 += batch) {
    const int64_t r0 = g0 * n_beams;
    p.n_groups = (int32_t)std::min<int64_t>(batch, n_groups - g0);
    p.logits = static_cast<const char*>(logits) + r0 * row_stride * elem;
    p.scores = scores + r0;
    p.finished = finished ? finished + r0 : nullptr;
    p.out_scores = out_scores + g0 * n_out;
    p.out_beams = out_beams + g0 * n_out;
    p.out_tokens = out_tokens + g0 * n_out;
    p.part_keys = reinterpret_cast<uint64_t*>(ws);
    p.part_sums = reinterpret_cast<float2*>(ws + (size_t)p.n_groups * n_beams * p.n_chunks * n_out * sizeof(uint64_t));
    if (launch_recorded(c, MIXATTN_K_SELECT, st, [&] { return launch_beam_select(p, elem, st); }) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

static int append_impl(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                       const int32_t* n_new, const void* k, const void* v, void* stream, double rope_log2_theta) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  int rc = c->cm.check_append(layer, n_seqs, seq_ids, n_new);
  if (rc != MIXATTN_OK) return rc;
  int64_t total = 0;
  for (int i = 0; i < n_seqs; ++i) total += n_new ? n_new[i] : 1;
  if (total > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
  if (!c->host_only) {
    if (total > 0 && (k == nullptr || v == nullptr)) return MIXATTN_ERR_INVALID_ARG;
    if (c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  }
  std::vector<int32_t> start(n_seqs);
  for (int i = 0; i < n_seqs; ++i) start[i] = c->cm.len(layer, seq_ids[i]);
  std::vector<PageGrant> grants;
  c->cm.apply_append(layer, n_seqs, seq_ids, n_new, &grants);
  ++c->cache_epoch;
  if (c->host_only) return MIXATTN_OK;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  return enqueue_append(c, layer, n_seqs, seq_ids, n_new, start, grants, k, v,
                        static_cast<cudaStream_t>(stream), rope_log2_theta);
}

int mixattn_append_kv(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                      const int32_t* n_new, const void* k, const void* v, void* stream) {
  return append_impl(c, layer, n_seqs, seq_ids, n_new, k, v, stream, 0.0);
}

int mixattn_append_kv_rope(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                           const int32_t* n_new, const void* k, const void* v, float rope_theta,
                           void* stream) {
  if (!(rope_theta > 1.f) || !isfinite(rope_theta)) return MIXATTN_ERR_INVALID_ARG;
  return append_impl(c, layer, n_seqs, seq_ids, n_new, k, v, stream, log2((double)rope_theta));
}

int mixattn_rope_qkv(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, const int32_t* n_new,
                     const int32_t* first_pos, const mixattn_rope* rope, const void* q, int64_t q_stride, const void* k,
                     int64_t k_stride, const void* v, int64_t v_stride, int32_t store, void* q_out, void* k_out,
                     void* v_out, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0 || (n_seqs > 0 && seq_ids == nullptr) || rope == nullptr ||
      (store != 0 && store != 1))
    return MIXATTN_ERR_INVALID_ARG;
  RopeParams p;
  p.rotary = rope->rotary_dim;
  if (p.rotary < 16 || p.rotary > c->cfg.head_dim || p.rotary % 16 != 0) return MIXATTN_ERR_INVALID_ARG;
  if (rope->inv_freq == nullptr && !(rope->theta > 1.0 && isfinite(rope->theta))) return MIXATTN_ERR_INVALID_ARG;
  if (!(rope->scale >= 0.f) || !isfinite(rope->scale)) return MIXATTN_ERR_INVALID_ARG;
  for (int i = 0; i < p.rotary / 2; ++i) {
    p.freq[i] = rope->inv_freq ? rope->inv_freq[i] : pow(rope->theta, -2.0 * i / p.rotary);
    if (!(fabs(p.freq[i]) <= 1e6)) return MIXATTN_ERR_INVALID_ARG;   // (NaN, or turns that a double does not count exactly)
  }
  p.scale = rope->scale > 0.f ? rope->scale : 1.f;
  p.halves = rope->halves != 0;
  const LayerInfo& li = c->cm.layer(layer);
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim, esz = c->geom.elem_bytes;
  if (store) {
    try {
      const int rc = c->cm.check_append(layer, n_seqs, seq_ids, n_new);
      if (rc != MIXATTN_OK) return rc;
    } catch (const std::bad_alloc&) {
      return MIXATTN_ERR_CUDA;
    }
  }
  int64_t total = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
    const int64_t n = n_new ? n_new[i] : 1, at = first_pos ? first_pos[i] : c->cm.len(layer, seq_ids[i]);
    if (n < 0 || at < 0 || at + n > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
    total += n;
  }
  if (total > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
  if (!c->host_only && c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (c->host_only && !store) return MIXATTN_ERR_CUDA;
  if (!c->host_only && total > 0) {
    if ((q == nullptr && k == nullptr && v == nullptr) || (store && (k == nullptr || v == nullptr)) ||
        (q_out != nullptr && q == nullptr) || (k_out != nullptr && k == nullptr) || (v_out != nullptr && v == nullptr))
      return MIXATTN_ERR_INVALID_ARG;
    const void* in[3] = {q, k, v};
    const int64_t stride[3] = {q_stride, k_stride, v_stride};
    for (int i = 0; i < 3; ++i) {
      if (in[i] == nullptr) continue;
      const int64_t least = (int64_t)(i == 0 ? Hq : Hkv) * D;
      if (total > 1 && (stride[i] < least || stride[i] > INT64_MAX / esz / total || stride[i] * esz % 16 != 0)) return MIXATTN_ERR_INVALID_ARG;
    }
    if (((size_t)q | (size_t)k | (size_t)v | (size_t)q_out | (size_t)k_out | (size_t)v_out) & 15) return MIXATTN_ERR_INVALID_ARG;
  }
  std::vector<int32_t> start;
  std::vector<PageGrant> grants;
  bool moved = false;
  try {
    start.resize(n_seqs);
    for (int i = 0; i < n_seqs; ++i) start[i] = c->cm.len(layer, seq_ids[i]);
    if (store) {
      moved = true;
      c->cm.apply_append(layer, n_seqs, seq_ids, n_new, &grants);
      ++c->cache_epoch;
    }
  } catch (const std::bad_alloc&) {   // no host memory: the bookkeeping may have moved
    if (moved) c->sticky_cuda_error = true;
    return MIXATTN_ERR_CUDA;
  }
  if (c->host_only || total == 0) return MIXATTN_OK;
  DeviceGuard g(c->device);
  if (!g.ok) {
    if (store) c->sticky_cuda_error = true;
    return MIXATTN_ERR_CUDA;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool ring = li.kind == MIXATTN_SLIDING;
  bool single = true;
  for (int i = 0; i < n_seqs; ++i) single = single && (n_new == nullptr || n_new[i] == 1);
  if (store && !ring && !single && !grants.empty()) {
    const int rc = enqueue_grants(c, grants, st);
    if (rc != MIXATTN_OK) return rc;
  }
  p.q_stride = total > 1 ? q_stride * esz : 0;
  p.k_stride = total > 1 ? k_stride * esz : 0;
  p.v_stride = total > 1 ? v_stride * esz : 0;
  // (inputs that nothing is done with are not read)
  p.q = static_cast<const char*>(q_out ? q : nullptr);
  p.k = static_cast<const char*>(k_out || store ? k : nullptr);
  p.v = static_cast<const char*>(v_out || store ? v : nullptr);
  p.q_out = static_cast<char*>(q_out);
  p.k_out = static_cast<char*>(k_out);
  p.v_out = static_cast<char*>(v_out);
  if (p.q == nullptr && p.k == nullptr && p.v == nullptr) return MIXATTN_OK;   // nothing is wanted
  p.pool = store ? c->owner_storage(layer) : nullptr;
  p.table = c->dev_table();
  p.table_stride = c->cm.max_blocks();
  p.is_ring = ring;
  p.window = ring ? li.window : 0;
  p.ring_pages = ring ? ring_pages_of(li.window) : 0;
  p.geom = c->geom;
  p.n_q_heads = Hq;
  int32_t row = 0;
  size_t gi = 0;
  for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
    p.n_entries = std::min(n_seqs - i0, kMaxCallSeqs);
    int most = 0;
    for (int j = 0; j < p.n_entries; ++j) {
      const int i = i0 + j;
      RopeEntry& e = p.e[j];
      e.seq = c->cm.slot(seq_ids[i]);
      e.start_pos = start[i];
      e.pos0 = first_pos ? first_pos[i] : start[i];
      e.n_new = n_new ? n_new[i] : 1;
      e.row0 = row;
      e.page_hint = e.tbl_idx = -1;
      if (store && !ring && single) {
        e.page_hint = c->cm.table_row(seq_ids[i])[e.start_pos / kPage];
        if (gi < grants.size() && grants[gi].seq == seq_ids[i]) {
          e.tbl_idx = e.seq * p.table_stride + grants[gi].block;
          ++gi;
        }
      }
      row += e.n_new;
      most = std::max(most, e.n_new);
    }
    if (most == 0) continue;
    if (launch_recorded(c, MIXATTN_K_ROPE, st, [&] { return launch_rope_qkv(p, most, st); }) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

int mixattn_adjust_logits(mixattn_ctx* c, int32_t n_rows, int32_t vocab, int32_t logits_dtype, const void* logits,
                          int64_t row_stride, int32_t out_dtype, void* out, int64_t out_stride,
                          const mixattn_logit_rules* rules, void* stream) {
  if (c == nullptr || rules == nullptr || n_rows < 0 || vocab < 1 || vocab > MIXATTN_MAX_VOCAB ||
      (logits_dtype != MIXATTN_F32 && logits_dtype != MIXATTN_BF16) || (out_dtype != MIXATTN_F32 && out_dtype != MIXATTN_BF16))
    return MIXATTN_ERR_INVALID_ARG;
  if (logits_dtype == MIXATTN_F32 && out_dtype == MIXATTN_BF16) return MIXATTN_ERR_UNSUPPORTED;
  const mixattn_logit_rules& r = *rules;
  const int64_t rows = std::max<int64_t>(n_rows, 1), limit = INT64_MAX / 8 / rows;
  if (rows > INT32_MAX / 8) return MIXATTN_ERR_INVALID_ARG;
  if (row_stride < vocab || out_stride < vocab || row_stride > limit || out_stride > limit) return MIXATTN_ERR_INVALID_ARG;
  if (r.max_tokens < 0 || r.max_tokens > MIXATTN_MAX_RULE_TOKENS || r.n_bias < 0 || r.n_bias > MIXATTN_MAX_RULE_BIASES)
    return MIXATTN_ERR_INVALID_ARG;
  if (r.tokens != nullptr ? (r.token_stride < r.max_tokens || r.token_stride > limit)
                          : (r.max_tokens != 0 || r.n_tokens != nullptr || r.n_prompt != nullptr))
    return MIXATTN_ERR_INVALID_ARG;
  if ((r.bias_tokens != nullptr) != (r.bias_values != nullptr) || (r.bias_tokens == nullptr && r.n_bias != 0)) return MIXATTN_ERR_INVALID_ARG;
  if (r.allowed != nullptr) {
    if (r.n_allowed < 1 || r.allowed_stride < ((int64_t)vocab + 31) / 32 || r.allowed_stride > INT64_MAX / 8 / r.n_allowed ||
        (r.allowed_rows == nullptr && r.n_allowed < n_rows))
      return MIXATTN_ERR_INVALID_ARG;
  } else if (r.n_allowed != 0 || r.allowed_rows != nullptr) {
    return MIXATTN_ERR_INVALID_ARG;
  }
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_rows == 0) return MIXATTN_OK;
  if (logits == nullptr || out == nullptr || (size_t)logits % (logits_dtype == MIXATTN_BF16 ? 2 : 4) != 0 ||
      (size_t)out % (out_dtype == MIXATTN_BF16 ? 2 : 4) != 0)
    return MIXATTN_ERR_INVALID_ARG;
  const void* words[9] = {r.tokens, r.n_tokens, r.n_prompt, r.repetition, r.frequency, r.presence, r.temperature, r.bias_tokens, r.allowed};
  for (const void* w : words)
    if ((size_t)w % 4 != 0) return MIXATTN_ERR_INVALID_ARG;
  if (((size_t)r.bias_values | (size_t)r.allowed_rows) % 4 != 0) return MIXATTN_ERR_INVALID_ARG;
  if (logits == out && (logits_dtype != out_dtype || row_stride != out_stride)) return MIXATTN_ERR_INVALID_ARG;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  AdjustParams p;
  p.logits = logits;
  p.out = out;
  p.row_stride = row_stride;
  p.out_stride = out_stride;
  p.n_rows = n_rows;
  p.vocab = vocab;
  p.in_place = logits == out;
  p.rules = r;
  if (r.max_tokens == 0) p.rules.tokens = nullptr;
  if (launch_recorded(c, MIXATTN_K_ADJUST, st, [&] { return launch_adjust_logits(p, logits_dtype, out_dtype, c->sm_count, st); }) != cudaSuccess)
    return MIXATTN_ERR_CUDA;
  return MIXATTN_OK;
}

// L2 policy of a decode launch (see l2_policy_of in decode_bf16.cu).  Only a ring that a later
// layer reads again (Section 3's cache sharing makes consecutive layers read the same bytes) is
// worth keeping: the leading part of its storage, up to a share of the L2 that a cyclic scan was
// measured to keep resident.  The last layer that reads the ring lets go of it.
static void set_l2_policy(const mixattn_ctx* c, int layer, DecodeParams* p) {
  p->l2_keep_bytes = 0;
  p->l2_pool_bytes = 0;
  const LayerInfo& li = c->cm.layer(layer);
  if (li.kind != MIXATTN_SLIDING || c->l2_bytes <= 0) return;
  bool read_again = false;
  for (int l = layer + 1; l < c->cfg.n_layers; ++l) read_again = read_again || c->cm.layer(l).owner == li.owner;
  if (!read_again) return;
  const uint64_t pool = c->plan.owner_bytes[li.owner_slot];
  // (measured on a 126 MB L2: a 67 MB ring stays resident under plain LRU, a 134 MB ring does not
  // at all; keeping 0.4-0.5 of the L2 of it gave the shortest step)
  const uint64_t fits = (uint64_t)(kL2FitsShare * (double)c->l2_bytes);
  const uint64_t room = (uint64_t)(kL2KeepShare * (double)c->l2_bytes);
  const uint64_t window = pool < 0xFFFFFF00ull ? pool : 0xFFFFFF00ull;   // the policy's sizes are 32-bit
  p->l2_pool_bytes = (uint32_t)window;
  p->l2_keep_bytes = (uint32_t)(window <= fits ? window : room);
}

// Kernel parameters of a layer's shaped scores; false = plain scores (nothing to pass).
static bool score_shape_of(const mixattn_ctx* c, int layer, ScoreShape* sh) {
  const LayerScores& ls = c->scores[layer];
  if (ls.plain()) return false;
  sh->pre = ls.softcap > 0.f ? c->scale / ls.softcap : c->scale * kLog2e;
  sh->post = ls.softcap * kLog2e;
  const double pre = sh->pre;
  bool normal = pre > 1e-18;   // (squares of products up to 1 / (2 pre) stay finite)
  double power = pre;
  for (int i = 0; i < 4; ++i, power *= pre * pre) {
    const double f = tanh_near_coefficient(i) * power * ls.softcap * (double)kLog2e;
    normal = normal && fabs(f) > 1e-36 && fabs(f) < 1e36;
    sh->near[i] = (float)f;
  }
  sh->near_sq = normal ? (float)(0.25 / (pre * pre)) : -1.f;
  sh->biased = !ls.slopes.empty();
  for (size_t h = 0; h < ls.slopes.size(); ++h) sh->slope[h] = ls.slopes[h] * kLog2e;
  return true;
}

// Where the keys of a decode launch sit relative to the query (sequences ids[0 .. nb)).
static void set_distances(const mixattn_ctx* c, int layer, const int32_t* ids, int nb, ShapedDecodeParams* p) {
  const LayerInfo& li = c->cm.layer(layer);
  p->wrap = li.kind == MIXATTN_SLIDING ? li.window : 0;
  for (int j = 0; j < nb; ++j) {
    const int32_t n = c->cm.len(layer, ids[j]);
    p->newest[j] = p->wrap ? (n - 1) % p->wrap : n - 1;
  }
}

// The split pass of a decode launch; `shaped`: the layer's scores are shaped.
static cudaError_t launch_split_pass(const mixattn_ctx* c, const ShapedDecodeParams& p, bool shaped, cudaStream_t st) {
  const ShapedDecodeParams* sp = shaped ? &p : nullptr;
  return c->cfg.dtype == MIXATTN_BF16 ? launch_decode_split_bf16(p, sp, c->sm_count, st)
                                      : launch_decode_split_f32(p, sp, st);
}

// Splits of a shared decode's own keys: about four items for each of the launch's CTAs, which evens out
// lengths from a few tokens to thousands (64 sequences of 16 to 2048 own tokens behind 32k: 79 us with splits of 2048, 77).
static int64_t own_split(const mixattn_ctx* c, int64_t total, const DecodeParams* p) {
  if (c->split_tokens > 0) return (c->split_tokens + kPage - 1) / kPage * kPage;
  const int64_t t = total * c->cfg.n_kv_heads * p->head_chunks / (4 * (int64_t)p->partial);
  return std::min<int64_t>(std::max<int64_t>((t + kPage - 1) / kPage * kPage, 512), kSplitTokens);
}

// The cutting itself: n_eff[0 .. nb) are set, `total` is their sum.
static int cut_splits(const mixattn_ctx* c, int layer, int nb, int64_t total, DecodeParams* p, bool* any_split) {
  const int Hkv = c->cfg.n_kv_heads;
  int64_t T = p->partial ? own_split(c, total, p) : c->split_tokens > 0 ? (c->split_tokens + kPage - 1) / kPage * kPage : kSplitTokens;
  // Shaped scores, and too few items of that size to even out over the SMs: half the size.  (17
  // sequences of 1 to 64k tokens, quantised cache: 86 -> 67 us; 5 of 9k to 20k: 68 -> 49; with
  // 14 items per SM it makes no difference.  Layers with plain scores keep the splits, and with them
  // the order of summation, that they have had.)
  if (!p->partial && c->split_tokens == 0 && !c->scores[layer].plain() &&
      total * c->cfg.n_kv_heads * p->head_chunks < (int64_t)kFewItems * c->sm_count * T)
    T = kSplitTokens / 2;
  const int64_t extra = p->partial ? kOwnExtraChunks : kWsExtraChunks;
  int64_t t_min = (total + extra - 1) / extra;
  t_min = (t_min + kPage - 1) / kPage * kPage;
  if (T < t_min) T = t_min;
  const int64_t pairs = (int64_t)nb * Hkv * p->head_chunks;
  int64_t nc_wave = c->split_tokens > 0 || p->partial ? 1 : c->sm_count / pairs;
  if (nc_wave > kWsWaveChunks / nb) nc_wave = kWsWaveChunks / nb;   // the workspace bounds the extra splits
  int base = 0;
  *any_split = false;
  for (int j = 0; j < nb; ++j) {
    const int64_t n = p->n_eff[j];
    int64_t nc = (n + T - 1) / T;
    if (nc < nc_wave) {
      int64_t by_len = n / kMinSplitTokens;
      nc = by_len < nc_wave ? by_len : nc_wave;
      if (nc < 1) nc = 1;
    }
    int64_t len = (n + nc - 1) / nc;
    len = (len + kPage - 1) / kPage * kPage;
    nc = (n + len - 1) / len;
    p->chunk_base[j] = base;
    p->chunk_len[j] = (int32_t)len;
    base += (int)nc;
    *any_split = *any_split || nc > 1;
  }
  p->chunk_base[nb] = base;
  p->n_seqs = nb;
  p->total_items = base * Hkv * p->head_chunks;
  return base;
}

// Split plan of one decode launch over sequences ids[0 .. nb): fills the per-sequence fields of
// *p (seq_id, n_eff, chunk_len, chunk_base, n_seqs, total_items; group and head_chunks must be
// set) and returns the number of split slots the launch writes; *any_split tells whether a
// combine pass is needed.  Long caches are cut into splits of kSplitTokens keys (large splits
// keep the per-item epilogue negligible; thousands of items balance over the SMs).  When there
// are fewer (sequence, KV head) pairs than SMs, short caches are cut further, but only up to one
// item per SM, so the launch stays a single wave.  Both decode entry points use this one
// function, so they add the partial results in the same order.
static int plan_splits(const mixattn_ctx* c, int layer, const int32_t* ids, int nb, DecodeParams* p,
                       bool* any_split) {
  int64_t total = 0;
  for (int j = 0; j < nb; ++j) {
    p->seq_id[j] = c->cm.slot(ids[j]);
    p->n_eff[j] = c->cm.n_attended(layer, ids[j]);
    total += p->n_eff[j];
  }
  return cut_splits(c, layer, nb, total, p, any_split);
}

static int decode_plain(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, const void* q, void* out,
                        void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0) return MIXATTN_ERR_INVALID_ARG;
  if (n_seqs > 0 && (seq_ids == nullptr || q == nullptr || out == nullptr)) return MIXATTN_ERR_INVALID_ARG;
  for (int i = 0; i < n_seqs; ++i) {
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
  }
  for (int i = 0; i < n_seqs; ++i) {
    if (c->cm.len(layer, seq_ids[i]) < 1) return MIXATTN_ERR_EMPTY_CONTEXT;
  }
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_seqs == 0) return MIXATTN_OK;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  const LayerInfo& li = c->cm.layer(layer);
  const bool ring = li.kind == MIXATTN_SLIDING;
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim;
  const size_t esz = c->geom.elem_bytes;

  ShapedDecodeParams p;
  const bool shaped = score_shape_of(c, layer, &p.shape);
  p.pool = c->owner_storage(layer);
  p.table = ring ? nullptr : c->dev_table();
  p.table_stride = c->cm.max_blocks();
  p.ring_pages = ring ? ring_pages_of(li.window) : 0;
  p.geom = c->geom;
  p.n_q_heads = Hq;
  p.group = Hq / Hkv;
  p.head_chunks = (p.group + kMaxGroupRows - 1) / kMaxGroupRows;
  p.scale_log2e = c->scale * kLog2e;
  p.part_o = reinterpret_cast<float*>(c->arena + c->plan.part_o_off);
  p.part_ml = reinterpret_cast<float2*>(c->arena + c->plan.part_ml_off);
  p.status = c->dev_status();
  set_l2_policy(c, layer, &p);

  for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
    const int nb = n_seqs - i0 < kMaxCallSeqs ? n_seqs - i0 : kMaxCallSeqs;
    bool any_split = false;
    const int base = plan_splits(c, layer, seq_ids + i0, nb, &p, &any_split);
    if (base > kWsChunks) return MIXATTN_ERR_UNSUPPORTED;   // (cannot happen: the plan is bounded by the workspace)
    if (shaped) set_distances(c, layer, seq_ids + i0, nb, &p);
    p.q = static_cast<const char*>(q) + (size_t)i0 * Hq * D * esz;
    p.out = static_cast<char*>(out) + (size_t)i0 * Hq * D * esz;
    const int cls = ring ? MIXATTN_K_DECODE_SLIDING : MIXATTN_K_DECODE_FULL;
    cudaError_t e = launch_recorded(c, cls, st, [&] { return launch_split_pass(c, p, shaped, st); });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
    if (any_split) {
      e = launch_recorded(c, MIXATTN_K_COMBINE, st,
                          [&] { return launch_decode_combine(p, c->cfg.dtype, st); });
      if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
    }
  }
  return MIXATTN_OK;
}

// Lays the items of a tree's pieces out on the line of work units (internal.h) and cuts the line into equal
// parts for at most max_ctas CTAs, fewer if the partial results would not fit `room` rows.  Items whose rows
// make several chunks read the same keys: where they are long, each begins with a CTA of its own, so that all
// chunks get to a key at about the same time and it comes from HBM once (128k keys, 64 sequences x 4 heads:
// 229 -> 198 us).  With `leaves` the pieces of a single sequence are left to the split pass.  Returns false if
// it does not fit at all.
static bool lay_out_shared(const ShareTree& t, bool leaves, int max_ctas, int64_t room, SharedDecodeParams* p, int* n_leaves) {
  const int Hkv = p->geom.n_kv_heads;
  std::vector<int32_t> at(t.pieces.size(), -1);   // node of each piece
  p->n_nodes = 0;
  for (size_t v = 0; v < t.pieces.size(); ++v) {
    const SharePiece& s = t.pieces[v];
    if (leaves && s.ns == 1) continue;
    at[v] = p->n_nodes;
    p->node[p->n_nodes++] = ShareNode{s.t0, s.t1, s.slot, s.s0, s.ns, s.parent < 0 ? -1 : at[s.parent], 0, 0, 0, 0};
  }
  int end = p->n_nodes;
  p->node[end] = ShareNode{0, 0, 0, 0, 0, -1, 0, 0, 0, 0};
  if (leaves)
    for (size_t v = 0; v < t.pieces.size(); ++v) {
      const SharePiece& s = t.pieces[v];
      if (s.ns != 1) continue;
      at[v] = ++end;
      p->node[end] = ShareNode{s.t0, s.t1, s.slot, s.s0, 1, s.parent < 0 ? -1 : at[s.parent], 0, 0, 0, -1};
    }
  *n_leaves = end - p->n_nodes;
  for (size_t i = 0; i < t.leaf.size(); ++i) p->leaf[i] = at[t.leaf[i]];

  // units and rows for a given quota
  auto lay = [&](int64_t quota, int64_t* units, int64_t* rows) {
    *units = *rows = 0;
    for (int v = 0; v < p->n_nodes; ++v) {
      ShareNode& nd = p->node[v];
      const int64_t tiles = ((int64_t)nd.t1 - nd.t0 + p->tile_keys - 1) / p->tile_keys;
      const int64_t chunks = ((int64_t)nd.ns * p->group + p->row_chunk - 1) / p->row_chunk;
      int64_t len = tiles + p->item_units;
      if (chunks > 1 && len > 2 * quota) {
        len = (len + quota - 1) / quota * quota;
        *units = (*units + quota - 1) / quota * quota;
      }
      if (*units + len * Hkv * chunks > (1 << 30)) return false;
      nd.unit0 = (int32_t)*units;
      nd.item_len = (int32_t)len;
      *units += len * Hkv * chunks;
      nd.max_segs = (int32_t)((tiles + quota - 2) / quota + 1);
      nd.row0 = (int32_t)std::min<int64_t>(*rows, INT32_MAX);
      *rows += (int64_t)nd.ns * p->n_q_heads * nd.max_segs;
    }
    p->node[p->n_nodes].unit0 = (int32_t)*units;
    return true;
  };
  int64_t units, rows;
  if (!lay(INT32_MAX, &units, &rows)) return false;
  int64_t quota = std::max<int64_t>((units + max_ctas - 1) / max_ctas, p->item_units + 1);
  for (int step = 0; step < 1000; ++step) {
    if (!lay(quota, &units, &rows)) return false;
    if ((units + quota - 1) / quota <= max_ctas && rows <= room) {
      p->quota = (int32_t)quota;
      p->n_ctas = (int32_t)((units + quota - 1) / quota);
      return true;
    }
    quota += 1 + (rows > room ? quota / 4 : quota / 64);
    if (quota > (1 << 30)) break;
  }
  return false;
}

// SMs that are left to the split pass of the sequences' own keys: the two kernels run side by side, and their
// shares follow what each has to do, in microseconds of an SM as measured: the split pass 1.0 for 128 keys and 3
// for an item (64 one-token items on four CTAs: 53 us), the tensor-core kernel 1.5 for a tile of few rows (its
// bytes), 1.75 for one of many (its products) and 4 for an item.
struct SharedCost {
  double own = 0, common = 0;   // per KV head
};
static SharedCost shared_cost(const ShareTree& t, const SharedDecodeParams& p, const DecodeParams& d, double few_rows, double many_rows) {
  SharedCost c;
  for (const SharePiece& s : t.pieces) {
    const double tiles = (s.t1 - s.t0) / 128.0;
    if (s.ns == 1) {
      c.own += (tiles + 3.0) * d.head_chunks;
    } else {
      const int rows = s.ns * p.group, chunks = (rows + p.row_chunk - 1) / p.row_chunk;
      c.common += (tiles * (rows > 64 ? many_rows : few_rows) + 4.0) * chunks;
    }
  }
  return c;
}
static int own_key_ctas(const ShareTree& t, const SharedDecodeParams& p, const DecodeParams& d, int sm_count) {
  const SharedCost c = shared_cost(t, p, d, 1.5, 1.75);
  if (c.own == 0) return 0;
  return std::min((int)(sm_count * c.own / (c.own + c.common)) + 1, sm_count - 1);
}

// Whether sharing pays: an estimate of either way in microseconds, from what either has to do.  The ordinary decode is
// not bound by the bytes (what the sequences have in common comes from L2) but by its keys: 19000 (quantised 28000) keys
// of a KV head per microsecond over all SMs, in rounds of an item per SM, all of a round as long as its items are.
// The shared one costs its pieces, as above (a quantised tile 2.3), and three launches, which together with the
// plan take the host 16 and a tenth per sequence.  Measured both ways at 504 points (2 to 64 sequences behind 512 to
// 32k tokens, nine layouts, 64 and 512 own tokens), calls that take the slower way: by more than 4 % in GPU or
// wall time, 1 shared (5 %); by more than 10 % in both, 12 ordinary (up to 28 %, one with less than 56 MB to save 75).
// With the bytes saved as the only measure, 39 (up to twice the time) and 7.  16 sequences behind 1k tokens of 8 heads
// x 128 (63 MB saved, but of 4 MB): 17.6 us shared, 11.3 ordinary; 8 behind 8k: 18.7 and 47.
static bool worth_sharing(const mixattn_ctx* c, int layer, int nb, const int32_t* ids, const ShareTree& t, const SharedDecodeParams& p,
                          ShapedDecodeParams* d) {
  bool any = false;
  d->partial = 0;
  plan_splits(c, layer, ids, nb, d, &any);
  int64_t keys = 0;
  int32_t longest = 0;
  for (int j = 0; j < nb; ++j) {
    keys += d->n_eff[j];
    longest = std::max(longest, d->chunk_len[j]);
  }
  const bool fp8 = c->geom.fp8 != 0;
  const int sms = c->sm_count, items = d->total_items;
  double work = (double)keys * c->cfg.n_kv_heads * d->head_chunks;
  if (!(items > sms && items <= 2 * sms && longest <= 2048))   // (those run two to an SM, in one round)
    work *= (double)((items + sms - 1) / sms) * sms / items;
  const double ordinary = 2.5 + work / (fp8 ? 28000.0 : 19000.0);
  const SharedCost cost = fp8 ? shared_cost(t, p, *d, 2.3, 2.3) : shared_cost(t, p, *d, 1.5, 1.75);
  const double shared = (fp8 ? 14.0 : 11.5) + (cost.own + cost.common) * c->cfg.n_kv_heads / sms;
  return ordinary > std::max(shared, 16.0 + 0.1 * nb);
}

// The keys that only one sequence has, as a launch of the ordinary split pass: each sequence with its block
// table from its first own page on, the longest ones first (the CTAs take the items in turns: 64
// sequences of 16 to 2048 own tokens in the caller's order kept some CTAs busy for 70 us and others for 39).
// Completes the nodes behind p's items.
static void plan_own_keys(const mixattn_ctx* c, int layer, int n_leaves, SharedDecodeParams* p, ShapedDecodeParams* d) {
  ShareNode* leaf = p->node + p->n_nodes + 1;
  int32_t by_length[kMaxCallSeqs];
  int64_t total = 0;
  for (int v = 0; v < n_leaves; ++v) {
    by_length[v] = v;
    total += leaf[v].t1 - leaf[v].t0;
  }
  std::sort(by_length, by_length + n_leaves, [&](int a, int b) {
    const int na = leaf[a].t1 - leaf[a].t0, nb = leaf[b].t1 - leaf[b].t0;
    return na != nb ? na > nb : a < b;
  });
  d->n_seqs = n_leaves;
  d->total_items = 0;
  if (n_leaves == 0) return;
  for (int i = 0; i < n_leaves; ++i) {
    const ShareNode& nd = leaf[by_length[i]];
    d->q_row[i] = p->order[nd.s0];
    d->seq_id[i] = nd.slot * p->table_stride + nd.t0 / kPage;   // (a table's entries are indexed in 32 bits)
    d->n_eff[i] = nd.t1 - nd.t0;
    d->newest[i] = p->newest[nd.s0] - nd.t0;
  }
  bool any = false;
  cut_splits(c, layer, n_leaves, total, d, &any);
  for (int i = 0; i < n_leaves; ++i) {
    leaf[by_length[i]].row0 = d->chunk_base[i];
    leaf[by_length[i]].max_segs = -(d->chunk_base[i + 1] - d->chunk_base[i]);
  }
}

static int decode_shared_impl(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, const void* q,
                              void* out, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0) return MIXATTN_ERR_INVALID_ARG;
  if (n_seqs > 0 && (seq_ids == nullptr || q == nullptr || out == nullptr)) return MIXATTN_ERR_INVALID_ARG;
  for (int i = 0; i < n_seqs; ++i)
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
  for (int i = 0; i < n_seqs; ++i)
    if (c->cm.len(layer, seq_ids[i]) < 1) return MIXATTN_ERR_EMPTY_CONTEXT;
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  // (nothing to share, or tensors that the wide accesses of these kernels cannot take)
  const bool tc = c->cfg.dtype == MIXATTN_BF16;
  if (n_seqs < 2 || c->cm.layer(layer).kind == MIXATTN_SLIDING || (((size_t)q | (size_t)out) & 15) != 0 || (tc && !shared_tc_supported(c->geom)))
    return decode_plain(c, layer, n_seqs, seq_ids, q, out, stream);
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim;
  const size_t row_bytes = (size_t)Hq * D * c->geom.elem_bytes;
  try {
    ShareTree tree;
    SharedDecodeParams p;
    ShapedDecodeParams d;
    p.pool = c->owner_storage(layer);
    p.table = c->dev_table();
    p.table_stride = c->cm.max_blocks();
    p.n_pages = c->cm.n_pages();
    p.geom = c->geom;
    p.n_q_heads = Hq;
    p.group = Hq / Hkv;
    p.scale_log2e = c->scale * kLog2e;
    p.split_o = reinterpret_cast<float*>(c->arena + c->plan.part_o_off);
    p.split_ml = reinterpret_cast<float2*>(c->arena + c->plan.part_ml_off);   // (tensor cores: set below)
    p.status = c->dev_status();
    p.shaped = score_shape_of(c, layer, &p.shape) ? 1 : 0;
    int64_t room;
    if (tc) {
      shared_tc_tiles(&p);
      const int64_t own_rows = (int64_t)kOwnChunks * Hq;
      char* own = c->arena + c->plan.part_o_off;
      char* shared = own + rows_bytes(own_rows, D);
      room = c->shared_room;
      p.split_ml = reinterpret_cast<float2*>(own + align_up((size_t)own_rows * D * sizeof(float)));
      p.part_o = reinterpret_cast<float*>(shared);
      p.part_ml = reinterpret_cast<float2*>(shared + align_up((size_t)room * D * sizeof(float)));
      d.pool = p.pool;
      d.table = p.table;
      d.table_stride = 1;
      d.ring_pages = 0;
      d.geom = c->geom;
      d.n_q_heads = Hq;
      d.group = p.group;
      d.head_chunks = (p.group + kMaxGroupRows - 1) / kMaxGroupRows;
      d.scale_log2e = p.scale_log2e;
      d.part_o = const_cast<float*>(p.split_o);
      d.part_ml = const_cast<float2*>(p.split_ml);
      d.status = p.status;
      d.l2_keep_bytes = d.l2_pool_bytes = 0;
      d.wrap = 0;
      // (always the kernel of shaped scores, here without cap or bias where the layer has none: it clears
      // what earlier sequences left behind the last key)
      if (p.shaped) {
        d.shape = p.shape;
      } else {
        d.shape.pre = p.scale_log2e;
        d.shape.post = 0.f;
        d.shape.biased = 0;
      }
    } else {
      p.tile_keys = 32;
      p.row_chunk = 32;
      p.item_units = 1;
      p.part_o = const_cast<float*>(p.split_o);
      p.part_ml = const_cast<float2*>(p.split_ml);
      room = (int64_t)kWsChunks * Hq;
    }
    // (launches of kMaxCallSeqs sequences: a larger batch is cut in the caller's order)
    for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
      const int nb = std::min(n_seqs - i0, kMaxCallSeqs);
      const int32_t* ids = seq_ids + i0;
      const char* qb = static_cast<const char*>(q) + (size_t)i0 * row_bytes;
      char* ob = static_cast<char*>(out) + (size_t)i0 * row_bytes;
      bool fits = false;
      int n_leaves = 0;
      for (int32_t least = MIXATTN_MIN_SHARED_TOKENS; !fits; least *= 2) {   // (deep trees of short pieces: only the longer ones)
        build_share_tree(c->cm, layer, nb, ids, least, &tree);
        if (!tree.shared) break;
        if (tc) {   // worth it?  (fp32: always, 14.5 against 28.8 us at 200 tokens of 2 sequences)
          int64_t apart = 0;
          for (int j = 0; j < nb; ++j) apart += c->cm.len(layer, ids[j]);
          const int64_t saved = (apart - tree.tokens) * (c->geom.page_bytes / kPage);
          if (saved < (c->share_min_bytes < 0 ? MIXATTN_MIN_SAVED_BYTES : c->share_min_bytes)) break;
          if (c->share_min_bytes < 0 && !worth_sharing(c, layer, nb, ids, tree, p, &d)) break;
        }
        const int own_ctas = tc ? own_key_ctas(tree, p, d, c->sm_count) : 0;
        d.partial = own_ctas;
        fits = lay_out_shared(tree, tc, tc ? c->sm_count - own_ctas : 2 * c->sm_count, room, &p, &n_leaves);
        if (least > (1 << 29)) break;
      }
      if (!fits) {
        const int rc = decode_plain(c, layer, nb, ids, qb, ob, stream);
        if (rc != MIXATTN_OK) return rc;
        continue;
      }
      p.q = qb;
      p.out = ob;
      p.n_seqs = nb;
      for (int j = 0; j < nb; ++j) {
        p.order[j] = tree.order[j];
        p.newest[j] = c->cm.len(layer, ids[tree.order[j]]) - 1;
      }
      cudaError_t e = launch_recorded(c, MIXATTN_K_SHARED, st, [&] {
        return tc ? launch_decode_shared_tc(p, st) : launch_decode_shared(p, st);
      });
      if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
      if (tc) {
        // The split pass comes right behind the tensor-core kernel, and nothing may come between: it reads q, the table and
        // the pages without a wait of its own, which is sound because that kernel lets its dependents start only after
        // its own wait for everything ahead of it (and each way out of the split pass waits for that kernel's end, which the
        // merge relies on).
        plan_own_keys(c, layer, n_leaves, &p, &d);
        d.q = qb;
        d.out = nullptr;
        if (d.total_items > 0) {
          e = launch_recorded(c, MIXATTN_K_DECODE_FULL, st, [&] { return launch_split_pass(c, d, true, st); });
          if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
        }
      }
      e = launch_recorded(c, MIXATTN_K_MERGE, st, [&] { return launch_merge_shared(p, c->cfg.dtype, c->sm_count, st); });
      if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
    }
  } catch (const std::bad_alloc&) {
    return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

int mixattn_decode(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                   const void* q, void* out, void* stream) {
  return c != nullptr && c->prefix_sharing ? decode_shared_impl(c, layer, n_seqs, seq_ids, q, out, stream)
                                           : decode_plain(c, layer, n_seqs, seq_ids, q, out, stream);
}

int mixattn_decode_shared(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                          const void* q, void* out, void* stream) {
  return decode_shared_impl(c, layer, n_seqs, seq_ids, q, out, stream);
}

int mixattn_set_prefix_sharing(mixattn_ctx* c, int32_t enable) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  c->prefix_sharing = enable != 0;
  return MIXATTN_OK;
}

int mixattn_set_share_min_bytes(mixattn_ctx* c, int64_t bytes) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  c->share_min_bytes = bytes;
  return MIXATTN_OK;
}

int mixattn_get_distinct_tokens(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, int64_t* tokens) {
  if (c == nullptr || tokens == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0 || (n_seqs > 0 && seq_ids == nullptr))
    return MIXATTN_ERR_INVALID_ARG;
  int64_t sum = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
    sum += c->cm.n_attended(layer, seq_ids[i]);
  }
  if (c->cm.layer(layer).kind == MIXATTN_FULL) {
    try {
      ShareTree tree;
      sum = 0;
      for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
        build_share_tree(c->cm, layer, std::min(n_seqs - i0, kMaxCallSeqs), seq_ids + i0, MIXATTN_MIN_SHARED_TOKENS, &tree);
        sum += tree.tokens;
      }
    } catch (const std::bad_alloc&) {
      return MIXATTN_ERR_CUDA;
    }
  }
  *tokens = sum;
  return MIXATTN_OK;
}

int mixattn_decode_layers(mixattn_ctx* c, int32_t layer_begin, int32_t layer_end, int32_t n_seqs,
                          const int32_t* seq_ids, const void* const* q, const void* const* k,
                          const void* const* v, void* const* out, void* stream, int32_t* layers_done) {
  if (layers_done != nullptr) *layers_done = 0;
  if (c == nullptr || layer_begin < 0 || layer_end < layer_begin || layer_end > c->cm.n_layers())
    return MIXATTN_ERR_INVALID_ARG;
  if (layer_end > layer_begin && (q == nullptr || out == nullptr || k == nullptr || v == nullptr))
    return MIXATTN_ERR_INVALID_ARG;
  for (int l = layer_begin; l < layer_end; ++l) {
    if (c->cm.layer(l).owner == l) {
      int rc = append_impl(c, l, n_seqs, seq_ids, nullptr, k[l], v[l], stream, 0.0);
      if (rc != MIXATTN_OK) return rc;
    }
    int rc = mixattn_decode(c, l, n_seqs, seq_ids, q[l], out[l], stream);
    if (rc != MIXATTN_OK) return rc;
    if (layers_done != nullptr) *layers_done = l - layer_begin + 1;
  }
  return MIXATTN_OK;
}

int mixattn_prefill(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                    const int32_t* seq_lens, const void* q, const void* k, const void* v,
                    void* out, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0) return MIXATTN_ERR_INVALID_ARG;
  if (n_seqs > 0 && (seq_ids == nullptr || seq_lens == nullptr)) return MIXATTN_ERR_INVALID_ARG;
  const LayerInfo& li = c->cm.layer(layer);
  const bool owner = li.owner == layer;
  int64_t total = 0;
  int max_len = 0;
  {
    std::vector<char> seen(c->cm.max_seqs(), 0);
    for (int i = 0; i < n_seqs; ++i) {
      if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
      if (seen[seq_ids[i]]) return MIXATTN_ERR_INVALID_ARG;
      seen[seq_ids[i]] = 1;
      if (seq_lens[i] < 1) return MIXATTN_ERR_INVALID_ARG;
      total += seq_lens[i];
      if (seq_lens[i] > max_len) max_len = seq_lens[i];
    }
  }
  if (total > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
  if (owner) {
    for (int i = 0; i < n_seqs; ++i)
      if (c->cm.len(layer, seq_ids[i]) != 0) return MIXATTN_ERR_UNSUPPORTED;
    int rc = c->cm.check_append(layer, n_seqs, seq_ids, seq_lens);
    if (rc != MIXATTN_OK) return rc;
  }
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_seqs == 0) return MIXATTN_OK;
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr) return MIXATTN_ERR_INVALID_ARG;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim;
  const size_t esz = c->geom.elem_bytes;
  PrefillParams p;
  ScoreShape shape;
  if (score_shape_of(c, layer, &shape)) p.shape = &shape;
  p.n_q_heads = Hq;
  p.n_kv_heads = Hkv;
  p.head_dim = D;
  p.window = li.kind == MIXATTN_SLIDING ? li.window : 0;
  p.scale_log2e = c->scale * kLog2e;
  p.status = c->dev_status();
  int64_t row = 0;
  for (int i0 = 0; i0 < n_seqs; i0 += kMaxCallSeqs) {
    const int nb = n_seqs - i0 < kMaxCallSeqs ? n_seqs - i0 : kMaxCallSeqs;
    int r = 0, mlen = 0;
    for (int j = 0; j < nb; ++j) {
      p.row0[j] = r;
      p.krow0[j] = r;
      p.prefix[j] = 0;
      r += seq_lens[i0 + j];
      if (seq_lens[i0 + j] > mlen) mlen = seq_lens[i0 + j];
    }
    p.row0[nb] = r;
    p.n_seqs = nb;
    p.q = static_cast<const char*>(q) + (size_t)row * Hq * D * esz;
    p.out = static_cast<char*>(out) + (size_t)row * Hq * D * esz;
    p.k = static_cast<const char*>(k) + (size_t)row * Hkv * D * esz;
    p.v = static_cast<const char*>(v) + (size_t)row * Hkv * D * esz;
    row += r;
    const int cls = p.window ? MIXATTN_K_PREFILL_SLIDING : MIXATTN_K_PREFILL_FULL;
    // bf16 runs on the tensor-core kernel, fp32 mode on the exact CUDA-core kernel
    const bool tc = prefill_tc_supported(c->cfg.dtype, D, p.q, p.k, p.v) && (((size_t)p.out) & 15) == 0;
    cudaError_t e = launch_recorded(c, cls, st, [&] {
      return tc ? launch_prefill_tc(p, mlen, c->sm_count, st) : launch_prefill_simple(p, c->cfg.dtype, mlen, st);
    });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
  }
  // The attention reads the caller's tensors, not the cache, so the cache is written after it:
  // the bookkeeping moves only once every attention launch (tensor maps included) has been
  // accepted.  A CUDA failure past this point leaves the context unusable (see the header).
  if (owner) {
    std::vector<int32_t> start(n_seqs, 0);
    std::vector<PageGrant> grants;
    c->cm.apply_append(layer, n_seqs, seq_ids, seq_lens, &grants);
    ++c->cache_epoch;
    int rc = enqueue_append(c, layer, n_seqs, seq_ids, seq_lens, start, grants, k, v, st);
    if (rc != MIXATTN_OK) return rc;
  }
  return MIXATTN_OK;
}

int mixattn_attend_chunk(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                         const int32_t* seq_lens, const void* q, const void* k, const void* v,
                         void* out, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0) return MIXATTN_ERR_INVALID_ARG;
  if (n_seqs > 0 && (seq_ids == nullptr || seq_lens == nullptr)) return MIXATTN_ERR_INVALID_ARG;
  const LayerInfo& li = c->cm.layer(layer);
  const bool ring = li.kind == MIXATTN_SLIDING;
  const int scratch = c->cfg.chunk_scratch_tokens;
  // cached keys each sequence's chunk needs: all of a paged cache, the last window - 1 of a ring
  std::vector<int32_t> n_prefix(n_seqs > 0 ? n_seqs : 0);
  {
    std::vector<char> seen(c->cm.max_seqs(), 0);
    int64_t total = 0;
    for (int i = 0; i < n_seqs; ++i) {
      if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
      if (seen[seq_ids[i]]) return MIXATTN_ERR_INVALID_ARG;
      seen[seq_ids[i]] = 1;
      if (seq_lens[i] < 1) return MIXATTN_ERR_INVALID_ARG;
      const int64_t n = c->cm.len(layer, seq_ids[i]);
      if (n + seq_lens[i] > c->cm.max_seq_len()) return MIXATTN_ERR_INVALID_ARG;
      total += seq_lens[i];
      n_prefix[i] = (int32_t)(ring ? (n < li.window - 1 ? n : li.window - 1) : n);
    }
    if (total > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;
  }
  if (scratch <= 0) return MIXATTN_ERR_UNSUPPORTED;
  for (int i = 0; i < n_seqs; ++i)
    if ((int64_t)n_prefix[i] + seq_lens[i] > scratch) return MIXATTN_ERR_TOO_LARGE;
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_seqs == 0) return MIXATTN_OK;
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr) return MIXATTN_ERR_INVALID_ARG;
  if ((((size_t)k) | ((size_t)v)) & 15) return MIXATTN_ERR_INVALID_ARG;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim;
  const size_t esz = c->geom.elem_bytes;
  char* ks = c->arena + c->plan.chunk_k_off;
  char* vs = c->arena + c->plan.chunk_v_off;

  GatherParams gp;
  gp.k_out = ks;
  gp.v_out = vs;
  gp.pool = c->owner_storage(layer);
  gp.table = c->dev_table();
  gp.table_stride = c->cm.max_blocks();
  gp.is_ring = ring;
  gp.window = ring ? li.window : 0;
  gp.ring_pages = ring ? ring_pages_of(li.window) : 0;
  gp.geom = c->geom;
  PrefillParams p;
  ScoreShape shape;
  if (score_shape_of(c, layer, &shape)) p.shape = &shape;
  p.n_q_heads = Hq;
  p.n_kv_heads = Hkv;
  p.head_dim = D;
  p.window = ring ? li.window : 0;
  p.scale_log2e = c->scale * kLog2e;
  p.status = c->dev_status();
  p.k = ks;
  p.v = vs;

  // The rows this call would copy are already in the scratch when the previous chunk call read
  // the same cache for the same sequences with the same chunk K/V, in one piece, on this stream,
  // and no cache has changed since (a reader layer right after its owner, or after another reader).
  bool one_piece = n_seqs <= kMaxCallSeqs;
  {
    int64_t rows = 0;
    for (int i = 0; i < n_seqs; ++i) rows += (int64_t)n_prefix[i] + seq_lens[i];
    one_piece = one_piece && rows <= scratch;
  }
  // A ring whose window is a whole number of key tiles is read where it is: a key tile of the
  // cached positions is eight consecutive pages of the sequence's ring, in the layout the tensor
  // cores take.  K / V of the chunk itself then come from the caller's tensors.
  const bool direct = ring && c->chunk_ring_direct && prefill_tc_ring_direct_supported(c->geom, li.window) &&
                      prefill_tc_supported(c->cfg.dtype, D, q, k, v) && (((size_t)out) & 15) == 0;
  mixattn_ctx::GatherKey dummy;
  mixattn_ctx::GatherKey& held = direct ? dummy : c->scratch_holds;
  const bool reuse = !direct && c->chunk_reuse && one_piece && held.valid && held.owner == li.owner &&
                     held.epoch == c->cache_epoch && held.k == k && held.v == v && held.st == st &&
                     held.ids.size() == (size_t)n_seqs &&
                     std::equal(held.ids.begin(), held.ids.end(), seq_ids) &&
                     std::equal(held.lens.begin(), held.lens.end(), seq_lens);
  if (!reuse) {
    held.valid = false;   // set again below, once the copy of a one-piece call has been issued
    held.owner = li.owner;
    held.epoch = c->cache_epoch;
    held.k = k;
    held.v = v;
    held.st = st;
    held.ids.assign(seq_ids, seq_ids + n_seqs);
    held.lens.assign(seq_lens, seq_lens + n_seqs);
  }

  // groups of consecutive sequences whose keys fit the scratch together; the stream orders
  // each group's attention before the next group's copy reuses the scratch
  int64_t row = 0;   // first chunk row of the group in q / k / v / out
  for (int i0 = 0; i0 < n_seqs;) {
    int nb = 0, mlen = 0, max_rows = 0;
    int32_t krow = 0, qrow = 0;
    while (i0 + nb < n_seqs && nb < kMaxCallSeqs) {
      const int i = i0 + nb;
      const int rows = n_prefix[i] + seq_lens[i];
      if (krow + rows > scratch) break;
      GatherEntry& e = gp.e[nb];
      e.seq = c->cm.slot(seq_ids[i]);
      e.n_prefix = n_prefix[i];
      e.pos0 = c->cm.len(layer, seq_ids[i]) - n_prefix[i];
      e.n_chunk = seq_lens[i];
      e.src_row0 = qrow;
      e.dst_row0 = krow;
      p.row0[nb] = qrow;
      p.krow0[nb] = direct ? qrow : krow;
      p.prefix[nb] = direct ? c->cm.len(layer, seq_ids[i]) : n_prefix[i];
      p.cached[nb] = p.prefix[nb];
      p.ring_page0[nb] = c->cm.slot(seq_ids[i]) * ring_pages_of(li.window);
      krow += rows;
      qrow += seq_lens[i];
      if (seq_lens[i] > mlen) mlen = seq_lens[i];
      if (rows > max_rows) max_rows = rows;
      ++nb;
    }
    p.row0[nb] = qrow;
    p.n_seqs = nb;
    gp.n_entries = nb;
    gp.k_chunk = static_cast<const char*>(k) + (size_t)row * Hkv * D * esz;
    gp.v_chunk = static_cast<const char*>(v) + (size_t)row * Hkv * D * esz;
    p.q = static_cast<const char*>(q) + (size_t)row * Hq * D * esz;
    p.out = static_cast<char*>(out) + (size_t)row * Hq * D * esz;
    if (direct) {
      p.k = gp.k_chunk;
      p.v = gp.v_chunk;
      p.ring_pool = gp.pool;
      p.ring_pages = gp.ring_pages;
      p.ring_total_pages = (int64_t)c->cm.max_seqs() * gp.ring_pages;
      p.geom = c->geom;
    }
    cudaError_t e = cudaSuccess;
    if (!reuse && !direct) {
      e = launch_recorded(c, MIXATTN_K_GATHER, st, [&] { return launch_gather(gp, max_rows, st); });
      if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
      held.valid = one_piece;
    }
    const int cls = p.window ? MIXATTN_K_PREFILL_SLIDING : MIXATTN_K_PREFILL_FULL;
    const bool tc = prefill_tc_supported(c->cfg.dtype, D, p.q, p.k, p.v) && (((size_t)p.out) & 15) == 0;
    if (direct && !tc) return MIXATTN_ERR_INVALID_ARG;   // (not reachable: the pointers were checked above)
    e = launch_recorded(c, cls, st, [&] {
      return tc ? launch_prefill_tc(p, mlen, c->sm_count, st) : launch_prefill_simple(p, c->cfg.dtype, mlen, st);
    });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
    row += qrow;
    i0 += nb;
  }
  return MIXATTN_OK;
}

int mixattn_get_len(mixattn_ctx* c, int32_t layer, int32_t seq, int32_t* len) {
  if (c == nullptr || len == nullptr || !c->cm.valid_layer(layer)) return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  *len = c->cm.len(layer, seq);
  return MIXATTN_OK;
}

int mixattn_get_stored(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids, int32_t* out) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0 || (n_seqs > 0 && (seq_ids == nullptr || out == nullptr)))
    return MIXATTN_ERR_INVALID_ARG;
  for (int i = 0; i < n_seqs; ++i)
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
  for (int i = 0; i < n_seqs; ++i) out[i] = c->cm.n_attended(layer, seq_ids[i]);
  return MIXATTN_OK;
}

int mixattn_get_block_table(mixattn_ctx* c, int32_t seq, int32_t* out, int32_t cap, int32_t* n_blocks) {
  if (c == nullptr || n_blocks == nullptr || cap < 0 || (cap > 0 && out == nullptr))
    return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  const int n = c->cm.n_blocks(seq);
  *n_blocks = n;
  const int m = n < cap ? n : cap;
  if (m > 0) memcpy(out, c->cm.table_row(seq), (size_t)m * sizeof(int32_t));
  return MIXATTN_OK;
}

int mixattn_get_n_free_pages(mixattn_ctx* c, int32_t* n_free) {
  if (c == nullptr || n_free == nullptr) return MIXATTN_ERR_INVALID_ARG;
  *n_free = c->cm.n_free();
  return MIXATTN_OK;
}

int mixattn_get_ring_state(mixattn_ctx* c, int32_t layer, int32_t seq, int32_t* next_slot, int32_t* n_valid) {
  if (c == nullptr || next_slot == nullptr || n_valid == nullptr || !c->cm.valid_layer(layer))
    return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  const LayerInfo& li = c->cm.layer(layer);
  if (li.kind != MIXATTN_SLIDING) return MIXATTN_ERR_INVALID_ARG;
  const int32_t n = c->cm.len(layer, seq);
  *next_slot = n % li.window;
  *n_valid = n < li.window ? n : li.window;
  return MIXATTN_OK;
}

int mixattn_locate(mixattn_ctx* c, int32_t layer, int32_t seq, int32_t pos, int32_t* page, int32_t* slot) {
  if (c == nullptr || page == nullptr || slot == nullptr || !c->cm.valid_layer(layer))
    return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  return c->cm.locate(layer, seq, pos, page, slot) ? MIXATTN_OK : MIXATTN_ERR_INVALID_ARG;
}

// Physical page (looked up in the DEVICE copy of the block table for a paged cache) and slot
// within it of a stored token; `slot` comes in as CacheManager::locate returned it.
static int stored_page_of(mixattn_ctx* c, int layer, int seq, int pos, int64_t* phys, int32_t* slot) {
  const LayerInfo& li = c->cm.layer(layer);
  if (li.kind == MIXATTN_FULL) {
    int32_t dev_page = -1;
    if (cudaMemcpy(&dev_page, c->dev_table() + (size_t)c->cm.slot(seq) * c->cm.max_blocks() + pos / kPage,
                   sizeof(int32_t), cudaMemcpyDeviceToHost) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
    *phys = dev_page;
  } else {
    *phys = (int64_t)c->cm.slot(seq) * ring_pages_of(li.window) + *slot / kPage;
    *slot = *slot % kPage;
  }
  return MIXATTN_OK;
}

// Copies one stored row (its 16-byte chunks put back in order) to `dst` (st_row_bytes bytes) and,
// for quantised storage, its shared exponent to *X.
static int read_stored_row(mixattn_ctx* c, const char* pool, int64_t phys, int gh, int which, int slot,
                           void* dst, int32_t* X) {
  const KvGeom& ge = c->geom;
  if (ge.fp8 && which == 1) {
    // quantised V is stored transposed: fetch the page's V^T and pick this token's column
    std::vector<unsigned char> vt((size_t)ge.head_dim * kPage);
    if (cudaMemcpy(vt.data(), pool + kv_fp8_v_offset(ge, phys, gh, 0, 0), vt.size(), cudaMemcpyDeviceToHost) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
    for (int d = 0; d < ge.head_dim; ++d) static_cast<unsigned char*>(dst)[d] = vt[(size_t)d * kPage + slot];
  } else {
    unsigned char row[512];
    if (ge.st_row_bytes > (int)sizeof(row)) return MIXATTN_ERR_UNSUPPORTED;
    // start of the stored row; its 16-byte chunks are permuted unless the cache is fp32
    const char* src = pool + phys * ge.page_bytes + (int64_t)gh * ge.blk_bytes +
                      (int64_t)(which * kPage + slot) * ge.st_row_bytes;
    if (cudaMemcpy(row, src, ge.st_row_bytes, cudaMemcpyDeviceToHost) != cudaSuccess) return MIXATTN_ERR_CUDA;
    const int chunks = ge.st_row_bytes / 16;
    for (int ch = 0; ch < chunks; ++ch) {
      const int phys_ch = !ge.swizzle ? ch : ge.fp8 ? (ch ^ fp8_k_swizzle(slot)) : (ch ^ (slot & 7));
      memcpy(static_cast<char*>(dst) + ch * 16, row + phys_ch * 16, 16);
    }
  }
  if (ge.fp8 && X != nullptr) {
    unsigned char xb = 0;
    if (cudaMemcpy(&xb, pool + kv_exp_offset(ge, phys, gh, which, slot), 1, cudaMemcpyDeviceToHost) != cudaSuccess)
      return MIXATTN_ERR_CUDA;
    *X = (int32_t)xb - 127;
  }
  return MIXATTN_OK;
}

// bf16 bit pattern of an E4M3 code times 2^X (host side of the debug read; the format is the
// OCP 8-bit float: exponent bias 7, subnormals m/8 * 2^-6, no infinity).
static uint16_t bf16_bits_of_e4m3(unsigned char code, int X) {
  const int e = (code >> 3) & 0xF, m = code & 7;
  float v = e == 0 ? ldexpf((float)m, -9) : ldexpf(1.0f + (float)m / 8.0f, e - 7);
  v = ldexpf(v, X);
  if (code & 0x80) v = -v;
  uint32_t bits;
  memcpy(&bits, &v, 4);
  return (uint16_t)(bits >> 16);   // exact: four significant bits
}

int mixattn_debug_read_kv(mixattn_ctx* c, int32_t layer, int32_t seq, int32_t pos, void* k_host, void* v_host) {
  if (c == nullptr || k_host == nullptr || v_host == nullptr || !c->cm.valid_layer(layer))
    return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  int32_t page, slot;
  if (!c->cm.locate(layer, seq, pos, &page, &slot)) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only) return MIXATTN_ERR_CUDA;
  DeviceGuard g(c->device);
  if (!g.ok || cudaDeviceSynchronize() != cudaSuccess) return MIXATTN_ERR_CUDA;
  const KvGeom& ge = c->geom;
  int64_t phys;
  if (stored_page_of(c, layer, seq, pos, &phys, &slot) != MIXATTN_OK) return MIXATTN_ERR_CUDA;
  const char* pool = c->owner_storage(layer);
  std::vector<unsigned char> codes(ge.st_row_bytes);
  for (int which = 0; which < 2; ++which) {
    char* dst = static_cast<char*>(which ? v_host : k_host);
    for (int gh = 0; gh < ge.n_kv_heads; ++gh) {
      if (!ge.fp8) {
        if (read_stored_row(c, pool, phys, gh, which, slot, dst + (size_t)gh * ge.row_bytes, nullptr) != MIXATTN_OK)
          return MIXATTN_ERR_CUDA;
        continue;
      }
      // quantised storage: element * 2^X, which is a bf16 number
      int32_t X = 0;
      if (read_stored_row(c, pool, phys, gh, which, slot, codes.data(), &X) != MIXATTN_OK) return MIXATTN_ERR_CUDA;
      uint16_t* out = reinterpret_cast<uint16_t*>(dst + (size_t)gh * ge.row_bytes);
      for (int d = 0; d < ge.head_dim; ++d) out[d] = bf16_bits_of_e4m3(codes[d], X);
    }
  }
  return MIXATTN_OK;
}

int mixattn_debug_read_kv_fp8(mixattn_ctx* c, int32_t layer, int32_t seq, int32_t pos, uint8_t* k_codes,
                              int32_t* k_exp, uint8_t* v_codes, int32_t* v_exp) {
  if (c == nullptr || k_codes == nullptr || k_exp == nullptr || v_codes == nullptr || v_exp == nullptr ||
      !c->cm.valid_layer(layer))
    return MIXATTN_ERR_INVALID_ARG;
  if (!c->cm.valid_seq(seq)) return MIXATTN_ERR_BAD_SEQ;
  if (!c->geom.fp8) return MIXATTN_ERR_UNSUPPORTED;
  int32_t page, slot;
  if (!c->cm.locate(layer, seq, pos, &page, &slot)) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only) return MIXATTN_ERR_CUDA;
  DeviceGuard g(c->device);
  if (!g.ok || cudaDeviceSynchronize() != cudaSuccess) return MIXATTN_ERR_CUDA;
  int64_t phys;
  if (stored_page_of(c, layer, seq, pos, &phys, &slot) != MIXATTN_OK) return MIXATTN_ERR_CUDA;
  const KvGeom& ge = c->geom;
  const char* pool = c->owner_storage(layer);
  for (int gh = 0; gh < ge.n_kv_heads; ++gh) {
    if (read_stored_row(c, pool, phys, gh, 0, slot, k_codes + (size_t)gh * ge.head_dim, &k_exp[gh]) != MIXATTN_OK ||
        read_stored_row(c, pool, phys, gh, 1, slot, v_codes + (size_t)gh * ge.head_dim, &v_exp[gh]) != MIXATTN_OK)
      return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

int mixattn_get_device_status(mixattn_ctx* c, int32_t* status) {
  if (c == nullptr || status == nullptr) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only) return MIXATTN_ERR_CUDA;
  DeviceGuard g(c->device);
  if (!g.ok || cudaDeviceSynchronize() != cudaSuccess) return MIXATTN_ERR_CUDA;
  if (cudaMemcpy(status, c->dev_status(), sizeof(int32_t), cudaMemcpyDeviceToHost) != cudaSuccess)
    return MIXATTN_ERR_CUDA;
  return MIXATTN_OK;
}

int mixattn_set_layer_scores(mixattn_ctx* c, int32_t layer, float softcap, const float* slopes) {
  if (c == nullptr || !c->cm.valid_layer(layer)) return MIXATTN_ERR_INVALID_ARG;
  if (!(softcap == 0.f || (softcap >= MIXATTN_SOFTCAP_MIN && softcap <= MIXATTN_SOFTCAP_MAX))) return MIXATTN_ERR_INVALID_ARG;
  if (softcap > 0.f && !isnormal(c->scale / softcap)) return MIXATTN_ERR_INVALID_ARG;
  const int Hq = c->cfg.n_q_heads;
  if (slopes != nullptr) {
    for (int h = 0; h < Hq; ++h)
      if (!(slopes[h] >= 0.f && slopes[h] <= MIXATTN_SLOPE_MAX)) return MIXATTN_ERR_INVALID_ARG;
    if (Hq > kMaxSlopeHeads) return MIXATTN_ERR_UNSUPPORTED;
  }
  try {
    LayerScores ls;
    ls.softcap = softcap;
    if (slopes != nullptr) ls.slopes.assign(slopes, slopes + Hq);
    c->scores[layer] = std::move(ls);
  } catch (const std::bad_alloc&) {
    return MIXATTN_ERR_INVALID_ARG;   // (as mixattn_create without host memory)
  }
  return MIXATTN_OK;
}

int mixattn_set_split_tokens(mixattn_ctx* c, int32_t tokens) {
  if (c == nullptr || tokens < 0) return MIXATTN_ERR_INVALID_ARG;
  c->split_tokens = tokens;
  return MIXATTN_OK;
}

int mixattn_set_chunk_gather_reuse(mixattn_ctx* c, int32_t enable) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  c->chunk_reuse = enable != 0;
  c->scratch_holds.valid = false;
  return MIXATTN_OK;
}

int mixattn_set_chunk_ring_direct(mixattn_ctx* c, int32_t enable) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  c->chunk_ring_direct = enable != 0;
  return MIXATTN_OK;
}

int mixattn_profile_enable(mixattn_ctx* c, int32_t enable) {
  if (c == nullptr) return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only) return MIXATTN_ERR_CUDA;
  for (auto& r : c->records) {
    if (r.start) c->event_pool.push_back(r.start);
    if (r.stop) c->event_pool.push_back(r.stop);
  }
  c->records.clear();
  c->profiling = enable != 0;
  return MIXATTN_OK;
}

int mixattn_profile_read(mixattn_ctx* c, int32_t cls, int32_t* launches, float* ms) {
  if (c == nullptr || launches == nullptr || ms == nullptr || cls < 0 || cls >= MIXATTN_K_COUNT)
    return MIXATTN_ERR_INVALID_ARG;
  if (c->host_only) return MIXATTN_ERR_CUDA;
  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  int n = 0;
  float total = 0.f;
  for (auto& r : c->records) {
    if (r.cls != cls || !r.start || !r.stop) continue;
    if (cudaEventSynchronize(r.stop) != cudaSuccess) return MIXATTN_ERR_CUDA;
    float t = 0.f;
    if (cudaEventElapsedTime(&t, r.start, r.stop) != cudaSuccess) return MIXATTN_ERR_CUDA;
    total += t;
    ++n;
  }
  *launches = n;
  *ms = total;
  return MIXATTN_OK;
}

// ---------------------------------------------------------------------------
// Decode with the split-KV scratch in a static device array (no arena workspace used).
// ---------------------------------------------------------------------------
namespace {

constexpr size_t kStaticScratchBytes = MIXATTN_STATIC_SCRATCH_BYTES;
constexpr int kMaxDevices = 64;

// Lives in every GPU context that loads this library, until the process exits.
static __device__ __align__(256) unsigned char g_decode_scratch[kStaticScratchBytes];

// Device address of g_decode_scratch per device ordinal.  In host code the array's name
// is only a handle for the runtime; the address a kernel can use comes from
// cudaGetSymbolAddress, asked once per device with that device current.
// Contexts on several threads may make their first call at once: the slots are atomic (every
// thread that asks gets the same address, so a relaxed load / store is enough).  The address is
// kept until the process exits; it does not survive a cudaDeviceReset of that device.
std::atomic<void*> g_decode_scratch_ptr[kMaxDevices];

int static_scratch_for_current_device(int device, void** out) {
  if (device < 0 || device >= kMaxDevices) return MIXATTN_ERR_INVALID_ARG;
  void* ptr = g_decode_scratch_ptr[device].load(std::memory_order_relaxed);
  if (ptr == nullptr) {
    if (cudaGetSymbolAddress(&ptr, g_decode_scratch) != cudaSuccess || ptr == nullptr) return MIXATTN_ERR_CUDA;
    g_decode_scratch_ptr[device].store(ptr, std::memory_order_relaxed);
  }
  *out = ptr;
  return MIXATTN_OK;
}

}  // namespace

int mixattn_decode_static_scratch(mixattn_ctx* c, int32_t layer, int32_t n_seqs, const int32_t* seq_ids,
                                  const void* q, void* out, void* stream) {
  if (c == nullptr || !c->cm.valid_layer(layer) || n_seqs < 0) return MIXATTN_ERR_INVALID_ARG;
  if (n_seqs > 0 && (seq_ids == nullptr || q == nullptr || out == nullptr)) return MIXATTN_ERR_INVALID_ARG;
  for (int i = 0; i < n_seqs; ++i) {
    if (!c->cm.valid_seq(seq_ids[i])) return MIXATTN_ERR_BAD_SEQ;
  }
  for (int i = 0; i < n_seqs; ++i) {
    if (c->cm.len(layer, seq_ids[i]) < 1) return MIXATTN_ERR_EMPTY_CONTEXT;
  }
  if (c->host_only || c->sticky_cuda_error) return MIXATTN_ERR_CUDA;
  if (n_seqs == 0) return MIXATTN_OK;
  if (n_seqs > kMaxCallSeqs) return MIXATTN_ERR_TOO_LARGE;

  const LayerInfo& li = c->cm.layer(layer);
  const bool ring = li.kind == MIXATTN_SLIDING;
  const int Hq = c->cfg.n_q_heads, Hkv = c->cfg.n_kv_heads, D = c->cfg.head_dim;

  ShapedDecodeParams p;
  const bool shaped = score_shape_of(c, layer, &p.shape);
  if (shaped) set_distances(c, layer, seq_ids, n_seqs, &p);
  p.group = Hq / Hkv;
  p.head_chunks = (p.group + kMaxGroupRows - 1) / kMaxGroupRows;
  // the split plan of mixattn_decode (one function), so both calls add the partial results in
  // the same order and give the same bits
  bool any_split = false;
  const int base = plan_splits(c, layer, seq_ids, n_seqs, &p, &any_split);
  // scratch needed: per split and query head, D partial outputs + (max, sum)
  const size_t part_o_bytes = align_up((size_t)base * Hq * D * sizeof(float));
  const size_t need = part_o_bytes + (size_t)base * Hq * sizeof(float2);
  if (need > kStaticScratchBytes) return MIXATTN_ERR_TOO_LARGE;

  DeviceGuard g(c->device);
  if (!g.ok) return MIXATTN_ERR_CUDA;
  void* scratch = nullptr;
  int rc = static_scratch_for_current_device(c->device, &scratch);
  if (rc != MIXATTN_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  p.q = q;
  p.out = out;
  p.pool = c->owner_storage(layer);
  p.table = ring ? nullptr : c->dev_table();
  p.table_stride = c->cm.max_blocks();
  p.ring_pages = ring ? ring_pages_of(li.window) : 0;
  p.geom = c->geom;
  p.n_q_heads = Hq;
  p.scale_log2e = c->scale * kLog2e;
  set_l2_policy(c, layer, &p);
  // every partial slot that the combine pass reads is written by the split pass of the
  // same call first, so nothing in the array has to start at zero
  p.part_o = reinterpret_cast<float*>(scratch);
  p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(scratch) + part_o_bytes);
  p.status = c->dev_status();
  const int cls = ring ? MIXATTN_K_DECODE_SLIDING : MIXATTN_K_DECODE_FULL;
  cudaError_t e = launch_recorded(c, cls, st, [&] { return launch_split_pass(c, p, shaped, st); });
  if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
  if (any_split) {
    e = launch_recorded(c, MIXATTN_K_COMBINE, st, [&] { return launch_decode_combine(p, c->cfg.dtype, st); });
    if (e != cudaSuccess) return MIXATTN_ERR_CUDA;
  }
  return MIXATTN_OK;
}

int mixattn_get_launch_count(mixattn_ctx* c, int64_t* launches) {
  if (c == nullptr || launches == nullptr) return MIXATTN_ERR_INVALID_ARG;
  *launches = c->launches;
  return MIXATTN_OK;
}

const char* mixattn_strerror(int code) {
  switch (code) {
    case MIXATTN_OK: return "ok";
    case MIXATTN_ERR_INVALID_ARG: return "invalid argument";
    case MIXATTN_ERR_INVALID_LAYOUT: return "invalid layer layout";
    case MIXATTN_ERR_NOT_OWNER: return "layer reuses another layer's KV cache and takes no K/V";
    case MIXATTN_ERR_OUT_OF_PAGES: return "not enough free pages";
    case MIXATTN_ERR_EMPTY_CONTEXT: return "sequence has no cached token";
    case MIXATTN_ERR_BAD_SEQ: return "sequence id out of range";
    case MIXATTN_ERR_UNSUPPORTED: return "unsupported request";
    case MIXATTN_ERR_CUDA: return "CUDA error or host-only context";
    case MIXATTN_ERR_TOO_LARGE: return "request needs more scratch than the static array holds";
    default: return "unknown status";
  }
}

}  // extern "C"
