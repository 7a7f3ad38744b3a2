// Host-side KV-cache bookkeeping: layout resolution, the FIFO page allocator, block
// tables, ring positions and per-owner length counters.  Pure C++ (no CUDA): the host
// copy is authoritative, the device only mirrors the block tables.
//
// Paper, Section 3: a layer either computes its own KV cache or reuses the cache of an
// earlier layer; a sliding-window cache keeps the past `window` tokens.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <deque>
#include <vector>

#include "mixattn.h"

namespace mixattn {

struct LayerInfo {
  int32_t kind;
  int32_t window;
  int32_t owner;       // layer whose cache this layer reads
  int32_t owner_slot;  // index of that owner among owners (storage handle)
};

struct PageGrant {     // a block-table entry set during an append
  int32_t seq;
  int32_t block;
  int32_t page;
};

// What a fork has to move on the device for one copy that could not simply take over its
// source's slot.  Blocks [0, n_shared) of the source's block table are shared (their pages gain
// a reference); of those, the first `same` were in the slot's row already (copies of one prompt
// mostly differ in their last pages).  The blocks from n_shared on, which an append may still
// write to, are copied: pages tail0 .. tail0 + n_tail - 1 of the plan.
struct ForkCopy {
  int32_t src_slot, dst_slot;
  int32_t same, n_shared;
  int32_t tail0, n_tail;
};
struct ForkPlan {
  std::vector<ForkCopy> copies;
  std::vector<int32_t> src_pages, dst_pages;
};

class CacheManager {
 public:
  static constexpr int kPageSize = 16;

  // Validates the config; returns MIXATTN_OK or an error code (then *this is unusable).
  // `allocate` false: only resolve the layout and sizes (for the byte-count queries).
  int init(const mixattn_config& cfg, bool allocate = true) {
    if (cfg.n_layers <= 0 || cfg.layers == nullptr) return MIXATTN_ERR_INVALID_LAYOUT;
    if (cfg.n_q_heads <= 0 || cfg.n_kv_heads <= 0 || cfg.n_q_heads % cfg.n_kv_heads != 0)
      return MIXATTN_ERR_INVALID_ARG;
    if (cfg.head_dim != 64 && cfg.head_dim != 128) return MIXATTN_ERR_INVALID_ARG;
    if (cfg.dtype != MIXATTN_F32 && cfg.dtype != MIXATTN_BF16) return MIXATTN_ERR_INVALID_ARG;
    if (cfg.page_size != kPageSize || cfg.max_seqs <= 0 || cfg.n_pages < 0 || cfg.max_seq_len < 0)
      return MIXATTN_ERR_INVALID_ARG;
    layers_.clear();
    owners_.clear();
    for (int l = 0; l < cfg.n_layers; ++l) {
      const mixattn_layer_desc& d = cfg.layers[l];
      if (d.kind != MIXATTN_FULL && d.kind != MIXATTN_SLIDING) return MIXATTN_ERR_INVALID_LAYOUT;
      if (d.kind == MIXATTN_SLIDING && d.window < 1) return MIXATTN_ERR_INVALID_LAYOUT;
      if (d.kv_owner_layer < 0 || d.kv_owner_layer > l) return MIXATTN_ERR_INVALID_LAYOUT;
      const mixattn_layer_desc& o = cfg.layers[d.kv_owner_layer];
      if (o.kv_owner_layer != d.kv_owner_layer) return MIXATTN_ERR_INVALID_LAYOUT;
      if (o.kind != d.kind) return MIXATTN_ERR_INVALID_LAYOUT;
      if (d.kind == MIXATTN_SLIDING && o.window != d.window) return MIXATTN_ERR_INVALID_LAYOUT;
      layers_.push_back(LayerInfo{d.kind, d.kind == MIXATTN_SLIDING ? d.window : 0, d.kv_owner_layer, -1});
    }
    for (int l = 0; l < cfg.n_layers; ++l) {
      if (layers_[l].owner == l) {
        layers_[l].owner_slot = (int32_t)owners_.size();
        owners_.push_back(l);
      }
    }
    for (auto& li : layers_) li.owner_slot = layers_[li.owner].owner_slot;
    n_full_owners_ = 0;
    for (int o : owners_) n_full_owners_ += layers_[o].kind == MIXATTN_FULL;
    max_seqs_ = cfg.max_seqs;
    n_pages_ = cfg.n_pages;
    int64_t cap = (int64_t)cfg.n_pages * kPageSize;
    int64_t msl = cfg.max_seq_len > 0 ? cfg.max_seq_len : cap;
    if (msl > INT32_MAX - kPageSize) return MIXATTN_ERR_INVALID_ARG;
    if (msl < 1) msl = 1;
    max_seq_len_ = (int32_t)msl;
    max_blocks_ = (max_seq_len_ + kPageSize - 1) / kPageSize;
    if ((int64_t)max_seqs_ * max_blocks_ > INT32_MAX) return MIXATTN_ERR_INVALID_ARG;   // table entries are indexed in 32 bits
    free_.clear();
    if (cfg.free_order) {
      std::vector<char> seen(cfg.n_pages, 0);
      for (int i = 0; i < cfg.n_pages; ++i) {
        int32_t pg = cfg.free_order[i];
        if (pg < 0 || pg >= cfg.n_pages || seen[pg]) return MIXATTN_ERR_INVALID_ARG;
        seen[pg] = 1;
        if (allocate) free_.push_back(pg);
      }
    } else if (allocate) {
      for (int i = 0; i < cfg.n_pages; ++i) free_.push_back(i);
    }
    if (allocate) {
      table_.assign((size_t)max_seqs_ * max_blocks_, -1);
      n_blocks_.assign(max_seqs_, 0);
      refs_.assign(n_pages_, 0);
      slot_.resize(max_seqs_);
      for (int i = 0; i < max_seqs_; ++i) slot_[i] = i;
      len_.assign(owners_.size() * (size_t)max_seqs_, 0);
    }
    return MIXATTN_OK;
  }

  int n_layers() const { return (int)layers_.size(); }
  const LayerInfo& layer(int l) const { return layers_[l]; }
  const std::vector<int>& owners() const { return owners_; }
  int n_full_owners() const { return n_full_owners_; }
  int max_seqs() const { return max_seqs_; }
  int n_pages() const { return n_pages_; }
  int max_blocks() const { return max_blocks_; }
  int max_seq_len() const { return max_seq_len_; }
  int n_free() const { return (int)free_.size(); }
  bool valid_layer(int l) const { return l >= 0 && l < (int)layers_.size(); }
  bool valid_seq(int s) const { return s >= 0 && s < max_seqs_; }

  // Storage slot of a sequence: the row of the device block table and the ring of every
  // sliding-window owner that hold its tokens.  Lengths and tables are kept per slot, so that a
  // fork hands a sequence on by renaming its slot.
  int32_t slot(int seq) const { return slot_[seq]; }
  int32_t len(int layer, int seq) const {
    return len_[(size_t)layers_[layer].owner_slot * max_seqs_ + slot_[seq]];
  }
  int32_t slot_len(int owner_slot, int slot) const { return len_[(size_t)owner_slot * max_seqs_ + slot]; }
  int32_t n_blocks(int seq) const { return n_blocks_[slot_[seq]]; }
  const int32_t* table_row(int seq) const { return &table_[(size_t)slot_[seq] * max_blocks_]; }

  // Keys a decode of `layer` attends to for `seq`: all of them, or the last `window`.
  int32_t n_attended(int layer, int seq) const {
    int32_t n = len(layer, seq);
    const LayerInfo& li = layers_[layer];
    return li.kind == MIXATTN_SLIDING && n > li.window ? li.window : n;
  }

  // Checks an append call; nothing changes.
  int check_append(int layer, int n_seqs, const int32_t* seq_ids, const int32_t* n_new) const {
    if (!valid_layer(layer) || n_seqs < 0 || (n_seqs > 0 && seq_ids == nullptr))
      return MIXATTN_ERR_INVALID_ARG;
    const LayerInfo& li = layers_[layer];
    if (li.owner != layer) return MIXATTN_ERR_NOT_OWNER;
    std::vector<char> seen(max_seqs_, 0);
    int64_t need = 0;
    for (int i = 0; i < n_seqs; ++i) {
      int s = seq_ids[i];
      if (!valid_seq(s)) return MIXATTN_ERR_BAD_SEQ;
      if (seen[s]) return MIXATTN_ERR_INVALID_ARG;
      seen[s] = 1;
      int64_t n = n_new ? n_new[i] : 1;
      if (n < 0) return MIXATTN_ERR_INVALID_ARG;
      int64_t end = (int64_t)len(layer, s) + n;
      if (end > max_seq_len_) return MIXATTN_ERR_INVALID_ARG;
      if (li.kind == MIXATTN_FULL) {
        int64_t blocks = (end + kPageSize - 1) / kPageSize;
        if (blocks > n_blocks(s)) need += blocks - n_blocks(s);
      }
    }
    if (need > (int64_t)free_.size()) return MIXATTN_ERR_OUT_OF_PAGES;
    return MIXATTN_OK;
  }

  // Applies an append that check_append accepted.  Pages are popped from the FIFO head,
  // sequences in call order, blocks in position order; every new table entry is
  // reported in `grants`.
  void apply_append(int layer, int n_seqs, const int32_t* seq_ids, const int32_t* n_new,
                    std::vector<PageGrant>* grants) {
    const LayerInfo& li = layers_[layer];
    for (int i = 0; i < n_seqs; ++i) {
      const int s = slot_[seq_ids[i]];
      int32_t n = n_new ? n_new[i] : 1;
      int32_t& L = len_[(size_t)li.owner_slot * max_seqs_ + s];
      int32_t end = L + n;
      if (li.kind == MIXATTN_FULL) {
        int32_t blocks = (end + kPageSize - 1) / kPageSize;
        while (n_blocks_[s] < blocks) {
          const int32_t pg = take_page();
          table_[(size_t)s * max_blocks_ + n_blocks_[s]] = pg;
          if (grants) grants->push_back(PageGrant{seq_ids[i], n_blocks_[s], pg});
          ++n_blocks_[s];
        }
      }
      L = end;
    }
  }

  void seq_reset(int seq) { release_slot(slot_[seq]); }

  // Checks a fork call (see apply_fork) apart from the pages it needs; nothing changes.
  int check_fork(int n, const int32_t* src, const int32_t* dst) const {
    if (n < 0 || (n > 0 && (src == nullptr || dst == nullptr))) return MIXATTN_ERR_INVALID_ARG;
    std::vector<char> seen(max_seqs_, 0);
    for (int i = 0; i < n; ++i) {
      if (!valid_seq(src[i]) || !valid_seq(dst[i])) return MIXATTN_ERR_BAD_SEQ;
      if (seen[dst[i]]) return MIXATTN_ERR_INVALID_ARG;
      seen[dst[i]] = 1;
    }
    return MIXATTN_OK;
  }

  // Every dst[i] becomes what src[i] was before the call (all assignments at once).  A source
  // that the call overwrites hands its slot to its first copy; every other copy gets the slot of
  // an overwritten sequence without copies, shares the source's pages that are full in every
  // full-attention owner (no append writes to those any more) and takes fresh pages for the
  // rest.  Order of the page movements: the overwritten sequences' pages return to the FIFO
  // tail in call order, then the copies take theirs from its head in call order.
  // Returns MIXATTN_OK, or OUT_OF_PAGES with nothing changed.
  int apply_fork(int n, const int32_t* src, const int32_t* dst, ForkPlan* plan) {
    std::vector<int32_t> from(n), to(n, -1);              // slots before and after, per entry
    std::vector<char> held(max_seqs_, 0);                 // slots that keep their contents
    std::vector<char> overwritten(max_seqs_, 0);          // sequences the call replaces
    for (int i = 0; i < n; ++i) {
      from[i] = slot_[src[i]];
      overwritten[dst[i]] = src[i] != dst[i];
    }
    for (int i = 0; i < n; ++i)                           // sources that stay (or map to themselves)
      if (!overwritten[src[i]]) {
        held[from[i]] = 1;
        if (src[i] == dst[i]) to[i] = from[i];
      }
    for (int i = 0; i < n; ++i)                           // an overwritten source: its first copy takes over
      if (to[i] < 0 && !held[from[i]]) {
        held[from[i]] = 1;
        to[i] = from[i];
      }
    // slots whose contents die, in call order, and the copies that move in (one each): a copy stays
    // in the slot its sequence had where it can
    std::vector<int32_t> dead;
    for (int i = 0; i < n; ++i)
      if (!held[slot_[dst[i]]]) dead.push_back(slot_[dst[i]]);
    std::vector<char> taken(max_seqs_, 0);
    for (int i = 0; i < n; ++i)
      if (to[i] < 0 && !held[slot_[dst[i]]]) {
        to[i] = slot_[dst[i]];
        taken[to[i]] = 1;
      }
    size_t at = 0;
    for (int i = 0; i < n; ++i)
      if (to[i] < 0) {
        while (taken[dead[at]]) ++at;
        to[i] = dead[at++];
      }
    auto row = [&](int slot) { return &table_[(size_t)slot * max_blocks_]; };
    std::vector<int32_t> same(dead.empty() ? 0 : max_seqs_, 0);   // per dead slot
    size_t n_tails = 0;
    plan->copies.reserve(dead.size());
    for (int i = 0; i < n; ++i) {
      if (to[i] == from[i]) continue;
      ForkCopy c;
      c.src_slot = from[i];
      c.dst_slot = to[i];
      c.n_shared = n_shared(from[i]);
      const int most = c.n_shared < n_blocks_[to[i]] ? c.n_shared : n_blocks_[to[i]];
      c.same = (int32_t)(std::mismatch(row(from[i]), row(from[i]) + most, row(to[i])).first - row(from[i]));
      c.n_tail = n_blocks_[from[i]] - c.n_shared;
      c.tail0 = (int32_t)n_tails;
      n_tails += c.n_tail;
      same[to[i]] = c.same;
      plan->copies.push_back(c);
    }
    plan->src_pages.reserve(n_tails);
    plan->dst_pages.reserve(n_tails);
    // Shared pages gain their references before the dead slots lose theirs (a page both hold keeps
    // its count).  Only where the FIFO is short are the pages the dead slots free counted first, so
    // that a call that cannot be served changes nothing.
    auto share = [&](int by) {
      for (const ForkCopy& c : plan->copies)
        for (int b = c.same; b < c.n_shared; ++b) refs_[row(c.src_slot)[b]] += by;
    };
    share(1);
    if (n_tails > free_.size()) {
      size_t freed = 0;
      for (int s : dead)
        for (int b = same[s]; b < n_blocks_[s]; ++b) freed += --refs_[row(s)[b]] == 0;
      for (int s : dead)
        for (int b = same[s]; b < n_blocks_[s]; ++b) ++refs_[row(s)[b]];
      if (n_tails > free_.size() + freed) {
        share(-1);
        plan->copies.clear();
        return MIXATTN_ERR_OUT_OF_PAGES;
      }
    }
    for (int s : dead) release_slot(s, same[s]);
    for (const ForkCopy& c : plan->copies) {
      int32_t* to_row = row(c.dst_slot);
      const int32_t* from_row = row(c.src_slot);
      std::copy(from_row + c.same, from_row + c.n_shared, to_row + c.same);
      for (int b = c.n_shared; b < c.n_shared + c.n_tail; ++b) {
        plan->src_pages.push_back(from_row[b]);
        plan->dst_pages.push_back(to_row[b] = take_page());
      }
      n_blocks_[c.dst_slot] = c.n_shared + c.n_tail;
      for (size_t o = 0; o < owners_.size(); ++o) len_[o * max_seqs_ + c.dst_slot] = len_[o * max_seqs_ + c.src_slot];
    }
    for (int i = 0; i < n; ++i) slot_[dst[i]] = to[i];
    return MIXATTN_OK;
  }

  // Page and slot of a stored token; false if it is not stored (any more).
  bool locate(int layer, int seq, int pos, int32_t* page, int32_t* slot) const {
    const LayerInfo& li = layers_[layer];
    int32_t n = len(layer, seq);
    int32_t lo = li.kind == MIXATTN_SLIDING && n > li.window ? n - li.window : 0;
    if (pos < lo || pos >= n) return false;
    if (li.kind == MIXATTN_FULL) {
      *page = table_row(seq)[pos / kPageSize];
      *slot = pos % kPageSize;
    } else {
      *page = -1;
      *slot = pos % li.window;
    }
    return true;
  }

 private:
  // Blocks of a slot whose 16 tokens are stored in every full-attention owner.
  int n_shared(int slot) const {
    int n = n_blocks_[slot];
    for (size_t o = 0; o < owners_.size(); ++o)
      if (layers_[owners_[o]].kind == MIXATTN_FULL) {
        const int full = len_[o * max_seqs_ + slot] / kPageSize;
        if (full < n) n = full;
      }
    return n;
  }
  int32_t take_page() {
    const int32_t pg = free_.front();
    free_.pop_front();
    refs_[pg] = 1;
    return pg;
  }
  // Empties a slot from block `first` on; a page returns to the FIFO tail when its last reference goes.
  void release_slot(int slot, int first = 0) {
    for (size_t o = 0; o < owners_.size(); ++o) len_[o * max_seqs_ + slot] = 0;
    int32_t* row = &table_[(size_t)slot * max_blocks_];
    for (int b = first; b < n_blocks_[slot]; ++b) {
      if (--refs_[row[b]] == 0) free_.push_back(row[b]);
      row[b] = -1;
    }
    n_blocks_[slot] = first < n_blocks_[slot] ? first : n_blocks_[slot];
  }

  std::vector<LayerInfo> layers_;
  std::vector<int> owners_;
  int n_full_owners_ = 0;
  int max_seqs_ = 0, n_pages_ = 0, max_seq_len_ = 0, max_blocks_ = 0;
  std::deque<int32_t> free_;
  std::vector<int32_t> table_;
  std::vector<int32_t> n_blocks_;
  std::vector<int32_t> len_;        // per owner and slot
  std::vector<int32_t> refs_;       // block tables that hold the page
  std::vector<int32_t> slot_;       // storage slot of each sequence
};

}  // namespace mixattn
