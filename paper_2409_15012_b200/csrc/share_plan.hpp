// The tree of shared prefixes behind a decode call (mixattn_decode_shared), from the block tables.
//
// A fork shares pages, and only whole rows from block 0 on: two rows that hold the same page in the same place hold the
// same pages in front of it too (a row changes by appending fresh pages behind its end or by being
// cut and taking over another row's continuation after equal blocks).  So the common prefix of two rows is found
// by bisection, and sorting the rows puts sequences with a common prefix next to each other.  Host
// code only; the cache itself is not looked at.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

#include "cache_manager.hpp"

namespace mixattn {

struct SharePiece {
  int32_t t0, t1, slot, s0, ns, parent;
};
struct ShareTree {
  std::vector<int32_t> order;        // sequences in tree order: index into the call's list
  std::vector<int32_t> leaf;         // per sequence in tree order: its last piece
  std::vector<SharePiece> pieces;    // a piece comes after its parent
  bool shared = false;               // some piece has several sequences
  int64_t rows = 0;                  // sum of ns over the pieces
  int64_t tokens = 0;                // sum of their lengths: the distinct keys of the call
};

// Tokens that two sequences have in common in the cache of `layer` (a paged one).
inline int32_t common_tokens(const CacheManager& cm, int layer, int a, int b) {
  const int32_t na = cm.len(layer, a), nb = cm.len(layer, b), least = std::min(na, nb);
  if (cm.slot(a) == cm.slot(b)) return least;
  const int32_t *ra = cm.table_row(a), *rb = cm.table_row(b);
  int32_t lo = 0, hi = (least + CacheManager::kPageSize - 1) / CacheManager::kPageSize;   // blocks [0, lo) agree, the answer is in [lo, hi]
  if (hi > 0 && ra[hi - 1] == rb[hi - 1]) return least;
  while (lo < hi) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (ra[mid] == rb[mid]) lo = mid + 1; else hi = mid;
  }
  return std::min(least, lo * CacheManager::kPageSize);
}

// Pieces shorter than min_tokens are not cut off for several sequences: each reads them itself.
inline void build_share_tree(const CacheManager& cm, int layer, int n, const int32_t* ids, int32_t min_tokens, ShareTree* t) {
  t->order.resize(n);
  t->leaf.assign(n, -1);
  t->pieces.clear();
  t->shared = false;
  t->rows = t->tokens = 0;
  for (int i = 0; i < n; ++i) t->order[i] = i;
  auto less = [&](int x, int y) {
    const int a = ids[x], b = ids[y];
    const int32_t na = cm.len(layer, a), nb = cm.len(layer, b);
    if (na == 0 || nb == 0) return na < nb;
    const int32_t *ra = cm.table_row(a), *rb = cm.table_row(b);
    if (ra[0] != rb[0]) return ra[0] < rb[0];
    const int32_t c = common_tokens(cm, layer, a, b);
    if (c == std::min(na, nb)) return na < nb;
    const int32_t blk = c / CacheManager::kPageSize;   // (the rows part at a whole block)
    return ra[blk] < rb[blk];
  };
  std::stable_sort(t->order.begin(), t->order.end(), less);
  std::vector<int32_t> common(n, 0);   // with the sequence in front
  for (int i = 1; i < n; ++i) common[i] = common_tokens(cm, layer, ids[t->order[i - 1]], ids[t->order[i]]);

  struct Range { int lo, hi; int32_t from, parent; };
  std::vector<Range> todo{{0, n, 0, -1}};
  while (!todo.empty()) {
    const Range r = todo.back();
    todo.pop_back();
    if (r.hi <= r.lo) continue;
    int32_t upto = cm.len(layer, ids[t->order[r.lo]]);   // of one sequence: its end
    for (int i = r.lo + 1; i < r.hi; ++i) upto = std::min(upto, common[i]);
    const int ns = r.hi - r.lo;
    int32_t from = r.from, parent = r.parent;
    if (upto > from && (ns == 1 || upto - from >= min_tokens)) {
      parent = (int32_t)t->pieces.size();
      t->pieces.push_back(SharePiece{from, upto, cm.slot(ids[t->order[r.lo]]), r.lo, ns, r.parent});
      t->shared = t->shared || ns > 1;
      t->rows += ns;
      t->tokens += upto - from;
      for (int i = r.lo; i < r.hi; ++i) t->leaf[i] = parent;
      from = upto;
    }
    if (ns == 1) continue;
    // split where the common prefix ends; what is left of the range is no shorter than before only in keys
    int first = r.lo;
    for (int i = r.lo + 1; i <= r.hi; ++i)
      if (i == r.hi || common[i] <= upto) {
        todo.push_back(Range{first, i, from, parent});
        first = i;
      }
  }
}

}  // namespace mixattn
