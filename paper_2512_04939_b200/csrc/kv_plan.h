// How the work of a batch over a paged K/V cache is cut: which rows of which sequence meet which keys in which CTA.  Host
// arithmetic only; the batch's arrays are made here once and serve every call that is made with it.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

namespace lv {

// A sequence of a batch: its rows in the packed tensors, the tokens that it holds, where its pages begin in the batch's list.
struct KvSeq {
  int row0, rows, len, page0;
};

// Keys [key0, key1) of rows [row0, row0 + rows) of one sequence and K/V head.  The `group` query heads that share the head
// are rows of their own, side by side: row = token * group + head within the group.
// A worker is told one number, that of its first piece, which is its own, and finds everything else in the pieces: what a CTA has
// to read before its first load of keys is this and the page.
struct alignas(16) KvPiece {
  KvSeq seq;
  int kv_head, row0, rows, key0;
  int key1;
  int slot;        // where its partial rows go, -1: the rows have no other piece
  int first_slot;  // of all pieces of the same rows
  int parts;       // how many they are,
  int join;        // and the counter of those that have come
  int next;        // the worker's next piece, -1: none
  int pad[2];
};
static_assert(sizeof(KvPiece) == 64, "four loads of 16 bytes");

// Tokens that row `token` of a sequence's chunk sees; none if it is negative.
#ifdef __CUDACC__
__host__ __device__
#endif
inline int kv_seen(int len, int rows, int causal_block, int token) {
  if (causal_block == 0) return len;
  const long long end = (long long)len - rows + (long long)(token / causal_block + 1) * causal_block;
  return end < len ? (int)end : len;
}

struct KvWork {
  std::vector<KvPiece> pieces;
  std::vector<int> first;  // [workers + 1] a worker's pieces; every worker that is launched has one
  int slots = 0, joins = 0;
  double cost = 0.0;       // of the worker with the most to do, in units
  int workers() const { return first.empty() ? 0 : (int)first.size() - 1; }
};

// The pieces as the device gets them: worker w's first one is number w, the others lie behind.
inline std::vector<KvPiece> kv_chain(const KvWork& work) {
  const int workers = work.workers();
  std::vector<KvPiece> out((size_t)workers);
  for (int w = 0; w < workers; ++w) {
    size_t last = (size_t)w;
    for (int i = work.first[(size_t)w]; i < work.first[(size_t)w + 1]; ++i) {
      if (i == work.first[(size_t)w]) {
        out[last] = work.pieces[(size_t)i];
      } else {
        out[last].next = (int)out.size();
        last = out.size();
        out.push_back(work.pieces[(size_t)i]);
      }
      out[last].next = -1;
    }
  }
  return out;
}

// What a kernel needs from the cutting.
struct KvCut {
  int row_block;   // rows of one piece at most
  int unit;        // keys: pieces begin at multiples of it
  int workers;     // at most
  int min_units;   // of a piece where rows are cut
  int max_units;
  double overhead; // of a piece, in units
};

// Cost of a unit of `rows` rows: what fills less than half of the rows takes less than the full block, but not half.
inline double kv_unit_cost(const KvCut& cut, int rows) { return 2 * rows <= cut.row_block ? 0.65 : 1.0; }

// What a pass over the rows found: the last worker takes what is left when the others have their shares.
inline double kv_cut_by(double share, const std::vector<KvSeq>& seqs, const std::vector<int>& which, int group, int kv_heads,
                        int causal_block, const KvCut& cut, KvWork* out) {
  KvWork& work = *out;
  work = KvWork();
  double spent = 0.0;   // of all shares
  double begun = 0.0;   // when the present worker began
  int worker = 0;
  work.first.push_back(0);
  auto next_worker = [&]() {
    if (worker + 1 >= cut.workers || (size_t)work.first.back() == work.pieces.size()) return false;
    work.first.push_back((int)work.pieces.size());
    ++worker;
    work.cost = std::max(work.cost, spent - begun);
    begun = spent;
    return true;
  };
  for (int s : which) {
    const KvSeq& q = seqs[(size_t)s];
    const int all = q.rows * group;
    for (int h = 0; h < kv_heads; ++h)
      for (long long first = 0; first < all; first += cut.row_block) {  // (the end of the last block may lie beyond 32 bits)
        const int r = (int)first, n = std::min(cut.row_block, all - r);
        const int seen = std::max(kv_seen(q.len, q.rows, causal_block, (r + n - 1) / group), 0);
        const int units = (int)(((long long)seen + cut.unit - 1) / cut.unit);
        const double cost = kv_unit_cost(cut, n);
        const size_t begin = work.pieces.size();
        int done = 0;
        do {
          const double left = (worker + 1) * share - spent - cut.overhead;
          int take = left > 0.0 ? (int)std::min(left / cost, (double)units) : 0;
          if (worker + 1 >= cut.workers) take = units;
          if (take < std::min(cut.min_units, units - done) && next_worker()) continue;
          if (units - done - take < cut.min_units) take = units - done;  // no crumbs
          take = std::min(std::max(take, std::min(cut.min_units, units - done)), std::min(units - done, cut.max_units));
          KvPiece p{};
          p.seq = q; p.kv_head = h; p.row0 = r; p.rows = n;
          p.key0 = done * cut.unit;
          p.key1 = (int)std::min((long long)(done + take) * cut.unit, (long long)seen);
          p.slot = -1;
          work.pieces.push_back(p);
          done += take;
          spent += take * cost + cut.overhead;
        } while (done < units);
        const int parts = (int)(work.pieces.size() - begin);
        if (parts > 1) {
          for (size_t i = begin; i < work.pieces.size(); ++i) {
            work.pieces[i].slot = work.slots + (int)(i - begin);
            work.pieces[i].first_slot = work.slots;
            work.pieces[i].parts = parts;
            work.pieces[i].join = work.joins;
          }
          work.slots += parts;
          ++work.joins;
        }
      }
  }
  work.first.push_back((int)work.pieces.size());
  work.cost = std::max(work.cost, spent - begun);
  return spent - begun;
}

// Cuts the rows of the sequences in `which` into pieces.  All pieces in a row, every worker takes an equal share of what
// they cost, so a launch ends at the same time everywhere whatever the lengths; a share's border cuts the keys of the
// rows that it falls into.
inline KvWork kv_cut(const std::vector<KvSeq>& seqs, const std::vector<int>& which, int group, int kv_heads, int causal_block,
                     const KvCut& cut) {
  KvWork work;
  double total = 0.0;
  for (int s : which) {
    const KvSeq& q = seqs[(size_t)s];
    const int all = q.rows * group;
    double one_head = 0.0;
    for (long long first = 0; first < all; first += cut.row_block) {
      const int r = (int)first, n = std::min(cut.row_block, all - r);
      const int seen = std::max(kv_seen(q.len, q.rows, causal_block, (r + n - 1) / group), 0);
      one_head += (double)(((long long)seen + cut.unit - 1) / cut.unit) * kv_unit_cost(cut, n) + cut.overhead;
    }
    total += one_head * kv_heads;
  }
  if (total <= 0.0) return work;
  // How many pieces the borders make is known only afterwards: what the last worker has too much goes to all.
  double share = std::max(total / cut.workers + cut.overhead, cut.min_units + cut.overhead);
  for (int pass = 0; pass < 4; ++pass) {
    const double last = kv_cut_by(share, seqs, which, group, kv_heads, causal_block, cut, &work);
    if (last <= 1.02 * share) break;
    share += (last - share) / cut.workers + 0.002 * share;
  }
  return work;
}

}  // namespace lv
