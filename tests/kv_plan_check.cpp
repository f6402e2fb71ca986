// Cuts a batch's work and prints the pieces as the device gets them, for test_kv_plan.py.
//   kv_plan_check group kv_heads causal_block row_block unit workers min_units max_units overhead rows,length ...
#include <cstdio>
#include <cstdlib>

#include "../paper_2512_04939_b200/csrc/kv_plan.h"

int main(int argc, char** argv) {
  using namespace lv;
  const int group = atoi(argv[1]), kv_heads = atoi(argv[2]), causal_block = atoi(argv[3]);
  const KvCut cut{atoi(argv[4]), atoi(argv[5]), atoi(argv[6]), atoi(argv[7]), atoi(argv[8]), atof(argv[9])};
  std::vector<KvSeq> seqs;
  std::vector<int> which;
  int row0 = 0;
  for (int i = 10; i < argc; ++i) {
    int rows = 0, len = 0;
    sscanf(argv[i], "%d,%d", &rows, &len);
    if (rows > 0) which.push_back((int)seqs.size());
    seqs.push_back(KvSeq{row0, rows, len, 0});
    row0 += rows;
  }
  const KvWork work = kv_cut(seqs, which, group, kv_heads, causal_block, cut);
  const std::vector<KvPiece> chain = kv_chain(work);
  printf("%d %zu %d %d\n", work.workers(), chain.size(), work.slots, work.joins);
  for (const KvPiece& p : chain)
    printf("%d %d %d %d %d %d %d %d %d %d %d\n", p.seq.row0, p.kv_head, p.row0, p.rows, p.key0, p.key1, p.slot, p.first_slot, p.parts, p.join,
           p.next);
  for (const KvSeq& q : seqs)
    for (int t = 0; t < q.rows; ++t) printf("%d%c", kv_seen(q.len, q.rows, causal_block, t), t + 1 < q.rows ? ' ' : '\n');
  return 0;
}
