// Cuts the work of one sequence of very many rows and prints how many pieces that makes, for test_kv_plan_large.py.
//   kv_plan_large_check rows length row_block workers
#include <cstdio>
#include <cstdlib>

#include "../paper_2512_04939_b200/csrc/kv_plan.h"

int main(int, char** argv) {
  using namespace lv;
  const KvCut cut{atoi(argv[3]), 128, atoi(argv[4]), 4, 512, 2.0};
  const std::vector<KvSeq> seqs{KvSeq{0, atoi(argv[1]), atoi(argv[2]), 0}};
  const KvWork work = kv_cut(seqs, {0}, 1, 1, 0, cut);
  long long rows = 0, units = 0;
  for (const KvPiece& p : work.pieces) rows += p.key0 == 0 ? p.rows : 0, units += (p.key1 - p.key0 + cut.unit - 1) / cut.unit;
  printf("%d %zu %lld %lld\n", work.workers(), work.pieces.size(), rows, units);
  return 0;
}
