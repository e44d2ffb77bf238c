// Prints what the rules of tree attention make of geometries given as "heads group nodes page stride
// sequences" on stdin: sequences a launch, and the stages that they have at most.
#include <stdio.h>

#include "cache_rules.h"

int main() {
  int heads, group, nodes, page, stride, seqs;
  while (scanf("%d %d %d %d %d %d", &heads, &group, &nodes, &page, &stride, &seqs) == 6) {
    dora_decode_desc d = {};
    d.num_seqs = seqs;
    d.num_q_heads = heads * group;
    d.num_kv_heads = heads;
    d.head_dim = 128;
    d.page_size = page;
    d.block_table_stride = stride;
    d.num_pages = 1;
    dora::TreeLayout t;
    dora::tree_layout(d, nodes, 256, &t);
    // as the kernels count them: full rows, all drafts, and the start of each segment
    const long long steps = ((long long)stride * page + 31) / 32 + (nodes + 31) / 32;
    const long long one = t.tiles == 1 ? (steps + 3) / 4 + dora::kTreeNarrowCost : steps + dora::kTreeWideCost;
    printf("%d %lld\n", t.seqs, one * t.blocks * heads * t.seqs);
  }
  return 0;
}
