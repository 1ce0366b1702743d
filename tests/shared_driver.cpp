// Prints the plan of a batch whose groups share prefixes: the records that a
// handle uploads, with the block ids of their ranges looked up as the kernels
// do, its merge records and its append units.
// Input: "nq nkv hd cu split_tile split_item share_all check R NG", then R lines "chunk context
// n_blocks id ...", then NG lines "first count prefix_len". check 1: check_shared only.
#include <algorithm>
#include <cstdio>
#include <vector>

#include "hb_plan.h"

using namespace hb;

int main() {
  hb_layer_config c{};
  int cu, all, check, n, ng;
  PlanOptions opt;
  if (scanf("%d %d %d %d %d %d %d %d %d %d", &c.n_q_heads, &c.n_kv_heads, &c.head_dim, &cu, &opt.split_tile,
            &opt.split_item, &all, &check, &n, &ng) != 10)
    return 2;
  opt.share_all = all;
  c.hidden = 64;
  c.ffn_dim = 16;
  c.kv_block_size = 16;
  c.rope_theta = 5e5f;
  c.max_batch_tokens = 1 << 16;
  c.max_requests = 1 << 16;
  Dims d;
  if (check_config(&c, &d) != HB_OK) return 3;
  std::vector<std::vector<int32_t>> tables(n);
  std::vector<hb_request> reqs(n);
  for (int r = 0; r < n; ++r) {
    if (scanf("%d %d %d", &reqs[r].chunk_len, &reqs[r].context_len, &reqs[r].n_blocks) != 3) return 4;
    tables[r].resize(reqs[r].n_blocks);
    for (int32_t& b : tables[r])
      if (scanf("%d", &b) != 1) return 5;
    reqs[r].block_table = tables[r].data();
  }
  std::vector<hb_prefix_group> groups(ng);
  for (hb_prefix_group& g : groups)
    if (scanf("%d %d %d", &g.first, &g.count, &g.prefix_len) != 3) return 6;
  int64_t T = 0;
  const hb_status st = check_shared(d, 1 << 20, reqs.data(), n, groups.data(), ng, &T);
  printf("status %d\n", (int)st);
  if (st != HB_OK || check) return 0;
  opt.fit_round = true;
  opt.groups = groups.data();
  opt.n_groups = ng;
  const hb_batch_desc desc{n, reqs.data(), nullptr, nullptr, HB_OUT_BF16};
  Plan p;
  build_plan(d, &desc, cu, &p, opt);
  printf("geom %d %d %d\n", p.half_tiles ? kTileCols / 2 : kTileCols, p.n_slots, (int)p.too_many_slots);
  if (p.too_many_slots) return 0;
  RecordPlan rp;
  build_records(p, &rp);
  int off = 0;
  const int n_append = build_append(reqs.data(), n, &rp.meta, &off);
  const int32_t* m = rp.meta.data();
  for (int i = 0; i < kItemsPerUnit * p.n_units; ++i) {
    const UnitRec& r = reinterpret_cast<const UnitRec*>(m)[i];
    const AttnItem& it = r.item;
    printf("wave %d %d %d %d %d %d %d %d", r.kind, it.kv_head, it.tok0, it.pos0, it.npos, it.kv_begin, it.kv_end, it.part);
    if (it.kv_begin < it.kv_end)
      for (int b = it.kv_begin / 16; b <= (it.kv_end - 1) / 16; ++b) {
        const int at = rp.off_bt + r.window + b;
        printf(" %d", at >= rp.off_bt && at < rp.off_merge ? m[at] : -1);
        const int k = b - it.kv_begin / 16;  // the ids at hand are those of the table
        const int step = r.kind == kRecTile ? 2 : 1, w = r.kind == kRecTile ? i % 4 & 1 : 0;
        if (k % step == w && k / step < 4 && r.ids[k / step] != m[at]) printf(" differs");
      }
    printf("\n");
  }
  for (int i = 0; i < p.n_merge_units; ++i) {
    const MergeGroup& g = reinterpret_cast<const MergeGroup*>(m + rp.off_merge)[i];
    printf("merge %d %d %d %d %d %d %d\n", g.part0, g.nparts, g.stride, g.tok0, g.npos, g.kv_head, g.cols);
  }
  for (int i = 0; i < n_append; ++i) {
    const AppendUnit& u = reinterpret_cast<const AppendUnit*>(m + off)[i];
    printf("append %d %d %d %d\n", u.tok0, u.pos0, u.n, u.block);
  }
  return 0;
}
