// Prints how the work units of one batch's plan are launched and joined: for a
// layer's plan the unit codes, items, groups and merge units, for a handle's
// (fit 1) the records that it uploads.
// Input: "H nq nkv hd F cu fit window sinks split_tile split_item R", then R lines "chunk context".
#include <algorithm>
#include <cstdio>
#include <vector>

#include "hb_plan.h"

using namespace hb;

int main() {
  hb_layer_config c{};
  int cu, fit, n;
  PlanOptions opt;
  if (scanf("%d %d %d %d %d %d %d %d %d %d %d %d", &c.hidden, &c.n_q_heads, &c.n_kv_heads, &c.head_dim, &c.ffn_dim, &cu,
            &fit, &opt.window.window, &opt.window.sinks, &opt.split_tile, &opt.split_item, &n) != 12)
    return 2;
  c.kv_block_size = 16;
  c.rope_theta = 5e5f;
  c.rms_eps = 1e-5f;
  c.max_requests = 1 << 16;
  opt.fit_round = fit;
  std::vector<hb_request> reqs(n);
  int longest = 0;
  for (hb_request& r : reqs) {
    if (scanf("%d %d", &r.chunk_len, &r.context_len) != 2) return 4;
    longest = std::max(longest, r.chunk_len + r.context_len);
    c.max_batch_tokens += r.chunk_len;
  }
  Dims d;
  if (check_config(&c, &d) != HB_OK) return 3;
  const std::vector<int32_t> table((longest + 15) / 16, 0);
  for (hb_request& r : reqs) {
    r.block_table = table.data();
    r.n_blocks = (int32_t)table.size();
  }
  int64_t T = 0;
  if (check_requests(d, 1, reqs.data(), n, opt.window, &T) != HB_OK) return 5;
  const hb_batch_desc desc{n, reqs.data(), nullptr, nullptr, HB_OUT_BF16};
  Plan p;
  build_plan(d, &desc, cu, &p, opt);
  printf("geom %d %d %d %d\n", p.half_tiles ? kTileCols / 2 : kTileCols, p.n_slots, p.n_tiles, p.n_items);
  auto item = [](const AttnItem& it) {
    printf(" %d %d %d %d %d %d %d %d", it.req, it.kv_head, it.tok0, it.pos0, it.npos, it.kv_begin, it.kv_end, it.part);
  };
  auto merge = [](const MergeGroup& g, int cols) {
    printf("merge %d %d %d %d %d %d %d\n", g.part0, g.nparts, g.stride, g.tok0, g.npos, g.kv_head, cols);
  };
  // a wave's work, in launch order: its kind, which tile or item it is, and that
  const int32_t* m = p.meta.data();
  const AttnItem* tiles = reinterpret_cast<const AttnItem*>(m + p.off_tiles);
  const AttnItem* items = reinterpret_cast<const AttnItem*>(m + p.off_items);
  RecordPlan rp;
  if (fit) build_records(p, &rp);
  for (int u = 0; u < p.n_units; ++u) {
    const int code = m[p.off_units + u];
    const bool tile = code >= 0;
    const int unit = tile ? code : (-1 - code) & ~kUnitMerged;
    for (int w = 0; w < kItemsPerUnit; ++w) {
      const int i = tile ? unit : kItemsPerUnit * unit + w;
      int kind = tile ? kRecTile : ((-1 - code) & kUnitMerged) ? kRecMerged : kRecSingle;
      AttnItem it = tile ? tiles[i] : items[i];
      if (fit) {
        const UnitRec& r = reinterpret_cast<const UnitRec*>(rp.meta.data())[kItemsPerUnit * u + w];
        kind = r.kind;
        it = r.item;
      }
      printf("wave %d %d", kind, i);
      item(it);
      printf("\n");
    }
  }
  for (int i = 0; i < p.n_merge_units; ++i) {
    const int mu = m[p.off_merge + i];
    if (fit) {
      const MergeGroup& g = reinterpret_cast<const MergeGroup*>(rp.meta.data() + rp.off_merge)[i];
      merge(g, g.cols);
    } else {
      merge(reinterpret_cast<const MergeGroup*>(m + p.off_groups)[mu >> 4], mu & 15);
    }
  }
  return 0;
}
