// Prints the plan of one batch under a sliding window as text, its block ids
// looked up the way the kernels look them up.
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <vector>

#include "hb_plan.h"

using namespace hb;

int main() {
  hb_layer_config c{};
  int cu, n, window, sinks, split_tile, split_item;
  if (scanf("%d %d %d %d %d %d %d %d %d %d %d", &c.hidden, &c.n_q_heads, &c.n_kv_heads, &c.head_dim, &c.ffn_dim, &cu, &n,
            &window, &sinks, &split_tile, &split_item) != 11)
    return 2;
  c.kv_block_size = 16;
  c.rope_theta = 5e5f;
  c.rms_eps = 1e-5f;
  c.max_batch_tokens = 1 << 18;
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
  PlanOptions opt;
  opt.split_tile = split_tile;
  opt.split_item = split_item;
  opt.window = {window, sinks};
  opt.fit_round = true;
  int64_t T = 0;
  const hb_status st = check_requests(d, 1 << 24, reqs.data(), n, opt.window, &T);
  printf("status %d\n", (int)st);
  if (st != HB_OK) return 0;
  hb_batch_desc desc{n, reqs.data(), nullptr, nullptr, HB_OUT_BF16};
  Plan p;
  build_plan(d, &desc, cu, &p, opt);
  const int32_t* m = p.meta.data();
  printf("geom %d %d %d %d\n", kTileCols, kItemsPerUnit, (int)p.windowed, p.sink_blocks);
  printf("work %.17g %.17g\n", p.flops, p.bytes);
  for (int off : {p.off_bt, p.off_req_bt, p.off_tiles, p.off_items, p.off_units, p.off_groups, p.off_merge,
                  p.off_tile_shift, p.off_item_shift})
    printf("off %d %d\n", off, (int)p.meta.size());
  auto unit = [&](const char* kind, int at, int shift_at, int i) {
    const AttnItem& it = reinterpret_cast<const AttnItem*>(m + at)[i];
    UnitShift sh{0, 0};
    if (p.windowed) sh = reinterpret_cast<const UnitShift*>(m + shift_at)[i];
    printf("%s %d %d %d %d %d %d %d %d", kind, it.req, it.kv_head, it.tok0, it.pos0, it.npos, it.kv_begin, it.kv_end,
           it.part);
    // block ids of the range's steps
    for (int b = it.kv_begin / 16; b < (it.kv_end + 15) / 16 && it.kv_begin < it.kv_end; ++b) {
      const int idx = b + (p.windowed ? (b < p.sink_blocks ? sh.sink : sh.window) : 0);
      const int at_bt = p.off_bt + m[p.off_req_bt + it.req] + idx;
      if (at_bt < p.off_bt || at_bt >= p.off_tiles) {
        printf(" out-of-table");
        continue;
      }
      printf(" %d", m[at_bt]);
    }
    printf("\n");
  };
  for (int i = 0; i < p.n_tiles; ++i) unit("tile", p.off_tiles, p.off_tile_shift, i);
  for (int i = 0; i < p.n_items; ++i) unit("item", p.off_items, p.off_item_shift, i);
  for (int i = 0; i < p.n_units; ++i) printf("unit %d\n", m[p.off_units + i]);
  // the records: the same units, in launch order, one per wave, with the same
  // block at every place of their ranges and the first of them at hand
  RecordPlan rp;
  build_records(p, &rp);
  const int32_t* o = rp.meta.data();
  bool same = (int)rp.meta.size() >= 64 * p.n_units && rp.off_bt == 64 * p.n_units;
  auto block = [&](const AttnItem& it, const UnitShift& sh, int b) {
    return m[p.off_bt + m[p.off_req_bt + it.req] + b + (p.windowed ? (b < p.sink_blocks ? sh.sink : sh.window) : 0)];
  };
  for (int u = 0; u < p.n_units; ++u) {
    const int code = m[p.off_units + u];
    const int unit = code >= 0 ? code : (-1 - code) & ~kUnitMerged;
    for (int w = 0; w < 4; ++w) {
      const UnitRec& r = reinterpret_cast<const UnitRec*>(o)[4 * u + w];
      const int i = code >= 0 ? unit : 4 * unit + w;
      const AttnItem& it = reinterpret_cast<const AttnItem*>(m + (code >= 0 ? p.off_tiles : p.off_items))[i];
      UnitShift sh{0, 0};
      if (p.windowed) sh = reinterpret_cast<const UnitShift*>(m + (code >= 0 ? p.off_tile_shift : p.off_item_shift))[i];
      same &= r.kind == (code >= 0 ? kRecTile : ((-1 - code) & kUnitMerged) ? kRecMerged : kRecSingle);
      same &= std::memcmp(&r.item, &it, sizeof it) == 0;
      if (it.kv_begin >= it.kv_end) continue;
      const int first = it.kv_begin / 16, last = (it.kv_end - 1) / 16;
      for (int b = first; b <= last; ++b) {
        const int at = rp.off_bt + b + (b < p.sink_blocks ? r.sink : r.window);
        same &= at >= rp.off_bt && at < rp.off_merge && o[at] == block(it, sh, b);
      }
      for (int k = 0; k < 4; ++k)
        same &= r.ids[k] == block(it, sh, std::min(last, first + (code >= 0 ? 2 * k + (w & 1) : k)));
    }
  }
  for (int i = 0; i < p.n_merge_units; ++i) {
    const int mu = m[p.off_merge + i];
    MergeGroup want = reinterpret_cast<const MergeGroup*>(m + p.off_groups)[mu >> 4];
    want.cols = mu & 15;
    same &= std::memcmp(o + rp.off_merge + 8 * i, &want, sizeof want) == 0;
  }
  printf("records %d\n", (int)same);
  for (int r = 0; r < n; ++r)  // the block a request's first new token goes to
    printf("slot %d\n", m[p.off_bt + m[p.off_req_bt + r] + reqs[r].context_len / 16]);
  return 0;
}
