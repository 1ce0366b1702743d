// Host-side validation and planning of a hybrid-batch iteration (no HIP).
#include "hb_plan.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <map>
#include <new>
#include <tuple>

namespace hb {

static thread_local std::string g_err;

hb_status fail(hb_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return st;
}

const char* last_error() { return g_err.c_str(); }

hb_status host_oom() { return fail(HB_ERR_OOM, "host allocation failed"); }

hb_status check_config(const hb_layer_config* c, Dims* d) {
  if (!c) return fail(HB_ERR_INVALID, "null layer config");
  if (c->hidden <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 ||
      c->ffn_dim <= 0 || c->max_batch_tokens <= 0 || c->max_requests <= 0)
    return fail(HB_ERR_INVALID, "layer config sizes must be positive");
  if (!(c->rope_theta > 1.f) || !(c->rms_eps >= 0.f))
    return fail(HB_ERR_INVALID, "rope_theta must exceed 1 and rms_eps be >= 0");
  if (c->kv_block_size != 16) return fail(HB_ERR_UNSUPPORTED, "kv_block_size must be 16 (got %d)", c->kv_block_size);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(HB_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", c->head_dim);
  if (c->n_q_heads % c->n_kv_heads)
    return fail(HB_ERR_UNSUPPORTED, "n_q_heads (%d) must be a multiple of n_kv_heads (%d)", c->n_q_heads, c->n_kv_heads);
  int G = c->n_q_heads / c->n_kv_heads;
  if (G > 16 || 16 % G)
    return fail(HB_ERR_UNSUPPORTED, "q heads per kv head (%d) must divide 16", G);
  if (c->hidden % 64) return fail(HB_ERR_UNSUPPORTED, "hidden must be a multiple of 64 (got %d)", c->hidden);
  if (c->ffn_dim % 16) return fail(HB_ERR_UNSUPPORTED, "ffn_dim must be a multiple of 16 (got %d)", c->ffn_dim);
  if (c->max_batch_tokens > (1 << 20) || c->max_requests > (1 << 20))
    return fail(HB_ERR_UNSUPPORTED, "max_batch_tokens / max_requests above 2^20");
  {
    // every GEMM operand within the buffer window: the four weight matrices
    // and the three activation operands (with their padding rows)
    const int64_t H = c->hidden, F = c->ffn_dim, qd = (int64_t)c->n_q_heads * c->head_dim;
    const int64_t qkv = (int64_t)(c->n_q_heads + 2 * c->n_kv_heads) * c->head_dim;
    const int64_t TA = (int64_t)c->max_batch_tokens + kGemmPadRows;
    hb_status st = check_window("w_qkv", qkv, H);
    if (st == HB_OK) st = check_window("w_o", H, qd);
    if (st == HB_OK) st = check_window("w_gate_up", 2 * F, H);
    if (st == HB_OK) st = check_window("w_down", H, F);
    if (st == HB_OK) st = check_window("normed activations (max_batch_tokens + 512 rows)", TA, H);
    if (st == HB_OK) st = check_window("attention output (max_batch_tokens + 512 rows)", TA, qd);
    if (st == HB_OK) st = check_window("SwiGLU activations (max_batch_tokens + 512 rows)", TA, F);
    if (st != HB_OK) return st;
  }
  d->H = c->hidden;
  d->nq = c->n_q_heads;
  d->nkv = c->n_kv_heads;
  d->hd = c->head_dim;
  d->F = c->ffn_dim;
  d->blk = 16;
  d->G = G;
  d->P = 16 / G;
  d->BQ = kTileCols / G;
  d->qkv_n = (d->nq + 2 * d->nkv) * d->hd;
  d->theta = c->rope_theta;
  d->eps = c->rms_eps;
  d->max_T = c->max_batch_tokens;
  d->max_R = c->max_requests;
  return HB_OK;
}

hb_status check_window(const char* what, int64_t rows, int64_t cols) {
  if (rows * cols * 2 > kOperandWindow)
    return fail(HB_ERR_UNSUPPORTED, "%s: %lld x %lld bf16 values exceed the %lld-byte GEMM operand window", what,
                (long long)rows, (long long)cols, (long long)kOperandWindow);
  return HB_OK;
}

static int64_t blocks_for(int64_t kv_len) { return (kv_len + 15) / 16; }

hb_status check_window_args(int window, int sinks) {
  if (window < 0 || sinks < 0) return fail(HB_ERR_INVALID, "window %d or sinks %d below 0", window, sinks);
  if (window > (1 << 30) || sinks > (1 << 30)) return fail(HB_ERR_INVALID, "window %d or sinks %d above 2^30", window, sinks);
  return HB_OK;
}

DeadBlocks dead_blocks(const Window& w, int pos) {
  if (w.window <= 0) return {};
  const int first = (w.sinks + 15) / 16, end = std::max(0, pos - w.window + 1) / 16;
  if (end <= first) return {};
  return {first, end - first};
}

hb_status check_requests(const Dims& d, int num_blocks, const hb_request* requests, int n, const Window& w,
                         int64_t* n_tokens) {
  if (n < 0) return fail(HB_ERR_INVALID, "n_requests < 0");
  if (n > d.max_R) return fail(HB_ERR_INVALID, "n_requests %d exceeds max_requests %d", n, d.max_R);
  if (n > 0 && !requests) return fail(HB_ERR_INVALID, "null request array");
  if (num_blocks <= 0) return fail(HB_ERR_INVALID, "pool has no blocks");
  int64_t T = 0, entries = 0;
  for (int r = 0; r < n; ++r) {
    const hb_request& q = requests[r];
    if (q.chunk_len < 1) return fail(HB_ERR_INVALID, "request %d: chunk_len %d < 1", r, q.chunk_len);
    if (q.context_len < 0) return fail(HB_ERR_INVALID, "request %d: context_len %d < 0", r, q.context_len);
    int64_t kv = (int64_t)q.context_len + q.chunk_len;
    if (kv > (int64_t)1 << 30) return fail(HB_ERR_INVALID, "request %d: context too long", r);
    if (!q.block_table) return fail(HB_ERR_INVALID, "request %d: null block_table", r);
    if (q.n_blocks < blocks_for(kv))
      return fail(HB_ERR_INVALID, "request %d: block table has %d blocks, needs %lld", r, q.n_blocks,
                  (long long)blocks_for(kv));
    const DeadBlocks dead = dead_blocks(w, q.context_len);
    for (int64_t i = 0; i < blocks_for(kv); ++i) {
      if (i == dead.first) i += dead.count;
      int32_t b = q.block_table[i];
      if (b < 0 || b >= num_blocks)
        return fail(HB_ERR_RANGE, "request %d: block_table[%lld] = %d outside [0, %d)", r, (long long)i, b, num_blocks);
    }
    T += q.chunk_len;
    entries += blocks_for(kv) - dead.count + kBtPad;
  }
  if (T > d.max_T) return fail(HB_ERR_INVALID, "batch has %lld tokens, max_batch_tokens is %d", (long long)T, d.max_T);
  if (entries > (int64_t)1 << 30)  // the plan counts its words in 32 bits
    return fail(HB_ERR_UNSUPPORTED, "block tables of %lld entries in one batch", (long long)entries);
  *n_tokens = T;
  return HB_OK;
}

hb_status check_batch(const Dims& d, int num_blocks, const hb_batch_desc* desc, SlotMarks* marks, const Window& w) {
  if (!desc) return fail(HB_ERR_INVALID, "null batch descriptor");
  const int R = desc->n_requests;
  if (R < 0) return fail(HB_ERR_INVALID, "n_requests < 0");
  if (R == 0) return HB_OK;
  if (R > d.max_R) return fail(HB_ERR_INVALID, "n_requests %d exceeds max_requests %d", R, d.max_R);
  if (!desc->requests) return fail(HB_ERR_INVALID, "null request array");
  if (!desc->x_in || !desc->x_out) return fail(HB_ERR_INVALID, "null x_in or x_out");
  if (desc->out_dtype != HB_OUT_F32 && desc->out_dtype != HB_OUT_BF16)
    return fail(HB_ERR_INVALID, "out_dtype must be HB_OUT_F32 or HB_OUT_BF16");
  int64_t T = 0;
  hb_status st = check_requests(d, num_blocks, desc->requests, R, w, &T);
  if (st != HB_OK) return st;
  // x_in (bf16) and x_out must not overlap
  {
    uintptr_t a0 = (uintptr_t)desc->x_in, a1 = a0 + (uintptr_t)T * d.H * 2;
    uintptr_t b0 = (uintptr_t)desc->x_out, b1 = b0 + (uintptr_t)T * d.H * (desc->out_dtype == HB_OUT_F32 ? 4 : 2);
    if (a0 < b1 && b0 < a1) return fail(HB_ERR_INVALID, "x_out overlaps x_in");
  }
  // no two new tokens may be written to the same physical slot
  SlotMarks local;
  SlotMarks* m = marks ? marks : &local;
  if ((int)m->mask.size() < num_blocks) m->mask.assign(num_blocks, 0);
  m->touched.clear();
  m->touched.reserve(T);  // nothing can fail while marks stand
  for (int r = 0; r < R && st == HB_OK; ++r) {
    const hb_request& q = desc->requests[r];
    for (int64_t p = q.context_len; p < (int64_t)q.context_len + q.chunk_len; ++p) {
      int32_t b = q.block_table[p / 16];
      uint16_t bit = (uint16_t)(1u << (p % 16));
      if (m->mask[b] == 0) m->touched.push_back(b);
      if (m->mask[b] & bit) {
        st = fail(HB_ERR_INVALID, "request %d writes slot %lld of block %d, already written by this batch", r,
                  (long long)(p % 16), b);
        break;
      }
      m->mask[b] |= bit;
    }
  }
  for (int32_t b : m->touched) m->mask[b] = 0;
  m->touched.clear();
  return st;
}

static hb_status plan_compaction(int num_blocks, int32_t* const* tables, const int32_t* n_blocks, int n_tables,
                                 int32_t* src, int32_t* dst, int32_t* n_moves, int32_t* n_used) {
  if (!src || !dst || !n_moves || !n_used) return fail(HB_ERR_INVALID, "hb_plan_compaction: null output pointer");
  if (num_blocks < 1 || n_tables < 0) return fail(HB_ERR_INVALID, "num_blocks %d < 1 or n_tables %d < 0", num_blocks, n_tables);
  if (n_tables > 0 && (!tables || !n_blocks)) return fail(HB_ERR_INVALID, "null tables or n_blocks");
  std::vector<int32_t> to(num_blocks, -1);  // -1: not named; else where the block goes
  int used = 0;
  for (int t = 0; t < n_tables; ++t) {
    if (n_blocks[t] < 0 || (n_blocks[t] > 0 && !tables[t])) return fail(HB_ERR_INVALID, "table %d: null or negative length", t);
    for (int i = 0; i < n_blocks[t]; ++i) {
      const int32_t b = tables[t][i];
      if (b < -1 || b >= num_blocks)
        return fail(HB_ERR_RANGE, "table %d: entry %d = %d outside [-1, %d)", t, i, b, num_blocks);
      if (b >= 0 && to[b] < 0) {
        to[b] = b;
        ++used;
      }
    }
  }
  int moves = 0;
  for (int b = used, hole = 0; b < num_blocks; ++b) {
    if (to[b] < 0) continue;
    while (to[hole] >= 0) ++hole;  // as many holes below `used` as named blocks from it on
    src[moves] = b;
    dst[moves++] = hole;
    to[b] = to[hole] = hole;  // (the latter for a table given twice, whose ids are new already)
    ++hole;
  }
  for (int t = 0; t < n_tables; ++t)
    for (int i = 0; i < n_blocks[t]; ++i)
      if (tables[t][i] >= 0) tables[t][i] = to[tables[t][i]];
  *n_moves = moves;
  *n_used = used;
  return HB_OK;
}

static int align16(int x) { return (x + 15) & ~15; }

void iteration_work(const Dims& d, const hb_request* reqs, int n, double* flops, double* bytes, const Window& w) {
  double T = 0, pairs = 0, kv_tokens = 0;
  for (int r = 0; r < n; ++r) {
    double c = reqs[r].chunk_len, x = reqs[r].context_len;
    T += c;
    pairs += c * x + c * (c + 1) / 2;
    kv_tokens += x + c;
    if (w.window > 0) {
      // the window hides h(p) = max(0, p + 1 - window - sinks) keys from the row at p:
      // h(x) of them from every row, and b the last row's
      const double a = std::max(0.0, x + 1 - w.window - w.sinks), b = std::max(0.0, x + c - w.window - w.sinks);
      const double hiding = std::min(c, b);  // rows from which something is hidden: h counts up to b over them
      pairs -= hiding * (2 * b - hiding + 1) / 2;
      kv_tokens -= a;
    }
  }
  double p_lin = (double)d.H * d.qkv_n + (double)d.nq * d.hd * d.H + 3.0 * d.H * d.F;
  *flops = 2.0 * T * p_lin + 4.0 * d.nq * d.hd * pairs;
  double kv_tok_bytes = 2.0 * d.nkv * d.hd * 2.0;  // K and V, bf16
  *bytes = 2.0 * p_lin + 2.0 * 2.0 * d.H         // weights and gains, bf16, once
           + kv_tokens * kv_tok_bytes            // cached + new K/V read once per (request, kv head)
           + T * kv_tok_bytes                    // new K/V written
           + T * d.H * 2.0 + T * d.H * 4.0;      // x_in bf16, y fp32
}

static int round_up(int64_t x, int m) { return (int)((x + m - 1) / m * m); }

// The rules of PlanOptions::fit_round. Their limits, in keys, were measured at head
// dimension 128; at 64, where a key is half the bytes and half the products, the
// same ones are used.

// Smallest split length from `finest` on (multiples of 64 keys, at most 1024) at
// which key ranges of these lengths, each in nkv kv heads, take `slots`
// workgroups at most, a workgroup taking `waves` splits; 0 where none does.
static int one_round_split(const std::vector<int>& lengths, int nkv, int64_t slots, double finest, int waves) {
  for (int S = std::max(64, round_up((int64_t)std::ceil(finest), 64)); S <= 1024; S += 64) {
    int64_t units = 0;
    for (int n : lengths) units += (n + (int64_t)S * waves - 1) / (S * waves);
    if (units * nkv <= slots) return S;
  }
  return 0;
}

// Split length of a launch of item ranges (lengths, each in nkv kv heads) that
// fits one round of workgroups, one per CU; 0 where it does not.
// A range of at most 576 keys stays one unit: its four waves, of up to 192 keys,
// are done before a merge kernel would be (cold caches, 300 keys 12.2 -> 9.3 us,
// 8 decodes behind a 500-key window 13.3 -> 11.8; at 1000 keys a unit takes 15.6
// and the split 13.0). Longer ones are split as finely as one round allows (4
// decodes of 3000 keys, 192 instead of 128 units 18.8 -> 17.4 us; a second
// round costs more than it divides: 1 x 20000 keys on eight heads, 320 units of
// 128 keys a wave 28.5, 216 of 192 23.1), but no finer than sqrt(keys): parts
// cost the merge about as much as a wave's keys cost it (1 x 30000 keys on one
// head, 64 keys a wave and 118 parts 25.0 us, 192 and 40 20.8).
static int fit_item_split(const std::vector<int>& lengths, int nkv, int cus) {
  int longest = 0;
  for (int n : lengths) longest = std::max(longest, n);
  if ((int64_t)lengths.size() * nkv > cus || longest == 0) return 0;
  if (longest <= 576) return round_up((longest + kItemsPerUnit - 1) / kItemsPerUnit, 64);
  return one_round_split(lengths, nkv, cus, std::sqrt((double)longest), kItemsPerUnit);
}

// The same for tiles that share the CUs with item units: `slots` workgroups are
// theirs. A tile step costs a third of an item's, and a part that the merge
// reads holds eight times an item's columns, so no finer than 3 sqrt(keys) (one
// kv head, cold caches: one tile of 2000 keys 29.2 -> 16.7 us, 4 of 16000 32.8 ->
// 27.5 at 384 and 28.7 at 256 keys; eight heads, 32 tiles of 2100: 30.9 -> 22.1
// at 384, one round, 24.4 at 256), and ranges of at most 576 keys stay whole
// (128 tiles of 544 keys, halved, 22.5 -> 24.2; 128 of 1000 28.2 -> 25.9).
static int fit_tile_split(const std::vector<int>& lengths, int nkv, int64_t slots) {
  int longest = 0;
  for (int n : lengths) longest = std::max(longest, n);
  return longest > 576 ? one_round_split(lengths, nkv, slots, 3.0 * std::sqrt((double)longest), 1) : 0;
}

// Item units of one round in an order that gives those that read the same keys to
// one die: workgroups go to the kDies dies in turn, each with an L2 of its own,
// and every die would fetch all of K and V otherwise (cold caches, 64 tokens
// behind 500 cached, eight kv heads, 128 units 13.1 -> 10.0 us; 70B heads behind
// 900 17.4 -> 12.6). Larger groups first, each to the die with the most room, the
// rest of it to the next. (Tiles share a key range four times less often: even
// with cold caches, 19.8 -> 23.2 us with warm ones, 64 tiles of 1000 keys.)
constexpr int kDies = 8;
template <typename F>
static std::vector<int32_t> by_die(const std::vector<int32_t>& units, F&& item_of) {
  const int n = (int)units.size();
  std::map<std::tuple<int, int, int>, int> known;
  std::vector<std::vector<int32_t>> groups;
  for (const int32_t u : units) {
    const AttnItem it = item_of(u);
    const auto at = known.insert({{it.req, it.kv_head, it.kv_begin}, (int)groups.size()}).first;
    if (at->second == (int)groups.size()) groups.emplace_back();
    groups[at->second].push_back(u);
  }
  std::stable_sort(groups.begin(), groups.end(), [](const auto& a, const auto& b) { return a.size() > b.size(); });
  int next[kDies], room[kDies];
  for (int x = 0; x < kDies; ++x) {
    next[x] = x;
    room[x] = (n - x + kDies - 1) / kDies;
  }
  std::vector<int32_t> order(n);
  for (const auto& group : groups) {
    int x = 0, left = 0;
    for (const int32_t u : group) {
      if (left == 0) {
        x = (int)(std::max_element(room, room + kDies) - room);
        left = room[x];
      }
      order[next[x]] = u;
      next[x] += kDies;
      --room[x];
      --left;
    }
  }
  return order;
}

void build_plan(const Dims& d, const hb_batch_desc* desc, int cu_count, Plan* p, const PlanOptions& opt) {
  const int R = desc->n_requests;
  const hb_request* rq = desc->requests;
  int T = 0, nbt = 0;
  std::vector<int> tok_start(R + 1, 0);
  const Window& win = opt.window;
  p->windowed = false;
  for (int r = 0; r < R; ++r) {
    tok_start[r] = T;
    T += rq[r].chunk_len;
    const int64_t kv = (int64_t)rq[r].context_len + rq[r].chunk_len;
    nbt += (int)blocks_for(kv) - dead_blocks(win, rq[r].context_len).count + kBtPad;
    p->windowed |= win.window > 0 && kv - win.window > win.sinks;  // the last row's window hides a key
  }
  p->window = win;
  p->sink_blocks = p->windowed ? (win.sinks + 15) / 16 : 0;
  tok_start[R] = T;
  p->T = T;
  p->R = R;

  const int cus = std::max(1, cu_count);
  // keys of the w rows from i0 on of request r
  auto range_len = [&](int r, int i0, int w) {
    const int x = rq[r].context_len;
    return x + std::min(rq[r].chunk_len, i0 + w) - 16 * dead_blocks(win, x + i0).count;
  };
  // A small launch is latency: a wave item starts sooner than a tile (its K and V
  // go straight to registers, no ring and barrier) and its four waves share the
  // key range, so a batch whose chunks, cut into items as well, make one round of
  // workgroups of at most 320 keys a wave takes no tiles. Eight kv heads, cold
  // caches: a fresh 100-token chunk 10.3 -> 8.2 us, 64 tokens behind 500 cached
  // 19.1 -> 10.0, behind 900 26.6 -> 13.2, 128 behind 1000 18.7 (split tiles) ->
  // 13.7. From 384 keys a wave on it depends (64 behind 2500 20.2 -> 20.5; sixteen
  // heads, 64 behind 2000 with 4 decodes of 3000 28.0 -> 30.9). With more items
  // than CUs, one round of two workgroups per CU, a unit to a range, does as well
  // up to 256 keys a wave (256 behind 200 17.8 -> 12.0, a fresh 256 13.3 -> 10.4; at
  // 320 128 behind 1000 beside 8 decodes of 1000 21.5 -> 23.8; with ranges split 128
  // behind 2000 22.3 -> 25.1; a second round 512 behind 300 23.4 -> 32.8).
  auto fills_tile = [&](int r) { return (int64_t)rq[r].chunk_len * d.G >= kTileCols / 2; };
  bool items_only = false;
  int S_items = 0;
  p->paired = false;
  const bool fit_chunks = opt.fit_round && opt.split_tile <= 0 && opt.split_item <= 0;
  if (fit_chunks) {
    int64_t n = 0;
    bool chunks = false;
    for (int r = 0; r < R; ++r) {
      n += (rq[r].chunk_len + d.P - 1) / d.P;
      chunks |= fills_tile(r);
    }
    if (chunks && n * d.nkv <= 2 * cus) {
      std::vector<int> all;
      for (int r = 0; r < R; ++r)
        for (int i0 = 0; i0 < rq[r].chunk_len; i0 += d.P) all.push_back(range_len(r, i0, d.P));
      const int longest = *std::max_element(all.begin(), all.end());
      p->paired = n * d.nkv > cus;
      S_items = p->paired ? round_up(((int64_t)longest + kItemsPerUnit - 1) / kItemsPerUnit, 64)
                          : fit_item_split(all, d.nkv, cus);
      items_only = S_items > 0 && S_items <= (p->paired ? 256 : 320);
      p->paired &= items_only;
    }
  }
  // Otherwise a chunk that fills at least half a workgroup tile goes to the
  // workgroup path; decodes and short chunks become 16-column wave items.
  auto is_tile = [&](int r) { return !items_only && fills_tile(r); };
  double tile_keys = 0, item_keys = 0;
  std::vector<int> item_lengths, tile_lengths;  // of one kv head
  for (int r = 0; r < R; ++r) {
    const int w = is_tile(r) ? d.BQ : d.P;
    for (int i0 = 0; i0 < rq[r].chunk_len; i0 += w) {
      const int len = range_len(r, i0, w);
      (is_tile(r) ? tile_keys : item_keys) += (double)d.nkv * len;
      if (opt.fit_round) (is_tile(r) ? tile_lengths : item_lengths).push_back(len);
    }
  }
  // split lengths (multiples of 64 keys): about one round of tile workgroups
  // (each split also writes kTileCols columns of fp32 partials). Items: a
  // wave advances one 32-key step per memory latency (about 1.2 us), so a
  // launch lasts at least that times its longest range, and at least its K/V
  // bytes at the HBM rate. S_i is where the first is about 0.6 of the second,
  // item_keys / (2.8 CUs) keys, between opt.min_item (64: shorter ranges gain
  // less than their merge costs) and 1024; from 1024 on most decodes, up to 4 S_i
  // keys, need no merge kernel, and S_i grows again with two wave slots' worth
  // of keys per wave. Attention + merge, at least 1024 keys -> this rule: 8
  // decodes of 512-8192 keys and one kv head 41 -> 13 us, 4 decodes of 8192
  // keys and eight kv heads 42 -> 29 us, 128 decodes and one kv head 50 -> 31
  // us, 32 decodes and eight kv heads 66 -> 63 us. When both kinds are present, tiles run
  // beside the bandwidth-bound items, and a tile is split only as far as it
  // would otherwise outlast the launch: the launch takes about the longer of
  // the items' K/V bytes at the HBM rate and the tile steps spread over the
  // workgroup slots (two per compute unit), and a tile step of 32 keys
  // (beside an item workgroup) takes about kMixedStepUs. Measured on MI355X
  // over chunk/decode mixes of the 8B and 70B layers and of their
  // tensor-parallel shards (item split 256 .. 4096, tile split 1024 .. 16384).
  constexpr double kMixedStepUs = 0.6, kItemBytesPerUs = 6.0e6;
  const bool mixed = tile_keys > 0 && item_keys > 0;
  double s_t = tile_keys / (1.0 * cus);
  if (mixed) {
    const double launch_us = std::max(item_keys * 4.0 * d.hd / kItemBytesPerUs,
                                      tile_keys / 32.0 * kMixedStepUs / (2.0 * cus));
    s_t = launch_us / kMixedStepUs * 32.0;
  }
  const int S_t_auto = std::max(1024, round_up((int64_t)std::min(s_t, 1.0e9) + 1, 64));
  const int S_i_fill = std::min(1024, std::max(opt.min_item, round_up((int64_t)(item_keys * d.hd / 128 / (2.8 * cus)), 64)));
  const int S_i_fit = items_only      ? S_items
                      : tile_keys > 0 ? 0
                                      : fit_item_split(item_lengths, d.nkv, cus);
  const int S_i = opt.split_item > 0 ? round_up(opt.split_item, 64)
                  : S_i_fit > 0      ? S_i_fit
                                     : std::max(S_i_fill, round_up((int64_t)std::min(item_keys / (16.0 * cus), 1.0e9) + 1, 64));
  // Longest range that one wave takes alone. With few item groups a lone wave of
  // S_i keys is what the launch ends on, so ranges above 256 keys are cut over a
  // unit's four waves already (beside a 512-token chunk, 64 decodes behind a
  // 1024-key window 55.8 -> 49.4 us; 300 + 100 decodes of 50-800 keys 34.4 ->
  // 29.5; 64 decodes behind 4096 138 -> 134.7). From four groups per CU on others
  // fill in behind it, and the merge in LDS is only a cost (128 decodes of 600
  // keys on eight heads 49.4 -> 52.0, 256 of 50-1000 82.4 -> 84.4).
  const bool few_items = opt.fit_round && item_lengths.size() * (size_t)d.nkv < 4 * (size_t)cus;
  const int S_1 = few_items ? std::min(S_i, 256) : S_i;
  // Tiles that leave CUs idle are split for one round too, beside the item units,
  // or, where that is sooner done, halved: one round of two half tiles per CU,
  // which hide each other's latencies (0.57 us a step of 32 keys; a tile alone
  // 0.61), with nothing to merge. Of t tiles a split spreads the keys over all
  // CUs, so halves win while (CUs - t) keys are few: eight kv heads, cold caches,
  // 128 tiles of 512 keys 17.9 -> 14.9 us, of 1000 25.9 -> 22.3, 2500 even; 192
  // of 1800 39.5 -> 33.8, of 2800 even; 256 of 9000 172 -> 161; 64 of 1250 lose.
  constexpr int64_t kHalfTileKeys = 160 * 1024;
  int S_t_fit = 0;
  p->half_tiles = false;
  if (fit_chunks) {
    int64_t quarters = 0;  // of item units
    for (int n : item_lengths)
      quarters += n <= S_1 ? 1 : ((n + S_i - 1) / S_i + kItemsPerUnit - 1) / kItemsPerUnit * kItemsPerUnit;
    const int64_t item_groups = quarters * d.nkv / kItemsPerUnit, t = (int64_t)tile_lengths.size() * d.nkv;
    const int longest = tile_lengths.empty() ? 0 : *std::max_element(tile_lengths.begin(), tile_lengths.end());
    p->half_tiles = t > 0 && t <= cus && (cus - t) * longest <= kHalfTileKeys &&
                    2 * t + item_groups <= 2 * cus;
    S_t_fit = p->half_tiles ? round_up(longest, 64) : fit_tile_split(tile_lengths, d.nkv, cus - item_groups);
  }
  const int S_t = opt.split_tile > 0 ? round_up(opt.split_tile, 64) : S_t_fit > 0 ? S_t_fit : S_t_auto;
  p->split_tile = S_t;
  p->split_item = S_i;

  // Tiles: one work unit per (request, kv head, position block, key split).
  // Items: a (request, kv head, position group) whose keys fit one split
  // length is one wave item, packed four to a unit with items of similar
  // length. A longer range is cut over k = ceil(n / 4) workgroups of four
  // waves (n = its split count); each workgroup's four waves take
  // consecutive sub-ranges and combine them in LDS, so only ranges that need
  // more than one workgroup leave partial results for the merge kernel.
  // In a windowed plan every length here is one of the unit's key axis (AttnItem).
  std::vector<AttnItem> tiles, singles;
  struct Unit {
    int64_t len;     // keys of the unit's longest wave
    int first;       // first item (merged) or first single
    bool merged;
  };
  std::vector<AttnItem> merged_items;
  std::vector<Unit> merged_units;
  struct SplitTile {
    int first, n, kv_len;  // its pieces are tiles[first .. first + n)
  };
  std::vector<SplitTile> split_tiles;
  std::vector<MergeGroup> groups;
  int slots = 0;
  for (int r = 0; r < R; ++r) {
    const int c = rq[r].chunk_len, x = rq[r].context_len;
    const bool tile = is_tile(r);
    const int w = !tile ? d.P : p->half_tiles ? d.BQ / 2 : d.BQ, S = tile ? S_t : S_i;
    for (int g = 0; g < d.nkv; ++g) {
      for (int i0 = 0; i0 < c; i0 += w) {
        const int npos = std::min(w, c - i0);
        const int gap = 16 * dead_blocks(win, x + i0).count;
        const int pos0 = x + i0 - gap, kv_len = pos0 + npos;
        const int nspl = (kv_len + S - 1) / S;
        if (tile) {
          int part0 = -1;
          if (nspl > 1) {
            part0 = slots;
            groups.push_back({slots, nspl, kTileCols, tok_start[r] + i0, npos, g, 0, 0});
            slots += nspl * kTileCols;
          }
          if (nspl > 1) split_tiles.push_back({(int)tiles.size(), nspl, kv_len});
          for (int s = 0; s < nspl; ++s)
            tiles.push_back({r, g, tok_start[r] + i0, pos0, npos, s * S, std::min(kv_len, (s + 1) * S),
                             nspl > 1 ? part0 + s * kTileCols : -1});
          continue;
        }
        if (kv_len <= S_1) {
          singles.push_back({r, g, tok_start[r] + i0, pos0, npos, 0, kv_len, -1});
          continue;
        }
        const int k = (nspl + kItemsPerUnit - 1) / kItemsPerUnit;
        const int wlen = round_up((kv_len + k - 1) / k, 64);
        int part0 = -1;
        if (k > 1) {
          part0 = slots;
          groups.push_back({slots, k, 16, tok_start[r] + i0, npos, g, 0, 0});
          slots += 16 * k;
        }
        for (int j = 0; j < k; ++j) {
          const int b = j * wlen, e = std::min(kv_len, b + wlen);
          const int plen = round_up((e - b + kItemsPerUnit - 1) / kItemsPerUnit, 64);
          merged_units.push_back({plen, (int)merged_items.size(), true});
          for (int q = 0; q < kItemsPerUnit; ++q) {
            const int pb = std::min(e, b + q * plen), pe = std::min(e, pb + plen);
            merged_items.push_back({r, g, tok_start[r] + i0, pos0, npos, pb, pe, k > 1 ? part0 + 16 * j : -1});
          }
        }
      }
    }
  }
  // A split tile is cut at multiples of S_t (full pieces and a shorter
  // last one). When every work unit gets a workgroup slot of its own (two
  // per compute unit), nothing queues behind a piece and the launch lasts as
  // long as the longest one, so the pieces are evened out instead (64-key
  // multiples, at most S_t; the piece count is unchanged). With more units
  // than slots, even pieces would add long units to the queue; the short
  // last pieces fill gaps there.
  const int64_t item_unit_count = (int64_t)merged_units.size() + ((int64_t)singles.size() + kItemsPerUnit - 1) / kItemsPerUnit;
  if ((int64_t)tiles.size() + item_unit_count <= 2 * (int64_t)std::max(1, cu_count)) {
    for (const SplitTile& st : split_tiles) {
      const int piece = round_up((st.kv_len + st.n - 1) / st.n, 64);
      for (int s = 0; s < st.n; ++s) {
        tiles[st.first + s].kv_begin = s * piece;
        tiles[st.first + s].kv_end = std::min(st.kv_len, (s + 1) * piece);
      }
    }
  }
  // longest first (greedy list scheduling over the compute units), and items
  // of similar length share a workgroup, which lasts as long as its longest
  auto longer = [](const AttnItem& x, const AttnItem& y) {
    return (x.kv_end - x.kv_begin) * (int64_t)x.npos > (y.kv_end - y.kv_begin) * (int64_t)y.npos;
  };
  std::stable_sort(tiles.begin(), tiles.end(), longer);
  std::stable_sort(singles.begin(), singles.end(), [](const AttnItem& x, const AttnItem& y) {
    return (x.kv_end - x.kv_begin) > (y.kv_end - y.kv_begin);
  });
  std::vector<Unit> item_units = merged_units;
  for (int i = 0; i < (int)singles.size(); i += kItemsPerUnit)
    item_units.push_back({singles[i].kv_end - singles[i].kv_begin, i, false});
  std::stable_sort(item_units.begin(), item_units.end(), [](const Unit& x, const Unit& y) { return x.len > y.len; });
  // items in unit order: unit v's items are 4 v .. 4 v + 3 (the last unit of
  // singles is padded with empty items)
  std::vector<AttnItem> items;
  std::vector<int32_t> item_unit_codes;
  items.reserve(merged_items.size() + singles.size() + kItemsPerUnit);
  for (const Unit& u : item_units) {
    const int v = (int)(items.size() / kItemsPerUnit);
    item_unit_codes.push_back(-1 - (u.merged ? (v | kUnitMerged) : v));
    const std::vector<AttnItem>& src = u.merged ? merged_items : singles;
    const int n = std::min<int>(kItemsPerUnit, (int)src.size() - u.first);
    for (int q = 0; q < n; ++q) items.push_back(src[u.first + q]);
    for (int q = n; q < kItemsPerUnit; ++q) {
      AttnItem e = src[u.first];
      e.kv_begin = e.kv_end;  // empty: the wave does nothing
      items.push_back(e);
    }
  }
  // work units: one per tile, one per item unit, in alternating runs of one
  // unit per CU: workgroups are handed out round-robin over the CUs, two per
  // CU, so a CU's first two workgroups are a compute-bound tile and a
  // bandwidth-bound item unit, which overlap well
  const int nt = (int)tiles.size(), ni_units = (int)item_unit_codes.size();
  std::vector<int32_t> units;
  units.reserve(nt + ni_units);
  const int run = opt.unit_block != 0 ? opt.unit_block : cus;
  if (run > 0 && ni_units == 0 && nt <= 2 * run) {
    // tiles alone, at most two per CU: CU i gets the i-th longest and the
    // i-th shortest (workgroups i and i + CUs share a CU), so that all CUs
    // hold about the same number of steps: a fresh 2048-token chunk of the 8B
    // layer, 512 tiles, 53.2 -> 50.8 us; longest first throughout gives the
    // first CU 96 steps and the last 34
    for (int a = 0; a < std::min(nt, run); ++a) units.push_back(a);
    for (int a = nt - 1; a >= run; --a) units.push_back(a);
  } else if (run > 0) {
    for (int a = 0, b = 0; a < nt || b < ni_units;) {
      for (int k = 0; k < run && a < nt; ++k) units.push_back(a++);
      for (int k = 0; k < run && b < ni_units; ++k) units.push_back(item_unit_codes[b++]);
    }
  } else {
    for (int a = 0, b = 0; a < nt || b < ni_units;) {
      if (b >= ni_units || (a < nt && (int64_t)a * ni_units <= (int64_t)b * nt)) units.push_back(a++);
      else units.push_back(item_unit_codes[b++]);
    }
  }
  if (items_only)
    units = by_die(units, [&](int32_t u) { return items[((-1 - u) & ~kUnitMerged) * kItemsPerUnit]; });
  p->n_tiles = nt;
  p->n_items = (int)items.size();
  p->n_units = (int)units.size();
  p->n_groups = (int)groups.size();
  p->n_slots = slots;
  std::vector<int32_t> merge;
  for (int gi = 0; gi < p->n_groups; ++gi)
    for (int cb = 0; cb * 16 < groups[gi].npos * d.G; ++cb) merge.push_back(gi * 16 + cb);
  p->n_merge_units = (int)merge.size();

  int off = 0;
  p->off_tok_pos = off;  off += align16(T);
  p->off_tok_req = off;  off += align16(T);
  p->off_req_bt = off;   off += align16(R);
  p->off_bt = off;       off += align16(nbt);
  p->off_tiles = off;    off += align16(8 * nt);
  p->off_items = off;    off += align16(8 * p->n_items);
  p->off_units = off;    off += align16(p->n_units);
  p->off_groups = off;   off += align16(8 * p->n_groups);
  p->off_merge = off;    off += align16(p->n_merge_units);
  p->off_tile_shift = off;  off += p->windowed ? align16(2 * nt) : 0;
  p->off_item_shift = off;  off += p->windowed ? align16(2 * p->n_items) : 0;
  p->meta.assign(off, 0);
  int32_t* m = p->meta.data();
  int bt_off = 0;
  for (int r = 0; r < R; ++r) {
    for (int i = 0; i < rq[r].chunk_len; ++i) {
      m[p->off_tok_pos + tok_start[r] + i] = rq[r].context_len + i;
      m[p->off_tok_req + tok_start[r] + i] = r;
    }
    // dead blocks are left out: block i behind them stands at req_bt + i all the same
    const DeadBlocks dead = dead_blocks(win, rq[r].context_len);
    const int nb = (int)blocks_for((int64_t)rq[r].context_len + rq[r].chunk_len);
    m[p->off_req_bt + r] = bt_off - dead.count;
    int32_t* bt = m + p->off_bt + bt_off;
    std::memcpy(bt, rq[r].block_table, sizeof(int32_t) * dead.first);
    std::memcpy(bt + dead.first, rq[r].block_table + dead.first + dead.count,
                sizeof(int32_t) * (nb - dead.first - dead.count));
    for (int i = 0; i < kBtPad; ++i) bt[nb - dead.count + i] = rq[r].block_table[nb - 1];
    bt_off += nb - dead.count + kBtPad;
  }
  if (p->windowed) {
    // a unit's first row: its token's position tells its own gap
    auto shifts = [&](const std::vector<AttnItem>& v, int at) {
      for (size_t i = 0; i < v.size(); ++i) {
        const int x = rq[v[i].req].context_len, pos = x + v[i].tok0 - tok_start[v[i].req];
        m[at + 2 * i] = dead_blocks(win, x).count;
        m[at + 2 * i + 1] = dead_blocks(win, pos).count;
      }
    };
    shifts(tiles, p->off_tile_shift);
    shifts(items, p->off_item_shift);
  }
  if (nt) std::memcpy(m + p->off_tiles, tiles.data(), sizeof(AttnItem) * nt);
  if (!items.empty()) std::memcpy(m + p->off_items, items.data(), sizeof(AttnItem) * items.size());
  if (!units.empty()) std::memcpy(m + p->off_units, units.data(), sizeof(int32_t) * units.size());
  if (!groups.empty()) std::memcpy(m + p->off_groups, groups.data(), sizeof(MergeGroup) * groups.size());
  if (!merge.empty()) std::memcpy(m + p->off_merge, merge.data(), sizeof(int32_t) * merge.size());
  iteration_work(d, rq, R, &p->flops, &p->bytes, win);
}

void build_records(const Plan& p, RecordPlan* out) {
  const int32_t* m = p.meta.data();
  const int n_bt = p.off_tiles - p.off_bt;  // with its padding
  int off = 16 * 4 * p.n_units;
  out->off_bt = off;     off += n_bt;
  out->off_merge = off;  off += align16(8 * p.n_merge_units);
  out->meta.assign(off, 0);
  if (off == 0) return;
  int32_t* o = out->meta.data();
  std::memcpy(o + out->off_bt, m + p.off_bt, sizeof(int32_t) * n_bt);
  const MergeGroup* groups = reinterpret_cast<const MergeGroup*>(m + p.off_groups);
  MergeGroup* merge = reinterpret_cast<MergeGroup*>(o + out->off_merge);
  for (int i = 0; i < p.n_merge_units; ++i) {
    const int mu = m[p.off_merge + i];
    merge[i] = groups[mu >> 4];
    merge[i].cols = mu & 15;
  }
  UnitRec* rec = reinterpret_cast<UnitRec*>(o);
  const AttnItem* tiles = reinterpret_cast<const AttnItem*>(m + p.off_tiles);
  const AttnItem* items = reinterpret_cast<const AttnItem*>(m + p.off_items);
  for (int u = 0; u < p.n_units; ++u) {
    const int code = m[p.off_units + u];
    const bool tile = code >= 0;
    const int unit = tile ? code : (-1 - code) & ~kUnitMerged;
    for (int w = 0; w < kItemsPerUnit; ++w) {
      UnitRec& r = rec[kItemsPerUnit * u + w];
      const int i = tile ? unit : kItemsPerUnit * unit + w;
      r.item = tile ? tiles[i] : items[i];
      r.kind = tile ? kRecTile : ((-1 - code) & kUnitMerged) ? kRecMerged : kRecSingle;
      r.sink = r.window = m[p.off_req_bt + r.item.req];
      if (p.windowed) {
        const int32_t* s = m + (tile ? p.off_tile_shift : p.off_item_shift) + 2 * i;
        r.sink += s[0];
        r.window += s[1];
      }
      if (r.item.kv_begin >= r.item.kv_end) continue;  // an empty item reads nothing
      const int first = r.item.kv_begin / 16, last = (r.item.kv_end - 1) / 16;
      for (int k = 0; k < 4; ++k) {
        const int b = std::min(last, first + (tile ? 2 * k + (w & 1) : k));
        r.ids[k] = m[p.off_bt + b + (b < p.sink_blocks ? r.sink : r.window)];
      }
    }
  }
}

}  // namespace hb

using namespace hb;

extern "C" hb_status hb_plan_compaction(int32_t num_blocks, int32_t* const* tables, const int32_t* n_blocks,
                                        int32_t n_tables, int32_t* src, int32_t* dst, int32_t* n_moves,
                                        int32_t* n_used) {
  try {
    return plan_compaction(num_blocks, tables, n_blocks, n_tables, src, dst, n_moves, n_used);
  } catch (const std::bad_alloc&) {
    return host_oom();
  }
}

extern "C" hb_status hb_window_dead_blocks(int32_t context_len, int32_t window, int32_t sinks, int32_t* first,
                                           int32_t* count) {
  if (!first || !count) return fail(HB_ERR_INVALID, "null first or count");
  if (context_len < 0) return fail(HB_ERR_INVALID, "context_len %d < 0", context_len);
  const hb_status st = check_window_args(window, sinks);
  if (st != HB_OK) return st;
  const DeadBlocks b = dead_blocks({window, sinks}, context_len);
  *first = b.first;
  *count = b.count;
  return HB_OK;
}
