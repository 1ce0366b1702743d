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
                         int64_t* n_tokens, const std::vector<int>* skip) {
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
    const DeadBlocks dead = skip ? DeadBlocks{0, (*skip)[r]} : dead_blocks(w, q.context_len);
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
  return check_slots(num_blocks, desc->requests, R, T, marks);
}

hb_status check_slots(int num_blocks, const hb_request* requests, int n, int64_t n_tokens, SlotMarks* marks) {
  hb_status st = HB_OK;
  SlotMarks local;
  SlotMarks* m = marks ? marks : &local;
  if ((int)m->mask.size() < num_blocks) m->mask.assign(num_blocks, 0);
  m->touched.clear();
  m->touched.reserve(n_tokens);  // nothing can fail while marks stand
  for (int r = 0; r < n && st == HB_OK; ++r) {
    const hb_request& q = requests[r];
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

hb_status check_shared(const Dims& d, int num_blocks, const hb_request* requests, int n, const hb_prefix_group* groups,
                       int n_groups, int64_t* n_tokens) {
  if (n < 0) return fail(HB_ERR_INVALID, "n_requests < 0");
  if (n > d.max_R) return fail(HB_ERR_INVALID, "n_requests %d exceeds max_requests %d", n, d.max_R);
  if (n_groups < 0 || (n_groups > 0 && !groups)) return fail(HB_ERR_INVALID, "n_groups < 0 or null groups");
  std::vector<int> skip(n, 0);
  int next = 0;
  for (int i = 0; i < n_groups; ++i) {
    const hb_prefix_group& g = groups[i];
    if (g.count < 1 || g.first < next || g.first > n - g.count)
      return fail(HB_ERR_INVALID, "group %d: requests [%d, %d + %d) are empty, outside the batch or in or before group %d's",
                  i, g.first, g.first, g.count, i - 1);
    if (g.prefix_len < 0 || g.prefix_len % 16)
      return fail(HB_ERR_INVALID, "group %d: prefix_len %d is no multiple of 16", i, g.prefix_len);
    next = g.first + g.count;
    if (!requests) break;  // (refused below)
    for (int r = g.first; r < next; ++r) {
      if (requests[r].context_len < g.prefix_len)
        return fail(HB_ERR_INVALID, "request %d: context_len %d below its group's prefix_len %d", r,
                    requests[r].context_len, g.prefix_len);
      if (r > g.first) skip[r] = g.prefix_len / 16;
    }
  }
  const hb_status st = check_requests(d, num_blocks, requests, n, Window(), n_tokens, &skip);
  if (st != HB_OK) return st;
  for (int i = 0; i < n_groups; ++i)
    for (int r = groups[i].first + 1; r < groups[i].first + groups[i].count; ++r)
      if (std::memcmp(requests[r].block_table, requests[groups[i].first].block_table,
                      sizeof(int32_t) * (groups[i].prefix_len / 16)) != 0)
        return fail(HB_ERR_INVALID, "request %d: its first %d blocks are not those of request %d, of its group", r,
                    groups[i].prefix_len / 16, groups[i].first);
  return HB_OK;
}

static hb_status check_rows(const char* name, const Rows& r) {
  if (r.stride < r.width || r.stride % 8 || r.stride > (int64_t)1 << 40)
    return fail(HB_ERR_INVALID, "%s: row stride %lld: a multiple of 8 from %lld to 2^40", name, (long long)r.stride,
                (long long)r.width);
  if (r.at % 16) return fail(HB_ERR_INVALID, "%s must be 16-byte aligned", name);
  return HB_OK;
}

// Whether some row of the one shares memory with some row of the other. (Rows of
// different strides that reach into each other's range are taken to.)
static bool rows_overlap(const Rows& x, const Rows& y, int T) {
  if (x.at >= y.end(T) || y.at >= x.end(T)) return false;
  if (x.stride != y.stride || T == 1) return true;
  const uintptr_t s = (uintptr_t)x.stride * 2, d = y.at >= x.at ? (y.at - x.at) % s : s - 1 - (x.at - y.at - 1) % s;
  return d < (uintptr_t)x.width * 2 || d + (uintptr_t)y.width * 2 > s;
}

hb_status check_append(const Dims& d, int num_blocks, int T, const hb_kv_pool* pool, const Rows& q, const Rows& k,
                       const Rows& v, const Rows& out) {
  if (!pool || !pool->k_pool || !pool->v_pool || !q.at || !k.at || !v.at || !out.at)
    return fail(HB_ERR_INVALID, "null pool, q, k, v or q_out");
  if (pool->num_blocks < num_blocks)
    return fail(HB_ERR_INVALID, "pool of %d blocks, the plan's tables are over %d", pool->num_blocks, num_blocks);
  const struct {
    const char* name;
    const Rows& rows;
  } all[] = {{"q", q}, {"k", k}, {"v", v}, {"q_out", out}};
  for (const auto& r : all) {
    const hb_status st = check_rows(r.name, r.rows);
    if (st != HB_OK) return st;
  }
  const uintptr_t kp = (uintptr_t)pool->k_pool, vp = (uintptr_t)pool->v_pool;
  const uintptr_t bytes = (uintptr_t)pool->num_blocks * d.nkv * 16 * d.hd * 2;
  if (kp % 16 || vp % 16) return fail(HB_ERR_INVALID, "pools must be 16-byte aligned");
  if (kp < vp + bytes && vp < kp + bytes) return fail(HB_ERR_INVALID, "the pools overlap");
  for (const auto& r : all)
    for (const uintptr_t p : {kp, vp})
      if (p < r.rows.end(T) && r.rows.at < p + bytes) return fail(HB_ERR_INVALID, "%s overlaps a pool", r.name);
  const bool in_place = out.at == q.at && (out.stride == q.stride || T == 1);
  if ((!in_place && rows_overlap(out, q, T)) || rows_overlap(out, k, T) || rows_overlap(out, v, T))
    return fail(HB_ERR_INVALID, "q_out overlaps k, v or part of q");
  return HB_OK;
}

hb_status check_rope(int head_dim, int rotary_dim, int layout, const double* inv_freq, double magnitude) {
  if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 16)
    return fail(HB_ERR_UNSUPPORTED, "rotary_dim %d: a multiple of 16 up to %d", rotary_dim, head_dim);
  if (layout != HB_ROPE_HALF && layout != HB_ROPE_INTERLEAVED) return fail(HB_ERR_INVALID, "unknown rotary layout %d", layout);
  if (rotary_dim > 0 && !inv_freq) return fail(HB_ERR_INVALID, "null inv_freq");
  if (!(magnitude >= 0 && std::isfinite((float)magnitude))) return fail(HB_ERR_INVALID, "magnitude %g", magnitude);
  for (int j = 0; j < rotary_dim / 2; ++j)
    if (!(inv_freq[j] >= 0 && inv_freq[j] <= 1 << 20)) return fail(HB_ERR_INVALID, "inv_freq[%d] = %g", j, inv_freq[j]);
  return HB_OK;
}

hb_status check_sample(int max_rows, int vocab, const hb_sample_desc* d) {
  if (!d) return fail(HB_ERR_INVALID, "null sample descriptor");
  const int n = d->n_rows;
  if (n < 0 || n > max_rows) return fail(HB_ERR_INVALID, "n_rows %d outside [0, %d]", n, max_rows);
  if (d->logits_dtype != HB_OUT_F32 && d->logits_dtype != HB_OUT_BF16)
    return fail(HB_ERR_INVALID, "logits_dtype must be HB_OUT_F32 or HB_OUT_BF16");
  if (n == 0) return HB_OK;
  if (!d->logits || !d->u || !d->tokens) return fail(HB_ERR_INVALID, "null logits, u or tokens");
  if (d->row_stride < vocab || d->row_stride > (int64_t)1 << 40)
    return fail(HB_ERR_INVALID, "row stride %lld: from %d to 2^40", (long long)d->row_stride, vocab);
  const uintptr_t size = d->logits_dtype == HB_OUT_F32 ? 4 : 2, x = (uintptr_t)d->logits, m = 4 * (uintptr_t)n;
  struct Range {
    uintptr_t at, bytes;
  };
  const Range in[] = {{x, ((uintptr_t)(n - 1) * d->row_stride + vocab) * size}, {(uintptr_t)d->u, m},
                      {(uintptr_t)d->temperature, m}, {(uintptr_t)d->top_k, m},
                      {(uintptr_t)d->top_p, m}, {(uintptr_t)d->min_p, m}};
  const Range out[] = {{(uintptr_t)d->tokens, m}, {(uintptr_t)d->probs, m}};
  auto overlap = [](const Range& a, const Range& b) {
    return a.at && b.at && a.at < b.at + b.bytes && b.at < a.at + a.bytes;
  };
  if (x % size) return fail(HB_ERR_INVALID, "misaligned logits");
  for (int i = 1; i < 6; ++i)
    if (in[i].at % 4) return fail(HB_ERR_INVALID, "misaligned u or settings");
  for (const Range& o : out) {
    if (o.at % 4) return fail(HB_ERR_INVALID, "misaligned tokens or probs");
    for (const Range& i : in)
      if (overlap(o, i)) return fail(HB_ERR_INVALID, "tokens or probs overlap an input");
  }
  if (overlap(out[0], out[1])) return fail(HB_ERR_INVALID, "tokens and probs overlap");
  return HB_OK;
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
// 900 17.4 -> 12.6). Each group goes to the die with the most room, the rest of it to
// the next. (Tiles share a key range four times less often: even
// with cold caches, 19.8 -> 23.2 us with warm ones, 64 tiles of 1000 keys.)
constexpr int kDies = 8;
// units[at[i]] are dealt anew over the places `at`, group by group: the largest first,
// which then lie whole on one die, or in the order in which they stand.
template <typename F>
static void by_die(std::vector<int32_t>* units, const std::vector<int>& at, bool largest_first, F&& item_of) {
  std::map<std::tuple<int, int, int>, int> known;
  std::vector<std::vector<int32_t>> groups;
  std::vector<int> places[kDies];
  for (const int i : at) {
    const int32_t u = (*units)[i];
    const AttnItem it = item_of(u);
    const auto found = known.insert({{it.req, it.kv_head, it.kv_begin}, (int)groups.size()}).first;
    if (found->second == (int)groups.size()) groups.emplace_back();
    groups[found->second].push_back(u);
    places[i % kDies].push_back(i);
  }
  if (largest_first)
    std::stable_sort(groups.begin(), groups.end(), [](const auto& a, const auto& b) { return a.size() > b.size(); });
  size_t next[kDies] = {}, room[kDies];
  for (int x = 0; x < kDies; ++x) room[x] = places[x].size();
  for (const auto& group : groups) {
    int x = 0;
    size_t left = 0;
    for (const int32_t u : group) {
      if (left == 0) {
        x = (int)(std::max_element(room, room + kDies) - room);
        left = room[x];
      }
      (*units)[places[x][next[x]++]] = u;
      --room[x];
      --left;
    }
  }
}

namespace {
// Rows that read one key range of one block table: a request's own, or those of
// consecutive requests over the prefix that they share.
struct Span {
  int r, tok0, rows;
  int x;    // position of the first row
  int lo;   // first key
  int end;  // end of the keys, every one of which each row sees; or -1: a row's keys end with itself
  int run;  // the shared run whose parts these rows leave, or -1
};
// Consecutive requests whose prefix is read for all of them at once. Column
// slots: part s of a column (row, head) of kv head g is slot
// base + (g parts + s) columns + column, the prefix's parts first.
struct Run {
  int first, count, len, rows;
  int prefix_parts = 0, parts = 0;
  int64_t base = 0;
};

// The requests of a group that are joined, as runs of consecutive ones. Joined rows
// need the merge kernel (2.5 to 3 us); requests alone need it from some 600 keys on, or
// where launches are large. So joining pays from 1024 shared keys on (cold caches, one
// call, alone / joined: 2 decodes of 8B heads behind 512 keys 6.9 / 9.6 us, 1024 10.3 /
// 9.1, 8192 13.8 / 12.6; 64 behind 1024 19.2 / 16.2, 8192 137 / 24) or where it saves
// as many K and V bytes as these take to read (64 behind 512: eight kv heads, 132 MB,
// 13.3 / 15.3; sixteen, 264 MB, 19.3 / 16.6). The rule looks at neither rows nor heads: over 504
// batches of one group (2 to 200 requests of 1 or 5 rows, prefixes of 1024 to 16384, seven
// sets of heads) joined takes 0.026 to 1.39 times as long, more than 1.05 in 24, at most 6.4 us
// more (three requests of 5 rows, 8B heads, 16384 keys 41.3 / 47.7; 64 decodes of one kv head
// of 16 behind 6000 15.8 / 22.0; 16 decodes of twelve heads of 64 behind 1024 8.6 / 11.1).
constexpr int kSharedKeys = 1024;
constexpr double kSharedBytes = 192e6;
std::vector<Run> shared_runs(const Dims& d, const hb_request* rq, const PlanOptions& opt) {
  std::vector<Run> runs;
  for (int i = 0; i < opt.n_groups; ++i) {
    const hb_prefix_group& g = opt.groups[i];
    int rows = 0, first = g.first;
    auto close = [&](int end) {
      const double saved = (end - first - 1.0) * g.prefix_len * 4 * d.nkv * d.hd;
      if (end - first > 1 && g.prefix_len > 0 && (opt.share_all || g.prefix_len >= kSharedKeys || saved >= kSharedBytes))
        runs.push_back({first, end - first, g.prefix_len, rows});
      first = end + 1;
      rows = 0;
    };
    for (int r = g.first; r < g.first + g.count; ++r) {
      if ((int64_t)rq[r].chunk_len * d.G >= kTileCols / 2) close(r);  // fills its own tiles: nothing to share
      else rows += rq[r].chunk_len;
    }
    close(g.first + g.count);
  }
  return runs;
}
}  // namespace

void build_plan(const Dims& d, const hb_batch_desc* desc, int cu_count, Plan* p, const PlanOptions& opt) {
  const int R = desc->n_requests;
  const hb_request* rq = desc->requests;
  int T = 0, nbt = 0;
  std::vector<int> tok_start(R + 1, 0);
  const Window& win = opt.window;
  p->windowed = false;
  // table entries that are not uploaded: hidden by the window, or uploaded with the
  // first request of a shared run
  std::vector<DeadBlocks> absent(R);
  std::vector<Run> runs = shared_runs(d, rq, opt);
  for (int r = 0; r < R; ++r) absent[r] = dead_blocks(win, rq[r].context_len);
  for (const Run& u : runs)
    for (int r = u.first + 1; r < u.first + u.count; ++r) absent[r] = {0, u.len / 16};
  for (int r = 0; r < R; ++r) {
    tok_start[r] = T;
    T += rq[r].chunk_len;
    const int64_t kv = (int64_t)rq[r].context_len + rq[r].chunk_len;
    nbt += (int)blocks_for(kv) - absent[r].count + kBtPad;
    p->windowed |= win.window > 0 && kv - win.window > win.sinks;  // the last row's window hides a key
  }
  p->window = win;
  p->sink_blocks = p->windowed ? (win.sinks + 15) / 16 : 0;
  tok_start[R] = T;
  p->T = T;
  p->R = R;

  const int cus = std::max(1, cu_count);
  std::vector<Span> spans;
  spans.reserve(R + runs.size());
  for (int r = 0, u = 0; r < R; ++r) {
    if (u < (int)runs.size() && r == runs[u].first + runs[u].count) ++u;
    const bool joined = u < (int)runs.size() && r >= runs[u].first;
    if (joined && r == runs[u].first)
      spans.push_back({r, tok_start[r], runs[u].rows, runs[u].len, 0, runs[u].len, u});
    spans.push_back({r, tok_start[r], rq[r].chunk_len, rq[r].context_len, joined ? runs[u].len : 0, -1, joined ? u : -1});
  }
  // keys of the w rows from i0 on of a span
  auto range_len = [&](const Span& s, int i0, int w) {
    if (s.end >= 0) return s.end - s.lo;
    return s.x + std::min(s.rows, i0 + w) - s.lo - 16 * dead_blocks(win, s.x + i0).count;
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
  auto fills_tile = [&](const Span& s) { return (int64_t)s.rows * d.G >= kTileCols / 2; };
  bool items_only = false;
  int S_items = 0;
  p->paired = false;
  const bool fit_chunks = opt.fit_round && opt.split_tile <= 0 && opt.split_item <= 0;
  if (fit_chunks) {
    int64_t n = 0;
    bool chunks = false;
    for (const Span& s : spans) {
      n += (s.rows + d.P - 1) / d.P;
      chunks |= fills_tile(s);
    }
    if (chunks && n * d.nkv <= 2 * cus) {
      std::vector<int> all;
      for (const Span& s : spans)
        for (int i0 = 0; i0 < s.rows; i0 += d.P) all.push_back(range_len(s, i0, d.P));
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
  auto is_tile = [&](const Span& s) { return !items_only && fills_tile(s); };
  double tile_keys = 0, item_keys = 0;
  std::vector<int> item_lengths, tile_lengths;  // of one kv head
  for (const Span& s : spans) {
    const int w = is_tile(s) ? d.BQ : d.P;
    for (int i0 = 0; i0 < s.rows; i0 += w) {
      const int len = range_len(s, i0, w);
      (is_tile(s) ? tile_keys : item_keys) += (double)d.nkv * len;
      if (opt.fit_round) (is_tile(s) ? tile_lengths : item_lengths).push_back(len);
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
  // A shared prefix's tiles: as many pieces as make one for each CU, all tiles taken
  // together (cold caches, 8B heads: 64 decodes behind 8192 shared keys, 16 tiles, 16
  // pieces each 24.3 us, 8 29.6, 32 29.3; 256 behind 16384 and up to 1000 of their own,
  // 64 tiles, 4 pieces 127, 8 140, 6 146, 16 167), but, beside items, none shorter than
  // what takes 0.6 of their time (64 behind 8192 and up to 2000 of their own: 6 pieces
  // 55.2, 5 63.5, 8 58.5, 16 65.9), and no finer than other tiles' parts (fit_tile_split).
  auto prefix_split = [&](int keys) {
    const double finest = std::max(3.0 * std::sqrt((double)keys), tile_keys / cus);
    const double least = item_keys * 4.0 * d.hd / kItemBytesPerUs * 32.0;
    const int n = (int)std::max(1.0, std::min(std::floor(keys / finest + 1e-6), std::ceil(keys / std::max(least, 64.0))));
    return round_up((keys + n - 1) / n, 64);
  };
  auto tile_split = [&](const Span& s) { return s.end >= 0 && opt.split_tile <= 0 ? prefix_split(s.end - s.lo) : S_t; };

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
    int first, n, begin, end;  // its pieces are tiles[first .. first + n), over these keys
    bool shared;
  };
  std::vector<SplitTile> split_tiles;
  std::vector<MergeGroup> groups;
  int slots = 0;
  // units that a range of `len` keys takes one after the other (for a wave alone: one)
  auto parts_of = [&](bool tile, int len, int split) {
    const int nspl = (len + split - 1) / split;
    return tile ? nspl : len <= S_1 ? 1 : (nspl + kItemsPerUnit - 1) / kItemsPerUnit;
  };
  // slots of the shared runs, every unit of which leaves parts
  int64_t run_slots = 0;
  for (const Span& s : spans) {
    if (s.run < 0) continue;
    Run& u = runs[s.run];
    if (s.end >= 0) u.parts = u.prefix_parts = parts_of(is_tile(s), s.end - s.lo, is_tile(s) ? tile_split(s) : S_i);
    else u.parts = std::max(u.parts, u.prefix_parts + parts_of(false, range_len(s, s.rows - 1, 1), S_i));
  }
  int64_t run_rows = 0;
  for (Run& u : runs) {
    u.base = run_slots;
    run_slots += (int64_t)u.parts * u.rows * d.G * d.nkv;
    run_rows += (int64_t)u.rows * d.nkv;
  }
  p->too_many_slots = run_slots > 1 << 30 || run_rows > 1 << 26;  // (merge units have 27 bits for a group)
  if (p->too_many_slots) {
    p->n_slots = 0;
    return;
  }
  slots = (int)run_slots;
  for (const Span& sp : spans) {
    const int r = sp.r, c = sp.rows, x = sp.x;
    const bool tile = is_tile(sp);
    const int w = !tile ? d.P : p->half_tiles ? d.BQ / 2 : d.BQ, S = tile ? tile_split(sp) : S_i;
    for (int g = 0; g < d.nkv; ++g) {
      for (int i0 = 0; i0 < c; i0 += w) {
        const int npos = std::min(w, c - i0), tok0 = sp.tok0 + i0;
        const int gap = 16 * dead_blocks(win, x + i0).count;
        const int pos0 = sp.end >= 0 ? x : x + i0 - gap, kv_end = sp.end >= 0 ? sp.end : pos0 + npos;
        const int kv_len = kv_end - sp.lo;
        const int nspl = (kv_len + S - 1) / S, k = parts_of(tile, kv_len, S);
        // where the unit's parts go: the first one's slots, and those between two of them
        int part0 = -1, stride = 0;
        if (sp.run >= 0) {
          const Run& u = runs[sp.run];
          const int row0 = tok0 - tok_start[u.first];
          stride = u.rows * d.G;
          part0 = (int)(u.base + (int64_t)g * u.parts * stride) + row0 * d.G;
          if (sp.end < 0) {
            groups.push_back({part0, u.prefix_parts + k, stride, tok0, npos, g, 0, 0});
            part0 += u.prefix_parts * stride;
          }
        } else if (k > 1) {
          part0 = slots;
          stride = tile ? kTileCols : 16;
          groups.push_back({slots, k, stride, tok0, npos, g, 0, 0});
          slots += k * stride;
        }
        if (tile) {
          if (nspl > 1) split_tiles.push_back({(int)tiles.size(), nspl, sp.lo, kv_end, sp.end >= 0});
          for (int s = 0; s < nspl; ++s)
            tiles.push_back({r, g, tok0, pos0, npos, sp.lo + s * S, std::min(kv_end, sp.lo + (s + 1) * S),
                             part0 < 0 ? -1 : part0 + s * stride});
          continue;
        }
        if (kv_len <= S_1) {
          singles.push_back({r, g, tok0, pos0, npos, sp.lo, kv_end, part0});
          continue;
        }
        const int wlen = round_up((kv_len + k - 1) / k, 64);
        for (int j = 0; j < k; ++j) {
          const int b = sp.lo + j * wlen, e = std::min(kv_end, b + wlen);
          const int plen = round_up((e - b + kItemsPerUnit - 1) / kItemsPerUnit, 64);
          merged_units.push_back({plen, (int)merged_items.size(), true});
          for (int q = 0; q < kItemsPerUnit; ++q) {
            const int pb = std::min(e, b + q * plen), pe = std::min(e, pb + plen);
            merged_items.push_back({r, g, tok0, pos0, npos, pb, pe, part0 < 0 ? -1 : part0 + j * stride});
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
  // (A shared prefix's pieces are even always: pieces of one length keep their order,
  // in which those of the same keys go to one die.)
  const bool one_round = (int64_t)tiles.size() + item_unit_count <= 2 * (int64_t)std::max(1, cu_count);
  for (const SplitTile& st : split_tiles) {
    if (one_round || st.shared) {
      const int piece = round_up((st.end - st.begin + st.n - 1) / st.n, 64);
      for (int s = 0; s < st.n; ++s) {
        tiles[st.first + s].kv_begin = st.begin + s * piece;
        tiles[st.first + s].kv_end = std::min(st.end, st.begin + (s + 1) * piece);
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
  if (items_only || !runs.empty()) {
    // All item units, which are one round. Or the tiles of the shared prefixes, whose keys
    // many tiles read: among the places that they hold and the longest first as before, since
    // they are a queue with the other tiles (8B heads, cold caches, 64 decodes behind 8192 shared
    // keys and a chunk of 777 behind 5234, all split tiles dealt anew, the most read first: 217 us,
    // so 172; with a fresh chunk of 2048 102, 75).
    auto of_run = [&](const AttnItem& t) { return t.part >= 0 && t.part < run_slots; };
    std::vector<int> at;
    for (int i = 0; i < (int)units.size(); ++i)
      if (items_only || (units[i] >= 0 && of_run(tiles[units[i]]))) at.push_back(i);
    by_die(&units, at, items_only, [&](int32_t u) { return u >= 0 ? tiles[u] : items[((-1 - u) & ~kUnitMerged) * kItemsPerUnit]; });
  }
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
    // absent blocks are left out: block i behind them stands at req_bt + i all the same
    const DeadBlocks dead = absent[r];
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
  for (const Run& u : runs) p->bytes -= (u.count - 1.0) * u.len * 4 * d.nkv * d.hd;
}

int build_append(const hb_request* requests, int n, std::vector<int32_t>* out, int* off) {
  *off = align16((int)out->size());
  int units = 0;
  for (int r = 0; r < n; ++r)
    units += (requests[r].context_len + requests[r].chunk_len - 1) / 16 - requests[r].context_len / 16 + 1;
  out->resize((size_t)*off + align16(4 * units), 0);
  AppendUnit* u = reinterpret_cast<AppendUnit*>(out->data() + *off);
  int tok = 0;
  for (int r = 0; r < n; ++r) {
    const hb_request& q = requests[r];
    for (int p = q.context_len, end = p + q.chunk_len; p < end;) {
      const int m = std::min(end, (p & ~15) + 16) - p;
      *u++ = {tok, p, m, q.block_table[p / 16]};
      tok += m;
      p += m;
    }
  }
  return units;
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

extern "C" hb_status hb_rope_frequencies(int32_t rotary_dim, double theta, const hb_rope_scaling* scaling,
                                         double* inv_freq) {
  if (!inv_freq) return fail(HB_ERR_INVALID, "null inv_freq");
  if (rotary_dim < 0 || rotary_dim % 2) return fail(HB_ERR_INVALID, "rotary_dim %d: even, from 0 on", rotary_dim);
  if (!(theta > 1 && std::isfinite(theta))) return fail(HB_ERR_INVALID, "theta %g: above 1 and finite", theta);
  const hb_rope_scaling s = scaling ? *scaling : hb_rope_scaling{};
  if (s.kind != HB_ROPE_UNSCALED && s.kind != HB_ROPE_LINEAR && s.kind != HB_ROPE_BY_PARTS)
    return fail(HB_ERR_INVALID, "unknown scaling %d", s.kind);
  if (s.kind != HB_ROPE_UNSCALED && !(s.factor > 0 && std::isfinite(s.factor)))
    return fail(HB_ERR_INVALID, "scaling factor %g", s.factor);
  if (s.kind == HB_ROPE_BY_PARTS && !(s.original_context >= 1 && s.low >= 0 && s.low < s.high && std::isfinite(s.high)))
    return fail(HB_ERR_INVALID, "scaling by parts: original_context %d, low %g, high %g", s.original_context, s.low, s.high);
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const double f = std::pow(theta, -2.0 * j / rotary_dim);
    double g = s.kind == HB_ROPE_UNSCALED ? 1.0 : 0.0;  // share of the frequency that is not scaled
    if (s.kind == HB_ROPE_BY_PARTS)
      g = std::min(1.0, std::max(0.0, (s.original_context * f / 6.283185307179586 - s.low) / (s.high - s.low)));
    inv_freq[j] = g == 1.0 ? f : f * (g + (1.0 - g) / s.factor);
  }
  return HB_OK;
}
