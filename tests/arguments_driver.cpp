// The argument checks of hb_run_append, hb_set_attention_rope and hb_sample, which
// make no HIP call. Reads lines and prints the status of each:
//   append nq nkv hd num_blocks T pool_blocks k_pool v_pool q qs k ks v vs out outs
//   rope head_dim rotary layout magnitude frequency (the last one's; the others are 1) null
//   sample max_rows vocab n dtype logits stride temperature top_k top_p min_p u tokens probs
// Addresses are numbers, never dereferenced.
#include <cstdio>
#include <cstring>
#include <vector>

#include "hb_plan.h"

using namespace hb;

int main() {
  char what[16];
  while (scanf("%15s", what) == 1) {
    if (!strcmp(what, "append")) {
      Dims d;
      int nb, T;
      hb_kv_pool pool{};
      unsigned long long kp, vp, at[4];
      long long st[4];
      if (scanf("%d %d %d %d %d %d %llu %llu", &d.nq, &d.nkv, &d.hd, &nb, &T, &pool.num_blocks, &kp, &vp) != 8) return 1;
      for (int i = 0; i < 4; ++i)
        if (scanf("%llu %lld", &at[i], &st[i]) != 2) return 1;
      pool.k_pool = (void*)kp;
      pool.v_pool = (void*)vp;
      const int64_t row = (int64_t)d.nq * d.hd, kv = (int64_t)d.nkv * d.hd;
      printf("%d\n", check_append(d, nb, T, &pool, {at[0], st[0], row}, {at[1], st[1], kv}, {at[2], st[2], kv},
                                  {at[3], st[3], row}));
    } else if (!strcmp(what, "rope")) {
      int hd, rotary, layout, null;
      double magnitude, f;
      if (scanf("%d %d %d %lf %lf %d", &hd, &rotary, &layout, &magnitude, &f, &null) != 6) return 1;
      std::vector<double> fs(rotary > 1 ? rotary / 2 : 1, 1.0);
      fs.back() = f;
      printf("%d\n", check_rope(hd, rotary, layout, null ? nullptr : fs.data(), magnitude));
    } else {
      hb_sample_desc s{};
      int rows, vocab;
      unsigned long long p[8];
      long long stride;
      if (scanf("%d %d %d %d %llu %lld", &rows, &vocab, &s.n_rows, &s.logits_dtype, &p[0], &stride) != 6) return 1;
      for (int i = 1; i < 8; ++i)
        if (scanf("%llu", &p[i]) != 1) return 1;
      s.logits = (void*)p[0];
      s.row_stride = stride;
      s.temperature = (float*)p[1];
      s.top_k = (int32_t*)p[2];
      s.top_p = (float*)p[3];
      s.min_p = (float*)p[4];
      s.u = (float*)p[5];
      s.tokens = (int32_t*)p[6];
      s.probs = (float*)p[7];
      printf("%d\n", check_sample(rows, vocab, &s));
    }
  }
  return 0;
}
