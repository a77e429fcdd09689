// Attention of a batch whose sequences begin with the same text, held once as a sequence of an FP8
// cache of its own.
//
// The softmax over a row's keys is taken in two sets, the prefix's and the row's own:
// with (M, L, O) the maximum, the sum of exp(s - M) and the sum of those times the
// values of each set, the result is sum_i e^(M_i - M) O_i / sum_i e^(M_i - M) L_i.
// First launch: all rows of the batch against the prefix as if they were one sequence's,
// split over its keys, (M, L, O) of every part to the workspace; second launch: every
// sequence's rows over its own cache, which joins the parts as it finishes a row.
// The prefix's codes are read once for 16 or 32 rows of a kv head, not once a sequence.
#include "attention8.h"

namespace specdec {

namespace {

template <typename T>
hipError_t launch_typed(AttnArgs own, const SharedAttn& sh, hipStream_t s) {
  SharedParts parts{sh.o, sh.ml, sh.prefix.len + sh.b, sh.max_len, 1, 1};
  if (sh.max_len > 0) {
    AttnArgs a = own;
    a.f8 = sh.prefix;
    a.rps = own.M;
    a.max_ctx = sh.max_len;
    a.o_part = sh.o;
    a.ml_part = sh.ml;
    const Plan p = plan_of(a.rps, 1, a.n_heads, a.n_kv_heads, a.head_dim, a.max_ctx);
    if (p.parts > sh.parts) return hipErrorInvalidValue;  // (the caller has checked)
    parts.keys = p.per * chunk_of(a.head_dim);
    parts.stride = p.parts;
    const hipError_t e = launch_plan(a, p, 1, PrefixPass<T>{sh.b}, s);
    if (e != hipSuccess) return e;
  }
  const int B = own.M / own.rps;
  const Plan p = plan_of(own.rps, B, own.n_heads, own.n_kv_heads, own.head_dim, own.max_ctx);
  if (p.parts > own.n_split) return hipErrorInvalidValue;
  return launch_plan(own, p, B, OwnPass<T>{parts}, s);
}

}  // namespace

bool attention_shared_fits(int64_t rows, int n_heads, int n_kv_heads) {
  // (rows of a kv head are numbered below 2^20, see div_small)
  return rows * (n_heads / n_kv_heads) < 1 << 20 && attention8_fits((int)rows, 1, n_heads, n_kv_heads);
}

int attention_shared_parts(int rows, int n_heads, int n_kv_heads, int head_dim, int max_len, bool bf16) {
  return plan_of(rows, 1, n_heads, n_kv_heads, head_dim, max_len).parts;
}

hipError_t launch_attention_shared(const AttnArgs& own, const SharedAttn& sh, hipStream_t s) {
  return sh.bf16 ? launch_typed<uint16_t>(own, sh, s) : launch_typed<float>(own, sh, s);
}

}  // namespace specdec
