// Host-only parts of daso_block.h: argument checks, and how the tensors of a clipping are cut.
#include "daso_block_host.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "daso_check.h"

namespace daso {
namespace host {
namespace {

// A buffer as rows that do not overlap, twice: as its tokens' (or its heads') rows whole, and, where all (token, head) rows
// lie a multiple of one distance apart, as those rows themselves (else as the first).  And the distances of neighbouring tokens
// and heads, 0 where there is one of them.
struct Rows {
  Block whole, each;
  int64_t token, head;
};
Rows line(const void* p, int64_t n, size_t esz) { return {flat(p, n, esz), flat(p, n, esz), 0, 0}; }

// Whether the rows lie as daso_heads says, and how.
bool rows_of_heads(const daso_heads& h, int64_t tokens, int64_t heads, int64_t dim, size_t esz, Rows* to) {
  const int64_t most = kMaxElems / (tokens * heads);
  const int64_t ts = tokens > 1 ? h.token_stride : 0, hs = heads > 1 ? h.head_stride : 0;
  if (ts < 0 || hs < 0 || ts > most || hs > most) return false;
  if ((tokens > 1 && ts < dim) || (heads > 1 && hs < dim)) return false;
  const int64_t token = (heads - 1) * hs + dim, head = (tokens - 1) * ts + dim;
  if (tokens == 1 || ts >= token) to->whole = rows_of(h.data, tokens, ts, token, esz);
  else if (heads == 1 || hs >= head) to->whole = rows_of(h.data, heads, hs, head, esz);
  else return false;
  to->each = to->whole, to->token = ts, to->head = hs;
  if (heads > 1 && tokens > 1 && ts % hs == 0) to->each = rows_of(h.data, tokens * heads, hs, dim, esz);
  else if (heads > 1 && tokens > 1 && hs % ts == 0) to->each = rows_of(h.data, tokens * heads, ts, dim, esz);
  return true;
}

bool meet(const Rows& a, const Rows& b) { return overlap(a.whole, b.whole) && !beside(a.each, b.each); }

// The same rows for the same tokens and heads.  (Both distances: with as many tokens as heads a buffer with the two
// exchanged has the same rows, which are other tokens'.)
bool same_rows(const Rows& a, const Rows& b) {
  return a.whole.p == b.whole.p && a.whole.esz == b.whole.esz && a.token == b.token && a.head == b.head;
}

// Outputs against inputs and each other.  The first `in_place` outputs may be the input of the same number, row for row.
int check_rows(std::initializer_list<Rows> outputs, std::initializer_list<Rows> inputs, int in_place) {
  int k = 0;
  for (const Rows* o = outputs.begin(); o != outputs.end(); ++o, ++k) {
    int i = 0;
    for (const Rows& in : inputs) {
      const bool allowed = i == k && k < in_place && same_rows(*o, in);
      if (!allowed && meet(*o, in)) return DASO_EALIAS;
      ++i;
    }
    for (const Rows* p = outputs.begin(); p != o; ++p)
      if (meet(*o, *p)) return DASO_EALIAS;
  }
  return DASO_OK;
}

int need_all(std::initializer_list<Rows> rows) {
  for (const Rows& r : rows)
    if (const int rc = need(r.whole)) return rc;
  return DASO_OK;
}

bool heads_ok(int32_t heads) { return heads >= 1 && heads <= DASO_MAX_HEADS; }
bool dim_ok(int32_t dim) { return dim >= 8 && dim <= DASO_MAX_HEAD_DIM && dim % 8 == 0; }

}  // namespace

// ------------------------------------------------------------------------- norm and rotation
int check_rotary_sizes(const daso_rotary_args& s) {
  if (s.tokens < 0 || s.tokens > DASO_MAX_TOKENS || !heads_ok(s.heads) || !heads_ok(s.kv_heads) || !dim_ok(s.dim) || !known(s.type))
    return DASO_EINVAL;
  if (s.rotated < 0 || s.rotated > s.dim || s.rotated % 8 != 0 || !finite_not_negative(s.eps)) return DASO_EINVAL;
  return (s.flags & ~DASO_ROTARY_INTERLEAVED) != 0 || s.reserved != 0 ? DASO_EINVAL : DASO_OK;
}

int check_rotary(const daso_rotary_args& s, bool backward) {
  int rc = check_rotary_sizes(s);
  if (rc != DASO_OK) return rc;
  const Rows qw = line(s.q_weight, s.dim, 4), kw = line(s.k_weight, s.dim, 4);
  const Rows dqw = line(backward ? s.dq_weight : nullptr, s.dim, 4), dkw = line(backward ? s.dk_weight : nullptr, s.dim, 4);
  if ((rc = first({need(dqw.whole, true), need(dkw.whole, true)})) != DASO_OK) return rc;
  if (s.tokens == 0) return check_rows({dqw, dkw}, {}, 0);
  const size_t e = bytes_of(s.type);
  Rows q, k, q_to, k_to, dq, dk;
  const auto heads = [&](const daso_heads& h, int32_t count, Rows* to) { return rows_of_heads(h, s.tokens, count, s.dim, e, to); };
  if (!heads(s.q, s.heads, &q) || !heads(s.k, s.kv_heads, &k)) return DASO_EINVAL;
  const Rows at = line(s.positions, s.tokens, 8), f = line(s.frequencies, s.rotated / 2, 8);
  rc = first({need(q.whole), need(k.whole), need(at.whole), need(f.whole, s.rotated == 0), need(qw.whole, true), need(kw.whole, true)});
  if (rc != DASO_OK) return rc;
  if (!backward) {
    if (!heads(s.q_out, s.heads, &q_to) || !heads(s.k_out, s.kv_heads, &k_to)) return DASO_EINVAL;
    if ((rc = need_all({q_to, k_to})) != DASO_OK) return rc;
    return check_rows({q_to, k_to}, {q, k, at, f, qw, kw}, 2);
  }
  if (!heads(s.dq_out, s.heads, &dq) || !heads(s.dk_out, s.kv_heads, &dk) || !heads(s.dq, s.heads, &q_to) ||
      !heads(s.dk, s.kv_heads, &k_to))
    return DASO_EINVAL;
  if ((rc = need_all({dq, dk, q_to, k_to})) != DASO_OK) return rc;
  return check_rows({q_to, k_to, dqw, dkw}, {dq, dk, q, k, at, f, qw, kw}, 2);
}

// ------------------------------------------------------------------------- attention
int check_attention_sizes(const daso_attention_args& s) {
  if (s.tokens < 0 || s.tokens > DASO_MAX_TOKENS || !heads_ok(s.heads) || !heads_ok(s.kv_heads) || s.heads % s.kv_heads != 0)
    return DASO_EINVAL;
  if (!dim_ok(s.dim) || !known(s.type) || !(s.scale > 0.0f) || !std::isfinite(2.0f * s.scale)) return DASO_EINVAL;
  if ((s.flags & ~(DASO_ATTENTION_CAUSAL | DASO_ATTENTION_ZERO_Q | DASO_ATTENTION_ZERO_K | DASO_ATTENTION_ZERO_V)) != 0 || s.reserved != 0 || s.sequences < 0 || s.sequences > DASO_MAX_SEQUENCES)
    return DASO_EINVAL;
  return (s.tokens / 32 + s.sequences) * s.heads < (int64_t(1) << 23) ? DASO_OK : DASO_EINVAL;
}

int check_attention(const daso_attention_args& s, bool backward) {
  int rc = check_attention_sizes(s);
  if (rc != DASO_OK) return rc;
  if (s.tokens == 0 || (s.sequences == 0 && s.offsets == nullptr)) return DASO_OK;
  if (s.offsets == nullptr && s.sequences != 1) return DASO_EINVAL;
  const size_t e = bytes_of(s.type);
  Rows q, k, v, out, dout, dq, dk, dv;
  const auto heads = [&](const daso_heads& h, int32_t count, Rows* to) {
    return (s.tokens <= 1 || h.token_stride <= kMaxTokenStride) && rows_of_heads(h, s.tokens, count, s.dim, e, to);
  };
  if (!heads(s.q, s.heads, &q) || !heads(s.k, s.kv_heads, &k) || !heads(s.v, s.kv_heads, &v) || !heads(s.out, s.heads, &out))
    return DASO_EINVAL;
  const Rows at = line(s.offsets, int64_t(s.sequences) + 1, 8), lse = line(s.lse, s.tokens * s.heads, 4);
  if ((rc = first({need_all({q, k, v, out, lse}), need(at.whole, true)})) != DASO_OK) return rc;
  if (!backward) return check_rows({out, lse}, {q, k, v, at}, 0);
  if (!heads(s.dout, s.heads, &dout) || !heads(s.dq, s.heads, &dq) || !heads(s.dk, s.kv_heads, &dk) || !heads(s.dv, s.kv_heads, &dv))
    return DASO_EINVAL;
  if ((rc = need_all({dout, dq, dk, dv})) != DASO_OK) return rc;
  return check_rows({dq, dk, dv}, {q, k, v, out, dout, lse, at}, 0);
}

// ------------------------------------------------------------------------- clipping
int check_clip_sizes(const daso_clip_args& s) {
  if (s.n < 0 || s.n > DASO_MAX_N || s.g < 1 || s.g > DASO_MAX_G || s.ntensors < 0 || (s.ntensors > 0 && s.tensors == nullptr))
    return DASO_EINVAL;
  int64_t at = 0;
  for (int32_t t = 0; t < s.ntensors; ++t) {
    const daso_span& span = s.tensors[t];
    if (span.start < at || span.start > s.n || span.n < 0 || span.n > s.n - span.start) return DASO_EINVAL;
    at = span.start + span.n;
  }
  return s.n / kPiece + 2 * int64_t(s.ntensors) < kMostPieces ? DASO_OK : DASO_EINVAL;
}

int check_clip(const daso_clip_args& s) {
  int rc = check_clip_sizes(s);
  if (rc != DASO_OK) return rc;
  if (!finite_not_negative(s.eps) || !(s.max_norm >= 0.0f)) return DASO_EINVAL;
  const int64_t norms = s.ntensors > 0 ? s.ntensors : 1;
  const Rows out = line(s.out, s.n, 4), norm = line(s.norm, 1, 4), each = line(s.norms, norms, 4);
  if ((rc = first({need(norm.whole), need(each.whole, true)})) != DASO_OK) return rc;
  if (s.n == 0) return check_rows({norm, each}, {}, 0);
  if (s.grads == nullptr) return DASO_EINVAL;
  for (int32_t r = 0; r < s.g; ++r) {
    if (s.grads[r] == nullptr) return DASO_EINVAL;
    if (!aligned(s.grads[r], 16)) return DASO_EALIGN;
    const Rows in = line(s.grads[r], s.n, 4);
    if (meet(norm, in) || meet(each, in) || (s.out != s.grads[r] && meet(out, in))) return DASO_EALIAS;
  }
  if (!aligned(s.out, 16)) return DASO_EALIGN;
  return check_rows({out, norm, each}, {}, 0);
}

int64_t pieces_of(const daso_clip_args& s) {
  if (s.ntensors == 0) return pieces_of(daso_span{0, s.n});
  int64_t pieces = 0;
  for (int32_t t = 0; t < s.ntensors; ++t) pieces += pieces_of(s.tensors[t]);
  return pieces;
}

int32_t fill_table(const daso_clip_args& s, int32_t tensor, bool merged, ClipTable* table) {
  const daso_span whole = {0, s.n};
  const daso_span* spans = s.ntensors > 0 ? s.tensors : &whole;
  const int32_t count = s.ntensors > 0 ? s.ntensors : 1;
  ClipTable& t = *table;
  t.tensor = tensor, t.runs = 0;
  t.bound[0] = spans[tensor].start, t.first[0] = 0;
  int32_t taken = 0;
  const auto run = [&t](int64_t end, int64_t pieces, int32_t number) {
    t.number[t.runs] = static_cast<int16_t>(number);
    t.bound[t.runs + 1] = end, t.first[t.runs + 1] = t.first[t.runs] + static_cast<int32_t>(pieces);
    ++t.runs;
  };
  for (; tensor + taken < count; ++taken) {
    const daso_span& span = spans[tensor + taken];
    const bool gap = span.start != t.bound[t.runs];
    if (merged && !gap && taken > 0) {
      const daso_span grown = {t.bound[t.runs - 1], span.start + span.n - t.bound[t.runs - 1]};
      t.bound[t.runs] = span.start + span.n;
      t.first[t.runs] = t.first[t.runs - 1] + static_cast<int32_t>(pieces_of(grown));
      continue;
    }
    if (t.runs + (gap ? 2 : 1) > kClipRuns) break;
    if (gap) run(span.start, 0, -1);
    run(span.start + span.n, pieces_of(span), taken);
  }
  return taken;
}

}  // namespace host
}  // namespace daso
