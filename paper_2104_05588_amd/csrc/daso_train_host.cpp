// Host-only parts of daso_train.h: argument checks and the plan of the Newton-Schulz rounds.
#include "daso_train_host.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <map>
#include <utility>

namespace daso {
namespace host {
namespace {

constexpr int64_t kMaxElems = DASO_MAX_N;

bool known(int32_t type) { return type == DASO_TYPE_F32 || type == DASO_TYPE_BF16; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// A buffer of `outer` blocks `outer_stride` apart, each of `rows` rows of `row` elements,
// `stride` apart.
struct Block {
  const void* p;
  int64_t outer, outer_stride, rows, stride, row;
  size_t esz;
};

Block rows_of(const void* p, int64_t rows, int64_t stride, int64_t row, size_t esz) {
  return {p, 1, 0, rows, stride, row, esz};
}
Block flat(const void* p, int64_t n, size_t esz) { return {p, 1, 0, 1, n, n, esz}; }

uintptr_t begin(const Block& b) { return reinterpret_cast<uintptr_t>(b.p); }
uintptr_t end(const Block& b) {
  if (b.outer == 0 || b.rows == 0 || b.row == 0) return begin(b);
  return begin(b) + static_cast<uintptr_t>((b.outer - 1) * b.outer_stride + (b.rows - 1) * b.stride + b.row) * b.esz;
}
// Rows the same distance apart, of which one buffer's lie beside the other's: columns of one wider buffer.
bool beside(const Block& a, const Block& b) {
  if (a.outer > 1 || b.outer > 1 || a.rows <= 1 || b.rows <= 1) return false;
  const uintptr_t apart = static_cast<uintptr_t>(a.stride) * a.esz;
  if (apart != static_cast<uintptr_t>(b.stride) * b.esz || apart == 0) return false;
  const uintptr_t behind = begin(b) >= begin(a) ? (begin(b) - begin(a)) % apart : (apart - (begin(a) - begin(b)) % apart) % apart;
  return behind >= static_cast<uintptr_t>(a.row) * a.esz && behind + static_cast<uintptr_t>(b.row) * b.esz <= apart;
}
// By their spans, but for such rows.
bool overlap(const Block& a, const Block& b) {
  return a.p != nullptr && b.p != nullptr && begin(a) < end(b) && begin(b) < end(a) && !beside(a, b);
}
bool same(const Block& a, const Block& b) {
  return a.p == b.p && a.esz == b.esz && (a.rows <= 1 || a.stride == b.stride) &&
         (a.outer <= 1 || a.outer_stride == b.outer_stride);
}

// DASO_OK, or what is wrong with a buffer that is needed (or, with optional, may be null).
int need(const Block& b, bool optional = false) {
  if (b.p == nullptr) return optional ? DASO_OK : DASO_EINVAL;
  return aligned(b.p, b.esz) ? DASO_OK : DASO_EALIGN;
}

// The first status that is not DASO_OK.
int first(std::initializer_list<int> codes) {
  for (int c : codes)
    if (c != DASO_OK) return c;
  return DASO_OK;
}

bool stride_ok(int64_t stride, int64_t row, int64_t rows) {
  return stride >= row && (rows == 0 || stride <= kMaxElems / std::max<int64_t>(rows, 1));
}

bool finite_not_negative(float v) { return v >= 0.0f && std::isfinite(v); }

// Outputs against inputs and each other; `in_place` is the one input that outputs[0] may be.  (Lists of the call's own: an
// entry point that only checks its arguments and launches allocates nothing that could throw.)
template <class Inputs>
int check_alias(std::initializer_list<Block> outputs, const Inputs& inputs, int in_place) {
  for (const Block* o = outputs.begin(); o != outputs.end(); ++o) {
    int i = 0;
    for (const Block& in : inputs) {
      const bool allowed = i++ == in_place && o == outputs.begin() && same(*o, in);
      if (!allowed && overlap(*o, in)) return DASO_EALIAS;
    }
    for (const Block* k = outputs.begin(); k != o; ++k)
      if (overlap(*o, *k)) return DASO_EALIAS;
  }
  return DASO_OK;
}
int check_alias(std::initializer_list<Block> outputs, std::initializer_list<Block> inputs, int in_place) {
  return check_alias<std::initializer_list<Block>>(outputs, inputs, in_place);
}

int64_t padded(int64_t k) { return std::max<int64_t>(128, (k + 63) / 64 * 64); }

}  // namespace

int check_workspace(const void* p, size_t bytes, size_t need_bytes) {
  if (need_bytes == 0) return DASO_OK;
  if (bytes < need_bytes) return DASO_ENOSPACE;
  if (p == nullptr) return DASO_EINVAL;
  return aligned(p, 256) ? DASO_OK : DASO_EALIGN;
}

// ------------------------------------------------------------------------- layer norm
int check_layer_norm(const daso_layer_norm_args& s) {
  if (s.rows < 0 || s.d < 0 || s.d > DASO_MAX_NORM_D || !known(s.type) || !finite_not_negative(s.eps)) return DASO_EINVAL;
  if (s.rows == 0 || s.d == 0) return DASO_OK;
  if (!stride_ok(s.x_stride, s.d, s.rows) || !stride_ok(s.y_stride, s.d, s.rows)) return DASO_EINVAL;
  const size_t e = bytes_of(s.type);
  const Block x = rows_of(s.x, s.rows, s.x_stride, s.d, e), y = rows_of(s.y, s.rows, s.y_stride, s.d, e);
  const Block w = flat(s.weight, s.d, 4), b = flat(s.bias, s.d, 4);
  const Block mean = flat(s.mean, s.rows, 4), rstd = flat(s.rstd, s.rows, 4);
  const int rc = first({need(x), need(y), need(w, true), need(b, true), need(mean, true), need(rstd, true)});
  if (rc != DASO_OK) return rc;
  return check_alias({y, mean, rstd}, {x, w, b}, 0);
}

int check_layer_norm_backward_sizes(const daso_layer_norm_backward_args& s) {
  return s.rows < 0 || s.d < 0 || s.d > DASO_MAX_NORM_D || !known(s.type) || s.reserved != 0 ? DASO_EINVAL : DASO_OK;
}

int check_layer_norm_backward(const daso_layer_norm_backward_args& s) {
  int rc = check_layer_norm_backward_sizes(s);
  if (rc != DASO_OK || s.d == 0) return rc;
  const Block dw = flat(s.dweight, s.d, 4), db = flat(s.dbias, s.d, 4);
  if ((rc = first({need(dw, true), need(db, true)})) != DASO_OK) return rc;
  if (s.rows == 0) return check_alias({dw, db}, {}, -1);
  if (!stride_ok(s.x_stride, s.d, s.rows) || !stride_ok(s.dy_stride, s.d, s.rows)) return DASO_EINVAL;
  if (s.dx != nullptr && !stride_ok(s.dx_stride, s.d, s.rows)) return DASO_EINVAL;
  const size_t e = bytes_of(s.type);
  const Block dy = rows_of(s.dy, s.rows, s.dy_stride, s.d, e), x = rows_of(s.x, s.rows, s.x_stride, s.d, e);
  const Block dx = rows_of(s.dx, s.rows, s.dx_stride, s.d, e), w = flat(s.weight, s.d, 4);
  const Block mean = flat(s.mean, s.rows, 4), rstd = flat(s.rstd, s.rows, 4);
  rc = first({need(dy), need(x), need(w, true), need(mean), need(rstd), need(dx, true)});
  if (rc != DASO_OK) return rc;
  return check_alias({dx, dw, db}, {dy, x, w, mean, rstd}, 0);
}

// ------------------------------------------------------------------------- the loss
int check_loss_sizes(const daso_loss_args& s) {
  if (s.tokens < 0 || s.tokens > kMaxLd || s.vocab < 1 || s.vocab > DASO_MAX_SIDE || s.d < 1 || s.d > DASO_MAX_SIDE)
    return DASO_EINVAL;
  if (!known(s.type) || !known(s.dweight_type)) return DASO_EINVAL;
  return DASO_OK;
}

int check_loss(const daso_loss_args& s, bool backward) {
  int rc = check_loss_sizes(s);
  if (rc != DASO_OK) return rc;
  const size_t e = bytes_of(s.type);
  const Block h = rows_of(s.hidden, s.tokens, s.hidden_stride, s.d, e), w = rows_of(s.weight, s.vocab, s.weight_stride, s.d, e);
  const Block t = flat(s.targets, s.tokens, 8), lse = flat(s.lse, s.tokens, 4);
  const Block dw = rows_of(s.dweight, s.vocab, s.dweight_stride, s.d, bytes_of(s.dweight_type));
  if (backward && s.dweight != nullptr) {
    if (!stride_ok(s.dweight_stride, s.d, s.vocab)) return DASO_EINVAL;
    if ((rc = need(dw)) != DASO_OK) return rc;
  }
  if (s.tokens == 0) return DASO_OK;
  if (!stride_ok(s.hidden_stride, s.d, s.tokens) || !stride_ok(s.weight_stride, s.d, s.vocab)) return DASO_EINVAL;
  if (s.hidden_stride > kMaxLd || s.weight_stride > kMaxLd) return DASO_EINVAL;
  if ((rc = first({need(h), need(w), need(t), need(lse)})) != DASO_OK) return rc;
  if (!backward) {
    const Block loss = flat(s.loss, s.tokens, 4);
    if ((rc = need(loss)) != DASO_OK) return rc;
    return check_alias({loss, lse}, {h, w, t}, -1);
  }
  const Block dloss = flat(s.dloss, s.tokens, 4), dh = rows_of(s.dhidden, s.tokens, s.dhidden_stride, s.d, e);
  if (s.dhidden != nullptr && !stride_ok(s.dhidden_stride, s.d, s.tokens)) return DASO_EINVAL;
  if ((rc = first({need(dloss), need(dh, true)})) != DASO_OK) return rc;
  return check_alias({dh, dw}, {h, w, t, lse, dloss}, -1);
}

// ------------------------------------------------------------------------- Newton-Schulz
namespace {
int check_steps(int32_t steps, float eps, const float* c) {
  if (steps < 1 || steps > DASO_MAX_SCHULZ_STEPS || !finite_not_negative(eps) || c == nullptr) return DASO_EINVAL;
  for (int32_t i = 0; i < 3 * steps; ++i)
    if (!std::isfinite(c[i])) return DASO_EINVAL;
  return DASO_OK;
}
}  // namespace

int check_orthogonalize_sizes(const daso_orthogonalize_args& s) {
  if (s.batch < 0 || s.batch > INT32_MAX || s.rows < 0 || s.cols < 0 || s.rows > DASO_MAX_SIDE || s.cols > DASO_MAX_SIDE)
    return DASO_EINVAL;
  return known(s.type) && known(s.out_type) ? DASO_OK : DASO_EINVAL;
}

int check_orthogonalize(const daso_orthogonalize_args& s) {
  int rc = check_orthogonalize_sizes(s);
  if (rc != DASO_OK) return rc;
  if ((rc = check_steps(s.steps, s.eps, s.coefficients)) != DASO_OK) return rc;
  if (s.batch == 0 || s.rows == 0 || s.cols == 0) return DASO_OK;
  const Block src = {s.src, s.batch, s.src_batch_stride, s.rows, s.src_stride, s.cols, bytes_of(s.type)};
  const Block out = {s.out, s.batch, s.out_batch_stride, s.rows, s.out_stride, s.cols, bytes_of(s.out_type)};
  for (const Block* b : {&src, &out}) {
    if (!stride_ok(b->stride, s.cols, s.rows)) return DASO_EINVAL;
    if (s.batch > 1 && !stride_ok(b->outer_stride, (s.rows - 1) * b->stride + s.cols, s.batch)) return DASO_EINVAL;
  }
  if ((rc = first({need(src), need(out)})) != DASO_OK) return rc;
  return check_alias({out}, {src}, 0);
}

int check_muon_sizes(const daso_muon_args& s) {
  if (s.n < 0 || s.n > DASO_MAX_N || s.g < 1 || s.g > DASO_MAX_G || s.nmatrices < 0) return DASO_EINVAL;
  if (s.nmatrices > 0 && s.matrices == nullptr) return DASO_EINVAL;
  std::vector<std::pair<int64_t, int64_t>> spans;
  spans.reserve(static_cast<size_t>(s.nmatrices));
  for (int32_t i = 0; i < s.nmatrices; ++i) {
    const daso_matrix& m = s.matrices[i];
    if (m.rows < 1 || m.cols < 1 || m.rows > DASO_MAX_SIDE || m.cols > DASO_MAX_SIDE || m.reserved != 0 || !std::isfinite(m.scale))
      return DASO_EINVAL;
    const int64_t k = int64_t(m.rows) * m.cols;
    if (m.start < 0 || m.start > s.n || k > s.n - m.start) return DASO_EINVAL;
    spans.emplace_back(m.start, m.start + k);
  }
  std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return DASO_EINVAL;
  return DASO_OK;
}

int check_muon(const daso_muon_args& s) {
  int rc = check_muon_sizes(s);
  if (rc != DASO_OK) return rc;
  if ((s.flags & ~DASO_MUON_NESTEROV) != 0 || !std::isfinite(s.lr) || !std::isfinite(s.mu) || !std::isfinite(s.weight_decay))
    return DASO_EINVAL;
  if ((rc = check_steps(s.steps, s.eps, s.coefficients)) != DASO_OK) return rc;
  if (s.n == 0 || s.nmatrices == 0) return DASO_OK;
  if (s.grads == nullptr || s.params == nullptr || s.momentum == nullptr) return DASO_EINVAL;
  std::vector<Block> inputs;
  for (int32_t r = 0; r < s.g; ++r) {
    if (s.grads[r] == nullptr) return DASO_EINVAL;
    if (!aligned(s.grads[r], 16)) return DASO_EALIGN;
    inputs.push_back(flat(s.grads[r], s.n, 4));
  }
  if (!aligned(s.params, 16) || !aligned(s.momentum, 16) || !aligned(s.wire, 16)) return DASO_EALIGN;
  return check_alias({flat(s.params, s.n, 4), flat(s.momentum, s.n, 4), flat(s.wire, s.n, 2)}, inputs, -1);
}

std::vector<SchulzRound> plan_rounds(const std::vector<Shape>& shapes, bool with_source, bool full) {
  // shapes in order of first appearance, each with its matrices
  std::map<std::pair<int64_t, int64_t>, size_t> at;
  std::vector<std::pair<Shape, std::vector<int32_t>>> kinds;
  for (size_t i = 0; i < shapes.size(); ++i) {
    const auto key = std::make_pair(shapes[i].rows, shapes[i].cols);
    auto it = at.find(key);
    if (it == at.end()) {
      it = at.emplace(key, kinds.size()).first;
      kinds.push_back({shapes[i], {}});
    }
    kinds[it->second].second.push_back(static_cast<int32_t>(i));
  }
  std::vector<SchulzRound> rounds;
  int64_t held = 0;
  for (const auto& kind : kinds) {
    const Shape& s = kind.first;
    const int64_t m = padded(std::min(s.rows, s.cols)), n = padded(std::max(s.rows, s.cols));
    const bool small = is_small(std::min(s.rows, s.cols), std::max(s.rows, s.cols), full);
    const int64_t each = small ? 1024 : m * n;  // (small ones hold no planes)
    for (size_t done = 0; done < kind.second.size();) {
      int64_t room = 0;
      if (!rounds.empty() && rounds.back().groups.size() < size_t(kRoundGroups))
        room = std::min((kRoundElems - held) / each, int64_t(kRoundMatrices) - int64_t(rounds.back().matrices.size()));
      if (room < 1) {
        rounds.push_back({});
        held = 0;
        room = std::max<int64_t>(1, std::min(kRoundElems / each, int64_t(kRoundMatrices)));
      }
      SchulzRound& r = rounds.back();
      SchulzGroup g = {};
      g.rows = s.rows, g.cols = s.cols, g.m = m, g.n = n, g.tall = s.rows > s.cols, g.small = small;
      g.count = static_cast<int32_t>(std::min<int64_t>(room, int64_t(kind.second.size() - done)));
      g.first = static_cast<int32_t>(r.matrices.size());
      for (int32_t k = 0; k < g.count; ++k) r.matrices.push_back(kind.second[done + size_t(k)]);
      r.groups.push_back(g);
      held += each * g.count;
      done += size_t(g.count);
    }
  }
  for (SchulzRound& r : rounds) {
    size_t to = (kRoundTables + 255) / 256 * 256;
    const auto take = [&to](int64_t bytes) {
      const size_t from = to;
      to += (static_cast<size_t>(bytes) + 255) / 256 * 256;
      return from;
    };
    for (SchulzGroup& g : r.groups) {
      if (with_source) g.source = take(4 * g.rows * g.cols * g.count);
      if (g.small) continue;
      for (int b = 0; b < 2; ++b)
        for (int p = 0; p < 2; ++p) g.x[b][p] = take(2 * g.m * g.n * g.count);
      for (int p = 0; p < 2 && g.tall; ++p) g.xt[p] = take(2 * g.m * g.n * g.count);
      for (int p = 0; p < 2; ++p) g.gram[p] = take(2 * g.m * g.m * g.count), g.poly[p] = take(2 * g.m * g.m * g.count);
      for (int p = 0; p < 2; ++p) g.rest[p] = take(4 * g.m * g.count);
    }
    // steps of the largest of a step's products, in tiles of 128 and three segments
    int64_t gram = 0, poly = 0, next = 0;
    for (const SchulzGroup& g : r.groups) {
      if (g.small) continue;
      const int64_t m = (g.m + 127) / 128, n = (g.n + 127) / 128;
      gram += g.count * (m * (m + 1) / 2) * 3 * (g.n / 64);
      poly += g.count * (m * (m + 1) / 2) * 3 * (g.m / 64);
      next += g.count * (m * n) * 3 * (g.m / 64);
    }
    r.sums_bytes = next > 0 ? sums_bytes(std::max({gram, poly, next})) : 0;
    r.sums = take(static_cast<int64_t>(r.sums_bytes));
    r.bytes = to;
  }
  return rounds;
}

SchulzBatch plan_batch(int64_t batch, const Shape& shape, bool full) {
  const auto round_of = [&](int64_t matrices) {
    return plan_rounds(std::vector<Shape>(static_cast<size_t>(matrices), shape), false, full)[0];
  };
  SchulzBatch b = {};
  b.full = round_of(std::min<int64_t>(batch, kRoundMatrices));
  b.each = static_cast<int64_t>(b.full.matrices.size());
  b.rounds = (batch + b.each - 1) / b.each;
  b.last = batch % b.each != 0 ? round_of(batch % b.each) : b.full;
  return b;
}

}  // namespace host
}  // namespace daso
