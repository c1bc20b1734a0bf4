// Exercises the host-only code of the training operators (argument checks, rounds and workspace offsets of the
// Newton-Schulz steps) under AddressSanitizer and UndefinedBehaviorSanitizer, and without memory.  Built with the host
// compiler alone; fake device addresses are never dereferenced.  Exit status 0 when every expectation holds.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <random>
#include <vector>

#include "daso_train.h"
#include "daso_train_host.h"

static int failures = 0;
#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) {                                                       \
      std::fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__,  \
                   __LINE__, #cond);                                     \
      ++failures;                                                        \
    }                                                                    \
  } while (0)

static bool no_memory = false;
void* operator new(size_t n) {
  void* p = no_memory ? nullptr : std::malloc(n ? n : 1);
  if (p == nullptr) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

using namespace daso::host;
typedef std::mt19937_64 Rng;

template <class T>
static T* at(uint64_t address) { return reinterpret_cast<T*>(address); }
static int64_t one_of(Rng& rng, std::initializer_list<int64_t> of) { return of.begin()[rng() % of.size()]; }
// A small address now and then null, odd or inside another buffer's; strides and sizes at the ends of their ranges too.
static uint64_t address(Rng& rng) { return rng() % 12 == 0 ? 0 : 0x10000000 + (rng() % 24) * 0x8000 + (rng() % 8 == 0 ? rng() % 64 : 0); }
static int64_t size_of(Rng& rng) { return one_of(rng, {-1, 0, 1, 2, 7, 64, 65, 1000, 65536, 65537, 1 << 20, (1 << 20) + 1, int64_t(1) << 40, INT64_MAX}); }

static daso_layer_norm_args layer_norm(Rng& rng) {
  return {size_of(rng), size_of(rng), int32_t(rng() % 3), 1e-5f, at<void>(address(rng)), size_of(rng), at<float>(address(rng)),
          at<float>(address(rng)), at<void>(address(rng)), size_of(rng), at<float>(address(rng)), at<float>(address(rng))};
}
static daso_layer_norm_backward_args layer_norm_backward(Rng& rng) {
  return {size_of(rng), size_of(rng), int32_t(rng() % 3), 0, at<void>(address(rng)), size_of(rng), at<void>(address(rng)), size_of(rng),
          at<float>(address(rng)), at<float>(address(rng)), at<float>(address(rng)), at<void>(address(rng)), size_of(rng),
          at<float>(address(rng)), at<float>(address(rng)), at<void>(address(rng)), rng()};
}
static daso_loss_args loss(Rng& rng) {
  return {size_of(rng), size_of(rng), size_of(rng), int32_t(rng() % 3), int32_t(rng() % 3), at<void>(address(rng)), size_of(rng),
          at<void>(address(rng)), size_of(rng), at<int64_t>(address(rng)), -100, at<float>(address(rng)), at<float>(address(rng)),
          at<float>(address(rng)), at<void>(address(rng)), size_of(rng), at<void>(address(rng)), size_of(rng), at<void>(address(rng)), rng()};
}
static float coefficients[3 * DASO_MAX_SCHULZ_STEPS] = {3.4445f, -4.775f, 2.0315f};
static daso_orthogonalize_args orthogonalize(Rng& rng) {
  return {size_of(rng), size_of(rng), size_of(rng), int32_t(rng() % 3), int32_t(rng() % 3), at<void>(address(rng)), size_of(rng),
          size_of(rng), at<void>(address(rng)), size_of(rng), size_of(rng), int32_t(rng() % 18), 0.0f, coefficients, at<void>(address(rng)), rng()};
}

static bool status(int rc) { return rc == DASO_OK || rc == DASO_EINVAL || rc == DASO_EALIGN || rc == DASO_EALIAS; }

// Every call ends in a status: no overflow, no read of what a null pointer names, and, without memory, no exception.
static void check_calls(Rng& rng, int trials) {
  int taken = 0;
  for (int t = 0; t < trials; ++t) {
    int rc[5];
    const auto norm = layer_norm(rng);
    const auto back = layer_norm_backward(rng);
    const auto ce = loss(rng);
    const auto ns = orthogonalize(rng);
    no_memory = true;
    try {
      rc[0] = check_layer_norm(norm), rc[1] = check_layer_norm_backward(back), rc[2] = check_loss(ce, false), rc[3] = check_loss(ce, true);
      rc[4] = check_orthogonalize(ns);
    } catch (const std::bad_alloc&) {
      no_memory = false;
      EXPECT(!"a check of arguments allocates");
      return;
    }
    no_memory = false;
    for (int k : rc) {
      EXPECT(status(k));
      taken += k == DASO_OK;
    }
  }
  EXPECT(taken > trials / 100);
}

// The pairs that may be one buffer, and a stride that makes them two that overlap.
static void alias_checks() {
  daso_layer_norm_args a = {10, 64, DASO_TYPE_F32, 1e-5f, at<void>(0x10000), 64, nullptr, nullptr, at<void>(0x10000), 64, nullptr, nullptr};
  EXPECT(check_layer_norm(a) == DASO_OK);
  a.y_stride = 65;
  EXPECT(check_layer_norm(a) == DASO_EALIAS);
  a.y_stride = 64, a.mean = at<float>(0x10000 + 4 * 64);
  EXPECT(check_layer_norm(a) == DASO_EALIAS);
  daso_layer_norm_backward_args b = {10, 64, DASO_TYPE_F32, 0, at<void>(0x10000), 64, at<void>(0x20000), 64, nullptr, at<float>(0x30000),
                                     at<float>(0x31000), at<void>(0x10000), 64, at<float>(0x40000), at<float>(0x41000), nullptr, 0};
  EXPECT(check_layer_norm_backward(b) == DASO_OK);
  b.dx = at<void>(0x20000);  // x is read by the sums too
  EXPECT(check_layer_norm_backward(b) == DASO_EALIAS);
  b.dx = nullptr, b.dbias = b.dweight;
  EXPECT(check_layer_norm_backward(b) == DASO_EALIAS);
  float c[3] = {1, 1, 1};
  daso_orthogonalize_args o = {2, 8, 8, DASO_TYPE_F32, DASO_TYPE_F32, at<void>(0x10000), 64, 8, at<void>(0x10000), 64, 8, 1, 0.0f, c, nullptr, 0};
  EXPECT(check_orthogonalize(o) == DASO_OK);
  o.out_type = DASO_TYPE_BF16;
  EXPECT(check_orthogonalize(o) == DASO_EALIAS);
}

// Two row blocks of one buffer are told apart element by element where their strides agree, and never taken as apart where
// they are not.
static void beside_checks(Rng& rng, int trials) {
  int apart = 0;
  for (int t = 0; t < trials; ++t) {
    const int64_t rows = 1 + int64_t(rng() % 5), d = 1 + int64_t(rng() % 6), xs = d + int64_t(rng() % 9), ys = rng() % 3 ? xs : d + int64_t(rng() % 9);
    const int64_t from = int64_t(rng() % 40);
    daso_layer_norm_args a = {rows, d, DASO_TYPE_F32, 1e-5f, at<void>(0x10000), xs, nullptr, nullptr, at<void>(0x10000 + 4 * from), ys, nullptr, nullptr};
    if (rng() % 2) {
      const void* x = a.x;
      a.x = a.y, a.y = const_cast<void*>(x);
      std::swap(a.x_stride, a.y_stride);
    }
    std::vector<char> used(400, 0);
    const auto element = [](const void* p, int64_t i) { return (reinterpret_cast<uintptr_t>(p) - 0x10000) / 4 + size_t(i); };
    bool meet = false;
    for (int64_t r = 0; r < rows; ++r)
      for (int64_t c = 0; c < d; ++c) used[element(a.x, r * a.x_stride + c)] = 1;
    for (int64_t r = 0; r < rows; ++r)
      for (int64_t c = 0; c < d; ++c) meet |= used[element(a.y, r * a.y_stride + c)] != 0;
    const bool same = a.x == a.y && (rows == 1 || a.x_stride == a.y_stride);
    const int rc = check_layer_norm(a);
    EXPECT(rc == DASO_OK || rc == DASO_EALIAS);
    if (meet && !same) EXPECT(rc == DASO_EALIAS);
    if (same || (!meet && a.x_stride == a.y_stride && rows > 1)) EXPECT(rc == DASO_OK);
    apart += rc == DASO_OK;
  }
  EXPECT(apart > trials / 10);
}

// A product's operands may have rows of kMaxLd elements: the loss's as they lie in memory, and hidden turned, of all tokens.
static void row_checks() {
  daso_loss_args a = {2, 3, 64, DASO_TYPE_BF16, DASO_TYPE_BF16, at<void>(0x100000000), kMaxLd, at<void>(0x200000000), kMaxLd,
                      at<int64_t>(0x300000000), -100, at<float>(0x400000000), at<float>(0x500000000), at<float>(0x600000000),
                      at<void>(0x700000000), 64, at<void>(0x800000000), 64, nullptr, 0};
  EXPECT(check_loss(a, false) == DASO_OK && check_loss(a, true) == DASO_OK);
  for (int64_t daso_loss_args::*field : {&daso_loss_args::hidden_stride, &daso_loss_args::weight_stride, &daso_loss_args::tokens}) {
    const int64_t was = a.*field;
    a.*field = kMaxLd + 1;
    EXPECT(check_loss(a, false) == DASO_EINVAL && check_loss(a, true) == DASO_EINVAL);
    a.*field = was;
  }
}

// Each matrix once, matrices of one shape together, and no two regions of a round's workspace overlap.
static void round_checks(Rng& rng, int trials) {
  struct Region {
    size_t from, bytes;
  };
  for (int t = 0; t < trials; ++t) {
    const bool source = rng() % 2, full = rng() % 2;
    std::vector<Shape> shapes;
    const int kinds = 1 + int(rng() % 12);
    for (int k = 0; k < kinds; ++k) {
      const int64_t top = one_of(rng, {1, 64, 640, 5000, 1 << 16});
      const Shape s = {1 + int64_t(rng() % top), 1 + int64_t(rng() % std::min<int64_t>(top, (int64_t(1) << 28) / top))};
      for (int i = int(rng() % 200); i >= 0; --i) shapes.push_back(s);
    }
    std::shuffle(shapes.begin(), shapes.end(), rng);
    std::vector<int> seen(shapes.size(), 0);
    for (const SchulzRound& r : plan_rounds(shapes, source, full)) {
      EXPECT(!r.groups.empty() && r.groups.size() <= size_t(kRoundGroups) && r.matrices.size() <= size_t(kRoundMatrices));
      std::vector<Region> taken = {{0, kRoundTables}};
      size_t first = 0;
      for (const SchulzGroup& g : r.groups) {
        EXPECT(g.count > 0 && size_t(g.first) == first);
        first += size_t(g.count);
        for (int32_t i = 0; i < g.count && first <= r.matrices.size(); ++i) {
          const int32_t m = r.matrices[size_t(g.first + i)];
          ++seen[size_t(m)];
          EXPECT(shapes[size_t(m)].rows == g.rows && shapes[size_t(m)].cols == g.cols);
        }
        EXPECT(g.tall == (g.rows > g.cols) && g.m >= std::min(g.rows, g.cols) && g.n >= std::max(g.rows, g.cols) && g.m % 64 == 0 && g.n % 64 == 0 && g.m >= 128);
        const size_t k = size_t(g.count), square = size_t(2 * g.m * g.m) * k, planes = size_t(2 * g.m * g.n) * k;
        if (source) taken.push_back({g.source, size_t(4 * g.rows * g.cols) * k});
        if (g.small) continue;
        for (int p = 0; p < 2; ++p) {
          taken.insert(taken.end(), {{g.x[0][p], planes}, {g.x[1][p], planes}, {g.gram[p], square}, {g.poly[p], square}, {g.rest[p], size_t(4 * g.m) * k}});
          if (g.tall) taken.push_back({g.xt[p], planes});
        }
      }
      EXPECT(first == r.matrices.size());
      taken.push_back({r.sums, r.sums_bytes});
      std::sort(taken.begin(), taken.end(), [](const Region& a, const Region& b) { return a.from < b.from || (a.from == b.from && a.bytes < b.bytes); });
      for (size_t i = 0; i < taken.size(); ++i) {
        EXPECT(taken[i].from % 256 == 0 && taken[i].from + taken[i].bytes <= r.bytes);
        if (i > 0) EXPECT(taken[i - 1].from + taken[i - 1].bytes <= taken[i].from);
      }
    }
    EXPECT(std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; }));
  }
}

// A batch of one shape: the rounds of plan_rounds, and as little memory for any number of matrices.
static void batch_checks(Rng& rng, int trials) {
  for (int t = 0; t < trials; ++t) {
    const int64_t top = one_of(rng, {1, 64, 640, 5000, 20000});
    const Shape s = {1 + int64_t(rng() % top), 1 + int64_t(rng() % top)};
    const bool full = rng() % 2;
    const int64_t batch = 1 + int64_t(rng() % 500);
    const std::vector<SchulzRound> rounds = plan_rounds(std::vector<Shape>(size_t(batch), s), false, full);
    const SchulzBatch b = plan_batch(batch, s, full);
    EXPECT(b.rounds == int64_t(rounds.size()));
    size_t most = 0;
    for (size_t k = 0; k < rounds.size(); ++k) {
      const SchulzRound& r = k + 1 < rounds.size() ? b.full : b.last;
      EXPECT(rounds[k].matrices[0] == int64_t(k) * b.each && r.groups.size() == 1 && r.groups[0].count == rounds[k].groups[0].count && r.bytes == rounds[k].bytes);
      most = std::max(most, r.bytes);
    }
    EXPECT(most == b.full.bytes);
  }
  const SchulzBatch many = plan_batch(INT32_MAX, {1, 1}, true);
  EXPECT(many.each == kRoundMatrices && many.rounds == (int64_t(INT32_MAX) + kRoundMatrices - 1) / kRoundMatrices);
}

int main() {
  Rng rng(20);
  check_calls(rng, 200000);
  alias_checks();
  row_checks();
  beside_checks(rng, 100000);
  round_checks(rng, 400);
  batch_checks(rng, 2000);
  if (failures == 0) std::printf("train host checks ok\n");
  return failures == 0 ? 0 : 1;
}
