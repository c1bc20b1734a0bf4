// Exercises the host-only code of the transformer block's operators (argument checks, how a clipping's tensors are cut)
// under AddressSanitizer and UndefinedBehaviorSanitizer, and without memory: it allocates nothing.  Built with the host
// compiler alone; fake device addresses are never dereferenced.  Exit status 0 when every expectation holds.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <random>
#include <vector>

#include "daso_block_host.h"

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

static int64_t one_of(Rng& rng, std::initializer_list<int64_t> of) { return of.begin()[rng() % of.size()]; }
template <class T>
static T* place(Rng& rng) {
  return reinterpret_cast<T*>(rng() % 20 == 0 ? 0 : 0x10000000 + (rng() % 64) * 0x100000 + (rng() % 8 == 0 ? rng() % 300 : 0));
}
static daso_heads heads(Rng& rng, int64_t dim) {
  daso_heads h;
  h.data = place<void>(rng);
  h.token_stride = one_of(rng, {dim, 8 * dim, 12 * dim, 0, -1, 1, INT64_MAX, INT64_MIN, int64_t(1) << 40, (int64_t(2) << 20) + 1});
  h.head_stride = one_of(rng, {dim, 3 * dim, 1000 * dim, 0, -1, INT64_MAX, INT64_MIN, int64_t(1) << 50});
  return h;
}

static int calls(Rng& rng) {
  int ok = 0;
  const int64_t dim = one_of(rng, {8, 64, 128, 64, 64, 0, 12, 136, -8, INT32_MAX});
  const int64_t tokens = one_of(rng, {0, 1, 2, 100, 4096, 1 << 24, (1 << 24) + 1, -1, INT64_MAX, INT64_MIN});
  const int32_t many = int32_t(one_of(rng, {1, 2, 8, 8, 1024, 0, -1, INT32_MAX})), few = int32_t(one_of(rng, {1, 2, 4, 8, 3, 0, INT32_MIN}));
  const float scale = float(one_of(rng, {1, 1, 1, 0, -1}));
  daso_rotary_args r = {};
  r.tokens = tokens, r.heads = many, r.kv_heads = few, r.dim = int32_t(dim), r.rotated = int32_t(one_of(rng, {0, 8, 64, dim, 4, -8, INT32_MAX}));
  r.type = int32_t(one_of(rng, {0, 1, 1, 2, -1})), r.eps = scale, r.flags = uint32_t(one_of(rng, {0, 1, 2})), r.reserved = rng() % 16 == 0;
  r.positions = place<int64_t>(rng), r.frequencies = place<double>(rng), r.q_weight = place<float>(rng), r.k_weight = place<float>(rng);
  for (daso_heads* h : {&r.q, &r.k, &r.q_out, &r.k_out, &r.dq_out, &r.dk_out, &r.dq, &r.dk}) *h = heads(rng, dim);
  r.dq_weight = place<float>(rng), r.dk_weight = place<float>(rng);
  ok += check_rotary(r, false) == DASO_OK, ok += check_rotary(r, true) == DASO_OK;
  daso_attention_args a = {};
  a.tokens = tokens, a.heads = many, a.kv_heads = few, a.dim = int32_t(dim), a.type = r.type, a.scale = scale;
  a.sequences = int32_t(one_of(rng, {0, 1, 1, 5, 1 << 20, (1 << 20) + 1, -1, INT32_MAX})), a.flags = uint32_t(one_of(rng, {0, 1, 15, 16}));
  a.offsets = place<int64_t>(rng), a.lse = place<float>(rng);
  for (daso_heads* h : {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv}) *h = heads(rng, dim);
  ok += check_attention(a, false) == DASO_OK, ok += check_attention(a, true) == DASO_OK;
  const float* grads[3] = {place<float>(rng), place<float>(rng), place<float>(rng)};
  daso_span spans[3];
  for (daso_span& s : spans) s = {one_of(rng, {0, 5, 100, -1, INT64_MAX, INT64_MIN}), one_of(rng, {0, 5, 50, -1, INT64_MAX, INT64_MIN})};
  daso_clip_args c = {};
  c.n = one_of(rng, {0, 1, 200, 200, int64_t(1) << 33, int64_t(1) << 56, INT64_MAX, -1}), c.g = int32_t(one_of(rng, {1, 2, 3, 0, -1}));
  c.ntensors = int32_t(one_of(rng, {0, 1, 2, 3, -1})), c.grads = rng() % 20 ? grads : nullptr, c.tensors = rng() % 20 ? spans : nullptr;
  c.out = place<float>(rng), c.norm = place<float>(rng), c.norms = place<float>(rng), c.max_norm = scale, c.eps = 0.0f;
  ok += check_clip(c) == DASO_OK;
  if (check_clip_sizes(c) == DASO_OK) EXPECT(pieces_of(c) >= 0);
  return ok;
}

// Every element of a tensor is in one piece of its run, and nothing else is; the launches' pieces come to the plan's.
static void cut(Rng& rng) {
  std::vector<daso_span> spans;
  int64_t at = 0;
  const int count = 1 + int(rng() % 700);
  for (int i = 0; i < count; ++i) {
    at += rng() % 3 == 0 ? int64_t(rng() % 5000) : 0;
    const int64_t n = one_of(rng, {0, 1, 3, 1023, 1024, 1025, int64_t(rng() % 20000)});
    spans.push_back({at, n});
    at += n;
  }
  daso_clip_args s = {};
  s.n = at, s.g = 1, s.ntensors = count, s.tensors = spans.data();
  EXPECT(check_clip_sizes(s) == DASO_OK);
  for (int merged = 0; merged < 2; ++merged) {
    std::vector<int> seen(size_t(at), 0), want(size_t(at), 0);
    std::vector<int> numbers(size_t(count), 0);
    int64_t pieces = 0;
    for (int32_t t = 0; t < count;) {
      static ClipTable table;
      const int32_t took = fill_table(s, t, merged != 0, &table);
      EXPECT(took > 0 && table.runs >= 1 && table.runs <= kClipRuns && table.tensor == t);
      for (int run = 0; run < table.runs; ++run) {
        const int64_t from = table.bound[run], to = table.bound[run + 1];
        const int32_t have = table.first[run + 1] - table.first[run];
        if (table.number[run] < 0) {
          EXPECT(have == 0);
          continue;
        }
        EXPECT(have == pieces_of(daso_span{from, to - from}));
        if (!merged) ++numbers[size_t(t + table.number[run])];
        for (int32_t p = 0; p < have; ++p) {
          const int64_t first = (from / kPiece + p) * kPiece;
          for (int64_t e = first < from ? from : first; e < first + kPiece && e < to; ++e) ++seen[size_t(e)];
        }
        pieces += have;
      }
      t += took;
    }
    for (const daso_span& span : spans)
      for (int64_t e = 0; e < span.n; ++e) ++want[size_t(span.start + e)];
    EXPECT(seen == want);
    if (!merged) {
      EXPECT(pieces == pieces_of(s));
      for (int k : numbers) EXPECT(k == 1);
    }
  }
}

int main() {
  Rng rng(7);
  int ok = 0;
  no_memory = true;
  for (int i = 0; i < 400000; ++i) ok += calls(rng);
  no_memory = false;
  EXPECT(ok > 100);
  for (int i = 0; i < 60; ++i) cut(rng);
  if (failures != 0) return 1;
  std::printf("block host checks ok: %d calls accepted\n", ok);
  return 0;
}
