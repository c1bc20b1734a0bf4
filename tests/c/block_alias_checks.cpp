// The aliasing rules of the transformer block's operators against every pair of rows, on random small layouts: of an accepted
// call no output's row touches another row, but for the row of the same token and head of the input that it may replace.
// Built with the host compiler alone; fake device addresses are never dereferenced.  Exit status 0 when every expectation holds.
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <random>

#include "daso_block_host.h"

using namespace daso::host;
typedef std::mt19937_64 Rng;

static int failures = 0, accepted = 0, in_place = 0;

struct Sides {
  int64_t tokens, dim;
  size_t bytes;
};
struct Operand {
  const daso_heads* rows;
  int64_t heads;
};

static uintptr_t row_at(const Operand& o, int64_t t, int64_t h, const Sides& s) {
  const int64_t at = (s.tokens > 1 ? t * o.rows->token_stride : 0) + (o.heads > 1 ? h * o.rows->head_stride : 0);
  return reinterpret_cast<uintptr_t>(o.rows->data) + uintptr_t(at) * s.bytes;
}

// Whether a row of `a` touches one of `b`; with `replaces`, other than the one of its token and head.
static bool touch(const Operand& a, const Operand& b, const Sides& s, bool replaces) {
  const uintptr_t row = uintptr_t(s.dim) * s.bytes;
  for (int64_t t = 0; t < s.tokens; ++t)
    for (int64_t h = 0; h < a.heads; ++h)
      for (int64_t u = 0; u < s.tokens; ++u)
        for (int64_t k = 0; k < b.heads; ++k) {
          const uintptr_t p = row_at(a, t, h, s), q = row_at(b, u, k, s);
          if (replaces && t == u && h == k && p == q) continue;
          if (p < q + row && q < p + row) return true;
        }
  return false;
}

static void check(std::initializer_list<Operand> outputs, std::initializer_list<Operand> inputs, int replaceable, const Sides& s) {
  ++accepted;
  int k = 0;
  for (const Operand* o = outputs.begin(); o != outputs.end(); ++o, ++k) {
    int i = 0;
    for (const Operand& in : inputs) {
      const bool replaces = i++ == k && k < replaceable;
      if (replaces && o->rows->data == in.rows->data) ++in_place;
      if (touch(*o, in, s, replaces)) ++failures;
    }
    for (const Operand* p = outputs.begin(); p != o; ++p)
      if (touch(*o, *p, s, false)) ++failures;
  }
}

static void random_call(Rng& rng) {
  const auto one_of = [&rng](std::initializer_list<int64_t> of) { return of.begin()[rng() % of.size()]; };
  const Sides s = {int64_t(1 + rng() % 4), 8, size_t(2 + 2 * (rng() % 2))};
  const int64_t kv = 1 + int64_t(rng() % 2), heads = kv * int64_t(1 + rng() % 3);
  const int64_t wide = one_of({(heads + kv) * 8, (heads + 2 * kv) * 8, heads * 8, 100});
  daso_heads of[8];
  for (daso_heads& h : of) {
    const int64_t token = one_of({8, 16, 24, 32, wide, wide, wide}), head = one_of({8, 8, 8, 16, 24, wide, s.tokens * 8});
    // (the parts of one buffer, or a buffer of its own)
    h = {reinterpret_cast<void*>(0x10000000 + one_of({0, 0, 0, 1, 2, 3, 4, 5, 6, 7}) * 0x100000 + uintptr_t(one_of({0, 0, 0, 8, 16, 24, 32, 48})) * s.bytes),
         token, head};
  }
  // often the buffer that an output may replace, as it is or with the distances exchanged
  const auto over = [&](int output, int input) {
    const uint64_t how = rng() % 4;
    if (how == 1) of[output] = of[input];
    if (how == 2) of[output] = {of[input].data, of[input].head_stride, of[input].token_stride};
  };
  const int64_t type = s.bytes == 2 ? DASO_TYPE_BF16 : DASO_TYPE_F32;
  daso_rotary_args r = {};
  r.tokens = s.tokens, r.heads = int32_t(heads), r.kv_heads = int32_t(kv), r.dim = 8, r.rotated = 8, r.type = int32_t(type);
  r.positions = reinterpret_cast<const int64_t*>(0x20000000), r.frequencies = reinterpret_cast<const double*>(0x21000000);
  over(2, 0), over(3, 1);
  r.q = of[0], r.k = of[1], r.q_out = of[2], r.k_out = of[3];
  const auto q = [&](const daso_heads& h) { return Operand{&h, heads}; };
  const auto k = [&](const daso_heads& h) { return Operand{&h, kv}; };
  if (check_rotary(r, false) == DASO_OK) check({q(r.q_out), k(r.k_out)}, {q(r.q), k(r.k)}, 2, s);
  over(6, 4), over(7, 5);
  r.dq_out = of[4], r.dk_out = of[5], r.dq = of[6], r.dk = of[7];
  if (check_rotary(r, true) == DASO_OK) check({q(r.dq), k(r.dk)}, {q(r.dq_out), k(r.dk_out), q(r.q), k(r.k)}, 2, s);
  daso_attention_args a = {};
  a.tokens = s.tokens, a.heads = int32_t(heads), a.kv_heads = int32_t(kv), a.dim = 8, a.type = int32_t(type), a.sequences = 1, a.scale = 1.0f;
  a.lse = reinterpret_cast<float*>(0x22000000);
  a.q = of[0], a.k = of[1], a.v = of[2], a.out = of[3], a.dout = of[4], a.dq = of[5], a.dk = of[6], a.dv = of[7];
  if (check_attention(a, false) == DASO_OK) check({q(a.out)}, {q(a.q), k(a.k), k(a.v)}, 0, s);
  if (check_attention(a, true) == DASO_OK)
    check({q(a.dq), k(a.dk), k(a.dv)}, {q(a.q), k(a.k), k(a.v), q(a.out), q(a.dout)}, 0, s);
}

int main() {
  Rng rng(11);
  for (int i = 0; i < 400000; ++i) random_call(rng);
  if (failures != 0 || accepted < 10000 || in_place < 1000) {
    std::fprintf(stderr, "%d rows touched in %d accepted calls, %d in place\n", failures, accepted, in_place);
    return 1;
  }
  std::printf("block alias checks ok: %d calls accepted, %d outputs in place\n", accepted, in_place);
  return 0;
}
