// Host-only argument checks of daso_train.h (no HIP calls).  Each returns DASO_OK or the
// status that the entry point returns; workspaces are checked by the entry points, which
// know their size.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "daso_train.h"

namespace daso {
namespace host {

inline size_t bytes_of(int32_t type) { return type == DASO_TYPE_BF16 ? 2 : 4; }

int check_layer_norm(const daso_layer_norm_args& s);
int check_layer_norm_backward(const daso_layer_norm_backward_args& s);
int check_loss(const daso_loss_args& s, bool backward);
int check_orthogonalize(const daso_orthogonalize_args& s);
int check_muon(const daso_muon_args& s);
// The shapes and counts alone, for the *_workspace functions.
int check_layer_norm_backward_sizes(const daso_layer_norm_backward_args& s);
int check_loss_sizes(const daso_loss_args& s);
int check_orthogonalize_sizes(const daso_orthogonalize_args& s);
int check_muon_sizes(const daso_muon_args& s);
int check_workspace(const void* p, size_t bytes, size_t need);

// The longest rows of a product's operands, in elements: the offsets of a tile's 256 rows stay in 32 bits.
constexpr int64_t kMaxLd = 4 * DASO_MAX_SIDE;
static_assert(255 * 2 * kMaxLd + 128 <= UINT32_MAX, "the last byte of a tile's last row");

// ------------------------------------------------------------------ sums of cut tiles
// Steps of a part of a tile, at the least, and the most parts of an XCD's pool, a workgroup
// (daso_product.h).
constexpr int kLeastPart = 6, kPoolParts = 3, kPlaces256 = 256;

// Bytes of the sums that a launch of so many steps of 128 tiles may leave; a 256 tile's step counts
// as four.
inline size_t sums_bytes(int64_t steps128) {
  const int64_t parts = steps128 / kLeastPart + 64, most = int64_t(kPoolParts) * kPlaces256 * 4;
  return static_cast<size_t>(parts < most ? parts : most) * 128 * 128 * 4;
}

// ------------------------------------------------------------------ Newton-Schulz plan
// Matrices of one shape that take their steps together.  Inside, X is m x n with m <= n,
// both padded with zeros to multiples of 64.
struct SchulzGroup {
  int64_t rows, cols;
  int64_t m, n;           // padded
  bool tall;              // X is the transpose
  bool small;             // all steps in one workgroup: no planes in the workspace
  int32_t count;          // matrices
  int32_t first;          // place of the first among the round's matrices
  // byte offsets in the workspace; planes: [0] hi, [1] lo
  size_t source;          // fp32 copies of what is orthogonalised, rows x cols (muon only)
  size_t x[2][2], xt[2], gram[2], poly[2];  // x: [buffer][plane]; xt: of tall ones, for the last step
  size_t rest[2];         // what the one plane of gram and of poly leaves of their diagonals
};

// What is worked on at a time: groups of up to kRoundElems elements in all.
struct SchulzRound {
  std::vector<SchulzGroup> groups;
  std::vector<int32_t> matrices;  // indexes into the caller's list, group by group
  size_t sums, sums_bytes;        // the products' sums: byte offset, and room
  size_t bytes;                   // of workspace
};

// (an update of 302M elements takes 20.7 ms, with 2^26 21.5, with 2^25 22.1, with 2^28 20.65)
constexpr int64_t kRoundElems = int64_t(1) << 27;  // up to 16 bytes of workspace each, and the squares
constexpr int32_t kRoundMatrices = 128;            // as many as kernel arguments hold
constexpr int32_t kRoundGroups = 8;
constexpr int32_t kSumParts = 256;                 // partial sums of squares a matrix, one a thread of who adds them
constexpr size_t kRoundTables = size_t(kRoundMatrices) * (16 + 8 * kSumParts);  // table and partial sums

struct Shape {
  int64_t rows, cols;
};
// Rounds over the given matrices, in order of first appearance of their shapes.  full: products in 22 bits.
std::vector<SchulzRound> plan_rounds(const std::vector<Shape>& shapes, bool with_source, bool full);

// Rounds over a batch of matrices of one shape, however many: all of them like `full` but, where there is one, the last.
struct SchulzBatch {
  SchulzRound full, last;
  int64_t each;    // matrices of a full round
  int64_t rounds;  // with the last
};
SchulzBatch plan_batch(int64_t batch, const Shape& shape, bool full);

// The matrices that one workgroup takes (daso_muon.hip): what they need of its LDS, and whether they fit.
constexpr int kSmallM = 64, kSmallGroups = 5;                        // m, and groups of 128 columns of n, at most
constexpr int kGramStride = kSmallM * 2 + 16;                        // bytes a row of the gram matrix
constexpr int small_stride(int n) { return (n + 63) / 64 * 128 + 16; }  // bytes a row of X
constexpr int small_lds(int n, bool full) {
  return (full ? 2 : 1) * (kSmallM * small_stride(n) + kSmallM * kGramStride) + 1024;
}
constexpr bool is_small(int64_t m, int64_t n, bool full) {
  return m <= kSmallM && n <= kSmallGroups * 128 && small_lds(static_cast<int>(n), full) <= 160 * 1024;
}

}  // namespace host
}  // namespace daso
