// Host-only argument checks and plans of daso_block.h (no HIP calls, nothing allocated).  Each check returns DASO_OK
// or the status that the entry point returns; workspaces are checked by the entry points.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "daso_block.h"
#include "daso_train_host.h"

namespace daso {
namespace host {

// The largest distance of two tokens' rows in an attention, in elements: the byte offsets of a workgroup's 128 rows stay
// below 2^31.
constexpr int64_t kMaxTokenStride = 2 * DASO_MAX_SIDE;
static_assert(127 * kMaxTokenStride * 4 + DASO_MAX_HEAD_DIM * 4 < (int64_t(1) << 31), "offsets of 31 bits");

int check_rotary_sizes(const daso_rotary_args& s);
int check_rotary(const daso_rotary_args& s, bool backward);
int check_attention_sizes(const daso_attention_args& s);
int check_attention(const daso_attention_args& s, bool backward);
int check_clip_sizes(const daso_clip_args& s);
int check_clip(const daso_clip_args& s);

// How the tensors of a clipping are cut: pieces of 1024 elements, counted from the buffer's start, of one tensor each: a workgroup
// and a partial sum of squares a piece.
constexpr int64_t kPiece = 1024;
constexpr int64_t kMostPieces = int64_t(1) << 24;
constexpr int64_t kJoined = 4096;  // pieces from which on their sums are added by kernels of their own
inline int64_t pieces_of(const daso_span& t) { return t.n == 0 ? 0 : (t.start + t.n - 1) / kPiece - t.start / kPiece + 1; }
int64_t pieces_of(const daso_clip_args& s);

// What of a clipping one launch takes: runs of elements between neighbouring boundaries, of which those that are a tensor
// have pieces and gaps between tensors none.
constexpr int kClipRuns = 208;
struct ClipTable {
  int64_t bound[kClipRuns + 1];  // run i: bound[i] <= element < bound[i + 1]
  int32_t first[kClipRuns + 1];  // its first piece, counted from the launch's first
  int16_t number[kClipRuns];     // its tensor, counted from the launch's first, or -1
  int32_t tensor;                // number of the first tensor
  int32_t runs;
};
// Fills the table with the tensors from `tensor` on that fit; returns how many.  merged: tensors next to each other are one run,
// whose pieces are not those of the tensors apart.
int32_t fill_table(const daso_clip_args& s, int32_t tensor, bool merged, ClipTable* table);

}  // namespace host
}  // namespace daso
