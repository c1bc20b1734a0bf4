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

// How the tensors of a clipping are cut: chunks of one tensor each, a partial sum of squares a chunk.
struct ClipPlan {
  int64_t chunk;   // elements
  int64_t chunks;  // of all tensors
};
constexpr int64_t kClipChunks = 2048;      // and one more a tensor, at most
constexpr int64_t kClipLeastChunk = 4096;  // elements
ClipPlan plan_clip(const daso_clip_args& s);
inline int64_t chunks_of(int64_t n, int64_t chunk) { return n / chunk + (n % chunk != 0); }

// What of a clipping one launch takes: runs of elements between neighbouring boundaries, of which those that are a tensor
// have chunks and gaps between tensors none.
constexpr int kClipRuns = 208;
struct ClipTable {
  int64_t bound[kClipRuns + 1];  // run i: bound[i] <= element < bound[i + 1]
  int32_t first[kClipRuns + 1];  // its first chunk, counted from the launch's first
  int16_t number[kClipRuns];     // its tensor, counted from the launch's first, or -1
  int32_t tensor;                // number of the first tensor
  int32_t runs;
};
// Fills the table with the tensors from `tensor` on that fit; returns how many.
int32_t fill_table(const daso_clip_args& s, int64_t chunk, int32_t tensor, ClipTable* table);

}  // namespace host
}  // namespace daso
