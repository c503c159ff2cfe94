// Shared by the token models' calls (embed.hip, scan.hip, act8.hip) and their host checks
// (tokens.cpp, plain C++): the finished mini-batches of a call, the checks of its buffers
// and the sizes of its workspaces.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "nbsgd.h"

#ifdef __HIPCC__
#define NBSGD_HD __host__ __device__ __forceinline__
#else
#define NBSGD_HD inline
#endif

namespace nbsgd {

constexpr int kMaxGroups = NBSGD_MAX_LEARNERS * NBSGD_MAX_MINIBATCHES;

// The finished mini-batches of a call, in order: i * m + j, two to a word (kernel
// arguments, read as 32-bit words only).
struct Groups {
  int32_t count, m;
  uint32_t w[kMaxGroups / 2];
};
#if defined(__HIP__)
__device__ __forceinline__ int group_id(const Groups& g, int e) {
  return (int)((g.w[e >> 1] >> (16 * (e & 1))) & 0xffffu);
}
#endif

// Checks n, m and the mask and fills *g.
nbsgd_status check_groups(int32_t n, int32_t m, const uint8_t* mask, Groups* g);

// Bytes of an element, 0 for an unknown type.
inline int dtype_size(int32_t dtype) {
  return dtype == NBSGD_F32 ? 4 : dtype == NBSGD_BF16 ? 2 : 0;
}

// A buffer of a call: `rows` rows of `width` bytes, `stride` bytes apart.
struct Rows {
  const char* name;
  const void* p;
  int64_t rows, width, stride;
};
// Whether no row of one buffer touches a row of the other; rows that lie side by side
// with one stride (two halves of a buffer) are apart.
bool rows_apart(const Rows& a, const Rows& b);
// Checks that the first `outs` buffers overlap neither each other nor the rest.  Null and
// empty ones pass.
nbsgd_status check_apart(const Rows* b, int count, int outs);

// Checks the parameters' row stride and alignment.
nbsgd_status check_params(const char* name, const void* p, int64_t ld, int64_t params);
// Checks an activation buffer: stride, width limit, alignment of its element; null only
// where it has no rows.
nbsgd_status check_rows(const char* name, const void* p, int64_t rows, int64_t width, int64_t ld,
                        int elem);
// Checks a workspace.
nbsgd_status check_workspace(const void* ws, size_t bytes, size_t need);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- embeddings: pieces of a mini-batch's sorted tokens (embed.hip)
constexpr int kMaxPiece = 32;
struct EmbedSpace {
  int32_t items;      // of a piece
  int64_t pieces;     // of one mini-batch
  size_t keys, sorted, flags, parts, total;  // byte offsets, and the whole
};
EmbedSpace embed_space(int64_t groups, int64_t T, int64_t dim);
nbsgd_status check_embed(int32_t T, int32_t vocab, int32_t dim);

// ---- recurrence: tiles of NBSGD_SCAN_INTERVAL tokens
constexpr int kScanTile = NBSGD_SCAN_INTERVAL;
constexpr int kScanWaves = 8;  // rows of bias-gradient sums that a tile leaves
struct ScanSpace {
  int64_t tiles;                      // of one sequence
  size_t pairs, carry, bias, total;   // byte offsets, and the whole
};
ScanSpace scan_space(int64_t seqs, int64_t T, int64_t dim);
nbsgd_status check_scan(int32_t n, int32_t m, int32_t batch, int32_t T, int32_t dim);

// ---- 8-bit activations
constexpr int kActBlock = 32;
struct Act8 {
  int64_t blocks;        // of 32 tokens
  int64_t scale, bytes;  // offset of the steps, and bytes of a mini-batch
};
inline Act8 act8_layout(int64_t T, int64_t dim) {
  Act8 a;
  a.blocks = ceil_div(T, kActBlock);
  a.scale = a.blocks * dim * kActBlock;
  a.bytes = (a.scale + ceil_div(a.blocks, 4) * dim * 4 + 15) / 16 * 16;
  return a;
}
nbsgd_status check_act8(int32_t T, int32_t dim);
// A tile of the weight gradient, columns c0 .. c0 + width of `cols`, reads rows of dY without looking
// at their ends, eight elements from every eighth column: up to seven of them follow the row's last.
// Where there are any they have to be the same mini-batch's, since the next one may be unfinished and is
// not read then: those of tokens below act8_border are.  The number of the first `tokens` tokens that
// are read so:
inline int32_t act8_border(int32_t T, int64_t ldy) { return T - (int32_t)ceil_div(7, ldy); }
NBSGD_HD int act8_sure(int tokens, int border, int c0, int width, int cols) {
  const bool ends = c0 + width <= cols || cols % 8 == 0;  // every load with its row, or before
  return ends || tokens < border ? tokens : border;
}
// Parts that the tokens of a weight gradient are summed in, by workgroups of their own where
// its smallest tiles (64 x 128) are few and the tokens many.  By the mini-batch's sizes alone,
// not by how many mini-batches a call has, so that a result does not depend on the others.
// One mini-batch of 16384 x 1024 x 1024: 71 us in four parts, 96 in two, 173 in one.  A part costs a
// write and a read of the gradient, 8 dim out bytes, so it has the tokens to read half as much again,
// dim + 2 out bytes each: 16 mini-batches of 4096 x 1024 x 1024 take 117 us in one part and
// 229 in four, of 8192 x 256 x 256 42 us in eight parts, 52 in two and 88 in one.
constexpr int64_t kSplitTiles = 512, kSplitTokens = 1024;
int act8_splits(int64_t T, int64_t dim, int64_t out);
size_t act8_space(int64_t groups, int64_t T, int64_t dim, int64_t out);

}  // namespace nbsgd
