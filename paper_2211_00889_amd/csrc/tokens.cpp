// Host checks and sizes of the token models' calls (plain C++, no HIP).
#include "tokens.h"

#include <string.h>

#include <algorithm>

#include "internal.h"

namespace nbsgd {

namespace {
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
}  // namespace

nbsgd_status check_groups(int32_t n, int32_t m, const uint8_t* mask, Groups* g) {
  if (nbsgd_status st = check_nm(n, m)) return st;
  if (!mask) return fail(NBSGD_E_ARG, "mask is null");
  memset(g, 0, sizeof *g);
  g->m = m;
  for (int32_t k = 0; k < n * m; ++k)
    if (mask[k]) {
      g->w[g->count >> 1] |= (uint32_t)k << (16 * (g->count & 1));
      ++g->count;
    }
  return NBSGD_OK;
}

bool rows_apart(const Rows& a, const Rows& b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return true;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  const uint64_t la = (uint64_t)(a.rows - 1) * a.stride + a.width;
  const uint64_t lb = (uint64_t)(b.rows - 1) * b.stride + b.width;
  if (a0 + la <= b0 || b0 + lb <= a0) return true;
  if (a.stride != b.stride) return false;
  // b's rows begin `off` bytes into a's period: they fit between two of a's rows
  const int64_t period = a.stride;
  const int64_t off = (int64_t)(((int64_t)(b0 - a0) % period + period) % period);
  return off >= a.width && off + b.width <= period;
}

nbsgd_status check_apart(const Rows* b, int count, int outs) {
  for (int i = 0; i < outs; ++i)
    for (int k = i + 1; k < count; ++k)
      if (!rows_apart(b[i], b[k]))
        return fail(NBSGD_E_ARG, "%s and %s overlap", b[i].name, b[k].name);
  return NBSGD_OK;
}

nbsgd_status check_params(const char* name, const void* p, int64_t ld, int64_t params) {
  if (ld < params || ld % 4)
    return fail(NBSGD_E_SHAPE, "row stride %lld must be a multiple of 4 and hold the %lld floats of %s",
                (long long)ld, (long long)params, name);
  if (ld > (int64_t)1 << 40)
    return fail(NBSGD_E_SHAPE, "row stride %lld of %s exceeds 2^40", (long long)ld, name);
  if (!p) return fail(NBSGD_E_ARG, "%s is null", name);
  if ((uintptr_t)p & 15) return fail(NBSGD_E_ALIGN, "%s must be 16-byte aligned", name);
  return NBSGD_OK;
}

nbsgd_status check_rows(const char* name, const void* p, int64_t rows, int64_t width, int64_t ld,
                        int elem) {
  if (ld < width || ld > (int64_t)1 << 31)
    return fail(NBSGD_E_SHAPE, "rows of %s: stride %lld must lie in [%lld, 2^31]", name, (long long)ld,
                (long long)width);
  if (!p && rows > 0) return fail(NBSGD_E_ARG, "%s is null", name);
  if ((uintptr_t)p & (uintptr_t)(elem - 1))
    return fail(NBSGD_E_ALIGN, "%s is not aligned to its element", name);
  return NBSGD_OK;
}

nbsgd_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return NBSGD_OK;
  if (!ws) return fail(NBSGD_E_ARG, "workspace is null");
  if ((uintptr_t)ws & 15) return fail(NBSGD_E_ALIGN, "workspace must be 16-byte aligned");
  if (bytes < need)
    return fail(NBSGD_E_ARG, "workspace of %zu bytes is below the %zu needed", bytes, need);
  return NBSGD_OK;
}

// ---------------------------------------------------------------- embeddings
nbsgd_status check_embed(int32_t T, int32_t vocab, int32_t dim) {
  if (T < 0 || vocab < 1 || dim < 1)
    return fail(NBSGD_E_SHAPE, "T=%d must be >= 0, vocab=%d and dim=%d >= 1", T, vocab, dim);
  if (T > NBSGD_MAX_TOKENS || vocab > NBSGD_MAX_VOCAB || dim > NBSGD_MAX_WIDTH)
    return fail(NBSGD_E_UNSUPPORTED, "T=%d, vocab=%d, dim=%d: at most %d, %d, %d", T, vocab, dim,
                NBSGD_MAX_TOKENS, NBSGD_MAX_VOCAB, NBSGD_MAX_WIDTH);
  return NBSGD_OK;
}

EmbedSpace embed_space(int64_t groups, int64_t T, int64_t dim) {
  EmbedSpace s;
  // of 32 tokens (16 mini-batches of 8192 x 512: 264 us, 16 tokens 267, 64 tokens 272); of 16
  // where a mini-batch has few and the time is a piece's own
  s.items = T < 64 * kMaxPiece ? 16 : kMaxPiece;
  s.pieces = ceil_div(T, s.items);
  s.keys = 0;
  s.sorted = s.keys + up256((size_t)groups * T * 8);
  s.flags = s.sorted + up256((size_t)groups * T * 8);
  s.parts = s.flags + up256((size_t)groups * s.pieces * 4);
  s.total = s.parts + up256((size_t)groups * s.pieces * 2 * dim * 4);
  return s;
}

// ---------------------------------------------------------------- recurrence
nbsgd_status check_scan(int32_t n, int32_t m, int32_t batch, int32_t T, int32_t dim) {
  if (nbsgd_status st = check_nm(n, m)) return st;
  if (batch < 1 || T < 0 || dim < 1)
    return fail(NBSGD_E_SHAPE, "batch=%d and dim=%d must be >= 1, T=%d >= 0", batch, dim, T);
  if (T > NBSGD_MAX_LENGTH || dim > NBSGD_MAX_WIDTH)
    return fail(NBSGD_E_UNSUPPORTED, "T=%d, dim=%d: at most %d, %d", T, dim, NBSGD_MAX_LENGTH,
                NBSGD_MAX_WIDTH);
  if ((int64_t)n * m * batch * ceil_div(dim, 64) > (int64_t)1 << 21)
    return fail(NBSGD_E_UNSUPPORTED, "n=%d, m=%d, batch=%d, dim=%d: too many sequences", n, m, batch,
                dim);
  return NBSGD_OK;
}

ScanSpace scan_space(int64_t seqs, int64_t T, int64_t dim) {
  ScanSpace s;
  s.tiles = ceil_div(T, kScanTile);
  const size_t cells = (size_t)seqs * s.tiles * dim;
  s.pairs = 0;
  s.carry = s.pairs + up256(cells * 8);
  s.bias = s.carry + up256(cells * 4);
  s.total = s.bias + up256(cells * 4 * kScanWaves);
  return s;
}

// ---------------------------------------------------------- 8-bit activations
nbsgd_status check_act8(int32_t T, int32_t dim) {
  if (T < 0 || dim < 1) return fail(NBSGD_E_SHAPE, "T=%d must be >= 0 and dim=%d >= 1", T, dim);
  if (T > NBSGD_MAX_TOKENS || dim > NBSGD_MAX_WIDTH)
    return fail(NBSGD_E_UNSUPPORTED, "T=%d, dim=%d: at most %d, %d", T, dim, NBSGD_MAX_TOKENS,
                NBSGD_MAX_WIDTH);
  return NBSGD_OK;
}

int act8_splits(int64_t T, int64_t dim, int64_t out) {
  const int64_t tiles = ceil_div(dim, 64) * ceil_div(out, 128);
  const int64_t tokens = std::max(kSplitTokens, 12 * dim * out / (dim + 2 * out));
  return (int)std::max<int64_t>(1, std::min(kSplitTiles / tiles, T / tokens));
}

size_t act8_space(int64_t groups, int64_t T, int64_t dim, int64_t out) {
  const int s = act8_splits(T, dim, out);
  return s > 1 ? up256((size_t)groups * s * dim * out * 4) : 0;
}

}  // namespace nbsgd

using namespace nbsgd;

extern "C" nbsgd_status nbsgd_embed_workspace_bytes(int32_t n, int32_t m, int32_t T, int32_t vocab,
                                                    int32_t dim, size_t* bytes) {
  clear_error();
  if (nbsgd_status st = check_nm(n, m)) return st;
  if (nbsgd_status st = check_embed(T, vocab, dim)) return st;
  if (!bytes) return fail(NBSGD_E_ARG, "bytes is null");
  *bytes = embed_space((int64_t)n * m, T, dim).total;
  return NBSGD_OK;
}

extern "C" nbsgd_status nbsgd_scan_workspace_bytes(int32_t n, int32_t m, int32_t batch, int32_t T,
                                                   int32_t dim, size_t* bytes) {
  clear_error();
  if (nbsgd_status st = check_scan(n, m, batch, T, dim)) return st;
  if (!bytes) return fail(NBSGD_E_ARG, "bytes is null");
  *bytes = scan_space((int64_t)n * m * batch, T, dim).total;
  return NBSGD_OK;
}

extern "C" nbsgd_status nbsgd_act_bytes(int32_t T, int32_t dim, int64_t* bytes) {
  clear_error();
  if (nbsgd_status st = check_act8(T, dim)) return st;
  if (!bytes) return fail(NBSGD_E_ARG, "bytes is null");
  *bytes = act8_layout(T, dim).bytes;
  return NBSGD_OK;
}

extern "C" nbsgd_status nbsgd_act_workspace_bytes(int32_t n, int32_t m, int32_t T, int32_t dim,
                                                   int32_t out, size_t* bytes) {
  clear_error();
  if (nbsgd_status st = check_nm(n, m)) return st;
  if (nbsgd_status st = check_act8(T, dim)) return st;
  if (out < 1 || out > NBSGD_MAX_WIDTH)
    return fail(out < 1 ? NBSGD_E_SHAPE : NBSGD_E_UNSUPPORTED, "out=%d must lie in [1, %d]", out,
                NBSGD_MAX_WIDTH);
  if (!bytes) return fail(NBSGD_E_ARG, "bytes is null");
  *bytes = act8_space((int64_t)n * m, T, dim, out);
  return NBSGD_OK;
}
