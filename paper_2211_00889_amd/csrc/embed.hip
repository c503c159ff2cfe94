// Embedding lookup with scaling and its gradient, per learner and mini-batch (gfx950).
#include "device_rows.h"

using namespace nbsgd;

namespace {

// Y[t][:] = scale * E[token[t]][:]: a team of L lanes a token, 16 bytes of Y a lane.  What
// bounds it is the store of Y; the table's rows of frequent tokens come from the caches.
template <typename T>
__global__ void __launch_bounds__(256)
    k_embed(const float* __restrict__ E, int64_t ld, int vocab, int dim, float scale,
            const int32_t* __restrict__ tokens, int Tn, T* __restrict__ Y, int64_t ldy, int L,
            Groups groups) {
  constexpr int V = Elem<T>::V;
  const int id = group_id(groups, blockIdx.y);
  const float* table = E + (int64_t)(id / groups.m) * ld;
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (t >= Tn) return;
  const int64_t row = (int64_t)id * Tn + t;
  const int tok = tokens[row];
  const bool inside = tok >= 0 && tok < vocab;
  const float* src = table + (int64_t)(inside ? tok : 0) * dim;
  T* dst = Y + row * ldy;
  for (int c = (threadIdx.x % L) * V; c < dim; c += L * V) {
    const int n = min(V, dim - c);
    float v[V];
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      float w[4] = {0.f, 0.f, 0.f, 0.f};
      if (inside && n > 4 * q) Elem<float>::expand(load16<float>(src + c + 4 * q, n - 4 * q), w);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[4 * q + k] = inside ? scale * w[k] : 0.f;
    }
    store16<T>(dst + c, Elem<T>::collapse(v), n);
  }
}

// One wave a row of the table: the mini-batch's tokens are searched 64 at a time and the
// rows of dY that match are added in their order.
template <typename T>
__global__ void __launch_bounds__(64)
    k_embed_rows(const T* __restrict__ dY, int64_t ldy, const int32_t* __restrict__ tokens, int Tn,
                 int dim, float scale, float* __restrict__ G, int64_t ld, Groups groups) {
  const int id = group_id(groups, blockIdx.y);
  const int v = blockIdx.x, lane = threadIdx.x;
  const int32_t* tok = tokens + (int64_t)id * Tn;
  const T* rows = dY + (int64_t)id * Tn * ldy;
  float* out = G + (int64_t)id * ld + (int64_t)v * dim;
  for (int c0 = 0; c0 < dim; c0 += 64) {
    const int c = c0 + lane;
    float sum = 0.f;
    for (int t0 = 0; t0 < Tn; t0 += 64) {
      uint64_t hit = __ballot(t0 + lane < Tn && tok[min(t0 + lane, Tn - 1)] == v);
      while (hit) {
        const int t = t0 + __builtin_ctzll(hit);
        hit &= hit - 1;
        if (c < dim) sum += Elem<T>::load(rows + (int64_t)t * ldy + c);
      }
    }
    if (c < dim) out[c] = scale * sum;
  }
}

}  // namespace

extern "C" nbsgd_status nbsgd_embed(const float* E, int64_t ld, int32_t n, int32_t m, int32_t vocab,
                                    int32_t dim, float scale, const int32_t* tokens, int32_t T,
                                    const uint8_t* mask, void* Y, int64_t ldy, int32_t dtype,
                                    void* stream) {
  clear_error();
  Groups g;
  if (nbsgd_status st = check_groups(n, m, mask, &g)) return st;
  if (nbsgd_status st = check_embed(T, vocab, dim)) return st;
  const int e = dtype_size(dtype);
  if (!e) return fail(NBSGD_E_ARG, "unknown dtype %d", dtype);
  const int64_t rows = (int64_t)n * m * T;
  if (nbsgd_status st = check_params("E", E, ld, (int64_t)vocab * dim)) return st;
  if (nbsgd_status st = check_rows("tokens", tokens, rows, 1, 1, 4)) return st;
  if (nbsgd_status st = check_rows("Y", Y, rows, dim, ldy, e)) return st;
  const Rows b[] = {{"Y", Y, rows, (int64_t)dim * e, ldy * e},
                    {"E", E, n, (int64_t)vocab * dim * 4, ld * 4},
                    {"tokens", tokens, 1, rows * 4, rows * 4}};
  if (nbsgd_status st = check_apart(b, 3, 1)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  if (!g.count || !T) return NBSGD_OK;
  const int V = 16 / e;
  int L = 8;
  while (L < 64 && L * V < dim) L *= 2;
  const dim3 grid((unsigned)ceil_div(T, 256 / L), g.count);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == NBSGD_F32)
    hipLaunchKernelGGL(k_embed<float>, grid, dim3(256), 0, s, E, ld, vocab, dim, scale, tokens, T,
                       static_cast<float*>(Y), ldy, L, g);
  else
    hipLaunchKernelGGL(k_embed<__bf16>, grid, dim3(256), 0, s, E, ld, vocab, dim, scale, tokens, T,
                       static_cast<__bf16*>(Y), ldy, L, g);
  return launched("nbsgd_embed");
}

extern "C" nbsgd_status nbsgd_embed_grad(const void* dY, int64_t ldy, int32_t dtype, int32_t n,
                                         int32_t m, int32_t T, const int32_t* tokens, int32_t vocab,
                                         int32_t dim, float scale, const uint8_t* mask, float* G,
                                         int64_t ld, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  clear_error();
  Groups g;
  if (nbsgd_status st = check_groups(n, m, mask, &g)) return st;
  if (nbsgd_status st = check_embed(T, vocab, dim)) return st;
  const int e = dtype_size(dtype);
  if (!e) return fail(NBSGD_E_ARG, "unknown dtype %d", dtype);
  const int64_t rows = (int64_t)n * m * T;
  if (nbsgd_status st = check_rows("dY", dY, rows, dim, ldy, e)) return st;
  if (nbsgd_status st = check_rows("tokens", tokens, rows, 1, 1, 4)) return st;
  if (nbsgd_status st = check_params("G", G, ld, (int64_t)vocab * dim)) return st;
  const EmbedSpace w = embed_space((int64_t)n * m, T, vocab, dim);
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, w.total)) return st;
  const Rows b[] = {{"G", G, (int64_t)n * m, (int64_t)vocab * dim * 4, ld * 4},
                    {"workspace", workspace, 1, (int64_t)w.total, (int64_t)w.total},
                    {"dY", dY, rows, (int64_t)dim * e, ldy * e},
                    {"tokens", tokens, 1, rows * 4, rows * 4}};
  if (nbsgd_status st = check_apart(b, 4, 2)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  if (!g.count) return NBSGD_OK;
  const dim3 grid(vocab, g.count);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == NBSGD_F32)
    hipLaunchKernelGGL(k_embed_rows<float>, grid, dim3(64), 0, s, static_cast<const float*>(dY), ldy,
                       tokens, T, dim, scale, G, ld, g);
  else
    hipLaunchKernelGGL(k_embed_rows<__bf16>, grid, dim3(64), 0, s, static_cast<const __bf16*>(dY),
                       ldy, tokens, T, dim, scale, G, ld, g);
  return launched("nbsgd_embed_grad");
}
