// Gated linear recurrence over long sequences and its backward pass (gfx950):
//   a_t = sigmoid(g_t + bias), h_t = a_t h_{t-1} + (1 - a_t) x_t, a state a channel.
#include "device_rows.h"

using namespace nbsgd;

namespace {

// Gate and complement of z, both accurate where they are small (1 - a would cancel).
struct Gate {
  float a, rest;
};
__device__ __forceinline__ Gate gate(float z) {
  const float e = expf(-fabsf(z));
  const float r = 1.f / (1.f + e), s = e * r;
  return z >= 0.f ? Gate{r, s} : Gate{s, r};
}

// What both passes are told of a call.
template <typename T>
struct Call {
  const T *x, *g;
  const float* bias;       // learner 0's, or null
  const int32_t* lengths;  // or null
  int64_t ldx, ld;
  int32_t batch, T_, dim, tiles;
  Groups groups;
};

template <typename T>
__global__ void __launch_bounds__(64)
    k_scan_serial(Call<T> c, const float* __restrict__ h0, T* __restrict__ h, int64_t ldh,
                  float* __restrict__ h_last, float* __restrict__ states) {
  const int cols = (c.dim + 63) / 64, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 64 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = c.bias ? c.bias[(int64_t)(id / c.groups.m) * c.ld + ch] : 0.f;
  const int len = c.lengths ? min(max(c.lengths[seq], 0), c.T_) : c.T_;
  float s = h0 ? h0[seq * c.dim + ch] : 0.f;
  for (int t = 0; t < c.T_; ++t) {
    if (states && t % kScanTile == 0) states[(seq * c.tiles + t / kScanTile) * c.dim + ch] = s;
    const int64_t row = seq * c.T_ + t;
    if (t < len) {
      const Gate q = gate(Elem<T>::load(c.g + row * c.ldx + ch) + bias);
      s = q.a * s + q.rest * Elem<T>::load(c.x + row * c.ldx + ch);
    }
    Elem<T>::store(h + row * ldh + ch, t < len ? s : 0.f);
  }
  if (h_last) h_last[seq * c.dim + ch] = s;
}

// From the last tile to the first: the tile's states again from the one before it, kept in
// LDS, then the gradients from its last token to its first.
template <typename T>
__global__ void __launch_bounds__(64)
    k_scan_grad_serial(Call<T> c, const float* __restrict__ states, const T* __restrict__ dh,
                       int64_t lddh, const float* __restrict__ dh_last, T* __restrict__ dx,
                       T* __restrict__ dg, float* __restrict__ dh0, float* __restrict__ part) {
  __shared__ float before[kScanTile][64];
  const int cols = (c.dim + 63) / 64, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 64 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = c.bias ? c.bias[(int64_t)(id / c.groups.m) * c.ld + ch] : 0.f;
  const int len = c.lengths ? min(max(c.lengths[seq], 0), c.T_) : c.T_;
  float mu = dh_last ? dh_last[seq * c.dim + ch] : 0.f;
  for (int tile = c.tiles - 1; tile >= 0; --tile) {
    const int t0 = tile * kScanTile, t1 = min(t0 + kScanTile, c.T_);
    float s = states[(seq * c.tiles + tile) * c.dim + ch], sum = 0.f;
    for (int t = t0; t < min(t1, len); ++t) {
      const int64_t row = (seq * c.T_ + t) * c.ldx + ch;
      before[t - t0][threadIdx.x] = s;
      const Gate q = gate(Elem<T>::load(c.g + row) + bias);
      s = q.a * s + q.rest * Elem<T>::load(c.x + row);
    }
    for (int t = t1 - 1; t >= t0; --t) {
      const int64_t row = (seq * c.T_ + t) * c.ldx + ch;
      float vx = 0.f, vg = 0.f;
      if (t < len) {
        const Gate q = gate(Elem<T>::load(c.g + row) + bias);
        const float lam = Elem<T>::load(dh + (seq * c.T_ + t) * lddh + ch) + mu;
        vx = lam * q.rest;
        vg = vx * q.a * (before[t - t0][threadIdx.x] - Elem<T>::load(c.x + row));
        mu = q.a * lam;
      }
      sum += vg;
      Elem<T>::store(dx + row, vx);
      Elem<T>::store(dg + row, vg);
    }
    part[(seq * c.tiles + tile) * c.dim + ch] = sum;
  }
  if (dh0) dh0[seq * c.dim + ch] = mu;
}

// Bias gradient of a mini-batch: its sequences' `rows` partial sums each, in order.
__global__ void __launch_bounds__(64)
    k_scan_bias(const float* __restrict__ part, int64_t rows, int dim, float* __restrict__ G,
                int64_t ld, Groups groups) {
  const int ch = blockIdx.x * 64 + threadIdx.x;
  if (ch >= dim) return;
  const int id = group_id(groups, blockIdx.y);
  const float* p = part + id * rows * dim + ch;
  float sum = 0.f;
  for (int64_t r = 0; r < rows; ++r) sum += p[r * dim];
  G[(int64_t)id * ld + ch] = sum;
}

template <typename T>
nbsgd_status fill_call(Call<T>* c, const void* x, const void* g, int64_t ldx, int32_t n, int32_t m,
                       int32_t batch, int32_t Tn, int32_t dim, const float* bias, int64_t ld,
                       const int32_t* lengths, const uint8_t* mask) {
  c->x = static_cast<const T*>(x);
  c->g = static_cast<const T*>(g);
  c->bias = bias;
  c->lengths = lengths;
  c->ldx = ldx;
  c->ld = ld;
  c->batch = batch;
  c->T_ = Tn;
  c->dim = dim;
  c->tiles = (int32_t)ceil_div(Tn, kScanTile);
  return check_groups(n, m, mask, &c->groups);
}

template <typename T>
nbsgd_status scan_forward(const void* x, const void* g, int64_t ldx, int32_t n, int32_t m,
                          int32_t batch, int32_t Tn, int32_t dim, const float* bias, int64_t ld,
                          const int32_t* lengths, const uint8_t* mask, const float* h0, void* h,
                          int64_t ldh, float* h_last, float* states, void* ws, hipStream_t s) {
  (void)ws;
  Call<T> c;
  if (nbsgd_status st = fill_call(&c, x, g, ldx, n, m, batch, Tn, dim, bias, ld, lengths, mask))
    return st;
  if (!c.groups.count) return NBSGD_OK;
  const unsigned cols = (unsigned)ceil_div(dim, 64);
  const dim3 grid(cols * c.groups.count * batch);
  hipLaunchKernelGGL(k_scan_serial<T>, grid, dim3(64), 0, s, c, h0, static_cast<T*>(h), ldh, h_last,
                     states);
  return launched("nbsgd_scan");
}

template <typename T>
nbsgd_status scan_backward(const void* x, const void* g, int64_t ldx, int32_t n, int32_t m,
                           int32_t batch, int32_t Tn, int32_t dim, const float* bias, int64_t ld,
                           const int32_t* lengths, const uint8_t* mask, const float* states,
                           const void* dh, int64_t lddh, const float* dh_last, void* dx, void* dg,
                           float* dh0, float* Gbias, void* ws, hipStream_t s) {
  Call<T> c;
  if (nbsgd_status st = fill_call(&c, x, g, ldx, n, m, batch, Tn, dim, bias, ld, lengths, mask))
    return st;
  if (!c.groups.count) return NBSGD_OK;
  const ScanSpace w = scan_space((int64_t)n * m * batch, Tn, dim);
  float* part = reinterpret_cast<float*>(static_cast<char*>(ws) + w.bias);
  const unsigned cols = (unsigned)ceil_div(dim, 64);
  const dim3 grid(cols * c.groups.count * batch);
  hipLaunchKernelGGL(k_scan_grad_serial<T>, grid, dim3(64), 0, s, c, states,
                     static_cast<const T*>(dh), lddh, dh_last, static_cast<T*>(dx),
                     static_cast<T*>(dg), dh0, part);
  if (Gbias)
    hipLaunchKernelGGL(k_scan_bias, dim3(cols, c.groups.count), dim3(64), 0, s, part,
                       (int64_t)batch * c.tiles, dim, Gbias, ld, c.groups);
  return launched("nbsgd_scan_grad");
}

}  // namespace

extern "C" nbsgd_status nbsgd_scan(const void* x, const void* g, int64_t ldx, int32_t dtype, int32_t n,
                                   int32_t m, int32_t batch, int32_t T, int32_t dim,
                                   const float* bias, int64_t ld, const int32_t* lengths,
                                   const uint8_t* mask, const float* h0, void* h, int64_t ldh,
                                   float* h_last, float* states, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  clear_error();
  if (nbsgd_status st = check_scan(n, m, batch, T, dim)) return st;
  const int e = dtype_size(dtype);
  if (!e) return fail(NBSGD_E_ARG, "unknown dtype %d", dtype);
  if (!mask) return fail(NBSGD_E_ARG, "mask is null");
  const int64_t seqs = (int64_t)n * m * batch, rows = seqs * T, width = (int64_t)dim * e;
  if (nbsgd_status st = check_rows("x", x, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_rows("g", g, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_rows("h", h, rows, dim, ldh, e)) return st;
  if (bias)
    if (nbsgd_status st = check_params("bias", bias, ld, dim)) return st;
  if (((uintptr_t)h0 | (uintptr_t)h_last | (uintptr_t)states | (uintptr_t)lengths) & 3)
    return fail(NBSGD_E_ALIGN, "h0, h_last, states and lengths must be 4-byte aligned");
  const ScanSpace w = scan_space(seqs, T, dim);
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, w.total)) return st;
  const int64_t kept = seqs * dim * 4, all = kept * w.tiles;
  const Rows b[] = {{"h", h, rows, width, ldh * e},
                    {"h_last", h_last, 1, kept, kept},
                    {"states", states, 1, all, all},
                    {"workspace", workspace, 1, (int64_t)w.total, (int64_t)w.total},
                    {"x", x, rows, width, ldx * e},
                    {"g", g, rows, width, ldx * e},
                    {"h0", h0 == h_last ? nullptr : h0, 1, kept, kept},
                    {"bias", bias, n, (int64_t)dim * 4, ld * 4},
                    {"lengths", lengths, 1, seqs * 4, seqs * 4}};
  if (nbsgd_status st = check_apart(b, 9, 4)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return dtype == NBSGD_F32
             ? scan_forward<float>(x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask, h0, h,
                                   ldh, h_last, states, workspace, s)
             : scan_forward<__bf16>(x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask, h0, h,
                                    ldh, h_last, states, workspace, s);
}

extern "C" nbsgd_status nbsgd_scan_grad(const void* x, const void* g, int64_t ldx, int32_t dtype,
                                        int32_t n, int32_t m, int32_t batch, int32_t T, int32_t dim,
                                        const float* bias, int64_t ld, const int32_t* lengths,
                                        const uint8_t* mask, const float* states, const void* dh,
                                        int64_t lddh, const float* dh_last, void* dx, void* dg,
                                        float* dh0, float* Gbias, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  clear_error();
  if (nbsgd_status st = check_scan(n, m, batch, T, dim)) return st;
  const int e = dtype_size(dtype);
  if (!e) return fail(NBSGD_E_ARG, "unknown dtype %d", dtype);
  if (!mask) return fail(NBSGD_E_ARG, "mask is null");
  const int64_t seqs = (int64_t)n * m * batch, rows = seqs * T, width = (int64_t)dim * e;
  if (nbsgd_status st = check_rows("x", x, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_rows("g", g, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_rows("dh", dh, rows, dim, lddh, e)) return st;
  if (nbsgd_status st = check_rows("dx", dx, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_rows("dg", dg, rows, dim, ldx, e)) return st;
  if (bias)
    if (nbsgd_status st = check_params("bias", bias, ld, dim)) return st;
  if (Gbias)
    if (nbsgd_status st = check_params("Gbias", Gbias, ld, dim)) return st;
  if (!states && rows) return fail(NBSGD_E_ARG, "states is null");
  if (((uintptr_t)dh0 | (uintptr_t)dh_last | (uintptr_t)states | (uintptr_t)lengths) & 3)
    return fail(NBSGD_E_ALIGN, "dh0, dh_last, states and lengths must be 4-byte aligned");
  const ScanSpace w = scan_space(seqs, T, dim);
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, w.total)) return st;
  const int64_t kept = seqs * dim * 4, all = kept * w.tiles;
  const Rows b[] = {{"dx", dx, rows, width, ldx * e},
                    {"dg", dg, rows, width, ldx * e},
                    {"dh0", dh0, 1, kept, kept},
                    {"Gbias", Gbias, (int64_t)n * m, (int64_t)dim * 4, ld * 4},
                    {"workspace", workspace, 1, (int64_t)w.total, (int64_t)w.total},
                    {"x", x, rows, width, ldx * e},
                    {"g", g, rows, width, ldx * e},
                    {"dh", dh, rows, width, lddh * e},
                    {"dh_last", dh_last == dh0 ? nullptr : dh_last, 1, kept, kept},
                    {"states", states, 1, all, all},
                    {"bias", bias, n, (int64_t)dim * 4, ld * 4},
                    {"lengths", lengths, 1, seqs * 4, seqs * 4}};
  if (nbsgd_status st = check_apart(b, 12, 5)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return dtype == NBSGD_F32
             ? scan_backward<float>(x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask, states,
                                    dh, lddh, dh_last, dx, dg, dh0, Gbias, workspace, s)
             : scan_backward<__bf16>(x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask, states,
                                     dh, lddh, dh_last, dx, dg, dh0, Gbias, workspace, s);
}
