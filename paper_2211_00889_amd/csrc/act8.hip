// Activations kept in 8 bits for the backward pass, and the weight gradient of a layer from
// them (gfx950).  Packed layout of a mini-batch: block of 32 tokens, channel, 32 int8; then
// group of four blocks, channel, four step exponents (k + 127; 255 for NaNs).
#include "device_rows.h"

using namespace nbsgd;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float step_of(uint32_t byte) {  // 2^(byte - 127), NaN for 255
  return byte == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
}

// Smallest k in [-126, 121] with rne(peak / 2^k) <= 127, plus 127; 255 for infinity and NaN.
__device__ __forceinline__ uint32_t step_byte(float peak) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, peak);
  const int e = (int)(bits >> 23);          // peak = m 2^(e - 126), m in [0.5, 1)
  if (e == 255) return 255u;
  // rne(peak / 2^k) reaches 128 where the top 8 significant bits are ones
  const int k = e - 126 - 7 + ((bits & 0x7fffffu) >= 0x7f0000u ? 1 : 0);
  return (uint32_t)(min(max(k, -126), 121) + 127);
}

// A thread a channel and block of 32 tokens.
template <typename T>
__global__ void __launch_bounds__(256)
    k_act8_pack(const T* __restrict__ A, int64_t lda, int Tn, int dim, uint8_t* __restrict__ packed,
                Act8 lay, Groups groups) {
  const int ch = blockIdx.x * 256 + threadIdx.x;
  if (ch >= dim) return;
  const int64_t blk = blockIdx.y;
  const int64_t id = group_id(groups, blockIdx.z);
  const int t0 = (int)blk * kActBlock, live = min(kActBlock, Tn - t0);
  const T* src = A + (id * Tn + t0) * lda + ch;
  float v[kActBlock];
  uint32_t peak = 0;  // as bits: a NaN stays the largest
#pragma unroll
  for (int t = 0; t < kActBlock; ++t) {
    v[t] = t < live ? Elem<T>::load(src + t * lda) : 0.f;
    peak = max(peak, __builtin_bit_cast(uint32_t, v[t]) & 0x7fffffffu);
  }
  const uint32_t byte = step_byte(__builtin_bit_cast(float, peak));
  const float inv = byte == 255u ? 0.f : __builtin_bit_cast(float, (254u - byte) << 23);
  uint8_t* base = packed + id * lay.bytes;
  uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (byte != 255u) {
#pragma unroll
    for (int t = 0; t < kActBlock; ++t) {
      const int q = (int)fminf(fmaxf(rintf(v[t] * inv), -127.f), 127.f);
      w[t >> 2] |= ((uint32_t)q & 0xffu) << (8 * (t & 3));
    }
  }
  u32x4* dst = reinterpret_cast<u32x4*>(base + (blk * dim + ch) * kActBlock);
  dst[0] = (u32x4){w[0], w[1], w[2], w[3]};
  dst[1] = (u32x4){w[4], w[5], w[6], w[7]};
  uint8_t* steps = base + lay.scale + ((blk >> 2) * dim + ch) * 4;
  steps[blk & 3] = (uint8_t)byte;
  if (blk == lay.blocks - 1)  // the rest of the last four
    for (int k = (int)(blk & 3) + 1; k < 4; ++k) steps[k] = 0;
}

template <typename T>
__global__ void __launch_bounds__(256)
    k_act8_unpack(const uint8_t* __restrict__ packed, int Tn, int dim, T* __restrict__ A, int64_t lda,
                  Act8 lay, Groups groups) {
  const int ch = blockIdx.x * 256 + threadIdx.x;
  if (ch >= dim) return;
  const int64_t blk = blockIdx.y;
  const int64_t id = group_id(groups, blockIdx.z);
  const int t0 = (int)blk * kActBlock, live = min(kActBlock, Tn - t0);
  const uint8_t* base = packed + id * lay.bytes;
  const u32x4* src = reinterpret_cast<const u32x4*>(base + (blk * dim + ch) * kActBlock);
  const u32x4 w[2] = {src[0], src[1]};
  const float step = step_of(base[lay.scale + ((blk >> 2) * dim + ch) * 4 + (blk & 3)]);
  T* dst = A + (id * Tn + t0) * lda + ch;
#pragma unroll
  for (int t = 0; t < kActBlock; ++t)
    if (t < live)
      Elem<T>::store(dst + t * lda, step * (float)(int8_t)(w[t >> 4][(t >> 2) & 3] >> (8 * (t & 3))));
}

// One wave 16 channels x 64 columns, MFMA 16x16x32 a block of 32 tokens.
// Operands (lane l, t = 0..7): A[l % 16][8 (l / 16) + t], B[8 (l / 16) + t][l % 16]; result
// D[4 (l / 16) + t][l % 16], t = 0..3.
__global__ void __launch_bounds__(64)
    k_act8_grad_plain(const uint8_t* __restrict__ packed, const __bf16* __restrict__ dY, int64_t ldy,
                      int Tn, int dim, int out, float* __restrict__ G, int64_t ld, Act8 lay,
                      Groups groups) {
  const int lane = threadIdx.x, i = lane & 15, g = lane >> 4;
  const int64_t id = group_id(groups, blockIdx.z);
  const int k0 = blockIdx.y * 16, c0 = blockIdx.x * 64;
  const uint8_t* base = packed + id * lay.bytes;
  const __bf16* rows = dY + id * Tn * ldy;
  const int64_t ch = min(k0 + i, dim - 1);
  f32x4 acc[4] = {};
  for (int64_t blk = 0; blk < lay.blocks; ++blk) {
    const u32x2 q = *reinterpret_cast<const u32x2*>(base + (blk * dim + ch) * kActBlock + 8 * g);
    const float step = step_of(base[lay.scale + ((blk >> 2) * dim + ch) * 4 + (blk & 3)]);
    bf16x8 a;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      a[t] = (__bf16)(step * (float)(int8_t)(q[t >> 2] >> (8 * (t & 3))));
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int col = c0 + 16 * f + i;
      bf16x8 b;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int64_t tok = blk * kActBlock + 8 * g + t;
        b[t] = tok < Tn && col < out ? rows[tok * ldy + col] : (__bf16)0.f;
      }
      acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc[f], 0, 0, 0);
    }
  }
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int k = k0 + 4 * g + t, col = c0 + 16 * f + i;
      if (k < dim && col < out) G[id * ld + (int64_t)k * out + col] = acc[f][t];
    }
}

template <typename T>
nbsgd_status pack_launch(const void* A, int64_t lda, int32_t Tn, int32_t dim, void* packed,
                         const Groups& g, hipStream_t s) {
  const Act8 lay = act8_layout(Tn, dim);
  const dim3 grid((unsigned)ceil_div(dim, 256), (unsigned)lay.blocks, g.count);
  hipLaunchKernelGGL(k_act8_pack<T>, grid, dim3(256), 0, s, static_cast<const T*>(A), lda, Tn, dim,
                     static_cast<uint8_t*>(packed), lay, g);
  return launched("nbsgd_act_pack");
}

template <typename T>
nbsgd_status unpack_launch(const void* packed, int32_t Tn, int32_t dim, void* A, int64_t lda,
                           const Groups& g, hipStream_t s) {
  const Act8 lay = act8_layout(Tn, dim);
  const dim3 grid((unsigned)ceil_div(dim, 256), (unsigned)lay.blocks, g.count);
  hipLaunchKernelGGL(k_act8_unpack<T>, grid, dim3(256), 0, s, static_cast<const uint8_t*>(packed), Tn,
                     dim, static_cast<T*>(A), lda, lay, g);
  return launched("nbsgd_act_unpack");
}

// Checks shared by the two directions.
nbsgd_status check_pack(const void* A, int64_t lda, int32_t dtype, int32_t n, int32_t m, int32_t Tn,
                        int32_t dim, const uint8_t* mask, const void* packed, void* stream,
                        Groups* g) {
  if (nbsgd_status st = check_groups(n, m, mask, g)) return st;
  if (nbsgd_status st = check_act8(Tn, dim)) return st;
  const int e = dtype_size(dtype);
  if (!e) return fail(NBSGD_E_ARG, "unknown dtype %d", dtype);
  const int64_t rows = (int64_t)n * m * Tn, bytes = (int64_t)n * m * act8_layout(Tn, dim).bytes;
  if (nbsgd_status st = check_rows("A", A, rows, dim, lda, e)) return st;
  if (!packed && bytes) return fail(NBSGD_E_ARG, "packed is null");
  if ((uintptr_t)packed & 15) return fail(NBSGD_E_ALIGN, "packed must be 16-byte aligned");
  const Rows b[] = {{"packed", packed, 1, bytes, bytes}, {"A", A, rows, (int64_t)dim * e, lda * e}};
  if (nbsgd_status st = check_apart(b, 2, 1)) return st;
  return check_stream(stream);
}

}  // namespace

extern "C" nbsgd_status nbsgd_act_pack(const void* A, int64_t lda, int32_t dtype, int32_t n, int32_t m,
                                        int32_t T, int32_t dim, const uint8_t* mask, void* packed,
                                        void* stream) {
  clear_error();
  Groups g;
  if (nbsgd_status st = check_pack(A, lda, dtype, n, m, T, dim, mask, packed, stream, &g)) return st;
  if (!g.count || !T) return NBSGD_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return dtype == NBSGD_F32 ? pack_launch<float>(A, lda, T, dim, packed, g, s)
                            : pack_launch<__bf16>(A, lda, T, dim, packed, g, s);
}

extern "C" nbsgd_status nbsgd_act_unpack(const void* packed, int32_t n, int32_t m, int32_t T,
                                          int32_t dim, const uint8_t* mask, void* A, int64_t lda,
                                          int32_t dtype, void* stream) {
  clear_error();
  Groups g;
  if (nbsgd_status st = check_pack(A, lda, dtype, n, m, T, dim, mask, packed, stream, &g)) return st;
  if (!g.count || !T) return NBSGD_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return dtype == NBSGD_F32 ? unpack_launch<float>(packed, T, dim, A, lda, g, s)
                            : unpack_launch<__bf16>(packed, T, dim, A, lda, g, s);
}

extern "C" nbsgd_status nbsgd_act_grad(const void* packed, const void* dY, int64_t ldy, int32_t n,
                                        int32_t m, int32_t T, int32_t dim, int32_t out,
                                        const uint8_t* mask, float* G, int64_t ld, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  clear_error();
  Groups g;
  if (nbsgd_status st = check_groups(n, m, mask, &g)) return st;
  if (nbsgd_status st = check_act8(T, dim)) return st;
  if (out < 1 || out > NBSGD_MAX_WIDTH)
    return fail(out < 1 ? NBSGD_E_SHAPE : NBSGD_E_UNSUPPORTED, "out=%d must lie in [1, %d]", out,
                NBSGD_MAX_WIDTH);
  const int64_t nm = (int64_t)n * m, rows = nm * T;
  const Act8 lay = act8_layout(T, dim);
  if (!packed && lay.bytes) return fail(NBSGD_E_ARG, "packed is null");
  if ((uintptr_t)packed & 15) return fail(NBSGD_E_ALIGN, "packed must be 16-byte aligned");
  if (nbsgd_status st = check_rows("dY", dY, rows, out, ldy, 2)) return st;
  if (nbsgd_status st = check_params("G", G, ld, (int64_t)dim * out)) return st;
  const size_t need = act8_space(nm, T, dim, out);
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, need)) return st;
  const Rows b[] = {{"G", G, nm, (int64_t)dim * out * 4, ld * 4},
                    {"workspace", workspace, 1, (int64_t)need, (int64_t)need},
                    {"packed", packed, 1, nm * lay.bytes, nm * lay.bytes},
                    {"dY", dY, rows, (int64_t)out * 2, ldy * 2}};
  if (nbsgd_status st = check_apart(b, 4, 2)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  if (!g.count) return NBSGD_OK;
  const dim3 grid((unsigned)ceil_div(out, 64), (unsigned)ceil_div(dim, 16), g.count);
  hipLaunchKernelGGL(k_act8_grad_plain, grid, dim3(64), 0, reinterpret_cast<hipStream_t>(stream),
                     static_cast<const uint8_t*>(packed), static_cast<const __bf16*>(dY), ldy, T, dim,
                     out, G, ld, lay, g);
  return launched("nbsgd_act_grad");
}
