// Activations kept in 8 bits for the backward pass, and the weight gradient of a layer from
// them (gfx950).  Packed layout of a mini-batch: block of 32 tokens, channel, 32 int8; then
// group of four blocks, channel, four step exponents (k + 127; 255 for NaNs).
#include <algorithm>
#include <type_traits>

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

// Packing and unpacking are copies with a transposition of 32 tokens: what bounds them is HBM.
// A thread takes V channels (8 bytes of a row in bf16, 16 in fp32) and 8 of a block's 32 tokens, four
// threads a block; the four put their parts of the peaks together by shuffles, and packing turns
// their 4 x 4 parts of 8 bytes, so that each writes the 32 bytes of one channel and a wave 16 V x 32
// contiguous ones.  A thread with a channel's whole block from the start (128 bytes a load of bf16)
// packed at 2.3 TB/s, this at 4.5.  It goes on to the next of four blocks, whose steps make one word.
template <typename T>
struct PackTile {
  static constexpr int V = 4, CH = 16 * V;  // channels of a wave
};

// The V elements at p, the first n of them; zeros behind.
__device__ __forceinline__ void load_v(const float* p, int n, float (&v)[4]) {
  Elem<float>::expand(load16(p, n), v);
}
__device__ __forceinline__ void load_v(const __bf16* p, int n, float (&v)[4]) {
  if (n >= 4) {
    const u32x2 r = *reinterpret_cast<const u32x2_any*>(p);
    v[0] = bf16_lo(r[0]), v[1] = bf16_hi(r[0]), v[2] = bf16_lo(r[1]), v[3] = bf16_hi(r[1]);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = k < n ? (float)p[k] : 0.f;
}
template <bool LINES>
__device__ __forceinline__ void store_v(float* p, int n, const float (&v)[4]) {
  if (LINES && n >= 4) __builtin_nontemporal_store(Elem<float>::collapse(v), reinterpret_cast<u32x4*>(p));
  else store16<float>(p, Elem<float>::collapse(v), n);
}
template <bool LINES>
__device__ __forceinline__ void store_v(__bf16* p, int n, const float (&v)[4]) {
  const u32x2 r = {pack2(v[0], v[1]), pack2(v[2], v[3])};
  if (n >= 4) {
    if (LINES) __builtin_nontemporal_store(r, reinterpret_cast<u32x2*>(p));
    else *reinterpret_cast<u32x2_any*>(p) = r;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) p[k] = (__bf16)v[k];
}

// The value of the lane whose number differs in bit D (0 or 1), within four lanes.
template <int D>
__device__ __forceinline__ uint32_t swap_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, D ? 0x4e : 0xb1, 0xf, 0xf, true);
}
// a of the lanes with bit D against b of those without it.
template <int D>
__device__ __forceinline__ void exchange(int lane, u32x2& a, u32x2& b) {
  const bool up = lane >> D & 1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t got = swap_lane<D>(up ? a[h] : b[h]);
    if (up) a[h] = got;
    else b[h] = got;
  }
}

// Lane: channels V (lane / 4) of the wave's, tokens 8 (lane % 4) of each of four blocks.
template <typename T>
__global__ void __launch_bounds__(256)
    k_act8_pack(const T* __restrict__ A, int64_t lda, int Tn, int dim, uint8_t* __restrict__ packed,
                Act8 lay, Groups groups) {
  constexpr int V = PackTile<T>::V, CH = PackTile<T>::CH;
  const int lane = threadIdx.x & 63, oct = lane & 3;
  const int ch = (blockIdx.x * 4 + (threadIdx.x >> 6)) * CH + (lane >> 2) * V;
  const int n = dim - ch;
  const int64_t id = group_id(groups, blockIdx.z);
  const T* src = A + id * Tn * lda + ch;
  uint8_t* base = packed + id * lay.bytes;
  const int64_t blk0 = 4 * (int64_t)blockIdx.y;
  uint32_t steps[V];
#pragma unroll
  for (int k = 0; k < V; ++k) steps[k] = 0u;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    if (blk0 + b >= lay.blocks) break;  // uniform
    const int t0 = (int)(blk0 + b) * kActBlock + 8 * oct;
    float v[8][V];
    uint32_t peak[V];  // as bits: a NaN stays the largest
#pragma unroll
    for (int k = 0; k < V; ++k) peak[k] = 0u;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (n > 0 && t0 + t < Tn) {
        load_v(src + (int64_t)(t0 + t) * lda, n, v[t]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[t][k] = 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int k = 0; k < V; ++k) peak[k] = max(peak[k], __builtin_bit_cast(uint32_t, v[t][k]) & 0x7fffffffu);
    u32x2 out[V];  // this lane's 8 tokens of its four channels
#pragma unroll
    for (int k = 0; k < V; ++k) {
      peak[k] = max(peak[k], swap_lane<0>(peak[k]));
      peak[k] = max(peak[k], swap_lane<1>(peak[k]));
      const uint32_t byte = step_byte(__builtin_bit_cast(float, peak[k]));
      steps[k] |= byte << (8 * b);
      const float inv = byte == 255u ? 0.f : __builtin_bit_cast(float, (254u - byte) << 23);
      uint32_t w[2] = {0u, 0u};
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int q = (int)fminf(fmaxf(rintf(v[t][k] * inv), -127.f), 127.f);
        w[t >> 2] |= ((uint32_t)q & 0xffu) << (8 * (t & 3));
      }
      out[k] = byte == 255u ? (u32x2){0u, 0u} : (u32x2){w[0], w[1]};
    }
    // four lanes turn their 4 x 4 parts, so that each has the 32 tokens of one channel
    exchange<0>(lane, out[0], out[1]);
    exchange<0>(lane, out[2], out[3]);
    exchange<1>(lane, out[0], out[2]);
    exchange<1>(lane, out[1], out[3]);
    if (oct < n) {
      u32x4* to = reinterpret_cast<u32x4*>(base + ((blk0 + b) * dim + ch + oct) * kActBlock);
      to[0] = (u32x4){out[0][0], out[0][1], out[1][0], out[1][1]};
      to[1] = (u32x4){out[2][0], out[2][1], out[3][0], out[3][1]};
    }
  }
  if (oct == 0) {
    uint32_t* to = reinterpret_cast<uint32_t*>(base + lay.scale) + (int64_t)blockIdx.y * dim + ch;
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k < n) to[k] = steps[k];
  }
}

// LINES: the rows are whole 128-byte lines, and go past the caches (32 mini-batches of 4096 x 1024
// bf16, packed before: 178 -> 164 us for both; rows of 1,000, off the lines, 117 -> 166).
template <typename T, bool LINES>
__global__ void __launch_bounds__(256)
    k_act8_unpack(const uint8_t* __restrict__ packed, int Tn, int dim, T* __restrict__ A, int64_t lda,
                  Act8 lay, Groups groups) {
  constexpr int V = PackTile<T>::V, CH = PackTile<T>::CH;
  const int lane = threadIdx.x & 63, oct = lane & 3;
  const int ch = (blockIdx.x * 4 + (threadIdx.x >> 6)) * CH + (lane >> 2) * V;
  const int n = dim - ch;
  if (n <= 0) return;
  const int64_t id = group_id(groups, blockIdx.z);
  const uint8_t* base = packed + id * lay.bytes;
  const uint32_t* from = reinterpret_cast<const uint32_t*>(base + lay.scale) + (int64_t)blockIdx.y * dim;
  const int64_t blk0 = 4 * (int64_t)blockIdx.y;
  uint32_t steps[V];
#pragma unroll
  for (int k = 0; k < V; ++k) steps[k] = from[min(ch + k, dim - 1)];
  T* dst = A + id * Tn * lda + ch;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    if (blk0 + b >= lay.blocks) break;  // uniform
    const int t0 = (int)(blk0 + b) * kActBlock + 8 * oct;
    u32x2 q[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
      q[k] = *reinterpret_cast<const u32x2*>(base + ((blk0 + b) * dim + min(ch + k, dim - 1)) * kActBlock + 8 * oct);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t0 + t >= Tn) break;
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k)
        v[k] = step_of(steps[k] >> (8 * b) & 0xffu) * (float)(int8_t)(q[k][t >> 2] >> (8 * (t & 3)));
      store_v<LINES>(dst + (int64_t)(t0 + t) * lda, n, v);
    }
  }
}

// Weight gradient dW = A^T dY: the tokens are the K of MFMA 16x16x32 (bf16, fp32 sums), 64 of
// them a stage of two steps.  Operands (lane l, g = l / 16, t = 0..7): A[l % 16][8 g + t], B[8 g +
// t][l % 16]; result D[4 g + t][l % 16], t = 0..3.  Which tokens a step's K are is free as long
// as both operands agree: of 64 tokens, octets 2 g of lanes g are step 0 and octets 2 g + 1 step 1,
// so that
//   A  (packed) is loaded 16 bytes a lane, 16 tokens of a channel, straight from memory, and
//      made bf16 in registers, q * 2^k exactly; every value once, since a wave has all columns
//      of its channels
//   B  (dY) comes a row a token: a thread turns 4 tokens x 8 columns and writes 8 bytes a
//      column to LDS, column 8 q + e of the tile to slot e * BN / 8 + q, so that the writes and
//      the fragment reads are contiguous and a lane's results of eight (or four) fragments are
//      consecutive columns.
// A wave takes 16 MT channels x 16 F columns, WM x WN waves a tile.  Two buffers of B; a stage's
// loads go out a whole stage before they are wanted.  Of eight waves, two on each SIMD (waves w
// and w + 4), the late half runs half a stage behind: while one wave of a SIMD multiplies, the
// other one unpacks, turns and loads, and two barriers a stage keep it so.
// 32 mini-batches of 4096 x 1024 x 2048: 473 us, 1.16 PFLOP/s (a library's bf16 product of
// 8192^3 reaches 1.17); 501-513 us over many passes, against 526 with both halves in step.  What
// bounds it is power: 0.92 million cycles at 1.95 GHz, 0.52 of them the MFMAs' own, where both
// halves in step and loads among the products took 1.21 million at 2.2 GHz.  Of 514 us, with an
// unpacking of as many instructions, no loads saved 94, half the MFMAs 63, no unpacking 56, no
// turning 32, no LDS reads 25.  128 tokens a stage, 64 channels x 256 or 128 columns a wave, two
// workgroups of four waves a CU took longer.
constexpr int kHB = 2, kStageTokens = kActBlock * kHB;
template <int MT, int F, int WM, int WN>
struct GradTile {
  static constexpr int kThreads = 64 * WM * WN, BM = 16 * MT * WM, BN = 16 * F * WN;
  static_assert(kStageTokens / 4 * (BN / 8) == kThreads, "a thread turns 4 tokens x 8 columns");
};

// What a launch is told: items (mini-batch, part of its tokens, tile), tiles fastest.
struct GradCall {
  const uint8_t* packed;
  const __bf16* dY;
  float* out;       // G, or the parts
  int64_t ldy, ld;  // of out: floats from one mini-batch to the next
  int64_t part;     // floats from one part to the next
  int32_t T, dim, cols, parts, per;  // per: blocks of a part, a multiple of four
  int32_t border;                    // act8_border
  int32_t tm, tn, items;
  Act8 lay;
  Groups groups;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// Eight bytes of a channel as bf16 on their step: q * 2^k exactly for every q and k, 127 * 2^121
// included (with 128 added to the bytes and its product taken off again, 128 * 2^121 is no fp32).
__device__ __forceinline__ bf16x8 unpack8(uint32_t q0, uint32_t q1, float step) {
  const uint32_t q[2] = {q0, q1};
  u32x4 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t u = q[h];
    r[2 * h] = pack2((float)(int8_t)u * step, (float)(int8_t)(u >> 8) * step);
    r[2 * h + 1] = pack2((float)(int8_t)(u >> 16) * step, (float)(int8_t)(u >> 24) * step);
  }
  return __builtin_bit_cast(bf16x8, r);
}

template <int MT, int F, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_act8_grad(GradCall c) {
  using S = GradTile<MT, F, WM, WN>;
  constexpr int BN = S::BN, Q = BN / 8, RING = 8, STEPS = kHB * F;
  __shared__ __attribute__((aligned(16))) u32x2 Bs[2][kStageTokens / 8][BN][2];
  // an XCD (workgroup b runs on XCD b % 8) takes a run of neighbouring tiles, which read the same
  // tokens through its L2
  const int xper = gridDim.x >> 3, item = (blockIdx.x & 7) * xper + (int)(blockIdx.x >> 3);
  if (item >= c.items) return;  // uniform
  const int tn = item % c.tn, tm = item / c.tn % c.tm, r = item / (c.tn * c.tm);
  const int part = r % c.parts;
  const int64_t id = group_id(c.groups, r / c.parts);
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int k0 = tm * S::BM + 16 * MT * wm, c0 = tn * BN;
  const int blk0 = part * c.per, blk1 = min(blk0 + c.per, (int)c.lay.blocks);
  const int tokens = min(blk1 * kActBlock, c.T);  // the next part's are left to it
  const int stages = (blk1 - blk0 + kHB - 1) / kHB;

  const uint8_t* base = c.packed + id * c.lay.bytes;
  const __bf16* rows = c.dY + id * c.T * c.ldy + c0;
  uint32_t aoff[MT], soff[MT];  // channels past the last read it: nothing stores what they give
#pragma unroll
  for (int a = 0; a < MT; ++a) {
    const uint32_t ch = (uint32_t)min(k0 + 16 * a + i, c.dim - 1);
    aoff[a] = ch * kActBlock + 16 * (g & 1);
    soff[a] = ch * 4;
  }
  const uint32_t aup = (uint32_t)(g >> 1) * (uint32_t)c.dim * kActBlock;  // to the lane's block of two
  const int four = tid / Q, q8 = tid % Q;  // the cell of B that this thread turns
  // cells past the last column turn the tile's first ones, and a cell at the border up to seven
  // elements of whatever follows its row: nothing stores what they give
  const uint32_t boff = 2u * (uint32_t)(4 * four * (int)c.ldy + (8 * q8 < c.cols - c0 ? 8 * q8 : 0));

  u32x4 qa[MT], rb[4];
  uint32_t sa[MT];
  // the first `plain` stages are read without looking
  const int plain = max(0, act8_sure(tokens, c.border, c0, BN, c.cols) / kActBlock - blk0) / kHB;
  auto load_rows = [&](int st) {
    const uint8_t* from = reinterpret_cast<const uint8_t*>(rows + (int64_t)(blk0 + kHB * st) * kActBlock * c.ldy);
#pragma unroll
    for (int t = 0; t < 4; ++t) rb[t] = *reinterpret_cast<const u32x4_any*>(from + 2 * t * c.ldy + boff);
  };
  auto load_packed = [&](int st) {
    const int64_t b = blk0 + kHB * st;
#pragma unroll
    for (int a = 0; a < MT; ++a) {
      qa[a] = *reinterpret_cast<const u32x4*>(base + b * c.dim * kActBlock + (aoff[a] + aup));
      sa[a] = *reinterpret_cast<const uint32_t*>(base + c.lay.scale + (b >> 2) * c.dim * 4 + soff[a]);
    }
  };
  // Any stage: blocks past the last are read as it, tokens and columns past the last as zeros
  auto any_rows = [&](int st) {
    const int b = blk0 + kHB * st, n = c.cols - c0 - 8 * q8;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int tok = b * kActBlock + 4 * four + t;
      rb[t] = (u32x4){0u, 0u, 0u, 0u};
      if (tok < tokens && n > 0) rb[t] = load16(rows + (int64_t)tok * c.ldy + 8 * q8, n);
    }
  };
  auto any_packed = [&](int st) {
    const int b = blk0 + kHB * st;
    const int blk = min(b + (g >> 1), blk1 - 1);
#pragma unroll
    for (int a = 0; a < MT; ++a) {
      qa[a] = *reinterpret_cast<const u32x4*>(base + (int64_t)blk * c.dim * kActBlock + aoff[a]);
      sa[a] = *reinterpret_cast<const uint32_t*>(base + c.lay.scale + (int64_t)(b >> 2) * c.dim * 4 + soff[a]);
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // tokens 2 p, 2 p + 1 of column e: the same half of two rows
      const uint32_t half = e & 1 ? 0x07060302u : 0x05040100u;
      Bs[buf][four >> 1][e * Q + q8][four & 1] = (u32x2){__builtin_amdgcn_perm(rb[1][e >> 1], rb[0][e >> 1], half),
                                                         __builtin_amdgcn_perm(rb[3][e >> 1], rb[2][e >> 1], half)};
    }
  };
  f32x4 acc[MT][F];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int f = 0; f < F; ++f) acc[a][f] = (f32x4){0.f, 0.f, 0.f, 0.f};
  bf16x8 A[kHB][MT];
  auto make_a = [&](int st) {
#pragma unroll
    for (int a = 0; a < MT; ++a) {
      const float step = step_of(sa[a] >> (16 * (st & 1) + 8 * (g >> 1)) & 0xffu);
      A[0][a] = unpack8(qa[a][0], qa[a][1], step);
      A[1][a] = unpack8(qa[a][2], qa[a][3], step);
    }
  };
  auto read_b = [&](int buf, int n) {
    const int h = n / F, f = wn * F + n % F;
    return *reinterpret_cast<const bf16x8*>(&Bs[buf][2 * g + h][f % 8 * Q + 16 * (f / 8) + i][0]);
  };
  // A stage's products, RING fragments read ahead
  auto multiply = [&](int buf) {
    __builtin_amdgcn_s_setprio(1);  // the products first
    bf16x8 B[RING];
#pragma unroll
    for (int n = 0; n < RING; ++n) B[n] = read_b(buf, n);
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
        acc[a][n % F] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[n / F][a], B[n % RING], acc[a][n % F], 0, 0, 0);
      if (n + RING < STEPS) B[n % RING] = read_b(buf, n + RING);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, RING, 0);  // LDS reads
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
      __builtin_amdgcn_sched_group_barrier(0x008, MT, 0);  // MFMAs
      if (n + RING < STEPS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  constexpr bool PAIR = WM * WN == 8;
  auto meet = [&]() {  // nothing of one side moves to the other
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  // The wave's way through the tile.  The first half multiplies stage st and then brings its part
  // of stage st + 1's B to LDS; the late half brings that part and multiplies stage st then.  So
  // B's buffer st + 1 is written after both halves' products of stage st - 1 and before theirs of
  // st + 1, and both meet equally often.
  auto walk = [&](auto half) {
    constexpr bool late = decltype(half)::value;
    if (stages > 0) {
      any_rows(0);
      any_packed(0);
      stage(0);
      if (!late) make_a(0);
    }
    if (stages > 1) {
      any_rows(1);
      if (!late) any_packed(1);
    }
    meet();
    int st = 0;
    for (; st + 2 < plain; ++st) {
      if (!late) multiply(st & 1);
      if (PAIR && !late) meet();
      stage(~st & 1);
      load_rows(st + 2);
      make_a(st + 1 - late);
      load_packed(st + 2 - late);
      if (late) meet();
      if (late) multiply(st & 1);
      meet();
    }
    for (; st < stages; ++st) {
      if (!late) multiply(st & 1);
      if (PAIR && !late) meet();
      if (st + 1 < stages) stage(~st & 1);
      if (st + 2 < stages) any_rows(st + 2);
      if (st + 1 - late < stages) make_a(st + 1 - late);
      if (st + 2 - late < stages) any_packed(st + 2 - late);
      if (late) meet();
      if (late) multiply(st & 1);
      meet();
    }
    float* out = c.out + id * c.ld + part * c.part;
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int ch = k0 + 16 * a + 4 * g + t;
        if (ch >= c.dim) continue;
#pragma unroll
        for (int f = 0; f < F; f += 4) {
          const int e = (wn * F + f) % 8, col = c0 + 8 * (16 * ((wn * F + f) / 8) + i) + e;
          float* p = out + (int64_t)ch * c.cols + col;
          if (col + 4 <= c.cols) {
            *reinterpret_cast<f32x4_any*>(p) = (f32x4){acc[a][f][t], acc[a][f + 1][t], acc[a][f + 2][t], acc[a][f + 3][t]};
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (col + k < c.cols) p[k] = acc[a][f + k][t];
          }
        }
      }
  };
  if constexpr (PAIR) {
    if (wave >= 4) return walk(std::true_type());
  }
  walk(std::false_type());
}

// The parts' sums in order.
__global__ void __launch_bounds__(256)
    k_act8_parts(const float* __restrict__ parts, int count, int64_t size, float* __restrict__ G, int64_t ld,
                 Groups groups) {
  const int64_t id = group_id(groups, blockIdx.y);
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < size; k += (int64_t)gridDim.x * 256) {
    const float* p = parts + id * count * size + k;
    float sum = p[0];
    for (int q = 1; q < count; ++q) sum += p[q * size];
    G[id * ld + k] = sum;
  }
}

template <int MT, int F, int WM, int WN>
void grad_launch(GradCall c, hipStream_t s) {
  using S = GradTile<MT, F, WM, WN>;
  c.tm = (int32_t)ceil_div(c.dim, S::BM);
  c.tn = (int32_t)ceil_div(c.cols, S::BN);
  c.items = c.tm * c.tn * c.parts * c.groups.count;
  hipLaunchKernelGGL((k_act8_grad<MT, F, WM, WN>), dim3(8 * (unsigned)ceil_div(c.items, 8)),
                     dim3(S::kThreads), 0, s, c);
}

template <typename T>
nbsgd_status pack_launch(const void* A, int64_t lda, int32_t Tn, int32_t dim, void* packed,
                         const Groups& g, hipStream_t s) {
  const Act8 lay = act8_layout(Tn, dim);
  const dim3 grid((unsigned)ceil_div(dim, 4 * PackTile<T>::CH), (unsigned)ceil_div(lay.blocks, 4), g.count);
  hipLaunchKernelGGL(k_act8_pack<T>, grid, dim3(256), 0, s, static_cast<const T*>(A), lda, Tn, dim,
                     static_cast<uint8_t*>(packed), lay, g);
  return launched("nbsgd_act_pack");
}

template <typename T>
nbsgd_status unpack_launch(const void* packed, int32_t Tn, int32_t dim, void* A, int64_t lda,
                           const Groups& g, hipStream_t s) {
  const Act8 lay = act8_layout(Tn, dim);
  const dim3 grid((unsigned)ceil_div(dim, 4 * PackTile<T>::CH), (unsigned)ceil_div(lay.blocks, 4), g.count);
  const auto kernel = on_lines(A, lda * sizeof(T)) ? k_act8_unpack<T, true> : k_act8_unpack<T, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, static_cast<const uint8_t*>(packed), Tn, dim,
                     static_cast<T*>(A), lda, lay, g);
  return launched("nbsgd_act_unpack");
}

constexpr int64_t kMaxStride = 1 << 22;  // 64 rows of dY lie within 32-bit offsets

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
  if (nm * dim * out > (int64_t)1 << 36)
    return fail(NBSGD_E_UNSUPPORTED, "n*m*dim*out = %lld floats of G exceed 2^36",
                (long long)(nm * dim * out));
  if (ldy > kMaxStride)
    return fail(NBSGD_E_UNSUPPORTED, "rows of dY: stride %lld exceeds %lld", (long long)ldy,
                (long long)kMaxStride);
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
  GradCall c;
  c.packed = static_cast<const uint8_t*>(packed);
  c.dY = static_cast<const __bf16*>(dY);
  c.ldy = ldy;
  c.T = T;
  c.dim = dim;
  c.cols = out;
  c.border = act8_border(T, ldy);
  c.parts = act8_splits(T, dim, out);
  c.per = (int32_t)(ceil_div(ceil_div(lay.blocks, c.parts), 4) * 4);
  c.lay = lay;
  c.groups = g;
  const int64_t size = (int64_t)dim * out;
  float* ws = static_cast<float*>(workspace);
  c.out = c.parts > 1 ? ws : G;
  c.ld = c.parts > 1 ? c.parts * size : ld;
  c.part = size;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // Which tile a call takes: the one whose tiles cost least.  A stage of a tile takes a full card
  // 8.6 ns (256 x 256), 3.2 (128 x 128) or 1.8 (64 x 128), 475 : 175 : 100, and a card with fewer
  // tiles than `least` is not full: one large tile a CU is, one middle or small one is not.
  //   1 mini-batch of 4096 x 2048 x 2048   large 89 us, middle 74, small 67
  //   8 of 4096 x 1024 x 1024              93, 93, 111
  //   64 of 512 x 512 x 512                29, 34, 36
  //   40 of 750 x 43 x 2225                52, 41, 29
  //   64 of 2048 x 256 x 256 in two parts  44, 41, 45
  const int64_t each = (int64_t)c.parts * g.count;
  const auto cost = [&](int64_t rows, int64_t columns, int64_t price, int64_t least) {
    return price * std::max(each * ceil_div(dim, rows) * ceil_div(out, columns), least);
  };
  const int64_t large = cost(256, 256, 475, 256), middle = cost(128, 128, 175, 362), small = cost(64, 128, 100, 416);
  if (large <= middle && large <= small) grad_launch<2, 16, 8, 1>(c, s);
  else if (middle <= small) grad_launch<4, 4, 2, 2>(c, s);
  else grad_launch<2, 4, 2, 2>(c, s);
  if (c.parts > 1)
    hipLaunchKernelGGL(k_act8_parts, dim3((unsigned)std::min<int64_t>(ceil_div(size, 256), 1024), g.count),
                       dim3(256), 0, s, ws, c.parts, size, G, ld, g);
  return launched("nbsgd_act_grad");
}
