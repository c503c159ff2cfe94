// Gated linear recurrence over long sequences and its backward pass (gfx950):
//   a_t = sigmoid(g_t + bias), h_t = a_t h_{t-1} + (1 - a_t) x_t, a state a channel.
//
// A token is the map h -> a h + b, and maps compose: (A, B) after (A', B') is
// (A A', A B' + B).  So a sequence is walked in tiles of 256 tokens x 128 bytes of channels by one
// workgroup, a wave 32 tokens of a tile and a lane 16 bytes of channels x a run of tokens:
//   1. each lane composes its run, the wave its lanes (shuffles) and the workgroup its
//      waves (LDS, one barrier a tile);
//   2. the state at the tile's start then gives every lane the state at its own, from
//      which it walks its run once more in registers.
// x and g cross HBM once, h once.  The next tile's rows are loaded before this tile's
// arithmetic.  The state goes from tile to tile as fma(A, h, B) of the tile's composition
// alone, so it does not depend on how tiles are dealt to workgroups.  Backward, the
// gradient mu_t = a_t (dh_t + mu_{t+1}) is the same kind of map from the last token to the
// first; the states inside a tile are recomputed from the one kept at its start.
#include <algorithm>

#include "device_rows.h"

using namespace nbsgd;

namespace {

// Gate and complement of z, both accurate where they are small (1 - a would cancel).
struct Gate {
  float a, rest;
};
// exp(-|z|) as 2^(z log2 e) on the hardware's exponential; EXACT adds what the product's and
// the constant's rounding lost (|z| 2^-24 of the value otherwise, below bf16's own step).
template <bool EXACT>
__device__ __forceinline__ Gate gate(float z) {
  const float y = -fabsf(z), kL = 1.44269502f, kLlo = 1.92596303e-8f;
  const float t = y * kL;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (EXACT) {
    // an infinite z has e = 0 already
    const float lost = fmaf(y, kLlo, fmaf(y, kL, -t)) * 0.693147181f;
    e = y > -200.f ? fmaf(e, lost, e) : e;
  }
  const float r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
  return z >= 0.f ? Gate{r, s} : Gate{s, r};
}
// The gate in one register: the smaller of the two, which keeps its accuracy, with z's sign.
// The other is at least 1/2, so that 1 - s is it to half a step.
template <bool EXACT>
__device__ __forceinline__ float fold_gate(float z) {
  const Gate q = gate<EXACT>(-fabsf(z));
  return __builtin_copysignf(q.a, z);
}
__device__ __forceinline__ Gate unfold_gate(float q) {
  const float s = fabsf(q), r = 1.f - s;
  return __builtin_bit_cast(int32_t, q) >= 0 ? Gate{r, s} : Gate{s, r};
}

// What both passes are told of a call.
struct Call {
  const void *x, *g;
  const float* bias;       // learner 0's, or null
  const int32_t* lengths;  // or null
  int64_t ldx, ld;
  int32_t batch, T, dim, tiles;
  int32_t chunk;           // tiles of a workgroup
  Groups groups;
};

// Lanes of a wave over a tile's part: eight lanes hold the CH channels of a token (128 bytes,
// one cache line), eight such sets take K consecutive tokens each.
template <typename T>
struct Lanes {
  static constexpr int V = Elem<T>::V, LV = 8, CH = LV * V, SUBS = 64 / LV, K = 32 / SUBS;
};

struct Where {
  int id, col, chunk;  // mini-batch, first channel, tiles chunk .. of the sequence
  int64_t seq;
  int len;
};
template <int CH>
__device__ __forceinline__ Where locate(const Call& c, int block) {
  Where w;
  const int cols = (c.dim + CH - 1) / CH, chunks = (c.tiles + c.chunk - 1) / c.chunk;
  w.col = block % cols * CH;
  const int r = block / cols;
  w.chunk = r % chunks;
  const int e = r / chunks;
  w.id = group_id(c.groups, e / c.batch);
  w.seq = (int64_t)w.id * c.batch + e % c.batch;
  w.len = c.lengths ? min(max(c.lengths[w.seq], 0), c.T) : c.T;
  return w;
}

// Rows of a tile: a uniform base and 32-bit lane offsets (kMaxStride keeps a tile in them),
// which leaves a load one address register where 64-bit row pointers took two each.
template <typename T>
__device__ __forceinline__ const T* row_at(const T* base, uint32_t bytes) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes);
}
template <typename T>
__device__ __forceinline__ T* row_at(T* base, uint32_t bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes);
}
// Bounds how far the scheduler mixes a run's steps: with all of them under way at once the
// registers spill.
__device__ __forceinline__ void step_fence() { __builtin_amdgcn_sched_barrier(0); }
// Keeps the compiler from holding on to what it derived from v: deriving it again is cheaper
// than the registers.
__device__ __forceinline__ float again(float v) {
  asm("" : "+v"(v));
  return v;
}
__device__ __forceinline__ u32x4 again(u32x4 v) {
  asm("" : "+v"(v));
  return v;
}

// The lane's V biases.
template <int V>
__device__ __forceinline__ void load_bias(const Call& c, const Where& w, int ch, float (&bias)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    bias[v] = c.bias && ch + v < c.dim ? c.bias[(int64_t)(w.id / c.groups.m) * c.ld + ch + v] : 0.f;
}

// The lane's rows of one operand, `off` bytes from the tile's first; of them `live` are taken,
// the others are zeros.  WHOLE (a row is a whole number of 16 bytes): without branches, lanes
// without a row or a channel read the tile's first 16 bytes instead; the branches for the
// parts of 16 bytes cost 7,000 instructions and the registers of their addresses.
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_run(const T* base, const uint32_t (&off)[Lanes<T>::K], int live,
                                         int n, u32x4 (&r)[Lanes<T>::K]) {
#pragma unroll
  for (int k = 0; k < Lanes<T>::K; ++k) {
    const bool ok = n > 0 && k < live;
    if constexpr (WHOLE) {
      const u32x4 v = *reinterpret_cast<const u32x4_any*>(row_at(base, ok ? off[k] : 0u));
#pragma unroll
      for (int q = 0; q < 4; ++q) r[k][q] = ok ? v[q] : 0u;
    } else {
      r[k] = ok ? load16<T>(row_at(base, off[k]), n) : (u32x4){0u, 0u, 0u, 0u};
    }
  }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_row(T* p, u32x4 r, int n) {
  if constexpr (WHOLE) *reinterpret_cast<u32x4_any*>(p) = r;
  else store16<T>(p, r, n);
}

// Inclusive composition of the maps (A, B) over the SUBS lane sets, first to last or last to
// first, and the exclusive one (what comes before the lane) in EA, EB.
template <typename T, bool UP>
__device__ __forceinline__ void compose(int sub, float (&A)[Lanes<T>::V], float (&B)[Lanes<T>::V],
                                        float (&EA)[Lanes<T>::V], float (&EB)[Lanes<T>::V]) {
  constexpr int V = Lanes<T>::V, LV = Lanes<T>::LV, SUBS = Lanes<T>::SUBS;
#pragma unroll
  for (int d = 1; d < SUBS; d *= 2) {
    const bool take = UP ? sub >= d : sub < SUBS - d;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float pa = UP ? __shfl_up(A[v], d * LV) : __shfl_down(A[v], d * LV);
      const float pb = UP ? __shfl_up(B[v], d * LV) : __shfl_down(B[v], d * LV);
      B[v] = take ? fmaf(A[v], pb, B[v]) : B[v];
      A[v] = take ? A[v] * pa : A[v];
    }
    step_fence();
  }
  const bool first = UP ? sub == 0 : sub == SUBS - 1;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float pa = UP ? __shfl_up(A[v], LV) : __shfl_down(A[v], LV);
    const float pb = UP ? __shfl_up(B[v], LV) : __shfl_down(B[v], LV);
    EA[v] = first ? 1.f : pa;
    EB[v] = first ? 0.f : pb;
  }
}

// V consecutive floats between a lane and LDS.
template <int V>
__device__ __forceinline__ void to_lds(float* p, const float (&v)[V]) {
#pragma unroll
  for (int q = 0; q < V / 4; ++q)
    reinterpret_cast<f32x4*>(p)[q] = (f32x4){v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
}
template <int V>
__device__ __forceinline__ void from_lds(const float* p, float (&v)[V]) {
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    const f32x4 r = reinterpret_cast<const f32x4*>(p)[q];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * q + k] = r[k];
  }
}
// Orders the wave's LDS writes before its later reads of other lanes' data.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Forward.  PAIRS: only each tile's composition, to `pairs` (the first of the three kernels
// that split a sequence over workgroups); otherwise the states, from `carry` (the state at the
// start of every tile) where the sequence is split, else from h0.
template <typename T, bool PAIRS, bool WHOLE>
__global__ void __launch_bounds__(64 * kScanWaves, 2)
    k_scan(Call c, const float* __restrict__ h0, const float* __restrict__ carry,
           float* __restrict__ pairs, T* __restrict__ h, int64_t ldh, float* __restrict__ h_last,
           float* __restrict__ states) {
  using L = Lanes<T>;
  constexpr int V = L::V, K = L::K, CH = L::CH;
  __shared__ __attribute__((aligned(16))) float tot[2][2][kScanWaves][CH];
  __shared__ __attribute__((aligned(16))) float start[kScanWaves][CH];
  const Where w = locate<CH>(c, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int o = lane % L::LV * V, sub = lane / L::LV;
  const int n = c.dim - (w.col + o);  // channels from the lane's first
  // the channel whose state this lane carries (twice over where a line has 32), and
  // whether it is the one that stores it
  const int oc = lane & (CH - 1), own = w.col + oc;
  const bool keeper = wave == 0 && lane < CH && own < c.dim;
  const int64_t row0 = w.seq * c.T;
  const T* x = static_cast<const T*>(c.x) + row0 * c.ldx + w.col;
  const T* g = static_cast<const T*>(c.g) + row0 * c.ldx + w.col;
  T* out0 = h + row0 * ldh + w.col;
  float bias[V];
  load_bias<V>(c, w, w.col + o, bias);
  const int tile0 = w.chunk * c.chunk, tile1 = min(tile0 + c.chunk, c.tiles);
  float s = 0.f;
  if (!PAIRS && own < c.dim) {
    if (carry) s = carry[(w.seq * c.tiles + tile0) * c.dim + own];
    else if (h0) s = h0[w.seq * c.dim + own];
  }
  const int at = 32 * wave + sub * K;  // the lane's first token of a tile
  uint32_t ix[K], ih[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    ix[k] = (uint32_t)((at + k) * (int)c.ldx + o) * (uint32_t)sizeof(T);
    ih[k] = (uint32_t)((at + k) * (int)ldh + o) * (uint32_t)sizeof(T);
  }
  u32x4 rx[K], rg[K];
  auto load_tile = [&](int tile) {
    const int t = tile * kScanTile;
    load_run<T, WHOLE>(x + t * c.ldx, ix, w.len - t - at, n, rx);
    load_run<T, WHOLE>(g + t * c.ldx, ix, w.len - t - at, n, rg);
  };
  load_tile(tile0);
  for (int tile = tile0; tile < tile1; ++tile) {
    const int t = tile * kScanTile + at, buf = tile & 1;
    float q[K][V], A[V], B[V];  // gates, folded; 0 (a = 1) past the length
    u32x4 cx[K];                // this tile's x
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, B[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float xv[V], gv[V];
      cx[k] = rx[k];
      Elem<T>::expand(cx[k], xv);
      Elem<T>::expand(rg[k], gv);
      const bool live = t + k < w.len;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        q[k][v] = live ? fold_gate<sizeof(T) == 4>(gv[v] + bias[v]) : 0.f;
        const Gate u = unfold_gate(q[k][v]);
        B[v] = fmaf(u.a, B[v], u.rest * xv[v]);
        A[v] *= u.a;
      }
      step_fence();
    }
    if (tile + 1 < tile1) load_tile(tile + 1);
    float EA[V], EB[V];
    compose<T, true>(sub, A, B, EA, EB);
    if (sub == L::SUBS - 1) {
      to_lds<V>(&tot[buf][0][wave][o], A);
      to_lds<V>(&tot[buf][1][wave][o], B);
    }
    __syncthreads();
    float TA = 1.f, TB = 0.f, mine = 0.f;
    for (int y = 0; y < waves; ++y) {
      if (y == wave) mine = fmaf(TA, s, TB);
      const float qa = tot[buf][0][y][oc], qb = tot[buf][1][y][oc];
      TB = fmaf(qa, TB, qb);
      TA *= qa;
    }
    if constexpr (PAIRS) {
      if (keeper) {
        const int64_t cell = (w.seq * c.tiles + tile) * c.dim + own;
        *reinterpret_cast<f32x2*>(pairs + 2 * cell) = (f32x2){TA, TB};
      }
      continue;
    }
    if (states && keeper) states[(w.seq * c.tiles + tile) * c.dim + own] = s;
    s = fmaf(TA, s, TB);
    start[wave][oc] = mine;
    wave_fence();
    float hv[V];
    from_lds<V>(&start[wave][o], hv);
    wave_fence();
#pragma unroll
    for (int v = 0; v < V; ++v) hv[v] = fmaf(EA[v], hv[v], EB[v]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float out[V], xv[V];
      Elem<T>::expand(again(cx[k]), xv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate u = unfold_gate(again(q[k][v]));
        hv[v] = fmaf(u.a, hv[v], u.rest * xv[v]);
        out[v] = t + k < w.len ? hv[v] : 0.f;
      }
      if (n > 0 && t + k < c.T)
        store_row<T, WHOLE>(row_at(out0 + tile * kScanTile * ldh, ih[k]), Elem<T>::collapse(out), n);
      step_fence();
    }
  }
  if (!PAIRS && h_last && tile1 == c.tiles && keeper) h_last[w.seq * c.dim + own] = s;
}

// State (or gradient, REVERSE) at the start of every tile of a split sequence, from the tiles'
// compositions.  A channel a thread.
template <bool REVERSE>
__global__ void __launch_bounds__(64)
    k_scan_carry(Call c, const float* __restrict__ pairs, const float* __restrict__ first,
                 float* __restrict__ carry) {
  const int cols = (c.dim + 63) / 64, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 64 + threadIdx.x;
  if (ch >= c.dim) return;
  const int64_t seq = (int64_t)group_id(c.groups, e / c.batch) * c.batch + e % c.batch;
  const f32x2* p = reinterpret_cast<const f32x2*>(pairs) + seq * c.tiles * c.dim + ch;
  float* out = carry + seq * c.tiles * c.dim + ch;
  float s = first ? first[seq * c.dim + ch] : 0.f;
  constexpr int U = 8;  // loads under way
  for (int k0 = 0; k0 < c.tiles; k0 += U) {
    f32x2 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + u, c.tiles - 1);
      q[u] = p[(int64_t)(REVERSE ? c.tiles - 1 - k : k) * c.dim];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u >= c.tiles) break;
      out[(int64_t)(REVERSE ? c.tiles - 1 - k0 - u : k0 + u) * c.dim] = s;
      s = fmaf(q[u][0], s, q[u][1]);
    }
  }
}

// Backward, tiles from the last to the first; PAIRS and carry as in k_scan, for mu.
template <typename T, bool PAIRS, bool WHOLE>
__global__ void __launch_bounds__(64 * kScanWaves, 2)
    k_scan_grad(Call c, const float* __restrict__ states, const T* __restrict__ dh, int64_t lddh,
                const float* __restrict__ dh_last, const float* __restrict__ carry,
                float* __restrict__ pairs, T* __restrict__ dx, T* __restrict__ dg,
                float* __restrict__ dh0, float* __restrict__ part) {
  using L = Lanes<T>;
  constexpr int V = L::V, K = L::K, CH = L::CH;
  __shared__ __attribute__((aligned(16))) float tot[2][4][kScanWaves][CH];
  __shared__ __attribute__((aligned(16))) float start[kScanWaves][2][CH];
  const Where w = locate<CH>(c, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int o = lane % L::LV * V, sub = lane / L::LV;
  const int n = c.dim - (w.col + o);
  const int oc = lane & (CH - 1), own = w.col + oc;
  const bool keeper = wave == 0 && lane < CH && own < c.dim;
  const int64_t row0 = w.seq * c.T;
  const T* x = static_cast<const T*>(c.x) + row0 * c.ldx + w.col;
  const T* g = static_cast<const T*>(c.g) + row0 * c.ldx + w.col;
  const T* d = dh + row0 * lddh + w.col;
  T *dx0 = dx + row0 * c.ldx + w.col, *dg0 = dg + row0 * c.ldx + w.col;
  float bias[V];
  load_bias<V>(c, w, w.col + o, bias);
  const int tile0 = w.chunk * c.chunk, tile1 = min(tile0 + c.chunk, c.tiles);
  float mu = 0.f;
  if (!PAIRS && own < c.dim) {
    if (carry) mu = carry[(w.seq * c.tiles + tile1 - 1) * c.dim + own];
    else if (dh_last) mu = dh_last[w.seq * c.dim + own];
  }
  const int at = 32 * wave + sub * K;
  uint32_t ix[K], id[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    ix[k] = (uint32_t)((at + k) * (int)c.ldx + o) * (uint32_t)sizeof(T);
    id[k] = (uint32_t)((at + k) * (int)lddh + o) * (uint32_t)sizeof(T);
  }
  u32x4 rx[K], rg[K], rd[K];
  float s = 0.f;
  auto load_tile = [&](int tile) {
    const int t = tile * kScanTile;
    if constexpr (!PAIRS) {
      load_run<T, WHOLE>(x + t * c.ldx, ix, w.len - t - at, n, rx);
      s = own < c.dim ? states[(w.seq * c.tiles + tile) * c.dim + own] : 0.f;
    }
    load_run<T, WHOLE>(g + t * c.ldx, ix, w.len - t - at, n, rg);
    load_run<T, WHOLE>(d + t * lddh, id, w.len - t - at, n, rd);
  };
  load_tile(tile1 - 1);
  for (int tile = tile1 - 1; tile >= tile0; --tile) {
    const int t = tile * kScanTile + at, buf = tile & 1;
    float q[K][V], A[V], B[V], RA[V], R[V];
    u32x4 cx[K], cd[K];  // this tile's x and dh, as they came
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, B[v] = R[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gv[V], xv[V];
      Elem<T>::expand(rg[k], gv);
      cd[k] = rd[k];
      if constexpr (!PAIRS) {
        cx[k] = rx[k];
        Elem<T>::expand(cx[k], xv);
      }
      const bool live = t + k < w.len;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        q[k][v] = live ? fold_gate<sizeof(T) == 4>(gv[v] + bias[v]) : 0.f;
        const Gate u = unfold_gate(q[k][v]);
        if constexpr (!PAIRS) B[v] = fmaf(u.a, B[v], u.rest * xv[v]);
        A[v] *= u.a;
      }
      step_fence();
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      float dv[V];
      Elem<T>::expand(again(cd[k]), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) R[v] = unfold_gate(again(q[k][v])).a * (dv[v] + R[v]);
      step_fence();
    }
    const float here = s;
    if (tile > tile0) load_tile(tile - 1);
#pragma unroll
    for (int v = 0; v < V; ++v) RA[v] = A[v];
    float EA[V], EB[V], FA[V], FR[V];
    compose<T, false>(sub, RA, R, FA, FR);
    if (sub == 0) {
      to_lds<V>(&tot[buf][0][wave][o], RA);
      to_lds<V>(&tot[buf][1][wave][o], R);
    }
    if constexpr (!PAIRS) {
      compose<T, true>(sub, A, B, EA, EB);
      if (sub == L::SUBS - 1) {
        to_lds<V>(&tot[buf][2][wave][o], A);
        to_lds<V>(&tot[buf][3][wave][o], B);
      }
    }
    __syncthreads();
    float TA = 1.f, TR = 0.f, mine = 0.f;
    for (int y = waves - 1; y >= 0; --y) {
      if (y == wave) mine = fmaf(TA, mu, TR);
      const float qa = tot[buf][0][y][oc], qr = tot[buf][1][y][oc];
      TR = fmaf(qa, TR, qr);
      TA *= qa;
    }
    if constexpr (PAIRS) {
      if (keeper) {
        const int64_t cell = (w.seq * c.tiles + tile) * c.dim + own;
        *reinterpret_cast<f32x2*>(pairs + 2 * cell) = (f32x2){TA, TR};
      }
      continue;
    }
    float PA = 1.f, PB = 0.f;
    for (int y = 0; y < wave; ++y) {
      const float qa = tot[buf][2][y][oc];
      PB = fmaf(qa, PB, tot[buf][3][y][oc]);
      PA *= qa;
    }
    mu = fmaf(TA, mu, TR);
    start[wave][0][oc] = fmaf(PA, here, PB);
    start[wave][1][oc] = mine;
    wave_fence();
    float hv[V], m[V], sum[V], gap[K][V];
    from_lds<V>(&start[wave][0][o], hv);
    from_lds<V>(&start[wave][1][o], m);
    wave_fence();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      hv[v] = fmaf(EA[v], hv[v], EB[v]);
      m[v] = fmaf(FA[v], m[v], FR[v]);
      sum[v] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float xv[V];
      Elem<T>::expand(again(cx[k]), xv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate u = unfold_gate(again(q[k][v]));
        gap[k][v] = hv[v] - xv[v];
        hv[v] = fmaf(u.a, hv[v], u.rest * xv[v]);
      }
      step_fence();
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      float ox[V], og[V], dv[V];
      Elem<T>::expand(again(cd[k]), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float lam = dv[v] + m[v];
        const Gate u = unfold_gate(again(q[k][v]));
        ox[v] = lam * u.rest;
        og[v] = ox[v] * u.a * gap[k][v];
        if (t + k >= w.len) ox[v] = og[v] = 0.f;
        sum[v] += og[v];
        m[v] = u.a * lam;
      }
      step_fence();
      if (n > 0 && t + k < c.T) {
        store_row<T, WHOLE>(row_at(dx0 + tile * kScanTile * c.ldx, ix[k]), Elem<T>::collapse(ox), n);
        store_row<T, WHOLE>(row_at(dg0 + tile * kScanTile * c.ldx, ix[k]), Elem<T>::collapse(og), n);
      }
    }
    if (part) {
#pragma unroll
      for (int dist = 1; dist < L::SUBS; dist *= 2)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += __shfl_xor(sum[v], dist * L::LV);
      if (sub == 0 && n > 0) {
        float* p = part + ((w.seq * c.tiles + tile) * waves + wave) * c.dim + w.col + o;
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v < n) p[v] = sum[v];
      }
    }
  }
  if (!PAIRS && dh0 && tile0 == 0 && keeper) dh0[w.seq * c.dim + own] = mu;
}

// Sequences of at most kShort tokens (a served step above all), a channel a thread: the tile
// kernels would leave most of their waves idle.
constexpr int kShort = 16;
template <typename T>
__global__ void __launch_bounds__(256)
    k_scan_short(Call c, const float* __restrict__ h0, T* __restrict__ h, int64_t ldh,
                 float* __restrict__ h_last, float* __restrict__ states) {
  const int cols = (c.dim + 255) / 256, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 256 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = c.bias ? c.bias[(int64_t)(id / c.groups.m) * c.ld + ch] : 0.f;
  const int len = c.lengths ? min(max(c.lengths[seq], 0), c.T) : c.T;
  const T* x = static_cast<const T*>(c.x) + seq * c.T * c.ldx + ch;
  const T* g = static_cast<const T*>(c.g) + seq * c.T * c.ldx + ch;
  float s = h0 ? h0[seq * c.dim + ch] : 0.f;
  if (states && c.T) states[seq * c.dim + ch] = s;
  for (int t = 0; t < c.T; ++t) {
    if (t < len) {
      const Gate q = gate<sizeof(T) == 4>(Elem<T>::load(g + t * c.ldx) + bias);
      s = fmaf(q.a, s, q.rest * Elem<T>::load(x + t * c.ldx));
    }
    Elem<T>::store(h + (seq * c.T + t) * ldh + ch, t < len ? s : 0.f);
  }
  if (h_last) h_last[seq * c.dim + ch] = s;
}

template <typename T>
__global__ void __launch_bounds__(256)
    k_scan_grad_short(Call c, const float* __restrict__ states, const T* __restrict__ dh,
                      int64_t lddh, const float* __restrict__ dh_last, T* __restrict__ dx,
                      T* __restrict__ dg, float* __restrict__ dh0, float* __restrict__ part) {
  const int cols = (c.dim + 255) / 256, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 256 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = c.bias ? c.bias[(int64_t)(id / c.groups.m) * c.ld + ch] : 0.f;
  const int len = c.lengths ? min(max(c.lengths[seq], 0), c.T) : c.T;
  const int64_t row0 = seq * c.T * c.ldx + ch;
  const T *x = static_cast<const T*>(c.x) + row0, *g = static_cast<const T*>(c.g) + row0;
  float mu = dh_last ? dh_last[seq * c.dim + ch] : 0.f, sum = 0.f;
  float before[kShort];
  float s = c.T ? states[seq * c.dim + ch] : 0.f;
#pragma unroll
  for (int t = 0; t < kShort; ++t) {
    before[t] = s;
    if (t < len) {
      const Gate q = gate<sizeof(T) == 4>(Elem<T>::load(g + t * c.ldx) + bias);
      s = fmaf(q.a, s, q.rest * Elem<T>::load(x + t * c.ldx));
    }
  }
#pragma unroll
  for (int t = kShort - 1; t >= 0; --t) {
    if (t >= c.T) continue;
    float vx = 0.f, vg = 0.f;
    if (t < len) {
      const Gate q = gate<sizeof(T) == 4>(Elem<T>::load(g + t * c.ldx) + bias);
      const float lam = Elem<T>::load(dh + (seq * c.T + t) * lddh + ch) + mu;
      vx = lam * q.rest;
      vg = vx * q.a * (before[t] - Elem<T>::load(x + t * c.ldx));
      mu = q.a * lam;
    }
    sum += vg;
    Elem<T>::store(dx + row0 + t * c.ldx, vx);
    Elem<T>::store(dg + row0 + t * c.ldx, vg);
  }
  if (part) part[seq * c.dim + ch] = sum;
  if (dh0) dh0[seq * c.dim + ch] = mu;
}

// Bias gradient of a mini-batch: its `rows` partial sums, every 16th by one wave, then the
// waves' sums in order.
__global__ void __launch_bounds__(1024)
    k_scan_bias(const float* __restrict__ part, int64_t rows, int dim, float* __restrict__ G,
                int64_t ld, Groups groups) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ch = blockIdx.x * 64 + lane;
  const int id = group_id(groups, blockIdx.y);
  const float* p = part + id * rows * dim + min(ch, dim - 1);
  float sum = 0.f;
#pragma unroll 4
  for (int64_t r = wave; r < rows; r += 16) sum += p[r * dim];
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave || ch >= dim) return;
  sum = 0.f;
  for (int q = 0; q < 16; ++q) sum += sums[q][lane];
  G[(int64_t)id * ld + ch] = sum;
}

// How a call's sequences are dealt: waves of a workgroup (fewer than eight only where a
// sequence is shorter than a tile), and tiles of a workgroup.  With at least kEnough
// workgroups every sequence is walked by one, and everything crosses HBM once; fewer would
// leave CUs idle, so the tiles are dealt to about kSplit workgroups, which costs a pass over
// x and g for the tiles' compositions first.
constexpr int kEnough = 512, kSplit = 1024;
struct Deal {
  int waves, chunk, chunks;
  int64_t cols, seqs;
};
Deal deal(const Call& c, int channels) {
  Deal d;
  d.cols = ceil_div(c.dim, channels);
  d.seqs = (int64_t)c.groups.count * c.batch;
  d.waves = (int)std::min<int64_t>(kScanWaves, ceil_div(c.T, 32));
  const int64_t walkers = d.cols * d.seqs;
  d.chunk = c.tiles;
  if (walkers < kEnough && c.tiles > 1)
    d.chunk = (int)std::max<int64_t>(1, ceil_div(walkers * c.tiles, kSplit));
  d.chunks = (int)ceil_div(c.tiles, d.chunk);
  return d;
}

// Checks one operand's rows; 256 of them have to lie within 32-bit byte offsets.
constexpr int64_t kMaxStride = 1 << 22;
nbsgd_status check_operand(const char* name, const void* p, int64_t rows, int64_t dim, int64_t ld,
                           int e) {
  if (ld > kMaxStride)
    return fail(NBSGD_E_UNSUPPORTED, "rows of %s: stride %lld exceeds %lld", name, (long long)ld,
                (long long)kMaxStride);
  return check_rows(name, p, rows, dim, ld, e);
}

nbsgd_status fill_call(Call* c, const void* x, const void* g, int64_t ldx, int32_t n, int32_t m,
                       int32_t batch, int32_t Tn, int32_t dim, const float* bias, int64_t ld,
                       const int32_t* lengths, const uint8_t* mask) {
  c->x = x;
  c->g = g;
  c->bias = bias;
  c->lengths = lengths;
  c->ldx = ldx;
  c->ld = ld;
  c->batch = batch;
  c->T = Tn;
  c->dim = dim;
  c->tiles = (int32_t)ceil_div(Tn, kScanTile);
  c->chunk = c->tiles;
  return check_groups(n, m, mask, &c->groups);
}

template <typename T, bool WHOLE>
nbsgd_status scan_forward(Call& c, const ScanSpace& w, const float* h0, void* h, int64_t ldh,
                          float* h_last, float* states, void* ws, hipStream_t s) {
  if (!c.groups.count) return NBSGD_OK;
  T* out = static_cast<T*>(h);
  const int64_t seqs = (int64_t)c.groups.count * c.batch;
  if (c.T <= kShort) {
    hipLaunchKernelGGL(k_scan_short<T>, dim3((unsigned)(ceil_div(c.dim, 256) * seqs)), dim3(256), 0, s,
                       c, h0, out, ldh, h_last, states);
    return launched("nbsgd_scan");
  }
  const Deal d = deal(c, Lanes<T>::CH);
  c.chunk = d.chunk;
  const dim3 grid((unsigned)(d.cols * d.seqs * d.chunks)), block(64 * d.waves);
  float* carry = nullptr;
  if (d.chunks > 1) {
    float* pairs = reinterpret_cast<float*>(static_cast<char*>(ws) + w.pairs);
    carry = reinterpret_cast<float*>(static_cast<char*>(ws) + w.carry);
    hipLaunchKernelGGL((k_scan<T, true, WHOLE>), grid, block, 0, s, c, h0, nullptr, pairs, out, ldh, nullptr,
                       nullptr);
    hipLaunchKernelGGL(k_scan_carry<false>, dim3((unsigned)(ceil_div(c.dim, 64) * d.seqs)), dim3(64), 0, s, c, pairs,
                       h0, carry);
  }
  hipLaunchKernelGGL((k_scan<T, false, WHOLE>), grid, block, 0, s, c, h0, carry, nullptr, out, ldh, h_last,
                     states);
  return launched("nbsgd_scan");
}

template <typename T, bool WHOLE>
nbsgd_status scan_backward(Call& c, const ScanSpace& w, const float* states, const void* dh,
                           int64_t lddh, const float* dh_last, void* dx, void* dg, float* dh0,
                           float* Gbias, int64_t ld, void* ws, hipStream_t s) {
  if (!c.groups.count) return NBSGD_OK;
  const T* d_in = static_cast<const T*>(dh);
  T *ox = static_cast<T*>(dx), *og = static_cast<T*>(dg);
  const int64_t seqs = (int64_t)c.groups.count * c.batch;
  float* part = Gbias ? reinterpret_cast<float*>(static_cast<char*>(ws) + w.bias) : nullptr;
  int64_t rows = c.batch;  // partial sums of a mini-batch's bias gradient
  if (c.T <= kShort) {
    if (!c.T) rows = 0;
    hipLaunchKernelGGL(k_scan_grad_short<T>, dim3((unsigned)(ceil_div(c.dim, 256) * seqs)), dim3(256), 0,
                       s, c, states, d_in, lddh, dh_last, ox, og, dh0, c.T ? part : nullptr);
  } else {
    const Deal d = deal(c, Lanes<T>::CH);
    c.chunk = d.chunk;
    rows *= (int64_t)c.tiles * d.waves;
    const dim3 grid((unsigned)(d.cols * d.seqs * d.chunks)), block(64 * d.waves);
    float* carry = nullptr;
    if (d.chunks > 1) {
      float* pairs = reinterpret_cast<float*>(static_cast<char*>(ws) + w.pairs);
      carry = reinterpret_cast<float*>(static_cast<char*>(ws) + w.carry);
      hipLaunchKernelGGL((k_scan_grad<T, true, WHOLE>), grid, block, 0, s, c, states, d_in, lddh, dh_last,
                         nullptr, pairs, ox, og, nullptr, nullptr);
      hipLaunchKernelGGL(k_scan_carry<true>, dim3((unsigned)(ceil_div(c.dim, 64) * d.seqs)), dim3(64), 0, s, c, pairs,
                         dh_last, carry);
    }
    hipLaunchKernelGGL((k_scan_grad<T, false, WHOLE>), grid, block, 0, s, c, states, d_in, lddh, dh_last, carry,
                       nullptr, ox, og, dh0, part);
  }
  if (Gbias)
    hipLaunchKernelGGL(k_scan_bias, dim3((unsigned)ceil_div(c.dim, 64), c.groups.count), dim3(1024), 0,
                       s, part, rows, c.dim, Gbias, ld, c.groups);
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
  if (nbsgd_status st = check_operand("x", x, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_operand("g", g, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_operand("h", h, rows, dim, ldh, e)) return st;
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
  Call c;
  if (nbsgd_status st = fill_call(&c, x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask)) return st;
  const auto run = dtype == NBSGD_F32 ? (dim % 4 ? scan_forward<float, false> : scan_forward<float, true>)
                                      : (dim % 8 ? scan_forward<__bf16, false> : scan_forward<__bf16, true>);
  return run(c, w, h0, h, ldh, h_last, states, workspace, s);
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
  if (nbsgd_status st = check_operand("x", x, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_operand("g", g, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_operand("dh", dh, rows, dim, lddh, e)) return st;
  if (nbsgd_status st = check_operand("dx", dx, rows, dim, ldx, e)) return st;
  if (nbsgd_status st = check_operand("dg", dg, rows, dim, ldx, e)) return st;
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
  Call c;
  if (nbsgd_status st = fill_call(&c, x, g, ldx, n, m, batch, T, dim, bias, ld, lengths, mask)) return st;
  const auto run = dtype == NBSGD_F32 ? (dim % 4 ? scan_backward<float, false> : scan_backward<float, true>)
                                      : (dim % 8 ? scan_backward<__bf16, false> : scan_backward<__bf16, true>);
  return run(c, w, states, dh, lddh, dh_last, dx, dg, dh0, Gbias, ld, workspace, s);
}
