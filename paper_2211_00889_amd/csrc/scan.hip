// Gated linear recurrence over long sequences and its backward pass (gfx950):
//   a_t = sigmoid(g_t + bias), h_t = a_t h_{t-1} + (1 - a_t) x_t, a state a channel.
//
// A token is the map h -> a h + b, and maps compose: (A, B) after (A', B') is
// (A A', A B' + B).  So a sequence is walked in tiles of 256 tokens x 128 bytes of channels by one
// workgroup, a wave 32 tokens of a tile and a lane 8 bytes of channels x a run of 8 tokens:
//   1. each lane composes its run, the wave its lanes (shuffles) and the workgroup its
//      waves (LDS, one barrier a tile);
//   2. the state at the tile's start then gives every lane the state at its own, from
//      which it walks its run once more in registers.
// x and g cross HBM once, h once.  The next tile's rows are loaded before this tile's
// arithmetic.  The state goes from tile to tile as fma(A, h, B) of the tile's composition
// alone, so it does not depend on how tiles are dealt to workgroups.  Backward, the
// gradient mu_t = a_t (dh_t + mu_{t+1}) is the same kind of map from the last token to the
// first; the states inside a tile are recomputed from the one kept at its start.
// What bounds it is memory: backward, 36 mini-batches of four sequences of 2048 x 1024 bf16, 614 us
// (3.03 GB, 4.93 TB/s; a large copy reaches 4.72); forward, 1900 x 1000 fp32 with ragged lengths,
// rows off the lines, 336 us (1.27 GB, 1.39 moved, 4.13 TB/s of them); one sequence
// of 65536 x 2048 bf16, read twice, 268 us (1.34 GB, 5.01 TB/s).  Far from it are rows narrower than
// a wave's 128 bytes, whose other lanes idle (20 sequences of 21265 x 19 bf16: 73 us for 48 MB,
// backward 100 for 81), and few sequences of some thousand tokens, three launches after each other.
#include <algorithm>
#include <type_traits>

#include "device_rows.h"

using namespace nbsgd;

// A tile's composition is computed by k_scan_pairs in a call that splits its sequences and by k_scan or
// k_scan_grad in one that does not, and has to be the same bit for bit: the maps' products and sums
// stand in one order in both, and where one is fused is written out, not left to the compiler.
#pragma clang fp contract(off)

namespace {

// Gate a = sigmoid(z) and its complement, both accurate where they are small (1 - a would
// cancel): with e = exp(-|z|) the larger is 1 / (1 + e) and the smaller e / (1 + e).  e is
// 2^(-|z| log2 e) on the hardware's exponential; EXACT (fp32 rows) adds what the product's and
// the constant's rounding lost and refines the reciprocal.  Of bf16 rows the smaller one may be off by
// (1.25 |z| + 6) 2^-24 of its value, in h_last, states, dh0 and the bias's gradient too, which are
// fp32; the larger one is taken as 1 - e r, to half a step but for the smaller one's error: a long
// sequence keeps products of gates near 1, and with 1 / (1 + e) as the hardware has it dh0 of 17,384
// tokens was 8.6e-7 off, with this 2.2e-7.  36 mini-batches of four sequences of 2048 x 1024 backward
// took 652 us with EXACT for bf16 too, 620 with this, 617 with neither.
struct Gate {
  float a, rest;
};
template <bool EXACT>
__device__ __forceinline__ Gate gate(float z) {
  const float y = -fabsf(z), kL = 1.44269502f, kLlo = 1.92596303e-8f;
  const float t = y * kL;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (EXACT) {
    // below -200 e is 0 already, and t may be infinite
    const float lost = fmaf(y, kLlo, fmaf(y, kL, -t)) * 0.693147181f;
    e = y > -200.f ? fmaf(e, lost, e) : e;
  }
  const float d = 1.f + e;
  float r = __builtin_amdgcn_rcpf(d);
  if constexpr (EXACT) r = fmaf(fmaf(-d, r, 1.f), r, r);  // the reciprocal's last place
  const float s = e * r;
  if constexpr (!EXACT) r = fmaf(-e, r, 1.f);
  return z >= 0.f ? Gate{r, s} : Gate{s, r};
}

// What both passes are told of a call.
struct Call {
  const void *x, *g;
  const float* bias;       // learner 0's, or null
  const int32_t* lengths;  // or null
  int64_t ldx, ld;
  int32_t batch, T, dim, tiles;
  int32_t chunk;           // tiles of a workgroup
  int32_t items;           // workgroups with work
  Groups groups;
};

// Lanes of a wave over its 32 tokens of a tile: sixteen lanes hold the CH channels of a token
// (128 bytes, one cache line; 8 bytes and V channels a lane), four such sets take K
// consecutive tokens each.  (16 bytes a lane and eight sets of half the tokens took one more
// step of composition on twice the channels: with everything in flight the arithmetic, not
// memory, was the bound.)
template <typename T>
struct Lanes {
  static constexpr int V = 8 / sizeof(T), LV = 16, CH = LV * V, SUBS = 64 / LV, K = 32 / SUBS;
};

struct Where {
  int id, col, chunk;  // mini-batch, first channel, tiles chunk .. of the sequence
  int64_t seq;
  int len;
};
// Workgroup b runs on XCD b % 8: each XCD takes a run of neighbours, so that the column blocks of
// one row, whose lines they share where rows are not whole lines, go through one L2.  FLIP:
// in the reverse order.
template <int CH>
__device__ __forceinline__ Where locate(const Call& c, bool flip) {
  Where w;
  const int per = gridDim.x >> 3, i = blockIdx.x >> 3;
  const int block = (blockIdx.x & 7) * per + (flip ? per - 1 - i : i);
  w.seq = -1;
  if (block >= c.items) return w;
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

// A uniform base and a 32-bit lane offset (kMaxStride keeps it in range): one address register
// for all the rows of a run, whose bases are uniform too.
template <typename T>
__device__ __forceinline__ const T* row_at(const T* base, uint32_t bytes) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes);
}
template <typename T>
__device__ __forceinline__ T* row_at(T* base, uint32_t bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes);
}

// A channel's bias.  -inf becomes the lowest finite value (a is 0 all the same), so that the gate
// of a token past the length, whose g is taken as +inf, is 1 with every bias.
__device__ __forceinline__ float bias_at(const Call& c, int id, int ch) {
  const float b = c.bias && ch < c.dim ? c.bias[(int64_t)(id / c.groups.m) * c.ld + ch] : 0.f;
  return b == -__builtin_inff() ? -3.40282347e38f : b;
}
template <int V>
__device__ __forceinline__ void load_bias(const Call& c, const Where& w, int ch, float (&bias)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) bias[v] = bias_at(c, w.id, ch + v);
}

__device__ __forceinline__ void expand(u32x2 r, float (&v)[4]) {
  v[0] = bf16_lo(r[0]), v[1] = bf16_hi(r[0]), v[2] = bf16_lo(r[1]), v[3] = bf16_hi(r[1]);
}
__device__ __forceinline__ void expand(u32x2 r, float (&v)[2]) {
  const uint32_t a = r[0], b = r[1];
  v[0] = __builtin_bit_cast(float, a), v[1] = __builtin_bit_cast(float, b);
}
__device__ __forceinline__ u32x2 collapse(const float (&v)[4]) {
  return (u32x2){pack2(v[0], v[1]), pack2(v[2], v[3])};
}
__device__ __forceinline__ u32x2 collapse(const float (&v)[2]) {
  return (u32x2){__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1])};
}
// Keeps the compiler from holding on to what it made of r earlier (32 registers of fp32 for 16
// of bf16): making it again is cheaper than spilling.
__device__ __forceinline__ u32x2 again(u32x2 r) {
  asm("" : "+v"(r));
  return r;
}
template <typename T>
struct Word;
template <>
struct Word<float> {
  typedef uint32_t bits;
  static constexpr uint32_t kPast = 0x7f800000u;  // infinities
};
template <>
struct Word<__bf16> {
  typedef uint16_t bits;
  static constexpr uint32_t kPast = 0x7f807f80u;
};

// What the host has found of a call's rows:
//   kTiny   shorter than a lane's 8 bytes
//   kOdd    not a whole number of them: a row's last lane reads the row's last 8 bytes and shifts
//           (by elements its loads wait for each other: 48 sequences of 386 x 1527 bf16 77 -> 62
//           us, backward 134 -> 103; 20 of 21265 x 19 126 -> 72, 187 -> 99)
//   kWhole  a whole number
//   kLines  and those that are written lie on whole 128-byte lines: stores past the caches.  128
//           sequences of 1,024 x 1,024 bf16: 168 -> 163 us, backward 286 -> 277; with rows off the
//           lines they lose what the caches put together (192 of 2,048 x 1,000: 495 -> 614 us)
//   kFar    and those that are read, once and more than the memory-side cache keeps: loads past
//           the caches too (163 -> 157, 277 -> 273; 128 of 512: 81 -> 93)
enum Kind { kTiny, kOdd, kWhole, kLines, kFar };

// Where a lane with n channels left from its first, `o` into the block, reads: `col` elements from
// the base of the rows (taken kBack before the block's first channel), and the bits that it
// shifts away.  Lanes past the last channel read the block's first ones, or the row's last.
template <typename T, Kind KIND>
struct Reads {
  static constexpr int kBack = KIND == kOdd ? Lanes<T>::V : 0;
  uint32_t col;
  int shift, n;
  __device__ __forceinline__ Reads(int o, int n_) : n(n_) {
    const int skip = KIND == kOdd && n > 0 && n < Lanes<T>::V ? Lanes<T>::V - n : 0;
    col = kBack + (n > 0 ? o - skip : KIND == kOdd ? o + n - Lanes<T>::V : 0);
    shift = 8 * (int)sizeof(T) * skip;
  }
  // What is read as the lane's channels; where it is used, not where it is loaded, which would
  // wait for it.
  __device__ __forceinline__ u32x2 take(u32x2 r) const {
    if constexpr (KIND == kOdd) return __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, r) >> shift);
    return r;
  }
};
// The K rows from `base`, `ld` elements apart, of a lane `off` bytes into them: the first
// `live` are read (all of them in a FULL tile), the others are `past` in every word.
template <typename T, Kind KIND>
__device__ __forceinline__ void load_run(const T* base, int64_t ld, uint32_t off, bool full, int live,
                                         const Reads<T, KIND>& at, uint32_t past, u32x2 (&r)[Lanes<T>::K]) {
  constexpr int K = Lanes<T>::K, V = Lanes<T>::V;
  auto load = [&](int k) -> u32x2 {
    const T* p = row_at(base + k * ld, off);
    const u32x2_any* q = reinterpret_cast<const u32x2_any*>(p);
    if constexpr (KIND == kFar) return __builtin_nontemporal_load(q);
    if constexpr (KIND != kTiny) return *q;
    typedef typename Word<T>::bits bits;
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int v = 0; v < V; ++v)  // the last element over and over
      w[v * sizeof(T) / 4] |= (uint32_t)__builtin_bit_cast(bits, p[max(min(v, at.n - 1), 0)]) << (8 * (v * sizeof(T) % 4));
    return (u32x2){w[0], w[1]};
  };
  if (KIND != kTiny && full) {  // uniform
#pragma unroll
    for (int k = 0; k < K; ++k) r[k] = load(k);
    return;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    r[k] = (u32x2){past, past};
    if (k < live) r[k] = load(k);
  }
}
template <typename T, Kind KIND>
__device__ __forceinline__ void store_row(T* p, u32x2 r, int n) {
  constexpr int V = Lanes<T>::V;
  if (KIND >= kLines) {
    __builtin_nontemporal_store(r, reinterpret_cast<u32x2*>(p));
    return;
  }
  if (KIND >= kWhole || n >= V) {
    *reinterpret_cast<u32x2_any*>(p) = r;
    return;
  }
  typedef typename Word<T>::bits bits;
  const uint32_t w[2] = {r[0], r[1]};
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (v < n) p[v] = __builtin_bit_cast(T, (bits)(w[v * sizeof(T) / 4] >> (8 * (v * sizeof(T) % 4))));
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
  typedef float vec __attribute__((ext_vector_type(V)));
  vec r;
#pragma unroll
  for (int k = 0; k < V; ++k) r[k] = v[k];
  *reinterpret_cast<vec*>(p) = r;
}
template <int V>
__device__ __forceinline__ void from_lds(const float* p, float (&v)[V]) {
  typedef float vec __attribute__((ext_vector_type(V)));
  const vec r = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = r[k];
}
// Forward, from h0, or from `carry` (the state at the start of every tile) where the sequence is
// split over workgroups.
template <typename T, Kind KIND>
__global__ void __launch_bounds__(64 * kScanWaves, 2)
    k_scan(Call c, const float* h0, const float* __restrict__ carry, T* __restrict__ h, int64_t ldh,
           float* h_last,
           float* __restrict__ states) {
  using L = Lanes<T>;
  constexpr int V = L::V, K = L::K, CH = L::CH;
  __shared__ __attribute__((aligned(16))) float tot[2][2][kScanWaves][CH];
  __shared__ __attribute__((aligned(16))) float start[kScanWaves][CH];
  // a split sequence's tiles in the reverse of the order that their compositions were made in:
  // the last ones are in the memory-side cache still
  const Where w = locate<CH>(c, carry != nullptr);
  if (w.seq < 0) return;  // uniform
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int o = lane % L::LV * V, sub = lane / L::LV;
  const int n = c.dim - (w.col + o);  // channels from the lane's first
  // the channel whose state this lane carries (twice over where a line has 32), and
  // whether it is the one that stores it
  const int oc = lane & (CH - 1), own = w.col + oc;
  const bool keeper = wave == 0 && lane < CH && own < c.dim;
  const int64_t row0 = w.seq * c.T;
  const Reads<T, KIND> in(o, n);
  const T* x = static_cast<const T*>(c.x) + row0 * c.ldx + w.col - in.kBack;
  const T* g = static_cast<const T*>(c.g) + row0 * c.ldx + w.col - in.kBack;
  T* out0 = h + row0 * ldh + w.col;
  float bias[V];
  load_bias<V>(c, w, w.col + o, bias);
  const int tile0 = w.chunk * c.chunk, tile1 = min(tile0 + c.chunk, c.tiles);
  float s = 0.f;
  if (own < c.dim) {
    if (carry) s = carry[(w.seq * c.tiles + tile0) * c.dim + own];
    else if (h0) s = h0[w.seq * c.dim + own];
  }
  const int at = 32 * wave + sub * K;  // the lane's first token of a tile
  const uint32_t ix = (uint32_t)(sub * K * (int)c.ldx + (int)in.col) * (uint32_t)sizeof(T);
  const uint32_t ih = (uint32_t)(sub * K * (int)ldh + o) * (uint32_t)sizeof(T);
  u32x2 rx[K], rg[K];
  auto load_tile = [&](int tile) {
    const int t = tile * kScanTile;
    const int64_t row = (int64_t)(t + 32 * wave) * c.ldx;
    const bool full = t + kScanTile <= w.len;
    load_run<T, KIND>(x + row, c.ldx, ix, full, w.len - t - at, in, 0u, rx);
    load_run<T, KIND>(g + row, c.ldx, ix, full, w.len - t - at, in, Word<T>::kPast, rg);
  };
  load_tile(tile0);
  for (int tile = tile0; tile < tile1; ++tile) {
    const int t = tile * kScanTile + at, buf = tile & 1;
    const bool full = (tile + 1) * kScanTile <= w.len;
    if (tile * kScanTile >= w.len) {  // uniform: nothing left of the sequence
      if (states && keeper) states[(w.seq * c.tiles + tile) * c.dim + own] = s;
      T* to = out0 + (int64_t)(tile * kScanTile + 32 * wave) * ldh;
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (n > 0 && t + k < c.T) store_row<T, KIND>(row_at(to + k * ldh, ih), (u32x2){0u, 0u}, n);
      continue;
    }
    float a[K][V], b[K][V], A[V], B[V];
    u32x2 cx[K], cg[K];  // this tile's rows; the next ones are on their way from here on
#pragma unroll
    for (int k = 0; k < K; ++k) cx[k] = in.take(rx[k]), cg[k] = in.take(rg[k]);
    if (tile + 1 < tile1) load_tile(tile + 1);
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, B[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float xv[V], gv[V];
      expand(cx[k], xv);
      expand(cg[k], gv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate u = gate<sizeof(T) == 4>(gv[v] + bias[v]);
        a[k][v] = u.a;
        b[k][v] = u.rest * xv[v];
        B[v] = fmaf(a[k][v], B[v], b[k][v]);
        A[v] *= a[k][v];
      }
    }
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
    if (states && keeper) states[(w.seq * c.tiles + tile) * c.dim + own] = s;
    s = fmaf(TA, s, TB);
    start[wave][oc] = mine;
    wave_fence();
    float hv[V];
    from_lds<V>(&start[wave][o], hv);
    wave_fence();
#pragma unroll
    for (int v = 0; v < V; ++v) hv[v] = fmaf(EA[v], hv[v], EB[v]);
    T* to = out0 + (int64_t)(tile * kScanTile + 32 * wave) * ldh;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int v = 0; v < V; ++v) hv[v] = fmaf(a[k][v], hv[v], b[k][v]);
      u32x2 r = collapse(hv);
      if (!full && t + k >= w.len) r = (u32x2){0u, 0u};
      if (n > 0 && (full || t + k < c.T)) store_row<T, KIND>(row_at(to + k * ldh, ih), r, n);
    }
  }
  if (h_last && tile1 == c.tiles) {  // uniform
    __syncthreads();  // h_last may be h0, which every wave has read by now
    if (keeper) h_last[w.seq * c.dim + own] = s;
  }
}

// Composition of every tile of a split sequence, to `pairs`: of h -> a h + (1 - a) x (p is x), or,
// REVERSE, of mu -> a (dh + mu) from a tile's last token to its first (p is dh).  As a rule a
// tile a workgroup, and few enough registers for four of them a CU: what it waits for is its rows.
template <typename T, bool REVERSE, Kind KIND>
__global__ void __launch_bounds__(64 * kScanWaves, 8)
    k_scan_pairs(Call c, const T* __restrict__ p, int64_t ldp, float* __restrict__ pairs) {
  using L = Lanes<T>;
  constexpr int V = L::V, K = L::K, CH = L::CH;
  __shared__ __attribute__((aligned(16))) float tot[2][kScanWaves][CH];
  const Where w = locate<CH>(c, false);
  if (w.seq < 0) return;  // uniform
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int o = lane % L::LV * V, sub = lane / L::LV;
  const int n = c.dim - (w.col + o), own = w.col + (lane & (CH - 1));
  const Reads<T, KIND> in(o, n);
  float bias[V];
  load_bias<V>(c, w, w.col + o, bias);
  for (int tile = w.chunk * c.chunk; tile < min((w.chunk + 1) * c.chunk, c.tiles); ++tile) {
    const int64_t row = w.seq * c.T + tile * kScanTile + 32 * wave;
    if (tile * kScanTile >= w.len) {  // uniform: behind the sequence; 1 s + -0 is s, of -0 too
      if (wave == 0 && lane < CH && own < c.dim)
        *reinterpret_cast<f32x2*>(pairs + 2 * ((w.seq * c.tiles + tile) * c.dim + own)) = (f32x2){1.f, -0.f};
      continue;
    }
    const bool full = (tile + 1) * kScanTile <= w.len;
    const int live = w.len - tile * kScanTile - 32 * wave - sub * K;
    u32x2 rp[K], rg[K];
    load_run<T, KIND>(p + row * ldp + w.col - in.kBack, ldp,
                      (uint32_t)(sub * K * (int)ldp + (int)in.col) * (uint32_t)sizeof(T), full, live, in, 0u, rp);
    load_run<T, KIND>(static_cast<const T*>(c.g) + row * c.ldx + w.col - in.kBack, c.ldx,
                      (uint32_t)(sub * K * (int)c.ldx + (int)in.col) * (uint32_t)sizeof(T), full, live, in,
                      Word<T>::kPast, rg);
    float A[V], B[V], last[V];  // last: the gate before
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = last[v] = 1.f, B[v] = 0.f;
#pragma unroll
    for (int q = 0; q < K; ++q) {
      const int k = REVERSE ? K - 1 - q : q;
      float pv[V], gv[V];
      expand(in.take(rp[k]), pv);
      expand(in.take(rg[k]), gv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate u = gate<sizeof(T) == 4>(gv[v] + bias[v]);
        B[v] = REVERSE ? fmaf(last[v], B[v], pv[v]) : fmaf(u.a, B[v], u.rest * pv[v]);
        A[v] *= u.a;
        last[v] = u.a;
      }
    }
    if (REVERSE) {
#pragma unroll
      for (int v = 0; v < V; ++v) B[v] *= last[v];
    }
    float EA[V], EB[V];
    compose<T, !REVERSE>(sub, A, B, EA, EB);
    if (sub == (REVERSE ? 0 : L::SUBS - 1)) {
      to_lds<V>(&tot[0][wave][o], A);
      to_lds<V>(&tot[1][wave][o], B);
    }
    __syncthreads();
    if (wave == 0 && lane < CH && own < c.dim) {
      float TA = 1.f, TB = 0.f;
      for (int y = 0; y < kScanWaves; ++y) {
        const int q = REVERSE ? kScanWaves - 1 - y : y;
        TB = fmaf(tot[0][q][lane], TB, tot[1][q][lane]);
        TA *= tot[0][q][lane];
      }
      *reinterpret_cast<f32x2*>(pairs + 2 * ((w.seq * c.tiles + tile) * c.dim + own)) = (f32x2){TA, TB};
    }
    __syncthreads();
  }
}

// State (or gradient, REVERSE) at the start of every tile of a split sequence, from the tiles'
// compositions, 64 channels a workgroup: eight waves bring 64 tiles' compositions at a time
// to LDS (the next ones are on their way meanwhile), one wave steps through them.
template <bool REVERSE>
__global__ void __launch_bounds__(512)
    k_scan_carry(Call c, const float* __restrict__ pairs, const float* __restrict__ first,
                 float* __restrict__ carry) {
  constexpr int W = 8, U = 8;
  __shared__ f32x2 stage[W * U][64];
  const int cols = (c.dim + 63) / 64, e = blockIdx.x / cols;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ch = min((int)(blockIdx.x % cols * 64) + lane, c.dim - 1);  // the last one over and over
  const int64_t seq = (int64_t)group_id(c.groups, e / c.batch) * c.batch + e % c.batch;
  const f32x2* p = reinterpret_cast<const f32x2*>(pairs) + seq * c.tiles * c.dim + ch;
  float* out = carry + seq * c.tiles * c.dim + ch;
  float s = first ? first[seq * c.dim + ch] : 0.f;
  f32x2 q[U];
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + wave * U + u, c.tiles - 1);
      q[u] = p[(int64_t)(REVERSE ? c.tiles - 1 - k : k) * c.dim];
    }
  };
  load(0);
  for (int k0 = 0; k0 < c.tiles; k0 += W * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) stage[wave * U + u][lane] = q[u];
    __syncthreads();
    load(k0 + W * U);
    if (wave == 0) {
      const int count = min(W * U, c.tiles - k0);
#pragma unroll 8
      for (int u = 0; u < count; ++u) {
        out[(int64_t)(REVERSE ? c.tiles - 1 - k0 - u : k0 + u) * c.dim] = s;
        const f32x2 r = stage[u][lane];
        s = fmaf(r[0], s, r[1]);
      }
    }
    __syncthreads();
  }
}

// Backward, tiles from the last to the first; carry as in k_scan, for mu.
template <typename T, Kind KIND>
__global__ void __launch_bounds__(64 * kScanWaves, 2)
    k_scan_grad(Call c, const float* __restrict__ states, const T* __restrict__ dh, int64_t lddh,
                const float* dh_last, const float* __restrict__ carry, T* __restrict__ dx,
                T* __restrict__ dg, float* dh0, float* __restrict__ part) {
  using L = Lanes<T>;
  constexpr int V = L::V, K = L::K, CH = L::CH;
  __shared__ __attribute__((aligned(16))) float tot[2][4][kScanWaves][CH];
  __shared__ __attribute__((aligned(16))) float start[kScanWaves][2][CH];
  // a split sequence's tiles in the reverse of the order that their compositions were made in:
  // the last ones are in the memory-side cache still
  const Where w = locate<CH>(c, carry != nullptr);
  if (w.seq < 0) return;  // uniform
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  const int o = lane % L::LV * V, sub = lane / L::LV;
  const int n = c.dim - (w.col + o);
  const int oc = lane & (CH - 1), own = w.col + oc;
  const bool keeper = wave == 0 && lane < CH && own < c.dim;
  const int64_t row0 = w.seq * c.T;
  const Reads<T, KIND> in(o, n);
  const T* x = static_cast<const T*>(c.x) + row0 * c.ldx + w.col - in.kBack;
  const T* g = static_cast<const T*>(c.g) + row0 * c.ldx + w.col - in.kBack;
  const T* d = dh + row0 * lddh + w.col - in.kBack;
  T *dx0 = dx + row0 * c.ldx + w.col, *dg0 = dg + row0 * c.ldx + w.col;
  float bias[V];
  load_bias<V>(c, w, w.col + o, bias);
  const int tile0 = w.chunk * c.chunk, tile1 = min(tile0 + c.chunk, c.tiles);
  float mu = 0.f;
  if (own < c.dim) {
    if (carry) mu = carry[(w.seq * c.tiles + tile1 - 1) * c.dim + own];
    else if (dh_last) mu = dh_last[w.seq * c.dim + own];
  }
  const int at = 32 * wave + sub * K;
  const uint32_t ix = (uint32_t)(sub * K * (int)c.ldx + (int)in.col) * (uint32_t)sizeof(T);
  const uint32_t id = (uint32_t)(sub * K * (int)lddh + (int)in.col) * (uint32_t)sizeof(T);
  const uint32_t iw = KIND == kOdd ? (uint32_t)(sub * K * (int)c.ldx + o) * (uint32_t)sizeof(T) : ix;  // written
  u32x2 rx[K], rg[K], rd[K];
  float s = 0.f;
  auto load_tile = [&](int tile) {
    const int t = tile * kScanTile;
    const int64_t row = (int64_t)(t + 32 * wave) * c.ldx;
    const bool full = t + kScanTile <= w.len;
    load_run<T, KIND>(x + row, c.ldx, ix, full, w.len - t - at, in, 0u, rx);
    s = own < c.dim ? states[(w.seq * c.tiles + tile) * c.dim + own] : 0.f;
    load_run<T, KIND>(g + row, c.ldx, ix, full, w.len - t - at, in, Word<T>::kPast, rg);
    load_run<T, KIND>(d + (int64_t)(t + 32 * wave) * lddh, lddh, id, full, w.len - t - at, in, 0u, rd);
  };
  load_tile(tile1 - 1);
  for (int tile = tile1 - 1; tile >= tile0; --tile) {
    const int t = tile * kScanTile + at, buf = tile & 1;
    const bool full = (tile + 1) * kScanTile <= w.len;
    T *tx = dx0 + (int64_t)(tile * kScanTile + 32 * wave) * c.ldx;
    T *tg = dg0 + (int64_t)(tile * kScanTile + 32 * wave) * c.ldx;
    const int64_t sums = ((w.seq * c.tiles + tile) * waves + wave) * c.dim + w.col + o;
    if (tile * kScanTile >= w.len) {  // uniform: behind the sequence
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (n > 0 && t + k < c.T) {
          store_row<T, KIND>(row_at(tx + k * c.ldx, iw), (u32x2){0u, 0u}, n);
          store_row<T, KIND>(row_at(tg + k * c.ldx, iw), (u32x2){0u, 0u}, n);
        }
      if (part && sub == 0)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v < n) part[sums + v] = 0.f;
      if (tile > tile0) load_tile(tile - 1);
      continue;
    }
    float a[K][V], rest[K][V], A[V], B[V], RA[V], R[V];
    u32x2 cx[K], cg[K], cd[K];  // this tile's rows; the next ones are on their way from here on
    const float here = s;
#pragma unroll
    for (int k = 0; k < K; ++k) cx[k] = in.take(rx[k]), cg[k] = in.take(rg[k]), cd[k] = in.take(rd[k]);
    if (tile > tile0) load_tile(tile - 1);
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, B[v] = R[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float gv[V], xv[V];
      expand(cg[k], gv);
      expand(cx[k], xv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate u = gate<sizeof(T) == 4>(gv[v] + bias[v]);
        a[k][v] = u.a;
        rest[k][v] = u.rest;
        B[v] = fmaf(u.a, B[v], u.rest * xv[v]);
      }
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {  // as in k_scan_pairs
      float dv[V];
      expand(again(cd[k]), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        R[v] = fmaf(k == K - 1 ? 1.f : a[min(k + 1, K - 1)][v], R[v], dv[v]);
        A[v] *= a[k][v];
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) RA[v] = A[v], R[v] *= a[0][v];
    float EA[V], EB[V], FA[V], FR[V];
    compose<T, false>(sub, RA, R, FA, FR);
    if (sub == 0) {
      to_lds<V>(&tot[buf][0][wave][o], RA);
      to_lds<V>(&tot[buf][1][wave][o], R);
    }
    compose<T, true>(sub, A, B, EA, EB);
    if (sub == L::SUBS - 1) {
      to_lds<V>(&tot[buf][2][wave][o], A);
      to_lds<V>(&tot[buf][3][wave][o], B);
    }
    __syncthreads();
    float TA = 1.f, TR = 0.f, mine = 0.f;
    for (int y = waves - 1; y >= 0; --y) {
      if (y == wave) mine = fmaf(TA, mu, TR);
      const float qa = tot[buf][0][y][oc], qr = tot[buf][1][y][oc];
      TR = fmaf(qa, TR, qr);
      TA *= qa;
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
      expand(again(cx[k]), xv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        gap[k][v] = hv[v] - xv[v];
        hv[v] = fmaf(a[k][v], hv[v], rest[k][v] * xv[v]);
      }
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      float ox[V], og[V], dv[V];
      expand(again(cd[k]), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        m[v] = fmaf(k == K - 1 ? 1.f : a[min(k + 1, K - 1)][v], m[v], dv[v]);  // l of token k
        ox[v] = m[v] * rest[k][v];
        og[v] = ox[v] * a[k][v] * gap[k][v];
      }
      if (!full && t + k >= w.len) {  // whatever comes from behind stays behind
#pragma unroll
        for (int v = 0; v < V; ++v) ox[v] = og[v] = 0.f;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) sum[v] += og[v];
      if (n > 0 && (full || t + k < c.T)) {
        store_row<T, KIND>(row_at(tx + k * c.ldx, iw), collapse(ox), n);
        store_row<T, KIND>(row_at(tg + k * c.ldx, iw), collapse(og), n);
      }
    }
    if (part) {
#pragma unroll
      for (int dist = 1; dist < L::SUBS; dist *= 2)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += __shfl_xor(sum[v], dist * L::LV);
      if (sub == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v < n) part[sums + v] = sum[v];
      }
    }
  }
  if (dh0 && tile0 == 0) {  // uniform
    __syncthreads();  // dh0 may be dh_last, which every wave has read by now
    if (keeper) dh0[w.seq * c.dim + own] = mu;
  }
}

// Sequences of at most kShort tokens (a served step above all), a channel a thread: the tile
// kernels would leave most of their waves idle.
constexpr int kShort = 16;
template <typename T>
__global__ void __launch_bounds__(256)
    k_scan_short(Call c, const float* h0, T* __restrict__ h, int64_t ldh, float* h_last,
                 float* __restrict__ states) {
  const int cols = (c.dim + 255) / 256, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 256 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = bias_at(c, id, ch);
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
                      int64_t lddh, const float* dh_last, T* __restrict__ dx, T* __restrict__ dg,
                      float* dh0, float* __restrict__ part) {
  const int cols = (c.dim + 255) / 256, e = blockIdx.x / cols;
  const int ch = blockIdx.x % cols * 256 + threadIdx.x;
  if (ch >= c.dim) return;
  const int id = group_id(c.groups, e / c.batch);
  const int64_t seq = (int64_t)id * c.batch + e % c.batch;
  const float bias = bias_at(c, id, ch);
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

// Grid of the compositions of a split call: a workgroup a tile, up to the limits of a grid.
dim3 tile_grid(Call* c, const Deal& d) {
  c->chunk = (int32_t)ceil_div(d.cols * d.seqs * c->tiles, 1 << 20);
  c->items = (int32_t)(d.cols * d.seqs * ceil_div(c->tiles, c->chunk));
  return dim3(8 * (unsigned)ceil_div(c->items, 8));
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
  c->items = 0;
  return check_groups(n, m, mask, &c->groups);
}

// Calls f with the rows' kind as a constant.  `written` and `read`: whether those rows lie on
// lines; `bytes`: what an unsplit call reads, against 1.5 times the memory-side cache.
template <typename T, typename F>
void by_kind(int dim, bool written, bool read, int64_t bytes, F f) {
  if (dim < Lanes<T>::V) f(std::integral_constant<Kind, kTiny>());
  else if (dim % Lanes<T>::V) f(std::integral_constant<Kind, kOdd>());
  else if (!written) f(std::integral_constant<Kind, kWhole>());
  else if (!read || bytes < (int64_t)384 << 20) f(std::integral_constant<Kind, kLines>());
  else f(std::integral_constant<Kind, kFar>());
}

template <typename T>
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
  c.items = (int32_t)(d.cols * d.seqs * d.chunks);
  const dim3 grid(8 * (unsigned)ceil_div(c.items, 8)), block(64 * d.waves);
  const bool split = d.chunks > 1;
  float* pairs = reinterpret_cast<float*>(static_cast<char*>(ws) + w.pairs);
  float* carry = split ? reinterpret_cast<float*>(static_cast<char*>(ws) + w.carry) : nullptr;
  const int64_t e = sizeof(T), bytes = split ? 0 : 2 * seqs * c.T * c.dim * e;
  by_kind<T>(c.dim, on_lines(h, ldh * e), on_lines(c.x, c.ldx * e) && on_lines(c.g, c.ldx * e), bytes, [&](auto kind) {
    constexpr Kind KIND = decltype(kind)::value;
    if (split) {
      Call each = c;
      hipLaunchKernelGGL((k_scan_pairs<T, false, std::min(KIND, kWhole)>), tile_grid(&each, d), block, 0, s, each,
                         static_cast<const T*>(c.x), c.ldx, pairs);
      hipLaunchKernelGGL(k_scan_carry<false>, dim3((unsigned)(ceil_div(c.dim, 64) * d.seqs)), dim3(512), 0, s, c,
                         pairs, h0, carry);
    }
    hipLaunchKernelGGL((k_scan<T, KIND>), grid, block, 0, s, c, h0, carry, out, ldh, h_last, states);
  });
  return launched("nbsgd_scan");
}

template <typename T>
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
    c.items = (int32_t)(d.cols * d.seqs * d.chunks);
    rows *= (int64_t)c.tiles * d.waves;
    const dim3 grid(8 * (unsigned)ceil_div(c.items, 8)), block(64 * d.waves);
    const bool split = d.chunks > 1;
    float* pairs = reinterpret_cast<float*>(static_cast<char*>(ws) + w.pairs);
    float* carry = split ? reinterpret_cast<float*>(static_cast<char*>(ws) + w.carry) : nullptr;
    const int64_t e = sizeof(T), bytes = split ? 0 : 3 * seqs * c.T * c.dim * e;
    const bool written = on_lines(dx, c.ldx * e) && on_lines(dg, c.ldx * e);
    const bool read = on_lines(c.x, c.ldx * e) && on_lines(c.g, c.ldx * e) && on_lines(dh, lddh * e);
    by_kind<T>(c.dim, written, read, bytes, [&](auto kind) {
      constexpr Kind KIND = decltype(kind)::value;
      if (split) {
        Call each = c;
        hipLaunchKernelGGL((k_scan_pairs<T, true, std::min(KIND, kWhole)>), tile_grid(&each, d), block, 0, s, each,
                           d_in, lddh, pairs);
        hipLaunchKernelGGL(k_scan_carry<true>, dim3((unsigned)(ceil_div(c.dim, 64) * d.seqs)), dim3(512), 0, s, c,
                           pairs, dh_last, carry);
      }
      hipLaunchKernelGGL((k_scan_grad<T, KIND>), grid, block, 0, s, c, states, d_in, lddh, dh_last, carry, ox, og,
                         dh0, part);
    });
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
  const size_t need = T > kScanTile ? w.total : 0;  // a sequence of one tile is not split
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, need)) return st;
  const int64_t kept = seqs * dim * 4, all = kept * w.tiles;
  const Rows b[] = {{"h", h, rows, width, ldh * e},
                    {"h_last", h_last, 1, kept, kept},
                    {"states", states, 1, all, all},
                    {"workspace", workspace, 1, (int64_t)need, (int64_t)need},
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
  const auto run = dtype == NBSGD_F32 ? scan_forward<float> : scan_forward<__bf16>;
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
  const auto run = dtype == NBSGD_F32 ? scan_backward<float> : scan_backward<__bf16>;
  return run(c, w, states, dh, lddh, dh_last, dx, dg, dh0, Gbias, ld, workspace, s);
}
