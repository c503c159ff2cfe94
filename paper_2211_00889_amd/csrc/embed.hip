// Embedding lookup with scaling and its gradient, per learner and mini-batch (gfx950).
#include <algorithm>

#include "device_rows.h"

using namespace nbsgd;

namespace {

// Y[t][:] = scale * E[token[t]][:]: a team of L lanes a token, 16 bytes of Y a lane.  What
// bounds it is the store of Y; the table's rows of frequent tokens come from the caches.  LINES:
// Y's rows are whole 128-byte lines, and go past the caches (36 mini-batches of 2048 tokens, 512
// bf16: 35 -> 31 us).
template <typename T, bool LINES>
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
      if (inside && n > 4 * q) Elem<float>::expand(load16(src + c + 4 * q, n - 4 * q), w);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[4 * q + k] = inside ? scale * w[k] : 0.f;
    }
    if (LINES && n == V) __builtin_nontemporal_store(Elem<T>::collapse(v), reinterpret_cast<u32x4*>(dst + c));
    else store16<T>(dst + c, Elem<T>::collapse(v), n);
  }
}

// ---- gradient of the lookup
//
// The tokens of a mini-batch are sorted (k_sort, stable, so that equal tokens keep their order)
// and the rows of dY added run by run, by teams of lanes that take equal pieces of the sorted
// tokens, so that every team has the same work whatever the tokens are.  A row whose tokens
// cross a piece's border is summed from the pieces' parts, in order, by k_embed_join; no atomics.
// What bounds it is the write of G, vocab x dim floats a mini-batch: workgroups beside the sort
// write zeros to all of it, and hide it, and the rows that have tokens are written again.  (With
// pieces of the tokens merged with the table's rows each row is written once, but after the sort:
// 16 x 8192 tokens, 32000 x 512, 289 against 264 us; with as many tokens as rows 125 against 115,
// with 16 times as many 106 against 108.)
// Sorted entry: token in the high word, position in the low; tokens outside the table as vocab.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

// Stable sort of up to 1024 x ITEMS tokens of a mini-batch by one workgroup, 8 bits a pass: a
// wave ranks its tokens against its lanes' equal digits by ballots and its own histogram, the
// histograms are added over waves and digits, and the tokens go to their places in LDS.
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads)
    k_sort(const int32_t* __restrict__ tokens, int Tn, int vocab, int bits, uint2* __restrict__ keys,
           float* __restrict__ G, int64_t ld, int64_t size, int fills, Groups groups) {
  constexpr int N = kSortThreads * ITEMS;
  const int runs = (Tn + N - 1) / N, sorts = runs * groups.count;
  if ((int)blockIdx.x >= sorts) {  // uniform: a part of a mini-batch's zeros
    const int f = blockIdx.x - sorts;
    float* to = G + (int64_t)group_id(groups, f / fills) * ld;
    const int64_t quads = size / 4, from = f % fills * (int64_t)kSortThreads + threadIdx.x;
    const int64_t each = (quads + fills - 1) / fills, q1 = min((f % fills + 1) * each, quads);
    for (int64_t k = f % fills * each + threadIdx.x; k < q1; k += kSortThreads)
      __builtin_nontemporal_store((f32x4){0.f, 0.f, 0.f, 0.f}, reinterpret_cast<f32x4*>(to) + k);
    if (from < size % 4) to[4 * quads + from] = 0.f;
    return;
  }
  __shared__ uint32_t tok[N];
  __shared__ uint16_t pos[N];
  __shared__ uint32_t hist[kSortWaves][256];
  __shared__ uint32_t wsum[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t id = group_id(groups, blockIdx.x / runs);
  const int first = blockIdx.x % runs * N, count = min(N, Tn - first);
  const int32_t* src = tokens + id * Tn + first;
  // wave w holds tokens 64 ITEMS w + 64 k + lane, k = 0 .. ITEMS - 1; the ones past the count sort last
  uint32_t key[ITEMS], at[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int p = 64 * (ITEMS * wave + k) + lane;
    const int32_t t = p < count ? src[p] : 0;
    key[k] = p >= count ? (uint32_t)vocab + 1 : t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab;
    at[k] = p;
  }
  for (int shift = 0; shift < bits; shift += 8) {
    for (int k = tid; k < kSortWaves * 256; k += kSortThreads) (&hist[0][0])[k] = 0;
    __syncthreads();
    uint32_t rank[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const uint32_t digit = key[k] >> shift & 0xffu;
      uint64_t same = ~0ull;  // lanes with this lane's digit
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint64_t set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
      }
      const uint64_t below = same & ((1ull << lane) - 1);
      const uint32_t before = hist[wave][digit];
      rank[k] = before + __popcll(below);
      wave_fence();
      if (!below) hist[wave][digit] = before + __popcll(same);
      wave_fence();
    }
    __syncthreads();
    // exclusive sums over (digit, wave): thread (q, d) of four takes waves 4 q .. 4 q + 3 of digit d
    {
      const int d = tid >> 2, q = tid & 3;
      uint32_t v[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = sum;
        sum += hist[4 * q + k][d];
      }
      uint32_t run = sum;  // inclusive over the wave's threads
#pragma unroll
      for (int dist = 1; dist < 64; dist *= 2) {
        const uint32_t up = __shfl_up(run, dist);
        if (lane >= dist) run += up;
      }
      if (lane == 63) wsum[wave] = run;
      __syncthreads();
      uint32_t base = run - sum;
      for (int k = 0; k < wave; ++k) base += wsum[k];
#pragma unroll
      for (int k = 0; k < 4; ++k) hist[4 * q + k][d] = base + v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const uint32_t to = hist[wave][key[k] >> shift & 0xffu] + rank[k];
      tok[to] = key[k];
      pos[to] = (uint16_t)at[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int p = 64 * (ITEMS * wave + k) + lane;
      key[k] = tok[p];
      at[k] = pos[p];
    }
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int p = 64 * (ITEMS * wave + k) + lane;
    if (p < count) keys[id * Tn + first + p] = make_uint2(at[k] + first, key[k]);
  }
}

// Places of the sorted runs' entries in the whole: an entry's own rank in its run and its rank in
// each other one, four runs searched at a time (the steps of one search wait for each other).
// Whole entries are compared, so there are no ties.
__global__ void __launch_bounds__(256)
    k_sort_join(const uint2* __restrict__ keys, int Tn, int run, uint2* __restrict__ sorted, Groups groups) {
  constexpr int U = 4;
  const int64_t id = group_id(groups, blockIdx.y);
  const int p = blockIdx.x * 256 + threadIdx.x;
  if (p >= Tn) return;
  const uint2* s = keys + id * Tn;
  const uint2 e = s[p];
  const int own = p / run, runs = (Tn + run - 1) / run;
  int to = p % run;
  for (int r0 = 0; r0 < runs; r0 += U) {
    int lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      lo[u] = 0;
      hi[u] = r0 + u < runs && r0 + u != own ? min(run, Tn - (r0 + u) * run) : 0;
    }
    for (int n = run; n > 0; n >>= 1) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (lo[u] >= hi[u]) continue;
        const int mid = (lo[u] + hi[u]) >> 1;
        const uint2 v = s[(r0 + u) * run + mid];
        if (v.y < e.y || (v.y == e.y && v.x < e.x)) lo[u] = mid + 1;
        else hi[u] = mid;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) to += lo[u];
  }
  sorted[id * Tn + to] = e;
}

// The first n (at most 4) elements at p, zeros behind them; and back.
__device__ __forceinline__ void load4(const float* p, int n, float (&v)[4]) {
  Elem<float>::expand(load16(p, n), v);
}
__device__ __forceinline__ void load4(const __bf16* p, int n, float (&v)[4]) {
  if (n >= 4) {
    const u32x2 r = *reinterpret_cast<const u32x2_any*>(p);
    v[0] = bf16_lo(r[0]), v[1] = bf16_hi(r[0]), v[2] = bf16_lo(r[1]), v[3] = bf16_hi(r[1]);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = k < n ? (float)p[k] : 0.f;
}
__device__ __forceinline__ void store4(float* p, int n, const float (&v)[4]) {
  store16<float>(p, Elem<float>::collapse(v), n);
}

// A piece of a row of G, which nothing reads again soon (269 -> 227 us for 1.05 GB).
__device__ __forceinline__ void store_row4(float* p, int n, const float (&v)[4]) {
  if (n == 4) __builtin_nontemporal_store(Elem<float>::collapse(v), reinterpret_cast<u32x4_any*>(p));
  else store4(p, n, v);
}

constexpr int kMinTeam = 16;

// What the gradient's kernels are told.
struct GradCall {
  const uint2* sorted;
  int32_t* flags;   // per piece: the row that it ended for an earlier piece, or -1
  float* parts;     // per piece: that row's share of the piece, and the piece's share of the row it leaves
  float* G;
  int64_t ldy, ld, pieces;
  int32_t T, vocab, dim, items, L;  // tokens of a piece, lanes of a team
  float scale;
  Groups groups;
};

// A team a piece: its entries to LDS, then the rows of dY in their order, U of them under way.
template <typename T>
__global__ void __launch_bounds__(256) k_embed_grad(const T* __restrict__ dY, GradCall c) {
  constexpr int V = 4, U = 8;
  __shared__ uint2 stage[256 / kMinTeam][kMaxPiece];
  const int64_t id = group_id(c.groups, blockIdx.y);
  const int team = threadIdx.x / c.L, l = threadIdx.x % c.L;
  const int64_t piece = (int64_t)blockIdx.x * (256 / c.L) + team;
  const uint2* s = c.sorted + id * c.T;
  const int k0 = (int)min(piece, c.pieces - 1) * c.items, k1 = min(k0 + c.items, c.T);
  uint2* mine = stage[team];
  for (int k = l; k < k1 - k0; k += c.L) mine[k] = s[k0 + k];
  const uint32_t before = k0 ? s[k0 - 1].y : ~0u, behind = k1 < c.T ? s[k1].y : ~0u;
  __syncthreads();
  if (piece >= c.pieces) return;
  int count = k1 - k0;  // tokens outside the table come last, and are not read
  while (count > 0 && mine[count - 1].y == (uint32_t)c.vocab) --count;
  const bool carried = count > 0 && before == mine[0].y;
  const bool open = count > 0 && behind == mine[count - 1].y;
  // the piece ends the row that it was handed, unless it goes on behind it
  const bool ends = carried && !(open && mine[0].y == mine[count - 1].y);
  if (l == 0) c.flags[id * c.pieces + piece] = ends ? (int)mine[0].y : -1;
  const T* rows = dY + id * c.T * c.ldy;
  float* part = c.parts + 2 * (id * c.pieces + piece) * c.dim;
  for (int col = V * l; col < c.dim; col += V * c.L) {
    const int n = min(V, c.dim - col);
    float sum[V] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < count; k += U) {
      float e[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u)
        load4(rows + (int64_t)mine[min(k + u, count - 1)].x * c.ldy + col, n, e[u]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k + u >= count) break;
        const uint32_t r = mine[k + u].y;
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += e[u][v];
        if (k + u + 1 < count ? mine[k + u + 1].y == r : open) continue;  // the row goes on
        if (ends && r == mine[0].y) {
          store4(part + col, n, sum);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) sum[v] *= c.scale;
          store_row4(c.G + id * c.ld + (int64_t)r * c.dim + col, n, sum);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = 0.f;
      }
    }
    if (open) store4(part + c.dim + col, n, sum);
  }
}

// The rows that more than one piece has tokens of: the earlier pieces' parts in order, then the
// last piece's.  A wave a piece; most of them end no such row.
__global__ void __launch_bounds__(256) k_embed_join(GradCall c) {
  const int64_t id = group_id(c.groups, blockIdx.y);
  const int lane = threadIdx.x & 63;
  const int64_t piece = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (piece >= c.pieces) return;
  const int r = c.flags[id * c.pieces + piece];
  if (r < 0) return;  // uniform in the wave
  const uint2* s = c.sorted + id * c.T;
  int lo = 0, hi = c.T;  // the first token of row r
  while (lo < hi) {
    const int n = hi - lo, p = n <= 64 ? min(lo + lane, hi - 1) : lo + (int)((int64_t)n * (lane + 1) / 65);
    const int below = __popcll(__ballot(s[p].y < (uint32_t)r));
    const int from = lo;
    if (n <= 64) {
      lo = hi = from + min(below, n);
    } else {
      if (below) lo = from + (int)((int64_t)n * below / 65) + 1;
      if (below < 64) hi = from + (int)((int64_t)n * (below + 1) / 65);
    }
  }
  const float* parts = c.parts + 2 * id * c.pieces * c.dim;
  for (int col = 4 * lane; col < c.dim; col += 256) {
    const int n = min(4, c.dim - col);
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, e[4];
#pragma unroll 16
    for (int64_t q = lo / c.items; q < piece; ++q) {
      load4(parts + (2 * q + 1) * c.dim + col, n, e);
#pragma unroll
      for (int v = 0; v < 4; ++v) sum[v] += e[v];
    }
    load4(parts + 2 * piece * c.dim + col, n, e);
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[v] = c.scale * (sum[v] + e[v]);
    store4(c.G + id * c.ld + (int64_t)r * c.dim + col, n, sum);
  }
}

// Few tokens: no sort, one launch (128 tokens and 1,000 rows of 64: 9 us, 18 through the sort; from
// 256 on, rows that many tokens share take longer than it: 32,000 x 512, 59 against 30 us).
// Every wave holds the mini-batch's tokens, up to two a lane, and goes through kFewRows rows of
// the table, a team a row: the ballots of the lanes whose token is the row's give the rows of
// dY, which are added in their order, U under way.
constexpr int kFewTokens = 128, kFewRows = 4;
template <typename T>
__global__ void __launch_bounds__(256)
    k_embed_grad_few(const T* __restrict__ dY, const int32_t* __restrict__ tokens, GradCall c) {
  constexpr int V = 4, U = 8, Q = kFewTokens / 64;
  const int64_t id = group_id(c.groups, blockIdx.y);
  const int lane = threadIdx.x & 63, teams = 64 / c.L, team = lane / c.L;
  const int v0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * kFewRows, v1 = min(v0 + kFewRows, c.vocab);
  const int32_t* src = tokens + id * c.T;
  const T* rows = dY + id * c.T * c.ldy;
  int tok[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) tok[q] = 64 * q + lane < c.T ? src[64 * q + lane] : -1;
  for (int v = v0; v < v1; v += teams) {
    uint64_t hit[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      hit[q] = 0;
      if (64 * q >= c.T) continue;  // uniform
      for (int t = 0; t < teams; ++t) {
        const uint64_t set = __ballot(tok[q] == v + t);
        hit[q] = t == team ? set : hit[q];
      }
    }
    if (v + team >= v1) continue;
    uint64_t any = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) any |= hit[q];
    const float scale = any ? c.scale : 0.f;  // a row without tokens is 0, of an infinite scale too
    float* to = c.G + id * c.ld + (int64_t)(v + team) * c.dim;
    for (int col = V * (lane % c.L); col < c.dim; col += V * c.L) {
      const int n = min(V, c.dim - col);
      float sum[V] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        uint64_t left = hit[q];
        while (left) {
          float e[U][V];
          int got = 0, t = 0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (left) {  // the last one once more behind it
              t = 64 * q + __builtin_ctzll(left);
              left &= left - 1;
              ++got;
            }
            load4(rows + (int64_t)t * c.ldy + col, n, e[u]);
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (u < got)
#pragma unroll
              for (int v4 = 0; v4 < V; ++v4) sum[v4] += e[u][v4];
        }
      }
#pragma unroll
      for (int v4 = 0; v4 < V; ++v4) sum[v4] *= scale;
      store_row4(to + col, n, sum);
    }
  }
}

template <int ITEMS>
void sort_launch(const int32_t* tokens, const GradCall& c, int bits, uint2* keys, hipStream_t s) {
  const int64_t size = (int64_t)c.vocab * c.dim;
  // about 2,048 workgroups of zeros, each with at least four rounds of stores
  const int64_t fills = std::min<int64_t>(ceil_div(2048, c.groups.count), ceil_div(size, 16 * kSortThreads));
  hipLaunchKernelGGL(k_sort<ITEMS>, dim3((unsigned)((ceil_div(c.T, kSortThreads * ITEMS) + fills) * c.groups.count)),
                     dim3(kSortThreads), 0, s, tokens, c.T, c.vocab, bits, keys, c.G, c.ld, size, (int)fills,
                     c.groups);
}

template <typename T>
void embed_grad_launch(const void* dY, const int32_t* tokens, GradCall c, const EmbedSpace& w, void* ws,
                       hipStream_t s) {
  uint2* keys = reinterpret_cast<uint2*>(static_cast<char*>(ws) + w.keys);
  uint2* sorted = reinterpret_cast<uint2*>(static_cast<char*>(ws) + w.sorted);
  c.flags = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + w.flags);
  c.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + w.parts);
  c.pieces = w.pieces;
  c.items = w.items;
  c.L = kMinTeam;
  if (c.T <= kFewTokens) {
    while (c.L < 64 && c.L * 4 < c.dim) c.L *= 2;
    hipLaunchKernelGGL(k_embed_grad_few<T>, dim3((unsigned)ceil_div(c.vocab, 4 * kFewRows), c.groups.count),
                       dim3(256), 0, s, static_cast<const T*>(dY), tokens, c);
    return;
  }
  int bits = 1;
  while ((c.vocab + 1) >> bits) ++bits;  // of vocab + 1, the largest key
  // one run up to 8,192 tokens: 18 us at that length, against 8 us for runs of 2,048 and 14 to
  // join them
  int run = kSortThreads;
  if (c.T <= kSortThreads) {
    sort_launch<1>(tokens, c, bits, keys, s);
  } else if (c.T <= 4 * kSortThreads) {
    sort_launch<4>(tokens, c, bits, keys, s);
    run = 4 * kSortThreads;
  } else {
    sort_launch<8>(tokens, c, bits, keys, s);
    run = 8 * kSortThreads;
  }
  c.sorted = keys;
  if (c.T > run) {
    hipLaunchKernelGGL(k_sort_join, dim3((unsigned)ceil_div(c.T, 256), c.groups.count), dim3(256), 0, s,
                       keys, c.T, run, sorted, c.groups);
    c.sorted = sorted;
  }
  while (c.L < 128 && c.L * 4 < c.dim) c.L *= 2;
  const dim3 grid((unsigned)ceil_div(c.pieces, 256 / c.L), c.groups.count);
  hipLaunchKernelGGL(k_embed_grad<T>, grid, dim3(256), 0, s, static_cast<const T*>(dY), c);
  hipLaunchKernelGGL(k_embed_join, dim3((unsigned)ceil_div(c.pieces, 4), c.groups.count), dim3(256), 0, s, c);
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
  const auto go = [&](auto kernel, auto y) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, E, ld, vocab, dim, scale, tokens, T, y, ldy, L, g);
  };
  const bool lines = on_lines(Y, ldy * e);
  if (dtype == NBSGD_F32) go(lines ? k_embed<float, true> : k_embed<float, false>, static_cast<float*>(Y));
  else go(lines ? k_embed<__bf16, true> : k_embed<__bf16, false>, static_cast<__bf16*>(Y));
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
  const EmbedSpace w = embed_space((int64_t)n * m, T, dim);
  if (nbsgd_status st = check_workspace(workspace, workspace_bytes, w.total)) return st;
  const Rows b[] = {{"G", G, (int64_t)n * m, (int64_t)vocab * dim * 4, ld * 4},
                    {"workspace", workspace, 1, (int64_t)w.total, (int64_t)w.total},
                    {"dY", dY, rows, (int64_t)dim * e, ldy * e},
                    {"tokens", tokens, 1, rows * 4, rows * 4}};
  if (nbsgd_status st = check_apart(b, 4, 2)) return st;
  if (nbsgd_status st = check_stream(stream)) return st;
  if (!g.count) return NBSGD_OK;
  GradCall c;
  c.G = G;
  c.ldy = ldy;
  c.ld = ld;
  c.T = T;
  c.vocab = vocab;
  c.dim = dim;
  c.scale = scale;
  c.groups = g;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == NBSGD_F32) embed_grad_launch<float>(dY, tokens, c, w, workspace, s);
  else embed_grad_launch<__bf16>(dY, tokens, c, w, workspace, s);
  return launched("nbsgd_embed_grad");
}
