// carve_short_conv.hip -- the short causal convolution of every channel over its last W
// inputs, with bias and SiLU:
//   p_t = bias + sum_j weight_j x_{t-W+1+j},  y_t = act(p_t)
// Inputs before a sequence's first row come from x0 (its last W - 1 inputs, oldest first)
// or are zero; x_T hands them on.  x0, x_T and the step's pool keep inputs as they are, in
// the token dtype: nothing is rounded there.  Backward for loss <dy, y> + <dx_T, x_T>:
//   dp_t = dy_t act'(p_t),  dx_t = sum_k weight_{W-1-k} dp_{t+k} + dx_T,
//   dweight_j = sum_t dp_t x_{t-W+1+j},  dbias = sum_t dp_t
// over the rows of the same sequence; p is formed again from x.
//
// Bound by HBM: the forward reads x and writes y, the backward reads x and dy and writes
// dx.  A thread takes 16 bytes of channels (8 bf16, 4 f32; 4 channels in the backward) and a
// run of rows, whose last W - 1 inputs it keeps in registers, so that every input is loaded
// once but for the few rows where runs meet (out of L2); four rows are worked on while the
// next four are on their way.  A workgroup is LW threads of channels by 256 / LW runs, LW up
// to 16, 32 in the backward (256 neighbouring bytes a row).  16384 rows of 2304 bf16 channels
// take 37 us (151 MB, 4.1 TB/s), their backward 61 (226 MB, 3.7 TB/s) and 5 for the weights'
// sums; row by row, with the window moved along, they took 44 and 84.  8192 rows of 2304 f32
// channels take 27 us forward and 99 in both directions (378 MB).  A step of a sequence
// takes 3 us, 8 with the call: its loads wait for one another (slot, inputs), no more.
#include "carve_ops.h"

namespace carve {
namespace {

constexpr int kThreads = 256;
constexpr int kBwdV = 4;   // channels of a thread in the backward

// V channels of a row (16 bytes, or 8 with V = 4 of bf16) and their values
template <typename T, int V>
struct Piece {
  static constexpr int words = V * (int)sizeof(T) / 4;
  typedef unsigned raw __attribute__((ext_vector_type(words)));
  static __device__ __forceinline__ raw ld(const T* p) { return *reinterpret_cast<const raw*>(p); }
  static __device__ __forceinline__ void unpack(raw r, float (&f)[V]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < words; ++i) {
        f[2 * i] = __builtin_bit_cast(float, r[i] << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, r[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const unsigned u = r[i];   // (of an element itself the cast takes the first one)
        f[i] = __builtin_bit_cast(float, u);
      }
    }
  }
  static __device__ __forceinline__ void st(T* p, const float (&f)[V]) {
    raw r;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < words; ++i) {
        const f32x2 v = {f[2 * i], f[2 * i + 1]};
        r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) r[i] = __builtin_bit_cast(unsigned, f[i]);
    }
    *reinterpret_cast<raw*>(p) = r;
  }
};
template <typename T, int V>
__device__ __forceinline__ void ld_row(const T* p, float (&f)[V]) {
  Piece<T, V>::unpack(Piece<T, V>::ld(p), f);
}

// weights of a thread's channels, by tap
template <int V, int W>
__device__ __forceinline__ void ld_weights(const float* weight, const float* bias, int c0, float (&w)[W][V], float (&b)[V]) {
  float flat[V * W];
#pragma unroll
  for (int i = 0; i < V * W; i += 4) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(weight + (size_t)c0 * W + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) flat[i + e] = x[e];
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][e] = flat[e * W + j];
    b[e] = 0.0f;
  }
  if (bias) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(bias + c0 + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) b[i + e] = x[e];
    }
  }
}

// Where a row lies: its sequence's rows [first, end) and the sequence, kept while rows
// come in ascending order.  in: whether the row belongs to a sequence.
struct Where {
  int n, first, end;
  bool in;
  __device__ __forceinline__ void at(const ConvArgs& a, int batch, int row) {
    if (!a.offsets) {
      n = batch, first = 0, end = a.T;
    } else {
      n = packed_find(a.offsets, a.nseq, a.T, row);
      packed_seq(a.offsets, n, a.T, first, end);
    }
    in = row >= first && row < end;
  }
  // the first row of a wave's runs of lw lanes (all lanes take part)
  __device__ __forceinline__ void start(const ConvArgs& a, int batch, int row, int lw) {
    if (!a.offsets) n = batch, first = 0, end = a.T;
    else packed_find_wave(a.offsets, a.nseq, a.T, row, lw, n, first, end);
    in = row >= first && row < end;
  }
  // the next row
  __device__ __forceinline__ void next(const ConvArgs& a, int batch, int row) {
    if (a.offsets && row >= end) at(a, batch, row);
    else in = row >= first && row < end;
  }
};

// Input of a sequence at position p of it, from x0 where p < 0.
template <typename T, int W, int V>
__device__ __forceinline__ void ld_past(const ConvArgs& a, const T* x, int n, int first, int p, int c0, float (&f)[V]) {
  if (p >= 0) {
    ld_row<T, V>(x + (size_t)(first + p) * a.x_token + c0, f);
  } else if (a.x0) {
    ld_row<T, V>(reinterpret_cast<const T*>(a.x0) + ((size_t)n * (W - 1) + (W - 1 + p)) * a.C + c0, f);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
  }
}

// A workgroup's place: blocks of channels within blocks of rows within batches, then (last)
// the blocks that make x_T or dx0, a sequence and row of it for each run.
struct Place {
  int batch, row0, c0;     // first row of the thread's run; its first channel
  long long item;          // the blocks of x_T or dx0, and any behind them: which row of them; else -1
};
template <int V>
__device__ __forceinline__ void place(const ConvArgs& a, int R, int lw, int rows_blocks, int batches, Place& p) {
  const int lane = threadIdx.x & (lw - 1), run = threadIdx.x / lw, runs = kThreads / lw;
  const int cblocks = (a.C / V + lw - 1) / lw;
  long long rb;
  int cb;
  if (gridDim.y == 1) {   // (a division of 32 bits)
    cb = blockIdx.x % (unsigned)cblocks, rb = blockIdx.x / (unsigned)cblocks;
  } else {
    const long long b = (long long)blockIdx.y * gridDim.x + blockIdx.x;
    cb = (int)(b % cblocks), rb = b / cblocks;
  }
  const long long main = (long long)rows_blocks * batches;
  p.c0 = (cb * lw + lane) * V;
  p.item = -1;
  p.batch = p.row0 = 0;
  if (rb < main) {
    p.batch = (int)(rb / rows_blocks);
    const long long r = (rb % rows_blocks) * (long long)(runs * R) + (long long)run * R;
    p.row0 = (int)min(r, (long long)a.T);
  } else {
    p.item = (rb - main) * runs + run;
  }
}

__device__ __forceinline__ float act_of(float p, int act) { return act ? silu_f(p) : p; }

// The rows of a run in ascending order.  Where all of a wave's runs lie within a sequence
// (but for its start), rows come by fours with the window in a ring of four, so that no
// value moves and no lane branches, and the next four are under way; else row by row.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) carve_short_conv_fwd_kernel(ConvArgs a, int R, int lw, int rows_blocks, int batches) {
  constexpr int V = Chunk16<T>::N;
  typedef Piece<T, V> P;
  Place pl;
  place<V>(a, R, lw, rows_blocks, batches, pl);
  const int c0 = min(pl.c0, a.C - V);   // (lanes behind the channels do and write what the last one does)
  if (pl.item >= 0) {   // x_T[n][j]: the input at position len - (W - 1) + j
    const long long n = pl.item / (W - 1);
    const int j = (int)(pl.item % (W - 1));
    if (n >= a.nseq || !a.x_T) return;
    int first = 0, end = a.T;
    if (a.offsets) packed_seq(a.offsets, (int)n, a.T, first, end);
    const T* x = reinterpret_cast<const T*>(a.x) + (a.offsets ? 0 : n * a.x_batch);
    float f[V];
    ld_past<T, W, V>(a, x, (int)n, first, end - first - (W - 1) + j, c0, f);
    P::st(reinterpret_cast<T*>(a.x_T) + ((size_t)n * (W - 1) + j) * a.C + c0, f);
    return;
  }
  const int row0 = pl.row0, rows = min(R, a.T - row0);   // (no rows: behind the tensor)
  const T* x = reinterpret_cast<const T*>(a.x) + pl.batch * a.x_batch;
  T* y = reinterpret_cast<T*>(a.y) + ((size_t)pl.batch * a.T + row0) * a.C + c0;
  // (the first rows on their way before the sequence is known)
  const T* xr = x + (size_t)row0 * a.x_token + c0;
  typename P::raw next[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) next[i] = P::ld(x + (size_t)min(row0 + i, a.T - 1) * a.x_token + c0);
  float w[W][V], b[V], past[W - 1][V];
  ld_weights<V, W>(a.weight, a.bias, c0, w, b);
  Where at;
  at.start(a, pl.batch, row0, min(lw, 64));
  if (at.in) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) ld_past<T, W, V>(a, x, at.n, at.first, row0 - at.first - (W - 1) + j, c0, past[j]);
  }
  if (__all(at.in && rows == R && row0 + R <= at.end)) {   // (R is a multiple of four)
    float ring[4][V];   // row r at r mod 4
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) ring[(j + 5 - W) & 3][e] = past[j][e];
#pragma unroll 1
    for (int i0 = 0; i0 < R; i0 += 4) {
      typename P::raw now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) now[i] = next[i];
      xr += 4 * a.x_token;
      if (i0 + 4 < R) {
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = P::ld(xr + (size_t)i * a.x_token);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        P::unpack(now[i], ring[i]);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float p = b[e];
#pragma unroll
          for (int j = 0; j < W; ++j) p += w[j][e] * ring[(i + 5 - W + j) & 3][e];
          o[e] = act_of(p, a.act);
        }
        P::st(y + (size_t)(i0 + i) * a.C, o);
      }
    }
    return;
  }
#pragma unroll 1
  for (int i = 0; i < rows; ++i) {
    const int row = row0 + i;
    if (i > 0) {
      at.next(a, pl.batch, row);
      if (at.in && row == at.first) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) ld_past<T, W, V>(a, x, at.n, at.first, j - (W - 1), c0, past[j]);
      }
    }
    if (!at.in) continue;   // (a row of no sequence is left as it was)
    float cur[V], o[V];
    ld_row<T, V>(x + (size_t)row * a.x_token + c0, cur);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float p = b[e] + w[W - 1][e] * cur[e];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) p += w[j][e] * past[j][e];
      o[e] = act_of(p, a.act);
    }
    P::st(y + (size_t)i * a.C, o);
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) past[j][e] = past[j + 1][e];
#pragma unroll
    for (int e = 0; e < V; ++e) past[W - 2][e] = cur[e];
  }
}

// dp of one row from its window
template <int V, int W>
__device__ __forceinline__ void row_dp(const float (&w)[W][V], const float (&b)[V], const float (&past)[W - 1][V],
                                       const float (&cur)[V], const float (&dy)[V], int act, float (&dp)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    dp[e] = dy[e];
    if (act) {
      float p = b[e] + w[W - 1][e] * cur[e];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) p += w[j][e] * past[j][e];
      dp[e] *= silu_grad_f(p);
    }
  }
}

// The rows of a run in ascending order, and W - 1 more that follow it (for dx alone): row
// u's dp goes to dx of rows u, u - 1, .. u - W + 1 of its sequence, of which acc[k] is that
// of row u - k; acc[W - 1] is then complete.  As in the forward, by fours with rings where
// all of a wave's runs and what follows them lie within a sequence and before its last
// W - 1 rows.  The sums of dweight and dbias over a workgroup's runs are added up in LDS in
// a fixed order and leave as one row of partials.  Four channels a thread: with eight the
// rings, weights and sums take 210 registers, and two waves a SIMD do not hide the loads.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) carve_short_conv_bwd_kernel(ConvArgs a, int lw, int rows_blocks, int batches) {
  constexpr int V = kBwdV, R = kConvBwdRows;
  typedef Piece<T, V> P;
  __shared__ float red[kThreads * (V + 1)];
  Place pl;
  place<V>(a, R, lw, rows_blocks, batches, pl);
  const int c0 = min(pl.c0, a.C - V);   // (lanes behind the channels do and write what the last one does)
  float w[W][V], b[V], past[W - 1][V];
  ld_weights<V, W>(a.weight, a.bias, c0, w, b);
  if (pl.item >= 0) {   // dx0[n][i], the input at position i - (W - 1)
    const long long n = pl.item / (W - 1);
    const int i = (int)(pl.item % (W - 1));
    if (n >= a.nseq || !a.dx0) return;
    int first = 0, end = a.T;
    if (a.offsets) packed_seq(a.offsets, (int)n, a.T, first, end);
    const long long batch = a.offsets ? 0 : n;
    const T* x = reinterpret_cast<const T*>(a.x) + batch * a.x_batch;
    const T* dy = reinterpret_cast<const T*>(a.dy) + (size_t)batch * a.T * a.C + c0;
    const int len = end - first;
    float d[V];
#pragma unroll
    for (int e = 0; e < V; ++e) d[e] = 0.0f;
    if (a.dx_T && i >= len) ld_row<T, V>(reinterpret_cast<const T*>(a.dx_T) + ((size_t)n * (W - 1) + i - len) * a.C + c0, d);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) ld_past<T, W, V>(a, x, (int)n, first, j - (W - 1), c0, past[j]);
#pragma unroll
    for (int u = 0; u < W - 1; ++u) {
      if (u >= len) break;
      float cur[V], g[V], dp[V];
      ld_row<T, V>(x + (size_t)(first + u) * a.x_token + c0, cur);
      ld_row<T, V>(dy + (size_t)(first + u) * a.C, g);
      row_dp<V, W>(w, b, past, cur, g, a.act, dp);
      // weight j of row u reads position u - (W - 1) + j
#pragma unroll
      for (int j = 0; j < W; ++j)
        if (u + j == i)
#pragma unroll
          for (int e = 0; e < V; ++e) d[e] += w[j][e] * dp[e];
#pragma unroll
      for (int j = 0; j + 1 < W - 1; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) past[j][e] = past[j + 1][e];
#pragma unroll
      for (int e = 0; e < V; ++e) past[W - 2][e] = cur[e];
    }
    P::st(reinterpret_cast<T*>(a.dx0) + ((size_t)n * (W - 1) + i) * a.C + c0, d);
    return;
  }
  const int row0 = pl.row0, rows = min(R, a.T - row0);
  const T* x = reinterpret_cast<const T*>(a.x) + pl.batch * a.x_batch + c0;
  const T* dy = reinterpret_cast<const T*>(a.dy) + (size_t)pl.batch * a.T * a.C + c0;
  T* dx = reinterpret_cast<T*>(a.dx) + (size_t)pl.batch * a.T * a.C + c0;
  float aw[W][V], ab[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    ab[e] = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) aw[j][e] = 0.0f;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) past[j][e] = 0.0f;
  }
  Where at;
  at.start(a, pl.batch, row0, min(lw, 64));
  if (at.in) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) ld_past<T, W, V>(a, x - c0, at.n, at.first, row0 - at.first - (W - 1) + j, c0, past[j]);
  }
  if (__all(at.in && rows == R && row0 + R + W - 1 <= at.end)) {
    float ring[4][V], acc[4][V];   // rows r's input and dx at r mod 4
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[j][e] = 0.0f;
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) ring[(j + 5 - W) & 3][e] = past[j][e];
    const T *xr = x + (size_t)row0 * a.x_token, *gr = dy + (size_t)row0 * a.C;
    T* dr = dx + (size_t)row0 * a.C;
    typename P::raw nx[4], ng[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) nx[i] = P::ld(xr + (size_t)i * a.x_token), ng[i] = P::ld(gr + (size_t)i * a.C);
    // row u0 + i, the run's (own) or behind it
    const auto row = [&](int i, typename P::raw rx, typename P::raw rg, bool own) {
      float g[V];
      P::unpack(rx, ring[i]);
      P::unpack(rg, g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float dp = g[e];
        if (a.act) {
          float p = b[e];
#pragma unroll
          for (int j = 0; j < W; ++j) p += w[j][e] * ring[(i + 5 - W + j) & 3][e];
          dp *= silu_grad_f(p);
        }
        if (own) {
          ab[e] += dp;
#pragma unroll
          for (int j = 0; j < W; ++j) aw[j][e] += dp * ring[(i + 5 - W + j) & 3][e];
          acc[i][e] = 0.0f;
        }
#pragma unroll
        for (int k = own ? 0 : 1; k < W; ++k) acc[(i - k) & 3][e] += w[W - 1 - k][e] * dp;
      }
    };
#pragma unroll 1
    for (int u0 = 0; u0 < R; u0 += 4) {
      typename P::raw rx[4], rg[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) rx[i] = nx[i], rg[i] = ng[i];
      xr += 4 * a.x_token, gr += 4 * a.C;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (behind the run only W - 1 rows are there)
        const int r = i < W - 1 ? i : u0 + 4 < R ? i : 0;
        nx[i] = P::ld(xr + (size_t)r * a.x_token), ng[i] = P::ld(gr + (size_t)r * a.C);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        row(i, rx[i], rg[i], true);
        if (u0 > 0 || i >= W - 1) P::st(dr + ((ptrdiff_t)u0 + i - (W - 1)) * a.C, acc[(i - (W - 1)) & 3]);
      }
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      row(i, nx[i], ng[i], false);
      P::st(dr + ((ptrdiff_t)R + i - (W - 1)) * a.C, acc[(i - (W - 1)) & 3]);
    }
  } else if (rows > 0) {
    float acc[W][V];
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[j][e] = 0.0f;
    unsigned ins = 0;   // bit k: whether row u - k belongs to a sequence and to this run
    const int last = row0 + rows + W - 1;   // (rows behind the tensor are of no sequence)
#pragma unroll 1
    for (int u = row0; u < last; ++u) {
      if (u > row0) {
        at.next(a, pl.batch, u);
        if (at.in && u == at.first) {
#pragma unroll
          for (int j = 0; j < W - 1; ++j) ld_past<T, W, V>(a, x - c0, at.n, at.first, j - (W - 1), c0, past[j]);
        }
      }
      const bool own = u < row0 + rows;
      ins = ins << 1 | (at.in && own);
      if (at.in) {
        float cur[V], g[V], dp[V];
        ld_row<T, V>(x + (size_t)u * a.x_token, cur);
        ld_row<T, V>(dy + (size_t)u * a.C, g);
        row_dp<V, W>(w, b, past, cur, g, a.act, dp);
        if (own) {
          const int j = u - at.end + W - 1;   // (one of the sequence's last W - 1 rows)
          if (a.dx_T && j >= 0) ld_row<T, V>(reinterpret_cast<const T*>(a.dx_T) + ((size_t)at.n * (W - 1) + j) * a.C + c0, acc[0]);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            ab[e] += dp[e];
            aw[W - 1][e] += dp[e] * cur[e];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) aw[j][e] += dp[e] * past[j][e];
          }
        }
#pragma unroll
        for (int k = 0; k < W; ++k)
          if (u - k >= at.first)   // (rows before the run take it too and are not written)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[k][e] += w[W - 1 - k][e] * dp[e];
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) past[j][e] = past[j + 1][e];
#pragma unroll
        for (int e = 0; e < V; ++e) past[W - 2][e] = cur[e];
      }
      if (ins >> (W - 1) & 1) P::st(dx + (size_t)(u - (W - 1)) * a.C, acc[W - 1]);
#pragma unroll
      for (int k = W - 1; k > 0; --k)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[k][e] = acc[k - 1][e];
#pragma unroll
      for (int e = 0; e < V; ++e) acc[0][e] = 0.0f;
    }
  }
  // the workgroup's sums, a tap at a time: a thread adds its channel's runs in order
  const int lane = threadIdx.x & (lw - 1), runs = kThreads / lw;
  const int cblocks = (a.C / V + lw - 1) / lw;
  const long long part = ((long long)blockIdx.y * gridDim.x + blockIdx.x) / cblocks;
  float* out = a.partial + (size_t)part * (W + 1) * a.C;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    if (j == W && !a.dbias) break;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) red[threadIdx.x * (V + 1) + e] = j < W ? aw[j < W ? j : 0][e] : ab[e];
    __syncthreads();
    for (int i = threadIdx.x; i < lw * V; i += kThreads) {
      const int l = i / V, e = i % V;
      float s = 0.0f;
      for (int r = 0; r < runs; ++r) s += red[(r * lw + l) * (V + 1) + e];
      const int col = (pl.c0 - lane * V) + i;
      if (col < a.C) out[(size_t)j * a.C + col] = s;
    }
  }
}

// dweight [C][W] and dbias [C] from the workgroups' partials, in order, in 64 bits: a dense
// batch of short sequences leaves a part for each of them, and 2^18 equal terms added up in f32
// are 2e-4 off
__global__ void __launch_bounds__(256) carve_short_conv_reduce_kernel(ConvArgs a, int W, long long parts) {
  __shared__ double red[4][64];
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + tx, n = (W + (a.dbias ? 1 : 0)) * a.C;
  const size_t step = (size_t)(W + 1) * a.C;
  double s = 0.0;
  if (col < n) {
    const float* p = a.partial + col;
    long long i = ty;
    for (; i + 28 < parts; i += 32) {   // eight loads in flight
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = p[(i + 4 * e) * step];
#pragma unroll
      for (int e = 0; e < 8; ++e) s += (double)f[e];
    }
    for (; i < parts; i += 4) s += (double)p[i * step];
  }
  red[ty][tx] = s;
  __syncthreads();
  if (ty == 0 && col < n) {
    s = (red[0][tx] + red[1][tx]) + (red[2][tx] + red[3][tx]);
    const int j = col / a.C, c = col % a.C;
    if (j < W) a.dweight[(size_t)c * W + j] = (float)s;
    else a.dbias[c] = (float)s;
  }
}

// T tokens of a sequence on its last inputs in the pool; a thread for 16 bytes of channels.
template <typename T, int W>
__global__ void __launch_bounds__(64) carve_short_conv_step_kernel(ConvStepArgs a) {
  constexpr int V = Chunk16<T>::N;
  const int c0 = ((int)blockIdx.x * 64 + (int)threadIdx.x) * V, b = blockIdx.y;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.pool || c0 >= a.C) return;
  T* st = reinterpret_cast<T*>(a.state) + (size_t)slot * (W - 1) * a.C + c0;
  const T* x = reinterpret_cast<const T*>(a.x) + b * a.x_batch + c0;
  T* y = reinterpret_cast<T*>(a.y) + (size_t)b * a.T * a.C + c0;
  typedef Piece<T, V> P;
  typename P::raw keep[W - 1], raw = P::ld(x);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) keep[j] = P::ld(st + (size_t)j * a.C);
  float w[W][V], bi[V];
  ld_weights<V, W>(a.weight, a.bias, c0, w, bi);
  for (int t = 0; t < a.T; ++t) {
    const typename P::raw now = raw;
    if (t + 1 < a.T) raw = P::ld(x + (size_t)(t + 1) * a.x_token);
    float cur[V], o[V];
    P::unpack(now, cur);
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = bi[e] + w[W - 1][e] * cur[e];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      float f[V];
      P::unpack(keep[j], f);
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] += w[j][e] * f[e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = act_of(o[e], a.act);
    P::st(y + (size_t)t * a.C, o);
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j) keep[j] = keep[j + 1];
    keep[W - 2] = now;
  }
#pragma unroll
  for (int j = 0; j < W - 1; ++j) *reinterpret_cast<typename P::raw*>(st + (size_t)j * a.C) = keep[j];
}

// threads side by side on a row, V channels each: a power of two, up to 256 bytes of it
int lanes_of(int C, int V, size_t esize) {
  int lw = 1;
  while (lw * V * (int)esize < 256 && lw * V < C) lw *= 2;
  return lw;
}

// blocks in two dimensions, each below 2^32 threads
bool grid_of(long long blocks, dim3& g) {
  const long long gx = blocks < (1 << 20) ? blocks : 1 << 20, gy = (blocks + gx - 1) / gx;
  if (gy > 65535) return false;
  g = dim3((unsigned)gx, (unsigned)gy);
  return true;
}

// Rows of a thread in the forward: runs of 16, but of 4 where those would be fewer workgroups
// than compute units.  (By 16 and by 4, on one input again and again, replayed from a graph:
// 16384 x 2304, 1152 workgroups by 16, 30 and 43 us; 16384 x 1024, 512: 15.8 and 21.8; 256: 10.0
// and 13.4; 192: 9.6 and 10.5; 128: 9.2 and 7.9; 64: 8.6 and 5.8; 2048 x 512, 32: 8.3 and 5.6.)
constexpr int kConvRows = 16, kConvFewRows = 4;
constexpr long long kConvFewBlocks = 256;

template <typename T, int W>
int launch_fwd(const ConvArgs& a, hipStream_t s) {
  constexpr int V = Chunk16<T>::N;
  const int lw = lanes_of(a.C, V, sizeof(T)), runs = kThreads / lw, cb = (a.C / V + lw - 1) / lw;
  const int batches = a.offsets ? 1 : a.nseq;
  const auto blocks = [&](int R) { return (a.T + (long long)runs * R - 1) / (runs * R); };
  const int R = blocks(kConvRows) * batches * cb < kConvFewBlocks ? kConvFewRows : kConvRows;
  const int rb = (int)blocks(R);
  const long long tail = a.x_T ? ((long long)a.nseq * (W - 1) + runs - 1) / runs : 0;
  dim3 g;
  if (!grid_of(((long long)rb * batches + tail) * cb, g)) return CARVE_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((carve_short_conv_fwd_kernel<T, W>), g, dim3(kThreads), 0, s, a, R, lw, rb, batches);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int W>
int launch_bwd(const ConvArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  constexpr int V = kBwdV;
  const int lw = lanes_of(a.C, V, sizeof(T)), runs = kThreads / lw;
  const int batches = a.offsets ? 1 : a.nseq, rows = runs * kConvBwdRows;
  const int rb = (int)((a.T + (long long)rows - 1) / rows), cb = (a.C / V + lw - 1) / lw;
  const long long tail = a.dx0 ? ((long long)a.nseq * (W - 1) + runs - 1) / runs : 0;
  dim3 g;
  if (!grid_of(((long long)rb * batches + tail) * cb, g)) return CARVE_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((carve_short_conv_bwd_kernel<T, W>), g, dim3(kThreads), 0, s, a, lw, rb, batches);
  if (hipGetLastError() != hipSuccess) return CARVE_ERR_HIP;
  mark(s);
  const int cols = (W + (a.dbias ? 1 : 0)) * a.C;
  hipLaunchKernelGGL(carve_short_conv_reduce_kernel, dim3((cols + 63) / 64), dim3(256), 0, s, a, W, (long long)rb * batches);
  if (hipGetLastError() != hipSuccess) return CARVE_ERR_HIP;
  mark(s);
  return CARVE_OK;
}
template <typename T, int W>
int launch_step(const ConvStepArgs& a, hipStream_t s) {
  const int chunks = a.C / Chunk16<T>::N;
  hipLaunchKernelGGL((carve_short_conv_step_kernel<T, W>), dim3((chunks + 63) / 64, a.B), dim3(64), 0, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}

}  // namespace

int conv_bwd_block_rows(int C, int dtype) { return kThreads / lanes_of(C, kBwdV, dtype == CARVE_BF16 ? 2 : 4) * kConvBwdRows; }
long long conv_parts(long long T, int batches, int C, int dtype) {
  const int rows = conv_bwd_block_rows(C, dtype);
  return (T + rows - 1) / rows * batches;
}

#define CARVE_BY_W(call)                                                  \
  switch (W) {                                                            \
    case 2: return dtype == CARVE_BF16 ? call(bf16_t, 2) : call(float, 2); \
    case 3: return dtype == CARVE_BF16 ? call(bf16_t, 3) : call(float, 3); \
    case 4: return dtype == CARVE_BF16 ? call(bf16_t, 4) : call(float, 4); \
    default: return CARVE_ERR_UNSUPPORTED;                                \
  }
int launch_short_conv_fwd(const ConvArgs& a, int W, int dtype, hipStream_t s) {
#define CALL(T, N) launch_fwd<T, N>(a, s)
  CARVE_BY_W(CALL)
#undef CALL
}
int launch_short_conv_bwd(const ConvArgs& a, int W, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
#define CALL(T, N) launch_bwd<T, N>(a, s, mark)
  CARVE_BY_W(CALL)
#undef CALL
}
int launch_short_conv_step(const ConvStepArgs& a, int W, int dtype, hipStream_t s) {
#define CALL(T, N) launch_step<T, N>(a, s)
  CARVE_BY_W(CALL)
#undef CALL
}
#undef CARVE_BY_W

}  // namespace carve
