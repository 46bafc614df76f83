// carve_block_norm.hip -- the norms before and after a block, fused with the
// block's gate and its scaled addition to the residual stream (rows of N):
//   n = y rsqrt(mean_group(y^2) + eps) weight        (groups of N / groups values)
//   t = n act(gate),  x = alpha residual + scale t
//   h = x rsqrt(mean(x^2) + eps) next_weight         (the next block's input)
// and backward for loss <dx, x> + <dh, h>, with everything formed again from y,
// gate and residual:
//   dX = dx + r2 (m - x r2^2 mean(m x)),  m = dh next_weight
//   dresidual = alpha dX,  dt = scale dX,  dgate = dt n act'(gate),  dn = dt act(gate)
//   dy = r1 (dn weight - y r1 mean_group(dn weight y r1))
//   dweight = sum dn y r1,  dscale = sum dX t,  dnext_weight = sum dh x r2
//
// Every row tensor is read once and written once.  16384 rows of 2048 in bf16, everything
// given: forward 335 MB in 71 us, 4.7 TB/s, bound by HBM and to a lesser part by its vector
// instructions (f32 rows of as many bytes, half as many values: 65 us; rows of 256 in bf16,
// which leave half of a wave idle, 97 us, in f32 61); backward with the parameters' sums 537
// MB in 129 us, 4.2 TB/s.  Norm and gate alone in 16 groups: 43 and 85 us for 201 and 336
// MB.  Of the same size, 4096 columns: 75 and 150 us; 8192: 93 and 238 us, where the
// registers of a row leave three waves a SIMD forward and one backward, which has no row
// loaded ahead beyond eight columns a thread; in f32, 2048, 4096 and 8192 columns: 65, 70,
// 79 and 117, 133, 198 us.
//
// NT threads (one wave, or four) hold a row in registers, NCH 16-byte chunks each; sums
// run over a group's lanes by DPP and over the waves through LDS.  Statistics, x and the
// gradients are f32 until they are stored; h comes from the unrounded x, and so
// does the backward, which forms x again instead of reading the rounded one.
#include "carve_kernels.h"

namespace carve {
namespace {

template <typename T>
struct Vec;
template <>
struct Vec<bf16_t> {
  static constexpr int n = 8;
};
template <>
struct Vec<float> {
  static constexpr int n = 4;
};

template <typename T>
__device__ __forceinline__ void ld_vec(const T* p, float* f) {
  Chunk16<T>::unpack(*reinterpret_cast<const u32x4_t*>(p), f);
}
template <typename T>
__device__ __forceinline__ void st_vec(T* p, const float* f) {
  *reinterpret_cast<u32x4_t*>(p) = Chunk16<T>::pack(f);
}
__device__ __forceinline__ void ld_f32(const float* p, float* f, int n) {
  for (int i = 0; i < n; i += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
    for (int e = 0; e < 4; ++e) f[i + e] = v[e];
  }
}

// sum over aligned groups of n lanes (n a power of two up to 64, uniform)
__device__ __forceinline__ float lanes_sum(float x, int n) {
  switch (n) {
    case 1: return x;
    case 2: return group_sum<2>(x);
    case 4: return group_sum<4>(x);
    case 8: return group_sum<8>(x);
    case 16: return group_sum<16>(x);
    case 32: return group_sum<32>(x);
    default: return group_sum<64>(x);
  }
}
// Sums over the row of two values at once, in every thread of the row.  One barrier: a
// buffer is written again only behind another of these sums' (the caller passes each
// sum of a row its own, and alternates where a row has one alone).
template <int NT>
__device__ __forceinline__ void row_sums(float& a, float& b, float* red) {
  a = group_sum<64>(a);
  b = group_sum<64>(b);
  if constexpr (NT > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      red[2 * w] = a;
      red[2 * w + 1] = b;
    }
    __syncthreads();
    a = red[0];
    b = red[1];
    for (int i = 1; i < NT / 64; ++i) {
      a += red[2 * i];
      b += red[2 * i + 1];
    }
  }
}

__device__ __forceinline__ float sigmoid_x(float z) { return 1.0f / (1.0f + expf(-z)); }

// Squares of large values leave the range of f32 (from 2^64 on, sums of them earlier), and
// with eps = 0 those of small ones lose their digits.  A row (or group) whose mean square
// with eps lies outside 2^-90 .. 2^87 is taken in another unit, 2^72 times as large or as
// small: its values are then at most 2^56 and their squares sum to less than 2^126.  A
// factor of a power of two rounds nothing, and what underflows is below 2^-36 of the mean.
// No row that models have is of that kind: it costs the others one comparison a sum.
__device__ __forceinline__ bool other_unit(float mean_eps) {   // (one comparison: of bits, as of values >= 0)
  constexpr unsigned lo = (127 - 90) << 23, hi = (127 + 87) << 23;
  return __builtin_bit_cast(unsigned, mean_eps) - lo > hi - lo;
}
__device__ __forceinline__ int unit_of(float mean_eps) { return mean_eps < 1.0f ? 72 : -72; }
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (127 + e) << 23); }

// y becomes y r1 and r1 is that of every chunk: over the whole row, or over the lanes of
// the chunk's group
template <typename T, int NT, int NCH>
__device__ __forceinline__ void group_norm(float (*y)[Vec<T>::n], float* r1, const BlockNormArgs& a, float* red) {
  constexpr int V = Vec<T>::n;
  const auto squares = [&](int ch) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < V; ++e) s += y[ch][e] * y[ch][e];
    return s;
  };
  const auto times = [&](int ch, float f) {
#pragma unroll
    for (int e = 0; e < V; ++e) y[ch][e] *= f;
  };
  const float inv = 1.0f / (float)(a.N / a.groups);
  if (a.groups == 1) {
    float s = 0.0f, z = 0.0f;
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) s += squares(ch);
    row_sums<NT>(s, z, red);
    const float mean_eps = s * inv + a.eps;
    float r = 1.0f / sqrtf(mean_eps), f = 1.0f;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(other_unit(mean_eps)) != 0, 0)) {   // (the row's: uniform)
      f = pow2(unit_of(mean_eps));
      s = 0.0f;
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        times(ch, f);
        s += squares(ch);
      }
      if (NT > 64) __syncthreads();   // (the first sums are read)
      row_sums<NT>(s, z, red);
      r = 1.0f / sqrtf(s * inv + a.eps * f * f);
    }
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      times(ch, r);
      r1[ch] = r * f;
    }
  } else {
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      float s = lanes_sum(squares(ch), a.lanes), f = 1.0f;
      const float mean_eps = s * inv + a.eps;
      float r = 1.0f / sqrtf(mean_eps);
      const bool other = other_unit(mean_eps);   // (the group's)
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(other) != 0, 0)) {
        f = other ? pow2(unit_of(mean_eps)) : 1.0f;
        times(ch, f);
        s = lanes_sum(squares(ch), a.lanes);
        r = 1.0f / sqrtf(s * inv + a.eps * f * f);
      }
      times(ch, r);
      r1[ch] = r * f;
    }
  }
}

template <typename T, int NT, int NCH>
__global__ void __launch_bounds__(256, NCH <= 2 ? 6 : 3) carve_block_norm_fwd_kernel(BlockNormArgs a) {
  constexpr int V = Vec<T>::n;
  __shared__ float red[16];
  const int tid = threadIdx.x % NT;
  const long long row = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (256 / NT) + threadIdx.x / NT;
  if (row >= a.rows) return;   // (whole waves; with NT = 256 whole workgroups)
  const T* yp = reinterpret_cast<const T*>(a.y) + row * a.y_stride;
  const T* zp = reinterpret_cast<const T*>(a.gate) + row * a.gate_stride;
  const T* rp = reinterpret_cast<const T*>(a.residual) + row * a.residual_stride;
  float y[NCH][V], z[NCH][V], rs[NCH][V];
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int c0 = (ch * NT + tid) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) y[ch][e] = z[ch][e] = rs[ch][e] = 0.0f;
    if (c0 < a.N) {
      ld_vec(yp + c0, y[ch]);
      if (a.gate) ld_vec(zp + c0, z[ch]);
      if (a.residual) ld_vec(rp + c0, rs[ch]);
    }
  }
  // (with one chunk a thread the parameters are on their way before the sums)
  constexpr bool AHEAD = NCH == 1;
  float pw[V], ps[V], pn[V];
  if (AHEAD && tid * V < a.N) {
    ld_f32(a.weight + tid * V, pw, V);
    if (a.scale) ld_f32(a.scale + tid * V, ps, V);
    if (a.next_weight) ld_f32(a.next_weight + tid * V, pn, V);
  }
  float r1[NCH];
  group_norm<T, NT, NCH>(y, r1, a, red);
  float ss = 0.0f, none = 0.0f;
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int c0 = (ch * NT + tid) * V;
    if (c0 >= a.N) continue;
    float wt[V], sc[V];
    if constexpr (AHEAD) {
#pragma unroll
      for (int e = 0; e < V; ++e) wt[e] = pw[e], sc[e] = ps[e];
    } else {
      ld_f32(a.weight + c0, wt, V);
      if (a.scale) ld_f32(a.scale + c0, sc, V);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float t = y[ch][e] * wt[e];
      if (a.gate) t *= a.act == CARVE_GATE_SILU ? z[ch][e] * sigmoid_x(z[ch][e]) : sigmoid_x(z[ch][e]);
      if (a.scale) t *= sc[e];
      y[ch][e] = a.residual ? a.alpha * rs[ch][e] + t : t;
      ss += y[ch][e] * y[ch][e];
    }
    st_vec(reinterpret_cast<T*>(a.x) + row * a.N + c0, y[ch]);
  }
  if (!a.next_weight) return;   // (uniform)
  row_sums<NT>(ss, none, red + 8);
  const float mean_eps = ss / (float)a.N + a.eps;
  float r2 = 1.0f / sqrtf(mean_eps);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(other_unit(mean_eps)) != 0, 0)) {   // (uniform)
    const float f = pow2(unit_of(mean_eps));
    ss = 0.0f;
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if ((ch * NT + tid) * V >= a.N) continue;
        y[ch][e] *= f;
        ss += y[ch][e] * y[ch][e];
      }
    if (NT > 64) __syncthreads();   // (the first sums are read)
    row_sums<NT>(ss, none, red + 8);
    r2 = 1.0f / sqrtf(ss / (float)a.N + a.eps * f * f);
  }
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int c0 = (ch * NT + tid) * V;
    if (c0 >= a.N) continue;
    float wt[V];
    if constexpr (AHEAD) {
#pragma unroll
      for (int e = 0; e < V; ++e) wt[e] = pn[e];
    } else {
      ld_f32(a.next_weight + c0, wt, V);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) y[ch][e] *= r2 * wt[e];
    st_vec(reinterpret_cast<T*>(a.h) + row * a.N + c0, y[ch]);
  }
}

// Workgroups take rows in turn and keep their share of the parameter gradients in
// registers; their partial rows, [group][3][N] (dweight, dscale, dnext_weight), are
// summed in order by the second launch, so reruns are bitwise identical.  With up to
// eight columns a thread the parameters stay in registers and the next row is on its way
// while this one's sums run (AHEAD).
template <typename T, int NT, int NCH>
__global__ void __launch_bounds__(256) carve_block_norm_bwd_kernel(BlockNormArgs a) {
  constexpr int V = Vec<T>::n;
  constexpr bool AHEAD = NCH * V <= 8;
  __shared__ float red[2][24];
  extern __shared__ __attribute__((aligned(16))) float sacc[];   // NT = 64: [4][N], a gradient at a time
  const int tid = threadIdx.x % NT, rw = threadIdx.x / NT;
  float aw[NCH][V], as[NCH][V], an[NCH][V];
  float pw[AHEAD ? NCH : 1][V], ps[AHEAD ? NCH : 1][V], pn[AHEAD ? NCH : 1][V];
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int c0 = (ch * NT + tid) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      aw[ch][e] = as[ch][e] = an[ch][e] = 0.0f;
      if (AHEAD) pw[AHEAD ? ch : 0][e] = pn[AHEAD ? ch : 0][e] = 0.0f, ps[AHEAD ? ch : 0][e] = 1.0f;
    }
    if (AHEAD && c0 < a.N) {
      ld_f32(a.weight + c0, pw[AHEAD ? ch : 0], V);
      if (a.scale) ld_f32(a.scale + c0, ps[AHEAD ? ch : 0], V);
      if (a.next_weight) ld_f32(a.next_weight + c0, pn[AHEAD ? ch : 0], V);
    }
  }
  const auto weight = [&](int ch, float* f) {
    if constexpr (AHEAD) for (int e = 0; e < V; ++e) f[e] = pw[ch][e];
    else ld_f32(a.weight + (ch * NT + tid) * V, f, V);
  };
  const auto scale = [&](int ch, float* f) {   // (1 where there is none)
    if constexpr (AHEAD) {
      for (int e = 0; e < V; ++e) f[e] = ps[ch][e];
    } else if (a.scale) {
      ld_f32(a.scale + (ch * NT + tid) * V, f, V);
    } else {
      for (int e = 0; e < V; ++e) f[e] = 1.0f;
    }
  };
  const auto next_weight = [&](int ch, float* f) {
    if constexpr (AHEAD) for (int e = 0; e < V; ++e) f[e] = pn[ch][e];
    else ld_f32(a.next_weight + (ch * NT + tid) * V, f, V);
  };
  // the row's chunks as they are in memory
  u32x4_t qy[NCH], qz[NCH], qr[NCH], qx[NCH], qh[NCH];
  const auto load = [&](long long row) {
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      const int c0 = (ch * NT + tid) * V;
      qy[ch] = qz[ch] = qr[ch] = qx[ch] = qh[ch] = u32x4_t{0, 0, 0, 0};
      if (c0 < a.N) {
        const auto at = [&](const void* p, long long stride) {
          return *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const T*>(p) + row * stride + c0);
        };
        qy[ch] = at(a.y, a.y_stride);
        if (a.gate) qz[ch] = at(a.gate, a.gate_stride);
        if (a.residual && a.next_weight) qr[ch] = at(a.residual, a.residual_stride);
        if (a.dx) qx[ch] = at(a.dx, a.N);
        if (a.dh) qh[ch] = at(a.dh, a.N);
      }
    }
  };
  const float invN = 1.0f / (float)a.N, invG = 1.0f / (float)(a.N / a.groups);
  const long long step = (long long)gridDim.x * (256 / NT), row0 = (long long)blockIdx.x * (256 / NT) + rw;
  if (AHEAD && row0 < a.rows) load(row0);
  int turn = 0;
  for (long long row = row0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) load(row);
    float y[NCH][V], z[NCH][V], x[NCH][V], dX[NCH][V], dh[NCH][V], sg[NCH][V];
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      Chunk16<T>::unpack(qy[ch], y[ch]);
      Chunk16<T>::unpack(qz[ch], z[ch]);
      Chunk16<T>::unpack(qr[ch], x[ch]);
      Chunk16<T>::unpack(qx[ch], dX[ch]);
      Chunk16<T>::unpack(qh[ch], dh[ch]);
    }
    if (AHEAD && row + step < a.rows) load(row + step);
    if (a.gate)
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch)
#pragma unroll
        for (int e = 0; e < V; ++e) sg[ch][e] = sigmoid_x(z[ch][e]);
    float r1[NCH];
    group_norm<T, NT, NCH>(y, r1, a, red[turn]);
    // through the next block's norm
    if (a.next_weight) {
      float ss = 0.0f, mx = 0.0f;
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        const int c0 = (ch * NT + tid) * V;
        if (c0 >= a.N) continue;
        float wt[V], sc[V], wn[V];
        weight(ch, wt);
        scale(ch, sc);
        next_weight(ch, wn);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float t = y[ch][e] * wt[e];
          if (a.gate) t *= a.act == CARVE_GATE_SILU ? z[ch][e] * sg[ch][e] : sg[ch][e];
          t *= sc[e];
          x[ch][e] = a.residual ? a.alpha * x[ch][e] + t : t;
          ss += x[ch][e] * x[ch][e];
          mx += dh[ch][e] * wn[e] * x[ch][e];
        }
      }
      row_sums<NT>(ss, mx, red[turn] + 8);
      const float mean_eps = ss * invN + a.eps;
      float r2 = 1.0f / sqrtf(mean_eps), r2f = r2;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(other_unit(mean_eps)) != 0, 0)) {   // (uniform)
        const float f = pow2(unit_of(mean_eps));
        ss = mx = 0.0f;
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
          if ((ch * NT + tid) * V >= a.N) continue;
          float wn[V];
          next_weight(ch, wn);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            x[ch][e] *= f;
            ss += x[ch][e] * x[ch][e];
            mx += dh[ch][e] * wn[e] * x[ch][e];
          }
        }
        if (NT > 64) __syncthreads();   // (the first sums are read)
        row_sums<NT>(ss, mx, red[turn] + 8);
        r2 = 1.0f / sqrtf(ss * invN + a.eps * f * f);
        r2f = r2 * f;
      }
      const float m2 = r2 * r2 * (mx * invN);
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        const int c0 = (ch * NT + tid) * V;
        if (c0 >= a.N) continue;
        float wn[V];
        next_weight(ch, wn);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dX[ch][e] += r2f * (dh[ch][e] * wn[e] - x[ch][e] * m2);
          an[ch][e] += dh[ch][e] * (x[ch][e] * r2);
        }
      }
    }
    float dot[NCH];
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      const int c0 = (ch * NT + tid) * V;
      dot[ch] = 0.0f;
      if (c0 >= a.N) continue;
      if (a.dresidual) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = a.alpha * dX[ch][e];
        st_vec(reinterpret_cast<T*>(a.dresidual) + row * a.N + c0, o);
      }
      float wt[V], sc[V];
      weight(ch, wt);
      scale(ch, sc);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float yh = y[ch][e], nv = yh * wt[e];
        float act = 1.0f, slope = 0.0f;
        if (a.gate) {
          const float s = sg[ch][e];
          act = a.act == CARVE_GATE_SILU ? z[ch][e] * s : s;
          slope = a.act == CARVE_GATE_SILU ? s * (1.0f + z[ch][e] * (1.0f - s)) : s * (1.0f - s);
        }
        as[ch][e] += dX[ch][e] * (nv * act);
        const float dt = dX[ch][e] * sc[e];
        z[ch][e] = dt * nv * slope;      // dgate
        const float dn = dt * act;
        aw[ch][e] += dn * yh;
        dX[ch][e] = dn * wt[e];          // through the weight
        dot[ch] += dX[ch][e] * yh;
      }
      if (a.dgate) st_vec(reinterpret_cast<T*>(a.dgate) + row * a.N + c0, z[ch]);
    }
    if (a.groups == 1) {
      float s = 0.0f, none = 0.0f;
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) s += dot[ch];
      row_sums<NT>(s, none, red[turn] + 16);
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) dot[ch] = s * invG;
    } else {
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) dot[ch] = lanes_sum(dot[ch], a.lanes) * invG;
    }
#pragma unroll
    for (int ch = 0; ch < NCH; ++ch) {
      const int c0 = (ch * NT + tid) * V;
      if (c0 >= a.N) continue;
#pragma unroll
      for (int e = 0; e < V; ++e) dX[ch][e] = r1[ch] * (dX[ch][e] - y[ch][e] * dot[ch]);
      st_vec(reinterpret_cast<T*>(a.dy) + row * a.N + c0, dX[ch]);
    }
  }
  // the workgroup's partial rows: one row of threads writes its share, four waves
  // with a row each are summed in wave order
  float* part = a.partial + (size_t)blockIdx.x * 3 * a.N;
  const auto put = [&](const float (*acc)[V], int which) {
    float* dst = part + (size_t)which * a.N;
    if constexpr (NT == 256) {
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        const int c0 = (ch * NT + tid) * V;
        if (c0 < a.N)
#pragma unroll
          for (int e = 0; e < V; ++e) dst[c0 + e] = acc[ch][e];
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        const int c0 = (ch * NT + tid) * V;
        if (c0 < a.N)
#pragma unroll
          for (int e = 0; e < V; ++e) sacc[rw * a.N + c0 + e] = acc[ch][e];
      }
      __syncthreads();
      for (int col = threadIdx.x; col < a.N; col += 256) {
        float s = sacc[col];
        for (int i = 1; i < 256 / NT; ++i) s += sacc[i * a.N + col];
        dst[col] = s;
      }
    }
  };
  put(aw, 0);
  if (a.dscale) put(as, 1);
  if (a.dnext_weight) put(an, 2);
}

// dweight, dscale, dnext_weight: the partial rows of every workgroup in order, as
// sixteen interleaved sums of a column that are added in order
constexpr int kReduceRows = 16;
__global__ void __launch_bounds__(64 * kReduceRows) carve_block_norm_reduce_kernel(BlockNormArgs a, int nparts) {
  __shared__ float red[kReduceRows][64];
  float* out = blockIdx.y == 0 ? a.dweight : blockIdx.y == 1 ? a.dscale : a.dnext_weight;
  if (!out) return;   // (uniform)
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + tx;
  const size_t step = 3 * (size_t)a.N;
  float s = 0.0f;
  if (col < a.N) {
    const float* p = a.partial + (size_t)blockIdx.y * a.N + col;
    int i = ty;
    for (; i + 3 * kReduceRows < nparts; i += 4 * kReduceRows) {
      const float a0 = p[i * step], a1 = p[(i + kReduceRows) * step];
      const float a2 = p[(i + 2 * kReduceRows) * step], a3 = p[(i + 3 * kReduceRows) * step];
      s += a0;
      s += a1;
      s += a2;
      s += a3;
    }
    for (; i < nparts; i += kReduceRows) s += p[i * step];
  }
  red[ty][tx] = s;
  __syncthreads();
  if (ty == 0 && col < a.N) {
    float t = red[0][tx];
    for (int y = 1; y < kReduceRows; ++y) t += red[y][tx];
    out[col] = t;
  }
}

constexpr unsigned kBlockNormGridX = 1u << 22;
// threads of a row and 16-byte chunks of a thread: one wave up to two chunks a lane
template <typename T>
bool wave_rows(int N) { return N <= 2 * 64 * Vec<T>::n; }

template <typename T, int NT, int NCH>
int fwd_t(const BlockNormArgs& a, hipStream_t s) {
  const long long nwg = (a.rows + 256 / NT - 1) / (256 / NT);
  // (a grid dimension has less than 2^32 threads)
  const unsigned nx = nwg < kBlockNormGridX ? (unsigned)nwg : kBlockNormGridX, ny = (unsigned)((nwg + nx - 1) / nx);
  hipLaunchKernelGGL((carve_block_norm_fwd_kernel<T, NT, NCH>), dim3(nx, ny), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int NT, int NCH>
int bwd_t(const BlockNormArgs& a, int nwg, hipStream_t s) {
  const size_t lds = NT == 64 ? (size_t)4 * a.N * sizeof(float) : 0;
  hipLaunchKernelGGL((carve_block_norm_bwd_kernel<T, NT, NCH>), dim3((unsigned)nwg), dim3(256), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T>
int fwd_d(const BlockNormArgs& a, hipStream_t s) {
  const int nch = (a.N + 256 * Vec<T>::n - 1) / (256 * Vec<T>::n);
  if (wave_rows<T>(a.N)) return a.N <= 64 * Vec<T>::n ? fwd_t<T, 64, 1>(a, s) : fwd_t<T, 64, 2>(a, s);
  if (nch <= 1) return fwd_t<T, 256, 1>(a, s);
  if (nch <= 2) return fwd_t<T, 256, 2>(a, s);
  if constexpr (sizeof(T) == 4)
    if (nch > 4) return fwd_t<T, 256, 8>(a, s);
  return fwd_t<T, 256, 4>(a, s);
}
template <typename T>
int bwd_d(const BlockNormArgs& a, int nwg, hipStream_t s) {
  const int nch = (a.N + 256 * Vec<T>::n - 1) / (256 * Vec<T>::n);
  if (wave_rows<T>(a.N)) return a.N <= 64 * Vec<T>::n ? bwd_t<T, 64, 1>(a, nwg, s) : bwd_t<T, 64, 2>(a, nwg, s);
  if (nch <= 1) return bwd_t<T, 256, 1>(a, nwg, s);
  if (nch <= 2) return bwd_t<T, 256, 2>(a, nwg, s);
  if constexpr (sizeof(T) == 4)
    if (nch > 4) return bwd_t<T, 256, 8>(a, nwg, s);
  return bwd_t<T, 256, 4>(a, nwg, s);
}

}  // namespace

int block_norm_groups(long long rows, int N, int dtype) {
  const bool wave = dtype == CARVE_BF16 ? wave_rows<bf16_t>(N) : wave_rows<float>(N);
  const long long need = wave ? (rows + 3) / 4 : rows;
  return (int)(need < kBlockNormGroups ? need : kBlockNormGroups);
}

int launch_block_norm_fwd(const BlockNormArgs& a, int dtype, hipStream_t s) {
  return dtype == CARVE_BF16 ? fwd_d<bf16_t>(a, s) : fwd_d<float>(a, s);
}

int launch_block_norm_bwd(const BlockNormArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
  const int nwg = block_norm_groups(a.rows, a.N, dtype);
  const int st = dtype == CARVE_BF16 ? bwd_d<bf16_t>(a, nwg, s) : bwd_d<float>(a, nwg, s);
  if (st) return st;
  mark(s);
  hipLaunchKernelGGL(carve_block_norm_reduce_kernel, dim3((a.N + 63) / 64, 3), dim3(64 * kReduceRows), 0, s, a, nwg);
  mark(s);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}

}  // namespace carve
