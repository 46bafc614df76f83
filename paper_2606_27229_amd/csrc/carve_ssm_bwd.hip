// carve_ssm_bwd.hip -- the chunked selective state space scan, backward for loss <dY, y> +
// <dS_T, S_T>.  Per chunk, with its start state S (kept by the forward), the gradient E of
// its end state, Q_ij = dy_i . x_j and E_t = e^{G_C - G_t}:
//   E <- e^{G_C} E + dY^T (e^G C)                                   (the chain)
//   dx_j = d_j (sum_{i >= j} L_ij (C_i . B_j) dy_i + E_j E B_j) + D dy_j
//   dB_j = d_j (sum_{i >= j} L_ij Q_ij C_i + E_j E^T x_j)           (summed over a group's heads)
//   dC_i = sum_{j <= i} L_ij d_j Q_ij B_j + e^{G_i} S^T dy_i        (likewise)
//   da_t = sum_{i >= t} e^{G_i} dy_i . S C_i + sum_{i >= t > j} M_ij d_j
//          + sum_{j < t} d_j E_j x_j . E B_j + e^{G_C} <E, S>,   M_ij = L_ij (C_i . B_j) Q_ij
//   dd_t = A da_t + sum_{i >= t} M_it + E_t x_t . E B_t,  ddt_t = dd_t softplus'(dt_t + dt_bias)
//   dA = sum d_t da_t,  ddt_bias = sum ddt_t,  dD = sum dy_t . x_t
// (da_t is summed over what the decay at t multiplies, and nothing else: as a suffix sum of
// gradients of G, what should cancel under hard decays would leave its rounding.)
// Launches: the chain of E (carve_ssm_fwd.hip), every chunk's gradients, the sums.
#include "carve_ssm.h"

namespace carve {
namespace {

constexpr int kPw = 32;   // value columns of a turn
constexpr int kPart = 4;  // floats of a (chunk, head) in SsmArgs::part

// One workgroup a chunk, group and share of the group's heads; wave w owns token tile w, as
// i of dC and as j of dB and dx (their work adds up to the same for every wave).  dB and dC
// stay in registers over the heads; a head comes in turns of 32 value columns, in which
// everything but L is linear: x, dy and the rows of S and E, loaded straight into LDS.
// Bound by HBM, the states S and E above all (N x P floats each, a chunk and head); two
// workgroups a compute unit load and compute by turns (bf16).
template <typename T, int N>
struct GradLds {
  typedef SsmRows<T, N, kSsmC> KR;     // B, C
  typedef SsmRows<T, kPw, kSsmC> VR;   // x, dy
  typedef SsmRows<T, N, kPw> SR;       // a plane of S or E
  static constexpr int state = SR::bytes * SsmState<T>::planes;
  static constexpr int B = 0, C = KR::bytes, X = 2 * KR::bytes, dY = X + VR::bytes, S = dY + VR::bytes, E = S + state;
  static constexpr int scal = E + state, sum = scal + kSmFloats * 4;
  // r_t, d_t E_t x.EB, their column sums, da's rectangles by wave, dy.x; <E, S> by wave
  static constexpr int total = sum + (8 * kSsmC + 4) * 4;
};

template <typename T, int N>
__device__ __forceinline__ Fi<T, kNear> state_tr(const char* lds, int j, int g, int c) {
  typedef typename GradLds<T, N>::SR SR;
  Fi<T, kNear> f;
#pragma unroll
  for (int i = 0; i < SsmState<T>::planes; ++i) f.x[i] = SR::tr32(lds + i * SR::bytes, 0, j, g, c);
  return f;
}
template <typename T, int N>
__device__ __forceinline__ Fi<T, kNear> state_nat(const char* lds, int i, int p, int g, int c) {
  typedef typename GradLds<T, N>::SR SR;
  Fi<T, kNear> f;
#pragma unroll
  for (int u = 0; u < SsmState<T>::planes; ++u) f.x[u] = SR::nat(lds + u * SR::bytes, i, p, g, c);
  return f;
}
__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]; }
__device__ __forceinline__ f32x4 four(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
// over the four lanes of a column
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <typename T, int N>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) carve_ssm_grad_kernel(SsmArgs a) {
  typedef GradLds<T, N> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef typename L::SR SR;
  constexpr int NP = N / 32, NT = N / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* sc = reinterpret_cast<float*>(smem + L::scal);
  float* sR = reinterpret_cast<float*>(smem + L::sum);
  float *sE = sR + kSsmC, *sM = sE + kSsmC, *sRect = sM + kSsmC, *sDiag = sRect + 4 * kSsmC, *sES = sDiag + kSsmC;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int slot = blockIdx.x, grp = blockIdx.y, part = blockIdx.z;
  const int rep = a.H / a.G, h0 = grp * rep + (int)((long long)rep * part / a.splits),
            h1 = grp * rep + (int)((long long)rep * (part + 1) / a.splits);
  const SsmSeq q = ssm_find(a, slot, kSsmC);
  const int ch = slot - ssm_slot0(a, q, kSsmC);
  if (ch < 0 || (long long)ch * kSsmC >= q.len) {   // a slot of no chunk
    for (int i = tid; i < (h1 - h0) * kPart; i += 256) a.part[((size_t)slot * a.H + h0) * kPart + i] = 0.0f;
    return;
  }
  const int first = q.first + ch * kSsmC, len = min(kSsmC, q.len - ch * kSsmC);
  const size_t row0 = (size_t)q.batch * a.T + first, pn = (size_t)a.P * N;
  const int tok = 16 * w + c;
  f32x4 dB[NT], dC[NT], CB[4];
#pragma unroll
  for (int j = 0; j < NT; ++j) dB[j] = dC[j] = zero4();
#pragma unroll
  for (int i = 0; i < 4; ++i) CB[i] = zero4();
  KR::template dma<4>(smem + L::B, reinterpret_cast<const T*>(a.Bm) + q.batch * a.bs[0] + first * a.bs[1] + grp * a.bs[2],
                      (int)(a.bs[1] * sizeof(T)), len, w, lane);
  KR::template dma<4>(smem + L::C, reinterpret_cast<const T*>(a.Cm) + q.batch * a.cs[0] + first * a.cs[1] + grp * a.cs[2],
                      (int)(a.cs[1] * sizeof(T)), len, w, lane);
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    const T* x = reinterpret_cast<const T*>(a.x) + q.batch * a.xs[0] + first * a.xs[1] + h * a.xs[2];
    const T* dy = reinterpret_cast<const T*>(a.dy) + (row0 * a.H + h) * a.P;
    T* dx = reinterpret_cast<T*>(a.dx) + (row0 * a.H + h) * a.P;
    const char* S = a.S_chunks + ((size_t)slot * a.H + h) * pn * 4;
    const char* E = a.E_chunks + ((size_t)slot * a.H + h) * pn * 4;
    const float skip = a.D ? a.D[h] : 0.0f, bias = a.dt_bias ? a.dt_bias[h] : 0.0f, A = a.A[h];
    float raw = 0.0f;
    if (w == 0 && lane < len) raw = (float)(reinterpret_cast<const T*>(a.dt) + q.batch * a.ds[0] + h)[(first + lane) * a.ds[1]];
    f32x4 QT[4], Q[4];       // Q of tile w's dy (columns) and of its x
    Fi<T, kNear> Lf[2];      // L C B^T, rows i, columns j of tile w
    f32x4 LC[4];
    float r = 0.0f, ex = 0.0f, es = 0.0f, dj = 0.0f, endj = 0.0f, gami = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) QT[i] = Q[i] = LC[i] = zero4();
#pragma unroll 1
    for (int p0 = 0; p0 < a.P; p0 += kPw) {
      __syncthreads();   // what the turn before read may be overwritten
      VR::template dma<4>(smem + L::X, x + p0, (int)(a.xs[1] * sizeof(T)), len, w, lane);
      VR::template dma<4>(smem + L::dY, dy + p0, (int)((long long)a.H * a.P * sizeof(T)), len, w, lane);
#pragma unroll
      for (int u = 0; u < SsmState<T>::planes; ++u) {
        const size_t at = (u * pn + (size_t)p0 * N) * sizeof(T);
        SR::template dma<4>(smem + L::S + u * SR::bytes, S + at, SR::RB, kPw, w, lane);
        SR::template dma<4>(smem + L::E + u * SR::bytes, E + at, SR::RB, kPw, w, lane);
      }
      if (p0 == 0 && w == 0) ssm_scalars(raw, lane < len, bias, A, a.softplus, lane, sc);
      vm_wait_all();
      __syncthreads();
      if (p0 == 0) {
        dj = sc[kSmD * kSsmC + tok], endj = sc[kSmEnd * kSsmC + tok], gami = sc[kSmGam * kSsmC + tok];
        if (h == h0) {
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const Fr<T> fb = KR::nat(smem + L::B, w, p, g, c);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i >= w) CB[i] = mma<T>(KR::nat(smem + L::C, i, p, g, c), fb, CB[i]);
          }
        }
        // L C B^T below the diagonal
        const float Gh = sc[kSmGh * kSsmC + tok], Gl = sc[kSmGl * kSsmC + tok];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i < w) continue;   // (uniform)
          const f32x4 gh = four(sc + kSmGh * kSsmC + 16 * i + 4 * g), gl = four(sc + kSmGl * kSsmC + 16 * i + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = 16 * i + 4 * g + e;
            LC[i][e] = t >= tok && t < len ? decay_exp((gh[e] - Gh) + (gl[e] - Gl)) * CB[i][e] : 0.0f;
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) Lf[s] = to_fi<T, kNear>(LC[2 * s], LC[2 * s + 1]);
      }
      const Fr<T> fx = VR::nat(smem + L::X, w, 0, g, c), fy = VR::nat(smem + L::dY, w, 0, g, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= w) Q[i] = mma<T>(VR::nat(smem + L::dY, i, 0, g, c), fx, Q[i]);
        if (i <= w) QT[i] = mma<T>(VR::nat(smem + L::X, i, 0, g, c), fy, QT[i]);
      }
      // dC and dB of the states, a tile of n at a time
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const f32x4 u = mma<T>(state_tr<T, N>(smem + L::S, j, g, c), fy, zero4()) * gami;
        dC[j] += u;
        r += dot4(u, Quad<T>::f32(KR::quad(smem + L::C, w, j, g, c)));
        const f32x4 v = mma<T>(state_tr<T, N>(smem + L::E, j, g, c), fx, zero4());
        dB[j] += v * (dj * endj);
      }
      // dx: two tiles of p
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x4 u = zero4(), z = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) u = mma<T>(state_nat<T, N>(smem + L::E, t, p, g, c), KR::nat(smem + L::B, w, p, g, c), u);
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (s >= w / 2) z = mma<T>(VR::tr32(smem + L::dY, s, t, g, c), Lf[s], z);
        u *= endj;
        ex += dot4(u, Quad<T>::f32(VR::quad(smem + L::X, w, t, g, c)));
        const f32x4 o = (u + z) * dj + Quad<T>::f32(VR::quad(smem + L::dY, w, t, g, c)) * skip;
        if (tok < len) Quad<T>::st(dx + (size_t)tok * a.H * a.P + p0 + 16 * t + 4 * g, Quad<T>::cvt(o));
      }
      // <E, S>, by pieces of 16 bytes (both lie alike in LDS)
      for (int i = tid; i < SR::bytes / 16; i += 256) {
        float e[Chunk16<T>::N], s[Chunk16<T>::N];
#pragma unroll
        for (int u = 0; u < Chunk16<T>::N; ++u) e[u] = s[u] = 0.0f;
#pragma unroll
        for (int pl = SsmState<T>::planes - 1; pl >= 0; --pl) {
          float fe[Chunk16<T>::N], fs[Chunk16<T>::N];
          Chunk16<T>::unpack(*reinterpret_cast<const u32x4_t*>(smem + L::E + pl * SR::bytes + 16 * i), fe);
          Chunk16<T>::unpack(*reinterpret_cast<const u32x4_t*>(smem + L::S + pl * SR::bytes + 16 * i), fs);
#pragma unroll
          for (int u = 0; u < Chunk16<T>::N; ++u) e[u] += fe[u], s[u] += fs[u];
        }
#pragma unroll
        for (int u = 0; u < Chunk16<T>::N; ++u) es += e[u] * s[u];
      }
    }
    // what pairs of tokens add: rows j (dC) and rows i (dB) against the wave's tile
    {
      const float Gh = sc[kSmGh * kSsmC + tok], Gl = sc[kSmGl * kSsmC + tok];
      f32x4 V[4], M[4];
      float cm = 0.0f, diag = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        V[i] = M[i] = zero4();
        const f32x4 gh = four(sc + kSmGh * kSsmC + 16 * i + 4 * g), gl = four(sc + kSmGl * kSsmC + 16 * i + 4 * g);
        const f32x4 d = four(sc + kSmD * kSsmC + 16 * i + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = 16 * i + 4 * g + e;
          if (i >= w) {
            const bool on = t >= tok && t < len;
            V[i][e] = on ? decay_exp((gh[e] - Gh) + (gl[e] - Gl)) * dj * Q[i][e] : 0.0f;
            M[i][e] = on ? LC[i][e] * Q[i][e] : 0.0f;
            cm += M[i][e];
            M[i][e] *= dj;
            if (t == tok) diag = Q[i][e];
          }
          if (i <= w) QT[i][e] = t <= tok ? decay_exp((Gh - gh[e]) + (Gl - gl[e])) * d[e] * QT[i][e] : 0.0f;
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s <= w / 2) {
          const Fi<T, kNear> f = to_fi<T, kNear>(QT[2 * s], QT[2 * s + 1]);
#pragma unroll
          for (int j = 0; j < NT; ++j) dC[j] = mma<T>(KR::tr32(smem + L::B, s, j, g, c), f, dC[j]);
        }
        if (s >= w / 2) {
          const Fi<T, kNear> f = to_fi<T, kNear>(V[2 * s], V[2 * s + 1]);
#pragma unroll
          for (int j = 0; j < NT; ++j) dB[j] = mma<T>(KR::tr32(smem + L::C, s, j, g, c), f, dB[j]);
        }
      }
      // sums of M over i >= t and j < t: suffix sums down each column, then along rows
      float carry = 0.0f;
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        f32x4 suf = zero4();
        if (i >= w) {   // (uniform)
          suf[3] = M[i][3];
#pragma unroll
          for (int e = 2; e >= 0; --e) suf[e] = M[i][e] + suf[e + 1];
          float in = suf[0];
          const float n1 = __shfl(in, (lane + 16) & 63);
          in += g < 3 ? n1 : 0.0f;
          const float n2 = __shfl(in, (lane + 32) & 63);
          in += g < 2 ? n2 : 0.0f;
          const float behind = __shfl(in, (lane + 16) & 63), whole = __shfl(in, c);
          const float more = carry + (g < 3 ? behind : 0.0f);
#pragma unroll
          for (int e = 0; e < 4; ++e) suf[e] = 16 * i + 4 * g + e > tok ? suf[e] + more : 0.0f;
          carry += whole;
        }
        const float rect = row_sum4(suf, c);
        if (c < 4) sRect[w * kSsmC + 16 * i + 4 * g + c] = rect;
      }
      r = col_sum(r), ex = col_sum(ex), cm = col_sum(cm), diag = col_sum(diag);
      es = group_sum<64>(es);
      if (g == 0) sR[tok] = r, sE[tok] = ex, sM[tok] = cm, sDiag[tok] = diag;
      if (lane == 0) sES[w] = es;
    }
    __syncthreads();
    if (w == 0) {   // (the next head's turns write these places behind their first barriers)
      const bool in = lane < len;
      const float d = sc[kSmD * kSsmC + lane], e = sE[lane];
      float suf = in ? sR[lane] : 0.0f, pre = in ? d * e : 0.0f;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) {
        const float dn = __shfl_down(suf, s), up = __shfl_up(pre, s);
        if (lane + s < 64) suf += dn;
        if (lane >= s) pre += up;
      }
      const float before = __shfl_up(pre, 1);
      const float es4 = sc[kSmWhole] * ((sES[0] + sES[1]) + (sES[2] + sES[3]));
      const float rect = (sRect[lane] + sRect[kSsmC + lane]) + (sRect[2 * kSsmC + lane] + sRect[3 * kSsmC + lane]);
      const float da = suf + (lane > 0 ? before : 0.0f) + rect + es4;
      float dd = A * da + (sM[lane] + e);
      if (a.softplus) {
        const float z = raw + bias, ez = expf(-fabsf(z));
        dd *= (z >= 0.0f ? 1.0f : ez) / (1.0f + ez);
      }
      if (in) reinterpret_cast<T*>(a.ddt)[(row0 + lane) * a.H + h] = (T)dd;
      const float sa = group_sum<64>(in ? d * da : 0.0f), sb = group_sum<64>(in ? dd : 0.0f), sd = group_sum<64>(in ? sDiag[lane] : 0.0f);
      if (lane == 0) *reinterpret_cast<f32x4*>(a.part + ((size_t)slot * a.H + h) * kPart) = f32x4{sa, sb, sd, 0.0f};
    }
  }
  if (tok < len) {
    const size_t at = ((row0 + tok) * a.G + grp) * N + 4 * g;
    if (a.splits == 1) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        Quad<T>::st(reinterpret_cast<T*>(a.dBm) + at + 16 * j, Quad<T>::cvt(dB[j]));
        Quad<T>::st(reinterpret_cast<T*>(a.dCm) + at + 16 * j, Quad<T>::cvt(dC[j]));
      }
    } else {
      const size_t all = (size_t)(a.offsets ? 1 : a.nseq) * a.T * a.G * N;
      float* out = a.dBp + (size_t)part * 2 * all + at;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<f32x4*>(out + 16 * j) = dB[j];
        *reinterpret_cast<f32x4*>(out + all + 16 * j) = dC[j];
      }
    }
  }
}

// dB, dC: the shares of the heads, in order; rows of no sequence are left as they were
template <typename T>
__global__ void __launch_bounds__(256) carve_ssm_sum_kernel(SsmArgs a) {
  const size_t per = (size_t)a.G * a.N, rows = (size_t)(a.offsets ? 1 : a.nseq) * a.T, all = rows * per;
  const size_t at = (((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= all) return;
  if (a.offsets) {
    const int row = (int)(at / per), n = packed_find(a.offsets, a.nseq, a.T, row);
    int first, end;
    packed_seq(a.offsets, n, a.T, first, end);
    if (row < first || row >= end) return;
  }
  f32x4 b = zero4(), d = zero4();
  for (int i = 0; i < a.splits; ++i) {
    b += *reinterpret_cast<const f32x4*>(a.dBp + (size_t)i * 2 * all + at);
    d += *reinterpret_cast<const f32x4*>(a.dBp + ((size_t)i * 2 + 1) * all + at);
  }
  Quad<T>::st(reinterpret_cast<T*>(a.dBm) + at, Quad<T>::cvt(b));
  Quad<T>::st(reinterpret_cast<T*>(a.dCm) + at, Quad<T>::cvt(d));
}

// dA, ddt_bias, dD of a head: its chunks' shares, in a fixed order, in 64 bits
__global__ void __launch_bounds__(256) carve_ssm_head_kernel(SsmArgs a) {
  __shared__ double red[3][256];
  const int h = blockIdx.x, tid = threadIdx.x;
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = tid; i < a.nslots; i += 256) {
    const f32x4 v = four(a.part + ((size_t)i * a.H + h) * kPart);
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] += (double)v[k];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) red[k][tid] = s[k];
  for (int n = 128; n > 0; n /= 2) {
    __syncthreads();
    if (tid < n)
#pragma unroll
      for (int k = 0; k < 3; ++k) red[k][tid] += red[k][tid + n];
  }
  if (tid == 0) {
    a.dA[h] = (float)red[0][0];
    if (a.ddt_bias) a.ddt_bias[h] = (float)red[1][0];
    if (a.dD) a.dD[h] = (float)red[2][0];
  }
}

int launched() { return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP; }

template <typename T, int N>
int launch_t(const SsmArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  constexpr int lds = GradLds<T, N>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_ssm_grad_kernel<T, N>;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CARVE_ERR_HIP;
  hipLaunchKernelGGL(kern, dim3(a.nslots, a.G, a.splits), dim3(256), lds, s, a);
  int st = launched();
  if (st) return st;
  mark(s);
  if (a.splits > 1) {
    const size_t blocks = ((size_t)(a.offsets ? 1 : a.nseq) * a.T * a.G * a.N / 4 + 255) / 256;
    const unsigned gx = blocks < (1 << 20) ? (unsigned)blocks : 1 << 20;
    hipLaunchKernelGGL(carve_ssm_sum_kernel<T>, dim3(gx, (unsigned)((blocks + gx - 1) / gx)), dim3(256), 0, s, a);
    st = launched();
    if (st) return st;
    mark(s);
  }
  hipLaunchKernelGGL(carve_ssm_head_kernel, dim3(a.H), dim3(256), 0, s, a);
  st = launched();
  mark(s);
  return st;
}

}  // namespace

int launch_ssm_bwd(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
  const int st = launch_ssm_spans_rev(a, dtype, s, mark);
  if (st) return st;
  const bool h = dtype == CARVE_BF16;
  switch (a.N) {
    case 32: return h ? launch_t<bf16_t, 32>(a, s, mark) : launch_t<float, 32>(a, s, mark);
    case 64: return h ? launch_t<bf16_t, 64>(a, s, mark) : launch_t<float, 64>(a, s, mark);
    case 128: return h ? launch_t<bf16_t, 128>(a, s, mark) : launch_t<float, 128>(a, s, mark);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}

}  // namespace carve
