// carve_gdr_bwd.hip -- the chunked gated delta rule, backward for loss <dO, o> +
// <dS_T, S_T>.  With dO' = scale dO, E_t = e^{G_C - G_t} and, per chunk, the start
// state S (kept by the forward) and the gradient dS of the end state:
//   dU = P^T dO' + E K dS^T,  dR = T^T dU,  dV = beta dR
//   dS <- e^{G_C} dS + dO'^T (e^G Q) - (beta e^G dR)^T K           (the chain)
//   dP = dO' U^T (j <= i),  dA = - dR U^T (j < i),  M = beta D dA
//   dQ = e^G dO' S + (D dP) K
//   dK = (D dP)^T Q + M K + M^T K + E U dS - beta e^G dR S
//   dbeta_t = dR_t.V_t - e^{G_t} k_t.(dR S)_t + sum_j dA_tj D_tj k_t.k_j
//   dG_t = q_t.(e^G dO' S)_t - k_t.(beta e^G dR S)_t - k_t.(E U dS)_t
//          + row sums - column sums of dP P + dA A
//   dG_C += e^{G_C} <dS, S> + sum_t k_t.(E U dS)_t,  dg_t = sum_{i >= t} dG_i
// Three launches: the triangles (carve_gdr_prep_kernel), the chain of state
// gradients, then every chunk's gradients at once.
#include "carve_gdr.h"

namespace carve {
namespace {

// ---------------------------------------------------------------------------------
// The chain of state gradients, the mirror of the forward's (carve_gdr_chain_kernel): a
// wave keeps dS^T[j][v] of 16 value columns in registers and runs the chunks from the
// last to the first; dS of every chunk's end goes to dS_chunks.
template <typename T, int DK, int NW>
struct BChainLds {
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, 16 * NW> VR;
  static constexpr int img = GdrWs<T>::bBytes - GdrWs<T>::bPt;   // P^T, T^T, scalars
  static constexpr int K = 0, Q = K + KR::bytes, O = Q + KR::bytes, I = O + VR::bytes;
  static constexpr int one = I + img;
  static constexpr int nbuf = 2 * one <= 160 * 1024 ? 2 : 1;
  static constexpr int total = nbuf * one;
};

template <typename T, int DK, int NW>
__global__ void __launch_bounds__(64 * NW, 1) carve_gdr_bchain_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef BChainLds<T, DK, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int ns = a.Dv / (16 * NW), idx = blockIdx.x;
  const int head = idx / (8 * ns) * 8 + idx % 8, slice = idx / 8 % ns;
  if (head >= a.nseq * a.Hv) return;
  const int n = head / a.Hv, hv = head % a.Hv, hk = hv / (a.Hv / a.Hk);
  const int vs = 16 * NW * slice, v0 = vs + 16 * w;
  const GdrSeq sq = gdr_seq(a, n);
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + sq.t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + sq.t0 * a.ks[1] + hk * a.ks[2];
  const T* dO = reinterpret_cast<const T*>(a.dO) + (((size_t)sq.batch * a.T + sq.t0) * a.Hv + hv) * a.Dv + vs;
  const size_t ors = (size_t)a.Hv * a.Dv;
  const size_t sm = (size_t)a.Dv * DK, soff = (size_t)(v0 + c) * DK + 4 * g;
  const int nch = (sq.len + kGdrC - 1) / kGdrC;

  const auto load = [&](int ch) {
    char* buf = smem + (L::nbuf == 2 ? (ch & 1) * L::one : 0);
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    KR::dma(buf + L::K, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, w, NW, lane);
    dma_flat(buf + L::I, a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per + WS::bPt, L::img, w, NW, lane);
    VR::dma(buf + L::O, dO + t0 * ors, (int)(ors * sizeof(T)), len, w, NW, lane);
    KR::dma(buf + L::Q, q + t0 * a.qs[1], (int)(a.qs[1] * sizeof(T)), len, w, NW, lane);
  };
  if (L::nbuf == 2 && nch > 0) load(nch - 1);

  f32x4 S[2 * NP];
#pragma unroll
  for (int j = 0; j < 2 * NP; ++j)
    S[j] = a.dS_T ? *reinterpret_cast<const f32x4*>(a.dS_T + (size_t)head * sm + soff + 16 * j) : zero4();
  for (int ch = nch - 1; ch >= 0; --ch) {
    const char* buf = smem + (L::nbuf == 2 ? (ch & 1) * L::one : 0);
    if constexpr (L::nbuf == 1) {
      __syncthreads();
      load(ch);
    }
    vm_wait_all();
    __syncthreads();
    if (L::nbuf == 2 && ch > 0) load(ch - 1);
    {
      float* s = a.dS_chunks + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * sm + soff;
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    const char* img = buf + L::I;
    const float* scal = reinterpret_cast<const float*>(img + (WS::bScal - WS::bPt));
    const int len = sq.len - ch * kGdrC;
    // dO[t][v] of this wave's columns, zeros behind the last token
    Fr<T> of[2] = {VR::tr32(buf + L::O, 0, w, g, c), VR::tr32(buf + L::O, 1, w, g, c)};
    if (len < kGdrC)
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (32 * s + 4 * g + e >= len) of[s].a[e] = (T)0.0f;
          if (32 * s + 16 + 4 * g + e >= len) of[s].b[e] = (T)0.0f;
        }
    Fi<T, kExact> Sf[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) Sf[p] = to_fi<T, kExact>(S[2 * p], S[2 * p + 1]);
    // dU = P^T dO' + E K dS^T
    f32x4 U[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 x = zero4(), y = zero4();
#pragma unroll
      for (int p = 0; p < NP; ++p) y = mma<T>(KR::nat(buf + L::K, i, p, g, c), Sf[p], y);
#pragma unroll
      for (int s = i / 2; s < 2; ++s) x = mma<T>(ld_img<T, kExact>(img, img_upper(i, s), lane), of[s], x);
      const f32x4 end = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
      U[i] = x * a.scale + y * end;
    }
    const Fi<T, kExact> Uf[2] = {to_fi<T, kExact>(U[0], U[1]), to_fi<T, kExact>(U[2], U[3])};
    // - beta e^G dR, dR = T^T dU, and e^G dO'
    f32x4 R[4], od[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 x = zero4();
#pragma unroll
      for (int s = i / 2; s < 2; ++s)
        x = mma<T>(ld_img<T, kExact>(img + (WS::bTt - WS::bPt), img_upper(i, s), lane), Uf[s], x);
      const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
      const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
      R[i] = -(x * gam * be);
      od[i] = Quad<T>::f32(i % 2 ? of[i / 2].b : of[i / 2].a) * (gam * a.scale);
    }
    const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(R[0], R[1]), to_fi<T, kExact>(R[2], R[3])};
    const Fi<T, kExact> Of[2] = {to_fi<T, kExact>(od[0], od[1]), to_fi<T, kExact>(od[2], od[3])};
    const float gend = scal[kScGam * kGdrC + kGdrC - 1];
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) {
      S[j] *= gend;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        S[j] = mma<T>(KR::tr32(buf + L::Q, s, j, g, c), Of[s], S[j]);
        S[j] = mma<T>(KR::tr32(buf + L::K, s, j, g, c), Rf[s], S[j]);
      }
    }
  }
  if (a.dS0) {
    float* s = a.dS0 + (size_t)head * sm + soff;
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
  }
}

// ---------------------------------------------------------------------------------
// Gradients of one chunk and key head (its value heads one after another, dq and dk
// summed in registers).  Eight waves, per value head and block of 128 value columns:
//   1. wave w: value columns 16 w ..: U and dR again from S and dS (both read here
//      once as B operands), into LDS transposed; dV; <dS, S>; dR.V
//   2. products over the value columns: dP and dA, tile by tile (lower tiles only),
//      and dO' S, U dS, dR S for the wave's key columns
// then, all columns done, D dP and M through LDS into dQ and dK.
constexpr int kVB = 128;   // value columns of a block

// [columns][tokens] tiles of an f32 intermediate in LDS
template <typename T>
struct InterT {
  static constexpr int LD = sizeof(T) == 2 ? kGdrC + 16 : kGdrC + 4;
  static __host__ __device__ constexpr int bytes(int cols, int n) { return cols * LD * (sizeof(T) == 2 ? 2 * n : 4); }
  // the four tokens 16 i + 4 g .. of column col, in N pieces
  template <int N>
  static __device__ __forceinline__ void put(char* m, int cols, int col, int i, int g, f32x4 x) {
    T* p = reinterpret_cast<T*>(m) + col * LD + 16 * i;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int y = 0; y < N; ++y) {
        const typename Quad<T>::q h = Quad<T>::cvt(x);
        Quad<T>::st(p + y * cols * LD + ((4 * g) ^ qswz<T>(col)), h);
        x -= Quad<T>::f32(h);
      }
    } else {
      Quad<T>::st(p + 4 * g, x);
    }
  }
  // lane (g, c): token 16 i + c, columns col0 + 4 g + e and col0 + 16 + 4 g + e
  template <int N>
  static __device__ __forceinline__ Fi<T, N> tok(const char* m, int cols, int i, int col0, int g, int c) {
    const T* p = reinterpret_cast<const T*>(m);
    Fi<T, N> f;
#pragma unroll
    for (int y = 0; y < (sizeof(T) == 2 ? N : 1); ++y) {
      f.x[y].a = Quad<T>::ld_tr_sw(p + y * cols * LD, LD, col0, 16 * i, g, c);
      f.x[y].b = Quad<T>::ld_tr_sw(p + y * cols * LD, LD, col0 + 16, 16 * i, g, c);
    }
    return f;
  }
  // lane (g, c): column col0 + c, tokens 32 s + 4 g + e and 32 s + 16 + 4 g + e
  template <int N>
  static __device__ __forceinline__ Fi<T, N> col(const char* m, int cols, int col0, int s, int g, int c) {
    const T* p = reinterpret_cast<const T*>(m) + (col0 + c) * LD + 32 * s + ((4 * g) ^ qswz<T>(col0 + c));
    Fi<T, N> f;
#pragma unroll
    for (int y = 0; y < (sizeof(T) == 2 ? N : 1); ++y) {
      f.x[y].a = Quad<T>::ld(p + y * cols * LD);
      f.x[y].b = Quad<T>::ld(p + y * cols * LD + 16);
    }
    return f;
  }
};

template <typename T>
struct GradLds {
  static constexpr int U = 0;
  static constexpr int R = U + InterT<T>::bytes(kVB, kExact);
  static constexpr int red = R + InterT<T>::bytes(kVB, kExact);
  static constexpr int W = 0;                                      // (D dP)^T: [j][i], over U
  static constexpr int M = W + InterT<T>::bytes(kGdrC, kNear);     // M^T: [j][i]
  // sums over values or keys: [wave][64] of dR.V, q.(dO' S), k.(U dS), k.(dR S), then
  // <dS, S> per wave; sums over tiles: [4][64] of rows of dP P + dA A, rows of dA A /
  // beta, columns of dP P + dA A; decays and beta
  static constexpr int floats = 4 * 8 * kGdrC + 8 + 3 * 4 * kGdrC + 3 * kGdrC;
  static constexpr int total = red + floats * 4;
};

template <typename T, int DK>
__global__ void __launch_bounds__(512, 1) carve_gdr_grad_kernel(GdrArgs a) {
  typedef InterT<T> IT;
  typedef GradLds<T> L;
  constexpr int NP = DK / 32;
  constexpr int NJ = DK / 16;      // key tiles
  constexpr int NI = NJ / 2;       // row tiles of a wave in the products over key columns
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* red = reinterpret_cast<float*>(smem + L::red);
  float* rRV = red;                        // [8][64]
  float* rQ = rRV + 8 * kGdrC;             // [8][64]
  float* rUK = rQ + 8 * kGdrC;             // [8][64]
  float* rRK = rUK + 8 * kGdrC;            // [8][64]
  float* rSS = rRK + 8 * kGdrC;            // [8]
  float* rRow = rSS + 8;                   // [4][64]
  float* rBeta = rRow + 4 * kGdrC;         // [4][64]
  float* rCol = rBeta + 4 * kGdrC;         // [4][64]
  float* sGh = rCol + 4 * kGdrC;           // [64]
  float* sGl = sGh + kGdrC;
  float* sBe = sGl + kGdrC;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int slot = blockIdx.x, hk = blockIdx.y, grp = a.Hv / a.Hk;
  GdrSeq sq;
  int n, chunk;
  if (!gdr_find(a, slot, sq, n, chunk)) return;   // (uniform)
  const int t0 = sq.t0 + chunk * kGdrC, len = min(kGdrC, sq.len - chunk * kGdrC);
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + t0 * a.ks[1] + hk * a.ks[2];
  const size_t row0 = (size_t)sq.batch * a.T + t0;
  const size_t sm = (size_t)a.Dv * DK;
  const size_t ors = (size_t)a.Hv * a.Dv;

  // this wave's key tile and row tiles
  const int jt = w % NJ, i0 = NI * (w / NJ);
  f32x4 dQ[NI], dK[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) dQ[i] = dK[i] = zero4();
  for (int hv = hk * grp; hv < (hk + 1) * grp; ++hv) {
    const size_t sh = (size_t)slot * a.Hv + hv;
    const char* ws = a.ws + sh * a.per;
    const float* scal = reinterpret_cast<const float*>(ws + GdrWs<T>::bScal);
    const T* v = reinterpret_cast<const T*>(a.v) + sq.batch * a.vs[0] + t0 * a.vs[1] + hv * a.vs[2];
    const T* dO = reinterpret_cast<const T*>(a.dO) + (row0 * a.Hv + hv) * a.Dv;
    T* dV = reinterpret_cast<T*>(a.dv) + (row0 * a.Hv + hv) * a.Dv;
    const float* S = a.S_chunks + sh * sm;
    const float* dS = a.dS_chunks + sh * sm;
    if (tid < kGdrC) {
      sGh[tid] = scal[kScGh * kGdrC + tid];
      sGl[tid] = scal[kScGl * kGdrC + tid];
      sBe[tid] = scal[kScBeta * kGdrC + tid];
    }
    f32x4 aP[2], aA[2];                     // tile tasks w and w + 8 (of ten)
    f32x4 a1[NI], a2[NI], a3[NI];           // dO S, U dS, dR S
#pragma unroll
    for (int x = 0; x < 2; ++x) aP[x] = aA[x] = zero4();
#pragma unroll
    for (int i = 0; i < NI; ++i) a1[i] = a2[i] = a3[i] = zero4();
    float rv[4][4], ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) rv[i][e] = 0.0f;

    for (int vb = 0; vb < a.Dv; vb += kVB) {
      const int cols = min(kVB, a.Dv - vb);
      // ---- 1. U, dR of columns vb + 16 w ..
      if (16 * w < cols) {
        const int v0 = vb + 16 * w;
        Fi<T, kExact> Sf[NP], Df[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const size_t at = (size_t)(v0 + c) * DK + 32 * p + 8 * g;
          const f32x4 s0 = *reinterpret_cast<const f32x4*>(S + at), s1 = *reinterpret_cast<const f32x4*>(S + at + 4);
          const f32x4 d0 = *reinterpret_cast<const f32x4*>(dS + at), d1 = *reinterpret_cast<const f32x4*>(dS + at + 4);
          for (int e = 0; e < 4; ++e) ss += s0[e] * d0[e] + s1[e] * d1[e];
          Sf[p] = to_fi<T, kExact>(s0, s1);
          Df[p] = to_fi<T, kExact>(d0, d1);
        }
        f32x4 R[4], U[4], vt[4], od[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = 16 * i + 4 * g + e;
            vt[i][e] = t < len ? (float)v[(size_t)t * a.vs[1] + v0 + c] : 0.0f;
            od[i][e] = t < len ? (float)dO[(size_t)t * ors + v0 + c] : 0.0f;
          }
        Fr<T> of[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          of[s].a = Quad<T>::cvt(od[2 * s]);
          of[s].b = Quad<T>::cvt(od[2 * s + 1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 16 * i + c;
          f32x4 x = zero4(), y = zero4(), z = zero4();
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const Fr<T> fk = ld_fr<T>(k + (size_t)r * a.ks[1] + 32 * p + 8 * g, r < len);
            x = mma<T>(fk, Sf[p], x);
            y = mma<T>(fk, Df[p], y);
          }
#pragma unroll
          for (int s = i / 2; s < 2; ++s) z = mma<T>(ld_img<T, kExact>(ws + GdrWs<T>::bPt, img_upper(i, s), lane), of[s], z);
          const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
          const f32x4 end = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
          const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
          R[i] = be * (vt[i] - gam * x);
          U[i] = z * a.scale + y * end;      // dU
        }
        const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(R[0], R[1]), to_fi<T, kExact>(R[2], R[3])};
        const Fi<T, kExact> Uf[2] = {to_fi<T, kExact>(U[0], U[1]), to_fi<T, kExact>(U[2], U[3])};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x = zero4(), y = zero4();
#pragma unroll
          for (int s = 0; s <= i / 2; ++s) x = mma<T>(ld_img<T, kExact>(ws, img_lower(i, s), lane), Rf[s], x);
#pragma unroll
          for (int s = i / 2; s < 2; ++s) y = mma<T>(ld_img<T, kExact>(ws + GdrWs<T>::bTt, img_upper(i, s), lane), Uf[s], y);
          IT::template put<kExact>(smem + L::U, kVB, 16 * w + c, i, g, x);
          IT::template put<kExact>(smem + L::R, kVB, 16 * w + c, i, g, y);
          const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = 16 * i + 4 * g + e;
            rv[i][e] += y[e] * vt[i][e];
            if (t < len) dV[(size_t)t * ors + v0 + c] = (T)(be[e] * y[e]);
          }
        }
      }
      __syncthreads();
      // ---- 2. products over these columns
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int y = w + 8 * x;
        if (y < 10) {
          const int i = tri_row_of(y, false), j = tri_col_of(y, false), r = 16 * i + c;
          for (int p = 0; p < cols / 32; ++p) {
            const Fi<T, kExact> fu = IT::template tok<kExact>(smem + L::U, kVB, j, 32 * p, g, c);
            aP[x] = mma<T>(ld_fr16<T>(dO + (size_t)r * ors + vb + 32 * p + 4 * g, r < len), fu, aP[x]);
            aA[x] = mma<T>(IT::template tok<kExact>(smem + L::R, kVB, i, 32 * p, g, c), fu, aA[x]);
          }
        }
      }
      for (int p = 0; p < cols / 32; ++p) {
        f32x4 s[2], d[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const size_t at = (size_t)(vb + 32 * p + 16 * h + 4 * g + e) * DK + 16 * jt + c;
            s[h][e] = S[at];
            d[h][e] = dS[at];
          }
        const Fi<T, kExact> fs = to_fi<T, kExact>(s[0], s[1]), fd = to_fi<T, kExact>(d[0], d[1]);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int r = 16 * (i0 + i) + c;
          a1[i] = mma<T>(ld_fr16<T>(dO + (size_t)r * ors + vb + 32 * p + 4 * g, r < len), fs, a1[i]);
          a2[i] = mma<T>(IT::template tok<kExact>(smem + L::U, kVB, i0 + i, 32 * p, g, c), fd, a2[i]);
          a3[i] = mma<T>(IT::template tok<kExact>(smem + L::R, kVB, i0 + i, 32 * p, g, c), fs, a3[i]);
        }
      }
      __syncthreads();
    }

    // ---- sums over the value columns and <dS, S>
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = group_sum<16>(rv[i][e]);
        if (c == 0) rRV[w * kGdrC + 16 * i + 4 * g + e] = x;
      }
    ss = group_sum<64>(ss);
    if (lane == 0) rSS[w] = ss;

    // ---- D dP and M of this wave's tiles, with their row and column sums; zeros in the
    // upper tiles (0, 1) and (2, 3), which the fragments reach
    if (w >= 4) {
      const int y = w - 4;
      IT::template put<kNear>(smem + (y & 1 ? L::M : L::W), kGdrC, 16 * (y < 2 ? 1 : 3) + c, y < 2 ? 0 : 2, g, zero4());
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int y = w + 8 * x;
      if (y < 10) {
        const int i = tri_row_of(y, false), j = tri_col_of(y, false), r = 16 * i + c, rj = 16 * j + c;
        f32x4 qk = zero4(), kk = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const Fr<T> fb = ld_fr<T>(k + (size_t)rj * a.ks[1] + 32 * p + 8 * g, rj < len);
          qk = mma<T>(ld_fr<T>(q + (size_t)r * a.qs[1] + 32 * p + 8 * g, r < len), fb, qk);
          kk = mma<T>(ld_fr<T>(k + (size_t)r * a.ks[1] + 32 * p + 8 * g, r < len), fb, kk);
        }
        f32x4 W, M;
        float col = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ti = 16 * i + 4 * g + e, tj = 16 * j + c;
          float D = 0.0f;
          if (tj <= ti) D = expf((sGh[ti] - sGh[tj]) + (sGl[ti] - sGl[tj]));
          const float be = sBe[ti], dA = tj < ti ? -aA[x][e] : 0.0f;
          W[e] = a.scale * (D * aP[x][e]);
          M[e] = be * (D * dA);
          const float pp = W[e] * qk[e], ab = D * dA * kk[e], s = pp + be * ab;
          col += s;
          const float rs = group_sum<16>(s), rb = group_sum<16>(ab);
          if (c == 0) {
            rRow[j * kGdrC + ti] = rs;
            rBeta[j * kGdrC + ti] = rb;
          }
        }
        col += __shfl_xor(col, 16);
        col += __shfl_xor(col, 32);
        if (g == 0) rCol[i * kGdrC + rj] = col;
        IT::template put<kNear>(smem + L::W, kGdrC, 16 * j + c, i, g, W);
        IT::template put<kNear>(smem + L::M, kGdrC, 16 * j + c, i, g, M);
      }
    }
    __syncthreads();

    // ---- dQ, dK of this wave's tiles
    {
      // K and Q as B operands: tokens 32 s + 4 g + e and + 16, column 16 jt + c
      Fr<T> fk[2], fq[2];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          typename Quad<T>::q xk, xq;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = 32 * s + 16 * h + 4 * g + e;
            xk[e] = t < len ? k[(size_t)t * a.ks[1] + 16 * jt + c] : (T)0.0f;
            xq[e] = t < len ? q[(size_t)t * a.qs[1] + 16 * jt + c] : (T)0.0f;
          }
          if (h == 0) fk[s].a = xk, fq[s].a = xq;
          else fk[s].b = xk, fq[s].b = xq;
        }
#pragma unroll
      for (int ii = 0; ii < NI; ++ii) {
        const int i = i0 + ii;
        const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
        const f32x4 end = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
        const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
        const f32x4 x1 = a1[ii] * gam * a.scale, x2 = a2[ii] * end, x3 = a3[ii] * gam;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = 16 * i + 4 * g + e;
          const float kt = t < len ? (float)k[(size_t)t * a.ks[1] + 16 * jt + c] : 0.0f;
          const float qt = t < len ? (float)q[(size_t)t * a.qs[1] + 16 * jt + c] : 0.0f;
          const float s1 = group_sum<16>(qt * x1[e]), s2 = group_sum<16>(kt * x2[e]), s3 = group_sum<16>(kt * x3[e]);
          if (c == 0) {
            rQ[jt * kGdrC + t] = s1;
            rUK[jt * kGdrC + t] = s2;
            rRK[jt * kGdrC + t] = s3;
          }
        }
        dQ[ii] += x1;
        dK[ii] += x2 - be * x3;
        for (int s = 0; s <= i / 2; ++s) {
          dQ[ii] = mma<T>(IT::template tok<kNear>(smem + L::W, kGdrC, i, 32 * s, g, c), fk[s], dQ[ii]);
          dK[ii] = mma<T>(IT::template tok<kNear>(smem + L::M, kGdrC, i, 32 * s, g, c), fk[s], dK[ii]);
        }
        for (int s = i / 2; s < 2; ++s) {
          dK[ii] = mma<T>(IT::template col<kNear>(smem + L::W, kGdrC, 16 * i, s, g, c), fq[s], dK[ii]);
          dK[ii] = mma<T>(IT::template col<kNear>(smem + L::M, kGdrC, 16 * i, s, g, c), fk[s], dK[ii]);
        }
      }
    }
    __syncthreads();

    // ---- dbeta, dg
    if (w == 0) {
      const int t = lane;
      float rv1 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f, sss = 0.0f, row = 0.0f, rb = 0.0f, col = 0.0f;
      for (int x = 0; x < 8; ++x) {
        rv1 += rRV[x * kGdrC + t];
        sss += rSS[x];
      }
      for (int x = 0; x < NJ; ++x) {
        s1 += rQ[x * kGdrC + t];
        s2 += rUK[x * kGdrC + t];
        s3 += rRK[x * kGdrC + t];
      }
      for (int x = 0; x < 4; ++x) {
        if (x <= t / 16) {
          row += rRow[x * kGdrC + t];
          rb += rBeta[x * kGdrC + t];
        }
        if (x >= t / 16) col += rCol[x * kGdrC + t];
      }
      const float be = sBe[t];
      float dG = s1 - be * s3 - s2 + row - col;
      float ends = group_sum<64>(s2);
      ends += scal[kScGam * kGdrC + kGdrC - 1] * sss;
      // suffix sums
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const float up = __shfl_down(dG, d);
        if (t + d < 64) dG += up;
      }
      if (t < len) {
        a.dg[(row0 + t) * a.Hv + hv] = dG + ends;
        reinterpret_cast<T*>(a.dbeta)[(row0 + t) * a.Hv + hv] = (T)(rv1 - s3 + rb);
      }
    }
    __syncthreads();
  }

  T* dq = reinterpret_cast<T*>(a.dq) + (row0 * a.Hk + hk) * DK + 16 * jt + c;
  T* dk = reinterpret_cast<T*>(a.dk) + (row0 * a.Hk + hk) * DK + 16 * jt + c;
#pragma unroll
  for (int ii = 0; ii < NI; ++ii)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = 16 * (i0 + ii) + 4 * g + e;
      if (t < len) {
        dq[(size_t)t * a.Hk * DK] = (T)dQ[ii][e];
        dk[(size_t)t * a.Hk * DK] = (T)dK[ii][e];
      }
    }
}

// dynamic LDS above 64 KB needs the attribute once per kernel and device
template <typename K>
int allow_lds(K kern, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) ==
                 hipSuccess
             ? CARVE_OK
             : CARVE_ERR_HIP;
}

template <typename T, int DK, int NW>
int launch_bchain_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = BChainLds<T, DK, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_bchain_kernel<T, DK, NW>;
  const int st = allow_lds(kern, lds);
  if (st) return st;
  const unsigned heads = (unsigned)a.nseq * a.Hv;
  hipLaunchKernelGGL(kern, dim3((heads + 7) / 8 * 8 * (a.Dv / (16 * NW))), dim3(64 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK>
int launch_bwd_t(const GdrArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  static_assert(GradLds<T>::total <= 160 * 1024, "LDS");
  int st = launch_gdr_prep(a, sizeof(T) == 2 ? CARVE_BF16 : CARVE_F32, true, s);
  if (st) return st;
  mark(s);
  st = gdr_chain_waves(a) == 4 ? launch_bchain_t<T, DK, 4>(a, s) : launch_bchain_t<T, DK, 2>(a, s);
  if (st) return st;
  mark(s);
  st = allow_lds(carve_gdr_grad_kernel<T, DK>, GradLds<T>::total);
  if (st) return st;
  hipLaunchKernelGGL((carve_gdr_grad_kernel<T, DK>), dim3(a.nslots, a.Hk), dim3(512), GradLds<T>::total, s, a);
  mark(s);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}

}  // namespace

int launch_gdr_bwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
  const bool h = dtype == CARVE_BF16;
  switch (a.Dk) {
    case 32: return h ? launch_bwd_t<bf16_t, 32>(a, s, mark) : launch_bwd_t<float, 32>(a, s, mark);
    case 64: return h ? launch_bwd_t<bf16_t, 64>(a, s, mark) : launch_bwd_t<float, 64>(a, s, mark);
    case 128: return h ? launch_bwd_t<bf16_t, 128>(a, s, mark) : launch_bwd_t<float, 128>(a, s, mark);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}

}  // namespace carve
