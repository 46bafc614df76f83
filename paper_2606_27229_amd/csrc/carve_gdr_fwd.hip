// carve_gdr_fwd.hip -- the chunked gated delta rule, forward: the chunk-local
// triangles (every chunk at once), then the chain of states.
#include "carve_gdr.h"

namespace carve {
namespace {

// ---------------------------------------------------------------------------------
// Chunk-local part: T = (I + A)^-1 and P of every (chunk slot, value head), as
// operand images, with the chunk's decay factors.  One workgroup of four waves each;
// wave w forms the row tile w of K K^T and Q K^T.  The diagonal 16 x 16 blocks are
// inverted by substitution (one lane a column, all four blocks in one wave), the
// blocks below by T21 = -T22 A21 T11 with f32 matrix-core products, twice.  f32
// throughout: T multiplies every value of the chunk.
// G is summed in 64 bits and kept as two floats, so that a decay between two tokens
// keeps its digits however strongly the tokens before them decay.
template <typename T, int DK, bool BWD>
__global__ void __launch_bounds__(256) carve_gdr_prep_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  constexpr int LD = kGdrC + 4;
  __shared__ __attribute__((aligned(16))) float sA[kGdrC * LD];
  __shared__ __attribute__((aligned(16))) float sT[kGdrC * LD];
  __shared__ __attribute__((aligned(16))) float sP[kGdrC * LD];
  __shared__ float sGh[kGdrC], sGl[kGdrC], sB[kGdrC];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int slot = blockIdx.x, hv = blockIdx.y, hk = hv / (a.Hv / a.Hk);
  GdrSeq sq;
  int n, chunk;
  if (!gdr_find(a, slot, sq, n, chunk)) return;   // (uniform)
  const int t0 = sq.t0 + chunk * kGdrC, len = min(kGdrC, sq.len - chunk * kGdrC);
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + t0 * a.ks[1] + hk * a.ks[2];
  const size_t row0 = ((size_t)sq.batch * a.T + t0) * a.Hv + hv;
  char* ws = a.ws + ((size_t)slot * a.Hv + hv) * a.per;
  typedef GdrWs<T> WS;
  float* scal = reinterpret_cast<float*>(ws + (BWD ? WS::bScal : WS::fScal));

  // row tile w against the column tiles up to it
  f32x4 kk[4], qk[4];
  {
    Fr<T> fk[NP], fq[NP];
    const int r = 16 * w + c;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      fk[p] = ld_fr<T>(k + r * a.ks[1] + 32 * p + 8 * g, r < len);
      fq[p] = ld_fr<T>(q + r * a.qs[1] + 32 * p + 8 * g, r < len);
    }
    if (w == 0) {   // decays: prefix sums over the wave's lanes
      const size_t at = row0 + (size_t)lane * a.Hv;
      float gt = lane < len ? a.g[at] : 0.0f;
      const float be = lane < len ? (float)reinterpret_cast<const T*>(a.beta)[at] : 0.0f;
      gt = gt < kGdrMinG ? kGdrMinG : gt;
      double G = (double)gt;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double up = __shfl_up(G, d);
        if (lane >= d) G += up;
      }
      const float Gh = (float)G, Gl = (float)(G - (double)Gh);
      const double Ge = __shfl(G, 63);
      sGh[lane] = Gh;
      sGl[lane] = Gl;
      sB[lane] = be;
      scal[kScGam * kGdrC + lane] = expf(Gh) * (1.0f + Gl);
      scal[kScEnd * kGdrC + lane] = expf((float)(Ge - G));
      scal[kScBeta * kGdrC + lane] = be;
      scal[kScGh * kGdrC + lane] = Gh;
      scal[kScGl * kGdrC + lane] = Gl;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      kk[s] = qk[s] = zero4();
      if (s <= w) {
        const int rb = 16 * s + c;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const Fr<T> fb = ld_fr<T>(k + rb * a.ks[1] + 32 * p + 8 * g, rb < len);
          kk[s] = mma<T>(fk[p], fb, kk[s]);
          qk[s] = mma<T>(fq[p], fb, qk[s]);
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 16 * w + 4 * g + e, j = 16 * s + c;
      float Av = 0.0f, Pv = 0.0f;
      if (j <= i) {
        const float D = expf((sGh[i] - sGh[j]) + (sGl[i] - sGl[j]));
        Pv = D * qk[s][e];
        if (j < i) Av = sB[i] * (D * kk[s][e]);
      }
      sA[i * LD + j] = Av;
      sP[i * LD + j] = Pv;
      sT[i * LD + j] = 0.0f;
    }
  __syncthreads();
  // P image by waves 1 - 3, the diagonal inverses by wave 0
  char* imgP = ws + (BWD ? WS::bPt : WS::fP);
  if (w > 0) {
    for (int x = tid - 64; x < 6 * 64; x += 192) {
      const int f = x >> 6, l = x & 63, lg = l >> 4, lc = l & 15;
      if constexpr (!BWD) {
        const int i = f < 2 ? f : 2 + (f - 2) / 2, s = f < 2 ? 0 : (f - 2) % 2;
        const float* r = sP + (16 * i + lc) * LD + 32 * s + 4 * lg;
        st_img<T, kNear>(imgP, f, l, *reinterpret_cast<const f32x4*>(r), *reinterpret_cast<const f32x4*>(r + 16));
      } else {
        const int i = f < 4 ? f / 2 : f - 2, s = f < 4 ? f % 2 : 1;
        const float* r = sP + (32 * s + 4 * lg) * LD + 16 * i + lc;
        const f32x4 x0 = {r[0], r[LD], r[2 * LD], r[3 * LD]};
        const f32x4 x1 = {r[16 * LD], r[17 * LD], r[18 * LD], r[19 * LD]};
        st_img<T, kExact>(imgP, f, l, x0, x1);
      }
    }
  } else {
    const float* A = sA + 16 * g * LD + 16 * g;
    float col[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = i == c ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < i; ++j) x -= A[i * LD + j] * col[j];
      col[i] = x;
      sT[(16 * g + i) * LD + 16 * g + c] = x;
    }
  }
  __syncthreads();
  // 16 x 16 operands in LDS: A operand rows, B operand columns
  const auto opA = [&](const float* m, int i, int j) {
    return *reinterpret_cast<const f32x4*>(m + (16 * i + c) * LD + 16 * j + 4 * g);
  };
  const auto opB = [&](const float* m, int i, int j) {
    const float* r = m + (16 * i + 4 * g) * LD + 16 * j + c;
    const f32x4 x = {r[0], r[LD], r[2 * LD], r[3 * LD]};
    return x;
  };
  const auto put = [&](int i, int j, f32x4 x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sT[(16 * i + 4 * g + e) * LD + 16 * j + c] = -x[e];
  };
  typedef Quad<float> QF;
  if (w < 2) {
    const f32x4 y = QF::mma16(opA(sA, 2 * w + 1, 2 * w), opB(sT, 2 * w, 2 * w), zero4());
    put(2 * w + 1, 2 * w, QF::mma16(opA(sT, 2 * w + 1, 2 * w + 1), y, zero4()));
  }
  __syncthreads();
  {
    const int j = w & 1, i = 2 + (w >> 1);   // wave w: block (i, j)
    f32x4 r = zero4();
#pragma unroll
    for (int kb = 2; kb < 4; ++kb) {
      if (kb > i) continue;
      f32x4 y = QF::mma16(opA(sA, kb, 1), opB(sT, 1, j), zero4());
      if (j == 0) y = QF::mma16(opA(sA, kb, 0), opB(sT, 0, 0), y);
      r = QF::mma16(opA(sT, i, kb), y, r);
    }
    put(i, j, r);
  }
  __syncthreads();
  for (int x = tid; x < 6 * 64; x += 256) {
    const int f = x >> 6, l = x & 63, lg = l >> 4, lc = l & 15;
    {
      const int i = f < 2 ? f : 2 + (f - 2) / 2, s = f < 2 ? 0 : (f - 2) % 2;
      const float* r = sT + (16 * i + lc) * LD + 32 * s + 4 * lg;
      st_img<T, kExact>(ws, f, l, *reinterpret_cast<const f32x4*>(r), *reinterpret_cast<const f32x4*>(r + 16));
    }
    if constexpr (BWD) {
      const int i = f < 4 ? f / 2 : f - 2, s = f < 4 ? f % 2 : 1;
      const float* r = sT + (32 * s + 4 * lg) * LD + 16 * i + lc;
      const f32x4 x0 = {r[0], r[LD], r[2 * LD], r[3 * LD]};
      const f32x4 x1 = {r[16 * LD], r[17 * LD], r[18 * LD], r[19 * LD]};
      st_img<T, kExact>(ws + WS::bTt, f, l, x0, x1);
    }
  }
}

// ---------------------------------------------------------------------------------
// The chain of states.  A workgroup runs one sequence and value head for 16 NW value
// columns, NW tiles of 16: value rows of S are independent, so the tiles share nothing
// but the chunk's rows.  Two waves a tile:
//   chain   R = beta (V - e^G K S^T), U = T R, S^T <- e^{G_C} S^T + K^T (e^{G_C - G} U)
//   helper  o = scale (e^G Q S^T + P U), one chunk behind, and all global memory: the
//           next chunk's keys, values, T and decays straight into LDS, its own queries
//           and P into registers, outputs and chunk start states out
// The chain is what the call takes (chunks follow each other), so the helper takes from
// it whatever it can; the two run on different SIMDs.  The chain's S^T[j][v] stays in the
// matrix-core result layout, where it is at once the B operand of K S^T (chain) and the
// A operand of (Q S^T)^T (helper): it needs no transposition, and U neither.  S and U
// pass to the helper through LDS as they lie in registers.  Barriers, two a chunk: (1)
// the chunk's rows are there and the chain has left S(ch), U(ch - 1); (2) the helper has
// taken them.
template <typename T, int DK, int NW>
struct ChainLds {
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, 16 * NW> VR;
  static constexpr int K = 0, V = K + KR::bytes, I = V + VR::bytes;   // I: T, scalars
  static constexpr int one = I + GdrWs<T>::fP;
  static constexpr int xS = 2 * one, xU = xS + NW * (DK / 16) * 1024;
  static constexpr int total = xU + NW * 4 * 1024;
};

template <typename T, int DK, int NW>
__global__ void __launch_bounds__(128 * NW, 1) carve_gdr_chain_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef ChainLds<T, DK, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool helper = wave >= NW;
  const int w = helper ? wave - NW : wave;   // tile
  const int g = lane >> 4, c = lane & 15;
  // blocks 8 apart share an XCD: the slices of a (sequence, head) follow each other there
  const int ns = a.Dv / (16 * NW), idx = blockIdx.x;
  const int head = idx / (8 * ns) * 8 + idx % 8, slice = idx / 8 % ns;
  if (head >= a.nseq * a.Hv) return;
  const int n = head / a.Hv, hv = head % a.Hv, hk = hv / (a.Hv / a.Hk);
  const int vs = 16 * NW * slice, v0 = vs + 16 * w;
  const GdrSeq sq = gdr_seq(a, n);
  const size_t sm = (size_t)a.Dv * DK;   // elements of a state
  const size_t soff = (size_t)(v0 + c) * DK + 4 * g;
  const int nch = (sq.len + kGdrC - 1) / kGdrC;
  f32x4* xS = reinterpret_cast<f32x4*>(smem + L::xS + w * (DK / 16) * 1024) + lane;
  f32x4* xU = reinterpret_cast<f32x4*>(smem + L::xU + w * 4 * 1024) + lane;

  if (!helper) {
    f32x4 S[2 * NP];
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) {
      S[j] = a.S0 ? *reinterpret_cast<const f32x4*>(a.S0 + (size_t)head * sm + soff + 16 * j) : zero4();
      xS[64 * j] = S[j];
    }
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
      const char* buf = smem + (ch & 1) * L::one;
      const float* scal = reinterpret_cast<const float*>(buf + L::I + WS::fScal);
      __syncthreads();   // (1)
      Fi<T, kExact> Sf[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) Sf[p] = to_fi<T, kExact>(S[2 * p], S[2 * p + 1]);
      __syncthreads();   // (2)
      f32x4 R[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 acc = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) acc = mma<T>(KR::nat(buf + L::K, i, p, g, c), Sf[p], acc);
        const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
        const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
        R[i] = be * (Quad<T>::f32(VR::tr(buf + L::V, 16 * i, w, g, c)) - gam * acc);
      }
      const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(R[0], R[1]), to_fi<T, kExact>(R[2], R[3])};
      f32x4 U[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        U[i] = zero4();
#pragma unroll
        for (int s = 0; s <= i / 2; ++s)
          U[i] = mma<T>(ld_img<T, kExact>(buf + L::I + WS::fT, img_lower(i, s), lane), Rf[s], U[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xU[64 * i] = U[i];
        U[i] *= *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
      }
      const float gend = scal[kScGam * kGdrC + kGdrC - 1];
      const Fi<T, kExact> Ue[2] = {to_fi<T, kExact>(U[0], U[1]), to_fi<T, kExact>(U[2], U[3])};
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j) {
        S[j] *= gend;
#pragma unroll
        for (int s = 0; s < 2; ++s) S[j] = mma<T>(KR::tr32(buf + L::K, s, j, g, c), Ue[s], S[j]);
        xS[64 * j] = S[j];
      }
    }
    __syncthreads();
    if (a.S_T) {
      float* s = a.S_T + (size_t)head * sm + soff;
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    return;
  }

  // ---- helper
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + sq.t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + sq.t0 * a.ks[1] + hk * a.ks[2];
  const T* v = reinterpret_cast<const T*>(a.v) + sq.batch * a.vs[0] + sq.t0 * a.vs[1] + hv * a.vs[2] + vs;
  T* o = reinterpret_cast<T*>(a.o) + (((size_t)sq.batch * a.T + sq.t0) * a.Hv + hv) * a.Dv + v0;
  const size_t ors = (size_t)a.Hv * a.Dv;
  const auto load = [&](int ch) {
    char* buf = smem + (ch & 1) * L::one;
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    KR::dma(buf + L::K, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, w, NW, lane);
    dma_flat(buf + L::I, a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per, WS::fP, w, NW, lane);
    VR::dma(buf + L::V, v + t0 * a.vs[1], (int)(a.vs[1] * sizeof(T)), len, w, NW, lane);
  };
  // queries of a chunk (any row behind the last token repeats it) and P with e^G
  struct Mine {
    Fr<T> q[4][NP];
    Fi<T, kNear> P[6];
    float gam[4];
  };
  const auto load_q = [&](Mine& m, int ch) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T* r = q + (size_t)min(ch * kGdrC + 16 * i + c, sq.len - 1) * a.qs[1] + 4 * g;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        m.q[i][p].a = Quad<T>::ld(r + 32 * p);
        m.q[i][p].b = Quad<T>::ld(r + 32 * p + 16);
      }
    }
  };
  const auto load_p = [&](Mine& m, int ch) {
    const char* img = a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per;
#pragma unroll
    for (int f = 0; f < 6; ++f) m.P[f] = ld_img<T, kNear>(img + WS::fP, f, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m.gam[i] = reinterpret_cast<const float*>(img + WS::fScal)[kScGam * kGdrC + 16 * i + c];
  };
  // with the registers for it (one wave a SIMD, bf16), loaded a chunk ahead
  constexpr bool AHEAD = NW == 2 && sizeof(T) == 2;
  Mine cur, nxt;
  f32x4 x[4];
  if (nch > 0) {
    load(0);
    if constexpr (AHEAD) load_q(nxt, 0);
  }
#pragma unroll 1
  for (int ch = 0; ch <= nch; ++ch) {
    vm_wait_all();
    __syncthreads();   // (1)
    f32x4 S[2 * NP], U[4];
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) S[j] = xS[64 * j];
#pragma unroll
    for (int i = 0; i < 4; ++i) U[i] = xU[64 * i];
    if (ch < nch) __syncthreads();   // (2)
    if (ch + 1 < nch) load(ch + 1);
    if constexpr (AHEAD) {
      // (the queries of this chunk and P of the last one)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int p = 0; p < NP; ++p) cur.q[i][p] = nxt.q[i][p];
#pragma unroll
      for (int f = 0; f < 6; ++f) cur.P[f] = nxt.P[f];
#pragma unroll
      for (int i = 0; i < 4; ++i) cur.gam[i] = nxt.gam[i];
      if (ch + 1 < nch) load_q(nxt, ch + 1);
      if (ch < nch) load_p(nxt, ch);
    }
    if (a.S_chunks && ch < nch) {
      float* s = a.S_chunks + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * sm + soff;
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    if (ch > 0) {   // o of the last chunk
      if constexpr (!AHEAD) load_p(cur, ch - 1);
      const Fi<T, kNear> Uf[2] = {to_fi<T, kNear>(U[0], U[1]), to_fi<T, kNear>(U[2], U[3])};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 y = zero4();
#pragma unroll
        for (int s = 0; s <= i / 2; ++s) y = mma<T>(Uf[s], cur.P[img_lower(i, s)], y);
        const int t = (ch - 1) * kGdrC + 16 * i + c;
        if (t < sq.len) Quad<T>::st(o + (size_t)t * ors + 4 * g, Quad<T>::cvt((x[i] * cur.gam[i] + y) * a.scale));
      }
    }
    if (ch < nch) {   // (Q S^T)^T: a lane holds four values of token 16 i + c
      if constexpr (!AHEAD) load_q(cur, ch);
      Fi<T, kNear> Sf[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) Sf[p] = to_fi<T, kNear>(S[2 * p], S[2 * p + 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) x[i] = mma<T>(Sf[p], cur.q[i][p], x[i]);
      }
    }
  }
}

template <typename T, int DK>
int launch_prep_t(const GdrArgs& a, bool bwd, hipStream_t s) {
  const dim3 grid(a.nslots, a.Hv);
  if (bwd) hipLaunchKernelGGL((carve_gdr_prep_kernel<T, DK, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((carve_gdr_prep_kernel<T, DK, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK, int NW>
int launch_chain_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = ChainLds<T, DK, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_chain_kernel<T, DK, NW>;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CARVE_ERR_HIP;
  const unsigned heads = (unsigned)a.nseq * a.Hv;
  hipLaunchKernelGGL(kern, dim3((heads + 7) / 8 * 8 * (a.Dv / (16 * NW))), dim3(128 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK>
int launch_fwd_t(const GdrArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  int st = launch_prep_t<T, DK>(a, false, s);
  if (st) return st;
  mark(s);
  if constexpr (sizeof(T) == 4 && DK == 128) st = launch_chain_t<T, DK, 2>(a, s);
  else st = gdr_chain_tiles(a, sizeof(T) == 4) == 4 ? launch_chain_t<T, DK, 4>(a, s) : launch_chain_t<T, DK, 2>(a, s);
  mark(s);
  return st;
}

}  // namespace

int launch_gdr_prep(const GdrArgs& a, int dtype, bool bwd, hipStream_t s) {
  const bool h = dtype == CARVE_BF16;
  switch (a.Dk) {
    case 32: return h ? launch_prep_t<bf16_t, 32>(a, bwd, s) : launch_prep_t<float, 32>(a, bwd, s);
    case 64: return h ? launch_prep_t<bf16_t, 64>(a, bwd, s) : launch_prep_t<float, 64>(a, bwd, s);
    case 128: return h ? launch_prep_t<bf16_t, 128>(a, bwd, s) : launch_prep_t<float, 128>(a, bwd, s);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}
int launch_gdr_fwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
  const bool h = dtype == CARVE_BF16;
  switch (a.Dk) {
    case 32: return h ? launch_fwd_t<bf16_t, 32>(a, s, mark) : launch_fwd_t<float, 32>(a, s, mark);
    case 64: return h ? launch_fwd_t<bf16_t, 64>(a, s, mark) : launch_fwd_t<float, 64>(a, s, mark);
    case 128: return h ? launch_fwd_t<bf16_t, 128>(a, s, mark) : launch_fwd_t<float, 128>(a, s, mark);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}

}  // namespace carve
