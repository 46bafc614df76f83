// carve_gdr_fwd.hip -- the chunked gated delta rule, forward: the chunk-local
// triangles (every chunk at once), then the chain of states.
#include "carve_gdr.h"

namespace carve {
namespace {

// ---------------------------------------------------------------------------------
// Chunk-local part: T = (I + A)^-1 and P of every (chunk slot, value head), as
// operand images, with the chunk's decay factors.  One workgroup of four waves each.
// Wave w forms the products of token tile w (as columns of the result, so that a lane
// holds four consecutive entries of a row of A and P: P's image needs no transposition).
// The diagonal 16 x 16 blocks are inverted by substitution (one lane a column, a block a
// wave), the blocks below by T21 = -T22 A21 T11 with f32 matrix-core
// products, twice.  f32 throughout: T multiplies every value of the chunk.  Bound by the
// latency of these steps, so what counts is how many workgroups a compute unit holds:
// A (below the diagonal) and T (transposed, above it) share 17 KB of LDS, where the rows
// were before.  The rows come through LDS because each wave needs most of them: loaded by
// every wave for itself, 16 rows at a time, they made it 86 us at 4096 chunks of 128 keys
// (bf16; 270 MB in and out), where it takes 57 us now; the backward form, which writes
// two more images, 72 us.
// G is summed in 64 bits and kept as two floats, so that a decay between two tokens
// keeps its digits however strongly the tokens before them decay.
template <typename T, int DK>
struct PrepLds {
  typedef GdrRows<T, DK> KR;
  static constexpr int LD = kGdrC + 4;
  static constexpr int K = 0, Q = KR::bytes, M = 0;   // M over the rows
  static constexpr int rows = 2 * KR::bytes > kGdrC * LD * 4 ? 2 * KR::bytes : kGdrC * LD * 4;
  static constexpr int total = rows + 3 * kGdrC * 4;
};

template <typename T, int DK, bool BWD>
__global__ void __launch_bounds__(256, 4) carve_gdr_prep_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef PrepLds<T, DK> L;
  typedef typename L::KR KR;
  typedef GdrWs<T> WS;
  constexpr int LD = L::LD;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* sM = reinterpret_cast<float*>(smem + L::M);
  float* sGh = reinterpret_cast<float*>(smem + L::rows);
  float* sGl = sGh + kGdrC;
  float* sB = sGl + kGdrC;
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
  float* scal = reinterpret_cast<float*>(ws + (BWD ? WS::bScal : WS::fScal));

  // KK[j]: tokens 16 j + 4 g + e against token 16 w + c; QK[j] the same with the queries
  // of token 16 w + c (forward), or queries 16 j + 4 g + e against key 16 w + c (backward)
  f32x4 KK[4], QK[4];
  {
    // (the decays first: their sums form while the rows are on their way)
    float gt = 0.0f, be = 0.0f, Gh, Gl, end;
    if (w == 0 && lane < len) {
      const size_t at = row0 + (size_t)lane * a.Hv;
      gt = a.g[at];
      be = (float)reinterpret_cast<const T*>(a.beta)[at];
    }
    // (rows behind the last token repeat it: beta is 0 there, and no token before them
    // sees them)
    KR::template dma<4>(smem + L::K, k, (int)(a.ks[1] * sizeof(T)), len, w, lane);
    KR::template dma<4>(smem + L::Q, q, (int)(a.qs[1] * sizeof(T)), len, w, lane);
    if (w == 0) {   // decays: prefix sums over the wave's lanes
      gt = gt < kGdrMinG ? kGdrMinG : gt;
      double G = (double)gt;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double up = __shfl_up(G, d);
        if (lane >= d) G += up;
      }
      Gh = (float)G;
      Gl = (float)(G - (double)Gh);
      end = (float)(__shfl(G, 63) - G);
      sGh[lane] = Gh;
      sGl[lane] = Gl;
      sB[lane] = be;
    }
    vm_wait_all();
    __syncthreads();
    if (w == 0) {   // (behind the wait, which would wait for these stores too)
      scal[kScGam * kGdrC + lane] = decay_exp(Gh) * (1.0f + Gl);
      scal[kScEnd * kGdrC + lane] = decay_exp(end);
      scal[kScBeta * kGdrC + lane] = be;
      scal[kScGh * kGdrC + lane] = Gh;
      scal[kScGl * kGdrC + lane] = Gl;
    }
    Fr<T> fk[NP], fq[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      fk[p] = KR::nat(smem + L::K, w, p, g, c);
      if (!BWD) fq[p] = KR::nat(smem + L::Q, w, p, g, c);
    }
    // (all four tiles for every wave, masked below: branches by wave cost more than the
    // products they save)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      KK[j] = QK[j] = zero4();
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const Fr<T> fa = KR::nat(smem + L::K, j, p, g, c);
        KK[j] = mma<T>(fa, fk[p], KK[j]);
        if constexpr (BWD) QK[j] = mma<T>(KR::nat(smem + L::Q, j, p, g, c), fk[p], QK[j]);
        else QK[j] = mma<T>(fa, fq[p], QK[j]);
      }
    }
  }
  __syncthreads();
  {
    const int t = 16 * w + c;
    const float Gh = sGh[t], Gl = sGl[t], be = sB[t];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 gh = *reinterpret_cast<const f32x4*>(sGh + 16 * j + 4 * g);
      const f32x4 gl = *reinterpret_cast<const f32x4*>(sGl + 16 * j + 4 * g);
      f32x4 A;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int s = 16 * j + 4 * g + e;
        // one exponential serves both: of the decay from s to t, or from t to s
        const float x = (Gh - gh[e]) + (Gl - gl[e]), D = decay_exp(s <= t ? x : -x);
        A[e] = s < t ? be * (D * KK[j][e]) : 0.0f;
        QK[j][e] = (BWD ? s >= t : s <= t) ? D * QK[j][e] : 0.0f;
      }
      if (j <= w) *reinterpret_cast<f32x4*>(sM + t * LD + 16 * j + 4 * g) = A;   // (uniform)
    }
    // P's rows, or P^T's, of this wave's tile
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (!BWD && s <= w / 2) st_img<T, kNear>(ws + WS::fP, img_lower(w, s), lane, QK[2 * s], QK[2 * s + 1]);
      if (BWD && s >= w / 2) st_img<T, kExact>(ws + WS::bPt, img_upper(w, s), lane, QK[2 * s], QK[2 * s + 1]);
    }
  }
  // the wave's own diagonal block, lane (g, c) column c of its inverse; A's block is this
  // wave's writes (LDS accesses of a wave are carried out in order) and is not read again
  asm volatile("" ::: "memory");
  {
    const float* A = sM + 16 * w * (LD + 1);
    float col[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = i == c ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < i; ++j) x -= A[i * LD + j] * col[j];
      col[i] = x;
    }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; i += 4)   // (T transposed, zeros below its diagonal)
      if (4 * g == i) *reinterpret_cast<f32x4*>(sM + (16 * w + c) * LD + 16 * w + i) = f32x4{col[i], col[i + 1], col[i + 2], col[i + 3]};
  }
  __syncthreads();
  // 16 x 16 operands: A's rows; T's rows and columns, zero above T's diagonal blocks
  const auto opA = [&](int i, int j) { return *reinterpret_cast<const f32x4*>(sM + (16 * i + c) * LD + 16 * j + 4 * g); };
  const auto rowT = [&](int i, int j) {
    const float* r = sM + (16 * j + 4 * g) * LD + 16 * i + c;
    const f32x4 x = {r[0], r[LD], r[2 * LD], r[3 * LD]};
    return i < j ? zero4() : x;
  };
  const auto colT = [&](int i, int j) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(sM + (16 * j + c) * LD + 16 * i + 4 * g);
    return i < j ? zero4() : x;
  };
  const auto put = [&](int i, int j, f32x4 x) { *reinterpret_cast<f32x4*>(sM + (16 * j + c) * LD + 16 * i + 4 * g) = -x; };
  typedef Quad<float> QF;
  if (w < 2) {
    const f32x4 y = QF::mma16(opA(2 * w + 1, 2 * w), colT(2 * w, 2 * w), zero4());
    put(2 * w + 1, 2 * w, QF::mma16(rowT(2 * w + 1, 2 * w + 1), y, zero4()));
  }
  __syncthreads();
  {
    const int j = w & 1, i = 2 + (w >> 1);   // wave w: block (i, j)
    f32x4 r = zero4();
#pragma unroll
    for (int kb = 2; kb < 4; ++kb) {
      if (kb > i) continue;
      f32x4 y = QF::mma16(opA(kb, 1), colT(1, j), zero4());
      if (j == 0) y = QF::mma16(opA(kb, 0), colT(0, 0), y);
      r = QF::mma16(rowT(i, kb), y, r);
    }
    put(i, j, r);
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (s <= w / 2) st_img<T, kExact>(ws, img_lower(w, s), lane, rowT(w, 2 * s), rowT(w, 2 * s + 1));
    if (BWD && s >= w / 2) st_img<T, kExact>(ws + WS::bTt, img_upper(w, s), lane, colT(2 * s, w), colT(2 * s + 1, w));
  }
}

// ---------------------------------------------------------------------------------
// The chain of states, keys of 32.  A workgroup runs one sequence and value head for 32
// value columns, two tiles of 16: value rows of S are independent, so the tiles share
// nothing but the chunk's rows.  Two waves a tile:
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
constexpr int kChainNW = 2;   // value tiles of a workgroup
template <typename T>
struct ChainLds {
  static constexpr int DK = 32, NW = kChainNW;
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, 16 * NW> VR;
  static constexpr int K = 0, V = K + KR::bytes, I = V + VR::bytes;   // I: T, scalars
  static constexpr int one = I + GdrWs<T>::fP;
  static constexpr int xS = 2 * one, xU = xS + NW * (DK / 16) * 1024;
  static constexpr int total = xU + NW * 4 * 1024;
};

template <typename T>
__global__ void __launch_bounds__(128 * kChainNW, 1) carve_gdr_chain_kernel(GdrArgs a) {
  typedef ChainLds<T> L;
  constexpr int DK = L::DK, NP = DK / 32, NW = L::NW;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool helper = wave >= NW;
  const int w = helper ? wave - NW : wave;   // tile
  const int g = lane >> 4, c = lane & 15;
  int n, hv, slice;
  if (!gdr_chain_block(a, a.Dv / (16 * NW), n, hv, slice)) return;
  const int hk = hv / (a.Hv / a.Hk), head = n * a.Hv + hv;
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
    KR::template dma<NW>(buf + L::K, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, w, lane);
    dma_flat<NW, WS::fP / 1024>(buf + L::I, a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per, w, lane);
    VR::template dma<NW>(buf + L::V, v + t0 * a.vs[1], (int)(a.vs[1] * sizeof(T)), len, w, lane);
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
  // loaded a chunk ahead where they take few registers (bf16)
  constexpr bool AHEAD = sizeof(T) == 2;
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

// ---------------------------------------------------------------------------------
// The same chain with two waves a tile on it and two helpers (keys of 64 and 128): a call
// waits for each chunk's chain, 500 to 600 instructions of a chain wave (128 keys, bf16)
// that depend on each other in long rows: 5200 cycles a chunk with a tile a workgroup, 6600
// with two, where the vector units issue in 14 and 37 % of them.  (With a tile a workgroup
// some 90 of the instructions move accumulators between the register files: launch bounds
// of one wave a SIMD leave the compiler that choice.)  Chain wave h keeps the state of the
// keys' half h.  K S^T
// is the sum of both halves' products; each wave finishes two token tiles of it, makes
// their R and multiplies by T's columns of these tokens; both then add up U and update
// their half of the state.  Helper wave h takes the outputs of two token tiles.
// Barriers (1) and (2) as above; with LDS for S and U of two chunks in turn the helpers have
// taken one before the chain writes it again behind the next (1), and (2) is not needed (one
// sequence of 256 chunks of 16 heads 588 -> 562 us).  The chain waves of a tile meet twice more,
// by flags in LDS: (3) the halves of K S^T are there; (4) the parts of U.  With barriers
// for these too the helpers, whose memory instructions wait for each other, held the chain
// up: 214 us for 64 sequences and heads of 64 chunks (128 keys, 128 values, bf16), where it
// takes 180 us now, 2.8 us a chunk (230 us with the states at chunk starts written out:
// 268 MB).  One chain wave a tile with four tiles in a workgroup, which
// fits more tiles on the card, loses also where there are many: 8 x 1024 tokens of 32 heads
// (2048 tiles) 318 us, this 239 us.
template <typename T, int DK, int NW>   // NW: tiles
struct PairLds {
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, 32> VR;    // (with one tile, its neighbour's values too)
  static constexpr int K = 0, V = K + KR::bytes, I = V + VR::bytes;   // I: T, scalars
  static constexpr int one = I + GdrWs<T>::fP;
  // KB of a tile: S, U (its last two tiles without the other wave's part), U's last two
  // tiles; with room for it once more, for the other parity of the chunk; the halves of
  // K S^T that the other wave takes, its part of U
  static constexpr int xS = 0, xU = DK / 16, xW = xU + 4, out = xW + 2;
  static constexpr bool q_lds = sizeof(T) == 2 || DK < 128;           // (f32 queries of 128: from memory)
  static constexpr int Q = 2 * one, qone = q_lds ? KR::bytes : 0, x = Q + 2 * qone;
  static constexpr bool twice = x + NW * ((2 * out + 6) * 1024 + 16) <= 160 * 1024;
  static constexpr int other = twice ? out : 0, xP = out + other, xV = xP + 4, kb = xV + 2;
  static constexpr int flags = x + NW * kb * 1024, total = flags + NW * 16;
};

template <typename T, int DK, int NW>
__global__ void __launch_bounds__(256 * NW, 1) carve_gdr_pair_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef PairLds<T, DK, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool helper = wave >= 2 * NW;
  const int w = (wave >> 1) & (NW - 1), h = wave & 1;   // tile, half
  const int g = lane >> 4, c = lane & 15;
  int n, hv, slice;
  if (!gdr_chain_block(a, a.Dv / (16 * NW), n, hv, slice)) return;
  const int hk = hv / (a.Hv / a.Hk), head = n * a.Hv + hv;
  const int v0 = 16 * (NW * slice + w), vs = v0 & ~31, vt0 = v0 & 16 ? 1 : 0;   // vt0: tile of the values' rows
  const GdrSeq sq = gdr_seq(a, n);
  const size_t sm = (size_t)a.Dv * DK;
  const size_t soff = (size_t)(v0 + c) * DK + 4 * g;
  const int nch = (sq.len + kGdrC - 1) / kGdrC;
  // KB number i of the tile's exchange area, this lane's 16 bytes
  f32x4* x = reinterpret_cast<f32x4*>(smem + L::x + w * L::kb * 1024) + lane;

  lds_flag* flags = (lds_flag*)lds_at(smem + L::flags + 16 * w);

  if (!helper) {
    flags[h] = 0;   // (seen by the other wave behind the first barrier)
    f32x4 S[NP];   // key tiles NP h ..
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      S[j] = a.S0 ? *reinterpret_cast<const f32x4*>(a.S0 + (size_t)head * sm + soff + 16 * (NP * h + j)) : zero4();
      x[64 * (L::xS + NP * h + j)] = S[j];
    }
#pragma unroll 1
    for (int ch = 0; ch < nch; ++ch) {
      const char* buf = smem + (ch & 1) * L::one;
      const float* scal = reinterpret_cast<const float*>(buf + L::I + WS::fScal);
      f32x4* const xu = x + 64 * L::other * (ch & 1);             // this chunk's U
      f32x4* const xs = x + 64 * L::other * ((ch + 1) & 1);       // the state behind it
      __syncthreads();   // (1)
      Fi<T, kExact> Sf[NP / 2];
#pragma unroll
      for (int p = 0; p < NP / 2; ++p) Sf[p] = to_fi<T, kExact>(S[2 * p], S[2 * p + 1]);
      if (!L::twice) __syncthreads();   // (2)
      f32x4 acc[4];      // the other wave's two token tiles, then this one's
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int i = (2 * (1 - h) + y) & 3;
        acc[y] = zero4();
#pragma unroll
        for (int p = 0; p < NP / 2; ++p) acc[y] = mma<T>(KR::nat(buf + L::K, i, NP / 2 * h + p, g, c), Sf[p], acc[y]);
        if (y < 2) x[64 * (L::xP + 2 * h + y)] = acc[y];
      }
      const float gend = scal[kScGam * kGdrC + kGdrC - 1];
#pragma unroll
      for (int j = 0; j < NP; ++j) S[j] *= gend;
      // (what a step needs besides the other wave's part is read before the two meet)
      f32x4 gam[2], be[2], vt[2];
      Fi<T, kExact> Tf[4];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int i = 2 * h + y;
        gam[y] = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
        be[y] = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
        vt[y] = Quad<T>::f32(VR::tr(buf + L::V, 16 * i, vt0, g, c));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= 2 || !h) Tf[i] = ld_img<T, kExact>(buf + L::I + WS::fT, img_lower(i, h), lane);   // (uniform)
      pair_meet(flags, h, 2 * ch + 1);   // (3)
      f32x4 R[2], U[4];
#pragma unroll
      for (int y = 0; y < 2; ++y) R[y] = be[y] * (vt[y] - gam[y] * (acc[2 + y] + x[64 * (L::xP + 2 * (1 - h) + y)]));
      const Fi<T, kExact> Rf = to_fi<T, kExact>(R[0], R[1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < 2 && h) continue;   // (uniform)
        U[i] = mma<T>(Tf[i], Rf, zero4());
        (h ? x + 64 * (L::xV + i - 2) : xu + 64 * (L::xU + i))[0] = U[i];
      }
      f32x4 end[4];
      Fr<T> Kt[NP][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) end[i] = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s) Kt[j][s] = KR::tr32(buf + L::K, s, NP * h + j, g, c);
      pair_meet(flags, h, 2 * ch + 2);   // (4)
      if (h == 0) {
        U[2] += x[64 * L::xV];
        U[3] += x[64 * (L::xV + 1)];
      } else {
        U[0] = xu[64 * L::xU];
        U[1] = xu[64 * (L::xU + 1)];
        U[2] += xu[64 * (L::xU + 2)];
        U[3] += xu[64 * (L::xU + 3)];
        xu[64 * L::xW] = U[2];
        xu[64 * (L::xW + 1)] = U[3];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) U[i] *= end[i];
      const Fi<T, kExact> Ue[2] = {to_fi<T, kExact>(U[0], U[1]), to_fi<T, kExact>(U[2], U[3])};
#pragma unroll
      for (int j = 0; j < NP; ++j) {
#pragma unroll
        for (int s = 0; s < 2; ++s) S[j] = mma<T>(Kt[j][s], Ue[s], S[j]);
        xs[64 * (L::xS + NP * h + j)] = S[j];
      }
    }
    __syncthreads();
    if (a.S_T) {
      float* s = a.S_T + (size_t)head * sm + soff + 16 * NP * h;
#pragma unroll
      for (int j = 0; j < NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    return;
  }

  // ---- helper: token tiles 2 h, 2 h + 1
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + sq.t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + sq.t0 * a.ks[1] + hk * a.ks[2];
  const T* v = reinterpret_cast<const T*>(a.v) + sq.batch * a.vs[0] + sq.t0 * a.vs[1] + hv * a.vs[2] + vs;
  T* o = reinterpret_cast<T*>(a.o) + (((size_t)sq.batch * a.T + sq.t0) * a.Hv + hv) * a.Dv + v0;
  const size_t ors = (size_t)a.Hv * a.Dv;
  const int part = wave - 2 * NW;
  const auto load_k = [&](int ch) {
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    KR::template dma<2 * NW>(smem + (ch & 1) * L::one + L::K, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, part, lane);
  };
  const auto load_t = [&](int ch) {   // T, decays, values
    char* buf = smem + (ch & 1) * L::one;
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    dma_flat<2 * NW, WS::fP / 1024>(buf + L::I, a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per, part, lane);
    VR::template dma<2 * NW>(buf + L::V, v + t0 * a.vs[1], (int)(a.vs[1] * sizeof(T)), len, part, lane);
  };
  struct Mine {
    Fi<T, kNear> P[2][2];   // (the second of a pair: only tiles 2 and 3)
    float gam[2];
  };
  // queries go through LDS like the keys: a wave that loads 16 rows' pieces of 8 bytes
  // itself takes as long as all else together (64 heads of 64 chunks 252 us, this 214)
  const auto load_q = [&](int ch) {
    if constexpr (L::q_lds) {
      const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
      KR::template dma<2 * NW>(smem + L::Q + (ch & 1) * L::qone, q + t0 * a.qs[1], (int)(a.qs[1] * sizeof(T)), len, part, lane);
    }
  };
  const auto query = [&](int ch, int y, int p) {
    if constexpr (L::q_lds) {
      return KR::nat(smem + L::Q + (ch & 1) * L::qone, 2 * h + y, p, g, c);
    } else {
      const T* r = q + (size_t)min(ch * kGdrC + 16 * (2 * h + y) + c, sq.len - 1) * a.qs[1] + 32 * p + 4 * g;
      return Fr<T>{Quad<T>::ld(r), Quad<T>::ld(r + 16)};
    }
  };
  const auto load_p = [&](Mine& m, int ch) {
    const char* img = a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int i = 2 * h + y;
      m.P[y][0] = ld_img<T, kNear>(img + WS::fP, img_lower(i, 0), lane);
      if (h) m.P[y][1] = ld_img<T, kNear>(img + WS::fP, img_lower(i, 1), lane);
      m.gam[y] = reinterpret_cast<const float*>(img + WS::fScal)[kScGam * kGdrC + 16 * i + c];
    }
  };
  Mine cur, nxt;
  f32x4 xo[2];
  // (o^T of a chunk goes out an iteration later, before the loads: the wait at (1) covers
  // stores too)
  typename Quad<T>::q oq[2];
  const auto store_o = [&](int ch) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int t = ch * kGdrC + 16 * (2 * h + y) + c;
      if (t < sq.len) Quad<T>::st(o + (size_t)t * ors + 4 * g, oq[y]);
    }
  };
  if (nch > 0) {
    load_k(0);
    load_t(0);
    load_q(0);
  }
#pragma unroll 1
  for (int ch = 0; ch <= nch; ++ch) {
    vm_wait_all();
    __syncthreads();   // (1)
    f32x4 S[2 * NP], U[4];
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) S[j] = x[64 * (L::other * (ch & 1) + L::xS + j)];
#pragma unroll
    for (int i = 0; i < 4; ++i) U[i] = x[64 * (L::other * ((ch + 1) & 1) + (i < 2 ? L::xU + i : L::xW + i - 2))];
    if (!L::twice && ch < nch) __syncthreads();   // (2)
    if (ch > 1) store_o(ch - 2);
    if (ch + 1 < nch) {
      load_k(ch + 1);
      load_t(ch + 1);
      load_q(ch + 1);
    }
    cur = nxt;   // (the last chunk's P)
    if (ch < nch) load_p(nxt, ch);
    if (a.S_chunks && ch < nch) {
      float* s = a.S_chunks + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * sm + soff;
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j)
        if (j / NP == h) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    if (ch > 0) {   // o of the last chunk
      const Fi<T, kNear> Uf[2] = {to_fi<T, kNear>(U[0], U[1]), to_fi<T, kNear>(U[2], U[3])};
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        f32x4 z = mma<T>(Uf[0], cur.P[y][0], zero4());
        if (h) z = mma<T>(Uf[1], cur.P[y][1], z);
        oq[y] = Quad<T>::cvt((xo[y] * cur.gam[y] + z) * a.scale);
      }
    }
    if (ch < nch) {
      Fi<T, kNear> Sf[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) Sf[p] = to_fi<T, kNear>(S[2 * p], S[2 * p + 1]);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        xo[y] = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) xo[y] = mma<T>(Sf[p], query(ch, y, p), xo[y]);
      }
    }
  }
  if (nch > 0) store_o(nch - 1);
}

template <typename T, int DK, bool BWD>
int launch_prep_b(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = PrepLds<T, DK>::total;
  const auto kern = carve_gdr_prep_kernel<T, DK, BWD>;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CARVE_ERR_HIP;
  hipLaunchKernelGGL(kern, dim3(a.nslots, a.Hv), dim3(256), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK>
int launch_prep_t(const GdrArgs& a, bool bwd, hipStream_t s) {
  return bwd ? launch_prep_b<T, DK, true>(a, s) : launch_prep_b<T, DK, false>(a, s);
}
template <typename T>
int launch_chain_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = ChainLds<T>::total, NW = kChainNW;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_chain_kernel<T>;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CARVE_ERR_HIP;
  const unsigned heads = (unsigned)a.nseq * a.Hv;
  hipLaunchKernelGGL(kern, dim3(gdr_chain_grid(heads, a.Dv / (16 * NW))), dim3(128 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK, int NW>
int launch_pair_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = PairLds<T, DK, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_pair_kernel<T, DK, NW>;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CARVE_ERR_HIP;
  const unsigned heads = (unsigned)a.nseq * a.Hv;
  hipLaunchKernelGGL(kern, dim3(gdr_chain_grid(heads, a.Dv / (16 * NW))), dim3(256 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK>
int launch_fwd_t(const GdrArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  int st = launch_prep_t<T, DK>(a, false, s);
  if (st) return st;
  mark(s);
  if constexpr (DK == 32) st = launch_chain_t<T>(a, s);   // (one pair of key tiles: no halves)
  else st = gdr_few_tiles(a) ? launch_pair_t<T, DK, 1>(a, s) : launch_pair_t<T, DK, 2>(a, s);
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
