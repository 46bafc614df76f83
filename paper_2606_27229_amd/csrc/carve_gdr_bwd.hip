// carve_gdr_bwd.hip -- the chunked gated delta rule, backward for loss <dO, o> +
// <dS_T, S_T>.  With dO' = scale dO, E_t = e^{G_C - G_t} and, per chunk, the start
// state S (kept by the forward) and the gradient dS of the end state:
//   dU = P^T dO' + E K dS^T,  dR = T^T dU,  dV = beta dR
//   dS <- e^{G_C} dS + dO'^T (e^G Q) - (beta e^G dR)^T K           (the chain)
//   dP = dO' U^T (j <= i),  dA = - dR U^T (j < i),  M = beta D dA
//   dQ = e^G dO' S + (D dP) K
//   dK = (D dP)^T Q + M K + M^T K + E U dS - beta e^G dR S
//   dbeta_t = dR_t.V_t - e^{G_t} k_t.(dR S)_t + sum_j dA_tj D_tj k_t.k_j
//   dg_t = sum_{i >= t} (q_i.(e^G dO' S)_i - k_i.(beta e^G dR S)_i) + sum_{i >= t > j} (dP P + dA A)_ij
//          + sum_{j < t} k_j.(E U dS)_j + e^{G_C} <dS, S>
// (each sum over what the decay at t multiplies, and nothing else: every term holds e^{g_t})
// Three launches: the triangles (carve_gdr_prep_kernel), the chain of state
// gradients, then every chunk's gradients at once.
#include "carve_gdr.h"

namespace carve {
namespace {

// ---------------------------------------------------------------------------------
// The chain of state gradients, the mirror of the forward's (carve_gdr_chain_kernel), from
// the last chunk to the first.  Two waves a tile of 16 value columns:
//   chain   dU = z + E K dS^T, dR = T^T dU, dS^T <- e^{G_C} dS^T + Y - K^T (beta e^G dR);
//           dS of every chunk's end and dR go out
//   helper  what does not need dS, one chunk ahead: z = P^T dO' and Y = Q^T (e^G dO');
//           it loads the next chunk's rows
// z and Y pass through LDS as they lie in registers.  Barriers, two a chunk: (1) z, Y and
// the chunk's rows are there; (2) the chain has taken z and Y.
// Two tiles a workgroup (keys of 32), or four where there are many (gdr_many_tiles).
template <typename T, int DK, int NW>
struct BChainLds {
  typedef GdrRows<T, DK> KR;
  static constexpr bool q_lds = sizeof(T) == 2 || DK < 128;       // (f32 queries of 128: from memory)
  static constexpr int K0 = 0, I = KR::bytes;                     // I: scalars, then T^T
  static constexpr int one = I + kGdrScal + GdrWs<T>::I3;
  static constexpr int Q = 2 * one, qone = q_lds ? KR::bytes : 0;
  static constexpr int xz = Q + 2 * qone, xY = xz + NW * 4 * 1024;
  static constexpr int total = xY + NW * (DK / 16) * 1024;
};

template <typename T, int DK, int NW>
__global__ void __launch_bounds__(128 * NW, 1) carve_gdr_bchain_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef BChainLds<T, DK, NW> L;
  typedef typename L::KR KR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool helper = wave >= NW;
  const int w = helper ? wave - NW : wave;
  const int g = lane >> 4, c = lane & 15;
  int n, hv, slice;
  if (!gdr_chain_block(a, a.Dv / (16 * NW), n, hv, slice)) return;
  const int hk = hv / (a.Hv / a.Hk), head = n * a.Hv + hv;
  const int v0 = 16 * (NW * slice + w);
  const GdrSeq sq = gdr_seq(a, n);
  const size_t sm = (size_t)a.Dv * DK, soff = (size_t)(v0 + c) * DK + 4 * g;
  const int nch = (sq.len + kGdrC - 1) / kGdrC;
  f32x4* xz = reinterpret_cast<f32x4*>(smem + L::xz + w * 4 * 1024) + lane;
  f32x4* xY = reinterpret_cast<f32x4*>(smem + L::xY + w * (DK / 16) * 1024) + lane;

  if (!helper) {
    f32x4 S[2 * NP];
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j)
      S[j] = a.dS_T ? *reinterpret_cast<const f32x4*>(a.dS_T + (size_t)head * sm + soff + 16 * j) : zero4();
    if (nch > 0) __syncthreads();   // (0)
#pragma unroll 1
    for (int ch = nch - 1; ch >= 0; --ch) {
      const char* buf = smem + (ch & 1) * L::one;
      const float* scal = reinterpret_cast<const float*>(buf + L::I);
      const size_t sh = (size_t)(sq.slot0 + ch) * a.Hv + hv;
      __syncthreads();   // (1)
      f32x4 U[4];
      Fi<T, kExact> Sf[NP];
      const float gend = scal[kScGam * kGdrC + kGdrC - 1];
      float* out = a.dS_chunks + sh * sm + soff;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        Sf[p] = to_fi<T, kExact>(S[2 * p], S[2 * p + 1]);
#pragma unroll
        for (int j = 2 * p; j < 2 * p + 2; ++j) {
          *reinterpret_cast<f32x4*>(out + 16 * j) = S[j];
          S[j] = S[j] * gend + xY[64 * j];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) U[i] = xz[64 * i];
      __syncthreads();   // (2)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 y = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) y = mma<T>(KR::nat(buf + L::K0, i, p, g, c), Sf[p], y);
        U[i] += y * *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
      }
      const Fi<T, kExact> Uf[2] = {to_fi<T, kExact>(U[0], U[1]), to_fi<T, kExact>(U[2], U[3])};
      f32x4 R[4];
      float* keep = a.dR + (sh * (a.Dv / 16) + v0 / 16) * 1024 + 4 * lane;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 x = zero4();
#pragma unroll
        for (int s = i / 2; s < 2; ++s)
          x = mma<T>(ld_img<T, kExact>(buf + L::I + kGdrScal, img_upper(i, s), lane), Uf[s], x);
        *reinterpret_cast<f32x4*>(keep + 256 * i) = x;
        const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
        const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
        R[i] = -(x * (gam * be));
      }
      const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(R[0], R[1]), to_fi<T, kExact>(R[2], R[3])};
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s) S[j] = mma<T>(KR::tr32(buf + L::K0, s, j, g, c), Rf[s], S[j]);
    }
    if (a.dS0) {
      float* s = a.dS0 + (size_t)head * sm + soff;
#pragma unroll
      for (int j = 0; j < 2 * NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    return;
  }

  // ---- helper
  if (nch == 0) return;   // (no barriers then)
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + sq.t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + sq.t0 * a.ks[1] + hk * a.ks[2];
  const T* dO = reinterpret_cast<const T*>(a.dO) + (((size_t)sq.batch * a.T + sq.t0) * a.Hv + hv) * a.Dv + v0 + c;
  const size_t ors = (size_t)a.Hv * a.Dv;
  const auto ws_of = [&](int ch) { return a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per; };
  const auto load = [&](int ch) {
    char* buf = smem + (ch & 1) * L::one;
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    KR::template dma<NW>(buf + L::K0, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, w, lane);
    dma_flat<NW, kGdrScal / 1024>(buf + L::I, ws_of(ch) + WS::bScal, w, lane);
    dma_flat<NW, WS::I3 / 1024>(buf + L::I + kGdrScal, ws_of(ch) + WS::bTt, w, lane);
  };
  const auto load_q = [&](int ch) {
    if constexpr (L::q_lds) {
      const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
      KR::template dma<NW>(smem + L::Q + (ch & 1) * L::qone, q + t0 * a.qs[1], (int)(a.qs[1] * sizeof(T)), len, w, lane);
    }
  };
  struct Mine {
    typename Quad<T>::q od[4];   // dO[t][v]: tokens 16 i + 4 g + e of column c
    Fi<T, kExact> Pt[6];
    f32x4 gam[4];
  };
  const auto load_m = [&](Mine& m, int ch) {
    const char* ws = ws_of(ch);
#pragma unroll
    for (int f = 0; f < 6; ++f) m.Pt[f] = ld_img<T, kExact>(ws + WS::bPt, f, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m.gam[i] = *reinterpret_cast<const f32x4*>(ws + WS::bScal + 4 * (kScGam * kGdrC + 16 * i + 4 * g));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (past the end: the last token, zeroed where it is used)
        m.od[i][e] = dO[(size_t)min(ch * kGdrC + 16 * i + 4 * g + e, sq.len - 1) * ors];
      }
    }
  };
  // z and Y of a chunk into LDS
  const auto work = [&](Mine& m, int ch) {
    const int len = sq.len - ch * kGdrC;
    f32x4 od[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (len < kGdrC)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * i + 4 * g + e >= len) m.od[i][e] = (T)0.0f;
      od[i] = Quad<T>::f32(m.od[i]) * (m.gam[i] * a.scale);
    }
    const Fr<T> of[2] = {{m.od[0], m.od[1]}, {m.od[2], m.od[3]}};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 x = zero4();
#pragma unroll
      for (int s = i / 2; s < 2; ++s) x = mma<T>(m.Pt[img_upper(i, s)], of[s], x);
      xz[64 * i] = x * a.scale;
    }
    const Fi<T, kExact> Of[2] = {to_fi<T, kExact>(od[0], od[1]), to_fi<T, kExact>(od[2], od[3])};
#pragma unroll
    for (int j = 0; j < 2 * NP; ++j) {
      f32x4 x = zero4();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        Fr<T> f;
        if constexpr (L::q_lds) {
          f = KR::tr32(smem + L::Q + (ch & 1) * L::qone, s, j, g, c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = ch * kGdrC + 32 * s + 4 * g + e;
            f.a[e] = q[(size_t)min(t, sq.len - 1) * a.qs[1] + 16 * j + c];
            f.b[e] = q[(size_t)min(t + 16, sq.len - 1) * a.qs[1] + 16 * j + c];
          }
        }
        x = mma<T>(f, Of[s], x);
      }
      xY[64 * j] = x;
    }
  };
  constexpr bool AHEAD = NW == 2 && sizeof(T) == 2;
  Mine cur, nxt;
  load(nch - 1);
  load_q(nch - 1);
  load_m(cur, nch - 1);
  vm_wait_all();
  __syncthreads();   // (0) the helpers' shares of the queries
  work(cur, nch - 1);
  if (nch > 1) {
    load_q(nch - 2);
    if constexpr (AHEAD) load_m(nxt, nch - 2);
  }
#pragma unroll 1
  for (int ch = nch - 1; ch >= 0; --ch) {
    vm_wait_all();
    __syncthreads();   // (1)
    __syncthreads();   // (2)
    if (ch == 0) break;
    load(ch - 1);
    if (ch > 1) load_q(ch - 2);
    if constexpr (AHEAD) {
      cur = nxt;
      if (ch > 1) load_m(nxt, ch - 2);
    } else {
      load_m(cur, ch - 1);
    }
    work(cur, ch - 1);
  }
}

// ---------------------------------------------------------------------------------
// The same chain with two waves a tile on it and two helpers, the mirror of
// carve_gdr_pair_kernel.  Chain wave h keeps dS of the keys' half h, finishes dU of the
// token tiles 2 h, 2 h + 1 and multiplies by T^T's columns of these tokens.  Helper wave
// h forms z of the same token tiles and Y of the same keys.
// Barriers (1) and, without LDS for z and Y of two chunks in turn, (2) as above; the chain
// waves of a tile meet by flags: (3)
// the halves of K dS^T are there; (4) the parts of dR.  Bound by the chunks following each
// other, 4.7 us each at 128 keys and values in bf16, where the 400 MB that go out (64
// sequences and heads of 64 chunks: 300 us) alone take 80 us; one chain wave: 372 us.
template <typename T, int DK, int NW>   // NW: tiles
struct BPairLds {
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, 32> VR;    // (with one tile, its neighbour's columns too)
  static constexpr bool q_lds = sizeof(T) == 2 || DK < 128;       // (f32 queries of 128: from memory)
  static constexpr int K0 = 0, I = KR::bytes;                     // I: scalars, then T^T
  static constexpr int one = I + kGdrScal + GdrWs<T>::I3;
  static constexpr int Q = 2 * one, qone = q_lds ? KR::bytes : 0;
  static constexpr int O = Q + 2 * qone, x = O + 2 * VR::bytes;   // O: dO of the workgroup's columns
  // KB of a tile: z, Y; with room for it once more, for the other parity of the chunk; the
  // halves of K dS^T that the other wave takes, dR of wave 1 (its first two tiles without
  // wave 0's part), that part
  static constexpr int xz = 0, xY = 4, in = xY + DK / 16;
  static constexpr bool twice = x + NW * ((2 * in + 10) * 1024 + 16) <= 160 * 1024;
  static constexpr int other = twice ? in : 0, xP = in + other, xU = xP + 4, xV = xU + 4, kb = xV + 2;
  static constexpr int flags = x + NW * kb * 1024, total = flags + NW * 16;
};

template <typename T, int DK, int NW>
__global__ void __launch_bounds__(256 * NW, 1) carve_gdr_bpair_kernel(GdrArgs a) {
  constexpr int NP = DK / 32;
  typedef BPairLds<T, DK, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef GdrWs<T> WS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool helper = wave >= 2 * NW;
  const int w = (wave >> 1) & (NW - 1), h = wave & 1;
  const int g = lane >> 4, c = lane & 15;
  int n, hv, slice;
  if (!gdr_chain_block(a, a.Dv / (16 * NW), n, hv, slice)) return;
  const int hk = hv / (a.Hv / a.Hk), head = n * a.Hv + hv;
  const int v0 = 16 * (NW * slice + w);
  const GdrSeq sq = gdr_seq(a, n);
  const int vt0 = v0 & 16 ? 1 : 0;   // tile of dO's columns
  const size_t sm = (size_t)a.Dv * DK, soff = (size_t)(v0 + c) * DK + 16 * NP * h + 4 * g;
  const int nch = (sq.len + kGdrC - 1) / kGdrC;
  f32x4* x = reinterpret_cast<f32x4*>(smem + L::x + w * L::kb * 1024) + lane;

  lds_flag* flags = (lds_flag*)lds_at(smem + L::flags + 16 * w);

  if (!helper) {
    flags[h] = 0;   // (seen by the other wave behind the first barrier)
    f32x4 S[NP];   // key tiles NP h ..
#pragma unroll
    for (int j = 0; j < NP; ++j)
      S[j] = a.dS_T ? *reinterpret_cast<const f32x4*>(a.dS_T + (size_t)head * sm + soff + 16 * j) : zero4();
    if (nch > 0) __syncthreads();   // (0)
#pragma unroll 1
    for (int ch = nch - 1; ch >= 0; --ch) {
      const char* buf = smem + (ch & 1) * L::one;
      const float* scal = reinterpret_cast<const float*>(buf + L::I);
      const size_t sh = (size_t)(sq.slot0 + ch) * a.Hv + hv;
      const f32x4* const xi = x + 64 * L::other * (ch & 1);   // this chunk's z and Y
      __syncthreads();   // (1)
      const float gend = scal[kScGam * kGdrC + kGdrC - 1];
      float* out = a.dS_chunks + sh * sm + soff;
      Fi<T, kExact> Sf[NP / 2];
#pragma unroll
      for (int p = 0; p < NP / 2; ++p) {
        Sf[p] = to_fi<T, kExact>(S[2 * p], S[2 * p + 1]);
#pragma unroll
        for (int j = 2 * p; j < 2 * p + 2; ++j) {
          *reinterpret_cast<f32x4*>(out + 16 * j) = S[j];
          S[j] = S[j] * gend + xi[64 * (L::xY + NP * h + j)];
        }
      }
      f32x4 U[2] = {xi[64 * (L::xz + 2 * h)], xi[64 * (L::xz + 2 * h + 1)]};
      if (!L::twice) __syncthreads();   // (2)
      f32x4 acc[4];      // the other wave's two token tiles, then this one's
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int i = (2 * (1 - h) + y) & 3;
        acc[y] = zero4();
#pragma unroll
        for (int p = 0; p < NP / 2; ++p) acc[y] = mma<T>(KR::nat(buf + L::K0, i, NP / 2 * h + p, g, c), Sf[p], acc[y]);
        if (y < 2) x[64 * (L::xP + 2 * h + y)] = acc[y];
      }
      // (what a step needs besides the other wave's part is read before the two meet)
      f32x4 end[2];
      Fi<T, kExact> Tf[4];
#pragma unroll
      for (int y = 0; y < 2; ++y) end[y] = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * (2 * h + y) + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < 2 || h) Tf[i] = ld_img<T, kExact>(buf + L::I + kGdrScal, img_upper(i, h), lane);   // (uniform)
      pair_meet(flags, h, 2 * (nch - 1 - ch) + 1);   // (3)
#pragma unroll
      for (int y = 0; y < 2; ++y) U[y] += (acc[2 + y] + x[64 * (L::xP + 2 * (1 - h) + y)]) * end[y];
      const Fi<T, kExact> Uf = to_fi<T, kExact>(U[0], U[1]);
      f32x4 R[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= 2 && !h) continue;   // (uniform)
        R[i] = mma<T>(Tf[i], Uf, zero4());
        x[64 * (h ? L::xU + i : L::xV + i)] = R[i];
      }
      f32x4 gb[4];
      Fr<T> Kt[NP][2];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        gb[i] = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g) *
                *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s) Kt[j][s] = KR::tr32(buf + L::K0, s, NP * h + j, g, c);
      pair_meet(flags, h, 2 * (nch - 1 - ch) + 2);   // (4)
      // dR whole; tiles 2 h, 2 h + 1 of it go out
      float* keep = a.dR + (sh * (a.Dv / 16) + v0 / 16) * 1024 + 4 * lane + 512 * h;
      if (h) {
        R[0] += x[64 * L::xV];
        R[1] += x[64 * (L::xV + 1)];
        *reinterpret_cast<f32x4*>(keep) = R[2];
        *reinterpret_cast<f32x4*>(keep + 256) = R[3];
      } else {
        R[0] += x[64 * L::xU];
        R[1] += x[64 * (L::xU + 1)];
        R[2] = x[64 * (L::xU + 2)];
        R[3] = x[64 * (L::xU + 3)];
        *reinterpret_cast<f32x4*>(keep) = R[0];
        *reinterpret_cast<f32x4*>(keep + 256) = R[1];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) R[i] *= -gb[i];
      const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(R[0], R[1]), to_fi<T, kExact>(R[2], R[3])};
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s) S[j] = mma<T>(Kt[j][s], Rf[s], S[j]);
    }
    if (a.dS0) {
      float* s = a.dS0 + (size_t)head * sm + soff;
#pragma unroll
      for (int j = 0; j < NP; ++j) *reinterpret_cast<f32x4*>(s + 16 * j) = S[j];
    }
    return;
  }

  // ---- helper
  if (nch == 0) return;   // (no barriers then)
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + sq.t0 * a.qs[1] + hk * a.qs[2];
  const T* k = reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + sq.t0 * a.ks[1] + hk * a.ks[2];
  const T* dO = reinterpret_cast<const T*>(a.dO) + (((size_t)sq.batch * a.T + sq.t0) * a.Hv + hv) * a.Dv + (v0 & ~31);
  const size_t ors = (size_t)a.Hv * a.Dv;
  const int part = wave - 2 * NW;
  const auto ws_of = [&](int ch) { return a.ws + ((size_t)(sq.slot0 + ch) * a.Hv + hv) * a.per; };
  const auto load = [&](int ch) {
    char* buf = smem + (ch & 1) * L::one;
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    KR::template dma<2 * NW>(buf + L::K0, k + t0 * a.ks[1], (int)(a.ks[1] * sizeof(T)), len, part, lane);
    dma_flat<2 * NW, kGdrScal / 1024>(buf + L::I, ws_of(ch) + WS::bScal, part, lane);
    dma_flat<2 * NW, WS::I3 / 1024>(buf + L::I + kGdrScal, ws_of(ch) + WS::bTt, part, lane);
  };
  const auto load_q = [&](int ch) {   // and dO
    const int t0 = ch * kGdrC, len = min(kGdrC, sq.len - t0);
    VR::template dma<2 * NW>(smem + L::O + (ch & 1) * VR::bytes, dO + t0 * ors, (int)(ors * sizeof(T)), len, part, lane);
    if constexpr (L::q_lds) {
      KR::template dma<2 * NW>(smem + L::Q + (ch & 1) * L::qone, q + t0 * a.qs[1], (int)(a.qs[1] * sizeof(T)), len, part,
                               lane);
    }
  };
  struct Mine {
    Fi<T, kExact> Pt[2][2];      // (the second of a pair: only tiles 0 and 1)
    f32x4 gam[4];
  };
  const auto load_m = [&](Mine& m, int ch) {
    const char* ws = ws_of(ch);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int i = 2 * h + y;
      m.Pt[y][0] = ld_img<T, kExact>(ws + WS::bPt, img_upper(i, h ? 1 : 0), lane);
      if (!h) m.Pt[y][1] = ld_img<T, kExact>(ws + WS::bPt, img_upper(i, 1), lane);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m.gam[i] = *reinterpret_cast<const f32x4*>(ws + WS::bScal + 4 * (kScGam * kGdrC + 16 * i + 4 * g));
  };
  typename Quad<T>::q od[4];   // dO[t][v]: tokens 16 i + 4 g + e of column c, zeros behind the last
  const auto work_z = [&](Mine& m, int ch) {
    const int len = sq.len - ch * kGdrC;
#pragma unroll
    for (int i = 0; i < 4; ++i) od[i] = VR::tr(smem + L::O + (ch & 1) * VR::bytes, 16 * i, vt0, g, c);
    if (len < kGdrC)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * i + 4 * g + e >= len) od[i][e] = (T)0.0f;
    const Fr<T> of[2] = {{od[0], od[1]}, {od[2], od[3]}};
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      f32x4 z = zero4();
      if (h) {
        z = mma<T>(m.Pt[y][0], of[1], z);
      } else {
        z = mma<T>(m.Pt[y][0], of[0], z);
        z = mma<T>(m.Pt[y][1], of[1], z);
      }
      x[64 * (L::other * (ch & 1) + L::xz + 2 * h + y)] = z * a.scale;
    }
  };
  const auto work_Y = [&](Mine& m, int ch) {
    f32x4 og[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) og[i] = Quad<T>::f32(od[i]) * (m.gam[i] * a.scale);
    const Fi<T, kExact> Of[2] = {to_fi<T, kExact>(og[0], og[1]), to_fi<T, kExact>(og[2], og[3])};
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      f32x4 y = zero4();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        Fr<T> f;
        if constexpr (L::q_lds) {
          f = KR::tr32(smem + L::Q + (ch & 1) * L::qone, s, NP * h + j, g, c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = ch * kGdrC + 32 * s + 4 * g + e;
            f.a[e] = q[(size_t)min(t, sq.len - 1) * a.qs[1] + 16 * (NP * h + j) + c];
            f.b[e] = q[(size_t)min(t + 16, sq.len - 1) * a.qs[1] + 16 * (NP * h + j) + c];
          }
        }
        y = mma<T>(f, Of[s], y);
      }
      x[64 * (L::other * (ch & 1) + L::xY + NP * h + j)] = y;
    }
  };
  Mine cur, nxt;
  load(nch - 1);
  load_q(nch - 1);
  load_m(cur, nch - 1);
  vm_wait_all();
  __syncthreads();   // (0) the helpers' shares of the queries
  work_z(cur, nch - 1);
  work_Y(cur, nch - 1);
  if (nch > 1) {
    load_q(nch - 2);
    load_m(nxt, nch - 2);
  }
#pragma unroll 1
  for (int ch = nch - 1; ch >= 0; --ch) {
    vm_wait_all();
    __syncthreads();   // (1)
    if (!L::twice) __syncthreads();   // (2)
    if (ch > 0) {
      load(ch - 1);
      cur = nxt;
      if (ch > 1) {
        load_q(ch - 2);
        load_m(nxt, ch - 2);
      }
    }
    if (ch > 0) {
      work_z(cur, ch - 1);
      work_Y(cur, ch - 1);
    }
  }
}

// ---------------------------------------------------------------------------------
// Gradients of one chunk and key head (its value heads one after another, dq and dk
// summed in registers).  Eight waves, per value head and block of VB value columns:
//   1. wave w: value columns 16 w ..: U again from S, beside dR from the chain; both
//      into LDS as pieces, transposed; sums over the value columns
//   2. products over the value columns: dP and dA, tile by tile (lower tiles only),
//      and dO' S, U dS, dR S for the wave's key columns
// then, all columns done, D dP and M through LDS into dQ and dK.
// dg is an f32 result: what reaches it (dP, dA, dO' S and U dS by their sums with q
// and k) is taken in three pieces; k.(dR S) is dR.(S k), summed where S k is at hand,
// so that dR S itself only reaches dk and is taken in two.
// LDS: U and dR in three pieces fill 96 KB at 128 columns, so the rest shares places:
// the values lie where U goes, the queries where T was.
// 4096 chunks and heads of 128 keys and values in bf16: 475 us for 1.5 GB, 3.2 TB/s.  Bound
// by one workgroup a compute unit (158 KB): its loads, its LDS reads (three pieces an
// operand) and its matrix products do not overlap beyond what two waves a SIMD give (vector
// units 38 %, matrix cores 17 % of the cycles).  0.4 GB of the traffic are registers that do
// not fit, 21 a lane here, 17 to 91 at 128 keys: dQ and dK live across the loop over the
// value heads.  With narrower keys none spill.  One workgroup a chunk and key head takes its
// value heads one after another, so a call takes whole turns of 256 such workgroups (5
// documents of 8191 tokens with 4 key heads: 528 of them, a third turn for 16).  Taken from
// memory without LDS, the token rows made it 5.4 ms.

// [VB columns][64 tokens] of an f32 intermediate in LDS
template <typename T, int VB>
struct InterT {
  static constexpr int LD = sizeof(T) == 2 ? kGdrC : kGdrC + 4;
  static constexpr int plane = VB * LD;
  static __host__ __device__ constexpr int bytes(int n) { return plane * (sizeof(T) == 2 ? 2 * n : 4); }
  // bf16 rows of 64 elements: quad y of column r at quad y ^ sw(r), which spreads the
  // 16 columns of a quad write or read, and the 8 columns x 4 quads of a read across
  // columns, over all banks
  static __device__ __forceinline__ int sw(int r) { return (((r >> 1) & 3) << 2) | (((r >> 3) & 1) << 1) | (r & 1); }
  // the four tokens 16 i + 4 g .. of column col, in N pieces
  template <int N>
  static __device__ __forceinline__ void put(char* m, int col, int i, int g, f32x4 x) {
    T* p = reinterpret_cast<T*>(m) + col * LD;
    if constexpr (sizeof(T) == 2) {
      p += 4 * ((4 * i + g) ^ sw(col));
#pragma unroll
      for (int y = 0; y < N; ++y) {
        const typename Quad<T>::q h = Quad<T>::cvt(x);
        Quad<T>::st(p + y * plane, h);
        if (y + 1 < N) x = bf16_rest(x, h);
      }
    } else {
      Quad<T>::st(p + 16 * i + 4 * g, x);
    }
  }
  // lane (g, c): token 16 i + c, columns col0 + 4 g + e and col0 + 16 + 4 g + e
  template <int N>
  static __device__ __forceinline__ Fi<T, N> tok(const char* m, int i, int col0, int g, int c) {
    const T* p = reinterpret_cast<const T*>(m);
    Fi<T, N> f;
    if constexpr (sizeof(T) == 2) {
      const int r = 4 * g + (c >> 2);
      p += (col0 + r) * LD + 4 * ((4 * i + (c & 3)) ^ sw(r));
#pragma unroll
      for (int y = 0; y < N; ++y) {
        f.x[y].a = Quad<T>::ld_tr_at(p + y * plane);
        f.x[y].b = Quad<T>::ld_tr_at(p + y * plane + 16 * LD);
      }
    } else {
      f.x[0].a = Quad<T>::ld_tr(p, LD, col0, 16 * i, g, c);
      f.x[0].b = Quad<T>::ld_tr(p, LD, col0 + 16, 16 * i, g, c);
    }
    return f;
  }
  // lane (g, c): token 16 i + c, the eight columns col0 + 8 g .., as f32 sums of N pieces
  template <int N>
  static __device__ __forceinline__ void eight(const char* m, int i, int col0, int g, int c, f32x4& lo, f32x4& hi) {
    const T* p = reinterpret_cast<const T*>(m);
    lo = hi = zero4();
    if constexpr (sizeof(T) == 2) {
      const int r = col0 + 8 * g + (c >> 2);
#pragma unroll
      for (int y = N - 1; y >= 0; --y) {
        lo += Quad<T>::f32(Quad<T>::ld_tr_at(p + y * plane + r * LD + 4 * ((4 * i + (c & 3)) ^ sw(r))));
        hi += Quad<T>::f32(Quad<T>::ld_tr_at(p + y * plane + (r + 4) * LD + 4 * ((4 * i + (c & 3)) ^ sw(r + 4))));
      }
    } else {
      const T* q = p + (col0 + 8 * g) * LD + 16 * i + c;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = q[e * LD];
        hi[e] = q[(4 + e) * LD];
      }
    }
  }
  // lane (g, c): column col0 + c, tokens 32 s + 4 g + e and 32 s + 16 + 4 g + e
  template <int N>
  static __device__ __forceinline__ Fi<T, N> col(const char* m, int col0, int s, int g, int c) {
    const T* p = reinterpret_cast<const T*>(m) + (col0 + c) * LD;
    Fi<T, N> f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int y = 0; y < N; ++y) {
        f.x[y].a = Quad<T>::ld(p + y * plane + 4 * ((8 * s + g) ^ sw(c)));
        f.x[y].b = Quad<T>::ld(p + y * plane + 4 * ((8 * s + 4 + g) ^ sw(c)));
      }
    } else {
      f.x[0].a = Quad<T>::ld(p + 32 * s + 4 * g);
      f.x[0].b = Quad<T>::ld(p + 32 * s + 16 + 4 * g);
    }
    return f;
  }
};

template <typename T, int DK, int VB>
struct GradLds {
  typedef GdrRows<T, DK> KR;
  typedef GdrRows<T, VB> VR;
  typedef InterT<T, VB> UT;
  typedef InterT<T, kGdrC> WT;
  static constexpr int U = 0, R = U + UT::bytes(kExact), V = U;
  static constexpr int W = U, M = W + WT::bytes(kNear);       // (D dP)^T, M^T: [j][i], over U and dR
  static constexpr int ur = 2 * UT::bytes(kExact) > 2 * WT::bytes(kNear) ? 2 * UT::bytes(kExact) : 2 * WT::bytes(kNear);
  static constexpr int K = ur > VR::bytes ? ur : VR::bytes;
  static constexpr int O = K + KR::bytes;
  static constexpr int scal = O + VR::bytes;
  static constexpr int Z = scal + kGdrScal;                    // T, then Q
  static constexpr int red = Z + (KR::bytes > GdrWs<T>::I3 ? KR::bytes : GdrWs<T>::I3);
  // sums over values, [wave][64]: dR.(V - e^G S k), dR.(e^G S k); over keys, [key tile]
  // [64]: q.(dO' S), k.(U dS); <dS, S> per wave; over tiles, [4][64]: rows of dP P + dA
  // A (of the diagonal tiles, sums over i >= t > j), rows of dA A / beta, columns of dP P +
  // dA A
  static constexpr int floats = 4 * 8 * kGdrC + 8 + 3 * 4 * kGdrC;
  static constexpr int total = red + floats * 4;
};

// NB: blocks of VB value columns (with one, no product has to live through another block's
// first part).  As many columns at once as LDS holds: 2 x 4096 tokens of 16 heads of 128 keys
// and values 249 us, in two blocks 325; 256 values of 8 heads in two 230, in four 246; 64
// values of 4 x 4096 tokens 374, in two 505.
template <typename T, int DK, int VB, int NB>
__global__ void __launch_bounds__(512, 1) carve_gdr_grad_kernel(GdrArgs a) {
  typedef GradLds<T, DK, VB> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  typedef typename L::UT UT;
  typedef typename L::WT WT;
  constexpr int NP = DK / 32;
  constexpr int NJ = DK / 16;      // key tiles
  constexpr int NI = NJ / 2;       // row tiles of a wave in the products over key columns
  constexpr int NV = VB / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const float* scal = reinterpret_cast<const float*>(smem + L::scal);
  float* rRV = reinterpret_cast<float*>(smem + L::red);   // [8][64]
  float* rRK = rRV + 8 * kGdrC;            // [8][64]
  float* rQ = rRK + 8 * kGdrC;             // [8][64]
  float* rUK = rQ + 8 * kGdrC;             // [8][64]
  float* rSS = rUK + 8 * kGdrC;            // [8]
  float* rRow = rSS + 8;                   // [4][64]
  float* rBeta = rRow + 4 * kGdrC;         // [4][64]
  float* rCol = rBeta + 4 * kGdrC;         // [4][64]
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int g = lane >> 4, c = lane & 15;
  const int slot = blockIdx.x, hk = blockIdx.y, grp = a.Hv / a.Hk;
  GdrSeq sq;
  int n, chunk;
  if (!gdr_find(a, slot, sq, n, chunk)) return;   // (uniform)
  const int t0 = sq.t0 + chunk * kGdrC, len = min(kGdrC, sq.len - chunk * kGdrC);
  const size_t row0 = (size_t)sq.batch * a.T + t0;
  const size_t sm = (size_t)a.Dv * DK;
  const size_t ors = (size_t)a.Hv * a.Dv;
  const T* q = reinterpret_cast<const T*>(a.q) + sq.batch * a.qs[0] + t0 * a.qs[1] + hk * a.qs[2];
  KR::template dma<8>(smem + L::K, reinterpret_cast<const T*>(a.k) + sq.batch * a.ks[0] + t0 * a.ks[1] + hk * a.ks[2],
          (int)(a.ks[1] * sizeof(T)), len, w, lane);

  // this wave's key tile and row tiles
  const int jt = w % NJ, i0 = NI * (w / NJ);
  f32x4 dQ[NI], dK[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) dQ[i] = dK[i] = zero4();

  // dbeta and dg of a value head, by one wave
  const auto finish = [&](int hv) {
    const int t = lane;
    float rv1 = 0.0f, rk1 = 0.0f, s1 = 0.0f, s2 = 0.0f, sss = 0.0f, row = 0.0f, rb = 0.0f, col = 0.0f;
    for (int x = 0; x < VB / 16; ++x) {
      rv1 += rRV[x * kGdrC + t];
      rk1 += rRK[x * kGdrC + t];
    }
    for (int x = 0; x < 8; ++x) sss += rSS[x];
    for (int x = 0; x < NJ; ++x) {
      s1 += rQ[x * kGdrC + t];
      s2 += rUK[x * kGdrC + t];
    }
    // (read whole, so that the reads wait for each other once; upper tiles hold nothing)
    f32x4 rows, betas, cols;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      rows[x] = rRow[x * kGdrC + t];
      betas[x] = rBeta[x * kGdrC + t];
      cols[x] = rCol[x * kGdrC + t];
    }
    float diag = rows[0];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      rb += x <= t / 16 ? betas[x] : 0.0f;
      row += x < t / 16 ? rows[x] : 0.0f;
      col += x > t / 16 ? cols[x] : 0.0f;
      if (x == t / 16) diag = rows[x];
    }
    const float be = scal[kScBeta * kGdrC + t];
    // dg_t: over i >= t what token i reads of the start state, over j < t the writes that
    // the end state keeps, and the pairs i >= t > j.  (As a suffix sum of dG alone, with a
    // pair a row term of G_i and a column term of G_j, the pairs that a decay at t leaves
    // alone would only cancel up to their rounding: nothing would be left of a small dg.)
    // The pairs by tiles (I, J): the diagonal tile's; I = t's, J before it, rows from t on;
    // J = t's, I behind it, columns before t; and whole tiles around t's.
    const float y0 = t >= 16 ? rows[0] : 0.0f, y1 = t >= 32 ? rows[1] : 0.0f;
    const auto of_lane = [](float x, int l) {
      return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
    };
    const float z0 = row_suffix(y0), z1 = row_suffix(y1);   // (whole tiles at their first rows)
    const float t30 = of_lane(z0, 48), in1 = of_lane(z0, 32) + t30, in2 = t30 + of_lane(z1, 48);
    float pairs = diag + row_suffix(row) + dpp<0x111>(row_scan(col));   // (0x111: of the lane before)
    pairs += t / 16 == 1 ? in1 : t / 16 == 2 ? in2 : 0.0f;
    float after = t < len ? s1 - be * rk1 : 0.0f;
    float before = __shfl_up(s2, 1);
    if (t == 0) before = 0.0f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const float x = __shfl_down(after, d), y = __shfl_up(before, d);
      if (t + d < 64) after += x;
      if (t >= d) before += y;
    }
    const float ends = scal[kScGam * kGdrC + kGdrC - 1] * sss;
    if (t < len) {
      a.dg[(row0 + t) * a.Hv + hv] = after + before + ends + pairs;
      reinterpret_cast<T*>(a.dbeta)[(row0 + t) * a.Hv + hv] = (T)(rv1 + rb);
    }
  };

  for (int hv = hk * grp; hv < (hk + 1) * grp; ++hv) {
    const size_t sh = (size_t)slot * a.Hv + hv;
    f32x4 aP[2], aA[2];                     // tile tasks w and w + 8 (of ten)
    f32x4 a1[NI], a2[NI], a3[NI];           // dO S, U dS, dR S
    float ss = 0.0f;
    const auto clear = [&] {
#pragma unroll
      for (int x = 0; x < 2; ++x) aP[x] = aA[x] = zero4();
#pragma unroll
      for (int i = 0; i < NI; ++i) a1[i] = a2[i] = a3[i] = zero4();
    };
    if (NB > 1) clear();

#pragma unroll 1
    for (int b = 0; b < NB; ++b) {
      const int vb = b * VB;
      // ---- 1. U and dR of columns vb + 16 w ..
      renew(g, c);
      const T* dO = reinterpret_cast<const T*>(a.dO) + (row0 * a.Hv + hv) * a.Dv + vb;
      VR::template dma<8>(smem + L::V, reinterpret_cast<const T*>(a.v) + sq.batch * a.vs[0] + t0 * a.vs[1] + hv * a.vs[2] + vb,
              (int)(a.vs[1] * sizeof(T)), len, w, lane);
      VR::template dma<8>(smem + L::O, dO, (int)(ors * sizeof(T)), len, w, lane);
      const char* ws = a.ws + sh * a.per;
      dma_flat<8, GdrWs<T>::I3 / 1024>(smem + L::Z, ws + GdrWs<T>::bT, w, lane);
      dma_flat<8, kGdrScal / 1024>(smem + L::scal, ws + GdrWs<T>::bScal, w, lane);
      const bool mine = 16 * w < VB;   // (uniform)
      const float* S = a.S_chunks + sh * sm + (size_t)vb * DK;
      const float* dS = a.dS_chunks + sh * sm + (size_t)vb * DK;
      f32x4 s[2 * NP], R[4], vt[4];
      if (mine) {
        const float* kept = a.dR + (sh * (a.Dv / 16) + vb / 16 + w) * 1024 + 4 * lane;
#pragma unroll
        for (int j = 0; j < 2 * NP; ++j) s[j] = *reinterpret_cast<const f32x4*>(S + (16 * w + c) * DK + 16 * j + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) R[i] = *reinterpret_cast<const f32x4*>(kept + 256 * i);
      }
      vm_wait_all();
      __syncthreads();
      if (mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) vt[i] = Quad<T>::f32(VR::tr(smem + L::V, 16 * i, w, g, c));
      }
      __syncthreads();   // (U goes where the values were)
      f32x4 sn[2], dn[2];   // S, dS of the next 32 value columns, on their way from here
      const auto columns = [&](int p) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int at = (32 * p + 16 * h + 4 * g + e) * DK + 16 * jt + c;
            sn[h][e] = S[at];
            dn[h][e] = dS[at];
          }
      };
      columns(0);
      if (mine) {
        Fi<T, kExact> Sf[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) Sf[p] = to_fi<T, kExact>(s[2 * p], s[2 * p + 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x = zero4();
#pragma unroll
          for (int p = 0; p < NP; ++p) x = mma<T>(KR::nat(smem + L::K, i, p, g, c), Sf[p], x);
          x *= *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
          const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
          vt[i] -= x;
          const float s1 = row_sum4(R[i] * vt[i], c), s2 = row_sum4(R[i] * x, c);
          if (c < 4) {
            const int at = w * kGdrC + 16 * i + 4 * g + c;
            rRV[at] = vb ? rRV[at] + s1 : s1;
            rRK[at] = vb ? rRK[at] + s2 : s2;
          }
          vt[i] *= be;
          UT::template put<kExact>(smem + L::R, 16 * w + c, i, g, R[i]);
        }
        const Fi<T, kExact> Rf[2] = {to_fi<T, kExact>(vt[0], vt[1]), to_fi<T, kExact>(vt[2], vt[3])};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x = zero4();
#pragma unroll
          for (int y = 0; y <= i / 2; ++y)
            x = mma<T>(ld_img<T, kExact>(smem + L::Z, img_lower(i, y), lane), Rf[y], x);
          UT::template put<kExact>(smem + L::U, 16 * w + c, i, g, x);
        }
      }
      __syncthreads();
      // ---- 2. products over these columns (queries on their way)
      if (NB == 1) clear();
      if (b + 1 == NB) KR::template dma<8>(smem + L::Z, q, (int)(a.qs[1] * sizeof(T)), len, w, lane);
#pragma unroll 1
      for (int p = 0; p < NV; ++p) {
        const Fi<T, kExact> fs = to_fi<T, kExact>(sn[0], sn[1]), fd = to_fi<T, kExact>(dn[0], dn[1]);
        if (w < NJ)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) ss += sn[h][e] * dn[h][e];
        if (p + 1 < NV) columns(p + 1);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          __builtin_amdgcn_sched_barrier(0);   // (the tiles' operands one tile at a time: all do not fit)
          a1[i] = mma<T>(VR::nat(smem + L::O, i0 + i, p, g, c), fs, a1[i]);
          a2[i] = mma<T>(UT::template tok<kExact>(smem + L::U, i0 + i, 32 * p, g, c), fd, a2[i]);
          a3[i] = mma<T>(UT::template tok<kNear>(smem + L::R, i0 + i, 32 * p, g, c), first<kNear>(fs), a3[i]);
        }
      }
      renew(g, c);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int y = w + 8 * x;
        if (y < 10) {
          const int i = tri_row_of(y, false), j = tri_col_of(y, false);
#pragma unroll 1
          for (int p = 0; p < NV; ++p) {
            const Fi<T, kExact> fu = UT::template tok<kExact>(smem + L::U, j, 32 * p, g, c);
            aP[x] = mma<T>(VR::nat(smem + L::O, i, p, g, c), fu, aP[x]);
            aA[x] = mma<T>(UT::template tok<kExact>(smem + L::R, i, 32 * p, g, c), fu, aA[x]);
          }
        }
      }
      // dV = beta dR, eight values of a token a lane
      for (int x = w; x < 4 * NV; x += 8) {
        const int i = x & 3, p = x >> 2, t = 16 * i + c;
        f32x4 lo, hi;
        UT::template eight<kExact>(smem + L::R, i, 32 * p, g, c, lo, hi);
        const float be = scal[kScBeta * kGdrC + t];
        if (t < len) st_eight(reinterpret_cast<T*>(a.dv) + ((row0 + t) * a.Hv + hv) * a.Dv + vb + 32 * p + 8 * g, lo * be, hi * be);
      }
      if (b + 1 == NB) vm_wait_all();
      __syncthreads();
    }

    // ---- <dS, S>
    renew(g, c);
    ss = group_sum<64>(ss);
    if (lane == 0) rSS[w] = ss;

    // ---- D dP and M of this wave's tiles, with their row and column sums; zeros in the
    // upper tiles (0, 1) and (2, 3), which the fragments reach
    if (w >= 4) {
      const int y = w - 4;
      WT::template put<kNear>(smem + (y & 1 ? L::M : L::W), 16 * (y < 2 ? 1 : 3) + c, y < 2 ? 0 : 2, g, zero4());
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int y = w + 8 * x;
      if (y < 10) {
        const int i = tri_row_of(y, false), j = tri_col_of(y, false), tj = 16 * j + c;
        f32x4 qk = zero4(), kk = zero4();
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const Fr<T> fb = KR::nat(smem + L::K, j, p, g, c);
          qk = mma<T>(KR::nat(smem + L::Z, i, p, g, c), fb, qk);
          kk = mma<T>(KR::nat(smem + L::K, i, p, g, c), fb, kk);
        }
        const float Ghj = scal[kScGh * kGdrC + tj], Glj = scal[kScGl * kGdrC + tj];
        f32x4 W, M, rows, betas;
        float col = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ti = 16 * i + 4 * g + e;
          float D = 0.0f;
          if (tj <= ti && ti < len) D = decay_exp((scal[kScGh * kGdrC + ti] - Ghj) + (scal[kScGl * kGdrC + ti] - Glj));
          const float be = scal[kScBeta * kGdrC + ti], dA = tj < ti ? -aA[x][e] : 0.0f;
          W[e] = a.scale * (D * aP[x][e]);
          M[e] = be * (D * dA);
          // (no decay lies between a token and itself)
          const float pp = tj < ti ? W[e] * qk[e] : 0.0f, ab = D * dA * kk[e], sum = pp + be * ab;
          col += sum;
          rows[e] = sum;
          betas[e] = ab;
        }
        if (i == j) {   // (uniform) the sums over i >= t > j for t = row: down the columns, then along t's row
          rows[2] += rows[3];
          rows[1] += rows[2];
          rows[0] += rows[1];
          const float d1 = __shfl_down(rows[0], 16), d2 = __shfl_down(rows[0], 32), d3 = __shfl_down(rows[0], 48);
          const float below = (g < 3 ? d1 : 0.0f) + (g < 2 ? d2 : 0.0f) + (g < 1 ? d3 : 0.0f);
#pragma unroll
          for (int e = 0; e < 4; ++e) rows[e] = c < 4 * g + e ? rows[e] + below : 0.0f;
        }
        const float rs = row_sum4(rows, c), rb = row_sum4(betas, c);
        if (c < 4) {
          rRow[j * kGdrC + 16 * i + 4 * g + c] = rs;
          rBeta[j * kGdrC + 16 * i + 4 * g + c] = rb;
        }
        col += __shfl_xor(col, 16);
        col += __shfl_xor(col, 32);
        if (g == 0) rCol[i * kGdrC + tj] = col;
        WT::template put<kNear>(smem + L::W, 16 * j + c, i, g, W);
        WT::template put<kNear>(smem + L::M, 16 * j + c, i, g, M);
      }
    }
    __syncthreads();

    // ---- dQ, dK of this wave's tiles
    renew(g, c);
#pragma unroll
    for (int ii = 0; ii < NI; ++ii) {
      const int i = i0 + ii;
      const f32x4 gam = *reinterpret_cast<const f32x4*>(scal + kScGam * kGdrC + 16 * i + 4 * g);
      const f32x4 end = *reinterpret_cast<const f32x4*>(scal + kScEnd * kGdrC + 16 * i + 4 * g);
      const f32x4 be = *reinterpret_cast<const f32x4*>(scal + kScBeta * kGdrC + 16 * i + 4 * g);
      const f32x4 x1 = a1[ii] * gam * a.scale, x2 = a2[ii] * end, x3 = a3[ii] * gam;
      const f32x4 kt = Quad<T>::f32(KR::tr(smem + L::K, 16 * i, jt, g, c));
      const f32x4 qt = Quad<T>::f32(KR::tr(smem + L::Z, 16 * i, jt, g, c));
      const float s1 = row_sum4(qt * x1, c), s2 = row_sum4(kt * x2, c);
      if (c < 4) {
        rQ[jt * kGdrC + 16 * i + 4 * g + c] = s1;
        rUK[jt * kGdrC + 16 * i + 4 * g + c] = s2;
      }
      dQ[ii] += x1;
      dK[ii] += x2 - be * x3;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const Fr<T> fk = KR::tr32(smem + L::K, y, jt, g, c);
        if (2 * y <= i) {    // (uniform)
          dQ[ii] = mma<T>(WT::template tok<kNear>(smem + L::W, i, 32 * y, g, c), fk, dQ[ii]);
          dK[ii] = mma<T>(WT::template tok<kNear>(smem + L::M, i, 32 * y, g, c), fk, dK[ii]);
        }
        if (2 * y + 1 >= i) {
          dK[ii] = mma<T>(WT::template col<kNear>(smem + L::W, 16 * i, y, g, c), KR::tr32(smem + L::Z, y, jt, g, c), dK[ii]);
          dK[ii] = mma<T>(WT::template col<kNear>(smem + L::M, 16 * i, y, g, c), fk, dK[ii]);
        }
      }
    }
    __syncthreads();

    if (hv + 1 < (hk + 1) * grp) {
      if (w == 0) finish(hv);
      __syncthreads();
    }
  }

  // out through LDS, 16 bytes a lane (from the results' layout a store would cover 32
  // bytes of each of 4 rows)
  typedef InterT<T, DK> DT;
  static_assert(2 * DT::bytes(1) <= L::scal, "over what is no longer needed");
#pragma unroll
  for (int ii = 0; ii < NI; ++ii) {
    DT::template put<1>(smem, 16 * jt + c, i0 + ii, g, dQ[ii]);
    DT::template put<1>(smem + DT::bytes(1), 16 * jt + c, i0 + ii, g, dK[ii]);
  }
  __syncthreads();
  for (int x = w; x < 8 * NP; x += 8) {
    const int i = x & 3, p = (x >> 2) % NP, t = 16 * i + c;
    const bool second = x >= 4 * NP;
    f32x4 lo, hi;
    DT::template eight<1>(smem + (second ? DT::bytes(1) : 0), i, 32 * p, g, c, lo, hi);
    T* out = reinterpret_cast<T*>(second ? a.dk : a.dq) + ((row0 + t) * a.Hk + hk) * DK + 32 * p + 8 * g;
    if (t < len) st_eight(out, lo, hi);
  }
  if (w == 7) finish((hk + 1) * grp - 1);
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
  hipLaunchKernelGGL(kern, dim3(gdr_chain_grid(heads, a.Dv / (16 * NW))), dim3(128 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK, int NW>
int launch_bpair_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = BPairLds<T, DK, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_bpair_kernel<T, DK, NW>;
  const int st = allow_lds(kern, lds);
  if (st) return st;
  const unsigned heads = (unsigned)a.nseq * a.Hv;
  hipLaunchKernelGGL(kern, dim3(gdr_chain_grid(heads, a.Dv / (16 * NW))), dim3(256 * NW), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK, int VB, int NB>
int launch_grad_t(const GdrArgs& a, hipStream_t s) {
  constexpr int lds = GradLds<T, DK, VB>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_gdr_grad_kernel<T, DK, VB, NB>;
  const int st = allow_lds(kern, lds);
  if (st) return st;
  hipLaunchKernelGGL(kern, dim3(a.nslots, a.Hk), dim3(512), lds, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T, int DK>
int launch_bwd_t(const GdrArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  int st = launch_gdr_prep(a, sizeof(T) == 2 ? CARVE_BF16 : CARVE_F32, true, s);
  if (st) return st;
  mark(s);
  if constexpr (DK == 32) {
    st = launch_bchain_t<T, DK, 2>(a, s);
  } else {
    constexpr bool four = sizeof(T) == 2 || DK < 128;   // (f32 rows of 128: four tiles' LDS does not fit)
    if (gdr_few_tiles(a)) st = launch_bpair_t<T, DK, 1>(a, s);
    else if (!four || !gdr_many_tiles(a)) st = launch_bpair_t<T, DK, 2>(a, s);
    else if constexpr (four) st = launch_bchain_t<T, DK, 4>(a, s);
  }
  if (st) return st;
  mark(s);
  if (a.Dv == 32) st = launch_grad_t<T, DK, 32, 1>(a, s);
  else if (a.Dv == 64) st = launch_grad_t<T, DK, 64, 1>(a, s);
  else if constexpr (sizeof(T) == 2) st = a.Dv == 128 ? launch_grad_t<T, DK, 128, 1>(a, s) : launch_grad_t<T, DK, 128, 2>(a, s);
  else st = a.Dv == 128 ? launch_grad_t<T, DK, 64, 2>(a, s) : launch_grad_t<T, DK, 64, 4>(a, s);   // (128 columns: 177 KB)
  mark(s);
  return st;
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
