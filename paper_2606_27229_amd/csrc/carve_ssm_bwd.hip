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

// One workgroup a chunk, group and share of the group's heads.  Waves 0 to 3 make dC and
// what pairs of tokens add to da, waves 4 to 7 dB and dx; wave w of each side owns token tile
// w, as i of dC and as j of dB and dx.  dB and dC stay in registers over the heads; a head
// comes in turns of 32 value columns, in which everything but L is linear: x, dy and the
// rows of S and E.  The other waves bring them a turn ahead: wave 8 rows straight into LDS (a
// wave that reads LDS waits for all the LDS loads it has under way, so the loads are
// others'); waves 9 and 10 the states, which pass their registers and become the matrix
// cores' operands on the way (with bf16 tokens three bf16 values each, StateRows); wave 11
// makes a head's ddt and its sums when the others have gone on.
// Bound by the latency of a turn's steps, most of all of its loads: the states S and E (N x P
// floats each, a chunk and head) are 0.54 of the 0.72 GB that 4 x 4096 tokens of 32 heads read in 248
// to 283 us, 264 on average (2.7 TB/s); vector instructions issue in 47 % of the cycles, matrix
// cores work in 22 %, LDS in 41 %.  Without the loads it takes as long as without the products.
template <typename T, int N>
struct GradLds {
  typedef SsmRows<T, N, kSsmC> KR;     // B, C
  typedef SsmRows<T, kPw, kSsmC> VR;   // x, dy
  typedef SsmRows<T, N, kPw> SR;       // a plane of S or E
  static constexpr int planes = sizeof(T) == 2 ? kExact : 1, state = SR::bytes * planes;
  static constexpr int B = 0, C = KR::bytes, turn = 2 * KR::bytes;
  static constexpr int X = 0, dY = VR::bytes, S = dY + VR::bytes, E = S + state, one = E + state;   // of a turn
  // of a head: r_t, E_t x.EB, dy.x, d_t, sums of M over i and da's rectangles by wave; <E, S>
  // by wave, e^{G_C}
  static constexpr int sums = 12 * kSsmC + 8, small = 2 * (kSmBwd + sums) * 4;
  // two turns' rows where they fit (else a turn's rows are waited for)
  static constexpr int bufs = turn + 2 * one + small <= 160 * 1024 ? 2 : 1;
  static constexpr int scal = turn + bufs * one, sum = scal + 2 * kSmBwd * 4, total = scal + small;
};
enum : int { kSuR = 0, kSuE = 1, kSuDiag = 2, kSuD = 3, kSuM = 4, kSuRect = 8, kSuES = 12 * kSsmC, kSuWhole = kSuES + 4 };

// The 32 rows of a turn's state, f32 in memory, by one wave: into its registers, then as
// planes into LDS (SsmRows' layout).
template <typename T, int N>
struct StateRows {
  typedef GradLds<T, N> L;
  typedef typename L::SR SR;
  static constexpr int n = kPw * N / 256;   // quads of a lane
  f32x4 v[n];
  // (read once: past the L2, which the rows of B, C, x and dy want; 280 -> 267 us)
  static __device__ __forceinline__ f32x4 quad(const float* from, int k, int lane) {
    return __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(from + 4 * (64 * k + lane)));
  }
  __device__ __forceinline__ void load(const float* from, int lane) {
#pragma unroll
    for (int k = 0; k < n; ++k) v[k] = quad(from, k, lane);
  }
  // next: the rows that take the registers as they become free
  __device__ __forceinline__ void put(char* lds, int lane, const float* next) {
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const int at = 64 * k + lane, row = at / (N / 4), q = at % (N / 4);
      if constexpr (sizeof(T) == 2) {
        char* to = lds + row * SR::RB + (((q >> 1) ^ SR::swz(row)) << 4) + ((q & 1) << 3);
        f32x4 x = v[k];
#pragma unroll
        for (int i = 0; i < L::planes; ++i) {
          const bf16x4 h = Quad<bf16_t>::cvt(x);
          *reinterpret_cast<bf16x4*>(to + i * SR::bytes) = h;
          if (i + 1 < L::planes) x = bf16_rest(x, h);
        }
      } else {
        *reinterpret_cast<f32x4*>(lds + row * SR::RB + ((q ^ SR::swz(row)) << 4)) = v[k];
      }
      v[k] = quad(next, k, lane);
    }
  }
};
// operands from the first M planes: columns n (rows p), and rows p in nat8's order
template <typename T, int N, int M>
__device__ __forceinline__ Fi<T, M> state_tr(const char* lds, int j, int g, int c) {
  typedef typename GradLds<T, N>::SR SR;
  Fi<T, M> f;
#pragma unroll
  for (int i = 0; i < (sizeof(T) == 2 ? M : 1); ++i) f.x[i] = SR::tr32(lds + i * SR::bytes, 0, j, g, c);
  return f;
}
template <typename T, int N>
__device__ __forceinline__ Fi<T, kExact> state_nat8(const char* lds, int i, int p, int g, int c) {
  typedef typename GradLds<T, N>::SR SR;
  Fi<T, kExact> f;
#pragma unroll
  for (int u = 0; u < GradLds<T, N>::planes; ++u) f.x[u] = SR::nat8(lds + u * SR::bytes, i, p, g, c);
  return f;
}
// f where sign is 1, -f where it is -1 (uniform)
template <typename T>
__device__ __forceinline__ Fr<T> with_sign(Fr<T> f, float sign) {
  if constexpr (sizeof(T) == 2) {
    const unsigned m = sign < 0.0f ? 0x80008000u : 0u;
    f.a = __builtin_bit_cast(bf16x4, __builtin_bit_cast(u32x2_t, f.a) ^ m);
    f.b = __builtin_bit_cast(bf16x4, __builtin_bit_cast(u32x2_t, f.b) ^ m);
  } else {
    f.a *= sign, f.b *= sign;
  }
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
__global__ void __launch_bounds__(768, 3) carve_ssm_grad_kernel(SsmArgs a) {
  typedef GradLds<T, N> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  constexpr int NP = N / 32, NT = N / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = wave & 3;
  int lane = tid & 63, g = lane >> 4, c = lane & 15, tok = 16 * w + c;
  // (coordinates the compiler takes as new: addresses are formed where they are used, not
  // all of them ahead of the loops and kept)
  const auto anew = [&]() {
    asm volatile("" : "+v"(lane));
    g = lane >> 4, c = lane & 15, tok = 16 * w + c;
  };
  const int slot = blockIdx.x, grp = blockIdx.y, part = blockIdx.z;
  const int rep = a.H / a.G, h0 = grp * rep + (int)((long long)rep * part / a.splits),
            h1 = grp * rep + (int)((long long)rep * (part + 1) / a.splits);
  const SsmSeq q = ssm_find(a, slot, kSsmC);
  const int ch = slot - ssm_slot0(a, q, kSsmC);
  if (ch < 0 || (long long)ch * kSsmC >= q.len) {   // a slot of no chunk
    for (int i = tid; i < (h1 - h0) * kPart; i += 768) a.part[((size_t)slot * a.H + h0) * kPart + i] = 0.0f;
    return;
  }
  const int first = q.first + ch * kSsmC, len = min(kSsmC, q.len - ch * kSsmC);
  const float sign = ssm_sign(slot);   // of E, and of dy where its products are summed into da
  const size_t row0 = (size_t)q.batch * a.T + first, pn = (size_t)a.P * N;
  const int turns = a.P / kPw, total = (h1 - h0) * turns;
  const auto rows = [&](int n) { return smem + L::turn + (L::bufs == 2 ? (n & 1) * L::one : 0); };
  const auto scal = [&](int h) { return reinterpret_cast<float*>(smem + L::scal) + (h & 1) * kSmBwd; };
  const auto sums = [&](int h) { return reinterpret_cast<float*>(smem + L::sum) + (h & 1) * L::sums; };

  if (wave == 8) {   // ---- rows
    KR::template dma<1>(smem + L::B, reinterpret_cast<const T*>(a.Bm) + q.batch * a.bs[0] + first * a.bs[1] + grp * a.bs[2],
                        (int)(a.bs[1] * sizeof(T)), len, 0, lane);
    KR::template dma<1>(smem + L::C, reinterpret_cast<const T*>(a.Cm) + q.batch * a.cs[0] + first * a.cs[1] + grp * a.cs[2],
                        (int)(a.cs[1] * sizeof(T)), len, 0, lane);
    const T* x = reinterpret_cast<const T*>(a.x) + q.batch * a.xs[0] + first * a.xs[1];
    const T* dy = reinterpret_cast<const T*>(a.dy) + row0 * a.H * a.P;
    const auto issue = [&](int n) {
      const int h = h0 + n / turns, p0 = n % turns * kPw;
      char* buf = rows(n);
      VR::template dma<1>(buf + L::X, x + h * a.xs[2] + p0, (int)(a.xs[1] * sizeof(T)), len, 0, lane);
      VR::template dma<1>(buf + L::dY, dy + h * a.P + p0, (int)((long long)a.H * a.P * sizeof(T)), len, 0, lane);
      if (p0 == 0) dma_flat<1, 3>(reinterpret_cast<char*>(scal(h)), a.scal + ((size_t)slot * a.H + h) * kSmBwd * 4, 0, lane);
    };
    if (L::bufs == 2) issue(0);
#pragma unroll 1
    for (int n = 0; n < total; ++n) {
      if (L::bufs == 1) {
        __syncthreads();   // (0) the rows of the turn before are no longer read
        issue(n);
      }
      vm_wait_all();
      __syncthreads();     // (1)
      if (L::bufs == 2 && n + 1 < total) issue(n + 1);
    }
    __syncthreads();       // (2)
    return;
  }
  if (wave == 9 || wave == 10) {   // ---- states
    const float* from = (wave == 9 ? a.S_chunks : a.E_chunks) + ((size_t)slot * a.H + h0) * pn;
    const int to = wave == 9 ? L::S : L::E;
    StateRows<T, N> st;
    // (a head's turns are one after another in memory)
    const auto at = [&](int n) { return from + (size_t)min(n, total - 1) * kPw * N; };   // (the last one again behind it)
    st.load(at(0), lane);
    if (L::bufs == 2) st.put(rows(0) + to, lane, at(1));
#pragma unroll 1
    for (int n = 0; n < total; ++n) {
      if (L::bufs == 1) {
        __syncthreads();   // (0)
        st.put(rows(n) + to, lane, at(n + 1));
      }
      __syncthreads();     // (1)
      if (L::bufs == 2 && n + 1 < total) st.put(rows(n + 1) + to, lane, at(n + 2));
    }
    __syncthreads();       // (2)
    return;
  }
  if (wave == 11) {   // ---- what remains of a head when all its sums are there
    const auto finish = [&](int h) {
      const float* su = sums(h);
      const bool in = lane < len;
      const float bias = a.dt_bias ? a.dt_bias[h] : 0.0f, A = a.A[h];
      const float raw = (float)(reinterpret_cast<const T*>(a.dt) + q.batch * a.ds[0] + h)[(first + min(lane, len - 1)) * a.ds[1]];
      const float d = su[kSuD * kSsmC + lane], e = su[kSuE * kSsmC + lane];
      float suf = in ? su[kSuR * kSsmC + lane] : 0.0f, pre = in ? d * e : 0.0f;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) {
        const float dn = __shfl_down(suf, s), up = __shfl_up(pre, s);
        if (lane + s < 64) suf += dn;
        if (lane >= s) pre += up;
      }
      const float before = __shfl_up(pre, 1);
      const float es = su[kSuWhole] * ((su[kSuES] + su[kSuES + 1]) + (su[kSuES + 2] + su[kSuES + 3]));
      const auto waves = [&](int k) {
        const float* p = su + k * kSsmC + lane;
        return (p[0] + p[kSsmC]) + (p[2 * kSsmC] + p[3 * kSsmC]);
      };
      const float da = suf + (lane > 0 ? before : 0.0f) + waves(kSuRect) + es;
      // (A may be -inf: nothing comes through decays of 0)
      float dd = (da != 0.0f ? A * da : 0.0f) + (waves(kSuM) + e);
      if (a.softplus) {
        const float z = raw + bias, ez = expf(-fabsf(z));
        dd *= (z >= 0.0f ? 1.0f : ez) / (1.0f + ez);
      }
      if (in) reinterpret_cast<T*>(a.ddt)[(row0 + lane) * a.H + h] = (T)dd;
      const float sa = group_sum<64>(in ? d * da : 0.0f), sb = group_sum<64>(in ? dd : 0.0f),
                  sd = group_sum<64>(in ? su[kSuDiag * kSsmC + lane] : 0.0f);
      if (lane == 0) *reinterpret_cast<f32x4*>(a.part + ((size_t)slot * a.H + h) * kPart) = f32x4{sa, sb, sd, 0.0f};
    };
#pragma unroll 1
    for (int h = h0; h < h1; ++h)
#pragma unroll 1
      for (int t = 0; t < turns; ++t) {
        if (L::bufs == 1) __syncthreads();   // (0)
        __syncthreads();                     // (1)
        if (t == 0 && h > h0) finish(h - 1);
      }
    __syncthreads();   // (2)
    finish(h1 - 1);
    return;
  }

  const bool back = wave >= 4;   // (uniform) dB and dx
  f32x4 acc[NT];                 // dC^T or dB^T: rows n, the tile's tokens
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = zero4();
  int n = 0;
  const char* cb = a.cb + ((size_t)slot * a.G + grp) * 2 * kSsmCB + 16 * lane;
  if (!back) {   // ---- dC, and what pairs of tokens add to da
    f32x4 CB[4];   // C B^T: rows j, the tile's columns i
#pragma unroll
    for (int i = 0; i < 4; ++i) CB[i] = i <= w ? *reinterpret_cast<const f32x4*>(cb + ssm_tile(w, i)) : zero4();
#pragma unroll 1
    for (int h = h0; h < h1; ++h) {
      f32x4 Q[4], ES = zero4(), U[NT];   // x (rows j) against the tile's dy; S against E; S^T dy
#pragma unroll
      for (int i = 0; i < 4; ++i) Q[i] = zero4();
#pragma unroll
      for (int j = 0; j < NT; ++j) U[j] = zero4();
      const float* sc = scal(h);
#pragma unroll 1
      for (int t = 0; t < turns; ++t, ++n) {
        const char* buf = rows(n);
        if (L::bufs == 1) __syncthreads();   // (0)
        __syncthreads();                     // (1)
        anew();
        const Fr<T> fy = with_sign<T>(VR::nat(buf + L::dY, w, 0, g, c), sign),
                    fy8 = with_sign<T>(VR::nat8(buf + L::dY, w, 0, g, c), sign);
#pragma unroll
        for (int i = 0; i < 4; ++i) Q[i] = mma<T>(VR::nat8(buf + L::X, i, 0, g, c), fy8, Q[i]);
        if (w < NP) {   // (uniform) <E, S> of 32 n: the diagonal of their product
#pragma unroll
          for (int v = 0; v < 2; ++v)
            ES = mma<T>(state_nat8<T, N>(buf + L::S, v, w, g, c), state_nat8<T, N>(buf + L::E, v, w, g, c), ES);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) U[j] = mma<T>(state_tr<T, N, kExact>(buf + L::S, j, g, c), fy, U[j]);
      }
      anew();
      const float Gh = sc[kSmGh * kSsmC + tok], Gl = sc[kSmGl * kSsmC + tok], gam = sc[kSmGam * kSsmC + tok] * sign;
      float* su = sums(h);
      float r = 0.0f, mine = 0.0f, carry = 0.0f;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        r += dot4(U[j], Quad<T>::f32(KR::quad(smem + L::C, w, j, g, c)));
        acc[j] += U[j] * gam;
      }
      // Q becomes L d Q.  M = L C B^T Q, summed over i (the tile's columns) for each j, and
      // d_j M over j < t and i >= t: prefix sums down each column, then along rows
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 pre = zero4(), ms = zero4();
        if (i <= w) {   // (uniform)
          const f32x4 d = four(sc + kSmD * kSsmC + 16 * i + 4 * g);
          Q[i] *= sign;
          if (i < w) {  // (uniform) from a tile before
            Q[i] *= four(sc + kSmF * kSsmC + 16 * i + 4 * g) * decay_between(Gh, Gl, sc[kSmTile + i], sc[kSmTile + 4 + i]);
          } else {
            const f32x4 gh = four(sc + kSmGh * kSsmC + 16 * i + 4 * g), gl = four(sc + kSmGl * kSsmC + 16 * i + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              mine += masked(4 * g + e == c, Q[i][e]);
              Q[i][e] = masked(4 * g + e <= c, decay_between(Gh, Gl, gh[e], gl[e]) * Q[i][e]);
            }
          }
          ms = CB[i] * Q[i];
          Q[i] *= d;
          const f32x4 m = ms * d;
          // (before each row of the quad, of the quads before it, of the tiles before it)
          pre[1] = m[0];
          pre[2] = m[0] + m[1];
          pre[3] = pre[2] + m[2];
          float in = pre[3] + m[3];
          const float p1 = __shfl(in, (lane - 16) & 63);
          in += g > 0 ? p1 : 0.0f;
          const float p2 = __shfl(in, (lane - 32) & 63);
          in += g > 1 ? p2 : 0.0f;
          const float ahead = __shfl(in, (lane - 16) & 63), whole = __shfl(in, 48 + c);
          const float more = carry + (g > 0 ? ahead : 0.0f);
#pragma unroll
          for (int e = 0; e < 4; ++e) pre[e] = masked((16 * i + 4 * g + e <= tok) & (tok < len), pre[e] + more);
          carry += whole;
#pragma unroll
          for (int e = 0; e < 4; ++e) ms[e] = masked(tok < len, ms[e]);
        }
        const float rect = row_sum4(pre, c), col = row_sum4(ms, c);
        if (c < 4) su[(kSuRect + w) * kSsmC + 16 * i + 4 * g + c] = rect, su[(kSuM + w) * kSsmC + 16 * i + 4 * g + c] = col;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s > w / 2) continue;   // (uniform)
        const Fi<T, kNear> f = to_fi<T, kNear>(Q[2 * s], 2 * s + 1 <= w ? Q[2 * s + 1] : zero4());
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = mma<T>(KR::tr32(smem + L::B, s, j, g, c), f, acc[j]);
      }
      r = col_sum(r) * gam, mine = col_sum(mine);
      float es = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) es += masked(4 * g + e == c, ES[e]);
      es = group_sum<64>(es);
      if (g == 0) su[kSuR * kSsmC + tok] = r, su[kSuDiag * kSsmC + tok] = mine, su[kSuD * kSsmC + tok] = sc[kSmD * kSsmC + tok];
      if (lane == 0) su[kSuES + w] = es, su[kSuWhole] = sc[kSmWhole] * sign;
    }
  } else {   // ---- dB, dx
    f32x4 CB[4];   // C B^T: rows i, the tile's columns j
#pragma unroll
    for (int i = 0; i < 4; ++i) CB[i] = i >= w ? *reinterpret_cast<const f32x4*>(cb + kSsmCB + ssm_tile(i, w)) : zero4();
#pragma unroll 1
    for (int h = h0; h < h1; ++h) {
      f32x4 Q[4];          // dy (rows i) against the tile's x
      Fi<T, kNear> Lf[2];  // L C B^T
      float ex = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) Q[i] = zero4();
      const float* sc = scal(h);
      // L of the tile's columns, applied to tile i
      const auto decayed = [&](int i, f32x4 v) {
        if (i < w) return zero4();   // (uniform)
        if (i > w) return v * (four(sc + (kSmDown + w) * kSsmC + 16 * i + 4 * g) * sc[kSmF * kSsmC + tok]);
        const float Gh = sc[kSmGh * kSsmC + tok], Gl = sc[kSmGl * kSsmC + tok];
        const f32x4 gh = four(sc + kSmGh * kSsmC + 16 * i + 4 * g), gl = four(sc + kSmGl * kSsmC + 16 * i + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = masked(4 * g + e >= c, decay_between(gh[e], gl[e], Gh, Gl) * v[e]);
        return v;
      };
#pragma unroll 1
      for (int t = 0; t < turns; ++t, ++n) {
        const char* buf = rows(n);
        if (L::bufs == 1) __syncthreads();   // (0)
        __syncthreads();                     // (1)
        anew();
        if (t == 0) {
#pragma unroll
          for (int s = 0; s < 2; ++s) Lf[s] = to_fi<T, kNear>(decayed(2 * s, CB[2 * s]), decayed(2 * s + 1, CB[2 * s + 1]));
        }
        const Fr<T> fx = VR::nat(buf + L::X, w, 0, g, c), fx8 = VR::nat8(buf + L::X, w, 0, g, c);
        const float dj = sc[kSmD * kSsmC + tok], endj = sc[kSmEnd * kSsmC + tok] * sign, endd = sc[kSmEndD * kSsmC + tok] * sign;
#pragma unroll
        for (int i = 0; i < 4; ++i) Q[i] = mma<T>(VR::nat8(buf + L::dY, i, 0, g, c), fx8, Q[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] += mma<T>(state_tr<T, N, kNear>(buf + L::E, j, g, c), fx, zero4()) * endd;
        // dx: two tiles of p
        const RowStore<T> dx(reinterpret_cast<T*>(a.dx) + (row0 * a.H + h) * a.P + t * kPw, (size_t)a.H * a.P, len, kPw);
        const float skip = a.D ? a.D[h] : 0.0f;
        f32x4 u[2] = {zero4(), zero4()}, z[2] = {zero4(), zero4()};
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const Fr<T> fb = KR::nat8(smem + L::B, w, p, g, c);
#pragma unroll
          for (int v = 0; v < 2; ++v) u[v] = mma<T>(state_nat8<T, N>(buf + L::E, v, p, g, c), fb, u[v]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int v = 0; v < 2; ++v) z[v] = mma<T>(VR::tr32(buf + L::dY, s, v, g, c), Lf[s], z[v]);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          u[v] *= endj;
          ex += dot4(u[v], Quad<T>::f32(VR::quad(buf + L::X, w, v, g, c)));
          dx.st(tok, 16 * v + 4 * g, (u[v] + z[v]) * dj + Quad<T>::f32(VR::quad(buf + L::dY, w, v, g, c)) * skip);
        }
      }
      anew();
      const float dj = sc[kSmD * kSsmC + tok];
#pragma unroll
      for (int i = 0; i < 4; ++i) Q[i] = decayed(i, Q[i] * dj);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s < w / 2) continue;   // (uniform)
        const Fi<T, kNear> f = to_fi<T, kNear>(Q[2 * s], Q[2 * s + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = mma<T>(KR::tr32(smem + L::C, s, j, g, c), f, acc[j]);
      }
      ex = col_sum(ex);
      if (g == 0) sums(h)[kSuE * kSsmC + tok] = ex;
    }
  }
  __syncthreads();   // (2)
  settle(acc);
  if (tok < len) {
    const size_t at = ((row0 + tok) * a.G + grp) * N + 4 * g;
    if (a.splits == 1) {
      T* out = reinterpret_cast<T*>(back ? a.dBm : a.dCm) + at;
#pragma unroll
      for (int j = 0; j < NT; ++j) Quad<T>::st(out + 16 * j, Quad<T>::cvt(acc[j]));
    } else {
      const size_t all = (size_t)(a.offsets ? 1 : a.nseq) * a.T * a.G * N;
      float* out = a.dBp + ((size_t)part * 2 + (back ? 0 : 1)) * all + at;
#pragma unroll
      for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(out + 16 * j) = acc[j];
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
  hipLaunchKernelGGL(kern, dim3(a.nslots, a.G, a.splits), dim3(768), lds, s, a);
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
