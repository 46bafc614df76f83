// carve_ssm_fwd.hip -- the chunked selective state space scan, forward, and the chains of
// states that both directions run: the spans' sums, their joining, and the outputs.
#include "carve_ssm.h"

namespace carve {
namespace {

// Wave w of a workgroup holds S^T[n][p] of 16 value rows p in the matrix-core result layout
// (lane (g, c): n = 16 j + 4 g + e, p = 16 w + c).
template <typename T, int N>
struct Tile {
  f32x4 S[N / 16];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < N / 16; ++j) S[j] = zero4();
  }
  __device__ __forceinline__ void load(const float* row) {   // row: of p, + 4 g
#pragma unroll
    for (int j = 0; j < N / 16; ++j) S[j] = *reinterpret_cast<const f32x4*>(row + 16 * j);
  }
  __device__ __forceinline__ void store(float* row) const {
#pragma unroll
    for (int j = 0; j < N / 16; ++j) *reinterpret_cast<f32x4*>(row + 16 * j) = S[j];
  }
  // S <- whole S + sum_t k_t (f_t v_t)^T over the chunk's rows k (N wide); v: the wave's 16
  // columns of the rows v, f(t): the factors of four tokens from t
  template <typename KR, typename F>
  __device__ __forceinline__ void add(const char* k, const Fr<T> (&v)[2], F f, float whole, int g, int c) {
    Fi<T, kExact> V[2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
      V[s] = to_fi<T, kExact>(Quad<T>::f32(v[s].a) * f(32 * s + 4 * g), Quad<T>::f32(v[s].b) * f(32 * s + 16 + 4 * g));
#pragma unroll
    for (int j = 0; j < N / 16; ++j) {
      S[j] *= whole;
#pragma unroll
      for (int s = 0; s < 2; ++s) S[j] = mma<T>(KR::tr32(k, s, j, g, c), V[s], S[j]);
    }
  }
};

__device__ __forceinline__ f32x4 four(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// The steps of a span's chunks, a chunk ahead: one wave holds the next chunk's dt and makes
// its scalars while the others' rows are on their way.
template <typename T>
struct Steps {
  const T* dt;             // of the span's first row
  long long stride;
  float A, bias;
  int softplus, len, lane;
  float raw;
  __device__ __forceinline__ void fetch(int ch) {
    const int t = ch * kSsmC + lane;
    raw = ch >= 0 && t < len ? (float)dt[t * stride] : 0.0f;
  }
  __device__ __forceinline__ void make(int ch, float* out) const {
    ssm_scalars(raw, ch * kSsmC + lane < len, bias, A, softplus, lane, out);
  }
};

template <typename T>
__device__ __forceinline__ Steps<T> steps_of(const SsmArgs& a, const SsmSpan& p, int h, int lane) {
  Steps<T> s;
  s.dt = reinterpret_cast<const T*>(a.dt) + p.q.batch * a.ds[0] + p.first * a.ds[1] + h;
  s.stride = a.ds[1];
  s.A = a.A[h];
  s.bias = a.dt_bias ? a.dt_bias[h] : 0.0f;
  s.softplus = a.softplus, s.len = p.len, s.lane = lane;
  return s;
}

// Chains of states without outputs.  Forward (REV false): what each span but a sequence's
// last adds to the state.  Reverse: E <- e^{G_C} E + dY^T (e^G C) from the last chunk to the
// first: what each span but the first adds (full = 0), or, from the span's own end, E of
// every chunk's end (full = 1), then dS0.
template <typename T, int N, int NW>
struct StateLds {
  typedef SsmRows<T, N, kSsmC> KR;
  typedef SsmRows<T, 16 * NW, kSsmC> VR;
  static constexpr int K = 0, V = KR::bytes, S = V + VR::bytes, total = S + 2 * kSmFloats * 4;
};
template <typename T, int N, int NW, bool REV>
__global__ void __launch_bounds__(64 * NW, 2) carve_ssm_state_kernel(SsmArgs a, int full) {
  typedef StateLds<T, N, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* scal = reinterpret_cast<float*>(smem + L::S);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int slices = a.P / (16 * NW);
  SsmSpan p;
  int rest;
  if (!ssm_block(a, a.H * slices, p, rest)) return;
  const int h = rest / slices, p0 = rest % slices * 16 * NW, grp = h / (a.H / a.G);
  if (!full && p.s == (REV ? 0 : p.nspan - 1)) return;
  const size_t pn = (size_t)a.P * N, row = (size_t)(p0 + 16 * w + c) * N + 4 * g;
  float* zs = a.Z + ((size_t)p.slot * a.H + h) * pn + row;
  Tile<T, N> t;
  if (!full) t.zero();
  else if (p.s < p.nspan - 1) t.load(zs);
  else if (a.dS_T) t.load(a.dS_T + ((size_t)p.q.n * a.H + h) * pn + row);
  else t.zero();
  const T* kb = REV ? reinterpret_cast<const T*>(a.Cm) + p.q.batch * a.cs[0] + p.first * a.cs[1] + grp * a.cs[2]
                    : reinterpret_cast<const T*>(a.Bm) + p.q.batch * a.bs[0] + p.first * a.bs[1] + grp * a.bs[2];
  const long long ks = REV ? a.cs[1] : a.bs[1], vs = REV ? (long long)a.H * a.P : a.xs[1];
  const T* vb = REV ? reinterpret_cast<const T*>(a.dy) + (((size_t)p.q.batch * a.T + p.first) * a.H + h) * a.P + p0
                    : reinterpret_cast<const T*>(a.x) + p.q.batch * a.xs[0] + p.first * a.xs[1] + h * a.xs[2] + p0;
  Steps<T> st = steps_of<T>(a, p, h, lane);
  const auto chunk = [&](int i) { return REV ? p.nch - 1 - i : i; };
  float decay = 1.0f;
  if (w == 0 && p.nch > 0) {
    st.fetch(chunk(0));
    st.make(chunk(0), scal);
    if (p.nch > 1) st.fetch(chunk(1));
  }
#pragma unroll 1
  for (int i = 0; i < p.nch; ++i) {
    const int ch = chunk(i), len = min(kSsmC, p.len - ch * kSsmC);
    const float* sc = scal + (i & 1) * kSmFloats;
    if (i > 0) __syncthreads();   // the rows of the chunk before are no longer read
    KR::template dma<NW>(smem + L::K, kb + (long long)ch * kSsmC * ks, (int)(ks * sizeof(T)), len, w, lane);
    VR::template dma<NW>(smem + L::V, vb + (long long)ch * kSsmC * vs, (int)(vs * sizeof(T)), len, w, lane);
    if (w == 0 && i + 1 < p.nch) {
      st.make(chunk(i + 1), scal + ((i + 1) & 1) * kSmFloats);
      if (i + 2 < p.nch) st.fetch(chunk(i + 2));
    }
    if (REV && full) {   // the gradient of the state behind this chunk
      SsmState<T, N>::st(a.E_chunks + ((size_t)(p.slot0 + ch) * a.H + h) * pn * 4, pn, p0 + 16 * w, t.S, lane);
    }
    vm_wait_all();
    __syncthreads();
    const Fr<T> v[2] = {VR::tr32(smem + L::V, 0, w, g, c), VR::tr32(smem + L::V, 1, w, g, c)};
    t.template add<KR>(smem + L::K, v, [&](int at) {
      return four(sc + (REV ? kSmGam : kSmEndD) * kSsmC + at);
    }, sc[kSmWhole], g, c);
    decay *= sc[kSmWhole];
  }
  settle();
  if (!full) {
    t.store(zs);
    if (tid == 0 && p0 == 0) a.Zg[(size_t)p.slot * a.H + h] = decay;
  } else if (p.s == 0 && a.dS0) {
    t.store(a.dS0 + ((size_t)p.q.n * a.H + h) * pn + row);
  }
}

// Joins the spans of every sequence: Z becomes the state each span starts from (REV: the
// gradient of the state it ends with).  Elementwise along the sequence: four values a
// thread; the spans next to come are loaded ahead of the sum that waits for them.
template <bool REV>
__global__ void __launch_bounds__(256) carve_ssm_join_kernel(SsmArgs a) {
  const size_t pn = (size_t)a.P * a.N;
  const int h = blockIdx.y;
  const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= pn) return;
  const float* from = REV ? a.dS_T : a.S0;
  constexpr int AHEAD = 4;
  for (int n = blockIdx.z; n < a.nseq; n += gridDim.z) {
    const SsmSeq q = ssm_seq(a, n);
    const int L = a.span * kSsmC, nspan = ssm_units(q.len, L), slot0 = ssm_slot0(a, q, L);
    if (nspan < 2) continue;
    f32x4 S = zero4();
    if (from) S = *reinterpret_cast<const f32x4*>(from + ((size_t)n * a.H + h) * pn + at);
    // span i (in order) adds Z_i with decay g_i; the next one starts from the sum
    const auto slot = [&](int i) { return (size_t)(slot0 + (REV ? nspan - 1 - i : i)) * a.H + h; };
    for (int i0 = 0; i0 < nspan - 1; i0 += AHEAD) {
      f32x4 buf[AHEAD];
      float dec[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const size_t z = slot(min(i0 + u, nspan - 2));
        buf[u] = *reinterpret_cast<const f32x4*>(a.Z + z * pn + at);
        dec[u] = a.Zg[z];
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (i0 + u < nspan - 1) {
          if (i0 + u > 0) *reinterpret_cast<f32x4*>(a.Z + slot(i0 + u) * pn + at) = S;
          S = S * dec[u] + buf[u];
        }
    }
    *reinterpret_cast<f32x4*>(a.Z + slot(nspan - 1) * pn + at) = S;
  }
}

// Outputs of a span: its chunks one after another, the state in registers.  A workgroup
// takes two units (a head's 16 NW value rows) of one group, which share B and C; waves hold
// 16 value rows each.  A chunk:
//   all waves   L d C B^T of both units, a pair of tiles a wave: operand images in LDS
//   its waves   Y^T = S (e^G C)^T + X^T (L d C B^T)^T + D X^T, then S as above
// Four more waves bring the next chunk's rows into LDS and make its scalars: a wave that
// reads LDS waits for all the LDS loads it has under way, so the loads are others'.
template <typename T, int N, int NW>
struct OutLds {
  typedef SsmRows<T, N, kSsmC> KR;
  typedef SsmRows<T, 16 * NW, kSsmC> VR;
  static constexpr int B = 0, C = KR::bytes, X = 2 * KR::bytes, one = X + 2 * VR::bytes;
  static constexpr int image = img_bytes<T>(kNear), small = 2 * image + 4 * kSmFloats * 4;
  static constexpr int bufs = 2 * one + small <= 160 * 1024 ? 2 : 1;
  static constexpr int P = bufs * one, S = P + 2 * image, total = S + 4 * kSmFloats * 4;
};
template <typename T, int N, int NW>
__global__ void __launch_bounds__(128 * NW + 256, NW == 4 ? 3 : 2) carve_ssm_out_kernel(SsmArgs a) {
  typedef OutLds<T, N, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  constexpr int NP = N / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slices = a.P / (16 * NW), rep = a.H / a.G, units = rep * slices, pairs = (units + 1) / 2;
  SsmSpan p;
  int rest;
  if (!ssm_block(a, a.G * pairs, p, rest)) return;
  const int grp = rest / pairs, u0 = 2 * (rest % pairs);   // the workgroup's first unit of the group
  const int have = min(2, units - u0);
  const auto scal = [&](int u, int ch) { return reinterpret_cast<float*>(smem + L::S) + (2 * u + (ch & 1)) * kSmFloats; };
  const auto rows = [&](int ch) { return smem + (L::bufs == 2 ? (ch & 1) * L::one : 0); };

  if (wave >= 2 * NW) {   // ---- rows and scalars
    const int k = wave - 2 * NW;
    const int h0 = grp * rep + u0 / slices, h1 = grp * rep + (u0 + have - 1) / slices;   // heads of the units
    const T* Bm = reinterpret_cast<const T*>(a.Bm) + p.q.batch * a.bs[0] + p.first * a.bs[1] + grp * a.bs[2];
    const T* Cm = reinterpret_cast<const T*>(a.Cm) + p.q.batch * a.cs[0] + p.first * a.cs[1] + grp * a.cs[2];
    const T* x = reinterpret_cast<const T*>(a.x) + p.q.batch * a.xs[0] + p.first * a.xs[1];
    const T* x0 = x + h0 * a.xs[2] + u0 % slices * 16 * NW;
    const T* x1 = x + h1 * a.xs[2] + (u0 + have - 1) % slices * 16 * NW;
    const auto issue = [&](int ch) {
      const int len = min(kSsmC, p.len - ch * kSsmC);
      char* to = rows(ch);
      if (k == 0) KR::template dma<1>(to + L::B, Bm + (long long)ch * kSsmC * a.bs[1], (int)(a.bs[1] * sizeof(T)), len, 0, lane);
      if (k == 1) KR::template dma<1>(to + L::C, Cm + (long long)ch * kSsmC * a.cs[1], (int)(a.cs[1] * sizeof(T)), len, 0, lane);
      if (k >= 2) VR::template dma<1>(to + L::X + (k - 2) * VR::bytes, (k == 2 ? x0 : x1) + (long long)ch * kSsmC * a.xs[1],
                                      (int)(a.xs[1] * sizeof(T)), len, 0, lane);
    };
    const int hs = k == 2 ? h0 : h1;   // waves 2 and 3: scalars of a unit
    Steps<T> st = steps_of<T>(a, p, hs, lane);
    if (k >= 2 && p.nch > 0) {
      st.fetch(0);
      st.make(0, scal(k - 2, 0));
      if (p.nch > 1) st.fetch(1);
    }
    if (L::bufs == 2 && p.nch > 0) issue(0);
#pragma unroll 1
    for (int ch = 0; ch < p.nch; ++ch) {
      if (L::bufs == 1) {
        __syncthreads();   // (0) the rows of the chunk before are no longer read
        issue(ch);
      }
      vm_wait_all();
      __syncthreads();     // (1)
      if (L::bufs == 2 && ch + 1 < p.nch) issue(ch + 1);
      if (k >= 2 && ch + 1 < p.nch) {
        st.make(ch + 1, scal(k - 2, ch + 1));
        if (ch + 2 < p.nch) st.fetch(ch + 2);
      }
      __syncthreads();     // (2)
    }
    return;
  }

  // ---- outputs and states
  const int g = lane >> 4, c = lane & 15, un = wave / NW, w = wave % NW;
  const bool mine = un < have;
  const int unit = min(u0 + un, units - 1), h = grp * rep + unit / slices, p0 = unit % slices * 16 * NW + 16 * w;
  const size_t pn = (size_t)a.P * N, row = (size_t)(p0 + c) * N + 4 * g;
  Tile<T, N> t;
  if (p.s > 0) t.load(a.Z + ((size_t)p.slot * a.H + h) * pn + row);
  else if (a.S0) t.load(a.S0 + ((size_t)p.q.n * a.H + h) * pn + row);
  else t.zero();
  T* y = reinterpret_cast<T*>(a.y) + (((size_t)p.q.batch * a.T + p.first) * a.H + h) * a.P + p0 + 4 * g;
  const size_t yrow = (size_t)a.H * a.P;
  const float skip = a.D ? a.D[h] : 0.0f;
#pragma unroll 1
  for (int ch = 0; ch < p.nch; ++ch) {
    const int len = min(kSsmC, p.len - ch * kSsmC);
    const char* buf = rows(ch);
    if (L::bufs == 1) __syncthreads();   // (0)
    if (a.S_chunks && mine) SsmState<T, N>::st(a.S_chunks + ((size_t)(p.slot0 + ch) * a.H + h) * pn * 4, pn, p0, t.S, lane);
    __syncthreads();   // (1) the chunk's rows and scalars are there, the images no longer read
    // L d C B^T: rows j of the result (tiles 2 s, 2 s + 1), columns the tokens i of a tile
    {
      constexpr int PER = 8 / (2 * NW);   // (i, s) of a wave: i = 0 .. 3, s = 0, 1
#pragma unroll
      for (int v = 0; v < PER; ++v) {
        const int id = wave + 2 * NW * v, i = id & 3, s = id >> 2;
        if (s > i / 2) continue;   // (uniform)
        f32x4 M[2] = {zero4(), zero4()};
#pragma unroll
        for (int q = 0; q < NP; ++q) {
          const Fr<T> fc = KR::nat(buf + L::C, i, q, g, c);
#pragma unroll
          for (int b = 0; b < 2; ++b) M[b] = mma<T>(KR::nat(buf + L::B, 2 * s + b, q, g, c), fc, M[b]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (u >= have) break;   // (uniform)
          const float* sc = scal(u, ch);
          const float Gh = sc[kSmGh * kSsmC + 16 * i + c], Gl = sc[kSmGl * kSsmC + 16 * i + c];
          f32x4 W[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int at = 32 * s + 16 * b + 4 * g;
            const f32x4 gh = four(sc + kSmGh * kSsmC + at), gl = four(sc + kSmGl * kSsmC + at), d = four(sc + kSmD * kSsmC + at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              W[b][e] = masked(at + e <= 16 * i + c, M[b][e] * (decay_between(Gh, Gl, gh[e], gl[e]) * d[e]));
          }
          st_img<T, kNear>(smem + L::P + u * L::image, img_lower(i, s), lane, W[0], W[1]);
        }
      }
    }
    Fi<T, kNear> Sf[NP];
#pragma unroll
    for (int q = 0; q < NP; ++q) Sf[q] = to_fi<T, kNear>(t.S[2 * q], t.S[2 * q + 1]);
    __syncthreads();   // (2)
    if (!mine) continue;
    const float* sc = scal(un, ch);
    const char* xb = buf + L::X + un * VR::bytes;
    const Fr<T> fx[2] = {VR::tr32(xb, 0, w, g, c), VR::tr32(xb, 1, w, g, c)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 o = zero4(), z = zero4();
#pragma unroll
      for (int q = 0; q < NP; ++q) o = mma<T>(Sf[q], KR::nat(buf + L::C, i, q, g, c), o);
#pragma unroll
      for (int s = 0; s <= i / 2; ++s) z = mma<T>(fx[s], ld_img<T, kNear>(smem + L::P + un * L::image, img_lower(i, s), lane), z);
      const int tok = 16 * i + c;
      const f32x4 xv = Quad<T>::f32(VR::quad(xb, i, w, g, c));
      o = o * sc[kSmGam * kSsmC + tok] + z + xv * skip;
      if (tok < len) Quad<T>::st(y + (size_t)(ch * kSsmC + tok) * yrow, Quad<T>::cvt(o));
    }
    t.template add<KR>(buf + L::B, fx, [&](int at) { return four(sc + kSmEndD * kSsmC + at); }, sc[kSmWhole], g, c);
  }
  settle();
  if (mine && a.S_T && p.s == p.nspan - 1) t.store(a.S_T + ((size_t)p.q.n * a.H + h) * pn + row);
}

template <typename K>
bool lds_attr(K kern, int lds) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
}
int launched() { return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP; }

template <typename T, int N, int NW, bool REV>
int launch_state(const SsmArgs& a, int full, hipStream_t s) {
  constexpr int lds = StateLds<T, N, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_ssm_state_kernel<T, N, NW, REV>;
  if (!lds_attr(kern, lds)) return CARVE_ERR_HIP;
  hipLaunchKernelGGL(kern, dim3(ssm_grid(a.nspans, a.H * (a.P / (16 * NW)))), dim3(64 * NW), lds, s, a, full);
  return launched();
}
template <bool REV>
int launch_join(const SsmArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((carve_ssm_join_kernel<REV>), dim3((unsigned)(((size_t)a.P * a.N / 4 + 255) / 256), a.H, a.nseq < 65535 ? a.nseq : 65535), dim3(256), 0, s, a);
  return launched();
}
// Whether any sequence can have more than one span (packed lengths are not known here)
bool split(const SsmArgs& a) { return a.T > a.span * kSsmC; }

template <typename T, int N, int NW, bool REV>
int launch_spans(const SsmArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  if (split(a)) {
    int st = launch_state<T, N, NW, REV>(a, 0, s);
    if (st) return st;
    mark(s);
    st = launch_join<REV>(a, s);
    if (st) return st;
    mark(s);
  }
  if (REV) {
    const int st = launch_state<T, N, NW, REV>(a, 1, s);
    if (st) return st;
    mark(s);
  }
  return CARVE_OK;
}
template <typename T, int N, int NW>
int launch_fwd_t(const SsmArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  int st = launch_spans<T, N, NW, false>(a, s, mark);
  if (st) return st;
  constexpr int lds = OutLds<T, N, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_ssm_out_kernel<T, N, NW>;
  if (!lds_attr(kern, lds)) return CARVE_ERR_HIP;
  const int pairs = (a.H / a.G * (a.P / (16 * NW)) + 1) / 2;
  hipLaunchKernelGGL(kern, dim3(ssm_grid(a.nspans, a.G * pairs)), dim3(128 * NW + 256), lds, s, a);
  st = launched();
  mark(s);
  return st;
}

}  // namespace

// value rows of a unit: 64, or 32 where P is no multiple of it, and with f32 keys of 128,
// whose products of 64 rows do not fit the registers (as in the C entry points' plan)
#define CARVE_SSM_BY(call)                                                      \
  const bool wide = a.P % 64 == 0;                                              \
  if (dtype == CARVE_BF16) {                                                    \
    switch (a.N) {                                                              \
      case 32: return wide ? call(bf16_t, 32, 4) : call(bf16_t, 32, 2);         \
      case 64: return wide ? call(bf16_t, 64, 4) : call(bf16_t, 64, 2);         \
      case 128: return wide ? call(bf16_t, 128, 4) : call(bf16_t, 128, 2);      \
    }                                                                           \
  } else {                                                                      \
    switch (a.N) {                                                              \
      case 32: return wide ? call(float, 32, 4) : call(float, 32, 2);           \
      case 64: return wide ? call(float, 64, 4) : call(float, 64, 2);           \
      case 128: return call(float, 128, 2);                                     \
    }                                                                           \
  }                                                                             \
  return CARVE_ERR_UNSUPPORTED;

int launch_ssm_fwd(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
#define CALL(T, N, NW) launch_fwd_t<T, N, NW>(a, s, mark)
  CARVE_SSM_BY(CALL)
#undef CALL
}
int launch_ssm_spans_rev(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t)) {
#define CALL(T, N, NW) launch_spans<T, N, NW, true>(a, s, mark)
  CARVE_SSM_BY(CALL)
#undef CALL
}
#undef CARVE_SSM_BY

}  // namespace carve
