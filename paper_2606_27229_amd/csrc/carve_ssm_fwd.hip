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
  __device__ __forceinline__ void scale(float by) {
#pragma unroll
    for (int j = 0; j < N / 16; ++j) S[j] *= by;
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

// Scalars and C B^T of every chunk slot: blockIdx.y < G a group's products, wave w making
// its column tile w; behind them the scalars of 16 heads, four a wave (4 x 4096 tokens of 32
// heads: 10 us, one after another of loads, sums by shuffles and stores; 6 of a few chunks).
constexpr int kPrepHeads = 16;
template <typename T, int N, bool BWD>
__global__ void __launch_bounds__(256) carve_ssm_prep_kernel(SsmArgs a) {
  typedef SsmRows<T, N, kSsmC> KR;
  constexpr int NP = N / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slot = blockIdx.x;
  const SsmSeq q = ssm_find(a, slot, kSsmC);
  const int ch = slot - ssm_slot0(a, q, kSsmC);
  if (ch < 0 || (long long)ch * kSsmC >= q.len) return;   // a slot of no chunk
  const int first = q.first + ch * kSsmC, len = min(kSsmC, q.len - ch * kSsmC);
  if ((int)blockIdx.y >= a.G) {
    const int h0 = ((int)blockIdx.y - a.G) * kPrepHeads + w;
    const T* dt = reinterpret_cast<const T*>(a.dt) + q.batch * a.ds[0] + (first + min(lane, len - 1)) * a.ds[1];
    float raw[kPrepHeads / 4], bias[kPrepHeads / 4], A[kPrepHeads / 4];
#pragma unroll
    for (int u = 0; u < kPrepHeads / 4; ++u) {
      const int h = min(h0 + 4 * u, a.H - 1);
      raw[u] = (float)dt[h], bias[u] = a.dt_bias ? a.dt_bias[h] : 0.0f, A[u] = a.A[h];
    }
    // (heads behind the last repeat it, so that the four of a wave run side by side)
#pragma unroll
    for (int u = 0; u < kPrepHeads / 4; ++u)
      ssm_scalars<BWD>(raw[u], lane < len, bias[u], A[u], a.softplus, lane,
                       reinterpret_cast<float*>(a.scal) + ((size_t)slot * a.H + min(h0 + 4 * u, a.H - 1)) * (BWD ? kSmBwd : kSmFwd));
    return;
  }
  const int grp = blockIdx.y, g = lane >> 4, c = lane & 15;
  KR::template dma<4>(smem, reinterpret_cast<const T*>(a.Bm) + q.batch * a.bs[0] + first * a.bs[1] + grp * a.bs[2],
                      (int)(a.bs[1] * sizeof(T)), len, w, lane);
  KR::template dma<4>(smem + KR::bytes, reinterpret_cast<const T*>(a.Cm) + q.batch * a.cs[0] + first * a.cs[1] + grp * a.cs[2],
                      (int)(a.cs[1] * sizeof(T)), len, w, lane);
  vm_wait_all();
  __syncthreads();
  char* out = a.cb + ((size_t)slot * a.G + grp) * (BWD ? 2 : 1) * kSsmCB + 16 * lane;
#pragma unroll
  for (int way = 0; way < (BWD ? 2 : 1); ++way) {   // rows j of B, then rows i of C
    const char *rows = smem + way * KR::bytes, *cols = smem + (1 - way) * KR::bytes;
    f32x4 M[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) M[i] = zero4();
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const Fr<T> f = KR::nat8(cols, w, p, g, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) M[i] = mma<T>(KR::nat8(rows, i, p, g, c), f, M[i]);
    }
    settle(M);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (way ? i >= w : i <= w) *reinterpret_cast<f32x4*>(out + (way ? kSsmCB + ssm_tile(i, w) : ssm_tile(w, i))) = M[i];
  }
}

// Chains of states without outputs.  Forward (REV false): what each span but a sequence's
// last adds to the state.  Reverse: E <- e^{G_C} E + dY^T (e^G C) from the last chunk to the
// first: what each span but the first adds, or (FULL), from the span's own end, E of every
// chunk's end, then dS0.
// (4 x 4096 tokens of 32 heads: 37 us for the spans' sums; 99 for every chunk's E, whose 268 MB a
// fill of memory takes 39 for.)
template <typename T, int N, int NW>
struct StateLds {
  typedef SsmRows<T, N, kSsmC> KR;
  typedef SsmRows<T, 16 * NW, kSsmC> VR;
  static constexpr int K = 0, V = KR::bytes, S = V + VR::bytes, total = S + kSmFwd * 4;
};
template <typename T, int N, int NW, bool REV, bool FULL>
__global__ void __launch_bounds__(64 * NW, 2) carve_ssm_state_kernel(SsmArgs a) {
  typedef StateLds<T, N, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const float* sc = reinterpret_cast<const float*>(smem + L::S);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int slices = a.P / (16 * NW);
  SsmSpan p;
  int rest;
  if (!ssm_block(a, a.H * slices, p, rest)) return;
  const int h = rest / slices, p0 = rest % slices * 16 * NW, grp = h / (a.H / a.G);
  if (!FULL && p.s == (REV ? 0 : p.nspan - 1)) return;
  const size_t pn = (size_t)a.P * N, row = (size_t)(p0 + 16 * w + c) * N + 4 * g;
  float* zs = a.Z + ((size_t)p.slot * a.H + h) * pn + row;
  Tile<T, N> t;
  if (!FULL) t.zero();
  else if (p.s < p.nspan - 1) t.load(zs);
  else if (a.dS_T) t.load(a.dS_T + ((size_t)p.q.n * a.H + h) * pn + row);
  else t.zero();
  const T* kb = REV ? reinterpret_cast<const T*>(a.Cm) + p.q.batch * a.cs[0] + p.first * a.cs[1] + grp * a.cs[2]
                    : reinterpret_cast<const T*>(a.Bm) + p.q.batch * a.bs[0] + p.first * a.bs[1] + grp * a.bs[2];
  const long long ks = REV ? a.cs[1] : a.bs[1], vs = REV ? (long long)a.H * a.P : a.xs[1];
  const T* vb = REV ? reinterpret_cast<const T*>(a.dy) + (((size_t)p.q.batch * a.T + p.first) * a.H + h) * a.P + p0
                    : reinterpret_cast<const T*>(a.x) + p.q.batch * a.xs[0] + p.first * a.xs[1] + h * a.xs[2] + p0;
  // (in reverse the state has the sign of the chunk that it is the gradient behind)
  float decay = 1.0f, sign = REV ? ssm_sign(p.slot0 + p.nch - 1) : 1.0f;
  if (FULL) t.scale(sign);
#pragma unroll 1
  for (int i = 0; i < p.nch; ++i) {
    const int ch = REV ? p.nch - 1 - i : i, len = min(kSsmC, p.len - ch * kSsmC);
    if (i > 0) __syncthreads();   // the rows of the chunk before are no longer read
    KR::template dma<NW>(smem + L::K, kb + (long long)ch * kSsmC * ks, (int)(ks * sizeof(T)), len, w, lane);
    VR::template dma<NW>(smem + L::V, vb + (long long)ch * kSsmC * vs, (int)(vs * sizeof(T)), len, w, lane);
    dma_flat<NW, 2>(smem + L::S, a.scal + ((size_t)(p.slot0 + ch) * a.H + h) * (REV ? kSmBwd : kSmFwd) * 4, w, lane);
    vm_wait_all();
    __syncthreads();
    // the gradient of the state behind this chunk (ahead of the barrier: 110 us, here 99)
    if (FULL) t.store(a.E_chunks + ((size_t)(p.slot0 + ch) * a.H + h) * pn + row);
    const Fr<T> v[2] = {VR::tr32(smem + L::V, 0, w, g, c), VR::tr32(smem + L::V, 1, w, g, c)};
    if (REV) sign = -sign;
    t.template add<KR>(smem + L::K, v, [&](int at) {
      return REV ? four(sc + kSmGam * kSsmC + at) * sign : four(sc + kSmEndD * kSsmC + at);
    }, REV ? -sc[kSmWhole] : sc[kSmWhole], g, c);
    decay *= sc[kSmWhole];
  }
  settle(t.S);
  if (REV) t.scale(sign);
  if (!FULL) {
    t.store(zs);
    if (tid == 0 && p0 == 0) a.Zg[(size_t)p.slot * a.H + h] = decay;
  } else if (p.s == 0 && a.dS0) {
    t.store(a.dS0 + ((size_t)p.q.n * a.H + h) * pn + row);
  }
}

// Joins the spans of every sequence: Z becomes the state each span starts from (REV: the
// gradient of the state it ends with).  Elementwise along the sequence: four values a
// thread; the spans next to come are loaded ahead of the sum that waits for them (8 spans of
// 4 sequences, 32 heads: 11 us, 67 MB).
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
//   all waves   L d C B^T of both units from C B^T, a pair of tiles a wave: operand images in LDS
//   its waves   Y^T = S (e^G C)^T + X^T (L d C B^T)^T + D X^T, then S as above
// Bound by the latency of these steps: two workgroups a compute unit take turns with loads
// and products (4 x 4096 tokens of 32 heads: 79 us, 130 with every chunk's state; without loads
// and stores 67 of 82; vector instructions issue in 32 % of the cycles, matrix cores work in 21 %).  One
// workgroup a compute unit with waves that load a chunk ahead took 97, one unit a workgroup 113.
// Of two waves the one that is further on in its chunk goes first, so that its workgroup's loads
// begin (82 -> 79 us, with states 142 -> 130).
template <typename T, int N, int NW>
struct OutLds {
  typedef SsmRows<T, N, kSsmC> KR;
  typedef SsmRows<T, 16 * NW, kSsmC> VR;
  static constexpr int B = 0, C = KR::bytes, X = 2 * KR::bytes;
  static constexpr int image = img_bytes<T>(kNear), P = X + 2 * VR::bytes, S = P + 2 * image, total = S + 2 * kSmFwd * 4;
};
template <typename T, int N, int NW, bool KEEP>
__global__ void __launch_bounds__(128 * NW, sizeof(T) == 2 && NW == 4 ? 4 : 2) carve_ssm_out_kernel(SsmArgs a) {
  typedef OutLds<T, N, NW> L;
  typedef typename L::KR KR;
  typedef typename L::VR VR;
  constexpr int NP = N / 32, WAVES = 2 * NW, PER = 8 / WAVES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15, un = wave / NW, w = wave % NW;
  const int slices = a.P / (16 * NW), rep = a.H / a.G, units = rep * slices, pairs = (units + 1) / 2;
  SsmSpan p;
  int rest;
  if (!ssm_block(a, a.G * pairs, p, rest)) return;
  const int grp = rest / pairs, u0 = 2 * (rest % pairs);   // the workgroup's first unit of the group
  const int have = min(2, units - u0);
  const bool mine = un < have;
  // (waves of a unit that is not there do the other's work and write nothing)
  const int unit = u0 + min(un, have - 1), h = grp * rep + unit / slices, slice0 = unit % slices * 16 * NW, p0 = slice0 + 16 * w;
  const size_t pn = (size_t)a.P * N, row = (size_t)(p0 + c) * N + 4 * g;
  const float* scal = reinterpret_cast<const float*>(smem + L::S);
  const float* sc = scal + un * kSmFwd;
  Tile<T, N> t;
  if (p.s > 0) t.load(a.Z + ((size_t)p.slot * a.H + h) * pn + row);
  else if (a.S0) t.load(a.S0 + ((size_t)p.q.n * a.H + h) * pn + row);
  else t.zero();
  const T* Bm = reinterpret_cast<const T*>(a.Bm) + p.q.batch * a.bs[0] + p.first * a.bs[1] + grp * a.bs[2];
  const T* Cm = reinterpret_cast<const T*>(a.Cm) + p.q.batch * a.cs[0] + p.first * a.cs[1] + grp * a.cs[2];
  const T* x = reinterpret_cast<const T*>(a.x) + p.q.batch * a.xs[0] + p.first * a.xs[1] + h * a.xs[2] + slice0;
  T* y = reinterpret_cast<T*>(a.y) + (((size_t)p.q.batch * a.T + p.first) * a.H + h) * a.P + p0;
  const size_t yrow = (size_t)a.H * a.P;
  const float skip = a.D ? a.D[h] : 0.0f;
  const char* xb = smem + L::X + un * VR::bytes;
#pragma unroll 1
  for (int ch = 0; ch < p.nch; ++ch) {
    const int len = min(kSsmC, p.len - ch * kSsmC);
    if (ch > 0) __syncthreads();   // (0) the chunk before is done with
    KR::template dma<WAVES>(smem + L::B, Bm + (long long)ch * kSsmC * a.bs[1], (int)(a.bs[1] * sizeof(T)), len, wave, lane);
    KR::template dma<WAVES>(smem + L::C, Cm + (long long)ch * kSsmC * a.cs[1], (int)(a.cs[1] * sizeof(T)), len, wave, lane);
    VR::template dma<NW>(smem + L::X + un * VR::bytes, x + (long long)ch * kSsmC * a.xs[1], (int)(a.xs[1] * sizeof(T)), len, w, lane);
    dma_flat<NW, 2>(smem + L::S + un * kSmFwd * 4, a.scal + ((size_t)(p.slot0 + ch) * a.H + h) * kSmFwd * 4, w, lane);
    // C B^T of the wave's tiles (i, j = 2 s, 2 s + 1), i = 0 .. 3, s = 0, 1
    f32x4 M[PER][2];
#pragma unroll
    for (int v = 0; v < PER; ++v) {
      const int id = wave + WAVES * v, i = id & 3, s = id >> 2;
      const char* cb = a.cb + ((size_t)(p.slot0 + ch) * a.G + grp) * kSsmCB + 16 * lane;
#pragma unroll
      for (int b = 0; b < 2; ++b) M[v][b] = 2 * s + b <= i ? *reinterpret_cast<const f32x4*>(cb + ssm_tile(i, 2 * s + b)) : zero4();
    }
    vm_wait_all();
    __syncthreads();   // (1) its rows and scalars are there
    __builtin_amdgcn_s_setprio(1);
    // (stores behind the barrier: ahead of it the loads, or what waits for them, take 159 us at 4 x
    // 4096 tokens of 32 heads, here 142; a unit that is not there writes the other's states, which are its own)
    if (KEEP) t.store(a.S_chunks + ((size_t)(p.slot0 + ch) * a.H + h) * pn + row);
    // L d C B^T: rows j of the result (tiles 2 s, 2 s + 1), columns the tokens i of a tile
#pragma unroll
    for (int v = 0; v < PER; ++v) {
      const int id = wave + WAVES * v, i = id & 3, s = id >> 2;
      if (s > i / 2) continue;   // (uniform)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float* su = scal + u * kSmFwd;
        const float Gh = su[kSmGh * kSsmC + 16 * i + c], Gl = su[kSmGl * kSsmC + 16 * i + c];
        f32x4 W[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int j = 2 * s + b, at = 16 * j + 4 * g;
          if (j < i) {   // (uniform) from a tile before: one exponential a token, F d of the other
            const float down = decay_between(Gh, Gl, su[kSmTile + j], su[kSmTile + 4 + j]);
            W[b] = M[v][b] * (four(su + kSmFD * kSsmC + at) * down);
          } else {       // within the tile, and nothing from behind it
            const f32x4 gh = four(su + kSmGh * kSsmC + at), gl = four(su + kSmGl * kSsmC + at), d = four(su + kSmD * kSsmC + at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              W[b][e] = masked(at + e <= 16 * i + c, M[v][b][e] * (decay_between(Gh, Gl, gh[e], gl[e]) * d[e]));
          }
        }
        st_img<T, kNear>(smem + L::P + u * L::image, img_lower(i, s), lane, W[0], W[1]);
      }
    }
    __syncthreads();   // (2) the images are there
    __builtin_amdgcn_s_setprio(2);
    const Fr<T> fx[2] = {VR::tr32(xb, 0, w, g, c), VR::tr32(xb, 1, w, g, c)};
    // (four token tiles side by side: a tile's products follow each other)
    f32x4 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = zero4();
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const Fi<T, kNear> Sf = to_fi<T, kNear>(t.S[2 * q], t.S[2 * q + 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = mma<T>(Sf, KR::nat(smem + L::C, i, q, g, c), o[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= sc[kSmGam * kSsmC + 16 * i + c];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 2 * s; i < 4; ++i) o[i] = mma<T>(fx[s], ld_img<T, kNear>(smem + L::P + un * L::image, img_lower(i, s), lane), o[i]);
    }
    if (mine) {
      const RowStore<T> out(y + (size_t)ch * kSsmC * yrow, yrow, len, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) out.st(16 * i + c, 4 * g, o[i] + Quad<T>::f32(VR::quad(xb, i, w, g, c)) * skip);
    }
    t.template add<KR>(smem + L::B, fx, [&](int at) { return four(sc + kSmEndD * kSsmC + at); }, sc[kSmWhole], g, c);
    __builtin_amdgcn_s_setprio(0);
  }
  settle(t.S);
  if (mine && a.S_T && p.s == p.nspan - 1) t.store(a.S_T + ((size_t)p.q.n * a.H + h) * pn + row);
}

template <typename K>
bool lds_attr(K kern, int lds) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
}
int launched() { return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP; }

template <typename T, int N, int NW, bool REV, bool FULL>
int launch_state(const SsmArgs& a, hipStream_t s) {
  constexpr int lds = StateLds<T, N, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_ssm_state_kernel<T, N, NW, REV, FULL>;
  if (!lds_attr(kern, lds)) return CARVE_ERR_HIP;
  hipLaunchKernelGGL(kern, dim3(ssm_grid(a.nspans, a.H * (a.P / (16 * NW)))), dim3(64 * NW), lds, s, a);
  return launched();
}
template <bool REV>
int launch_join(const SsmArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((carve_ssm_join_kernel<REV>), dim3((unsigned)(((size_t)a.P * a.N / 4 + 255) / 256), a.H, a.nseq < 65535 ? a.nseq : 65535), dim3(256), 0, s, a);
  return launched();
}
// Whether any sequence can have more than one span (packed lengths are not known here)
bool split(const SsmArgs& a) { return a.T > a.span * kSsmC; }

template <typename T, int N, bool BWD>
int launch_prep(const SsmArgs& a, hipStream_t s) {
  constexpr int lds = 2 * SsmRows<T, N, kSsmC>::bytes;
  const auto kern = carve_ssm_prep_kernel<T, N, BWD>;
  if (!lds_attr(kern, lds)) return CARVE_ERR_HIP;
  hipLaunchKernelGGL(kern, dim3(a.nslots, a.G + (a.H + kPrepHeads - 1) / kPrepHeads), dim3(256), lds, s, a);
  return launched();
}
template <typename T, int N, int NW, bool REV>
int launch_spans(const SsmArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  {
    const int st = launch_prep<T, N, REV>(a, s);
    if (st) return st;
    mark(s);
  }
  if (split(a)) {
    int st = launch_state<T, N, NW, REV, false>(a, s);
    if (st) return st;
    mark(s);
    st = launch_join<REV>(a, s);
    if (st) return st;
    mark(s);
  }
  if constexpr (REV) {
    const int st = launch_state<T, N, NW, true, true>(a, s);
    if (st) return st;
    mark(s);
  }
  return CARVE_OK;
}
template <typename T, int N, int NW, bool KEEP>
int launch_out(const SsmArgs& a, hipStream_t s) {
  constexpr int lds = OutLds<T, N, NW>::total;
  static_assert(lds <= 160 * 1024, "LDS");
  const auto kern = carve_ssm_out_kernel<T, N, NW, KEEP>;
  if (!lds_attr(kern, lds)) return CARVE_ERR_HIP;
  const int pairs = (a.H / a.G * (a.P / (16 * NW)) + 1) / 2;
  hipLaunchKernelGGL(kern, dim3(ssm_grid(a.nspans, a.G * pairs)), dim3(128 * NW), lds, s, a);
  return launched();
}
template <typename T, int N, int NW>
int launch_fwd_t(const SsmArgs& a, hipStream_t s, void (*mark)(hipStream_t)) {
  int st = launch_spans<T, N, NW, false>(a, s, mark);
  if (st) return st;
  st = a.S_chunks ? launch_out<T, N, NW, true>(a, s) : launch_out<T, N, NW, false>(a, s);
  mark(s);
  return st;
}

}  // namespace

// value rows of a unit: 64, or 32 where P is no multiple of it, and with f32 states of 128 (as
// in the C entry points' plan, which has the figures)
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
