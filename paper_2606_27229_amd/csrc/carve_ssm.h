// carve_ssm.h -- shared pieces of the selective state space scan (a matrix state a head,
// one decay a token and head):
//   d_t = softplus(dt_t + dt_bias),  a_t = d_t A,
//   S_t = e^{a_t} S_{t-1} + d_t x_t B_t^T  (P x N),  y_t = S_t C_t + D x_t
// Chunk form over C = 64 tokens, G = prefix sums of a inside the chunk, L_ij = e^{G_i - G_j}
// for j <= i:
//   Y = e^G C S^T + (L d_j C B^T) X + D X
//   S <- e^{G_C} S + X^T (e^{G_C - G} d B)
// Unlike a delta rule's, a chunk's writes do not depend on the state, so spans of chunks
// run side by side: each adds up what it writes, one pass joins them along the sequence,
// and each then makes its outputs from its start state.  A span keeps its state in
// registers; only spans' states go through memory.
//
// Precision as in the gated delta rule (carve_gdr.h): decays and steps multiply f32 values;
// with bf16 tokens the f32 intermediates enter the matrix cores as sums of bf16 values,
// three towards f32 results and two towards bf16 ones; with f32 tokens every product is
// f32.  G is summed in 64 bits and kept as two floats.
#pragma once
#include "carve_gdr.h"
#include "carve_ops.h"

namespace carve {

constexpr int kSsmC = kGdrC;              // tokens of a chunk

struct SsmArgs {
  const void *x, *dt, *Bm, *Cm, *dy;
  const float *A, *D, *dt_bias, *S0, *dS_T;
  const int* offsets;      // packed sequences: [nseq + 1]; dense: NULL
  void *y, *dx, *ddt, *dBm, *dCm;
  float *S_T, *dA, *dD, *ddt_bias, *dS0;
  float *S_chunks, *E_chunks;   // [nslots][H][P][N]: states at chunk starts, state gradients at chunk ends (ssm_sign)
  float* Z;                // [nspans][H][P][N]: what a span adds, then the state it starts from
  float* Zg;               // [nspans][H]: its decay
  char* scal;              // [nslots][H]: scalars; cb: [nslots][G], C B^T (backward: twice)
  char* cb;
  float* part;             // [nslots][H][4]: a chunk's share of dA, ddt_bias, dD
  float* dBp;              // [splits][rows][G][N], dCp behind it: shares of dB, dC
  long long xs[3], bs[3], cs[3], ds[2];   // strides of batch, token, head (or group)
  int T, G, H, P, N, nseq, nslots, nspans, span, splits;   // span: chunks of a span
  int softplus;
};

// ---- sequences, chunk slots and spans --------------------------------------------------
// As for the gated delta rule: a sequence's units of L rows are slots floor(first / L) +
// sequence + unit where sequences are packed, sequence * units + unit else.
struct SsmSeq {
  int n, batch, first, len;
};
__device__ __forceinline__ SsmSeq ssm_seq(const SsmArgs& a, int n) {
  SsmSeq s;
  s.n = n;
  if (!a.offsets) {
    s.batch = n, s.first = 0, s.len = a.T;
  } else {
    int end;
    packed_seq(a.offsets, n, a.T, s.first, end);
    s.batch = 0, s.len = end - s.first;
  }
  return s;
}
__device__ __forceinline__ int ssm_units(int len, int L) { return (int)(((long long)len + L - 1) / L); }
__device__ __forceinline__ int ssm_slot0(const SsmArgs& a, const SsmSeq& s, int L) {
  return a.offsets ? s.first / L + s.n : s.n * ssm_units(a.T, L);
}
// sequence of a slot; its unit there may lie behind the sequence's last
__device__ __forceinline__ SsmSeq ssm_find(const SsmArgs& a, int slot, int L) {
  if (!a.offsets) return ssm_seq(a, slot / ssm_units(a.T, L));
  int lo = 0, hi = a.nseq - 1;   // the last n whose first slot is not behind this one
  while (lo < hi) {
    const int m = (lo + hi + 1) >> 1;
    if (min(max(a.offsets[m], 0), a.T) / L + m <= slot) lo = m;
    else hi = m - 1;
  }
  return ssm_seq(a, lo);
}

// ---- what chunks are made from: scalars of the heads, products of the groups -----------------
// Made once a call by carve_ssm_prep_kernel, as several kernels need them.
// Scalars of a (slot, head), floats.  Of every token: d; G / log 2 as two floats (far below
// any other behind the last token, so that what decays from a token before to one there is
// 0); e^G (0 there); E = e^{G_C - G}; E d; F d with F = e^{g - G}, g being G at the end of
// the token's tile of 16.  Then g / log 2 of every tile as two floats, and e^{G_C}; for the
// backward also F, and e^{G - g} of tiles 0, 1 and 2 at the tokens behind them.
enum : int { kSmD = 0, kSmGh = 1, kSmGl = 2, kSmGam = 3, kSmEnd = 4, kSmEndD = 5, kSmFD = 6, kSmTile = 7 * kSsmC,
             kSmWhole = kSmTile + 8, kSmFwd = 8 * kSsmC, kSmF = 8, kSmDown = 9, kSmBwd = 12 * kSsmC };
constexpr float kSmNever = -1e7f;   // (64 tokens reach -10^6)
// C B^T of a (slot, group): its ten tiles on and below the diagonal, 1 KB each as result
// tiles (rows j, columns i); tile (i, j) at ssm_tile(i, j).  For the backward the same with
// rows i, columns j behind them.
constexpr int kSsmCB = 10 * 1024;
__host__ __device__ constexpr int ssm_tile(int i, int j) { return (i * (i + 1) / 2 + j) * 1024; }

__device__ __forceinline__ float ssm_step_of(float z, int softplus) {
  return softplus ? fmaxf(z, 0.0f) + log1pf(expf(-fabsf(z))) : z;
}
// by one wave, a token a lane; raw: its dt
template <bool BWD>
__device__ __forceinline__ void ssm_scalars(float raw, bool in, float bias, float A, int softplus, int lane, float* out) {
  const float d = in ? ssm_step_of(raw + bias, softplus) : 0.0f;
  float ga = in ? d * A : 0.0f;
  ga = ga < kGdrMinG ? kGdrMinG : ga;
  double G = (double)ga * 1.4426950408889634;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const double up = __shfl_up(G, s);
    if (lane >= s) G += up;
  }
  const double all = __shfl(G, 63), tile = __shfl(G, lane | 15);
  const float Gh = (float)G, Gl = (float)(G - (double)Gh), end = exp2_f((float)(all - G)), f = exp2_f((float)(tile - G));
  out[kSmD * kSsmC + lane] = d;
  out[kSmGh * kSsmC + lane] = in ? Gh : kSmNever;
  out[kSmGl * kSsmC + lane] = in ? Gl : 0.0f;
  out[kSmGam * kSsmC + lane] = in ? exp2_f(Gh) * (1.0f + Gl * 0.69314718f) : 0.0f;
  out[kSmEnd * kSsmC + lane] = end;
  out[kSmEndD * kSsmC + lane] = end * d;
  out[kSmFD * kSsmC + lane] = f * d;
  if ((lane & 15) == 15) out[kSmTile + lane / 16] = Gh, out[kSmTile + 4 + lane / 16] = Gl;
  if (lane == 0) out[kSmWhole] = exp2_f((float)all);
  if (BWD) {
    out[kSmF * kSsmC + lane] = f;
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      const double gt = __shfl(G, 16 * t + 15);
      out[(kSmDown + t) * kSsmC + lane] = in && lane / 16 > t ? exp2_f((float)(G - gt)) : 0.0f;
    }
  }
}
// The matrix cores leave sums of bf16 products a little low (by up to a step of f32, whatever
// their sign).  x, B and C have means, so that all tokens' da would be low together, and dA,
// which adds them up, off by ten times what rounding leaves: in the backward every other
// chunk's E is kept, and its products with dy are made, negated.  (At 4 x 4096 tokens of 32
// heads dA is 8e-7 to 2e-6 off without, 5e-8 to 2e-7 with.)
__device__ __forceinline__ float ssm_sign(int slot) { return slot & 1 ? -1.0f : 1.0f; }
// e^{G_i - G_j}
__device__ __forceinline__ float decay_between(float ih, float il, float jh, float jl) { return exp2_f((ih - jh) + (il - jl)); }

// ---- LDS tiles -------------------------------------------------------------------------
// GdrRows of ROWS rows (its layout and operand reads); rows behind the last of `len`
// repeat it.
template <typename T, int COLS, int ROWS>
struct SsmRows : GdrRows<T, COLS> {
  typedef GdrRows<T, COLS> R;
  static constexpr int bytes = ROWS * R::RB;
  static_assert(bytes % 1024 == 0, "whole pieces of 1 KB");
  template <int NW>
  static __device__ __forceinline__ void dma(char* lds, const void* base, int stride, int len, int w, int lane) {
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (len - 1) * stride + R::RB, 0x00027000);
    constexpr int RPI = 1024 / R::RB;   // rows of a piece
#pragma unroll
    for (int u = 0; u < (bytes / 1024 + NW - 1) / NW; ++u) {
      const int i = w + NW * u;
      if ((bytes / 1024) % NW != 0 && i >= bytes / 1024) break;   // (uniform)
      const int row = i * RPI + lane / R::NCH, x = (lane % R::NCH) ^ R::swz(row);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_at(lds + 1024 * i), 16, (int)__umul24(min(row, len - 1), stride) + 16 * x, 0, 0, 0);
    }
  }
  // lane (g, c): row 16 i + c, columns 32 p + 8 g + e, e < 8: for products both of whose
  // operands are read so (16 bytes at once, where nat's order is that of result tiles)
  static __device__ __forceinline__ Fr<T> nat8(const char* lds, int i, int p, int g, int c) {
    Fr<T> f;
    if constexpr (sizeof(T) == 2) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(lds + (16 * i + c) * R::RB + (((4 * p + g) ^ R::swz(c)) << 4));
      f.a = __builtin_shufflevector(v, v, 0, 1, 2, 3);
      f.b = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    } else {
      f.a = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * R::RB + (((8 * p + 2 * g) ^ R::swz(c)) << 4)));
      f.b = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * R::RB + (((8 * p + 2 * g + 1) ^ R::swz(c)) << 4)));
    }
    return f;
  }
  // lane (g, c): row 16 i + c, columns 16 j + 4 g + e
  static __device__ __forceinline__ typename Quad<T>::q quad(const char* lds, int i, int j, int g, int c) {
    int o;
    if constexpr (sizeof(T) == 2) o = (((2 * j + (g >> 1)) ^ R::swz(c)) << 4) + ((g & 1) << 3);
    else o = ((4 * j + g) ^ R::swz(c)) << 4;
    return Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * R::RB + o));
  }
};

// ---- odds and ends ------------------------------------------------------------------------
// v where `on`, else 0, without a branch around what v takes (the compiler makes one of a
// plain choice: sixteen of them cost more than the exponentials that they skip)
__device__ __forceinline__ float masked(bool on, float v) {
  asm("" : "+v"(v));
  return on ? v : 0.0f;
}
// Eight wait states between products and the stores that follow and read their results, where
// the compiler has left one too few behind a loop.  The results pass through: the products
// cannot sink below the wait, nor what reads them rise above it.
template <int n>
__device__ __forceinline__ void settle(f32x4 (&v)[n]) {
  static_assert(n == 2 || n == 4 || n == 8, "accumulators of a wave");
  if constexpr (n == 2)
    asm volatile("s_nop 7" : "+v"(v[0]), "+v"(v[1]));
  else if constexpr (n == 4)
    asm volatile("s_nop 7" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
  else
    asm volatile("s_nop 7" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}

// Rows of a chunk to memory, four values a lane, without a branch around the store (which
// would part what the compiler may reorder): a buffer of the rows there are, behind which
// stores are dropped.  base: the chunk's first row (uniform); row: values of a row; cols:
// values from a row's base that lanes write at most.
template <typename T>
struct RowStore {
  __amdgpu_buffer_rsrc_t r;
  unsigned bytes;          // of a row
  __device__ __forceinline__ RowStore(T* base, size_t row, int len, int cols)
      : r(__builtin_amdgcn_make_buffer_rsrc(base, 0, (int)((unsigned)(len - 1) * (unsigned)(row * sizeof(T)) + cols * (unsigned)sizeof(T)), 0x00027000)),
        bytes((unsigned)(row * sizeof(T))) {}
  __device__ __forceinline__ void st(int tok, int col, f32x4 v) const {
    const int off = (int)((unsigned)tok * bytes + (unsigned)col * (unsigned)sizeof(T));
    if constexpr (sizeof(T) == 2)
      __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2_t, Quad<T>::cvt(v)), r, off, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_g, v), r, off, 0, 0);
  }
};

// ---- workgroups of the scans -------------------------------------------------------------
// Workgroup -> (span, head, slice of PW value rows).  Blocks 8 apart share an XCD: with many
// spans each goes to one XCD with all its heads, which read the same B and C from one L2;
// with few the heads are spread (by one XCD and spread: 32 spans of 4 x 4096 tokens of 32 heads
// 114 and 113 us, of 16381 tokens in two groups 119 and 123; 22 spans of 9 prompts 48 and 46).
constexpr int kSsmManySpans = 32;
__host__ __device__ inline unsigned ssm_grid(int nspans, int per) {
  return nspans >= kSsmManySpans ? (unsigned)((nspans + 7) / 8 * 8) * per : (unsigned)nspans * per;
}
struct SsmSpan {
  SsmSeq q;
  int slot, s, nspan;      // span slot; the span's number in its sequence, of nspan (at least 1)
  int first, len, nch;     // rows (of the sequence's batch) and chunks of the span
  int slot0;               // its first chunk's slot
};
__device__ __forceinline__ bool ssm_block(const SsmArgs& a, int per, SsmSpan& p, int& rest) {
  int b = blockIdx.x;
  if (a.nspans >= kSsmManySpans) {
    const int at = b / 8;
    p.slot = at / per * 8 + b % 8;
    rest = at % per;
  } else {
    p.slot = b / per;
    rest = b % per;
  }
  if (p.slot >= a.nspans) return false;
  const int L = a.span * kSsmC;
  p.q = ssm_find(a, p.slot, L);
  p.s = p.slot - ssm_slot0(a, p.q, L);
  p.nspan = max(ssm_units(p.q.len, L), 1);
  if (p.s < 0 || p.s >= p.nspan) return false;
  p.first = p.q.first + p.s * L;
  p.len = min(p.q.len - p.s * L, L);
  p.nch = (p.len + kSsmC - 1) / kSsmC;
  p.slot0 = ssm_slot0(a, p.q, kSsmC) + p.s * a.span;
  return true;
}

struct SsmStepArgs {
  const void *x, *dt, *Bm, *Cm;
  const float *A, *D, *dt_bias;
  const int* slots;
  float* state;
  void* y;
  long long xs[3], bs[3], cs[3], ds[2];
  int B, T, G, H, P, pool, softplus;
};

int launch_ssm_fwd(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_ssm_bwd(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_ssm_step(const SsmStepArgs& a, int N, int dtype, hipStream_t s);
// scalars and C B^T for the backward, then the chain of state gradients: spans' sums and
// their joining, E of every chunk, dS0
int launch_ssm_spans_rev(const SsmArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));

}  // namespace carve
