// carve_gdr.h -- shared pieces of the gated delta rule kernels (scalar decay per
// token and value head, decay before the prediction):
//   S~ = e^{g_t} S_{t-1},  u_t = beta_t (v_t - S~ k_t),  S_t = S~ + u_t k_t^T,
//   o_t = scale S_t q_t
// Chunk form over C = 64 tokens, G = prefix sums of g inside the chunk, D_ij =
// e^{G_i - G_j} for j <= i:
//   A_ij = beta_i D_ij k_i.k_j (j < i),  T = (I + A)^-1,  P_ij = D_ij q_i.k_j (j <= i)
//   R = beta (V - e^G K S^T),  U = T R,  O = scale (e^G Q S^T + P U)
//   S <- e^{G_C} S + U^T (e^{G_C - G} K)
//
// Precision.  Every decay factor scales rows of f32 results, never an operand, so
// q, k, v and dO enter the matrix cores as they are.  With bf16 tokens the f32
// intermediates (S, T, P, R, U and their adjoints) enter as the sum of two bf16
// values (Fi): what that leaves out is 2^-18 of a value, and the product of two
// such operands leaves out their low parts' product, 2^-18 again.  One bf16 value
// would leave out 2^-9, which states and decay gradients (f32 outputs) do not
// bear.  With f32 tokens every product is an f32 matrix-core product.
#pragma once
#include "../../include/carve.h"
#include "carve_dev.h"

namespace carve {

constexpr int kGdrC = 64;                 // tokens of a chunk
constexpr int kGdrImg = 6 * 2 * 1024;     // bytes of a triangular operand image (6 fragments of 2 planes)
constexpr int kGdrScal = 5 * kGdrC * 4;   // bytes of a chunk's scalars
constexpr float kGdrMinG = -1e4f;         // e^-1e4 is 0 in f32: a decay of -inf is taken as this

struct GdrArgs {
  const void *q, *k, *v, *beta, *dO;
  const float *g, *S0, *dS_T;
  const int* offsets;      // packed sequences: [nseq + 1]; dense: NULL
  void *o, *dq, *dk, *dv, *dbeta;
  float *S_T, *S_chunks, *dg, *dS0;
  char* ws;                // images and scalars of every (chunk slot, value head)
  float* dS_chunks;        // [nslots][Hv][Dv][Dk]: the state gradients at chunk ends (backward)
  long long qs[3], ks[3], vs[3];   // strides of batch, token, head
  int T, Hk, Hv, Dk, Dv, nseq, nslots, per;   // per: bytes of one (slot, head) in ws
  float scale;
};

// ---- sequences and chunk slots ----------------------------------------------------
// Dense: sequence n is batch n, its chunk c is slot n * ceil(T / C) + c.  Packed:
// sequence n is rows [offsets[n], offsets[n+1]) and its chunk c is slot
// floor(offsets[n] / C) + n + c, which leaves room for every sequence's last
// partial chunk without a sum over the sequences before it.  Offsets are device
// data, so they are clamped to the rows here: any values stay within the tensors,
// the chunk slots and (being found by search) the sequences.
struct GdrSeq {
  int batch, t0, len, slot0;   // batch index of the strided tensors, first row, rows, first slot
};
__device__ __forceinline__ GdrSeq gdr_seq(const GdrArgs& a, int n) {
  GdrSeq s;
  if (!a.offsets) {
    s.batch = n;
    s.t0 = 0;
    s.len = a.T;
    s.slot0 = n * ((a.T + kGdrC - 1) / kGdrC);
  } else {
    const int b = min(max(a.offsets[n], 0), a.T);
    s.batch = 0;
    s.t0 = b;
    s.len = min(max(a.offsets[n + 1], b), a.T) - b;
    s.slot0 = b / kGdrC + n;
  }
  return s;
}
// sequence of a slot and the chunk in it; false where the slot holds no tokens
__device__ __forceinline__ bool gdr_find(const GdrArgs& a, int slot, GdrSeq& s, int& n, int& chunk) {
  if (!a.offsets) {
    n = slot / ((a.T + kGdrC - 1) / kGdrC);
  } else {
    int lo = 0, hi = a.nseq - 1;   // the last n whose first slot is not behind this one
    while (lo < hi) {
      const int m = (lo + hi + 1) >> 1;
      if (min(max(a.offsets[m], 0), a.T) / kGdrC + m <= slot) lo = m;
      else hi = m - 1;
    }
    n = lo;
  }
  s = gdr_seq(a, n);
  chunk = slot - s.slot0;
  return chunk >= 0 && chunk * kGdrC < s.len;
}

// ---- matrix-core operands of depth 32 ------------------------------------------------
// A token fragment (Fr): lane (g, c) holds the eight elements k = 8 g .. 8 g + 7 (or
// any other eight, the same on both sides of a product) of row / column c.
template <typename T>
struct Fr {
  typename Quad<T>::q a, b;
};
// An f32 intermediate as an operand: two bf16 values whose sum it is, or f32.
template <typename T>
struct Fi;
template <>
struct Fi<bf16_t> {
  Fr<bf16_t> hi, lo;
};
template <>
struct Fi<float> {
  Fr<float> x;
};

__device__ __forceinline__ void split4(f32x4 x, bf16x4& hi, bf16x4& lo) {
  hi = Quad<bf16_t>::cvt(x);
  lo = Quad<bf16_t>::cvt(x - Quad<bf16_t>::f32(hi));
}
template <typename T>
__device__ __forceinline__ Fi<T> to_fi(f32x4 a, f32x4 b) {
  Fi<T> f;
  if constexpr (sizeof(T) == 2) {
    split4(a, f.hi.a, f.lo.a);
    split4(b, f.hi.b, f.lo.b);
  } else {
    f.x.a = a;
    f.x.b = b;
  }
  return f;
}
template <typename T>
__device__ __forceinline__ f32x4 mma(Fr<T> a, Fr<T> b, f32x4 c) {
  return Quad<T>::mma32(a.a, a.b, b.a, b.b, c);
}
template <typename T>
__device__ __forceinline__ f32x4 mma(const Fi<T>& a, Fr<T> b, f32x4 c) {
  if constexpr (sizeof(T) == 2) return mma<T>(a.hi, b, mma<T>(a.lo, b, c));
  else return mma<T>(a.x, b, c);
}
template <typename T>
__device__ __forceinline__ f32x4 mma(Fr<T> a, const Fi<T>& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) return mma<T>(a, b.hi, mma<T>(a, b.lo, c));
  else return mma<T>(a, b.x, c);
}
template <typename T>
__device__ __forceinline__ f32x4 mma(const Fi<T>& a, const Fi<T>& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) return mma<T>(a.hi, b.hi, mma<T>(a.hi, b.lo, mma<T>(a.lo, b.hi, c)));
  else return mma<T>(a.x, b.x, c);
}

// eight consecutive elements of a token row (16-byte aligned), zeros if !ok
template <typename T>
__device__ __forceinline__ Fr<T> ld_fr(const T* p, bool ok) {
  Fr<T> f;
  if constexpr (sizeof(T) == 2) {
    u32x4_t v = {0, 0, 0, 0};
    if (ok) v = *reinterpret_cast<const u32x4_t*>(p);
    const bf16x8 b = __builtin_bit_cast(bf16x8, v);
    f.a = __builtin_shufflevector(b, b, 0, 1, 2, 3);
    f.b = __builtin_shufflevector(b, b, 4, 5, 6, 7);
  } else {
    f.a = f.b = zero4();
    if (ok) {
      f.a = *reinterpret_cast<const f32x4*>(p);
      f.b = *reinterpret_cast<const f32x4*>(p + 4);
    }
  }
  return f;
}
// four consecutive elements at p and four 16 further on
template <typename T>
__device__ __forceinline__ Fr<T> ld_fr16(const T* p, bool ok) {
  Fr<T> f;
  f.a = f.b = Quad<T>::cvt(zero4());
  if (ok) {
    f.a = Quad<T>::ld(p);
    f.b = Quad<T>::ld(p + 16);
  }
  return f;
}

// ---- triangular operand images ----------------------------------------------------------
// A 64 x 64 triangle as A operands of depth 32 over its columns: fragment (i, s)
// holds rows 16 i .. and columns 32 s .. + 31, lane (g, c) the columns 32 s + 4 g + e
// and 32 s + 16 + 4 g + e of row 16 i + c.  Lower: s <= i / 2; upper: s >= i / 2.
__host__ __device__ constexpr int img_lower(int i, int s) { return i < 2 ? i : 2 + 2 * (i - 2) + s; }
__host__ __device__ constexpr int img_upper(int i, int s) { return i < 2 ? 2 * i + s : i + 2; }
template <typename T>
__device__ __forceinline__ Fi<T> ld_img(const char* img, int f, int lane) {
  const char* p = img + f * 2048 + lane * 16;
  Fi<T> x;
  if constexpr (sizeof(T) == 2) {
    const bf16x8 h = *reinterpret_cast<const bf16x8*>(p), l = *reinterpret_cast<const bf16x8*>(p + 1024);
    x.hi.a = __builtin_shufflevector(h, h, 0, 1, 2, 3);
    x.hi.b = __builtin_shufflevector(h, h, 4, 5, 6, 7);
    x.lo.a = __builtin_shufflevector(l, l, 0, 1, 2, 3);
    x.lo.b = __builtin_shufflevector(l, l, 4, 5, 6, 7);
  } else {
    x.x.a = *reinterpret_cast<const f32x4*>(p);
    x.x.b = *reinterpret_cast<const f32x4*>(p + 1024);
  }
  return x;
}
template <typename T>
__device__ __forceinline__ void st_img(char* img, int f, int lane, f32x4 a, f32x4 b) {
  char* p = img + f * 2048 + lane * 16;
  const Fi<T> x = to_fi<T>(a, b);
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<bf16x8*>(p) = __builtin_shufflevector(x.hi.a, x.hi.b, 0, 1, 2, 3, 4, 5, 6, 7);
    *reinterpret_cast<bf16x8*>(p + 1024) = __builtin_shufflevector(x.lo.a, x.lo.b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    *reinterpret_cast<f32x4*>(p) = x.x.a;
    *reinterpret_cast<f32x4*>(p + 1024) = x.x.b;
  }
}

// one (slot, head) of the workspace: images, then scalars [5][64]: e^G, e^{G_C - G},
// beta, and G as a sum of two floats
enum : int { kScGam = 0, kScEnd = 1, kScBeta = 2, kScGh = 3, kScGl = 4 };

// ---- token rows in LDS for reads across rows --------------------------------------------
// A [64][DK] token tile whose 16-column tiles (p, h) = columns 32 p + 8 q + 4 h + i
// (q, i = 0..3) are read transposed: as A operands K^T[j][t].  bf16: quad (p, q, h)
// of row r sits at quad 8 p + 4 h + (q ^ ((r >> 2) & 3)), rows 16 (mod 32) elements
// apart, which keeps the transposing reads free of bank conflicts.  f32: as it is,
// rows padded by 16 bytes.
template <typename T, int DK>
struct GdrRows {
  static constexpr int LD = sizeof(T) == 2 ? DK + 16 : DK + 4;
  static constexpr int bytes = kGdrC * LD * (int)sizeof(T);
  // the row's eight elements 32 p + 8 q ..
  static __device__ __forceinline__ void put(T* t, int r, int p, int q, Fr<T> f) {
    if constexpr (sizeof(T) == 2) {
      T* d = t + r * LD + 32 * p + 4 * (q ^ ((r >> 2) & 3));
      Quad<T>::st(d, f.a);
      Quad<T>::st(d + 16, f.b);
    } else {
      T* d = t + r * LD + 32 * p + 8 * q;
      Quad<T>::st(d, f.a);
      Quad<T>::st(d + 4, f.b);
    }
  }
  // lane (g, c): column c of tile (p, h), rows r0 + 4 g + e
  static __device__ __forceinline__ typename Quad<T>::q tr(const T* t, int r0, int p, int h, int g, int c) {
    if constexpr (sizeof(T) == 2) {
      return Quad<T>::ld_tr_at(t + (r0 + 4 * g + (c >> 2)) * LD + 32 * p + 16 * h + 4 * ((c & 3) ^ g));
    } else {
      const T* d = t + (r0 + 4 * g) * LD + 32 * p + 8 * (c >> 2) + 4 * h + (c & 3);
      typename Quad<T>::q o = {d[0], d[LD], d[2 * LD], d[3 * LD]};
      return o;
    }
  }
  static __device__ __forceinline__ Fr<T> frag(const T* t, int s, int p, int h, int g, int c) {
    Fr<T> f;
    f.a = tr(t, 32 * s, p, h, g, c);
    f.b = tr(t, 32 * s + 16, p, h, g, c);
    return f;
  }
};

// launches (carve_gdr_*.hip); mark: called after every launch
int launch_gdr_fwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_gdr_bwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_gdr_prep(const GdrArgs& a, int dtype, bool bwd, hipStream_t s);

struct GdrStepArgs {
  const void *q, *k, *v, *beta;
  const float* g;
  const int* slots;
  float* state;
  void* o;
  long long qs[3], ks[3], vs[3];
  int B, T, Hk, Hv, Dv, nslots;
  float scale;
};
int launch_gdr_step(const GdrStepArgs& a, int Dk, int dtype, hipStream_t s);

}  // namespace carve
