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
// intermediates (S, T, R, U and their adjoints) enter as sums of bf16 values (Fi):
// three of them hold 24 bits, as f32 does; what only reaches bf16 results is taken
// as two (16 bits: what is left out is 2^-18 of a value, far below the rounding of
// the result).  Products of two such operands leave out the pairs of pieces that lie
// below the last piece.  One bf16 value would leave out 2^-9, which states and decay
// gradients (f32 outputs) do not bear; two left 4e-6 of a state and 1e-5 of dg.  With
// f32 tokens every product is an f32 matrix-core product.
#pragma once
#include "../../include/carve.h"
#include "carve_dev.h"

namespace carve {

constexpr int kGdrC = 64;                 // tokens of a chunk
constexpr int kGdrScal = 2048;            // bytes of a chunk's scalars ([5][64] floats, to whole KB)
constexpr float kGdrMinG = -1e4f;         // e^-1e4 is 0 in f32: a decay of -inf is taken as this

struct GdrArgs {
  const void *q, *k, *v, *beta, *dO;
  const float *g, *S0, *dS_T;
  const int* offsets;      // packed sequences: [nseq + 1]; dense: NULL
  void *o, *dq, *dk, *dv, *dbeta;
  float *S_T, *S_chunks, *dg, *dS0;
  char* ws;                // images and scalars of every (chunk slot, value head)
  float* dS_chunks;        // [nslots][Hv][Dv][Dk]: the state gradients at chunk ends (backward)
  float* dR;               // [nslots][Hv][Dv / 16][4][64][4]: dR as result tiles (backward)
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
// An f32 intermediate as an operand: N bf16 values whose sum it is, or f32.
template <typename T, int N>
struct Fi {
  Fr<T> x[sizeof(T) == 2 ? N : 1];
};
constexpr int kExact = 3, kNear = 2;   // pieces towards f32 and towards bf16 results

// x minus its bf16 rounding h, exactly: one two-term product a value, which also
// widens h (a shift or mask and a subtraction otherwise; the constants are the pairs
// (-1, 0) and (0, -1), set up here because as literals the assembler takes the pair's
// low half for an f32 constant)
__device__ __forceinline__ f32x4 bf16_rest(f32x4 x, bf16x4 h) {
  unsigned c0, c1;
  asm("s_mov_b32 %0, 0xbf80" : "=s"(c0));
  asm("s_mov_b32 %0, 0xbf800000" : "=s"(c1));
  const bf16x2 m0 = __builtin_bit_cast(bf16x2, c0), m1 = __builtin_bit_cast(bf16x2, c1);
  const bf16x2 lo = __builtin_shufflevector(h, h, 0, 1), hi = __builtin_shufflevector(h, h, 2, 3);
  const f32x4 r = {__builtin_amdgcn_fdot2_f32_bf16(lo, m0, x[0], false), __builtin_amdgcn_fdot2_f32_bf16(lo, m1, x[1], false),
                   __builtin_amdgcn_fdot2_f32_bf16(hi, m0, x[2], false), __builtin_amdgcn_fdot2_f32_bf16(hi, m1, x[3], false)};
  return r;
}
template <typename T, int N>
__device__ __forceinline__ Fi<T, N> to_fi(f32x4 a, f32x4 b) {
  Fi<T, N> f;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f.x[i].a = Quad<T>::cvt(a);
      f.x[i].b = Quad<T>::cvt(b);
      if (i + 1 < N) {
        a = bf16_rest(a, f.x[i].a);
        b = bf16_rest(b, f.x[i].b);
      }
    }
  } else {
    f.x[0].a = a;
    f.x[0].b = b;
  }
  return f;
}
// the first M pieces
template <int M, typename T, int N>
__device__ __forceinline__ Fi<T, M> first(const Fi<T, N>& f) {
  Fi<T, M> r;
  if constexpr (sizeof(T) == 2)
    for (int i = 0; i < M; ++i) r.x[i] = f.x[i];
  else r.x[0] = f.x[0];
  return r;
}
template <typename T>
__device__ __forceinline__ f32x4 mma(Fr<T> a, Fr<T> b, f32x4 c) {
  return Quad<T>::mma32(a.a, a.b, b.a, b.b, c);
}
// (small pieces first)
template <typename T, int N>
__device__ __forceinline__ f32x4 mma(const Fi<T, N>& a, Fr<T> b, f32x4 c) {
#pragma unroll
  for (int i = (sizeof(T) == 2 ? N : 1) - 1; i >= 0; --i) c = mma<T>(a.x[i], b, c);
  return c;
}
template <typename T, int N>
__device__ __forceinline__ f32x4 mma(Fr<T> a, const Fi<T, N>& b, f32x4 c) {
#pragma unroll
  for (int i = (sizeof(T) == 2 ? N : 1) - 1; i >= 0; --i) c = mma<T>(a, b.x[i], c);
  return c;
}
template <typename T, int N>
__device__ __forceinline__ f32x4 mma(const Fi<T, N>& a, const Fi<T, N>& b, f32x4 c) {
  constexpr int P = sizeof(T) == 2 ? N : 1;
#pragma unroll
  for (int s = P - 1; s >= 0; --s)
#pragma unroll
    for (int i = s; i >= 0; --i) c = mma<T>(a.x[i], b.x[s - i], c);
  return c;
}

template <typename T>
__device__ __forceinline__ void st_eight(T* p, f32x4 lo, f32x4 hi) {
  if constexpr (sizeof(T) == 2) {
    const bf16x4 a = Quad<T>::cvt(lo), b = Quad<T>::cvt(hi);
    *reinterpret_cast<bf16x8*>(p) = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    *reinterpret_cast<f32x4*>(p) = lo;
    *reinterpret_cast<f32x4*>(p + 4) = hi;
  }
}

// ---- triangular operand images ----------------------------------------------------------
// A 64 x 64 triangle as A operands of depth 32 over its columns: fragment (i, s)
// holds rows 16 i .. and columns 32 s .. + 31, lane (g, c) the columns 32 s + 4 g + e
// and 32 s + 16 + 4 g + e of row 16 i + c.  Lower: s <= i / 2; upper: s >= i / 2.
__host__ __device__ constexpr int img_lower(int i, int s) { return i < 2 ? i : 2 + 2 * (i - 2) + s; }
__host__ __device__ constexpr int img_upper(int i, int s) { return i < 2 ? 2 * i + s : i + 2; }
// bytes of an image of N pieces: planes of 1 KB a fragment, a piece each (bf16) or the
// two quads of a lane (f32)
template <typename T>
__host__ __device__ constexpr int img_planes(int N) { return sizeof(T) == 2 ? N : 2; }
template <typename T>
__host__ __device__ constexpr int img_bytes(int N) { return 6 * 1024 * img_planes<T>(N); }
template <typename T, int N>
__device__ __forceinline__ Fi<T, N> ld_img(const char* img, int f, int lane) {
  const char* p = img + f * 1024 * img_planes<T>(N) + lane * 16;
  Fi<T, N> x;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bf16x8 h = *reinterpret_cast<const bf16x8*>(p + 1024 * i);
      x.x[i].a = __builtin_shufflevector(h, h, 0, 1, 2, 3);
      x.x[i].b = __builtin_shufflevector(h, h, 4, 5, 6, 7);
    }
  } else {
    x.x[0].a = *reinterpret_cast<const f32x4*>(p);
    x.x[0].b = *reinterpret_cast<const f32x4*>(p + 1024);
  }
  return x;
}
template <typename T, int N>
__device__ __forceinline__ void st_img(char* img, int f, int lane, f32x4 a, f32x4 b) {
  char* p = img + f * 1024 * img_planes<T>(N) + lane * 16;
  const Fi<T, N> x = to_fi<T, N>(a, b);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      *reinterpret_cast<bf16x8*>(p + 1024 * i) = __builtin_shufflevector(x.x[i].a, x.x[i].b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    *reinterpret_cast<f32x4*>(p) = x.x[0].a;
    *reinterpret_cast<f32x4*>(p + 1024) = x.x[0].b;
  }
}
// one (slot, head) of the workspace.  Forward: T, scalars, P (towards o); backward: T,
// scalars, P^T, T^T
template <typename T>
struct GdrWs {
  static constexpr int I3 = img_bytes<T>(kExact), I2 = img_bytes<T>(kNear);
  static constexpr int fT = 0, fScal = I3, fP = I3 + kGdrScal, fBytes = fP + I2;
  static constexpr int bT = 0, bScal = I3, bPt = bScal + kGdrScal, bTt = bPt + I3, bBytes = bTt + I3;
};

// e^x of a decay (x <= 0): one hardware exp2.  The product's rounding moves e^x by
// |x| 2^-24 of itself, at most 0.4 * 2^-24 in all
__device__ __forceinline__ float decay_exp(float x) { return exp2_f(x * kLog2e); }

// scalars [5][64] of a chunk: e^G, e^{G_C - G}, beta, and G as a sum of two floats
enum : int { kScGam = 0, kScEnd = 1, kScBeta = 2, kScGh = 3, kScGl = 4 };

// Sums over the 16 lanes of a row of four values at once: lane c gets that of value
// c mod 4.  Neighbouring lanes swap the values the other one keeps, twice, and the four
// quads of the row are added up (11 operations; each value's butterfly on its own 16 to 24).
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum4(f32x4 v, int c) {
  const bool b0 = c & 1, b1 = c & 2;
  const float r0 = (b0 ? v[1] : v[0]) + dpp<0xB1>(b0 ? v[0] : v[1]);   // lane ^ 1
  const float r1 = (b0 ? v[3] : v[2]) + dpp<0xB1>(b0 ? v[2] : v[3]);
  float q = (b1 ? r1 : r0) + dpp<0x4E>(b1 ? r0 : r1);                  // lane ^ 2
  q += dpp<0x128>(q);                                                  // the row turned by 8 lanes
  return q + dpp<0x124>(q);                                            // and by 4
}

// lane coordinates the compiler takes as new: what is computed from them is computed
// where it is used, not ahead of a loop and kept
__device__ __forceinline__ void renew(int& g, int& c) { asm volatile("" : "+v"(g), "+v"(c)); }

// an LDS address as the direct loads take it (the low half of the generic address)
typedef __attribute__((address_space(3))) void* lds_ptr;
__device__ __forceinline__ lds_ptr lds_at(const char* p) { return (lds_ptr)(uintptr_t)(unsigned)(uintptr_t)p; }

// ---- token rows in LDS ------------------------------------------------------------------
// A [64][COLS] token tile loaded straight into LDS (16 bytes a lane, no registers):
// 16-byte piece x of row r sits at piece x ^ swz(r) of the row, so that both kinds of
// bf16 operand reads are free of bank conflicts: along a row (16 rows x 2 neighbouring
// quads at a time) and across rows (8 rows x 4 neighbouring quads).
template <typename T, int COLS>
struct GdrRows {
  static constexpr int RB = COLS * (int)sizeof(T);     // bytes of a row
  static constexpr int NCH = RB / 16;
  static constexpr int bytes = kGdrC * RB;
  static constexpr int PER = RB < 256 ? 256 / RB : 1;  // rows of a turn over the banks
  static constexpr int MASK = NCH / 2 - 1 < 7 ? NCH / 2 - 1 : 7;
  static_assert(NCH >= 4 && 1024 % RB == 0, "rows of 64 bytes to 1 KB");
  static __device__ __forceinline__ int swz(int r) { return (((r / PER) & MASK) * 2) ^ ((r >> 3) & 1); }

  // wave w of NW takes its share of the 1 KB pieces; rows behind the last of `len`
  // repeat it.  base: the first row; stride in bytes, below 2^24
  template <int NW>
  static __device__ __forceinline__ void dma(char* lds, const T* base, int stride, int len, int w, int lane) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<void*>(reinterpret_cast<const void*>(base)), 0, (len - 1) * stride + RB, 0x00027000);
    constexpr int RPI = 1024 / RB;   // rows of a piece
#pragma unroll
    for (int u = 0; u < (bytes / 1024 + NW - 1) / NW; ++u) {
      const int i = w + NW * u;
      if ((bytes / 1024) % NW != 0 && i >= bytes / 1024) break;   // (uniform)
      const int row = i * RPI + lane / NCH, x = (lane % NCH) ^ swz(row);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_at(lds + 1024 * i), 16,
                                               (int)__umul24(min(row, len - 1), stride) + 16 * x, 0, 0, 0);
    }
  }
  // lane (g, c): row 16 i + c, columns 32 p + 4 g + e and 32 p + 16 + 4 g + e
  static __device__ __forceinline__ Fr<T> nat(const char* lds, int i, int p, int g, int c) {
    Fr<T> f;
    if constexpr (sizeof(T) == 2) {
      const int o = (((4 * p + (g >> 1)) ^ swz(c)) << 4) + ((g & 1) << 3);
      f.a = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * RB + o));
      f.b = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * RB + (o ^ 32)));
    } else {
      f.a = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * RB + (((8 * p + g) ^ swz(c)) << 4)));
      f.b = Quad<T>::ld(reinterpret_cast<const T*>(lds + (16 * i + c) * RB + (((8 * p + 4 + g) ^ swz(c)) << 4)));
    }
    return f;
  }
  // lane (g, c): column 16 j + c, rows r0 + 4 g + e (r0 a multiple of 16)
  static __device__ __forceinline__ typename Quad<T>::q tr(const char* lds, int r0, int j, int g, int c) {
    if constexpr (sizeof(T) == 2) {
      const int r = 4 * g + (c >> 2);
      const int o = (((2 * j + ((c >> 1) & 1)) ^ swz(r)) << 4) + ((c & 1) << 3);
      return Quad<T>::ld_tr_at(reinterpret_cast<const T*>(lds + (r0 + r) * RB + o));
    } else {
      typename Quad<T>::q o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = r0 + 4 * g + e;
        o[e] = *reinterpret_cast<const T*>(lds + r * RB + (((4 * j + (c >> 2)) ^ swz(r)) << 4) + ((c & 3) << 2));
      }
      return o;
    }
  }
  // both for the 32 tokens from 32 s
  static __device__ __forceinline__ Fr<T> tr32(const char* lds, int s, int j, int g, int c) {
    Fr<T> f;
    f.a = tr(lds, 32 * s, j, g, c);
    f.b = tr(lds, 32 * s + 16, j, g, c);
    return f;
  }
};
// KB * 1024 bytes of global memory as they are, wave w of NW its share
template <int NW, int KB>
__device__ __forceinline__ void dma_flat(char* lds, const char* src, int w, int lane) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), 0, 1024 * KB, 0x00027000);
#pragma unroll
  for (int u = 0; u < (KB + NW - 1) / NW; ++u) {
    const int i = w + NW * u;
    if (KB % NW != 0 && i >= KB) break;   // (uniform)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_at(lds + 1024 * i), 16, 16 * lane, 1024 * i, 0, 0);
  }
}

// ---- two waves of a workgroup meeting ---------------------------------------------------
// Wave `me` (0 or 1) tells the other that its LDS writes so far are done and waits for the
// same word of it.  A wave's LDS accesses are carried out in order, so the flag (the
// `turn`-th meeting, counted from 1) follows the data.  Both waves belong to one workgroup
// and meet equally often, so the wait ends; it costs the other waves nothing, where a
// barrier would hold them to these two waves' pace.
typedef volatile __attribute__((address_space(3))) int lds_flag;
__device__ __forceinline__ void pair_meet(lds_flag* flags, int me, int turn) {
  asm volatile("" ::: "memory");
  flags[me] = turn;
  while (__builtin_amdgcn_readfirstlane(flags[1 - me]) < turn) {
  }
  asm volatile("" ::: "memory");
}

// ---- workgroups of the chains ---------------------------------------------------------
// Workgroup -> (sequence, value head) and value slice (of ns).  Blocks 8 apart share an
// XCD, which takes all slices of a head one after another: they read the same rows from
// one L2.  Packed sequences come longest first: a call takes as long as its last chain,
// and one that is long and starts late waits for a compute unit first.  Every wave ranks
// the sequences' chunk counts for itself, a sequence a lane; beyond 64 sequences they come
// as they are.
__host__ __device__ inline unsigned gdr_chain_grid(unsigned heads, int ns) { return (heads + 7) / 8 * 8 * ns; }
__device__ __forceinline__ bool gdr_chain_block(const GdrArgs& a, int ns, int& n, int& hv, int& slice) {
  const int at = blockIdx.x / 8, head = at / ns * 8 + (int)(blockIdx.x % 8);
  n = head / a.Hv;
  hv = head % a.Hv;
  slice = at % ns;
  if (n >= a.nseq) return false;
  if (a.offsets && a.nseq > 1 && a.nseq <= 64) {
    const int lane = threadIdx.x & 63;
    const int len = lane < a.nseq ? (gdr_seq(a, lane).len + kGdrC - 1) / kGdrC : -1;
    int rank = 0;
    for (int i = 0; i < a.nseq; ++i) {
      const int other = __builtin_amdgcn_readlane(len, i);
      rank += other > len || (other == len && i < lane);
    }
    // (the lanes without a sequence rank behind all that have one)
    n = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == n));
  }
  return true;
}

// launches (carve_gdr_*.hip); mark: called after every launch
int launch_gdr_fwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_gdr_bwd(const GdrArgs& a, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_gdr_prep(const GdrArgs& a, int dtype, bool bwd, hipStream_t s);
// Whether a call has no more value tiles than the card compute units (256): then a tile a
// workgroup runs a chunk faster than two, and beyond it they wait for each other (forward,
// one / two, us: 128 tiles of 4096 tokens 146 / 153, 256 149 / 154, in f32 with 1024 tokens
// 69 / 87; 320 tiles 271 / 166).
inline bool gdr_few_tiles(const GdrArgs& a) { return (long long)a.nseq * a.Hv * (a.Dv / 16) <= 256; }
// Whether a call of the backward's chain has more value tiles than workgroups of two can
// run at once (512): then four tiles a workgroup, one chain wave each, give more per compute
// unit; below it two chain waves a tile run a chunk faster.  Both sides (us, pairs / four;
// 128 values, bf16): 512 tiles of 4 x 2048 tokens 149 / 189; 640 of 5 x 1024 116 / 93; 1024
// of 8 x 1024 147 / 115, with keys of 64 105 / 83.  Packed sequences differ in length, so
// that the call waits for the longest ones' chains far beyond that: 5 documents, 640 tiles,
// 321 / 465, keys of 64 251 / 317; 11 documents, 1408 tiles 137 / 177, 2816 tiles 121 / 134;
// 40 documents, 5120 tiles 198 / 149.
inline bool gdr_many_tiles(const GdrArgs& a) {
  return a.Dv % 64 == 0 && (long long)a.nseq * a.Hv * (a.Dv / 16) > (a.offsets ? 4096 : 512);
}

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
