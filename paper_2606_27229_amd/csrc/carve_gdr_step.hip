// carve_gdr_step.hip -- the gated delta rule token by token, on states in a pool:
//   S <- e^g S;  u = beta (v - S k);  S <- S + u k^T;  o = scale S q
// in f32.  One pass over the state serves both products of a token, as the new
// state's read-out is that of the old one plus the write's:
//   S_new q = e^g (S q) + u (k.q),  S k before the write = e^g (S k).
//
// Bound by HBM: every state is read and written once a call, whatever T (64 states of
// 32 heads of 128 x 128 and their tokens, 270 MB: 56 us, 4.8 TB/s; 43 us on the states of the
// call before, which the last-level cache still holds).  One state of 16 heads takes 4.3 us,
// 8.3 with the call.  A token's rows are loaded when the token before it is done, so that
// several tokens wait for memory in turn (24 x 4 tokens of 8 f32 heads of 64: 6.3 us).  A row of
// S (Dk floats) is spread over Dk / 8 lanes, two 16-byte loads each, so that a wave
// load covers whole rows; a lane holds kStepRows rows, 8 loads in flight; a row's two
// sums run over its lanes by DPP.
#include "carve_gdr.h"

namespace carve {
namespace {

constexpr int kStepRows = 4;    // rows a lane holds a piece of
constexpr int kStepWaves = 4;

template <typename T>
__device__ __forceinline__ f32x4 ld4(const T* p) {
  return Quad<T>::f32(Quad<T>::ld(p));
}

template <typename T, int DK>
__global__ void __launch_bounds__(64 * kStepWaves) carve_gdr_step_kernel(GdrStepArgs a) {
  constexpr int LPR = DK / 8;            // lanes of a row
  constexpr int RPW = 64 / LPR;          // rows of a wave load
  constexpr int R = kStepRows;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = lane % LPR, r0 = ((int)blockIdx.x * kStepWaves + w) * RPW * R + lane / LPR;
  const int hv = blockIdx.y, b = blockIdx.z, hk = hv / (a.Hv / a.Hk);
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.nslots) return;   // (uniform) a padding row of the batch
  float* S = a.state + ((size_t)slot * a.Hv + hv) * a.Dv * DK + 4 * c;
  const T* q = reinterpret_cast<const T*>(a.q) + b * a.qs[0] + hk * a.qs[2] + 4 * c;
  const T* k = reinterpret_cast<const T*>(a.k) + b * a.ks[0] + hk * a.ks[2] + 4 * c;
  const T* v = reinterpret_cast<const T*>(a.v) + b * a.vs[0] + hv * a.vs[2];
  f32x4 s0[R], s1[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + i * RPW;
    s0[i] = s1[i] = zero4();
    if (r < a.Dv) {
      s0[i] = *reinterpret_cast<const f32x4*>(S + (size_t)r * DK);
      s1[i] = *reinterpret_cast<const f32x4*>(S + (size_t)r * DK + DK / 2);
    }
  }
  for (int t = 0; t < a.T; ++t) {
    const size_t row = ((size_t)b * a.T + t) * a.Hv + hv;
    const f32x4 k0 = ld4(k + t * a.ks[1]), k1 = ld4(k + t * a.ks[1] + DK / 2);
    const f32x4 q0 = ld4(q + t * a.qs[1]), q1 = ld4(q + t * a.qs[1] + DK / 2);
    const float al = expf(a.g[row]), be = (float)reinterpret_cast<const T*>(a.beta)[row];
    float vr[R];
#pragma unroll
    for (int i = 0; i < R; ++i) vr[i] = r0 + i * RPW < a.Dv ? (float)v[t * a.vs[1] + r0 + i * RPW] : 0.0f;
    float kq = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) kq += k0[e] * q0[e] + k1[e] * q1[e];
    kq = group_sum<LPR>(kq);
    float out = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float p = 0.0f, x = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p += s0[i][e] * k0[e] + s1[i][e] * k1[e];
        x += s0[i][e] * q0[e] + s1[i][e] * q1[e];
      }
      p = group_sum<LPR>(p);
      x = group_sum<LPR>(x);
      const float u = be * (vr[i] - al * p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s0[i][e] = al * s0[i][e] + u * k0[e];
        s1[i][e] = al * s1[i][e] + u * k1[e];
      }
      // row i's output from the row's lane i
      if (c == i) out = a.scale * (al * x + u * kq);
    }
    const int r = r0 + c * RPW;
    if (c < R && r < a.Dv) reinterpret_cast<T*>(a.o)[row * a.Dv + r] = (T)out;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + i * RPW;
    if (r < a.Dv) {
      *reinterpret_cast<f32x4*>(S + (size_t)r * DK) = s0[i];
      *reinterpret_cast<f32x4*>(S + (size_t)r * DK + DK / 2) = s1[i];
    }
  }
}

template <typename T, int DK>
int launch_t(const GdrStepArgs& a, hipStream_t s) {
  static_assert(DK / 8 >= kStepRows, "a row's lanes write its rows' outputs");
  const int rows = 64 / (DK / 8) * kStepRows * kStepWaves;
  hipLaunchKernelGGL((carve_gdr_step_kernel<T, DK>), dim3((a.Dv + rows - 1) / rows, a.Hv, a.B), dim3(64 * kStepWaves), 0,
                     s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T>
int launch_d(const GdrStepArgs& a, int Dk, hipStream_t s) {
  switch (Dk) {
    case 32: return launch_t<T, 32>(a, s);
    case 64: return launch_t<T, 64>(a, s);
    case 128: return launch_t<T, 128>(a, s);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}

}  // namespace

int launch_gdr_step(const GdrStepArgs& a, int Dk, int dtype, hipStream_t s) {
  return dtype == CARVE_BF16 ? launch_d<bf16_t>(a, Dk, s) : launch_d<float>(a, Dk, s);
}

}  // namespace carve
