// carve_ssm_step.hip -- the selective state space scan token by token, on states in a pool:
//   S <- e^{d A} S + d x B^T;  y = S C + D x
// in f32.  Bound by HBM: every state is read and written once a call, whatever T.  A row of
// S (N floats) is spread over N / 8 lanes, two 16-byte loads each, so that a wave load
// covers whole rows; a lane holds kRows rows, 8 loads in flight; a row's sum runs over its
// lanes by DPP.  One token for each of 64 sequences of 32 heads of 64 x 128 (135 MB): 24 us,
// 5.7 TB/s, part of the states in the last-level cache.  Small states wait longer for what they
// move: 64 x 64 (68 MB) 14 us, 64 x 32 (34 MB) 11, 32 x 32 (17 MB) 9, with rows for one of a
// workgroup's four waves.
#include "carve_ssm.h"

namespace carve {
namespace {

constexpr int kRows = 4;    // rows a lane holds a piece of
constexpr int kWaves = 4;

template <typename T>
__device__ __forceinline__ f32x4 ld4(const T* p) {
  return Quad<T>::f32(Quad<T>::ld(p));
}

template <typename T, int N>
__global__ void __launch_bounds__(64 * kWaves) carve_ssm_step_kernel(SsmStepArgs a) {
  constexpr int LPR = N / 8;             // lanes of a row
  constexpr int RPW = 64 / LPR;          // rows of a wave load
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = lane % LPR, r0 = ((int)blockIdx.x * kWaves + w) * RPW * kRows + lane / LPR;
  const int h = blockIdx.y, b = blockIdx.z, grp = h / (a.H / a.G);
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.pool) return;   // (uniform) a padding row of the batch
  float* S = a.state + ((size_t)slot * a.H + h) * a.P * N + 4 * c;
  const T* x = reinterpret_cast<const T*>(a.x) + b * a.xs[0] + h * a.xs[2];
  const T* Bm = reinterpret_cast<const T*>(a.Bm) + b * a.bs[0] + grp * a.bs[2] + 4 * c;
  const T* Cm = reinterpret_cast<const T*>(a.Cm) + b * a.cs[0] + grp * a.cs[2] + 4 * c;
  const T* dt = reinterpret_cast<const T*>(a.dt) + b * a.ds[0] + h;
  f32x4 s0[kRows], s1[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + i * RPW;
    s0[i] = s1[i] = zero4();
    if (r < a.P) {
      s0[i] = *reinterpret_cast<const f32x4*>(S + (size_t)r * N);
      s1[i] = *reinterpret_cast<const f32x4*>(S + (size_t)r * N + N / 2);
    }
  }
  const float A = a.A[h], bias = a.dt_bias ? a.dt_bias[h] : 0.0f, D = a.D ? a.D[h] : 0.0f;
  for (int t = 0; t < a.T; ++t) {
    const f32x4 b0 = ld4(Bm + t * a.bs[1]), b1 = ld4(Bm + t * a.bs[1] + N / 2);
    const f32x4 c0 = ld4(Cm + t * a.cs[1]), c1 = ld4(Cm + t * a.cs[1] + N / 2);
    float xr[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) xr[i] = r0 + i * RPW < a.P ? (float)x[t * a.xs[1] + r0 + i * RPW] : 0.0f;
    const float d = ssm_step_of((float)dt[t * a.ds[1]] + bias, a.softplus), al = expf(d * A);
    float out = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float u = d * xr[i];
      float p = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s0[i][e] = al * s0[i][e] + u * b0[e];
        s1[i][e] = al * s1[i][e] + u * b1[e];
        p += s0[i][e] * c0[e] + s1[i][e] * c1[e];
      }
      p = group_sum<LPR>(p) + D * xr[i];
      if (c == i) out = p;   // row i's output from the row's lane i
    }
    const int r = r0 + c * RPW;
    if (c < kRows && r < a.P) reinterpret_cast<T*>(a.y)[(((size_t)b * a.T + t) * a.H + h) * a.P + r] = (T)out;
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + i * RPW;
    if (r < a.P) {
      *reinterpret_cast<f32x4*>(S + (size_t)r * N) = s0[i];
      *reinterpret_cast<f32x4*>(S + (size_t)r * N + N / 2) = s1[i];
    }
  }
}

template <typename T, int N>
int launch_t(const SsmStepArgs& a, hipStream_t s) {
  static_assert(N / 8 >= kRows, "a row's lanes write its rows' outputs");
  const int rows = 64 / (N / 8) * kRows * kWaves;
  hipLaunchKernelGGL((carve_ssm_step_kernel<T, N>), dim3((a.P + rows - 1) / rows, a.H, a.B), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
template <typename T>
int launch_n(const SsmStepArgs& a, int N, hipStream_t s) {
  switch (N) {
    case 32: return launch_t<T, 32>(a, s);
    case 64: return launch_t<T, 64>(a, s);
    case 128: return launch_t<T, 128>(a, s);
    default: return CARVE_ERR_UNSUPPORTED;
  }
}

}  // namespace

int launch_ssm_step(const SsmStepArgs& a, int N, int dtype, hipStream_t s) {
  return dtype == CARVE_BF16 ? launch_n<bf16_t>(a, N, s) : launch_n<float>(a, N, s);
}

}  // namespace carve
