// carve_rotary.hip -- rotary positions of queries and keys: the pairs of values of a head's
// first `rot` are turned by the angle position * freq_i,
//   (a, b) -> m (a cos - b sin, b cos + a sin),
// pairs being values i and i + rot / 2 ("half") or 2 i and 2 i + 1 ("interleaved"); what
// lies behind `rot` is kept.  m: an amplitude.  Turned the other way (sign -1) it is the
// backward: the transposed map.
//
// Angles are formed and brought to one turn in 64 bits: position * freq reaches 10^6, of
// which f32 keeps a sixteenth; sines and cosines, of less than half a turn, are f32.
// Bound by HBM: every value is read and written once (and by the call for few tokens: 4 us of
// the kernel, 9 to 10 with the call).  A thread makes the sines of one row's 8 (bf16) or 4
// (f32) pairs once and turns those pairs of two heads, of the queries and the keys alike;
// 16-byte accesses.
#include "carve_ops.h"

namespace carve {
namespace {

constexpr int kThreads = 256;
// Heads of a thread.  The sines are about 300 operations, but threads that load more than two
// heads' pairs one after another keep fewer loads under way than the memory has room for:
// 4 x 4096 tokens of 16 + 16 bf16 heads of 128 (268 MB) take 48 us with 2 heads (5.5 TB/s),
// 59 with 1, 53 with 3, 55 with 4 and 59 with 8; 8191 rows of 16 + 4 f32 heads 28 us with 2,
// 29 with 1 or 4; one token a sequence the same with any.
constexpr int kHeads = 2;

template <typename T>
__global__ void __launch_bounds__(kThreads) carve_rotary_kernel(RotaryArgs a, int chunks, int turns, int groups) {
  constexpr int V = Chunk16<T>::N;
  const long long b64 = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  // thread -> (row, group of heads, piece of a head), pieces next to each other
  const long long id0 = b64 * kThreads;
  const int per = chunks * groups;   // threads of a row
  const long long base = id0 / per;
  const int off = (int)(id0 - base * per) + (int)threadIdx.x;
  const long long row = base + off / per;
  const int in_row = off % per, group = in_row / chunks, piece = in_row % chunks;
  if (row >= (long long)a.B * a.T) return;
  const int batch = (int)(row / a.T), t = (int)(row % a.T);
  long long pos = 0;   // (a start and a row together may pass 32 bits)
  if (a.positions) {
    pos = a.positions[row];
  } else if (a.offsets) {
    const int n = packed_find(a.offsets, a.nseq, a.T, t);
    int first, end;
    packed_seq(a.offsets, n, a.T, first, end);
    if (t < first || t >= end) return;   // a row of no sequence
    pos = (long long)(t - first) + (a.start ? a.start[n] : 0);
  } else {
    pos = (long long)t + (a.start ? a.start[batch] : 0);
  }
  const bool turn = piece < turns;
  // first values of the thread's two 16-byte pieces
  int v0, v1;
  bool second = true;
  if (turn) {
    v0 = a.interleaved ? 2 * V * piece : V * piece;
    v1 = a.interleaved ? v0 + V : v0 + a.rot / 2;
  } else {
    v0 = a.rot + 2 * V * (piece - turns);
    v1 = v0 + V;
    second = v1 < a.D;
  }
  float cs[V], sn[V];
  if (turn) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const double turns64 = (double)pos * a.freq[V * piece + i] * 0.15915494309189533577;   // 1 / (2 pi)
      const float r = (float)(turns64 - rint(turns64));
      float s, c;
      sincospif(2.0f * r, &s, &c);
      cs[i] = a.amplitude * c;
      sn[i] = a.sign * a.amplitude * s;
    }
  }
  const auto one = [&](const T* in, T* out) {
    u32x4_t x0 = *reinterpret_cast<const u32x4_t*>(in + v0), x1 = {};
    if (second) x1 = *reinterpret_cast<const u32x4_t*>(in + v1);
    if (turn) {
      float f0[V], f1[V];
      Chunk16<T>::unpack(x0, f0);
      Chunk16<T>::unpack(x1, f1);
      if (a.interleaved) {
        float g0[V], g1[V];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          g0[2 * i] = f0[2 * i] * cs[i] - f0[2 * i + 1] * sn[i];
          g0[2 * i + 1] = f0[2 * i + 1] * cs[i] + f0[2 * i] * sn[i];
          g1[2 * i] = f1[2 * i] * cs[V / 2 + i] - f1[2 * i + 1] * sn[V / 2 + i];
          g1[2 * i + 1] = f1[2 * i + 1] * cs[V / 2 + i] + f1[2 * i] * sn[V / 2 + i];
        }
        x0 = Chunk16<T>::pack(g0);
        x1 = Chunk16<T>::pack(g1);
      } else {
        float g0[V], g1[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          g0[i] = f0[i] * cs[i] - f1[i] * sn[i];
          g1[i] = f1[i] * cs[i] + f0[i] * sn[i];
        }
        x0 = Chunk16<T>::pack(g0);
        x1 = Chunk16<T>::pack(g1);
      }
    }
    *reinterpret_cast<u32x4_t*>(out + v0) = x0;
    if (second) *reinterpret_cast<u32x4_t*>(out + v1) = x1;
  };
  const T* q = reinterpret_cast<const T*>(a.q) + batch * a.qs[0] + t * a.qs[1];
  const T* k = reinterpret_cast<const T*>(a.k) + batch * a.ks[0] + t * a.ks[1];
  T* qo = reinterpret_cast<T*>(a.qo) + batch * a.qos[0] + t * a.qos[1];
  T* ko = reinterpret_cast<T*>(a.ko) + batch * a.kos[0] + t * a.kos[1];
  // heads, the keys' behind the queries'
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = group * kHeads + i;
    if (h < a.Hq) one(q + h * a.qs[2], qo + h * a.qos[2]);
    else if (h < a.Hq + a.Hk) one(k + (h - a.Hq) * a.ks[2], ko + (h - a.Hq) * a.kos[2]);
  }
}

template <typename T>
int launch_t(const RotaryArgs& a, hipStream_t s) {
  constexpr int V = Chunk16<T>::N;
  const int turns = a.rot / 2 / V, chunks = turns + (a.copy ? ((a.D - a.rot) / V + 1) / 2 : 0);
  const int groups = (a.Hq + a.Hk + kHeads - 1) / kHeads;
  const long long threads = (long long)a.B * a.T * chunks * groups, blocks = (threads + kThreads - 1) / kThreads;
  const long long gx = blocks < (1 << 20) ? blocks : 1 << 20, gy = (blocks + gx - 1) / gx;
  if (gy > 65535) return CARVE_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(carve_rotary_kernel<T>, dim3((unsigned)gx, (unsigned)gy), dim3(kThreads), 0, s, a, chunks, turns, groups);
  return hipGetLastError() == hipSuccess ? CARVE_OK : CARVE_ERR_HIP;
}
}  // namespace

int launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  return dtype == CARVE_BF16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace carve
