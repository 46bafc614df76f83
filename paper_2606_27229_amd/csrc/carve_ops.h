// carve_ops.h -- arguments and launches of the short causal convolution and the rotary
// positions, and the sequences of packed rows as both see them.
#pragma once
#include "../../include/carve.h"
#include "carve_dev.h"

namespace carve {

// Sequence n of packed rows: [first, end).  Offsets are device data, so they are clamped
// to the rows here, in the same way for every kernel: any values stay within the tensors.
__device__ __forceinline__ void packed_seq(const int* offsets, int n, int T, int& first, int& end) {
  first = min(max(offsets[n], 0), T);
  end = min(max(offsets[n + 1], first), T);
}
// the last sequence that starts at or before a row (the row may lie behind its end)
__device__ __forceinline__ int packed_find(const int* offsets, int nseq, int T, int row) {
  int lo = 0, hi = nseq - 1;
  while (lo < hi) {
    const int m = (lo + hi + 1) >> 1;
    if (min(max(offsets[m], 0), T) <= row) lo = m;
    else hi = m - 1;
  }
  return lo;
}

// The same for every lane of a wave at once, with the sequence's rows: up to 63 sequences
// come with one load, and each row (the same in runs of lw lanes) is counted by a ballot,
// where the search waits for memory at every step.  All lanes take part.
__device__ __forceinline__ void packed_find_wave(const int* offsets, int nseq, int T, int row, int lw, int& n, int& first, int& end) {
  if (nseq > 63) {
    n = packed_find(offsets, nseq, T, row);
    packed_seq(offsets, n, T, first, end);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int v = min(max(offsets[min(lane, nseq)], 0), T);
  n = 0;
  for (int r = 0; r < 64; r += lw) {
    const int at = __builtin_amdgcn_readlane(row, r);
    const int count = __popcll(__builtin_amdgcn_ballot_w64(lane < nseq && v <= at));
    if ((lane & ~(lw - 1)) == r) n = max(count - 1, 0);
  }
  first = __shfl(v, n);
  end = max(__shfl(v, n + 1), first);
}

struct ConvArgs {
  const void *x, *x0, *dy, *dx_T;
  const float *weight, *bias;
  const int* offsets;      // packed sequences: [nseq + 1]; dense: NULL
  void *y, *x_T, *dx, *dx0;
  float *dweight, *dbias, *partial;
  long long x_batch, x_token;
  int T, C, nseq, act;
};
struct ConvStepArgs {
  const void* x;
  const float *weight, *bias;
  const int* slots;
  void *state, *y;
  long long x_batch, x_token;
  int B, T, C, pool, act;
};
constexpr int kConvBwdRows = 24;   // rows of a thread in the backward (16384 x 2304: 62 us; 16 rows 69, 32 rows 75)
// rows of a workgroup of the backward, which leaves one row of partial sums for them
int conv_bwd_block_rows(int C, int dtype);
long long conv_parts(long long rows_of_a_batch, int batches, int C, int dtype);
int launch_short_conv_fwd(const ConvArgs& a, int W, int dtype, hipStream_t s);
int launch_short_conv_bwd(const ConvArgs& a, int W, int dtype, hipStream_t s, void (*mark)(hipStream_t));
int launch_short_conv_step(const ConvStepArgs& a, int W, int dtype, hipStream_t s);

struct RotaryArgs {
  const void *q, *k;
  const double* freq;
  const int *positions, *start, *offsets;
  void *qo, *ko;
  long long qs[3], ks[3], qos[3], kos[3];   // strides of batch, token, head
  int B, T, Hq, Hk, D, rot, nseq, interleaved;
  float amplitude, sign;
  bool copy;               // whether the part of the heads behind `rot` is copied
};
int launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s);

}  // namespace carve
