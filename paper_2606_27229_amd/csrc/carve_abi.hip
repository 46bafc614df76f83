// carve_abi.hip -- the C ABI of libcarve: argument validation, workspace
// sizing, kernel selection and launch.  No allocation, no synchronisation.
#include <stdint.h>

#include <utility>

#include "carve_gdr.h"
#include "carve_kernels.h"
#include "carve_ssm.h"

using namespace carve;

namespace {

constexpr size_t kMaxLds = 160 * 1024;

int round_rp(int R) { return (R + 31) / 32 * 32; }

size_t esize(carve_dtype_t dt) { return dt == CARVE_BF16 ? 2 : 4; }

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// 16-token tiles of the backward's WY blocks (1, 2 or 4, dividing the chunk):
// the largest whose LDS layout fits
int pick_nb(const carve_dims_t* d) {
  const int RP = round_rp(d->R);
  for (int nb = 4; nb >= 1; nb /= 2) {
    if (16 * nb > d->L || d->L % (16 * nb)) continue;
    if (bwd_lds_bytes(d->dtype, d->Dk, nb, RP) <= kMaxLds) return nb;
  }
  return 0;
}

// backward workspace: d[Ub; Uw] partials per (b,h, chunk split) | dVb, dVw
// partials per (b,h, token split) | chunk records of the recompute | ready
// flags, ticket counter and adjoint positions of the fused recompute + adjoint
// launch | dA, dtau partials | the adjoints' parameter operands
struct BwdWs {
  size_t part, partV, rec, sync, partG, opnd, total;
};

BwdWs bwd_workspace_layout(const carve_dims_t* d) {
  BwdWs l{};
  const size_t nbh = (size_t)d->B * d->H;
  const size_t nch = (size_t)(d->T / d->L);
  size_t off = 0;
  const size_t npart = nbh * param_splits(d->B * d->H);
  l.part = off;  off += align256(npart * part_floats(d->R, d->Dk) * 4);
  l.partV = off; off += align256(npart * part_floats(d->R, d->Dk) * 4);
  // records of the full layer (2RP fold rows); the scalar-write records are smaller
  l.rec = off;   off += align256(nbh * nch * chunk_rec_bytes(d->dtype, d->Dk, d->L, 2 * round_rp(d->R), pick_nb(d)));
  l.sync = off;  off += align256(sync_ints(nbh, nch) * sizeof(int));
  l.partG = off; off += align256(nbh * 2 * (size_t)d->Dk * 4);   // dA, dtau partials (gated)
  l.opnd = off;  off += align256(nbh * adj_opnd_bytes(d->Dk, 2 * round_rp(d->R), esize(d->dtype)));
  l.total = off;
  return l;
}

int check_dims(const carve_dims_t* d) {
  if (!d) return CARVE_ERR_NULL;
  if (d->B <= 0 || d->T <= 0 || d->H <= 0 || d->Dk <= 0 || d->Dv <= 0 || d->R <= 0 || d->L <= 0)
    return CARVE_ERR_SHAPE;
  if (d->dtype != CARVE_F32 && d->dtype != CARVE_BF16) return CARVE_ERR_UNSUPPORTED;
  if (d->T % d->L != 0) return CARVE_ERR_SHAPE;
  if (d->Dk != d->Dv) return CARVE_ERR_UNSUPPORTED;
  if (d->Dk != 32 && d->Dk != 64 && d->Dk != 128) return CARVE_ERR_UNSUPPORTED;
  if (d->R > 64) return CARVE_ERR_UNSUPPORTED;
  if (d->L != 16 && d->L != 32 && d->L != 64 && d->L != 128) return CARVE_ERR_UNSUPPORTED;
  // the grid is B*H workgroups; inside one (batch, head) the kernels address
  // token tensors with 32-bit offsets
  if ((long long)d->B * d->H > (1LL << 30)) return CARVE_ERR_UNSUPPORTED;
  if ((long long)d->T * d->H * (d->Dk > d->Dv ? d->Dk : d->Dv) >= (1LL << 31)) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}

// compute units of the current device (the fused backward sizes its grid by it)
int device_cus(int* cus) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return CARVE_ERR_HIP;
  if (hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return CARVE_ERR_HIP;
  if (*cus < 1) *cus = 1;
  return CARVE_OK;
}

// largest WY block (<= 64 tokens, dividing L) whose chain-forward LDS layout fits
int pick_wb(const carve_dims_t* d) {
  const int RP = round_rp(d->R);
  for (int wb = 64; wb >= 16; wb /= 2) {
    if (wb > d->L || d->L % wb) continue;
    if (chain_lds_bytes(d->dtype, d->Dk, wb, RP) <= kMaxLds) return wb;
  }
  return 0;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// launch-boundary events of the next call on this thread (carve_profile_events);
// the handles are copied when the hook is armed
constexpr int kMaxProfEvents = 16;
thread_local hipEvent_t g_prof_events[kMaxProfEvents];
thread_local int g_prof_capacity = 0;
thread_local int g_prof_count = 0;

void prof_mark(hipStream_t stream) {
  if (g_prof_count < g_prof_capacity) hipEventRecord(g_prof_events[g_prof_count++], stream);
}

// the hook covers exactly one call: it is cleared when that call returns,
// whatever its status
struct ProfClear {
  ~ProfClear() { g_prof_capacity = 0; }
};

// bound of the backward's wait for a chunk record, for the calls made on this
// thread (carve_set_ready_wait_limit)
thread_local int g_wait_limit = kReadySpinLimit;

struct Range {
  const void* p;
  size_t bytes;
};

bool overlap(const Range& a, const Range& b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, a1 = a0 + a.bytes, b0 = (uintptr_t)b.p, b1 = b0 + b.bytes;
  return a0 < b1 && b0 < a1;
}

bool any_overlap(const Range* outs, int nout, const Range* ins, int nin) {
  for (int i = 0; i < nout; ++i) {
    for (int j = 0; j < nin; ++j)
      if (overlap(outs[i], ins[j])) return true;
    for (int j = i + 1; j < nout; ++j)
      if (overlap(outs[i], outs[j])) return true;
  }
  return false;
}

}  // namespace

extern "C" {

const char* carve_status_string(int status) {
  switch (status) {
    case CARVE_OK: return "ok";
    case CARVE_ERR_NULL: return "a required pointer is NULL";
    case CARVE_ERR_SHAPE: return "invalid shape (non-positive size or T not a multiple of L)";
    case CARVE_ERR_UNSUPPORTED: return "unsupported configuration (dtype, head size, rank or chunk length)";
    case CARVE_ERR_ALIGN: return "a pointer is not 16-byte aligned";
    case CARVE_ERR_WORKSPACE: return "workspace missing or too small";
    case CARVE_ERR_HIP: return "HIP runtime error";
    case CARVE_ERR_ARG: return "conflicting or invalid argument values (both of two alternative inputs given, or eps)";
    default: return "unknown status";
  }
}

int carve_profile_events(hipEvent_t* events, int capacity) {
  g_prof_capacity = 0;
  if (capacity < 0 || (capacity > 0 && !events)) return CARVE_ERR_NULL;
  if (capacity > kMaxProfEvents) return CARVE_ERR_UNSUPPORTED;
  for (int i = 0; i < capacity; ++i) g_prof_events[i] = events[i];
  g_prof_capacity = capacity;
  g_prof_count = 0;
  return CARVE_OK;
}

int carve_set_ready_wait_limit(int polls) {
  const int prev = g_wait_limit;
  g_wait_limit = polls < 0 ? kReadySpinLimit : polls;
  return prev;
}

int carve_bwd_wait_status(const carve_dims_t* d, const void* workspace, hipStream_t stream, int* timed_out) {
  if (!d || !workspace || !timed_out) return CARVE_ERR_NULL;
  int st = check_dims(d);
  if (st) return st;
  if (!pick_nb(d)) return CARVE_ERR_UNSUPPORTED;
  const BwdWs wl = bwd_workspace_layout(d);
  const int* word = reinterpret_cast<const int*>(reinterpret_cast<const char*>(workspace) + wl.sync) +
                    sync_timeout_word((size_t)d->B * d->H, (size_t)(d->T / d->L));
  int h = 0;
  if (hipMemcpyAsync(&h, word, sizeof(int), hipMemcpyDeviceToHost, stream) != hipSuccess) return CARVE_ERR_HIP;
  if (hipStreamSynchronize(stream) != hipSuccess) return CARVE_ERR_HIP;
  *timed_out = h != 0 ? 1 : 0;
  return CARVE_OK;
}

size_t carve_workspace_size(const carve_dims_t* d, int for_backward) {
  if (check_dims(d) != CARVE_OK) return 0;
  if (!for_backward) return 0;
  if (!pick_nb(d)) return 0;
  return bwd_workspace_layout(d).total;
}

}  // extern "C"

namespace {

// the decay input: g itself, or its raw logit f with A, tau_f (Eq. decay_gate)
struct Decay {
  const float* g;
  const void* f;
  const float *A, *tau_f;
  bool gated() const { return f != nullptr; }
};

// kernel variant of a call
int variant_of(const Decay& dc, bool sw, bool act) {
  return (dc.gated() ? kVarGated : 0) | (sw ? kVarScalarW : 0) | (act ? kVarAct : 0);
}

// sw: the scalar write gate (wx [B,T,H], no Uw, Vw); act: q, k, v are the raw
// projections (the kernels apply the input activations)
int fwd_impl(const carve_dims_t* d, const void* q, const void* k, const void* v, const void* beta,
             const Decay& dc, const void* bx, const void* wx, const float* Ub, const float* Uw,
             const float* Vb, const float* Vw, const float* S0, void* o, float* S_T, float* S_chunks,
             bool sw, bool act, hipStream_t stream) {
  ProfClear pc;
  int st = check_dims(d);
  if (st) return st;
  if (!q || !k || !v || !beta || !bx || !wx || !Ub || !Vb || !o) return CARVE_ERR_NULL;
  if (!sw && (!Uw || !Vw)) return CARVE_ERR_NULL;
  if (dc.gated() ? (!dc.A || !dc.tau_f) : !dc.g) return CARVE_ERR_NULL;
  const void* ptrs[] = {q, k, v, beta, dc.g, dc.f, dc.A, dc.tau_f, bx, wx, Ub, Uw, Vb, Vw, S0, o, S_T, S_chunks};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t es = esize(d->dtype);
  const size_t ntok = (size_t)d->B * d->T * d->H;
  const size_t nst = (size_t)d->B * d->H * d->Dv * d->Dk;
  const size_t HD = (size_t)d->H * d->Dk * 4;
  const Range ins[] = {{q, ntok * d->Dk * es}, {k, ntok * d->Dk * es}, {v, ntok * d->Dv * es},
                       {beta, ntok * es}, {dc.g, ntok * d->Dk * 4}, {dc.f, ntok * d->Dk * es},
                       {dc.A, HD}, {dc.tau_f, HD}, {bx, ntok * d->Dk * es},
                       {wx, ntok * (sw ? 1 : d->Dv) * es}, {Ub, (size_t)d->R * d->Dv * 4},
                       {Uw, (size_t)d->R * d->Dv * 4}, {Vb, (size_t)d->Dk * d->R * 4},
                       {Vw, (size_t)d->Dv * d->R * 4}, {S0, nst * 4}};
  const Range outs[] = {{o, ntok * d->Dv * es}, {S_T, nst * 4}, {S_chunks, nst * (d->T / d->L) * 4}};
  if (any_overlap(outs, 3, ins, 15)) return CARVE_ERR_UNSUPPORTED;
  const int wb = pick_wb(d);
  if (!wb) return CARVE_ERR_UNSUPPORTED;
  FwdArgs a;
  a.q = q; a.k = k; a.v = v; a.beta = beta; a.bx = bx; a.wx = wx;
  a.g = dc.g; a.Ub = Ub; a.Uw = Uw; a.Vb = Vb; a.Vw = Vw; a.S0 = S0;
  a.f = dc.f; a.A = dc.A; a.tau_f = dc.tau_f;
  a.o = o; a.S_T = S_T; a.S_chunks = S_chunks;
  a.B = d->B; a.T = d->T; a.H = d->H; a.R = d->R; a.RP = round_rp(d->R); a.L = d->L;
  a.rec = nullptr;
  prof_mark(stream);
  st = launch_chain_fwd(a, d->dtype, d->Dk, wb, variant_of(dc, sw, act), stream);
  prof_mark(stream);
  return st;
}

// decay gradient: dg, or df with dA, dtau (gated)
struct DecayGrad {
  float* dg;
  void* df;
  float *dA, *dtau;
};

int bwd_impl(const carve_dims_t* d, const void* q, const void* k, const void* v, const void* beta,
             const Decay& dc, const void* bx, const void* wx, const float* Ub, const float* Uw,
             const float* Vb, const float* Vw, const float* S_chunks, const void* dO, const float* dS_T,
             void* dq, void* dk, void* dv, void* dbeta, const DecayGrad& dd, void* dbx, void* dwx,
             float* dUb, float* dUw, float* dVb, float* dVw, float* dS0, void* workspace,
             size_t workspace_bytes, bool sw, bool act, hipStream_t stream) {
  ProfClear pc;
  int st = check_dims(d);
  if (st) return st;
  if (!q || !k || !v || !beta || !bx || !wx || !Ub || !Vb || !S_chunks || !dO ||
      !dq || !dk || !dv || !dbeta || !dbx || !dwx || !dUb || !dVb)
    return CARVE_ERR_NULL;
  if (!sw && (!Uw || !Vw || !dUw || !dVw)) return CARVE_ERR_NULL;
  if (dc.gated() ? (!dc.A || !dc.tau_f || !dd.df || !dd.dA || !dd.dtau) : (!dc.g || !dd.dg)) return CARVE_ERR_NULL;
  const void* ptrs[] = {q, k, v, beta, dc.g, dc.f, dc.A, dc.tau_f, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO, dS_T,
                        dq, dk, dv, dbeta, dd.dg, dd.df, dd.dA, dd.dtau, dbx, dwx, dUb, dUw, dVb, dVw, dS0,
                        workspace};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_workspace_size(d, 1);
  if (need && (!workspace || workspace_bytes < need)) return CARVE_ERR_WORKSPACE;
  const size_t es = esize(d->dtype);
  const size_t ntok = (size_t)d->B * d->T * d->H;
  const size_t nst = (size_t)d->B * d->H * d->Dv * d->Dk;
  const size_t RDv = (size_t)d->R * d->Dv * 4;
  const size_t HD = (size_t)d->H * d->Dk * 4;
  const size_t nwx = ntok * (sw ? 1 : d->Dv) * es;   // bytes of wx and of dwx
  const Range ins[] = {{q, ntok * d->Dk * es}, {k, ntok * d->Dk * es}, {v, ntok * d->Dv * es},
                       {beta, ntok * es}, {dc.g, ntok * d->Dk * 4}, {dc.f, ntok * d->Dk * es},
                       {dc.A, HD}, {dc.tau_f, HD}, {bx, ntok * d->Dk * es},
                       {wx, nwx}, {Ub, RDv}, {Uw, RDv}, {Vb, RDv}, {Vw, RDv},
                       {S_chunks, nst * (d->T / d->L) * 4}, {dO, ntok * d->Dv * es},
                       {dS_T, nst * 4}, {workspace, need}};
  const Range outs[] = {{dq, ntok * d->Dk * es}, {dk, ntok * d->Dk * es}, {dv, ntok * d->Dv * es},
                        {dbeta, ntok * es}, {dd.dg, ntok * d->Dk * 4}, {dd.df, ntok * d->Dk * es},
                        {dd.dA, HD}, {dd.dtau, HD}, {dbx, ntok * d->Dk * es},
                        {dwx, nwx}, {dUb, RDv}, {dUw, RDv}, {dVb, RDv},
                        {dVw, RDv}, {dS0, nst * 4}};
  if (any_overlap(outs, 15, ins, 18)) return CARVE_ERR_UNSUPPORTED;
  const int nb = pick_nb(d);
  if (!nb) return CARVE_ERR_UNSUPPORTED;
  int cus = 0;
  st = device_cus(&cus);
  if (st) return st;
  const BwdWs wl = bwd_workspace_layout(d);
  char* wsb = reinterpret_cast<char*>(workspace);
  const int RP = round_rp(d->R);
  // 1-2. chunk-parallel recompute -> chunk records, overlapped with the adjoint
  FwdArgs f;
  f.q = q; f.k = k; f.v = v; f.beta = beta; f.bx = bx; f.wx = wx;
  f.g = dc.g; f.Ub = Ub; f.Uw = Uw; f.Vb = Vb; f.Vw = Vw; f.S0 = nullptr;
  f.f = dc.f; f.A = dc.A; f.tau_f = dc.tau_f;
  f.o = nullptr; f.S_T = nullptr; f.S_chunks = const_cast<float*>(S_chunks);
  f.rec = wsb + wl.rec;
  f.B = d->B; f.T = d->T; f.H = d->H; f.R = d->R; f.RP = RP; f.L = d->L;
  BwdArgs a;
  a.v = v; a.Ub = Ub; a.Uw = Uw; a.Vb = Vb; a.Vw = Vw; a.S_chunks = S_chunks;
  a.f = dc.f; a.A = dc.A; a.tau_f = dc.tau_f;
  a.dO = dO; a.dS_T = dS_T;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dbeta = dbeta; a.dbx = dbx; a.dwx = dwx; a.dg = dd.dg; a.dS0 = dS0;
  a.df = dd.df;
  a.part = reinterpret_cast<float*>(wsb + wl.part);
  a.partV = reinterpret_cast<float*>(wsb + wl.partV);
  a.partG = reinterpret_cast<float*>(wsb + wl.partG);
  a.rec = wsb + wl.rec;
  a.opnd = wsb + wl.opnd;
  a.B = d->B; a.T = d->T; a.H = d->H; a.R = d->R; a.RP = RP; a.L = d->L; a.NB = nb;
  a.splits = param_splits(d->B * d->H);
  a.wait_limit = g_wait_limit;
  int* sync = reinterpret_cast<int*>(wsb + wl.sync);
  prof_mark(stream);
  st = launch_sync_clear(sync, sync_ints((size_t)d->B * d->H, (size_t)(d->T / d->L)), stream);
  if (st) return st;
  prof_mark(stream);
  st = launch_bwd_fused(f, a, sync, cus, d->dtype, d->Dk, nb, variant_of(dc, sw, act), stream);
  if (st) return st;
  prof_mark(stream);
  // 3. in one launch: d[Ub; Uw] from the per-chunk dF, dVb, dVw from dbx, dwx
  //    and tau (dUb, dVb only with the scalar write gate)
  st = launch_bwd_param(a, d->dtype, d->Dk, sw, stream);
  if (st) return st;
  prof_mark(stream);
  // 4. fixed-order reductions of the partials
  const int nbh = d->B * d->H;
  const size_t RD = (size_t)d->R * d->Dk;
  st = launch_param_reduce(a.part, nbh * a.splits, a.partV, nbh * a.splits, RD, dUb, sw ? nullptr : dUw, dVb,
                           sw ? nullptr : dVw, stream);
  if (st) return st;
  prof_mark(stream);
  // 5. (gated) dA, dtau summed over the batch
  if (dc.gated()) {
    st = launch_gate_reduce(a.partG, d->B, d->H, d->Dk, dd.dA, dd.dtau, stream);
    if (st) return st;
    prof_mark(stream);
  }
  // 6. (input activations) dq, dk through the L2 normalisation and SiLU
  if (act) {
    st = launch_act_bwd(q, k, dq, dk, (size_t)d->B * d->T * d->H, d->Dk, d->dtype, stream);
    prof_mark(stream);
  }
  return st;
}

}  // namespace

extern "C" {

int carve_chunk_fwd(const carve_dims_t* d, const void* q, const void* k, const void* v,
                    const void* beta, const float* g, const void* bx, const void* wx,
                    const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                    const float* S0, void* o, float* S_T, float* S_chunks, void* workspace,
                    size_t workspace_bytes, hipStream_t stream) {
  (void)workspace;
  (void)workspace_bytes;
  return fwd_impl(d, q, k, v, beta, Decay{g, nullptr, nullptr, nullptr}, bx, wx, Ub, Uw, Vb, Vw, S0, o, S_T,
                  S_chunks, false, false, stream);
}

int carve_chunk_fwd_gated(const carve_dims_t* d, const void* q, const void* k, const void* v,
                          const void* beta, const void* f, const float* A, const float* tau_f,
                          const void* bx, const void* wx, const float* Ub, const float* Uw,
                          const float* Vb, const float* Vw, const float* S0, void* o, float* S_T,
                          float* S_chunks, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  (void)workspace;
  (void)workspace_bytes;
  if (!f) {
    ProfClear pc;
    return CARVE_ERR_NULL;
  }
  return fwd_impl(d, q, k, v, beta, Decay{nullptr, f, A, tau_f}, bx, wx, Ub, Uw, Vb, Vw, S0, o, S_T, S_chunks,
                  false, false, stream);
}

int carve_chunk_bwd(const carve_dims_t* d, const void* q, const void* k, const void* v,
                    const void* beta, const float* g, const void* bx, const void* wx,
                    const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                    const float* S_chunks, const void* dO, const float* dS_T, void* dq, void* dk,
                    void* dv, void* dbeta, float* dg, void* dbx, void* dwx, float* dUb,
                    float* dUw, float* dVb, float* dVw, float* dS0, void* workspace,
                    size_t workspace_bytes, hipStream_t stream) {
  return bwd_impl(d, q, k, v, beta, Decay{g, nullptr, nullptr, nullptr}, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO,
                  dS_T, dq, dk, dv, dbeta, DecayGrad{dg, nullptr, nullptr, nullptr}, dbx, dwx, dUb, dUw, dVb,
                  dVw, dS0, workspace, workspace_bytes, false, false, stream);
}

int carve_chunk_bwd_gated(const carve_dims_t* d, const void* q, const void* k, const void* v,
                          const void* beta, const void* f, const float* A, const float* tau_f,
                          const void* bx, const void* wx, const float* Ub, const float* Uw,
                          const float* Vb, const float* Vw, const float* S_chunks, const void* dO,
                          const float* dS_T, void* dq, void* dk, void* dv, void* dbeta, void* df,
                          float* dA, float* dtau, void* dbx, void* dwx, float* dUb, float* dUw,
                          float* dVb, float* dVw, float* dS0, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  if (!f) {
    ProfClear pc;
    return CARVE_ERR_NULL;
  }
  return bwd_impl(d, q, k, v, beta, Decay{nullptr, f, A, tau_f}, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO, dS_T,
                  dq, dk, dv, dbeta, DecayGrad{nullptr, df, dA, dtau}, dbx, dwx, dUb, dUw, dVb, dVw, dS0,
                  workspace, workspace_bytes, false, false, stream);
}

int carve_chunk_fwd_sw(const carve_dims_t* d, const void* q, const void* k, const void* v,
                       const void* beta, const float* g, const void* f, const float* A,
                       const float* tau_f, const void* bx, const void* wx, const float* Ub,
                       const float* Vb, const float* S0, void* o, float* S_T, float* S_chunks,
                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  (void)workspace;
  (void)workspace_bytes;
  if (!g == !f) {
    ProfClear pc;
    return g ? CARVE_ERR_ARG : CARVE_ERR_NULL;
  }
  const Decay dc = g ? Decay{g, nullptr, nullptr, nullptr} : Decay{nullptr, f, A, tau_f};
  return fwd_impl(d, q, k, v, beta, dc, bx, wx, Ub, nullptr, Vb, nullptr, S0, o, S_T, S_chunks, true, false, stream);
}

int carve_chunk_bwd_sw(const carve_dims_t* d, const void* q, const void* k, const void* v,
                       const void* beta, const float* g, const void* f, const float* A,
                       const float* tau_f, const void* bx, const void* wx, const float* Ub,
                       const float* Vb, const float* S_chunks, const void* dO, const float* dS_T,
                       void* dq, void* dk, void* dv, void* dbeta, float* dg, void* df, float* dA,
                       float* dtau, void* dbx, void* dwx, float* dUb, float* dVb, float* dS0,
                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!g == !f) {
    ProfClear pc;
    return g ? CARVE_ERR_ARG : CARVE_ERR_NULL;
  }
  const Decay dc = g ? Decay{g, nullptr, nullptr, nullptr} : Decay{nullptr, f, A, tau_f};
  const DecayGrad dd = g ? DecayGrad{dg, nullptr, nullptr, nullptr} : DecayGrad{nullptr, df, dA, dtau};
  return bwd_impl(d, q, k, v, beta, dc, bx, wx, Ub, nullptr, Vb, nullptr, S_chunks, dO, dS_T, dq, dk, dv, dbeta, dd,
                  dbx, dwx, dUb, nullptr, dVb, nullptr, dS0, workspace, workspace_bytes, true, false, stream);
}

int carve_chunk_fwd_act(const carve_dims_t* d, const void* q, const void* k, const void* v,
                        const void* beta, const float* g, const void* bx, const void* wx,
                        const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                        const float* S0, void* o, float* S_T, float* S_chunks, void* workspace,
                        size_t workspace_bytes, hipStream_t stream) {
  (void)workspace;
  (void)workspace_bytes;
  return fwd_impl(d, q, k, v, beta, Decay{g, nullptr, nullptr, nullptr}, bx, wx, Ub, Uw, Vb, Vw, S0, o, S_T,
                  S_chunks, false, true, stream);
}

int carve_chunk_bwd_act(const carve_dims_t* d, const void* q, const void* k, const void* v,
                        const void* beta, const float* g, const void* bx, const void* wx,
                        const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                        const float* S_chunks, const void* dO, const float* dS_T, void* dq, void* dk,
                        void* dv, void* dbeta, float* dg, void* dbx, void* dwx, float* dUb,
                        float* dUw, float* dVb, float* dVw, float* dS0, void* workspace,
                        size_t workspace_bytes, hipStream_t stream) {
  return bwd_impl(d, q, k, v, beta, Decay{g, nullptr, nullptr, nullptr}, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO,
                  dS_T, dq, dk, dv, dbeta, DecayGrad{dg, nullptr, nullptr, nullptr}, dbx, dwx, dUb, dUw, dVb,
                  dVw, dS0, workspace, workspace_bytes, false, true, stream);
}

}  // extern "C"

// ---- output RMS normalisation (Alg. carve_fwd output step, hoisted) --------

namespace {

// rows and row length of reshape(o) [B*T, H*Dv]; only B, T, H, Dv and dtype
// of the dims are read
int norm_dims(const carve_dims_t* d, long* rows, int* N) {
  if (!d) return CARVE_ERR_NULL;
  if (d->B <= 0 || d->T <= 0 || d->H <= 0 || d->Dv <= 0) return CARVE_ERR_SHAPE;
  if (d->dtype != CARVE_F32 && d->dtype != CARVE_BF16) return CARVE_ERR_UNSUPPORTED;
  const long long n = (long long)d->H * d->Dv;
  if (n > (1 << 20) || !rmsnorm_supported(d->dtype, (int)n)) return CARVE_ERR_UNSUPPORTED;
  const long long r = (long long)d->B * d->T;
  if (r * n >= (1LL << 62)) return CARVE_ERR_UNSUPPORTED;
  *rows = (long)r;
  *N = (int)n;
  return CARVE_OK;
}

bool eps_ok(float eps) { return eps >= 0.0f && eps <= 3.0e38f; }   // false for NaN and +Inf

}  // namespace

extern "C" {

size_t carve_rmsnorm_workspace_size(const carve_dims_t* d) {
  long rows = 0;
  int N = 0;
  if (norm_dims(d, &rows, &N) != CARVE_OK) return 0;
  return align256((size_t)rmsnorm_bwd_groups(rows) * N * sizeof(float));
}

int carve_rmsnorm_fwd(const carve_dims_t* d, const void* o, const float* weight, float eps, void* y,
                      hipStream_t stream) {
  ProfClear pc;
  long rows = 0;
  int N = 0;
  int st = norm_dims(d, &rows, &N);
  if (st) return st;
  if (!o || !weight || !y) return CARVE_ERR_NULL;
  if (!eps_ok(eps)) return CARVE_ERR_ARG;
  if (!aligned16(o) || !aligned16(weight) || !aligned16(y)) return CARVE_ERR_ALIGN;
  const size_t es = esize(d->dtype);
  const Range ins[] = {{o, (size_t)rows * N * es}, {weight, (size_t)N * 4}};
  const Range outs[] = {{y, (size_t)rows * N * es}};
  if (any_overlap(outs, 1, ins, 2)) return CARVE_ERR_UNSUPPORTED;
  prof_mark(stream);
  st = launch_rmsnorm_fwd(o, weight, y, rows, N, eps, d->dtype, stream);
  prof_mark(stream);
  return st;
}

int carve_rmsnorm_bwd_noalloc(const carve_dims_t* d, const void* o, const float* weight, float eps, const void* dy,
                              void* d_o, float* dweight, hipStream_t stream) {
  long rows = 0;
  int N = 0;
  int st = norm_dims(d, &rows, &N);
  if (st) {
    ProfClear pc;
    return st;
  }
  const size_t need = carve_rmsnorm_workspace_size(d);
  if (need > kNormScratchBytes) {
    ProfClear pc;
    return CARVE_ERR_WORKSPACE;
  }
  float* ws = nullptr;
  st = norm_scratch(&ws);
  if (st) {
    ProfClear pc;
    return st;
  }
  return carve_rmsnorm_bwd(d, o, weight, eps, dy, d_o, dweight, ws, kNormScratchBytes, stream);
}

int carve_rmsnorm_bwd(const carve_dims_t* d, const void* o, const float* weight, float eps, const void* dy,
                      void* d_o, float* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ProfClear pc;
  long rows = 0;
  int N = 0;
  int st = norm_dims(d, &rows, &N);
  if (st) return st;
  if (!o || !weight || !dy || !d_o || !dweight) return CARVE_ERR_NULL;
  if (!eps_ok(eps)) return CARVE_ERR_ARG;
  const void* ptrs[] = {o, weight, dy, d_o, dweight, workspace};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_rmsnorm_workspace_size(d);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t es = esize(d->dtype);
  const size_t nx = (size_t)rows * N * es;
  const Range ins[] = {{o, nx}, {weight, (size_t)N * 4}, {dy, nx}, {workspace, need}};
  const Range outs[] = {{d_o, nx}, {dweight, (size_t)N * 4}};
  if (any_overlap(outs, 2, ins, 4)) return CARVE_ERR_UNSUPPORTED;
  prof_mark(stream);
  st = launch_rmsnorm_bwd(o, weight, dy, d_o, reinterpret_cast<float*>(workspace), dweight, rows, N, eps, d->dtype,
                          stream, prof_mark);
  prof_mark(stream);
  return st;
}

}  // extern "C"

// ---- the gated delta rule ----------------------------------------------------

namespace {

// largest offset + 1 of a strided [B, T, H, D] tensor, in bytes
size_t span(long long sb, long long st, long long sh, int B, int T, int H, int D, size_t es) {
  return ((size_t)(B - 1) * sb + (size_t)(T - 1) * st + (size_t)(H - 1) * sh + D) * es;
}

int check_gdr(const carve_gdr_dims_t* d) {
  if (!d) return CARVE_ERR_NULL;
  if (d->B <= 0 || d->T <= 0 || d->N < 0 || d->Hk <= 0 || d->Hv <= 0 || d->Dk <= 0 || d->Dv <= 0) return CARVE_ERR_SHAPE;
  if (d->N > 0 && d->B != 1) return CARVE_ERR_SHAPE;
  if (d->dtype != CARVE_F32 && d->dtype != CARVE_BF16) return CARVE_ERR_UNSUPPORTED;
  if (d->Dk != 32 && d->Dk != 64 && d->Dk != 128) return CARVE_ERR_UNSUPPORTED;
  if (d->Dv != 32 && d->Dv != 64 && d->Dv != 128 && d->Dv != 256) return CARVE_ERR_UNSUPPORTED;
  if (d->Hv % d->Hk || d->Hv > 65535) return CARVE_ERR_UNSUPPORTED;
  if (!(d->scale >= -3.0e38f && d->scale <= 3.0e38f)) return CARVE_ERR_ARG;
  const long long strides[] = {d->q_batch, d->q_token, d->q_head, d->k_batch, d->k_token,
                               d->k_head,  d->v_batch, d->v_token, d->v_head};
  const long long vec = 16 / (long long)esize(d->dtype);
  for (const long long s : strides) {
    if (s < 0) return CARVE_ERR_ARG;
    if (s % vec) return CARVE_ERR_ALIGN;
  }
  // (no tensor reaches 2^45 elements: the spans below stay within 64 bits)
  const int counts[] = {d->B, d->T, d->Hk, d->B, d->T, d->Hk, d->B, d->T, d->Hv};
  for (int i = 0; i < 9; ++i)
    if ((double)strides[i] * (counts[i] - 1) >= 3.5e13) return CARVE_ERR_UNSUPPORTED;
  // (a chunk's rows are addressed with 32 bits)
  for (const long long s : {d->q_token, d->k_token, d->v_token, (long long)d->Hv * d->Dv})
    if (s >= (1LL << 24) / (long long)esize(d->dtype)) return CARVE_ERR_UNSUPPORTED;
  // (row and slot numbers are ints)
  if ((long long)d->B * d->T >= (1LL << 31)) return CARVE_ERR_UNSUPPORTED;
  if ((long long)d->B * ((d->T + kGdrC - 1) / kGdrC) + d->N >= (1LL << 31)) return CARVE_ERR_UNSUPPORTED;
  const long long seqs = d->N ? d->N : d->B;
  if (seqs * d->Hv * (d->Dv / 32) >= (1LL << 30)) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}

size_t gdr_chunks(const carve_gdr_dims_t* d) {
  return d->N ? (size_t)(d->T / kGdrC) + d->N : (size_t)d->B * ((d->T + kGdrC - 1) / kGdrC);
}
// the chunk form's: a launch has less than 2^32 threads, 512 a chunk slot and 512 a
// (sequence, head, 32 value columns)
int check_gdr_chunk(const carve_gdr_dims_t* d) {
  const int st = check_gdr(d);
  if (st) return st;
  const long long heads = (d->N ? d->N : (long long)d->B) * d->Hv;
  if ((heads + 7) / 8 * 8 * (d->Dv / 32) >= (1LL << 23) || gdr_chunks(d) >= (1u << 23)) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}
// workspace bytes of one (chunk slot, value head)
size_t gdr_per(const carve_gdr_dims_t* d, bool bwd) {
  if (d->dtype == CARVE_BF16) return bwd ? GdrWs<bf16_t>::bBytes : GdrWs<bf16_t>::fBytes;
  return bwd ? GdrWs<float>::bBytes : GdrWs<float>::fBytes;
}
size_t gdr_state(const carve_gdr_dims_t* d) { return (size_t)d->Hv * d->Dv * d->Dk * 4; }   // bytes, all heads

void gdr_args(GdrArgs& a, const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
              const void* beta, const int* offsets, void* ws, bool bwd) {
  a = GdrArgs{};
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.offsets = offsets;
  a.qs[0] = d->q_batch, a.qs[1] = d->q_token, a.qs[2] = d->q_head;
  a.ks[0] = d->k_batch, a.ks[1] = d->k_token, a.ks[2] = d->k_head;
  a.vs[0] = d->v_batch, a.vs[1] = d->v_token, a.vs[2] = d->v_head;
  a.T = d->T, a.Hk = d->Hk, a.Hv = d->Hv, a.Dk = d->Dk, a.Dv = d->Dv;
  a.nseq = d->N ? d->N : d->B;
  a.nslots = (int)gdr_chunks(d);
  a.scale = d->scale;
  a.ws = static_cast<char*>(ws);
  a.per = (int)gdr_per(d, bwd);
}

// the input ranges that every entry point has
int gdr_inputs(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
               const void* beta, Range* r) {
  const size_t es = esize(d->dtype), rows = (size_t)d->B * d->T;
  r[0] = {q, span(d->q_batch, d->q_token, d->q_head, d->B, d->T, d->Hk, d->Dk, es)};
  r[1] = {k, span(d->k_batch, d->k_token, d->k_head, d->B, d->T, d->Hk, d->Dk, es)};
  r[2] = {v, span(d->v_batch, d->v_token, d->v_head, d->B, d->T, d->Hv, d->Dv, es)};
  r[3] = {g, rows * d->Hv * 4};
  r[4] = {beta, rows * d->Hv * es};
  return 5;
}

}  // namespace

extern "C" {

size_t carve_gdr_chunk_count(const carve_gdr_dims_t* d) { return check_gdr_chunk(d) == CARVE_OK ? gdr_chunks(d) : 0; }

size_t carve_gdr_workspace_size(const carve_gdr_dims_t* d, int for_backward) {
  if (check_gdr_chunk(d) != CARVE_OK) return 0;
  const size_t n = gdr_chunks(d);
  const size_t images = align256(n * d->Hv * gdr_per(d, for_backward != 0));
  return for_backward ? images + n * gdr_state(d) + n * d->Hv * d->Dv * kGdrC * 4 : images;
}

int carve_gdr_chunk_fwd(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                  const void* beta, const float* S0, const int* offsets, void* o, float* S_T, float* S_chunks,
                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ProfClear pc;
  int st = check_gdr_chunk(d);
  if (st) return st;
  if (!q || !k || !v || !g || !beta || !o || (d->N > 0 && !offsets)) return CARVE_ERR_NULL;
  if (d->N == 0 && offsets) return CARVE_ERR_ARG;
  const void* ptrs[] = {q, k, v, g, beta, S0, offsets, o, S_T, S_chunks, workspace};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_gdr_workspace_size(d, 0);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t seqs = d->N ? d->N : d->B, state = gdr_state(d);
  Range ins[7];
  int nin = gdr_inputs(d, q, k, v, g, beta, ins);
  ins[nin++] = {S0, seqs * state};
  ins[nin++] = {offsets, (size_t)(d->N + 1) * 4};
  const Range outs[] = {{o, (size_t)d->B * d->T * d->Hv * d->Dv * esize(d->dtype)},
                        {S_T, seqs * state},
                        {S_chunks, gdr_chunks(d) * state},
                        {workspace, need}};
  if (any_overlap(outs, 4, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  GdrArgs a;
  gdr_args(a, d, q, k, v, g, beta, offsets, workspace, false);
  a.S0 = S0, a.o = o, a.S_T = S_T, a.S_chunks = S_chunks;
  prof_mark(stream);
  return launch_gdr_fwd(a, d->dtype, stream, prof_mark);
}

int carve_gdr_chunk_bwd(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                  const void* beta, const float* S_chunks, const int* offsets, const void* dO, const float* dS_T,
                  void* dq, void* dk, void* dv, float* dg, void* dbeta, float* dS0, void* workspace,
                  size_t workspace_bytes, hipStream_t stream) {
  ProfClear pc;
  int st = check_gdr_chunk(d);
  if (st) return st;
  if (!q || !k || !v || !g || !beta || !S_chunks || !dO || !dq || !dk || !dv || !dg || !dbeta ||
      (d->N > 0 && !offsets))
    return CARVE_ERR_NULL;
  if (d->N == 0 && offsets) return CARVE_ERR_ARG;
  const void* ptrs[] = {q, k, v, g, beta, S_chunks, offsets, dO, dS_T, dq, dk, dv, dg, dbeta, dS0, workspace};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_gdr_workspace_size(d, 1);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t es = esize(d->dtype), rows = (size_t)d->B * d->T;
  const size_t seqs = d->N ? d->N : d->B, state = gdr_state(d);
  Range ins[9];
  int nin = gdr_inputs(d, q, k, v, g, beta, ins);
  ins[nin++] = {S_chunks, gdr_chunks(d) * state};
  ins[nin++] = {offsets, (size_t)(d->N + 1) * 4};
  ins[nin++] = {dO, rows * d->Hv * d->Dv * es};
  ins[nin++] = {dS_T, seqs * state};
  const Range outs[] = {{dq, rows * d->Hk * d->Dk * es}, {dk, rows * d->Hk * d->Dk * es},
                        {dv, rows * d->Hv * d->Dv * es}, {dg, rows * d->Hv * 4},
                        {dbeta, rows * d->Hv * es},      {dS0, seqs * state},
                        {workspace, need}};
  if (any_overlap(outs, 7, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  GdrArgs a;
  gdr_args(a, d, q, k, v, g, beta, offsets, workspace, true);
  a.S_chunks = const_cast<float*>(S_chunks);   // (read only)
  a.dS_chunks = reinterpret_cast<float*>(a.ws + align256(gdr_chunks(d) * d->Hv * gdr_per(d, true)));
  a.dR = a.dS_chunks + gdr_chunks(d) * (gdr_state(d) / 4);
  a.dO = dO, a.dS_T = dS_T, a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dS0 = dS0;
  prof_mark(stream);
  return launch_gdr_bwd(a, d->dtype, stream, prof_mark);
}

int carve_gdr_step(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                   const void* beta, const int* slots, int pool, float* state, void* o, hipStream_t stream) {
  ProfClear pc;
  int st = check_gdr(d);
  if (st) return st;
  if (d->N != 0 || pool <= 0 || (!slots && pool < d->B)) return CARVE_ERR_SHAPE;
  if (d->B > 65535) return CARVE_ERR_UNSUPPORTED;
  if (!q || !k || !v || !g || !beta || !state || !o) return CARVE_ERR_NULL;
  const void* ptrs[] = {q, k, v, g, beta, state, o};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  if (slots && ((uintptr_t)slots & 3u)) return CARVE_ERR_ALIGN;
  Range ins[6];
  int nin = gdr_inputs(d, q, k, v, g, beta, ins);
  ins[nin++] = {slots, (size_t)d->B * 4};
  const Range outs[] = {{o, (size_t)d->B * d->T * d->Hv * d->Dv * esize(d->dtype)}, {state, (size_t)pool * gdr_state(d)}};
  if (any_overlap(outs, 2, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  GdrStepArgs a = {};
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.slots = slots, a.state = state, a.o = o;
  a.qs[0] = d->q_batch, a.qs[1] = d->q_token, a.qs[2] = d->q_head;
  a.ks[0] = d->k_batch, a.ks[1] = d->k_token, a.ks[2] = d->k_head;
  a.vs[0] = d->v_batch, a.vs[1] = d->v_token, a.vs[2] = d->v_head;
  a.B = d->B, a.T = d->T, a.Hk = d->Hk, a.Hv = d->Hv, a.Dv = d->Dv, a.nslots = pool, a.scale = d->scale;
  prof_mark(stream);
  st = launch_gdr_step(a, d->Dk, d->dtype, stream);
  prof_mark(stream);
  return st;
}

}  // extern "C"

// ---- the norms around a block ---------------------------------------------------

namespace {

int check_block_norm(const carve_block_norm_dims_t* d) {
  if (!d) return CARVE_ERR_NULL;
  if (d->rows <= 0 || d->N <= 0 || d->groups <= 0 || d->N % d->groups) return CARVE_ERR_SHAPE;
  if (d->dtype != CARVE_F32 && d->dtype != CARVE_BF16) return CARVE_ERR_UNSUPPORTED;
  const int vec = 16 / (int)esize(d->dtype);
  if (d->N % vec || d->N > kBlockNormMaxN || d->rows >= (1LL << 31)) return CARVE_ERR_UNSUPPORTED;
  const int size = d->N / d->groups;
  if (d->groups > 1 && (size % vec || size / vec > 64 || ((size / vec) & (size / vec - 1)))) return CARVE_ERR_UNSUPPORTED;
  if (!eps_ok(d->eps)) return CARVE_ERR_ARG;
  return CARVE_OK;
}

// what the forward and the backward check alike; fills the arguments and the input ranges
int block_norm_args(const carve_block_norm_dims_t* d, const void* y, const float* weight, const void* gate,
                    const void* residual, const float* scale, const float* next_weight, BlockNormArgs& a, Range* ins) {
  if (!y || !weight) return CARVE_ERR_NULL;
  if (gate && d->gate_act != CARVE_GATE_SILU && d->gate_act != CARVE_GATE_SIGMOID) return CARVE_ERR_ARG;
  if (residual && !(d->alpha >= -3.0e38f && d->alpha <= 3.0e38f)) return CARVE_ERR_ARG;
  const void* ptrs[] = {y, weight, gate, residual, scale, next_weight};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t es = esize(d->dtype);
  const long long vec = 16 / (long long)es;
  const struct {
    const void* p;
    long long stride;
  } rows[] = {{y, d->y_stride}, {gate, d->gate_stride}, {residual, d->residual_stride}};
  for (int i = 0; i < 3; ++i) {
    ins[i] = {nullptr, 0};
    if (!rows[i].p) continue;
    if (rows[i].stride < 0) return CARVE_ERR_ARG;
    if (rows[i].stride % vec) return CARVE_ERR_ALIGN;
    if ((double)rows[i].stride * (d->rows - 1) >= 3.5e13) return CARVE_ERR_UNSUPPORTED;   // (no tensor reaches that)
    ins[i] = {rows[i].p, ((size_t)(d->rows - 1) * rows[i].stride + d->N) * es};
  }
  ins[3] = {weight, (size_t)d->N * 4};
  ins[4] = {scale, (size_t)d->N * 4};
  ins[5] = {next_weight, (size_t)d->N * 4};
  a = BlockNormArgs{};
  a.y = y, a.gate = gate, a.residual = residual, a.weight = weight, a.scale = scale, a.next_weight = next_weight;
  a.rows = d->rows, a.N = d->N, a.groups = d->groups, a.lanes = (int)(d->N / d->groups / vec), a.act = d->gate_act;
  a.y_stride = d->y_stride, a.gate_stride = d->gate_stride, a.residual_stride = d->residual_stride;
  a.eps = d->eps, a.alpha = d->alpha;
  return CARVE_OK;
}

}  // namespace

extern "C" {

size_t carve_block_norm_workspace_size(const carve_block_norm_dims_t* d) {
  if (check_block_norm(d) != CARVE_OK) return 0;
  return align256((size_t)block_norm_groups(d->rows, d->N, d->dtype) * 3 * d->N * 4);
}

int carve_block_norm_fwd(const carve_block_norm_dims_t* d, const void* y, const float* weight, const void* gate,
                         const void* residual, const float* scale, const float* next_weight, void* x, void* h,
                         hipStream_t stream) {
  ProfClear pc;
  int st = check_block_norm(d);
  if (st) return st;
  if (!x) return CARVE_ERR_NULL;
  if (!next_weight != !h) return CARVE_ERR_ARG;
  BlockNormArgs a;
  Range ins[6];
  st = block_norm_args(d, y, weight, gate, residual, scale, next_weight, a, ins);
  if (st) return st;
  if (!aligned16(x) || !aligned16(h)) return CARVE_ERR_ALIGN;
  const size_t nx = (size_t)d->rows * d->N * esize(d->dtype);
  const Range outs[] = {{x, nx}, {h, nx}};
  if (any_overlap(outs, 2, ins, 6)) return CARVE_ERR_UNSUPPORTED;
  a.x = x, a.h = h;
  prof_mark(stream);
  st = launch_block_norm_fwd(a, d->dtype, stream);
  prof_mark(stream);
  return st;
}

int carve_block_norm_bwd(const carve_block_norm_dims_t* d, const void* y, const float* weight, const void* gate,
                         const void* residual, const float* scale, const float* next_weight, const void* dx,
                         const void* dh, void* dy, void* dgate, void* dresidual, float* dweight, float* dscale,
                         float* dnext_weight, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ProfClear pc;
  int st = check_block_norm(d);
  if (st) return st;
  if (!dy || !dweight || (!dx && !dh)) return CARVE_ERR_NULL;
  if (!next_weight != !dh || !next_weight != !dnext_weight || !gate != !dgate || !residual != !dresidual ||
      !scale != !dscale)
    return CARVE_ERR_ARG;
  BlockNormArgs a;
  Range ins[8];
  st = block_norm_args(d, y, weight, gate, residual, scale, next_weight, a, ins);
  if (st) return st;
  const void* ptrs[] = {dx, dh, dy, dgate, dresidual, dweight, dscale, dnext_weight, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_block_norm_workspace_size(d);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t nx = (size_t)d->rows * d->N * esize(d->dtype), np = (size_t)d->N * 4;
  ins[6] = {dx, nx};
  ins[7] = {dh, nx};
  const Range outs[] = {{dy, nx}, {dgate, nx}, {dresidual, nx}, {dweight, np}, {dscale, np}, {dnext_weight, np}, {workspace, need}};
  if (any_overlap(outs, 7, ins, 8)) return CARVE_ERR_UNSUPPORTED;
  a.dx = dx, a.dh = dh, a.dy = dy, a.dgate = dgate, a.dresidual = dresidual;
  a.dweight = dweight, a.dscale = dscale, a.dnext_weight = dnext_weight;
  a.partial = static_cast<float*>(workspace);
  prof_mark(stream);
  return launch_block_norm_bwd(a, d->dtype, stream, prof_mark);
}

}  // extern "C"

// ---- the short causal convolution --------------------------------------------------

namespace {

// sizes that packed and dense rows share: B, T, N of every operator beside the layer
int check_rows(int B, int T, int N, carve_dtype_t dtype) {
  if (B <= 0 || T <= 0 || N < 0) return CARVE_ERR_SHAPE;
  if (N > 0 && B != 1) return CARVE_ERR_SHAPE;
  if (dtype != CARVE_F32 && dtype != CARVE_BF16) return CARVE_ERR_UNSUPPORTED;
  if ((long long)B * T >= (1LL << 31)) return CARVE_ERR_UNSUPPORTED;   // (row numbers are ints)
  return CARVE_OK;
}
// a stride of `count` steps: not negative, whole pieces of 16 bytes (vec elements)
int check_stride(long long stride, int count, long long vec) {
  if (stride < 0) return CARVE_ERR_ARG;
  if (stride % vec) return CARVE_ERR_ALIGN;
  // (no tensor reaches 2^45 elements: spans stay within 64 bits)
  if ((double)stride * (count - 1) >= 3.5e13) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}

int check_conv(const carve_short_conv_dims_t* d) {
  if (!d) return CARVE_ERR_NULL;
  if (d->C <= 0 || d->W <= 0) return CARVE_ERR_SHAPE;
  int st = check_rows(d->B, d->T, d->N, d->dtype);
  if (st) return st;
  const long long vec = 16 / (long long)esize(d->dtype);
  if (d->W < 2 || d->W > 4 || d->C % vec || d->C >= (1 << 20)) return CARVE_ERR_UNSUPPORTED;
  // (the kernels count up to a run's rows and W - 1 more behind the last one, in ints)
  if ((long long)d->T > (1LL << 31) - 64) return CARVE_ERR_UNSUPPORTED;
  if (d->activation != CARVE_CONV_LINEAR && d->activation != CARVE_CONV_SILU) return CARVE_ERR_ARG;
  st = check_stride(d->x_batch, d->B, vec);
  return st ? st : check_stride(d->x_token, d->T, vec);
}
size_t conv_seqs(const carve_short_conv_dims_t* d) { return d->N ? d->N : d->B; }
size_t conv_kept(const carve_short_conv_dims_t* d) { return (size_t)(d->W - 1) * d->C * esize(d->dtype); }
Range conv_x(const carve_short_conv_dims_t* d, const void* x) {
  return {x, ((size_t)(d->B - 1) * d->x_batch + (size_t)(d->T - 1) * d->x_token + d->C) * esize(d->dtype)};
}
void conv_args(ConvArgs& a, const carve_short_conv_dims_t* d, const void* x, const float* weight, const float* bias,
               const void* x0, const int* offsets) {
  a = ConvArgs{};
  a.x = x, a.weight = weight, a.bias = bias, a.x0 = x0, a.offsets = offsets;
  a.x_batch = d->x_batch, a.x_token = d->x_token;
  a.T = d->T, a.C = d->C, a.nseq = (int)conv_seqs(d), a.act = d->activation;
}

}  // namespace

extern "C" {

int carve_short_conv_fwd(const carve_short_conv_dims_t* d, const void* x, const float* weight, const float* bias,
                         const void* x0, const int* offsets, void* y, void* x_T, hipStream_t stream) {
  ProfClear pc;
  int st = check_conv(d);
  if (st) return st;
  if (!x || !weight || !y || (d->N > 0 && !offsets)) return CARVE_ERR_NULL;
  if (d->N == 0 && offsets) return CARVE_ERR_ARG;
  const void* ptrs[] = {x, weight, bias, x0, offsets, y, x_T};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t kept = conv_seqs(d) * conv_kept(d);
  const Range ins[] = {conv_x(d, x), {weight, (size_t)d->C * d->W * 4}, {bias, (size_t)d->C * 4}, {x0, kept}, {offsets, (size_t)(d->N + 1) * 4}};
  const Range outs[] = {{y, (size_t)d->B * d->T * d->C * esize(d->dtype)}, {x_T, kept}};
  if (any_overlap(outs, 2, ins, 5)) return CARVE_ERR_UNSUPPORTED;
  ConvArgs a;
  conv_args(a, d, x, weight, bias, x0, offsets);
  a.y = y, a.x_T = x_T;
  prof_mark(stream);
  st = launch_short_conv_fwd(a, d->W, d->dtype, stream);
  prof_mark(stream);
  return st;
}

size_t carve_short_conv_workspace_size(const carve_short_conv_dims_t* d) {
  if (check_conv(d) != CARVE_OK) return 0;
  return align256((size_t)conv_parts(d->T, d->B, d->C, d->dtype) * (d->W + 1) * d->C * 4);
}

int carve_short_conv_bwd(const carve_short_conv_dims_t* d, const void* x, const float* weight, const float* bias,
                         const void* x0, const int* offsets, const void* dy, const void* dx_T, void* dx,
                         float* dweight, float* dbias, void* dx0, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  ProfClear pc;
  int st = check_conv(d);
  if (st) return st;
  if (!x || !weight || !dy || !dx || !dweight || (d->N > 0 && !offsets)) return CARVE_ERR_NULL;
  if ((d->N == 0 && offsets) || !bias != !dbias) return CARVE_ERR_ARG;
  const void* ptrs[] = {x, weight, bias, x0, offsets, dy, dx_T, dx, dweight, dbias, dx0, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_short_conv_workspace_size(d);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t kept = conv_seqs(d) * conv_kept(d), rows = (size_t)d->B * d->T * d->C * esize(d->dtype);
  const size_t nw = (size_t)d->C * d->W * 4, nb = (size_t)d->C * 4;
  const Range ins[] = {conv_x(d, x), {weight, nw}, {bias, nb}, {x0, kept}, {offsets, (size_t)(d->N + 1) * 4}, {dy, rows}, {dx_T, kept}};
  const Range outs[] = {{dx, rows}, {dweight, nw}, {dbias, nb}, {dx0, kept}, {workspace, need}};
  if (any_overlap(outs, 5, ins, 7)) return CARVE_ERR_UNSUPPORTED;
  ConvArgs a;
  conv_args(a, d, x, weight, bias, x0, offsets);
  a.dy = dy, a.dx_T = dx_T, a.dx = dx, a.dweight = dweight, a.dbias = dbias, a.dx0 = dx0;
  a.partial = static_cast<float*>(workspace);
  prof_mark(stream);
  return launch_short_conv_bwd(a, d->W, d->dtype, stream, prof_mark);
}

int carve_short_conv_step(const carve_short_conv_dims_t* d, const void* x, const float* weight, const float* bias,
                          const int* slots, int pool, void* state, void* y, hipStream_t stream) {
  ProfClear pc;
  int st = check_conv(d);
  if (st) return st;
  if (d->N != 0 || pool <= 0 || (!slots && pool < d->B)) return CARVE_ERR_SHAPE;
  if (d->B > 65535) return CARVE_ERR_UNSUPPORTED;
  if (!x || !weight || !state || !y) return CARVE_ERR_NULL;
  const void* ptrs[] = {x, weight, bias, state, y};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  if ((uintptr_t)slots & 3u) return CARVE_ERR_ALIGN;
  const Range ins[] = {conv_x(d, x), {weight, (size_t)d->C * d->W * 4}, {bias, (size_t)d->C * 4}, {slots, (size_t)d->B * 4}};
  const Range outs[] = {{y, (size_t)d->B * d->T * d->C * esize(d->dtype)}, {state, pool * conv_kept(d)}};
  if (any_overlap(outs, 2, ins, 4)) return CARVE_ERR_UNSUPPORTED;
  ConvStepArgs a = {};
  a.x = x, a.weight = weight, a.bias = bias, a.slots = slots, a.state = state, a.y = y;
  a.x_batch = d->x_batch, a.x_token = d->x_token;
  a.B = d->B, a.T = d->T, a.C = d->C, a.pool = pool, a.act = d->activation;
  prof_mark(stream);
  st = launch_short_conv_step(a, d->W, d->dtype, stream);
  prof_mark(stream);
  return st;
}

}  // extern "C"

// ---- rotary positions ------------------------------------------------------------------

namespace {

// whether every element of a strided [.., D] tensor has a place of its own (st, n: strides
// and counts of its three outer dimensions)
bool places_apart(const long long* st, const int* n, long long D) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (st[order[j]] > st[order[j + 1]]) std::swap(order[j], order[j + 1]);
  long long extent = D;
  for (const int i : order) {
    if (n[i] <= 1) continue;
    if (st[i] < extent) return false;
    extent += st[i] * (n[i] - 1);
  }
  return true;
}
// whether two such tensors are slices of one fused tensor's rows without meeting: their
// heads one after another, and what lies from the first head to the last one of them apart
// from every other row's
bool rows_apart(const void* p, const long long* sp, int hp, const void* r, const long long* sr, int hr, const int* n, int D,
                size_t es) {
  if ((uintptr_t)p > (uintptr_t)r) return rows_apart(r, sr, hr, p, sp, hp, n, D, es);
  const size_t off = ((uintptr_t)r - (uintptr_t)p) / es;   // (whole elements: both are 16-byte aligned)
  if ((size_t)(hp - 1) * sp[2] + D > off) return false;
  for (int i = 0; i < 2; ++i)
    if (n[i] > 1 && sp[i] != sr[i]) return false;
  const long long rows[] = {sp[0], sp[1], 0};
  const int counts[] = {n[0], n[1], 1};
  return places_apart(rows, counts, (long long)off + (long long)(hr - 1) * sr[2] + D);
}

}  // namespace

extern "C" {

int carve_rotary(const carve_rotary_dims_t* d, const void* q, const void* k, const double* freq, const int* positions,
                 const int* start, const int* offsets, int backward, void* q_out, void* k_out, hipStream_t stream) {
  ProfClear pc;
  if (!d) return CARVE_ERR_NULL;
  if (d->Hq <= 0 || d->Hk < 0 || d->D <= 0 || d->rot <= 0 || d->rot > d->D) return CARVE_ERR_SHAPE;
  int st = check_rows(d->B, d->T, d->N, d->dtype);
  if (st) return st;
  const size_t es = esize(d->dtype);
  const int vec = (int)(16 / es);
  if (d->D % vec || d->D > 1024 || d->rot % (2 * vec) || (long long)d->Hq + d->Hk > 65535) return CARVE_ERR_UNSUPPORTED;
  if (!(d->amplitude >= -3.0e38f && d->amplitude <= 3.0e38f)) return CARVE_ERR_ARG;
  const long long strides[] = {d->q_batch,  d->q_token,  d->q_head,  d->k_batch,  d->k_token,  d->k_head,
                               d->qo_batch, d->qo_token, d->qo_head, d->ko_batch, d->ko_token, d->ko_head};
  const int counts[] = {d->B, d->T, d->Hq, d->B, d->T, d->Hk > 0 ? d->Hk : 1};
  for (int i = 0; i < 12; ++i) {
    st = check_stride(strides[i], counts[i % 6], vec);
    if (st) return st;
  }
  if (!q || !freq || !q_out || (d->Hk > 0 && (!k || !k_out)) || (d->N > 0 && !offsets)) return CARVE_ERR_NULL;
  if (d->Hk == 0 && (k || k_out)) return CARVE_ERR_ARG;
  if ((d->N == 0 && offsets) || (positions && (start || offsets))) return CARVE_ERR_ARG;
  const void* ptrs[] = {q, k, freq, q_out, k_out};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  for (const int* p : {positions, start, offsets})
    if ((uintptr_t)p & 3u) return CARVE_ERR_ALIGN;
  const size_t nq = span(d->q_batch, d->q_token, d->q_head, d->B, d->T, d->Hq, d->D, es);
  const size_t nqo = span(d->qo_batch, d->qo_token, d->qo_head, d->B, d->T, d->Hq, d->D, es);
  const size_t nk = d->Hk ? span(d->k_batch, d->k_token, d->k_head, d->B, d->T, d->Hk, d->D, es) : 0;
  const size_t nko = d->Hk ? span(d->ko_batch, d->ko_token, d->ko_head, d->B, d->T, d->Hk, d->D, es) : 0;
  const int nqd[] = {d->B, d->T, d->Hq}, nkd[] = {d->B, d->T, d->Hk};
  if (!places_apart(strides + 6, nqd, d->D) || (d->Hk > 0 && !places_apart(strides + 9, nkd, d->D))) return CARVE_ERR_ARG;
  const bool in_place = q_out == q;
  if (d->Hk > 0 && in_place != (k_out == k)) return CARVE_ERR_ARG;
  if (in_place)
    for (int i = 0; i < 6; ++i)
      if ((i < 3 ? nqd[i] : nkd[i - 3]) > 1 && strides[i] != strides[6 + i]) return CARVE_ERR_ARG;
  const Range others[] = {{freq, (size_t)(d->rot / 2) * 8}, {positions, (size_t)d->B * d->T * 4},
                          {start, (size_t)(d->N ? d->N : d->B) * 4}, {offsets, (size_t)(d->N + 1) * 4},
                          {q, in_place ? 0 : nq}, {k, in_place ? 0 : nk}};
  const Range qo = {q_out, nqo}, ko = {k_out, nko};
  if (any_overlap(&qo, 1, others, 6) || any_overlap(&ko, 1, others, 6)) return CARVE_ERR_UNSUPPORTED;
  // (both may be slices of one tensor)
  if (overlap(qo, ko) && !rows_apart(q_out, strides + 6, d->Hq, k_out, strides + 9, d->Hk, nqd, d->D, es))
    return CARVE_ERR_UNSUPPORTED;
  RotaryArgs a = {};
  a.q = q, a.k = k, a.freq = freq, a.positions = positions, a.start = start, a.offsets = offsets, a.qo = q_out, a.ko = k_out;
  for (int i = 0; i < 3; ++i) a.qs[i] = strides[i], a.ks[i] = strides[3 + i], a.qos[i] = strides[6 + i], a.kos[i] = strides[9 + i];
  a.B = d->B, a.T = d->T, a.Hq = d->Hq, a.Hk = d->Hk, a.D = d->D, a.rot = d->rot, a.nseq = d->N ? d->N : d->B;
  a.interleaved = d->interleaved, a.amplitude = d->amplitude, a.sign = backward ? -1.0f : 1.0f, a.copy = !in_place;
  prof_mark(stream);
  st = launch_rotary(a, d->dtype, stream);
  prof_mark(stream);
  return st;
}

}  // extern "C"

// ---- the selective state space scan -------------------------------------------------------

namespace {

int check_ssm(const carve_ssm_dims_t* d) {
  if (!d) return CARVE_ERR_NULL;
  if (d->G <= 0 || d->H <= 0 || d->P <= 0 || d->S <= 0) return CARVE_ERR_SHAPE;
  int st = check_rows(d->B, d->T, d->N, d->dtype);
  if (st) return st;
  if (d->S != 32 && d->S != 64 && d->S != 128) return CARVE_ERR_UNSUPPORTED;
  if (d->P % 32 || d->P > 256 || d->H % d->G || d->H > 65535) return CARVE_ERR_UNSUPPORTED;
  const long long vec = 16 / (long long)esize(d->dtype);
  const struct {
    long long s;
    int n;
    long long vec;
  } strides[] = {{d->x_batch, d->B, vec}, {d->x_token, d->T, vec},  {d->x_head, d->H, vec},   {d->b_batch, d->B, vec},
                 {d->b_token, d->T, vec}, {d->b_group, d->G, vec},  {d->c_batch, d->B, vec},  {d->c_token, d->T, vec},
                 {d->c_group, d->G, vec}, {d->dt_batch, d->B, 1}, {d->dt_token, d->T, 1}};
  for (const auto& x : strides) {
    st = check_stride(x.s, x.n, x.vec);
    if (st) return st;
  }
  // (a chunk's rows are addressed with 32 bits)
  for (const long long s : {d->x_token, d->b_token, d->c_token, (long long)d->H * d->P})
    if (s >= (1LL << 24) / (long long)esize(d->dtype)) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}

// Value rows of a unit: 64, or 32 where P is no multiple of it and with f32 states of 128.  (By
// 64 rows and by 32, outputs of 32 heads of 64: bf16, 4 x 4096 tokens, 112 and 125 us with
// states of 128, 82 and 101 of 64, 73 and 90 of 32; f32, 4 x 1024 tokens, 71 and 66 with states
// of 64, 51 and 51 of 32, 107 and 114 of 128: f32 is within a tenth either way.)
bool ssm_wide(const carve_ssm_dims_t* d) { return d->P % 64 == 0 && !(d->dtype == CARVE_F32 && d->S == 128); }

// chunks of a span, spans (slots of them) and shares of a group's heads
struct SsmPlan {
  size_t chunks, spans;
  int span, splits;
};
// Spans: as many as let every compute unit hold two workgroups of the outputs (a pair of
// units each, see carve_ssm_fwd.hip), none shorter than kSsmMinSpan chunks.  (Replayed from a
// graph, for 512 workgroups, 256 and 1024: 115, 129 and 135 us at 4 x 4096 tokens of 32 heads,
// training 571, 584 and 598; 116, 132 and 134 at 16381 tokens.  For spans of at least 2 chunks,
// 1 and 4: 19, 22 and 19 us at 128 tokens of 8 heads, 28, 23 and 27 at 256, 30, 28 and 39 at
// 1024; 45, 52 and 49 at 4096 of 16, 47, 51 and 48 for 9 prompts of 1777 tokens; training, 74,
// 64 and 72 at 256 of 8, 131, 145 and 138 at 2048 of 32: a chunk a span is a little better for
// the smallest calls alone.)
constexpr long long kSsmGroups = 512;
constexpr int kSsmMinSpan = 2;
SsmPlan ssm_plan(const carve_ssm_dims_t* d) {
  SsmPlan p;
  const long long units = (d->T + (long long)kSsmC - 1) / kSsmC;
  p.chunks = d->N ? (size_t)(d->T / kSsmC) + d->N : (size_t)(d->B * units);
  const long long per = (long long)d->G * ((d->H / d->G * (d->P / (ssm_wide(d) ? 64 : 32)) + 1) / 2) * d->B;
  long long n = kSsmGroups / per;
  if (n > (units + kSsmMinSpan - 1) / kSsmMinSpan) n = (units + kSsmMinSpan - 1) / kSsmMinSpan;
  if (n < 1) n = 1;
  p.span = (int)((units + n - 1) / n);
  const long long L = (long long)p.span * kSsmC;
  p.spans = d->N ? (size_t)(d->T / L) + d->N : (size_t)(d->B * ((d->T + L - 1) / L));
  // Shares of a group's heads: the gradients run one workgroup a compute unit, in turns of
  // 256, each of which takes its heads and about as long as one more to begin and end (32
  // heads, forward and backward: 2048 tokens 134 us, 295 undivided; 8192 tokens 307 and 384).
  const long long rep = d->H / d->G, wgs = (long long)p.chunks * d->G;
  double best = 0.0;
  p.splits = 1;
  for (long long s = 1; s <= rep && s <= 64; s *= 2) {
    const double cost = (double)((wgs * s + 255) / 256) * ((double)((rep + s - 1) / s) + 1.0);
    if (s == 1 || cost < 0.95 * best) best = cost, p.splits = (int)s;
  }
  return p;
}
// the chunk form's: a launch has less than 2^32 threads of each dimension (the gradients 768 a chunk)
constexpr long long kSsmMaxChunks = 5LL << 20;
int check_ssm_chunk(const carve_ssm_dims_t* d) {
  const int st = check_ssm(d);
  if (st) return st;
  if ((long long)(d->T / kSsmC) + d->N >= kSsmMaxChunks || (long long)d->B * ((d->T + kSsmC - 1) / kSsmC) >= kSsmMaxChunks)
    return CARVE_ERR_UNSUPPORTED;
  const SsmPlan p = ssm_plan(d);
  if ((long long)(p.spans + 8) * d->H * (d->P / 32) >= (1LL << 23) || d->G > 61000) return CARVE_ERR_UNSUPPORTED;
  return CARVE_OK;
}
size_t ssm_state(const carve_ssm_dims_t* d) { return (size_t)d->H * d->P * d->S * 4; }   // bytes, all heads
bool ssm_split(const carve_ssm_dims_t* d, const SsmPlan& p) { return (long long)d->T > (long long)p.span * kSsmC; }

// workspace: scalars and C B^T of the chunks | spans' states and decays | state gradients | shares of the head sums | of dB, dC
struct SsmWs {
  size_t scal, cb, Z, Zg, E, part, dBp, total;
};
SsmWs ssm_ws(const carve_ssm_dims_t* d, bool bwd) {
  const SsmPlan p = ssm_plan(d);
  SsmWs w{};
  size_t off = 0;
  const bool split = ssm_split(d, p);
  w.scal = off, off += align256(p.chunks * d->H * (bwd ? kSmBwd : kSmFwd) * 4);
  w.cb = off, off += align256(p.chunks * d->G * (bwd ? 2 : 1) * kSsmCB);
  w.Z = off, off += split ? align256(p.spans * ssm_state(d)) : 0;
  w.Zg = off, off += split ? align256(p.spans * d->H * 4) : 0;
  if (bwd) {
    w.E = off, off += align256(p.chunks * ssm_state(d));
    w.part = off, off += align256(p.chunks * d->H * 16);
    w.dBp = off, off += p.splits > 1 ? align256((size_t)p.splits * 2 * d->B * d->T * d->G * d->S * 4) : 0;
  }
  w.total = off;
  return w;
}
void ssm_args(SsmArgs& a, const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm,
              const void* Cm, const float* D, const float* dt_bias, const int* offsets, void* workspace, bool bwd) {
  a = SsmArgs{};
  a.x = x, a.dt = dt, a.A = A, a.Bm = Bm, a.Cm = Cm, a.D = D, a.dt_bias = dt_bias, a.offsets = offsets;
  a.xs[0] = d->x_batch, a.xs[1] = d->x_token, a.xs[2] = d->x_head;
  a.bs[0] = d->b_batch, a.bs[1] = d->b_token, a.bs[2] = d->b_group;
  a.cs[0] = d->c_batch, a.cs[1] = d->c_token, a.cs[2] = d->c_group;
  a.ds[0] = d->dt_batch, a.ds[1] = d->dt_token;
  a.T = d->T, a.G = d->G, a.H = d->H, a.P = d->P, a.N = d->S, a.softplus = d->softplus;
  const SsmPlan p = ssm_plan(d);
  a.nseq = d->N ? d->N : d->B;
  a.nslots = (int)p.chunks, a.nspans = (int)p.spans, a.span = p.span, a.splits = p.splits;
  const SsmWs w = ssm_ws(d, bwd);
  char* ws = static_cast<char*>(workspace);
  a.Z = reinterpret_cast<float*>(ws + w.Z), a.Zg = reinterpret_cast<float*>(ws + w.Zg);
  a.scal = ws + w.scal, a.cb = ws + w.cb;
  a.E_chunks = reinterpret_cast<float*>(ws + w.E), a.part = reinterpret_cast<float*>(ws + w.part), a.dBp = reinterpret_cast<float*>(ws + w.dBp);
}
int ssm_inputs(const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm,
               const float* D, const float* dt_bias, Range* r) {
  const size_t es = esize(d->dtype), nh = (size_t)d->H * 4;
  r[0] = {x, span(d->x_batch, d->x_token, d->x_head, d->B, d->T, d->H, d->P, es)};
  r[1] = {dt, span(d->dt_batch, d->dt_token, 0, d->B, d->T, 1, d->H, es)};
  r[2] = {Bm, span(d->b_batch, d->b_token, d->b_group, d->B, d->T, d->G, d->S, es)};
  r[3] = {Cm, span(d->c_batch, d->c_token, d->c_group, d->B, d->T, d->G, d->S, es)};
  r[4] = {A, nh}, r[5] = {D, nh}, r[6] = {dt_bias, nh};
  return 7;
}
// pointers every entry point takes: whole pieces of 16 bytes, but the scalars a head and dt
int ssm_aligned(const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm, const void* Cm,
                const float* D, const float* dt_bias) {
  if (!aligned16(x) || !aligned16(Bm) || !aligned16(Cm) || (uintptr_t)dt % esize(d->dtype)) return CARVE_ERR_ALIGN;
  for (const float* p : {A, D, dt_bias})
    if ((uintptr_t)p & 3u) return CARVE_ERR_ALIGN;
  return CARVE_OK;
}

}  // namespace

extern "C" {

size_t carve_ssm_chunk_count(const carve_ssm_dims_t* d) { return check_ssm_chunk(d) == CARVE_OK ? ssm_plan(d).chunks : 0; }

size_t carve_ssm_workspace_size(const carve_ssm_dims_t* d, int for_backward) {
  return check_ssm_chunk(d) == CARVE_OK ? ssm_ws(d, for_backward != 0).total : 0;
}

int carve_ssm_chunk_fwd(const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm,
                        const void* Cm, const float* D, const float* dt_bias, const float* S0, const int* offsets,
                        void* y, float* S_T, float* S_chunks, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  ProfClear pc;
  int st = check_ssm_chunk(d);
  if (st) return st;
  if (!x || !dt || !A || !Bm || !Cm || !y || (d->N > 0 && !offsets)) return CARVE_ERR_NULL;
  if (d->N == 0 && offsets) return CARVE_ERR_ARG;
  st = ssm_aligned(d, x, dt, A, Bm, Cm, D, dt_bias);
  if (st) return st;
  const void* ptrs[] = {S0, offsets, y, S_T, S_chunks, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  const size_t need = carve_ssm_workspace_size(d, 0);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t seqs = d->N ? d->N : d->B, state = ssm_state(d);
  Range ins[9];
  int nin = ssm_inputs(d, x, dt, A, Bm, Cm, D, dt_bias, ins);
  ins[nin++] = {S0, seqs * state};
  ins[nin++] = {offsets, (size_t)(d->N + 1) * 4};
  const Range outs[] = {{y, (size_t)d->B * d->T * d->H * d->P * esize(d->dtype)},
                        {S_T, seqs * state},
                        {S_chunks, ssm_plan(d).chunks * state},
                        {workspace, need}};
  if (any_overlap(outs, 4, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  SsmArgs a;
  ssm_args(a, d, x, dt, A, Bm, Cm, D, dt_bias, offsets, workspace, false);
  a.S0 = S0, a.y = y, a.S_T = S_T, a.S_chunks = S_chunks;
  prof_mark(stream);
  return launch_ssm_fwd(a, d->dtype, stream, prof_mark);
}

int carve_ssm_chunk_bwd(const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm,
                        const void* Cm, const float* D, const float* dt_bias, const float* S_chunks, const int* offsets,
                        const void* dy, const float* dS_T, void* dx, void* ddt, float* dA, void* dBm, void* dCm,
                        float* dD, float* ddt_bias, float* dS0, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  ProfClear pc;
  int st = check_ssm_chunk(d);
  if (st) return st;
  if (!x || !dt || !A || !Bm || !Cm || !S_chunks || !dy || !dx || !ddt || !dA || !dBm || !dCm || (d->N > 0 && !offsets))
    return CARVE_ERR_NULL;
  if ((d->N == 0 && offsets) || !D != !dD || !dt_bias != !ddt_bias) return CARVE_ERR_ARG;
  st = ssm_aligned(d, x, dt, A, Bm, Cm, D, dt_bias);
  if (st) return st;
  const void* ptrs[] = {S_chunks, offsets, dy, dS_T, dx, ddt, dBm, dCm, dS0, workspace};
  for (const void* p : ptrs)
    if (!aligned16(p)) return CARVE_ERR_ALIGN;
  for (const float* p : {dA, dD, ddt_bias})
    if ((uintptr_t)p & 3u) return CARVE_ERR_ALIGN;
  const size_t need = carve_ssm_workspace_size(d, 1);
  if (!workspace || workspace_bytes < need) return CARVE_ERR_WORKSPACE;
  const size_t es = esize(d->dtype), rows = (size_t)d->B * d->T, seqs = d->N ? d->N : d->B, state = ssm_state(d);
  Range ins[11];
  int nin = ssm_inputs(d, x, dt, A, Bm, Cm, D, dt_bias, ins);
  ins[nin++] = {S_chunks, ssm_plan(d).chunks * state};
  ins[nin++] = {offsets, (size_t)(d->N + 1) * 4};
  ins[nin++] = {dy, rows * d->H * d->P * es};
  ins[nin++] = {dS_T, seqs * state};
  const size_t nb = rows * d->G * d->S * es, nh = (size_t)d->H * 4;
  const Range outs[] = {{dx, rows * d->H * d->P * es}, {ddt, rows * d->H * es}, {dA, nh}, {dBm, nb}, {dCm, nb},
                        {dD, nh}, {ddt_bias, nh}, {dS0, seqs * state}, {workspace, need}};
  if (any_overlap(outs, 9, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  SsmArgs a;
  ssm_args(a, d, x, dt, A, Bm, Cm, D, dt_bias, offsets, workspace, true);
  a.S_chunks = const_cast<float*>(S_chunks);   // (read only)
  a.dy = dy, a.dS_T = dS_T, a.dx = dx, a.ddt = ddt, a.dA = dA, a.dBm = dBm, a.dCm = dCm, a.dD = dD;
  a.ddt_bias = ddt_bias, a.dS0 = dS0;
  prof_mark(stream);
  return launch_ssm_bwd(a, d->dtype, stream, prof_mark);
}

int carve_ssm_step(const carve_ssm_dims_t* d, const void* x, const void* dt, const float* A, const void* Bm,
                   const void* Cm, const float* D, const float* dt_bias, const int* slots, int pool, float* state,
                   void* y, hipStream_t stream) {
  ProfClear pc;
  int st = check_ssm(d);
  if (st) return st;
  if (d->N != 0 || pool <= 0 || (!slots && pool < d->B)) return CARVE_ERR_SHAPE;
  if (d->B > 65535) return CARVE_ERR_UNSUPPORTED;
  if (!x || !dt || !A || !Bm || !Cm || !state || !y) return CARVE_ERR_NULL;
  st = ssm_aligned(d, x, dt, A, Bm, Cm, D, dt_bias);
  if (st) return st;
  if (!aligned16(state) || !aligned16(y) || ((uintptr_t)slots & 3u)) return CARVE_ERR_ALIGN;
  Range ins[8];
  int nin = ssm_inputs(d, x, dt, A, Bm, Cm, D, dt_bias, ins);
  ins[nin++] = {slots, (size_t)d->B * 4};
  const Range outs[] = {{y, (size_t)d->B * d->T * d->H * d->P * esize(d->dtype)}, {state, (size_t)pool * ssm_state(d)}};
  if (any_overlap(outs, 2, ins, nin)) return CARVE_ERR_UNSUPPORTED;
  SsmStepArgs a = {};
  a.x = x, a.dt = dt, a.Bm = Bm, a.Cm = Cm, a.A = A, a.D = D, a.dt_bias = dt_bias, a.slots = slots, a.state = state, a.y = y;
  a.xs[0] = d->x_batch, a.xs[1] = d->x_token, a.xs[2] = d->x_head;
  a.bs[0] = d->b_batch, a.bs[1] = d->b_token, a.bs[2] = d->b_group;
  a.cs[0] = d->c_batch, a.cs[1] = d->c_token, a.cs[2] = d->c_group;
  a.ds[0] = d->dt_batch, a.ds[1] = d->dt_token;
  a.B = d->B, a.T = d->T, a.G = d->G, a.H = d->H, a.P = d->P, a.pool = pool, a.softplus = d->softplus;
  prof_mark(stream);
  st = launch_ssm_step(a, d->S, d->dtype, stream);
  prof_mark(stream);
  return st;
}

}  // extern "C"
