// ea_api.hip -- the C ABI: argument checks, buffer sizes and the launch
// sequence of the forward (tau solver with the mask's row tables -> sparse
// forward with the column tables) and backward (delta -> dK/dV -> dQ) passes.
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include <mutex>

#include "../../include/entmax_attn.h"
#include "ea_internal.h"

// Scratch of entmax_attn_bwd_noalloc: delta (one fp32 per row) lives here
// instead of in a caller workspace.  Each device holds its own copy for the
// life of the process.  In host code `scratch` only names the symbol: its
// device address comes from hipGetSymbolAddress (scratch_for below), taken
// once per device with that device current, and only that address is passed
// to kernels.
static __device__ __align__(256) float scratch[EA_NOALLOC_MAX_ROWS];

namespace ea {

int gamma_kind(float alpha) {
  if (alpha == 2.0f) return 1;
  if (alpha == 1.5f) return 2;
  if (alpha == 1.25f) return 4;
  return 0;
}

namespace {

constexpr int DEFAULT_MAX_ITER = 12;
constexpr float DEFAULT_TOL = 1e-5f;
constexpr int MAX_ITER_CAP = 64;
// Candidate-cache entries per list (see entmax_attn_sizes); a slot holds
// two lists per row of a workgroup.
constexpr int SOLVE_QUAD_CAP = 96;
static_assert(SOLVE_QUAD_CAP % 8 == 0, "the solver reads lists in batches of 8 quads");
constexpr size_t SOLVE_SLOT_BYTES = solve_slot_bytes(SOLVE_QUAD_CAP);
static_assert(SOLVE_SLOT_BYTES % (2 * SOLVE_THREADS * sizeof(CandEntry) * 8) == 0,
              "a refilled slot holds a multiple of 8 single entries per list");

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct Dims {
  int64_t BH, n, d, T, elems;
  int dtype;
  size_t esize;
};

ea_status check_params(const ea_params* p) {
  if (!std::isfinite(p->alpha) || !(p->alpha > 1.0f)) return EA_ERR_INVALID_ARG;
  if (!std::isfinite(p->scale) || !(p->scale > 0.0f)) return EA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return EA_ERR_INVALID_ARG;
  if (p->need_bwd != 0 && p->need_bwd != 1) return EA_ERR_INVALID_ARG;
  if (p->max_iter < 0 || p->max_iter > MAX_ITER_CAP) return EA_ERR_INVALID_ARG;
  if (!std::isfinite(p->tol) || p->tol < 0.0f) return EA_ERR_INVALID_ARG;
  return EA_OK;
}

ea_status check_shape(const ea_shape* s, const ea_params* p, Dims* out) {
  if (!s || !p) return EA_ERR_INVALID_ARG;
  if (s->batch < 1 || s->heads < 1 || s->seqlen < 1 || s->head_dim < 1) return EA_ERR_INVALID_ARG;
  if (s->dtype != EA_BF16 && s->dtype != EA_F32) return EA_ERR_UNSUPPORTED;
  if (s->head_dim != 64 && s->head_dim != 128) return EA_ERR_UNSUPPORTED;
  if (s->seqlen > MAX_SEQLEN) return EA_ERR_UNSUPPORTED;
  const ea_status st = check_params(p);
  if (st != EA_OK) return st;
  const int64_t BH = (int64_t)s->batch * s->heads;
  const int64_t n = s->seqlen;
  const int64_t T = (n + 63) / 64;
  // grid sizes and in-kernel offsets use 32-bit block counts
  if (BH * ((n + 63) / 64) > (int64_t)INT32_MAX / 2) return EA_ERR_UNSUPPORTED;
  out->BH = BH;
  out->n = n;
  out->d = s->head_dim;
  out->T = T;
  out->elems = BH * n * s->head_dim;
  out->dtype = s->dtype;
  out->esize = s->dtype == EA_BF16 ? 2 : 4;
  return EA_OK;
}

// delta, one fp32 per row
size_t bwd_ws_bytes(const Dims& d) { return (size_t)(d.BH * d.n) * 4; }

// One cache slot per solver tile of 256 rows, at most MAX_SOLVE_SLOTS: two
// co-resident workgroups per CU of a 256-CU MI355X.  With fewer slots than
// tiles the solver runs in launches of one workgroup per slot, so the workspace
// does not grow with B * H * n.  (Sequences that the solver for short ones takes
// use none of it.)
constexpr int64_t MAX_SOLVE_SLOTS = 512;
int64_t solve_tiles(const Dims& d) { return d.BH * ((d.n + SOLVE_ROWS - 1) / SOLVE_ROWS); }
int64_t solve_slots(const Dims& d) {
  return solve_tiles(d) < MAX_SOLVE_SLOTS ? solve_tiles(d) : MAX_SOLVE_SLOTS;
}

void fill_sizes(const Dims& d, ea_sizes* z) {
  z->tau = (size_t)(d.BH * d.n) * 4;
  z->o2 = (size_t)d.elems * 4;
  z->block_mask = (size_t)(d.BH * d.T * d.T);
  z->q_count = (size_t)(d.BH * d.T) * 4;
  z->q_index = (size_t)(d.BH * d.T * d.T) * 4;
  z->k_count = z->q_count;
  z->k_index = z->q_index;
  z->stats = (size_t)(2 * d.BH * d.T) * 4;
  z->ws_fwd = (size_t)solve_slots(d) * SOLVE_SLOT_BYTES;
  z->ws_bwd = bwd_ws_bytes(d);
  z->tau_lo = d.dtype == EA_F32 ? (size_t)(d.BH * d.n) * 4 : 0;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// The parts of one buffer, each 256-byte aligned; `at` sums up its size.
struct Parts {
  char* base;
  size_t at = 0;
  template <typename T>
  T* take(size_t count) {
    char* p = base ? base + at : nullptr;
    at += up256(count * sizeof(T));
    return reinterpret_cast<T*>(p);
  }
};

// Element lists: one ListBlock per query block, then what each serves.
size_t lists_bytes_of(const Dims& d) {
  if (d.n > LIST_MAX_SEQLEN) return 0;
  const size_t blocks = (size_t)(d.BH * d.T);
  return up256(blocks * sizeof(ListBlock)) + blocks * 4;
}
int32_t* lists_use(const Dims& d, void* lists) {
  return lists ? reinterpret_cast<int32_t*>(static_cast<char*>(lists) +
                                            up256((size_t)(d.BH * d.T) * sizeof(ListBlock)))
               : nullptr;
}

// A backward's workspace with element lists: delta, then the buckets that it
// sorts the lists into, each part 256-byte aligned.  Returns its size (that of
// delta alone where there are no lists); fills *b, if given, from `ws`.
size_t bwd_lists_ws(const Dims& d, char* ws, Buckets* b) {
  if (d.n > LIST_MAX_SEQLEN) return bwd_ws_bytes(d);
  const size_t blocks = (size_t)(d.BH * d.T);
  size_t at = up256(bwd_ws_bytes(d));
  auto part = [&](size_t bytes) {
    char* p = ws ? ws + at : nullptr;
    at += up256(bytes);
    return p;
  };
  Buckets t;
  t.used = reinterpret_cast<int32_t*>(part(blocks * 4));
  t.heads = reinterpret_cast<int32_t*>(part((size_t)d.BH * 4));
  t.off = reinterpret_cast<uint16_t*>(part(blocks * (size_t)(d.T + 1) * 2));
  t.z = reinterpret_cast<float*>(part(blocks * LIST_ENTRIES * 4));
  t.code = reinterpret_cast<uint16_t*>(part(blocks * LIST_ENTRIES * 2));
  if (b) *b = t;
  return at;
}

bool tensor_ok(const void* p) { return p && aligned(p, 16); }
bool small_ok(const void* p) { return p && aligned(p, 4); }

ea_status check_tables(const ea_residuals* r, const Dims& d) {
  if (!r) return EA_ERR_INVALID_ARG;
  if (!small_ok(r->tau) || !r->block_mask || !small_ok(r->q_count) || !small_ok(r->q_index) ||
      !small_ok(r->k_count) || !small_ok(r->k_index))
    return EA_ERR_INVALID_ARG;
  if (r->stats && !aligned(r->stats, 4)) return EA_ERR_INVALID_ARG;
  if (d.dtype == EA_F32 && !small_ok(r->tau_lo)) return EA_ERR_INVALID_ARG;
  return EA_OK;
}

// fp64 parameters of the fp32 inputs' refinement, from the fp32 values given
double c64_of(const ea_params* p) { return ((double)p->alpha - 1.0) * (double)p->scale; }
double g64_of(const ea_params* p) { return 1.0 / ((double)p->alpha - 1.0); }
const float* tau_lo_of(const ea_residuals* r, const Dims& d) {
  return d.dtype == EA_F32 ? r->tau_lo : nullptr;
}

// HIP error behind the calling thread's most recent EA_ERR_HIP.
thread_local hipError_t last_hip_error = hipSuccess;

// Checks shared by the row-wise entry points; fills the kernel arguments.
ea_status prep_rows(int64_t rows, int32_t n, ea_dtype dtype, const ea_params* params,
                    const void* s, RowsArgs* ra) {
  if (!params) return EA_ERR_INVALID_ARG;
  ea_status st = check_params(params);
  if (st != EA_OK) return st;
  if (rows < 1 || n < 1) return EA_ERR_INVALID_ARG;
  if (dtype != EA_BF16 && dtype != EA_F32) return EA_ERR_UNSUPPORTED;
  if (n > MAX_ROW_LEN || rows > (int64_t)INT32_MAX) return EA_ERR_UNSUPPORTED;
  if (!tensor_ok(s)) return EA_ERR_INVALID_ARG;
  *ra = RowsArgs{};
  ra->s = s;
  ra->rows = rows;
  ra->n = n;
  ra->alpha = params->alpha;
  ra->gamma = 1.0f / (params->alpha - 1.0f);
  ra->scale = params->scale;
  ra->c = (params->alpha - 1.0f) * params->scale;
  ra->tol = params->tol;
  ra->max_iter = params->max_iter;
  ra->gk = gamma_kind(params->alpha);
  return EA_OK;
}

ea_status from_hip(hipError_t e) {
  if (e == hipSuccess) return EA_OK;
  last_hip_error = e;
  return EA_ERR_HIP;
}

constexpr int MAX_DEVICES = 64;
std::mutex scratch_mutex;
float* scratch_ptr[MAX_DEVICES] = {};

// Device address of `scratch` on the device that `stream` belongs to (the
// current device for the null stream); null on failure with *err set.
float* scratch_for(hipStream_t stream, hipError_t* err) {
  int dev = 0;
  *err = stream ? hipStreamGetDevice(stream, &dev) : hipGetDevice(&dev);
  if (*err != hipSuccess) return nullptr;
  if (dev < 0 || dev >= MAX_DEVICES) {
    *err = hipErrorInvalidDevice;
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(scratch_mutex);
  if (scratch_ptr[dev]) return scratch_ptr[dev];
  int cur = 0;
  if ((*err = hipGetDevice(&cur)) != hipSuccess) return nullptr;
  if (cur != dev && (*err = hipSetDevice(dev)) != hipSuccess) return nullptr;
  void* p = nullptr;
  *err = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
  if (cur != dev) {
    const hipError_t e2 = hipSetDevice(cur);
    if (*err == hipSuccess) *err = e2;
  }
  if (*err != hipSuccess) return nullptr;
  scratch_ptr[dev] = static_cast<float*>(p);
  return scratch_ptr[dev];
}

}  // namespace
}  // namespace ea

using namespace ea;

extern "C" {

void entmax_attn_default_params(ea_params* p) {
  if (!p) return;
  p->alpha = 1.5f;
  p->scale = 0.125f;
  p->causal = 0;
  p->max_iter = DEFAULT_MAX_ITER;
  p->tol = DEFAULT_TOL;
  p->need_bwd = 1;
}

ea_status entmax_attn_sizes(const ea_shape* shape, const ea_params* params, ea_sizes* out) {
  Dims d;
  ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (!out) return EA_ERR_INVALID_ARG;
  fill_sizes(d, out);
  return EA_OK;
}

namespace {

// Checks shared by the forward entry points; fills the kernel arguments.
ea_status prep_fwd(const ea_shape* shape, const ea_params* params, const void* q, const void* k,
                   const void* v, void* o, const ea_residuals* res, const void* workspace,
                   Dims* d) {
  ea_status st = check_shape(shape, params, d);
  if (st != EA_OK) return st;
  if (workspace && !aligned(workspace, 16)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(q) || !tensor_ok(k) || !tensor_ok(v) || !tensor_ok(o)) return EA_ERR_INVALID_ARG;
  if ((st = check_tables(res, *d)) != EA_OK) return st;
  if (params->need_bwd && !tensor_ok(res->o2)) return EA_ERR_INVALID_ARG;
  return EA_OK;
}

ea_status run_fwd_stage(int stage, const Dims& d, const ea_params* params, const void* q,
                        const void* k, const void* v, void* o, const ea_residuals* res,
                        void* workspace, size_t ws_bytes, ListBlock* lists, hipStream_t s) {
  const float c = (params->alpha - 1.0f) * params->scale;
  const float gamma = 1.0f / (params->alpha - 1.0f);
  const int gk = gamma_kind(params->alpha);
  if (stage == 0) {
    // The cache is optional: tiles without a slot (all of them when there is
    // no workspace) stream K on every solver pass.
    int64_t slots = workspace ? (int64_t)(ws_bytes / SOLVE_SLOT_BYTES) : 0;
    const int64_t most = solve_tiles(d);
    if (slots > most) slots = most;
    void* cand = slots > 0 ? workspace : nullptr;
    TauArgs ta{q, k, res->tau, res->block_mask, res->stats, cand,
               SOLVE_QUAD_CAP, (int)slots, /*tile0=*/0,
               (int)d.BH, (int)d.n, (int)d.T, c, params->alpha, gamma, params->causal,
               params->max_iter, params->tol, gk,
               const_cast<float*>(tau_lo_of(res, d)), c64_of(params), g64_of(params),
               res->q_count, res->q_index, lists, lists_use(d, lists)};
    return from_hip(launch_tau(ta, d.dtype, (int)d.d, s));
  }
  FwdArgs fa{q, k, v, o, params->need_bwd ? res->o2 : nullptr, res->tau, res->q_count,
             res->q_index, (int)d.BH, (int)d.n, (int)d.T, c, gamma, params->causal, gk,
             tau_lo_of(res, d), c64_of(params), g64_of(params),
             res->block_mask, res->k_count, res->k_index, lists, lists_use(d, lists)};
  return from_hip(launch_fwd(fa, d.dtype, (int)d.d, params->need_bwd != 0, s));
}

// Checks of the backward's tensors and residuals (not its workspace).
ea_status prep_bwd_args(const ea_shape* shape, const ea_params* params, const void* q,
                        const void* k, const void* v, const void* dout, const ea_residuals* res,
                        const float* dq, const float* dk, const float* dv, Dims* d) {
  ea_status st = check_shape(shape, params, d);
  if (st != EA_OK) return st;
  if (!tensor_ok(q) || !tensor_ok(k) || !tensor_ok(v) || !tensor_ok(dout)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(dq) || !tensor_ok(dk) || !tensor_ok(dv)) return EA_ERR_INVALID_ARG;
  if ((st = check_tables(res, *d)) != EA_OK) return st;
  if (!tensor_ok(res->o2)) return EA_ERR_INVALID_ARG;
  return EA_OK;
}

ea_status prep_bwd(const ea_shape* shape, const ea_params* params, const void* q, const void* k,
                   const void* v, const void* dout, const ea_residuals* res, const float* dq,
                   const float* dk, const float* dv, const void* workspace, size_t ws_bytes,
                   Dims* d) {
  ea_status st = prep_bwd_args(shape, params, q, k, v, dout, res, dq, dk, dv, d);
  if (st != EA_OK) return st;
  if (!workspace || !aligned(workspace, 16)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < bwd_ws_bytes(*d)) return EA_ERR_WORKSPACE;
  return EA_OK;
}

ea_status run_bwd_stage(int stage, const Dims& d, const ea_params* params, const void* q,
                        const void* k, const void* v, const void* dout, const ea_residuals* res,
                        float* dq, float* dk, float* dv, void* workspace, void* lists_buf,
                        hipStream_t s) {
  // (with lists, the workspace has room for their buckets)
  float* delta = static_cast<float*>(workspace);
  const ListBlock* lists = static_cast<const ListBlock*>(lists_buf);
  Buckets buckets{};
  if (lists) bwd_lists_ws(d, static_cast<char*>(workspace), &buckets);
  if (stage == 0) {
    DeltaArgs da{dout, res->o2, delta, d.BH * d.n, lists, lists_use(d, lists_buf), res->tau, buckets,
                 (int)d.BH, (int)d.n, (int)d.T};
    return from_hip(launch_delta(da, d.dtype, (int)d.d, s));
  }
  const float c = (params->alpha - 1.0f) * params->scale;
  const float gamma = 1.0f / (params->alpha - 1.0f);
  BwdArgs ba{q, k, v, dout, res->tau, delta, res->q_count, res->q_index, res->k_count,
             res->k_index, dq, dk, dv, (int)d.BH, (int)d.n, (int)d.T, c, gamma,
             params->scale, params->causal, gamma_kind(params->alpha), tau_lo_of(res, d),
             c64_of(params), g64_of(params), lists, buckets};
  if (stage == 1) {
    const ea_status st = from_hip(launch_bwd_dkdv(ba, d.dtype, (int)d.d, s));
    if (st != EA_OK || !lists) return st;
    return from_hip(launch_bwd_dkdv_lists(ba, d.dtype, (int)d.d, s));
  }
  return from_hip(launch_bwd_dq(ba, d.dtype, (int)d.d, s));
}

}  // namespace

ea_status entmax_attn_fwd(const ea_shape* shape, const ea_params* params, const void* q,
                          const void* k, const void* v, void* o, const ea_residuals* res,
                          void* workspace, size_t ws_bytes, void* stream) {
  Dims d;
  ea_status st = prep_fwd(shape, params, q, k, v, o, res, workspace, &d);
  if (st != EA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int stage = 0; stage < 2; ++stage)
    if ((st = run_fwd_stage(stage, d, params, q, k, v, o, res, workspace, ws_bytes, nullptr, s)) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_fwd_stage(int stage, const ea_shape* shape, const ea_params* params,
                                const void* q, const void* k, const void* v, void* o,
                                const ea_residuals* res, void* workspace, size_t ws_bytes,
                                void* stream) {
  if (stage < 0 || stage > 1) return EA_ERR_INVALID_ARG;
  Dims d;
  ea_status st = prep_fwd(shape, params, q, k, v, o, res, workspace, &d);
  if (st != EA_OK) return st;
  return run_fwd_stage(stage, d, params, q, k, v, o, res, workspace, ws_bytes, nullptr,
                       static_cast<hipStream_t>(stream));
}

ea_status entmax_attn_bwd(const ea_shape* shape, const ea_params* params, const void* q,
                          const void* k, const void* v, const void* dout,
                          const ea_residuals* res, float* dq, float* dk, float* dv,
                          void* workspace, size_t ws_bytes, void* stream) {
  Dims d;
  ea_status st = prep_bwd(shape, params, q, k, v, dout, res, dq, dk, dv, workspace, ws_bytes, &d);
  if (st != EA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int stage = 0; stage < 3; ++stage)
    if ((st = run_bwd_stage(stage, d, params, q, k, v, dout, res, dq, dk, dv, workspace, nullptr, s)) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_bwd_stage(int stage, const ea_shape* shape, const ea_params* params,
                                const void* q, const void* k, const void* v, const void* dout,
                                const ea_residuals* res, float* dq, float* dk, float* dv,
                                void* workspace, size_t ws_bytes, void* stream) {
  if (stage < 0 || stage > 2) return EA_ERR_INVALID_ARG;
  Dims d;
  ea_status st = prep_bwd(shape, params, q, k, v, dout, res, dq, dk, dv, workspace, ws_bytes, &d);
  if (st != EA_OK) return st;
  return run_bwd_stage(stage, d, params, q, k, v, dout, res, dq, dk, dv, workspace, nullptr,
                       static_cast<hipStream_t>(stream));
}

ea_status entmax_attn_lists_bytes(const ea_shape* shape, const ea_params* params, size_t* bytes) {
  Dims d;
  const ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  *bytes = lists_bytes_of(d);
  return EA_OK;
}

ea_status entmax_attn_bwd_lists_workspace(const ea_shape* shape, const ea_params* params, size_t* bytes) {
  Dims d;
  const ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  *bytes = bwd_lists_ws(d, nullptr, nullptr);
  return EA_OK;
}

namespace {

// Checks of a lists buffer (null: no lists).
ea_status check_lists(const Dims& d, const void* lists, size_t lists_bytes) {
  if (!lists) return EA_OK;
  const size_t need = lists_bytes_of(d);
  if (need == 0) return EA_ERR_UNSUPPORTED;
  if (!aligned(lists, 16)) return EA_ERR_INVALID_ARG;
  return lists_bytes < need ? EA_ERR_WORKSPACE : EA_OK;
}

// The stages of one call: all of them, or one.
int first_stage(int stage) { return stage == EA_ALL_STAGES ? 0 : stage; }
int last_stage(int stage, int last) { return stage == EA_ALL_STAGES ? last : stage; }

}  // namespace

ea_status entmax_attn_fwd_lists(int stage, const ea_shape* shape, const ea_params* params, const void* q,
                                const void* k, const void* v, void* o, const ea_residuals* res,
                                void* lists, size_t lists_bytes, void* workspace, size_t ws_bytes,
                                void* stream) {
  if (stage < EA_ALL_STAGES || stage > 1) return EA_ERR_INVALID_ARG;
  Dims d;
  ea_status st = prep_fwd(shape, params, q, k, v, o, res, workspace, &d);
  if (st != EA_OK || (st = check_lists(d, lists, lists_bytes)) != EA_OK) return st;
  for (int x = first_stage(stage); x <= last_stage(stage, 1); ++x)
    if ((st = run_fwd_stage(x, d, params, q, k, v, o, res, workspace, ws_bytes,
                            static_cast<ListBlock*>(lists), static_cast<hipStream_t>(stream))) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_bwd_lists(int stage, const ea_shape* shape, const ea_params* params, const void* q,
                                const void* k, const void* v, const void* dout, const ea_residuals* res,
                                void* lists, size_t lists_bytes, float* dq, float* dk, float* dv,
                                void* workspace, size_t ws_bytes, void* stream) {
  if (stage < EA_ALL_STAGES || stage > 2) return EA_ERR_INVALID_ARG;
  Dims d;
  ea_status st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (workspace || stage != EA_ALL_STAGES) {
    st = prep_bwd(shape, params, q, k, v, dout, res, dq, dk, dv, workspace, ws_bytes, &d);
    if (st != EA_OK || (st = check_lists(d, lists, lists_bytes)) != EA_OK) return st;
  } else {  // delta in the library's scratch, as in entmax_attn_bwd_noalloc
    if ((st = check_shape(shape, params, &d)) != EA_OK) return st;
    if (d.BH * d.n > (int64_t)EA_NOALLOC_MAX_ROWS) return EA_ERR_UNSUPPORTED;
    if ((st = prep_bwd_args(shape, params, q, k, v, dout, res, dq, dk, dv, &d)) != EA_OK) return st;
    if ((st = check_lists(d, lists, lists_bytes)) != EA_OK) return st;
    hipError_t e = hipSuccess;
    workspace = scratch_for(s, &e);
    if (!workspace) return from_hip(e);
    ws_bytes = 0;
  }
  if (ws_bytes < bwd_lists_ws(d, nullptr, nullptr)) lists = nullptr;  // no room to sort them
  for (int x = first_stage(stage); x <= last_stage(stage, 2); ++x)
    if ((st = run_bwd_stage(x, d, params, q, k, v, dout, res, dq, dk, dv, workspace, lists, s)) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_bwd_noalloc(const ea_shape* shape, const ea_params* params, const void* q,
                                  const void* k, const void* v, const void* dout,
                                  const ea_residuals* res, float* dq, float* dk, float* dv,
                                  void* stream) {
  Dims d;
  ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (d.BH * d.n > (int64_t)EA_NOALLOC_MAX_ROWS) return EA_ERR_UNSUPPORTED;
  if ((st = prep_bwd_args(shape, params, q, k, v, dout, res, dq, dk, dv, &d)) != EA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  float* delta = scratch_for(s, &e);
  if (!delta) return from_hip(e);
  for (int stage = 0; stage < 3; ++stage)
    if ((st = run_bwd_stage(stage, d, params, q, k, v, dout, res, dq, dk, dv, delta, nullptr, s)) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_rows_fwd(int64_t rows, int32_t n, ea_dtype dtype, const ea_params* params,
                          const void* s, float* p, float* tau, void* stream) {
  RowsArgs ra;
  ea_status st = prep_rows(rows, n, dtype, params, s, &ra);
  if (st != EA_OK) return st;
  if (!tensor_ok(p) || !tensor_ok(tau)) return EA_ERR_INVALID_ARG;
  ra.p = p;
  ra.tau = tau;
  return from_hip(launch_rows_fwd(ra, dtype, static_cast<hipStream_t>(stream)));
}

ea_status entmax_rows_bwd(int64_t rows, int32_t n, ea_dtype dtype, const ea_params* params,
                          const void* s, const float* tau, const float* dp, float* ds,
                          void* stream) {
  RowsArgs ra;
  ea_status st = prep_rows(rows, n, dtype, params, s, &ra);
  if (st != EA_OK) return st;
  if (!tensor_ok(tau) || !tensor_ok(dp) || !tensor_ok(ds)) return EA_ERR_INVALID_ARG;
  ra.tau = const_cast<float*>(tau);  // read only by the backward kernel
  ra.dp = dp;
  ra.ds = ds;
  return from_hip(launch_rows_bwd(ra, dtype, static_cast<hipStream_t>(stream)));
}

// The no-mask mode: the same stages without a mask or tables.
ea_status entmax_attn_fwd_dense_lists(const ea_shape* shape, const ea_params* params, const void* q,
                                      const void* k, const void* v, void* o, float* tau, float* tau_lo,
                                      float* o2, void* lists, size_t lists_bytes, void* workspace,
                                      size_t ws_bytes, void* stream) {
  Dims d;
  ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (!tensor_ok(q) || !tensor_ok(k) || !tensor_ok(v) || !tensor_ok(o)) return EA_ERR_INVALID_ARG;
  if (!small_ok(tau)) return EA_ERR_INVALID_ARG;
  if (d.dtype == EA_F32 && !small_ok(tau_lo)) return EA_ERR_INVALID_ARG;
  if (params->need_bwd && !tensor_ok(o2)) return EA_ERR_INVALID_ARG;
  if (workspace && !aligned(workspace, 16)) return EA_ERR_INVALID_ARG;
  if ((st = check_lists(d, lists, lists_bytes)) != EA_OK) return st;
  ea_residuals res{};
  res.tau = tau;
  res.tau_lo = tau_lo;
  res.o2 = o2;
  for (int stage = 0; stage < 2; ++stage)
    if ((st = run_fwd_stage(stage, d, params, q, k, v, o, &res, workspace, ws_bytes,
                            static_cast<ListBlock*>(lists), static_cast<hipStream_t>(stream))) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_fwd_dense(const ea_shape* shape, const ea_params* params, const void* q,
                                const void* k, const void* v, void* o, float* tau, float* tau_lo,
                                float* o2, void* workspace, size_t ws_bytes, void* stream) {
  return entmax_attn_fwd_dense_lists(shape, params, q, k, v, o, tau, tau_lo, o2, nullptr, 0, workspace,
                                     ws_bytes, stream);
}

ea_status entmax_attn_bwd_dense_lists(const ea_shape* shape, const ea_params* params, const void* q,
                                      const void* k, const void* v, const void* dout, const float* tau,
                                      const float* tau_lo, const float* o2, void* lists, size_t lists_bytes,
                                      float* dq, float* dk, float* dv, void* workspace, size_t ws_bytes,
                                      void* stream) {
  Dims d;
  ea_status st = check_shape(shape, params, &d);
  if (st != EA_OK) return st;
  if (!tensor_ok(q) || !tensor_ok(k) || !tensor_ok(v) || !tensor_ok(dout)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(dq) || !tensor_ok(dk) || !tensor_ok(dv)) return EA_ERR_INVALID_ARG;
  if (!small_ok(tau) || !tensor_ok(o2)) return EA_ERR_INVALID_ARG;
  if (d.dtype == EA_F32 && !small_ok(tau_lo)) return EA_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 16)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < bwd_ws_bytes(d)) return EA_ERR_WORKSPACE;
  if ((st = check_lists(d, lists, lists_bytes)) != EA_OK) return st;
  if (ws_bytes < bwd_lists_ws(d, nullptr, nullptr)) lists = nullptr;  // no room to sort them
  // no tables: the kernels visit every valid block that has no lists
  ea_residuals res{};
  res.tau = const_cast<float*>(tau);
  res.tau_lo = const_cast<float*>(tau_lo);
  res.o2 = const_cast<float*>(o2);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (lists) {
    Buckets buckets{};
    bwd_lists_ws(d, static_cast<char*>(workspace), &buckets);
    CollectArgs ca{q, k, tau, tau_lo_of(&res, d), static_cast<ListBlock*>(lists), lists_use(d, lists),
                   buckets.used /* (written after this) */, (int)d.BH, (int)d.n, (int)d.T, (params->alpha - 1.0f) * params->scale, params->causal,
                   gamma_kind(params->alpha), c64_of(params)};
    if ((st = from_hip(launch_collect(ca, d.dtype, (int)d.d, s))) != EA_OK) return st;
  }
  for (int stage = 0; stage < 3; ++stage)
    if ((st = run_bwd_stage(stage, d, params, q, k, v, dout, &res, dq, dk, dv, workspace, lists, s)) != EA_OK)
      return st;
  return EA_OK;
}

ea_status entmax_attn_bwd_dense(const ea_shape* shape, const ea_params* params, const void* q,
                                const void* k, const void* v, const void* dout, const float* tau,
                                const float* tau_lo, const float* o2, float* dq, float* dk,
                                float* dv, void* workspace, size_t ws_bytes, void* stream) {
  return entmax_attn_bwd_dense_lists(shape, params, q, k, v, dout, tau, tau_lo, o2, nullptr, 0, dq, dk, dv,
                                     workspace, ws_bytes, stream);
}

// ------------------------------------------------ norm and rotation

namespace {

constexpr int64_t MAX_STRIDE = (int64_t)1 << 40;
// Strides of rows of `esize`-byte elements that start at multiples of 16 bytes.
bool strides_ok(const ea_strides* s, size_t esize) {
  const int64_t vec = 16 / (int64_t)esize;
  return s && s->row >= 0 && s->head >= 0 && s->row % vec == 0 && s->head % vec == 0 && s->row <= MAX_STRIDE &&
         s->head <= MAX_STRIDE;
}

bool dtype_ok(int32_t t) { return t == EA_BF16 || t == EA_F32; }
size_t size_of(int32_t t) { return t == EA_BF16 ? 2 : 4; }

ea_status check_rotary(const ea_rotary* r) {
  if (!r) return EA_ERR_INVALID_ARG;
  if (r->tokens < 0 || r->heads < 1 || r->kv_heads < 1) return EA_ERR_INVALID_ARG;
  if (!dtype_ok(r->dtype) || (r->head_dim != 64 && r->head_dim != 128)) return EA_ERR_UNSUPPORTED;
  if (r->weight_dtype != r->dtype && r->weight_dtype != EA_F32) return EA_ERR_UNSUPPORTED;
  if (r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 16 != 0) return EA_ERR_INVALID_ARG;
  if (r->interleaved != 0 && r->interleaved != 1) return EA_ERR_INVALID_ARG;
  if (!std::isfinite(r->eps) || r->eps < 0.0f) return EA_ERR_INVALID_ARG;
  if (r->axes < 1 || r->axes > ROT_MAX_AXES) return EA_ERR_INVALID_ARG;
  int64_t pairs = 0;
  for (int a = 0; a < r->axes; ++a) {
    if (r->sections[a] < 0) return EA_ERR_INVALID_ARG;
    pairs += r->sections[a];
  }
  if (2 * pairs != r->rot_dim) return EA_ERR_INVALID_ARG;
  // a launch has fewer than 2^32 threads, 64 of them to a token
  if ((int64_t)r->heads + r->kv_heads > (1 << 20) || r->tokens > (1 << 25)) return EA_ERR_UNSUPPORTED;
  return EA_OK;
}

ea_status prep_rotary(const ea_rotary* r, const void* q, const ea_strides* qs, const void* k, const ea_strides* ks,
                      const int32_t* positions, int64_t position_stride, const float* freqs, const void* q_weight,
                      const void* k_weight, RotaryArgs* out) {
  const size_t es = size_of(r->dtype);
  if (!tensor_ok(q) || !tensor_ok(k) || !strides_ok(qs, es) || !strides_ok(ks, es)) return EA_ERR_INVALID_ARG;
  if (r->rot_dim && (!small_ok(positions) || !small_ok(freqs))) return EA_ERR_INVALID_ARG;
  if (position_stride < 0) return EA_ERR_INVALID_ARG;
  if ((q_weight && !tensor_ok(q_weight)) || (k_weight && !tensor_ok(k_weight))) return EA_ERR_INVALID_ARG;
  RotaryArgs a{};
  a.q = {const_cast<void*>(q), qs->row, qs->head};
  a.k = {const_cast<void*>(k), ks->row, ks->head};
  a.positions = positions;
  a.position_stride = position_stride;
  a.freqs = freqs;
  int end = 0;
  for (int x = 0; x < r->axes; ++x) a.axis_end[x] = end += r->sections[x];
  a.axes = r->axes;
  a.tokens = r->tokens;
  a.hq = r->heads;
  a.hk = r->kv_heads;
  a.d = r->head_dim;
  a.rot = r->rot_dim;
  a.interleaved = r->interleaved;
  a.eps = r->eps;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.weight_f32 = r->weight_dtype == EA_F32;
  *out = a;
  return EA_OK;
}

size_t rotary_ws(const ea_rotary* r) { return (size_t)rotary_partials(r->tokens) * 2 * r->head_dim * 4; }

}  // namespace

ea_status entmax_norm_rotary(const ea_rotary* r, const void* q, const ea_strides* q_strides, const void* k,
                             const ea_strides* k_strides, const int32_t* positions, int64_t position_stride,
                             const float* freqs, const void* q_weight, const void* k_weight, void* q_out,
                             const ea_strides* q_out_strides, void* k_out, const ea_strides* k_out_strides,
                             void* stream) {
  ea_status st = check_rotary(r);
  if (st != EA_OK || r->tokens == 0) return st;
  RotaryArgs a;
  st = prep_rotary(r, q, q_strides, k, k_strides, positions, position_stride, freqs, q_weight, k_weight, &a);
  if (st != EA_OK) return st;
  const size_t es = size_of(r->dtype);
  if (!tensor_ok(q_out) || !tensor_ok(k_out) || !strides_ok(q_out_strides, es) || !strides_ok(k_out_strides, es))
    return EA_ERR_INVALID_ARG;
  a.q_out = {q_out, q_out_strides->row, q_out_strides->head};
  a.k_out = {k_out, k_out_strides->row, k_out_strides->head};
  return from_hip(launch_rotary_fwd(a, r->dtype, static_cast<hipStream_t>(stream)));
}

ea_status entmax_norm_rotary_workspace(const ea_rotary* r, size_t* bytes) {
  const ea_status st = check_rotary(r);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  *bytes = rotary_ws(r);
  return EA_OK;
}

ea_status entmax_norm_rotary_bwd(const ea_rotary* r, const void* dq_out, const ea_strides* dq_out_strides,
                                 const void* dk_out, const ea_strides* dk_out_strides, const void* q,
                                 const ea_strides* q_strides, const void* k, const ea_strides* k_strides,
                                 const int32_t* positions, int64_t position_stride, const float* freqs,
                                 const void* q_weight, const void* k_weight, void* dq, void* dk,
                                 float* dq_weight, float* dk_weight, void* workspace, size_t ws_bytes,
                                 void* stream) {
  ea_status st = check_rotary(r);
  if (st != EA_OK) return st;
  if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return EA_ERR_INVALID_ARG;
  RotaryArgs a{};
  if (r->tokens == 0) {  // (the sums of no terms)
    a.d = r->head_dim;
    a.dq_weight = dq_weight;
    a.dk_weight = dk_weight;
    return from_hip(launch_rotary_bwd(a, r->dtype, static_cast<hipStream_t>(stream)));
  }
  st = prep_rotary(r, q, q_strides, k, k_strides, positions, position_stride, freqs, q_weight, k_weight, &a);
  if (st != EA_OK) return st;
  const size_t es = size_of(r->dtype);
  if (!tensor_ok(dq_out) || !tensor_ok(dk_out) || !strides_ok(dq_out_strides, es) || !strides_ok(dk_out_strides, es))
    return EA_ERR_INVALID_ARG;
  if (!tensor_ok(dq) || !tensor_ok(dk)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(workspace)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < rotary_ws(r)) return EA_ERR_WORKSPACE;
  const int64_t d = r->head_dim;
  a.dq = {const_cast<void*>(dq_out), dq_out_strides->row, dq_out_strides->head};
  a.dk = {const_cast<void*>(dk_out), dk_out_strides->row, dk_out_strides->head};
  a.q_out = {dq, r->heads * d, d};
  a.k_out = {dk, r->kv_heads * d, d};
  a.partials = static_cast<float*>(workspace);
  a.partial_count = rotary_partials(r->tokens);
  a.dq_weight = dq_weight;
  a.dk_weight = dk_weight;
  return from_hip(launch_rotary_bwd(a, r->dtype, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------ packed sequences

namespace {

ea_status check_plan(int32_t tokens, int32_t seqs) {
  if (tokens < 1 || seqs < 1) return EA_ERR_INVALID_ARG;
  if (seqs > MAX_SEQS) return EA_ERR_UNSUPPORTED;
  // tiles and rows are 32-bit numbers
  return (int64_t)tokens / 64 + seqs > (1 << 26) ? EA_ERR_UNSUPPORTED : EA_OK;
}

size_t plan_parts(int32_t tokens, int32_t seqs, void* base, PlanArgs* a) {
  Parts p{static_cast<char*>(base)};
  a->header = p.take<PackedHeader>(1);
  a->seqs = p.take<PackedSeq>((size_t)seqs);
  for (int z = 0; z < 2; ++z) a->tiles[z] = p.take<PackedTile>((size_t)packed_tiles(tokens, seqs, z));
  return p.at;
}

struct PackedResiduals {
  float *tau, *tau_lo, *o2;
  int32_t *q_count, *q_index, *k_count, *k_index;
  uint8_t* mask;
};

size_t residual_parts(const ea_packed_shape* s, const ea_params* p, void* base, PackedResiduals* r) {
  const size_t rows = (size_t)s->heads * s->tokens, width = ((size_t)s->max_seqlen + 63) / 64;
  const size_t blocks = (size_t)s->heads * packed_tiles(s->tokens, s->seqs, 0);
  Parts x{static_cast<char*>(base)};
  r->tau = x.take<float>(rows);
  r->tau_lo = x.take<float>(s->dtype == EA_F32 ? rows : 0);
  r->q_count = x.take<int32_t>(blocks);
  r->q_index = x.take<int32_t>(blocks * width);
  r->mask = x.take<uint8_t>(blocks * width);
  r->o2 = x.take<float>(p->need_bwd ? rows * s->head_dim : 0);
  r->k_count = x.take<int32_t>(p->need_bwd ? blocks : 0);
  r->k_index = x.take<int32_t>(p->need_bwd ? blocks * width : 0);
  return x.at;
}

ea_status check_packed(const ea_packed_shape* s, const ea_params* p) {
  if (!s || !p) return EA_ERR_INVALID_ARG;
  ea_status st = check_plan(s->tokens, s->seqs);
  if (st != EA_OK) return st;
  if (s->max_seqlen < 1 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads != 0) return EA_ERR_INVALID_ARG;
  if (!dtype_ok(s->dtype) || (s->head_dim != 64 && s->head_dim != 128)) return EA_ERR_UNSUPPORTED;
  if (s->max_seqlen > MAX_SEQLEN) return EA_ERR_UNSUPPORTED;
  if ((st = check_params(p)) != EA_OK) return st;
  // a launch has fewer than 2^32 threads: up to 512 to a tile, 16 to a row
  if ((int64_t)s->heads * packed_tiles(s->tokens, s->seqs, 0) >= (1 << 22)) return EA_ERR_UNSUPPORTED;
  return EA_OK;
}

size_t packed_lists_bytes(const ea_packed_shape* s) {
  if (s->max_seqlen > LIST_MAX_SEQLEN) return 0;
  const size_t blocks = (size_t)s->heads * packed_tiles(s->tokens, s->seqs, 0);
  return up256(blocks * sizeof(ListBlock)) + blocks * 4;
}
int32_t* packed_lists_use(const ea_packed_shape* s, const void* lists) {
  const size_t blocks = (size_t)s->heads * packed_tiles(s->tokens, s->seqs, 0);
  return reinterpret_cast<int32_t*>(static_cast<char*>(const_cast<void*>(lists)) + up256(blocks * sizeof(ListBlock)));
}
ea_status check_packed_lists(const ea_packed_shape* s, const void* lists, size_t bytes) {
  if (!lists) return EA_OK;
  const size_t need = packed_lists_bytes(s);
  if (need == 0) return EA_ERR_UNSUPPORTED;
  if (!aligned(lists, 16)) return EA_ERR_INVALID_ARG;
  return bytes < need ? EA_ERR_WORKSPACE : EA_OK;
}

int packed_parts(const ea_packed_shape* s) {
  return dkdv_packed_parts(s->tokens, s->seqs, s->heads, s->kv_heads, s->dtype, s->head_dim);
}

// The solver's workgroups of 128 rows use half a slot each, and no more of them
// run at a time than packed_solvers().
int64_t packed_slots(const ea_packed_shape* s, const ea_params* p) {
  const int64_t tiles = (int64_t)s->heads * packed_tiles(s->tokens, s->seqs, 1);
  const int64_t most = packed_solvers(s->dtype == EA_F32, s->head_dim, gamma_kind(p->alpha));
  return ((tiles < most ? tiles : most) + 1) / 2;
}
// The backward's workspace: delta, the parts of dK and dV where there are some
// (with element lists always, and one more), and with lists their buckets.
struct PackedBwdWs {
  float *delta, *dk, *dv;
  int32_t* wrote;
  Buckets buckets;
};
size_t packed_ws_bwd(const ea_packed_shape* s, bool lists, void* base, PackedBwdWs* w) {
  const int parts = packed_parts(s);
  const size_t blocks = (size_t)s->heads * packed_tiles(s->tokens, s->seqs, 0);
  const size_t sums = (size_t)(lists ? parts + 1 : parts > 1 ? parts : 0) * s->tokens * s->kv_heads * s->head_dim;
  Parts p{static_cast<char*>(base)};
  w->delta = p.take<float>((size_t)s->heads * s->tokens);
  w->dk = p.take<float>(sums);
  w->dv = p.take<float>(sums);
  if (!lists) return p.at;
  w->wrote = p.take<int32_t>((size_t)parts * blocks / s->heads * s->kv_heads);
  w->buckets.used = p.take<int32_t>(blocks);
  w->buckets.heads = p.take<int32_t>((size_t)s->heads * s->seqs);
  w->buckets.off = p.take<uint16_t>(blocks * (((size_t)s->max_seqlen + 63) / 64 + 1));
  w->buckets.z = p.take<float>(blocks * LIST_ENTRIES);
  w->buckets.code = p.take<uint16_t>(blocks * LIST_ENTRIES);
  return p.at;
}

// A tile copy's offsets are 32-bit numbers of elements.
bool packed_strides_ok(const ea_packed_strides* st, size_t es) {
  if (!st) return false;
  for (const ea_strides* s : {&st->q, &st->k, &st->v, &st->o})
    if (!strides_ok(s, es) || s->row > (1 << 24)) return false;
  return true;
}

PackedArgs packed_args(const ea_packed_shape* s, const void* plan, const ea_packed_strides* st, int32_t zero_rest) {
  PlanArgs parts{};
  plan_parts(s->tokens, s->seqs, const_cast<void*>(plan), &parts);
  PackedArgs a{};
  a.header = parts.header;
  a.seqs = parts.seqs;
  for (int z = 0; z < 2; ++z) a.lists[z] = parts.tiles[z];
  a.seq_count = s->seqs;
  a.heads = s->heads;
  a.kv_heads = s->kv_heads;
  a.group = s->heads / s->kv_heads;
  a.tokens = s->tokens;
  a.blocks = packed_tiles(s->tokens, s->seqs, 0);
  a.width = (s->max_seqlen + 63) / 64;
  auto strides = [](const ea_strides& x) { return Strides{(int)x.row, x.head}; };
  a.q = strides(st->q);
  a.k = strides(st->k);
  a.v = strides(st->v);
  a.o = strides(st->o);
  a.zero_rest = zero_rest;
  a.parts = 1;
  return a;
}

// Checks shared by the two passes.
ea_status prep_packed(const ea_packed_shape* shape, const ea_params* params, const void* plan, const void* q,
                      const void* k, const void* v, const void* o, const ea_packed_strides* strides,
                      const void* residuals, size_t residual_bytes, PackedResiduals* r) {
  const ea_status st = check_packed(shape, params);
  if (st != EA_OK) return st;
  if (!tensor_ok(plan) || !tensor_ok(q) || !tensor_ok(k) || !tensor_ok(v) || !tensor_ok(o) || !tensor_ok(residuals))
    return EA_ERR_INVALID_ARG;
  if (!packed_strides_ok(strides, size_of(shape->dtype))) return EA_ERR_INVALID_ARG;
  return residual_bytes < residual_parts(shape, params, const_cast<void*>(residuals), r) ? EA_ERR_WORKSPACE : EA_OK;
}

}  // namespace

ea_status entmax_packed_plan_bytes(int32_t tokens, int32_t seqs, size_t* bytes) {
  const ea_status st = check_plan(tokens, seqs);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  PlanArgs a{};
  *bytes = plan_parts(tokens, seqs, nullptr, &a);
  return EA_OK;
}

ea_status entmax_packed_plan(int32_t tokens, int32_t seqs, int32_t max_seqlen, int32_t causal, const int32_t* cu,
                             void* plan, size_t plan_bytes, void* stream) {
  const ea_status st = check_plan(tokens, seqs);
  if (st != EA_OK) return st;
  if (max_seqlen < 1 || (causal != 0 && causal != 1)) return EA_ERR_INVALID_ARG;
  if (max_seqlen > MAX_SEQLEN) return EA_ERR_UNSUPPORTED;
  if (!small_ok(cu) || !tensor_ok(plan)) return EA_ERR_INVALID_ARG;
  PlanArgs a{};
  if (plan_bytes < plan_parts(tokens, seqs, plan, &a)) return EA_ERR_WORKSPACE;
  a.cu = cu;
  a.seq_count = seqs;
  a.tokens = tokens;
  a.max_seqlen = max_seqlen;
  a.causal = causal;
  return from_hip(launch_plan(a, static_cast<hipStream_t>(stream)));
}

ea_status entmax_packed_sizes(const ea_packed_shape* shape, const ea_params* params, ea_packed_sizes* out) {
  const ea_status st = check_packed(shape, params);
  if (st != EA_OK) return st;
  if (!out) return EA_ERR_INVALID_ARG;
  PackedResiduals r;
  out->residuals = residual_parts(shape, params, nullptr, &r);
  out->ws_fwd = (size_t)packed_slots(shape, params) * SOLVE_SLOT_BYTES;
  out->lists = packed_lists_bytes(shape);
  PackedBwdWs w;
  out->ws_bwd = packed_ws_bwd(shape, false, nullptr, &w);
  out->ws_bwd_lists = out->lists ? packed_ws_bwd(shape, true, nullptr, &w) : out->ws_bwd;
  return EA_OK;
}

ea_status entmax_packed_fwd(const ea_packed_shape* shape, const ea_params* params, const void* plan, const void* q,
                            const void* k, const void* v, void* o, const ea_packed_strides* strides,
                            int32_t zero_rest, void* residuals, size_t residual_bytes, void* lists,
                            size_t lists_bytes, void* workspace, size_t ws_bytes, void* stream) {
  PackedResiduals r;
  ea_status st = prep_packed(shape, params, plan, q, k, v, o, strides, residuals, residual_bytes, &r);
  if (st != EA_OK) return st;
  if (workspace && !aligned(workspace, 16)) return EA_ERR_INVALID_ARG;
  if ((st = check_packed_lists(shape, lists, lists_bytes)) != EA_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const PackedArgs pk = packed_args(shape, plan, strides, zero_rest);
  const int64_t most = packed_slots(shape, params);
  int64_t slots = workspace ? (int64_t)(ws_bytes / SOLVE_SLOT_BYTES) : 0;
  if (slots > most) slots = most;
  Packed<TauArgs> ta{};
  ta.pk = pk;
  ta.q = q;
  ta.k = k;
  ta.tau = r.tau;
  ta.tau_lo = r.tau_lo;
  ta.mask = r.mask;
  ta.q_count = r.q_count;
  ta.q_index = r.q_index;
  ta.cand = slots > 0 ? workspace : nullptr;
  ta.cap = SOLVE_QUAD_CAP;
  ta.slots = (int)slots;
  ta.c = (params->alpha - 1.0f) * params->scale;
  ta.alpha = params->alpha;
  ta.gamma = 1.0f / (params->alpha - 1.0f);
  ta.causal = params->causal;
  ta.max_iter = params->max_iter;
  ta.tol = params->tol;
  ta.gk = gamma_kind(params->alpha);
  ta.c64 = c64_of(params);
  ta.g64 = g64_of(params);
  if (lists) {
    ta.lists = static_cast<ListBlock*>(lists);
    ta.use = packed_lists_use(shape, lists);
  }
  if ((st = from_hip(launch_tau_packed(ta, shape->dtype, shape->head_dim, s))) != EA_OK) return st;
  Packed<FwdArgs> fa{};
  fa.pk = pk;
  fa.q = q;
  fa.k = k;
  fa.v = v;
  fa.o = o;
  fa.o2 = r.o2;
  fa.tau = r.tau;
  fa.tau_lo = shape->dtype == EA_F32 ? r.tau_lo : nullptr;
  fa.q_count = r.q_count;
  fa.q_index = r.q_index;
  fa.mask = r.mask;
  fa.k_count = r.k_count;
  fa.k_index = r.k_index;
  fa.c = ta.c;
  fa.gamma = ta.gamma;
  fa.causal = params->causal;
  fa.gk = ta.gk;
  fa.c64 = ta.c64;
  fa.g64 = ta.g64;
  fa.lists = ta.lists;
  fa.use = ta.use;
  return from_hip(launch_fwd_packed(fa, shape->dtype, shape->head_dim, params->need_bwd != 0, s));
}

ea_status entmax_packed_bwd(const ea_packed_shape* shape, const ea_params* params, const void* plan, const void* q,
                            const void* k, const void* v, const void* dout, const ea_packed_strides* strides,
                            int32_t zero_rest, const void* residuals, size_t residual_bytes, const void* lists,
                            size_t lists_bytes, void* dq, void* dk, void* dv, void* workspace, size_t ws_bytes,
                            void* stream) {
  PackedResiduals r;
  ea_status st = prep_packed(shape, params, plan, q, k, v, dout, strides, residuals, residual_bytes, &r);
  if (st != EA_OK) return st;
  if (!params->need_bwd || !tensor_ok(dq) || !tensor_ok(dk) || !tensor_ok(dv) || !tensor_ok(workspace))
    return EA_ERR_INVALID_ARG;
  if ((st = check_packed_lists(shape, lists, lists_bytes)) != EA_OK) return st;
  PackedBwdWs w{};
  if (lists && ws_bytes < packed_ws_bwd(shape, true, workspace, &w)) lists = nullptr;  // no room to sort them
  if (!lists && ws_bytes < packed_ws_bwd(shape, false, workspace, &w)) return EA_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Packed<DeltaArgs> da{};
  da.pk = packed_args(shape, plan, strides, zero_rest);
  da.dout = dout;
  da.o2 = r.o2;
  da.delta = w.delta;
  if (lists) {
    da.lists = static_cast<const ListBlock*>(lists);
    da.use = packed_lists_use(shape, lists);
    da.buckets = w.buckets;
  }
  da.rows = (int64_t)shape->heads * shape->tokens;
  if ((st = from_hip(launch_delta_packed(da, shape->dtype, shape->head_dim, s))) != EA_OK) return st;
  Packed<BwdArgs> ba{};
  ba.pk = da.pk;
  ba.pk.parts = packed_parts(shape);
  ba.pk.dk_part = w.dk;
  ba.pk.dv_part = w.dv;
  ba.q = q;
  ba.k = k;
  ba.v = v;
  ba.dout = dout;
  ba.tau = r.tau;
  ba.tau_lo = shape->dtype == EA_F32 ? r.tau_lo : nullptr;
  ba.delta = da.delta;
  ba.q_count = r.q_count;
  ba.q_index = r.q_index;
  ba.k_count = r.k_count;
  ba.k_index = r.k_index;
  ba.dq = static_cast<float*>(dq);  // (of the inputs' type: see the kernels)
  ba.dk = static_cast<float*>(dk);
  ba.dv = static_cast<float*>(dv);
  ba.c = (params->alpha - 1.0f) * params->scale;
  ba.gamma = 1.0f / (params->alpha - 1.0f);
  ba.scale = params->scale;
  ba.causal = params->causal;
  ba.gk = gamma_kind(params->alpha);
  ba.c64 = c64_of(params);
  ba.g64 = g64_of(params);
  if (lists) {
    ba.lists = da.lists;
    ba.buckets = w.buckets;
    ba.pk.use = da.use;
    ba.pk.wrote = w.wrote;
  }
  if ((st = from_hip(launch_bwd_dkdv_packed(ba, shape->dtype, shape->head_dim, s))) != EA_OK) return st;
  return from_hip(launch_bwd_dq_packed(ba, shape->dtype, shape->head_dim, s));
}

// ------------------------------------------------ single tokens

namespace {

// The sizes of a call.
DecodeArgs decode_sizes(const ea_decode_shape* s) {
  DecodeArgs a{};
  a.requests = s->requests;
  a.heads = s->heads;
  a.kv_heads = s->kv_heads;
  a.group = s->heads / s->kv_heads;
  a.prefix = s->prefix;
  a.capacity = s->capacity;
  static_assert(DEC_RUN == 4, "a run's maxima are 16 bytes");
  constexpr int RUN_KEYS = DEC_KEYS * DEC_RUN;
  a.prefix_runs = (s->prefix + RUN_KEYS - 1) / RUN_KEYS;
  a.own_runs = (s->capacity + RUN_KEYS - 1) / RUN_KEYS;
  return a;
}

ea_status check_decode(const ea_decode_shape* s) {
  if (!s) return EA_ERR_INVALID_ARG;
  if (s->requests < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads != 0) return EA_ERR_INVALID_ARG;
  if (s->prefix < 0 || s->capacity < 0) return EA_ERR_INVALID_ARG;
  if (!dtype_ok(s->dtype) || (s->head_dim != 64 && s->head_dim != 128)) return EA_ERR_UNSUPPORTED;
  if ((int64_t)s->prefix + s->capacity > MAX_SEQLEN) return EA_ERR_UNSUPPORTED;
  // a launch has fewer than 2^32 threads: 256 to a row, 64 to a workgroup over keys
  if ((int64_t)s->requests * s->heads >= (1 << 23)) return EA_ERR_UNSUPPORTED;
  if (decode_maxima_wgs(decode_sizes(s), s->dtype) >= (1 << 26)) return EA_ERR_UNSUPPORTED;
  return EA_OK;
}

size_t decode_parts(const ea_decode_shape* s, void* base, DecodeArgs* a) {
  const size_t rows = (size_t)s->requests * s->heads;
  const size_t pb = ((size_t)s->prefix + DEC_KEYS - 1) / DEC_KEYS, ob = ((size_t)s->capacity + DEC_KEYS - 1) / DEC_KEYS;
  const size_t p_wide = (pb + DEC_RUN - 1) / DEC_RUN * DEC_RUN, o_wide = (ob + DEC_RUN - 1) / DEC_RUN * DEC_RUN;
  Parts p{static_cast<char*>(base)};
  a->pq = p.take<uint8_t>(rows * p_wide * (DEC_KEYS / 4));
  a->oq = p.take<uint8_t>(rows * o_wide * (DEC_KEYS / 4));
  a->pm = p.take<float>(rows * p_wide);
  a->om = p.take<float>(rows * o_wide);
  a->spill = p.take<float>(rows * (pb + ob) * DEC_KEYS);
  return p.at;
}

}  // namespace

ea_status entmax_prefix_decode_workspace(const ea_decode_shape* shape, size_t* bytes) {
  const ea_status st = check_decode(shape);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  DecodeArgs a{};
  *bytes = decode_parts(shape, nullptr, &a);
  return EA_OK;
}

ea_status entmax_prefix_decode(const ea_decode_shape* shape, const ea_params* params,
                               const ea_decode_strides* st, const void* q, const void* k, const void* v,
                               const int32_t* lengths, const void* k_prefix, const void* v_prefix, void* o,
                               void* workspace, size_t ws_bytes, void* stream) {
  ea_status status = check_decode(shape);
  if (status != EA_OK) return status;
  if (!params) return EA_ERR_INVALID_ARG;
  if ((status = check_params(params)) != EA_OK) return status;
  if (shape->requests == 0) return EA_OK;
  const size_t es = size_of(shape->dtype);
  const int64_t vec = 16 / (int64_t)es;
  if (!st || !strides_ok(&st->q, es) || !strides_ok(&st->o, es)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(q) || !tensor_ok(o) || !small_ok(lengths)) return EA_ERR_INVALID_ARG;
  // (a block's offsets are 32-bit numbers)
  constexpr int64_t MAX_KEY_ROW = 1 << 24;
  if (shape->capacity && st->k.row > MAX_KEY_ROW) return EA_ERR_INVALID_ARG;
  if (shape->prefix && st->k_prefix.row > MAX_KEY_ROW) return EA_ERR_INVALID_ARG;
  if (shape->capacity) {
    if (!tensor_ok(k) || !tensor_ok(v) || !strides_ok(&st->k, es) || !strides_ok(&st->v, es)) return EA_ERR_INVALID_ARG;
    for (int64_t x : {st->k_request, st->v_request})
      if (x < 0 || x % vec != 0 || x > MAX_STRIDE) return EA_ERR_INVALID_ARG;
  }
  if (shape->prefix && (!tensor_ok(k_prefix) || !tensor_ok(v_prefix) || !strides_ok(&st->k_prefix, es) ||
                        !strides_ok(&st->v_prefix, es)))
    return EA_ERR_INVALID_ARG;
  DecodeArgs a = decode_sizes(shape);
  const size_t need = decode_parts(shape, workspace, &a);
  if (need && !tensor_ok(workspace)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < need) return EA_ERR_WORKSPACE;
  a.q = q;
  a.k = k;
  a.v = v;
  a.pk = k_prefix;
  a.pv = v_prefix;
  a.o = o;
  a.q_row = st->q.row;
  a.q_head = st->q.head;
  a.o_row = st->o.row;
  a.o_head = st->o.head;
  a.k_batch = st->k_request;
  a.k_row = st->k.row;
  a.k_head = st->k.head;
  a.v_batch = st->v_request;
  a.v_row = st->v.row;
  a.v_head = st->v.head;
  a.pk_row = st->k_prefix.row;
  a.pk_head = st->k_prefix.head;
  a.pv_row = st->v_prefix.row;
  a.pv_head = st->v_prefix.head;
  a.lengths = lengths;
  a.c = (params->alpha - 1.0f) * params->scale;
  a.alpha = params->alpha;
  a.gamma = 1.0f / (params->alpha - 1.0f);
  a.tol = params->tol;
  a.max_iter = params->max_iter;
  a.gk = gamma_kind(params->alpha);
  a.c64 = c64_of(params);
  a.g64 = g64_of(params);
  return from_hip(launch_decode(a, shape->dtype, shape->head_dim, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------ a cache in pages and 4 bits

namespace {

ea_status check_cache(const ea_cache* c, PageDims* out) {
  if (!c || c->pages < 1 || c->page_size < 1 || c->kv_heads < 1) return EA_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return EA_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return EA_ERR_UNSUPPORTED;
  if (c->kv_heads > 1 << 16) return EA_ERR_UNSUPPORTED;
  int shift = 4;
  while (1 << shift < c->page_size) ++shift;
  // (a token's place in the pool is a 32-bit number)
  if ((int64_t)c->pages << shift > INT32_MAX) return EA_ERR_UNSUPPORTED;
  *out = PageDims{c->pages, shift, c->kv_heads, c->head_dim};
  return EA_OK;
}

ea_status check_table(const ea_page_table* t, const int32_t* ids, const PageDims& c, PageTable* out) {
  if (!t || t->rows < 1 || t->width < 1 || t->stride < 0 || t->stride > MAX_STRIDE) return EA_ERR_INVALID_ARG;
  if (!small_ok(ids)) return EA_ERR_INVALID_ARG;
  if ((int64_t)t->width << c.shift > MAX_SEQLEN || t->rows > 1 << 20) return EA_ERR_UNSUPPORTED;
  *out = PageTable{ids, t->rows, t->width, t->stride};
  return EA_OK;
}

ea_status cache_rows(const ea_cache* c, const void* cache, const ea_page_table* t, const int32_t* table, int32_t tokens,
                     int32_t dtype, const int32_t* rows, const int32_t* positions, const void* k, const ea_strides* ks,
                     const void* v, const ea_strides* vs, bool append, void* stream) {
  CacheRowsArgs a{};
  ea_status st = check_cache(c, &a.c);
  if (st != EA_OK || (st = check_table(t, table, a.c, &a.t)) != EA_OK) return st;
  if (!dtype_ok(dtype)) return EA_ERR_UNSUPPORTED;
  if (tokens < 0) return EA_ERR_INVALID_ARG;
  // a launch has fewer than 2^32 threads: at least 16 tokens to 256 of them
  if ((int64_t)tokens * c->kv_heads >= (int64_t)1 << 27) return EA_ERR_UNSUPPORTED;
  if (tokens == 0) return EA_OK;
  const size_t es = size_of(dtype);
  if (!strides_ok(ks, es) || !strides_ok(vs, es)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(cache) || !tensor_ok(k) || !tensor_ok(v) || !small_ok(rows) || !small_ok(positions))
    return EA_ERR_INVALID_ARG;
  a.cache = static_cast<uint8_t*>(const_cast<void*>(cache));
  a.k = const_cast<void*>(k);
  a.v = const_cast<void*>(v);
  a.k_row = ks->row;
  a.k_head = ks->head;
  a.v_row = vs->row;
  a.v_head = vs->head;
  a.rows = rows;
  a.positions = positions;
  a.tokens = tokens;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return from_hip(append ? launch_cache_append(a, dtype, s) : launch_cache_read(a, dtype, s));
}

size_t update_parts(const PageDims& c, int rows, void* base, CacheUpdateArgs* a) {
  const size_t pairs = rows > c.pages ? rows : c.pages;
  Parts p{static_cast<char*>(base)};
  a->marks = p.take<int32_t>(UPDATE_MARKS);
  a->holders = p.take<int32_t>(c.pages);
  a->writers = p.take<int32_t>(c.pages);
  a->lowest = p.take<int32_t>(c.pages);
  a->furthest = p.take<int32_t>(c.pages);
  a->free_list = p.take<int32_t>(c.pages);
  a->before = p.take<int32_t>(rows);
  a->source = p.take<int32_t>(pairs);
  a->target = p.take<int32_t>(pairs);
  return p.at;
}

// The arguments that an update and a compaction have in common.
ea_status table_args(const ea_cache* c, int32_t layers, void* cache, const ea_page_table* t,
                     const int32_t* table, const int32_t* lengths, int32_t rows, int32_t* table_out, int64_t out_stride, void* workspace,
                     size_t ws_bytes, CacheUpdateArgs* a) {
  ea_status st = check_cache(c, &a->c);
  if (st != EA_OK || (st = check_table(t, table, a->c, &a->t)) != EA_OK) return st;
  if (layers < 1 || rows < 0 || out_stride < t->width || out_stride > MAX_STRIDE) return EA_ERR_INVALID_ARG;
  if (layers > 1 << 16 || rows > 1 << 20) return EA_ERR_UNSUPPORTED;
  if (!tensor_ok(cache) || !small_ok(lengths) || (rows && !small_ok(table_out))) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(workspace)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < update_parts(a->c, rows, workspace, a)) return EA_ERR_WORKSPACE;
  a->layers = layers;
  a->cache = static_cast<uint8_t*>(cache);
  a->lengths = lengths;
  a->table_out = table_out;
  a->out_stride = out_stride;
  a->rows_out = rows;
  return EA_OK;
}

ea_status check_paged(const ea_paged_shape* s, const ea_cache* c, PagedArgs* a) {
  if (!s) return EA_ERR_INVALID_ARG;
  const ea_status st = check_cache(c, &a->c);
  if (st != EA_OK) return st;
  if (s->queries < 0 || s->heads < 1 || s->heads % c->kv_heads != 0 || s->longest < 0) return EA_ERR_INVALID_ARG;
  if (!dtype_ok(s->dtype) || s->longest > MAX_SEQLEN) return EA_ERR_UNSUPPORTED;
  // a launch has fewer than 2^32 threads: 256 to a workgroup
  if ((int64_t)s->queries * s->heads >= 1 << 23) return EA_ERR_UNSUPPORTED;
  a->queries = s->queries;
  a->heads = s->heads;
  a->group = s->heads / c->kv_heads;
  a->longest = s->longest;
  a->regions = (s->longest + PAGED_REGION - 1) / PAGED_REGION;
  if (paged_score_wgs(*a) >= 1 << 24) return EA_ERR_UNSUPPORTED;
  return EA_OK;
}

size_t paged_parts(void* base, PagedArgs* a) {
  const size_t lists = (size_t)a->queries * a->heads * a->regions;
  Parts p{static_cast<char*>(base)};
  a->tops = p.take<u32x4_t>(lists);
  a->list = p.take<u32x2_t>(lists * PAGED_REGION);
  return p.at;
}

}  // namespace

ea_status entmax_cache_page_bytes(const ea_cache* c, size_t* bytes) {
  PageDims d;
  const ea_status st = check_cache(c, &d);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  *bytes = (size_t)page_bytes(d);
  return EA_OK;
}

ea_status entmax_cache_append(const ea_cache* c, void* cache, const ea_page_table* t,
                              const int32_t* table, int32_t tokens, int32_t dtype, const int32_t* rows,
                              const int32_t* positions, const void* k, const ea_strides* ks, const void* v, const ea_strides* vs, void* stream) {
  return cache_rows(c, cache, t, table, tokens, dtype, rows, positions, k, ks, v, vs, true, stream);
}

ea_status entmax_cache_read(const ea_cache* c, const void* cache, const ea_page_table* t,
                            const int32_t* table, int32_t tokens, int32_t dtype, const int32_t* rows,
                            const int32_t* positions, void* k, const ea_strides* ks, void* v, const ea_strides* vs, void* stream) {
  return cache_rows(c, cache, t, table, tokens, dtype, rows, positions, k, ks, v, vs, false, stream);
}

ea_status entmax_cache_workspace(const ea_cache* c, int32_t rows, size_t* bytes) {
  PageDims d;
  const ea_status st = check_cache(c, &d);
  if (st != EA_OK) return st;
  if (rows < 0 || !bytes) return EA_ERR_INVALID_ARG;
  if (rows > 1 << 20) return EA_ERR_UNSUPPORTED;
  CacheUpdateArgs a{};
  *bytes = update_parts(d, rows, nullptr, &a);
  return EA_OK;
}

ea_status entmax_cache_update(const ea_cache* c, int32_t layers, void* cache, const ea_page_table* t,
                              const int32_t* table, const int32_t* lengths, int32_t rows_out, const int32_t* parents, const int32_t* counts,
                              int32_t* table_out, int64_t out_stride, int32_t* lengths_out, int32_t* missing,
                              void* workspace, size_t ws_bytes, void* stream) {
  CacheUpdateArgs a{};
  const ea_status st =
      table_args(c, layers, cache, t, table, lengths, rows_out, table_out, out_stride, workspace, ws_bytes, &a);
  if (st != EA_OK) return st;
  if (rows_out == 0) return EA_OK;
  if (!small_ok(parents) || !small_ok(counts) || !small_ok(lengths_out) || !small_ok(missing))
    return EA_ERR_INVALID_ARG;
  a.parents = parents;
  a.counts = counts;
  a.lengths_out = lengths_out;
  a.missing = missing;
  return from_hip(launch_cache_update(a, static_cast<hipStream_t>(stream)));
}

ea_status entmax_cache_compact(const ea_cache* c, int32_t layers, void* cache, const ea_page_table* t,
                               const int32_t* table, const int32_t* lengths, int32_t* table_out, int64_t out_stride, int32_t* used,
                               void* workspace, size_t ws_bytes, void* stream) {
  CacheUpdateArgs a{};
  const ea_status st = table_args(c, layers, cache, t, table, lengths, t ? t->rows : 0, table_out, out_stride,
                                  workspace, ws_bytes, &a);
  if (st != EA_OK) return st;
  if (!small_ok(used)) return EA_ERR_INVALID_ARG;
  a.missing = used;
  return from_hip(launch_cache_compact(a, static_cast<hipStream_t>(stream)));
}

ea_status entmax_paged_decode_workspace(const ea_paged_shape* shape, const ea_cache* c, size_t* bytes) {
  PagedArgs a{};
  const ea_status st = check_paged(shape, c, &a);
  if (st != EA_OK) return st;
  if (!bytes) return EA_ERR_INVALID_ARG;
  *bytes = paged_parts(nullptr, &a);
  return EA_OK;
}

ea_status entmax_paged_decode(const ea_paged_shape* shape, const ea_params* params, const ea_cache* c,
                              const void* cache, const ea_page_table* t, const int32_t* table, const void* q,
                              const ea_strides* qs, const int32_t* lengths, const int32_t* rows, void* o, const ea_strides* os,
                              void* workspace, size_t ws_bytes, void* stream) {
  PagedArgs a{};
  ea_status st = check_paged(shape, c, &a);
  if (st != EA_OK || (st = check_table(t, table, a.c, &a.t)) != EA_OK) return st;
  if (!params) return EA_ERR_INVALID_ARG;
  if ((st = check_params(params)) != EA_OK) return st;
  if (params->alpha > 2.0f) return EA_ERR_UNSUPPORTED;
  if (shape->queries == 0) return EA_OK;
  const size_t es = size_of(shape->dtype);
  if (!strides_ok(qs, es) || !strides_ok(os, es) || !tensor_ok(q) || !tensor_ok(o)) return EA_ERR_INVALID_ARG;
  if (!tensor_ok(cache) || !small_ok(lengths) || (rows && !small_ok(rows))) return EA_ERR_INVALID_ARG;
  const size_t need = paged_parts(workspace, &a);
  if (need && !tensor_ok(workspace)) return EA_ERR_INVALID_ARG;
  if (ws_bytes < need) return EA_ERR_WORKSPACE;
  a.cache = static_cast<const uint8_t*>(cache);
  a.q = q;
  a.o = o;
  a.q_row = qs->row;
  a.q_head = qs->head;
  a.o_row = os->row;
  a.o_head = os->head;
  a.lengths = lengths;
  a.rows = rows;
  a.scale_c = (params->alpha - 1.0f) * params->scale;
  a.alpha = params->alpha;
  a.gamma = 1.0f / (params->alpha - 1.0f);
  a.tol = params->tol;
  a.max_iter = params->max_iter;
  a.gk = gamma_kind(params->alpha);
  return from_hip(launch_paged_decode(a, shape->dtype, static_cast<hipStream_t>(stream)));
}

const char* entmax_attn_status_string(ea_status s) {
  switch (s) {
    case EA_OK: return "ok";
    case EA_ERR_INVALID_ARG: return "invalid argument";
    case EA_ERR_UNSUPPORTED: return "unsupported shape or dtype";
    case EA_ERR_WORKSPACE: return "workspace too small";
    case EA_ERR_HIP: return "HIP launch failure";
  }
  return "unknown status";
}

const char* entmax_attn_last_hip_error(void) {
  return last_hip_error == hipSuccess ? "" : hipGetErrorName(last_hip_error);
}

}  // extern "C"
