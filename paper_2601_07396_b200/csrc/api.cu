// The extern "C" surface: argument validation, layout queries, dispatch to the kernels.
#include <algorithm>
#include <atomic>
#include <cstdio>
#include <cmath>
#include <cstring>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "fp8.cuh"
#include "internal.cuh"

namespace svdc {

static std::atomic<uint64_t> g_launches{0};
static std::atomic<int> g_path{0};
static std::atomic<int> g_last_path{0};
static thread_local char g_cuda_error[256] = "";

void count_launch(int n) { g_launches.fetch_add((uint64_t)n, std::memory_order_relaxed); }

int record_cuda(cudaError_t e) {
    if (e == cudaSuccess) return SVDCACHE_OK;
    std::snprintf(g_cuda_error, sizeof(g_cuda_error), "%s: %s", cudaGetErrorName(e), cudaGetErrorString(e));
    return SVDCACHE_ERR_CUDA;
}

int check_last_launch() { return record_cuda(cudaGetLastError()); }

// An NVTX range around an entry point (costs nothing unless a profiler is attached): the kernels
// of a call show up under its name in a timeline.
struct NvtxRange {
    explicit NvtxRange(const char *name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
};

static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static int check_shape(int64_t N, int D, int k, int dtype) {
    if (dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) return SVDCACHE_ERR_INVALID_ARG;
    if (N < 1 || D < 8 || D > 16384 || (D % 8) != 0) return SVDCACHE_ERR_BAD_SHAPE;
    if (k < 8 || k > 256 || (k % 8) != 0 || k > D) return SVDCACHE_ERR_BAD_SHAPE;
    return SVDCACHE_OK;
}

static int check_pitch(int64_t ld, int D, int dtype) {
    if (ld < D) return SVDCACHE_ERR_BAD_SHAPE;
    if (((size_t)ld * elem_bytes(dtype)) % 16 != 0) return SVDCACHE_ERR_BAD_ALIGN;
    return SVDCACHE_OK;
}

static int dispatch(const StepArgs &a_in, bool full, cudaStream_t s) {
    StepArgs a = a_in;
    const int want = g_path.load();
    const bool can_umma = umma_supported(a, full);
    if (want == 2 && !can_umma) return SVDCACHE_ERR_BAD_SHAPE;
    const bool use_umma = (want == 2) || (want == 0 && can_umma);
    g_last_path.store(use_umma ? 2 : 1);
    if (use_umma) return full ? umma_full_step(a, s) : umma_cached_step(a, s);
    return full ? simt_full_step(a, s) : simt_cached_step(a, s);
}

__global__ void state_reset_kernel(StateHeader *h, int64_t N, int D, int k, int dtype) {
    if (threadIdx.x == 0 && blockIdx.x == 0) {
        h->magic = kStateMagic;
        h->dtype = dtype;
        h->N = N;
        h->D = D;
        h->k = k;
        h->full_steps = 0;
        h->status = SVDCACHE_OK;
        h->done = 0;
        h->pad = 0;
        h->exits = 0;
    }
}

}  // namespace svdc

using namespace svdc;

extern "C" {

const char *svdcache_status_string(int status) {
    switch (status) {
        case SVDCACHE_OK: return "ok";
        case SVDCACHE_ERR_INVALID_ARG: return "invalid argument";
        case SVDCACHE_ERR_BAD_SHAPE: return "shape outside the supported limits";
        case SVDCACHE_ERR_BAD_ALIGN: return "pointer or pitch not 16-byte aligned";
        case SVDCACHE_ERR_STATE: return "cached step on a state that has seen no full step";
        case SVDCACHE_ERR_WORKSPACE: return "workspace or buffer too small";
        case SVDCACHE_ERR_TIMEOUT: return "a bounded in-kernel wait ran out";
        case SVDCACHE_ERR_CUDA: return "CUDA call failed";
        case SVDCACHE_ERR_NOT_CONVERGED: return "eigen-solver did not converge";
        case SVDCACHE_ERR_SCRATCH_LIMIT: return "problem needs more scratch than the library carries built in";
        default: return "unknown status";
    }
}

const char *svdcache_last_cuda_error(void) { return g_cuda_error; }

uint64_t svdcache_kernel_launches(void) { return g_launches.load(); }
int svdcache_set_path(int path) {
    if (path < 0 || path > 2) return SVDCACHE_ERR_INVALID_ARG;
    return g_path.exchange(path);
}
int svdcache_last_path(void) { return g_last_path.load(); }

int svdcache_selftest_wait_timeout(void *state, int64_t limit_cycles, void *stream) {
    if (!state) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(state) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    if (limit_cycles < 1 || limit_cycles > 200000000LL) return SVDCACHE_ERR_INVALID_ARG;   // at most ~0.1 s
    return umma_wait_selftest(state, (long long)limit_cycles, (cudaStream_t)stream);
}

/* ----------------------------------------------------------------- calibration --- */

int svdcache_calibrate_workspace_bytes(int D, int k, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_shape(1, D, k, SVDCACHE_F32);
    if (rc) return rc;
    *bytes = calib_workspace_bytes(D, k);
    return SVDCACHE_OK;
}

static int check_ws(int D, int k, void *ws, size_t bytes) {
    int rc = check_shape(1, D, k, SVDCACHE_F32);
    if (rc) return rc;
    if (!ws) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    if (bytes < calib_workspace_bytes(D, k)) return SVDCACHE_ERR_WORKSPACE;
    return SVDCACHE_OK;
}

int svdcache_calibrate_begin(int D, int k, void *ws, size_t bytes, void *stream) {
    int rc = check_ws(D, k, ws, bytes);
    if (rc) return rc;
    return calib_begin(D, k, ws, (cudaStream_t)stream);
}

int svdcache_calibrate_accumulate(const void *F, int64_t M, int D, int64_t ld, int dtype, void *ws,
                                  size_t bytes, void *stream) {
    NvtxRange range("svdcache_calibrate_accumulate");
    if (dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) return SVDCACHE_ERR_INVALID_ARG;
    if (M < 0 || D < 8 || D > 16384 || (D % 8) != 0) return SVDCACHE_ERR_BAD_SHAPE;
    if (!ws) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    if (bytes < calib_workspace_bytes(D, 8)) return SVDCACHE_ERR_WORKSPACE;
    if (M == 0) return SVDCACHE_OK;
    if (!F) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_pitch(ld, D, dtype);
    if (rc) return rc;
    if (!aligned16(F)) return SVDCACHE_ERR_BAD_ALIGN;
    return calib_accumulate(F, M, D, ld, dtype, ws, (cudaStream_t)stream);
}

int svdcache_calibrate_finish(int D, int k, float *Vk, double *lambda, double *trace, double *info,
                              void *ws, size_t bytes, void *stream) {
    NvtxRange range("svdcache_calibrate_finish");
    int rc = check_ws(D, k, ws, bytes);
    if (rc) return rc;
    if (!Vk) return SVDCACHE_ERR_INVALID_ARG;
    if (!aligned16(Vk)) return SVDCACHE_ERR_BAD_ALIGN;
    return calib_finish(D, k, Vk, lambda, trace, info, ws, (cudaStream_t)stream);
}

int svdcache_calibrate(const void *Fstack, int64_t M, int D, int64_t ld, int dtype, int k, float *Vk,
                       double *lambda, double *trace, double *info, void *ws, size_t bytes,
                       void *stream) {
    if (M < 1) return SVDCACHE_ERR_BAD_SHAPE;
    int rc = svdcache_calibrate_begin(D, k, ws, bytes, stream);
    if (rc) return rc;
    rc = svdcache_calibrate_accumulate(Fstack, M, D, ld, dtype, ws, bytes, stream);
    if (rc) return rc;
    return svdcache_calibrate_finish(D, k, Vk, lambda, trace, info, ws, bytes, stream);
}

int svdcache_calibrate_gram_region(int D, size_t *offset, size_t *bytes) {
    if (!offset || !bytes) return SVDCACHE_ERR_INVALID_ARG;
    if (D < 8 || D > 16384 || (D % 8) != 0) return SVDCACHE_ERR_BAD_SHAPE;
    *offset = calib_gram_offset();
    *bytes = (size_t)D * D * sizeof(double);
    return SVDCACHE_OK;
}

int svdcache_basis_similarity(const float *VkA, const double *lambdaA, const float *VkB, const double *lambdaB, int D,
                              int k, double *column_cos, double *out, void *stream) {
    if (!VkA || !VkB || !lambdaA || !lambdaB || !column_cos || !out) return SVDCACHE_ERR_INVALID_ARG;
    if (D < 1 || k < 1 || k > D || k > 16384) return SVDCACHE_ERR_BAD_SHAPE;
    int rc = column_cosines_launch(VkA, VkB, D, k, column_cos, (cudaStream_t)stream);
    if (rc) return rc;
    // the spectra are k numbers each: their statistic is formed on the host
    std::vector<double> la(k), lb(k), cs(k);
    rc = record_cuda(cudaMemcpyAsync(la.data(), lambdaA, k * sizeof(double), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    if (!rc) rc = record_cuda(cudaMemcpyAsync(lb.data(), lambdaB, k * sizeof(double), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    if (!rc) rc = record_cuda(cudaMemcpyAsync(cs.data(), column_cos, k * sizeof(double), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    if (!rc) rc = record_cuda(cudaStreamSynchronize((cudaStream_t)stream));
    if (rc) return rc;
    double ab = 0.0, aa = 0.0, bb = 0.0, mean = 0.0;
    for (int i = 0; i < k; ++i) {
        const double sa = la[i] > 0.0 ? std::sqrt(la[i]) : 0.0, sb = lb[i] > 0.0 ? std::sqrt(lb[i]) : 0.0;
        ab += sa * sb; aa += sa * sa; bb += sb * sb;
        mean += cs[i];
    }
    const double na = std::sqrt(aa), nb = std::sqrt(bb);
    out[0] = (na > 0.0 && nb > 0.0) ? (ab / (na * nb)) * (na < nb ? na / nb : nb / na) : 0.0;
    out[1] = mean / k;
    return SVDCACHE_OK;
}

int svdcache_rank_for_energy(const double *lambda, int n, double trace, double tau, int *k_out) {
    if (!lambda || !k_out || n < 1 || !(trace > 0.0) || !(tau >= 0.0) || !(tau <= 1.0))
        return SVDCACHE_ERR_INVALID_ARG;
    double acc = 0.0;
    *k_out = n;
    for (int i = 0; i < n; ++i) {
        acc += lambda[i];
        if (acc / trace >= tau) { *k_out = i + 1; break; }
    }
    return SVDCACHE_OK;
}

/* ------------------------------------------------------------------------ basis --- */

int svdcache_basis_bytes(int D, int k, int dtype, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_shape(1, D, k, dtype);
    if (rc) return rc;
    *bytes = basis_layout(D, k, dtype).total;
    return SVDCACHE_OK;
}

int svdcache_basis_layout(int D, int k, int dtype, size_t *v32, size_t *vt32, size_t *v16, size_t *vt16) {
    int rc = check_shape(1, D, k, dtype);
    if (rc) return rc;
    const BasisLayout L = basis_layout(D, k, dtype);
    if (v32) *v32 = L.v_f32;
    if (vt32) *vt32 = L.vt_f32;
    if (v16) *v16 = (dtype == SVDCACHE_BF16) ? L.v_bf16 : 0;
    if (vt16) *vt16 = (dtype == SVDCACHE_BF16) ? L.vt_bf16 : 0;
    return SVDCACHE_OK;
}

int svdcache_basis_prepare(const float *Vk, int D, int k, int dtype, void *basis, size_t bytes, void *stream) {
    int rc = check_shape(1, D, k, dtype);
    if (rc) return rc;
    if (!Vk || !basis) return SVDCACHE_ERR_INVALID_ARG;
    if (!aligned16(Vk) || (reinterpret_cast<uintptr_t>(basis) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    if (bytes < basis_layout(D, k, dtype).total) return SVDCACHE_ERR_WORKSPACE;
    return basis_prepare(Vk, D, k, dtype, basis, (cudaStream_t)stream);
}

/* ------------------------------------------------------------------------ state --- */

int svdcache_state_bytes(int64_t N, int D, int k, int dtype, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_shape(N, D, k, dtype);
    if (rc) return rc;
    *bytes = state_layout(N, D, k, dtype).total;
    return SVDCACHE_OK;
}

int svdcache_state_layout(int64_t N, int D, int k, int dtype, size_t *chat_offset, size_t *r_offset) {
    int rc = check_shape(N, D, k, dtype);
    if (rc) return rc;
    const StateLayout L = state_layout(N, D, k, dtype);
    if (chat_offset) *chat_offset = L.chat;
    if (r_offset) *r_offset = L.r;
    return SVDCACHE_OK;
}

int svdcache_state_reset(void *state, int64_t N, int D, int k, int dtype, void *stream) {
    int rc = check_shape(N, D, k, dtype);
    if (rc) return rc;
    if (!state) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(state) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    state_reset_kernel<<<1, 32, 0, (cudaStream_t)stream>>>((StateHeader *)state, N, D, k, dtype);
    count_launch();
    return check_last_launch();
}

int svdcache_state_query(const void *state, void *stream, int64_t *full_steps, int *status) {
    if (!state) return SVDCACHE_ERR_INVALID_ARG;
    StateHeader h;
    int rc = record_cuda(cudaMemcpyAsync(&h, state, sizeof(h), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    if (rc) return rc;
    rc = record_cuda(cudaStreamSynchronize((cudaStream_t)stream));
    if (rc) return rc;
    if (h.magic != kStateMagic) return SVDCACHE_ERR_STATE;
    if (full_steps) *full_steps = (int64_t)h.full_steps;
    if (status) *status = h.status;
    return SVDCACHE_OK;
}

/* ------------------------------------------------------------------------ steps --- */

static int check_step(const StepArgs &a, bool full) {
    int rc = check_shape(a.N, a.D, a.k, a.dtype);
    if (rc) return rc;
    if (a.nblocks < 1) return SVDCACHE_ERR_BAD_SHAPE;
    if (!a.basis || !a.state || (full ? !a.F : !a.Fhat)) return SVDCACHE_ERR_INVALID_ARG;
    rc = check_pitch(a.ld, a.D, a.dtype);
    if (rc) return rc;
    if (!aligned16(full ? a.F : (const void *)a.Fhat)) return SVDCACHE_ERR_BAD_ALIGN;
    if ((reinterpret_cast<uintptr_t>(a.basis) & 255u) || (reinterpret_cast<uintptr_t>(a.state) & 255u))
        return SVDCACHE_ERR_BAD_ALIGN;
    if (a.C_out && !aligned16(a.C_out)) return SVDCACHE_ERR_BAD_ALIGN;
    if (full && !(a.beta >= 0.0f && a.beta <= 1.0f)) return SVDCACHE_ERR_INVALID_ARG;
    if (a.nblocks > 1) {
        const size_t strides[5] = {a.F_stride, a.Fhat_stride, a.basis_stride, a.state_stride, a.C_stride};
        for (size_t st : strides)
            if (st % 256 != 0) return SVDCACHE_ERR_BAD_ALIGN;
        if (a.basis_stride < basis_layout(a.D, a.k, a.dtype).total) return SVDCACHE_ERR_BAD_SHAPE;
        if (a.state_stride < state_layout(a.N, a.D, a.k, a.dtype).total) return SVDCACHE_ERR_BAD_SHAPE;
        const size_t need = ((size_t)(a.N - 1) * a.ld + a.D) * elem_bytes(a.dtype);
        if ((full ? a.F_stride : a.Fhat_stride) < need) return SVDCACHE_ERR_BAD_SHAPE;
        if (a.C_out && a.C_stride < (size_t)a.N * a.k * 4) return SVDCACHE_ERR_BAD_SHAPE;
    }
    return SVDCACHE_OK;
}

int svdcache_full_step_batched(int nblocks, const void *F, int64_t ld, size_t F_stride, const void *basis,
                               size_t basis_stride, void *state, size_t state_stride, float *C_out,
                               size_t C_stride, int64_t N, int D, int k, int dtype, float beta,
                               void *stream) {
    NvtxRange range("svdcache_full_step_batched");
    StepArgs a{};
    a.F = F; a.ld = ld; a.F_stride = F_stride; a.basis = basis; a.basis_stride = basis_stride;
    a.state = state; a.state_stride = state_stride; a.C_out = C_out; a.C_stride = C_stride;
    a.N = N; a.D = D; a.k = k; a.dtype = dtype; a.beta = beta; a.nblocks = nblocks;
    int rc = check_step(a, true);
    if (rc) return rc;
    return dispatch(a, true, (cudaStream_t)stream);
}

int svdcache_cached_step_batched(int nblocks, const void *state, size_t state_stride, const void *basis,
                                 size_t basis_stride, void *Fhat, int64_t ld, size_t Fhat_stride,
                                 int64_t N, int D, int k, int dtype, int steps_since_full, void *stream) {
    NvtxRange range("svdcache_cached_step_batched");
    (void)steps_since_full;  // the EMA forecast does not depend on it
    StepArgs a{};
    a.Fhat = Fhat; a.ld = ld; a.Fhat_stride = Fhat_stride; a.basis = basis; a.basis_stride = basis_stride;
    a.state = const_cast<void *>(state); a.state_stride = state_stride;
    a.N = N; a.D = D; a.k = k; a.dtype = dtype; a.nblocks = nblocks;
    int rc = check_step(a, false);
    if (rc) return rc;
    return dispatch(a, false, (cudaStream_t)stream);
}

int svdcache_full_step_residual_ema_batched(int nblocks, const void *F, int64_t ld, size_t F_stride,
                                            const void *basis, size_t basis_stride, void *state,
                                            size_t state_stride, float *C_out, size_t C_stride, int64_t N,
                                            int D, int k, int dtype, float beta, float beta_r, void *stream) {
    NvtxRange range("svdcache_full_step_residual_ema_batched");
    if (!(beta_r >= 0.0f && beta_r <= 1.0f)) return SVDCACHE_ERR_INVALID_ARG;
    StepArgs a{};
    a.F = F; a.ld = ld; a.F_stride = F_stride; a.basis = basis; a.basis_stride = basis_stride;
    a.state = state; a.state_stride = state_stride; a.C_out = C_out; a.C_stride = C_stride;
    a.N = N; a.D = D; a.k = k; a.dtype = dtype; a.beta = beta; a.beta_r = beta_r; a.nblocks = nblocks;
    int rc = check_step(a, true);
    if (rc) return rc;
    return dispatch(a, true, (cudaStream_t)stream);
}

int svdcache_forecast_weights(int predictor, int order, int steps_since_full, int interval, double *w) {
    if (!w || interval < 1 || steps_since_full < 0) return SVDCACHE_ERR_INVALID_ARG;
    return forecast_weights(predictor, order, (double)steps_since_full / (double)interval, w);
}

int svdcache_forecast_bytes(int64_t N, int k, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    if (N < 1 || k < 8 || k > 256 || (k % 8) != 0) return SVDCACHE_ERR_BAD_SHAPE;
    *bytes = forecast_layout(N, k).total;
    return SVDCACHE_OK;
}

int svdcache_cached_step_forecast_batched(int nblocks, const void *state, size_t state_stride, const void *basis,
                                          size_t basis_stride, void *Fhat, int64_t ld, size_t Fhat_stride,
                                          int64_t N, int D, int k, int dtype, const float *const *C_hist,
                                          size_t C_stride, int predictor, int order, int steps_since_full,
                                          int interval, void *forecast, size_t forecast_stride, void *stream) {
    NvtxRange range("svdcache_cached_step_forecast_batched");
    StepArgs a{};
    a.Fhat = Fhat; a.ld = ld; a.Fhat_stride = Fhat_stride; a.basis = basis; a.basis_stride = basis_stride;
    a.state = const_cast<void *>(state); a.state_stride = state_stride;
    a.N = N; a.D = D; a.k = k; a.dtype = dtype; a.nblocks = nblocks;
    int rc = check_step(a, false);
    if (rc) return rc;
    if (predictor == SVDCACHE_PREDICT_EMA) return dispatch(a, false, (cudaStream_t)stream);   // the state's own forecast
    if (!C_hist || !forecast || interval < 1 || steps_since_full < 0) return SVDCACHE_ERR_INVALID_ARG;
    double w[8];
    rc = forecast_weights(predictor, order, (double)steps_since_full / (double)interval, w);
    if (rc) return rc;
    for (int j = 0; j <= order; ++j) {
        if (!C_hist[j]) return SVDCACHE_ERR_INVALID_ARG;
        if (!aligned16(C_hist[j])) return SVDCACHE_ERR_BAD_ALIGN;
    }
    if ((reinterpret_cast<uintptr_t>(forecast) & 255u) != 0) return SVDCACHE_ERR_BAD_ALIGN;
    if (nblocks > 1) {
        if (C_stride % 256 != 0 || forecast_stride % 256 != 0) return SVDCACHE_ERR_BAD_ALIGN;
        if (C_stride < (size_t)N * k * 4 || forecast_stride < forecast_layout(N, k).total) return SVDCACHE_ERR_BAD_SHAPE;
    }
    rc = forecast_launch(C_hist, C_stride, w, order, N, k, dtype, nblocks, forecast, forecast_stride, (cudaStream_t)stream);
    if (rc) return rc;
    a.coef = forecast;
    a.coef_stride = forecast_stride;
    return dispatch(a, false, (cudaStream_t)stream);
}

int svdcache_singular_values(const double *lambda, int k, double *sigma, void *stream) {
    if (!lambda || !sigma) return SVDCACHE_ERR_INVALID_ARG;
    if (k < 1 || k > 16384) return SVDCACHE_ERR_BAD_SHAPE;
    return sigma_launch(lambda, k, sigma, (cudaStream_t)stream);
}

int svdcache_left_factors(const float *C, const double *sigma, int64_t N, int k, float *U, void *stream) {
    if (!C || !sigma || !U) return SVDCACHE_ERR_INVALID_ARG;
    if (N < 1 || k < 1 || k > 16384) return SVDCACHE_ERR_BAD_SHAPE;
    return left_factors_launch(C, sigma, N, k, U, (cudaStream_t)stream);
}

/* ----------------------------------------------------------- 8-bit linear path --- */

static const int64_t kFp8MaxRows = 0x7FFFFFFFLL - 256;
static const int kFp8MaxCols = 131072;

static int check_fp8_shape(int64_t rows, int cols) {
    return rows < 0 || rows >= kFp8MaxRows || cols < 1 || cols > kFp8MaxCols ? SVDCACHE_ERR_BAD_SHAPE : SVDCACHE_OK;
}

// a matrix of `elem`-byte values: pointer and pitch
static int check_matrix(const void *p, int64_t ld, int cols, int elem) {
    if (!p) return SVDCACHE_ERR_INVALID_ARG;
    if (ld < cols || ld > (1LL << 36)) return SVDCACHE_ERR_BAD_SHAPE;
    return aligned16(p) && (ld * elem) % 16 == 0 ? SVDCACHE_OK : SVDCACHE_ERR_BAD_ALIGN;
}

static int check_fp8_matrix(const void *q, int64_t ld, int cols, const void *s) {
    if (!s) return SVDCACHE_ERR_INVALID_ARG;
    const int rc = check_matrix(q, ld, cols, 1);
    return rc ? rc : aligned16(s) ? SVDCACHE_OK : SVDCACHE_ERR_BAD_ALIGN;
}

int svdcache_fp8_scale_bytes(int64_t rows, int cols, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    const int rc = check_fp8_shape(rows, cols);
    if (rc) return rc;
    *bytes = fp8_scale_bytes(rows, cols);
    return SVDCACHE_OK;
}

int svdcache_quantize_fp8(const void *X, int64_t rows, int cols, int64_t ld, int dtype, int tile_rows, void *Q,
                          int64_t ldq, void *S, void *stream) {
    NvtxRange range("svdcache_quantize_fp8");
    if ((dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) || (tile_rows != 1 && tile_rows != kScaleRows))
        return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(rows, cols);
    if (rc || rows == 0) return rc;
    rc = check_matrix(X, ld, cols, (int)elem_bytes(dtype));
    if (!rc) rc = check_fp8_matrix(Q, ldq, cols, S);
    if (rc) return rc;
    return quantize_fp8_launch(X, rows, cols, ld, dtype, tile_rows, Q, ldq, S, (cudaStream_t)stream);
}

int svdcache_residual_rmsnorm_fp8(const void *H, int64_t ldh, const void *X, int64_t ldx, void *H_out, int64_t ldo,
                                  const float *weight, float eps, void *Q, int64_t ldq, void *S, int64_t rows, int D,
                                  int dtype, void *stream) {
    NvtxRange range("svdcache_residual_rmsnorm_fp8");
    if ((dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) || !(eps >= 0.0f)) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(rows, D);
    if (rc) return rc;
    if (D < 8 || D > 16384 || (D % 8) != 0) return SVDCACHE_ERR_BAD_SHAPE;
    if (rows == 0) return SVDCACHE_OK;
    rc = check_matrix(H, ldh, D, (int)elem_bytes(dtype));
    if (!rc && X) rc = check_matrix(X, ldx, D, (int)elem_bytes(dtype));
    if (!rc && H_out) rc = check_matrix(H_out, ldo, D, (int)elem_bytes(dtype));
    if (!rc) rc = check_fp8_matrix(Q, ldq, D, S);
    if (!rc && weight && !aligned16(weight)) rc = SVDCACHE_ERR_BAD_ALIGN;
    if (rc) return rc;
    return rmsnorm_fp8_launch(H, ldh, X, ldx, H_out, ldo, weight, eps, Q, ldq, S, rows, D, dtype, (cudaStream_t)stream);
}

// every check of a product's arguments; args is filled where there is something to launch (M > 0)
static int check_gemm_fp8(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB, const float *bias, int act,
                          void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K, int32_t *status, GemmFp8Args *args) {
    if (act != SVDCACHE_ACT_NONE && act != SVDCACHE_ACT_GELU) return SVDCACHE_ERR_INVALID_ARG;
    if (out_dtype != SVDCACHE_F32 && out_dtype != SVDCACHE_BF16 && out_dtype != SVDCACHE_FP8) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(M, K);
    if (!rc) rc = check_fp8_shape(M, N);
    if (rc || M == 0) return rc;
    if (!status) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(status) & 3u) || (reinterpret_cast<uintptr_t>(bias) & 3u)) return SVDCACHE_ERR_BAD_ALIGN;
    rc = check_fp8_matrix(A, lda, K, SA);
    if (!rc) rc = check_fp8_matrix(B, ldb, K, SB);
    if (!rc) rc = out_dtype == SVDCACHE_FP8 ? check_fp8_matrix(C, ldc, N, SC) : check_matrix(C, ldc, N, (int)elem_bytes(out_dtype));
    GemmFp8Args a{};
    a.A = A; a.B = B; a.SA = SA; a.SB = SB; a.lda = lda; a.ldb = ldb; a.ldc = ldc; a.bias = bias; a.C = C; a.SC = SC;
    a.M = M; a.N = N; a.K = K; a.act = act; a.out = out_dtype; a.status = status;
    *args = a;
    return rc;
}

int svdcache_gemm_fp8(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB,
                      const float *bias, int act, void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K,
                      int32_t *status, void *stream) {
    NvtxRange range("svdcache_gemm_fp8");
    GemmFp8Args a;
    const int rc = check_gemm_fp8(A, lda, SA, B, ldb, SB, bias, act, C, ldc, out_dtype, SC, M, N, K, status, &a);
    return rc || M == 0 ? rc : gemm_fp8_launch(a, nullptr, (cudaStream_t)stream);
}

/* ------------------------------------------------- adapters beside a projection --- */

static const int kMaxAdapterRank = 128, kMaxAdapters = 65536, kMaxRequests = 65536;

static int check_adapters(const svdcache_adapters *p, int N, int K) {
    if (!p) return SVDCACHE_ERR_INVALID_ARG;
    if (p->count < 0 || p->count > kMaxAdapters || p->rank < 8 || p->rank > kMaxAdapterRank || p->rank % 8) return SVDCACHE_ERR_BAD_SHAPE;
    if (p->count == 0) return SVDCACHE_OK;
    if (!p->factor) return SVDCACHE_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->factor) & 3u) return SVDCACHE_ERR_BAD_ALIGN;
    int rc = check_fp8_matrix(p->down, p->down_ld, K, p->down_scales);
    if (!rc) rc = check_matrix(p->up, p->up_ld, p->rank, 2);
    if (rc) return rc;
    const int64_t most = 1LL << 38;
    if (p->down_stride < p->down_ld * (p->rank - 1) + K || p->down_stride > most || p->scales_stride < (int64_t)fp8_scale_bytes(p->rank, K) || p->scales_stride > most ||
        p->up_stride < p->up_ld * ((int64_t)N - 1) + p->rank || p->up_stride > most)
        return SVDCACHE_ERR_BAD_SHAPE;
    return p->down_stride % 16 || p->scales_stride % 16 || p->up_stride % 8 ? SVDCACHE_ERR_BAD_ALIGN : SVDCACHE_OK;
}

/* rows for the highest tiles, tiles and slots for the lowest: room for any plan */
static size_t adapters_need(int64_t M, int rank, int requests, int parts) {
    const AdapterLayout high = adapter_layout(M, 256, rank, requests, parts), low = adapter_layout(M, 16, rank, requests, parts);
    return high.tile_slots + align_up((size_t)low.tiles * 16, kAlign) + align_up((size_t)low.slots * 8, kAlign) + kAlign;
}

int svdcache_adapters_workspace_bytes(int64_t M, int rank, int requests, size_t *bytes) {
    if (!bytes) return SVDCACHE_ERR_INVALID_ARG;
    const int rc = check_fp8_shape(M, 1);
    if (rc || rank < 8 || rank > kMaxAdapterRank || rank % 8 || requests < 0 || requests > kMaxRequests) return SVDCACHE_ERR_BAD_SHAPE;
    *bytes = adapters_need(M, rank, requests, 3);
    return SVDCACHE_OK;
}

static int run_gemm_fp8_adapters(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB, const float *bias, int act,
                                 void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K, const svdcache_adapters *adapters,
                                 const int32_t *row_start, const int32_t *adapter, int requests, void *workspace, size_t workspace_bytes,
                                 int32_t *status, const int32_t *plan, int64_t limit_cycles, void *stream) {
    GemmFp8Args a;
    int rc = check_gemm_fp8(A, lda, SA, B, ldb, SB, bias, act, C, ldc, out_dtype, SC, M, N, K, status, &a);
    if (!rc) rc = check_adapters(adapters, N, K);
    if (!rc && (requests < 0 || requests > kMaxRequests)) rc = SVDCACHE_ERR_BAD_SHAPE;
    if (rc || M == 0) return rc;
    if ((requests == 0 || adapters->count == 0) && !plan) return gemm_fp8_launch(a, nullptr, (cudaStream_t)stream);
    if (requests == 0 || adapters->count == 0) return SVDCACHE_ERR_BAD_SHAPE;      /* a named plan with nothing to add */
    if (!row_start || !adapter || !workspace) return SVDCACHE_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(row_start) & 3u) || (reinterpret_cast<uintptr_t>(adapter) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return SVDCACHE_ERR_BAD_ALIGN;
    if (workspace_bytes < adapters_need(M, adapters->rank, requests, 2)) return SVDCACHE_ERR_WORKSPACE;
    if (adapter_layout(M, 256, adapters->rank, requests, 2).narrow_rows > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    const AdapterCall c{*adapters, row_start, adapter, requests, workspace, workspace_bytes, 0};
    const GemmFp8Plan named{plan && plan[0] != 0, plan ? plan[1] : 0, plan ? plan[2] : 0, 0, 0};
    a.limit = limit_cycles;
    return gemm_fp8_adapters_launch(a, c, plan ? &named : nullptr, (cudaStream_t)stream);
}

int svdcache_gemm_fp8_adapters(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB, const float *bias, int act,
                               void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K, const svdcache_adapters *adapters,
                               const int32_t *row_start, const int32_t *adapter, int requests, void *workspace, size_t workspace_bytes,
                               int32_t *status, void *stream) {
    NvtxRange range("svdcache_gemm_fp8_adapters");
    return run_gemm_fp8_adapters(A, lda, SA, B, ldb, SB, bias, act, C, ldc, out_dtype, SC, M, N, K, adapters, row_start, adapter, requests, workspace,
                                 workspace_bytes, status, nullptr, 0, stream);
}

int svdcache_selftest_gemm_fp8_adapters(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB, const float *bias, int act,
                                        void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K, const svdcache_adapters *adapters,
                                        const int32_t *row_start, const int32_t *adapter, int requests, void *workspace, size_t workspace_bytes,
                                        int32_t *status, const int32_t *plan, int64_t limit_cycles, void *stream) {
    if (!plan || limit_cycles < 0 || limit_cycles > 200000000LL) return SVDCACHE_ERR_INVALID_ARG;   /* at most ~0.1 s */
    return run_gemm_fp8_adapters(A, lda, SA, B, ldb, SB, bias, act, C, ldc, out_dtype, SC, M, N, K, adapters, row_start, adapter, requests, workspace,
                                 workspace_bytes, status, plan, limit_cycles, stream);
}

int svdcache_selftest_adapters_sizes(int64_t M, int N, int K, int rank, int requests, int out_dtype, const int32_t *plan, int brief, int sms, int64_t *sizes) {
    if (!plan || !sizes || (out_dtype != SVDCACHE_F32 && out_dtype != SVDCACHE_BF16 && out_dtype != SVDCACHE_FP8)) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(M, K);
    if (!rc) rc = check_fp8_shape(1, N);
    if (rc || M == 0 || rank < 8 || rank > kMaxAdapterRank || rank % 8 || requests < 1 || requests > kMaxRequests || sms < 2) return SVDCACHE_ERR_BAD_SHAPE;
    const bool pairs = plan[0] != 0;
    auto in = [](int v, std::initializer_list<int> of) { return std::find(of.begin(), of.end(), v) != of.end(); };
    if (pairs ? plan[2] != 2 || !in(plan[1], {128, 192, 256}) : !in(plan[1], {16, 32, 64, 128}) || !in(plan[2], {1, 2, 3, 4, 6, 8}) || plan[2] > fp8_groups(K)) return SVDCACHE_ERR_INVALID_ARG;
    KernelSize size[2];
    gemm_fp8_adapters_size(M, N, K, rank, requests, out_dtype, {pairs, plan[1], plan[2], 0, 0}, brief != 0, sms, size);
    for (const KernelSize &k : size)
        for (int64_t v : {k.ctas, (int64_t)k.cluster, (int64_t)k.columns, (int64_t)k.shared}) *sizes++ = v;
    return SVDCACHE_OK;
}

int svdcache_selftest_adapters_slots(const int32_t *row_start, const int32_t *adapter, int requests, int64_t first, int64_t M, int count, int tile_rows,
                                     int32_t *tasks, int32_t *tiles, int32_t *list, int32_t *tile_list) {
    if (!row_start || !adapter || !tasks || !tiles || !list || !tile_list) return SVDCACHE_ERR_INVALID_ARG;
    if (requests < 1 || requests > kMaxRequests || first < 0 || M < 1 || M > 0x7FFFFFFFLL || count < 0) return SVDCACHE_ERR_BAD_SHAPE;
    Requests q{row_start, adapter, first, M, requests, count, 0};
    while (q.tile_shift < 8 && (1 << q.tile_shift) < tile_rows) ++q.tile_shift;
    if ((1 << q.tile_shift) != tile_rows || tile_rows < 16) return SVDCACHE_ERR_BAD_SHAPE;
    const int all = (int)((M + tile_rows - 1) / tile_rows);
    for (int i = 0; i < all + requests; ++i) {
        const Task t = find_task(OneThread{}, q, all, i);
        memcpy(tasks + 4 * (size_t)i, &t, sizeof t);
    }
    for (int i = 0; i < all; ++i) {
        int2 from;
        write_tile_slots(OneThread{}, q, i, reinterpret_cast<int4 *>(tiles), reinterpret_cast<int2 *>(list));
        int32_t *own = tile_list + (size_t)i * (2 * tile_rows + 1);
        own[0] = tile_slots_of(OneThread{}, q, i, tile_rows, from, [&](int place, int, int2 slot) { own[1 + 2 * place] = slot.x; own[2 + 2 * place] = slot.y; });
    }
    return SVDCACHE_OK;
}

int svdcache_adapter_load(const svdcache_adapters *adapters, int index, const void *down, int64_t ldd, const void *up, int64_t ldu, int r,
                          float factor, int N, int K, int dtype, void *stream) {
    NvtxRange range("svdcache_adapter_load");
    if (dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(1, N);
    if (!rc) rc = check_fp8_shape(1, K);
    if (!rc) rc = check_adapters(adapters, N, K);
    if (rc) return rc;
    if (index < 0 || index >= adapters->count) return SVDCACHE_ERR_INVALID_ARG;
    if (r < 1 || r > adapters->rank || ldu < r || ldu > (1LL << 36)) return SVDCACHE_ERR_BAD_SHAPE;
    if (!up) return SVDCACHE_ERR_INVALID_ARG;
    rc = check_matrix(down, ldd, K, (int)elem_bytes(dtype));
    if (!rc && (reinterpret_cast<uintptr_t>(up) & (elem_bytes(dtype) - 1))) rc = SVDCACHE_ERR_BAD_ALIGN;
    if (rc) return rc;
    return adapter_load_launch(*adapters, index, down, ldd, up, ldu, r, factor, N, K, dtype, (cudaStream_t)stream);
}

int svdcache_gemm_fp8_plan(int64_t M, int N, int K, int64_t lda, int64_t ldb, int out_dtype, int32_t *plan) {
    if (!plan || (out_dtype != SVDCACHE_F32 && out_dtype != SVDCACHE_BF16 && out_dtype != SVDCACHE_FP8)) return SVDCACHE_ERR_INVALID_ARG;
    int rc = check_fp8_shape(M, K);
    if (!rc) rc = check_fp8_shape(M, N);
    if (rc) return rc;
    if (M == 0 || lda < K || ldb < K) return SVDCACHE_ERR_BAD_SHAPE;
    GemmFp8Args a{};
    a.M = M; a.N = N; a.K = K; a.lda = lda; a.ldb = ldb; a.out = out_dtype;
    GemmFp8Plan p{};
    rc = gemm_fp8_plan(a, &p);
    if (rc) return rc;
    plan[0] = p.pairs; plan[1] = p.size; plan[2] = p.splits; plan[3] = (int32_t)(p.rounds < 0x7FFFFFFF ? p.rounds : 0x7FFFFFFF);
    return SVDCACHE_OK;
}

int svdcache_selftest_gemm_fp8(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB,
                               const float *bias, int act, void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K,
                               int32_t *status, const int32_t *plan, int64_t limit_cycles, void *stream) {
    if (!plan || limit_cycles < 0 || limit_cycles > 200000000LL) return SVDCACHE_ERR_INVALID_ARG;   // at most ~0.1 s
    GemmFp8Args a;
    const int rc = check_gemm_fp8(A, lda, SA, B, ldb, SB, bias, act, C, ldc, out_dtype, SC, M, N, K, status, &a);
    if (rc || M == 0) return rc;
    const GemmFp8Plan p{plan[0] != 0, plan[1], plan[2], 0, 0};
    a.limit = limit_cycles;
    return gemm_fp8_launch(a, &p, (cudaStream_t)stream);
}

int svdcache_gemm_fp8_status_word(int32_t **word) {
    if (!word) return SVDCACHE_ERR_INVALID_ARG;
    return gemm_fp8_status_word(word);
}

int svdcache_gemm_fp8_status_query(int32_t *status) {
    if (!status) return SVDCACHE_ERR_INVALID_ARG;
    int *word = nullptr;
    int rc = gemm_fp8_status_word(&word);
    if (!rc) rc = record_cuda(cudaDeviceSynchronize());
    if (!rc) rc = record_cuda(cudaMemcpy(status, word, sizeof(*status), cudaMemcpyDeviceToHost));
    return rc;
}

/* ------------------------------------------------------------- queries and keys --- */

int svdcache_rotary_table(const void *positions, int64_t tokens, int64_t ld, int position_type, int axes, const int *dims, const double *bases,
                          float *table, int64_t ldt, void *stream) {
    NvtxRange range("svdcache_rotary_table");
    if (!dims || !bases || position_type < SVDCACHE_POSITION_I32 || position_type > SVDCACHE_POSITION_F32) return SVDCACHE_ERR_INVALID_ARG;
    if (axes < 1 || axes > SVDCACHE_ROTARY_MAX_AXES || tokens < 0 || tokens > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    int r = 0;
    for (int i = 0; i < axes; ++i) {
        if (dims[i] < 2 || dims[i] > SVDCACHE_ROTARY_MAX_DIM || dims[i] % 2) return SVDCACHE_ERR_BAD_SHAPE;
        if (!(bases[i] > 0.0) || !std::isfinite(bases[i])) return SVDCACHE_ERR_INVALID_ARG;
        r += dims[i];
    }
    if (r > SVDCACHE_ROTARY_MAX_DIM || r % 8) return SVDCACHE_ERR_BAD_SHAPE;
    if (tokens == 0) return SVDCACHE_OK;
    if (!positions || !table) return SVDCACHE_ERR_INVALID_ARG;
    if (ld < axes || ld > (1LL << 36) || ldt < r || ldt > (1LL << 36)) return SVDCACHE_ERR_BAD_SHAPE;
    if (!aligned16(table) || ldt % 4 || (reinterpret_cast<uintptr_t>(positions) & (position_type == SVDCACHE_POSITION_I64 ? 7u : 3u)))
        return SVDCACHE_ERR_BAD_ALIGN;
    return rotary_table_launch(positions, tokens, ld, position_type, axes, dims, bases, table, ldt, (cudaStream_t)stream);
}

static int check_heads(const svdcache_heads *h, int64_t batch, int64_t tokens, int dtype, bool written) {
    if (!h || !h->data) return SVDCACHE_ERR_INVALID_ARG;
    if (h->heads < 1 || h->heads > 65536) return SVDCACHE_ERR_BAD_SHAPE;
    const int64_t unit = dtype == SVDCACHE_BF16 ? 8 : 4, most = 1LL << 40;
    const int64_t strides[3] = {h->batch_stride, h->token_stride, h->head_stride}, sizes[3] = {batch, tokens, h->heads};
    if (!aligned16(h->data)) return SVDCACHE_ERR_BAD_ALIGN;
    for (int i = 0; i < 3; ++i) {
        if (sizes[i] == 1) continue;                     /* never used */
        if (strides[i] < (written ? 1 : 0) || strides[i] > most) return SVDCACHE_ERR_BAD_SHAPE;
        if (strides[i] % unit) return SVDCACHE_ERR_BAD_ALIGN;
    }
    return SVDCACHE_OK;
}

/* whether `out` is `in` itself, or begins elsewhere */
static bool in_place_or_apart(const svdcache_heads *in, const svdcache_heads *out, int64_t batch, int64_t tokens) {
    return in->data != out->data || ((batch == 1 || in->batch_stride == out->batch_stride) && (tokens == 1 || in->token_stride == out->token_stride) &&
                                     (in->heads == 1 || in->head_stride == out->head_stride));
}

/* Q (and K, unless null) of `dim` elements a head; `norm` or not */
static int run_rotary(const svdcache_heads *Q, const svdcache_heads *Q_out, const float *q_weight, const svdcache_heads *K, const svdcache_heads *K_out,
                      const float *k_weight, bool norm, float eps, int64_t batch, int64_t tokens, int dim, int dtype, const svdcache_rotation *rotation,
                      void *stream) {
    if ((dtype != SVDCACHE_F32 && dtype != SVDCACHE_BF16) || (norm && !(eps >= 0.0f)) || (K != nullptr) != (K_out != nullptr)) return SVDCACHE_ERR_INVALID_ARG;
    if (dim < 8 || dim > SVDCACHE_ROTARY_MAX_DIM || dim % 8 || batch < 0 || batch > 65535 || tokens < 0 || tokens > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    if (rotation) {
        if (rotation->flags & ~(SVDCACHE_ROTARY_HALVES | SVDCACHE_ROTARY_INVERSE)) return SVDCACHE_ERR_INVALID_ARG;
        if (rotation->r < 8 || rotation->r > dim || rotation->r % 8 || rotation->first < 0 || rotation->tokens < 0 || rotation->first > tokens ||
            rotation->tokens > tokens - rotation->first)
            return SVDCACHE_ERR_BAD_SHAPE;
    }
    if (batch == 0 || tokens == 0) return SVDCACHE_OK;
    int rc = check_heads(Q, batch, tokens, dtype, false);
    if (!rc) rc = check_heads(Q_out, batch, tokens, dtype, true);
    if (!rc && K) rc = check_heads(K, batch, tokens, dtype, false);
    if (!rc && K) rc = check_heads(K_out, batch, tokens, dtype, true);
    if (!rc && (Q->heads != Q_out->heads || (K && K->heads != K_out->heads))) rc = SVDCACHE_ERR_BAD_SHAPE;
    if (!rc && (!in_place_or_apart(Q, Q_out, batch, tokens) || (K && !in_place_or_apart(K, K_out, batch, tokens)))) rc = SVDCACHE_ERR_INVALID_ARG;
    if (!rc && ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight)))) rc = SVDCACHE_ERR_BAD_ALIGN;
    if (rc) return rc;
    if (rotation && rotation->tokens > 0) {
        if (!rotation->table) return SVDCACHE_ERR_INVALID_ARG;
        if (rotation->batch_stride < 0 || rotation->batch_stride > (1LL << 40) || rotation->token_stride > (1LL << 36) ||
            (rotation->tokens > 1 && rotation->token_stride < rotation->r))
            return SVDCACHE_ERR_BAD_SHAPE;
        if (!aligned16(rotation->table) || (batch > 1 && rotation->batch_stride % 4) || (rotation->tokens > 1 && rotation->token_stride % 4))
            return SVDCACHE_ERR_BAD_ALIGN;
    }
    const svdcache_heads *const in[2] = {Q, K}, *const out[2] = {Q_out, K_out};
    const float *const weight[2] = {q_weight, k_weight};
    return rotary_launch(in, out, weight, norm, eps, batch, tokens, dim, dtype, rotation, (cudaStream_t)stream);
}

int svdcache_rotary(const svdcache_heads *X, const svdcache_heads *out, int64_t batch, int64_t tokens, int dim, int dtype,
                    const svdcache_rotation *rotation, void *stream) {
    NvtxRange range("svdcache_rotary");
    if (!rotation) return SVDCACHE_ERR_INVALID_ARG;
    return run_rotary(X, out, nullptr, nullptr, nullptr, nullptr, false, 0.0f, batch, tokens, dim, dtype, rotation, stream);
}

int svdcache_qk_rmsnorm_rotary(const svdcache_heads *Q, const svdcache_heads *Q_out, const float *q_weight, const svdcache_heads *K,
                               const svdcache_heads *K_out, const float *k_weight, float eps, int64_t batch, int64_t tokens, int dim, int dtype,
                               const svdcache_rotation *rotation, void *stream) {
    NvtxRange range("svdcache_qk_rmsnorm_rotary");
    return run_rotary(Q, Q_out, q_weight, K, K_out, k_weight, true, eps, batch, tokens, dim, dtype, rotation, stream);
}

/* Blocks of different rank in one call: consecutive blocks of equal rank form one batched launch. */
int svdcache_full_step_ranked_batched(int nblocks, const void *F, int64_t ld, size_t F_stride, const void *basis,
                                      size_t basis_stride, void *state, size_t state_stride, float *C_out,
                                      size_t C_stride, int64_t N, int D, const int *k_per_block, int dtype,
                                      float beta, void *stream) {
    if (!k_per_block || nblocks < 1) return SVDCACHE_ERR_INVALID_ARG;
    for (int b0 = 0; b0 < nblocks;) {
        int b1 = b0 + 1;
        while (b1 < nblocks && k_per_block[b1] == k_per_block[b0]) ++b1;
        const int rc = svdcache_full_step_batched(
            b1 - b0, (const char *)F + (size_t)b0 * F_stride, ld, F_stride, (const char *)basis + (size_t)b0 * basis_stride,
            basis_stride, (char *)state + (size_t)b0 * state_stride, state_stride,
            C_out ? reinterpret_cast<float *>((char *)C_out + (size_t)b0 * C_stride) : nullptr, C_stride, N, D,
            k_per_block[b0], dtype, beta, stream);
        if (rc) return rc;
        b0 = b1;
    }
    return SVDCACHE_OK;
}

int svdcache_cached_step_ranked_batched(int nblocks, const void *state, size_t state_stride, const void *basis,
                                        size_t basis_stride, void *Fhat, int64_t ld, size_t Fhat_stride, int64_t N,
                                        int D, const int *k_per_block, int dtype, int steps_since_full, void *stream) {
    if (!k_per_block || nblocks < 1) return SVDCACHE_ERR_INVALID_ARG;
    for (int b0 = 0; b0 < nblocks;) {
        int b1 = b0 + 1;
        while (b1 < nblocks && k_per_block[b1] == k_per_block[b0]) ++b1;
        const int rc = svdcache_cached_step_batched(
            b1 - b0, (const char *)state + (size_t)b0 * state_stride, state_stride,
            (const char *)basis + (size_t)b0 * basis_stride, basis_stride, (char *)Fhat + (size_t)b0 * Fhat_stride, ld,
            Fhat_stride, N, D, k_per_block[b0], dtype, steps_since_full, stream);
        if (rc) return rc;
        b0 = b1;
    }
    return SVDCACHE_OK;
}

int svdcache_full_step(const void *F, int64_t ld, const void *basis, void *state, float *C_out, int64_t N,
                       int D, int k, int dtype, float beta, void *stream) {
    return svdcache_full_step_batched(1, F, ld, 0, basis, 0, state, 0, C_out, 0, N, D, k, dtype, beta, stream);
}

int svdcache_cached_step(const void *state, const void *basis, void *Fhat, int64_t ld, int64_t N, int D,
                         int k, int dtype, int steps_since_full, void *stream) {
    return svdcache_cached_step_batched(1, state, 0, basis, 0, Fhat, ld, 0, N, D, k, dtype, steps_since_full,
                                        stream);
}

}  // extern "C"
