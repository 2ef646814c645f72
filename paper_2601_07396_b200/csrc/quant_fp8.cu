// Eight-bit outputs of elementwise and row-wise work (format: fp8.cuh):
//   quantize_rows_kernel    a matrix as e4m3 with a scale per 1 x 128 group (activations)
//   quantize_tiles_kernel   the same with one scale per 128 x 128 tile, repeated for its rows (weights)
//   rmsnorm_kernel          h' = h + x;  y = h' * rsqrt(mean(h'^2) + eps) * w;  y as e4m3 with a scale per group
// All three read every input once and write every output once: bandwidth-bound.  The common step is a chunk of
// eight elements per thread, so that 16 neighbouring lanes hold one group and its maximum takes four shuffles.
// Arithmetic is fp32 throughout; h' is rounded to the I/O type only where it is stored, and y is formed from
// the unrounded h'.
#include "fp8.cuh"

namespace svdc {
namespace {

constexpr int kChunk = 8;                           // elements per thread and step: 16 bytes of bf16, 32 of fp32
constexpr int kGroupLanes = kFp8Group / kChunk;     // 16 lanes hold a group
constexpr int kThreads = 256;

template <bool BF16> struct Raw;                    // a chunk as it lies in memory
template <> struct Raw<true> { uint4 a; };
template <> struct Raw<false> { float4 a, b; };

template <bool BF16> __device__ __forceinline__ Raw<BF16> load_chunk(const void *row, int c0) {
    Raw<BF16> r;
    if constexpr (BF16) {
        r.a = *reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(row) + c0);
    } else {
        r.a = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(row) + c0);
        r.b = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(row) + c0 + 4);
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ void to_float(const Raw<BF16> &r, float (&v)[kChunk]) {
    if constexpr (BF16) {
        const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
        v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
        v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
    }
}
template <bool BF16> __device__ __forceinline__ void store_chunk(void *row, int c0, const float (&v)[kChunk]) {
    if constexpr (BF16) {
        __nv_bfloat162 p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(row) + c0) = *reinterpret_cast<const uint4 *>(p);
    } else {
        float *o = reinterpret_cast<float *>(row) + c0;
        *reinterpret_cast<float4 *>(o) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// chunk c0 of a row `cols` long, zeros beyond its end; a chunk that the end cuts is read element by element
template <bool BF16> __device__ __forceinline__ void load_cut_chunk(const void *row, int c0, int cols, float (&v)[kChunk]) {
    if (c0 + kChunk <= cols) {
        to_float<BF16>(load_chunk<BF16>(row, c0), v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        v[i] = 0.0f;
        if (c0 + i < cols) {
            if constexpr (BF16) v[i] = __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(row)[c0 + i]);
            else v[i] = reinterpret_cast<const float *>(row)[c0 + i];
        }
    }
}
__device__ __forceinline__ void store_cut_bytes(uint8_t *row, int c0, int cols, uint2 w) {
    if (c0 + kChunk <= cols) {
        *reinterpret_cast<uint2 *>(row + c0) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
        if (c0 + i < cols) row[c0 + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

__device__ __forceinline__ float largest(const float (&v)[kChunk]) {   // NaN is passed over, Inf is not
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) m = fmaxf(m, fabsf(v[i]));
    return m;
}
// over the 16 lanes of a group
__device__ __forceinline__ float group_max(float m) {
#pragma unroll
    for (int o = kGroupLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    return m;
}
__device__ __forceinline__ bool is_inf(float m) { return __float_as_uint(m) == 0x7F800000u; }
// the maximum over the group's finite values; elements that are Inf become NaN.  Called by whole warps.
__device__ __forceinline__ float finite_group_max(float (&v)[kChunk]) {
    float m = group_max(largest(v));
    if (__any_sync(0xFFFFFFFFu, is_inf(m))) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = fp8_nan_if_not_finite(v[i]);
        m = group_max(largest(v));
    }
    return m;
}
__device__ __forceinline__ uint2 scaled_bytes(const float (&v)[kChunk], uint32_t byte) {
    const float inv = fp8_inverse_scale(byte);
    uint2 w;
    w.x = fp8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    w.y = fp8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    return w;
}

// ------------------------------------------------------------------------------------------ quantiser ---

struct QuantArgs {
    const void *X;
    uint8_t *Q, *S;
    int64_t rows, ld, ldq;
    int cols, groups, rows_per_cta;
    int64_t pieces;
};

// A CTA takes rows_per_cta rows; 16 lanes take a group at a time.
template <bool BF16> __global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const QuantArgs a) {
    const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_cta;
    const int nrows = (int)(a.rows - row0 < a.rows_per_cta ? a.rows - row0 : a.rows_per_cta);
    const int units = nrows * a.groups, lane = threadIdx.x % kGroupLanes;
    constexpr int kAtOnce = kThreads / kGroupLanes;
    for (int u0 = 0; u0 < units; u0 += kAtOnce) {   // the same number of steps for every lane of a warp
        const int u = u0 + (int)threadIdx.x / kGroupLanes;
        const bool live = u < units;
        const int r = live ? u / a.groups : 0, g = live ? u - r * a.groups : 0;
        const int64_t m = row0 + r;
        const int c0 = g * kFp8Group + lane * kChunk;
        float v[kChunk] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (live)
            load_cut_chunk<BF16>(reinterpret_cast<const char *>(a.X) + (size_t)m * a.ld * (BF16 ? 2 : 4), c0, a.cols, v);
        const uint32_t byte = fp8_scale_byte(finite_group_max(v));
        if (live) {
            store_cut_bytes(a.Q + (size_t)m * a.ldq, c0, a.cols, scaled_bytes(v, byte));
            if (lane == 0) a.S[fp8_scale_offset(m, g, a.pieces)] = (uint8_t)byte;
        }
    }
}

// One CTA per 128 x 128 tile, held in registers between the maximum and the rounding.
template <bool BF16> __global__ void __launch_bounds__(kThreads) quantize_tiles_kernel(const QuantArgs a) {
    constexpr int kRowsAtOnce = kThreads / kGroupLanes, kSteps = kScaleRows / kRowsAtOnce;   // 16 rows, 8 steps
    __shared__ float part[kThreads / 32];
    const int64_t row0 = (int64_t)(blockIdx.x / a.groups) * kScaleRows;
    const int g = (int)(blockIdx.x % a.groups), lane = threadIdx.x % kGroupLanes;
    const int c0 = g * kFp8Group + lane * kChunk;
    float v[kSteps][kChunk];
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t m = row0 + i * kRowsAtOnce + threadIdx.x / kGroupLanes;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[i][j] = 0.0f;
        if (m < a.rows)
            load_cut_chunk<BF16>(reinterpret_cast<const char *>(a.X) + (size_t)m * a.ld * (BF16 ? 2 : 4), c0, a.cols, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) top = fmaxf(top, finite_group_max(v[i]));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, kGroupLanes));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, part[w]);
    const uint32_t byte = fp8_scale_byte(top);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t m = row0 + i * kRowsAtOnce + threadIdx.x / kGroupLanes;
        if (m < a.rows) store_cut_bytes(a.Q + (size_t)m * a.ldq, c0, a.cols, scaled_bytes(v[i], byte));
    }
    if (threadIdx.x < kScaleRows && row0 + threadIdx.x < a.rows)
        a.S[fp8_scale_offset(row0 + threadIdx.x, g, a.pieces)] = (uint8_t)byte;
}

// ------------------------------------------------------------------- residual addition and RMS norm ---

struct NormArgs {
    const void *H, *X;      // X null: no addition
    void *H_out;            // null: h' is not stored
    const float *weight;    // null: ones
    uint8_t *Q, *S;
    int64_t ldh, ldx, ldo, ldq, rows;
    int D;
    float eps;
    int64_t pieces;
};

// TPR threads per row, V chunks of 8 elements per thread, held in fp32 registers from the load to the rounding.
template <bool BF16, int TPR, int V> __global__ void __launch_bounds__(TPR > kThreads ? TPR : kThreads) rmsnorm_kernel(const NormArgs a) {
    constexpr int kCta = TPR > kThreads ? TPR : kThreads, kRows = kCta / TPR, kWarps = TPR / 32;
    __shared__ float part[kCta / 32];
    const int64_t m = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    const int t = threadIdx.x % TPR;
    const bool live = m < a.rows;
    constexpr int e = BF16 ? 2 : 4;
    const char *h_row = reinterpret_cast<const char *>(a.H) + (size_t)m * a.ldh * e;
    const char *x_row = reinterpret_cast<const char *>(a.X) + (size_t)m * a.ldx * e;
    float v[V][kChunk];
    float sum = 0.0f;
    {
        Raw<BF16> rh[V], rx[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * TPR + t) * kChunk;
            if (live && c0 < a.D) {
                rh[j] = load_chunk<BF16>(h_row, c0);
                if (a.X) rx[j] = load_chunk<BF16>(x_row, c0);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * TPR + t) * kChunk;
            const bool in = live && c0 < a.D;
            float x[kChunk];
            if (in) to_float<BF16>(rh[j], v[j]);
            if (in && a.X) {
                to_float<BF16>(rx[j], x);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[j][i] += x[i];
            }
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                if (!in) v[j][i] = 0.0f;
                sum = fmaf(v[j][i], v[j][i], sum);
            }
            if (in && a.H_out) store_chunk<BF16>(reinterpret_cast<char *>(a.H_out) + (size_t)m * a.ldo * e, c0, v[j]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if constexpr (kWarps > 1) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
        __syncthreads();
        const int w0 = threadIdx.x / TPR * kWarps;
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += part[w0 + w];
    }
    const float inv_rms = rsqrtf(sum / (float)a.D + a.eps);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * TPR + t) * kChunk;
        const bool in = live && c0 < a.D;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[j][i] *= inv_rms;
        if (in && a.weight) {
            const float4 w0 = *reinterpret_cast<const float4 *>(a.weight + c0), w1 = *reinterpret_cast<const float4 *>(a.weight + c0 + 4);
            v[j][0] *= w0.x; v[j][1] *= w0.y; v[j][2] *= w0.z; v[j][3] *= w0.w;
            v[j][4] *= w1.x; v[j][5] *= w1.y; v[j][6] *= w1.z; v[j][7] *= w1.w;
        }
        if (!in) {   // lanes beyond the row hold 0 * inv_rms, which is not 0 in a row that is not finite
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[j][i] = 0.0f;
        }
        const uint32_t byte = fp8_scale_byte(finite_group_max(v[j]));
        if (in) {
            *reinterpret_cast<uint2 *>(a.Q + (size_t)m * a.ldq + c0) = scaled_bytes(v[j], byte);
            if (t % kGroupLanes == 0) a.S[fp8_scale_offset(m, c0 / kFp8Group, a.pieces)] = (uint8_t)byte;
        }
    }
}

template <bool BF16, int TPR> int norm_launch_v(const NormArgs &a, int v, cudaStream_t s) {
    constexpr int kCta = TPR > kThreads ? TPR : kThreads;
    const int64_t grid = (a.rows + kCta / TPR - 1) / (kCta / TPR);
    if (grid > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    switch (v) {
        case 1: rmsnorm_kernel<BF16, TPR, 1><<<(unsigned)grid, kCta, 0, s>>>(a); break;
        case 2: rmsnorm_kernel<BF16, TPR, 2><<<(unsigned)grid, kCta, 0, s>>>(a); break;
        case 3: rmsnorm_kernel<BF16, TPR, 3><<<(unsigned)grid, kCta, 0, s>>>(a); break;
        default: rmsnorm_kernel<BF16, TPR, 4><<<(unsigned)grid, kCta, 0, s>>>(a); break;
    }
    count_launch();
    return check_last_launch();
}

// The fewest threads per row (a power of two of warps) that hold a row in four chunks each.
template <bool BF16> int norm_launch(const NormArgs &a, cudaStream_t s) {
    const int chunks = a.D / kChunk;
    int tpr = 32;
    while ((chunks + tpr - 1) / tpr > 4) tpr *= 2;
    const int v = (chunks + tpr - 1) / tpr;
    switch (tpr) {
        case 32: return norm_launch_v<BF16, 32>(a, v, s);
        case 64: return norm_launch_v<BF16, 64>(a, v, s);
        case 128: return norm_launch_v<BF16, 128>(a, v, s);
        case 256: return norm_launch_v<BF16, 256>(a, v, s);
        default: return norm_launch_v<BF16, 512>(a, v, s);
    }
}

}  // namespace

int quantize_fp8_launch(const void *X, int64_t rows, int cols, int64_t ld, int dtype, int tile_rows, void *Q, int64_t ldq,
                        void *S, cudaStream_t s) {
    QuantArgs a{};
    a.X = X; a.Q = (uint8_t *)Q; a.S = (uint8_t *)S; a.rows = rows; a.ld = ld; a.ldq = ldq; a.cols = cols;
    a.groups = (int)fp8_groups(cols); a.pieces = fp8_piece_cols(cols);
    const bool bf = dtype == SVDCACHE_BF16;
    if (tile_rows == 1) {
        // about four steps per CTA, so that each warp has several loads to wait for
        constexpr int kUnits = 4 * kThreads / kGroupLanes;
        a.rows_per_cta = a.groups >= kUnits ? 1 : kUnits / a.groups;
        const int64_t grid = (rows + a.rows_per_cta - 1) / a.rows_per_cta;
        if (grid > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
        if (bf) quantize_rows_kernel<true><<<(unsigned)grid, kThreads, 0, s>>>(a);
        else quantize_rows_kernel<false><<<(unsigned)grid, kThreads, 0, s>>>(a);
    } else {
        const int64_t grid = (rows + kScaleRows - 1) / kScaleRows * a.groups;
        if (grid > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
        if (bf) quantize_tiles_kernel<true><<<(unsigned)grid, kThreads, 0, s>>>(a);
        else quantize_tiles_kernel<false><<<(unsigned)grid, kThreads, 0, s>>>(a);
    }
    count_launch();
    return check_last_launch();
}

int rmsnorm_fp8_launch(const void *H, int64_t ldh, const void *X, int64_t ldx, void *H_out, int64_t ldo, const float *weight,
                       float eps, void *Q, int64_t ldq, void *S, int64_t rows, int D, int dtype, cudaStream_t s) {
    NormArgs a{};
    a.H = H; a.X = X; a.H_out = H_out; a.weight = weight; a.Q = (uint8_t *)Q; a.S = (uint8_t *)S;
    a.ldh = ldh; a.ldx = ldx; a.ldo = ldo; a.ldq = ldq; a.rows = rows; a.D = D; a.eps = eps; a.pieces = fp8_piece_cols(D);
    return dtype == SVDCACHE_BF16 ? norm_launch<true>(a, s) : norm_launch<false>(a, s);
}

}  // namespace svdc
