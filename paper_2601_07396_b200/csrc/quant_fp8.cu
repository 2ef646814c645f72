// Eight-bit outputs of elementwise and row-wise work (format: fp8.cuh):
//   rows_kernel<.., false>   a matrix as e4m3 with a scale per 1 x 128 group (activations)
//   rows_kernel<.., true>    h' = h + x;  y = h' * rsqrt(mean(h'^2) + eps) * w;  y as e4m3 with a scale per group
//   tiles_kernel             a matrix with one scale per 128 x 128 tile, repeated for its rows (weights)
// All of it reads every input once and writes every output once: bandwidth-bound.  The common step is a chunk of
// eight elements per thread, so that 16 neighbouring lanes hold one group and its maximum takes four shuffles.
// Arithmetic is fp32 throughout; h' is rounded to the I/O type only where it is stored, and y is formed from
// the unrounded h'.
#include <cstring>
#include <type_traits>

#include "fp8.cuh"

namespace svdc {
namespace {

constexpr int kChunk = 8;                           // elements per thread and step: 16 bytes of bf16, 32 of fp32
constexpr int kGroupLanes = kFp8Group / kChunk;     // 16 lanes hold a group
constexpr int kThreads = 256;                       // of a CTA of tiles_kernel
constexpr int kRowWarps = 4;                        // of a CTA of rows_kernel, or what one row takes where that is more
constexpr int kMaxCta = 512;                        // 16 warps of four chunks per lane: a row of 16384

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

// Chunk c0 of a row `cols` long, zeros beyond its end and where `live` is false.  CUT: cols is not a multiple of 8,
// so that the end may cut a chunk, which is then read element by element.
template <bool BF16, bool CUT>
__device__ __forceinline__ Raw<BF16> load_live_chunk(const void *row, int c0, int cols, bool live) {
    Raw<BF16> r{};
    if (live && c0 + (CUT ? kChunk : 1) <= cols) r = load_chunk<BF16>(row, c0);
    else if (CUT && live) {
        using T = typename std::conditional<BF16, __nv_bfloat16, float>::type;
        T e[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) e[i] = c0 + i < cols ? reinterpret_cast<const T *>(row)[c0 + i] : T(0.0f);
        memcpy(&r, e, sizeof(r));
    }
    return r;
}
template <bool CUT> __device__ __forceinline__ void store_live_bytes(uint8_t *row, int c0, int cols, uint2 w) {
    if (c0 + (CUT ? kChunk : 1) <= cols) *reinterpret_cast<uint2 *>(row + c0) = w;
    else if (CUT) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (c0 + i < cols) row[c0 + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
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
__device__ __forceinline__ void drop_infinities(float (&v)[kChunk]) {   // they become NaN, which the format has
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = fp8_nan_if_not_finite(v[i]);
}
__device__ __forceinline__ uint2 scaled_bytes(const float (&v)[kChunk], uint32_t byte) {
    const float inv = fp8_inverse_scale(byte);
    uint2 w;
    w.x = fp8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    w.y = fp8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    return w;
}

// ----------------------------------------------------------------------------------------------- rows ---

struct RowsArgs {
    const void *H, *X;      // NORM: X null: no addition
    void *H_out;            // NORM: null: h' is not stored
    const float *weight;    // NORM: null: ones
    uint8_t *Q, *S;
    int64_t ldh, ldx, ldo, ldq, rows;
    int cols, warps;        // warps per row
    float eps;
    int64_t pieces;
};

// A row (NORM) or a segment of one (blockIdx.y) belongs to a.warps warps, V chunks per lane, consecutive runs of 32
// chunks per warp and step: 64 bytes of bf16 in flight per lane and input at V = 4.  Where a row is no more than one
// warp's and V is less, a warp takes R rows at once instead (V R = 4: 100000 x 264: 35 -> 29 us).  Values stay in fp32
// registers from the load to the rounding.
template <bool BF16, bool CUT, bool NORM, int V, int R> __global__ void __launch_bounds__(kMaxCta) rows_kernel(const RowsArgs a) {
    __shared__ float part[kMaxCta / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int warps = R > 1 ? 1 : a.warps;
    const int in_cta = warp / warps, at = warp - in_cta * warps;            // row of the CTA, warp of the row
    const int64_t m0 = ((int64_t)blockIdx.x * (blockDim.x / 32 / warps) + in_cta) * R;
    const int step0 = (blockIdx.y * warps + at) * V, first = (step0 * 32 + lane) * kChunk;     // this lane's columns: first + 256 j
    constexpr int e = BF16 ? 2 : 4;
    float v[R][V][kChunk];
    previous_done();
    next_may_launch();
    {
        Raw<BF16> rh[R][V], rx[NORM ? R : 1][NORM ? V : 1];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const char *h_row = reinterpret_cast<const char *>(a.H) + (size_t)(m0 + r) * a.ldh * e;
#pragma unroll
            for (int j = 0; j < V; ++j) rh[r][j] = load_live_chunk<BF16, CUT>(h_row, first + 256 * j, a.cols, m0 + r < a.rows);
        }
        if constexpr (NORM) {
            if (a.X) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const char *x_row = reinterpret_cast<const char *>(a.X) + (size_t)(m0 + r) * a.ldx * e;
#pragma unroll
                    for (int j = 0; j < V; ++j) rx[r][j] = load_live_chunk<BF16, CUT>(x_row, first + 256 * j, a.cols, m0 + r < a.rows);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                to_float<BF16>(rh[r][j], v[r][j]);
                if constexpr (NORM) {
                    if (a.X) {
                        float x[kChunk];
                        to_float<BF16>(rx[r][j], x);
#pragma unroll
                        for (int i = 0; i < kChunk; ++i) v[r][j][i] += x[i];
                    }
                }
            }
    }
    if constexpr (NORM) {
        // The sum of squares as a tree: a lane's element i of each chunk in a chain of its own (at most four additions deep),
        // the eight chains in three, the lanes in five, the warps in four: fewer than 16 that depend on one another, where a
        // chain per lane and one across the warps made 52.  (Squares of 1 and 2^-24 in a row of 16384: off by 4 * 2^-24, not
        // 46 * 2^-24.  118800 x 3072 bf16 365.6 -> 369.4 us, 4000 x 16384 80.0 -> 78.3.)
        float sum[R], inv_rms[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float chain[kChunk];
#pragma unroll
            for (int j = 0; j < V; ++j) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) chain[i] = j == 0 ? v[r][j][i] * v[r][j][i] : fmaf(v[r][j][i], v[r][j][i], chain[i]);
                if (a.H_out && m0 + r < a.rows && first + 256 * j < a.cols)
                    store_chunk<BF16>(reinterpret_cast<char *>(a.H_out) + (size_t)(m0 + r) * a.ldo * e, first + 256 * j, v[r][j]);
            }
            sum[r] = ((chain[0] + chain[1]) + (chain[2] + chain[3])) + ((chain[4] + chain[5]) + (chain[6] + chain[7]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] += __shfl_xor_sync(0xFFFFFFFFu, sum[r], o);
        if (R == 1 && warps > 1) {
            if (lane == 0) part[warp] = sum[0];
            __syncthreads();
            const int w = lane & (kMaxCta / 32 - 1);                         // 16 warps at most, so each half of the lanes sums all
            sum[0] = w < warps ? part[in_cta * warps + w] : 0.0f;
#pragma unroll
            for (int o = kMaxCta / 64; o > 0; o >>= 1) sum[0] += __shfl_xor_sync(0xFFFFFFFFu, sum[0], o);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) inv_rms[r] = rsqrtf(sum[r] / (float)a.cols + a.eps);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const bool in = first + 256 * j < a.cols;
            float w[kChunk] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (a.weight && in) to_float<false>(load_chunk<false>(a.weight, first + 256 * j), w);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[r][j][i] = in ? v[r][j][i] * inv_rms[r] * w[i] : 0.0f;   // 0 * inv_rms is not 0 in every row
        }
    }
    float top[R][V], most = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            top[r][j] = group_max(largest(v[r][j]));
            most = fmaxf(most, top[r][j]);
        }
    if (__any_sync(0xFFFFFFFFu, is_inf(most))) {   // a group's scale is that of its finite values
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                drop_infinities(v[r][j]);
                top[r][j] = group_max(largest(v[r][j]));
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t m = m0 + r;
        const bool live = m < a.rows;
        uint8_t *q_row = a.Q + (size_t)m * a.ldq;
        uint8_t *s_row = a.S + fp8_scale_offset(m, 0, a.pieces);
        uint32_t byte[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            byte[j] = fp8_scale_byte(top[r][j]);
            if (live) store_live_bytes<CUT>(q_row, first + 256 * j, a.cols, scaled_bytes(v[r][j], byte[j]));
        }
        // group 2 (step0 + j) + lane / 16.  Two steps from an even one on make a whole word of four scales, unless the
        // row ends inside it.
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int g = 2 * (step0 + j), off = g / kScaleGroups * kScalePieceBytes + (g & 3);
            if (V % 2 == 0 && (j & 1) == 0 && (g + 3) * kFp8Group < a.cols) {
                const uint32_t both = byte[j] | byte[(j + 1) % V] << 16, other = __shfl_xor_sync(0xFFFFFFFFu, both, 16);
                if (live && lane == 0) *reinterpret_cast<uint32_t *>(s_row + off) = both | other << 8;
                ++j;
            } else if (live && lane % kGroupLanes == 0 && first + 256 * j < a.cols) {
                s_row[off + lane / kGroupLanes] = (uint8_t)byte[j];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- tiles ---

struct TilesArgs {
    const void *X;
    uint8_t *Q, *S;
    int64_t rows, ld, ldq;
    int cols, groups;
    int64_t pieces;
};

// One CTA per 128 x 128 tile, held in registers as it was read between the maximum and the rounding.
template <bool BF16, bool CUT> __global__ void __launch_bounds__(kThreads) tiles_kernel(const TilesArgs a) {
    constexpr int kRowsAtOnce = kThreads / kGroupLanes, kSteps = kScaleRows / kRowsAtOnce;   // 16 rows, 8 steps
    __shared__ float part[kThreads / 32];
    const int64_t row0 = (int64_t)(blockIdx.x / a.groups) * kScaleRows;
    const int g = (int)(blockIdx.x % a.groups), lane = threadIdx.x % kGroupLanes;
    const int c0 = g * kFp8Group + lane * kChunk;
    Raw<BF16> raw[kSteps];
    previous_done();
    next_may_launch();
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t m = row0 + i * kRowsAtOnce + threadIdx.x / kGroupLanes;
        raw[i] = load_live_chunk<BF16, CUT>(reinterpret_cast<const char *>(a.X) + (size_t)m * a.ld * (BF16 ? 2 : 4), c0, a.cols, m < a.rows);
    }
    float v[kChunk], top = 0.0f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        to_float<BF16>(raw[i], v);
        top = fmaxf(top, largest(v));
    }
    const bool inf = __syncthreads_or(is_inf(top));   // an Inf anywhere in the tile: the maximum over what is finite
    if (inf) {
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            to_float<BF16>(raw[i], v);
            drop_infinities(v);
            top = fmaxf(top, largest(v));
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, part[w]);
    const uint32_t byte = fp8_scale_byte(top);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t m = row0 + i * kRowsAtOnce + threadIdx.x / kGroupLanes;
        to_float<BF16>(raw[i], v);
        if (inf) drop_infinities(v);
        if (m < a.rows) store_live_bytes<CUT>(a.Q + (size_t)m * a.ldq, c0, a.cols, scaled_bytes(v, byte));
    }
    if (threadIdx.x < kScaleRows && row0 + threadIdx.x < a.rows)
        a.S[fp8_scale_offset(row0 + threadIdx.x, g, a.pieces)] = (uint8_t)byte;
}

// Lanes hold four chunks (8 KB of values per warp and input: the loads that hide the memory's latency at eight warps a
// row of the CTA); fewer where the row is short.  Rows longer than `most` warps are cut into segments, which a norm
// cannot be.
template <bool BF16, bool CUT, bool NORM> int rows_launch(RowsArgs a, int most, cudaStream_t s) {
    constexpr int kSteps = 4;
    const int steps = (a.cols + 255) / 256, segments = (steps + most * kSteps - 1) / (most * kSteps);
    const int per = (steps + segments - 1) / segments;               // steps of a segment
    a.warps = (per + kSteps - 1) / kSteps;
    const int v = (per + a.warps - 1) / a.warps;
    const int each = v == 1 ? 4 : v == 2 ? 2 : 1;                    // rows of a warp (two or more warps per row: v is 3 or 4)
    const int at_once = a.warps < kRowWarps ? kRowWarps / a.warps : 1;
    const int64_t grid = (a.rows + at_once * each - 1) / (at_once * each);
    const dim3 blocks((unsigned)grid, (unsigned)((steps + a.warps * v - 1) / (a.warps * v))), threads(32 * a.warps * at_once);
    switch (v) {
        case 1: return launch_early(rows_kernel<BF16, CUT, NORM, 1, 4>, blocks, threads, 0, 1, s, a);
        case 2: return launch_early(rows_kernel<BF16, CUT, NORM, 2, 2>, blocks, threads, 0, 1, s, a);
        case 3: return launch_early(rows_kernel<BF16, CUT, NORM, 3, 1>, blocks, threads, 0, 1, s, a);
        default: return launch_early(rows_kernel<BF16, CUT, NORM, 4, 1>, blocks, threads, 0, 1, s, a);
    }
}

template <bool BF16> int tiles_launch(const TilesArgs &a, cudaStream_t s) {
    const int64_t grid = (a.rows + kScaleRows - 1) / kScaleRows * a.groups;
    if (grid > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    return launch_early(a.cols % kChunk ? tiles_kernel<BF16, true> : tiles_kernel<BF16, false>, dim3((unsigned)grid), dim3(kThreads), 0, 1, s, a);
}

}  // namespace

int quantize_fp8_launch(const void *X, int64_t rows, int cols, int64_t ld, int dtype, int tile_rows, void *Q, int64_t ldq,
                        void *S, cudaStream_t s) {
    const bool bf = dtype == SVDCACHE_BF16;
    if (tile_rows != 1) {
        TilesArgs a{};
        a.X = X; a.Q = (uint8_t *)Q; a.S = (uint8_t *)S; a.rows = rows; a.ld = ld; a.ldq = ldq; a.cols = cols;
        a.groups = (int)fp8_groups(cols); a.pieces = fp8_piece_cols(cols);
        return bf ? tiles_launch<true>(a, s) : tiles_launch<false>(a, s);
    }
    RowsArgs a{};
    a.H = X; a.Q = (uint8_t *)Q; a.S = (uint8_t *)S; a.rows = rows; a.ldh = ld; a.ldq = ldq; a.cols = cols; a.pieces = fp8_piece_cols(cols);
    if (cols % kChunk) return bf ? rows_launch<true, true, false>(a, 1, s) : rows_launch<false, true, false>(a, 1, s);
    return bf ? rows_launch<true, false, false>(a, 1, s) : rows_launch<false, false, false>(a, 1, s);
}

int rmsnorm_fp8_launch(const void *H, int64_t ldh, const void *X, int64_t ldx, void *H_out, int64_t ldo, const float *weight,
                       float eps, void *Q, int64_t ldq, void *S, int64_t rows, int D, int dtype, cudaStream_t s) {
    RowsArgs a{};
    a.H = H; a.X = X; a.H_out = H_out; a.weight = weight; a.Q = (uint8_t *)Q; a.S = (uint8_t *)S;
    a.ldh = ldh; a.ldx = ldx; a.ldo = ldo; a.ldq = ldq; a.rows = rows; a.cols = D; a.eps = eps; a.pieces = fp8_piece_cols(D);
    return dtype == SVDCACHE_BF16 ? rows_launch<true, false, true>(a, kMaxCta / 32, s) : rows_launch<false, false, true>(a, kMaxCta / 32, s);
}

}  // namespace svdc
