// Between the product that makes queries and keys and the attention that reads them:
//   table_kernel   (cos, sin) of pos * base^(-2 i / d) for each token and pair, positions of several axes
//   heads_kernel   y = x * rsqrt(mean(x^2) + eps) * w for each head (NORM), then the rotation of y's pairs by the table:
//                  (a, b) -> (a c - b s, a s + b c); its inverse, which is its gradient too, takes -s for s
// Both read every input once and write every output once: bandwidth-bound.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "fp8.cuh"

namespace svdc {
namespace {

// ---------------------------------------------------------------------------------------------- table ---

constexpr int kTableThreads = 256, kTableSteps = 4;      // of a CTA; tokens that a thread has under way
constexpr int kTableCtas = 592;                          // at most: all that are at work at once (of int64 positions 444 are)

struct TableArgs {
    double2 turns[SVDCACHE_ROTARY_MAX_DIM / 4];          // of two neighbouring pairs, per unit of position
    const void *positions;
    float *table;
    int64_t tokens, ld, ldt;
    int columns, at_once;                                // r / 4; tokens that the CTA's threads hold at a time
    int begins[SVDCACHE_ROTARY_MAX_AXES];                // an axis's first pair (beyond the last axis: of no pair)
};

// cos and sin of 2 pi t.  t is reduced in 64 bits to an eighth of a turn, so that far positions cost nothing, and the rest x,
// |x| <= pi / 4, rounded to 32 (off by pi / 4 2^-24).  There Taylor's series to x^9 and x^10 leave 2^-29; both values are good to
// 2^-23.  The quarter is rounded by adding 1.5 * 2^52, whose last bits then are the whole number: conversions between 64-bit
// floats and integers are many times slower than additions.  (sincospif in the series' place reduces its argument again, on the
// pipe that is busiest here: 118800 tokens 21.8 us.)
__device__ __forceinline__ float2 cos_sin_of_turns(double t) {
    constexpr double kWhole = 6755399441055744.0;
    const double shifted = fma(t, 4.0, kWhole);
    const int q = __double2loint(shifted);
    float x = (float)(fma(shifted - kWhole, -0.25, t) * 6.283185307179586476925);
    x = fabsf(x) > 1.0f ? 0.0f : x;                                          // t beyond 2^49, where kWhole rounds to no whole number
    const float z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const float2 v = q & 1 ? make_float2(s, c) : make_float2(c, s);          // q: (c, s), (-s, c), (-c, -s), (s, -c)
    return make_float2(__uint_as_float(__float_as_uint(v.x) ^ ((uint32_t)(q + 1) << 30 & 0x80000000u)),
                       __uint_as_float(__float_as_uint(v.y) ^ ((uint32_t)q << 30 & 0x80000000u)));
}

// A thread keeps two neighbouring pairs, whose speeds it reads once (lanes that read different words of the parameters wait
// for one another: reading them for four tokens each made 48 us of 118800 tokens), and walks over the tokens, the next ones'
// positions on their way meanwhile (118800 tokens of 64 pairs: 20 -> 16 us, 3.9 TB/s, int64 18).  The bytes
// would take 9.6 and the 2.6 64-bit and 40 32-bit instructions of a pair 8.6 of issue, beside one another; the rest is half of an SM's threads, or
// fewer (64 registers, 76 for int64), and 592 CTAs that walk 6.3 rounds as seven.
template <typename P> __global__ void __launch_bounds__(kTableThreads) table_kernel(const __grid_constant__ TableArgs a) {
    const int row = (int)threadIdx.x / a.columns, column = (int)threadIdx.x - row * a.columns;
    if (row >= a.at_once) return;
    const double2 turn = a.turns[column];
    int axis0 = -1, axis1 = -1;
#pragma unroll
    for (int i = 0; i < SVDCACHE_ROTARY_MAX_AXES; ++i) {
        axis0 += 2 * column >= a.begins[i];
        axis1 += 2 * column + 1 >= a.begins[i];
    }
    previous_done();
    next_may_launch();
    const int64_t n0 = (int64_t)blockIdx.x * (a.at_once * kTableSteps) + row, step = (int64_t)gridDim.x * (a.at_once * kTableSteps);
    const P *in = reinterpret_cast<const P *>(a.positions) + n0 * a.ld;
    float *out = a.table + n0 * a.ldt + 4 * column;
    const int64_t in_step = a.at_once * a.ld, out_step = a.at_once * a.ldt;
    int64_t left = a.tokens - n0;
    P p0[kTableSteps], p1[kTableSteps];
    auto request = [&] {
#pragma unroll
        for (int i = 0; i < kTableSteps; ++i) {
            if (i * a.at_once >= left) continue;
            p0[i] = in[i * in_step + axis0];
            p1[i] = in[i * in_step + axis1];
        }
    };
    request();
    while (left > 0) {
        double x0[kTableSteps], x1[kTableSteps];
        const int64_t now = left;
#pragma unroll
        for (int i = 0; i < kTableSteps; ++i) {
            x0[i] = x1[i] = (double)p0[i];
            if (axis0 != axis1) x1[i] = (double)p1[i];
        }
        left -= step;
        in += step * a.ld;
        request();                                       // of the next round, on their way meanwhile
#pragma unroll
        for (int i = 0; i < kTableSteps; ++i) {
            if (i * a.at_once >= now) break;
            const float2 u = cos_sin_of_turns(x0[i] * turn.x), v = cos_sin_of_turns(x1[i] * turn.y);
            *reinterpret_cast<float4 *>(out + i * out_step) = make_float4(u.x, u.y, v.x, v.y);
        }
        out += step * a.ldt;
    }
}

// ---------------------------------------------------------------------------------------------- heads ---

// Heads of a CTA's tokens: eight of bf16 or four of fp32, 128 bytes in flight per lane (118800 x 48 x 128 bf16 with norm: 669, 550, 489
// us at 2, 4, 8, and 463 with the heads of a token in neighbouring CTAs: 6.4 TB/s in a short run, 5.6 to 5.9 in long ones, 502 to 532 us), fewer where that would leave SMs without work
// (one token of 24 heads: 2.2 us with eight, 1.5 with one).
constexpr int kHeadThreads = 128, kFillingCtas = 592;

struct HeadsOf {                 // queries or keys: [batch, tokens, heads, dim], strides in elements
    const void *in;
    void *out;
    int64_t in_batch, in_token, in_head, out_batch, out_token, out_head;
    const float *weight;         // NORM: null: ones
    int heads, each;             // heads that a CTA takes at most
    uint32_t blocks;             // of heads
};
struct HeadsArgs {
    HeadsOf of[2];
    const float *table;
    int64_t table_batch, table_token, first, count;      // tokens [first, first + count) are rotated
    uint32_t tokens, blocks;
    int dim, r;
    int lanes, groups, reach;    // lanes of a head, heads of a warp; half of the power of two that holds `lanes`, or 0 where they are one
    float inv_dim, eps, sign;    // sign -1: the inverse rotation
};

// eight elements of a head as fp32: a run of eight, or two runs of four, `at` and `at2`
template <bool BF16> struct Eight {
    static constexpr int kWords = BF16 ? 2 : 4;          // of a run of four
    uint32_t w[2][kWords];
};
template <bool BF16, bool HALVES> __device__ __forceinline__ Eight<BF16> load_eight(const void *p, int64_t at, int64_t at2) {
    Eight<BF16> e;
    if constexpr (BF16) {
        const __nv_bfloat16 *x = reinterpret_cast<const __nv_bfloat16 *>(p);
        if constexpr (HALVES) {
            const uint2 lo = *reinterpret_cast<const uint2 *>(x + at), hi = *reinterpret_cast<const uint2 *>(x + at2);
            e.w[0][0] = lo.x; e.w[0][1] = lo.y; e.w[1][0] = hi.x; e.w[1][1] = hi.y;
        } else {
            const uint4 v = *reinterpret_cast<const uint4 *>(x + at);
            e.w[0][0] = v.x; e.w[0][1] = v.y; e.w[1][0] = v.z; e.w[1][1] = v.w;
        }
    } else {
        const float *x = reinterpret_cast<const float *>(p);
        const uint4 lo = *reinterpret_cast<const uint4 *>(x + at), hi = *reinterpret_cast<const uint4 *>(x + at2);
        e.w[0][0] = lo.x; e.w[0][1] = lo.y; e.w[0][2] = lo.z; e.w[0][3] = lo.w;
        e.w[1][0] = hi.x; e.w[1][1] = hi.y; e.w[1][2] = hi.z; e.w[1][3] = hi.w;
    }
    return e;
}
template <bool BF16> __device__ __forceinline__ void to_float(const Eight<BF16> &e, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < Eight<BF16>::kWords; ++i) {
            if constexpr (BF16) {
                v[4 * h + 2 * i] = __uint_as_float(e.w[h][i] << 16);
                v[4 * h + 2 * i + 1] = __uint_as_float(e.w[h][i] & 0xFFFF0000u);
            } else {
                v[4 * h + i] = __uint_as_float(e.w[h][i]);
            }
        }
}
template <bool BF16, bool HALVES> __device__ __forceinline__ void store_eight(void *p, int64_t at, int64_t at2, const float (&v)[8]) {
    if constexpr (BF16) {
        __nv_bfloat16 *x = reinterpret_cast<__nv_bfloat16 *>(p);
        __nv_bfloat162 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        if constexpr (HALVES) {
            *reinterpret_cast<uint2 *>(x + at) = *reinterpret_cast<const uint2 *>(w);
            *reinterpret_cast<uint2 *>(x + at2) = *reinterpret_cast<const uint2 *>(w + 2);
        } else {
            *reinterpret_cast<uint4 *>(x + at) = *reinterpret_cast<const uint4 *>(w);
        }
    } else {
        float *x = reinterpret_cast<float *>(p);
        *reinterpret_cast<float4 *>(x + at) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(x + at2) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// A lane holds eight elements of a head that make four whole pairs: a run of eight for pairs of neighbours, four of either
// half for pairs of halves (and a run of eight of what is not rotated); `lanes` lanes hold a head and stay with its token, as
// many tokens of a warp side by side as have room (60000 x 32 heads of 72: 151 us with 16 lanes a head, 112 with 9), so that
// the token's row of the table and the weights lie in registers for up to R of its heads, whose loads are all under way at
// once.  Values stay in fp32 from the load to the one rounding.
template <bool BF16, bool NORM, bool HALVES, int R> __global__ void __launch_bounds__(kHeadThreads) heads_kernel(const __grid_constant__ HeadsArgs a) {
    const uint32_t tb = blockIdx.x / a.blocks, hb = blockIdx.x - tb * a.blocks;
    const bool second = hb >= a.of[0].blocks;
    const HeadsOf &h = a.of[second];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = lane / a.lanes, in_head = lane - group * a.lanes, chunks = a.dim / 8;
    const bool turns = in_head < a.r / 8;                                    // this lane's elements are rotated
    const int at = HALVES && turns ? 4 * in_head : 8 * in_head, at2 = HALVES && turns ? a.r / 2 + at : at + 4;
    const uint32_t token = (tb * (kHeadThreads / 32) + warp) * (uint32_t)a.groups + (uint32_t)group;
    const int head0 = (int)(hb - (second ? a.of[0].blocks : 0u)) * h.each, count = min(h.each, h.heads - head0);
    const bool live = group < a.groups && in_head < chunks && token < a.tokens;
    constexpr int e = BF16 ? 2 : 4;
    const char *in = reinterpret_cast<const char *>(h.in) + ((int64_t)blockIdx.z * h.in_batch + (int64_t)token * h.in_token + (int64_t)head0 * h.in_head) * e;
    char *out = reinterpret_cast<char *>(h.out) + ((int64_t)blockIdx.z * h.out_batch + (int64_t)token * h.out_token + (int64_t)head0 * h.out_head) * e;
    const int64_t place = (int64_t)token - a.first;
    const bool rotate = live && turns && place >= 0 && place < a.count;
    previous_done();
    next_may_launch();
    Eight<BF16> raw[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        raw[i] = Eight<BF16>{};
        if (live && i < count) raw[i] = load_eight<BF16, HALVES>(in + i * h.in_head * e, at, at2);
    }
    float4 t0 = make_float4(1.f, 0.f, 1.f, 0.f), t1 = t0;
    if (rotate) {
        const float4 *row = reinterpret_cast<const float4 *>(a.table + blockIdx.z * a.table_batch + place * a.table_token + 8 * in_head);
        t0 = __ldg(row);
        t1 = __ldg(row + 1);
    }
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (NORM && h.weight && live) {
        const float4 lo = __ldg(reinterpret_cast<const float4 *>(h.weight + at)), hi = __ldg(reinterpret_cast<const float4 *>(h.weight + at2));
        w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w; w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
    }
    const float c[4] = {t0.x, t0.z, t1.x, t1.z}, s[4] = {a.sign * t0.y, a.sign * t0.w, a.sign * t1.y, a.sign * t1.w};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (i >= count) break;                                               // the same for the whole CTA
        float v[8];
        to_float<BF16>(raw[i], v);
        if constexpr (NORM) {
            float sum = ((v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3])) + ((v[4] * v[4] + v[5] * v[5]) + (v[6] * v[6] + v[7] * v[7]));
            if (a.reach == 0) {
                for (int o = a.lanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            } else {
                for (int o = a.reach; o > 0; o >>= 1) {
                    const float other = __shfl_down_sync(0xFFFFFFFFu, sum, o);
                    if (in_head + o < a.lanes) sum += other;
                }
                sum = __shfl_sync(0xFFFFFFFFu, sum, lane - in_head);
            }
            const float inv_rms = rsqrtf(sum * a.inv_dim + a.eps);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * inv_rms * w[j];
        }
        if (rotate) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float &x = v[HALVES ? j : 2 * j], &y = v[HALVES ? 4 + j : 2 * j + 1];
                const float x0 = x;
                x = x0 * c[j] - y * s[j];
                y = x0 * s[j] + y * c[j];
            }
        }
        if (live) store_eight<BF16, HALVES>(out + i * h.out_head * e, at, at2, v);
    }
}

template <bool BF16, bool NORM, bool HALVES> int heads_launch(HeadsArgs a, int64_t batch, cudaStream_t s) {
    constexpr int R = BF16 ? 8 : 4;
    const int64_t per = kHeadThreads / 32 * a.groups, token_blocks = (a.tokens + per - 1) / per;
    for (int most = R;; most /= 2) {
        a.blocks = 0;
        for (HeadsOf &h : a.of) {
            h.blocks = (uint32_t)((h.heads + most - 1) / most);
            h.each = h.blocks ? (h.heads + (int)h.blocks - 1) / (int)h.blocks : 0;
            a.blocks += h.blocks;
        }
        if (most == 1 || token_blocks * a.blocks * batch >= kFillingCtas) break;
    }
    if (token_blocks * a.blocks > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    return launch_early(heads_kernel<BF16, NORM, HALVES, R>, dim3((unsigned)(token_blocks * a.blocks), 1, (unsigned)batch), dim3(kHeadThreads), 0, 1, s, a);
}

}  // namespace

int rotary_table_launch(const void *positions, int64_t tokens, int64_t ld, int type, int axes, const int *dims, const double *bases,
                        float *table, int64_t ldt, cudaStream_t s) {
    TableArgs a{};
    a.positions = positions; a.table = table; a.tokens = tokens; a.ld = ld; a.ldt = ldt;
    int pairs = 0;
    double *turns = &a.turns[0].x;
    for (int i = 0; i < SVDCACHE_ROTARY_MAX_AXES; ++i) {
        a.begins[i] = i < axes ? pairs : SVDCACHE_ROTARY_MAX_DIM;
        for (int j = 0; i < axes && j < dims[i] / 2; ++j) turns[pairs++] = std::pow(bases[i], -2.0 * j / dims[i]) / 6.283185307179586476925;
    }
    a.columns = pairs / 2;
    a.at_once = kTableThreads / a.columns;
    const int64_t each = (int64_t)a.at_once * kTableSteps, grid = std::min((tokens + each - 1) / each, (int64_t)kTableCtas);
    const dim3 blocks((unsigned)grid), threads(kTableThreads);
    if (type == SVDCACHE_POSITION_I32) return launch_early(table_kernel<int32_t>, blocks, threads, 0, 1, s, a);
    if (type == SVDCACHE_POSITION_I64) return launch_early(table_kernel<int64_t>, blocks, threads, 0, 1, s, a);
    return launch_early(table_kernel<float>, blocks, threads, 0, 1, s, a);
}

int rotary_launch(const svdcache_heads *const (&in)[2], const svdcache_heads *const (&out)[2], const float *const (&weight)[2], bool norm, float eps,
                  int64_t batch, int64_t tokens, int dim, int dtype, const svdcache_rotation *rotation, cudaStream_t s) {
    HeadsArgs a{};
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        HeadsOf &h = a.of[i];
        h.in = in[i]->data; h.in_batch = in[i]->batch_stride; h.in_token = in[i]->token_stride; h.in_head = in[i]->head_stride;
        h.out = out[i]->data; h.out_batch = out[i]->batch_stride; h.out_token = out[i]->token_stride; h.out_head = out[i]->head_stride;
        h.weight = weight[i]; h.heads = in[i]->heads;
    }
    a.sign = 1.0f;
    bool halves = false;
    if (rotation) {
        a.table = rotation->table; a.table_batch = rotation->batch_stride; a.table_token = rotation->token_stride;
        a.first = rotation->first; a.count = rotation->tokens; a.r = rotation->r;
        halves = (rotation->flags & SVDCACHE_ROTARY_HALVES) != 0;
        if (rotation->flags & SVDCACHE_ROTARY_INVERSE) a.sign = -1.0f;
    }
    a.tokens = (uint32_t)tokens; a.dim = dim; a.inv_dim = 1.0f / (float)dim; a.eps = eps;
    // as many lanes as the head has chunks where more heads then fit in a warp, else up to a power of two, whose sums take one step less
    // (60000 x 24 heads of 96: 125 us with 16 lanes, 138 with 12)
    int power = 1;
    while (8 * power < dim) power *= 2;
    const bool exact = 32 / (dim / 8) > 32 / power;
    a.lanes = exact ? dim / 8 : power;
    a.groups = 32 / a.lanes;
    a.reach = exact ? power / 2 : 0;
    const int kind = (dtype == SVDCACHE_BF16 ? 4 : 0) | (norm ? 2 : 0) | (halves ? 1 : 0);
    switch (kind) {
        case 0: return heads_launch<false, false, false>(a, batch, s);
        case 1: return heads_launch<false, false, true>(a, batch, s);
        case 2: return heads_launch<false, true, false>(a, batch, s);
        case 3: return heads_launch<false, true, true>(a, batch, s);
        case 4: return heads_launch<true, false, false>(a, batch, s);
        case 5: return heads_launch<true, false, true>(a, batch, s);
        case 6: return heads_launch<true, true, false>(a, batch, s);
        default: return heads_launch<true, true, true>(a, batch, s);
    }
}

}  // namespace svdc
