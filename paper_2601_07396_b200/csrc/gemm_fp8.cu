// Matrix product of two 8-bit matrices (format: fp8.cuh) on the tensor cores of sm_100a:
//     C[m, n] = act( sum_g sA[m, g] sB[n, g] sum_{k in g} A[m, k] B[n, k]  +  bias[n] )
// with act the identity or gelu(x) = x / (1 + exp(-2u)), u = sqrt(2 / pi) (x + 0.044715 x^3) (the tanh form), and
// C in fp32, bf16 or 8 bits again with a scale per row and 128 columns.  The scales are powers of two, so
// kind::mxf8f6f4 applies them: an MMA of K = 32 takes one scale byte per row of either operand, and a piece of
// 128 rows x 4 groups reaches tensor memory as it is stored (tcgen05.cp), one word per row whose byte g % 4 the
// four MMAs of group g name.  Sums are fp32 in tensor memory.
//
// tile_kernel: the lanes of the accumulator are 128 columns of C (rows of B), its columns 16, 32, 64 or 128 rows of C, so
// that few rows of C waste little tensor work (one row pays for 16, 33 for 64).  One CTA per tile; where that leaves SMs idle, the S CTAs of a
// cluster share a tile: CTA r takes the groups r, r + S, ... of K (together they read whole runs of B's rows), sends
// every CTA the rows of its sum that are that one's to finish (a bulk copy into its shared memory), and finishes its own
// share, adding the parts in rank order: no atomics, the same sum in every run.  No CTA leaves before all have their parts.
// Warps: 0 TMA producer, 1 MMA issuer, 2-5 accumulator -> shared memory; then all of them write C.
#include <algorithm>
#include <atomic>
#include <cstring>
#include <type_traits>

#include "fp8.cuh"
#include "umma.cuh"

namespace svdc {

using namespace sm100;

namespace {

constexpr int kSmemLimit = 227 * 1024 - 7 * 1024;     // dynamic; the static part of any of the kernels is below 7 KB
constexpr int kTileN = 128;                           // columns of C per tile: MMA M
constexpr int kStageK = 128;                          // bytes of K per pipeline stage: one scale group
constexpr uint32_t kBBytes = kTileN * kStageK;
constexpr int kTileThreads = 192;
constexpr int kMaxStages = 12;

struct TileParams {
    int64_t M, ldc;
    int N, groups, splits, n_tiles, tile_m, stages, tmem_cols;
    int64_t pieces;                 // scale pieces along K
    uint32_t a_bytes, stage_bytes;
    const uint8_t *SA, *SB;
    const float *bias;
    void *C;
    uint8_t *SC;
    int64_t pieces_c;
    int act, out;
    int *status;
    int limit, withhold;            // of every wait, in units of 1024 cycles; `withhold`: nothing is loaded, so that they run out
};

// A wait ran out: tell the host, and give what is in flight (loads, sums under way, MMAs) time to land before the memory
// and the tensor memory go.  By all threads of a CTA.
__device__ __forceinline__ void settle(int *status) {
    if ((threadIdx.x & 31) == 0) {
        atomicExch(status, SVDCACHE_ERR_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < kWaitCycles / 100) {}
    }
    __syncwarp();
}

// four neighbouring columns n .. n + 3 of row m of C (n a multiple of 4): plain types
__device__ __forceinline__ void store_plain(const TileParams &p, int64_t m, int n, const float (&v)[4]) {
    if (p.out == SVDCACHE_F32) {
        float *o = reinterpret_cast<float *>(p.C) + m * p.ldc + n;
        if (n + 4 <= p.N) *reinterpret_cast<float4 *>(o) = make_float4(v[0], v[1], v[2], v[3]);
        else
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) o[i] = v[i];
    } else {
        __nv_bfloat16 *o = reinterpret_cast<__nv_bfloat16 *>(p.C) + m * p.ldc + n;
        if (n + 4 <= p.N) {
            const __nv_bfloat162 w[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
            *reinterpret_cast<uint2 *>(o) = *reinterpret_cast<const uint2 *>(w);
        } else {
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) o[i] = __float2bfloat16_rn(v[i]);
        }
    }
}

// The rows of a tile are dealt to its cluster's S CTAs in runs of ceil(tile_m / S), and within a CTA to the warps, R at a
// time, four columns per lane.  `parts`: S blocks [run][128] of sums, one from every CTA.
template <int S, int R>
__device__ __forceinline__ void finish_rows(const TileParams &p, uint32_t parts, int rank, int64_t m0, int n_tile, const float (&bias)[4]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = (p.tile_m + S - 1) / S;
    const int64_t m_first = m0 + rank * per;
    const int own = min(per, p.tile_m - rank * per);
    const int rows = (int)(p.M - m_first < own ? p.M - m_first : own);
    const int n = n_tile * kTileN + 4 * lane;
    for (int r0 = warp * R; r0 < rows; r0 += kTileThreads / 32 * R) {
        float4 part[R][S];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int x = 0; x < S; ++x)
                part[i][x] = shared_load(parts + (uint32_t)((x * per + min(r0 + i, per - 1)) * kTileN + 4 * lane) * 4u);
        float v[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            v[i][0] = part[i][0].x; v[i][1] = part[i][0].y; v[i][2] = part[i][0].z; v[i][3] = part[i][0].w;
#pragma unroll
            for (int x = 1; x < S; ++x) {
                v[i][0] += part[i][x].x; v[i][1] += part[i][x].y; v[i][2] += part[i][x].z; v[i][3] += part[i][x].w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] += bias[j];
        }
        if (p.act == SVDCACHE_ACT_GELU) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                pair_to(gelu_tanh(pair_of(v[i][0], v[i][1])), v[i][0], v[i][1]);
                pair_to(gelu_tanh(pair_of(v[i][2], v[i][3])), v[i][2], v[i][3]);
            }
        }
        if (p.out != SVDCACHE_FP8) {
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (r0 + i < rows) store_plain(p, m_first + r0 + i, n, v[i]);
            continue;
        }
        float top[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            top[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][j] = n + j < p.N ? fp8_nan_if_not_finite(v[i][j]) : 0.0f;
                top[i] = fmaxf(top[i], fabsf(v[i][j]));
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) top[i] = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top[i])));   // none is negative
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint32_t byte = fp8_scale_byte(top[i]);
            const float inv = fp8_inverse_scale(byte);
            const uint32_t w = fp8_pack4(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
            if (r0 + i >= rows) break;
            const int64_t m = m_first + r0 + i;
            uint8_t *o = reinterpret_cast<uint8_t *>(p.C) + m * p.ldc + n;
            if (n + 4 <= p.N) *reinterpret_cast<uint32_t *>(o) = w;
            else
                for (int j = 0; j < 4; ++j)
                    if (n + j < p.N) o[j] = (uint8_t)(w >> (8 * j));
            if (lane == 0) p.SC[fp8_scale_offset(m, n_tile, p.pieces_c)] = (uint8_t)byte;
        }
    }
}

// one group of K of the tile into ring slot s
__device__ __forceinline__ void request_group(const CUtensorMap &tm_a, const CUtensorMap &tm_b, const TileParams &p, uint32_t dst, uint32_t bar,
                                              int g, bool scales, int64_t m0, int n_tile) {
    mbar_arrive_expect_tx(bar, kBBytes + p.a_bytes + (scales ? 2 * kScalePieceBytes : 0));
    tma_load_2d(dst, &tm_b, bar, g * kStageK, n_tile * kTileN);
    tma_load_2d(dst + kBBytes, &tm_a, bar, g * kStageK, (int)m0);
    if (scales) {
        const uint32_t sdst = dst + kBBytes + p.a_bytes;
        const int64_t at = g / kScaleGroups;
        bulk_load(sdst, p.SB + ((size_t)n_tile * p.pieces + at) * kScalePieceBytes, kScalePieceBytes, bar);
        bulk_load(sdst + kScalePieceBytes, p.SA + ((size_t)(m0 / kScaleRows) * p.pieces + at) * kScalePieceBytes, kScalePieceBytes, bar);
    }
}

__global__ void __launch_bounds__(kTileThreads)
tile_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const TileParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) unsigned long long bar_mem[2 * kMaxStages + 2];
    __shared__ uint32_t tmem_slot_mem;
    __shared__ int control_mem[2];               // abort flag, limit of the waits
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(bar_mem), empty = full + 8 * kMaxStages, done_bar = empty + 8 * kMaxStages, parts_bar = done_bar + 8;
    volatile int *control = control_mem;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    const int S = p.splits;
    const int rank = (int)(blockIdx.x % (unsigned)S);                   // = rank in the cluster
    const int tile = (int)(blockIdx.x / (unsigned)S);
    const int n_tile = tile % p.n_tiles;
    const int64_t m0 = (int64_t)(tile / p.n_tiles) * p.tile_m;
    const int count = (p.groups - rank + S - 1) / S;                    // groups rank, rank + S, ... of K: at least one
    const int loaded = p.withhold ? 0 : count;
    const int per = (p.tile_m + S - 1) / S, own = min(per, p.tile_m - rank * per);   // rows that a CTA finishes
    // the CTA's own sum goes where the ring was (all loads have been consumed by then); the parts that others send, behind
    // both
    const uint32_t parts = S == 1 ? base : base + max((uint32_t)p.stages * p.stage_bytes, (uint32_t)p.tile_m * kTileN * 4u);

    if (warp == 0 && elect_one()) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        mbar_init(done_bar, 1);
        mbar_init(parts_bar, 1);
        control_mem[0] = 0;
        control_mem[1] = p.limit;
        fence_barrier_init();
        if (S > 1) mbar_arrive_expect_tx(parts_bar, (uint32_t)(S * own) * kTileN * 4u);   // this CTA's rows from all S of them
        prefetch_tensormap(&tm_a);
        prefetch_tensormap(&tm_b);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_slot_mem), (uint32_t)p.tmem_cols);
        tmem_relinquish();
    }
    __syncwarp();
    previous_done();
    // the empty ring is filled before anything else is set up; a piece of scales comes with every group that is the
    // CTA's first in it
    if (warp == 0 && elect_one())
        for (int i = 0; i < p.stages && i < loaded; ++i)
            request_group(tm_a, tm_b, p, base + i * p.stage_bytes, full + 8 * i, rank + i * S, i == 0 || (rank + i * S) % kScaleGroups < S, m0, n_tile);
    tc_fence_before();
    __syncthreads();
    next_may_launch();
    tc_fence_after();
    if (S > 1) cluster_arrive();                                        // this CTA's barriers exist
    const uint32_t tmem = *(volatile uint32_t *)&tmem_slot_mem;
    float bias[4] = {0.f, 0.f, 0.f, 0.f};                               // of the four columns that finish_rows gives this lane
    if (p.bias)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n_tile * kTileN + 4 * lane + j < p.N) bias[j] = p.bias[n_tile * kTileN + 4 * lane + j];

    if (warp == 0) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0;
            for (int i = p.stages; i < loaded; ++i) {
                if (!mbar_wait_control(empty + 8 * s, ph, control, 1)) break;
                const int g = rank + i * S;
                request_group(tm_a, tm_b, p, base + s * p.stage_bytes, full + 8 * s, g, g % kScaleGroups < S, m0, n_tile);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0;
            // scale words: four columns for B, then four for A; two sets that alternate
            const uint32_t sf = tmem + (uint32_t)p.tmem_cols - 32u;
            const uint32_t a_word = (uint32_t)(m0 % kScaleRows) / 32u;   // 0 or 2: a tile of 64 rows may begin in the middle of a piece
            uint32_t set = 1;
            // An instruction's operands (uniform registers) stay taken until the queue of MMAs reaches it, and a loop that
            // writes the same registers again waits for that: 290 cycles a group.  Four copies of the body use four sets
            // (1 x 128 x 9216 5.65 -> 5.1 us, 64 x 2048 x 4608 7.85 -> 7.2 us; 5.6 and 6.9 now).
#pragma unroll 4
            for (int i = 0; i < count; ++i) {
                const int g = rank + i * S;
                if (!mbar_wait_control(full + 8 * s, ph, control, 2)) break;
                tc_fence_after();
                const uint32_t src = base + s * p.stage_bytes;
                if (i == 0 || g % kScaleGroups < S) {
                    set ^= 1u;
                    const uint32_t ssrc = src + kBBytes + p.a_bytes;
                    tmem_cp_scales(sf + 16 * set, smem_desc_scales(ssrc));
                    tmem_cp_scales(sf + 16 * set + 4, smem_desc_scales(ssrc + kScalePieceBytes));
                }
                const uint64_t bd = smem_desc_kmajor(src, 128), ad = smem_desc_kmajor(src + kBBytes, 128);
                const uint32_t idesc = idesc_mxf8(kTileN, p.tile_m, g & 3);
#pragma unroll
                for (int ks = 0; ks < kStageK / 32; ++ks)
                    mma_mxf8_ss(tmem, bd + 2 * ks, ad + 2 * ks, idesc, sf + 16 * set, sf + 16 * set + 4 + a_word,
                                (i > 0 || ks > 0) ? 1u : 0u);
                mma_commit(empty + 8 * s);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
            mma_commit(done_bar);
        }
        __syncwarp();
    }
    // every wait below is passed by all CTAs of the cluster in the same order, also after a time-out in one of them
    if (S > 1) cluster_wait();                                          // the other CTAs' barriers exist
    if (warp >= 2) {
        const int q = warp & 3;
        const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_control(done_bar, 0u, control, 3));
        tc_fence_after();
        for (int c = 0; ok && c < p.tile_m; c += 32) {
            uint32_t acc[32];
            tmem_ld_32x32(tmem + ((uint32_t)(q * 32) << 16) + c, acc);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (c + i < p.tile_m) shared_store1(base + (uint32_t)((c + i) * kTileN + q * 32 + lane) * 4u, acc[i]);
        }
        tc_fence_before();
        if (S > 1) {
            fence_proxy_async();
            named_barrier(1, 128);
            if (warp == 2 && lane < S) {        // to CTA `lane`: its rows of this CTA's sum
                const uint32_t run = (uint32_t)(per * kTileN) * 4u, last = (uint32_t)((p.tile_m - lane * per) * kTileN) * 4u;
                bulk_send(cluster_addr(parts + (uint32_t)rank * run, (uint32_t)lane), base + (uint32_t)lane * run, min(run, last),
                          cluster_addr(parts_bar, (uint32_t)lane));
            }
        }
    }
    __syncthreads();
    if (control[0]) settle(p.status);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
    }
    if (S > 1 && !__all_sync(0xFFFFFFFFu, mbar_wait_cluster(parts_bar, 0u, control))) settle(p.status);
    if (S > 1) cluster_arrive();                                        // this CTA has all its parts (or has waited long enough)
    switch (S) {
        case 1: finish_rows<1, 4>(p, parts, rank, m0, n_tile, bias); break;
        case 2: finish_rows<2, 4>(p, parts, rank, m0, n_tile, bias); break;
        case 3: finish_rows<3, 2>(p, parts, rank, m0, n_tile, bias); break;
        case 4: finish_rows<4, 2>(p, parts, rank, m0, n_tile, bias); break;
        case 6: finish_rows<6, 1>(p, parts, rank, m0, n_tile, bias); break;
        default: finish_rows<8, 1>(p, parts, rank, m0, n_tile, bias); break;
    }
    // What a CTA sent is reported to the receiver alone: only when every CTA has its parts has this one's shared memory been
    // read to the end, and may go to another CTA.
    __syncwarp();
    if (S > 1) cluster_wait();
}

// ---------------------------------------------------------------------- pairs of CTAs ---
//
// pair_kernel: a persistent cluster of two CTAs computes tiles of 256 x BN of C with cta_group::2 MMAs: each CTA
// holds 128 rows of the tile in its tensor memory and loads its 128 rows of A and half of the tile's rows of B, so
// a group of K costs an SM 32 KB at BN = 256 instead of the 48 KB of a one-CTA 128 x 256 tile -- the traffic between
// L2 and the SMs is what bounds such a kernel first.
// Tensor memory (512 columns) holds two accumulators, so that a tile's epilogue runs beside the next tile's MMAs, and two
// sets of scale words in the last 32 columns.
//   BN = 128, 192   accumulators side by side; the two epilogue groups (warps 2-5, 6-9) take alternate tiles
//   BN = 256        only for 8-bit C, whose groups of 128 columns a tile of 192 would cut: columns [0, 256) and
//                   [224, 480) share 32.  The groups take the two column halves of every tile; the next tile's MMAs start
//                   when the group whose half holds the shared columns has all its 128 columns in registers
// Warps: 0 TMA producer, 1 MMA issuer (the first CTA's, for both), 2-9 epilogue.

constexpr int kPairM = 256;
constexpr int kPairThreads = 320;
constexpr uint32_t kPairABytes = 128 * kStageK;                                   // each CTA's share
constexpr uint32_t kStoreBytes = 32 * 128;                                        // a warp's box of C: 32 rows of 128 bytes
constexpr uint32_t kScaleCol = 480;
constexpr int kMaxPairStages = 7;

template <int BN> struct Pair {
    static constexpr bool kHalves = BN == 256;
    static constexpr uint32_t kBBytes = BN / 2 * kStageK;                         // each CTA's share
    static constexpr int kBPieces = (BN + 127) / 128;                             // of scales: all rows of B, in both CTAs
    static constexpr uint32_t kScaleBytes = (1 + kBPieces) * kScalePieceBytes;
    static constexpr uint32_t kStageBytes = (kPairABytes + kBBytes + kScaleBytes + 1023) / 1024 * 1024;
    static constexpr int kFit = (int)((kSmemLimit - 1024 - 8 * kStoreBytes) / kStageBytes);
    static constexpr int kStages = kFit < kMaxPairStages ? kFit : kMaxPairStages;
    static constexpr uint32_t kSmem = 1024 + kStages * kStageBytes + 8 * kStoreBytes;
    static constexpr uint32_t kAccStep = kHalves ? 224 : BN;
    static constexpr int kWarpCols = kHalves ? 128 : BN;                          // columns of a tile that a warp finishes
    static_assert(kStages >= 4 && (BN == 256 || 2 * BN <= (int)kScaleCol), "shared and tensor memory");
};
// Tiles are walked in bands of tile rows, column by column: the clusters at work share a few columns of B's tiles and the
// band's rows of A.  High bands read B fewer times (4608 x 12288 x 3072 into bf16: 134 us with bands of 8 rows, 130 with
// one of 18; into 8 bits with gelu 138 and 136), up to where a band's A no longer stays in L2 (4608 x 3072 x 12288: 128 us
// with 57 MB in one band, 123 with bands of 25 or 31 MB).
constexpr int kBandRows = 20;
constexpr int64_t kBandBytes = 32 << 20;

// Quotients by a divisor that the host knows, without the device's division (three of which a tile cost 400 cycles):
// with 2^l the least power of two >= d and m = 2^32 (2^l - d) / d + 1, n / d = (umulhi(m, n) + n) >> l (Granlund and
// Montgomery), for 0 <= n < 2^31.
struct Divisor {
    uint32_t d, m, l;
    __host__ static Divisor of(int d) {
        uint32_t l = 0;
        while ((1u << l) < (uint32_t)d) ++l;
        return {(uint32_t)d, (uint32_t)((((1ull << l) - (uint64_t)d) << 32) / (uint64_t)d + 1), l};
    }
    __device__ __forceinline__ int quotient(int n) const { return (int)((__umulhi(m, (uint32_t)n) + (uint32_t)n) >> l); }
};

struct PairParams {
    int64_t M, ldc;
    void *C;
    int N, groups, tiles, bands;
    Divisor band_tiles, band_rows, last_rows;        // tiles of a band; tile rows of a band, of the last one
    const float *bias;
    uint8_t *SC;
    int64_t pieces_c;
    int act;
    int *status;
    int limit, withhold;                             // as in TileParams
};

struct TileAt { int m, n; };
__device__ __forceinline__ TileAt pair_tile(const PairParams &p, int t) {
    const int b = p.band_tiles.quotient(t), in = t - b * (int)p.band_tiles.d;
    const bool last = b == p.bands - 1;
    const int n = last ? p.last_rows.quotient(in) : p.band_rows.quotient(in);
    return {b * (int)p.band_rows.d + in - n * (int)(last ? p.last_rows.d : p.band_rows.d), n};
}

// v += bias (shared memory, the same for every lane), then the activation
template <int N> __device__ __forceinline__ void add_bias_and_act(float *v, const float *bias, int act) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(bias + i);
        pair_to(pair_add(pair_of(v[i], v[i + 1]), pair_of(b.x, b.y)), v[i], v[i + 1]);
        pair_to(pair_add(pair_of(v[i + 2], v[i + 3]), pair_of(b.z, b.w)), v[i + 2], v[i + 3]);
    }
    if (act == SVDCACHE_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; i += 2) pair_to(gelu_tanh(pair_of(v[i], v[i + 1])), v[i], v[i + 1]);
    }
}

// the largest magnitude of a group (NaN is passed over), as eight chains
__device__ __forceinline__ float largest_of(const float (&v)[128]) {
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = fabsf(v[i]);
#pragma unroll
    for (int i = 8; i < 128; ++i) m[i & 7] = fmaxf(m[i & 7], fabsf(v[i]));
    return fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), fmaxf(fmaxf(m[4], m[5]), fmaxf(m[6], m[7])));
}

// A warp's box of C (32 rows of 128 bytes, 16-byte pieces swizzled), written by all its lanes, on its way out.  A TMA
// store ends at a multiple of 16 bytes, not at the matrix's last column: of a box that the last column cuts elsewhere
// each lane writes a row, so that nothing beyond column N changes.
template <typename T>
__device__ __forceinline__ void send_box(const CUtensorMap *tm_c, const PairParams &p, uint32_t box, int n, int64_t row0, int lane) {
    constexpr int kCols = 128 / (int)sizeof(T), kPiece = 16 / (int)sizeof(T);
    const bool live = n < p.N && row0 < p.M, whole = n + kCols <= p.N || (p.N * (int)sizeof(T)) % 16 == 0;
    if (live && whole) {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(tm_c, box, n, (int)row0);
            tma_store_commit();
        }
    } else if (live) {
        if (row0 + lane < p.M) {
            T *out = reinterpret_cast<T *>(p.C) + (row0 + lane) * p.ldc + n;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int left = p.N - n - c * kPiece;       // columns from this piece on
                if (left <= 0) break;
                const float4 f = shared_load(box + (uint32_t)lane * 128u + (uint32_t)(c ^ (lane & 7)) * 16u);
                T *o = out + c * kPiece;
                if (left >= kPiece) {
                    *reinterpret_cast<float4 *>(o) = f;
                    continue;
                }
                // the first left * sizeof(T) bytes: 8, 4, 2 and 1 of them, as that number's bits say
                uint32_t w[4];
                memcpy(w, &f, 16);
                const int bytes = left * (int)sizeof(T);
                uint8_t *b = reinterpret_cast<uint8_t *>(o);
                if (bytes & 8) {
                    *reinterpret_cast<uint2 *>(b) = make_uint2(w[0], w[1]);
                    w[0] = w[2]; w[1] = w[3]; b += 8;
                }
                if (bytes & 4) {
                    *reinterpret_cast<uint32_t *>(b) = w[0];
                    w[0] = w[1]; b += 4;
                }
                if (bytes & 2) {
                    *reinterpret_cast<uint16_t *>(b) = (uint16_t)w[0];
                    w[0] >>= 16; b += 2;
                }
                if (bytes & 1) *b = (uint8_t)w[0];
            }
        }
        __syncwarp();
    }
}

template <int OUT, int BN>
__global__ void __launch_bounds__(kPairThreads, 1)
pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
            const __grid_constant__ CUtensorMap tm_sa, const __grid_constant__ CUtensorMap tm_sb,
            const __grid_constant__ CUtensorMap tm_c, const PairParams p) {
    extern __shared__ uint8_t smem_raw[];
    using T = Pair<BN>;
    constexpr bool kHalves = T::kHalves;
    __shared__ __align__(8) unsigned long long bar_mem[2 * kMaxPairStages + 4];
    __shared__ __align__(16) float bias_mem[8][T::kWarpCols];
    __shared__ uint32_t tmem_slot_mem;
    __shared__ int control_mem[2];               // abort flag, limit of the waits
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(bar_mem), empty = full + 8 * kMaxPairStages, acc_full = empty + 8 * kMaxPairStages, acc_empty = acc_full + 16;
    volatile int *control = control_mem;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1u;           // in the cluster
    const int cluster = (int)(blockIdx.x >> 1), clusters = (int)(gridDim.x >> 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < T::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) {                // halves: the first of each serves both accumulators in turn
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, kHalves ? 16 : 8);   // the epilogue warps of both CTAs that read it
        }
        control_mem[0] = 0;
        control_mem[1] = p.limit;
        fence_barrier_init();
        prefetch_tensormap(&tm_a);
        prefetch_tensormap(&tm_b);
        prefetch_tensormap(&tm_sa);
        prefetch_tensormap(&tm_sb);
        prefetch_tensormap(&tm_c);
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(&tmem_slot_mem), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                  // both CTAs' barriers exist
    tc_fence_after();
    previous_done();
    next_may_launch();
    const uint32_t tmem = *(volatile uint32_t *)&tmem_slot_mem;

    if (warp == 0) {
        if (!p.withhold && elect_one()) {
            int s = 0;
            uint32_t ph = 1;
            for (int t = cluster; t < p.tiles; t += clusters) {
                const TileAt at = pair_tile(p, t);
                const int row_a = at.m * kPairM + (int)rank * 128, row_b = at.n * BN + (int)rank * (BN / 2);
                // unrolled as tile_kernel's loop over groups is, here and in the issuer (256 x 3072 x 12288 22.6 -> 21.8 us)
#pragma unroll 4
                for (int g = 0; g < p.groups; ++g) {
                    if (!mbar_wait_control(empty + 8 * s, ph, control, 1)) goto done;
                    const uint32_t dst = base + s * T::kStageBytes, bar = cluster_addr(full + 8 * s, 0);
                    const bool scales = (g & (kScaleGroups - 1)) == 0;
                    if (rank == 0)
                        mbar_arrive_expect_tx(full + 8 * s, 2 * (kPairABytes + T::kBBytes + (scales ? T::kScaleBytes : 0)));
                    tma_load_2d_pair(dst, &tm_a, bar, g * kStageK, row_a);
                    tma_load_2d_pair(dst + kPairABytes, &tm_b, bar, g * kStageK, row_b);
                    if (scales) {
                        // the scale buffers as rows of pieces, g / 4 the piece of the row
                        const uint32_t sdst = dst + kPairABytes + T::kBBytes;
                        const int c = g / kScaleGroups * (kScalePieceBytes / 4);
                        tma_load_2d_pair(sdst, &tm_sa, bar, c, at.m * 2 + (int)rank);
#pragma unroll
                        for (int i = 0; i < T::kBPieces; ++i)
                            tma_load_2d_pair(sdst + (1 + i) * kScalePieceBytes, &tm_sb, bar, c, at.n * BN / 128 + i);
                    }
                    if (++s == T::kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            int s = 0;
            uint32_t ph = 0, it = 0, set = 1;
            for (int t = cluster; t < p.tiles; t += clusters, ++it) {
                const uint32_t b = it & 1u;
                if (kHalves) {
                    if (it > 0 && !mbar_wait_control(acc_empty, b ^ 1u, control, 2)) goto done;
                } else {
                    if (it > 1 && !mbar_wait_control(acc_empty + 8 * b, (it >> 1 & 1u) ^ 1u, control, 2)) goto done;
                }
                tc_fence_after();
                const uint32_t acc = tmem + b * T::kAccStep;
                const uint32_t b_word = BN == 192 ? (uint32_t)(pair_tile(p, t).n & 1) * 2u : 0u;   // a tile of 192 may begin in the middle of a piece
#pragma unroll 4
                for (int g = 0; g < p.groups; ++g) {
                    if (!mbar_wait_control(full + 8 * s, ph, control, 3)) goto done;
                    tc_fence_after();
                    const uint32_t src = base + s * T::kStageBytes;
                    if ((g & (kScaleGroups - 1)) == 0) {
                        set ^= 1u;
                        const uint32_t ssrc = src + kPairABytes + T::kBBytes, sf = tmem + kScaleCol + 16 * set;
#pragma unroll
                        for (int i = 0; i <= T::kBPieces; ++i) tmem_cp_scales_pair(sf + 4 * i, smem_desc_scales(ssrc + i * kScalePieceBytes));
                    }
                    const uint32_t sf = tmem + kScaleCol + 16 * set;
                    const uint64_t ad = smem_desc_kmajor(src, 128), bd = smem_desc_kmajor(src + kPairABytes, 128);
                    const uint32_t idesc = idesc_mxf8(kPairM, BN, g & 3);
#pragma unroll
                    for (int ks = 0; ks < kStageK / 32; ++ks)
                        mma_mxf8_ss_pair(acc, ad + 2 * ks, bd + 2 * ks, idesc, sf, sf + 4 + b_word, (g > 0 || ks > 0) ? 1u : 0u);
                    mma_commit_pair(empty + 8 * s);
                    if (++s == T::kStages) { s = 0; ph ^= 1u; }
                }
                mma_commit_pair(acc_full + (kHalves ? 0 : 8 * b));
            }
        }
    } else {
        const int q = warp & 3, group = (warp - 2) >> 2;
        const uint32_t store = base + T::kStages * T::kStageBytes + (uint32_t)(warp - 2) * kStoreBytes;
        const uint32_t store_row = store + (uint32_t)lane * 128u;
        float *bias = bias_mem[warp - 2];
        const uint32_t acc_empty_first = cluster_addr(acc_empty + (kHalves ? 0 : 8 * group), 0);
        constexpr int kBlocks = T::kWarpCols / 32;                                          // column blocks of a tensor-memory load
        float next_bias[kBlocks];
        auto request_bias = [&](int t) {
            const int n0 = t < p.tiles ? pair_tile(p, t).n * BN + (kHalves ? group * 128 : 0) + lane : p.N;
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) next_bias[j] = p.bias && n0 + j * 32 < p.N ? __ldg(p.bias + n0 + j * 32) : 0.0f;
        };
        request_bias(cluster + (kHalves ? 0 : group * clusters));
        uint32_t it = 0;
        for (int t = cluster; t < p.tiles; t += clusters, ++it) {
            if (!kHalves && (int)(it & 1u) != group) continue;
            const TileAt at = pair_tile(p, t);
            const int64_t row0 = (int64_t)at.m * kPairM + rank * 128 + q * 32;
            const int col0 = at.n * BN + (kHalves ? group * 128 : 0);
            // this tile's bias was requested a tile ago
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) bias[j * 32 + lane] = next_bias[j];
            __syncwarp();
            request_bias(t + (kHalves ? 1 : 2) * clusters);
            if (!__all_sync(0xFFFFFFFFu, mbar_wait_control(acc_full + (kHalves ? 0 : 8 * group), (kHalves ? it : it >> 1) & 1u, control, 4))) goto done;
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (it & 1u) * T::kAccStep + (kHalves ? group * 128 : 0);
            // halves: the columns that the next accumulator shares are the last 32 of the first one and the first 32 of
            // the second; the group that does not hold them has nothing to release
            const bool shares = kHalves && group == (int)((it & 1u) ^ 1u);
            auto release = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty_first);
            };
            if (kHalves && !shares) release();
            if constexpr (OUT == SVDCACHE_FP8) {
                float v[128];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t r[32];
                    tmem_ld_32x32(acc + j * 32, r);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[j * 32 + i] = __uint_as_float(r[i]);
                }
                tmem_wait_ld();
                if (!kHalves || shares) release();
#pragma unroll
                for (int j = 0; j < 4; ++j) add_bias_and_act<32>(v + 32 * j, bias + 32 * j, p.act);
                if (col0 + 128 > p.N) {
#pragma unroll
                    for (int j = 0; j < 128; j += 32) {
                        if (col0 + j + 32 <= p.N) continue;
#pragma unroll
                        for (int i = j; i < j + 32; ++i)
                            if (col0 + i >= p.N) v[i] = 0.0f;
                    }
                }
                float top = largest_of(v);
                if (__float_as_uint(top) == 0x7F800000u) {
#pragma unroll
                    for (int i = 0; i < 128; ++i) v[i] = fp8_nan_if_not_finite(v[i]);
                    top = largest_of(v);
                }
                const uint32_t byte = fp8_scale_byte(top);
                const uint64_t inv = pair_of(fp8_inverse_scale(byte), fp8_inverse_scale(byte));
                if (lane == 0) tma_store_wait_read<0>();      // the last box has left
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = c * 16 + i * 4;
                        float x[4];
                        pair_to(pair_mul(pair_of(v[k], v[k + 1]), inv), x[0], x[1]);
                        pair_to(pair_mul(pair_of(v[k + 2], v[k + 3]), inv), x[2], x[3]);
                        w[i] = fp8_pack4(x[0], x[1], x[2], x[3]);
                    }
                    shared_store(store_row + (uint32_t)(c ^ (lane & 7)) * 16u, w);
                }
                send_box<uint8_t>(&tm_c, p, store, col0, row0, lane);   // its fence waits for earlier stores: the scale's comes after
                if (row0 + lane < p.M && col0 < p.N) p.SC[fp8_scale_offset(row0 + lane, col0 / kFp8Group, p.pieces_c)] = (uint8_t)byte;
            } else {
                // a block of 32 columns at a time, the next one on its way from tensor memory meanwhile; a box holds two
                // blocks of bf16 (128 bytes of a row: 64 were 5-13 % slower where C's bytes count) or one of fp32
                using C = typename std::conditional<OUT == SVDCACHE_BF16, __nv_bfloat16, float>::type;
                constexpr int kPerBox = OUT == SVDCACHE_BF16 ? 2 : 1;
                auto finish = [&](const uint32_t (&r)[32], int j, bool second) {
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
                    add_bias_and_act<32>(v, bias + j * 32, p.act);
                    if (kPerBox == 1 || !second) {
                        if (lane == 0) tma_store_wait_read<0>();      // the last box has left
                        __syncwarp();
                    }
                    const uint32_t c0 = kPerBox == 2 && second ? 4u : 0u;
#pragma unroll
                    for (int c = 0; c < 8 / kPerBox; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (OUT == SVDCACHE_BF16) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(v[c * 8 + 2 * i], v[c * 8 + 2 * i + 1]);
                                w[i] = *reinterpret_cast<const uint32_t *>(&h);
                            } else {
                                w[i] = __float_as_uint(v[c * 4 + i]);
                            }
                        }
                        shared_store(store_row + ((c0 + c) ^ (uint32_t)(lane & 7)) * 16u, w);
                    }
                    if (kPerBox == 1 || second) send_box<C>(&tm_c, p, store, col0 + (j - (kPerBox - 1)) * 32, row0, lane);
                };
                uint32_t even[32], odd[32];
                tmem_ld_32x32(acc, even);
#pragma unroll 1
                for (int j = 0; j < kBlocks; j += 2) {
                    tmem_wait_ld();
                    tmem_ld_32x32(acc + (j + 1) * 32, odd);
                    finish(even, j, false);
                    tmem_wait_ld();
                    if (j + 2 < kBlocks) tmem_ld_32x32(acc + (j + 2) * 32, even);
                    else release();
                    finish(odd, j + 1, true);
                }
            }
        }
        if (lane == 0) tma_store_wait<0>();
    }

done:
    __syncwarp();
    __syncthreads();
    if (control[0]) settle(p.status);
    tc_fence_before();
    cluster_sync();      // neither CTA signals the other any more
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ------------------------------------------------------------------------- host side ---

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(ptr);
        return (EncodeTiledFn) nullptr;
    }();
    return fn;
}

// bytes [rows x cols], rows `ld` bytes apart, boxes of 128 bytes x box_rows with the 128-byte swizzle; bytes
// beyond the matrix read as zero, which is e4m3's zero.  Where rows begin at multiples of 256 bytes, L2 fetches so many
// at a time, two groups of K that are read one after the other (1 x 18432 x 9216 31.7 -> 29.5 us); elsewhere half of such
// a fetch may belong to another row (256 x 6912 x 9000 27.1 -> 29.3 us, 40 x 18432 x 400 4.8 -> 5.2).
int byte_map(CUtensorMap *m, const void *base, int64_t rows, int cols, int64_t ld, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return SVDCACHE_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kStageK, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          ld % 256 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SVDCACHE_OK : SVDCACHE_ERR_CUDA;
}

// CTAs per tile of tile_kernel.  (3 and 6 for numbers of tiles that leave SMs to 2 and 4: 256 x 1152 x 9000 16.6 -> 13.2 us.)
constexpr int kSplits[] = {1, 2, 3, 4, 6, 8}, kSplitKinds = 6;

// The status word of products that are given none: part of the library's image on each device, zero when that is loaded, so
// that no first call has to allocate one or wait for its zero (which a stream capture forbids).
__device__ int default_status;

// What the launches ask of a device, once: its SMs, how many clusters of so many CTAs of tile_kernel it runs at the same
// time, where the default status word lies, and leave to use an SM's shared memory.
struct Device {
    int sms, clusters[kSplitKinds];
    int *status;
};
constexpr int kMaxDevices = 64;

int ask_device(Device *d) {
    int dev = 0;
    int rc = record_cuda(cudaGetDevice(&dev));
    if (!rc) rc = record_cuda(cudaGetSymbolAddress((void **)&d->status, default_status));
    if (!rc) rc = record_cuda(cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev));
    for (const void *k : {(const void *)tile_kernel, (const void *)pair_kernel<SVDCACHE_F32, 128>, (const void *)pair_kernel<SVDCACHE_F32, 192>,
                          (const void *)pair_kernel<SVDCACHE_BF16, 128>, (const void *)pair_kernel<SVDCACHE_BF16, 192>,
                          (const void *)pair_kernel<SVDCACHE_FP8, 128>, (const void *)pair_kernel<SVDCACHE_FP8, 256>})
        if (!rc) rc = record_cuda(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit));
    for (int i = 0; i < kSplitKinds && !rc; ++i) {
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3(24 * (unsigned)d->sms);
        cfg.blockDim = dim3(kTileThreads);
        cfg.dynamicSmemBytes = kSmemLimit;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)kSplits[i];
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        rc = record_cuda(cudaOccupancyMaxActiveClusters(&d->clusters[i], tile_kernel, &cfg));
    }
    return rc;
}

int device(Device *d) {
    static Device known[kMaxDevices];
    static std::atomic<int> state[kMaxDevices];      // 0: not asked, 1: one thread is asking, 2: known
    int dev = 0;
    int rc = record_cuda(cudaGetDevice(&dev));
    if (rc) return rc;
    if (dev < kMaxDevices && state[dev].load(std::memory_order_acquire) == 2) {
        *d = known[dev];
        return SVDCACHE_OK;
    }
    rc = ask_device(d);
    int zero = 0;
    if (!rc && dev < kMaxDevices && state[dev].compare_exchange_strong(zero, 1)) {
        known[dev] = *d;
        state[dev].store(2, std::memory_order_release);
    }
    return rc;
}

// in units of 1024 cycles
int wait_limit(const GemmFp8Args &a) { return (int)((a.limit > 0 ? a.limit : kWaitCycles) / 1024); }

int tile_launch(const GemmFp8Args &a, int tile_m, int splits, cudaStream_t s) {
    TileParams p{};
    p.M = a.M; p.N = a.N; p.ldc = a.ldc;
    p.SA = (const uint8_t *)a.SA; p.SB = (const uint8_t *)a.SB; p.bias = a.bias; p.C = a.C; p.SC = (uint8_t *)a.SC;
    p.act = a.act; p.out = a.out; p.status = a.status; p.limit = wait_limit(a); p.withhold = a.limit > 0;
    p.groups = (int)fp8_groups(a.K); p.splits = splits; p.n_tiles = (a.N + kTileN - 1) / kTileN; p.tile_m = tile_m;
    const int64_t tiles = (a.M + tile_m - 1) / tile_m * p.n_tiles;
    p.pieces = fp8_piece_cols(a.K); p.pieces_c = fp8_piece_cols(a.N);
    if (tiles * p.splits > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    p.a_bytes = (uint32_t)p.tile_m * kStageK;
    p.stage_bytes = kBBytes + p.a_bytes + 1024u;
    p.tmem_cols = p.tile_m <= 32 ? 64 : 2 * p.tile_m;                     // the accumulator and 32 columns of scales
    const size_t sums = (size_t)p.tile_m * kTileN * 4;                    // pass through the ring,
    const size_t parts = p.splits == 1 ? 0 : (size_t)((p.tile_m + p.splits - 1) / p.splits * p.splits) * kTileN * 4;   // others' arrive behind it
    static_assert((kSmemLimit - 1024 - 132 * kTileN * 4) / (kBBytes + 128 * kStageK + 1024) >= 2, "a ring has at least two stages");
    p.stages = (int)((kSmemLimit - 1024 - parts) / p.stage_bytes);
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    const int longest = (p.groups + p.splits - 1) / p.splits;
    if (p.stages > longest) p.stages = longest;
    size_t smem = (size_t)p.stages * p.stage_bytes;
    smem = 1024 + std::max(smem, sums) + parts;

    CUtensorMap tm_a, tm_b;
    int rc = byte_map(&tm_a, a.A, a.M, a.K, a.lda, p.tile_m);
    if (!rc) rc = byte_map(&tm_b, a.B, a.N, a.K, a.ldb, kTileN);
    if (rc) return rc;
    return launch_early(tile_kernel, dim3((unsigned)(tiles * p.splits)), dim3(kTileThreads), smem, p.splits, s, tm_a, tm_b, p);
}

// a scale buffer as rows of 128-row strips, each `pieces` pieces of 128 words; boxes of one piece.  Pieces beyond
// the buffer read as zero.
int scale_map(CUtensorMap *m, const void *base, int64_t rows, int64_t pieces) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return SVDCACHE_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)pieces * (kScalePieceBytes / 4), (cuuint64_t)((rows + kScaleRows - 1) / kScaleRows)};
    const cuuint64_t strides[1] = {(cuuint64_t)pieces * kScalePieceBytes};
    const cuuint32_t box[2] = {kScalePieceBytes / 4, 1};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, const_cast<void *>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SVDCACHE_OK : SVDCACHE_ERR_CUDA;
}

// C in boxes of 32 rows x 128 bytes; what lies beyond M or N is not written
int out_map(CUtensorMap *m, const GemmFp8Args &a) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return SVDCACHE_ERR_CUDA;
    const int elem = a.out == SVDCACHE_FP8 ? 1 : a.out == SVDCACHE_BF16 ? 2 : 4;
    const CUtensorMapDataType t = a.out == SVDCACHE_FP8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                  : a.out == SVDCACHE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const cuuint64_t dims[2] = {(cuuint64_t)a.N, (cuuint64_t)a.M};
    const cuuint64_t strides[1] = {(cuuint64_t)a.ldc * elem};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / elem), 32};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, t, 2, a.C, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SVDCACHE_OK : SVDCACHE_ERR_CUDA;
}

template <int OUT, int BN> int pair_launch(const GemmFp8Args &a, int clusters, cudaStream_t s) {
    PairParams p{};
    p.M = a.M; p.N = a.N; p.groups = (int)fp8_groups(a.K); p.C = a.C; p.ldc = a.ldc;
    const int n_tiles = (a.N + BN - 1) / BN;
    const int64_t tiles = (a.M + kPairM - 1) / kPairM * n_tiles;
    if (tiles > 0x3FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    const int m_tiles = (int)((a.M + kPairM - 1) / kPairM);
    p.tiles = (int)tiles;
    const int64_t fit = kBandBytes / ((int64_t)kPairM * a.K), most = fit < 4 ? 4 : fit > kBandRows ? kBandRows : fit;
    const int bands = (int)((m_tiles + most - 1) / most);
    const int rows = (m_tiles + bands - 1) / bands;
    p.bands = (m_tiles + rows - 1) / rows;
    p.band_tiles = Divisor::of(rows * n_tiles);
    p.band_rows = Divisor::of(rows);
    p.last_rows = Divisor::of(m_tiles - (p.bands - 1) * rows);
    p.bias = a.bias; p.SC = (uint8_t *)a.SC; p.pieces_c = fp8_piece_cols(a.N); p.act = a.act; p.status = a.status;
    p.limit = wait_limit(a); p.withhold = a.limit > 0;
    CUtensorMap tm_a, tm_b, tm_sa, tm_sb, tm_c;
    int rc = byte_map(&tm_a, a.A, a.M, a.K, a.lda, 128);
    if (!rc) rc = byte_map(&tm_b, a.B, a.N, a.K, a.ldb, BN / 2);
    if (!rc) rc = scale_map(&tm_sa, a.SA, a.M, fp8_piece_cols(a.K));
    if (!rc) rc = scale_map(&tm_sb, a.SB, a.N, fp8_piece_cols(a.K));
    if (!rc) rc = out_map(&tm_c, a);
    if (rc) return rc;
    if (clusters > p.tiles) clusters = p.tiles;
    return launch_early(pair_kernel<OUT, BN>, dim3(2 * (unsigned)clusters), dim3(kPairThreads), Pair<BN>::kSmem, 2, s, tm_a, tm_b, tm_sa,
                        tm_sb, tm_c, p);
}

// Rows of tile_kernel's tiles: what M needs, up to 64 or 128.  (Fewer only where M has no more: an MMA's scale words begin at
// an even column of tensor memory, 32 rows each, so a tile begins at a multiple of 64.)
int least_tile_rows(int64_t M) { return M <= 16 ? 16 : M <= 32 ? 32 : 64; }
int most_tile_rows(int64_t M) { return M <= 64 ? least_tile_rows(M) : 128; }

// Whether kSplits[i] CTAs may share a tile: all clusters run at the same time and each CTA has two groups of K.
bool split_allowed(int64_t tiles, int groups, const Device &d, int i) {
    return d.clusters[i] > 0 && (i == 0 || (tiles <= d.clusters[i] && groups >= 2 * kSplits[i]));
}

// Which kernel and tile take less time, by a model of both in units of 10 ns whose numbers were measured (M from 1 to 4000,
// N from 128 to 18432, K from 100 to 9216; over 200 other shapes of that range, every plan of each timed, the choice takes 1.6 % more
// than the best on average, nothing at the median, 7 % at the 90th percentile and 22 % at worst):
//   pairs       3.1 us from launch to end, and per round of the clusters 0.4 and for a group of K 0.20 us at BN = 128, 0.23
//               at 192, 0.35 at 256, two fifths more where rows do not begin at multiples of 128 bytes (a box's row then
//               lies in two lines); or 4 us and B's bytes at 4 TB/s, where that is more: a pair's ring holds little of B
//   small tiles 2.1 us, 1.5 us per 100 rows of a tile and 0.4 (8-bit C: 1.5) per 100 rows that a CTA finishes, 1.2 more where
//               CTAs exchange sums; and per group of a CTA's share of K 0.20 us at 16 rows, 0.32 at 64, 0.48 at 128, or
//               B's bytes at 5.6 TB/s, where that is more
// N = 500, K = 100, M = 40: 3.9 us by pairs, 3.8 by small tiles.  N = 500, K = 9000, M = 1 / 40 / 512: 15.0 / 17.7 / 24.3 and
// 6.2 / 7.4 / 11.2.  N = 18432, K = 3072, M = 1 / 40 / 256: 27.0 / 21.7 / 16.8 and 12.0 / 12.8 / 24.4.
GemmFp8Plan plan_pair(const GemmFp8Args &a, const Device &d) {
    const int64_t m_tiles = (a.M + kPairM - 1) / kPairM, groups = fp8_groups(a.K), clusters = d.sms / 2;
    const int64_t fifths = (a.lda | a.ldb) % 128 ? 7 : 5;
    auto plan = [&](int bn, int64_t group) {
        const int64_t rounds = (m_tiles * ((a.N + bn - 1) / bn) + clusters - 1) / clusters, work = rounds * (40 + groups * group * fifths / 5);
        // the last term: fewer rounds where memory decides
        return GemmFp8Plan{true, bn, 2, rounds, std::max(310 + work, 400 + (int64_t)a.N * a.K / 40000 + work / 16)};
    };
    const GemmFp8Plan wide = a.out == SVDCACHE_FP8 ? plan(256, 35) : plan(192, 23), narrow = plan(128, 20);
    return wide.time < narrow.time ? wide : narrow;
}

GemmFp8Plan plan_tile(const GemmFp8Args &a, const Device &d) {
    GemmFp8Plan best{};
    const int groups = (int)fp8_groups(a.K), n_tiles = (a.N + kTileN - 1) / kTileN;
    for (int tile_m = least_tile_rows(a.M); tile_m <= most_tile_rows(a.M); tile_m *= 2) {
        const int64_t tiles = (a.M + tile_m - 1) / tile_m * n_tiles;
        for (int i = 0; i < kSplitKinds; ++i) {
            const int splits = kSplits[i], fit = d.clusters[i];
            if (!split_allowed(tiles, groups, d, i)) continue;
            const int own = (tile_m + splits - 1) / splits, each = (groups + splits - 1) / splits;
            const int64_t rounds = (tiles + fit - 1) / fit;
            const int64_t ends = 210 + (splits > 1 ? 120 : 0) + tile_m * 3 / 2 + (a.out == SVDCACHE_FP8 ? own * 3 / 2 : own * 2 / 5);
            const int64_t time = ends + std::max(rounds * each * (16 + tile_m / 4), (int64_t)a.N * a.K / 56000);
            if (!best.splits || time < best.time) best = {false, tile_m, splits, rounds, time};
        }
    }
    return best;
}

GemmFp8Plan choose(const GemmFp8Args &a, const Device &d) {
    const GemmFp8Plan t = plan_tile(a, d), p = plan_pair(a, d);
    return t.splits > 0 && t.time < p.time ? t : p;
}

bool allowed(const GemmFp8Args &a, const GemmFp8Plan &plan, const Device &d) {
    if (plan.pairs) return plan.splits == 2 && (plan.size == 128 || plan.size == (a.out == SVDCACHE_FP8 ? 256 : 192));
    if (plan.size != least_tile_rows(a.M) && plan.size != most_tile_rows(a.M)) return false;
    const int64_t tiles = (a.M + plan.size - 1) / plan.size * ((a.N + kTileN - 1) / kTileN);
    for (int i = 0; i < kSplitKinds; ++i)
        if (plan.splits == kSplits[i]) return split_allowed(tiles, (int)fp8_groups(a.K), d, i);
    return false;
}

int run(const GemmFp8Args &a, const GemmFp8Plan &plan, const Device &d, cudaStream_t s) {
    if (!plan.pairs) return tile_launch(a, plan.size, plan.splits, s);
    const int clusters = d.sms / 2;
    if (a.out == SVDCACHE_FP8) return plan.size == 256 ? pair_launch<SVDCACHE_FP8, 256>(a, clusters, s) : pair_launch<SVDCACHE_FP8, 128>(a, clusters, s);
    if (a.out == SVDCACHE_BF16) return plan.size == 192 ? pair_launch<SVDCACHE_BF16, 192>(a, clusters, s) : pair_launch<SVDCACHE_BF16, 128>(a, clusters, s);
    return plan.size == 192 ? pair_launch<SVDCACHE_F32, 192>(a, clusters, s) : pair_launch<SVDCACHE_F32, 128>(a, clusters, s);
}

}  // namespace

int gemm_fp8_status_word(int **word) {
    Device d;
    const int rc = device(&d);
    if (!rc) *word = d.status;
    return rc;
}

int gemm_fp8_plan(const GemmFp8Args &a, GemmFp8Plan *plan) {
    Device d;
    const int rc = device(&d);
    if (!rc) *plan = choose(a, d);
    return rc;
}

int gemm_fp8_launch(const GemmFp8Args &a, const GemmFp8Plan *plan, cudaStream_t s) {
    Device d;
    const int rc = device(&d);
    if (rc) return rc;
    if (plan && !allowed(a, *plan, d)) return SVDCACHE_ERR_INVALID_ARG;
    return run(a, plan ? *plan : choose(a, d), d, s);
}

}  // namespace svdc
