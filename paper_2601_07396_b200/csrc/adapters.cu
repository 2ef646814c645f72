// Low-rank adapters of many requests: the first, narrow product t = factor_a A down_a^T of each request's rows, and the loading of
// an adapter into its pool.  The second product, t up_a^T, belongs to the shared projection's kernels (gemm_fp8.cu), whose
// accumulators it is added to.
//
// down_kernel: bound by the bytes of A.  A task is a slot (tile x request) or, where tiles are of 256 rows, half of one; 128 rows of
// A lie on the lanes of the accumulator, the rank on its columns.  As in the projection, K is dealt in groups to the CTAs of a
// cluster where tasks are few; each then adds up a share of the rows from all of them, in rank order.  t leaves as a sum of bf16
// values, since its other factor is held in bf16 (in 32 bits it would need tf32 MMAs at half of bf16's rate with `up` widened).
// Warps: 0 finds the task, TMA producer; 1 MMA issuer; 2-5 accumulator -> t.
#include <algorithm>
#include <atomic>

#include "fp8.cuh"
#include "maps.cuh"
#include "umma.cuh"

namespace svdc {

using namespace sm100;

namespace {

constexpr int kThreads = 192;
constexpr int kStageK = 128;                          // bytes of K per stage: one scale group
constexpr int kMaxStages = 12;
// Dynamic shared memory of a CTA at most: alone on an SM (the projection's pairs need all of one themselves), two on one where there are
// more tasks than SMs, and beside a CTA of the projection's small tiles.  (64 x 18432 x 3072, eight adapters of rank 64: 30.7 us with 50 KB,
// 26.6 with 70, 24.7 with 90.)
constexpr int kAlone = 220 * 1024, kTwoOfAnSm = 110 * 1024, kBesideProjection = 90 * 1024;

struct DownParams {
    Requests q;
    int tiles, slots, halves, sub;                    // rows of a tile: 1 << q.tile_shift = halves * sub
    int rank, parts, width, chunks, groups, splits, stages, tmem_cols;
    uint32_t x_bytes, stage_bytes;
    int64_t pieces;                                   // scale pieces along K
    const uint8_t *SX, *SD;
    int64_t sd_stride;
    const float *factor;
    __nv_bfloat16 *narrow;
    int4 *tile_slots;                                 // null: nobody asks.  Of a tile: where its slots are listed, how many they are, the first one's number and adapter
    int2 *slot_list;                                  // number and adapter
    int *status;
    int limit, withhold;                              // of every wait, in units of 1024 cycles; `withhold`: nothing is loaded, so that they run out
};

// where column n of the rank begins in a row (width 16 or 32)
__device__ __forceinline__ int place_of(int n, int width) { return (width == 16 ? n >> 4 : n >> 5) * kChunkRow + (n & (width - 1)); }
// A finite value that would round to bf16's infinity begins with the largest bf16; the rest of an infinity is 0.
__device__ __forceinline__ float within_bf16(float v) {
    constexpr float kLargest = 3.38953139e38f;          // (2 - 2^-7) 2^127
    return fabsf(v) > kLargest && fabsf(v) < __int_as_float(0x7F800000) ? copysignf(kLargest, v) : v;
}
__device__ __forceinline__ float rest_of(float v, float part) { return fabsf(v) == __int_as_float(0x7F800000) ? 0.0f : v - part; }
// eight values -> their parts in bf16, `width` apart, each the rounded rest of those before
__device__ __forceinline__ void store_parts(__nv_bfloat16 *out, int parts, int width, float (&v)[8]) {
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        if (p >= parts) break;
        __nv_bfloat162 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __floats2bfloat162_rn(within_bf16(v[2 * i]), within_bf16(v[2 * i + 1]));
            v[2 * i] = rest_of(v[2 * i], __low2float(w[i]));
            v[2 * i + 1] = rest_of(v[2 * i + 1], __high2float(w[i]));
        }
        *reinterpret_cast<uint4 *>(out + p * width) = *reinterpret_cast<const uint4 *>(w);
    }
}

__device__ __forceinline__ void request_group(const CUtensorMap &tm_x, const CUtensorMap &tm_d, const DownParams &p, uint32_t dst, uint32_t bar,
                                              int g, bool scales, int64_t m0, int adapter) {
    const uint32_t d_bytes = (uint32_t)p.rank * kStageK;
    mbar_arrive_expect_tx(bar, p.x_bytes + d_bytes + (scales ? 2 * kScalePieceBytes : 0));
    tma_load_2d(dst, &tm_x, bar, g * kStageK, (int)m0);
    tma_load_3d(dst + p.x_bytes, &tm_d, bar, g * kStageK, 0, adapter);
    if (scales) {
        const uint32_t sdst = dst + p.stage_bytes - 2 * kScalePieceBytes;
        const int64_t at = g / kScaleGroups;
        bulk_load(sdst, p.SX + ((size_t)(m0 / kScaleRows) * p.pieces + at) * kScalePieceBytes, kScalePieceBytes, bar);
        bulk_load(sdst + kScalePieceBytes, p.SD + (size_t)adapter * p.sd_stride + (size_t)at * kScalePieceBytes, kScalePieceBytes, bar);
    }
}

// the rows of a task that a CTA adds up from all S CTAs of its cluster, in rank order, eight columns at a time
struct Share {
    uint32_t sums;                                    // where they lie in each CTA's shared memory, `pitch` floats a row
    __nv_bfloat16 *out;
    int pitch, ldt, row0, rows, in_lo, in_hi, parts, width, blocks, rank;
    float factor;
};
template <int S> __device__ __forceinline__ void finish_share(const Share &h) {
    for (int i = (int)threadIdx.x; i < h.rows * h.blocks; i += kThreads) {
        const int row = h.row0 + i / h.blocks, b = i % h.blocks;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (row >= h.in_lo && row < h.in_hi && 8 * b < h.rank) {
            const uint32_t src = h.sums + (uint32_t)(row * h.pitch + 8 * b) * 4u;
            float4 part[S][2];
#pragma unroll
            for (int x = 0; x < S; ++x) {
                const uint32_t from = cluster_addr(src, (uint32_t)x);
                part[x][0] = cluster_load(from);
                part[x][1] = cluster_load(from + 16u);
            }
#pragma unroll
            for (int x = 0; x < S; ++x) {
                v[0] += part[x][0].x; v[1] += part[x][0].y; v[2] += part[x][0].z; v[3] += part[x][0].w;
                v[4] += part[x][1].x; v[5] += part[x][1].y; v[6] += part[x][1].z; v[7] += part[x][1].w;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= h.factor;
        }
        store_parts(h.out + (int64_t)row * h.ldt + place_of(8 * b, h.width), h.parts, h.width, v);
    }
}

__global__ void __launch_bounds__(kThreads)
down_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_d, const __grid_constant__ DownParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) unsigned long long bar_mem[2 * kMaxStages + 1];
    __shared__ uint32_t tmem_slot_mem;
    __shared__ int control_mem[2];               // abort flag, limit of the waits
    __shared__ Task task_mem;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(bar_mem), empty = full + 8 * kMaxStages, done_bar = empty + 8 * kMaxStages;
    volatile int *control = control_mem;
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    const int S = p.splits;
    const int rank = (int)(blockIdx.x % (unsigned)S);                   // = rank in the cluster
    const int at = (int)(blockIdx.x / (unsigned)S), slot = at / p.halves, half = at - slot * p.halves;
    const int count = (p.groups - rank + S - 1) / S;                    // groups rank, rank + S, ... of K: at least one
    const int loaded = p.withhold ? 0 : count;

    if (warp == 0 && elect_one()) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        mbar_init(done_bar, 1);
        control_mem[0] = 0;
        control_mem[1] = p.limit;
        fence_barrier_init();
        prefetch_tensormap(&tm_x);
        prefetch_tensormap(&tm_d);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_slot_mem), (uint32_t)p.tmem_cols);
        tmem_relinquish();
    }
    __syncwarp();
    previous_done();
    // The projection's kernel, which may begin now, takes for granted that all before this one is done, and that this one
    // holds its tensor memory.
    if (warp == 1) next_may_launch();
    if (warp == 0) {
        const Task t = find_task(Warp{lane}, p.q, p.tiles, slot);
        const int64_t m0 = ((int64_t)t.tile << p.q.tile_shift) + half * p.sub;
        if (lane == 0) task_mem = t;
        if (t.adapter >= 0 && t.lo < m0 + p.sub && t.hi > m0 && elect_one())
            for (int i = 0; i < p.stages && i < loaded; ++i)
                request_group(tm_x, tm_d, p, base + i * p.stage_bytes, full + 8 * i, rank + i * S, i == 0 || (rank + i * S) % kScaleGroups < S, m0, t.adapter);
    } else if (warp == 2 && p.tile_slots) {
        for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) write_tile_slots(Warp{lane}, p.q, (int)t, p.tile_slots, p.slot_list);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&tmem_slot_mem;
    const Task t = task_mem;
    const int64_t m0 = ((int64_t)t.tile << p.q.tile_shift) + half * p.sub;
    const bool live = t.adapter >= 0 && t.lo < m0 + p.sub && t.hi > m0;  // the same in all CTAs of the cluster
    const int ldt = p.chunks * kChunkRow, blocks32 = (p.rank + 31) / 32;
    __nv_bfloat16 *out = p.narrow + (((int64_t)slot << p.q.tile_shift) + half * p.sub) * ldt;
    const int per = (p.sub + S - 1) / S, row0 = rank * per, rows = min(per, p.sub - row0);   // of the task, that this CTA writes
    if (!live) {
        if (t.adapter >= 0)                                              // the slot's rows in the other half: zeros here
            for (int i = (int)threadIdx.x; i < rows * ldt / 8; i += kThreads) *reinterpret_cast<uint4 *>(out + (int64_t)row0 * ldt + i * 8) = make_uint4(0, 0, 0, 0);
        if (warp == 1) tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
        return;
    }
    const float factor = p.factor[t.adapter];
    const int in_lo = (int)(t.lo - m0), in_hi = (int)(t.hi - m0);       // rows of the task that are the request's

    if (warp == 0) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0;
            for (int i = p.stages; i < loaded; ++i) {
                if (!mbar_wait_control(empty + 8 * s, ph, control, 1)) break;
                const int g = rank + i * S;
                request_group(tm_x, tm_d, p, base + s * p.stage_bytes, full + 8 * s, g, g % kScaleGroups < S, m0, t.adapter);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0, set = 1;
            // scale words: four columns for A, which are read up to two columns further where x_word is 2, and from the eighth on four for down; two
            // sets that alternate
            const uint32_t sf = tmem + (uint32_t)p.tmem_cols - 32u;
            const uint32_t x_word = (uint32_t)(m0 % kScaleRows) / 32u;   // 0 or 2: a task of 64 rows may begin in the middle of a piece
            const int n = (p.rank + 15) / 16 * 16;                       // columns beyond the rank come from rows that were not loaded
#pragma unroll 4
            for (int i = 0; i < count; ++i) {
                const int g = rank + i * S;
                if (!mbar_wait_control(full + 8 * s, ph, control, 2)) break;
                tc_fence_after();
                const uint32_t src = base + s * p.stage_bytes;
                if (i == 0 || g % kScaleGroups < S) {
                    set ^= 1u;
                    const uint32_t ssrc = src + p.stage_bytes - 2 * kScalePieceBytes;
                    tmem_cp_scales(sf + 16 * set + 8, smem_desc_scales(ssrc + kScalePieceBytes));
                    tmem_cp_scales(sf + 16 * set, smem_desc_scales(ssrc));
                }
                const uint64_t xd = smem_desc_kmajor(src, 128), dd = smem_desc_kmajor(src + p.x_bytes, 128);
                const uint32_t idesc = idesc_mxf8(128, n, g & 3);
#pragma unroll
                for (int ks = 0; ks < kStageK / 32; ++ks)
                    mma_mxf8_ss(tmem, xd + 2 * ks, dd + 2 * ks, idesc, sf + 16 * set + x_word, sf + 16 * set + 8, (i > 0 || ks > 0) ? 1u : 0u);
                mma_commit(empty + 8 * s);
                if (++s == p.stages) { s = 0; ph ^= 1u; }
            }
            mma_commit(done_bar);
        }
        __syncwarp();
    }
    const int pitch = blocks32 * 32 + 4;                                // of a row of sums in shared memory, in floats
    if (warp >= 2) {
        const int q = warp & 3, row = q * 32 + lane;
        const bool ok = __all_sync(0xFFFFFFFFu, mbar_wait_control(done_bar, 0u, control, 3));
        tc_fence_after();
        for (int c = 0; ok && c < blocks32; ++c) {
            uint32_t acc[32];
            tmem_ld_32x32(tmem + ((uint32_t)(q * 32) << 16) + c * 32, acc);
            tmem_wait_ld();
            const bool in = row >= in_lo && row < in_hi;
            if (S > 1 && row < p.sub) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const uint32_t w[4] = {acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
                    shared_store(base + (uint32_t)(row * pitch + c * 32 + i) * 4u, w);
                }
            } else if (row < p.sub) {
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    const int n = c * 32 + i;
                    if (n >= p.chunks * p.width) break;
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = in && n < p.rank ? __uint_as_float(acc[i + j]) * factor : 0.0f;
                    store_parts(out + (int64_t)row * ldt + place_of(n, p.width), p.parts, p.width, v);
                }
            }
            __syncwarp();
        }
        tc_fence_before();
    }
    if (S > 1) {
        __syncwarp();
        cluster_sync();                                                 // every CTA's sums lie in its shared memory
        const Share share{base, out, pitch, ldt, row0, rows, in_lo, in_hi, p.parts, p.width, p.chunks * p.width / 8, p.rank, factor};
        switch (S) {
            case 2: finish_share<2>(share); break;
            case 4: finish_share<4>(share); break;
            default: finish_share<8>(share); break;
        }
        // No CTA's sums are read any more: they are in registers.  (With a release the arrival waits for the stores of t, 8 us
        // where the projection's loads keep the memory busy.)
        __syncwarp();
        cluster_arrive_relaxed();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (control[0] && lane == 0) {
        // a wait ran out: tell the host, and let what is in flight land before the memory goes
        atomicExch(p.status, SVDCACHE_ERR_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < kWaitCycles / 100) {}
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
    }
}

// ------------------------------------------------------------------------------- loading an adapter ---

struct LoadArgs {
    const void *up;
    int64_t ldu, up_ld, down_ld;
    __nv_bfloat16 *to;
    uint8_t *down, *scales;
    float *factor_to;
    float factor;
    int r, rank, N, K;
    int64_t pieces;
};

// rows r .. rank - 1 of down: zeros, whose groups have scale 1; and the factor
__global__ void pad_kernel(const LoadArgs a) {
    previous_done();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i == 0) *a.factor_to = a.factor;
    const int row = a.r + (int)(i / a.K), c = (int)(i % a.K);
    if (row >= a.rank) return;
    a.down[(int64_t)row * a.down_ld + c] = 0;
    if (c % kFp8Group == 0) a.scales[fp8_scale_offset(row, c / kFp8Group, a.pieces)] = 127;
}

// N x r of up into bf16, zeros behind r; runs after pad_kernel
template <typename T> __global__ void up_kernel(const LoadArgs a) {
    previous_done();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t n = i / a.rank;
    const int c = (int)(i % a.rank);
    if (n >= a.N) return;
    const __nv_bfloat16 v = c < a.r ? __float2bfloat16_rn((float)reinterpret_cast<const T *>(a.up)[n * a.ldu + c]) : __nv_bfloat16(0.0f);
    const bool finite = fabsf(__bfloat162float(v)) < __int_as_float(0x7F800000);
    a.to[n * a.up_ld + c] = finite ? v : __nv_bfloat16(0.0f);
    if (!finite) *a.factor_to = __int_as_float(0x7FC00000);
}

// ------------------------------------------------------------------------- host side ---

// leave to use an SM's shared memory, asked for once per device
int allow_shared_memory() {
    static std::atomic<bool> done[64];
    int dev = 0;
    int rc = record_cuda(cudaGetDevice(&dev));
    if (rc || (dev < 64 && done[dev].load(std::memory_order_acquire))) return rc;
    rc = record_cuda(cudaFuncSetAttribute((const void *)down_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kAlone));
    // An SM divides its memory into L1 and shared when a kernel comes to it, and keeps that while it runs: the projection's CTAs,
    // which need most of it, could not join this kernel's on the share that these need.
    if (!rc) rc = record_cuda(cudaFuncSetAttribute((const void *)down_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    if (!rc && dev < 64) done[dev].store(true, std::memory_order_release);
    return rc;
}

}  // namespace

AdapterLayout adapter_layout(int64_t M, int tile_rows, int rank, int requests, int parts) {
    AdapterLayout l{};
    l.tiles = (M + tile_rows - 1) / tile_rows;
    l.slots = l.tiles + requests;
    l.narrow_rows = l.slots * tile_rows;
    l.parts = parts;
    l.width = l.parts == 3 || rank <= 16 ? 16 : 32;
    l.chunks = (rank + l.width - 1) / l.width;
    l.tile_slots = (size_t)l.narrow_rows * l.chunks * kChunkRow * 2;          // a multiple of 2048
    l.slot_list = align_up(l.tile_slots + (size_t)l.tiles * sizeof(int4), kAlign);
    l.total = align_up(l.slot_list + (size_t)l.slots * sizeof(int2), kAlign);
    return l;
}

Requests requests_of(const GemmFp8Args &a, const AdapterCall &c, int tile_rows) {
    Requests q{c.row_start, c.adapter, c.first, a.M, c.requests, c.pool.count, 0};
    while ((1 << q.tile_shift) < tile_rows) ++q.tile_shift;
    return q;
}

namespace {
int down_columns(int rank) { return rank <= 32 ? 64 : rank <= 96 ? 128 : 256; }
uint32_t down_stage_bytes(int tile_rows, int rank) { return (uint32_t)(std::min(tile_rows, 128) + (rank + 15) / 16 * 16) * kStageK + 2 * kScalePieceBytes; }
}  // namespace

size_t adapter_down_beside(int rank) { return shared_for(kBesideProjection, down_columns(rank)); }

KernelSize adapter_down_size(const AdapterLayout &l, int K, int rank, int requests, int tile_rows, int splits, bool brief, int sms) {
    const int sub = std::min(tile_rows, 128), halves = tile_rows / sub, groups = (int)fp8_groups(K);
    const uint32_t stage_bytes = down_stage_bytes(tile_rows, rank);
    KernelSize k{};
    k.columns = down_columns(rank);
    // tasks that have work: a tile's, and one more where a request begins in the middle of a tile
    const int64_t tasks = l.slots * halves, busy = l.tiles * halves + requests - 1;
    // K is shared by as many CTAs as there are SMs beside a projection of 25 us or less (2048 x 1152 x 4608: 17.9 us with four CTAs a task,
    // 21.0 with one), and where K is long; beside longer ones fewer CTAs leave more SMs to the projection, which begins on those that
    // are free (4608 x 9216 x 3072: 104.6 us with four, 102.4 with one; 4608 x 3072 x 12288: 148.7 with one, 144.7 with two, 147.2 with
    // four).  Beside small tiles half of the SMs (64 x 18432 x 3072, 64 adapters: 40.1 us with two, 37.4 with one); beside shared ones no more
    // CTAs than share the projection's tiles, and than there are SMs (64 x 512 x 2048, 64 requests of rank 128: 44.7 us with eight, 40.1 with two).
    k.cluster = 1;
    while (k.cluster < 8 && groups >= 4 * k.cluster && (splits > 1 ? 2 * k.cluster <= splits && busy * k.cluster * 2 <= sms : busy * k.cluster * 2 <= (splits == 1 ? sms / 2 : brief || groups > 48 * k.cluster ? sms : 0)))
        k.cluster *= 2;
    k.ctas = tasks * k.cluster;
    const int longest = (groups + k.cluster - 1) / k.cluster;
    // an MMA reads 128 rows whatever there are of A: what follows them then stands in rows of the sum that nobody reads
    const int beyond = (128 - sub) * kStageK;
    const int most = tile_rows <= 128 ? kBesideProjection : busy * k.cluster > sms ? kTwoOfAnSm : kAlone;
    k.stages = std::min({(int)((most - 1024 - beyond) / stage_bytes), kMaxStages, longest});
    const size_t ring = (size_t)k.stages * stage_bytes + (size_t)beyond;
    const size_t sums = k.cluster == 1 ? 0 : (size_t)sub * ((rank + 31) / 32 * 32 + 4) * 4;
    k.shared = shared_for(1024 + std::max(ring, sums), k.columns);
    return k;
}

int adapter_down_launch(const GemmFp8Args &a, const AdapterCall &c, const AdapterLayout &l, int tile_rows, int splits, bool brief, int sms, cudaStream_t s) {
    int rc = allow_shared_memory();
    if (rc) return rc;
    const KernelSize k = adapter_down_size(l, a.K, c.pool.rank, c.requests, tile_rows, splits, brief, sms);
    DownParams p{};
    p.q = requests_of(a, c, tile_rows);
    p.tiles = (int)l.tiles; p.slots = (int)l.slots;
    p.sub = tile_rows < 128 ? tile_rows : 128;
    p.halves = tile_rows / p.sub;
    p.rank = c.pool.rank; p.parts = l.parts; p.width = l.width; p.chunks = l.chunks; p.groups = (int)fp8_groups(a.K);
    p.splits = k.cluster; p.stages = k.stages; p.tmem_cols = k.columns;
    p.x_bytes = (uint32_t)p.sub * kStageK;
    p.stage_bytes = down_stage_bytes(tile_rows, p.rank);
    p.pieces = fp8_piece_cols(a.K);
    p.SX = (const uint8_t *)a.SA; p.SD = (const uint8_t *)c.pool.down_scales; p.sd_stride = c.pool.scales_stride;
    p.factor = c.pool.factor;
    char *ws = (char *)c.workspace;
    p.narrow = (__nv_bfloat16 *)ws; p.tile_slots = tile_rows > 128 ? (int4 *)(ws + l.tile_slots) : nullptr; p.slot_list = (int2 *)(ws + l.slot_list);
    p.status = a.status; p.limit = (int)((a.limit > 0 ? a.limit : kWaitCycles) / 1024); p.withhold = a.limit > 0;
    if (k.ctas > 0x7FFFFFFFLL) return SVDCACHE_ERR_BAD_SHAPE;
    CUtensorMap tm_x, tm_d;
    rc = byte_map(&tm_x, a.A, a.M, a.K, a.lda, p.sub);
    if (!rc) rc = byte_map(&tm_d, c.pool.down, c.pool.rank, a.K, c.pool.down_ld, c.pool.rank, c.pool.count, c.pool.down_stride);
    if (rc) return rc;
    return launch_early(down_kernel, dim3((unsigned)k.ctas), dim3(kThreads), k.shared, k.cluster, s, tm_x, tm_d, p);
}

int adapter_load_launch(const svdcache_adapters &pool, int index, const void *down, int64_t ldd, const void *up, int64_t ldu, int r, float factor,
                        int N, int K, int dtype, cudaStream_t s) {
    LoadArgs a{};
    a.up = up; a.ldu = ldu; a.up_ld = pool.up_ld; a.down_ld = pool.down_ld; a.factor = factor; a.r = r; a.rank = pool.rank; a.N = N; a.K = K;
    a.pieces = fp8_piece_cols(K);
    a.to = (__nv_bfloat16 *)pool.up + (int64_t)index * pool.up_stride;
    a.down = (uint8_t *)pool.down + (int64_t)index * pool.down_stride;
    a.scales = (uint8_t *)pool.down_scales + (int64_t)index * pool.scales_stride;
    a.factor_to = pool.factor + index;
    int rc = quantize_fp8_launch(down, r, K, ldd, dtype, 1, a.down, pool.down_ld, a.scales, s);
    const int64_t pad = (int64_t)(pool.rank - r) * K, cells = (int64_t)N * pool.rank;
    if (!rc) rc = launch_early(pad_kernel, dim3((unsigned)(pad / 256 + 1)), dim3(256), 0, 1, s, a);
    if (!rc)
        rc = launch_early(dtype == SVDCACHE_BF16 ? up_kernel<__nv_bfloat16> : up_kernel<float>, dim3((unsigned)((cells + 255) / 256)), dim3(256), 0, 1, s, a);
    return rc;
}

}  // namespace svdc
