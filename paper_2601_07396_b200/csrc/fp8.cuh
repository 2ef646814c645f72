// The 8-bit matrices of the library: e4m3 values with one power-of-two scale per 1 x 128 group of a row.
//
//   scale = 2^e with e the smallest integer for which 448 * 2^e >= the group's largest finite magnitude
//   (e = 0 for a group without one, e >= -127), stored as the byte e + 127 (E8M0)
//   value = e4m3(y / scale), round to nearest even; Inf and NaN become the NaN code, so they stay with
//   their element and reach every sum it enters
//
// A power of two costs no bit of an e4m3 value's mantissa (the format floats on its own; what is given up is
// at most one of its 18 binades at the low end), the division is exact, value * scale is exact in bf16, and
// the tensor cores take such a scale as an operand of the product.
//
// Scales lie in pieces of 512 bytes, one per 128 rows and 4 groups, pieces of the same rows side by side.
// The byte of row m and group g is byte (m % 32) * 16 + (m / 32 % 4) * 4 + g % 4 of piece (m / 128, g / 4):
// the layout that tcgen05.cp carries into tensor memory with one instruction per piece, so that the product
// reads the scales as they are stored.  Bytes of rows and groups that do not exist are never written, and
// never reach a result.
#pragma once

#include <cuda_fp8.h>

#include "internal.cuh"
#include "slots.cuh"

namespace svdc {

constexpr int kFp8Group = 128;          // elements of a row that share a scale
constexpr int kScaleRows = 128;         // rows of a piece of scales
constexpr int kScaleGroups = 4;         // groups of a piece of scales
constexpr int kScalePieceBytes = kScaleRows * kScaleGroups;

__host__ __device__ inline int64_t fp8_groups(int64_t cols) { return (cols + kFp8Group - 1) / kFp8Group; }
__host__ __device__ inline int64_t fp8_piece_cols(int64_t cols) { return (fp8_groups(cols) + kScaleGroups - 1) / kScaleGroups; }
inline size_t fp8_scale_bytes(int64_t rows, int64_t cols) {
    return (size_t)((rows + kScaleRows - 1) / kScaleRows) * (size_t)fp8_piece_cols(cols) * kScalePieceBytes;
}

// byte offset of the scale of row m, group g; `pieces` = fp8_piece_cols(cols)
__device__ __forceinline__ int64_t fp8_scale_offset(int64_t m, int g, int64_t pieces) {
    const int r = (int)(m & (kScaleRows - 1));
    return ((m / kScaleRows) * pieces + g / kScaleGroups) * kScalePieceBytes + (r & 31) * 16 + (r >> 5) * 4 + (g & 3);
}

// Scale byte of a group whose largest finite magnitude is `top` (not NaN, not Inf): 448 = 1.75 * 2^8, so with
// top = 1.f * 2^k the exponent is k - 8, and one more where the fraction f is above 0.75.
__device__ __forceinline__ uint32_t fp8_scale_byte(float top) {
    if (!(top > 0.0f)) return 127u;
    const int e = (int)((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 8;
    return e > 0 ? (uint32_t)e : 0u;
}
// 1 / scale: exact, and finite for every byte that fp8_scale_byte returns (0 .. 247)
__device__ __forceinline__ float fp8_inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

__device__ __forceinline__ float fp8_nan_if_not_finite(float v) {
    return fabsf(v) < __int_as_float(0x7F800000) ? v : __int_as_float(0x7FC00000);
}
// four values -> four e4m3 bytes, the first in the low byte (NaN -> 0x7F or 0xFF; |v| <= 448 otherwise)
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}

// Two fp32 values in one 64-bit register, and the arithmetic that takes such pairs in one instruction.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void pair_to(uint64_t p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// x / (1 + exp(-2u)) by ex2 and rcp (each good to a few 2^-23): exp(-2u) = 2^(x (a + b x^2)).  Beyond the range of
// exp the quotient is 0 or x.  The ftz forms are one instruction each; what they flush (exp below 2^-126 beside the 1, a
// quotient below |x| 2^-126) is far below the sum's own rounding.
__device__ __forceinline__ uint64_t gelu_tanh(uint64_t x) {
    constexpr float kA = -2.3022082f, kB = -0.10294324f;           // -2 sqrt(2 / pi) log2(e) {1, 0.044715}
    float t0, t1, e0, e1;
    pair_to(pair_mul(x, pair_fma(pair_mul(x, x), pair_of(kB, kB), pair_of(kA, kA))), t0, t1);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t0));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t1));
    pair_to(pair_add(pair_of(e0, e1), pair_of(1.0f, 1.0f)), e0, e1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(e0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(e1));
    return pair_mul(x, pair_of(e0, e1));
}

// These kernels are short and follow one another, so each may be launched while the one before it still runs: what
// does not touch memory of the stream's other work (barriers, tensor memory, descriptors) comes before
// previous_done(), everything else after it, and next_may_launch() lets the following kernel begin its own such part.
// previous_done() returns when all earlier work of the stream is complete and visible.
__device__ __forceinline__ void previous_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void next_may_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
int launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const int rc = record_cuda(cudaLaunchKernelEx(&cfg, kernel, P(args)...));
    if (rc) return rc;
    count_launch();
    return check_last_launch();
}

// launches (quant_fp8.cu, gemm_fp8.cu)
int quantize_fp8_launch(const void *X, int64_t rows, int cols, int64_t ld, int dtype, int tile_rows, void *Q, int64_t ldq,
                        void *S, cudaStream_t s);
int rmsnorm_fp8_launch(const void *H, int64_t ldh, const void *X, int64_t ldx, void *H_out, int64_t ldo, const float *weight,
                       float eps, void *Q, int64_t ldq, void *S, int64_t rows, int D, int dtype, cudaStream_t s);

// launches (rotary.cu): queries and keys (null: none), norm and rotation
int rotary_table_launch(const void *positions, int64_t tokens, int64_t ld, int type, int axes, const int *dims, const double *bases,
                        float *table, int64_t ldt, cudaStream_t s);
int rotary_launch(const svdcache_heads *const (&in)[2], const svdcache_heads *const (&out)[2], const float *const (&weight)[2], bool norm, float eps,
                  int64_t batch, int64_t tokens, int dim, int dtype, const svdcache_rotation *rotation, cudaStream_t s);

struct GemmFp8Args {
    const void *A, *B;      // e4m3 [M x K], [N x K]
    const void *SA, *SB;    // their scales
    int64_t lda, ldb, ldc;
    const float *bias;      // N, or null
    void *C, *SC;           // output, and its scales where it is 8-bit
    int64_t M;
    int N, K;
    int act, out;           // SVDCACHE_ACT_*, dtype of C
    int *status;            // device word that receives SVDCACHE_ERR_TIMEOUT if a bounded wait runs out
    long long limit;        // 0, or for a test of that: cycles after which the waits run out, for loads that are not made
};
// How a product is taken: by pairs of CTAs in tiles of 256 x `size`, or in tiles of `size` rows x 128 that `splits` CTAs
// share; tiles that follow one another on an SM (at most), and the model's time.
struct GemmFp8Plan {
    bool pairs;
    int size, splits;
    int64_t rounds, time;
};
int gemm_fp8_plan(const GemmFp8Args &a, GemmFp8Plan *plan);        // the one that the model chooses (A, B, C and status are not used)
int gemm_fp8_launch(const GemmFp8Args &a, const GemmFp8Plan *plan, cudaStream_t s);   // plan null: the model's; else one that it may choose
int gemm_fp8_status_word(int **word);   // the current device's default status word

// A product with adapters: what lies in the workspace, for tiles of `tile_rows` rows and their slots (slots.cuh).
// `narrow` holds tile_rows rows for each slot with an adapter: factor * A down^T where the row is the
// request's, zeros elsewhere, as a sum of bf16 values.  For bf16 output two (off by 2^-16 of the value at most; one would be off by
// 2^-8, as much as the output's rounding), in chunks of 32 of the rank, or of 16 where that holds it.  For fp32 and 8-bit output
// three (2^-24), in chunks of 16: a value near a rounding boundary of e4m3 moves by a whole step, and with two parts 7 in 10^5 did,
// with three 1.4 (9216 x 12288 x 3072, rank 32: 268 and 271 us); two for 8-bit output where the caller's workspace holds no more.  A row of a
// chunk is kChunkRow values: the first of the two or three, then the seconds, ...
constexpr int kChunkRow = 64;
struct AdapterLayout {
    int64_t tiles, slots, narrow_rows;
    int parts, width, chunks;
    size_t tile_slots, slot_list, total;             // offsets in bytes; narrow lies at 0
};
AdapterLayout adapter_layout(int64_t M, int tile_rows, int rank, int requests, int parts);

struct AdapterCall {
    svdcache_adapters pool;
    const int32_t *row_start, *adapter;
    int requests;
    void *workspace;
    size_t room;                                     // its bytes
    int64_t first;                                   // row of the caller's that the launch begins with
};
// how a kernel is launched: CTAs, how many of them a cluster has, dynamic shared memory and columns of tensor memory of each
struct KernelSize {
    int64_t ctas;
    int cluster, columns, stages;
    size_t shared;
};
// The narrow product's, for a projection by small tiles that `splits` CTAs share, or by pairs (0); brief: that takes little time.
KernelSize adapter_down_size(const AdapterLayout &l, int K, int rank, int requests, int tile_rows, int splits, bool brief, int sms);
// the most that it asks for beside small tiles
size_t adapter_down_beside(int rank);
// both kernels' for a plan, by numbers alone
void gemm_fp8_adapters_size(int64_t M, int N, int K, int rank, int requests, int out, const GemmFp8Plan &plan, bool brief, int sms, KernelSize (&size)[2]);
int adapter_down_launch(const GemmFp8Args &a, const AdapterCall &c, const AdapterLayout &l, int tile_rows, int splits, bool brief, int sms, cudaStream_t s);
Requests requests_of(const GemmFp8Args &a, const AdapterCall &c, int tile_rows);
int adapter_load_launch(const svdcache_adapters &pool, int index, const void *down, int64_t ldd, const void *up, int64_t ldu, int r, float factor,
                        int N, int K, int dtype, cudaStream_t s);
int gemm_fp8_adapters_launch(const GemmFp8Args &a, const AdapterCall &c, const GemmFp8Plan *plan, cudaStream_t s);   // plan as above

}  // namespace svdc
