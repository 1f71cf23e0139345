// Product of 8-bit matrices with a scale for each block of 128 (perf_gemm_fp8):
//     C[m][n] = alpha * sum_j scaleA[m][j] * scaleB[n or n / 128][j] * sum_{k in block j} A[m][k] * B[n][k].
// A block of K is one v_mfma_f32_16x16x128_f8f6f4: its result, started from zero, is scaled on the vector units and added to
// the fp32 sums.  The rows of B are the instruction's first operand, so that a lane holds four neighbouring n of one m: the
// scale of A is one value per lane and 16 rows, and C leaves in runs of four.  Which lane holds which k of a block does not
// matter as long as both operands agree.
//
// What the matrix instruction does with a block is less than fp32: of eight products it keeps what reaches down to 2^-13 of
// the largest and drops the rest before they are added (measured with single products; on normal operands the result is off
// by 1.3e-5 of its norm, whatever K).  Below the rounding of a bf16 C, 1.6e-3, that does not show.  For an fp32 C the operands
// are widened to bf16, exactly, and multiplied by v_mfma_f32_16x16x32_bf16, whose sums are fp32 (3e-8): half the rate.
//
//  * gemm_fp8_tile_kernel: operands pass through LDS, two or four stages of one block of K; a workgroup tile of 256 x 256 (bf16 C)
//    or 128 x 128 (fp32 C: or 128 x 96).  Bound by the matrix units at the clock that their power leaves (1.55 to 1.83 GHz) and by
//    the additions beside them: 4096^3 bf16 C 62 to 67 us (2.1 PFLOP/s), fp32 C 120 to 130 us (1.1 PFLOP/s).
//  * gemm_fp8_waves_kernel: few output tiles or few rows; the waves of a workgroup share one tile and divide the blocks
//    of K, each with LDS of its own to load through; their sums are added through LDS in the waves' order.  Bound by the
//    operands' bytes: 64 x 14336 x 4096 14.2 us (4.3 TB/s); 1 x 4096 x 4096 5.4 us, of which half is the launch.
#include <atomic>
#include "fp8.h"
#include "mfma_tile.h"
#include "host_utils.h"

namespace perf {

typedef int int8v_t __attribute__((ext_vector_type(8)));
typedef int int4v_t __attribute__((ext_vector_type(4)));

struct Gemm8Args {
    const uint8_t *A, *B;
    const float *sa, *sb;
    void *C;
    int M, N, K;
    int64_t lda, ldsa, ldb, ldsb, ldc, strideA, strideSA, strideB, strideSB, strideC;
    int64_t batch;
    int b_block_rows;
    float alpha;
};

// A lane's share of 16 rows of an operand in a block, as the matrix instruction takes it: 32 bytes, or with WIDE 32 bf16.
template <bool WIDE> struct Fragment { int8v_t v; };
template <> struct Fragment<true> { bf16x8_t v[4]; };

// Elements 2 w and 2 w + 1 of a fragment's eight from 8 q on, times a power of two, as bf16, exactly: one instruction
template <bool E5M2>
__device__ __forceinline__ void widen_two(Fragment<true> &f, int8v_t v, int q, int w, float power = 1.0f)
{
    const int src = v[2 * q + (w >> 1)];
    if constexpr (E5M2) {
        const auto two = (w & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(src, power, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(src, power, false);
        f.v[q][2 * w] = two[0], f.v[q][2 * w + 1] = two[1];
    } else {
        const auto two = (w & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(src, power, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(src, power, false);
        f.v[q][2 * w] = two[0], f.v[q][2 * w + 1] = two[1];
    }
}
template <bool WIDE, bool E5M2>
__device__ __forceinline__ Fragment<WIDE> as_fragment(int8v_t v, float power = 1.0f)
{
    Fragment<WIDE> f;
    if constexpr (!WIDE) {
        f.v = v;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int w = 0; w < 4; ++w) widen_two<E5M2>(f, v, q, w, power);
    }
    return f;
}

// 16 x 16 sums of a block: rows of B (e4m3) by rows of A (e4m3, or e5m2 with A5), times 2^(exponent - 127)
template <bool WIDE, bool A5>
__device__ __forceinline__ float4_t mma_block(const Fragment<WIDE> &b, const Fragment<WIDE> &a, int exponent = 127)
{
    float4_t c = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[q], a.v[q], c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, c, 0, A5 ? 1 : 0, 0, exponent, 0, 127);
    }
    return c;
}

// Clears the elements of 16 from `n` on.
__device__ __forceinline__ int4v_t keep_first(int4v_t v, int n)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int m = n - 4 * w;
        v[w] &= m >= 4 ? -1 : m <= 0 ? 0 : (1 << (8 * m)) - 1;
    }
    return v;
}

// Bytes of an operand's rows as a buffer: to the last row's last element, rounded up to whole words (a word that holds an
// element is readable).  What lies behind reads as zero.
__device__ __forceinline__ int operand_bytes(int rows, int64_t ld, int K)
{
    return (int)(((int64_t)(rows - 1) * ld + K + 3) & ~(int64_t)3);
}

template <typename CT> __device__ __forceinline__ void store_four(CT *p, const float (&v)[4], int n);
template <> __device__ __forceinline__ void store_four<float>(float *p, const float (&v)[4], int n)
{
    if (n >= 4) {
        __builtin_nontemporal_store(float4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<float4_at4 *>(p));
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) p[e] = v[e];
    }
}
template <> __device__ __forceinline__ void store_four<uint16_t>(uint16_t *p, const float (&v)[4], int n)
{
    if (n >= 4) {
        *reinterpret_cast<uint2_at2 *>(p) = uint2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) p[e] = f32_to_bf16(v[e]);
    }
}

// A half fragment's elements behind the row's end are cleared: `left` of them from the block's start on are inside.
__device__ __forceinline__ int8v_t masked_fragment(int8v_t v, int left, int lane)
{
    const int4v_t lo = keep_first(int4v_t{v[0], v[1], v[2], v[3]}, left - 16 * (lane >> 4));
    const int4v_t hi = keep_first(int4v_t{v[4], v[5], v[6], v[7]}, left - 16 * (lane >> 4) - 64);
    return int8v_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// All of this wave's LDS accesses are done; its loads stay in flight.
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// TM x TN groups of 16 rows of A and of B per workgroup; its W waves take every W-th block of K, each through a stage of LDS of
// its own, and meet no barrier until their sums are added.  A stage: the rows, 128 bytes each, loaded eight lanes to a row (a
// load of 16 bytes from each of 16 rows, as the fragments lie, moves a third of that per clock) with their chunks permuted
// (swz64), then the scales, loaded a lane to a row.  A block's fragments go to registers at once and the next block's loads
// follow them, so that every wave has a stage in flight while it multiplies (a second stage each: no faster).
constexpr int waves_stage_bytes(int TM, int TN) { return (TM + TN) * 16 * kBlock8 + 512; }

template <int TM, int TN, int W, bool B128, bool A5, typename CT>
__global__ __launch_bounds__(64 * W) void gemm_fp8_waves_kernel(const Gemm8Args g, int tiles_m, int tiles_n)
{
    constexpr bool WIDE = sizeof(CT) == 4;
    constexpr int kStage = waves_stage_bytes(TM, TN);
    extern __shared__ __attribute__((aligned(1024))) char smem[];  // (one array, as in the tile kernel)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t bz = blockIdx.y;
    int tm, tn;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm), tn = __builtin_amdgcn_readfirstlane(tn);  // (divisions leave vector registers)
    const int m0 = tm * 16 * TM, n0 = tn * 16 * TN;
    const int rows_m = min(16 * TM, g.M - m0), rows_n = min(16 * TN, g.N - n0);
    const int blocks = (g.K + kBlock8 - 1) / kBlock8;
    const uint8_t *tile_a = g.A + bz * g.strideA + (int64_t)m0 * g.lda, *tile_b = g.B + bz * g.strideB + (int64_t)n0 * g.ldb;
    const int bytes_a = operand_bytes(rows_m, g.lda, g.K), bytes_b = operand_bytes(rows_n, g.ldb, g.K);
    rsrc_t from_a[2 * TM], from_b[2 * TN];  // the operand from row 8 i on
#pragma unroll
    for (int i = 0; i < 2 * TM; ++i) from_a[i] = make_rsrc(tile_a + (int64_t)(8 * i) * g.lda, max(bytes_a - 8 * i * (int)g.lda, 0));
#pragma unroll
    for (int i = 0; i < 2 * TN; ++i) from_b[i] = make_rsrc(tile_b + (int64_t)(8 * i) * g.ldb, max(bytes_b - 8 * i * (int)g.ldb, 0));
    // rows 8 i + lane / 8: the permutation of odd i is that of even i with its third bit turned
    const uint32_t chunk = (lane & 7) ^ swz64(lane >> 3), row8 = lane >> 3;
    const uint32_t off_a[2] = {(uint32_t)(row8 * g.lda) + chunk * 16, (uint32_t)(row8 * g.lda) + (chunk ^ 4) * 16};
    const uint32_t off_b[2] = {(uint32_t)(row8 * g.ldb) + chunk * 16, (uint32_t)(row8 * g.ldb) + (chunk ^ 4) * 16};
    const rsrc_t scales_a = make_rsrc(g.sa + bz * g.strideSA + (int64_t)m0 * g.ldsa, (uint32_t)(((rows_m - 1) * g.ldsa + blocks) * 4));
    const int first_b = B128 ? n0 / kBlock8 : n0, last_b = B128 ? (n0 + rows_n - 1) / kBlock8 : n0 + rows_n - 1;
    const rsrc_t scales_b = make_rsrc(g.sb + bz * g.strideSB + (int64_t)first_b * g.ldsb, (uint32_t)(((last_b - first_b) * g.ldsb + blocks) * 4));
    const uint32_t off_sa = (uint32_t)(min(lane, rows_m - 1) * g.ldsa * 4);
    const uint32_t off_sb = (uint32_t)(((B128 ? (n0 + min(lane, rows_n - 1)) / kBlock8 : n0 + min(lane, rows_n - 1)) - first_b) * g.ldsb * 4);

    char *const mine = smem + wave * kStage;
    auto load = [&](int kb) {  // (past the last block out of range: nothing is moved)
        const uint32_t at = kb < blocks ? (uint32_t)kb * kBlock8 : kOutOfRange, at_s = kb < blocks ? (uint32_t)kb * 4 : kOutOfRange;
        char *to = mine;
#pragma unroll
        for (int i = 0; i < 2 * TM; ++i) issue_load_to(from_a[i], off_a[i & 1] + at, 0, to + i * 1024);
#pragma unroll
        for (int i = 0; i < 2 * TN; ++i) issue_load_to(from_b[i], off_b[i & 1] + at, 0, to + (2 * TM + i) * 1024);
        to += (TM + TN) * 16 * kBlock8;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(scales_a, (__attribute__((address_space(3))) void *)to, 4, off_sa + at_s, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(scales_b, (__attribute__((address_space(3))) void *)(to + 256), 4, off_sb + at_s, 0, 0, 0);
    };
    float4_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = float4_t{0.f, 0.f, 0.f, 0.f};
    const int place[2] = {frag_offset64(lane & 15, lane >> 4), frag_offset64(lane & 15, (lane >> 4) + 4)};
    load(wave);
    for (int kb = wave; kb < blocks; kb += W) {
        wait_vmem<0>();  // the stage has arrived
        asm volatile("" ::: "memory");
        const char *at = mine;
        auto read = [&](int group) {
            const int4v_t lo = *reinterpret_cast<const int4v_t *>(at + group * 16 * kBlock8 + place[0]);
            const int4v_t hi = *reinterpret_cast<const int4v_t *>(at + group * 16 * kBlock8 + place[1]);
            return int8v_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        int8v_t raw_a[TM], raw_b[TN];
        float fa[TM];
        float4_t fb[TN];
        const char *scales = at + (TM + TN) * 16 * kBlock8;
#pragma unroll
        for (int i = 0; i < TM; ++i) raw_a[i] = read(i), fa[i] = *reinterpret_cast<const float *>(scales + (16 * i + (lane & 15)) * 4);
#pragma unroll
        for (int j = 0; j < TN; ++j) raw_b[j] = read(TM + j), fb[j] = *reinterpret_cast<const float4_t *>(scales + 256 + (16 * j + 4 * (lane >> 4)) * 4);
        wait_lds();  // it is in registers: the stage is free
        asm volatile("" ::: "memory");
        load(kb + W);
        const int left = g.K - kb * kBlock8;
        if (left < kBlock8) {
#pragma unroll
            for (int i = 0; i < TM; ++i) raw_a[i] = masked_fragment(raw_a[i], left, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) raw_b[j] = masked_fragment(raw_b[j], left, lane);
        }
        Fragment<WIDE> b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = as_fragment<WIDE, false>(raw_b[j]);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const Fragment<WIDE> a = as_fragment<WIDE, A5>(raw_a[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const float4_t p = mma_block<WIDE, A5>(b[j], a);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(p[e] * fa[i], fb[j][e], acc[i][j][e]);
            }
        }
    }
    wait_vmem_and_lds<0>();  // (loads into LDS end before its next use)
    wg_barrier();
    float4_t(&sums)[W][TM * TN][64] = *reinterpret_cast<float4_t(*)[W][TM * TN][64]>(smem);
    static_assert(sizeof(sums) <= W * kStage, "the sums fit the stages");
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) sums[wave][i * TN + j][lane] = acc[i][j];
    __syncthreads();
    CT *C = (CT *)g.C + bz * g.strideC;
    for (int t = wave; t < TM * TN; t += W) {
        const int i = t / TN, j = t - i * TN;
        float4_t s = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) s += sums[w][t][lane];
        const int m = m0 + 16 * i + (lane & 15), n = n0 + 16 * j + 4 * (lane >> 4);
        const float v[4] = {g.alpha * s[0], g.alpha * s[1], g.alpha * s[2], g.alpha * s[3]};
        if (m < g.M) store_four<CT>(C + (int64_t)m * g.ldc + n, v, g.N - n);
    }
}

constexpr int tile_stage_bytes(int BM, int BN) { return BM + BN <= 256 ? 256 * kBlock8 : 512 * kBlock8; }  // a power of two
constexpr int scale_stage_bytes(int waves) { return waves * 256; }  // the scales of a block: a lane's each
// S stages of operands and twice as many of scales: those of a block are read when its operands are in registers already
constexpr int tile_lds_bytes(int BM, int BN, int S, int waves) { return S * tile_stage_bytes(BM, BN) + 2 * S * scale_stage_bytes(waves); }

// WM x WN waves, each with TM x TN groups of 16 rows of A and of B.  LDS: S stages of a block of K, rows of 128 bytes whose
// 16-byte chunks are permuted as in mfma_tile.h (swz64), and the blocks' scales.
//
// A step multiplies a block: B's fragments stay in registers, A's pass by, up to four groups ahead; a sum is scaled and
// added behind the third product after its own (a sum can be used some 50 cycles after its instruction; behind the fourth it
// is no faster and takes 16 more registers, in front of that product a lone wave needs 37 cycles for each and not 33).  The waves
// meet once, before the last of these groups, whose fragments are in registers by then: the next stage has arrived, this one is
// free.  Its reload is spread over those groups: in a burst the loads fill the texture path, and a wave whose load cannot
// issue holds back the products behind it.
//
// The scale of a 128 x 128 tile of B (B128) is the same for all sums of a wave: its exponent goes into the matrix
// instruction (WIDE: into B's elements as they are widened), its mantissa into the factor of A's scale, which leaves one
// multiply-add per sum, and no product of two scales that could leave fp32's range.  A block's sum is at most 128 x 57344 x 448,
// less than 2^32: the exponent is taken up to 2^95, down to 2^-60, and what is beyond stays in the factor, which A's scales of
// up to 2^95 keep finite, and whose product with a sum of 2^-60 underflows only where the result does.
template <int TM, int TN, int WM, int WN, int S, bool B128, bool A5, typename CT>
__global__ __launch_bounds__(64 * WM * WN, 2) void gemm_fp8_tile_kernel(const Gemm8Args g, int tiles_m, int tiles_n)
{
    constexpr bool WIDE = sizeof(CT) == 4;
    constexpr int NW = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN;
    constexpr int kStage = tile_stage_bytes(BM, BN), kLoadsA = BM / (8 * NW), kLoadsB = BN / (8 * NW);
    // groups of A that are in registers or on their way there: four, or what the sums and B's scales leave room for
    constexpr int kAhead = TM == 8 && !B128 ? 2 : 4;
    constexpr int kScaleStage = scale_stage_bytes(NW), kScalesAt = 0, kTilesAt = 2 * S * kScaleStage;
    constexpr int kInFlight = kLoadsA + kLoadsB + 1;  // loads of a block
    static_assert((S & (S - 1)) == 0 && (kStage & (kStage - 1)) == 0 && (kScaleStage & (kScaleStage - 1)) == 0, "places wrap by a mask");
    static_assert(kLoadsA == 4 && kLoadsB == TN && (B128 ? BM + 64 : BM + BN) <= 64 * NW, "the loads divide among the waves");
    static_assert(TM == 4 || TM == 8, "the schedule of the loads");
    static_assert(TN == 4 || (TN == 3 && WIDE && !B128), "the order of the sums; a wave's rows of B in one tile of scales");
    // (one array of dynamic size: of several the compiler knows that a load into LDS and a read are of the same one, and waits
    // for every load in flight before each read, whatever their places in it)
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    char *const scales = smem + kScalesAt, *const tiles = smem + kTilesAt;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int64_t bz = blockIdx.y;
    int tm, tn;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm), tn = __builtin_amdgcn_readfirstlane(tn);  // (divisions leave vector registers)
    const int m0 = tm * BM, n0 = tn * BN;
    const int rows_m = min(BM, g.M - m0), rows_n = min(BN, g.N - n0);
    const int blocks = (g.K + kBlock8 - 1) / kBlock8;
    const uint8_t *tile_a = g.A + bz * g.strideA + (int64_t)m0 * g.lda, *tile_b = g.B + bz * g.strideB + (int64_t)n0 * g.ldb;
    const int bytes_a = operand_bytes(rows_m, g.lda, g.K), bytes_b = operand_bytes(rows_n, g.ldb, g.K);
    // this lane's row and chunk in a load of its wave: 8 rows; the wave's loads of a block are 8 NW rows apart
    const int row = wave * 8 + (lane >> 3), chunk_at = ((lane & 7) ^ swz64(row)) << 4;
    const uint32_t off_a = (uint32_t)(row * g.lda) + chunk_at, off_b = (uint32_t)(row * g.ldb) + chunk_at;
    static_assert(NW * 8 % 16 == 0, "the permutation repeats after 16 rows");
    // the row of scales that this lane fetches for all: A's, then B's, of which a tile of B128 has one for 128 rows
    const int slot = wave * 64;
    const bool of_a = slot < BM;
    auto scale_row = [&](int slot) {
        if (of_a) return m0 + min(slot, rows_m - 1);
        return B128 ? min(n0 / kBlock8 + slot - BM, (g.N - 1) / kBlock8) : n0 + min(slot - BM, rows_n - 1);
    };
    const int first_scale = scale_row(slot);
    const int64_t ld_scales = of_a ? g.ldsa : g.ldsb;
    const rsrc_t from_scales = make_rsrc((of_a ? g.sa + bz * g.strideSA : g.sb + bz * g.strideSB) + first_scale * ld_scales,
                                         (uint32_t)(((scale_row(slot + 63) - first_scale) * ld_scales + blocks) * 4));
    const uint32_t off_scale = (uint32_t)((scale_row(slot + lane) - first_scale) * ld_scales * 4);
    // Load i of a block begins with row 8 NW i and ends with the operand: what is behind (rows past the matrix among it) reads
    // as zero.  A load of a block past the last one is out of range altogether: it moves nothing, and the number in flight is
    // the same.
    rsrc_t from_a[kLoadsA], from_b[kLoadsB];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int skip_a = i * NW * 8 * (int)g.lda, skip_b = i * NW * 8 * (int)g.ldb;
        from_a[i] = make_rsrc(tile_a + skip_a, max(bytes_a - skip_a, 0));
        if (i < kLoadsB) from_b[i] = make_rsrc(tile_b + skip_b, max(bytes_b - skip_b, 0));
    }
    auto load = [&](int kb, int i) {
        const uint32_t at = kb < blocks ? (uint32_t)kb * kBlock8 : kOutOfRange;
        char *to = tiles + (kb & (S - 1)) * kStage + (i * NW + wave) * 1024;
        issue_load_to(from_a[i], off_a + at, 0, to);
        if (i < kLoadsB) issue_load_to(from_b[i], off_b + at, 0, to + BM * kBlock8);
    };
    auto load_scale = [&](int kb) {
        const uint32_t at = kb < blocks ? (uint32_t)kb * 4 : kOutOfRange;
        char *to = scales + (kb & (2 * S - 1)) * kScaleStage + wave * 256;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from_scales, (__attribute__((address_space(3))) void *)to, 4, off_scale + at, 0, 0, 0);
    };

    // This lane's places in a stage: of its half fragments of A and B (rows are 16 apart from group to group, which leaves the
    // permutation as it is) and of the scales of its row of A and its four of B.
    const int row_a = wm * 16 * TM, row_b = BM + wn * 16 * TN;
    int at_a[2], at_b[2], at_sa = (row_a + (lane & 15)) * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        at_a[h] = row_a * kBlock8 + frag_offset64(lane & 15, (lane >> 4) + 4 * h);
        at_b[h] = row_b * kBlock8 + frag_offset64(lane & 15, (lane >> 4) + 4 * h);
    }
    const int at_sb = B128 ? (BM + wn * 16 * TN / kBlock8) * 4 : (row_b + 4 * (lane >> 4)) * 4;  // from the stage's scales on
    auto next_stage = [&](int (&at)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) at[h] = S == 2 ? at[h] ^ kStage : (at[h] + kStage) & (S * kStage - 1);
    };
    auto read = [&](const int (&at)[2], int row) {
        const int4v_t lo = *reinterpret_cast<const int4v_t *>(tiles + at[0] + row * kBlock8);
        const int4v_t hi = *reinterpret_cast<const int4v_t *>(tiles + at[1] + row * kBlock8);
        return int8v_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    int8v_t a[kAhead], b[TN];
    float fa[kAhead], next128 = 1.f;
    auto read_a = [&](int i) {
        a[i % kAhead] = read(at_a, 16 * i);
        fa[i % kAhead] = *reinterpret_cast<const float *>(scales + at_sa + 64 * i);
    };
    auto read_128 = [&](int kb) {
        if constexpr (B128) next128 = *reinterpret_cast<const float *>(scales + (kb & (2 * S - 1)) * kScaleStage + at_sb);
    };

    // p: the last four sums, not yet added (WIDE: a group's are begun together and added during the next)
    float4_t acc[TM][TN], p[WIDE ? 2 * TN : TN], fb[TN];
    float factor = 0.f;                   // of the group before
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j] = float4_t{0.f, 0.f, 0.f, 0.f};
        fb[j] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < (WIDE ? 2 * TN : TN); ++j) p[j] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto add = [&](int i, int j, float f) {  // sum j of group i; the empty asm keep the compiler from doing it earlier or later
        float4_t &sum = p[WIDE ? (i & 1) * TN + j : j];
        asm volatile("" : "+v"(sum));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (B128)
                acc[i][j][e] = __builtin_fmaf(sum[e], f, acc[i][j][e]);
            else
                acc[i][j][e] = __builtin_fmaf(sum[e] * f, fb[j][e], acc[i][j][e]);
        }
        asm volatile("" : "+v"(acc[i][j]));
    };

    // the first S blocks; the first is waited for
#pragma unroll
    for (int kb = 0; kb < S; ++kb) {
        load_scale(kb);
#pragma unroll
        for (int i = 0; i < 4; ++i) load(kb, i);
    }
    wait_vmem<(S - 1) * kInFlight>();
    wg_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j) b[j] = read(at_b, 16 * j);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read_a(i);
    read_128(0);

    auto take_scales_b = [&](int kb) {
        if constexpr (!B128) {
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = *reinterpret_cast<const float4_t *>(scales + (kb & (2 * S - 1)) * kScaleStage + at_sb + 64 * j);
        }
    };
    Fragment<WIDE> next_a;  // (WIDE) the next group's fragment, widened during this one's products
    auto step = [&](int kb, auto mask) {
        constexpr bool MASK = decltype(mask)::value;
        const int left = g.K - kb * kBlock8;
        int exponent = 127;
        float mantissa = 1.f;
        if constexpr (B128) {
            const uint32_t bits = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, next128));
            mantissa = __builtin_bit_cast(float, bits);
            exponent = min(max((int)(bits >> 23 & 0xff), 127 - 60), 127 + 95);
            mantissa = __builtin_ldexpf(mantissa, 127 - exponent);
        }
        Fragment<WIDE> fragment_b[WIDE ? TN : 1];
        if constexpr (MASK) {
#pragma unroll
            for (int j = 0; j < TN; ++j) b[j] = masked_fragment(b[j], left, lane);
        }
        if constexpr (WIDE) {
#pragma unroll
            for (int j = 0; j < TN; ++j) fragment_b[j] = as_fragment<WIDE, false>(b[j], __builtin_bit_cast(float, exponent << 23));
            if constexpr (MASK) a[0] = masked_fragment(a[0], left, lane);
            next_a = as_fragment<WIDE, A5>(a[0]);
        }
        unrolled<TM>([&](auto group) {
            constexpr int i = decltype(group)::value;
            if constexpr (i == TM - kAhead) {
                wait_vmem<(S - 2) * kInFlight>();
                wait_lds();
                wg_barrier();
                load_scale(kb + S);
            }
            if constexpr (i >= TM - kAhead) {
#pragma unroll
                for (int l = 0; l < 4 / kAhead; ++l) load(kb + S, (i - (TM - kAhead)) * (4 / kAhead) + l);
            }
            const float f = fa[i % kAhead] * mantissa;
            auto read_next = [&](int j) {  // into the places of what has been used for the last time
                if constexpr (i == TM - 1) {
                    if (j == 0) next_stage(at_b);
                    b[j] = read(at_b, 16 * j);
                }
                if (j == TN - 1) {
                    if constexpr (i == TM - kAhead) next_stage(at_a), at_sa = (at_sa + kScaleStage) & (2 * S * kScaleStage - 1);
                    read_a((i + kAhead) % TM);
                    if constexpr (i == TM - 1) read_128(kb + 1);
                }
            };
            if constexpr (WIDE) {
                static_assert(!WIDE || kAhead == TM, "fragments of the next group are there");
                const Fragment<WIDE> fragment_a = next_a;
                if constexpr (MASK && i < TM - 1) a[(i + 1) % kAhead] = masked_fragment(a[(i + 1) % kAhead], left, lane);
                float4_t *sums = p + (i & 1) * TN;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const float4_t zero = {0.f, 0.f, 0.f, 0.f};
                        sums[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fragment_b[j].v[q], fragment_a.v[q], q ? sums[j] : zero, 0, 0, 0);
                        asm volatile("" : "+v"(sums[j]));  // (the product is begun here)
                    }
                    // (one by one between the products this is no faster)
                    if constexpr (i < TM - 1) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) widen_two<A5>(next_a, a[(i + 1) % kAhead], q, w);
                    }
                    if (q < TN) {
                        add((i + TM - 1) % TM, q, factor);  // of the group before, or of the step before
                        read_next(q);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (i == 0) take_scales_b(kb);
            } else {
                if constexpr (MASK) a[i % kAhead] = masked_fragment(a[i % kAhead], left, lane);
                const Fragment<WIDE> fragment_a = as_fragment<WIDE, A5>(a[i % kAhead]);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    Fragment<WIDE> whole;
                    whole.v = b[j];
                    p[j] = mma_block<WIDE, A5>(whole, fragment_a, exponent);
                    asm volatile("" : "+v"(p[j]));  // (the product is begun here)
                    read_next(j);
                    if (j < TN - 1) {
                        add((i + TM - 1) % TM, j + 1, factor);  // of the group before, or of the step before
                    } else {
                        if constexpr (i == 0) take_scales_b(kb);
                        add(i, 0, f);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            factor = f;
        });
    };
    const int whole = g.K / kBlock8;
    for (int kb = 0; kb < whole; ++kb) step(kb, std::false_type{});
    if (whole < blocks) step(whole, std::true_type{});
#pragma unroll
    for (int j = WIDE ? 0 : 1; j < TN; ++j) add(TM - 1, j, factor);

    // C through this wave's part of LDS, so that it leaves 16 bytes per lane in whole rows of 16 TN columns: written from the
    // registers, 8 or 16 bytes per lane in 16 rows, it took 10 to 17 thousand cycles of the 126 thousand of 4096 x 4096 x 4096.
    wait_vmem_and_lds<0>();
    wg_barrier();  // (everyone's loads into LDS have ended)
    constexpr int kPer = 16 / (int)sizeof(CT), kChunks = 16 * 4 / kPer, kRowsOut = 64 / kChunks;  // (rows of TN = 3 as long as of 4)
    static_assert(NW * 16 * TM * kChunks * 16 <= S * kStage, "the tile fits the stages");
    char *const out = tiles + wave * (16 * TM * kChunks * 16);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int n = 16 * j + 4 * (lane >> 4), chunk = (n / kPer) ^ (row & (kChunks - 1));
            const float v[4] = {g.alpha * acc[i][j][0], g.alpha * acc[i][j][1], g.alpha * acc[i][j][2], g.alpha * acc[i][j][3]};
            char *at = out + (row * kChunks + chunk) * 16;
            if constexpr (sizeof(CT) == 4)
                *reinterpret_cast<float4_t *>(at) = float4_t{v[0], v[1], v[2], v[3]};
            else
                *reinterpret_cast<uint2_t *>(at + (n % kPer) * 2) = uint2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
    }
    wait_lds();
    asm volatile("" ::: "memory");
    CT *C = (CT *)g.C + bz * g.strideC;
    const int chunk = lane % kChunks, n = n0 + wn * 16 * TN + chunk * kPer;
#pragma unroll
    for (int r = 0; r < 16 * TM; r += kRowsOut) {
        const int row_out = r + lane / kChunks, m = m0 + wm * 16 * TM + row_out;
        const uint4_t v = *reinterpret_cast<const uint4_t *>(out + (row_out * kChunks + (chunk ^ (row_out & (kChunks - 1)))) * 16);
        if (m >= g.M || n >= g.N || (TN < 4 && chunk * kPer >= 16 * TN)) continue;
        CT *to = C + (int64_t)m * g.ldc + n;
        if (n + kPer <= g.N) {
            if constexpr (sizeof(CT) == 4)  // (past the caches, two whole lines: 16 x 2113 x 1152 x 264 68 -> 50 us; bf16's single ones: no gain)
                __builtin_nontemporal_store(v, reinterpret_cast<uint4_at4 *>(to));
            else
                *reinterpret_cast<uint4_at2 *>(to) = v;
        } else {
#pragma unroll
            for (int e = 0; e < kPer - 1; ++e)
                if (n + e < g.N) {
                    if constexpr (sizeof(CT) == 4)
                        reinterpret_cast<uint32_t *>(to)[e] = v[e];
                    else
                        to[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                }
        }
    }
}

// Raises a kernel's limit of dynamic LDS, an idempotent setting, at its first launch on each device.
template <auto KERNEL>
static bool allow_lds(int bytes)
{
    static std::atomic<uint64_t> done{0};
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return false;
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

template <int TM, int TN, int WM, int WN, int S, bool A5, typename CT>
static perf_status launch_tile(const Gemm8Args &g, hipStream_t stream)
{
    const int64_t tiles_m = (g.M + 16 * TM * WM - 1) / (16 * TM * WM), tiles_n = (g.N + 16 * TN * WN - 1) / (16 * TN * WN);
    if (tiles_m * tiles_n > max_blocks(64 * WM * WN)) return PERF_ERR_UNSUPPORTED;
    for (int64_t b = 0; b < g.batch; b += kMaxGridYZ) {
        Gemm8Args p = g;
        p.A += b * g.strideA, p.B += b * g.strideB, p.sa += b * g.strideSA, p.sb += b * g.strideSB;
        p.C = (CT *)g.C + b * g.strideC;
        const dim3 grid((unsigned)(tiles_m * tiles_n), (unsigned)std::min(kMaxGridYZ, g.batch - b));
        constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN;
        constexpr int lds = tile_lds_bytes(BM, BN, S, WM * WN);
        if (TN == 4 && g.b_block_rows == kBlock8) {
            if (!allow_lds<gemm_fp8_tile_kernel<TM, 4, WM, WN, S, true, A5, CT>>(lds)) return PERF_ERR_LAUNCH;
            gemm_fp8_tile_kernel<TM, 4, WM, WN, S, true, A5, CT><<<grid, 64 * WM * WN, lds, stream>>>(p, (int)tiles_m, (int)tiles_n);
        } else {
            if (!allow_lds<gemm_fp8_tile_kernel<TM, TN, WM, WN, S, false, A5, CT>>(lds)) return PERF_ERR_LAUNCH;
            gemm_fp8_tile_kernel<TM, TN, WM, WN, S, false, A5, CT><<<grid, 64 * WM * WN, lds, stream>>>(p, (int)tiles_m, (int)tiles_n);
        }
        const perf_status st = launch_status();
        if (st != PERF_OK) return st;
    }
    return PERF_OK;
}

template <int TM, int TN, bool A5, typename CT>
static perf_status launch_waves(const Gemm8Args &g, hipStream_t stream)
{
    constexpr int W = 8;
    const int64_t tiles_m = (g.M + 16 * TM - 1) / (16 * TM), tiles_n = (g.N + 16 * TN - 1) / (16 * TN);
    if (tiles_m * tiles_n > max_blocks(64 * W)) return PERF_ERR_UNSUPPORTED;
    const int lds = W * waves_stage_bytes(TM, TN);
    for (int64_t b = 0; b < g.batch; b += kMaxGridYZ) {
        Gemm8Args p = g;
        p.A += b * g.strideA, p.B += b * g.strideB, p.sa += b * g.strideSA, p.sb += b * g.strideSB;
        p.C = (CT *)g.C + b * g.strideC;
        const dim3 grid((unsigned)(tiles_m * tiles_n), (unsigned)std::min(kMaxGridYZ, g.batch - b));
        if (g.b_block_rows == kBlock8) {
            if (!allow_lds<gemm_fp8_waves_kernel<TM, TN, W, true, A5, CT>>(lds)) return PERF_ERR_LAUNCH;
            gemm_fp8_waves_kernel<TM, TN, W, true, A5, CT><<<grid, 64 * W, lds, stream>>>(p, (int)tiles_m, (int)tiles_n);
        } else {
            if (!allow_lds<gemm_fp8_waves_kernel<TM, TN, W, false, A5, CT>>(lds)) return PERF_ERR_LAUNCH;
            gemm_fp8_waves_kernel<TM, TN, W, false, A5, CT><<<grid, 64 * W, lds, stream>>>(p, (int)tiles_m, (int)tiles_n);
        }
        const perf_status st = launch_status();
        if (st != PERF_OK) return st;
    }
    return PERF_OK;
}

// The widest tile that leaves enough workgroups: 768 x 1024 x 1024 takes 8.4 us with 192 of them and 9.4 with 384 of half the
// size, 128 x 4096 x 4096 12.0 with 128 and 9.4 with 256, 64 x 4096 x 4096 9.4 with 128 and 8.4 with 256.
template <int TM, bool A5, typename CT>
static perf_status waves_by_columns(const Gemm8Args &g, hipStream_t stream)
{
    constexpr int64_t kEnough = 160;
    const int64_t tiles_m = (g.M + 16 * TM - 1) / (16 * TM) * g.batch, widest = tiles_m * ((g.N + 63) / 64);
    // Of the widest, whose LDS takes a CU, no more than one round for few rows: of half the size there are two or three to a CU, and
    // one loads while another adds its sums (1 x 65536 x 2048 32 -> 26.5 us, 1 x 32768 x 4096 31 -> 29; 160 tiles, 1 x 10240 x 8192:
    // 14.3 with them and 16.3 with 320 of half the size).
    if (widest >= kEnough && (TM > 2 || widest <= 256)) return launch_waves<TM, 4, A5, CT>(g, stream);
    if (tiles_m * ((g.N + 31) / 32) >= kEnough) return launch_waves<TM, 2, A5, CT>(g, stream);
    return launch_waves<TM, 1, A5, CT>(g, stream);
}

template <bool A5, typename CT>
static perf_status gemm8(const Gemm8Args &g, hipStream_t stream)
{
    constexpr bool WIDE = sizeof(CT) == 4;
    const int64_t big = ((g.M + 255) / 256) * ((g.N + 255) / 256) * g.batch, mid = ((g.M + 127) / 128) * ((g.N + 127) / 128) * g.batch;
    const int64_t blocks = (g.K + kBlock8 - 1) / kBlock8;
    // A round of 256 tiles of 256 x 256 takes as long as 2.4 of 128 x 128 (K = 4096, N = 4096: 50 us; 41 for two of the latter, 63
    // for three), so the larger ones pay from three rounds of the smaller on.
    if constexpr (!WIDE) {
        if (12 * ((big + 255) / 256) < 5 * ((mid + 255) / 256)) return launch_tile<8, 4, 2, 4, 2, A5, CT>(g, stream);
    }
    // A tile takes its time however few there are, the waves that divide K theirs for each.  192 tiles, K = 3000: 19.5 us against
    // 30.7 (bf16 C); 128 tiles: K = 1024 8.6 against 12.7, K = 4096 21.3 against 23.2, K = 14336 66 against 60; fp32 C: 256 tiles,
    // K = 4096 38 against 54, 128 tiles, K = 700 13.0 against 14.1, K = 4096 37 against 27.  64 tiles, K = 8192: 36 against 20.
    // Few rows leave a tile part empty: 256 tiles of 32 rows, K = 4096 36 against 33 (fp32 50 against 33), 512 of them, K = 1024 15.4
    // against 21; 128 of 64 rows, K = 4096 21 against 15.4, 256 of them, K = 2048 17.4 against 20.
    // The waves' 64 x 64 tiles take a CU each: beyond 256 of them a second round begins.  700 x 1500 x 300 8.5 us in tiles against 11
    // (both C), 2700 x 400 x 713 9.1 against 12.8, 1024 x 1536 x 2048 15.4 against 16.8 (bf16), 18.5 in both (fp32).
    // (and a launch of the waves, whose tiles are smaller, does not hold 2^29 columns)
    const int64_t waves = ((g.M + 63) / 64) * ((g.N + 63) / 64) * g.batch;
    const bool tiles = mid >= 200 ? g.M > 32 || blocks <= 8 || mid > (1 << 20)
                                  : g.M > 64 && (mid >= (WIDE ? 176 : 140) || (mid >= 100 && blocks <= (WIDE ? 8 : 32)) ||
                                                 (waves > 256 && blocks <= (WIDE ? 8 : 16)));
    // Tiles of 128 x 96, a quarter less work in a round of 256, where there are no more rounds of them: 1999 x 2999 x 5003 (384 or 512
    // tiles) 92 and 78 us, 2176 x 2048 x 500 (272, 374) 13.6 and 11.6; with 256 and 352 tiles (K = 4096) 47 and 55.
    if constexpr (WIDE) {
        const int64_t narrow = ((g.M + 127) / 128) * ((g.N + 95) / 96) * g.batch;
        if (tiles && g.b_block_rows == 1 && 4 * ((narrow + 255) / 256) < 5 * ((mid + 255) / 256))
            return launch_tile<4, 3, 2, 2, 2, A5, CT>(g, stream);
    }
    // One workgroup to a CU, so that its stages can be four: 1024 x 4096 x 4096 27.7 -> 24 us.  (Of two to a CU one hides the other's
    // loads: 2048 x 4096 x 4096 41.5 us with two stages each, 47 with four.)
    if (tiles && mid <= 256) return launch_tile<4, 4, 2, 2, 4, A5, CT>(g, stream);
    if (tiles) return launch_tile<4, 4, 2, 2, 2, A5, CT>(g, stream);
    if (g.M <= 16) return waves_by_columns<1, A5, CT>(g, stream);
    if (g.M <= 32) return waves_by_columns<2, A5, CT>(g, stream);
    return waves_by_columns<4, A5, CT>(g, stream);
}

}  // namespace perf

extern "C" perf_status perf_gemm_fp8(const void *A, const float *scaleA, const void *B, const float *scaleB, void *C, int64_t M,
                                     int64_t N, int64_t K, int64_t lda, int64_t ldsa, int64_t ldb, int64_t ldsb, int64_t ldc,
                                     int64_t b_block_rows, int64_t batch, int64_t strideA, int64_t strideSA, int64_t strideB,
                                     int64_t strideSB, int64_t strideC, float alpha, perf_dtype a_dt, perf_dtype b_dt,
                                     perf_dtype c_dt, perf_stream stream)
{
    using namespace perf;
    if (!A || !scaleA || !B || !scaleB || !C) return PERF_ERR_NULL;
    if (M < 1 || N < 1 || K < 1 || batch < 1 || M > kMaxExtent8 || N > kMaxExtent8 || K > kMaxExtent8) return PERF_ERR_SHAPE;
    const int64_t blocks = (K + kBlock8 - 1) / kBlock8;
    if (lda < K || ldb < K || ldsa < blocks || ldsb < blocks || ldc < N) return PERF_ERR_SHAPE;
    if (b_block_rows != 1 && b_block_rows != kBlock8) return PERF_ERR_SHAPE;
    if (strideA < 0 || strideSA < 0 || strideB < 0 || strideSB < 0 || strideC < 0) return PERF_ERR_SHAPE;
    if (!addressable(M, lda) || !addressable(N, ldb) || !addressable(M, ldsa) || !addressable(N, ldsb) || !addressable(M, ldc))
        return PERF_ERR_SHAPE;
    if (batch > 1 && (!addressable(batch, strideA) || !addressable(batch, strideSA) || !addressable(batch, strideB) ||
                      !addressable(batch, strideSB) || !addressable(batch, strideC) || strideC < (M - 1) * ldc + N))
        return PERF_ERR_SHAPE;
    if (!std::isfinite(alpha)) return PERF_ERR_SHAPE;
    if (!dtype8_ok(a_dt) || !dtype8_ok(b_dt) || !dtype_ok(c_dt)) return PERF_ERR_DTYPE;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(scaleA, 4) || !aligned(scaleB, 4) || !aligned(C, dtype_size(c_dt)))
        return PERF_ERR_ALIGN;
    if (b_dt != PERF_E4M3 || lda % 16 || ldb % 16 || lda >= (1 << 23) || ldb >= (1 << 23) || ldsa >= (1 << 23) || ldsb >= (1 << 23))
        return PERF_ERR_UNSUPPORTED;
    if (batch > 1 && (strideA % 16 || strideB % 16)) return PERF_ERR_UNSUPPORTED;
    const Gemm8Args g{(const uint8_t *)A, (const uint8_t *)B, scaleA, scaleB, C, (int)M, (int)N, (int)K, lda, ldsa, ldb, ldsb, ldc,
                      strideA, strideSA, strideB, strideSB, strideC, batch, (int)b_block_rows, alpha};
    const hipStream_t st = (hipStream_t)stream;
    const bool a5 = a_dt == PERF_E5M2;
    if (c_dt == PERF_BF16) return a5 ? gemm8<true, uint16_t>(g, st) : gemm8<false, uint16_t>(g, st);
    return a5 ? gemm8<true, float>(g, st) : gemm8<false, float>(g, st);
}
