// Quantisation to 8-bit floating point with one fp32 scale for each block of 128: the operands of perf_gemm_fp8.
//     s = max(amax / F, 2^-126),  q = round(x * (1 / s)),   F = 448 (e4m3) or 57344 (e5m2),
// over blocks of 1 x 128 of the matrix as it is read (row orientation), of its transpose (transposed orientation), or
// 128 x 128 tiles, which are the same in both.  Bound by HBM: each element is read once, whatever orientations are written.
//
//  * quantize_rows_kernel (row orientation, 1 x 128): eight lanes own a block, 16 elements each, so that every lane
//    writes 16 bytes; the largest magnitude passes through three DPP steps.
//  * quantize_tile_kernel (everything else): a workgroup of four waves owns a tile of 128 x 128 in its registers; a lane
//    holds 4 rows x 16 columns, so that the four rows of a column are one register of the transposed tile.  Column maxima
//    cross the lanes by DPP and permlane swaps and the waves through LDS; the transposed tile passes through LDS and
//    leaves in runs of 128 bytes.
// x * (1 / s) instead of x / s: a division per element is ten instructions more, which with two orientations would be
// as long as the memory time; the product differs from the quotient by one rounding of fp32 (2^-24), the values by more
// only where that falls on a tie.
#include "fp8.h"
#include "host_utils.h"

namespace perf {

template <typename T> struct Sixteen {
    Eight<T> h[2];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        h[0].load(p, n);
        h[1].load(p + 8, n - 8);
    }
    __device__ __forceinline__ void clear() { h[0].clear(), h[1].clear(); }
    __device__ __forceinline__ void get(float (&v)[16]) const
    {
        float a[8], b[8];
        h[0].get(a), h[1].get(b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = a[e], v[8 + e] = b[e];
    }
};

template <typename T, bool E5M2>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, uint8_t *__restrict__ q,
                                                            float *__restrict__ scales, int64_t items, int cols, int64_t ldx,
                                                            int64_t ldq, int64_t lds, int blocks, uint32_t blocks_magic)
{
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (item >= items) return;  // whole groups of eight lanes
    const int id = (int)(item >> 3), part = threadIdx.x & 7;
    const int row = div_by(id, blocks, blocks_magic), block = id - row * blocks;
    const int col = block * kBlock8 + part * 16;
    Sixteen<T> raw;
    raw.load(x + (int64_t)row * ldx + col, cols - col);
    float v[16];
    raw.get(v);
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) amax = max(amax, magnitude(v[e]));
    amax = group_max_u32<8>(amax);
    const float s = Fp8<E5M2>::scale(amax), inv = 1.0f / s;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        w[k] = Fp8<E5M2>::pack(v[4 * k] * inv, v[4 * k + 1] * inv, v[4 * k + 2] * inv, v[4 * k + 3] * inv);
    store_bytes<16>(q + (int64_t)row * ldq + col, w, cols - col);
    if (part == 0) scales[(int64_t)row * lds + block] = s;
}

// Largest over the lanes whose number differs in bits 3, 4 and 5 only (lanes of the same column group).
__device__ __forceinline__ uint32_t column_max_u32(uint32_t v)
{
    v = dpp_max_u32<0x128>(v);  // row_ror:8
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const uint32_t p0 = p[0], p1 = p[1];
    v = max(p0, p1);
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return max(r0, r1);
}

template <typename T, bool E5M2, bool TILE, bool ROW, bool TRANSPOSED>
__global__ __launch_bounds__(256) void quantize_tile_kernel(const T *__restrict__ x, uint8_t *__restrict__ q,
                                                            float *__restrict__ scales, uint8_t *__restrict__ qt,
                                                            float *__restrict__ scales_t, int rows, int cols, int64_t ldx,
                                                            int64_t ldq, int64_t lds, int64_t ldqt, int64_t ldst, int tiles_c)
{
    __shared__ uint32_t col_amax[TILE ? 4 : 4 * 128];
    __shared__ uint32_t turned[TRANSPOSED ? 128 * 32 : 1];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c;
    const int r0 = tile_r * 128, c0 = tile_c * 128;
    const int part = tid & 7, quad = tid >> 3;
    const int row = r0 + 4 * quad, col = c0 + 16 * part;

    Sixteen<T> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row + i < rows)
            raw[i].load(x + (int64_t)(row + i) * ldx + col, cols - col);
        else
            raw[i].clear();
    }
    uint32_t row_amax[4] = {0, 0, 0, 0}, cmax[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) cmax[e] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[16];
        raw[i].get(v);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t m = magnitude(v[e]);
            if constexpr (ROW || TILE) row_amax[i] = max(row_amax[i], m);
            if constexpr (TRANSPOSED && !TILE) cmax[e] = max(cmax[e], m);
        }
    }
    float inv_row[4], inv_col[16];
    if constexpr (TILE) {
        uint32_t m = max(max(row_amax[0], row_amax[1]), max(row_amax[2], row_amax[3]));
        m = column_max_u32(group_max_u32<8>(m));
        if ((tid & 63) == 0) col_amax[wave] = m;
        __syncthreads();
        m = max(max(col_amax[0], col_amax[1]), max(col_amax[2], col_amax[3]));
        const float s = Fp8<E5M2>::scale(m), inv = 1.0f / s;
#pragma unroll
        for (int i = 0; i < 4; ++i) inv_row[i] = inv;
#pragma unroll
        for (int e = 0; e < 16; ++e) inv_col[e] = inv;
        if (tid == 0) {
            if constexpr (ROW) scales[(int64_t)tile_r * lds + tile_c] = s;
            if constexpr (TRANSPOSED) scales_t[(int64_t)tile_c * ldst + tile_r] = s;
        }
    } else {
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int e = 0; e < 16; ++e) cmax[e] = column_max_u32(cmax[e]);
            if ((tid & 63) < 8) {
#pragma unroll
                for (int e = 0; e < 16; ++e) col_amax[wave * 128 + 16 * part + e] = cmax[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = 16 * part + e;
                const uint32_t m = max(max(col_amax[c], col_amax[128 + c]), max(col_amax[256 + c], col_amax[384 + c]));
                const float s = Fp8<E5M2>::scale(m);
                inv_col[e] = 1.0f / s;
                if (quad == 0 && col + e < cols) scales_t[(int64_t)(col + e) * ldst + tile_r] = s;
            }
        }
        if constexpr (ROW) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float s = Fp8<E5M2>::scale(group_max_u32<8>(row_amax[i]));
                inv_row[i] = 1.0f / s;
                if (part == 0 && row + i < rows) scales[(int64_t)(row + i) * lds + tile_c] = s;
            }
        }
    }
    if constexpr (ROW) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[16];
            raw[i].get(v);
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = Fp8<E5M2>::pack(v[4 * k] * inv_row[i], v[4 * k + 1] * inv_row[i], v[4 * k + 2] * inv_row[i],
                                       v[4 * k + 3] * inv_row[i]);
            if (row + i < rows) store_bytes<16>(q + (int64_t)(row + i) * ldq + col, w, cols - col);
        }
    }
    if constexpr (TRANSPOSED) {
        float v[4][16];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i].get(v[i]);
        // The transposed tile: 128 rows (columns of x) of 32 words; word `quad` of a row lies at chunk (quad / 4) ^ part,
        // so that the eight lanes of a row of x, 16 columns apart, do not meet in one bank.
#pragma unroll
        for (int e = 0; e < 16; ++e)
            turned[(16 * part + e) * 32 + ((((quad >> 2) ^ part) << 2) | (quad & 3))] =
                Fp8<E5M2>::pack(v[0][e] * inv_col[e], v[1][e] * inv_col[e], v[2][e] * inv_col[e], v[3][e] * inv_col[e]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 32 * i + (tid >> 3), chunk = tid & 7;
            const uint4_t t = *reinterpret_cast<const uint4_t *>(&turned[c * 32 + ((chunk ^ (c >> 4)) << 2)]);
            const uint32_t w[4] = {t[0], t[1], t[2], t[3]};
            if (c0 + c < cols) store_bytes<16>(qt + (int64_t)(c0 + c) * ldqt + r0 + 16 * chunk, w, rows - r0 - 16 * chunk);
        }
    }
}

struct QuantizeArgs {
    const void *x;
    uint8_t *q, *qt;
    float *scales, *scales_t;
    int64_t rows, cols, ldx, ldq, lds, ldqt, ldst;
    hipStream_t stream;
};

template <typename T, bool E5M2>
static perf_status launch_rows(const QuantizeArgs &a)
{
    const int64_t blocks = (a.cols + kBlock8 - 1) / kBlock8;
    // a launch covers fewer than 2^31 blocks, and no more than 2^32 threads
    const int64_t most = (int64_t)((1ll << 29) - 1) / blocks;
    for (int64_t r = 0; r < a.rows; r += most) {
        const int64_t rows = std::min(most, a.rows - r), items = rows * blocks * 8;
        quantize_rows_kernel<T, E5M2><<<(unsigned)((items + 255) / 256), 256, 0, a.stream>>>(
            (const T *)a.x + r * a.ldx, a.q + r * a.ldq, a.scales + r * a.lds, items, (int)a.cols, a.ldx, a.ldq, a.lds, (int)blocks,
            div_magic(blocks));
        const perf_status st = launch_status();
        if (st != PERF_OK) return st;
    }
    return PERF_OK;
}

template <typename T, bool E5M2, bool TILE>
static perf_status launch_tiles(const QuantizeArgs &a)
{
    const int64_t tiles_r = (a.rows + 127) / 128, tiles_c = (a.cols + 127) / 128;
    const int64_t most = std::max<int64_t>(1, max_blocks(256) / tiles_c);  // rows of tiles of a launch
    for (int64_t t = 0; t < tiles_r; t += most) {
        const int64_t n = std::min(most, tiles_r - t), r = t * 128;
        const T *x = (const T *)a.x + r * a.ldx;
        const int64_t ro = TILE ? t : r;
        const dim3 grid((unsigned)(n * tiles_c));
        const int rows = (int)std::min<int64_t>(n * 128, a.rows - r), cols = (int)a.cols;
        if (a.q && a.qt)
            quantize_tile_kernel<T, E5M2, TILE, true, true><<<grid, 256, 0, a.stream>>>(
                x, a.q + r * a.ldq, a.scales + ro * a.lds, a.qt + r, a.scales_t + t, rows, cols, a.ldx, a.ldq, a.lds, a.ldqt, a.ldst,
                (int)tiles_c);
        else if (a.q)
            quantize_tile_kernel<T, E5M2, TILE, true, false><<<grid, 256, 0, a.stream>>>(
                x, a.q + r * a.ldq, a.scales + ro * a.lds, nullptr, nullptr, rows, cols, a.ldx, a.ldq, a.lds, 0, 0, (int)tiles_c);
        else
            quantize_tile_kernel<T, E5M2, TILE, false, true><<<grid, 256, 0, a.stream>>>(
                x, nullptr, nullptr, a.qt + r, a.scales_t + t, rows, cols, a.ldx, 0, 0, a.ldqt, a.ldst, (int)tiles_c);
        const perf_status st = launch_status();
        if (st != PERF_OK) return st;
    }
    return PERF_OK;
}

template <typename T, bool E5M2>
static perf_status quantize(const QuantizeArgs &a, bool tile)
{
    if (tile) return launch_tiles<T, E5M2, true>(a);
    if (a.qt) return launch_tiles<T, E5M2, false>(a);
    return launch_rows<T, E5M2>(a);
}

}  // namespace perf

extern "C" perf_status perf_quantize_fp8(const void *x, void *q, float *scales, void *qt, float *scales_t, int64_t rows, int64_t cols,
                                         int64_t ldx, int64_t ldq, int64_t lds, int64_t ldqt, int64_t ldst, int64_t block_rows,
                                         perf_dtype x_dt, perf_dtype q_dt, perf_stream stream)
{
    using namespace perf;
    if (!x || (!q && !qt) || !q != !scales || !qt != !scales_t) return PERF_ERR_NULL;
    if (rows < 1 || cols < 1 || rows > kMaxExtent8 || cols > kMaxExtent8 || ldx < cols) return PERF_ERR_SHAPE;
    if (block_rows != 1 && block_rows != kBlock8) return PERF_ERR_SHAPE;
    const int64_t row_blocks = (rows + kBlock8 - 1) / kBlock8, col_blocks = (cols + kBlock8 - 1) / kBlock8;
    if (q && (ldq < cols || lds < col_blocks)) return PERF_ERR_SHAPE;
    if (qt && (ldqt < rows || ldst < row_blocks)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype8_ok(q_dt)) return PERF_ERR_DTYPE;
    if (!aligned(x, dtype_size(x_dt)) || !aligned(scales, 4) || !aligned(scales_t, 4)) return PERF_ERR_ALIGN;
    const QuantizeArgs a{x, (uint8_t *)q, (uint8_t *)qt, scales, scales_t, rows, cols, ldx, ldq, lds, ldqt, ldst, (hipStream_t)stream};
    const bool tile = block_rows == kBlock8, e5 = q_dt == PERF_E5M2;
    if (x_dt == PERF_BF16) return e5 ? quantize<uint16_t, true>(a, tile) : quantize<uint16_t, false>(a, tile);
    return e5 ? quantize<float, true>(a, tile) : quantize<float, false>(a, tile);
}
