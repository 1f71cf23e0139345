// Quantisation to 8-bit floating point with one fp32 scale for each block of 128: the operands of perf_gemm_fp8.
//     s = max(amax / F, 2^-126),  q = round(x * (1 / s)),   F = 448 (e4m3) or 57344 (e5m2),
// over blocks of 1 x 128 of the matrix as it is read (row orientation), of its transpose (transposed orientation), or
// 128 x 128 tiles, which are the same in both.  Bound by HBM: each element is read once, whatever orientations are written.
//
//  * quantize_rows_kernel (row orientation, 1 x 128): eight lanes own a block, 16 elements each, so that every lane
//    writes 16 bytes; the largest magnitude passes through three DPP steps.
//  * quantize_tile_kernel (everything else): a workgroup of four waves owns a tile of 128 x 128 in its registers; a lane
//    holds 8 rows x 8 columns, so that the eight rows of a column are two registers of the transposed tile, which passes
//    through LDS and leaves in runs of 128 bytes.
// The maxima of a tile's rows and columns meet in LDS, where each thread makes one scale: done by every lane that needs it, the
// divisions would be five operations per element.  Tiles that an XCD has at a time form a patch, so that the scales of
// neighbouring tiles, four bytes each in a line, meet in its L2.
// x * (1 / s) instead of x / s: a division per element is ten instructions more, which with two orientations would be
// as long as the memory time; the product differs from the quotient by one rounding of fp32 (2^-24), the values by more
// only where that falls on a tie.
// Measured: 8192 x 4096 bf16, rows 18.8 us (5.4 TB/s), both orientations 29 us (4.7 TB/s); 2999 x 5003 fp32 in tiles, both, 20.5 us
// (4.4 TB/s: one round of workgroups, whose loads and stores do not overlap).
#include "fp8.h"
#include "host_utils.h"
#include "mfma_tile.h"

namespace perf {

template <typename T> struct Sixteen {
    Eight<T> h[2];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        h[0].load(p, n);
        h[1].load(p + 8, n - 8);
    }
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

// Takes the words' values where it stands: a chain of maxima is not joined into trees, which would hold all their operands
__device__ __forceinline__ void pin(uint4_t &w)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t one = w[e];
        asm volatile("" : "+v"(one));
        w[e] = one;
    }
}

// Magnitudes of a lane's eight elements, for maxima: those of bf16 stay packed, two to a register
template <typename T> struct Eight8;
template <> struct Eight8<uint16_t> {
    typedef uint16_t Words __attribute__((ext_vector_type(8)));
    Words m;
    __device__ __forceinline__ explicit Eight8(const Eight<uint16_t> &x) : m(__builtin_bit_cast(Words, x.raw & 0x7fff7fffu)) {}
    __device__ __forceinline__ void take(const Eight8 &o)
    {
        uint4_t w = __builtin_bit_cast(uint4_t, __builtin_elementwise_max(m, o.m));
        pin(w);
        m = __builtin_bit_cast(Words, w);
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        typedef uint16_t Pair __attribute__((ext_vector_type(2)));
        const uint4_t w = __builtin_bit_cast(uint4_t, m);
        Pair p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t one = w[e];
            p[e] = __builtin_bit_cast(Pair, one);
        }
        const Pair a = __builtin_elementwise_max(__builtin_elementwise_max(p[0], p[1]), __builtin_elementwise_max(p[2], p[3]));
        return (uint32_t)max(a[0], a[1]) << 16;
    }
    __device__ __forceinline__ uint32_t at(int e) const { return (uint32_t)m[e] << 16; }
};
template <> struct Eight8<float> {
    uint4_t lo, hi;
    __device__ __forceinline__ explicit Eight8(const Eight<float> &x) : lo(x.lo & 0x7fffffffu), hi(x.hi & 0x7fffffffu) {}
    __device__ __forceinline__ void take(const Eight8 &o)
    {
        lo = __builtin_elementwise_max(lo, o.lo);
        hi = __builtin_elementwise_max(hi, o.hi);
        pin(lo), pin(hi);
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        const uint4_t a = __builtin_elementwise_max(lo, hi);
        return max(max(a[0], a[1]), max(a[2], a[3]));
    }
    __device__ __forceinline__ uint32_t at(int e) const { return e < 4 ? lo[e & 3] : hi[e & 3]; }
};

// Largest over the four lanes with the same low four bits of their number
__device__ __forceinline__ uint32_t column_max_u32(uint32_t v)
{
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const uint32_t p0 = p[0], p1 = p[1];
    v = max(p0, p1);
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return max(r0, r1);
}

// Lane `part` of sixteen holds the columns 8 part .. 8 part + 7 (bf16) or, so that a load of sixteen lanes is one run of memory
// there too, 4 part .. 4 part + 3 and those plus 64 (fp32), of the rows 8 * (thread / 16) and the seven after it.  Rows and
// columns behind the last one read the last one again, which changes no maximum, and are not written.
template <typename T, bool E5M2, bool TILE, bool ROW, bool TRANSPOSED>
__global__ __launch_bounds__(256) void quantize_tile_kernel(const T *__restrict__ x, uint8_t *__restrict__ q,
                                                            float *__restrict__ scales, uint8_t *__restrict__ qt,
                                                            float *__restrict__ scales_t, int rows, int cols, int64_t ldx,
                                                            int64_t ldq, int64_t lds, int64_t ldqt, int64_t ldst, int tiles_r,
                                                            int tiles_c)
{
    constexpr int kRuns = sizeof(T) / 2, kRun = 8 / kRuns, kFar = 128 / kRuns;  // a lane's runs of columns, kFar apart
    __shared__ uint32_t amax[TILE ? 4 : 5 * 128];  // of the rows, then of the columns by wave
    __shared__ float inv[TILE ? 1 : 2 * 128];      // of the rows, then of the columns
    __shared__ uint64_t turned[TRANSPOSED ? 128 * 16 : 1];
    const int tid = threadIdx.x, wave = tid >> 6;
    int tile_r, tile_c;
    tile_of_block(blockIdx.x, tiles_r, tiles_c, tile_r, tile_c);
    tile_r = __builtin_amdgcn_readfirstlane(tile_r), tile_c = __builtin_amdgcn_readfirstlane(tile_c);
    const int r0 = tile_r * 128, c0 = tile_c * 128;
    const int part = tid & 15, team = tid >> 4;
    const int row = r0 + 8 * team, col = c0 + kRun * part;
    const bool whole_cols = c0 + 128 <= cols, whole_rows = r0 + 128 <= rows;

    Eight<T> raw[8];
    const T *base = x + (int64_t)r0 * ldx + c0;
    if (whole_cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i].load_runs(base + (int64_t)(min(row + i, rows - 1) - r0) * ldx + kRun * part, kFar);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            raw[i].load_runs(base + (int64_t)(min(row + i, rows - 1) - r0) * ldx, kRun * part, kFar, cols - 1 - c0);
            if (i % 2) __builtin_amdgcn_sched_barrier(0);  // (fewer registers)
        }
    }
    Eight8<T> cmax(raw[0]);
    uint32_t rmax[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const Eight8<T> m(raw[i]);
        if (i) cmax.take(m);
        rmax[i] = m.largest();
        __builtin_amdgcn_sched_barrier(0);  // (fewer registers)
    }
    float inv_row[8], inv_col[8];
    if constexpr (TILE) {
        const uint32_t mine = column_max_u32(group_max_u32<16>(cmax.largest()));
        if ((tid & 63) == 0) amax[wave] = mine;
        __syncthreads();
        const float s = Fp8<E5M2>::scale(max(max(amax[0], amax[1]), max(amax[2], amax[3]))), r = 1.0f / s;
#pragma unroll
        for (int e = 0; e < 8; ++e) inv_row[e] = inv_col[e] = r;
        if (tid == 0) {
            if constexpr (ROW) scales[(int64_t)tile_r * lds + tile_c] = s;
            if constexpr (TRANSPOSED) scales_t[(int64_t)tile_c * ldst + tile_r] = s;
        }
    } else {
        // the maxima meet in LDS, where each thread makes the scale of one row or column
        if constexpr (ROW) {
#pragma unroll
            for (int i = 0; i < 8; ++i) rmax[i] = group_max_u32<16>(rmax[i]);
            if (part == 0) {
                *reinterpret_cast<uint4_t *>(&amax[8 * team]) = uint4_t{rmax[0], rmax[1], rmax[2], rmax[3]};
                *reinterpret_cast<uint4_t *>(&amax[8 * team + 4]) = uint4_t{rmax[4], rmax[5], rmax[6], rmax[7]};
            }
        }
        uint32_t c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = column_max_u32(cmax.at(e));
        if ((tid & 63) < 16) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
                *reinterpret_cast<uint4_t *>(&amax[128 * (1 + wave) + (kRuns == 2 ? 64 * r + 4 * part : 8 * part + 4 * r)]) =
                    uint4_t{c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]};
        }
        __syncthreads();
        const int line = tid & 127;
        if (tid < 128) {
            if constexpr (ROW) {
                const float s = Fp8<E5M2>::scale(amax[line]);
                inv[line] = 1.0f / s;
                if (r0 + line < rows) scales[(int64_t)(r0 + line) * lds + tile_c] = s;
            }
        } else {
            const float s = Fp8<E5M2>::scale(max(max(amax[128 + line], amax[256 + line]), max(amax[384 + line], amax[512 + line])));
            inv[128 + line] = 1.0f / s;
            if (c0 + line < cols) scales_t[(int64_t)(c0 + line) * ldst + tile_r] = s;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if constexpr (ROW) Elem<float>::unpack(*reinterpret_cast<const uint4_t *>(&inv[8 * team + 4 * r]), inv_row + 4 * r);
            Elem<float>::unpack(*reinterpret_cast<const uint4_t *>(&inv[128 + (kRuns == 2 ? 64 * r + 4 * part : 8 * part + 4 * r)]),
                                inv_col + 4 * r);
        }
    }
    if constexpr (ROW) {
        uint8_t *base = q + (int64_t)r0 * ldq + c0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            raw[i].renew();  // (what was unpacked is not kept from one use to the next)
            float v[8];
            raw[i].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= inv_row[i];
            const uint32_t w[2] = {Fp8<E5M2>::pack(v[0], v[1], v[2], v[3]), Fp8<E5M2>::pack(v[4], v[5], v[6], v[7])};
            uint8_t *p = base + (int64_t)(row + i - r0) * ldq + kRun * part;
            if (whole_rows || row + i < rows) {
                if (whole_cols) {
                    if constexpr (kRuns == 1) {
                        *reinterpret_cast<uint2_at1 *>(p) = uint2_t{w[0], w[1]};
                    } else {
                        *reinterpret_cast<uint32_at1 *>(p) = w[0];
                        *reinterpret_cast<uint32_at1 *>(p + kFar) = w[1];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((e / kRun) * kFar + e % kRun < cols - col) p[(e / kRun) * kFar + e % kRun] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        }
    }
    if constexpr (TRANSPOSED) {
        // The transposed tile: a line of 128 bytes for each column of x, in 16 pieces of 8 rows.  Lane `part` permutes the pieces
        // of its lines by `part` and swaps neighbouring lines where it is odd: the sixteen lanes of a row of x, whose lines are
        // a multiple of 512 bytes apart, then write to different banks.
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i].renew();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int line = (e / kRun) * (kFar) + kRun * part + e % kRun;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = raw[i].one(e) * inv_col[e];
            turned[(line ^ (part & 1)) * 16 + (team ^ part)] =
                (uint64_t)Fp8<E5M2>::pack(v[4], v[5], v[6], v[7]) << 32 | Fp8<E5M2>::pack(v[0], v[1], v[2], v[3]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int line = 32 * i + (tid >> 3), piece = tid & 7, by = line / kRun & 15;  // the lane that wrote the line
            const uint4_t t = *reinterpret_cast<const uint4_t *>(&turned[(line ^ (by & 1)) * 16 + ((2 * piece ^ by) & ~1)]);
            const uint32_t w[4] = {by & 1 ? t[2] : t[0], by & 1 ? t[3] : t[1], by & 1 ? t[0] : t[2], by & 1 ? t[1] : t[3]};
            uint8_t *p = qt + (int64_t)(c0 + line) * ldqt + r0 + 16 * piece;
            if (whole_cols || c0 + line < cols) {
                if (whole_rows)
                    *reinterpret_cast<uint4_at1 *>(p) = uint4_t{w[0], w[1], w[2], w[3]};
                else
                    store_bytes<16>(p, w, rows - r0 - 16 * piece);
            }
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
    // rows of a launch, which is less than 2^32 threads: a workgroup quantises 32 blocks
    const int64_t most = max_blocks(256) * 32 / blocks;
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
        const int nr = (int)n, nc = (int)tiles_c;
        const int rows = (int)std::min<int64_t>(n * 128, a.rows - r), cols = (int)a.cols;
        if (a.q && a.qt)
            quantize_tile_kernel<T, E5M2, TILE, true, true><<<grid, 256, 0, a.stream>>>(
                x, a.q + r * a.ldq, a.scales + ro * a.lds, a.qt + r, a.scales_t + t, rows, cols, a.ldx, a.ldq, a.lds, a.ldqt, a.ldst,
                nr, nc);
        else if constexpr (TILE) {
            if (a.q)
                quantize_tile_kernel<T, E5M2, true, true, false><<<grid, 256, 0, a.stream>>>(
                    x, a.q + r * a.ldq, a.scales + ro * a.lds, nullptr, nullptr, rows, cols, a.ldx, a.ldq, a.lds, 0, 0, nr, nc);
        }
        if (!a.q)
            quantize_tile_kernel<T, E5M2, TILE, false, true><<<grid, 256, 0, a.stream>>>(
                x, nullptr, nullptr, a.qt + r, a.scales_t + t, rows, cols, a.ldx, 0, 0, a.ldqt, a.ldst, nr, nc);
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
    if (!addressable(rows, ldx) || (q && (!addressable(rows, ldq) || !addressable(rows, lds))) ||
        (qt && (!addressable(cols, ldqt) || !addressable(cols, ldst))))
        return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype8_ok(q_dt)) return PERF_ERR_DTYPE;
    if (!aligned(x, dtype_size(x_dt)) || !aligned(scales, 4) || !aligned(scales_t, 4)) return PERF_ERR_ALIGN;
    const QuantizeArgs a{x, (uint8_t *)q, (uint8_t *)qt, scales, scales_t, rows, cols, ldx, ldq, lds, ldqt, ldst, (hipStream_t)stream};
    const bool tile = block_rows == kBlock8, e5 = q_dt == PERF_E5M2;
    if (x_dt == PERF_BF16) return e5 ? quantize<uint16_t, true>(a, tile) : quantize<uint16_t, false>(a, tile);
    return e5 ? quantize<float, true>(a, tile) : quantize<float, false>(a, tile);
}
