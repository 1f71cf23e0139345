// Attention of new tokens' queries over a paged cache in 8 bits (perf_cache_attention_fp8).  For query i of sequence s, at
// position p = lengths[s] + i, and head h, over the keys j <= p (with a window: j > p - window) whose page the table has:
//     S_j = scale * q . k_j,   m = max S_j,   l = sum exp(S_j - m),   o = sum exp(S_j - m) v_j / l,   lse = m + log l.
// A query without keys gets o = 0 and lse = -inf.
#include "cache.h"
#include "fp8.h"
#include "mfma_tile.h"

namespace perf {

struct AttentionArgs {
    PageTable t;
    const void *q;
    const uint8_t *k_pages, *v_pages, *k_scales, *v_scales;
    void *o;
    float *lse;
    int64_t ldq, ldo;
    int q_heads, kv_heads, max_tokens, window;
    float scale;
    // scratch: tiles of the few rows' kernel before each sequence, and sums that workgroups leave
    int64_t *before;
    float *partial;
};

// Elements d .. d + 3 of a query and head from the sums of weights and of weighted values
template <typename T>
__device__ __forceinline__ void finish(const AttentionArgs &a, int token, int head, int d, int D, float4_t v, float top, float sum)
{
    const float r = sum == 0.f ? 0.f : 1.0f / sum;
    T *const o = reinterpret_cast<T *>(a.o) + (int64_t)token * a.ldo + (int64_t)head * D + d;
    const float w[4] = {v[0] * r, v[1] * r, v[2] * r, v[3] * r};
    store_row_chunk<true, T, 4>(o, w);
    if (a.lse && d == 0) a.lse[(int64_t)token * a.q_heads + head] = __builtin_fmaf(top, fabsf(a.scale), logf(sum));
}

// ---- what both kernels share ----------------------------------------------------------------------------------------------

typedef int int2v_t __attribute__((ext_vector_type(2)));
typedef int int4v_t __attribute__((ext_vector_type(4)));

// Four values of 8 bits times a power of two as bf16, exactly, in elements 4 h .. 4 h + 3 of an operand
__device__ __forceinline__ void widen_four(bf16x8_t &f, int h, int w, float power)
{
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true);
    f[4 * h] = lo[0], f[4 * h + 1] = lo[1], f[4 * h + 2] = hi[0], f[4 * h + 3] = hi[1];
}
__device__ __forceinline__ bf16x8_t widen_eight(int w0, int w1, float p0, float p1)
{
    bf16x8_t f;
    widen_four(f, 0, w0, p0);
    widen_four(f, 1, w1, p1);
    return f;
}

// x as the sum of N bf16, each the nearest to what the ones before leave: three hold all of an fp32
template <int N>
__device__ __forceinline__ void split_eight(const float (&x)[8], bf16x8_t (&part)[N])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float left = x[e];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            part[n][e] = (__bf16)left;
            left -= (float)part[n][e];
        }
    }
}

// All of this wave's LDS accesses are done; its loads stay in flight.
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }
__device__ __forceinline__ void fence() { asm volatile("" ::: "memory"); }

// Scores are held without their scale, queries with its sign (0: zeros); this is what turns them into powers of two.
__device__ __forceinline__ float log2_scale(const AttentionArgs &a) { return a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.44269504088896341f; }
// exp2 of a difference of scores in units of log 2; -infinity gives 0
__device__ __forceinline__ float weight(float s, float c, float top_c) { return __builtin_amdgcn_exp2f(__builtin_fmaf(s, c, -top_c)); }

// Of the two lane groups 16 apart and of those 32 apart: the largest, or the sum
__device__ __forceinline__ float across_groups_max(float v)
{
    float a, b;
    swap16(v, a, b);
    v = __builtin_fmaxf(a, b);
    swap32(v, a, b);
    return __builtin_fmaxf(a, b);
}
__device__ __forceinline__ float across_groups_sum(float v)
{
    float a, b;
    swap16(v, a, b);
    v = a + b;
    swap32(v, a, b);
    return a + b;
}

// Rows of a cache block lie in LDS as they come, D bytes each, their chunks of 16 permuted: chunk c of row r at c ^ f(r).  A load
// of K takes one chunk of 16 rows, a transposing load of V one chunk of rows 4 g .. 4 g + 3 and 16 more for two g at a time; either
// then falls on all sixteen slots of a bank line.
template <int D> __device__ __forceinline__ constexpr int turn_k(int r)
{
    return D == 64 ? (r >> 2) & 3 : D == 128 ? ((r >> 1) & 3) | ((((r >> 3) ^ (r >> 4)) & 1) << 2) : r & 15;
}
template <int D> __device__ __forceinline__ constexpr int turn_v(int r)
{
    return D == 64 ? ((r >> 2) & 1) | (((r >> 4) & 1) << 1) : D == 128 ? turn_k<128>(r) : (r & 7) | (((r >> 4) & 1) << 3);
}

__device__ __forceinline__ rsrc_t block_rsrc(const uint8_t *pages, const AttentionArgs &a, int page, int head, int D)
{
    const int64_t block = (int64_t)max(page, 0) * a.kv_heads + head;
    return make_rsrc(pages + (block << a.t.page_shift) * D, page < 0 ? 0 : (uint32_t)D << a.t.page_shift);
}

// The part of a sequence that a call computes, with its keys [begin, end); begin is on a border of 32.
struct Span {
    Sequence q;
    int begin, end;
};
__device__ __forceinline__ Span span(const AttentionArgs &a, int s)
{
    Span r;
    r.q = sequence(a.t, s);
    r.q.count = min(r.q.count, a.max_tokens);
    r.end = (int)min((int64_t)r.q.held + r.q.count, (int64_t)a.t.columns << a.t.page_shift);
    r.begin = a.window ? max(r.q.held - a.window + 1, 0) & ~31 : 0;
    return r;
}

// ---- few rows: up to 16 of (token, head of a group) ---------------------------------------------------------------------
// Decoding: bound by the bytes of the cache.  The keys of all sequences and heads, in tiles of 128, are one list that is cut into
// equal runs, a workgroup each, whatever the lengths are; a run that begins or ends inside a head's keys leaves its sums in the
// workspace, and the second kernel joins them in order.  Inside a workgroup each of four waves takes 32 keys of a tile through LDS
// of its own, loaded kStages - 1 blocks ahead; they meet where a head ends.
//
// S^T = K Q^T and o^T = V^T P^T on v_mfma_f32_16x16x32_bf16, queries in the columns: a lane has one query, keys 4 g .. 4 g + 3 of
// both halves of the 32 (g = lane / 16), whose weights are its share of the second product's operand as they are.  The rows of V
// come transposed from LDS (ds_read_b64_tr_b8: eight rows of one element) in the same order of keys.
constexpr int kFewRows = 16, kFewWaves = 4, kFewKeys = 32 * kFewWaves;

template <int D> constexpr int few_stages() { return D == 64 ? 4 : 2; }
template <int D> constexpr int few_lds() { return kFewWaves * few_stages<D>() * 64 * D; }
template <int D> constexpr int few_workers() { return D == 256 ? 256 : 512; }  // as many as are on the chip at a time
template <int D> constexpr int partial_floats() { return kFewRows * (D + 2); }

__device__ __forceinline__ bool is_few(const AttentionArgs &a, int count) { return count * (int64_t)(a.q_heads / a.kv_heads) <= kFewRows; }

// Tiles of one head of a sequence: at least one if it has queries
__device__ __forceinline__ int few_tiles(const AttentionArgs &a, const Span &r)
{
    if (r.q.count == 0 || !is_few(a, r.q.count)) return 0;
    return max((r.end - r.begin + kFewKeys - 1) / kFewKeys, 1);
}

// The run of a worker begins here, and none is empty: as many workers as tiles, if those are fewer.  The worker of a tile is the
// last whose run begins at it or before.
__device__ __forceinline__ int workers_of(int64_t total, int workers) { return (int)min(total, (int64_t)workers); }
__device__ __forceinline__ int64_t run_start(int64_t total, int worker, int workers) { return total * worker / workers; }
__device__ __forceinline__ int worker_of(int64_t total, int64_t tile, int workers) { return (int)(((tile + 1) * workers - 1) / total); }

// Tiles before each sequence, and of all of them: a thread adds up a run of sequences.  The sequence that tile `x` lies in and the
// tiles before it are found on the way; `list` receives all of them, [sequences + 1].
struct Place { int64_t total, before; int s; };
__device__ __forceinline__ Place few_place(const AttentionArgs &a, int64_t (&sums)[kFewWaves + 3], int worker, int most, int64_t *list)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.t.sequences + 255) / 256, from = min(tid * each, a.t.sequences), to = min(from + each, a.t.sequences);
    int64_t mine = 0;
    for (int s = from; s < to; ++s) mine += (int64_t)few_tiles(a, span(a, s)) * a.kv_heads;
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up((long long)upto, d);
        upto += lane >= d ? v : 0;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        upto += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    const int workers = workers_of(total, most);
    const int64_t x = worker < workers ? run_start(total, worker, workers) : total;
    int64_t before = upto - mine;
    if (list || (x >= before && x < upto))
        for (int s = from; s < to; ++s) {
            const int64_t n = (int64_t)few_tiles(a, span(a, s)) * a.kv_heads;
            if (list) list[s] = before;
            if (x >= before && x < before + n) sums[kFewWaves] = before, sums[kFewWaves + 1] = s;
            before += n;
        }
    if (list && tid == 0) list[a.t.sequences] = total;
    __syncthreads();
    return Place{total, sums[kFewWaves], (int)sums[kFewWaves + 1]};
}

template <int D, typename T>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_attention_few_kernel(const AttentionArgs a)
{
    constexpr int kStages = few_stages<D>(), kStage = 64 * D, kLoads = D / 16;  // loads of a block: K, then V
    constexpr int kQ = sizeof(T) == 4 ? 3 : 1, kP = sizeof(T) == 4 ? 3 : 2;      // bf16 parts of a query's element and of a weight
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
    const int worker = blockIdx.x, group = a.q_heads / a.kv_heads, shift = a.t.page_shift, in_page = (1 << shift) - 1;
    int64_t(&sums)[kFewWaves + 3] = *reinterpret_cast<int64_t(*)[kFewWaves + 3]>(smem);
    const Place place = few_place(a, sums, worker, gridDim.x, worker == 0 ? a.before : nullptr);
    const int workers = workers_of(place.total, gridDim.x);
    if (worker >= workers) return;
    int64_t x = run_start(place.total, worker, workers);
    const int64_t stop = run_start(place.total, worker + 1, workers);
    __syncthreads();

    char *const ring = smem + wave * kStages * kStage;
    // a lane's 16 bytes of load i: row of the block's half and chunk
    uint32_t off_k[kLoads / 2], off_v[kLoads / 2];
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) {
        const int row = (i * 64 + lane) / (D / 16), at = lane % (D / 16);
        off_k[i] = (row & 15) * D + ((at ^ turn_k<D>(row)) << 4);
        off_v[i] = (row & 15) * D + ((at ^ turn_v<D>(row)) << 4);
    }
    const int v_row = (col >> 1 & 3) + 4 * g + (col >> 3) * 16;
    const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f, c = log2_scale(a);

    int s = __builtin_amdgcn_readfirstlane(place.s);
    Span r = span(a, s);
    int tiles = few_tiles(a, r);
    int head = (int)((x - place.before) / tiles), t0 = (int)((x - place.before) - (int64_t)head * tiles);
    bool first = true;
    while (x < stop) {
        const int n = (int)min((int64_t)(tiles - t0), stop - x), rows = r.q.count * group;
        const int held = __builtin_amdgcn_readfirstlane(r.q.held), end = __builtin_amdgcn_readfirstlane(r.end);
        const int from = __builtin_amdgcn_readfirstlane(r.begin) + t0 * kFewKeys + 32 * wave;  // this wave's first key

        // this lane's query (columns without one repeat another)
        const int token = col / group, position = held + token, last = held + r.q.count - 1;
        bf16x8_t q[D / 32][kQ];
        {
            const T *row = reinterpret_cast<const T *>(a.q) + (int64_t)(r.q.first + min(token, r.q.count - 1)) * a.ldq + (int64_t)(head * group + col % group) * D;
            Eight<T> raw[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) raw[i].load_cached(row + 64 * (i >> 1) + 16 * g + 8 * (i & 1), 8);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                float v[8];
                raw[i].get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= sign;
                split_eight(v, q[i]);
            }
        }

        // Pages and scales of 64 blocks, one a lane: those of block i are in lane i % 64
        int page0 = -1, page1 = -1;
        uint32_t scales = 0;  // bytes: K and V of the first half, K and V of the second
        auto look_up = [&](int base) {
            const int i = base + lane, k = from + i * kFewKeys;
            page0 = i < n && k < end ? page_at(a.t, s, k >> shift) : -1;
            page1 = i < n && k + 16 < end ? page_at(a.t, s, (k + 16) >> shift) : -1;
            uint32_t b[4] = {0, 0, 0, 0};
            if (page0 >= 0) b[0] = a.k_scales[(int64_t)page0 * a.kv_heads + head], b[1] = a.v_scales[(int64_t)page0 * a.kv_heads + head];
            if (page1 >= 0) b[2] = a.k_scales[(int64_t)page1 * a.kv_heads + head], b[3] = a.v_scales[(int64_t)page1 * a.kv_heads + head];
            scales = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
            wait_vmem<0>();
            asm volatile("" : "+v"(page0), "+v"(page1), "+v"(scales));
        };
        struct Block { uint32_t scales; int pages; };  // pages: bit h: half h is there
        auto issue = [&](int i) {  // (blocks past the end move nothing: the number in flight stays the same)
            if ((i & 63) == 0) look_up(i);
            const int p0 = __builtin_amdgcn_readlane(page0, i & 63), p1 = __builtin_amdgcn_readlane(page1, i & 63);
            const int k = from + i * kFewKeys;
            char *const to = ring + (i % kStages) * kStage;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int p = h ? p1 : p0;
                const rsrc_t in_k = block_rsrc(a.k_pages, a, p, head, D), in_v = block_rsrc(a.v_pages, a, p, head, D);
                const uint32_t at = (uint32_t)((k + 16 * h) & in_page) * D;
#pragma unroll
                for (int j = h * kLoads / 4; j < (h + 1) * kLoads / 4; ++j) issue_load_to(in_k, off_k[j], at, to + j * 1024);
#pragma unroll
                for (int j = h * kLoads / 4; j < (h + 1) * kLoads / 4; ++j) issue_load_to(in_v, off_v[j], at, to + (kLoads / 2 + j) * 1024);
            }
            return Block{(uint32_t)__builtin_amdgcn_readlane((int)scales, i & 63), (p0 >= 0 ? 1 : 0) | (p1 >= 0 ? 2 : 0)};
        };

        float4_t o[D / 16];
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] = float4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        Block ahead[kStages];
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) ahead[i] = issue(i);
        for (int i = 0; i < n; ++i) {
            wait_lds();  // the block before this one has been read
            fence();
            ahead[kStages - 1] = issue(i + kStages - 1);
            wait_vmem<(kStages - 1) * kLoads>();
            fence();
            const Block now = ahead[0];
#pragma unroll
            for (int j = 0; j + 1 < kStages; ++j) ahead[j] = ahead[j + 1];
            const int k = from + i * kFewKeys;
            if (k >= end) continue;
            const char *const in_k = ring + (i % kStages) * kStage, *const in_v = in_k + 32 * D;

            float4_t sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float power = scale_of(now.scales >> (16 * h) & 255);
                const int row = 16 * h + col;
                sc[h] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const int4v_t w = *reinterpret_cast<const int4v_t *>(in_k + row * D + (((4 * j + g) ^ turn_k<D>(row)) << 4));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bf16x8_t f = widen_eight(w[2 * e], w[2 * e + 1], power, power);
#pragma unroll
                        for (int p = kQ - 1; p >= 0; --p) sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[2 * j + e][p], sc[h], 0, 0, 0);
                    }
                }
            }
            int keep[2] = {-1, -1};  // bytes of V that are keys
            if (now.pages != 3 || k + 31 > held || (a.window && k <= last - a.window)) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = k + 16 * h + 4 * g + e;
                        const bool there = key < end && (now.pages >> h & 1), seen = there && key <= position && (!a.window || key > position - a.window);
                        if (!there) keep[h] &= ~(255 << (8 * e));
                        sc[h][e] = seen ? sc[h][e] : -INFINITY;
                    }
            }
            float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(sc[0][0], sc[0][1]), __builtin_fmaxf(sc[0][2], sc[0][3])),
                                        __builtin_fmaxf(__builtin_fmaxf(sc[1][0], sc[1][1]), __builtin_fmaxf(sc[1][2], sc[1][3])));
            top = __builtin_fmaxf(across_groups_max(top), m);
            const float top_c = top == -INFINITY ? 0.f : top * c;
            if (__ballot(top > m)) {
                const float shrink = weight(m, c, top_c);
                l *= shrink;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) o[d] *= shrink;
                m = top;
            }
            float p[8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[4 * h + e] = weight(sc[h][e], c, top_c);
            l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            bf16x8_t w[kP];
            split_eight(p, w);
            const float power0 = scale_of(now.scales >> 8 & 255), power1 = scale_of(now.scales >> 24);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                int2v_t v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (__attribute__((address_space(3))) int2v_t *)(in_v + v_row * D + ((d ^ turn_v<D>(v_row)) << 4) + (col & 1) * 8));
                const bf16x8_t f = widen_eight(v[0] & keep[0], v[1] & keep[1], power0, power1);
#pragma unroll
                for (int e = kP - 1; e >= 0; --e) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, w[e], o[d], 0, 0, 0);
            }
        }

        // The four waves' sums meet: the ring holds them by now, rows of D + 4 apart
        constexpr int kRow = D + 4, kSums = kFewRows * kRow + 2 * kFewRows;
        static_assert(kSums * 4 <= kStages * kStage, "a wave's sums fit its ring");
        wait_vmem_and_lds<0>();
        fence();
        l = across_groups_sum(l);
        float *const mine = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<float4_t *>(mine + col * kRow + 16 * d + 4 * g) = o[d];
        if (lane < kFewRows) mine[kFewRows * kRow + lane] = m, mine[kFewRows * kRow + kFewRows + lane] = l;
        __syncthreads();
        const bool whole = n == tiles;
        float *const out = whole ? nullptr : a.partial + (int64_t)(2 * worker + !first) * partial_floats<D>();
        for (int i = tid; i < rows * (D / 4); i += 256) {
            const int row = i / (D / 4), d = 4 * (i % (D / 4));
            float mw[kFewWaves], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                mw[w] = reinterpret_cast<float *>(smem + w * kStages * kStage)[kFewRows * kRow + row];
                top = __builtin_fmaxf(top, mw[w]);
            }
            const float top_c = top == -INFINITY ? 0.f : top * c;
            float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float *of = reinterpret_cast<float *>(smem + w * kStages * kStage);
                const float f = weight(mw[w], c, top_c);
                v += f * *reinterpret_cast<const float4_t *>(of + row * kRow + d);
                sum += f * of[kFewRows * kRow + kFewRows + row];
            }
            if (whole) {
                finish<T>(a, r.q.first + row / group, head * group + row % group, d, D, v, top, sum);
            } else {
                *reinterpret_cast<float4_t *>(out + row * D + d) = v;
                if (d == 0) out[kFewRows * D + row] = top, out[kFewRows * (D + 1) + row] = sum;
            }
        }
        __syncthreads();
        first = false;
        x += n, t0 = 0;
        if (x < stop && ++head == a.kv_heads) {
            head = 0;
            do r = span(a, ++s), tiles = few_tiles(a, r);
            while (tiles == 0);
        }
    }
}

// Joins what several workgroups have left of one query and head: in their order, their maxima first.
template <int D, typename T>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(const AttentionArgs a, int most)
{
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes;  // lanes that share a query, and teams that share the workgroups
    __shared__ float factor[few_workers<D>()], of_wave[2][4];
    __shared__ float4_t sums[kTeams][kLanes];
    const int tid = threadIdx.x, token = blockIdx.x / a.q_heads, of_all = blockIdx.x - token * a.q_heads, group = a.q_heads / a.kv_heads;
    const int s = find_sequence(a.t.sequences, token, [&](int i) { return first_token(a.t, i); });
    const Span r = span(a, s);
    const int tiles = few_tiles(a, r);
    if (token < r.q.first || token >= r.q.first + r.q.count || tiles == 0) return;
    const int head = of_all / group, row = (token - r.q.first) * group + of_all % group;
    const int64_t total = a.before[a.t.sequences], start = a.before[s] + (int64_t)head * tiles;
    const int workers = workers_of(total, most);
    const int from = worker_of(total, start, workers), count = worker_of(total, start + tiles - 1, workers) - from + 1;
    if (count == 1) return;
    const auto partial = [&](int i) {
        return a.partial + (int64_t)(2 * (from + i) + (run_start(total, from + i, workers) < start)) * partial_floats<D>();
    };
    const float c = log2_scale(a);
    float top = -INFINITY;
    for (int i = tid; i < count; i += 256) {
        factor[i] = partial(i)[kFewRows * D + row];
        top = __builtin_fmaxf(top, factor[i]);
    }
    top = wave_allreduce(top, OpMax());
    if ((tid & 63) == 0) of_wave[0][tid >> 6] = top;
    __syncthreads();
    top = __builtin_fmaxf(__builtin_fmaxf(of_wave[0][0], of_wave[0][1]), __builtin_fmaxf(of_wave[0][2], of_wave[0][3]));
    const float top_c = top == -INFINITY ? 0.f : top * c;
    float sum = 0.f;
    for (int i = tid; i < count; i += 256) {
        factor[i] = weight(factor[i], c, top_c);
        sum += factor[i] * partial(i)[kFewRows * (D + 1) + row];
    }
    sum = wave_allreduce(sum, OpSum());
    if ((tid & 63) == 0) of_wave[1][tid >> 6] = sum;
    __syncthreads();
    sum = (of_wave[1][0] + of_wave[1][1]) + (of_wave[1][2] + of_wave[1][3]);
    const int d = tid % kLanes, team = tid / kLanes;
    float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = team; i < count; i += kTeams) v += factor[i] * *reinterpret_cast<const float4_t *>(partial(i) + row * D + 4 * d);
    sums[team][d] = v;
    __syncthreads();
    if (team == 0) {
#pragma unroll
        for (int i = 1; i < kTeams; ++i) v += sums[i][d];
        finish<T>(a, token, of_all, 4 * d, D, v, top, sum);
    }
}

// One workgroup for a query and head: keys 256 at a time, one a thread; values an element a thread.
template <int D, typename T>
__global__ __launch_bounds__(256) void cache_attention_kernel(const AttentionArgs a)
{
    __shared__ float q[D], p[256], of_wave[4], part[256];
    const int tid = threadIdx.x;
    const int token = blockIdx.x / a.q_heads, head = blockIdx.x - token * a.q_heads, kv = head / (a.q_heads / a.kv_heads);
    const int s = find_sequence(a.t.sequences, token, [&](int i) { return first_token(a.t, i); });
    Sequence seq = sequence(a.t, s);
    seq.count = min(seq.count, a.max_tokens);
    if (token < seq.first || token >= seq.first + seq.count || is_few(a, seq.count)) return;
    const int position = seq.held + token - seq.first, shift = a.t.page_shift;
    const int end = (int)min((int64_t)position + 1, (int64_t)a.t.columns << shift);
    const int begin = a.window ? max(position - a.window + 1, 0) : 0;
    if (tid < D) q[tid] = Elem<T>::load1(reinterpret_cast<const T *>(a.q) + token * a.ldq + head * D + tid) * a.scale;
    __syncthreads();
    constexpr int kParts = 256 / D;  // threads that share an element
    const int d = tid % D, mine = tid / D;
    float m = -INFINITY, l = 0.f, acc = 0.f;
    for (int from = begin; from < end; from += 256) {
        const int j = from + tid, page = j < end ? page_at(a.t, s, j >> shift) : -1;
        float v = -INFINITY;
        if (page >= 0) {
            const int64_t block = (int64_t)page * a.kv_heads + kv;
            const uint8_t *row = a.k_pages + ((block << shift) + (j & ((1 << shift) - 1))) * D;
            float sum = 0.f;
            for (int c = 0; c < D; c += 16) {
                const uint4_t w = *reinterpret_cast<const uint4_t *>(row + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float k[4];
                    unpack_e4m3(w[e], k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum = fmaf(q[c + 4 * e + i], k[i], sum);
                }
            }
            v = sum * scale_of(a.k_scales[block]);
        }
        float top = wave_allreduce(v, OpMax());
        if ((tid & 63) == 0) of_wave[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
        const float next = fmaxf(m, top), keep = next == -INFINITY ? 1.f : expf(m - next);
        p[tid] = page >= 0 ? expf(v - next) : 0.f;
        l = l * keep + p[tid];
        acc *= keep;
        m = next;
        __syncthreads();
        for (int i = mine; i < min(256, end - from); i += kParts) {
            const int at = from + i, vp = page_at(a.t, s, at >> shift);
            if (vp < 0) continue;
            const int64_t block = (int64_t)vp * a.kv_heads + kv;
            float v4[4];
            unpack_e4m3(a.v_pages[((block << shift) + (at & ((1 << shift) - 1))) * D + d], v4);
            acc = fmaf(p[i], v4[0] * scale_of(a.v_scales[block]), acc);
        }
        __syncthreads();
    }
    l = wave_allreduce(l, OpSum());
    if ((tid & 63) == 0) of_wave[tid >> 6] = l;
    part[tid] = acc;
    __syncthreads();
    l = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
    if (tid < D) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) o += part[i * D + tid];
        Elem<T>::store1(reinterpret_cast<T *>(a.o) + token * a.ldo + head * D + tid, l == 0.f ? 0.f : o / l);
    }
    if (a.lse && tid == 0) a.lse[(int64_t)token * a.q_heads + head] = m + logf(l);
}

// Scratch in bytes: tiles before each sequence, then the few rows' sums
static int64_t list_bytes(int64_t sequences) { return (8 * (sequences + 1) + 15) / 16 * 16; }
template <int D> static int64_t scratch(int64_t sequences) { return list_bytes(sequences) + 8ll * few_workers<D>() * partial_floats<D>(); }

template <int D, typename T>
static perf_status attention(const AttentionArgs &a, hipStream_t st)
{
    const int64_t group = a.q_heads / a.kv_heads, rows = (int64_t)a.t.tokens * a.q_heads;
    if (rows > max_blocks(256)) return PERF_ERR_UNSUPPORTED;
    const bool many = a.max_tokens * group > kFewRows;  // (whether a sequence of as many tokens is for the other kernel)
    if (!allow_lds<cache_attention_few_kernel<D, T>>(few_lds<D>())) return PERF_ERR_LAUNCH;
    cache_attention_few_kernel<D, T><<<few_workers<D>(), 256, few_lds<D>(), st>>>(a);
    cache_attention_join_kernel<D, T><<<(uint32_t)rows, 256, 0, st>>>(a, few_workers<D>());
    if (many) cache_attention_kernel<D, T><<<(uint32_t)rows, 256, 0, st>>>(a);
    return launch_status();
}

}  // namespace perf

using namespace perf;

static bool attention_shape_ok(const CacheShape &c, int64_t max_tokens)
{
    return cache_shape_ok(c) && c.head_dim <= kMaxExtent8 / kMaxHeads && max_tokens >= 1;
}

extern "C" int64_t perf_cache_attention_fp8_workspace_bytes(int64_t tokens, int64_t sequences, int64_t max_tokens, int64_t q_heads,
                                                            int64_t kv_heads, int64_t head_dim, int64_t page_size, int64_t table_pages)
{
    const CacheShape c{tokens, sequences, q_heads, kv_heads, head_dim, 1, page_size, table_pages, table_pages};
    if (!attention_shape_ok(c, max_tokens) || !cache_supported(c)) return -1;
    return head_dim == 64 ? scratch<64>(sequences) : head_dim == 128 ? scratch<128>(sequences) : scratch<256>(sequences);
}

extern "C" perf_status perf_cache_attention_fp8(const void *q, const void *k_pages, const void *v_pages, const uint8_t *k_scales,
                                                const uint8_t *v_scales, const int32_t *table, const int32_t *lengths, const int32_t *cu,
                                                void *o, float *lse, void *workspace, int64_t tokens, int64_t sequences,
                                                int64_t max_tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t ldq,
                                                int64_t ldo, int64_t pages, int64_t page_size, int64_t table_pages, int64_t ldt,
                                                int64_t window, float scale, perf_dtype x_dt, perf_stream stream)
{
    if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lengths || !cu || !o || !workspace) return PERF_ERR_NULL;
    const CacheShape c{tokens, sequences, q_heads, kv_heads, head_dim, pages, page_size, table_pages, ldt};
    if (!attention_shape_ok(c, max_tokens)) return PERF_ERR_SHAPE;
    if (window < 0 || window > kMaxPosition || !std::isfinite(scale)) return PERF_ERR_SHAPE;
    if (ldq < q_heads * head_dim || ldo < q_heads * head_dim || !addressable(tokens, ldq) || !addressable(tokens, ldo)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt)) return PERF_ERR_DTYPE;
    const int64_t size = dtype_size(x_dt);
    if (!aligned(q, size) || !aligned(o, size) || !aligned(lse, 4) || !aligned(workspace, 16) || !aligned(k_pages, 16) ||
        !aligned(v_pages, 16) || !aligned(table, 4) || !aligned(lengths, 4) || !aligned(cu, 4))
        return PERF_ERR_ALIGN;
    if (!cache_supported(c)) return PERF_ERR_UNSUPPORTED;
    AttentionArgs a{};
    a.t = PageTable{table, lengths, cu, ldt, (int)tokens, (int)sequences, (int)pages, (int)table_pages, __builtin_ctzll(page_size)};
    a.q = q, a.o = o, a.lse = lse, a.ldq = ldq, a.ldo = ldo;
    a.k_pages = (const uint8_t *)k_pages, a.v_pages = (const uint8_t *)v_pages, a.k_scales = k_scales, a.v_scales = v_scales;
    a.q_heads = (int)q_heads, a.kv_heads = (int)kv_heads, a.max_tokens = (int)std::min(max_tokens, tokens), a.window = (int)window, a.scale = scale;
    a.before = (int64_t *)workspace, a.partial = (float *)((char *)workspace + list_bytes(sequences));
    const hipStream_t st = (hipStream_t)stream;
    const auto with = [&](auto one) {
        using T = decltype(one);
        return head_dim == 64 ? attention<64, T>(a, st) : head_dim == 128 ? attention<128, T>(a, st) : attention<256, T>(a, st);
    };
    return x_dt == PERF_BF16 ? with(uint16_t{}) : with(float{});
}
