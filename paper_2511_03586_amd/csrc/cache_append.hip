// Keys and values appended to a paged cache in 8 bits, with the position rotation on the way (perf_cache_append_fp8):
//     x1' = x1 c - x2 s,  x2' = x2 c + x1 s   for the pairs of a rotated part, c and s from the table's row of the position;
//     b = least byte >= 1 with max |x| <= 448 * 2^(b - 127) over a page and head, and no less than it was;
//     held as e4m3(x * 2^(127 - b)).
// Every product and sum of the rotation is rounded by itself, so that scales and bytes do not depend on what the compiler
// contracts.  A scale is a power of two: what a page holds is moved to a larger one exactly but for subnormals, so that a page
// that is filled token by token does not drift, and its values are exact in bf16.
//
// One launch: teams of waves for each (page that new tokens reach, head, keys or values), whose tokens stay in registers between
// the maximum and the rounding, and waves of (token, part of a query row) behind them.  Bound by bytes for long runs (4 of about 2048
// tokens, 32 + 2 x 8 heads of 128 in bf16: 39-44 us, 187 MB at 4.3-4.8 TB/s, most of them the queries), by the launch and four
// trips to memory one behind the other for single tokens (2 of them 3.5 us, 192 of them 6.7 us): place, page, what the page holds.
#include "cache.h"
#include "fp8.h"

namespace perf {

struct AppendArgs {
    PageTable t;
    const void *q, *k, *v;
    const float *rotation;
    void *q_out;
    uint8_t *k_pages, *v_pages, *k_scales, *v_scales;
    int64_t ldq, ldk, ldv, ldq_out;
    int q_heads, kv_heads, rotary, positions, q_waves;
    bool interleaved, by_token;
    uint32_t append_blocks;
};

// Rotates eight elements of a head from element d on, a multiple of 8; `row` is the table's row of their position: cosines,
// then sines.  The partners of halves lie in a lane `rotary / 16` away, whose eight are handed over.
template <typename T>
__device__ __forceinline__ void rotate(float (&x)[8], const float *row, int d, int rotary, bool interleaved)
{
#pragma clang fp contract(off)
    const int half = rotary >> 1;
    if (interleaved) {
        if (d >= rotary) return;
        const float4_t c = *reinterpret_cast<const float4_at4 *>(row + (d >> 1)), s = *reinterpret_cast<const float4_at4 *>(row + half + (d >> 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x1 = x[2 * i], x2 = x[2 * i + 1];
            x[2 * i] = x1 * c[i] - x2 * s[i];
            x[2 * i + 1] = x2 * c[i] + x1 * s[i];
        }
        return;
    }
    // all lanes take part in the exchange; those of the part that is not rotated drop what they get
    const int lane = threadIdx.x & (kWave - 1), away = half >> 3;
    const int from = d >= rotary ? lane : d < half ? lane + away : lane - away;
    float other[8];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // (bf16 values as they came: two to a register)
            const uint32_t mine = (__builtin_bit_cast(uint32_t, x[2 * i]) >> 16) | (__builtin_bit_cast(uint32_t, x[2 * i + 1]) & 0xffff0000u);
            const uint32_t got = (uint32_t)__shfl((int)mine, from);
            other[2 * i] = bf16_lo(got), other[2 * i + 1] = bf16_hi(got);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl(x[i], from);
    }
    if (d >= rotary) return;
    const int j = d < half ? d : d - half;
    float c[8], s[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float4_t cc = *reinterpret_cast<const float4_at4 *>(row + j + 4 * h), ss = *reinterpret_cast<const float4_at4 *>(row + half + j + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[4 * h + i] = cc[i], s[4 * h + i] = ss[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = x[i] * c[i], b = other[i] * s[i];
        x[i] = d < half ? a - b : a + b;
    }
}

constexpr int kQueryChunks = 4;  // groups of eight elements that a lane takes of a query row

// A wave's share of the queries: 64 * kQueryChunks groups of eight of one token's row.
template <int D, typename T>
__device__ __forceinline__ void rotate_queries(const AppendArgs &a, int64_t wave)
{
    const int lane = threadIdx.x & (kWave - 1);
    const int token = (int)(wave / a.q_waves), part = (int)(wave - (int64_t)token * a.q_waves);
    if (token >= a.t.tokens) return;
    const int s = find_sequence(a.t.sequences, token, [&](int i) { return first_token(a.t, i); });
    const Sequence q = sequence(a.t, s);
    if (token < q.first || token >= q.first + q.count) return;
    const int position = q.held + token - q.first;
    if (a.rotary && position >= a.positions) return;
    const float *row = a.rotation + (int64_t)position * a.rotary;
    const T *in = reinterpret_cast<const T *>(a.q) + token * a.ldq;
    T *out = reinterpret_cast<T *>(a.q_out) + token * a.ldq_out;
    const int groups = a.q_heads * (D / 8), d = 8 * lane % D;
    Eight<T> x[kQueryChunks];
#pragma unroll
    for (int i = 0; i < kQueryChunks; ++i) {
        const int g = (part * kQueryChunks + i) * kWave + lane;
        x[i].load(in + 8 * min(g, groups - 1), 8);
    }
#pragma unroll
    for (int i = 0; i < kQueryChunks; ++i) {
        const int g = (part * kQueryChunks + i) * kWave + lane;
        float v[8];
        x[i].get(v);
        if (a.rotary) rotate<T>(v, row, d, a.rotary, a.interleaved);
        if (g < groups) store_eight(out + 8 * g, v, 8);
    }
}

// The tokens of one page and head, keys or values: up to kChunks groups of eight a thread stay in registers; of more, which a team
// of one wave meets where a sequence brings many tokens among many that bring one, all are read a second time.
constexpr int kChunks = 8;

template <int D, int THREADS, typename T>
struct PageTokens {
    const T *in;
    const float *rotation;  // row of the first token's position; nullptr: not rotated
    int64_t ld;
    int groups, rotary;
    bool interleaved;
    __device__ __forceinline__ void load(Eight<T> &raw, int i) const
    {
        const int g = min(i, groups - 1);
        raw.load(in + (int64_t)(g / (D / 8)) * ld + 8 * (g % (D / 8)), 8);
    }
    __device__ __forceinline__ void get(const Eight<T> &raw, int i, float (&x)[8]) const
    {
        // (groups past the end repeat the last one; their partners then are not what they should be: not counted, not stored)
        raw.get(x);
        if (rotation) rotate<T>(x, rotation + (int64_t)(min(i, groups - 1) / (D / 8)) * rotary, 8 * (i % (D / 8)), rotary, interleaved);
    }
};

__device__ __forceinline__ uint32_t largest(const float (&x)[8])
{
    uint32_t v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) v = max(v, magnitude(x[e]));
    return v;
}

template <int D>
__device__ __forceinline__ void store_group(uint8_t *to, int g, const float (&x)[8], float up)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = Fp8<false>::pack(x[4 * h] * up, x[4 * h + 1] * up, x[4 * h + 2] * up, x[4 * h + 3] * up);
    *reinterpret_cast<uint2_t *>(to + 8 * g) = uint2_t{w[0], w[1]};
}

// THREADS to a team: 64 (four teams to a workgroup), or the workgroup's 256 or 1024
template <int D, int THREADS, typename T>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void cache_append_kernel(const AppendArgs a)
{
    constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kTeams = kBlock / THREADS;
    if (blockIdx.x >= a.append_blocks) {
        rotate_queries<D, T>(a, (int64_t)(blockIdx.x - a.append_blocks) * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
        return;
    }
    const int tid = kTeams == 1 ? threadIdx.x : threadIdx.x & (THREADS - 1), page_shift = a.t.page_shift, page_size = 1 << page_shift;
    const int index = kTeams == 1 ? blockIdx.x : blockIdx.x * kTeams + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    const bool values = index & 1;
    const int u = __builtin_amdgcn_readfirstlane((index >> 1) / a.kv_heads), head = (index >> 1) - u * a.kv_heads;
    if (kTeams > 1 && a.by_token && u >= a.t.tokens) return;
    const T *const rows = reinterpret_cast<const T *>(values ? a.v : a.k) + (int64_t)head * D;
    const int64_t ld = values ? a.ldv : a.ldk;
    // A unit is a page that new tokens reach.  By token: where `u` is the first new one of its page; its first elements are on
    // their way before anything else is known.  Else sequence s has the units from cu[s] / page_size + 2 s on: a run of n tokens
    // reaches at most n / page_size + 2 pages.
    Eight<T> early;
    if (a.by_token) early.load(rows + (int64_t)min(u + tid / (D / 8), a.t.tokens - 1) * ld + 8 * (tid % (D / 8)), 8);
    const auto start = [&](int s) { return a.by_token ? first_token(a.t, s) : (first_token(a.t, s) >> page_shift) + 2 * s; };
    const int s = find_sequence(a.t.sequences, u, start);
    const Sequence q = sequence(a.t, s);
    const int column = a.by_token ? (q.held + u - q.first) >> page_shift : (q.held >> page_shift) + u - start(s);
    const int at = column << page_shift;  // position of the page's first slot
    const int last = a.rotary ? min(q.held + q.count, a.positions) : q.held + q.count;
    const int slot0 = max(q.held - at, 0), slot1 = min(last - at, page_size);  // new tokens
    if (q.count == 0 || slot0 >= slot1 || (a.by_token && u != q.first + at + slot0 - q.held)) return;
    const bool turn = a.rotary && !values;
    const PageTokens<D, THREADS, T> tokens{rows + (int64_t)(q.first + at + slot0 - q.held) * ld, turn ? a.rotation + (int64_t)(at + slot0) * a.rotary : nullptr, ld,
                                           (slot1 - slot0) * (D / 8), a.rotary, a.interleaved};
    const int groups = tokens.groups;
    Eight<T> raw[kChunks];  // (on their way before the page is known)
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
        if (i * THREADS < groups) {
            if (i == 0 && a.by_token)
                raw[0] = early;
            else
                tokens.load(raw[i], tid + i * THREADS);
        }
    const int page = page_at(a.t, s, column);
    if (page < 0) return;
    const int64_t block = (int64_t)page * a.kv_heads + head;
    uint8_t *const to = (values ? a.v_pages : a.k_pages) + (block << page_shift) * D;
    uint8_t *const scale = (values ? a.v_scales : a.k_scales) + block;
    const int before = slot0 ? *scale : 0;
    float x[kChunks][8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
        if (i * THREADS < groups) {
            tokens.get(raw[i], tid + i * THREADS, x[i]);
            amax = max(amax, tid + i * THREADS < groups ? largest(x[i]) : 0);
        }
#pragma unroll 1
    for (int i = kChunks * THREADS; i < groups; i += THREADS) {
        Eight<T> more;
        float y[8];
        tokens.load(more, tid + i);
        tokens.get(more, tid + i, y);
        amax = max(amax, tid + i < groups ? largest(y) : 0);
    }
    amax = group_max_u32<32>(amax);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
    if constexpr (kTeams == 1) {
        __shared__ uint32_t of_wave[THREADS / kWave];
        if ((tid & 63) == 0) of_wave[tid >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / kWave; ++w) amax = max(amax, of_wave[w]);
    }

    // 448 is 1.75 * 2^8
    const int need = amax >= 0x7f800000u ? kNoNumber : max((int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u), 1);
    const int b = max(before, need);
    if (tid == 0 && b != before) *scale = (uint8_t)b;
    if (b > before && slot0 && b != kNoNumber) {  // what the page holds goes over to the larger scale
        const float shrink = b - before > 126 ? 0.f : __builtin_bit_cast(float, (uint32_t)(127 - (b - before)) << 23);
#pragma unroll 1
        for (int i = tid; i < slot0 * (D / 16); i += THREADS) {
            uint4_t w = *reinterpret_cast<const uint4_t *>(to + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v[4];
                unpack_e4m3(w[e], v);
                w[e] = Fp8<false>::pack(v[0] * shrink, v[1] * shrink, v[2] * shrink, v[3] * shrink);
            }
            *reinterpret_cast<uint4_t *>(to + 16 * i) = w;
        }
    }
    const float up = __builtin_bit_cast(float, (uint32_t)max(254 - b, 1) << 23);
    uint8_t *const new_rows = to + (int64_t)slot0 * D;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
        if (tid + i * THREADS < groups) store_group<D>(new_rows, tid + i * THREADS, x[i], up);
#pragma unroll 1
    for (int i = kChunks * THREADS; i < groups; i += THREADS) {
        Eight<T> more;
        float y[8];
        tokens.load(more, tid + i);
        tokens.get(more, tid + i, y);
        if (tid + i < groups) store_group<D>(new_rows, tid + i, y, up);
    }
}

template <int D, int THREADS, typename T>
static perf_status launch_append(AppendArgs &a, int64_t units, hipStream_t st)
{
    constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kTeams = kBlock / THREADS;
    const int64_t blocks = (units * a.kv_heads * 2 + kTeams - 1) / kTeams;
    const int64_t query_blocks = ((int64_t)a.t.tokens * a.q_waves * kWave + kBlock - 1) / kBlock;
    if (blocks + query_blocks > max_blocks(kBlock)) return PERF_ERR_UNSUPPORTED;
    a.append_blocks = (uint32_t)blocks;
    cache_append_kernel<D, THREADS, T><<<(uint32_t)(blocks + query_blocks), kBlock, 0, st>>>(a);
    return launch_status();
}

// A wave to a page where a sequence brings about one token (192 sequences, 8 heads of 128: 19.4 us with a workgroup each and two
// units to a sequence); else as many threads as hold a page's tokens in registers.
template <int D, typename T>
static perf_status append(AppendArgs &a, hipStream_t st)
{
    const int64_t by_page = (a.t.tokens >> a.t.page_shift) + 2 * (int64_t)a.t.sequences;
    a.q_waves = a.q ? (int)((a.q_heads * (D / 8) + kWave * kQueryChunks - 1) / (kWave * kQueryChunks)) : 0;
    a.by_token = a.t.tokens <= by_page;
    if (a.by_token) return launch_append<D, 64, T>(a, a.t.tokens, st);
    if ((D << a.t.page_shift) > kChunks * 8 * 256) return launch_append<D, 1024, T>(a, by_page, st);
    return launch_append<D, 256, T>(a, by_page, st);
}

}  // namespace perf

extern "C" perf_status perf_cache_append_fp8(const void *q, const void *k, const void *v, const float *rotation, void *q_out,
                                             void *k_pages, void *v_pages, uint8_t *k_scales, uint8_t *v_scales,
                                             const int32_t *table, const int32_t *lengths, const int32_t *cu, int64_t tokens,
                                             int64_t sequences, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t ldq,
                                             int64_t ldk, int64_t ldv, int64_t ldq_out, int64_t pages, int64_t page_size,
                                             int64_t table_pages, int64_t ldt, int64_t rotary_dim, int64_t positions,
                                             int interleaved, perf_dtype x_dt, perf_stream stream)
{
    using namespace perf;
    if (!k || !v || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lengths || !cu) return PERF_ERR_NULL;
    if (!q != !q_out || (rotary_dim != 0 && !rotation)) return PERF_ERR_NULL;
    const CacheShape c{tokens, sequences, q_heads, kv_heads, head_dim, pages, page_size, table_pages, ldt};
    if (!cache_shape_ok(c) || head_dim > kMaxExtent8 / kMaxHeads) return PERF_ERR_SHAPE;
    if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 2 || interleaved < 0 || interleaved > 1) return PERF_ERR_SHAPE;
    if (rotary_dim && (positions < 1 || positions > kMaxPosition)) return PERF_ERR_SHAPE;
    if (ldk < kv_heads * head_dim || ldv < kv_heads * head_dim || !addressable(tokens, ldk) || !addressable(tokens, ldv)) return PERF_ERR_SHAPE;
    if (q && (ldq < q_heads * head_dim || ldq_out < q_heads * head_dim || !addressable(tokens, ldq) || !addressable(tokens, ldq_out)))
        return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt)) return PERF_ERR_DTYPE;
    const int64_t size = dtype_size(x_dt);
    if (!aligned(q, size) || !aligned(q_out, size) || !aligned(k, size) || !aligned(v, size) || !aligned(rotation, 4) ||
        !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(table, 4) || !aligned(lengths, 4) || !aligned(cu, 4))
        return PERF_ERR_ALIGN;
    if (!cache_supported(c) || rotary_dim % 16) return PERF_ERR_UNSUPPORTED;
    AppendArgs a{};
    a.t = PageTable{table, lengths, cu, ldt, (int)tokens, (int)sequences, (int)pages, (int)table_pages, __builtin_ctzll(page_size)};
    a.q = q, a.k = k, a.v = v, a.rotation = rotation, a.q_out = q_out;
    a.k_pages = (uint8_t *)k_pages, a.v_pages = (uint8_t *)v_pages, a.k_scales = k_scales, a.v_scales = v_scales;
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.ldq_out = ldq_out;
    a.q_heads = (int)q_heads, a.kv_heads = (int)kv_heads, a.rotary = (int)rotary_dim, a.positions = (int)positions;
    a.interleaved = interleaved != 0;
    const hipStream_t st = (hipStream_t)stream;
    const auto with = [&](auto one) {
        using T = decltype(one);
        return head_dim == 64 ? append<64, T>(a, st) : head_dim == 128 ? append<128, T>(a, st) : append<256, T>(a, st);
    };
    return x_dt == PERF_BF16 ? with(uint16_t{}) : with(float{});
}
