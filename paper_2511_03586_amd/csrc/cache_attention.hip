// Attention of new tokens' queries over a paged cache in 8 bits (perf_cache_attention_fp8).  For query i of sequence s, at
// position p = lengths[s] + i, and head h, over the keys j <= p (with a window: j > p - window) whose page the table has:
//     S_j = scale * q . k_j,   m = max S_j,   l = sum exp(S_j - m),   o = sum exp(S_j - m) v_j / l,   lse = m + log l.
// A query without keys gets o = 0 and lse = -inf.
#include "cache.h"
#include "fp8.h"

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
};

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
    if (token < seq.first || token >= seq.first + seq.count) return;
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
    return 16;
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
    const hipStream_t st = (hipStream_t)stream;
    if (tokens * q_heads > max_blocks(256)) return PERF_ERR_UNSUPPORTED;
    const dim3 grid((uint32_t)(tokens * q_heads));
    const auto with = [&](auto one) {
        using T = decltype(one);
        if (head_dim == 64)
            cache_attention_kernel<64, T><<<grid, 256, 0, st>>>(a);
        else if (head_dim == 128)
            cache_attention_kernel<128, T><<<grid, 256, 0, st>>>(a);
        else
            cache_attention_kernel<256, T><<<grid, 256, 0, st>>>(a);
        return launch_status();
    };
    return x_dt == PERF_BF16 ? with(uint16_t{}) : with(float{});
}
