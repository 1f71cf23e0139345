// Attention of new tokens' queries over a paged cache in 8 bits (perf_cache_attention_fp8).  For query i of sequence s, at
// position p = lengths[s] + i, and head h, over the keys j <= p (with a window: j > p - window) whose page the table has:
//     S_j = scale * q . k_j,   m = max S_j,   l = sum exp(S_j - m),   o = sum exp(S_j - m) v_j / l,   lse = m + log l.
// A query without keys gets o = 0 and lse = -inf.
//
// Two pairs of kernels, by the rows that a sequence brings to a head of the cache (new tokens x queries that share the head): up to
// 16, or more; each pair takes its sequences from the whole batch, on the device, so that nothing of the lengths is needed on the
// host.  max_tokens leaves the second pair out where no sequence can be for it; the first pair takes 4.7 + 4.6 us where none is
// (reading the lengths, and idle workgroups).
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
    uint32_t group_magic;  // of div_by: rows of a sequence are (token, head of its group)
    float scale;
    // scratch of the kernels for few and for many rows: what is to be joined, and the sums that workgroups leave
    struct Join *few_join, *many_join;
    float *few_partial, *many_partial;
};

// A tile of rows whose keys several workgroups have: the first of them left its sums in slot 2 from + odd, the others of `count`
// in slots 2 (from + 1), 2 (from + 2), ...  Written by the second of them; count is 0 where a run cuts no tile or not first.
struct Join {
    int count, from, odd;
    int first, row0, rows, head;  // the sequence's first token; the tile's first row, and its rows; head of the cache
    int unused;
};

// lse: -infinity without keys, whose maximum is -infinity, for a scale of 0 too
__device__ __forceinline__ float log_of_sum(const AttentionArgs &a, float top, float sum)
{
    return sum == 0.f ? -INFINITY : __builtin_fmaf(top, fabsf(a.scale), logf(sum));
}

// Elements d .. d + 3 of a query and head from the sums of weights and of weighted values
template <typename T>
__device__ __forceinline__ void finish(const AttentionArgs &a, int token, int head, int d, int D, float4_t v, float top, float sum)
{
    const float r = sum == 0.f ? 0.f : 1.0f / sum;
    T *const o = reinterpret_cast<T *>(a.o) + (int64_t)token * a.ldo + (int64_t)head * D + d;
    const float w[4] = {v[0] * r, v[1] * r, v[2] * r, v[3] * r};
    store_row_chunk<true, T, 4>(o, w);
    if (a.lse && d == 0) a.lse[(int64_t)token * a.q_heads + head] = log_of_sum(a, top, sum);
}

template <typename T>
__device__ __forceinline__ void finish_eight(const AttentionArgs &a, int token, int head, int d, int D, float4_t lo, float4_t hi, float top, float sum)
{
    const float r = sum == 0.f ? 0.f : 1.0f / sum;
    const float w[8] = {lo[0] * r, lo[1] * r, lo[2] * r, lo[3] * r, hi[0] * r, hi[1] * r, hi[2] * r, hi[3] * r};
    store_row_chunk<true, T, 8>(reinterpret_cast<T *>(a.o) + (int64_t)token * a.ldo + (int64_t)head * D + d, w);
    if (a.lse && d == 0) a.lse[(int64_t)token * a.q_heads + head] = log_of_sum(a, top, sum);
}

__device__ __forceinline__ int token_of(const AttentionArgs &a, int row, int group) { return div_by(row, group, a.group_magic); }

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

// Transposing loads from LDS (ds_read_b64_tr_b8: of 16 lanes, whose addresses are those of eight rows' halves, lane c gets column c),
// four of them: at four addresses, or at one and kStep, 2 kStep, 3 kStep behind it.  Written out, and waited for at once, because
// in front of the builtin the compiler waits for every load into LDS that is on its way.
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p; }
__device__ __forceinline__ void read_transposed(int2v_t *to, uint32_t at0, uint32_t at1, uint32_t at2, uint32_t at3)
{
    asm volatile("ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(to[0]), "=&v"(to[1]), "=&v"(to[2]), "=&v"(to[3])
                 : "v"(at0), "v"(at1), "v"(at2), "v"(at3)
                 : "memory");
}
template <int kStep>
__device__ __forceinline__ void read_transposed(int2v_t *to, uint32_t at)
{
    asm volatile("ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %4 offset:%5\n\tds_read_b64_tr_b8 %2, %4 offset:%6\n\tds_read_b64_tr_b8 %3, %4 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(to[0]), "=&v"(to[1]), "=&v"(to[2]), "=&v"(to[3])
                 : "v"(at), "n"(kStep), "n"(2 * kStep), "n"(3 * kStep)
                 : "memory");
}

// Values that are the same in all lanes, in scalar registers
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
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
    // (64-bit products are made in vector registers, and a resource that lies there is read lane by lane)
    const int64_t block = uniform((int64_t)max(page, 0) * a.kv_heads + head);
    return make_rsrc(pages + (block << a.t.page_shift) * D, page < 0 ? 0 : (uint32_t)D << a.t.page_shift);
}

// The part of a sequence that a call computes, with its keys [begin, end); begin is on a border of 32, and keys below `low` are
// none: no query sees them, and what lies in their places may be no number, under any scale.
struct Span {
    Sequence q;
    int begin, low, end;
};
__device__ __forceinline__ Span span(const AttentionArgs &a, Sequence q)
{
    Span r;
    r.q = q;
    r.q.count = min(r.q.count, a.max_tokens);
    r.end = (int)min((int64_t)r.q.held + r.q.count, (int64_t)a.t.columns << a.t.page_shift);
    r.low = a.window ? max(r.q.held - a.window + 1, 0) : 0;
    r.begin = r.low & ~31;
    return r;
}
__device__ __forceinline__ Span span(const AttentionArgs &a, int s) { return span(a, sequence(a.t, s)); }
__device__ __forceinline__ Span uniform(Span r)
{
    return Span{Sequence{uniform(r.q.first), uniform(r.q.count), uniform(r.q.held)}, uniform(r.begin), uniform(r.low), uniform(r.end)};
}

// A kernel's tiles, of all items one after the other, are cut into one run for each worker, and none is empty: as many workers as
// tiles, if those are fewer.  Runs are equal, or, of a list that is long enough, by the Shares of the workers: of each XCD's, those
// of the first round of workgroups (32 of them, one to a CU), of the second, of the third.
template <int... kOfRound>
struct Shares {
    static constexpr int kRounds = sizeof...(kOfRound), kOf[kRounds] = {kOfRound...}, kOfXcd = 32 * (kOfRound + ...), kAll = 8 * kOfXcd;
    // shares of the workers before this one; the worker that has this share
    static __device__ __forceinline__ int before(int worker)
    {
        int xcd = worker / (32 * kRounds), at = worker - xcd * 32 * kRounds, sum = xcd * kOfXcd;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) sum += kOf[r] * min(max(at - 32 * r, 0), 32);
        return sum;
    }
    static __device__ __forceinline__ int worker(int share)
    {
        int xcd = share / kOfXcd, at = share - xcd * kOfXcd, found = xcd * 32 * kRounds;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            found += min(at, 32 * kOf[r] - (r + 1 < kRounds ? 0 : 1)) / kOf[r];
            at = max(at - 32 * kOf[r], 0);
        }
        return found;
    }
};
template <typename S>
struct Runs {
    int64_t total;
    int workers;
    bool by_shares;
    __device__ __forceinline__ Runs(int64_t tiles, int most) : total(tiles), workers((int)min(tiles, (int64_t)most)), by_shares(S::kRounds > 1 && tiles >= 2 * S::kAll) {}
    __device__ __forceinline__ int64_t start(int worker) const
    {
        return by_shares ? total * S::before(worker) / S::kAll : total * worker / workers;
    }
    // the worker of a tile: the last whose run begins at it or before
    __device__ __forceinline__ int worker(int64_t tile) const
    {
        return by_shares ? S::worker((int)(((tile + 1) * S::kAll - 1) / total)) : (int)(((tile + 1) * workers - 1) / total);
    }
};

// Tiles of each of `items` (each thread adds up a run of them) and of all, `copies` times over.  The item in which the run of
// `worker` begins and the tiles before it are found on the way.
struct Place {
    int64_t total, start, stop;  // tiles of all copies, and this worker's run of them
    int64_t before;              // of one copy, before the item
    int copy, item;
};
struct PlaceScratch { int64_t of_wave[4], before, item; };
template <typename S, typename Tiles>
__device__ __forceinline__ Place find_place(PlaceScratch &at, int items, int copies, int worker, int most, Tiles &&tiles_of)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (items + 255) / 256, from = min(tid * each, items), to = min(from + each, items);
    int64_t mine = 0;
    tiles_of(from, to, [&](int, int64_t n) { mine += n; });
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up((long long)upto, d);
        upto += lane >= d ? v : 0;
    }
    if (lane == 63) at.of_wave[wave] = upto;
    __syncthreads();
    int64_t one = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        upto += w < wave ? at.of_wave[w] : 0;
        one += at.of_wave[w];
    }
    Place p;
    p.total = one * copies;
    const Runs<S> runs(p.total, most);
    const bool some = worker < runs.workers;
    p.start = some ? runs.start(worker) : 0;
    p.stop = some ? runs.start(worker + 1) : 0;
    p.copy = some ? (int)(p.start / one) : 0;
    const int64_t x = p.start - p.copy * one;
    int64_t before = upto - mine;
    if (some && x >= before && x < upto)
        tiles_of(from, to, [&](int i, int64_t n) {
            if (x >= before && x < before + n) at.before = before, at.item = i;
            before += n;
        });
    __syncthreads();
    p.total = uniform(p.total), p.start = uniform(p.start), p.stop = uniform(p.stop), p.copy = uniform(p.copy);
    p.before = uniform(at.before), p.item = uniform((int)at.item);
    __syncthreads();
    return p;
}

// A tile of rows takes some places of the list before those of its tiles of keys: what a workgroup spends on its beginning and
// end, in tiles of keys.  (With none, 64 sequences of 64 to 32768 tokens took 160-165 us, for 134 so, where 64 of 5242 took 125:
// workgroups that met short sequences met many.)  Lists so short that a run has fewer places than a setup leave workgroups without
// keys: 53 of 256 where six sequences bring 39 tiles of keys to each of ten heads.
constexpr int kFewSetup = 3, kManySetup = 5;

// What has to be joined where the run of `worker` begins, in a tile of rows whose places, `setup` and `tiles`, begin with `start`
template <typename S>
__device__ __forceinline__ Join join_at(const Place &p, const Runs<S> &runs, int worker, int64_t start, int setup, int tiles, Join j)
{
    j.count = 0, j.from = worker - 1, j.odd = 0, j.unused = 0;
    const int64_t before = worker ? runs.start(worker - 1) : 0, first = start + setup;
    if (worker && first < p.start && first >= before) {
        // (the last of them at most: where cu does not ascend, tiles may be other ones than those counted)
        j.count = min(runs.worker(first + tiles - 1), runs.workers - 1) - j.from + 1;
        j.odd = before < start;
    }
    return j;
}

// The sequences' first tokens and lengths in LDS, where they fit
constexpr int kSequencesInLds = 512;
constexpr int kSequencesBytes = (2 * kSequencesInLds + 1) * 4;
struct Sequences {
    const AttentionArgs &a;
    int *firsts, *lengths;
    bool in_lds;
    __device__ __forceinline__ Sequences(const AttentionArgs &args, char *lds) : a(args), firsts(reinterpret_cast<int *>(lds)), lengths(firsts + kSequencesInLds + 1)
    {
        in_lds = a.t.sequences <= kSequencesInLds;
        if (in_lds) {
            for (int i = threadIdx.x; i <= a.t.sequences; i += 256) firsts[i] = first_token(a.t, i);
            for (int i = threadIdx.x; i < a.t.sequences; i += 256) lengths[i] = a.t.lengths[i];
            __syncthreads();
        }
    }
    __device__ __forceinline__ int first(int s) const { return in_lds ? firsts[s] : first_token(a.t, s); }
    __device__ __forceinline__ Span span(int s) const
    {
        return in_lds ? perf::span(a, sequence(firsts[s], firsts[s + 1], lengths[s])) : perf::span(a, s);
    }
};

// ---- few rows: up to 16 of (token, head of a group) ---------------------------------------------------------------------
// Decoding: bound by the bytes of the cache.  The keys of all sequences and heads, in tiles of 128, are one list that is cut into
// equal runs, a workgroup each, whatever the lengths are; a run that begins or ends inside a head's keys leaves its sums in the
// workspace, and the second kernel joins them in order.  Inside a workgroup each of four waves takes 32 keys of a tile through LDS
// of its own, kStages blocks at a time on their way: a block goes to registers whole before the next one of its stage is asked for.
// The waves meet where a head ends.  Sequences' rows and lengths lie in LDS, of up to 512: walking from one to the next then costs
// no trip to memory.
//
// 64 sequences of 64 to 32768 tokens, 8 heads of 128, 32 queries: 134 us, 5.4 TB/s (a copy of 1 GiB reaches 6.4); one of 131071
// tokens 55 us, 5.1 TB/s; 16 of 2048 to 6000 tokens 30-31 us, 4.0 TB/s, of which 10 pass before the first key (lengths, then the run's
// place, then pages, then keys) and 11 with the eight tiles of a run.
//
// S^T = K Q^T and o^T = V^T P^T on v_mfma_f32_16x16x32_bf16, queries in the columns: a lane has one query, keys 4 g .. 4 g + 3 of
// both halves of the 32 (g = lane / 16), whose weights are its share of the second product's operand as they are.  The rows of V
// come transposed from LDS (ds_read_b64_tr_b8: eight rows of one element) in the same order of keys.
constexpr int kFewRows = 16, kFewWaves = 4, kFewKeys = 32 * kFewWaves;

template <int D> constexpr int few_stages() { return D == 64 ? 4 : 2; }
template <int D> constexpr int few_ring() { return kFewWaves * few_stages<D>() * 64 * D; }
template <int D> constexpr int few_lds() { return few_ring<D>() + kSequencesBytes; }
template <int D> constexpr int few_workers() { return D == 256 ? 256 : 512; }  // as many as are on the chip at a time
using FewShares = Shares<1>;
constexpr int partial_floats(int rows, int D) { return rows * (D + 2); }  // sums of a tile of rows, maxima, sums of weights

__device__ __forceinline__ bool is_few(const AttentionArgs &a, int count) { return count * (int64_t)(a.q_heads / a.kv_heads) <= kFewRows; }

// Tiles of one head of a sequence: at least one if it has queries
__device__ __forceinline__ int few_tiles(const AttentionArgs &a, const Span &r)
{
    if (r.q.count == 0 || !is_few(a, r.q.count)) return 0;
    return max((r.end - r.begin + kFewKeys - 1) / kFewKeys, 1);
}

template <int D, typename T>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_attention_few_kernel(const AttentionArgs a)
{
    constexpr int kStages = few_stages<D>(), kStage = 64 * D, kLoads = D / 16;  // loads of a block: K, then V
    constexpr int kQ = sizeof(T) == 4 ? 3 : 1, kP = sizeof(T) == 4 ? 3 : 2;      // bf16 parts of a query's element and of a weight
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
    const int worker = blockIdx.x, group = uniform(a.q_heads / a.kv_heads), shift = a.t.page_shift, in_page = (1 << shift) - 1;
    const Sequences sequences(a, smem + few_ring<D>());
    const Place place = find_place<FewShares>(*reinterpret_cast<PlaceScratch *>(smem), a.t.sequences, 1, worker, gridDim.x, [&](int i, int to, auto &&take) {
        for (; i < to; ++i) {
            const int tiles = few_tiles(a, sequences.span(i));
            take(i, tiles ? (int64_t)(kFewSetup + tiles) * a.kv_heads : 0);
        }
    });
    const int64_t stop = place.stop;
    if (place.start >= stop) {
        if (tid == 0) a.few_join[worker].count = 0;
        return;
    }

    char *const ring = smem + wave * kStages * kStage;
    // a lane's 16 bytes of load i: row of the block's half and chunk
    uint32_t off_k[kLoads / 2], off_v[kLoads / 2];
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) {
        const int row = (i * 64 + lane) / (D / 16), at = lane % (D / 16);
        off_k[i] = (row & 15) * D + ((at ^ turn_k<D>(row)) << 4);
        off_v[i] = (row & 15) * D + ((at ^ turn_v<D>(row)) << 4);
    }
    // where it finds its operands in a stage
    int at_k[2][D / 64], at_v[D / 16];
    const int v_row = (col >> 1 & 3) + 4 * g + (col >> 3) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) at_k[h][j] = (16 * h + col) * D + (((4 * j + g) ^ turn_k<D>(16 * h + col)) << 4);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) at_v[d] = 32 * D + v_row * D + ((d ^ turn_v<D>(v_row)) << 4) + (col & 1) * 8;
    const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f, c = log2_scale(a);

    int s = place.item;
    Span r = uniform(sequences.span(s));
    int tiles = few_tiles(a, r);
    int head = uniform((int)((place.start - place.before) / (kFewSetup + tiles)));
    int64_t start = place.before + (int64_t)head * (kFewSetup + tiles);  // of the head's places
    int t0 = uniform((int)max(place.start - start - kFewSetup, (int64_t)0));
    if (tid == 0)
        a.few_join[worker] = join_at(place, Runs<FewShares>(place.total, gridDim.x), worker, start, kFewSetup, tiles, Join{0, 0, 0, r.q.first, 0, r.q.count * group, head, 0});
    bool first = true;

    // Pages and scales of 64 blocks, one a lane: those of block i are in lane i % 64
    int page0, page1, n, from;
    uint32_t scales;  // bytes: K and V of the first half, K and V of the second
    const auto look_up_pages = [&](int base) {
        const int i = base + lane, k = from + i * kFewKeys;
        page0 = i < n && k < r.end && k + 16 > r.low ? page_at(a.t, s, k >> shift) : -1;
        page1 = i < n && k + 16 < r.end ? page_at(a.t, s, (k + 16) >> shift) : -1;
    };
    const auto look_up_scales = [&] {
        uint32_t b[4] = {0, 0, 0, 0};
        if (page0 >= 0) b[0] = a.k_scales[(int64_t)page0 * a.kv_heads + head], b[1] = a.v_scales[(int64_t)page0 * a.kv_heads + head];
        if (page1 >= 0) b[2] = a.k_scales[(int64_t)page1 * a.kv_heads + head], b[3] = a.v_scales[(int64_t)page1 * a.kv_heads + head];
        scales = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    };
    // the run's tiles of this head, and the pages that this wave meets first
    const auto begin = [&] {
        n = uniform((int)min((int64_t)(tiles - t0), stop - (start + kFewSetup + t0)));
        from = r.begin + t0 * kFewKeys + 32 * wave;
        if (n > 0) look_up_pages(0);
    };
    begin();
    while (n > 0) {
        const int rows = r.q.count * group, held = r.q.held, low = r.low, end = r.end;
        const int token = token_of(a, col, group), position = held + token, last = held + r.q.count - 1;
        asm volatile("" : "+v"(page0), "+v"(page1));

        struct Block { uint32_t scales; int pages; };  // pages: bit h: half h is there
        const auto block_of = [&](int i) {
            return Block{(uint32_t)__builtin_amdgcn_readlane((int)scales, i & 63),
                         (__builtin_amdgcn_readlane(page0, i & 63) >= 0 ? 1 : 0) | (__builtin_amdgcn_readlane(page1, i & 63) >= 0 ? 2 : 0)};
        };
        auto issue = [&](int i) {  // (blocks past the end move nothing: the number in flight stays the same)
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
        };
#pragma unroll
        for (int i = 0; i < kStages; ++i) issue(i);
        look_up_scales();

        // this lane's query (columns without one repeat another)
        bf16x8_t q[D / 32][kQ];
        {
            const T *row = reinterpret_cast<const T *>(a.q) + (int64_t)(r.q.first + min(token, r.q.count - 1)) * a.ldq + (int64_t)(head * group + col - token * group) * D;
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
        wait_vmem<0>();
        asm volatile("" : "+v"(scales));

        float4_t o[D / 16];
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] = float4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        Block ahead[kStages];
#pragma unroll
        for (int i = 0; i < kStages; ++i) ahead[i] = block_of(i);
        int stage = 0;
        for (int i = 0; i < n; ++i) {
            wait_vmem<(kStages - 1) * kLoads>();
            fence();
            // the block goes to registers at once, and the next one of its stage is on its way while it is computed
            int4v_t raw_k[2][D / 64];
            int2v_t raw_v[D / 16];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < D / 64; ++j) raw_k[h][j] = *reinterpret_cast<const int4v_t *>(ring + stage + at_k[h][j]);
            const uint32_t in_stage = lds_address(ring) + stage;
#pragma unroll
            for (int d = 0; d < D / 16; d += 4)
                read_transposed(raw_v + d, in_stage + at_v[d], in_stage + at_v[d + 1], in_stage + at_v[d + 2], in_stage + at_v[d + 3]);
            wait_lds();
            fence();
            const Block now = ahead[0];
#pragma unroll
            for (int j = 0; j + 1 < kStages; ++j) ahead[j] = ahead[j + 1];
            if (((i + kStages) & 63) == 0) {
                look_up_pages(i + kStages);
                look_up_scales();
                wait_vmem<0>();
                asm volatile("" : "+v"(page0), "+v"(page1), "+v"(scales));
            }
            issue(i + kStages);
            ahead[kStages - 1] = block_of(i + kStages);
            stage = stage + kStage == kStages * kStage ? 0 : stage + kStage;
            const int k = from + i * kFewKeys;
            if (k >= end) continue;

            float4_t sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float power = scale_of(now.scales >> (16 * h) & 255);
                sc[h] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bf16x8_t f = widen_eight(raw_k[h][j][2 * e], raw_k[h][j][2 * e + 1], power, power);
#pragma unroll
                        for (int p = kQ - 1; p >= 0; --p) sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[2 * j + e][p], sc[h], 0, 0, 0);
                    }
                }
            }
            int keep[2] = {-1, -1};  // bytes of V that are keys (a weight of zero does not cancel a NaN)
            if (now.pages != 3 || k + 31 > held || (a.window && k <= last - a.window)) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = k + 16 * h + 4 * g + e;
                        const bool there = key >= low && key < end && (now.pages >> h & 1);
                        const bool seen = there && key <= position && (!a.window || key > position - a.window);
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
                const bf16x8_t f = widen_eight(raw_v[d][0] & keep[0], raw_v[d][1] & keep[1], power0, power1);
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
        const bool whole = n == tiles;
        float *const out = whole ? nullptr : a.few_partial + (int64_t)(2 * worker + !first) * partial_floats(kFewRows, D);
        const int of_token = r.q.first, of_head = head * group;
        first = false;
        // the next head's first pages are on their way while this one's sums are joined
        start += kFewSetup + tiles, t0 = 0;
        if (start < stop) {
            if (++head == a.kv_heads) {
                head = 0;
                do {
                    if (++s >= a.t.sequences) return;  // (there is one, unless the lengths change meanwhile)
                    r = uniform(sequences.span(s)), tiles = few_tiles(a, r);
                } while (tiles == 0);
            }
        }
        begin();
        __syncthreads();
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
                finish<T>(a, of_token + token_of(a, row, group), of_head + row - token_of(a, row, group) * group, d, D, v, top, sum);
            } else {
                *reinterpret_cast<float4_t *>(out + row * D + d) = v;
                if (d == 0) out[kFewRows * D + row] = top, out[kFewRows * (D + 1) + row] = sum;
            }
        }
        __syncthreads();
    }
}

// ---- many rows --------------------------------------------------------------------------------------------------------------
// Prompts: bound by the matrix units and by the vector work beside them.  Tiles of 128 rows of (token, head of a group) and one head
// of the cache meet its keys 64 at a time, which pass through three stages of LDS, loaded by all four waves, one barrier to a block;
// each wave has 32 of the rows.  The blocks of all row tiles and heads are one list, cut into equal runs as above, heads first: an
// XCD's workgroups take neighbouring runs, which share keys in its L2.
//
// 4 prompts of about 2048 tokens, 8 heads of 128, 32 queries: 208-230 us, 0.60-0.66 PFLOP/s of what is seen (a large library product
// in bf16: 1.2).  Beside the 32 products of a wave and block (0.49 us) stand some 320 vector instructions for widening keys and
// values, exponentials and maxima, which two waves of a SIMD hide from each other in part: 1.15 us a block and SIMD, by what a
// longer context adds.  Blocks are two thirds of the time here, beginnings and ends of row tiles, five to a workgroup, the rest.
// 64 rows to a wave, which widen half as often, leave one wave to a SIMD: 334 us.  Keys widened once for two waves, weights
// through LDS: 240 us.  With fp32 queries, for the same operations, 506 us (heads of 64: 302, half the operations; of 256: 497, though
// 71 registers of a lane go to memory there); heads of 256 in bf16, one wave to a SIMD, 246.
//
// The products are those above on v_mfma_f32_32x32x16_bf16: a lane has one query, and keys 4 g .. 4 g + 3 of every eight (g =
// lane / 32).  The weights of bf16 queries are rounded to bf16 once (the few rows' kernel, which waits for memory, keeps 16 bits
// of them): another product with what that leaves makes 214 us 274 (20 mixed sequences 162 -> 201, 32 of 512 tokens 71 -> 79), and
// the error against 64 bits 0.0019 instead of 0.00166, most of which is the rounding of o.  A running maximum is raised only by more
// than 2^8 in weights, which fp32 sums carry as well: the sums are then seldom scaled.
constexpr int kManyKeys = 64, kManyStages = 3;
constexpr int kManyRows = 128;
// workgroups to a CU, by the registers that a wave needs for its queries and sums
template <int D, typename T> constexpr int many_per_cu() { return D == 256 || (D == 128 && sizeof(T) == 4) ? 1 : D == 64 && sizeof(T) == 2 ? 3 : 2; }
// Of workgroups that share a CU the one that came first is served first: with equal runs it ended after 167 us and the second after
// 217 (4 prompts of about 2048 tokens, heads of 128), and the second's waves, then alone, hide nothing.  Equal runs, then these, a call:
// 4 x 2048 tokens 228 -> 216 us, on 1024 tokens 378 -> 361, on 4096 827 -> 803; with three to a CU (heads of 64) 32 x 512 80 -> 70, on
// 2048 276 -> 260.  6 : 5 and 3 : 2 are slower.  8 x 512 on 8192, whose row tiles have 129 blocks and more, lose: 675 -> 686.  The
// kernel for few rows, which waits for memory, gains nothing by it.
template <int D, typename T>
using ManyShares = std::conditional_t<many_per_cu<D, T>() == 1, Shares<1>, std::conditional_t<many_per_cu<D, T>() == 2, Shares<4, 3>, Shares<7, 4, 3>>>;
template <int D, typename T> constexpr int many_workers() { return 256 * many_per_cu<D, T>(); }
// (three stages; for heads of 64 a little more, which the sums need on their way out)
template <int D> constexpr int many_ring() { return std::max(kManyStages * 2 * kManyKeys * D, 4 * (32 * 68 + 64) * 4); }
template <int D> constexpr int many_lds() { return many_ring<D>() + kSequencesBytes; }

template <int D> __device__ __forceinline__ constexpr int turn_many_v(int r)
{
    return D == 64 ? (((r >> 3) & 1) << 1) | ((r >> 2) & 1) : D == 128 ? (((r >> 1) & 1) << 1) | (((r >> 3) & 1) << 2) | ((r >> 2) & 1) : ((r & 3) << 1) | (((r >> 3) & 1) << 3) | ((r >> 2) & 1);
}

// Row tiles of a sequence, whose first new token is `first`, begin at this number: those of `count` tokens are at most
// count * group / rows + 1.  (Where cu does not ascend they overlap or leave gaps: then some rows are not computed, and nothing
// below relies on their order.)
__device__ __forceinline__ int many_start(int first, int group, int rows, int s) { return s == 0 ? 0 : (int)((int64_t)first * group / rows) + s; }
inline int64_t many_units(int64_t tokens, int64_t sequences, int64_t group, int rows) { return tokens * group / rows + sequences; }

// The keys that a row tile needs: [begin, end), begin on a border of 64, and those below `low` none as above
struct Keys { int begin, low, end, tiles; };
__device__ __forceinline__ Keys uniform(Keys k) { return Keys{uniform(k.begin), uniform(k.low), uniform(k.end), uniform(k.tiles)}; }
__device__ __forceinline__ Keys many_keys(const AttentionArgs &a, const Span &r, int group, int tile, int tile_rows)
{
    const int rows = r.q.count * group, row = tile * tile_rows;
    Keys k{0, 0, 0, 0};
    if (row >= rows || is_few(a, r.q.count)) return k;
    const int token0 = token_of(a, row, group), token1 = token_of(a, min(row + tile_rows, rows) - 1, group);
    k.end = (int)min((int64_t)r.q.held + token1 + 1, (int64_t)a.t.columns << a.t.page_shift);
    k.low = a.window ? max(r.q.held + token0 - a.window + 1, 0) : 0;
    k.begin = k.low & ~(kManyKeys - 1);
    k.tiles = max((k.end - k.begin + kManyKeys - 1) / kManyKeys, 1);
    return k;
}

template <int D, typename T>
__global__ __launch_bounds__(256, (many_per_cu<D, T>())) void cache_attention_many_kernel(const AttentionArgs a, int units)
{
    constexpr int kStage = 2 * kManyKeys * D, kLoads = D / 32;                  // loads of a wave and block: K, then V
    constexpr int kQ = sizeof(T) == 4 ? 3 : 1, kP = sizeof(T) == 4 ? 3 : 1;     // bf16 parts of a query's element and of a weight
    constexpr int kRows = kManyRows;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, col = lane & 31;
    const int group = uniform(a.q_heads / a.kv_heads), shift = a.t.page_shift, in_page = (1 << shift) - 1, sequences = a.t.sequences;
    const int worker = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);  // (a multiple of 8 workgroups)

    const Sequences all(a, smem + many_ring<D>());
    const auto start_of = [&](int s) { return many_start(all.first(s), group, kRows, s); };
    const Place place = find_place<ManyShares<D, T>>(*reinterpret_cast<PlaceScratch *>(smem), units, a.kv_heads, worker, gridDim.x, [&](int u, int to, auto &&take) {
        if (u >= to) return;
        int s = 0;  // the last sequence that begins at u or before
        for (int n = sequences; n > 1;) {
            const int half = n >> 1;
            if (start_of(s + half) <= u) s += half, n -= half; else n = half;
        }
        for (; u < to; ++u) {
            while (s + 1 < sequences && start_of(s + 1) <= u) ++s;
            const int tiles = many_keys(a, all.span(s), group, u - start_of(s), kRows).tiles;
            take(u, tiles ? kManySetup + tiles : 0);
        }
    });
    const int64_t stop = place.stop;
    if (place.start >= stop) {
        if (tid == 0) a.many_join[worker].count = 0;
        return;
    }

    // a lane's 16 bytes of load i of its wave's 16 rows
    uint32_t off_k[kLoads / 2], off_v[kLoads / 2];
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) {
        const int row = (i * 64 + lane) / (D / 16), at = lane % (D / 16);
        off_k[i] = row * D + ((at ^ turn_k<D>(row + 16 * wave)) << 4);
        off_v[i] = row * D + ((at ^ turn_many_v<D>(row + 16 * wave)) << 4);
    }
    // where it finds its operands in a stage: of the first 32 keys, and of the first 16
    int at_k[D / 32], at_v[D / 32];
    const int v_row = 4 * g + (lane >> 1 & 3) + (lane >> 3 & 1) * 8;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        at_k[j] = col * D + (((2 * j + g) ^ turn_k<D>(col)) << 4);
        at_v[j] = (kManyKeys + v_row) * D + (((2 * j + (lane >> 4 & 1)) ^ turn_many_v<D>(v_row)) << 4) + (lane & 1) * 8;
    }
    const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f, c = log2_scale(a);

    int head = place.copy, u = place.item;
    int s = find_sequence(sequences, u, start_of);
    Span r = uniform(all.span(s));
    int tile = u - uniform(start_of(s));
    int64_t start = head * (place.total / a.kv_heads) + place.before;  // of the row tile's places
    int t0 = uniform((int)max(place.start - start - kManySetup, (int64_t)0));
    Keys keys = uniform(many_keys(a, r, group, tile, kRows));
    if (tid == 0)
        a.many_join[worker] = join_at(place, Runs<ManyShares<D, T>>(place.total, gridDim.x), worker, start, kManySetup, keys.tiles,
                                      Join{0, 0, 0, r.q.first, tile * kRows, min(r.q.count * group - tile * kRows, kRows), head, 0});
    bool first = true;

    // Pages and scales of 64 pieces of 16 keys, one a lane: 16 blocks, and of the 16 behind them
    struct Pieces {
        int page;
        uint32_t scales;  // bytes of K and V; bit 16: the page is there
    };
    Pieces pieces{-1, 0}, ahead{-1, 0};
    int n, from;
    const auto look_up_page = [&](Pieces &p, int i) {
        const int k = from + i * kManyKeys + 16 * lane;
        p.page = k < keys.end && k + 16 > keys.low ? page_at(a.t, s, k >> shift) : -1;
    };
    const auto look_up_scales = [&](Pieces &p) {
        const int64_t block = (int64_t)p.page * a.kv_heads + head;
        p.scales = 0;
        if (p.page >= 0) p.scales = 0x10000 | a.k_scales[block] | (uint32_t)a.v_scales[block] << 8;
    };
    // the run's tiles of keys of this row tile, and the first pages
    const auto begin = [&] {
        n = uniform((int)min((int64_t)(keys.tiles - t0), stop - (start + kManySetup + t0)));
        from = keys.begin + t0 * kManyKeys;
        if (n > 0) look_up_page(pieces, 0);
    };
    begin();
    while (n > 0) {
        const int held = r.q.held, low_key = keys.low, end = keys.end, rows = r.q.count * group;
        const int row0 = tile * kRows + 32 * wave, row = min(row0 + col, rows - 1);  // this wave's first row, and this lane's
        const bool active = row0 < rows;
        const int token = token_of(a, row, group), of_group = row - token * group, position = held + token;
        // positions of the wave's first and last row, by which its blocks are taken, masked or left out
        const int low = __builtin_amdgcn_readfirstlane(position), high = __builtin_amdgcn_readlane(position, 31);

        struct Block { uint32_t scales0, scales1, scales2, scales3; };  // of its four pieces
        const auto block_of = [&](int i) {
            const auto of = [&](int j) { return (uint32_t)__builtin_amdgcn_readlane((int)pieces.scales, 4 * (i & 15) + j); };
            return Block{of(0), of(1), of(2), of(3)};
        };
        int to_stage = 0, stage = 0;
        auto issue = [&](int i) {
            // (scalar multiplications: unsigned, of 32 bits each)
            const int p = __builtin_amdgcn_readlane(pieces.page, 4 * (i & 15) + wave);
            const uint64_t block = ((uint64_t)(uint32_t)max(p, 0) * (uint32_t)a.kv_heads + (uint32_t)head) << shift << __builtin_ctz(D);
            const uint32_t bytes = p < 0 ? 0 : (uint32_t)D << shift;
            const rsrc_t in_k = make_rsrc(a.k_pages + block, bytes), in_v = make_rsrc(a.v_pages + block, bytes);
            const uint32_t at = (uint32_t)((from + i * kManyKeys + 16 * wave) & in_page) * D;
            char *const to = smem + to_stage + wave * 16 * D;
            to_stage = to_stage + kStage == kManyStages * kStage ? 0 : to_stage + kStage;
#pragma unroll
            for (int j = 0; j < kLoads / 2; ++j) issue_load_to(in_k, off_k[j], at, to + j * 1024);
#pragma unroll
            for (int j = 0; j < kLoads / 2; ++j) issue_load_to(in_v, off_v[j], at, to + kManyKeys * D + j * 1024);
        };
        issue(0), issue(1);
        look_up_scales(pieces);

        // this lane's query
        bf16x8_t q[D / 16][kQ];
        {
            const T *in = reinterpret_cast<const T *>(a.q) + (int64_t)(r.q.first + token) * a.ldq + (int64_t)(head * group + of_group) * D;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                Eight<T> raw;
                raw.load_cached(in + 32 * (i >> 1) + 16 * g + 8 * (i & 1), 8);
                float v[8];
                raw.get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= sign;
                split_eight(v, q[i]);
            }
        }
        wait_vmem<0>();
        asm volatile("" : "+v"(pieces.scales));

        float16_t o[D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] = float16_t{};
        float m = -INFINITY, l = 0.f;
        // A maximum that rises by more than 2^8 leaves the loop, which takes the block up again behind it: sums that are scaled on
        // one of two paths inside would be copied on the other, all of them for each block.
        Block now = block_of(0), next = block_of(1), of = now;
        int in = 0;
        bool loaded = false, there = true;
        int i = 0;
        while (i < n) {
            float raised = -INFINITY;
            for (; i < n; ++i) {
                const int k = from + i * kManyKeys;
                if (!loaded) {
                    wait_vmem<kLoads>();  // this wave's part of the block has arrived, and what it read of the one before
                    wait_lds();
                    wg_barrier();
                    // (the pieces of the next 16 blocks: pages, then scales, then both)
                    if ((i & 15) == 3) look_up_page(ahead, (i & ~15) + 16);
                    if ((i & 15) == 8) look_up_scales(ahead);
                    if ((i & 15) == 14) pieces = ahead;
                    issue(i + 2);
                    of = now, now = next, next = block_of(i + 2);
                    in = stage;
                    stage = stage + kStage == kManyStages * kStage ? 0 : stage + kStage;
                    there = (of.scales0 & of.scales1 & of.scales2 & of.scales3) >> 16;
                    if (!there || k < low_key || k + kManyKeys > end) {
                        // values that are not there or that no row sees: zeros, whatever lies in their places (a weight of zero does not cancel a NaN)
                        const uint32_t s0 = of.scales0, s1 = of.scales1, s2 = of.scales2, s3 = of.scales3, piece = wave < 2 ? (wave == 0 ? +s0 : +s1) : (wave == 2 ? +s2 : +s3);
                        for (int j = lane; j < D; j += 64) {  // this wave's 16 keys, 16 bytes at a time
                            const int key = 16 * wave + j / (D / 16);
                            if (!(piece >> 16) || k + key < low_key || k + key >= end) *reinterpret_cast<uint4_t *>(smem + in + (kManyKeys + 16 * wave) * D + 16 * j) = uint4_t{0, 0, 0, 0};
                        }
                        wait_lds();
                        wg_barrier();
                    }
                }
                loaded = false;
                if (!active || k > high || (a.window && k + kManyKeys - 1 <= low - a.window)) continue;

                const uint32_t of_piece[4] = {of.scales0, of.scales1, of.scales2, of.scales3};
                int4v_t raw_k[2][D / 32];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) raw_k[h][j] = *reinterpret_cast<const int4v_t *>(smem + in + at_k[j] + 32 * h * D);
                float16_t sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float power = col < 16 ? scale_of(of_piece[2 * h] & 255) : scale_of(of_piece[2 * h + 1] & 255);
                    sc[h] = float16_t{};
#pragma unroll
                    for (int j = 0; j < D / 32; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const bf16x8_t f = widen_eight(raw_k[h][j][2 * e], raw_k[h][j][2 * e + 1], power, power);
#pragma unroll
                            for (int p = kQ - 1; p >= 0; --p) sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[2 * j + e][p], sc[h], 0, 0, 0);
                        }
                }
                // (while the last products run)
                int2v_t raw_v[D / 32][4];
#pragma unroll
                for (int d = 0; d < D / 32; ++d) read_transposed<16 * D>(raw_v[d], lds_address(smem) + in + at_v[d]);
                if (!there || k + kManyKeys - 1 > low || (a.window && k <= high - a.window)) {
                    // keys of a lane, counted from its first, that the row sees: those above `over`, up to `upto`
                    int upto = min(position, end - 1) - k - 4 * g, over = a.window ? position - a.window - k - 4 * g : -1;
                    asm("" : "+v"(upto), "+v"(over));
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int key = 32 * h + 8 * (e >> 2) + (e & 3);
                            const bool seen = (of_piece[2 * h + (e >> 3)] >> 16) && key <= upto && key > over;
                            sc[h][e] = seen ? sc[h][e] : -INFINITY;
                        }
                }
                float top = sc[0][0];
#pragma unroll
                for (int e = 1; e < 32; ++e) top = __builtin_fmaxf(top, sc[e >> 4][e & 15]);
                float t_a, t_b;
                swap32(top, t_a, t_b);
                top = __builtin_fmaxf(t_a, t_b);
                if (__ballot(m > -INFINITY && (top - m) * c > 8.f)) {
                    raised = top;
                    break;
                }
                m = m == -INFINITY ? top : m;  // (its sums are zeros so far)
                const float top_c = m == -INFINITY ? 0.f : m * c;
#pragma unroll
                for (int step = 0; step < 4; ++step) {
                    float p[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = weight(sc[step >> 1][8 * (step & 1) + e], c, top_c);
                    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                    bf16x8_t w[kP];
                    split_eight(p, w);
                    const float power = scale_of(of_piece[step] >> 8 & 255);
#pragma unroll
                    for (int d = 0; d < D / 32; ++d) {
                        const bf16x8_t f = widen_eight(raw_v[d][step][0], raw_v[d][step][1], power, power);
#pragma unroll
                        for (int e = kP - 1; e >= 0; --e) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, w[e], o[d], 0, 0, 0);
                    }
                }
            }
            if (i == n) break;
            loaded = true;
            raised = __builtin_fmaxf(m, raised);
            const float shrink = m == -INFINITY ? 1.f : weight(m, c, raised * c);
            l *= shrink;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= shrink;
            m = raised;
        }
        const bool whole = n == keys.tiles;
        const int in_tile0 = 32 * wave, last_row = rows - row0;  // (rows of the wave, if positive)
        float *const out = whole ? nullptr : a.many_partial + (int64_t)(2 * worker + !first) * partial_floats(kRows, D);
        const int of_first = r.q.first, of_head = head * group;
        first = false;
        // the next row tile that has keys, whose first pages are on their way while this one's sums are stored
        start += kManySetup + keys.tiles, t0 = 0;
        if (start < stop) {
            do {
                if (++u == units) {
                    u = 0, s = 0;
                    if (++head == a.kv_heads) return;  // (only where cu does not ascend)
                    r = uniform(all.span(s));
                }
                while (s + 1 < sequences && uniform(start_of(s + 1)) <= u) r = uniform(all.span(++s));
                tile = u - uniform(start_of(s));
                keys = uniform(many_keys(a, r, group, tile, kRows));
            } while (keys.tiles == 0);
        }
        begin();
        wait_vmem_and_lds<0>();
        wg_barrier();  // the stages are free

        // The wave's sums pass through LDS of its own, 64 elements of its 32 rows at a time, so that rows are stored in long runs
        float l_a, l_b;
        swap32(l, l_a, l_b);
        l = l_a + l_b;
        constexpr int kPitch = 68;
        float *const staged = reinterpret_cast<float *>(smem) + wave * (32 * kPitch + 64);
        static_assert(4 * (32 * kPitch + 64) * 4 <= many_ring<D>(), "the stages hold them");
        if (g == 0) staged[32 * kPitch + col] = m, staged[32 * kPitch + 32 + col] = l;
#pragma unroll
        for (int d = 0; d < D; d += 64) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                *reinterpret_cast<float4_t *>(staged + col * kPitch + 8 * e + 4 * g) =
                    float4_t{o[d / 32 + e / 4][4 * (e & 3)], o[d / 32 + e / 4][4 * (e & 3) + 1], o[d / 32 + e / 4][4 * (e & 3) + 2], o[d / 32 + e / 4][4 * (e & 3) + 3]};
            wait_lds();
            fence();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int of = 8 * j + (lane >> 3), at = 8 * (lane & 7);
                const float4_t lo = *reinterpret_cast<const float4_t *>(staged + of * kPitch + at), hi = *reinterpret_cast<const float4_t *>(staged + of * kPitch + at + 4);
                const float top = staged[32 * kPitch + of], sum = staged[32 * kPitch + 32 + of];
                if (of < last_row) {
                    if (whole) {
                        const int token = token_of(a, row0 + of, group);
                        finish_eight<T>(a, of_first + token, of_head + row0 + of - token * group, d + at, D, lo, hi, top, sum);
                    } else {
                        float *const to = out + (in_tile0 + of) * D + d + at;
                        *reinterpret_cast<float4_t *>(to) = lo, *reinterpret_cast<float4_t *>(to + 4) = hi;
                        if (d + at == 0) out[kRows * D + in_tile0 + of] = top, out[kRows * (D + 1) + in_tile0 + of] = sum;
                    }
                }
            }
            wait_lds();
            fence();
        }
        wg_barrier();  // before the next row tile's keys come
    }
}

// ---- both ----------------------------------------------------------------------------------------------------------------------
// Joins what several workgroups have left of one tile of rows, in their order, the largest maximum first: for each beginning of
// a run as many workgroups as the grid's other dimension has, which deal out its rows.  What few workgroups left is added by the
// D / 4 lanes of a row; of more, all teams of so many take a share.  Bound by trips to memory for few rows (3.3-5 us) and by the sums'
// bytes for many: 51 MB in 17-18 us after 4 prompts of about 2048 tokens.  (A fourth of the workgroups for few rows, where most are
// idle, 1.7 for 4.6 us, makes a mixed batch's join 10.6 for 5.7 us.)
template <int D, typename T, bool MANY>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(const AttentionArgs a)
{
    constexpr int kTile = MANY ? kManyRows : kFewRows, kWorkers = MANY ? many_workers<D, T>() : few_workers<D>();
    constexpr int kLanes = D / 4, kTeams = 256 / kLanes, kSerial = 8;
    __shared__ float factor[kWorkers], of_wave[2][4];
    __shared__ float4_t sums[kTeams][kLanes];
    const int tid = threadIdx.x, group = a.q_heads / a.kv_heads;
    const Join j = (MANY ? a.many_join : a.few_join)[blockIdx.x];
    const int count = j.count, rows = j.rows;
    if (count == 0) return;
    const float *const partials = MANY ? a.many_partial : a.few_partial;
    const auto partial = [&](int i) { return partials + (int64_t)(2 * (j.from + i) + (i == 0 ? j.odd : 0)) * partial_floats(kTile, D); };
    const float c = log2_scale(a);
    const int d = tid % kLanes, team = tid / kLanes;
    const auto put = [&](int row, float4_t v, float top, float sum) {
        const int of_all = j.row0 + row, token = token_of(a, of_all, group);
        finish<T>(a, j.first + token, j.head * group + of_all - token * group, 4 * d, D, v, top, sum);
    };
    if (count <= kSerial) {
        for (int row = blockIdx.y * kTeams + team; row < rows; row += gridDim.y * kTeams) {
            float m[kSerial], l[kSerial], top = -INFINITY, sum = 0.f;
            float4_t o[kSerial];
#pragma unroll
            for (int i = 0; i < kSerial; ++i) {
                const float *const of = partial(min(i, count - 1));
                m[i] = of[kTile * D + row], l[i] = of[kTile * (D + 1) + row], o[i] = *reinterpret_cast<const float4_t *>(of + row * D + 4 * d);
                top = __builtin_fmaxf(top, m[i]);
            }
            const float top_c = top == -INFINITY ? 0.f : top * c;
            float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kSerial; ++i)
                if (i < count) {
                    const float f = weight(m[i], c, top_c);
                    v += f * o[i], sum += f * l[i];
                }
            put(row, v, top, sum);
        }
        return;
    }
    for (int row = blockIdx.y; row < rows; row += gridDim.y) {
        float top = -INFINITY;
        for (int i = tid; i < count; i += 256) {
            factor[i] = partial(i)[kTile * D + row];
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
            sum += factor[i] * partial(i)[kTile * (D + 1) + row];
        }
        sum = wave_allreduce(sum, OpSum());
        if ((tid & 63) == 0) of_wave[1][tid >> 6] = sum;
        __syncthreads();
        sum = (of_wave[1][0] + of_wave[1][1]) + (of_wave[1][2] + of_wave[1][3]);
        float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = team; i < count; i += kTeams) v += factor[i] * *reinterpret_cast<const float4_t *>(partial(i) + row * D + 4 * d);
        sums[team][d] = v;
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int i = 1; i < kTeams; ++i) v += sums[i][d];
            put(row, v, top, sum);
        }
        __syncthreads();
    }
}

// Scratch: what is to be joined, then the sums
struct Scratch { int64_t many_join, few_partial, many_partial, bytes; };  // where these begin, in bytes
template <int D>
static Scratch scratch(int64_t tokens, int64_t max_tokens, int64_t group)
{
    const bool many = std::min(max_tokens, tokens) * group > kFewRows;
    constexpr int kMany = many_workers<D, uint16_t>();  // (as many as of any type)
    Scratch s;
    s.many_join = few_workers<D>() * sizeof(Join);
    s.few_partial = s.many_join + kMany * sizeof(Join);
    s.many_partial = s.few_partial + 8ll * few_workers<D>() * partial_floats(kFewRows, D);
    s.bytes = s.many_partial + (many ? 8ll * kMany * partial_floats(kManyRows, D) : 0);
    return s;
}

template <int D, typename T>
static perf_status attention(AttentionArgs &a, char *workspace, hipStream_t st)
{
    const int64_t group = a.q_heads / a.kv_heads, units = many_units(a.t.tokens, a.t.sequences, group, kManyRows);
    a.group_magic = div_magic(group);
    const Scratch at = scratch<D>(a.t.tokens, a.max_tokens, group);
    a.few_join = (Join *)workspace, a.many_join = (Join *)(workspace + at.many_join);
    a.few_partial = (float *)(workspace + at.few_partial), a.many_partial = (float *)(workspace + at.many_partial);
    const bool many = a.max_tokens * group > kFewRows;  // (whether a sequence of as many tokens is for the other kernel)
    if (!allow_lds<cache_attention_few_kernel<D, T>>(few_lds<D>())) return PERF_ERR_LAUNCH;
    cache_attention_few_kernel<D, T><<<few_workers<D>(), 256, few_lds<D>(), st>>>(a);
    const uint32_t rows = (uint32_t)std::min<int64_t>(kFewRows, a.max_tokens * group);
    cache_attention_join_kernel<D, T, false><<<dim3(few_workers<D>(), rows), 256, 0, st>>>(a);
    if (many) {
        if (!allow_lds<cache_attention_many_kernel<D, T>>(many_lds<D>())) return PERF_ERR_LAUNCH;
        cache_attention_many_kernel<D, T><<<many_workers<D, T>(), 256, many_lds<D>(), st>>>(a, (int)units);
        cache_attention_join_kernel<D, T, true><<<dim3(many_workers<D, T>(), 16), 256, 0, st>>>(a);
    }
    return launch_status();
}

}  // namespace perf

using namespace perf;

static bool attention_shape_ok(const CacheShape &c, int64_t max_tokens)
{
    return cache_shape_ok(c) && c.head_dim <= kMaxExtent8 / kMaxHeads && max_tokens >= 1;
}

// (rows of a sequence are counted in 31 bits)
static bool attention_supported(const CacheShape &c) { return cache_supported(c) && c.tokens * (c.q_heads / c.kv_heads) <= kMaxExtent8; }

extern "C" int64_t perf_cache_attention_fp8_workspace_bytes(int64_t tokens, int64_t sequences, int64_t max_tokens, int64_t q_heads,
                                                            int64_t kv_heads, int64_t head_dim, int64_t page_size, int64_t table_pages)
{
    const CacheShape c{tokens, sequences, q_heads, kv_heads, head_dim, 1, page_size, table_pages, table_pages};
    if (!attention_shape_ok(c, max_tokens) || !attention_supported(c)) return -1;
    const int64_t group = q_heads / kv_heads;
    return (head_dim == 64    ? scratch<64>(tokens, max_tokens, group)
            : head_dim == 128 ? scratch<128>(tokens, max_tokens, group)
                              : scratch<256>(tokens, max_tokens, group))
        .bytes;
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
    if (!attention_supported(c)) return PERF_ERR_UNSUPPORTED;
    AttentionArgs a{};
    a.t = PageTable{table, lengths, cu, ldt, (int)tokens, (int)sequences, (int)pages, (int)table_pages, __builtin_ctzll(page_size)};
    a.q = q, a.o = o, a.lse = lse, a.ldq = ldq, a.ldo = ldo;
    a.k_pages = (const uint8_t *)k_pages, a.v_pages = (const uint8_t *)v_pages, a.k_scales = k_scales, a.v_scales = v_scales;
    a.q_heads = (int)q_heads, a.kv_heads = (int)kv_heads, a.max_tokens = (int)std::min(max_tokens, tokens), a.window = (int)window, a.scale = scale;
    const hipStream_t st = (hipStream_t)stream;
    const auto with = [&](auto one) {
        using T = decltype(one);
        char *const ws = (char *)workspace;
        return head_dim == 64 ? attention<64, T>(a, ws, st) : head_dim == 128 ? attention<128, T>(a, ws, st) : attention<256, T>(a, ws, st);
    };
    return x_dt == PERF_BF16 ? with(uint16_t{}) : with(float{});
}
