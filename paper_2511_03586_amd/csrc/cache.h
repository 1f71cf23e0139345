// A cache of keys and values in pages of 8-bit values (e4m3), shared by the kernels that append to it and that attend to it.
// A page holds `page_size` tokens (a power of two) of every head, [kv_heads][page_size][head_dim]; a byte b for each page and
// head is their scale 2^(b - 127), 255 that of a block that took a value which is no finite number.  Sequence s holds
// lengths[s] tokens and brings those from cu[s] to cu[s + 1], at the positions that follow; position p lies in slot
// p % page_size of page table[s][p / page_size].
//
// lengths, cu and table lie on the device and cannot be checked before a launch: nothing they hold leads outside the buffers.
#pragma once
#include "device_utils.h"
#include "host_utils.h"

namespace perf {

constexpr int64_t kMaxTokens = 1 << 28;      // rows of a call
constexpr int64_t kMaxSequences = 1 << 24;
constexpr int64_t kMaxHeads = 1024;
constexpr int64_t kMaxPosition = 1 << 30;    // pages of a sequence x tokens of a page
constexpr int kNoNumber = 255;               // scale of a block that took an infinity or a NaN

struct PageTable {
    const int32_t *table, *lengths, *cu;
    int64_t ldt;
    int tokens, sequences, pages, columns, page_shift;
};

struct Sequence {
    int first, count, held;  // first of its new tokens, how many, and how many tokens it holds before them
};

__device__ __forceinline__ int first_token(const PageTable &t, int s) { return min(max(t.cu[s], 0), t.tokens); }

__device__ __forceinline__ Sequence sequence(int first, int next, int length)
{
    return Sequence{first, length < 0 ? 0 : max(next - first, 0), min(length, (int)kMaxPosition)};
}
__device__ __forceinline__ Sequence sequence(const PageTable &t, int s) { return sequence(first_token(t, s), first_token(t, s + 1), t.lengths[s]); }

// Page of a sequence's column, or -1 where the table has none
__device__ __forceinline__ int page_at(const PageTable &t, int s, int column)
{
    if (column >= t.columns) return -1;
    const int p = t.table[s * t.ldt + column];
    return (uint32_t)p < (uint32_t)t.pages ? p : -1;
}

// The last sequence whose start(s) is at most `u`, where start ascends from at most u: a lane looks at up to four at a time, so
// that 256 sequences cost one trip to memory.
template <typename Start>
__device__ __forceinline__ int find_sequence(int sequences, int u, Start &&start)
{
    constexpr int kEach = 4;
    const int lane = threadIdx.x & (kWave - 1);
    int from = 0, n = sequences;
    while (n > 1) {
        const int step = n <= kWave * kEach ? 1 : (n + kWave * kEach - 1) / (kWave * kEach);
        int last = 0;
        bool at_most[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = (j * kWave + lane) * step;
            at_most[j] = i < n && start(from + i) <= u;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint64_t b = __ballot(at_most[j]);
            if (b) last = (j * kWave + 63 - __builtin_clzll(b)) * step;
        }
        from += last;
        n = min(step, n - last);
    }
    return __builtin_amdgcn_readfirstlane(from);
}

// The scale that a byte stands for, as the conversions from 8 bits take it
__device__ __forceinline__ float scale_of(int b) { return __builtin_bit_cast(float, b == kNoNumber ? 0x7fc00000u : (uint32_t)b << 23); }

// Four e4m3 values of a register as fp32
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float (&v)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
}

// Host side: what both operators check of the cache
struct CacheShape {
    int64_t tokens, sequences, q_heads, kv_heads, head_dim, pages, page_size, columns, ldt;
};
inline bool cache_shape_ok(const CacheShape &c)
{
    if (c.tokens < 1 || c.tokens > kMaxTokens || c.sequences < 1 || c.sequences > kMaxSequences) return false;
    if (c.kv_heads < 1 || c.q_heads < 1 || c.q_heads > kMaxHeads || c.q_heads % c.kv_heads) return false;
    if (c.head_dim < 1 || c.pages < 1 || c.pages > kMaxExtent8 || c.page_size < 1 || c.page_size > kMaxPosition) return false;
    if (c.columns < 1 || c.columns > kMaxPosition / c.page_size || c.ldt < c.columns) return false;
    return addressable(c.sequences, c.ldt);
}
inline bool cache_supported(const CacheShape &c)
{
    const bool dim = c.head_dim == 64 || c.head_dim == 128 || c.head_dim == 256;
    const bool page = c.page_size >= 16 && c.page_size <= 256 && (c.page_size & (c.page_size - 1)) == 0;
    return dim && page;
}

}  // namespace perf
