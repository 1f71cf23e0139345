// 8-bit floating point shared by the quantiser, the norms and the block-scaled product: the OCP formats e4m3 (largest
// value 448, no infinities) and e5m2 (largest finite value 57344), blocks of 128 elements with one fp32 scale, and
// groups of 8 elements of a row as a lane holds them.
#pragma once
#include <type_traits>
#include "row_io.h"

namespace perf {

constexpr int kBlock8 = 128;  // elements of a row that share a scale

typedef uint32_t uint4_at1 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t uint4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uint2_at1 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t uint32_at1 __attribute__((aligned(1)));

template <bool E5M2> struct Fp8 {
    static constexpr float kLargest = E5M2 ? 57344.f : 448.f;
    // four values in a register, each rounded to nearest even; a NaN stays one
    __device__ static __forceinline__ uint32_t pack(float a, float b, float c, float d)
    {
        if constexpr (E5M2) {
            const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, lo, true);
        } else {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
        }
    }
    // The scale of a block whose largest magnitude has the bits `amax`: amax / largest, and no less than the least normal
    // number, so that its reciprocal is finite.  Magnitudes are compared as integers, which puts infinities and NaN above
    // all numbers: their block gets a scale that is no number (an infinite scale with values of zero and NaN reads back as
    // NaN), so that an overflow is seen behind a product and not lost.
    __device__ static __forceinline__ float scale(uint32_t amax)
    {
        const float s = __builtin_bit_cast(float, amax) / kLargest;
        return s < 0x1p-126f ? 0x1p-126f : s;  // (false for NaN)
    }
};

// Largest of an unsigned value over groups of 8, 16 or 32 neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);  // (all lanes have a source)
    return v > o ? v : o;
}
template <int LANES>
__device__ __forceinline__ uint32_t group_max_u32(uint32_t v)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32, "half a DPP row, one, or two");
    v = dpp_max_u32<0xB1>(v);   // quad_perm [1,0,3,2]
    v = dpp_max_u32<0x4E>(v);   // quad_perm [2,3,0,1]
    v = dpp_max_u32<0x141>(v);  // row_half_mirror
    if constexpr (LANES >= 16) v = dpp_max_u32<0x140>(v);  // row_mirror
    if constexpr (LANES == 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        const uint32_t p0 = p[0], p1 = p[1];
        v = max(p0, p1);
    }
    return v;
}

// Eight neighbouring elements of a row, n of them inside it (the others read as zero and are not written).  Any alignment
// of the elements; only the lane with the ragged end takes the element loop.
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
    uint4_t raw;
    // makes the compiler take the elements for new ones: it then unpacks them again and does not keep what it unpacked before
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w = raw[e];
            asm("" : "+v"(w));
            raw[e] = w;
        }
    }
    __device__ __forceinline__ void load(const uint16_t *p, int n)  // (read once: past the caches)
    {
        if (n >= 8)
            raw = __builtin_nontemporal_load(reinterpret_cast<const uint4_at2 *>(p));
        else
            load_ragged(p, n);
    }
    __device__ __forceinline__ void load_cached(const uint16_t *p, int n)
    {
        if (n >= 8)
            raw = *reinterpret_cast<const uint4_at2 *>(p);
        else
            load_ragged(p, n);
    }
    __device__ __forceinline__ void load_ragged(const uint16_t *p, int n)
    {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        raw = uint4_t{w[0], w[1], w[2], w[3]};
    }
    // columns in runs, one here, two `far` apart in fp32 (read once); or columns c on, those behind `last` as that one
    __device__ __forceinline__ void load_runs(const uint16_t *p, int) { load(p, 8); }
    __device__ __forceinline__ void load_runs(const uint16_t *row, int c, int, int last)
    {
#pragma unroll
        for (int e = 0; e < 8; e += 2) raw[e >> 1] = (uint32_t)row[min(c + e + 1, last)] << 16 | row[min(c + e, last)];
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { Elem<uint16_t>::unpack(raw, v); }
    __device__ __forceinline__ float one(int e) const { return e & 1 ? bf16_hi(raw[e >> 1]) : bf16_lo(raw[e >> 1]); }
    __device__ __forceinline__ void get_half(int q, float (&v)[4]) const  // elements 4q .. 4q + 3
    {
        const uint32_t a = raw[2 * q], b = raw[2 * q + 1];
        v[0] = bf16_lo(a), v[1] = bf16_hi(a), v[2] = bf16_lo(b), v[3] = bf16_hi(b);
    }
};
template <> struct Eight<float> {
    uint4_t lo, hi;
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w = lo[e], v = hi[e];
            asm("" : "+v"(w), "+v"(v));
            lo[e] = w, hi[e] = v;
        }
    }
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= 8) {
            lo = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(p));
            hi = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(p) + 1);
        } else {
            load_ragged(p, n);
        }
    }
    __device__ __forceinline__ void load_cached(const float *p, int n)
    {
        if (n >= 8) {
            lo = *reinterpret_cast<const uint4_at4 *>(p);
            hi = *(reinterpret_cast<const uint4_at4 *>(p) + 1);
        } else {
            load_ragged(p, n);
        }
    }
    __device__ __forceinline__ void load_ragged(const float *p, int n)
    {
        uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e] = reinterpret_cast<const uint32_t *>(p)[e];
        lo = uint4_t{w[0], w[1], w[2], w[3]};
        hi = uint4_t{w[4], w[5], w[6], w[7]};
    }
    __device__ __forceinline__ void load_runs(const float *p, int far)
    {
        lo = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(p));
        hi = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(p + far));
    }
    __device__ __forceinline__ void load_runs(const float *row, int c, int far, int last)
    {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(row);
#pragma unroll
        for (int e = 0; e < 4; ++e) lo[e] = w[min(c + e, last)], hi[e] = w[min(c + far + e, last)];
    }
    __device__ __forceinline__ float one(int e) const { return __builtin_bit_cast(float, (uint32_t)(e < 4 ? lo[e & 3] : hi[e & 3])); }
    __device__ __forceinline__ void get_half(int q, float (&v)[4]) const { Elem<float>::unpack(q ? hi : lo, v); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        Elem<float>::unpack(lo, v);
        Elem<float>::unpack(hi, v + 4);
    }
};

template <typename T>
__device__ __forceinline__ void store_eight(T *p, const float (&v)[8], int n)
{
    if (n >= 8) {
        store_row_chunk<true, T, 8>(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) Elem<T>::store1(p + e, v[e]);
    }
}

// Element c >= 0 of a row that is the same for a wave: a scalar base and an unsigned 32-bit offset are one address operand
template <typename T>
__device__ __forceinline__ T *offset_by(T *row, int c)
{
    using Byte = std::conditional_t<std::is_const_v<T>, const char, char>;
    return reinterpret_cast<T *>(reinterpret_cast<Byte *>(row) + (uint32_t)c * (uint32_t)sizeof(T));
}

// N bytes (8 or 16), n of them inside the row, at any address
template <int N>
__device__ __forceinline__ void store_bytes(uint8_t *p, const uint32_t (&w)[N / 4], int n)
{
    if (n >= N) {
        if constexpr (N == 16)
            *reinterpret_cast<uint4_at1 *>(p) = uint4_t{w[0], w[1], w[2], w[3]};
        else
            *reinterpret_cast<uint2_at1 *>(p) = uint2_t{w[0], w[1]};
    } else {
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
            if (e < n) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
    }
}

// Where a lane's eight elements lie in rows of at least eight: one run of eight (bf16) or two of four (fp32, so that a load
// of a wave is one run of memory), the runs of `threads` lanes side by side.  The run that would overhang the row (RAG)
// starts as many elements before its end instead; its first `dup` elements are its neighbour's too: computed by both, left out
// of sums over the row and stored by the neighbour.  Runs behind the row load others' elements and drop them: a load on one
// of two paths of a loop would make the compiler wait for all that are in flight.
template <typename T, bool RAG> struct Group {
    static constexpr int kRuns = sizeof(T) / 2, kRun = 8 / kRuns;
    int at[kRuns], dup[kRuns];
    Group() = default;
    __device__ __forceinline__ Group(int lane, int threads, int cols)
    {
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            const int c = kRun * (lane + r * threads);
            at[r] = RAG ? min(c, cols - kRun) : c < cols ? c : 0;
            dup[r] = RAG ? c - at[r] : c < cols ? 0 : kRun;
        }
    }
    __device__ __forceinline__ bool in(int e) const { return dup[e / kRun] < kRun; }  // whether the run of element e is in the row
    __device__ __forceinline__ float once(int e, float v) const { return !RAG || e % kRun >= dup[e / kRun] ? v : 0.f; }
    __device__ __forceinline__ void load(Eight<T> &g, const T *row) const  // (read once: past the caches)
    {
        if constexpr (kRuns == 1) {
            g.raw = __builtin_nontemporal_load(reinterpret_cast<const uint4_at2 *>(offset_by(row, at[0])));
        } else {
            g.lo = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(offset_by(row, at[0])));
            g.hi = __builtin_nontemporal_load(reinterpret_cast<const uint4_at4 *>(offset_by(row, at[1])));
        }
    }
    __device__ __forceinline__ void keep(Eight<T> &g, bool in_row) const  // or zeros
    {
        if constexpr (kRuns == 1)
            g.raw = in_row && in(0) ? g.raw : uint4_t{0, 0, 0, 0};
        else
            g.lo = in_row && in(0) ? g.lo : uint4_t{0, 0, 0, 0}, g.hi = in_row && in(4) ? g.hi : uint4_t{0, 0, 0, 0};
    }
    // the same elements of another row, of any type, as fp32; zeros behind the row's end
    template <typename P>
    __device__ __forceinline__ void load_as(const P *row, float (&v)[8]) const
    {
        typedef P Some __attribute__((ext_vector_type(kRun), aligned(sizeof(P))));
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            const Some w = *reinterpret_cast<const Some *>(offset_by(row, at[r]));
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                const P one = w[e];
                v[kRun * r + e] = in(kRun * r) ? Elem<P>::load1(&one) : 0.f;
            }
        }
    }
    template <typename P>
    __device__ __forceinline__ void store(P *row, const float (&v)[8]) const
    {
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            P *p = offset_by(row, at[r]);
            const float *f = v + kRun * r;
            if (dup[r] == 0) {
                store_row_chunk<true, P, kRun>(p, f);
            } else if constexpr (RAG) {
#pragma unroll
                for (int e = 1; e < kRun; ++e)
                    if (e >= dup[r]) Elem<P>::store1(p + e, f[e]);
            }
        }
    }
    // fp32 that this lane reads again
    __device__ __forceinline__ void store_cached(float *row, const float (&v)[8]) const
    {
#pragma unroll
        for (int r = 0; r < kRuns; ++r)
#pragma unroll
            for (int e = 0; e < kRun; ++e)
                if (dup[r] <= (RAG ? e : 0)) offset_by(row, at[r])[e] = v[kRun * r + e];
    }
    // the eight as bytes w
    __device__ __forceinline__ void store_bytes(uint8_t *row, const uint32_t (&w)[2]) const
    {
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            uint8_t *p = offset_by(row, at[r]);
            if (dup[r] == 0) {
                if constexpr (kRun == 8)
                    *reinterpret_cast<uint2_at1 *>(p) = uint2_t{w[0], w[1]};
                else
                    *reinterpret_cast<uint32_at1 *>(p) = w[r];
            } else if constexpr (RAG) {
#pragma unroll
                for (int e = 1; e < kRun; ++e)
                    if (e >= dup[r]) p[e] = (uint8_t)(w[(kRun * r + e) >> 2] >> (8 * (e & 3)));
            }
        }
    }
};

// Magnitude bits of a value as they are compared for a block's largest
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

}  // namespace perf
