// 8-bit floating point shared by the quantiser, the norms and the block-scaled product: the OCP formats e4m3 (largest
// value 448, no infinities) and e5m2 (largest finite value 57344), blocks of 128 elements with one fp32 scale, and
// groups of 8 elements of a row as a lane holds them.
#pragma once
#include "row_io.h"

namespace perf {

constexpr int kBlock8 = 128;  // elements of a row that share a scale

typedef uint32_t uint4_at1 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t uint4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uint2_at1 __attribute__((ext_vector_type(2), aligned(1)));

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

// Largest of an unsigned value over groups of 8 or 16 neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
    return v > o ? v : o;
}
template <int LANES>
__device__ __forceinline__ uint32_t group_max_u32(uint32_t v)
{
    static_assert(LANES == 8 || LANES == 16, "a DPP row or half of one");
    v = dpp_max_u32<0xB1>(v);   // quad_perm [1,0,3,2]
    v = dpp_max_u32<0x4E>(v);   // quad_perm [2,3,0,1]
    v = dpp_max_u32<0x141>(v);  // row_half_mirror
    if constexpr (LANES == 16) v = dpp_max_u32<0x140>(v);  // row_mirror
    return v;
}

// Eight neighbouring elements of a row, n of them inside it (the others read as zero and are not written).  Any alignment
// of the elements; only the lane with the ragged end takes the element loop.
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
    uint4_t raw;
    __device__ __forceinline__ void clear() { raw = uint4_t{0, 0, 0, 0}; }
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
    __device__ __forceinline__ void keep(bool in)  // or zeros
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[e] = in ? raw[e] : 0u;
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
    __device__ __forceinline__ void get(float (&v)[8]) const { Elem<uint16_t>::unpack(raw, v); }
    __device__ __forceinline__ void get_half(int q, float (&v)[4]) const  // elements 4q .. 4q + 3
    {
        const uint32_t a = raw[2 * q], b = raw[2 * q + 1];
        v[0] = bf16_lo(a), v[1] = bf16_hi(a), v[2] = bf16_lo(b), v[3] = bf16_hi(b);
    }
};
template <> struct Eight<float> {
    uint4_t lo, hi;
    __device__ __forceinline__ void clear() { lo = hi = uint4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w = lo[e], v = hi[e];
            asm("" : "+v"(w), "+v"(v));
            lo[e] = w, hi[e] = v;
        }
    }
    __device__ __forceinline__ void keep(bool in)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) lo[e] = in ? lo[e] : 0u, hi[e] = in ? hi[e] : 0u;
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
    return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(row) + (uint32_t)c * (uint32_t)sizeof(T));
}

// A group of a row at element c, n = cols - c: RAG takes any number of columns; without it there are whole groups only, and
// one behind the row's end loads the row's first instead, to be masked later: a load on one of two paths of a loop would
// make the compiler wait for all that are in flight.
template <bool RAG, typename T>
__device__ __forceinline__ void load_group(Eight<T> &g, const T *row, int c, int n)
{
    if constexpr (RAG)
        g.load(row + c, n);
    else
        g.load(offset_by(row, n > 0 ? c : 0), 8);
}
// ... and its way back: nothing is written of what lies behind the row's end
template <bool RAG, typename T>
__device__ __forceinline__ void store_group(T *row, const float (&v)[8], int c, int n)
{
    if constexpr (RAG) {
        store_eight(row + c, v, n);
    } else {
        if (n > 0) store_row_chunk<true, T, 8>(offset_by(row, c), v);
    }
}
// ... as fp32, zeros unless `in`
template <typename T>
__device__ __forceinline__ void get_group(const Eight<T> &g, float (&v)[8], bool in)
{
    g.get(v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = in ? v[e] : 0.f;
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

// Magnitude bits of a value as they are compared for a block's largest
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

}  // namespace perf
