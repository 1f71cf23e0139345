// The RMS norms before and after a block of a network, joined with the block's gate and the scaled residual:
//     n = u r1 gamma_post,   h = residual_scale x + gate n,   y = h r2 gamma_pre,
//     r1 = (mean u^2 + eps)^(-1/2),   r2 = (mean h^2 + eps)^(-1/2),
// u the block's output, x the residual stream before it, h the stream behind it, y the next block's input, in x's type or
// in 8 bits with a scale for each 128 elements.  And the gradient: with t = dy gamma_pre, hn = h r2, un = u r1,
//     H = dh + r2 (t - hn mean(t hn)),   dx = residual_scale H,    dgamma_pre = sum over rows of dy hn,
//     D = gate H,  v = D gamma_post,     du = r1 (v - un mean(v un)),  dgamma_post = sum of D un,  dgate = sum of n H.
// (gamma_post left out: n = u, du = D.)  Bound by HBM: each operand is read once and each result written once.
//
//  * residual_norm_kernel / residual_norm_grad_kernel<W, NC>: W waves own a row, NC groups of 8 elements per lane, so that
//    a row is in registers between its two sums; 8 / W rows side by side in a workgroup of 8 waves.  The gains and the
//    gate stay in registers for all rows that share them.
//  * The gradient's sums over rows: a workgroup owns a run of rows and sums them in registers; its sums go to the
//    workspace and are added in the order of the rows by residual_norm_sums_kernel.  No atomics.
//  * residual_norm_any_kernel and its gradient: rows beyond 16 waves' registers, several passes over memory.
// Statistics, h on its way into y, and all sums are fp32; y is computed from h before it is rounded to its type.
#include "fp8.h"
#include "host_utils.h"

namespace perf {

// A vector of parameters of either type, element j at p + j (PERF_F32 or PERF_BF16: the same for a whole launch).
struct Param {
    const void *p;
    int bf16;
    __device__ __forceinline__ float at(int64_t j) const
    {
        return bf16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(p)[j]) : reinterpret_cast<const float *>(p)[j];
    }
    // n of the eight elements from j on, the others zero; RAG as for rows
    template <bool RAG = true>
    __device__ __forceinline__ void eight(int64_t j, int n, float (&v)[8]) const
    {
        if constexpr (!RAG) j = n > 0 ? j : 0, n = n > 0 ? 8 : 0;
        if (bf16) {
            Eight<uint16_t> e;
            e.load_cached(reinterpret_cast<const uint16_t *>(p) + j, RAG ? n : 8);
            get_group(e, v, RAG || n > 0);
        } else {
            Eight<float> e;
            e.load_cached(reinterpret_cast<const float *>(p) + j, RAG ? n : 8);
            get_group(e, v, RAG || n > 0);
        }
    }
    __device__ __forceinline__ void four(int64_t j, int n, float (&v)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < n ? at(j + e) : 0.f;
    }
    __device__ __forceinline__ void put(int64_t j, float v) const
    {
        if (bf16)
            reinterpret_cast<uint16_t *>(const_cast<void *>(p))[j] = f32_to_bf16(v);
        else
            reinterpret_cast<float *>(const_cast<void *>(p))[j] = v;
    }
    template <bool RAG>
    __device__ __forceinline__ void put_eight(int64_t at, const float (&v)[8], int c, int n) const
    {
        if (bf16)
            store_group<RAG>(reinterpret_cast<uint16_t *>(const_cast<void *>(p)) + at, v, c, n);
        else
            store_group<RAG>(reinterpret_cast<float *>(const_cast<void *>(p)) + at, v, c, n);
    }
};

struct NormArgs {
    const void *u, *x;
    Param gate, post, pre;  // p is null where there is none
    void *h, *y;
    float *y_scales, *r_post, *r_pre;
    int64_t rows, ldu, ldx, ldg, gate_rows, ldh, ldy, lds;
    int cols;
    float residual_scale, eps;
};

// Sum over the W waves of a team, the same in all of them.  `red` has a float for each wave of the workgroup; two arrays
// that are used in turn need one barrier each: a wave writes one again only behind the barrier of the other.
template <int W>
__device__ __forceinline__ float team_sum(float v, float *red)
{
    v = wave_allreduce(v, OpSum{});
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        const float *team = red + wave / W * W;
        v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += team[w];
    }
    return v;
}

// Y8: y is e4m3 with scales (else of x's type)
template <typename T, int W, int NC, bool Y8, bool RAG>
__global__ __launch_bounds__(W > 8 ? 64 * W : 512) void residual_norm_kernel(const NormArgs a)
{
    constexpr int kWaves = W > 8 ? W : 8, kTeams = kWaves / W, kThreads = 64 * W;
    __shared__ float red[2][kWaves];
    // (the same in all lanes of a wave: rows and their addresses are scalars)
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / W, lane = threadIdx.x - team * kThreads;
    const float inv_cols = 1.0f / (float)a.cols;
    int n[NC];  // elements of group k inside the row
    float post[NC][8], pre[NC][8], gate[NC][8];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int c = 8 * (k * kThreads + lane);
        n[k] = a.cols - c;
#pragma unroll
        for (int e = 0; e < 8; ++e) post[k][e] = pre[k][e] = gate[k][e] = 1.f;
        if (a.post.p) a.post.template eight<RAG>(c, n[k], post[k]);
        if (a.pre.p) a.pre.template eight<RAG>(c, n[k], pre[k]);
    }
    int64_t held = -1;  // the group of rows whose gate is in `gate`
    const int64_t step = (int64_t)gridDim.x * kTeams;
    Eight<T> u[NC], x[NC];
    auto load = [&](int64_t r) {
        r = min(r, a.rows - 1);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const int c = 8 * (k * kThreads + lane);
            load_group<RAG>(u[k], (const T *)a.u + r * a.ldu, c, n[k]);
            load_group<RAG>(x[k], (const T *)a.x + r * a.ldx, c, n[k]);
        }
    };
    // teams of a workgroup take neighbouring rows and run the same number of rounds: its barriers are met by all
    int64_t row = (int64_t)blockIdx.x * kTeams + team;
    load(row);
    for (int64_t first = (int64_t)blockIdx.x * kTeams; first < a.rows; first += step, row += step) {
        const bool live = row < a.rows;
        if (a.gate.p && live) {
            const int64_t g = a.gate_rows == 1 ? row : row / a.gate_rows;
            if (g != held) {
#pragma unroll
                for (int k = 0; k < NC; ++k) a.gate.template eight<RAG>(g * a.ldg + 8 * (k * kThreads + lane), n[k], gate[k]);
                held = g;
            }
        }
        float v[NC][8], h[NC][8], s = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            get_group(u[k], v[k], n[k] > 0);
            get_group(x[k], h[k], n[k] > 0);
        }
        load(row + step);  // the next row's loads fly during this row's sums
        if (a.post.p) {
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) s = __builtin_fmaf(v[k][e], v[k][e], s);
            s = team_sum<W>(s, red[0]);
            const float r1 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
            if (live && lane == 0 && a.r_post) a.r_post[row] = r1;
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] *= r1 * post[k][e];
        } else if (W > 1) {
            __syncthreads();  // the one sum's array is written again in the next round
        }
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[k][e] = __builtin_fmaf(gate[k][e], v[k][e], a.residual_scale * h[k][e]);
                s = __builtin_fmaf(h[k][e], h[k][e], s);
            }
        if (a.h && live) {
#pragma unroll
            for (int k = 0; k < NC; ++k) store_group<RAG>((T *)a.h + row * a.ldh, h[k], 8 * (k * kThreads + lane), n[k]);
        }
        if (!a.y) {
            if (W > 1) __syncthreads();  // the first sums' array is written again in the next round
            continue;
        }
        s = team_sum<W>(s, red[1]);
        const float r2 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
        if (live && lane == 0 && a.r_pre) a.r_pre[row] = r2;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const int c = 8 * (k * kThreads + lane);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h[k][e] * r2 * pre[k][e];
            if constexpr (!Y8) {
                if (live) store_group<RAG>((T *)a.y + row * a.ldy, y, c, n[k]);
            } else {
                using F = Fp8<false>;
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, n[k] > e ? magnitude(y[e]) : 0u);
                const float q = F::scale(group_max_u32<16>(m)), inv = 1.0f / q;  // sixteen lanes hold a block
                const uint32_t w[2] = {F::pack(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                                       F::pack(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
                if (live) {
                    store_bytes<8>((uint8_t *)a.y + row * a.ldy + c, w, n[k]);
                    if ((lane & 15) == 0 && n[k] > 0) a.y_scales[row * a.lds + c / kBlock8] = q;
                }
            }
        }
    }
}

// Rows of any length: a workgroup per row, three passes.  What a pass needs of an earlier one is computed again from u and
// x, so that h and y may take the place of either: an element is read for the last time by the lane that writes it.
template <typename T, bool Y8>
__global__ __launch_bounds__(1024) void residual_norm_any_kernel(const NormArgs a)
{
    __shared__ float red[2][16];
    const float inv_cols = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *u = (const T *)a.u + row * a.ldu, *x = (const T *)a.x + row * a.ldx;
        const int64_t g = a.gate.p ? row / a.gate_rows * a.ldg : 0;
        const int end = (a.cols + kBlock8 - 1) / kBlock8 * kBlock8;  // whole blocks: their lanes take part in the maximum
        float s = 0.f, r1 = 1.f;
        if (a.post.p) {
            for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * 1024) {
                Eight<T> raw;
                float v[8];
                raw.load_cached(u + c, a.cols - c);
                raw.get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = __builtin_fmaf(v[e], v[e], s);
            }
        }
        s = team_sum<16>(s, red[0]);
        if (a.post.p) {
            r1 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
            if (threadIdx.x == 0 && a.r_post) a.r_post[row] = r1;
        }
        auto stream = [&](int c, float (&h)[8]) {
            const int n = a.cols - c;
            Eight<T> raw;
            float v[8], p[8], gate[8];
            raw.load_cached(u + c, n);
            raw.get(v);
            raw.load_cached(x + c, n);
            raw.get(h);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = gate[e] = 1.f;
            if (a.post.p) {
                a.post.eight(c, n, p);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= r1 * p[e];
            }
            if (a.gate.p) a.gate.eight(g + c, n, gate);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = __builtin_fmaf(gate[e], v[e], a.residual_scale * h[e]);
        };
        s = 0.f;
        if (a.y) {
            for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * 1024) {
                float h[8];
                stream(c, h);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = __builtin_fmaf(h[e], h[e], s);
            }
        }
        s = team_sum<16>(s, red[1]);
        const float r2 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
        if (a.y && threadIdx.x == 0 && a.r_pre) a.r_pre[row] = r2;
        for (int c = 8 * threadIdx.x; c < end; c += 8 * 1024) {
            const int n = a.cols - c;
            float h[8], y[8], pre[8];
            stream(c, h);
            if (a.h) store_eight((T *)a.h + row * a.ldh + c, h, n);
            if (!a.y) continue;
            a.pre.eight(c, n, pre);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h[e] * r2 * pre[e];
            if constexpr (!Y8) {
                store_eight((T *)a.y + row * a.ldy + c, y, n);
            } else {
                using F = Fp8<false>;
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, n > e ? magnitude(y[e]) : 0u);
                const float q = F::scale(group_max_u32<16>(m)), inv = 1.0f / q;
                const uint32_t w[2] = {F::pack(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                                       F::pack(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
                store_bytes<8>((uint8_t *)a.y + row * a.ldy + c, w, n);
                if ((threadIdx.x & 15) == 0) a.y_scales[row * a.lds + c / kBlock8] = q;
            }
        }
    }
}

// ---- gradient ------------------------------------------------------------------------------------------------------
struct GradArgs {
    const void *dy, *dh, *h, *u;  // one that is not given has u's place (and row stride): it is loaded like the others and dropped
    bool has_dy, has_dh;
    Param gate, post, pre;
    const float *r_post, *r_pre;
    void *dx, *du;
    Param dgate;  // p is null where it is not asked for
    float *dpost, *dpre;
    float *ws;  // [2 runs][cols] sums of dgamma_pre and dgamma_post, then [2 runs][cols] of dgate
    int64_t rows, lddy, lddh, ldh, ldu, ldg, gate_rows, lddx, lddu, lddg;
    int64_t run;  // rows of a workgroup
    int runs, cols;
    bool whole_groups;  // runs are whole groups of gate rows, and a team takes a group by itself
    float residual_scale;
};

// Where a workgroup's sum of a gate's gradient goes: a group that lies within its run straight to the result; of a group
// that goes on beyond it, slot 2 run + 1 (it begins here) or 2 run (it began before).
__device__ __forceinline__ float *gate_slot(const GradArgs &a, int64_t run, bool begins)
{
    return a.ws + (2 * (int64_t)a.runs + 2 * run + (begins ? 1 : 0)) * a.cols;
}

// A row stays in registers as it came and is unpacked for each of its three uses; the gains and the gate lie in LDS, every
// lane's own where it alone reads them (for rows of two groups per lane, which leave no room there, in the caches), and so do
// two of the three sums of such rows.  With all of it in registers the kernel spilled 50 to 300 of them per lane.
template <typename T, int W, int NC, bool RAG>
__global__ __launch_bounds__(W > 8 ? 64 * W : 512, W <= 8 ? 2 : 4) void residual_norm_grad_kernel(const GradArgs a)
{
    constexpr int kWaves = W > 8 ? W : 8, kTeams = kWaves / W, kThreads = 64 * W, kAll = 64 * kWaves;
    constexpr bool kWide = NC > 1;
    __shared__ float red[2][kWaves];
    __shared__ float joined[kTeams > 1 ? kAll * 8 : 1];
    __shared__ float4_t own[kWide ? 2 : 3][2 * NC][kAll];  // gamma_post, gamma_pre, gate; of wide rows the sums of post and gate
    const int tid = threadIdx.x, team = __builtin_amdgcn_readfirstlane(tid >> 6) / W, lane = tid - team * kThreads;
    const float inv_cols = 1.0f / (float)a.cols;
    const bool has_post = a.post.p != nullptr, has_gate = a.gate.p != nullptr;
    auto col = [&](int k) { return 8 * (k * kThreads + lane); };
    auto get_own = [&](int which, int k, int q, float (&v)[4]) {
        const float4_t f = own[which][2 * k + q][tid];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = f[e];
    };
    auto put_own = [&](int which, int k, int q, const float (&v)[4]) { own[which][2 * k + q][tid] = float4_t{v[0], v[1], v[2], v[3]}; };
    auto get_own8 = [&](int which, int k, float (&v)[8]) {
        float lo[4], hi[4];
        get_own(which, k, 0, lo), get_own(which, k, 1, hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = lo[e], v[4 + e] = hi[e];
    };
    auto put_own8 = [&](int which, int k, const float (&v)[8]) {
        const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
        put_own(which, k, 0, lo), put_own(which, k, 1, hi);
    };
    int64_t g = 0;  // the group of rows whose gate is in use
    auto param = [&](int which, int k, int q, float (&v)[4]) {
        if constexpr (!kWide) {
            get_own(which, k, q, v);
        } else {
            const Param &p = which == 0 ? a.post : which == 1 ? a.pre : a.gate;
            const bool has = which == 0 ? has_post : which == 1 ? a.has_dy : has_gate;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = 1.f;
            if (has) p.four((which == 2 ? g * a.ldg : 0) + col(k) + 4 * q, a.cols - col(k) - 4 * q, v);
        }
    };
    float sum_pre[NC][8], sum_post[kWide ? 1 : NC][8], sum_gate[kWide ? 1 : NC][8];
    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto clear_gate_sum = [&]() {
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            if constexpr (kWide) {
                put_own8(1, k, zeros);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum_gate[k][e] = 0.f;
            }
        }
    };
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum_pre[k][e] = 0.f;
        if constexpr (kWide) {
            put_own8(0, k, zeros);
        } else {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 1.f, sum_post[k][e] = 0.f;
            put_own8(2, k, v);
            if (has_post) a.post.template eight<RAG>(col(k), a.cols - col(k), v);
            put_own8(0, k, v);
            if (a.has_dy) a.pre.template eight<RAG>(col(k), a.cols - col(k), v);
            put_own8(1, k, v);
        }
    }

    Eight<T> dy[NC], dh[NC], h[NC], u[NC], next_dy[NC], next_dh[NC], next_h[NC], next_u[NC];
    auto load = [&](int64_t r) {
        r = min(r, a.rows - 1);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const int c = col(k), n = a.cols - c;
            load_group<RAG>(next_dy[k], (const T *)a.dy + r * a.lddy, c, n);
            load_group<RAG>(next_h[k], (const T *)a.h + r * a.ldh, c, n);
            load_group<RAG>(next_dh[k], (const T *)a.dh + r * a.lddh, c, n);
            load_group<RAG>(next_u[k], (const T *)a.u + r * a.ldu, c, n);
        }
    };
    // one row of this team (a dead one adds nothing and writes nothing); `next` is loaded meanwhile
    auto one = [&](int64_t row, bool live, int64_t next) {
        const float r2 = a.has_dy && live ? a.r_pre[row] : 0.f, r1 = !has_post ? 1.f : live ? a.r_post[row] : 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const bool in = live && a.cols > col(k);
            dy[k] = next_dy[k], h[k] = next_h[k], dh[k] = next_dh[k], u[k] = next_u[k];
            dy[k].keep(in && a.has_dy), h[k].keep(in && a.has_dy), dh[k].keep(in && a.has_dh), u[k].keep(in);
        }
        load(next);
        float s = 0.f;
        if (a.has_dy) {
#pragma unroll
            for (int k = 0; k < NC; ++k) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float t[4], hn[4], pre[4];
                    dy[k].get_half(q, t), h[k].get_half(q, hn), param(1, k, q, pre);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hn[e] *= r2;
                        sum_pre[k][4 * q + e] = __builtin_fmaf(t[e], hn[e], sum_pre[k][4 * q + e]);
                        s = __builtin_fmaf(t[e] * pre[e], hn[e], s);
                    }
                    __builtin_amdgcn_sched_barrier(0);  // (reads of the next half's operands ahead of here cost registers)
                }
            }
            s = team_sum<W>(s, red[0]);
        } else if (W > 1) {
            __syncthreads();  // the one sum's array is written again in the next row
        }
        const float mean2 = s * inv_cols;
        auto into_h = [&](int k, int q, float (&H)[4]) {
            float t[4], hn[4], pre[4];
            dy[k].get_half(q, t), h[k].get_half(q, hn), dh[k].get_half(q, H), param(1, k, q, pre);
#pragma unroll
            for (int e = 0; e < 4; ++e) H[e] = __builtin_fmaf(r2, t[e] * pre[e] - hn[e] * r2 * mean2, H[e]);
        };
        auto renew = [&]() {
#pragma unroll
            for (int k = 0; k < NC; ++k) dy[k].renew(), h[k].renew(), dh[k].renew(), u[k].renew();
        };
        renew();
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float dx[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float H[4], un[4], post[4], gate[4], more_post[4], more_gate[4];
                into_h(k, q, H);
                u[k].get_half(q, un), param(0, k, q, post), param(2, k, q, gate);
                if constexpr (kWide) get_own(0, k, q, more_post), get_own(1, k, q, more_gate);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    un[e] *= r1;
                    const float d = H[e] * gate[e];
                    float &to_post = kWide ? more_post[e] : sum_post[kWide ? 0 : k][4 * q + e];
                    float &to_gate = kWide ? more_gate[e] : sum_gate[kWide ? 0 : k][4 * q + e];
                    to_post = __builtin_fmaf(d, un[e], to_post);
                    to_gate = __builtin_fmaf(un[e] * post[e], H[e], to_gate);
                    s = __builtin_fmaf(d * post[e], un[e], s);
                    dx[4 * q + e] = a.residual_scale * H[e];
                }
                if constexpr (kWide) put_own(0, k, q, more_post), put_own(1, k, q, more_gate);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (live) store_group<RAG>((T *)a.dx + row * a.lddx, dx, col(k), a.cols - col(k));
        }
        float mean1 = 0.f;
        if (has_post)
            mean1 = team_sum<W>(s, red[1]) * inv_cols;
        else if (W > 1)
            __syncthreads();  // as above
        renew();
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float du[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float H[4], un[4], post[4], gate[4];
                into_h(k, q, H);
                u[k].get_half(q, un), param(0, k, q, post), param(2, k, q, gate);
#pragma unroll
                for (int e = 0; e < 4; ++e) du[4 * q + e] = r1 * (H[e] * gate[e] * post[e] - un[e] * r1 * mean1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (live) store_group<RAG>((T *)a.du + row * a.lddu, du, col(k), a.cols - col(k));
        }
    };
    // the teams' sums v, added in the teams' order; the first team has them
    auto join = [&](float (&v)[8]) {
        if constexpr (kTeams > 1) {
            static_assert(NC == 1, "teams of fewer than eight waves hold one group per lane");
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) joined[e * kAll + tid] = v[e];
            __syncthreads();
            if (team == 0) {
                for (int o = 1; o < kTeams; ++o)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += joined[e * kAll + o * kThreads + lane];
            }
        }
    };

    // Groups of few rows (whole_groups): a team takes every kTeams-th group by itself.  Otherwise the rows of the run that
    // share a gate are dealt to the teams in turn.  All teams run the same number of rounds.
    const int64_t begin = (int64_t)blockIdx.x * a.run, end = min(a.rows, begin + a.run);
    const int64_t per = has_gate ? a.gate_rows : a.rows;
    const bool each = a.whole_groups;
    g = begin / per + (each ? team : 0);
    int64_t row = each ? g * per : begin + team;
    int64_t from = begin;  // the round's first row, the same for all teams
    load(row);
    while (from < end) {
        const int64_t stop = min(end, (g + 1) * per);
        if constexpr (!kWide) {
            if (has_gate && g * per < end) {
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    float v[8];
                    a.gate.template eight<RAG>(g * a.ldg + col(k), a.cols - col(k), v);
                    put_own8(2, k, v);
                }
            }
        }
        clear_gate_sum();
        const int64_t rounds = each ? per : (stop - from + kTeams - 1) / kTeams;
        for (int64_t i = rounds; i > 0; --i) {
            const int64_t next = each ? (i > 1 ? row + 1 : (g + kTeams) * per) : (i > 1 ? row + kTeams : stop + team);
            one(row, row < stop, next);
            row = next;
        }
        if (a.dgate.p) {
            const bool begins = g * per >= begin, ends = min(a.rows, (g + 1) * per) <= end;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                float v[8];
                if constexpr (kWide)
                    get_own8(1, k, v);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = sum_gate[k][e];
                if (!each) join(v);
                if (each ? g * per < end : team == 0) {
                    if (begins && ends)
                        a.dgate.template put_eight<RAG>(g * a.lddg, v, col(k), a.cols - col(k));
                    else
                        store_group<RAG>(gate_slot(a, blockIdx.x, begins), v, col(k), a.cols - col(k));
                }
            }
        }
        g += each ? kTeams : 1;
        from = each ? (g - team) * per : stop;
    }
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        if (a.dpre && a.has_dy) {
            join(sum_pre[k]);
            if (team == 0) store_group<RAG>(a.ws + (int64_t)blockIdx.x * a.cols, sum_pre[k], col(k), a.cols - col(k));
        }
        if (a.dpost) {
            float v[8];
            if constexpr (kWide)
                get_own8(0, k, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = sum_post[k][e];
            join(v);
            if (team == 0) store_group<RAG>(a.ws + ((int64_t)a.runs + blockIdx.x) * a.cols, v, col(k), a.cols - col(k));
        }
    }
}

// The runs' sums, added in the order of the rows.  blockIdx.y: 0 = dgamma_pre, 1 = dgamma_post, 2 + t = the gate of the group
// that begins in run t and goes on beyond it.  64 columns and four parts of the runs per workgroup, the parts added in order.
__global__ __launch_bounds__(256) void residual_norm_sums_kernel(const GradArgs a)
{
    const int64_t col = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int part = threadIdx.x >> 6, which = blockIdx.y;
    const float *from;
    int64_t count, step = a.cols, g = 0;
    __shared__ float parts[3][64];
    const bool in = col < a.cols;
    if (which < 2) {
        float *to = which ? a.dpost : a.dpre;
        if (!to) return;
        from = a.ws + (int64_t)which * a.runs * a.cols;
        count = which == 0 && !a.has_dy ? 0 : a.runs;
    } else {
        const int64_t t = which - 2, last = min(a.rows, (t + 1) * a.run) - 1;
        g = last / a.gate_rows;
        const int64_t begin = g * a.gate_rows, end = min(a.rows, begin + a.gate_rows);
        if (begin < t * a.run || end <= last + 1) return;
        from = nullptr;
        count = (end - 1) / a.run - t + 1;
    }
    const int64_t per = (count + 3) / 4, lo = part * per, hi = min(count, lo + per);
    float s = 0.f;
    if (in) {
        if (from) {
#pragma unroll 8
            for (int64_t i = lo; i < hi; ++i) s += from[i * step + col];
        } else {
            const int64_t t = which - 2;
            for (int64_t i = lo; i < hi; ++i) s += gate_slot(a, t + i, i == 0)[col];
        }
    }
    if (part) parts[part - 1][threadIdx.x & 63] = s;
    __syncthreads();
    if (part || !in) return;
    s = ((s + parts[0][threadIdx.x]) + parts[1][threadIdx.x]) + parts[2][threadIdx.x];
    if (which == 0)
        a.dpre[col] = s;
    else if (which == 1)
        a.dpost[col] = s;
    else
        a.dgate.put(g * a.lddg + col, s);
}

// Rows of any length, in three kernels: every row's mean(t hn) into the workspace; a lane per column, which computes H
// again and sums a run of rows; dx and du, a workgroup per row.  In this order dx and du may take the place of dh and dy.
template <typename T>
__device__ __forceinline__ float grad_into_h(const GradArgs &a, int64_t row, int64_t c, float r2, float mean)
{
    const float dh = a.has_dh ? Elem<T>::load1((const T *)a.dh + row * a.lddh + c) : 0.f;
    if (!a.has_dy) return dh;
    const float t = Elem<T>::load1((const T *)a.dy + row * a.lddy + c) * a.pre.at(c);
    const float hn = Elem<T>::load1((const T *)a.h + row * a.ldh + c) * r2;
    return __builtin_fmaf(r2, t - hn * mean, dh);
}

template <typename T, bool MEANS>
__global__ __launch_bounds__(1024) void residual_norm_grad_any_kernel(const GradArgs a, float *means)
{
    __shared__ float red[1][16];
    const float inv_cols = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float r2 = a.has_dy ? a.r_pre[row] : 0.f, r1 = a.post.p ? a.r_post[row] : 1.f;
        const int64_t g = a.gate.p ? row / a.gate_rows * a.ldg : 0;
        float s = 0.f;
        if constexpr (MEANS) {
            if (a.has_dy) {
                for (int c = threadIdx.x; c < a.cols; c += 1024)
                    s = __builtin_fmaf(Elem<T>::load1((const T *)a.dy + row * a.lddy + c) * a.pre.at(c),
                                       Elem<T>::load1((const T *)a.h + row * a.ldh + c) * r2, s);
            }
            s = team_sum<16>(s, red[0]) * inv_cols;
            if (threadIdx.x == 0) means[row] = s;
            __syncthreads();  // the sum's array is written again for the next row
            continue;
        }
        const float mean = means[row];
        if (a.post.p) {
            for (int c = threadIdx.x; c < a.cols; c += 1024) {
                const float d = grad_into_h<T>(a, row, c, r2, mean) * (a.gate.p ? a.gate.at(g + c) : 1.f);
                s = __builtin_fmaf(d * a.post.at(c), Elem<T>::load1((const T *)a.u + row * a.ldu + c) * r1, s);
            }
        }
        s = team_sum<16>(s, red[0]) * inv_cols;
        __syncthreads();  // ... and this one
        for (int c = threadIdx.x; c < a.cols; c += 1024) {
            const float H = grad_into_h<T>(a, row, c, r2, mean), d = H * (a.gate.p ? a.gate.at(g + c) : 1.f);
            float du = d;
            if (a.post.p) du = r1 * (d * a.post.at(c) - Elem<T>::load1((const T *)a.u + row * a.ldu + c) * r1 * s);
            Elem<T>::store1((T *)a.dx + row * a.lddx + c, a.residual_scale * H);
            Elem<T>::store1((T *)a.du + row * a.lddu + c, du);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void residual_norm_grad_cols_kernel(const GradArgs a, const float *means)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const int64_t begin = (int64_t)blockIdx.y * a.run, end = min(a.rows, begin + a.run);
    const int64_t per = a.gate.p ? a.gate_rows : a.rows;
    const float post = a.post.p ? a.post.at(c) : 1.f;
    float sum_pre = 0.f, sum_post = 0.f;
    for (int64_t from = begin; from < end;) {
        const int64_t g = from / per, to = min(end, (g + 1) * per);
        const float gate = a.gate.p ? a.gate.at(g * a.ldg + c) : 1.f;
        float sum_gate = 0.f;
        for (int64_t row = from; row < to; ++row) {
            const float r2 = a.has_dy ? a.r_pre[row] : 0.f, r1 = a.post.p ? a.r_post[row] : 1.f;
            const float H = grad_into_h<T>(a, row, c, r2, means[row]);
            const float un = Elem<T>::load1((const T *)a.u + row * a.ldu + c) * r1;
            if (a.has_dy)
                sum_pre = __builtin_fmaf(Elem<T>::load1((const T *)a.dy + row * a.lddy + c),
                                         Elem<T>::load1((const T *)a.h + row * a.ldh + c) * r2, sum_pre);
            sum_post = __builtin_fmaf(H * gate, un, sum_post);
            sum_gate = __builtin_fmaf(un * post, H, sum_gate);
        }
        if (a.dgate.p) {
            const bool begins = g * per >= begin, ends = min(a.rows, (g + 1) * per) <= end;
            if (begins && ends)
                a.dgate.put(g * a.lddg + c, sum_gate);
            else
                gate_slot(a, blockIdx.y, begins)[c] = sum_gate;
        }
        from = to;
    }
    if (a.has_dy) a.ws[(int64_t)blockIdx.y * a.cols + c] = sum_pre;
    a.ws[((int64_t)a.runs + blockIdx.y) * a.cols + c] = sum_post;
}

// ---- entry points --------------------------------------------------------------------------------------------------
constexpr int kWidest = 16 * 64 * 8;  // columns that a team of 16 waves holds

// f(waves of a team, groups per lane) for rows of `cols` elements within kWidest
template <typename F>
static void with_team(int64_t cols, F &&f)
{
    using std::integral_constant;
    if (cols <= 512)
        f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    else if (cols <= 1024)
        f(integral_constant<int, 2>{}, integral_constant<int, 1>{});
    else if (cols <= 2048)
        f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (cols <= 4096)
        f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else
        f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
}

template <typename T, bool Y8>
static void launch_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.cols > kWidest) {
        residual_norm_any_kernel<T, Y8><<<(unsigned)std::min<int64_t>(a.rows, 65536), 1024, 0, stream>>>(a);
        return;
    }
    with_team(a.cols, [&](auto w, auto nc) {
        constexpr int W = w, NC = nc, kTeams = W > 8 ? 1 : 8 / W, kThreads = W > 8 ? 1024 : 512;
        const int64_t grid = std::min<int64_t>((a.rows + kTeams - 1) / kTeams, 1024 * 512 / kThreads);
        if (a.cols % 8)
            residual_norm_kernel<T, W, NC, Y8, true><<<(unsigned)grid, kThreads, 0, stream>>>(a);
        else
            residual_norm_kernel<T, W, NC, Y8, false><<<(unsigned)grid, kThreads, 0, stream>>>(a);
    });
}

// Rows of a workgroup's run in the gradient, and whether the runs are whole groups of a gate.
struct RunPlan {
    int64_t run;
    int runs;
    bool whole_groups;
};
static RunPlan plan_runs(int64_t rows, int64_t cols, int64_t gate_rows)
{
    const int64_t teams = cols <= 512 ? 8 : cols <= 1024 ? 4 : cols <= 2048 ? 2 : 1;
    const int64_t most = cols <= 4096 ? 512 : 256;
    RunPlan p;
    p.whole_groups = gate_rows <= 16;
    const int64_t unit = teams * (p.whole_groups ? gate_rows : 1);
    p.run = ((rows + most - 1) / most + unit - 1) / unit * unit;
    p.runs = (int)((rows + p.run - 1) / p.run);
    return p;
}
static int64_t gate_rows_or_all(int64_t gate_rows, int64_t rows) { return gate_rows < 1 || gate_rows > rows ? rows : gate_rows; }

template <typename T>
static void launch_grad(GradArgs a, hipStream_t stream)
{
    if (a.cols > kWidest) {
        float *means = a.ws + 4 * (int64_t)a.runs * a.cols;
        const unsigned grid = (unsigned)std::min<int64_t>(a.rows, 65536);
        residual_norm_grad_any_kernel<T, true><<<grid, 1024, 0, stream>>>(a, means);
        residual_norm_grad_cols_kernel<T><<<dim3((a.cols + 255) / 256, a.runs), 256, 0, stream>>>(a, means);
        residual_norm_grad_any_kernel<T, false><<<grid, 1024, 0, stream>>>(a, means);
    } else {
        with_team(a.cols, [&](auto w, auto nc) {
            constexpr int W = w, NC = nc;
            if (a.cols % 8)
                residual_norm_grad_kernel<T, W, NC, true><<<a.runs, W > 8 ? 1024 : 512, 0, stream>>>(a);
            else
                residual_norm_grad_kernel<T, W, NC, false><<<a.runs, W > 8 ? 1024 : 512, 0, stream>>>(a);
        });
    }
    const unsigned blocks = (unsigned)((a.cols + 63) / 64);
    // (a gate whose groups lie within runs has its sums already)
    const unsigned gates = a.dgate.p && !(a.cols <= kWidest && a.whole_groups) ? a.runs : 0;
    if (a.dpre || a.dpost || gates) residual_norm_sums_kernel<<<dim3(blocks, 2 + gates), 256, 0, stream>>>(a);
}

}  // namespace perf

extern "C" perf_status perf_residual_norm(const void *u, const void *x, const void *gate, const void *gamma_post, const void *gamma_pre,
                                          void *h, void *y, float *y_scales, float *rrms_post, float *rrms_pre, int64_t rows,
                                          int64_t cols, int64_t ldu, int64_t ldx, int64_t ldg, int64_t gate_rows, int64_t ldh,
                                          int64_t ldy, int64_t lds, float residual_scale, float eps, perf_dtype x_dt,
                                          perf_dtype gate_dt, perf_dtype param_dt, perf_dtype y_dt, perf_stream stream)
{
    using namespace perf;
    const bool y8 = y && y_dt == PERF_E4M3;
    if (!u || !x || (!h && !y) || (y && !gamma_pre) || (y8 && !y_scales)) return PERF_ERR_NULL;
    if (rows < 1 || cols < 1 || cols > kMaxExtent8 || ldu < cols || ldx < cols || (h && ldh < cols) || (y && ldy < cols))
        return PERF_ERR_SHAPE;
    if (gate && (ldg < cols || gate_rows < 1)) return PERF_ERR_SHAPE;
    if (y8 && lds < (cols + kBlock8 - 1) / kBlock8) return PERF_ERR_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(residual_scale)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype_ok(param_dt) || (gate && !dtype_ok(gate_dt)) || (y && !dtype_ok(y_dt) && !dtype8_ok(y_dt)))
        return PERF_ERR_DTYPE;
    const int64_t sz = dtype_size(x_dt), psz = dtype_size(param_dt);
    if (!aligned(u, sz) || !aligned(x, sz) || !aligned(h, sz) || (y && !y8 && !aligned(y, sz)) || (gate && !aligned(gate, dtype_size(gate_dt))) ||
        !aligned(gamma_post, psz) || (y && !aligned(gamma_pre, psz)) || !aligned(rrms_post, 4) || !aligned(rrms_pre, 4) ||
        (y8 && !aligned(y_scales, 4)))
        return PERF_ERR_ALIGN;
    if (y && !y8 && y_dt != x_dt) return PERF_ERR_UNSUPPORTED;
    const int pb = param_dt == PERF_BF16;
    const NormArgs a{u, x, Param{gate, gate_dt == PERF_BF16}, Param{gamma_post, pb}, Param{y ? gamma_pre : nullptr, pb}, h, y, y_scales,
                     rrms_post, rrms_pre, rows, ldu, ldx, ldg, gate ? gate_rows_or_all(gate_rows, rows) : rows, ldh, ldy, lds,
                     (int)cols, residual_scale, eps};
    const hipStream_t st = (hipStream_t)stream;
    if (x_dt == PERF_BF16) {
        if (y8)
            launch_norm<uint16_t, true>(a, st);
        else
            launch_norm<uint16_t, false>(a, st);
    } else {
        if (y8)
            launch_norm<float, true>(a, st);
        else
            launch_norm<float, false>(a, st);
    }
    return launch_status();
}

extern "C" int64_t perf_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    using namespace perf;
    if (rows < 1 || cols < 1 || cols > kMaxExtent8) return -1;
    // (runs of whole groups are longer, so there are no more of them)
    const RunPlan p = plan_runs(rows, cols, INT64_MAX);
    return 4 * (4 * (int64_t)p.runs * cols + (cols > kWidest ? rows : 0));
}

extern "C" perf_status perf_residual_norm_backward(const void *dy, const void *dh, const void *h, const void *u, const void *gate,
                                                   const void *gamma_post, const void *gamma_pre, const float *rrms_post,
                                                   const float *rrms_pre, void *dx, void *du, void *dgate, float *dgamma_post,
                                                   float *dgamma_pre, void *workspace, int64_t rows, int64_t cols, int64_t lddy,
                                                   int64_t lddh, int64_t ldh, int64_t ldu, int64_t ldg, int64_t gate_rows,
                                                   int64_t lddx, int64_t lddu, int64_t lddg, float residual_scale, perf_dtype x_dt,
                                                   perf_dtype gate_dt, perf_dtype param_dt, perf_stream stream)
{
    using namespace perf;
    if ((!dy && !dh) || !u || !dx || !du || !workspace) return PERF_ERR_NULL;
    if (dy && (!h || !gamma_pre || !rrms_pre)) return PERF_ERR_NULL;
    if ((gamma_post && !rrms_post) || (dgate && !gate) || (dgamma_post && !gamma_post) || (dgamma_pre && !dy)) return PERF_ERR_NULL;
    if (rows < 1 || cols < 1 || cols > kMaxExtent8 || (dy && (lddy < cols || ldh < cols)) || (dh && lddh < cols) || ldu < cols ||
        lddx < cols || lddu < cols)
        return PERF_ERR_SHAPE;
    if (gate && (ldg < cols || gate_rows < 1 || (dgate && lddg < cols))) return PERF_ERR_SHAPE;
    if (!std::isfinite(residual_scale)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype_ok(param_dt) || (gate && !dtype_ok(gate_dt))) return PERF_ERR_DTYPE;
    const int64_t sz = dtype_size(x_dt), psz = dtype_size(param_dt), gsz = gate ? dtype_size(gate_dt) : 1;
    if (!aligned(dy, sz) || !aligned(dh, sz) || (dy && !aligned(h, sz)) || !aligned(u, sz) || !aligned(dx, sz) || !aligned(du, sz) ||
        !aligned(gate, gsz) || !aligned(dgate, gsz) || !aligned(gamma_post, psz) || (dy && !aligned(gamma_pre, psz)) ||
        (gamma_post && !aligned(rrms_post, 4)) || (dy && !aligned(rrms_pre, 4)) || !aligned(dgamma_post, 4) ||
        !aligned(dgamma_pre, 4) || !aligned(workspace, 4))
        return PERF_ERR_ALIGN;
    const int pb = param_dt == PERF_BF16, gb = gate_dt == PERF_BF16;
    const int64_t per = gate ? gate_rows_or_all(gate_rows, rows) : rows;
    const RunPlan p = plan_runs(rows, cols, per);
    GradArgs a{dy ? dy : u, dh ? dh : u, dy ? h : u, u, dy != nullptr, dh != nullptr, Param{gate, gb}, Param{gamma_post, pb},
               Param{gamma_pre, pb}, rrms_post, rrms_pre, dx, du, Param{dgate, gb}, dgamma_post, dgamma_pre, (float *)workspace, rows,
               dy ? lddy : ldu, dh ? lddh : ldu, dy ? ldh : ldu, ldu, ldg, per, lddx, lddu, lddg, p.run, p.runs, (int)cols,
               gate && p.whole_groups, residual_scale};
    if (x_dt == PERF_BF16)
        launch_grad<uint16_t>(a, (hipStream_t)stream);
    else
        launch_grad<float>(a, (hipStream_t)stream);
    return launch_status();
}
