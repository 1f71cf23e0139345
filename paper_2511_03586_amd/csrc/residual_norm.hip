// The RMS norms before and after a block of a network, joined with the block's gate and the scaled residual:
//     n = u r1 gamma_post,   h = residual_scale x + gate n,   y = h r2 gamma_pre,
//     r1 = (mean u^2 + eps)^(-1/2),   r2 = (mean h^2 + eps)^(-1/2),
// u the block's output, x the residual stream before it, h the stream behind it, y the next block's input, in x's type or
// in 8 bits with a scale for each 128 elements.  And the gradient: with t = dy gamma_pre, hn = h r2, un = u r1,
//     H = dh + r2 (t - hn mean(t hn)),   dx = residual_scale H,    dgamma_pre = sum over rows of dy hn,
//     D = gate H,  v = D gamma_post,     du = r1 (v - un mean(v un)),  dgamma_post = sum of D un,  dgate = sum of n H.
// (gamma_post left out: n = u, du = D.)  Bound by HBM: each operand is read once and each result written once.
//
//  * residual_norm_kernel / residual_norm_grad_kernel<W>: W waves own a row, 8 elements per lane (16 from 8193 columns on), so
//    that a row is in registers between its two sums; workgroups of 8 waves (gradient: 16) take the rows of several teams
//    side by side.  The gains and the gate are read once for all rows that share them.
//  * The gradient's sums over rows: a workgroup owns a run of rows and sums them in registers; its sums go to the
//    workspace and are added in the order of the rows by residual_norm_sums_kernel.  No atomics.
//  * residual_norm_any_kernel and its gradient: rows of fewer than 8 elements and those beyond 16 waves' registers, in several
//    passes over memory.
// Statistics, h on its way into y, and all sums are fp32; y is computed from h before it is rounded to its type.
// Measured (bf16, one gate for all rows): 8192 x 4096 forward 46 us (5.8 TB/s), gradient 80 us (5.0 TB/s, 75 + 5 in its two
// kernels); 2048 x 16384 50 and 102 us, where several passes over memory took 73 and 530.
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
    // n of the eight elements from j on, the others zero
    __device__ __forceinline__ void eight(int64_t j, int n, float (&v)[8]) const
    {
        if (bf16) {
            Eight<uint16_t> e;
            e.load_cached(reinterpret_cast<const uint16_t *>(p) + j, n);
            e.get(v);
        } else {
            Eight<float> e;
            e.load_cached(reinterpret_cast<const float *>(p) + j, n);
            e.get(v);
        }
    }
    // a lane's group of the row that begins at `row`
    template <typename G>
    __device__ __forceinline__ void group(int64_t row, const G &at, float (&v)[8]) const
    {
        if (bf16)
            at.load_as(reinterpret_cast<const uint16_t *>(p) + row, v);
        else
            at.load_as(reinterpret_cast<const float *>(p) + row, v);
    }
    template <typename G>
    __device__ __forceinline__ void put_group(int64_t row, const G &at, const float (&v)[8]) const
    {
        if (bf16)
            at.store(reinterpret_cast<uint16_t *>(const_cast<void *>(p)) + row, v);
        else
            at.store(reinterpret_cast<float *>(const_cast<void *>(p)) + row, v);
    }
    __device__ __forceinline__ void put(int64_t j, float v) const
    {
        if (bf16)
            reinterpret_cast<uint16_t *>(const_cast<void *>(p))[j] = f32_to_bf16(v);
        else
            reinterpret_cast<float *>(const_cast<void *>(p))[j] = v;
    }
};

struct NormArgs {
    const void *u, *x;
    Param gate, post, pre;  // p is null where there is none
    void *h, *y;
    float *y_scales, *r_post, *r_pre;
    int64_t ldu, ldx, ldg, ldh, ldy, lds;
    int rows, cols, gate_rows;
    uint32_t gate_magic;  // of a division by gate_rows: one of 64 bits runs on the vector units, and every row's address behind it
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

// G: groups of eight elements per lane.  Y8: y is e4m3 with scales (else of x's type); RAG: rows that are no whole groups of 8
template <typename T, int W, int G, bool Y8, bool RAG>
__global__ __launch_bounds__(W > 8 ? 64 * W : 512) void residual_norm_kernel(const NormArgs a)
{
    constexpr int kWaves = W > 8 ? W : 8, kTeams = kWaves / W, kThreads = 64 * W;
    __shared__ float red[2][kWaves];
    // (the same in all lanes of a wave: rows and their addresses are scalars)
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / W, lane = threadIdx.x - team * kThreads;
    const float inv_cols = 1.0f / (float)a.cols;
    using Own = Group<T, RAG>;
    Own own[G];
    float post[G][8], pre[G][8], gate[G][8];
#pragma unroll
    for (int k = 0; k < G; ++k) {
        own[k] = Own(lane + k * Own::kRuns * kThreads, kThreads, a.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) post[k][e] = pre[k][e] = gate[k][e] = 1.f;
        if (a.post.p) a.post.group(0, own[k], post[k]);
        if (a.pre.p) a.pre.group(0, own[k], pre[k]);
    }
    int held = -1;  // the group of rows whose gate is in `gate`
    const int step = gridDim.x * kTeams;
    constexpr bool kAhead = G * sizeof(T) <= 4;  // (two groups of fp32 leave no registers for the next row's operands)
    Eight<T> u[G], x[G];
    auto load = [&](int to) {
        const int64_t r = min(to, a.rows - 1);
#pragma unroll
        for (int k = 0; k < G; ++k) {
            own[k].load(u[k], (const T *)a.u + r * a.ldu);
            own[k].load(x[k], (const T *)a.x + r * a.ldx);
        }
    };
    // teams of a workgroup take neighbouring rows and run the same number of rounds: its barriers are met by all
    int at = blockIdx.x * kTeams + team;
    if constexpr (kAhead) load(at);
    for (int first = blockIdx.x * kTeams; first < a.rows; first += step, at += step) {
        const int64_t row = at;
        const bool live = at < a.rows;
        if (a.gate.p && live) {
            const int g = div_by(at, a.gate_rows, a.gate_magic);
            if (g != held) {
#pragma unroll
                for (int k = 0; k < G; ++k) a.gate.group((int64_t)g * a.ldg, own[k], gate[k]);
                held = g;
            }
        }
        if constexpr (!kAhead) load(at);
        float v[G][8], h[G][8], s = 0.f;
#pragma unroll
        for (int k = 0; k < G; ++k) {
            own[k].keep(u[k], true), own[k].keep(x[k], true);
            u[k].get(v[k]), x[k].get(h[k]);
        }
        if constexpr (kAhead) load(at + step);  // the next row's loads fly during this row's sums
        if (a.post.p) {
#pragma unroll
            for (int k = 0; k < G; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) s = __builtin_fmaf(own[k].once(e, v[k][e]), v[k][e], s);
            s = team_sum<W>(s, red[0]);
            const float r1 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
            if (live && lane == 0 && a.r_post) a.r_post[row] = r1;
#pragma unroll
            for (int k = 0; k < G; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] *= r1 * post[k][e];
        } else if (W > 1) {
            __syncthreads();  // the one sum's array is written again in the next round
        }
        s = 0.f;
#pragma unroll
        for (int k = 0; k < G; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[k][e] = __builtin_fmaf(gate[k][e], v[k][e], a.residual_scale * h[k][e]);
                s = __builtin_fmaf(own[k].once(e, h[k][e]), h[k][e], s);
            }
            if (a.h && live) own[k].store((T *)a.h + row * a.ldh, h[k]);
        }
        if (!a.y) {
            if (W > 1) __syncthreads();  // as above
            continue;
        }
        s = team_sum<W>(s, red[1]);
        const float r2 = 1.0f / __builtin_sqrtf(s * inv_cols + a.eps);
        if (live && lane == 0 && a.r_pre) a.r_pre[row] = r2;
#pragma unroll
        for (int k = 0; k < G; ++k) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = h[k][e] * r2 * pre[k][e];
            if constexpr (!Y8) {
                if (live) own[k].store((T *)a.y + row * a.ldy, y);
            } else {
                using F = Fp8<false>;
                // a block is sixteen lanes' groups (bf16), or thirty-two lanes' halves of theirs (fp32)
                float inv[8];
                constexpr int kRun = Own::kRun, kLanes = kBlock8 / kRun;
#pragma unroll
                for (int r = 0; r < 8; r += kRun) {
                    uint32_t m = 0;
#pragma unroll
                    for (int e = r; e < r + kRun; ++e) m = max(m, magnitude(own[k].in(e) ? own[k].once(e, y[e]) : 0.f));
                    const float q = F::scale(group_max_u32<kLanes>(m));
#pragma unroll
                    for (int e = r; e < r + kRun; ++e) inv[e] = 1.0f / q;
                    if (live && lane % kLanes == 0 && own[k].in(r))
                        a.y_scales[row * a.lds + (lane + (k * Own::kRuns + r / kRun) * kThreads) / kLanes] = q;
                }
                const uint32_t w[2] = {F::pack(y[0] * inv[0], y[1] * inv[1], y[2] * inv[2], y[3] * inv[3]),
                                       F::pack(y[4] * inv[4], y[5] * inv[5], y[6] * inv[6], y[7] * inv[7])};
                if (live) own[k].store_bytes((uint8_t *)a.y + row * a.ldy, w);
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
    for (int at = blockIdx.x; at < a.rows; at += gridDim.x) {
        const int64_t row = at;
        const T *u = (const T *)a.u + row * a.ldu, *x = (const T *)a.x + row * a.ldx;
        const int64_t g = a.gate.p ? (int64_t)div_by(at, a.gate_rows, a.gate_magic) * a.ldg : 0;
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
    int64_t lddy, lddh, ldh, ldu, ldg, lddx, lddu, lddg;
    int rows, cols, gate_rows;
    uint32_t gate_magic;
    int run, runs;  // rows of a workgroup, and workgroups
    bool whole_groups;  // runs are whole groups of gate rows, and a team takes a group by itself
    float residual_scale;
};

// Where a workgroup's sum of a gate's gradient goes: a group that lies within its run straight to the result; of a group
// that goes on beyond it, slot 2 run + 1 (it begins here) or 2 run (it began before).
__device__ __forceinline__ float *gate_slot(const GradArgs &a, int64_t run, bool begins)
{
    return a.ws + (2 * (int64_t)a.runs + 2 * run + (begins ? 1 : 0)) * a.cols;
}

// A row stays in registers as it came and is unpacked where it is used; gamma_pre, gate gamma_post and the sum that grows by
// groups lie in LDS, every lane's own where it alone reads them: a lane has 128 registers.  Of the
// three sums over rows two grow by the row, dy hn and H un: while the gate is the same, dgate is gamma_post times the latter
// and dgamma_post the gate times it.
// With two groups of eight to a lane (G) there is no LDS left for the sum by groups, which lies in the workspace then.
template <typename T, int W, int G, bool RAG>
__global__ __launch_bounds__(1024) void residual_norm_grad_kernel(const GradArgs a)
{
    constexpr int kWaves = 16, kTeams = kWaves / W, kThreads = 64 * W, kAll = 64 * kWaves;
    enum { kPre, kGatePost, kSumPost, kPlanes = G == 1 ? 3 : 2 };
    constexpr bool kAhead = G == 1;  // (two groups leave no registers for the next row's operands)
    constexpr bool kTwice = G * sizeof(T) > 4;  // (... of fp32, none for u from one sum to the next: it is read again)
    __shared__ float red[2][kWaves];
    __shared__ float4_t own[kPlanes][G][2][kAll];
    const int tid = threadIdx.x, team = __builtin_amdgcn_readfirstlane(tid >> 6) / W, lane = tid - team * kThreads;
    const float inv_cols = 1.0f / (float)a.cols;
    const bool has_post = a.post.p != nullptr, has_gate = a.gate.p != nullptr;
    using Own = Group<T, RAG>;
    Own here[G];
#pragma unroll
    for (int k = 0; k < G; ++k) here[k] = Own(lane + k * Own::kRuns * kThreads, kThreads, a.cols);
    auto get_own = [&](int which, int k, int q, float (&v)[4]) {
        const float4_t f = own[which][k][q][tid];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = f[e];
    };
    auto put_own = [&](int which, int k, const float (&v)[8]) {
        own[which][k][0][tid] = float4_t{v[0], v[1], v[2], v[3]};
        own[which][k][1][tid] = float4_t{v[4], v[5], v[6], v[7]};
    };
    // the sums of this run, of which a single one has the results; posts grows by groups, each lane its own columns
    const bool only = a.runs == 1;
    float *const pres = only ? a.dpre : a.ws + (int64_t)blockIdx.x * a.cols;
    float *const posts = only ? a.dpost : a.ws + ((int64_t)a.runs + blockIdx.x) * a.cols;
    auto get_sum_post = [&](int k, float (&v)[8]) {
        if constexpr (G == 1) {
            float lo[4], hi[4];
            get_own(kSumPost, 0, 0, lo), get_own(kSumPost, 0, 1, hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = lo[e], v[4 + e] = hi[e];
        } else {
            here[k].load_as(posts, v);
        }
    };
    auto put_sum_post = [&](int k, const float (&v)[8]) {
        if constexpr (G == 1)
            put_own(kSumPost, 0, v);
        else
            here[k].store_cached(posts, v);
    };
    float sum_pre[G][8], sum_un[G][8], v8[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v8[e] = 0.f;
#pragma unroll
        for (int k = 0; k < G; ++k) sum_pre[k][e] = 0.f;
    }
    // gamma_post, or one, or the gate of group g, or one
    auto get_post = [&](int k, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.f;
        if (has_post) a.post.group(0, here[k], v);
    };
    auto get_gate = [&](int g, int k, float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 1.f;
        if (has_gate) a.gate.group((int64_t)g * a.ldg, here[k], v);
    };
    const bool all_in = a.cols == 8 * G * kThreads && a.has_dy && a.has_dh;

    Eight<T> next_dy[G], next_dh[G], next_h[G], next_u[G];
    float next_r2, next_r1;
    auto load = [&](int to) {
        const int64_t r = min(to, a.rows - 1);
#pragma unroll
        for (int k = 0; k < G; ++k) {
            // (a new value to the compiler for each row: it would keep a 64-bit address for every operand and lane otherwise)
            asm volatile("" : "+v"(here[k].at[0]));
            if constexpr (Own::kRuns > 1) asm volatile("" : "+v"(here[k].at[1]));
            here[k].load(next_dy[k], (const T *)a.dy + r * a.lddy);
            here[k].load(next_h[k], (const T *)a.h + r * a.ldh);
            here[k].load(next_dh[k], (const T *)a.dh + r * a.lddh);
            here[k].load(next_u[k], (const T *)a.u + r * a.ldu);
        }
        // (not given: some other number, not used)
        next_r2 = *(a.has_dy ? a.r_pre + r : a.ws), next_r1 = *(has_post ? a.r_post + r : a.ws);
    };
    // Groups of few rows (whole_groups): a team takes every kTeams-th group by itself.  Otherwise the rows of the run that
    // share a gate are dealt to the teams in turn.  Where all rows share it (spread), the rows are dealt to all teams of the
    // chip instead, which then read one stretch of memory together (8192 x 4096: 90 us, with runs of neighbours 95).  All teams of a
    // workgroup run the same number of rounds.
    const int begin = blockIdx.x * a.run, end = min(a.rows, begin + a.run), per = a.gate_rows;
    const bool each = a.whole_groups, spread = !each && per >= a.rows;
    const int step = spread ? gridDim.x * kTeams : kTeams;
    int g = div_by(begin, per, a.gate_magic) + (each ? team : 0);  // the group of rows whose gate is in use
    int row = each ? g * per : (spread ? blockIdx.x * kTeams : begin) + team;
    int from = begin;  // the round's first row, the same for all teams
    if constexpr (kAhead) load(row);  // (ahead of the parameters: both fly together)
#pragma unroll
    for (int k = 0; k < G; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v8[e] = 0.f;
        if (a.dpost) put_sum_post(k, v8);
        if (a.has_dy) a.pre.group(0, here[k], v8);
        put_own(kPre, k, v8);
    }

    // one row of this team (a dead one adds nothing and writes nothing); `next` is loaded meanwhile
    auto one = [&](int64_t row, bool live, int next) {
        if constexpr (!kAhead) load((int)row);
        const float r2 = a.has_dy && live ? next_r2 : 0.f, r1 = !has_post ? 1.f : live ? next_r1 : 0.f;
        Eight<T> dy[G], h[G], dh[G], u[G];
#pragma unroll
        for (int k = 0; k < G; ++k) {
            dy[k] = next_dy[k], h[k] = next_h[k], dh[k] = next_dh[k], u[k] = next_u[k];
            if (!(live && all_in)) {
                here[k].keep(dy[k], live && a.has_dy), here[k].keep(h[k], live && a.has_dy);
                here[k].keep(dh[k], live && a.has_dh), here[k].keep(u[k], live);
            }
        }
        if constexpr (kAhead) load(next);
        float s = 0.f;
        if (a.has_dy) {
#pragma unroll
            for (int p = 0; p < 2 * G; ++p) {
                const int k = p >> 1, q = p & 1;
                float t[4], hv[4], pre[4];
                dy[k].get_half(q, t), h[k].get_half(q, hv), get_own(kPre, k, q, pre);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float th = t[e] * hv[e];
                    sum_pre[k][4 * q + e] = __builtin_fmaf(th, r2, sum_pre[k][4 * q + e]);
                    s = __builtin_fmaf(here[k].once(4 * q + e, th), pre[e], s);
                }
                __builtin_amdgcn_sched_barrier(0);  // (reads of the next half's operands ahead of here cost registers)
            }
            s = team_sum<W>(s, red[0]);
        } else if (W > 1) {
            __syncthreads();  // the one sum's array is written again in the next row
        }
        const float of_h = -r2 * r2 * (r2 * s * inv_cols);  // H = dh + r2 t - r2 hn mean(t hn)
        s = 0.f;
        float v[G][8];
#pragma unroll
        for (int k = 0; k < G; ++k) {
            dy[k].renew(), h[k].renew();
            float dx[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float t[4], hv[4], H[4], pre[4], un[4], gp[4];
                dy[k].get_half(q, t), h[k].get_half(q, hv), dh[k].get_half(q, H), u[k].get_half(q, un);
                get_own(kPre, k, q, pre), get_own(kGatePost, k, q, gp);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    H[e] = __builtin_fmaf(hv[e], of_h, __builtin_fmaf(t[e] * pre[e], r2, H[e]));
                    un[e] *= r1;
                    sum_un[k][4 * q + e] = __builtin_fmaf(H[e], un[e], sum_un[k][4 * q + e]);
                    v[k][4 * q + e] = H[e] * gp[e];
                    s = __builtin_fmaf(here[k].once(4 * q + e, v[k][4 * q + e]), un[e], s);
                    dx[4 * q + e] = a.residual_scale * H[e];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (live) here[k].store((T *)a.dx + row * a.lddx, dx);
        }
        if (has_post) {
            const float of_u = -r1 * r1 * (team_sum<W>(s, red[1]) * inv_cols);  // du = r1 v - r1 un mean(v un)
#pragma unroll
            for (int k = 0; k < G; ++k) {
                if constexpr (kTwice)
                    here[k].load(u[k], (const T *)a.u + min((int)row, a.rows - 1) * a.ldu);
                else
                    u[k].renew();
                float uv[8];
                u[k].get(uv);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] = __builtin_fmaf(uv[e], of_u, r1 * v[k][e]);
            }
        } else if (W > 1) {
            __syncthreads();  // as above
        }
        if (live) {
#pragma unroll
            for (int k = 0; k < G; ++k) here[k].store((T *)a.du + row * a.lddu, v[k]);
        }
    };
    // the teams' sums v, added in the teams' order: the first team has them.  The gate's place serves, until the next one comes
    auto join = [&](float (&v)[8]) {
        if constexpr (kTeams > 1) {  // (one group a lane)
            __syncthreads();
            put_own(kGatePost, 0, v);
            __syncthreads();
            if (team == 0) {
                for (int o = 1; o < kTeams; ++o)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += own[kGatePost][0][e >> 2][o * kThreads + lane][e & 3];
            }
            __syncthreads();
        }
    };

    while (from < end) {
        const int stop = spread ? a.rows : min(end, (g + 1) * per), first = spread ? blockIdx.x * kTeams : from;
#pragma unroll
        for (int k = 0; k < G; ++k) {
            if (g * per < end) {
                float gate[8];
                get_gate(g, k, gate), get_post(k, v8);
#pragma unroll
                for (int e = 0; e < 8; ++e) v8[e] *= gate[e];
                put_own(kGatePost, k, v8);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum_un[k][e] = 0.f;
        }
        const int rounds = each ? per : (stop - first + step - 1) / step;
        for (int i = rounds; i > 0; --i) {
            const int next = each ? (i > 1 ? row + 1 : (g + kTeams) * per) : (i > 1 ? row + step : stop + team);
            one(row, row < stop, next);
            row = next;
        }
#pragma unroll
        for (int k = 0; k < G; ++k) {
            if (a.dpost && g * per < end) {
                float sum[8];
                get_gate(g, k, v8), get_sum_post(k, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf(v8[e], sum_un[k][e], sum[e]);
                put_sum_post(k, sum);
            }
            if (a.dgate.p) {
                if (!each) join(sum_un[k]);
                const bool begins = g * per >= begin, ends = min(a.rows, (g + 1) * per) <= end;
                if (each ? g * per < end : team == 0) {
                    get_post(k, v8);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum_un[k][e] *= v8[e];
                    if (begins && ends)
                        a.dgate.put_group((int64_t)g * a.lddg, here[k], sum_un[k]);
                    else
                        here[k].store(gate_slot(a, blockIdx.x, begins), sum_un[k]);
                }
            }
        }
        g += each ? kTeams : 1;
        from = each ? (g - team) * per : stop;
    }
#pragma unroll
    for (int k = 0; k < G; ++k) {
        if (a.dpre && a.has_dy) {
            join(sum_pre[k]);
            if (team == 0) here[k].store(pres, sum_pre[k]);
        }
        if (a.dpost && G == 1) {
            get_sum_post(k, v8);
            join(v8);
            if (team == 0) here[k].store(posts, v8);
        }
    }
}

// The runs' sums, added in the order of the rows, 64 columns per workgroup, from column `first` on.  blockIdx.y: 0 = dgamma_pre,
// 1 = dgamma_post, sixteen parts of the runs side by side; then the gates of groups that begin in one run and go on beyond it, by
// group or (by_run) by the run in which it begins, whichever are fewer: one gate in sixteen parts, or sixteen gates (each_part) of
// few runs.
__global__ __launch_bounds__(1024) void residual_norm_sums_kernel(const GradArgs a, bool by_run, bool each_part, int gates, int first)
{
    constexpr int kParts = 16;
    __shared__ float parts[kParts][64];
    const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = first + blockIdx.x * 64 + lane;
    const bool gamma = blockIdx.y < 2, post = blockIdx.y == 1;
    const int gate = each_part ? (blockIdx.y - 2) * kParts + part : blockIdx.y - 2;
    int count = a.runs, g = 0;
    const float *from = a.ws + (post ? (int64_t)a.runs * a.cols : 0);  // the sums of run i lie `step` after those of run i - 1
    int64_t step = a.cols;
    if (gamma) {
        if (!(post ? a.dpost : a.dpre)) return;
    } else {
        if (gate >= gates) return;  // (whole waves, and no barrier behind)
        g = by_run ? div_by(min(a.rows, (gate + 1) * a.run) - 1, a.gate_rows, a.gate_magic) : gate;
        const int begin = g * a.gate_rows, end = min(a.rows, begin + a.gate_rows), t = begin / a.run;
        if ((by_run && t != gate) || end <= (t + 1) * a.run) return;
        from = gate_slot(a, t, true);  // ... of the first, one row of slots early for the others
        step = 2 * (int64_t)a.cols;
        count = (end - 1) / a.run - t + 1;
    }
    const bool alone = !gamma && each_part;
    const int per = alone ? count : (count + kParts - 1) / kParts, lo = alone ? 0 : part * per, hi = min(count, lo + per);
    float s = 0.f;
    if (col < a.cols) {
#pragma unroll 8
        for (int i = lo; i < hi; ++i) s += from[i * step - (!gamma && i > 0 ? a.cols : 0) + col];
    }
    if (!alone) {
        parts[part][lane] = s;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int p = 1; p < kParts; ++p) s += parts[p][lane];
    }
    if (col >= a.cols) return;
    if (!gamma)
        a.dgate.put((int64_t)g * a.lddg + col, s);
    else if (post)
        a.dpost[col] = s;
    else
        a.dpre[col] = s;
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
    for (int at = blockIdx.x; at < a.rows; at += gridDim.x) {
        const int64_t row = at;
        const float r2 = a.has_dy ? a.r_pre[row] : 0.f, r1 = a.post.p ? a.r_post[row] : 1.f;
        const int64_t g = a.gate.p ? (int64_t)div_by(at, a.gate_rows, a.gate_magic) * a.ldg : 0;
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
    const int begin = blockIdx.y * a.run, end = min(a.rows, begin + a.run), per = a.gate_rows;
    const float post = a.post.p ? a.post.at(c) : 1.f;
    float sum_pre = 0.f, sum_post = 0.f;
    for (int from = begin; from < end;) {
        const int g = div_by(from, per, a.gate_magic), to = min(end, (g + 1) * per);
        const float gate = a.gate.p ? a.gate.at((int64_t)g * a.ldg + c) : 1.f;
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
                a.dgate.put((int64_t)g * a.lddg + c, sum_gate);
            else
                gate_slot(a, blockIdx.y, begins)[c] = sum_gate;
        }
        from = to;
    }
    if (a.has_dy) a.ws[(int64_t)blockIdx.y * a.cols + c] = sum_pre;
    a.ws[((int64_t)a.runs + blockIdx.y) * a.cols + c] = sum_post;
}

// ---- entry points --------------------------------------------------------------------------------------------------
// columns of the kernels that hold a row: a group of eight, and what 16 waves have room for
constexpr int kNarrowest = 8, kWidest = 16 * 64 * 8 * 2;
inline bool row_fits(int64_t cols) { return cols >= kNarrowest && cols <= kWidest; }

// f(waves of a team, groups of eight to a lane) for rows that fit one
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
    else if (cols <= 8192)
        f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else
        f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
}

template <typename T, bool Y8>
static void launch_norm(const NormArgs &a, hipStream_t stream)
{
    if (!row_fits(a.cols)) {
        residual_norm_any_kernel<T, Y8><<<(unsigned)std::min<int64_t>(a.rows, 65536), 1024, 0, stream>>>(a);
        return;
    }
    with_team(a.cols, [&](auto w, auto groups) {
        constexpr int W = w, G = groups, kTeams = W > 8 ? 1 : 8 / W, kThreads = W > 8 ? 1024 : 512;
        // One workgroup per CU: more of them read more places of memory at once (8192 x 4096 bf16: 46.7 us with 256, 48.5 with
        // 512, 53 with 1024).  A gate that changes after a few rows is waited for, which a second one hides (of every element's
        // own: 56 us with 512, 79 with 256).
        const int64_t most = a.gate.p && a.gate_rows < 16 ? 512 : 256;
        const int64_t grid = std::min<int64_t>((a.rows + kTeams - 1) / kTeams, most);
        if (a.cols % 8)
            residual_norm_kernel<T, W, G, Y8, true><<<(unsigned)grid, kThreads, 0, stream>>>(a);
        else
            residual_norm_kernel<T, W, G, Y8, false><<<(unsigned)grid, kThreads, 0, stream>>>(a);
    });
}

// Rows of a workgroup's run in the gradient, and whether the runs are whole groups of a gate.
struct RunPlan {
    int run, runs;
    bool whole_groups;
};
// A run for each CU.  Teams that take whole groups by themselves add a gate's sums in their registers, but hold all its rows; if
// all teams share a group's rows, its sums meet in LDS behind it, for about the time of two rows.  The fewer rows in turn: 5000 x
// 512 with 16 rows to a gate take 41 us by groups and 23 by rows, 300 x 512 with 2 rows to a gate 13 and 39.
static RunPlan plan_runs(int64_t rows, int64_t cols, int64_t gate_rows, bool gate)
{
    const int64_t teams = cols <= 512 ? 16 : cols <= 1024 ? 8 : cols <= 2048 ? 4 : cols <= 4096 ? 2 : 1, most = 256;
    auto run_of = [&](int64_t unit) { return ((rows + most - 1) / most + unit - 1) / unit * unit; };
    RunPlan p;
    p.run = (int)run_of(teams);
    p.whole_groups = false;
    if (gate && gate_rows <= 16) {
        const int64_t whole = run_of(teams * gate_rows);
        p.whole_groups = whole / teams <= p.run / teams + 2 * ((p.run - 1) / gate_rows + 1);
        if (p.whole_groups) p.run = (int)whole;
    }
    p.runs = (int)((rows + p.run - 1) / p.run);
    return p;
}

template <typename T>
static void launch_grad(GradArgs a, hipStream_t stream)
{
    if (!row_fits(a.cols)) {
        float *means = a.ws + 4 * (int64_t)a.runs * a.cols;
        const unsigned grid = (unsigned)std::min<int64_t>(a.rows, 65536);
        residual_norm_grad_any_kernel<T, true><<<grid, 1024, 0, stream>>>(a, means);
        residual_norm_grad_cols_kernel<T><<<dim3((a.cols + 255) / 256, a.runs), 256, 0, stream>>>(a, means);
        residual_norm_grad_any_kernel<T, false><<<grid, 1024, 0, stream>>>(a, means);
    } else {
        with_team(a.cols, [&](auto w, auto groups) {
            constexpr int W = w, G = groups;
            if (a.cols % 8)
                residual_norm_grad_kernel<T, W, G, true><<<a.runs, 1024, 0, stream>>>(a);
            else
                residual_norm_grad_kernel<T, W, G, false><<<a.runs, 1024, 0, stream>>>(a);
        });
    }
    // (a gate whose groups lie within runs has its sums already)
    const int groups = (a.rows + a.gate_rows - 1) / a.gate_rows;
    const bool by_run = groups > a.runs;
    const int gates = a.dgate.p && !a.whole_groups ? std::min(groups, a.runs) : 0;
    if (a.runs == 1 && row_fits(a.cols)) return;  // (the run's sums are the results)
    // Sixteen gates to a workgroup where a gate has few runs: 2000 x 2048, 7 rows to a gate, 46 us with a workgroup for each, 27 so;
    // 1920 x 136 with about nine runs to a gate 17 and 18.5.
    const bool each_part = a.gate_rows <= 6 * a.run;
    if (!a.dpre && !a.dpost && !gates) return;
    constexpr int kMost = (int)max_blocks(1024) * 64;  // columns of a launch, which is less than 2^32 threads
    for (int64_t first = 0; first < a.cols; first += kMost)
        residual_norm_sums_kernel<<<dim3(((int)std::min<int64_t>(kMost, a.cols - first) + 63) / 64, 2 + (each_part ? (gates + 15) / 16 : gates)),
                                    1024, 0, stream>>>(a, by_run, each_part, gates, (int)first);
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
    if (rows < 1 || cols < 1 || rows > kMaxExtent8 || cols > kMaxExtent8 || ldu < cols || ldx < cols || (h && ldh < cols) || (y && ldy < cols))
        return PERF_ERR_SHAPE;
    if (gate && (ldg < cols || gate_rows < 1)) return PERF_ERR_SHAPE;
    if (y8 && (lds < (cols + kBlock8 - 1) / kBlock8 || !addressable(rows, lds))) return PERF_ERR_SHAPE;
    if (!addressable(rows, ldu) || !addressable(rows, ldx) || (h && !addressable(rows, ldh)) || (y && !addressable(rows, ldy)) ||
        (gate && !addressable(rows, ldg)))
        return PERF_ERR_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(residual_scale)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype_ok(param_dt) || (gate && !dtype_ok(gate_dt)) || (y && !dtype_ok(y_dt) && !dtype8_ok(y_dt)))
        return PERF_ERR_DTYPE;
    const int64_t sz = dtype_size(x_dt), psz = dtype_size(param_dt);
    if (!aligned(u, sz) || !aligned(x, sz) || !aligned(h, sz) || (y && !y8 && !aligned(y, sz)) || (gate && !aligned(gate, dtype_size(gate_dt))) ||
        !aligned(gamma_post, psz) || (y && !aligned(gamma_pre, psz)) || !aligned(rrms_post, 4) || !aligned(rrms_pre, 4) ||
        (y8 && !aligned(y_scales, 4)))
        return PERF_ERR_ALIGN;
    if (y && !y8 && y_dt != x_dt) return PERF_ERR_UNSUPPORTED;
    const int pb = param_dt == PERF_BF16, per = (int)(gate ? std::min(gate_rows, rows) : rows);
    const NormArgs a{u, x, Param{gate, gate_dt == PERF_BF16}, Param{gamma_post, pb}, Param{y ? gamma_pre : nullptr, pb}, h, y, y_scales,
                     rrms_post, rrms_pre, ldu, ldx, ldg, ldh, ldy, lds, (int)rows, (int)cols, per, div_magic(per), residual_scale, eps};
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
    if (rows < 1 || cols < 1 || rows > kMaxExtent8 || cols > kMaxExtent8) return -1;
    // (runs of whole groups are longer: there are no more of them)
    const RunPlan p = plan_runs(rows, cols, rows, false);
    return 4 * (4 * (int64_t)p.runs * cols + (row_fits(cols) ? 0 : rows));
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
    if (rows < 1 || cols < 1 || rows > kMaxExtent8 || cols > kMaxExtent8 || (dy && (lddy < cols || ldh < cols)) || (dh && lddh < cols) || ldu < cols ||
        lddx < cols || lddu < cols)
        return PERF_ERR_SHAPE;
    if (gate && (ldg < cols || gate_rows < 1 || (dgate && lddg < cols))) return PERF_ERR_SHAPE;
    if ((dy && (!addressable(rows, lddy) || !addressable(rows, ldh))) || (dh && !addressable(rows, lddh)) || !addressable(rows, ldu) ||
        !addressable(rows, lddx) || !addressable(rows, lddu) || (gate && !addressable(rows, ldg)) || (dgate && !addressable(rows, lddg)))
        return PERF_ERR_SHAPE;
    if (!std::isfinite(residual_scale)) return PERF_ERR_SHAPE;
    if (!dtype_ok(x_dt) || !dtype_ok(param_dt) || (gate && !dtype_ok(gate_dt))) return PERF_ERR_DTYPE;
    const int64_t sz = dtype_size(x_dt), psz = dtype_size(param_dt), gsz = gate ? dtype_size(gate_dt) : 1;
    if (!aligned(dy, sz) || !aligned(dh, sz) || (dy && !aligned(h, sz)) || !aligned(u, sz) || !aligned(dx, sz) || !aligned(du, sz) ||
        !aligned(gate, gsz) || !aligned(dgate, gsz) || !aligned(gamma_post, psz) || (dy && !aligned(gamma_pre, psz)) ||
        (gamma_post && !aligned(rrms_post, 4)) || (dy && !aligned(rrms_pre, 4)) || !aligned(dgamma_post, 4) ||
        !aligned(dgamma_pre, 4) || !aligned(workspace, 4))
        return PERF_ERR_ALIGN;
    const int pb = param_dt == PERF_BF16, gb = gate_dt == PERF_BF16;
    const int per = (int)(gate ? std::min(gate_rows, rows) : rows);
    const RunPlan p = plan_runs(rows, cols, per, gate != nullptr);
    GradArgs a{dy ? dy : u, dh ? dh : u, dy ? h : u, u, dy != nullptr, dh != nullptr, Param{gate, gb}, Param{gamma_post, pb},
               Param{gamma_pre, pb}, rrms_post, rrms_pre, dx, du, Param{dgate, gb}, dgamma_post, dgamma_pre, (float *)workspace,
               dy ? lddy : ldu, dh ? lddh : ldu, dy ? ldh : ldu, ldu, ldg, lddx, lddu, lddg, (int)rows, (int)cols, per, div_magic(per),
               p.run, p.runs, p.whole_groups, residual_scale};
    if (x_dt == PERF_BF16)
        launch_grad<uint16_t>(a, (hipStream_t)stream);
    else
        launch_grad<float>(a, (hipStream_t)stream);
    return launch_status();
}
