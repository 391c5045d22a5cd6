// Layer normalisation over the channels of a channels-last map, forward on a frame's active
// blocks and backward on every pixel.
//
//   forward   y = act((x - mean) rstd gamma + beta (+ residual)), mean and variance over the
//             c channels of one pixel (a row), rstd = 1 / sqrt(var + eps);
//   backward  with g = dy' gamma, dy' = dy [y > 0] behind a ReLU, xhat = (x - mean) rstd:
//             dx = rstd (g - mean(g) - xhat mean(g xhat)),
//             dgamma = sum over rows of dy' xhat, dbeta = sum over rows of dy'.
//
// Both are bound by memory: a row is read once, kept in registers, and its statistics are
// taken in two passes over the registers (the mean, then the squares of the differences), in
// fp32 whatever the storage (the mean by a division: a row of one value has no variance,
// which 1 / c rounded would give it). The backward pass computes the statistics again from x, which
// it has to read in any case.
//
// A row belongs to L lanes with NV vectors of 16 bytes each: 8 to 64 lanes of a wave, whose
// sums are register exchanges, or a workgroup of 256 threads for longer rows (partial sums
// through LDS), or one that passes over a still longer row three times. A row whose length
// is no multiple of a vector ends in a vector that starts earlier and overlaps its
// neighbour: the overlapped elements are left out of the sums, and both store the same value.
//
// Weight gradients: a workgroup keeps the sums of its rows in registers (a lane has the same
// columns in every row), its groups meet in LDS, each workgroup writes one partial row, and
// a second kernel adds those in their order: no atomics, equal bits in every run.
//
// Measured: forward 5.1 to 5.5 TB/s on maps of 50 MB and more (16384 x 4096 in fp16 49 us,
// 8191 x 1001 in fp32 12.3), backward 4.5 to 4.9 (16384 x 4096 84 us and 4 for the partial
// rows; 16384 x 1024 in fp32 41.5), where a large copy reaches 4.9. Calls of a few hundred
// rows take 2.7 us forward and 5.6 backward, launches of which little is work.
#include <algorithm>

#include "bc_internal.h"
#include "rows.h"

namespace bc {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t row_count(const NormGeom &g)
{
    return g.idx ? (uint32_t)*g.count * (uint32_t)(g.bh * g.bw) : g.rows;
}

// Sums of N values over the L lanes of a row: part of a wave, or two or four waves (through
// `lds`, their slots, free for reuse after the next sum's barrier; the whole workgroup calls).
template <int L, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (&lds)[N][4])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane_sum<(L < 64 ? L : 64)>(v[i]);
    if constexpr (L > 64) {
        static_assert(L == 128 || L == 256, "a row belongs to a wave's lanes, to two waves or to four");
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[i][threadIdx.x % L >> 6] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lds[i][0] + lds[i][1];
            if constexpr (L == 256) v[i] += lds[i][2] + lds[i][3];
        }
    }
}

// Which elements of a row a lane holds: vector v covers [at, at + VEC), the first `skip` of
// them belonging to a neighbour (all of them where the row has no such vector).
struct Span {
    int at, skip;
};

template <int VEC, int L, bool FULL>
__device__ __forceinline__ Span span_of(int v, int c)
{
    const int lane = threadIdx.x % L, begin = (v * L + lane) * VEC;
    if constexpr (FULL) return {begin, 0};
    if (begin >= c) return {max(0, c - VEC), VEC};
    const int at = min(begin, c - VEC);
    return {at, begin - at};
}

// Gains (or offsets) of a lane's columns. Rows of one vector per lane keep them in registers;
// longer rows read them again for each row, from the L1, and leave the registers to rows in
// flight (the pointer is made opaque, or the compiler would keep them all the same).
template <int VEC>
__device__ __forceinline__ void load_columns(const float *p, int at, float other, float (&out)[VEC])
{
    if (p) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[j] = p[at + j];
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[j] = other;
    }
}

__device__ __forceinline__ const float *again(const float *p)
{
    asm volatile("" : "+s"(p));
    return p;
}

// Rows of several 16-bit vectors stay as stored between the passes: the words are made opaque, or the
// compiler would keep the converted values too, at twice the registers.
template <int FMT, int VEC, int NV>
__device__ __forceinline__ void keep_stored(Raw<FMT, VEC> (&r)[NV])
{
    if constexpr (FMT != kF32 && NV >= 2) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(r[v].w[i]));
    }
}

// ---------------------------------------------------------------- forward

template <int FMT, int VEC, int L, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void k_norm(const void *x, const float *__restrict__ gamma,
                                                   const float *__restrict__ beta, const void *res,
                                                   void *out, NormGeom g)
{
    constexpr int kGroups = kThreads / L;
    constexpr bool kKeep = NV <= 2;                       // gains and offsets in registers
    __shared__ float sums[L > 64 ? kGroups : 1][2][1][4];
    const int group = threadIdx.x / L;
    auto &lds = sums[L > 64 ? group : 0];
    const uint32_t rows = row_count(g);
    Span sp[NV];
    float ga[kKeep ? NV : 1][VEC], be[kKeep ? NV : 1][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        sp[v] = span_of<VEC, L, FULL>(v, g.c);
        if constexpr (kKeep) {
            load_columns(gamma, sp[v].at, 1.f, ga[v]);
            load_columns(beta, sp[v].at, 0.f, be[v]);
        }
    }
    // the workgroup's groups take neighbouring rows, all of them as many turns (a barrier may
    // be in them): past the last row a group reads the last one again and keeps nothing
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < rows; r0 += gridDim.x * kGroups) {
        const bool live = r0 + group < rows;
        const size_t base = (size_t)row_pixel(g, live ? r0 + group : rows - 1) * g.c;
        Raw<FMT, VEC> rx[NV], rr[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) rx[v] = load_raw<FMT, VEC>(x, base + sp[v].at);
        if (res)
#pragma unroll
            for (int v = 0; v < NV; ++v) rr[v] = load_raw<FMT, VEC>(res, base + sp[v].at);
        float s[1] = {0.f}, q[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += FULL || j >= sp[v].skip ? get(rx[v], j) : 0.f;
        row_sum<L>(s, lds[0]);
        const float mean = s[0] / (float)g.c;
        keep_stored(rx);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = get(rx[v], j) - mean;
                q[0] += FULL || j >= sp[v].skip ? d * d : 0.f;
            }
        row_sum<L>(q, lds[1]);
        const float rstd = rsqrtf(q[0] * g.inv_c + g.eps);
        keep_stored(rx);
        const float *gp = gamma, *bp = beta;
        if constexpr (!kKeep) gp = again(gamma), bp = again(beta);
        if (!live) continue;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!FULL && sp[v].skip == VEC) continue;
            auto &gain = ga[kKeep ? v : 0], &offset = be[kKeep ? v : 0];
            if constexpr (!kKeep) {
                load_columns(gp, sp[v].at, 1.f, gain);
                load_columns(bp, sp[v].at, 0.f, offset);
            }
            float y[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                y[j] = (get(rx[v], j) - mean) * rstd * gain[j] + offset[j];
                if (res) y[j] += get(rr[v], j);
                // a NaN passes (fmaxf would drop it)
                if (g.relu) y[j] = y[j] < 0.f ? 0.f : y[j];
            }
            store_raw<FMT, VEC>(out, base + sp[v].at, pack<FMT, VEC>(y));
        }
    }
}

// A row longer than a workgroup's registers: three passes over it, the last two from the L2.
template <int FMT>
__global__ __launch_bounds__(kThreads) void k_norm_long(const void *x, const float *__restrict__ gamma,
                                                        const float *__restrict__ beta, const void *res,
                                                        void *out, NormGeom g)
{
    __shared__ float lds[2][1][4];
    const uint32_t rows = row_count(g), c = g.c;           // i passes 31 bits behind the last channels
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const size_t base = (size_t)row_pixel(g, r) * g.c;
        float s[1] = {0.f}, q[1] = {0.f};
        for (uint32_t i = threadIdx.x; i < c; i += kThreads) s[0] += get(load_raw<FMT, 1>(x, base + i), 0);
        row_sum<kThreads>(s, lds[0]);
        const float mean = s[0] / (float)g.c;
        for (uint32_t i = threadIdx.x; i < c; i += kThreads) {
            const float d = get(load_raw<FMT, 1>(x, base + i), 0) - mean;
            q[0] += d * d;
        }
        row_sum<kThreads>(q, lds[1]);
        const float rstd = rsqrtf(q[0] * g.inv_c + g.eps);
        for (uint32_t i = threadIdx.x; i < c; i += kThreads) {
            float y[1] = {(get(load_raw<FMT, 1>(x, base + i), 0) - mean) * rstd * (gamma ? gamma[i] : 1.f) +
                          (beta ? beta[i] : 0.f)};
            if (res) y[0] += get(load_raw<FMT, 1>(res, base + i), 0);
            if (g.relu) y[0] = y[0] < 0.f ? 0.f : y[0];
            store_raw<FMT, 1>(out, base + i, pack<FMT, 1>(y));
        }
    }
}

// ---------------------------------------------------------------- backward

// dy behind a ReLU: the stored bits where y > 0, zero elsewhere (a NaN there is not used).
template <int FMT, int VEC>
__device__ __forceinline__ Raw<FMT, VEC> masked(Raw<FMT, VEC> dy, const Raw<FMT, VEC> &y)
{
    if constexpr (FMT == kF32 || VEC == 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (!(get(y, j) > 0.f)) dy.w[j] = 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = get(y, 2 * i) > 0.f ? 0xFFFFu : 0u, hi = get(y, 2 * i + 1) > 0.f ? 0xFFFF0000u : 0u;
            dy.w[i] &= lo | hi;
        }
    }
    return dy;
}

// Threads of a workgroup whose rows take L lanes with NV vectors each
template <int L, int NV> constexpr int kGradThreads = NV == 8 ? 256 : 512;

// Sum over the lanes of a wave that hold the same columns (groups of L lanes).
template <int L>
__device__ __forceinline__ float group_sum(float v)
{
    if constexpr (L <= 8) v += dpp<0x128>(v);            // row_ror 8: lane ^ 8
    if constexpr (L <= 16) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (L <= 32) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// One row's stored vectors of a lane, requested together.
template <int FMT, int VEC, int NV>
struct GradRow {
    Raw<FMT, VEC> x[NV], dy[NV], y[NV];

    __device__ __forceinline__ void load(const NormGradArgs &a, const Span (&sp)[NV], size_t base)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            x[v] = load_raw<FMT, VEC>(a.x, base + sp[v].at);
            dy[v] = load_raw<FMT, VEC>(a.dy, base + sp[v].at);
        }
        if (a.y)
#pragma unroll
            for (int v = 0; v < NV; ++v) y[v] = load_raw<FMT, VEC>(a.y, base + sp[v].at);
    }
};

// Partial sums of dgamma and dbeta: [workgroup][2][c] in `part`. The next row is requested
// before the present one is worked on (but for rows that fill the registers).
template <int FMT, int VEC, int L, int NV, bool FULL>
__global__ __launch_bounds__((kGradThreads<L, NV>)) void k_norm_grad(NormGradArgs a, NormGeom g, float *__restrict__ part)
{
    constexpr int T = kGradThreads<L, NV>, kGroups = T / L, kWaves = T / 64;
    constexpr bool kAhead = NV <= 4;
    constexpr bool kKeep = NV <= 2;                       // gains in registers
    __shared__ float sum1[L > 64 ? kGroups : 1][1][4], sum3[L > 64 ? kGroups : 1][3][4];
    const int group = threadIdx.x / L;
    Span sp[NV];
    float sg[NV][VEC], sb[NV][VEC], ga[kKeep ? NV : 1][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        sp[v] = span_of<VEC, L, FULL>(v, g.c);
        if constexpr (kKeep) load_columns(a.gamma, sp[v].at, 1.f, ga[v]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sg[v][j] = sb[v][j] = 0.f;
    }
    // every group takes as many turns as the workgroup (a barrier may be in them); past the
    // last row a group reads the last one again and keeps nothing
    auto base_of = [&](uint32_t r) { return (size_t)min(r, g.rows - 1) * g.c; };
    const uint32_t stride = gridDim.x * kGroups;
    GradRow<FMT, VEC, NV> row, next;
    next.load(a, sp, base_of(blockIdx.x * kGroups + group));
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < g.rows; r0 += stride) {
        const uint32_t r = r0 + group;
        const size_t base = base_of(r);
        row = next;
        if (kAhead && r0 + stride < g.rows) next.load(a, sp, base_of(r + stride));
        // behind a ReLU: from here on row.dy holds dy'
        if (a.y)
#pragma unroll
            for (int v = 0; v < NV; ++v) row.dy[v] = masked(row.dy[v], row.y[v]);
        float one[1] = {0.f}, three[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) one[0] += FULL || j >= sp[v].skip ? get(row.x[v], j) : 0.f;
        row_sum<L>(one, sum1[L > 64 ? group : 0]);
        const float mean = one[0] / (float)g.c;
        keep_stored(row.x);
        const float *gp = a.gamma;
        if constexpr (!kKeep) gp = again(gp);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            auto &gain = ga[kKeep ? v : 0];
            if constexpr (!kKeep) load_columns(gp, sp[v].at, 1.f, gain);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const bool mine = FULL || j >= sp[v].skip;
                const float d = mine ? get(row.x[v], j) - mean : 0.f, gr = mine ? get(row.dy[v], j) * gain[j] : 0.f;
                three[0] += d * d;
                three[1] += gr;
                three[2] += gr * d;
            }
        }
        row_sum<L>(three, sum3[L > 64 ? group : 0]);
        const float rstd = rsqrtf(three[0] * g.inv_c + g.eps), mean_g = three[1] * g.inv_c;
        const float mean_gx = three[2] * rstd * g.inv_c;
        keep_stored(row.x);
        keep_stored(row.dy);
        if (r < g.rows) {
            if constexpr (!kKeep) gp = again(gp);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!FULL && sp[v].skip == VEC) continue;
                auto &gain = ga[kKeep ? v : 0];
                if constexpr (!kKeep) load_columns(gp, sp[v].at, 1.f, gain);
                float dx[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    // the difference first: x rstd - mean rstd would leave the rounding of mean rstd
                    // in xhat (0.06 in a row of one value 4096.3), or pass fp32's range
                    const float xhat = (get(row.x[v], j) - mean) * rstd, dy = get(row.dy[v], j);
                    dx[j] = rstd * (dy * gain[j] - (xhat * mean_gx + mean_g));
                    sg[v][j] += dy * xhat;
                    sb[v][j] += dy;
                }
                store_raw<FMT, VEC>(a.dx, base + sp[v].at, pack<FMT, VEC>(dx));
                if (a.dres) store_raw<FMT, VEC>(a.dres, base + sp[v].at, row.dy[v]);
            }
        }
        if (!kAhead && r0 + stride < g.rows) next.load(a, sp, base_of(r + stride));
    }
    if (!part) return;
    // a wave's groups by register exchanges, then the waves (or groups) through LDS, in
    // their order: side by side for one vector per lane, else one after the other
    extern __shared__ float cols[];                       // [waves or 1][2][c]
    constexpr bool kApart = NV == 1 && L <= 64;
    constexpr int kTurns = kApart ? 1 : T / (L < 64 ? 64 : L);
    const int turn_of = threadIdx.x / (L < 64 ? 64 : L);
    if constexpr (L < 64)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sg[v][j] = group_sum<L>(sg[v][j]);
                sb[v][j] = group_sum<L>(sb[v][j]);
            }
    float *mine = cols + (kApart ? (threadIdx.x >> 6) * 2 * g.c : 0);
    for (int turn = 0; turn < kTurns; ++turn) {
        if (turn) __syncthreads();
        if ((!kApart && turn_of != turn) || (L < 64 && (threadIdx.x & 63) >= L)) continue;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (!FULL && j < sp[v].skip) continue;
                const int i = sp[v].at + j;
                mine[i] = (turn ? mine[i] : 0.f) + sg[v][j];
                mine[g.c + i] = (turn ? mine[g.c + i] : 0.f) + sb[v][j];
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * g.c; i += T) {
        float s = cols[i];
        if constexpr (kApart)
            for (int w = 1; w < kWaves; ++w) s += cols[w * 2 * g.c + i];
        part[(size_t)blockIdx.x * 2 * g.c + i] = s;
    }
}

// Rows longer than a workgroup's registers: their mean, rstd, mean(g) and mean(g xhat) first,
template <int FMT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_stats(NormGradArgs a, NormGeom g, float4 *__restrict__ stats)
{
    __shared__ float lds[2][2][4];
    const uint32_t c = g.c;
    for (uint32_t r = blockIdx.x; r < g.rows; r += gridDim.x) {
        const size_t base = (size_t)r * g.c;
        auto x_at = [&](uint32_t i) { return get(load_raw<FMT, 1>(a.x, base + i), 0); };
        auto g_at = [&](uint32_t i) {
            if (a.y && !(get(load_raw<FMT, 1>(a.y, base + i), 0) > 0.f)) return 0.f;
            return get(load_raw<FMT, 1>(a.dy, base + i), 0) * (a.gamma ? a.gamma[i] : 1.f);
        };
        float one[2] = {0.f, 0.f}, two[2] = {0.f, 0.f};
        for (uint32_t i = threadIdx.x; i < c; i += kThreads) {
            one[0] += x_at(i);
            one[1] += g_at(i);
        }
        row_sum<kThreads>(one, lds[0]);
        const float mean = one[0] / (float)g.c, mean_g = one[1] * g.inv_c;
        for (uint32_t i = threadIdx.x; i < c; i += kThreads) {
            const float d = x_at(i) - mean;
            two[0] += d * d;
            two[1] += g_at(i) * d;
        }
        row_sum<kThreads>(two, lds[1]);
        const float rstd = rsqrtf(two[0] * g.inv_c + g.eps);
        const float mean_gx = two[1] * rstd * g.inv_c;
        if (threadIdx.x == 0) stats[r] = make_float4(mean, rstd, mean_g, mean_gx);
    }
}

// then dx and the column sums, one column per thread over a run of rows.
template <int FMT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_cols(NormGradArgs a, NormGeom g,
                                                             const float4 *__restrict__ stats, float *__restrict__ part)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= (uint32_t)g.c) return;
    const float ga = a.gamma ? a.gamma[i] : 1.f;
    float sg = 0.f, sb = 0.f;
    for (uint32_t r = blockIdx.y; r < g.rows; r += gridDim.y) {
        const size_t at = (size_t)r * g.c + i;
        const float4 st = stats[r];
        float dy[1] = {get(load_raw<FMT, 1>(a.dy, at), 0)};
        if (a.y && !(get(load_raw<FMT, 1>(a.y, at), 0) > 0.f)) dy[0] = 0.f;
        const float xhat = (get(load_raw<FMT, 1>(a.x, at), 0) - st.x) * st.y;
        float dx[1] = {st.y * (dy[0] * ga - st.z - xhat * st.w)};
        sg += dy[0] * xhat;
        sb += dy[0];
        store_raw<FMT, 1>(a.dx, at, pack<FMT, 1>(dx));
        if (a.dres) store_raw<FMT, 1>(a.dres, at, pack<FMT, 1>(dy));
    }
    if (part) {
        part[(size_t)blockIdx.y * 2 * g.c + i] = sg;
        part[(size_t)blockIdx.y * 2 * g.c + g.c + i] = sb;
    }
}

// Adds the partial rows in their order: 32 of the 2 c columns per workgroup, from `first` on, and
// 32 runs of rows each (each summed in order), then the runs in order. (Columns as such count to
// 2^32; in turns of a loop instead of several launches for them the kernel took 0.3 us more.)
constexpr int kRuns = 32;
__global__ __launch_bounds__(32 * kRuns) void k_norm_grad_join(const float *__restrict__ part, int parts, uint32_t c, uint32_t first,
                                                               float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                               int accumulate)
{
    __shared__ float lds[kRuns][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const uint32_t cols = 2 * c, i = first + blockIdx.x * 32 + lane;
    const int each = (parts + kRuns - 1) / kRuns, lo = run * each, hi = min(parts, lo + each);
    float s = 0.f;
    if (i < cols)
#pragma unroll 8
        for (int p = lo; p < hi; ++p) s += part[(size_t)p * cols + i];
    lds[run][lane] = s;
    __syncthreads();
    if (run || i >= cols) return;
    for (int k = 1; k < kRuns; ++k) s += lds[k][lane];
    float *to = i < c ? dgamma : dbeta;
    if (!to) return;
    to += i < c ? i : i - c;
    *to = accumulate ? *to + s : s;
}

// Its launches: one of 2^32 threads or more does not take place.
void launch_join(const float *part, int parts, uint32_t c, float *dgamma, float *dbeta, int accumulate, hipStream_t s)
{
    constexpr uint32_t kMost = 1 << 21;                   // workgroups, 2^31 threads
    const uint32_t groups = (uint32_t)(((uint64_t)2 * c + 31) / 32);
    for (uint32_t at = 0; at < groups; at += kMost)
        hipLaunchKernelGGL(k_norm_grad_join, dim3(std::min(kMost, groups - at)), dim3(32 * kRuns), 0, s, part, parts, c,
                           at * 32, dgamma, dbeta, accumulate);
}

// ---------------------------------------------------------------- choice of form

// Calls f(vector elements, lanes per row, vectors per lane, full) with the form for rows of
// c elements, or returns false where a row exceeds a workgroup's registers. The fewest lanes
// that hold a row in one vector each, or 256 lanes with the fewest vectors. With other forms,
// us forward and backward: 32768 rows of 64 in bf16 with 8 lanes 3.9 and 8.8, with 64 lanes
// 11.9 and 23.1; 16384 of 1024 with 128 lanes 13.4 and 27.3, with 256 21.0 and 42.4; 16384 of
// 4096 held in registers 49 and 88, in three passes 168 and 399.
template <int FMT, typename F>
bool with_form(int c, F &&f)
{
    constexpr int V = kVec<FMT>;
    auto go = [&](auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value;
        if (c == L * NV * V) f(std::integral_constant<int, V>{}, lanes, vecs, std::true_type{});
        else f(std::integral_constant<int, V>{}, lanes, vecs, std::false_type{});
    };
    using std::integral_constant;
    if (c < V) {
        f(integral_constant<int, 1>{}, integral_constant<int, 8>{}, integral_constant<int, 1>{}, std::false_type{});
        return true;
    }
    const int nv = c / V + (c % V != 0);
    auto with = [&](auto lanes, auto vecs) { go(lanes, vecs); return true; };
    using one = integral_constant<int, 1>;
    using wave = integral_constant<int, 64>;
    using group = integral_constant<int, 256>;
    if (nv <= 8) return with(integral_constant<int, 8>{}, one{});
    if (nv <= 16) return with(integral_constant<int, 16>{}, one{});
    if (nv <= 32) return with(integral_constant<int, 32>{}, one{});
    if (nv <= 64) return with(wave{}, one{});
    if (nv <= 128) return with(integral_constant<int, 128>{}, one{});
    if (nv <= 256) return with(group{}, one{});
    if (nv <= 512) return with(group{}, integral_constant<int, 2>{});
    if (nv <= 1024) return with(group{}, integral_constant<int, 4>{});
    if (nv <= 2048) return with(group{}, integral_constant<int, 8>{});
    return false;
}

// Workgroups of the forward pass at most. Every pixel: 32 per CU, of which eight run (16384 rows
// of 4096 in fp16 57 us with 2048 workgroups, 51 with 4096, 49 with 8192, 53 with one per
// row; 30000 of 3000 88, 76, 71 and 80). Active blocks, whose number only the device knows:
// 8 per CU, for those without work cost more than they bring (38 of 128 blocks of
// 32 x 32 x 256: 11.0 us with 2048, 12.4 with 8192).
unsigned most_groups(const NormGeom &g) { return g.idx ? 2048 : 8192; }

constexpr int kLongParts = 64;

// Workgroups of the backward pass, each with a partial row; *held: its form keeps the row.
unsigned parts_of(int fmt, uint32_t rows, int c, bool *held)
{
    return with_format(fmt, [&](auto f) {
        unsigned parts = std::min<uint32_t>(rows, kLongParts);
        *held = with_form<decltype(f)::value>(c, [&](auto, auto lanes, auto vecs, auto) {
            constexpr int L = decltype(lanes)::value, kGroups = kGradThreads<L, decltype(vecs)::value> / L;
            // 512, two per CU, where each has two turns at least (32768 rows of 64: 9.8 us
            // with 512, 9.0 with 256) and rows leave room for two (4096 of 8192: 74 and 61)
            const unsigned most = decltype(vecs)::value <= 2 && rows / (2 * kGroups) > 256 ? 512 : 256;
            parts = std::min<uint32_t>({(rows + kGroups - 1) / kGroups, most, std::max(256u, rows / (2 * kGroups))});
        });
        return parts;
    });
}

}  // namespace

hipError_t launch_norm(const void *x, const float *gamma, const float *beta, const void *res, void *out,
                       const NormGeom &g, int fmt, hipStream_t s)
{
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        const bool held = with_form<FMT>(g.c, [&](auto vec, auto lanes, auto vecs, auto full) {
            constexpr int L = decltype(lanes)::value;
            const unsigned grid = std::min<uint32_t>((g.rows + kThreads / L - 1) / (kThreads / L), most_groups(g));
            hipLaunchKernelGGL((k_norm<FMT, decltype(vec)::value, L, decltype(vecs)::value, decltype(full)::value>),
                               dim3(grid), dim3(kThreads), 0, s, x, gamma, beta, res, out, g);
        });
        if (!held)
            hipLaunchKernelGGL(k_norm_long<FMT>, dim3(std::min<uint32_t>(g.rows, most_groups(g))), dim3(kThreads), 0, s,
                               x, gamma, beta, res, out, g);
        return hipGetLastError();
    });
}

size_t norm_grad_work(int fmt, uint32_t rows, int c)
{
    bool held = false;
    const size_t parts = parts_of(fmt, rows, c, &held);
    return (held ? 0 : (size_t)rows * sizeof(float4)) + parts * 2 * c * sizeof(float);
}

hipError_t launch_norm_grad(const NormGradArgs &a, float *dgamma, float *dbeta, int accumulate, void *work,
                            const NormGeom &g, int fmt, hipStream_t s)
{
    bool held = false;
    const unsigned parts = parts_of(fmt, g.rows, g.c, &held);
    const bool sums = dgamma || dbeta;
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        hipError_t e = hipSuccess;
        float *part = sums ? (float *)work : nullptr;
        with_form<FMT>(g.c, [&](auto vec, auto lanes, auto vecs, auto full) {
            constexpr int L = decltype(lanes)::value, NV = decltype(vecs)::value;
            auto kern = k_norm_grad<FMT, decltype(vec)::value, L, NV, decltype(full)::value>;
            const size_t tables = !sums ? 0 : NV == 1 && L <= 64 ? kGradThreads<L, NV> / 64 : 1;
            const size_t lds = tables * 2 * g.c * sizeof(float);
            if ((e = allow_lds((const void *)kern, lds)) == hipSuccess)
                hipLaunchKernelGGL(kern, dim3(parts), dim3(kGradThreads<L, NV>), lds, s, a, g, part);
        });
        if (e != hipSuccess) return e;
        if (!held) {
            float4 *stats = (float4 *)work;
            part = sums ? (float *)(stats + g.rows) : nullptr;
            hipLaunchKernelGGL(k_norm_grad_stats<FMT>, dim3(std::min<uint32_t>(g.rows, most_groups(g))), dim3(kThreads), 0,
                               s, a, g, stats);
            hipLaunchKernelGGL(k_norm_grad_cols<FMT>, dim3(((uint32_t)g.c + kThreads - 1) / kThreads, parts), dim3(kThreads), 0,
                               s, a, g, stats, part);
        }
        if (sums)
            launch_join(part, (int)parts, (uint32_t)g.c, dgamma, dbeta, accumulate, s);
        return hipGetLastError();
    });
}

}  // namespace bc
