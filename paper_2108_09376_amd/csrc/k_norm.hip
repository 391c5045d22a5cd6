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

// Pixel of row r: itself, or the pixel of an active block.
__device__ __forceinline__ uint32_t row_pixel(const NormGeom &g, uint32_t r)
{
    if (!g.idx) return r;
    const uint32_t bpx = g.bh * g.bw, k = r / bpx, p = r - k * bpx;
    const uint32_t id = g.idx[k], bpi = g.gh * g.gw;
    const uint32_t img = id / bpi, b = id - img * bpi, gy = b / g.gw, gx = b - gy * g.gw;
    const uint32_t py = p / g.bw, px = p - py * g.bw;
    return (img * (g.gh * g.bh) + gy * g.bh + py) * (g.gw * g.bw) + gx * g.bw + px;
}

// Sum over the L lanes of a row: part of a wave, or the workgroup's four waves (through
// `lds`, a slot of four floats that is free for reuse two sums later).
template <int L>
__device__ __forceinline__ float row_sum(float v, float *lds)
{
    if constexpr (L <= 64) {
        return lane_sum<L>(v);
    } else {
        static_assert(L == kThreads, "a row belongs to a wave's lanes or to the workgroup");
        v = lane_sum<64>(v);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        return (lds[0] + lds[1]) + (lds[2] + lds[3]);
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

// ---------------------------------------------------------------- forward

template <int FMT, int VEC, int L, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void k_norm(const void *x, const float *__restrict__ gamma,
                                                   const float *__restrict__ beta, const void *res,
                                                   void *out, NormGeom g)
{
    constexpr int kGroups = kThreads / L;
    __shared__ float lds[2][4];
    const int group = threadIdx.x / L;
    const uint32_t rows = row_count(g);
    Span sp[NV];
    float ga[NV][VEC], be[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        sp[v] = span_of<VEC, L, FULL>(v, g.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            ga[v][j] = gamma ? gamma[sp[v].at + j] : 1.f;
            be[v][j] = beta ? beta[sp[v].at + j] : 0.f;
        }
    }
    // the workgroup's groups take neighbouring rows
    for (uint32_t r = blockIdx.x * kGroups + group; r < rows; r += gridDim.x * kGroups) {
        const size_t base = (size_t)row_pixel(g, r) * g.c;
        Raw<FMT, VEC> rx[NV], rr[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) rx[v] = load_raw<FMT, VEC>(x, base + sp[v].at);
        if (res)
#pragma unroll
            for (int v = 0; v < NV; ++v) rr[v] = load_raw<FMT, VEC>(res, base + sp[v].at);
        float d[NV][VEC], s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                d[v][j] = get(rx[v], j);
                s += FULL || j >= sp[v].skip ? d[v][j] : 0.f;
            }
        const float mean = row_sum<L>(s, lds[0]) / (float)g.c;
        float q = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                d[v][j] -= mean;
                q += FULL || j >= sp[v].skip ? d[v][j] * d[v][j] : 0.f;
            }
        const float rstd = 1.f / sqrtf(row_sum<L>(q, lds[1]) * g.inv_c + g.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!FULL && sp[v].skip == VEC) continue;
            float y[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                y[j] = d[v][j] * rstd * ga[v][j] + be[v][j];
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
    __shared__ float lds[2][4];
    const uint32_t rows = row_count(g);
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const size_t base = (size_t)row_pixel(g, r) * g.c;
        float s = 0.f, q = 0.f;
        for (int i = threadIdx.x; i < g.c; i += kThreads) s += get(load_raw<FMT, 1>(x, base + i), 0);
        const float mean = row_sum<kThreads>(s, lds[0]) / (float)g.c;
        for (int i = threadIdx.x; i < g.c; i += kThreads) {
            const float d = get(load_raw<FMT, 1>(x, base + i), 0) - mean;
            q += d * d;
        }
        const float rstd = 1.f / sqrtf(row_sum<kThreads>(q, lds[1]) * g.inv_c + g.eps);
        for (int i = threadIdx.x; i < g.c; i += kThreads) {
            float y[1] = {(get(load_raw<FMT, 1>(x, base + i), 0) - mean) * rstd * (gamma ? gamma[i] : 1.f) +
                          (beta ? beta[i] : 0.f)};
            if (res) y[0] += get(load_raw<FMT, 1>(res, base + i), 0);
            if (g.relu) y[0] = y[0] < 0.f ? 0.f : y[0];
            store_raw<FMT, 1>(out, base + i, pack<FMT, 1>(y));
        }
    }
}

// ---------------------------------------------------------------- backward

// Partial sums of dgamma and dbeta: [workgroup][2][c] in `part`.
template <int FMT, int VEC, int L, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void k_norm_grad(NormGradArgs a, NormGeom g, float *__restrict__ part)
{
    constexpr int kGroups = kThreads / L;
    __shared__ float lds[4][4];
    const int group = threadIdx.x / L;
    Span sp[NV];
    float ga[NV][VEC], sg[NV][VEC], sb[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        sp[v] = span_of<VEC, L, FULL>(v, g.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            ga[v][j] = a.gamma ? a.gamma[sp[v].at + j] : 1.f;
            sg[v][j] = sb[v][j] = 0.f;
        }
    }
    for (uint32_t r = blockIdx.x * kGroups + group; r < g.rows; r += gridDim.x * kGroups) {
        const size_t base = (size_t)r * g.c;
        Raw<FMT, VEC> rx[NV], rd[NV], ry[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            rx[v] = load_raw<FMT, VEC>(a.x, base + sp[v].at);
            rd[v] = load_raw<FMT, VEC>(a.dy, base + sp[v].at);
        }
        if (a.y)
#pragma unroll
            for (int v = 0; v < NV; ++v) ry[v] = load_raw<FMT, VEC>(a.y, base + sp[v].at);
        float d[NV][VEC], dy[NV][VEC], s = 0.f, t = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const bool mine = FULL || j >= sp[v].skip;
                d[v][j] = get(rx[v], j);
                dy[v][j] = get(rd[v], j);
                if (a.y && !(get(ry[v], j) > 0.f)) dy[v][j] = 0.f;
                s += mine ? d[v][j] : 0.f;
                t += mine ? dy[v][j] * ga[v][j] : 0.f;
            }
        const float mean = row_sum<L>(s, lds[0]) / (float)g.c;
        const float mean_g = row_sum<L>(t, lds[1]) * g.inv_c;
        float q = 0.f, u = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const bool mine = FULL || j >= sp[v].skip;
                d[v][j] -= mean;
                q += mine ? d[v][j] * d[v][j] : 0.f;
                u += mine ? dy[v][j] * ga[v][j] * d[v][j] : 0.f;
            }
        const float rstd = 1.f / sqrtf(row_sum<L>(q, lds[2]) * g.inv_c + g.eps);
        const float mean_gx = row_sum<L>(u, lds[3]) * rstd * g.inv_c;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!FULL && sp[v].skip == VEC) continue;
            float dx[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float xhat = d[v][j] * rstd;
                dx[j] = rstd * (dy[v][j] * ga[v][j] - mean_g - xhat * mean_gx);
                sg[v][j] += dy[v][j] * xhat;
                sb[v][j] += dy[v][j];
            }
            store_raw<FMT, VEC>(a.dx, base + sp[v].at, pack<FMT, VEC>(dx));
            if (a.dres) store_raw<FMT, VEC>(a.dres, base + sp[v].at, pack<FMT, VEC>(dy[v]));
        }
    }
    if (!part) return;
    // the groups' sums, one after the other in LDS, then one row of the partial table
    extern __shared__ float cols[];                       // [2][c]
    for (int turn = 0; turn < kGroups; ++turn) {
        __syncthreads();
        if (group != turn) continue;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (!FULL && j < sp[v].skip) continue;
                const int i = sp[v].at + j;
                cols[i] = (turn ? cols[i] : 0.f) + sg[v][j];
                cols[g.c + i] = (turn ? cols[g.c + i] : 0.f) + sb[v][j];
            }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * g.c; i += kThreads) part[(size_t)blockIdx.x * 2 * g.c + i] = cols[i];
}

// Rows longer than a workgroup's registers: their mean, rstd, mean(g) and mean(g xhat) first,
template <int FMT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_stats(NormGradArgs a, NormGeom g, float4 *__restrict__ stats)
{
    __shared__ float lds[4][4];
    for (uint32_t r = blockIdx.x; r < g.rows; r += gridDim.x) {
        const size_t base = (size_t)r * g.c;
        auto x_at = [&](int i) { return get(load_raw<FMT, 1>(a.x, base + i), 0); };
        auto g_at = [&](int i) {
            if (a.y && !(get(load_raw<FMT, 1>(a.y, base + i), 0) > 0.f)) return 0.f;
            return get(load_raw<FMT, 1>(a.dy, base + i), 0) * (a.gamma ? a.gamma[i] : 1.f);
        };
        float s = 0.f, t = 0.f, q = 0.f, u = 0.f;
        for (int i = threadIdx.x; i < g.c; i += kThreads) {
            s += x_at(i);
            t += g_at(i);
        }
        const float mean = row_sum<kThreads>(s, lds[0]) / (float)g.c;
        const float mean_g = row_sum<kThreads>(t, lds[1]) * g.inv_c;
        for (int i = threadIdx.x; i < g.c; i += kThreads) {
            const float d = x_at(i) - mean;
            q += d * d;
            u += g_at(i) * d;
        }
        const float rstd = 1.f / sqrtf(row_sum<kThreads>(q, lds[2]) * g.inv_c + g.eps);
        const float mean_gx = row_sum<kThreads>(u, lds[3]) * rstd * g.inv_c;
        if (threadIdx.x == 0) stats[r] = make_float4(mean, rstd, mean_g, mean_gx);
    }
}

// then dx and the column sums, one column per thread over a run of rows.
template <int FMT>
__global__ __launch_bounds__(kThreads) void k_norm_grad_cols(NormGradArgs a, NormGeom g,
                                                             const float4 *__restrict__ stats, float *__restrict__ part)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= g.c) return;
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

// Adds the partial rows in their order: 32 columns per workgroup, eight runs of rows each
// (each summed in order), then the runs in order.
__global__ __launch_bounds__(kThreads) void k_norm_grad_join(const float *__restrict__ part, int parts, int c,
                                                             float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                             int accumulate)
{
    __shared__ float lds[8][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    const int each = (parts + 7) / 8, lo = run * each, hi = min(parts, lo + each);
    float s = 0.f;
    if (i < 2 * c)
        for (int p = lo; p < hi; ++p) s += part[(size_t)p * 2 * c + i];
    lds[run][lane] = s;
    __syncthreads();
    if (run || i >= 2 * c) return;
    for (int k = 1; k < 8; ++k) s += lds[k][lane];
    float *to = i < c ? dgamma : dbeta;
    if (!to) return;
    to += i < c ? i : i - c;
    *to = accumulate ? *to + s : s;
}

// ---------------------------------------------------------------- choice of form

// Calls f(vector elements, lanes per row, vectors per lane, full) with the form for rows of
// c elements, or returns false where a row exceeds a workgroup's registers.
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
    const int nv = (c + V - 1) / V;
    if (nv <= 8) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (nv <= 16) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (nv <= 32) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (nv <= 64) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (nv <= 128) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (nv <= 256) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (nv <= 512) go(integral_constant<int, kThreads>{}, integral_constant<int, 2>{});
    else if (nv <= 1024) go(integral_constant<int, kThreads>{}, integral_constant<int, 4>{});
    else if (nv <= 2048) go(integral_constant<int, kThreads>{}, integral_constant<int, 8>{});
    else return false;
    return true;
}

constexpr unsigned kMostForward = 2048;      // eight workgroups per CU
constexpr unsigned kMostBackward = 512;
constexpr int kLongParts = 64;

// Rows per workgroup and turn of the form for rows of c elements; 0: the long form.
int row_groups(int fmt, int c)
{
    const int v = fmt == kF32 ? kVec<kF32> : kVec<kBF16>;
    if (c < v) return 32;
    const int nv = (c + v - 1) / v;
    if (nv <= 8) return 32;
    if (nv <= 16) return 16;
    if (nv <= 32) return 8;
    if (nv <= 256) return 4;
    return nv <= 2048 ? 1 : 0;
}

unsigned parts_of(int fmt, uint32_t rows, int c)
{
    const int groups = row_groups(fmt, c);
    if (!groups) return std::min<uint32_t>(rows, kLongParts);
    return std::min<uint32_t>((rows + groups - 1) / groups, kMostBackward);
}

}  // namespace

hipError_t launch_norm(const void *x, const float *gamma, const float *beta, const void *res, void *out,
                       const NormGeom &g, int fmt, hipStream_t s)
{
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        const bool held = with_form<FMT>(g.c, [&](auto vec, auto lanes, auto vecs, auto full) {
            constexpr int L = decltype(lanes)::value;
            const unsigned grid = std::min<uint32_t>((g.rows + kThreads / L - 1) / (kThreads / L), kMostForward);
            hipLaunchKernelGGL((k_norm<FMT, decltype(vec)::value, L, decltype(vecs)::value, decltype(full)::value>),
                               dim3(grid), dim3(kThreads), 0, s, x, gamma, beta, res, out, g);
        });
        if (!held)
            hipLaunchKernelGGL(k_norm_long<FMT>, dim3(std::min<uint32_t>(g.rows, kMostForward)), dim3(kThreads), 0, s,
                               x, gamma, beta, res, out, g);
        return hipGetLastError();
    });
}

size_t norm_grad_work(int fmt, uint32_t rows, int c)
{
    const size_t stats = row_groups(fmt, c) ? 0 : (size_t)rows * sizeof(float4);
    return stats + (size_t)parts_of(fmt, rows, c) * 2 * c * sizeof(float);
}

hipError_t launch_norm_grad(const NormGradArgs &a, float *dgamma, float *dbeta, int accumulate, void *work,
                            const NormGeom &g, int fmt, hipStream_t s)
{
    const unsigned parts = parts_of(fmt, g.rows, g.c);
    const bool sums = dgamma || dbeta;
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        hipError_t e = hipSuccess;
        float *part = sums ? (float *)work : nullptr;
        const size_t lds = sums ? (size_t)2 * g.c * sizeof(float) : 0;
        const bool held = with_form<FMT>(g.c, [&](auto vec, auto lanes, auto vecs, auto full) {
            auto kern = k_norm_grad<FMT, decltype(vec)::value, decltype(lanes)::value, decltype(vecs)::value,
                                    decltype(full)::value>;
            if ((e = allow_lds((const void *)kern, lds)) == hipSuccess)
                hipLaunchKernelGGL(kern, dim3(parts), dim3(kThreads), lds, s, a, g, part);
        });
        if (e != hipSuccess) return e;
        if (!held) {
            float4 *stats = (float4 *)work;
            part = sums ? (float *)(stats + g.rows) : nullptr;
            hipLaunchKernelGGL(k_norm_grad_stats<FMT>, dim3(std::min<uint32_t>(g.rows, kMostForward)), dim3(kThreads), 0,
                               s, a, g, stats);
            hipLaunchKernelGGL(k_norm_grad_cols<FMT>, dim3((g.c + kThreads - 1) / kThreads, parts), dim3(kThreads), 0,
                               s, a, g, stats, part);
        }
        if (sums)
            hipLaunchKernelGGL(k_norm_grad_join, dim3((2 * g.c + 31) / 32), dim3(kThreads), 0, s, part, (int)parts,
                               g.c, dgamma, dbeta, accumulate);
        return hipGetLastError();
    });
}

}  // namespace bc
