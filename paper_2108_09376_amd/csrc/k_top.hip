// A teacher's record of a score map: the k largest scores of each pixel with their classes, and
// the logarithm of the sum of exp(score / temperature) over the others.
//
// Scores are compared as integer keys of the same order (the bits, negative numbers reversed,
// -0 as 0); a key and the complement of the class are one 64-bit number, larger for the larger
// score and, among equal ones, for the lower class. The next entry of a record is the largest
// such number below the last.
#include "score_rows.h"

namespace bc {
namespace {

using Key = unsigned long long;

__device__ __forceinline__ Key key_of(float z, int cls)
{
    const int x = __float_as_int(z), s = x >> 31;
    const uint32_t order = (uint32_t)(((x & 0x7FFFFFFF) ^ s) - s) ^ 0x80000000u;
    return (Key)order << 32 | (0xFFFFFFFFu - (uint32_t)cls);
}

__device__ __forceinline__ float score_of(Key k)
{
    const int o = (int)((uint32_t)(k >> 32) ^ 0x80000000u);
    return __int_as_float(o < 0 ? (int)(0x80000000u | (uint32_t)-o) : o);
}

__device__ __forceinline__ int class_of(Key k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

template <int W>
__device__ __forceinline__ Key lane_max_key(Key k)
{
    for (int d = 1; d < W; d <<= 1) {
        const Key o = __shfl_xor(k, d, W);
        k = o > k ? o : k;
    }
    return k;
}

template <int FMT>
__device__ __forceinline__ void put(const TopArgs &a, size_t at, Key k)
{
    const float y[1] = {score_of(k)};
    store_raw<FMT, 1>(a.top, at, pack<FMT, 1>(y));
    a.index[at] = class_of(k);
}

__device__ __forceinline__ float rest_of(const TopArgs &a, const Stats &st)
{
    return st.s == 0.f ? -kInf : st.m * a.inv_t + __logf(st.s);
}

template <int FMT, int L, int NV, int PASS>
__global__ __launch_bounds__((kThreadsOf<L>)) void k_top(TopArgs a, ScoreGeom g)
{
    using Row = ScoreRow<FMT, L, NV>;
    constexpr int VEC = kVec<FMT>, T = kThreadsOf<L>, G = L <= 64 ? T / L : 1, W = L < 64 ? L : 64;
    __shared__ Key best[L > 64 ? L / 64 : 1];
    __shared__ Stats waves[L > 64 ? L / 64 : 1];
    const int group = L <= 64 ? threadIdx.x / L : 0;
    const float k2 = kLog2e * a.inv_t;
    const size_t rows = a.idx ? (size_t)*a.count * (size_t)(a.bh * a.bw) : (size_t)g.images * g.hw;
    const size_t items = PASS == kWhole ? (rows + G - 1) / G : rows * g.chunks;
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        const size_t r = PASS == kWhole ? item * G + group : item / g.chunks;
        if (r >= rows) continue;
        const int chunk = PASS == kWhole ? 0 : (int)(item % g.chunks);
        const size_t px = row_pixel(a, (uint32_t)r);
        const Chunk c = chunk_of<PASS>(g, px, chunk);
        Row row;
        row.load(a.x, c.base, c.len, c.live);
        const int nvec = c.len / VEC, lane = Row::lane();
        // f(score, class) of every element that this lane holds
        auto each = [&](auto f) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int e = (v * L + lane) * VEC + j;
                    if (e < c.live && v * L + lane < nvec) f(get(row.v[v], j), c.off + e);
                }
            const int e = nvec * VEC + lane;
            if (e < c.live) f(get(row.t, 0), c.off + e);
        };
        Key last = ~(Key)0;
        for (int i = 0; i < a.k; ++i) {
            Key k = 0;
            each([&](float z, int cls) {
                const Key o = key_of(z, cls);
                k = o < last && o > k ? o : k;
            });
            k = lane_max_key<W>(k);
            if constexpr (L > 64) {
                __syncthreads();
                if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = k;
                __syncthreads();
                for (int w = 0; w < L / 64; ++w) k = best[w] > k ? best[w] : k;
            }
            last = k;
            if (lane == 0) {
                if constexpr (PASS == kFirst) a.keys[item * a.k + i] = k;
                else put<FMT>(a, px * a.k + i, k);
            }
        }
        if (a.rest) {
            each([&](float z, int cls) {
                if (key_of(z, cls) >= last) row.mask(cls - c.off, c.len);
            });
            const Stats st = team_stats<L, false>(row.template stats<false>(k2), waves, k2);
            if (lane == 0) {
                if constexpr (PASS == kFirst) a.stats[item] = make_float4(st.m, st.s, 0.f, 0.f);
                else a.rest[px] = rest_of(a, st);
            }
        }
        if constexpr (L > 64) __syncthreads();
    }
}

// The chunks' records of a row joined, by a wave.
template <int FMT>
__global__ __launch_bounds__(64) void k_top_join(TopArgs a, ScoreGeom g)
{
    const float k2 = kLog2e * a.inv_t;
    const size_t rows = a.idx ? (size_t)*a.count * (size_t)(a.bh * a.bw) : (size_t)g.images * g.hw;
    for (size_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const size_t px = row_pixel(a, (uint32_t)r);
        const Key *keys = a.keys + r * g.chunks * a.k;
        const int n = g.chunks * a.k;
        Key last = ~(Key)0;
        for (int i = 0; i < a.k; ++i) {
            Key k = 0;
            for (int e = threadIdx.x; e < n; e += 64) {
                const Key o = keys[e];
                k = o < last && o > k ? o : k;
            }
            last = lane_max_key<64>(k);
            if (threadIdx.x == 0) put<FMT>(a, px * a.k + i, last);
        }
        if (!a.rest) continue;
        // the others: outside every chunk's record, and inside one but not of this record
        Stats st = {-kInf, 0.f, 0.f};
        for (int i = threadIdx.x; i < g.chunks; i += 64) {
            const float4 p = a.stats[r * g.chunks + i];
            st = join<false>(st, {p.x, p.y, 0.f}, k2);
        }
        for (int e = threadIdx.x; e < n; e += 64)
            if (keys[e] < last && keys[e]) {
                const float z = score_of(keys[e]);
                if (z != -kInf) st = join<false>(st, {z, 1.f, 0.f}, k2);
            }
        const float m = lane_max<64>(st.m);
        const float s = lane_sum<64>(st.m == -kInf ? st.s : st.s * exp2_of(st.m, m, k2));
        if (threadIdx.x == 0) a.rest[px] = rest_of(a, {m, s, 0.f});
    }
}

}  // namespace

ScorePlan top_plan(ScoreGeom &g, int fmt, int k)
{
    ScorePlan p = score_plan(g, fmt, 0, false);
    if (p.split) {
        p.pick = p.bytes;
        p.bytes += (size_t)g.images * g.hw * g.chunks * (size_t)k * sizeof(Key);
    }
    return p;
}

hipError_t launch_top(TopArgs a, ScoreGeom g, const ScorePlan &p, void *work, int fmt, hipStream_t s)
{
    uint8_t *w = (uint8_t *)work;
    a.stats = (float4 *)(w + p.stats);
    a.keys = (unsigned long long *)(w + p.pick);
    const size_t rows = (size_t)g.images * g.hw;
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        if (p.split) {
            constexpr int L = kForms[kChunkForm].lanes, NV = kForms[kChunkForm].nv;
            hipLaunchKernelGGL((k_top<FMT, L, NV, kFirst>), dim3(grid_of(rows * g.chunks)), dim3(L), 0, s, a, g);
            hipLaunchKernelGGL((k_top_join<FMT>), dim3(grid_of(rows)), dim3(64), 0, s, a, g);
            return hipGetLastError();
        }
        return with_form(p.form, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, NV = decltype(n)::value, G = L <= 64 ? kThreadsOf<L> / L : 1;
            hipLaunchKernelGGL((k_top<FMT, L, NV, kWhole>), dim3(grid_of((rows + G - 1) / G)), dim3(kThreadsOf<L>), 0, s, a, g);
            return hipGetLastError();
        });
    });
}

}  // namespace bc
