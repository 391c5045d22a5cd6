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

// Pixels of the map that a call runs on.
__device__ __forceinline__ uint32_t pixel_count(const TopArgs &a, const ScoreGeom &g)
{
    return a.idx ? (uint32_t)*a.count * (uint32_t)(a.bh * a.bw) : g.images * g.hw;
}

// Rows of a few lanes: each entry is the largest key below the last.
template <int FMT, int L>
__global__ __launch_bounds__(256) void k_top_lanes(TopArgs a, ScoreGeom g)
{
    constexpr int G = kGroupsOf<L>, VEC = kVec<FMT>;
    const uint32_t r = item_of() * G + threadIdx.x / L;
    if (r >= pixel_count(a, g)) return;
    const size_t px = row_pixel(a, r);
    ScoreRow<FMT, L, 1> row;
    row.load(a.x, px * (size_t)g.c, g.len, g.classes);
    const int lane = row.lane(), nvec = g.len / VEC, tail = nvec * VEC + lane;
    Key key[VEC + 1], last = ~(Key)0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) key[j] = lane < nvec && lane * VEC + j < g.classes ? key_of(get(row.v[0], j), lane * VEC + j) : 0;
    key[VEC] = tail < g.classes ? key_of(get(row.t, 0), tail) : 0;
    for (int i = 0; i < a.k; ++i) {
        Key top = 0;
#pragma unroll
        for (int j = 0; j <= VEC; ++j) top = key[j] < last && key[j] > top ? key[j] : top;
        last = lane_max_key<L>(top);
        if (lane == 0) put<FMT>(a, px * a.k + i, last);
    }
    if (!a.rest) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (key[j] >= last) mask_elem<FMT, VEC>(row.v[0], j);
    if (key[VEC] >= last) row.t = masked_raw<FMT, 1>();
    const Stats st = row.template stats<false>(kLog2e * a.inv_t);
    if (lane == 0) a.rest[px] = rest_of(a, st);
}

// Rows of a wave or a workgroup. Every wave finds the q-th largest of its lanes' maxima, q
// enough that all waves together have k; the least of these is a score that at least k scores reach,
// and few more than that do. Those that reach it are collected in LDS, and each one's place among
// them is the number of larger keys. Where more reach it than LDS holds (long runs of equal
// scores, parts of a row masked out), or fewer than k (NaN), the record is found by rounds.
constexpr int kCandidates = 1024;

template <int FMT, int L, int NV, int PASS>
__global__ __launch_bounds__(L, L > 64 ? 8 : 4) void k_top(TopArgs a, ScoreGeom g)
{
    using Row = ScoreRow<FMT, L, NV>;
    constexpr int VEC = kVec<FMT>, W = L / 64;
    __shared__ __attribute__((aligned(16))) Key cand[kCandidates];
    __shared__ Key record[64];
    __shared__ Key best[W];
    __shared__ float least[W];
    __shared__ Stats waves[W];
    __shared__ int head[L], next[64], count;
    uint32_t r = item_of();
    int chunk = 0;
    if constexpr (PASS == kFirst) {
        const uint32_t i = r;
        r = div(i, g.by_chunks);
        chunk = (int)(i - r * (uint32_t)g.chunks);
    }
    if (r >= pixel_count(a, g)) return;
    const size_t px = row_pixel(a, r);
    const Chunk c = chunk_of<PASS>(g, px, chunk);
    Row row;
    row.load(a.x, c.base, c.len, c.live);
    const int lane = Row::lane(), nvec = c.len / VEC, k = min(a.k, c.live);
    head[lane] = 0;
    if (lane == 0) count = 0;

    float m = get(row.t, 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (v < row.used)
#pragma unroll
            for (int j = 0; j < VEC; ++j) m = fmaxf(m, get(row.v[v], j));
        __builtin_amdgcn_sched_barrier(0);
    }
    row.keep();
    // waves whose lanes all hold a vector
    const int full = min(W, nvec / 64);
    float bar = -kInf;
    if (full) {
        float x = m;
        const int q = (k + full - 1) / full;
        for (int i = 0; i < q; ++i) {
            bar = lane_max<64>(x);
            const unsigned long long at = __ballot(x == bar);
            if (at && (int)(threadIdx.x & 63) == __ffsll(at) - 1) x = -kInf;
        }
    }
    if ((threadIdx.x & 63) == 0) least[threadIdx.x >> 6] = bar;
    __syncthreads();
    bar = least[0];
    for (int w = 1; w < full; ++w) bar = fminf(bar, least[w]);
    if (m >= bar) {
        auto add = [&](float z, int e) {
            const int at = atomicAdd(&count, 1);
            if (at < kCandidates) cand[at] = key_of(z, c.off + e);
        };
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = (v * L + lane) * VEC;
            uint32_t hit = 0;
            if (v < row.used && v * L + lane < nvec)
#pragma unroll
                for (int j = 0; j < VEC; ++j) hit |= get(row.v[v], j) >= bar && at + j < c.live ? 1u << j : 0u;
            if (hit)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (hit >> j & 1) add(get(row.v[v], j), at + j);
            __builtin_amdgcn_sched_barrier(0);
        }
        const int e = nvec * VEC + lane;
        if (e < c.live && get(row.t, 0) >= bar) add(get(row.t, 0), e);
    }
    __syncthreads();
    const int n = count;
    if (n >= k && n <= kCandidates) {
        for (int i = lane; i < n; i += L) {
            const Key mine = cand[i];
            int place = 0;
            for (int o = 0; o < n; ++o) place += cand[o] > mine;
            if (place < k) {
                record[place] = mine;
                const int e = class_of(mine) - c.off;
                next[place] = atomicExch(&head[Row::owner(e, c.len)], place + 1);
            }
        }
        __syncthreads();
    } else {
        // each entry the largest key below the last, over the row in memory: it is seldom needed,
        // and would take the registers from the other way
        Key last = ~(Key)0;
        for (int i = 0; i < k; ++i) {
            Key top = 0;
            for (int e = lane; e < c.live; e += L) {
                const Key o = key_of(load_elem(a.x, FMT, c.base + e), c.off + e);
                top = o < last && o > top ? o : top;
            }
            top = lane_max_key<64>(top);
            __syncthreads();
            if ((lane & 63) == 0) best[lane >> 6] = top;
            __syncthreads();
            last = best[0];
            for (int w = 1; w < W; ++w) last = best[w] > last ? best[w] : last;
            if (lane == 0) {
                record[i] = last;
                const int own = Row::owner(class_of(last) - c.off, c.len);
                next[i] = head[own];
                head[own] = i + 1;
            }
        }
        __syncthreads();
    }
    if constexpr (PASS == kFirst) {
        if (lane < a.k) a.keys[((size_t)r * g.chunks + chunk) * a.k + lane] = lane < k ? record[lane] : 0;
    } else {
        if (lane < a.k) put<FMT>(a, px * a.k + lane, record[lane]);
    }
    if (!a.rest) return;
    for (int h = head[lane]; h; h = next[h - 1]) row.mask(class_of(record[h - 1]) - c.off, c.len);
    const Stats st = team_stats<L, false>(row.template stats<false>(kLog2e * a.inv_t), waves, kLog2e * a.inv_t);
    if (lane == 0) {
        if constexpr (PASS == kFirst) a.stats[(size_t)r * g.chunks + chunk] = make_float4(st.m, st.s, 0.f, 0.f);
        else a.rest[px] = rest_of(a, st);
    }
}

// A pixel of few classes to four lanes, eight classes each: k times the largest of what is left. Of
// a 16-bit score the key's upper bits and the class make one 32-bit number, whose next largest is a
// select and a maximum per class. A workgroup is one wave: a frame's active blocks
// spread over the whole device.
template <int FMT>
__global__ __launch_bounds__(64) void k_top_quad(TopArgs a, ScoreGeom g)
{
    using Scores = QuadScores<FMT>;
    const uint32_t total = pixel_count(a, g), r = item_of() * 16 + (threadIdx.x >> 2);
    if (r >= total) return;
    const size_t px = row_pixel(a, r);
    const int lane = threadIdx.x & 3, at = Scores::first();
    Scores own;
    own.load(a.x, px * (size_t)g.c, g.c, g.classes);
    constexpr int kNone = (int)0x80000000u;                      // below every key
    int key[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        key[j] = (int)((uint32_t)(key_of(own.z[j], 0) >> 32) ^ 0x80000000u);
        // a 16-bit score's lowest 16 (bf16) or 13 (fp16) bits as fp32 are 0: room for the class, the
        // lower one on top
        if constexpr (FMT != kF32) key[j] |= 31 - (at + j);
        if (at + j >= g.classes) key[j] = kNone;
    }
    uint32_t taken = 0;                                          // of this lane's eight
    for (int i = 0; i < a.k; ++i) {
        int top = kNone, best = 0;
        if constexpr (FMT != kF32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, taken >> j & 1 ? kNone : key[j]);
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0xB1, 0xF, 0xF, false));
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0x4E, 0xF, 0xF, false));
            best = 31 - (top & 31);
        } else {
#pragma unroll
            for (int j = 7; j >= 0; --j)
                if (!(taken >> j & 1) && key[j] >= top) {
                    top = key[j];
                    best = at + j;
                }
            auto meet = [&](int t, int b) {                      // the larger, of equal ones the lower class
                const bool other = t > top || (t == top && b < best);
                top = other ? t : top;
                best = other ? b : best;
            };
            meet(__builtin_amdgcn_mov_dpp(top, 0xB1, 0xF, 0xF, false), __builtin_amdgcn_mov_dpp(best, 0xB1, 0xF, 0xF, false));
            meet(__builtin_amdgcn_mov_dpp(top, 0x4E, 0xF, 0xF, false), __builtin_amdgcn_mov_dpp(best, 0x4E, 0xF, 0xF, false));
        }
        if (best >> 3 == lane) {                                 // its lane writes it
            taken |= 1u << (best & 7);
            float y[1] = {own.z[0]};
#pragma unroll
            for (int j = 1; j < 8; ++j) y[0] = (best & 7) == j ? own.z[j] : y[0];
            store_raw<FMT, 1>(a.top, px * a.k + i, pack<FMT, 1>(y));
            a.index[px * a.k + i] = best;
        }
    }
    if (!a.rest) return;
    float m = -kInf, s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, taken >> j & 1 ? -kInf : own.z[j]);
    m = lane_max<4>(m);
    const float ref = m == -kInf ? 0.f : m;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += taken >> j & 1 ? 0.f : exp2_of(own.z[j], ref, kLog2e * a.inv_t);
    s = lane_sum<4>(s);
    if (lane == 0) a.rest[px] = rest_of(a, {m, s, 0.f});
}

// The chunks' records of a row joined, by a wave.
template <int FMT>
__global__ __launch_bounds__(64) void k_top_join(TopArgs a, ScoreGeom g)
{
    const float k2 = kLog2e * a.inv_t;
    {
        const size_t r = item_of();
        if (r >= pixel_count(a, g)) return;
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
        if (!a.rest) return;
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
    ScorePlan p = score_plan(g, fmt, 0, false, false, 16);
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
            hipLaunchKernelGGL((k_top<FMT, L, NV, kFirst>), grid_of(rows * g.chunks), dim3(L), 0, s, a, g);
            hipLaunchKernelGGL((k_top_join<FMT>), grid_of(rows), dim3(64), 0, s, a, g);
            return hipGetLastError();
        }
        if (p.form == 0) {
            hipLaunchKernelGGL((k_top_quad<FMT>), grid_of((rows + 15) / 16), dim3(64), 0, s, a, g);
            return hipGetLastError();
        }
        return with_form(p.form, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, NV = decltype(n)::value, G = kGroupsOf<L>;
            if constexpr (NV == 0)
                return hipErrorInvalidValue;                     // not planned here
            else if constexpr (L < 64)
                hipLaunchKernelGGL((k_top_lanes<FMT, L>), grid_of((rows + G - 1) / G), dim3(256), 0, s, a, g);
            else
                hipLaunchKernelGGL((k_top<FMT, L, NV, kWhole>), grid_of(rows), dim3(L), 0, s, a, g);
            return hipGetLastError();
        });
    });
}

}  // namespace bc
