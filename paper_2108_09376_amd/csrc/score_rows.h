// Rows of class scores in registers, and what the kernels on score maps share: the maximum
// and the sum of exponentials of a row over the lanes that hold it.
#pragma once

#include <algorithm>

#include "bc_internal.h"
#include "rows.h"

namespace bc {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

// -inf as stored, in one element or twice in a word.
template <int FMT> constexpr uint32_t kMaskedWord = FMT == kF32 ? 0xFF800000u : FMT == kBF16 ? 0xFF80FF80u : 0xFC00FC00u;
template <int FMT> constexpr uint32_t kMaskedElem = FMT == kF32 ? kMaskedWord<FMT> : kMaskedWord<FMT> & 0xFFFFu;

template <int FMT, int VEC>
__device__ __forceinline__ Raw<FMT, VEC> masked_raw()
{
    Raw<FMT, VEC> r;
    if constexpr (VEC == 1) r.w[0] = kMaskedElem<FMT>;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = kMaskedWord<FMT>;
    return r;
}

// Element j (known at compile time after unrolling) of a stored vector to -inf.
template <int FMT, int VEC>
__device__ __forceinline__ void mask_elem(Raw<FMT, VEC> &r, int j)
{
    if constexpr (FMT == kF32 || VEC == 1) r.w[j] = kMaskedElem<FMT>;
    else r.w[j >> 1] = j & 1 ? (r.w[j >> 1] & 0xFFFFu) | (kMaskedWord<FMT> & 0xFFFF0000u)
                             : (r.w[j >> 1] & 0xFFFF0000u) | (kMaskedWord<FMT> & 0xFFFFu);
}

template <int L>
__device__ __forceinline__ float lane_max(float v)
{
    if constexpr (L >= 2) v = fmaxf(v, dpp<0xB1>(v));
    if constexpr (L >= 4) v = fmaxf(v, dpp<0x4E>(v));
    if constexpr (L >= 8) v = fmaxf(v, dpp<0x141>(v));
    if constexpr (L >= 16) v = fmaxf(v, dpp<0x140>(v));
    if constexpr (L >= 32) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (L >= 64) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}

// What a wave knows of a row, or of its part: the maximum, the sum of exp2((z - max) k2),
// and the sum of those times (z - max) where an entropy is wanted. Nothing above -inf: the
// maximum is -inf and the sums are 0.
struct Stats {
    float m, s, sx;
};

__device__ __forceinline__ float exp2_of(float z, float m, float k2) { return __builtin_amdgcn_exp2f((z - m) * k2); }

// b's part of the row added to a's.
template <bool SX>
__device__ __forceinline__ Stats join(const Stats &a, const Stats &b, float k2)
{
    const float m = fmaxf(a.m, b.m);
    const float fa = a.m == -kInf ? 0.f : exp2_of(a.m, m, k2), fb = b.m == -kInf ? 0.f : exp2_of(b.m, m, k2);
    Stats r = {m, a.s * fa + b.s * fb, 0.f};
    if constexpr (SX) {
        // a distance past fp32's range belongs to a factor of 0
        const float da = fmaxf(a.m - m, -1e30f), db = fmaxf(b.m - m, -1e30f);
        r.sx = fa * (a.sx + da * a.s) + fb * (b.sx + db * b.s);
    }
    return r;
}

// A row, or a chunk of it, held by L lanes of a wave (or by a workgroup of L threads) in NV
// vectors of 16 bytes each and one element of the row's last len % VEC. Vector i of the row
// is v[i / L] of lane i % L. Elements at `live` and beyond are -inf and are not read.
template <int FMT, int L, int NV>
struct ScoreRow {
    static constexpr int VEC = kVec<FMT>;
    Raw<FMT, VEC> v[NV];
    Raw<FMT, 1> t;
    int used;                                  // vectors of a lane that some lane has a score in

    static __device__ __forceinline__ int lane() { return threadIdx.x % L; }
    // the lane that holds element e
    static __device__ __forceinline__ int owner(int e, int len)
    {
        const int nvec = len / VEC, i = e / VEC;
        return i < nvec ? i % L : e - nvec * VEC;
    }

    __device__ __forceinline__ void load(const void *x, size_t base, int len, int live)
    {
        const int nvec = len / VEC, here = min(nvec, (live + VEC - 1) / VEC);
        if (here == NV * L) {
#pragma unroll
            for (int k = 0; k < NV; ++k) v[k] = load_raw<FMT, VEC>(x, base + (size_t)(k * L + lane()) * VEC);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                v[k] = masked_raw<FMT, VEC>();
                if (k * L + lane() < here) v[k] = load_raw<FMT, VEC>(x, base + (size_t)(k * L + lane()) * VEC);
            }
        }
        const int e = nvec * VEC + lane();
        t = masked_raw<FMT, 1>();
        if (e < len && e < live) t = load_raw<FMT, 1>(x, base + e);
        if (live < len)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int at = (k * L + lane()) * VEC;
                if (at < live && at + VEC > live)
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (at + j >= live) mask_elem<FMT, VEC>(v[k], j);
            }
        used = (here + L - 1) / L;
    }

    // Between two passes over a row it stays as stored: the words are made opaque, or the compiler
    // would keep the converted values too, at twice the registers.
    __device__ __forceinline__ void keep()
    {
        if constexpr (FMT != kF32 && NV >= 2) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(v[k].w[i]));
        }
    }

    // Element e of a row that this lane holds to -inf.
    __device__ __forceinline__ void mask(int e, int len)
    {
        const int nvec = len / VEC, i = e / VEC, at = i / L;
        if (i >= nvec) {
            t = masked_raw<FMT, 1>();
            return;
        }
        // selects, not branches: the compiler would turn those into an array in memory
        const int word = FMT == kF32 ? e % VEC : e % VEC >> 1;
        const uint32_t keep = FMT == kF32 ? 0u : e & 1 ? 0xFFFFu : 0xFFFF0000u;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = v[k].w[i];
                v[k].w[i] = k == at && i == word ? (w & keep) | (kMaskedWord<FMT> & ~keep) : w;
            }
    }

    // Statistics over the lanes of a wave that hold the row (all of them if L >= 64).
    template <bool SX>
    __device__ __forceinline__ Stats stats(float k2)
    {
        constexpr int W = L < 64 ? L : 64;
        float m = get(t, 0);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k < used)
#pragma unroll
                for (int j = 0; j < VEC; ++j) m = fmaxf(m, get(v[k], j));
            __builtin_amdgcn_sched_barrier(0);
        }
        m = lane_max<W>(m);
        keep();
        const float ref = m == -kInf ? 0.f : m;
        float s = 0.f, sx = 0.f;
        auto add = [&](float z) {
            const float x = z - ref, e = __builtin_amdgcn_exp2f(x * k2);
            s += e;
            if constexpr (SX) sx += e * fmaxf(x, -1e30f);   // e = 0 at -inf
        };
        add(get(t, 0));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k < used)
#pragma unroll
                for (int j = 0; j < VEC; ++j) add(get(v[k], j));
            __builtin_amdgcn_sched_barrier(0);
        }
        keep();
        s = lane_sum<W>(s);
        if constexpr (SX) sx = lane_sum<W>(sx);
        return {m, s, sx};
    }

    // out[base + e] = value(score e) for every element of the row, 0 at `live` and beyond.
    template <typename F>
    __device__ __forceinline__ void store(void *out, size_t base, int len, int live, F value) const
    {
        const int nvec = len / VEC;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = k * L + lane(), at = i * VEC;
            if (i >= nvec) continue;
            float y[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) y[j] = value(get(v[k], j));
            if (at + VEC > live)
#pragma unroll
                for (int j = 0; j < VEC; ++j) y[j] = at + j < live ? y[j] : 0.f;
            store_raw<FMT, VEC>(out, base + at, pack<FMT, VEC>(y));
            __builtin_amdgcn_sched_barrier(0);
        }
        const int e = nvec * VEC + lane();
        if (e < len) {
            const float y[1] = {e < live ? value(get(t, 0)) : 0.f};
            store_raw<FMT, 1>(out, base + e, pack<FMT, 1>(y));
        }
    }

    static __device__ __forceinline__ void store_zeros(void *out, size_t base, int len)
    {
        const int nvec = len / VEC;
        Raw<FMT, VEC> z = {};
        Raw<FMT, 1> z1 = {};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = k * L + lane();
            if (i < nvec) store_raw<FMT, VEC>(out, base + (size_t)i * VEC, z);
        }
        const int e = nvec * VEC + lane();
        if (e < len) store_raw<FMT, 1>(out, base + e, z1);
    }
};

// One element of any format, told at run time.
__device__ __forceinline__ float load_elem(const void *p, int fmt, size_t i)
{
    if (fmt == kF32) return ((const float *)p)[i];
    if (fmt == kBF16) return get(load_raw<kBF16, 1>(p, i), 0);
    return get(load_raw<kF16, 1>(p, i), 0);
}

// Forms of a row: a thread to itself (up to kPixelClasses scores); or lanes (threads of a
// workgroup from 128 on) and vectors of each.
constexpr int kPixelClasses = 32;
struct Form {
    int lanes, nv;
};
constexpr Form kForms[] = {{1, 0}, {8, 1}, {32, 1}, {64, 2}, {64, 8}, {256, 8}, {512, 8}, {1024, 8}, {1024, 16}};
constexpr int kFormCount = 9, kChunkForm = 5;

template <int L> constexpr int kThreadsOf = L <= 64 ? 256 : L;
template <int L> constexpr int kGroupsOf = L <= 64 ? 256 / L : 1;  // rows of a workgroup

// Which part of the work a launch does: whole rows; a chunk's statistics; a chunk's gradient.
enum Pass { kWhole, kFirst, kSecond };

// A workgroup's rows (or chunk of a row) in the map.
struct Chunk {
    size_t row, base;                          // row of the map, its first element (of the chunk)
    int off, len, live;                        // first class, elements, class scores
};

template <int PASS>
__device__ __forceinline__ Chunk chunk_of(const ScoreGeom &g, size_t row, int chunk)
{
    Chunk c = {row, row * (size_t)g.c, 0, g.len, g.classes};
    if constexpr (PASS != kWhole) {
        c.off = chunk * g.chunk;
        c.len = min(g.chunk, g.len - c.off);
        c.live = max(0, min(g.classes - c.off, c.len));
        c.base += c.off;
    }
    return c;
}

// Statistics of a row over its workgroup (L > 64; through lds, read by the first wave only,
// after a barrier that every thread passes), or over its lanes.
template <int L, bool SX>
__device__ __forceinline__ Stats team_stats(Stats st, Stats *lds, float k2)
{
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = st;
        __syncthreads();
        if (threadIdx.x < 64) {
            st = lds[0];
#pragma unroll
            for (int i = 1; i < L / 64; ++i) st = join<SX>(st, lds[i], k2);
        }
    }
    return st;
}

// A chunk's statistics of all chunks of a row, by the first wave.
template <bool SX>
__device__ __forceinline__ Stats row_stats(const float4 *part, int chunks, float k2)
{
    Stats st = {-kInf, 0.f, 0.f};
    for (int i = 0; i < chunks; ++i) {
        const float4 p = part[i];
        st = join<SX>(st, {p.x, p.y, p.z}, k2);
    }
    return st;
}

// A launch of any number of workgroups below 2^32, and a workgroup's own number.
inline dim3 grid_of(size_t items)
{
    const unsigned x = (unsigned)std::min<size_t>(std::max<size_t>(items, 1), 1u << 16);
    return dim3(x, (unsigned)((items + x - 1) / x));
}

__device__ __forceinline__ uint32_t item_of() { return blockIdx.y * gridDim.x + blockIdx.x; }

// f(lanes, vectors) of a form of rows that lanes share, as integral constants.
template <typename F>
hipError_t with_form(int form, F &&f)
{
    using std::integral_constant;
    switch (form) {
    case 1: return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    case 2: return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    case 3: return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    case 4: return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    case 5: return f(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    case 6: return f(integral_constant<int, 512>{}, integral_constant<int, 8>{});
    case 7: return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
    default: return f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
    }
}

// f(classes of a pixel in registers, as an integral constant).
template <typename F>
hipError_t with_pixel(int classes, F &&f)
{
    if (classes <= 8) return f(std::integral_constant<int, 8>{});
    if (classes <= 16) return f(std::integral_constant<int, 16>{});
    if (classes <= 24) return f(std::integral_constant<int, 24>{});
    return f(std::integral_constant<int, 32>{});
}

// The scores of a thread's own pixel, -inf past its classes.
template <int FMT, int N>
struct PixelScores {
    static constexpr int VEC = kVec<FMT>;
    float z[N];

    __device__ __forceinline__ void load(const void *x, size_t base, int c, int classes)
    {
#pragma unroll
        for (int at = 0; at < N; at += VEC) {
            if (at >= classes) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) z[at + j] = -kInf;
            } else if (at + VEC <= c) {
                const Raw<FMT, VEC> r = load_raw<FMT, VEC>(x, base + at);
#pragma unroll
                for (int j = 0; j < VEC; ++j) z[at + j] = at + j < classes ? get(r, j) : -kInf;
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    z[at + j] = at + j < classes ? get(load_raw<FMT, 1>(x, base + at + j), 0) : -kInf;
            }
        }
    }
};

// Rows [first, first + rows) of `out`, c elements each, by a workgroup of 256 threads:
// value(row, j) for j < classes, 0 past them. by_out: by the vectors of a row, or its elements if it is not
// whole vectors.
template <int FMT, typename F>
__device__ __forceinline__ void store_pixels(void *out, size_t first, uint32_t rows, int c, int classes, const Divisor &by_out,
                                             F value)
{
    auto go = [&](auto w) {
        constexpr int W = decltype(w)::value;
        const uint32_t per = (uint32_t)c / W;
        for (uint32_t f = threadIdx.x; f < rows * per; f += 256) {
            const uint32_t r = div(f, by_out), at = (f - r * per) * W;
            float y[W];
#pragma unroll
            for (int j = 0; j < W; ++j) y[j] = (int)at + j < classes ? value(r, (int)at + j) : 0.f;
            store_raw<FMT, W>(out, (first + r) * (size_t)c + at, pack<FMT, W>(y));
        }
    };
    if (c % kVec<FMT> == 0) go(std::integral_constant<int, kVec<FMT>>{});
    else go(std::integral_constant<int, 1>{});
}

}  // namespace bc
