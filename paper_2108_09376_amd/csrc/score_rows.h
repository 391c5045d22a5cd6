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

// A barrier for what passes through LDS alone: stores to memory need not be done by then, as
// __syncthreads would have it.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
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

// The largest of the elements seen. 16-bit ones are compared two at once as integers: among signed
// ones a number that is not negative is right; where all are negative, the smallest unsigned one is
// the largest number.
template <int FMT>
struct Largest {
    typedef short S2 __attribute__((ext_vector_type(2)));
    typedef unsigned short U2 __attribute__((ext_vector_type(2)));
    float f = -kInf;
    S2 up = {(short)0x8000, (short)0x8000};
    U2 low = {0xFFFF, 0xFFFF};

    __device__ __forceinline__ void see(const Raw<FMT, kVec<FMT>> &r)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FMT == kF32) {
                f = fmaxf(f, __uint_as_float(r.w[i]));
            } else {
                up = __builtin_elementwise_max(up, __builtin_bit_cast(S2, r.w[i]));
                low = __builtin_elementwise_min(low, __builtin_bit_cast(U2, r.w[i]));
            }
        }
    }

    // together with one more (a NaN may or may not be passed on)
    __device__ __forceinline__ float with(float other) const
    {
        if constexpr (FMT == kF32) return fmaxf(f, other);
        const short u = up.x > up.y ? up.x : up.y;
        const unsigned short l = low.x < low.y ? low.x : low.y;
        Raw<FMT, 1> r;
        r.w[0] = u >= 0 ? (uint16_t)u : l;
        return fmaxf(l == 0xFFFF && u < 0 ? -kInf : get(r, 0), other);
    }
};

// The statistics of a wave's lanes joined.
template <bool SX>
__device__ __forceinline__ Stats wave_join(const Stats &a, float k2)
{
    const float m = lane_max<64>(a.m), all = m == -kInf ? 0.f : m, f = exp2_of(a.m, all, k2);
    const bool none = a.m == -kInf;                              // its sums are 0, or a NaN
    Stats r = {m, lane_sum<64>(none ? a.s : a.s * f), 0.f};
    if constexpr (SX) r.sx = lane_sum<64>(none ? a.sx : f * (a.sx + fmaxf(a.m - all, -1e30f) * a.s));
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

    // The largest score that this lane holds.
    __device__ __forceinline__ float largest() const
    {
        Largest<FMT> l;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k < used) l.see(v[k]);
            __builtin_amdgcn_sched_barrier(0);
        }
        return l.with(get(t, 0));
    }

    // This lane's sum of exp2((z - m) k2) against the largest score m that it holds.
    __device__ __forceinline__ float own_sum(float m, float k2) const
    {
        const float ref = m == -kInf ? 0.f : m;
        float s = exp2_of(get(t, 0), ref, k2);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k < used)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += exp2_of(get(v[k], j), ref, k2);
            __builtin_amdgcn_sched_barrier(0);
        }
        return s;
    }

    // Statistics over the lanes of a wave that hold the row (all of them if L >= 64).
    template <bool SX, typename M>
    __device__ __forceinline__ Stats stats(const void *, size_t, int len, int, float k2, M masked)
    {
        masked([&](int e) { mask(e, len); });
        return stats<SX>(k2);
    }

    template <bool SX>
    __device__ __forceinline__ Stats stats(float k2)
    {
        constexpr int W = L < 64 ? L : 64;
        const float m = lane_max<W>(largest());
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
    __device__ __forceinline__ void store(const void *, void *out, size_t base, int len, int live, F value) const
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

// A row of any length, passed over twice in memory: nothing of it stays in registers but B vectors of
// a lane at a time. The statistics keep a running maximum, the sums corrected where a batch
// raises it. Same interface as ScoreRow; elements to be masked are told one by one before the
// statistics (`masked` says which the lane has).
template <int FMT, int L, int B>
struct StreamRow {
    static constexpr int VEC = kVec<FMT>;

    static __device__ __forceinline__ int lane() { return threadIdx.x % L; }
    static __device__ __forceinline__ int owner(int e, int len)
    {
        const int nvec = len / VEC, i = e / VEC;
        return i < nvec ? i % L : e - nvec * VEC;
    }

    // The batch of vectors from v0 on: -inf past the live ones.
    static __device__ __forceinline__ void load(Raw<FMT, VEC> (&r)[B], const void *x, size_t base, int v0, int here, int live)
    {
        if (v0 + B * L <= here) {
#pragma unroll
            for (int k = 0; k < B; ++k) r[k] = load_raw<FMT, VEC>(x, base + (size_t)(v0 + k * L + lane()) * VEC);
        } else {
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const int i = v0 + k * L + lane();
                r[k] = masked_raw<FMT, VEC>();
                if (i < here) r[k] = load_raw<FMT, VEC>(x, base + (size_t)i * VEC);
                if (i < here && (i + 1) * VEC > live)
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (i * VEC + j >= live) mask_elem<FMT, VEC>(r[k], j);
            }
        }
    }

    // masked(f): calls f(e) for every element of the row that this lane holds and that is to count as -inf.
    template <bool SX, typename M>
    static __device__ __forceinline__ Stats stats(const void *x, size_t base, int len, int live, float k2, M masked)
    {
        const int nvec = len / VEC, here = min(nvec, (live + VEC - 1) / VEC), last = nvec * VEC + lane();
        float m = -kInf, ref = 0.f, s = 0.f, sx = 0.f;
        for (int v0 = 0; v0 < here; v0 += B * L) {
            Raw<FMT, VEC> r[B];
            load(r, x, base, v0, here, live);
            masked([&](int e) {
                const int i = e / VEC - v0, word = FMT == kF32 ? e % VEC : e % VEC >> 1;
                const uint32_t keep = FMT == kF32 ? 0u : e & 1 ? 0xFFFFu : 0xFFFF0000u;
#pragma unroll
                for (int k = 0; k < B; ++k)
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        r[k].w[w] = i == k * L + lane() && w == word && e < nvec * VEC
                                        ? (r[k].w[w] & keep) | (kMaskedWord<FMT> & ~keep) : r[k].w[w];
            });
            Largest<FMT> l;
#pragma unroll
            for (int k = 0; k < B; ++k) l.see(r[k]);
            const float up = l.with(m);
            const float to = up == -kInf ? 0.f : up, f = exp2_of(m, to, k2);
            if constexpr (SX) sx = f * (sx + fmaxf(m - to, -1e30f) * s);
            s *= f;
            m = up;
            ref = to;
#pragma unroll
            for (int k = 0; k < B; ++k) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = get(r[k], j) - ref, e = __builtin_amdgcn_exp2f(d * k2);
                    s += e;
                    if constexpr (SX) sx += e * fmaxf(d, -1e30f);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        Stats one = {-kInf, 0.f, 0.f};
        if (last < len && last < live) {
            float z = get(load_raw<FMT, 1>(x, base + last), 0);
            masked([&](int e) { z = e == last ? -kInf : z; });
            one = {z, z == -kInf ? 0.f : 1.f, 0.f};
            if (z != z) one = {-kInf, z, z};                     // a NaN is in the sums, not in the maximum
        }
        const Stats mine = join<SX>({m, s, sx}, one, k2);
        return wave_join<SX>(mine, k2);
    }

    // out[base + e] = value(score e), 0 at `live` and beyond; out may be x.
    template <typename F>
    static __device__ __forceinline__ void store(const void *x, void *out, size_t base, int len, int live, F value)
    {
        const int nvec = len / VEC, here = min(nvec, (live + VEC - 1) / VEC), last = nvec * VEC + lane();
        for (int v0 = 0; v0 < nvec; v0 += B * L) {
            Raw<FMT, VEC> r[B];
            load(r, x, base, v0, here, live);
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const int i = v0 + k * L + lane();
                if (i < nvec) {
                    float y[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) y[j] = value(get(r[k], j));
                    if ((i + 1) * VEC > live)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) y[j] = i * VEC + j < live ? y[j] : 0.f;
                    store_raw<FMT, VEC>(out, base + (size_t)i * VEC, pack<FMT, VEC>(y));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (last < len) {
            const float y[1] = {last < live ? value(get(load_raw<FMT, 1>(x, base + last), 0)) : 0.f};
            store_raw<FMT, 1>(out, base + last, pack<FMT, 1>(y));
        }
    }

    static __device__ __forceinline__ void store_zeros(void *out, size_t base, int len)
    {
        const int nvec = len / VEC, last = nvec * VEC + lane();
        const Raw<FMT, VEC> z = {};
        const Raw<FMT, 1> z1 = {};
        for (int i = lane(); i < nvec; i += L) store_raw<FMT, VEC>(out, base + (size_t)i * VEC, z);
        if (last < len) store_raw<FMT, 1>(out, base + last, z1);
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
// workgroup from 128 on) and vectors of each, 0 for a row of any length, which is not held.
constexpr int kPixelClasses = 32;
struct Form {
    int lanes, nv;
};
constexpr Form kForms[] = {{1, 0}, {8, 1}, {32, 1}, {64, 2}, {64, 8}, {256, 8}, {512, 8}, {1024, 8}, {1024, 0}};
constexpr int kFormCount = 8, kChunkForm = 5, kSmallChunk = -1;

template <int L> constexpr int kThreadsOf = L <= 64 ? 256 : L;
template <int L> constexpr int kGroupsOf = L <= 64 ? 256 / L : 1;  // rows of a workgroup

// NV = 0: rows of any length, of which a workgroup passes over its own twice.
template <int FMT, int L, int NV>
using RowOf = std::conditional_t<NV == 0, StreamRow<FMT, L, 4>, ScoreRow<FMT, L, NV ? NV : 1>>;

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

// Statistics of a row over its workgroup (L > 64; through lds, known to the first wave only,
// after a barrier that every thread passes), or over its lanes.
template <int L, bool SX>
__device__ __forceinline__ Stats team_stats(Stats st, Stats *lds, float k2)
{
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = st;
        lds_barrier();
        if (threadIdx.x < 64) {
            st = {-kInf, 0.f, 0.f};
            if (threadIdx.x < L / 64) st = lds[threadIdx.x];
            st = wave_join<SX>(st, k2);
        }
    }
    return st;
}

// Statistics of a row from those of its chunks, by a whole wave.
template <bool SX>
__device__ __forceinline__ Stats row_stats(const float4 *part, int chunks, float k2)
{
    Stats st = {-kInf, 0.f, 0.f};
    for (int i = threadIdx.x & 63; i < chunks; i += 64) {
        const float4 p = part[i];
        st = join<SX>(st, {p.x, p.y, p.z}, k2);
    }
    return wave_join<SX>(st, k2);
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
    default: return f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
    }
}

// f(lanes, vectors) of a chunk.
template <typename F>
hipError_t with_chunk(int form, F &&f)
{
    constexpr std::integral_constant<int, kForms[kChunkForm].lanes> lanes{};
    if (form == kSmallChunk) return f(lanes, std::integral_constant<int, 2>{});
    return f(lanes, std::integral_constant<int, kForms[kChunkForm].nv>{});
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

    // All requests before the first use: the conditions are the same for every pixel.
    __device__ __forceinline__ void load(const void *x, size_t base, int c, int classes)
    {
        if ((classes + VEC - 1) / VEC * VEC <= c) {
            Raw<FMT, VEC> r[N / VEC];
#pragma unroll
            for (int v = 0; v < N / VEC; ++v) {
                r[v] = masked_raw<FMT, VEC>();
                if (v * VEC < classes) r[v] = load_raw<FMT, VEC>(x, base + v * VEC);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = j < classes ? get(r[j / VEC], j % VEC) : -kInf;
        } else {
            Raw<FMT, 1> r[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                r[j] = masked_raw<FMT, 1>();
                if (j < classes) r[j] = load_raw<FMT, 1>(x, base + j);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = get(r[j], 0);
        }
    }
};

// The scores of a pixel of up to 32 classes over four lanes, eight to a lane; -inf past its classes.
template <int FMT>
struct QuadScores {
    static constexpr int VEC = kVec<FMT>, NV = 8 / VEC;
    float z[8];

    static __device__ __forceinline__ int first() { return (threadIdx.x & 3) * 8; }

    __device__ __forceinline__ void load(const void *x, size_t base, int c, int classes)
    {
        Raw<FMT, VEC> r[NV];
        Raw<FMT, 1> e[8];
        const int at = first();
        const bool whole = c % VEC == 0;                         // the same for every pixel
        if (whole) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                r[v] = masked_raw<FMT, VEC>();
                if (at + v * VEC < classes) r[v] = load_raw<FMT, VEC>(x, base + at + v * VEC);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = masked_raw<FMT, 1>();
                if (at + j < classes) e[j] = load_raw<FMT, 1>(x, base + at + j);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = at + j < classes ? (whole ? get(r[j / VEC], j % VEC) : get(e[j], 0)) : -kInf;
    }

    // y where there are classes, 0 in the row's other channels
    static __device__ __forceinline__ void store(void *out, size_t base, int c, int classes, float (&y)[8])
    {
        const int at = first();
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = at + j < classes ? y[j] : 0.f;
        if (c % VEC == 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = y[v * VEC + j];
                if (at + v * VEC < c) store_raw<FMT, VEC>(out, base + at + v * VEC, pack<FMT, VEC>(w));
            }
            const Raw<FMT, VEC> zero = {};
            for (int i = 32 + (threadIdx.x & 3) * VEC; i < c; i += 4 * VEC) store_raw<FMT, VEC>(out, base + i, zero);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w[1] = {y[j]};
                if (at + j < c) store_raw<FMT, 1>(out, base + at + j, pack<FMT, 1>(w));
            }
            const Raw<FMT, 1> zero = {};
            for (int i = 32 + (threadIdx.x & 3); i < c; i += 4) store_raw<FMT, 1>(out, base + i, zero);
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
