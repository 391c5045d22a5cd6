// Rows of a channels-last map in registers: element formats, vectors of 16 bytes at any
// element alignment, and sums over the lanes that share a row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace bc {

// Storage formats, numbered as bc_dtype.
constexpr int kF32 = 0, kBF16 = 1, kF16 = 2;

template <int FMT> constexpr int kElem = FMT == kF32 ? 4 : 2;        // bytes per element
template <int FMT> constexpr int kVec = 16 / kElem<FMT>;             // elements per 16 bytes

// 16 bytes at an element's alignment: gfx950 loads and stores four dwords at any byte
// address with one request.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };

template <int FMT, int VEC>
struct Raw {                        // VEC elements as stored: 16 bytes, or one element
    uint32_t w[VEC == 1 ? 1 : 4];
};

template <int FMT, int VEC>
__device__ __forceinline__ Raw<FMT, VEC> load_raw(const void *p, size_t elem)
{
    Raw<FMT, VEC> r;
    const uint8_t *q = (const uint8_t *)p + elem * kElem<FMT>;
    if constexpr (VEC == 1) {
        if constexpr (FMT == kF32) r.w[0] = *(const uint32_t *)q;
        else r.w[0] = *(const uint16_t *)q;
    } else {
        static_assert(VEC == kVec<FMT>, "vectors have 16 bytes");
        const Bytes16 b = *(const Bytes16 *)q;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = b.w[i];
    }
    return r;
}

template <int FMT, int VEC>
__device__ __forceinline__ void store_raw(void *p, size_t elem, const Raw<FMT, VEC> &r)
{
    uint8_t *q = (uint8_t *)p + elem * kElem<FMT>;
    if constexpr (VEC == 1) {
        if constexpr (FMT == kF32) *(uint32_t *)q = r.w[0];
        else *(uint16_t *)q = (uint16_t)r.w[0];
    } else {
        Bytes16 b;
#pragma unroll
        for (int i = 0; i < 4; ++i) b.w[i] = r.w[i];
        *(Bytes16 *)q = b;
    }
}

// Element j of a stored vector as fp32.
template <int FMT, int VEC>
__device__ __forceinline__ float get(const Raw<FMT, VEC> &r, int j)
{
    if constexpr (FMT == kF32) {
        return __uint_as_float(r.w[j]);
    } else {
        const uint32_t d = r.w[j >> 1];
        if constexpr (FMT == kBF16)
            return __uint_as_float(j & 1 ? d & 0xFFFF0000u : d << 16);
        else
            return (float)__builtin_bit_cast(_Float16, (uint16_t)(j & 1 ? d >> 16 : d));
    }
}

// fp32 values to a stored vector, each rounded once to nearest even (NaN stays NaN).
template <int FMT, int VEC>
__device__ __forceinline__ Raw<FMT, VEC> pack(const float (&v)[VEC])
{
    Raw<FMT, VEC> r;
    auto half = [](float f) -> uint32_t {
        if constexpr (FMT == kBF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
        else return __builtin_bit_cast(uint16_t, (_Float16)f);
    };
    if constexpr (FMT == kF32) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) r.w[j] = __float_as_uint(v[j]);
    } else if constexpr (VEC == 1) {
        r.w[0] = half(v[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = half(v[2 * i]) | (half(v[2 * i + 1]) << 16);
    }
    return r;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, false));
}

// Sum over each aligned group of L lanes of a wave, in every lane of the group. The lanes
// meet by exchanges in the register file (within quads, eights, sixteens, then halves).
template <int L>
__device__ __forceinline__ float lane_sum(float v)
{
    if constexpr (L >= 2) v += dpp<0xB1>(v);             // lane ^ 1
    if constexpr (L >= 4) v += dpp<0x4E>(v);             // lane ^ 2
    if constexpr (L >= 8) v += dpp<0x141>(v);            // mirrored within eight
    if constexpr (L >= 16) v += dpp<0x140>(v);           // mirrored within sixteen
    if constexpr (L >= 32) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (L >= 64) {
        const uint32_t u = __float_as_uint(v);
        const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// f(integral_constant of the format) for a bc_dtype.
template <typename F>
auto with_format(int fmt, F &&f)
{
    if (fmt == kF32) return f(std::integral_constant<int, kF32>{});
    if (fmt == kBF16) return f(std::integral_constant<int, kBF16>{});
    return f(std::integral_constant<int, kF16>{});
}

}  // namespace bc
