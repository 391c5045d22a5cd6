// Orthogonalised updates: a matrix G pushed towards the nearest orthogonal matrix by
// Newton-Schulz products, alone or as an optimiser's step (momentum, weights) over many
// weight matrices.
//
//   X_0 = G / (|G|_F + eps), transposed where it has more rows than columns (m <= n);
//   X <- a X + (b A + c A^2) X with A = X X^T, `steps` times; the result is X.
//
// The form computed. With B = (b/a) A + (c/a) A^2 a step is X <- a (I + B) X. B is a
// polynomial of A, so all factors commute, and the next step's A is a^2 (I + B)^2 A: a span
// of k steps can run on the m x m side alone, and one product applies its factor,
//   P <- P + B + B P,   R = A + B A,   A <- a^2 (R + B R),   X <- a^k (X + P X).
// Every product but the last is symmetric: the tiles on and above the diagonal are computed
// and written twice. In units of 2 m^3 operations, five steps in spans of 3 and 2 take
// 3 n/m + 7, in spans of one (products on X in every step) 7.5 n/m + 2.5. Directions of X
// that are small beside the largest lose digits in A as the square of their size, and a
// step multiplies such an error by up to a^2, so a new A is taken from X after three steps, after
// two once the small directions have grown, and after every step where that would still be less
// exact than plain fp32 (steps_direct has the figures).
//
// Arithmetic: an fp32 value x is held as two fp16 numbers, hi = half(x), lo = half(x - hi),
// about 22 bits, all scaled by 2^12, and a product is hi hi + hi lo + lo hi on the matrix
// cores: fp32 accuracy at a third of the fp16 rate, five times the fp32 rate. What is left
// out, lo lo, is below 2^-22 of the product. A matrix instruction rounds its running sum by
// more than an ulp, so the sums of every four chunks of K start at zero and join the tile's
// totals in fp32 (512 x 4608, five steps, difference to 64 bits: 1.7e-6; the textbook form in
// fp32 3.2e-6). Entries stay within 16 (the host has checked the coefficients), as |X|_2 <= 1 at
// the start.
#include <algorithm>
#include <cmath>

#include "bc_internal.h"
#include "lds_dma.h"
#include "rows.h"

namespace bc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;                      // edge of small tiles, and of the first kernel's
constexpr int kPad = 128;                      // matrices are padded to it with zeros
constexpr float kScale = 4096.f;
constexpr int kSpan = 3;                       // most steps between two A taken from X
constexpr int kSumParts = 1024;                // partial sums of squares per matrix at most
constexpr int kSumEach = 8192;                 // and elements of each at least
// Chunks of K per range at least: the sums of a range cost as much as some of its chunks. 8 / 16
// / 32, us: 64 x 4096 100 / 96 / 107, 64 x 2048 88 / 91 / 121, 256 x 2304 108 / 108 / 143, the
// policy network's step 146 / 149 / 175; 128 x 1024 84 / 92 / 93, 1024 x 1280 221 / 191 / 191.
constexpr int kLeastChunks = 16;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The workspace's shared part; the fp32 sums of K ranges follow it.
constexpr int kMostSplit = 1024;               // workgroups of a launch that splits K: 512 and one more per tile
struct OrthHead {
    uint32_t count[kMostSplit];                // arrivals per tile
};
static_assert(sizeof(OrthHead) % 256 == 0, "what follows is aligned");

// A matrix's part of the workspace: partial sums, two X and five squares, each two planes
// (hi, lo) of halves.
struct Slot {
    int m, n;                                  // rows <= columns of X, padded
    bool flip;                                 // X is the transpose
};

__host__ __device__ inline Slot slot_of(int rows, int cols)
{
    const bool flip = rows > cols;
    const int m = flip ? cols : rows, n = flip ? rows : cols, e = kPad;
    return {(m + e - 1) / e * e, (n + e - 1) / e * e, flip};
}

enum Buf { kX0, kX1, kA, kR, kB0, kB1, kP, kNone };

__host__ __device__ inline size_t buf_at(const Slot &s, int b)
{
    const size_t x = (size_t)s.m * s.n * 4, q = (size_t)s.m * s.m * 4, head = kSumParts * sizeof(double);
    return head + (b <= kX1 ? b * x : 2 * x + (b - kA) * q);
}

__host__ __device__ inline size_t slot_bytes(const Slot &s) { return buf_at(s, kNone); }

// Matrices lie in blocks of 32 x 32, row of blocks after row of blocks, each block its hi
// plane (2 KB), then its lo plane, as LDS holds them: a tile's chunk of K is whole blocks,
// which requests to LDS take in order, a kilobyte each. Within a plane the four 16-byte units
// of row r are stored at unit ^ (-(r / 4) mod 4). A read of 16 bytes per lane is served for
// rows 0-3 and 12-15 of one unit with rows 4-11 of the next (and the other way round), a
// transposing one for rows 0-3 and 8-11 (4-7 and 12-15): both then meet every bank once.
constexpr int kBlock = 32, kBlockPlane = kBlock * kBlock * 2, kBlockBytes = 2 * kBlockPlane;

__device__ __forceinline__ int in_block(int r, int c)
{
    return (r & 31) * 64 + ((((c & 31) >> 3) ^ (-(r >> 2) & 3)) << 4) + (c & 7) * 2;
}

// Byte address of (r, c) of the hi plane in a matrix of ld columns.
__device__ __forceinline__ size_t blocked(int r, int c, int ld)
{
    return ((size_t)(r >> 5) * (ld >> 5) + (c >> 5)) * kBlockBytes + in_block(r, c);
}

// Spans of one step (true) or of 3, 2, 2, ... for a matrix. Spans save products along n and cost
// accuracy. Difference to 64 bits after five steps on normal values, one by one / in spans / the
// textbook form in fp32: 140 x 200 9.8e-7 / 2.0e-6 / 1.6e-6, 256 x 256 8.6e-7 / 2.5e-6 / 1.8e-6,
// 320 x 5000 1.5e-6 / 3.6e-6 / 2.7e-6, 384 x 1536 1.3e-6 / 2.9e-6 / 3.0e-6, 512 x 512 8.2e-7 /
// 2.8e-6 / 2.3e-6, 512 x 4608 1.5e-6 / 3.5e-6 / 4.4e-6, 1024 x 4096 9.1e-7 / 2.0e-6 / 3.7e-6. So
// they are left to matrices on which they stay with fp32: both sides above 384, one of them well
// above the other; near squares have nothing to save either. us one by one / in spans: 512 x 640
// 117 / 129, 1024 x 1280 189 / 197, 1024 x 2048 243 / 218, 2048 x 2048 664 / 740, 512 x 4608
// 187 / 157; 256 x 2304 107 / 105 and ResNet-50's step 972 / 888, the price of the accuracy.
__host__ __device__ inline bool steps_direct(int rows, int cols)
{
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return m <= 384 || (long long)4 * n <= (long long)5 * m;
}

// Small matrices: M x C of X in LDS, hi and lo. kR x kC fragments of 16 x 16 of X per wave,
// kWR x kWC waves; kAR x kAC fragments of A.
template <int M_, int C_>
struct Fused {
    static constexpr int M = M_, C = C_;
    static constexpr int kThreads = 512, kWaves = 8;
    static constexpr int kB = M / kBlock, kCB = C / kBlock;
    static constexpr int kWC = M == 128 ? 2 : C == 512 ? 8 : 4, kWR = kWaves / kWC;
    static constexpr int kR = M / 16 / kWR, kC = C / 16 / kWC;
    static constexpr int kAR = M == 128 ? 2 : 1, kAC = M == 128 ? 4 : 2;
    static constexpr int kX = M * C * 4, kSquare = M * M * 4;
    static constexpr int kLds = kX + kSquare * (M == 128 ? 1 : 2);
    static_assert(kLds <= 160 * 1024, "one workgroup per CU");
};

// Whether a matrix fits one of the forms.
__host__ __device__ inline bool fits(const OrthShape &e, int m, int c)
{
    return (e.rows < e.cols ? e.rows : e.cols) <= m && (e.rows < e.cols ? e.cols : e.rows) <= c;
}

// v as hi + lo, to 22 bits. The compiler must see one v: an instruction that rounds a product
// or a sum to 16 bits at once would make a hi that differs, now and then, from v rounded twice,
// and lo would then miss by an ulp of hi.
struct Halves {
    _Float16 hi, lo;
};
__device__ __forceinline__ Halves halves_of(float v)
{
    asm("" : "+v"(v));
    const _Float16 hi = (_Float16)v;
    return {hi, (_Float16)(v - (float)hi)};
}

// The same value in every lane, told to the compiler.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p)
{
    const uint64_t u = (uint64_t)p;
    return (const uint8_t *)((uint64_t)(uint32_t)uniform((int)(u >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)u));
}

// What a kernel's launch is about, in its arguments: one shape with its batch, or a table. A
// chain of reads of the arguments costs a microsecond each, so every lane reads its entry of
// the whole table at once.
template <bool MANY>
struct Matrices {
    OrthShape e[MANY ? kMaxParams : 1];
    OrthParam p[MANY ? kMaxParams : 1];
    uint32_t first[MANY ? kMaxParams : 1];     // first workgroup of an entry; behind the last: their number
    uint8_t *work;                             // the matrices' parts
    const void *g;                             // bc_orthogonalize's tensors
    void *out;
};

// The matrix that workgroup `at` of a launch works on, and its number within the matrix.
struct Where {
    OrthShape e;
    int t, img;                                // place in the table, matrix of the batch
    uint32_t local;
};

// per: workgroups of each matrix of a batch.
template <bool MANY>
__device__ __forceinline__ Where find(const Matrices<MANY> &M, uint32_t at, uint32_t per)
{
    Where w;
    if constexpr (MANY) {
        static_assert(kMaxParams == 64, "one entry per lane");
        const int lane = threadIdx.x & 63;
        const OrthShape mine = M.e[lane];
        const uint32_t first = M.first[lane];
        w.t = uniform(__popcll(__ballot(first <= at)) - 1);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, w.t); };
        w.e = {of(mine.rows), of(mine.cols), 1, (uint32_t)of(mine.off)};
        w.img = 0;
        w.local = at - (uint32_t)of(first);
    } else {
        w.e = M.e[0];
        w.t = 0;
        w.img = M.e[0].batch == 1 ? 0 : at / per;
        w.local = at - w.img * per;
    }
    return w;
}

template <bool MANY>
__device__ __forceinline__ uint8_t *slot_base(const Matrices<MANY> &M, const Where &w, const Slot &s)
{
    return M.work + w.e.off * (size_t)256 + (size_t)w.img * slot_bytes(s);
}

// ---------------------------------------------------------------- the start: momentum, norm, X_0

// Several kernels compute these, and what a matrix becomes does not depend on which: fused
// operations are written as such, here and in the products' last steps.
//
// mom <- mu mom + grad, and u of the momentum form: nesterov ? grad + mu mom : mom.
__device__ __forceinline__ float moved(const OrthStep &h, float grad, float mom) { return __builtin_fmaf(h.momentum, mom, grad); }
__device__ __forceinline__ float look_ahead(const OrthStep &h, float grad, float mom)
{
    return h.nesterov ? __builtin_fmaf(h.momentum, mom, grad) : mom;
}

// The start's factor kScale / (norm + eps) as f 2^x: in 32 bits no step leaves their range.
struct Factor {
    float f;
    int x;
};
__device__ __forceinline__ Factor factor_of(double squares, double eps)
{
    Factor r;
    r.f = (float)frexp((double)kScale / (sqrt(squares) + eps), &r.x);
    return r;
}
__device__ __forceinline__ float scaled(float u, const Factor &by) { return ldexpf(u, by.x) * by.f; }

// The element behind a step: decay and update.
__device__ __forceinline__ float stepped(const OrthStep &h, float rate, float was, float x)
{
    return __builtin_fmaf(-rate, x, h.keep * was);
}

// Elements i .. i + 3 of p as fp32 (those below n; p is not read past it).
template <int FMT>
__device__ __forceinline__ void load4(const void *p, size_t i, size_t n, float (&v)[4])
{
    if (i + 4 <= n) {
        if constexpr (FMT == kF32) {
            const Raw<FMT, 4> r = load_raw<FMT, 4>(p, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = get(r, j);
        } else {
            struct __attribute__((packed, aligned(2))) Bytes8 { uint32_t w[2]; };
            const Bytes8 b = *(const Bytes8 *)((const uint8_t *)p + i * 2);
            Raw<FMT, 8> r{{b.w[0], b.w[1], 0u, 0u}};
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = get(r, j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j < n ? get(load_raw<FMT, 1>(p, i + j), 0) : 0.f;
    }
}

__device__ __forceinline__ void store4(float *p, size_t i, size_t n, const float (&v)[4])
{
    if (i + 4 <= n) {
        store_raw<kF32, 4>(p, i, pack<kF32, 4>(v));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < n) p[i + j] = v[j];
    }
}

__host__ __device__ inline int sum_parts(size_t count)
{
    const size_t parts = (count + kSumEach - 1) / kSumEach;
    return (int)(parts < kSumParts ? parts : kSumParts);
}

// Elements of each part: four per thread and turn, so the last part may be short or empty.
__host__ __device__ inline size_t sum_each(size_t count)
{
    const size_t parts = sum_parts(count);
    return ((count + parts - 1) / parts + 3) / 4 * 4;
}

__host__ __device__ inline uint32_t start_tiles(const OrthShape &e)
{
    const Slot s = slot_of(e.rows, e.cols);
    return (uint32_t)(s.m / kTile) * (uint32_t)(s.n / kTile);
}

__device__ __forceinline__ double wave_sum(double v)
{
    for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k, 64);
    return v;
}

// Sum of squares of one of a matrix's parts, in 64 bits: no fp32 gradient overflows it. A
// step's new momentum is written on the way.
template <bool MANY, int FMT>
__global__ __launch_bounds__(kThreads) void k_orth_sums(Matrices<MANY> M, OrthHead *head, OrthStep h, uint32_t per)
{
    __shared__ double lds[4];
    if (blockIdx.x == 0)                                  // for the launches after this one
        for (int i = threadIdx.x; i < kMostSplit; i += kThreads) head->count[i] = 0u;
    const Where w = find(M, blockIdx.x, per);
    const OrthShape &e = w.e;
    const size_t count = (size_t)e.rows * e.cols, each = sum_each(count);
    const size_t lo = w.local * each, hi = lo + each < count ? lo + each : count;
    double sum = 0.0;
#pragma unroll 2
    for (size_t i = lo + threadIdx.x * 4; i < hi; i += kThreads * 4) {
        float u[4];
        if constexpr (MANY) {
            const OrthParam &p = M.p[w.t];
            float g[4], m[4];
            load4<kF32>(p.grad, i, hi, g);
            load4<kF32>(p.mom, i, hi, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m[j] = moved(h, g[j], m[j]);
                u[j] = look_ahead(h, g[j], m[j]);
            }
            store4(p.mom, i, hi, m);
        } else {
            load4<FMT>((const uint8_t *)M.g + w.img * count * kElem<FMT>, i, hi, u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += (double)u[j] * u[j];
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) ((double *)slot_base(M, w, slot_of(e.rows, e.cols)))[w.local] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Elements i .. i + 3 (those below n) rounded to a 16-bit format, or as they are.
__device__ __forceinline__ void store4_as(int fmt, void *p, size_t i, size_t n, const float (&v)[4])
{
    if (fmt == kF32) {
        store4((float *)p, i, n, v);
        return;
    }
    struct __attribute__((packed, aligned(2))) Halves { uint16_t h[4]; } o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float one[1] = {v[j]};
        o.h[j] = (uint16_t)(fmt == kBF16 ? pack<kBF16, 1>(one).w[0] : pack<kF16, 1>(one).w[0]);
    }
    uint16_t *to = (uint16_t *)p + i;
    if (i + 4 <= n) {
        *(Halves *)to = o;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < n) to[j] = o.h[j];
    }
}

// X_0 from G, one 64 x 64 tile per workgroup.
template <bool MANY, int FMT>
__global__ __launch_bounds__(kThreads) void k_orth_start(Matrices<MANY> M, OrthStep h, double eps, uint32_t per)
{
    __shared__ float tile[kTile][kTile + 1];
    __shared__ double lds[4];
    const Where w = find(M, blockIdx.x, per);
    const OrthShape &e = w.e;
    const Slot s = slot_of(e.rows, e.cols);
    uint8_t *base = slot_base(M, w, s);
    const size_t count = (size_t)e.rows * e.cols;
    const int tiles_n = s.n / kTile, ti = w.local / tiles_n, tj = w.local - ti * tiles_n;
    // the tile of G behind tile (ti, tj) of X: four elements of a row at a time
    const int r0 = (s.flip ? tj : ti) * kTile, c0 = (s.flip ? ti : tj) * kTile;
    constexpr int kTurns = kTile * kTile / 4 / kThreads;
    float u[kTurns][4];
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
        const int q = k * kThreads + threadIdx.x, r = r0 + q / (kTile / 4), c = c0 + q % (kTile / 4) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[k][j] = 0.f;
        if (r >= e.rows || c >= e.cols) continue;
        const size_t i = (size_t)r * e.cols + c, end = (size_t)(r + 1) * e.cols;
        if constexpr (MANY) {
            const OrthParam &p = M.p[w.t];
            float g[4], m[4], zero[4] = {0.f, 0.f, 0.f, 0.f};
            load4<kF32>(p.grad, i, end, g);
            load4<kF32>(p.mom, i, end, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) u[k][j] = look_ahead(h, g[j], m[j]);
            store4(p.grad, i, end, zero);
        } else {
            load4<FMT>((const uint8_t *)M.g + w.img * count * kElem<FMT>, i, end, u[k]);
        }
    }
    // the norm, from the parts in their order
    double sum = 0.0;
    for (int i = threadIdx.x; i < sum_parts(count); i += kThreads) sum += ((const double *)base)[i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    const Factor by = factor_of((lds[0] + lds[1]) + (lds[2] + lds[3]), eps);
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
        const int q = k * kThreads + threadIdx.x, r = q / (kTile / 4), c = q % (kTile / 4) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = scaled(u[k][j], by);
            if (s.flip) tile[c + j][r] = v;
            else tile[r][c + j] = v;
        }
    }
    __syncthreads();
    uint8_t *x = base + buf_at(s, kX0);
    for (int q = threadIdx.x; q < kTile * kTile / 8; q += kThreads) {
        const int r = q / 8, c = q % 8 * 8;
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = tile[r][c + j];
            const Halves part = halves_of(v);
            hi[j] = part.hi;
            lo[j] = part.lo;
        }
        uint8_t *to = x + blocked(ti * kTile + r, tj * kTile + c, s.n);
        *(f16x8 *)to = hi;
        *(f16x8 *)(to + kBlockPlane) = lo;
    }
}

// ---------------------------------------------------------------- products
//
// D = s1 E1 + s2 E2 + s3 L R over square tiles of every matrix, two jobs at most per matrix
// and launch. Symmetric products (all but the last of a span) take L R as L R^T, rows of
// both, and write a tile on or above the diagonal and its mirror image. The last one takes
// R = X as it lies, rows along K, and writes X, the result, or the weights.
//
//  * A workgroup of four waves owns a tile of 32 FI x 32 FJ, each wave a quarter of it. Chunks
//    of 32 of K, FI blocks of L and FJ of R, go straight from memory to LDS, a few deep, one
//    barrier per chunk; a wave waits for its own requests only. Between the matrix
//    instructions of a chunk lie the reads of the next chunk's fragments and the requests of
//    the chunk that takes the present one's place, evenly: a wave that does one after the other
//    leaves its matrix core idle (2048 x 2048, 128 x 128 tiles: 38 us a product, 24 of them
//    the instructions).
//  * What is added to the product, E1 and E2, follows the last chunk into LDS. The finished
//    tile takes E1's place there and goes to memory in whole blocks, its mirror image through
//    transposing reads.
//  * Matrix instructions want eight values of K per lane. Rows along K (X as R) are read
//    through the transposing ds_read_b64_tr_b16.
//  * The matrix instruction gets R's fragment first, so that a lane holds four consecutive
//    columns of a row of D.
//  * Where tiles are few and K is long (X X^T of a wide matrix), K is split over several
//    workgroups. Each writes its fp32 sums through to the device-coherent level, and the last
//    to arrive (a counter per tile) adds all of them in order: the result does not depend on
//    the order of arrival.
//  * Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, so
//    that its L2 serves their common rows and columns. us so and with neighbours on different
//    XCDs: ResNet-50's step 988 and 1036, 512 x 4608 157 and 171, 12 of 193 x 301 102 and 122,
//    2048 x 2048 681 and 676. The runs are equal in tiles, not in work: in ResNet-50's launches
//    one XCD gets 1.5 to 2.0 times the mean's chunks.
//
// What bounds them is the latency of a workgroup's waves, not a unit. A symmetric product of
// 2048 x 2048 (272 tiles on 256 CUs, 41 to 51 us) keeps the matrix cores busy for 26000 cycles
// of each SIMD and LDS for 14000 of each CU, while a wave lives 58000: one wave per SIMD waits
// out its chunks' way; the product with X, two waves per SIMD, 49000 of 87000. In all 2048 x 2048,
// 670 us, is 255 TFLOP/s of the textbook's products, three fp16 products each. ResNet-50's step,
// 980 us: 100 for the two passes over momentum and gradients, which memory bounds, the rest the
// products, 25 to 126 us each, with XCDs that end early. Few tiles: 5 to 11 us for each of 15 or
// 17 products; a wave lives 17000 cycles, 400 to 2000 of its SIMD's in matrix instructions, the
// rest a launch, the way to LDS and the tile's way out.

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kK = kBlock;                     // depth of a chunk
constexpr int kFold = 4;                       // chunks with running sums of their own
constexpr int kExtent = 0x7FFFFF00;            // every request lies within its (padded) matrix
constexpr int kCoherent = 16;                  // cache policy SC1: device-coherent access

// A tile's form: FI x FJ fragments of 16 x 16 per wave. LDS for two workgroups per CU.
template <int FI, int FJ>
struct Tile {
    static constexpr int I = 32 * FI, J = 32 * FJ;        // rows, columns
    static constexpr int kPer = FI + FJ;                  // blocks of a chunk, requests of a wave for it
    static constexpr int kStages = FI + FJ > 4 ? 3 : 4;   // chunks in LDS
    static constexpr int kStage = kPer * kBlockBytes;
    static constexpr int kBlocks = FI * FJ;               // of the tile
    static constexpr int kRing = kStages * kPer;          // blocks of LDS
    static constexpr size_t kLds = (size_t)kStages * kStage;
    static_assert(2 * kBlocks <= kRing, "two addends fit where the chunks were");
};

__device__ __forceinline__ f16x8 read_tr(const uint8_t *lo, const uint8_t *hi)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 *lds_p;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(__attribute__((address_space(3))) uint8_t *)lo);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(__attribute__((address_space(3))) uint8_t *)hi);
    const f16x4 x = __builtin_bit_cast(f16x4, a), y = __builtin_bit_cast(f16x4, b);
    return f16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// All of this wave's requests but the youngest N have arrived and its LDS reads are done;
// past the barrier that holds for every wave.
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// Where a tile's blocks lie: the first of chunk 0, and the distances (in blocks) from one of
// a chunk's blocks to the next and from chunk to chunk.
struct Operand {
    const uint8_t *at;
    size_t next, step;
};

// The tile's blocks of E1 and E2 (nullptr: none), `pitch` blocks from row to row.
struct Addends {
    const uint8_t *at[2];
    int pitch;
};

// A lane's address in a 32 x 32 block for transposed reads: it gets rows 8 g + 4 k .. + 3
// (g = lane / 16) of column 16 h + lane % 16 from what its group of 16 lanes points to,
// lane 16 g + 4 j + a to row 8 g + 4 k + j, columns 16 h + 4 a .. + 3.
__device__ __forceinline__ int transposed(int lane, int h, int k)
{
    return in_block(8 * (lane >> 4) + 4 * k + (lane >> 2 & 3), 16 * h + (lane & 3) * 4);
}

template <int FI, int FJ>
struct Fragments {
    f16x8 l[2][FI], r[2][FJ];                             // [hi, lo][16 rows or columns]
};

// Sums of chunks [c0, c1) of the tile, a multiple of kFold and at least one fold. E1's blocks,
// then E2's, are left in LDS behind the last chunk, from block *behind of the ring on.
template <int FI, int FJ, bool SYM>
__device__ __forceinline__ void multiply(uint8_t *smem, const Operand &L, const Operand &R, const Addends &X, int c0,
                                         int c1, f32x4 (&tot)[FI][FJ], int *behind)
{
    using T = Tile<FI, FJ>;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const uint32_t lbase = uniform((int)lds_addr(smem));
    // request q of wave w: kilobyte w (0, 1: hi; 2, 3: lo) of L's block q or R's block q - FI
    int off[T::kPer];
#pragma unroll
    for (int q = 0; q < T::kPer; ++q)
        off[q] = (int)(q < FI ? q * L.next : (q - FI) * R.next) * kBlockBytes + wave * 1024 + lane * 16;
    const uint8_t *pl = L.at + c0 * L.step * kBlockBytes, *pr = R.at + c0 * R.step * kBlockBytes;
    i32x4 dl, dr;
    auto next_chunk = [&] {
        dl = raw_desc(pl, kExtent);
        dr = raw_desc(pr, kExtent);
        pl += L.step * kBlockBytes;
        pr += R.step * kBlockBytes;
    };
    auto request = [&](uint32_t to, int q) { dma16(q < FI ? dl : dr, to + q * kBlockBytes, off[q]); };
    // block x of the addends; one that is not there is zeros, from no memory
    auto request_addend = [&](uint32_t to, int q, int x) {
        const int b = x % T::kBlocks;
        const uint8_t *e = x < T::kBlocks ? X.at[0] : x < 2 * T::kBlocks ? X.at[1] : nullptr;
        dma16(raw_desc(e, e ? kExtent : 0), to + q * kBlockBytes,
              ((b / FJ) * X.pitch + b % FJ) * kBlockBytes + wave * 1024 + lane * 16);
    };
    // fragments of a chunk, 2 (FI + FJ): plane, 16 rows (or columns) of this wave's
    const int wi = (wave >> 1) * FI, wj = (wave & 1) * FJ;
    const int frag = in_block(lane & 15, (lane >> 4) * 8);
    int tr[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k) tr[h][k] = transposed(lane, h, k);
    auto read = [&](const uint8_t *b, Fragments<FI, FJ> &f, int q) {
        if (q < 2 * FI) {                                 // FI and FJ are even: the half of a block is i & 1
            const int p = q / FI, i = q % FI;
            f.l[p][i] = *(const f16x8 *)(b + ((wi + i) >> 1) * kBlockBytes + p * kBlockPlane + (i & 1) * 1024 + frag);
        } else {
            const int p = (q - 2 * FI) / FJ, i = (q - 2 * FI) % FJ;
            const uint8_t *br = b + (FI + ((wj + i) >> 1)) * kBlockBytes + p * kBlockPlane;
            if constexpr (SYM) f.r[p][i] = *(const f16x8 *)(br + (i & 1) * 1024 + frag);
            else f.r[p][i] = read_tr(br + tr[i & 1][0], br + tr[i & 1][1]);
        }
    };
#pragma unroll
    for (int i = 0; i < FI * FJ; ++i) tot[i / FJ][i % FJ] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < T::kStages; ++d) {
        next_chunk();
#pragma unroll
        for (int q = 0; q < T::kPer; ++q) request(lbase + d * T::kStage + wave * 1024, q);
    }
    Fragments<FI, FJ> f[2];
    arrived<(T::kStages - 1) * T::kPer>();
#pragma unroll
    for (int q = 0; q < 2 * T::kPer; ++q) read(smem, f[0], q);
    int at = 0;                                           // byte of LDS where chunk c lies
    // a chunk: its fragments are in `now`; the next one's are read meanwhile. Past the barrier
    // every wave has read the present chunk, so its place in LDS takes the chunk kStages ahead,
    // or the addends' blocks from AHEAD on.
    auto step = [&](Fragments<FI, FJ> &now, Fragments<FI, FJ> &next, f32x4 (&acc)[FI][FJ], auto ahead) {
        constexpr int kAhead = decltype(ahead)::value;
        arrived<(T::kStages - 2) * T::kPer>();
        const uint32_t to = lbase + at + wave * 1024;
        at = at + T::kStage == (int)T::kLds ? 0 : at + T::kStage;
        const uint8_t *b = smem + at;
        if constexpr (kAhead < 0) next_chunk();
        constexpr int kEach = 3 * FI * FJ / T::kPer;      // matrix instructions per group
        static_assert(kEach * T::kPer == 3 * FI * FJ, "groups are equal");
#pragma unroll
        for (int q = 0; q < T::kPer; ++q) {
            read(b, next, 2 * q);
            read(b, next, 2 * q + 1);
            if constexpr (kAhead < 0) request(to, q);
            else request_addend(to, q, kAhead + q);
#pragma unroll
            for (int k = q * kEach; k < (q + 1) * kEach; ++k) {
                const int p = k / (FI * FJ), i = k / FJ % FI, j = k % FJ;      // lo hi, hi lo, hi hi
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.r[p == 1][j], now.l[p == 0][i], acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // kFold chunks with sums of their own, written out: sums carried around a loop would be
    // moved between registers in every turn
    auto fold = [&](auto last) {
        f32x4 acc[FI][FJ];
#pragma unroll
        for (int i = 0; i < FI * FJ; ++i) acc[i / FJ][i % FJ] = f32x4{0.f, 0.f, 0.f, 0.f};
        static_assert(kFold == 4 && T::kStages <= 4, "the last fold's requests reach the addends");
        constexpr int kFirst = decltype(last)::value ? (T::kStages - kFold) * T::kPer : -4 * T::kPer;
        step(f[0], f[1], acc, std::integral_constant<int, kFirst>{});
        step(f[1], f[0], acc, std::integral_constant<int, kFirst + T::kPer>{});
        step(f[0], f[1], acc, std::integral_constant<int, kFirst + 2 * T::kPer>{});
        step(f[1], f[0], acc, std::integral_constant<int, kFirst + 3 * T::kPer>{});
#pragma unroll
        for (int i = 0; i < FI * FJ; ++i) tot[i / FJ][i % FJ] += acc[i / FJ][i % FJ];
    };
    for (int c = c0 + kFold; c < c1; c += kFold) fold(std::false_type{});
    fold(std::true_type{});
    arrived<0>();
    *behind = at / kBlockBytes;
}

// Chunks of K of a product, tiles of a matrix with `jobs` of them, and K ranges of `each` chunks
// (0: whole) where there are three at least: a shorter product is whole in every launch, so its
// bits do not depend on the longer ones beside it (in ranges as well: the policy network's step
// 144 us for 150, steps of other networks 0 to 2 % slower).
__host__ __device__ inline int chunks_of(const OrthPlan &p, const Slot &s) { return (p.job[0].L <= kX1 ? s.n : s.m) / kK; }

// Row i of a symmetric product's tiles holds those that reach the diagonal: i I / J .. m / J - 1.
template <int FI, int FJ>
__host__ __device__ inline uint32_t tiles_of(const OrthPlan &p, const Slot &s)
{
    static_assert(FI % FJ == 0, "whole tiles left of the diagonal");
    const uint32_t i = s.m / (32 * FI), j = p.sym ? s.m / (32 * FJ) : s.n / (32 * FJ);
    return p.sym ? i * j - FI / FJ * (i * (i - 1) / 2) : i * j;
}

__host__ __device__ inline int ranges_of(int chunks, int each) { return each && chunks >= 3 * each ? (chunks + each - 1) / each : 1; }

template <int FI, int FJ>
__host__ __device__ inline uint32_t products_of(const OrthPlan &p, const OrthShape &e, int each)
{
    const Slot s = slot_of(e.rows, e.cols);
    return p.jobs ? p.jobs * tiles_of<FI, FJ>(p, s) * ranges_of(chunks_of(p, s), each) : 0;
}

template <int FI, int FJ, bool MANY>
__global__ __launch_bounds__(kThreads) void k_orth_product(Matrices<MANY> M, OrthStage S, OrthHead *head, OrthStep h, uint32_t per)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int last;
    // run of neighbouring tiles for each XCD
    const uint32_t xcd = blockIdx.x % 8, runs = gridDim.x / 8, longer = gridDim.x % 8;
    const uint32_t wg = xcd * runs + min(xcd, longer) + blockIdx.x / 8;
    auto plan_of = [&](const OrthShape &e) -> const OrthPlan & {
        return S.plan[MANY && steps_direct(e.rows, e.cols)];
    };
    const Where w = find(M, wg, per);
    const OrthShape &e = w.e;
    const OrthPlan &plan = plan_of(e);
    const Slot s = slot_of(e.rows, e.cols);
    uint8_t *base = slot_base(M, w, s);
    using Form = Tile<FI, FJ>;
    // number within the matrix = (range * jobs + job) * tiles + tile, so that neighbours read
    // the same columns of X
    const int chunks = chunks_of(plan, s), ranges = ranges_of(chunks, S.each);
    const uint32_t tiles = tiles_of<FI, FJ>(plan, s), all = tiles * plan.jobs;
    uint32_t which = w.local, split = 0;
    if (ranges > 1) {
        split = w.local / all;
        which = w.local - split * all;
    }
    const int second = which >= tiles;
    const OrthJob job = plan.job[second];
    uint32_t tile = which - second * tiles;
    int ti, tj;
    if (plan.sym) {
        ti = 0;
        uint32_t row = s.m / Form::J;                      // tiles of row ti
        for (; tile >= row; row -= FI / FJ, ++ti) tile -= row;
        tj = ti * (FI / FJ) + tile;
    } else {
        const int tiles_m = s.m / Form::I;                 // down the columns of X
        tj = tile / tiles_m;
        ti = tile - tj * tiles_m;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // a lane's part of the tile: [i][j][q] is row wi + 16 i + lane % 16, column
    // wj + 16 j + 4 (lane / 16) + q
    const int wi = (wave >> 1) * 16 * FI, wj = (wave & 1) * 16 * FJ;
    const int ld = plan.sym ? s.m : s.n;
    const int gi = ti * FI, gj = tj * FJ;                  // the tile's first block
    auto block_at = [&](int b, int bi, int bj) {           // block (bi, bj) of a buffer
        return base + buf_at(s, b) + ((size_t)bi * (ld / kBlock) + bj) * kBlockBytes;
    };
    const Addends X = {{job.E1 == kNone ? nullptr : uniform(block_at(job.E1, gi, gj)),
                        job.E2 == kNone ? nullptr : uniform(block_at(job.E2, gi, gj))}, ld / kBlock};
    const int c0 = uniform(split * S.each), c1 = uniform(ranges > 1 ? min(chunks, c0 + S.each) : chunks);
    f32x4 tot[FI][FJ];
    int behind;
    const Operand L = {uniform(base + buf_at(s, job.L) + (size_t)gi * chunks * kBlockBytes), (size_t)chunks, 1};
    if (uniform(plan.sym)) {
        const Operand R = {uniform(base + buf_at(s, job.R) + (size_t)gj * chunks * kBlockBytes), (size_t)chunks, 1};
        multiply<FI, FJ, true>(smem, L, R, X, c0, c1, tot, &behind);
    } else {
        const Operand R = {uniform(base + buf_at(s, job.R) + (size_t)gj * kBlockBytes), 1, (size_t)s.n / kBlock};
        multiply<FI, FJ, false>(smem, L, R, X, c0, c1, tot, &behind);
    }
    if (ranges > 1) {
        const uint32_t slot = wg - w.local + which * ranges;   // the tile's first place
        const __amdgpu_buffer_rsrc_t part = __builtin_amdgcn_make_buffer_rsrc(
            (void *)((f32x4 *)(head + 1) + (size_t)slot * (FI * FJ * kThreads)), (short)0,
            ranges * FI * FJ * kThreads * 16, kBufferFlags);
        auto place = [&](int k, int i) { return ((k * FI * FJ + i) * kThreads + tid) * 16; };
#pragma unroll
        for (int i = 0; i < FI * FJ; ++i)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, tot[i / FJ][i % FJ]), part, place(split, i), 0, kCoherent);
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) {
            uint32_t *count = head->count + slot;
            last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)ranges - 1;
            if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
        }
        __syncthreads();
        if (!last) return;
#pragma unroll
        for (int i = 0; i < FI * FJ; ++i) tot[i / FJ][i % FJ] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = 0; k < ranges; ++k)
#pragma unroll
            for (int i = 0; i < FI * FJ; ++i)
                tot[i / FJ][i % FJ] += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, place(k, i), 0, kCoherent));
    }
    // behind the last chunk LDS holds E1's blocks, which the result replaces, then E2's
    auto in_lds = [&](int b) {                             // block b of them
        const int at = behind + b;
        return smem + (at < Form::kRing ? at : at - Form::kRing) * kBlockBytes;
    };
    // where a lane's [i][j] lies in block (wi + 16 i) / 32, (wj + 16 j) / 32 of the tile
    auto mine = [&](int i, int j, int add) {
        const int r = wi + i * 16, c = wj + j * 16;
        return in_lds(add * Form::kBlocks + (r >> 5) * FJ + (c >> 5)) + in_block(r + (lane & 15), c + (lane >> 4) * 4);
    };
    auto add = [&](int which, float by) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                const uint8_t *at = mine(i, j, which);
                const f16x4 hi = *(const f16x4 *)at, lo = *(const f16x4 *)(at + kBlockPlane);
#pragma unroll
                for (int q = 0; q < 4; ++q) tot[i][j][q] = __builtin_fmaf(by, (float)hi[q] + (float)lo[q], tot[i][j][q]);
            }
    };
#pragma unroll
    for (int i = 0; i < FI * FJ; ++i) tot[i / FJ][i % FJ] *= job.s3 * (1.f / kScale);
    if (job.E1 != kNone) add(0, job.s1);
    if (job.E2 != kNone) add(1, job.s2);
    if (!plan.last) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                f16x4 hi, lo;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const Halves part = halves_of(tot[i][j][q]);
                    hi[q] = part.hi;
                    lo[q] = part.lo;
                }
                uint8_t *at = mine(i, j, 0);
                *(f16x4 *)at = hi;
                *(f16x4 *)(at + kBlockPlane) = lo;
            }
        __syncthreads();
        // half a plane of a block per wave and turn: 16 rows, a unit of 16 bytes per lane
        const int r = lane & 15, u = lane >> 4;
#pragma unroll
        for (int k = 0; k < Form::kBlocks; ++k) {
            const int h = wave & 1, p = wave >> 1, bi = gi + k / FJ, bj = gj + k % FJ;
            const uint8_t *from = in_lds(k) + p * kBlockPlane;
            const int in = p * kBlockPlane + in_block(16 * h + r, 8 * u);
            uint8_t *d = block_at(job.D, bi, bj) + in;
            f16x8 v = *(const f16x8 *)(from + in_block(16 * h + r, 8 * u));
            if (!plan.sym) {
                *(f16x8 *)d = v;
                continue;
            }
            // the blocks above the diagonal, and their mirror images; on it the upper half stands
            // for both: what is stored is symmetric
            if (bi > bj) continue;
            const f16x8 m = read_tr(from + transposed(lane, h, 0), from + transposed(lane, h, 1));
            if (bi == bj) {
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (8 * u + q < 16 * h + r) v[q] = m[q];
            } else {
                *(f16x8 *)(block_at(job.D, bj, bi) + in) = m;
            }
            *(f16x8 *)d = v;
        }
        return;
    }
    // the result: in fp32 through LDS, in rows of the result (columns of X where that is the
    // transpose), four elements per thread and turn
    static_assert((size_t)Form::I * (Form::J + 4) * 4 <= Form::kLds && (size_t)Form::J * (Form::I + 4) * 4 <= Form::kLds,
                  "the tile fits");
    float *rows = (float *)smem;
    __syncthreads();                                       // E1 and E2 have been read
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int r = wi + i * 16 + (lane & 15), c = wj + j * 16 + (lane >> 4) * 4;
            tot[i][j] *= 1.f / kScale;
            if (!s.flip) {
                *(f32x4 *)(rows + r * (Form::J + 4) + c) = tot[i][j];
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) rows[(c + q) * (Form::I + 4) + r] = tot[i][j][q];
            }
        }
    __syncthreads();
    const int width = s.flip ? Form::I : Form::J;
    const int row0 = s.flip ? tj * Form::J : ti * Form::I, col0 = s.flip ? ti * Form::I : tj * Form::J;
    const float tall = e.rows > e.cols ? (float)e.rows / (float)e.cols : 1.f;
    const float rate = h.lr * sqrtf(tall);
#pragma unroll
    for (int k = 0; k < Form::I * Form::J / 4 / kThreads; ++k) {
        const int q = (k * kThreads + tid) * 4, r = q / width, c = q - r * width;
        if (row0 + r >= e.rows || col0 + c >= e.cols) continue;
        const f32x4 x = *(const f32x4 *)(rows + r * (width + 4) + c);
        const size_t o = (size_t)(row0 + r) * e.cols + col0 + c, end = (size_t)(row0 + r + 1) * e.cols;
        float v[4] = {x[0], x[1], x[2], x[3]};
        if constexpr (MANY) {
            const OrthParam &p = M.p[w.t];
            float was[4];
            load4<kF32>(p.w, o, end, was);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = stepped(h, rate, was[j], v[j]);
            store4(p.w, o, end, v);
            if (p.w16) store4_as(S.fmt, p.w16, o, end, v);
        } else {
            store4_as(S.fmt, (uint8_t *)M.out + (size_t)w.img * e.rows * e.cols * (S.fmt == kF32 ? 4 : 2), o, end, v);
        }
    }
}

// ---------------------------------------------------------------- small matrices, in one launch
//
// The products of small matrices are shorter than the launches for them. Here a workgroup of
// eight waves keeps 64 or 128 rows of X in LDS, with A and B beside it, and runs a matrix from
// G to the result in one launch.
//
// X' = a (X + B X), B = (b/a) A + (c/a) A^2, as the products above in spans of one step, and
// with their sums, order and roundings, the norm's among them: the same bits. (Products this
// short are never split over K.) The workgroup's latency bounds it: of a step of 64 x 64 (6500 cycles) the matrix
// instructions take some 1500, the rest is fragments on their way from LDS, the split into
// halves, and four barriers.
struct FusedStage {
    float a, b, c;                             // a, b / a, c / a
    double eps;
    int steps, fmt;
};

// acc += product t of the three of halves, l r^T of one block of K: lo hi, hi lo, hi hi. The
// mirror image of a fragment has the first two the other way round.
__device__ __forceinline__ void multiply(f32x4 &acc, const f16x8 (&l)[2], const f16x8 (&r)[2], int t)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[t == 1], l[t == 0], acc, 0, 0, 0);
}
__device__ __forceinline__ int mirrored(int t) { return t == 2 ? 2 : 1 - t; }

template <typename F, bool MANY, int FMT>
__global__ __launch_bounds__(F::kThreads) void k_orth_fused(Matrices<MANY> Ms, FusedStage S, OrthStep h, uint32_t per)
{
    constexpr int M = F::M, kR = F::kR, kC = F::kC, kAR = F::kAR, kAC = F::kAC;
    extern __shared__ __align__(16) uint8_t smem[];
    // X, A, and B: in A's place with 128 rows
    uint8_t *const X = smem, *const A = smem + F::kX, *const B = M == 128 ? A : A + F::kSquare;
    const Where w = find(Ms, blockIdx.x, per);
    const OrthShape &e = w.e;
    const bool flip = e.rows > e.cols;
    const int m = flip ? e.cols : e.rows, n = flip ? e.rows : e.cols;      // of X, not padded
    const int cols = (n + kBlock - 1) / kBlock * kBlock;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const size_t count = (size_t)e.rows * e.cols;
    const int frag = in_block(lane & 15, (lane >> 4) * 8);
    const int rr = lane & 15, cc = (lane >> 4) * 4;        // a lane's place in a fragment of sums
    // 16 rows of a block (half hf) as they lie, 16 columns of a block transposed
    auto rows_of = [&](const uint8_t *b, int p, int hf) { return *(const f16x8 *)(b + p * kBlockPlane + hf * 1024 + frag); };
    auto columns_of = [&](const uint8_t *b, int p, int hf) {
        return read_tr(b + p * kBlockPlane + transposed(lane, hf, 0), b + p * kBlockPlane + transposed(lane, hf, 1));
    };
    // fragment (i, j) of a matrix of ld blocks per row
    auto place = [&](uint8_t *at, int i, int j, int ld) {
        return at + ((i >> 1) * ld + (j >> 1)) * kBlockBytes + in_block((i & 1) * 16 + rr, (j & 1) * 16 + cc);
    };
    // four values of a row to hi and lo, and what these hold
    auto put = [](uint8_t *at, f32x4 &v) {
        f16x4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const Halves part = halves_of(v[q]);
            hi[q] = part.hi;
            lo[q] = part.lo;
        }
        *(f16x4 *)at = hi;
        *(f16x4 *)(at + kBlockPlane) = lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)hi[q] + (float)lo[q];
    };
    auto take = [](const uint8_t *at) {
        const f16x4 hi = *(const f16x4 *)at, lo = *(const f16x4 *)(at + kBlockPlane);
        f32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (float)hi[q] + (float)lo[q];
        return v;
    };

    // X to LDS: eight columns of a row of a block per thread and turn
    constexpr int kTurns = M * F::C / 8 / F::kThreads;
    static_assert(kTurns >= 1 && F::kThreads == 512, "four blocks a turn");
    {
        float u[kTurns][8];
        // row and first column of X, neighbours along a row of G
        struct Cell {
            int r, c;
        };
        auto cell = [&](int t) -> Cell {
            const int blk = t * 4 + wave / 2, k = tid & 127;
            return {blk / F::kCB * kBlock + (flip ? k & 31 : k >> 2), blk % F::kCB * kBlock + (flip ? k >> 5 : k & 3) * 8};
        };
        // The norm: the squares in the order in which k_orth_sums and k_orth_start take them, four
        // waves for each of four parts at most, or the last bits would depend on the kernel. The
        // elements are read again for it, all at once (through LDS instead, from the lanes that
        // hold them: 64 x 147 30.3 us, 64 x 512 58.7).
        double *const sums = (double *)A;                  // [part][wave of four]
        constexpr int kParts = M * F::C <= kSumEach ? 1 : M * F::C / kSumEach, kReads = kSumEach / 1024;
        static_assert(kParts <= 4 && M * F::C <= kParts * kSumEach, "parts of a matrix");
        auto squares = [&] {
            const int each = (int)sum_each(count);
#pragma unroll 1
            for (int part = wave >> 2; part < kParts; part += 2) {
                const int lo = part * each + (tid & 255) * 4, hi = min((int)count, (part + 1) * each);
                float v[kReads][4];
#pragma unroll
                for (int k = 0; k < kReads; ++k) {
                    const int i = lo + k * 1024;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[k][j] = 0.f;
                    if (i >= hi) continue;
                    if constexpr (MANY) {
                        const OrthParam &p = Ms.p[w.t];
                        float g[4], mom[4];
                        load4<kF32>(p.grad, i, hi, g);
                        load4<kF32>(p.mom, i, hi, mom);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[k][j] = look_ahead(h, g[j], moved(h, g[j], mom[j]));
                    } else {
                        load4<FMT>((const uint8_t *)Ms.g + w.img * count * kElem<FMT>, i, hi, v[k]);
                    }
                }
                double sum = 0.0;
#pragma unroll
                for (int k = 0; k < kReads; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum += (double)v[k][j] * v[k][j];
                sum = wave_sum(sum);
                if (lane == 0) sums[part * 4 + (wave & 3)] = sum;
            }
        };
        if constexpr (MANY) {                              // before the gradients and momenta are written
            squares();
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const auto [xr, xc] = cell(t);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[t][j] = 0.f;
            if (xr >= m || xc >= n) continue;
            if (flip) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (xc + j >= n) continue;
                    const size_t i = (size_t)(xc + j) * e.cols + xr;
                    if constexpr (MANY) {
                        const OrthParam &p = Ms.p[w.t];
                        const float g = p.grad[i], mom = moved(h, g, p.mom[i]);
                        u[t][j] = look_ahead(h, g, mom);
                        p.mom[i] = mom;
                        p.grad[i] = 0.f;
                    } else {
                        u[t][j] = get(load_raw<FMT, 1>(Ms.g, w.img * count + i), 0);
                    }
                }
                continue;
            }
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const size_t i = (size_t)xr * e.cols + xc + v * 4, end = (size_t)(xr + 1) * e.cols;
                if (i >= end) continue;
                float g[4];
                if constexpr (MANY) {
                    const OrthParam &p = Ms.p[w.t];
                    float mom[4], zero[4] = {0.f, 0.f, 0.f, 0.f};
                    load4<kF32>(p.grad, i, end, g);
                    load4<kF32>(p.mom, i, end, mom);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mom[j] = moved(h, g[j], mom[j]);
                        g[j] = look_ahead(h, g[j], mom[j]);
                    }
                    store4(p.mom, i, end, mom);
                    store4(p.grad, i, end, zero);
                } else {
                    load4<FMT>((const uint8_t *)Ms.g + w.img * count * kElem<FMT>, i, end, g);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) u[t][v * 4 + j] = g[j];
            }
        }
        if constexpr (!MANY) squares();
        __syncthreads();
        auto part_sum = [&](int k) {
            return k < kParts ? (sums[4 * k] + sums[4 * k + 1]) + (sums[4 * k + 2] + sums[4 * k + 3]) : 0.0;
        };
        const double sum = (part_sum(0) + part_sum(2)) + (part_sum(1) + part_sum(3));
        const Factor by = factor_of(sum, S.eps);
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            f16x8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = scaled(u[t][j], by);
                const Halves part = halves_of(v);
                hi[j] = part.hi;
                lo[j] = part.lo;
            }
            const auto [xr, xc] = cell(t);
            if (xc / kBlock * kBlock >= cols) continue;
            uint8_t *at = X + ((xr >> 5) * F::kCB + (xc >> 5)) * kBlockBytes + in_block(xr, xc);
            *(f16x8 *)at = hi;
            *(f16x8 *)(at + kBlockPlane) = lo;
        }
    }
    __syncthreads();

    // The wave's part of X, as it lies in LDS: both terms of X + B X have the same X.
    const int x_i = wave / F::kWC * kR, x_j = wave % F::kWC * kC;
    f32x4 x[kR][kC];
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int j = 0; j < kC; ++j)
            x[i][j] = (x_j + j) * 16 < cols ? take(place(X, x_i + i, x_j + j, F::kCB)) : f32x4{0.f, 0.f, 0.f, 0.f};

    // Sums of S S^T over `blocks` of K for the wave's part of A, the upper half standing for both:
    // below the diagonal the products come in the order that makes them its mirror image, and
    // fragments on the diagonal in either.
    const int a_i = M == 128 ? wave / 2 * 2 : wave / 2, a_j = M == 128 ? wave % 2 * 4 : wave % 2 * 2;
    auto square = [&](const uint8_t *from, int ld, int blocks, f32x4 (&tot)[kAR][kAC]) {
#pragma unroll
        for (int i = 0; i < kAR * kAC; ++i) tot[i / kAC][i % kAC] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int k0 = 0; k0 < blocks; k0 += kFold) {
            f32x4 acc[kAR][kAC], other[kAR];               // other: fragment (i, i) in the other order
#pragma unroll
            for (int i = 0; i < kAR * kAC; ++i) acc[i / kAC][i % kAC] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kAR; ++i) other[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int k = k0; k < min(k0 + kFold, blocks); ++k) {
                f16x8 l[kAR][2], r[kAC][2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
#pragma unroll
                    for (int i = 0; i < kAR; ++i) l[i][p] = rows_of(from + (((a_i + i) >> 1) * ld + k) * kBlockBytes, p, (a_i + i) & 1);
#pragma unroll
                    for (int j = 0; j < kAC; ++j) r[j][p] = rows_of(from + (((a_j + j) >> 1) * ld + k) * kBlockBytes, p, j & 1);
                }
#pragma unroll
                for (int j0 = 0; j0 < kAC; j0 += 2) {      // a block of 32 columns, one branch for it
                    // below(i, j): fragments below the diagonal; diagonal(i): a row's fragment on it
                    auto block = [&](auto below, auto diagonal) {
#pragma unroll
                        for (int t = 0; t < 3; ++t)
#pragma unroll
                            for (int i = 0; i < kAR; ++i) {
#pragma unroll
                                for (int j = 0; j < 2; ++j)
                                    multiply(acc[i][j0 + j], l[i], r[j0 + j], below(i, j) ? mirrored(t) : t);
                                if (diagonal(i) >= 0) multiply(other[i], l[i], r[j0 + diagonal(i)], mirrored(t));
                            }
                    };
                    const int d = (a_i >> 1) - ((a_j + j0) >> 1);
                    constexpr auto none = [](int) { return -1; };
                    if (d < 0) block([](int, int) { return false; }, none);
                    else if (d > 0) block([](int, int) { return true; }, none);
                    else if (kAR == 2) block([](int i, int j) { return i > j; }, [](int i) { return i; });
                    else if (a_i & 1) block([](int, int j) { return j == 0; }, [](int) { return 1; });
                    else block([](int, int) { return false; }, [](int) { return 0; });
                }
            }
#pragma unroll
            for (int i = 0; i < kAR; ++i)
#pragma unroll
                for (int j = 0; j < kAC; ++j) {
                    if (a_i + i == a_j + j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[i][j][q] = rr > cc + q ? other[i][q] : acc[i][j][q];
                    tot[i][j] += acc[i][j];
                }
        }
    };
    f32x4 sq[kAR][kAC];
    auto gram = [&] {
        square(X, F::kCB, cols / kBlock, sq);
#pragma unroll
        for (int i = 0; i < kAR * kAC; ++i) sq[i / kAC][i % kAC] *= 1.f / kScale;
    };

    gram();
    for (int step = 0; step < S.steps; ++step) {
#pragma unroll
        for (int i = 0; i < kAR; ++i)
#pragma unroll
            for (int j = 0; j < kAC; ++j) put(place(A, a_i + i, a_j + j, F::kB), sq[i][j]);
        __syncthreads();
        // B = (b/a) A + (c/a) A^2
        f32x4 b[kAR][kAC];
        square(A, F::kB, F::kB, b);
        if constexpr (M == 128) __syncthreads();           // B replaces A
#pragma unroll
        for (int i = 0; i < kAR; ++i)
#pragma unroll
            for (int j = 0; j < kAC; ++j) {
#pragma unroll
                for (int q = 0; q < 4; ++q) b[i][j][q] = __builtin_fmaf(S.b, sq[i][j][q], b[i][j][q] * (S.c * (1.f / kScale)));
                put(place(B, a_i + i, a_j + j, F::kB), b[i][j]);
            }
        __syncthreads();
        // X' = a (X + B X)
        constexpr int kJ = kR * kC > 8 ? 2 : kC;           // at once: registers for the sums
#pragma unroll
        for (int j0 = 0; j0 < kC; j0 += kJ) {
            if ((x_j + j0) * 16 >= cols) continue;
            f32x4 acc[kR][kJ];
#pragma unroll
            for (int i = 0; i < kR * kJ; ++i) acc[i / kJ][i % kJ] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int k = 0; k < F::kB; ++k) {
                f16x8 l[kR][2], r[kJ][2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
#pragma unroll
                    for (int i = 0; i < kR; ++i) l[i][p] = rows_of(B + (((x_i + i) >> 1) * F::kB + k) * kBlockBytes, p, (x_i + i) & 1);
#pragma unroll
                    for (int j = 0; j < kJ; ++j) r[j][p] = columns_of(X + (k * F::kCB + ((x_j + j0 + j) >> 1)) * kBlockBytes, p, j & 1);
                }
#pragma unroll
                for (int t = 0; t < 3; ++t)
#pragma unroll
                    for (int i = 0; i < kR; ++i)
#pragma unroll
                        for (int j = 0; j < kJ; ++j) multiply(acc[i][j], l[i], r[j], t);
            }
#pragma unroll
            for (int i = 0; i < kR; ++i)
#pragma unroll
                for (int j = 0; j < kJ; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        x[i][j0 + j][q] = __builtin_fmaf(S.a, x[i][j0 + j][q], acc[i][j][q] * (S.a * (1.f / kScale)));
        }
        if (step + 1 == S.steps) break;
        if constexpr (F::kWR > 1) __syncthreads();         // other waves read these columns too
#pragma unroll
        for (int i = 0; i < kR; ++i)
#pragma unroll
            for (int j = 0; j < kC; ++j)
                if ((x_j + j) * 16 < cols) put(place(X, x_i + i, x_j + j, F::kCB), x[i][j]);
        __syncthreads();
        gram();
    }
    const float tall = e.rows > e.cols ? (float)e.rows / (float)e.cols : 1.f;
    const float rate = h.lr * sqrtf(tall);
    auto write = [&](size_t i, size_t end, float (&v)[4]) {      // elements i .. i + 3 below end
        if constexpr (MANY) {
            const OrthParam &p = Ms.p[w.t];
            float was[4];
            load4<kF32>(p.w, i, end, was);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = stepped(h, rate, was[q], v[q]);
            store4(p.w, i, end, v);
            if (p.w16) store4_as(S.fmt, p.w16, i, end, v);
        } else {
            store4_as(S.fmt, (uint8_t *)Ms.out + w.img * count * (S.fmt == kF32 ? 4 : 2), i, end, v);
        }
    };
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int j = 0; j < kC; ++j) {
            const int r = (x_i + i) * 16 + rr, c = (x_j + j) * 16 + cc;
            if (r >= m || c >= n) continue;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = x[i][j][q] * (1.f / kScale);
            if (!flip) {
                write((size_t)r * e.cols + c, (size_t)(r + 1) * e.cols, v);
                continue;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c + q < n) {
                    float one[4] = {v[q], 0.f, 0.f, 0.f};
                    const size_t to = (size_t)(c + q) * e.cols + r;
                    write(to, to + 1, one);
                }
        }
}

// ---------------------------------------------------------------- host: what is launched when

// A list of at most N, in place: nothing here allocates, so no call can end in an exception.
template <typename T, int N>
struct List {
    T at[N];
    int n = 0;

    void add(const T &x) { at[n++] = x; }
    const T *begin() const { return at; }
    const T *end() const { return at + n; }
};

// Launches of products at most: 64 steps in spans of 3, 2, 2, ... take 10 + 30 * 7 + 3, one by
// one 3 each.
constexpr int kMostLaunches = 224;

// Steps of the span that begins at step `at` of `steps`.
int span_steps(int at, int steps, bool direct) { return std::min(steps - at, direct ? 1 : at == 0 ? kSpan : 2); }

// The products of a matrix in order, one entry per launch.
List<OrthPlan, kMostLaunches> plans_of(const NewtonSchulz &ns, bool direct)
{
    List<OrthPlan, kMostLaunches> all;
    auto symmetric = [&](std::initializer_list<OrthJob> jobs) {
        OrthPlan p{};
        p.sym = 1;
        for (const OrthJob &j : jobs) p.job[p.jobs++] = j;
        all.add(p);
    };
    int x = kX0;
    for (int at = 0, k; at < ns.steps; at += k) {
        k = span_steps(at, ns.steps, direct);
        int p = kNone;
        symmetric({{x, x, kNone, kNone, kA, 0.f, 0.f, 1.f}});
        for (int i = 0; i < k; ++i) {
            const int b = i & 1 ? kB1 : kB0;
            symmetric({{kA, kA, kA, kNone, b, ns.b / ns.a, 0.f, ns.c / ns.a}});
            // P of step 0 is B; then it goes where neither B nor the old P lies
            const int to = i == 1 ? kP : kB1;
            const OrthJob grow = {b, p, p, b, to, 1.f, 1.f, 1.f}, half = {b, kA, kA, kNone, kR, 1.f, 0.f, 1.f};
            const bool last = i + 1 == k;
            if (i > 0 && !last) symmetric({half, grow});
            else if (i > 0) symmetric({grow});
            else if (!last) symmetric({half});
            p = i == 0 ? b : to;
            const float aa = ns.a * ns.a;
            if (!last) symmetric({{b, kR, kR, kNone, kA, aa, 0.f, aa}});
        }
        const float ak = std::pow(ns.a, (float)k);
        const int to = x == kX0 ? kX1 : kX0;
        OrthPlan q{};
        q.jobs = 1;
        q.last = at + k == ns.steps;
        q.job[0] = {p, x, x, kNone, to, ak, 0.f, ak};
        all.add(q);
        x = to;
    }
    return all;
}

// Numbers a launch: count(shape) workgroups for each matrix. *per: of the first entry's.
template <bool MANY, typename F>
unsigned number(Matrices<MANY> &M, const OrthTable &T, uint32_t *per, F &&count)
{
    uint64_t at = 0;
    for (int t = 0; t < T.n; ++t) {
        const uint32_t c = count(T.e[t]);
        if (t == 0) *per = c;
        M.first[t] = (uint32_t)at;
        at += (uint64_t)c * T.e[t].batch;
    }
    if constexpr (MANY)
        for (int t = T.n; t < kMaxParams; ++t) M.first[t] = (uint32_t)at;
    return (unsigned)at;
}

// Tiles of 128 x 64 read three quarters of the bytes of 64 x 64 ones per product, where they
// are enough for the chip. us with the large ones and with the small ones only: 2048 x 2048 681
// and 811, ResNet-50's step 981 and 1011, 1024 x 2048 219 and 224; 1500 x 1700, 156 large tiles
// in its symmetric products, 395 and 408; the policy network's step, where only the products
// along n take them, 149 and 145. (128 x 128, one workgroup per CU: 2048 x 2048 half as slow again.)
constexpr uint64_t kEnough = 192;

// The products of one launch: the plans of its matrices (those taken in spans, those taken step
// by step; a plan that is done has no jobs), the tiles, and the K ranges.
struct Launch {
    OrthPlan plan[2];
    bool large;
    int each;
    size_t part_bytes;                         // of the sums of K ranges
};

List<Launch, kMostLaunches> launches_of(const OrthTable &T, const NewtonSchulz &ns)
{
    List<OrthPlan, kMostLaunches> plans[2];
    for (int t = 0; t < T.n; ++t) {
        const bool direct = steps_direct(T.e[t].rows, T.e[t].cols);
        if (!plans[direct].n) plans[direct] = plans_of(ns, direct);
    }
    List<Launch, kMostLaunches> all;
    for (int i = 0; i < std::max(plans[0].n, plans[1].n); ++i) {
        Launch l{};
        for (int d = 0; d < 2; ++d) l.plan[d] = i < plans[d].n ? plans[d].at[i] : OrthPlan{};
        auto total = [&](auto count) {
            uint64_t n = 0;
            for (int t = 0; t < T.n; ++t) {
                const OrthPlan &p = l.plan[steps_direct(T.e[t].rows, T.e[t].cols)];
                if (p.jobs) n += (uint64_t)count(p, T.e[t]) * T.e[t].batch;
            }
            return n;
        };
        auto chunks = [](const OrthPlan &p, const OrthShape &e) { return (uint64_t)chunks_of(p, slot_of(e.rows, e.cols)); };
        auto tiles = [&](bool large, int each) {
            return total([&](const OrthPlan &p, const OrthShape &e) {
                return large ? products_of<4, 2>(p, e, each) : products_of<2, 2>(p, e, each);
            });
        };
        auto work = [&](bool large) {
            return total([&](const OrthPlan &p, const OrthShape &e) {
                return (large ? products_of<4, 2>(p, e, 0) : products_of<2, 2>(p, e, 0)) * chunks(p, e);
            });
        };
        uint64_t longest = 0;
        for (int t = 0; t < T.n; ++t) {
            const OrthPlan &p = l.plan[steps_direct(T.e[t].rows, T.e[t].cols)];
            if (p.jobs) longest = std::max(longest, chunks(p, T.e[t]));
        }
        l.large = tiles(true, 0) >= kEnough;
        const uint64_t wgs = tiles(l.large, 0);
        // K in ranges, of whole folds, where the longest workgroup would far outlast the chip's
        // share of the work (twice as long: 1024 x 2048 254 us whole, 265 in ranges)
        const uint64_t share = std::max<uint64_t>(kLeastChunks, ((work(l.large) + 511) / 512 + kFold - 1) / kFold * kFold);
        l.each = longest >= 3 * share && wgs <= 512 ? (int)share : 0;
        const uint64_t places = tiles(l.large, l.each);
        l.part_bytes = l.each ? places * kThreads * sizeof(f32x4) * (l.large ? 8 : 4) : 0;
        all.add(l);
    }
    return all;
}

template <int FI, int FJ, bool MANY>
hipError_t launch_product(const OrthTable &T, Matrices<MANY> &M, OrthHead *head, const OrthStep &h, const OrthStage &S,
                          hipStream_t s)
{
    uint32_t per = 0;
    const unsigned grid = number(M, T, &per, [&](const OrthShape &e) {
        return products_of<FI, FJ>(S.plan[MANY && steps_direct(e.rows, e.cols)], e, S.each);
    });
    const hipError_t e = allow_lds((const void *)k_orth_product<FI, FJ, MANY>, Tile<FI, FJ>::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_orth_product<FI, FJ, MANY>), dim3(grid), dim3(kThreads), (unsigned)(Tile<FI, FJ>::kLds), s, M, S,
                       head, h, per);
    return hipGetLastError();
}

template <bool MANY>
hipError_t launch_products(const OrthTable &T, Matrices<MANY> &M, OrthHead *head, const OrthStep &h, int out_fmt,
                           const NewtonSchulz &ns, hipStream_t s)
{
    OrthStage S{};
    S.fmt = out_fmt;
    for (const Launch &l : launches_of(T, ns)) {
        S.each = l.each;
        for (int d = 0; d < 2; ++d) S.plan[d] = l.plan[d];
        if (!MANY && !S.plan[0].jobs) S.plan[0] = S.plan[1];      // one shape has its plan in the first place
        const hipError_t e = l.large ? launch_product<4, 2, MANY>(T, M, head, h, S, s)
                                     : launch_product<2, 2, MANY>(T, M, head, h, S, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Whether all matrices are small. With larger ones beside them their products share the
// larger ones' launches and cost nothing. By themselves, us in the launches of products and
// here: 64 x 64 68 and 18, 64 x 147 74 and 28, 64 x 512 80 and 54, 128 x 128 69 and 54,
// 256 of 64 x 64 164 and 20. (In a step the 64 x 512 form keeps 272 bytes a lane in scratch
// memory: three of 64 x 512 97 us, one of 512 x 64 118.)
bool all_fused(const OrthTable &T)
{
    for (int t = 0; t < T.n; ++t)
        if (!fits(T.e[t], 64, 512) && !fits(T.e[t], 128, 128)) return false;
    return true;
}

template <typename F, bool MANY, int FMT>
hipError_t launch_fused(const OrthTable &T, Matrices<MANY> &Ms, const OrthStep &h, int out_fmt, const NewtonSchulz &ns,
                        hipStream_t s)
{
    const hipError_t e = allow_lds((const void *)k_orth_fused<F, MANY, FMT>, F::kLds);
    if (e != hipSuccess) return e;
    uint32_t per = 0;
    const unsigned grid = number(Ms, T, &per, [&](const OrthShape &e) {
        // the smallest form that fits
        const bool is = fits(e, 64, 128)   ? F::M == 64 && F::C == 128
                        : fits(e, 64, 256) ? F::C == 256
                        : fits(e, 64, 512) ? F::C == 512
                                           : F::M == 128;
        return (uint32_t)is;
    });
    if (!grid) return hipSuccess;
    const FusedStage S = {ns.a, ns.b / ns.a, ns.c / ns.a, (double)ns.eps, ns.steps, out_fmt};
    hipLaunchKernelGGL((k_orth_fused<F, MANY, FMT>), dim3(grid), dim3(F::kThreads), (unsigned)F::kLds, s, Ms, S, h, per);
    return hipGetLastError();
}

}  // namespace

size_t orth_layout(OrthTable &T, int steps)
{
    const bool fused = all_fused(T);
    size_t at = sizeof(OrthHead), part = 0;
    if (!fused)
        for (const Launch &l : launches_of(T, NewtonSchulz{steps, 1.f, 1.f, 1.f, 0.f})) part = std::max(part, l.part_bytes);
    T.parts = at + part;                       // where the matrices' parts begin
    at = 0;
    for (int t = 0; t < T.n; ++t) {
        T.e[t].off = (uint32_t)(at / 256);
        if (!fused) at += slot_bytes(slot_of(T.e[t].rows, T.e[t].cols)) * T.e[t].batch;
    }
    return T.parts + at;
}

unsigned orth_tiles(int rows, int cols)
{
    const Slot s = slot_of(rows, cols);
    return (unsigned)(s.m / kTile) * (unsigned)(s.n / kTile);
}

bool orth_supported(const NewtonSchulz &ns, const char **why)
{
    const double a = ns.a, b = ns.b, c = ns.c, most = 15.0;   // of the 16 that fp16 holds at kScale
    if (!(std::isfinite(a) && std::isfinite(b) && std::isfinite(c)) || a <= 0.0) {
        *why = "the coefficients must be finite and a positive";
        return false;
    }
    // Bounds over the singular values in [0, top]: 1 + B at the ends and the vertex of its
    // parabola, the step's polynomial at the ends and where its derivative is zero.
    // The factors of a span's steps multiply up in P.
    double top = 1.0, factors = 1.0;
    for (int i = 0, next_span = 0; i < ns.steps; ++i) {
        if (i == next_span) {
            factors = 1.0;
            next_span += span_steps(i, ns.steps, false);
        }
        const double lam = top * top;
        auto factor = [&](double t) { return 1.0 + (b * t + c * t * t) / a; };
        double f = std::max(1.0, std::fabs(factor(lam)));
        if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < lam) f = std::max(f, std::fabs(factor(-b / (2 * c))));
        auto step = [&](double t) { return std::fabs(a * factor(t) * std::sqrt(t)); };
        double next = step(lam);
        const double disc = 9 * b * b - 20 * a * c;          // of 5 c t^2 + 3 b t + a
        if (c != 0.0 && disc >= 0.0) {
            for (double sign : {-1.0, 1.0}) {
                const double t = (-3 * b + sign * std::sqrt(disc)) / (10 * c);
                if (t > 0.0 && t < lam) next = std::max(next, step(t));
            }
        } else if (c == 0.0 && b < 0.0 && -a / (3 * b) < lam) {
            next = std::max(next, step(-a / (3 * b)));
        }
        factors *= f;
        top = next;
        if (!(lam <= most && f * lam <= most && factors + 1.0 <= most && top * top <= most)) {
            *why = "the coefficients let entries of the products pass 15, beyond the 16 bits they are held in";
            return false;
        }
    }
    return true;
}

template <bool MANY>
static hipError_t launch(const OrthTable &T, const OrthStep &h, int in_fmt, int out_fmt, const NewtonSchulz &ns, hipStream_t s)
{
    hipError_t e = hipSuccess;
    const bool fused = all_fused(T);
    OrthHead *head = (OrthHead *)T.work;
    Matrices<MANY> M{};
    M.work = T.work + T.parts;
    M.g = T.g;
    M.out = T.out;
    for (int t = 0; t < T.n; ++t) {
        M.e[t] = T.e[t];
        M.p[t] = T.p[t];
    }
    with_format(in_fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        if constexpr (!MANY || FMT == kF32) {                 // gradients and momentum are fp32
            if (fused) {
                e = launch_fused<Fused<64, 128>, MANY, FMT>(T, M, h, out_fmt, ns, s);
                if (e == hipSuccess) e = launch_fused<Fused<64, 256>, MANY, FMT>(T, M, h, out_fmt, ns, s);
                if (e == hipSuccess) e = launch_fused<Fused<64, 512>, MANY, FMT>(T, M, h, out_fmt, ns, s);
                if (e == hipSuccess) e = launch_fused<Fused<128, 128>, MANY, FMT>(T, M, h, out_fmt, ns, s);
                return;
            }
            uint32_t per = 0;
            unsigned grid = number(M, T, &per, [](const OrthShape &e) { return (uint32_t)sum_parts((size_t)e.rows * e.cols); });
            hipLaunchKernelGGL((k_orth_sums<MANY, FMT>), dim3(grid), dim3(kThreads), 0, s, M, head, h, per);
            if ((e = hipGetLastError()) != hipSuccess) return;
            grid = number(M, T, &per, start_tiles);
            hipLaunchKernelGGL((k_orth_start<MANY, FMT>), dim3(grid), dim3(kThreads), 0, s, M, h, (double)ns.eps, per);
            e = hipGetLastError();
        }
    });
    if (e != hipSuccess || fused) return e;
    return launch_products<MANY>(T, M, head, h, out_fmt, ns, s);
}

hipError_t launch_orth(const OrthTable &T, const OrthStep &h, bool step, int in_fmt, int out_fmt, const NewtonSchulz &ns,
                       hipStream_t s)
{
    return step ? launch<true>(T, h, in_fmt, out_fmt, ns, s) : launch<false>(T, h, in_fmt, out_fmt, ns, s);
}

}  // namespace bc
