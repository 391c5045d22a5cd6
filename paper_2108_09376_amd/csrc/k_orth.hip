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
// step multiplies such an error by up to a^2, so a new A is taken from X after three steps,
// and after two once the small directions have grown (spans_of has the figures).
//
// Arithmetic: an fp32 value x is held as two fp16 numbers, hi = half(x), lo = half(x - hi),
// about 22 bits, all scaled by 2^12, and a product is hi hi + hi lo + lo hi on the matrix
// cores: fp32 accuracy at a third of the fp16 rate, five times the fp32 rate. What is left
// out, lo lo, is below 2^-22 of the product. A matrix instruction rounds its running sum by
// more than an ulp, so the sums of each chunk of K start at zero and join the tile's totals
// in fp32 (512 x 4608, five steps, difference to 64 bits: 1.5e-6, with one running sum
// 3.3e-6; the textbook form in fp32 3.2e-6). Entries stay within 16 (the host has checked
// the coefficients), as |X|_2 <= 1 at the start.
#include <algorithm>
#include <cmath>

#include "bc_internal.h"
#include "rows.h"

namespace bc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;                      // tile edge; matrices are padded to it with zeros
constexpr float kScale = 4096.f;
constexpr int kSpan = 3;                       // most steps between two A taken from X
constexpr int kSumParts = 64;                  // partial sums of squares per matrix

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ constexpr int padded(int n) { return (n + kTile - 1) / kTile * kTile; }

// A matrix's part of the workspace: partial sums, two X and five squares, each two planes
// (hi, lo) of halves.
struct Slot {
    int m, n;                                  // rows <= columns of X, padded
    bool flip;                                 // X is the transpose
};

__host__ __device__ inline Slot slot_of(int rows, int cols)
{
    const bool flip = rows > cols;
    return {padded(flip ? cols : rows), padded(flip ? rows : cols), flip};
}

enum Buf { kX0, kX1, kA, kR, kB0, kB1, kP, kNone };

__host__ __device__ inline size_t buf_at(const Slot &s, int b)
{
    const size_t x = (size_t)s.m * s.n * 4, q = (size_t)s.m * s.m * 4, head = kSumParts * sizeof(double);
    return head + (b <= kX1 ? b * x : 2 * x + (b - kA) * q);
}

__host__ __device__ inline size_t slot_bytes(const Slot &s) { return buf_at(s, kNone); }

// The matrix that workgroup `at` of a launch works on, and its number within the matrix.
struct Where {
    int t;                                     // table entry
    int img;                                   // matrix of the entry's batch
    uint32_t local;
};

__device__ __forceinline__ Where find(const OrthTable &T, uint32_t at)
{
    int t = 0;
    while (t + 1 < T.n && at >= T.e[t + 1].first) ++t;
    const uint32_t per = T.e[t].per, in = at - T.e[t].first;
    const int img = in / per;
    return {t, img, in - img * per};
}

__device__ __forceinline__ uint8_t *slot_base(const OrthTable &T, const Where &w, const Slot &s)
{
    return T.work + T.e[w.t].off * 256 + (size_t)w.img * slot_bytes(s);
}

// ---------------------------------------------------------------- the start: momentum, norm, X_0

// u of the momentum form: nesterov ? grad + mu m : m, m the new momentum
__device__ __forceinline__ float look_ahead(const OrthStep &h, float grad, float mom)
{
    return h.nesterov ? grad + h.momentum * mom : mom;
}

// Sum of squares of one of a matrix's parts, in 64 bits: no fp32 gradient overflows it.
template <bool STEP, int FMT>
__global__ __launch_bounds__(kThreads) void k_orth_sums(OrthTable T, OrthStep h)
{
    __shared__ double lds[4];
    const Where w = find(T, blockIdx.x);
    const OrthEntry &e = T.e[w.t];
    const Slot s = slot_of(e.rows, e.cols);
    const size_t count = (size_t)e.rows * e.cols;
    const size_t each = ((count + e.per - 1) / e.per + 3) / 4 * 4;
    const size_t lo = w.local * each, hi = lo + each < count ? lo + each : count;
    double sum = 0.0;
    for (size_t i = lo + threadIdx.x; i < hi; i += kThreads) {
        float u;
        if constexpr (STEP) {
            const OrthParam &p = T.p[w.t];
            const float g = p.grad[i], m = h.momentum * p.mom[i] + g;
            p.mom[i] = m;
            u = look_ahead(h, g, m);
        } else {
            u = get(load_raw<FMT, 1>(T.g, w.img * count + i), 0);
        }
        sum += (double)u * u;
    }
    for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) ((double *)slot_base(T, w, s))[w.local] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__device__ __forceinline__ void store_split(_Float16 *hi, size_t plane, size_t at, float v)
{
    const _Float16 h = (_Float16)v;
    hi[at] = h;
    hi[at + plane] = (_Float16)(v - (float)h);
}

// X_0 from G, one padded tile per workgroup.
template <bool STEP, int FMT>
__global__ __launch_bounds__(kThreads) void k_orth_start(OrthTable T, OrthStep h, double eps, int parts_each)
{
    __shared__ float tile[kTile][kTile + 1];
    const Where w = find(T, blockIdx.x);
    const OrthEntry &e = T.e[w.t];
    const Slot s = slot_of(e.rows, e.cols);
    uint8_t *base = slot_base(T, w, s);
    const size_t count = (size_t)e.rows * e.cols;
    const int parts = (int)((count + parts_each - 1) / parts_each < kSumParts ? (count + parts_each - 1) / parts_each : kSumParts);
    double sum = 0.0;
    for (int i = 0; i < parts; ++i) sum += ((const double *)base)[i];
    const double inv = (double)kScale / (sqrt(sum) + eps);
    const int tiles_n = s.n / kTile, ti = w.local / tiles_n, tj = w.local - ti * tiles_n;
    // the tile of G behind tile (ti, tj) of X
    const int r0 = (s.flip ? tj : ti) * kTile, c0 = (s.flip ? ti : tj) * kTile;
    for (int k = threadIdx.x; k < kTile * kTile; k += kThreads) {
        const int r = k / kTile, c = k - r * kTile;
        float u = 0.f;
        if (r0 + r < e.rows && c0 + c < e.cols) {
            const size_t i = (size_t)(r0 + r) * e.cols + c0 + c;
            if constexpr (STEP) {
                const OrthParam &p = T.p[w.t];
                u = look_ahead(h, p.grad[i], p.mom[i]);
                p.grad[i] = 0.f;
            } else {
                u = get(load_raw<FMT, 1>(T.g, w.img * count + i), 0);
            }
            u = (float)(u * inv);
        }
        if (s.flip) tile[c][r] = u;
        else tile[r][c] = u;
    }
    __syncthreads();
    _Float16 *x = (_Float16 *)(base + buf_at(s, kX0));
    const size_t plane = (size_t)s.m * s.n;
    for (int k = threadIdx.x; k < kTile * kTile; k += kThreads) {
        const int r = k / kTile, c = k - r * kTile;
        store_split(x, plane, (size_t)(ti * kTile + r) * s.n + tj * kTile + c, tile[r][c]);
    }
}

// ---------------------------------------------------------------- products

constexpr int kK = 64;                         // depth of a chunk
constexpr int kPitch = kK + 8;                 // halves per LDS row: reads of 16 rows meet no bank twice

// D = s1 E1 + s2 E2 + s3 L R over 64 x 64 tiles of every matrix. Symmetric products take
// L R as L R^T (rows of both) and write a tile and its mirror image; the last one takes
// R = X as it lies, and writes X, the result, or the weights.
enum Out { kPlanes, kResult, kWeights };

template <bool SYM, int OUT, int FMT>
__global__ __launch_bounds__(kThreads) void k_orth_product(OrthTable T, OrthJobs J, OrthStep h)
{
    __shared__ _Float16 lds[2][2][kTile][kPitch];          // [operand][hi, lo][row][k]
    const Where w = find(T, blockIdx.x);
    const OrthJob &job = J.job[blockIdx.y];
    const OrthEntry &e = T.e[w.t];
    const Slot s = slot_of(e.rows, e.cols);
    uint8_t *base = slot_base(T, w, s);
    int ti, tj;
    if constexpr (SYM) {
        ti = 0;
        uint32_t t = w.local, row = s.m / kTile;           // row ti holds tiles ti .. m/64 - 1
        while (t >= row) { t -= row--; ++ti; }
        tj = ti + t;
    } else {
        const int tiles_n = s.n / kTile;
        ti = w.local / tiles_n;
        tj = w.local - ti * tiles_n;
    }
    const int depth = job.L <= kX1 ? s.n : s.m;            // columns of L
    const int ld_r = SYM ? depth : s.n;
    const _Float16 *L = (const _Float16 *)(base + buf_at(s, job.L));
    const _Float16 *R = (const _Float16 *)(base + buf_at(s, job.R));
    const size_t plane_l = (size_t)s.m * depth, plane_r = SYM ? plane_l : (size_t)s.m * s.n;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
    f32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < depth; k0 += kK) {
        f32x4 part[2][2] = {};
        __syncthreads();
        for (int p = 0; p < 2; ++p)
            for (int q = tid; q < kTile * kK / 8; q += kThreads) {
                const int r = q / (kK / 8), c = q % (kK / 8) * 8;
                *(f16x8 *)&lds[0][p][r][c] =
                    *(const f16x8 *)(L + p * plane_l + (size_t)(ti * kTile + r) * depth + k0 + c);
                if constexpr (SYM) {
                    *(f16x8 *)&lds[1][p][r][c] =
                        *(const f16x8 *)(R + p * plane_r + (size_t)(tj * kTile + r) * ld_r + k0 + c);
                } else {
                    const f16x8 v = *(const f16x8 *)(R + p * plane_r + (size_t)(k0 + r) * ld_r + tj * kTile + c);
                    for (int i = 0; i < 8; ++i) lds[1][p][c + i][r] = v[i];
                }
            }
        __syncthreads();
        for (int k = 0; k < kK; k += 32) {
            const int kk = k + (lane >> 4) * 8;
            f16x8 a[2][2], b[2][2];                        // [hi, lo][tile]
            for (int p = 0; p < 2; ++p)
                for (int i = 0; i < 2; ++i) {
                    a[p][i] = *(const f16x8 *)&lds[0][p][wi + i * 16 + (lane & 15)][kk];
                    b[p][i] = *(const f16x8 *)&lds[1][p][wj + i * 16 + (lane & 15)][kk];
                }
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < 2; ++j) {
                    part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[1][i], b[0][j], part[i][j], 0, 0, 0);
                    part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0][i], b[1][j], part[i][j], 0, 0, 0);
                    part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0][i], b[0][j], part[i][j], 0, 0, 0);
                }
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) acc[i][j] += part[i][j];
    }
    // acc[i][j][q]: row wi + 16 i + 4 (lane / 16) + q, column wj + 16 j + lane % 16
    const int ld = SYM ? s.m : s.n;
    const size_t plane = (size_t)s.m * ld;
    auto value = [&](int b, size_t at) {
        const _Float16 *p = (const _Float16 *)(base + buf_at(s, b));
        return (float)p[at] + (float)p[at + plane];
    };
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int q = 0; q < 4; ++q) {
                const int r = ti * kTile + wi + i * 16 + (lane >> 4) * 4 + q, c = tj * kTile + wj + j * 16 + (lane & 15);
                // on the diagonal the upper half stands for both: what is stored is symmetric
                if (SYM && c < r) continue;
                const size_t at = (size_t)r * ld + c;
                float v = job.s3 * (1.f / kScale) * acc[i][j][q];
                if (job.E1 != kNone) v += job.s1 * value(job.E1, at);
                if (job.E2 != kNone) v += job.s2 * value(job.E2, at);
                if constexpr (OUT == kPlanes) {
                    _Float16 *d = (_Float16 *)(base + buf_at(s, job.D));
                    store_split(d, plane, at, v);
                    if (SYM && c != r) store_split(d, plane, (size_t)c * ld + r, v);
                } else {
                    const int row = s.flip ? c : r, col = s.flip ? r : c;
                    if (row >= e.rows || col >= e.cols) continue;
                    const size_t o = (size_t)row * e.cols + col;
                    v *= 1.f / kScale;
                    if constexpr (OUT == kResult) {
                        const float y[1] = {v};
                        store_raw<FMT, 1>(T.out, (size_t)w.img * e.rows * e.cols + o, pack<FMT, 1>(y));
                    } else {
                        const OrthParam &p = T.p[w.t];
                        const float tall = e.rows > e.cols ? (float)e.rows / (float)e.cols : 1.f;
                        const float wn = h.keep * p.w[o] - h.lr * sqrtf(tall) * v;
                        p.w[o] = wn;
                        const float y[1] = {wn};
                        if (p.w16) store_raw<FMT, 1>(p.w16, o, pack<FMT, 1>(y));
                    }
                }
            }
}

// Numbers the workgroups of a launch: `per` of entry t for each matrix of its batch.
template <typename F>
unsigned number(OrthTable &T, F &&per)
{
    uint64_t at = 0;
    for (int t = 0; t < T.n; ++t) {
        T.e[t].first = (uint32_t)at;
        T.e[t].per = per(T.e[t]);
        at += (uint64_t)T.e[t].per * T.e[t].batch;
    }
    return (unsigned)at;
}

constexpr int kSumEach = 4096;

uint32_t sum_parts(const OrthEntry &e)
{
    return (uint32_t)std::min<size_t>(((size_t)e.rows * e.cols + kSumEach - 1) / kSumEach, kSumParts);
}

uint32_t tiles_x(const OrthEntry &e)
{
    const Slot s = slot_of(e.rows, e.cols);
    return (uint32_t)(s.m / kTile) * (uint32_t)(s.n / kTile);
}

uint32_t tiles_sym(const OrthEntry &e)
{
    const uint32_t t = slot_of(e.rows, e.cols).m / kTile;
    return t * (t + 1) / 2;
}

// Spans of one step (true) or of 3, 2, 2, ... for a matrix. Difference to 64 bits after five
// steps, in spans of one / of 3 and 2 / of the textbook form in fp32: 8 x 16 6.8e-7 / 6.7e-6
// / 6.6e-7, 64 x 147 6.9e-7 / 1.9e-6 / 1.1e-6, 193 x 301 8.3e-7 / 1.5e-6 / 1.6e-6,
// 512 x 512 6.8e-7 / 1.5e-6 / 2.0e-6: small matrices take the steps one by one.
bool steps_direct(const OrthEntry &e) { return slot_of(e.rows, e.cols).m <= 128; }

hipError_t launch_steps(OrthTable &T, const OrthStep &h, bool step, int out_fmt, const NewtonSchulz &ns, bool direct,
                        hipStream_t s)
{
    hipError_t e = hipSuccess;
    const dim3 block(kThreads);
    const unsigned grid_x = number(T, tiles_x);
    OrthTable S = T;                           // the same table numbered by symmetric tiles
    const unsigned grid_s = number(S, tiles_sym);
    auto symmetric = [&](std::initializer_list<OrthJob> jobs) {
        OrthJobs J{};
        unsigned n = 0;
        for (const OrthJob &j : jobs) J.job[n++] = j;
        hipLaunchKernelGGL((k_orth_product<true, kPlanes, kF32>), dim3(grid_s, n), block, 0, s, S, J, h);
        return hipGetLastError();
    };
    int x = kX0;
    for (int left = ns.steps, most = direct ? 1 : kSpan; left; most = std::min(most, 2)) {
        const int k = std::min(left, most);
        left -= k;
        int p = kNone;
        if ((e = symmetric({{x, x, kNone, kNone, kA, 0.f, 0.f, 1.f}})) != hipSuccess) return e;
        for (int i = 0; i < k; ++i) {
            const int b = i & 1 ? kB1 : kB0;
            if ((e = symmetric({{kA, kA, kA, kNone, b, ns.b / ns.a, 0.f, ns.c / ns.a}})) != hipSuccess) return e;
            // P of step 0 is B; then it goes where neither B nor the old P lies
            const int to = i == 1 ? kP : kB1;
            const OrthJob grow = {b, p, p, b, to, 1.f, 1.f, 1.f}, half = {b, kA, kA, kNone, kR, 1.f, 0.f, 1.f};
            const bool last = i + 1 == k;
            if (i > 0 && !last) e = symmetric({half, grow});
            else if (i > 0) e = symmetric({grow});
            else if (!last) e = symmetric({half});
            if (e != hipSuccess) return e;
            p = i == 0 ? b : to;
            const float aa = ns.a * ns.a;
            if (!last && (e = symmetric({{b, kR, kR, kNone, kA, aa, 0.f, aa}})) != hipSuccess) return e;
        }
        const float ak = std::pow(ns.a, (float)k);
        OrthJobs J{};
        J.job[0] = {p, x, x, kNone, x == kX0 ? kX1 : kX0, ak, 0.f, ak};
        if (left) {
            hipLaunchKernelGGL((k_orth_product<false, kPlanes, kF32>), dim3(grid_x), block, 0, s, T, J, h);
            x = x == kX0 ? kX1 : kX0;
        } else {
            with_format(out_fmt, [&](auto f) {
                constexpr int FMT = decltype(f)::value;
                if (step) hipLaunchKernelGGL((k_orth_product<false, kWeights, FMT>), dim3(grid_x), block, 0, s, T, J, h);
                else hipLaunchKernelGGL((k_orth_product<false, kResult, FMT>), dim3(grid_x), block, 0, s, T, J, h);
            });
        }
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t orth_work(int rows, int cols) { return slot_bytes(slot_of(rows, cols)); }

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
    double top = 1.0, factors = 1.0;
    for (int i = 0; i < ns.steps; ++i) {
        if (i % kSpan == 0) factors = 1.0;
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

hipError_t launch_orth(OrthTable &T, const OrthStep &h, bool step, int in_fmt, int out_fmt, const NewtonSchulz &ns,
                       hipStream_t s)
{
    hipError_t e = hipSuccess;
    const dim3 block(kThreads);
    unsigned grid = number(T, sum_parts);
    if (step) hipLaunchKernelGGL((k_orth_sums<true, kF32>), dim3(grid), block, 0, s, T, h);
    else
        with_format(in_fmt, [&](auto f) {
            hipLaunchKernelGGL((k_orth_sums<false, decltype(f)::value>), dim3(grid), block, 0, s, T, h);
        });
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const unsigned grid_x = number(T, tiles_x);
    if (step) hipLaunchKernelGGL((k_orth_start<true, kF32>), dim3(grid_x), block, 0, s, T, h, (double)ns.eps, kSumEach);
    else
        with_format(in_fmt, [&](auto f) {
            hipLaunchKernelGGL((k_orth_start<false, decltype(f)::value>), dim3(grid_x), block, 0, s, T, h, (double)ns.eps,
                               kSumEach);
        });
    if ((e = hipGetLastError()) != hipSuccess) return e;

    // the matrices of each way of taking the steps, one after the other
    for (const bool direct : {true, false}) {
        OrthTable part = T;
        part.n = 0;
        for (int t = 0; t < T.n; ++t) {
            if (steps_direct(T.e[t]) != direct) continue;
            part.e[part.n] = T.e[t];
            part.p[part.n++] = T.p[t];
        }
        if (part.n && (e = launch_steps(part, h, step, out_fmt, ns, direct, s)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bc
