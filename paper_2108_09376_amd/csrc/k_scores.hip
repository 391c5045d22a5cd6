// Losses on maps of class scores, with their gradients: the divergence from a teacher's record
// and the clipped policy loss; and the log probabilities of decisions.
//
//   s = sum over the classes but the action a of exp(z - m), m their maximum, x = s exp(m - z_a):
//   log pi(a) = -log(1 + x), 1 - pi(a) = x / (1 + x), exact for a probability near 1 too;
//   entropy = log s - sum of exp(z - m) (z - m) / s over all classes.
// Every gradient is, away from a few classes that are known by their index, one factor of the
// row times exp(z - m): F = -g (1 - pi(a)) / s for the policy loss (its derivative g by log pi(a);
// the action itself gets g (1 - pi(a))); for the divergence, with everything scaled by
// 1 / temperature, F = w (q_rest - p_rest) / s_rest, where s_rest runs over the classes outside the
// record alone (a difference of sums would lose it where the record holds nearly everything), and a
// class of the record gets w (q_j - p_j).
//
// All are bound by memory: a row is read once, kept in registers, and its gradient written
// from there. A row belongs to 8 to 64 lanes of a wave, or to a workgroup of up to 1024
// threads. Few rows, and rows too long for a workgroup's registers, are split into chunks:
// one launch leaves each chunk's maximum and sum, a second joins them and writes the gradient.
//
// A row's loss goes to its workgroup's sum, and the workgroups' sums are added by a launch of their
// own, each in its order and in fp64: no atomics, equal bits in every run.
#include "score_rows.h"

namespace bc {
namespace {

constexpr int kMaxTop = 64;

// The sums of a workgroup's groups (first thread of each) in the order of the groups.
template <int L>
__device__ __forceinline__ void write_part(double loss, double kl, double2 *out)
{
    constexpr int G = kThreadsOf<L> / (L <= 64 ? L : kThreadsOf<L>);
    __shared__ double2 sums[G];
    if (threadIdx.x % L == 0) sums[threadIdx.x / L] = make_double2(loss, kl);
    __syncthreads();
    if (threadIdx.x == 0) {
        double2 s = sums[0];
        for (int i = 1; i < G; ++i) {
            s.x += sums[i].x;
            s.y += sums[i].y;
        }
        *out = s;
    }
    __syncthreads();
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// exp(x) - 1 - x, at full relative accuracy near 0 too (x^2 / 2 + x^3 / 6 + ...).
__device__ __forceinline__ float exp_above_line(float x)
{
    if (fabsf(x) < 0.25f) {
        float s = 1.f / 40320.f;
        s = fmaf(s, x, 1.f / 5040.f);
        s = fmaf(s, x, 1.f / 720.f);
        s = fmaf(s, x, 1.f / 120.f);
        s = fmaf(s, x, 1.f / 24.f);
        s = fmaf(s, x, 1.f / 6.f);
        s = fmaf(s, x, 0.5f);
        return s * x * x;
    }
    return exp_of(x) - 1.f - x;
}

// ---------------------------------------------------------------- divergence from a record

// The entries of a group's record, as its lanes share them.
struct Record {
    int index[kMaxTop];                        // within the chunk; -1: not this entry's to write
    int next[kMaxTop];                         // entry + 1 that the same lane holds, 0: none
    float fix[kMaxTop];                        // the class's gradient
};

template <int FMT, int L, int NV, int PASS>
__global__ __launch_bounds__((kThreadsOf<L>)) void k_distill(DistillArgs a, ScoreGeom g)
{
    using Row = ScoreRow<FMT, L, NV>;
    constexpr int T = kThreadsOf<L>, G = L <= 64 ? T / L : 1;
    constexpr int EL = L < 64 ? L : 64, SLOTS = kMaxTop / EL;    // lanes that hold entries, entries of each
    __shared__ int head[T];                    // a thread's first entry + 1 (0: none)
    __shared__ Record records[G];
    __shared__ Stats waves[L > 64 ? L / 64 : 1];
    __shared__ float pub[2];
    const int group = L <= 64 ? threadIdx.x / L : 0, lane = threadIdx.x % L;
    Record &rec = records[group];
    const bool holder = L <= 64 || threadIdx.x < 64;             // of entries
    const float k2 = kLog2e * a.inv_t;
    auto meet = [] {
        if constexpr (L > 64) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    };
    head[threadIdx.x] = 0;
    __syncthreads();

    const size_t items = PASS == kWhole ? (size_t)g.images * g.per : (size_t)g.images * g.hw * g.chunks;
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        double loss = 0.0;
        const size_t first = PASS == kWhole ? item / g.per * g.hw : item / g.chunks;
        const int chunk = PASS == kWhole ? 0 : (int)(item % g.chunks);
        uint32_t p = PASS == kWhole ? (uint32_t)(item % g.per) * G + group : 0;
        // groups of one wave end at rows of their own; a workgroup has one group
        for (; p < (PASS == kWhole ? g.hw : 1u); p += g.per * G) {
            const Chunk c = chunk_of<PASS>(g, first + p, chunk);
            const float wt = a.weight ? a.weight[c.row] : 1.f;
            if (wt == 0.f) {
                if (PASS != kFirst && a.grad) Row::store_zeros(a.grad, c.base, c.len);
                continue;
            }
            if (L > 64) __syncthreads();                         // the last row's entries are done with
            Row row;
            row.load(a.x, c.base, c.len, c.live);
            // entries: class, teacher's score, student's score
            int idx[SLOTS];
            float tt[SLOTS], zk[SLOTS];
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                const int e = s * EL + lane;
                idx[s] = -1;
                tt[s] = zk[s] = -kInf;
                if (!holder || e >= a.k) continue;
                const int i = a.index[c.row * a.k + e];
                const bool valid = (unsigned)i < (unsigned)g.classes;
                if (valid) {
                    idx[s] = i;
                    tt[s] = load_elem(a.top, a.top_fmt, c.row * a.k + e) * a.inv_t;
                    if constexpr (PASS == kSecond) zk[s] = a.pick[c.row * a.k + e];
                    else zk[s] = load_elem(a.x, FMT, c.row * (size_t)g.c + i);
                }
                const int local = valid && i >= c.off && i < c.off + c.len ? i - c.off : -1;
                rec.index[e] = local;
                if (local >= 0) rec.next[e] = atomicExch(&head[group * L + Row::owner(local, c.len)], e + 1);
                if constexpr (PASS == kFirst)
                    if (local >= 0) a.pick[c.row * a.k + e] = zk[s];
            }
            meet();
            Stats st = {};
            if constexpr (PASS != kSecond) {
                for (int h = head[threadIdx.x]; h; h = rec.next[h - 1]) row.mask(rec.index[h - 1], c.len);
                st = team_stats<L, false>(row.template stats<false>(k2), waves, k2);
            }
            if constexpr (PASS == kFirst) {
                if (threadIdx.x == 0) a.stats[item] = make_float4(st.m, st.s, 0.f, 0.f);
                meet();
                head[threadIdx.x] = 0;
                continue;
            }
            float F = 0.f, m_r = 0.f;
            if (holder) {
                if constexpr (PASS == kSecond) st = row_stats<false>(a.stats + c.row * g.chunks, g.chunks, k2);
                // a class's first entry stands for it; entries of one class that no chunk shares are
                // found by their index
                bool lead[SLOTS];
                float M = st.m, Mt = a.rest ? a.rest[c.row] : -kInf;
                const float rest = Mt;
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) {
                    lead[s] = idx[s] >= 0;
                    if (s * EL >= a.k) continue;
                    M = fmaxf(M, zk[s]);
                    Mt = fmaxf(Mt, tt[s]);
                }
                M = lane_max<EL>(M);
                Mt = lane_max<EL>(Mt);
                M = M == -kInf ? 0.f : M;
                Mt = Mt == -kInf ? 0.f : Mt;
                bool twice = false;
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) {
                    if (s * EL >= a.k) continue;
                    if constexpr (PASS == kWhole) {
                        if (idx[s] < 0) continue;
                        const int e = s * EL + lane;
                        for (int h = head[group * L + Row::owner(idx[s], c.len)]; h; h = rec.next[h - 1])
                            if (h - 1 < e && rec.index[h - 1] == idx[s]) lead[s] = false;
                    } else {
                        for (int e = 0; e < a.k; ++e)
                            if (e < s * EL + lane && idx[s] >= 0 && a.index[c.row * a.k + e] == idx[s]) lead[s] = false;
                    }
                    twice |= idx[s] >= 0 && !lead[s];
                }
                float top = 0.f, tp = 0.f;                       // sums of exponentials over the record
                float ek[SLOTS], pk[SLOTS];
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) {
                    ek[s] = pk[s] = 0.f;
                    if (s * EL >= a.k) continue;
                    if (idx[s] >= 0) {
                        ek[s] = exp2_of(zk[s], M, k2);
                        pk[s] = exp_of(tt[s] - Mt);
                    }
                    top += lead[s] ? ek[s] : 0.f;
                    tp += pk[s];
                }
                top = lane_sum<EL>(top);
                tp = lane_sum<EL>(tp);
                const float er = st.m == -kInf ? st.s : st.s * exp2_of(st.m, M, k2);
                const float total = top + er, tr = a.rest ? exp_of(rest - Mt) : 0.f, ttotal = tp + tr;
                const bool part = total != 0.f && ttotal != 0.f;    // a NaN takes part
                const float inv = 1.f / total, tinv = 1.f / ttotal;
                const float logs = __logf(total) - __logf(ttotal);
                const float q_r = er * inv, p_r = tr * tinv, scale = wt * a.scale;
                // q_rest - p_rest from the side that does not cancel
                float each = 0.f, diff = 0.f;
#pragma unroll
                for (int s = 0; s < SLOTS; ++s) {
                    if (s * EL >= a.k) continue;
                    const float q = ek[s] * inv, pp = pk[s] * tinv;
                    // log(p / q), and p log(p / q) - p + q: both distributions sum to 1
                    const float d = (tt[s] - Mt) - (zk[s] - M) * a.inv_t + logs;
                    if (idx[s] >= 0) {
                        each += lead[s] ? (pp > 0.f ? pp * exp_above_line(-d) : q + pp) : (pp > 0.f ? pp * (d - 1.f) : pp);
                        diff += pp - (lead[s] ? q : 0.f);
                    }
                }
                each = lane_sum<EL>(each);
                diff = lane_sum<EL>(diff);
                const float dr = (rest - Mt) - ((st.m - M) * a.inv_t + __logf(st.s)) + logs;
                each += p_r > 0.f ? (st.s == 0.f ? kInf : p_r * exp_above_line(-dr)) : q_r + p_r;
                if (!(q_r > 0.5f)) diff = q_r - p_r;
                if (part) loss += (double)(scale * each);
                const float by = scale * a.inv_t;
                F = part && st.s != 0.f ? by * diff / st.s : 0.f;
                m_r = st.m == -kInf ? 0.f : st.m;
                if (a.grad) {
                    const bool doubled = __any(twice);
#pragma unroll
                    for (int s = 0; s < SLOTS; ++s) {
                        if (s * EL >= a.k || idx[s] < 0) continue;
                        const int e = s * EL + lane;
                        float pp = pk[s] * tinv;
                        if (doubled && lead[s]) {
                            pp = 0.f;
                            for (int o = 0; o < a.k; ++o)
                                if (a.index[c.row * a.k + o] == idx[s])
                                    pp += exp_of(load_elem(a.top, a.top_fmt, c.row * a.k + o) * a.inv_t - Mt) * tinv;
                        }
                        rec.fix[e] = part ? by * (ek[s] * inv - pp) : 0.f;
                        if (!lead[s]) rec.index[e] = -1;
                    }
                }
                if (L > 64 && threadIdx.x == 0) {
                    pub[0] = F;
                    pub[1] = m_r;
                }
            }
            meet();
            if constexpr (L > 64) {
                F = pub[0];
                m_r = pub[1];
            }
            if (a.grad) {
                row.store(a.grad, c.base, c.len, c.live,
                          [&](float z) { return F == 0.f ? 0.f : exp2_of(z, m_r, k2) * F; });
                // the record's own, over what the same thread has just stored there
                for (int h = head[threadIdx.x]; h; h = rec.next[h - 1])
                    if (rec.index[h - 1] >= 0) {
                        const float y[1] = {rec.fix[h - 1]};
                        store_raw<FMT, 1>(a.grad, c.base + rec.index[h - 1], pack<FMT, 1>(y));
                    }
            }
            head[threadIdx.x] = 0;
        }
        if (PASS == kWhole && a.part) write_part<L>(loss, 0.0, a.part + item);
        if (PASS == kSecond && a.part && chunk == 0 && threadIdx.x == 0) a.part[item / g.chunks] = make_double2(loss, 0.0);
    }
}

// ---------------------------------------------------------------- policy

// Log probability of an action with score za above -inf, and 1 - its probability, from the
// statistics of the other classes.
struct Chosen {
    double l, other;
};

__device__ __forceinline__ Chosen chosen(float za, const Stats &st)
{
    if (st.s == 0.f) return {0.0, 0.0};
    const double d = (double)st.m - (double)za;
    if (d > 0.0) {                                               // exp(-d) below s: past exp's range too
        const double t = exp(-d), s = (double)st.s + t;
        return {-d - log(s), (double)st.s / s};
    }
    const double x = (double)st.s * exp(d);
    return {-log1p(x), x / (1.0 + x)};
}

// The clipped loss of one decision with log probability l, and its derivative by l.
struct Decision {
    double loss, kl, slope;
};

__device__ __forceinline__ Decision decide(const ClipArgs &a, size_t row, double l)
{
    const double adv = a.advantage[row], r = exp(l - (double)a.old_logp[row]);
    const double lo = 1.0 - (double)a.low, hi = 1.0 + (double)a.high;
    const double kept = r * adv, held = (r < lo ? lo : r > hi ? hi : r) * adv;
    const bool open = !(kept > held);                            // a NaN stays one
    Decision d = {-(open ? kept : held), 0.0, open ? -kept : 0.0};
    if (a.ref_logp) {
        const double x = (double)a.ref_logp[row] - l, up = expm1(x);
        d.kl = up - x;
        d.loss += (double)a.beta * d.kl;
        d.slope -= (double)a.beta * up;
    }
    return d;
}

template <int FMT, int L, int NV, int PASS>
__global__ __launch_bounds__((kThreadsOf<L>)) void k_clip(ClipArgs a, ScoreGeom g)
{
    using Row = ScoreRow<FMT, L, NV>;
    constexpr int T = kThreadsOf<L>, G = L <= 64 ? T / L : 1;
    __shared__ Stats waves[L > 64 ? L / 64 : 1];
    __shared__ float pub[3];
    const int group = L <= 64 ? threadIdx.x / L : 0;
    const int32_t *action = (const int32_t *)a.action;
    const size_t items = PASS == kWhole ? (size_t)g.images * g.per : (size_t)g.images * g.hw * g.chunks;
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        double loss = 0.0, kl = 0.0;
        const size_t first = PASS == kWhole ? item / g.per * g.hw : item / g.chunks;
        const int chunk = PASS == kWhole ? 0 : (int)(item % g.chunks);
        uint32_t p = PASS == kWhole ? (uint32_t)(item % g.per) * G + group : 0;
        for (; p < (PASS == kWhole ? g.hw : 1u); p += g.per * G) {
            const Chunk c = chunk_of<PASS>(g, first + p, chunk);
            const float wt = a.weight ? a.weight[c.row] : 1.f;
            const int act = action[c.row];
            if (wt == 0.f || (unsigned)act >= (unsigned)g.classes) {
                if (PASS != kFirst && a.grad) Row::store_zeros(a.grad, c.base, c.len);
                continue;
            }
            Row row;
            row.load(a.x, c.base, c.len, c.live);
            float za = -kInf;
            if constexpr (PASS == kSecond) za = a.pick[c.row];
            else if (PASS == kWhole || (act >= c.off && act < c.off + c.len)) za = load_elem(a.x, FMT, c.row * (size_t)g.c + act);
            const int at = act - c.off;                          // the action's place in the chunk
            const bool mine = at >= 0 && at < c.len && Row::owner(at, c.len) == Row::lane();
            Stats st = {};
            if constexpr (PASS != kSecond) {
                if (mine) row.mask(at, c.len);
                st = team_stats<L, false>(row.template stats<false>(kLog2e), waves, kLog2e);
            }
            if constexpr (PASS == kFirst) {
                if (threadIdx.x == 0) {
                    a.stats[item] = make_float4(st.m, st.s, 0.f, 0.f);
                    if (at >= 0 && at < c.len) a.pick[c.row] = za;
                }
                __syncthreads();
                continue;
            }
            float F = 0.f, own = 0.f, m = 0.f;
            if (L <= 64 || threadIdx.x < 64) {
                if constexpr (PASS == kSecond) st = row_stats<false>(a.stats + c.row * g.chunks, g.chunks, kLog2e);
                if (za != -kInf) {                               // a masked class was not chosen here
                    const Chosen ch = chosen(za, st);
                    const Decision d = decide(a, c.row, ch.l);
                    const double by = (double)wt * (double)a.scale;
                    loss += by * d.loss;
                    kl += by * d.kl;
                    own = (float)(by * d.slope * ch.other);
                    F = st.s == 0.f ? 0.f : (float)(-by * d.slope * ch.other / (double)st.s);
                    m = st.m == -kInf ? 0.f : st.m;
                }
                if (L > 64 && threadIdx.x == 0) {
                    pub[0] = F;
                    pub[1] = own;
                    pub[2] = m;
                }
            }
            if constexpr (L > 64) {
                __syncthreads();
                F = pub[0];
                own = pub[1];
                m = pub[2];
            }
            if (a.grad) {
                row.store(a.grad, c.base, c.len, c.live,
                          [&](float z) { return F == 0.f ? 0.f : exp2_of(z, m, kLog2e) * F; });
                // the action's own, over what the same thread has just stored there
                if (mine) {
                    const float y[1] = {own};
                    store_raw<FMT, 1>(a.grad, c.base + at, pack<FMT, 1>(y));
                }
            }
        }
        if (PASS == kWhole && a.part) write_part<L>(loss, kl, a.part + item);
        if (PASS == kSecond && a.part && chunk == 0 && threadIdx.x == 0) a.part[item / g.chunks] = make_double2(loss, kl);
    }
}

// st: of all classes but a valid action.
__device__ __forceinline__ void finish_logp(const LogpArgs &a, size_t row, bool valid, float za, Stats st)
{
    a.logp[row] = !valid ? 0.f : za == -kInf ? -kInf : (float)chosen(za, st).l;
    if (!a.entropy) return;
    if (za != -kInf) st = join<true>(st, {za, 1.f, 0.f}, kLog2e);
    const double h = log((double)st.s) - (double)st.sx / (double)st.s;
    a.entropy[row] = st.s == 0.f || h < 0.0 ? 0.f : (float)h;
}

template <int FMT, int L, int NV, int PASS>
__global__ __launch_bounds__((kThreadsOf<L>)) void k_logp(LogpArgs a, ScoreGeom g)
{
    using Row = ScoreRow<FMT, L, NV>;
    constexpr int T = kThreadsOf<L>, G = L <= 64 ? T / L : 1;
    __shared__ Stats waves[L > 64 ? L / 64 : 1];
    const int group = L <= 64 ? threadIdx.x / L : 0;
    const int32_t *action = (const int32_t *)a.action;
    const size_t rows = (size_t)g.images * g.hw, items = PASS == kWhole ? (rows + G - 1) / G : rows * g.chunks;
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        const size_t r = PASS == kWhole ? item * G + group : item / g.chunks;
        if (r >= rows) continue;
        const int chunk = PASS == kWhole ? 0 : (int)(item % g.chunks);
        const Chunk c = chunk_of<PASS>(g, r, chunk);
        const int act = action[r], at = act - c.off;
        const bool valid = (unsigned)act < (unsigned)g.classes, here = valid && at >= 0 && at < c.len;
        Row row;
        row.load(a.x, c.base, c.len, c.live);
        const float za = here ? load_elem(a.x, FMT, c.row * (size_t)g.c + act) : -kInf;
        if (here && Row::owner(at, c.len) == Row::lane()) row.mask(at, c.len);
        Stats st = a.entropy ? team_stats<L, true>(row.template stats<true>(kLog2e), waves, kLog2e)
                             : team_stats<L, false>(row.template stats<false>(kLog2e), waves, kLog2e);
        if (Row::lane() == 0) {
            if constexpr (PASS == kFirst) {
                a.stats[item] = make_float4(st.m, st.s, st.sx, 0.f);
                if (here) a.pick[r] = za;
            } else {
                finish_logp(a, r, valid, za, st);
            }
        }
        if constexpr (L > 64) __syncthreads();
    }
}

// The chunks of each row joined, one row per thread.
__global__ __launch_bounds__(64) void k_logp_join(LogpArgs a, ScoreGeom g)
{
    const size_t rows = (size_t)g.images * g.hw;
    for (size_t r = (size_t)blockIdx.x * 64 + threadIdx.x; r < rows; r += (size_t)gridDim.x * 64) {
        const Stats st = row_stats<true>(a.stats + r * g.chunks, g.chunks, kLog2e);
        const bool valid = (unsigned)((const int32_t *)a.action)[r] < (unsigned)g.classes;
        finish_logp(a, r, valid, valid ? a.pick[r] : -kInf, st);
    }
}

// Decisions to execute a block or not: pi(1) = sigmoid(z). A pixel belongs to one thread, which
// writes its channels' gradient too (0 past the first).
struct Binary {
    double l, other;                           // log pi(action), 1 - pi(action)
};

__device__ __forceinline__ Binary binary(float z, bool executed)
{
    const double x = executed ? (double)z : -(double)z, t = exp(-fabs(x));
    return {(x < 0.0 ? x : 0.0) - log1p(t), (x < 0.0 ? 1.0 : t) / (1.0 + t)};
}

template <int FMT>
__global__ __launch_bounds__(256) void k_logp_binary(LogpArgs a, ScoreGeom g)
{
    const size_t rows = (size_t)g.images * g.hw;
    for (size_t r = (size_t)blockIdx.x * 256 + threadIdx.x; r < rows; r += (size_t)gridDim.x * 256) {
        const float z = load_elem(a.x, FMT, r * (size_t)g.c);
        const Binary b = binary(z, ((const uint8_t *)a.action)[r] != 0);
        a.logp[r] = (float)b.l;
        if (a.entropy) {
            // both outcomes: the likelier one's log plus what the other's adds
            const Binary up = binary(fabsf(z), true);
            const double far = up.other * fabs((double)z);
            a.entropy[r] = (float)(-up.l + (z - z == 0.f ? far : 0.0) + (z != z ? (double)z : 0.0));
        }
    }
}

template <int FMT>
__global__ __launch_bounds__(256) void k_clip_binary(ClipArgs a, ScoreGeom g)
{
    constexpr int VEC = kVec<FMT>;
    const size_t items = (size_t)g.images * g.per;
    for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
        double loss = 0.0, kl = 0.0;
        const size_t first = item / g.per * g.hw;
        for (uint32_t p = (uint32_t)(item % g.per) * 256 + threadIdx.x; p < g.hw; p += g.per * 256) {
            const size_t r = first + p, base = r * (size_t)g.c;
            const float wt = a.weight ? a.weight[r] : 1.f;
            float y[1] = {0.f};
            if (wt != 0.f) {
                const bool executed = ((const uint8_t *)a.action)[r] != 0;
                const float z = load_elem(a.x, FMT, base);
                const Binary b = binary(z, executed);
                if (b.l != -(double)kInf) {
                    const Decision d = decide(a, r, b.l);
                    const double by = (double)wt * (double)a.scale;
                    loss += by * d.loss;
                    kl += by * d.kl;
                    y[0] = (float)(by * d.slope * (executed ? b.other : -b.other));
                }
            }
            if (a.grad) {
                store_raw<FMT, 1>(a.grad, base, pack<FMT, 1>(y));
                const Raw<FMT, 1> zero = {};
                const Raw<FMT, VEC> zeros = {};
                int e = 1;
                for (; e + VEC <= g.c; e += VEC) store_raw<FMT, VEC>(a.grad, base + e, zeros);
                for (; e < g.c; ++e) store_raw<FMT, 1>(a.grad, base + e, zero);
            }
        }
        if (a.part) write_part<1>(loss, kl, a.part + item);
    }
}

// ---------------------------------------------------------------- sums of the losses

__global__ __launch_bounds__(256) void k_loss_sum(const double2 *part, uint32_t images, uint32_t per, float *loss,
                                                  float *kl)
{
    __shared__ double2 lds[256];
    for (uint32_t i = blockIdx.x; i < images; i += gridDim.x) {
        double2 s = make_double2(0.0, 0.0);
        for (uint32_t p = threadIdx.x; p < per; p += 256) {
            const double2 v = part[(size_t)i * per + p];
            s.x += v.x;
            s.y += v.y;
        }
        lds[threadIdx.x] = s;
        __syncthreads();
        for (int w = 128; w; w >>= 1) {
            if ((int)threadIdx.x < w) {
                lds[threadIdx.x].x += lds[threadIdx.x + w].x;
                lds[threadIdx.x].y += lds[threadIdx.x + w].y;
            }
            __syncthreads();
        }
        if (threadIdx.x == 0) {
            if (loss) loss[i] = (float)lds[0].x;
            if (kl) kl[i] = (float)lds[0].y;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- launches

hipError_t launch_sum(const ScoreGeom &g, const double2 *part, uint32_t per, float *loss, float *kl, hipStream_t s)
{
    hipLaunchKernelGGL(k_loss_sum, dim3(grid_of(g.images)), dim3(256), 0, s, part, g.images, per, loss, kl);
    return hipGetLastError();
}

}  // namespace

// Rows in whole where there are many, in chunks where few would leave most of the device idle
// or where one does not fit a workgroup's registers.
ScorePlan score_plan(ScoreGeom &g, int fmt, int picks, bool sums)
{
    const int vec = fmt == kF32 ? 4 : 8;
    const size_t rows = (size_t)g.images * g.hw;
    ScorePlan p = {};
    const int nvec = g.len / vec;
    p.form = 0;
    while (p.form < kFormCount && kForms[p.form].lanes * kForms[p.form].nv < nvec) ++p.form;
    g.chunks = 1;
    g.chunk = g.len;
    const int least = kForms[kChunkForm].lanes * kForms[kChunkForm].nv * vec;
    if (p.form == kFormCount || (p.form > kChunkForm && rows < 128)) {
        p.form = kChunkForm;
        g.chunk = least;
        g.chunks = (int)(((int64_t)g.len + least - 1) / least);
    }
    p.split = g.chunks > 1;
    const int lanes = kForms[p.form].lanes, groups = g.classes == 1 ? 256 : lanes <= 64 ? 256 / lanes : 1;
    g.per = p.split ? g.hw : std::min<uint32_t>((g.hw + groups - 1) / groups, lanes <= 64 ? 1024u : 8192u);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    if (p.split) {
        p.stats = take(rows * g.chunks * 16);
        p.pick = take(rows * (size_t)picks * 4);
    }
    if (sums) p.part = take((size_t)g.images * g.per * 16);
    p.bytes = at;
    return p;
}

hipError_t launch_distill(DistillArgs a, ScoreGeom g, const ScorePlan &p, void *work, float *loss, int fmt, hipStream_t s)
{
    uint8_t *w = (uint8_t *)work;
    a.stats = (float4 *)(w + p.stats);
    a.pick = (float *)(w + p.pick);
    a.part = loss ? (double2 *)(w + p.part) : nullptr;
    const size_t rows = (size_t)g.images * g.hw;
    hipError_t e = with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        if (p.split) {
            constexpr int L = kForms[kChunkForm].lanes, NV = kForms[kChunkForm].nv;
            const dim3 grid(grid_of(rows * g.chunks));
            hipLaunchKernelGGL((k_distill<FMT, L, NV, kFirst>), grid, dim3(L), 0, s, a, g);
            hipLaunchKernelGGL((k_distill<FMT, L, NV, kSecond>), grid, dim3(L), 0, s, a, g);
            return hipGetLastError();
        }
        return with_form(p.form, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, NV = decltype(n)::value;
            hipLaunchKernelGGL((k_distill<FMT, L, NV, kWhole>), dim3(grid_of((size_t)g.images * g.per)),
                               dim3(kThreadsOf<L>), 0, s, a, g);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || !loss) return e;
    return launch_sum(g, a.part, g.per, loss, nullptr, s);
}

hipError_t launch_clip(ClipArgs a, ScoreGeom g, const ScorePlan &p, void *work, float *loss, float *kl, int fmt, hipStream_t s)
{
    uint8_t *w = (uint8_t *)work;
    a.stats = (float4 *)(w + p.stats);
    a.pick = (float *)(w + p.pick);
    a.part = loss || kl ? (double2 *)(w + p.part) : nullptr;
    const size_t rows = (size_t)g.images * g.hw;
    hipError_t e = with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        if (g.classes == 1) {
            hipLaunchKernelGGL((k_clip_binary<FMT>), dim3(grid_of((size_t)g.images * g.per)), dim3(256), 0, s, a, g);
            return hipGetLastError();
        }
        if (p.split) {
            constexpr int L = kForms[kChunkForm].lanes, NV = kForms[kChunkForm].nv;
            const dim3 grid(grid_of(rows * g.chunks));
            hipLaunchKernelGGL((k_clip<FMT, L, NV, kFirst>), grid, dim3(L), 0, s, a, g);
            hipLaunchKernelGGL((k_clip<FMT, L, NV, kSecond>), grid, dim3(L), 0, s, a, g);
            return hipGetLastError();
        }
        return with_form(p.form, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, NV = decltype(n)::value;
            hipLaunchKernelGGL((k_clip<FMT, L, NV, kWhole>), dim3(grid_of((size_t)g.images * g.per)),
                               dim3(kThreadsOf<L>), 0, s, a, g);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || !a.part) return e;
    return launch_sum(g, a.part, g.per, loss, kl, s);
}

hipError_t launch_logp(LogpArgs a, ScoreGeom g, const ScorePlan &p, void *work, int fmt, hipStream_t s)
{
    uint8_t *w = (uint8_t *)work;
    a.stats = (float4 *)(w + p.stats);
    a.pick = (float *)(w + p.pick);
    const size_t rows = (size_t)g.images * g.hw;
    return with_format(fmt, [&](auto f) {
        constexpr int FMT = decltype(f)::value;
        if (g.classes == 1) {
            hipLaunchKernelGGL((k_logp_binary<FMT>), dim3(grid_of((rows + 255) / 256)), dim3(256), 0, s, a, g);
            return hipGetLastError();
        }
        if (p.split) {
            constexpr int L = kForms[kChunkForm].lanes, NV = kForms[kChunkForm].nv;
            hipLaunchKernelGGL((k_logp<FMT, L, NV, kFirst>), dim3(grid_of(rows * g.chunks)), dim3(L), 0, s, a, g);
            hipLaunchKernelGGL(k_logp_join, dim3(grid_of((rows + 63) / 64)), dim3(64), 0, s, a, g);
            return hipGetLastError();
        }
        return with_form(p.form, [&](auto l, auto n) {
            constexpr int L = decltype(l)::value, NV = decltype(n)::value, G = L <= 64 ? kThreadsOf<L> / L : 1;
            hipLaunchKernelGGL((k_logp<FMT, L, NV, kWhole>), dim3(grid_of((rows + G - 1) / G)), dim3(kThreadsOf<L>), 0, s, a,
                               g);
            return hipGetLastError();
        });
    });
}

}  // namespace bc
