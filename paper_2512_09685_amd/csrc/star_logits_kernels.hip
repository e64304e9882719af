// Losses on the logits of the taken tokens, and their gradients.
//
// A row of logits l_0 .. l_{V-1} gives, with k = log2(e) / temperature and m = max l,
//     e_j = 2^((l_j - m) k),   s = sum e_j,   logp = (l_y - m) / temperature - log s,   p_j = e_j / s
// and every loss here is a function of the rows' logp, so that its gradient is one number c a row:
//     dl_j = c / temperature ([j = y] - p_j).
// All of it is bound by memory: 2 or 4 bytes an element in, as many out, against about 4 operations.
#include <hip/hip_runtime.h>

#include "star_logits.h"

namespace star {

namespace {

// Up to this many rows are cut into sections, if they have at least so many chunks: for the policy loss, which is two launches either
// way (whole rows against sections, us: 1 x 131072, bf16: 20.6 / 10.7; 64 / 96 / 128 x 131072, bf16: 21.3 / 11.2, 21.7 / 12.5, 22.1 / 15.9, fp32:
// 24.3 / 14.2, 30.7 / 24.4, 33.8 / 30.5; x 32000 of either type 11.8 / 11.0 at 64 and 11.1 / 10.6 at 128), and for log-probabilities, where the second
// launch has to pay (1 x 131072, fp32: 12.6 / 9.8, bf16 9.9 / 9.1; 48 x 32000, fp32: 6.4 / 9.0).  Beyond the turn the policy loss still gains
// a little up to 160 rows (129 x 131072, bf16: 22.3 / 18.1, 160: 23.2 / 21.6, 200: 26.8 / 27.5; fp32, 129: 36.1 / 32.4, 255: equal), but log-probabilities
// lose (128 x 131072, bf16: 11.1 / 10.3, fp32: 14.3 / 15.8; 160: 11.8 / 13.8 and 14.9 / 18.5).
constexpr int64_t kFewTokens = 128, kPolicySections = 2048, kLogprobsSections = 16384;

// Whether token t counts.
__device__ __forceinline__ bool counts(const Logits& l, int64_t t, int64_t y) {
    return y >= 0 && y < l.vocab && (!l.weights || l.weights[t] != 0.f);
}

// One token's loss, KL estimate, whether it is clipped, and its derivative by logp (unweighted).
struct PolicyTerm {
    float loss, kl, clipped, slope;
};
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& a, int64_t t, const Two& logp) {
    const float A = a.advantages[t], r = expf((logp.high - a.old_logp[t]) + logp.low);
    const float held = fminf(fmaxf(r, a.low), a.high);
    // (an advantage of 0 costs nothing, also where the ratio has run over; where there is no ratio there is no cost to tell)
    const bool none = A == 0.f && r == r;
    const float free_cost = none ? 0.f : -A * r, held_cost = none ? 0.f : -A * held;
    PolicyTerm p;
    p.clipped = free_cost < held_cost ? 1.f : 0.f;
    p.loss = free_cost < held_cost ? held_cost : free_cost;
    p.slope = free_cost < held_cost ? 0.f : free_cost;
    p.kl = 0.f;
    if (a.kl != 0.f) {
        const float d = (a.ref_logp[t] - logp.high) - logp.low, q = expm1f(d);
        p.kl = kl_of(d, q);
        p.loss += a.kl * p.kl;
        p.slope -= a.kl * q;
    }
    return p;
}

// One chunk of the gradient from its elements but for the target: `c` more at element `at` of it, rounded.
template <class E>
__device__ __forceinline__ u32x4 finish_chunk(float (&v)[E::VEC], float c, int at) {
    if (at >= 0 && at < E::VEC)
        static_for<0, E::VEC>([&](auto I) { v[decltype(I)::value] += at == decltype(I)::value ? c : 0.f; });
    return E::pack(v);
}

// dl_j = scaled * 2^(l_j k - e), plus `c` at the target: one chunk, one element.  Where a product with k would not hold the row's
// values (`far`), scaled * 2^((l_j - m) k).
struct Slope {
    float k, e, m, scaled, c;
    int y;
    bool far;
    __device__ __forceinline__ float operator()(float l) const {
        return scaled * __builtin_amdgcn_exp2f(far ? (l - m) * k : __builtin_fmaf(l, k, -e));
    }
};
// Of a row whose sum of 2^((l_j - m) k) is s.
__device__ __forceinline__ Slope slope_of(float k, const MaxSum& all, float c, int64_t y) {
    const bool far = is_far(all.m * k);
    const float e = far ? 0.f : rintf(all.m * k), off = far ? 0.f : __builtin_fmaf(all.m, k, -e);
    return Slope{k, e, all.m, -c / all.s * __builtin_amdgcn_exp2f(-off), c, (int)y, far};
}
template <class E>
__device__ __forceinline__ u32x4 slope_chunk(const u32x4& x, const Slope& p, int first) {
    float v[E::VEC];
    if (p.far)
        static_for<0, E::VEC>([&](auto I) { v[decltype(I)::value] = p(E::template get<decltype(I)::value>(x)); });
    else
        static_for<0, E::VEC>([&](auto I) {
            v[decltype(I)::value] = p.scaled * __builtin_amdgcn_exp2f(__builtin_fmaf(E::template get<decltype(I)::value>(x), p.k, -p.e));
        });
    return finish_chunk<E>(v, p.c, p.y - first);
}
template <class E, int NT, int C>
__device__ __forceinline__ void store_slopes(const u32x4 (&x)[C], char* out, const RowSpan& sp, const Slope& p, int first) {
    u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        const int at = first + i * NT;
        if (at < sp.chunks) __builtin_nontemporal_store(slope_chunk<E>(x[i], p, sp.head + at * E::VEC), to + at);
    });
}
// The gradient of chunks that were scanned, read again from their end.
template <class E, int NT>
__device__ __forceinline__ void store_again(const char* row, char* out, const RowSpan& sp, const Slope& p, int tid) {
    for (int first = (sp.chunks - 1) / (4 * NT) * (4 * NT); first >= 0; first -= 4 * NT) {
        u32x4 z[4];
        load_chunks<E, NT>(z, row, sp, first + tid);
        store_slopes<E, NT>(z, out, sp, p, first + tid);
    }
}
template <class E>
__device__ __forceinline__ void store_slope(float l, char* out, const RowSpan& sp, const Slope& p, int tid) {
    const int j = sp.edge_element(tid);
    E::put(out, j, j == p.y ? p(l) + p.c : p(l));
}

enum class RowWork { Logprobs, Policy };

struct RowArgs {
    Logits l;
    PolicyArgs policy;
    float *logp, *logp_low, *lse;  // the last two may be null
    MaxSum* sums;                  // may be null
    char* dlogits;
    int64_t ld_out, first, rows;   // rows [first, first + rows)
    bool again;                    // the rows are read again by the gradient's launch
    const float *lse_in, *dlogp;   // of the gradient alone, as are
    const MaxSum* sums_in;         // the rows' maxima and sums, or lse_in (Normaliser)
    MaxSum* parts;                 // of rows that several workgroups share: [rows][sections]
    float* picked;                 // of such rows: the target's logit, which a gradient in place would be written over
    int sections, lanes;           // lanes that join a row's sections: a power of two, no more than a wave's
    float* stats;
    PairLoss loss;                 // of the pairs whose gradient this is; its output null: none
    unsigned int* ticket;          // cleared for the launch behind this one; null: it needs none
};

__device__ __forceinline__ const char* row_of(const RowArgs& a, int64_t t, int bytes) {
    return reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * bytes;
}
__device__ __forceinline__ float scaled_weight(const RowArgs& a, int64_t t) { return a.policy.scale * (a.l.weights ? a.l.weights[t] : 1.f); }

// logp and lse from the row's maximum and log sum exp(z - max z); `ly`: the target's logit.
__device__ __forceinline__ Two logp_of(const RowArgs& a, float m, const Two& log_s, float ly) {
    return add(scaled_difference(a.l, ly, m), log_s, -1.f);
}
__device__ __forceinline__ float lse_of(const RowArgs& a, float m, const Two& log_s) { return add(scaled_difference(a.l, m, 0.f), log_s, 1.f).high; }
__device__ __forceinline__ void put_row(const RowArgs& a, int64_t t, const Two& logp, float lse) {
    a.logp[t] = logp.high;
    if (a.logp_low) a.logp_low[t] = logp.low;
    if (a.lse) a.lse[t] = lse;
}
__device__ __forceinline__ void put_sum(const RowArgs& a, int64_t t, float m, float s) {
    if (a.sums) a.sums[t] = MaxSum{m, s};
}

__device__ __forceinline__ void clear_ticket(const RowArgs& a) {
    if (a.ticket && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0u;
}

// The whole row in registers, C chunks a thread: read once, written once.  NT threads a row, ROWS rows a workgroup.
// Registers and not LDS, because a unit has three times as much of them; rows of up to 8192 chunks let two workgroups of
// 1024 threads share a unit, of which one reads while the other writes, and rows of up to 13312 two of 512.
// Beside the memory it is the vector instructions that count (an exponential takes four turns of the others), so an
// exponent is one multiply-add, l k - e with e = round(max l k), a whole number that costs the sum no rounding; and
// where the registers allow it, fp32 rows and bf16 rows of up to 4 chunks, the exponentials are kept for the gradient
// in the logits' place.  Rows with a maximum that no product with k would hold (is_far: nothing but a mask's value, say) are taken
// relative to it first, which loses nothing: differences that count are exact, in bf16 too, where they are then 0.
template <class E, int NT, int C, int ROWS, RowWork WORK>
__global__ __launch_bounds__(NT* ROWS, C <= 8 ? 8 : 4) void logits_held_kernel(const RowArgs a) {
    constexpr bool KEEP = WORK == RowWork::Policy && (E::VEC == 4 || C <= 4);
    __shared__ float shared[2][NT / 64];
    clear_ticket(a);
    const int V = (int)a.l.vocab, tid = threadIdx.x % NT;
    const int64_t in = NT >= 512 ? die_run(blockIdx.x) : (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0);
    if (ROWS > 1 && in >= a.rows) return;
    const int64_t t = a.first + in, y = a.l.targets[t];
    const char* row = row_of(a, t, E::BYTES);
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const float k = a.l.k;
    if (!counts(a.l, t, y)) {
        if (tid == 0) put_row(a, t, Two{0.f, 0.f}, 0.f);
        if (WORK == RowWork::Policy) zero_row<E, NT>(out, V, tid);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    u32x4 x[C];
    if (WORK == RowWork::Logprobs && a.again) load_chunks<E, NT, Reading::Again>(x, row, sp, tid);
    else load_chunks<E, NT>(x, row, sp, tid);
    float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    const float ly = E::one(row, y);
    const float m = fold_row<NT>(max_of<E>(x, edge), shared[0], [](float p, float q) { return fmaxf(p, q); });
    keep_packed(x);
    const bool far = is_far(m * k);
    if (far) {
        static_for<0, C>([&](auto I) {
            float v[E::VEC];
            static_for<0, E::VEC>([&](auto J) { v[decltype(J)::value] = E::template get<decltype(J)::value>(x[decltype(I)::value]) - m; });
            x[decltype(I)::value] = E::pack(v);
        });
        edge -= m;
    }
    const float e = far ? 0.f : rintf(m * k);
    float kept[KEEP ? C * E::VEC : 1];
    const float kept_edge = __builtin_amdgcn_exp2f(__builtin_fmaf(edge, k, -e));
    float s = kept_edge;
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) {
            constexpr int i = decltype(I)::value, j = decltype(J)::value;
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(E::template get<j>(x[i]), k, -e));
            if constexpr (KEEP) kept[i * E::VEC + j] = v;
            s += v;
        });
    });
    s = fold_row<NT>(s, shared[1], [](float p, float q) { return p + q; });
    // log sum exp(z - max z): the sum is that of 2^(z' - e)
    Two log_s = two_log(s);
    const float off = far ? 0.f : __builtin_fmaf(m, k, -e);
    log_s.low -= off * kLn2;
    const Two logp = logp_of(a, m, log_s, ly);
    if (tid == 0) {
        put_row(a, t, logp, lse_of(a, m, log_s));
        if (WORK == RowWork::Logprobs) put_sum(a, t, m, s * __builtin_amdgcn_exp2f(-off));
    }
    if constexpr (WORK == RowWork::Policy) {
        const float c = scaled_weight(a, t) * policy_term(a.policy, t, logp).slope * a.l.inv_t, scaled = -c / s;
        if constexpr (!KEEP) keep_packed(x);
        u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int at = tid + i * NT;
            if (at < sp.chunks) {
                float v[E::VEC];
                static_for<0, E::VEC>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    if constexpr (KEEP) v[j] = scaled * kept[i * E::VEC + j];
                    else v[j] = scaled * __builtin_amdgcn_exp2f(__builtin_fmaf(E::template get<j>(x[i]), k, -e));
                });
                __builtin_nontemporal_store(finish_chunk<E>(v, c, (int)y - sp.head - at * E::VEC), to + at);
            }
        });
        if (tid < sp.edge) {
            const int j = sp.edge_element(tid);
            E::put(out, j, j == (int)y ? scaled * kept_edge + c : scaled * kept_edge);
        }
    }
}

// Rows too long for that: a workgroup a row, H chunks a thread of its end in registers; for its gradient the rest of the row is read a second
// time, from its end, which the caches still hold.  (2048 x 131072, fp32, before the first reading left the rest in the memory-side
// cache: 560 us with nothing in registers, 523 / 467 / 443 with H = 8 / 14 / 20, whose registers no longer all fit; now 345.)
template <class E, int NT, int H, RowWork WORK>
__global__ __launch_bounds__(NT, 4) void logits_scan_kernel(const RowArgs a) {
    __shared__ MaxSum shared[NT / 64];
    clear_ticket(a);
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    const int64_t t = a.first + die_run(blockIdx.x), y = a.l.targets[t];
    const char* row = row_of(a, t, E::BYTES);
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const float k = a.l.k;
    if (!counts(a.l, t, y)) {
        if (tid == 0) put_row(a, t, Two{0.f, 0.f}, 0.f);
        if (WORK == RowWork::Policy) zero_row<E, NT>(out, V, tid);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    const int rest = max(sp.chunks - H * NT, 0);
    const float ly = E::one(row, y), edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    RowSpan before = sp;
    before.chunks = rest;
    MaxSum mine = WORK == RowWork::Policy || a.again ? scan_chunks<E, NT, Reading::Again>(row, before, k, tid) : scan_chunks<E, NT>(row, before, k, tid);
    u32x4 x[H > 0 ? H : 1];
    if constexpr (H > 0) {
        load_chunks<E, NT>(x, row, sp, rest + tid);
        const float m = max_of<E>(x, fmaxf(mine.m, edge)), base = m == -INFINITY ? 0.f : m;
        keep_packed(x);
        mine = MaxSum{m, mine.s * __builtin_amdgcn_exp2f((mine.m - base) * k) + sum_from<E>(x, edge, m, k)};
    } else {
        mine = with_element(mine, edge, k);
    }
    const MaxSum all = join_group<NT>(mine, k, shared);
    const Two log_s = two_log(all.s), logp = logp_of(a, all.m, log_s, ly);
    if (tid == 0) {
        put_row(a, t, logp, lse_of(a, all.m, log_s));
        if (WORK == RowWork::Logprobs) put_sum(a, t, all.m, all.s);
    }
    if constexpr (WORK == RowWork::Policy) {
        const float c = scaled_weight(a, t) * policy_term(a.policy, t, logp).slope * a.l.inv_t;
        const Slope p = slope_of(k, all, c, y);
        if constexpr (H > 0) {
            keep_packed(x);
            store_slopes<E, NT>(x, out, sp, p, rest + tid);
        }
        store_again<E, NT>(row, out, before, p, tid);
        if (tid < sp.edge) store_slope<E>(edge, out, sp, p, tid);
    }
}

// Few rows: a row's chunks are cut into sections of NT C, a workgroup each.  First launch: every section's maximum and sum.
constexpr int kSectionThreads = 256;
template <class E, int C>
__global__ __launch_bounds__(kSectionThreads) void logits_part_kernel(const RowArgs a) {
    constexpr int NT = kSectionThreads;
    __shared__ MaxSum shared[NT / 64];
    const int V = (int)a.l.vocab, tid = threadIdx.x, section = (int)(blockIdx.x % (unsigned)a.sections);
    const int64_t in = blockIdx.x / (unsigned)a.sections, t = a.first + in, y = a.l.targets[t];
    if (!counts(a.l, t, y)) return;
    const char* row = row_of(a, t, E::BYTES);
    const float k = a.l.k;
    const RowSpan sp = row_span<E, NT>(row, V);
    u32x4 x[C];
    load_chunks<E, NT, Reading::Again>(x, row, sp, section * NT * C + tid);
    const float edge = section == 0 && tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    MaxSum mine{max_of<E>(x, edge), 0.f};
    keep_packed(x);
    mine.s = sum_from<E>(x, edge, mine.m, k);
    const MaxSum all = join_group<NT>(mine, k, shared);
    if (tid == 0) a.parts[in * a.sections + section] = all;
    if (tid == 0 && section == 0) a.picked[in] = E::one(row, y);
}

// The sections of a row joined by `a.lanes` lanes side by side, four sections of each on their way at a time; every lane gets the whole.
// All launches of a call join a row this way, with as many lanes: the gradient and the sums then rest on the same bits.
__device__ __forceinline__ MaxSum join_parts(const RowArgs& a, int64_t in, float k) {
    const MaxSum* p = a.parts + in * a.sections;
    const int lane = (int)threadIdx.x & (a.lanes - 1);
    MaxSum mine{-INFINITY, 0.f};
    for (int first = lane; first < a.sections; first += 4 * a.lanes) {
        MaxSum x[4];
        float m = mine.m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = first + i * a.lanes < a.sections ? p[first + i * a.lanes] : MaxSum{-INFINITY, 0.f};
            m = fmaxf(m, x[i].m);
        }
        const float base = m == -INFINITY ? 0.f : m;
        mine = MaxSum{m, mine.s * __builtin_amdgcn_exp2f((mine.m - base) * k)};
#pragma unroll
        for (int i = 0; i < 4; ++i) mine.s += x[i].s * __builtin_amdgcn_exp2f((x[i].m - base) * k);
    }
    float m = mine.m;
    for (int d = a.lanes / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    float s = mine.s * __builtin_amdgcn_exp2f((mine.m - (m == -INFINITY ? 0.f : m)) * k);
    for (int d = a.lanes / 2; d; d >>= 1) s += __shfl_xor(s, d);
    return MaxSum{m, s};
}

// Second launch of the log-probabilities: one workgroup, `a.lanes` lanes a row.
__global__ __launch_bounds__(kSectionThreads) void logits_join_kernel(const RowArgs a) {
    const int64_t in = threadIdx.x / (unsigned)a.lanes, t = a.first + in;
    if (in >= a.rows) return;
    const int64_t y = a.l.targets[t];
    const bool live = counts(a.l, t, y);
    const MaxSum all = live ? join_parts(a, in, a.l.k) : MaxSum{0.f, 1.f};
    const Two log_s = two_log(all.s);
    if ((threadIdx.x & (a.lanes - 1)) == 0) {
        put_row(a, t, live ? logp_of(a, all.m, log_s, a.picked[in]) : Two{0.f, 0.f}, live ? lse_of(a, all.m, log_s) : 0.f);
        put_sum(a, t, all.m, all.s);
    }
}

// ---------------------------------------------------------------- sums over tokens
constexpr int kSumThreads = 1024;

// What a token adds to the four sums of the policy loss.
__device__ __forceinline__ void add_policy_term(double (&sum)[4], const PolicyTerm& p, double w) {
    sum[0] += w * p.loss;
    sum[1] += w * p.kl;
    sum[2] += w * p.clipped;
    sum[3] += w;
}

// Second launch of the policy loss on few rows: every section's gradient, and, by one workgroup more, the log-probabilities and
// sums.
template <class E, int C>
__global__ __launch_bounds__(kSectionThreads) void policy_section_kernel(const RowArgs a) {
    constexpr int NT = kSectionThreads;
    __shared__ double shared[NT / 64][4];
    const int V = (int)a.l.vocab, tid = threadIdx.x, section = (int)(blockIdx.x % (unsigned)a.sections);
    const int64_t in = blockIdx.x / (unsigned)a.sections;
    const float k = a.l.k;
    if (in >= a.rows) {
        double sum[4] = {0, 0, 0, 0};
        const int64_t t = tid / a.lanes;
        if (t < a.rows) {
            // (everything is read before anything is decided: this workgroup is the one that the others wait for; what a row that does not
            // count left in the workspace is not used)
            const int64_t y = a.l.targets[t];
            const double w = a.l.weights ? (double)a.l.weights[t] : 1.0;
            const MaxSum all = join_parts(a, t, k);
            const Two logp = logp_of(a, all.m, two_log(all.s), a.picked[t]);
            const PolicyTerm p = policy_term(a.policy, t, logp);
            const bool live = y >= 0 && y < a.l.vocab && w != 0.0;
            if ((tid & (a.lanes - 1)) == 0) {
                a.logp[t] = live ? logp.high : 0.f;
                if (live) add_policy_term(sum, p, w);
            }
        }
        group_sums<NT>(sum, shared);
        if (tid == 0)
            for (int i = 0; i < 4; ++i) a.stats[i] = (float)(sum[i] * a.policy.scale);
        return;
    }
    const int64_t t = in, y = a.l.targets[t];
    const char* row = row_of(a, t, E::BYTES);
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const int first = section * NT * C;
    if (!counts(a.l, t, y)) {
        // (the output's own chunks, which need not lie as the row's do)
        zero_row<E, NT>(out, V, tid, first, section + 1 == a.sections ? 0x7fffffff : first + NT * C);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    u32x4 x[C];
    load_chunks<E, NT>(x, row, sp, first + tid);
    const float edge = section == 0 && tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    const MaxSum all = join_parts(a, in, k);
    const float c = scaled_weight(a, t) * policy_term(a.policy, t, logp_of(a, all.m, two_log(all.s), a.picked[in])).slope * a.l.inv_t;
    const Slope p = slope_of(k, all, c, y);
    store_slopes<E, NT>(x, out, sp, p, first + tid);
    if (section == 0 && tid < sp.edge) store_slope<E>(edge, out, sp, p, tid);
}

// The pairs' terms joined, by a workgroup of kBlock threads.
__device__ __forceinline__ void join_pair_loss(const PairLoss& p) {
    __shared__ double shared[kBlock / 64][1];
    double sum[1] = {0.0};
    for (int b = threadIdx.x; b < p.pairs; b += kBlock) sum[0] += p.terms[b];
    group_sums<kBlock>(sum, shared);
    if (threadIdx.x == 0) *p.out = (float)(sum[0] * p.scale);
}

// What a row's probabilities are taken from: the maxima and sums that the call's own first reading left, or a normaliser that the caller hands in.
// (Two kernels of it: one that asks took 326 against 321 us for the preference loss of 12288 x 32768, bf16.)
enum class Normaliser { Sums, Lse };

// The gradient alone, which needs nothing of the rest of its row: NT threads to a section of C chunks each, ROWS rows a workgroup.  The
// last rows come first: the memory-side cache may still hold them.
// A normaliser that the caller hands in is one fp32 number, which holds a row's sum the worse the larger it is: rounding it enters every p as |lse|
// 2^-24.  From 64 on (4e-6), of bf16 rows from 1024 on (6e-5, a 64th of what rounding the result to bf16 adds), the row's sum is formed again, by
// the threads of its first section, which then take all of the row: no other ones read it, so that it may be written in place.  (1023 x 50021,
// fp32: 114 against 78 us; bf16, 12288 x 32768: 452 / 281, 8192 x 65536: 1166 / 379; 1 x 131072: 34 / 7.5.)
template <class E>
constexpr float kMostLse = E::VEC == 4 ? 64.f : 1024.f;
template <class E, int NT, int C, int ROWS, Normaliser FROM>
__global__ __launch_bounds__(NT* ROWS) void logits_grad_kernel(const RowArgs a) {
    __shared__ MaxSum shared[NT / 64];
    const int V = (int)a.l.vocab, tid = threadIdx.x % NT, section = (int)(blockIdx.x % (unsigned)a.sections);
    const int64_t in = (int64_t)(blockIdx.x / (unsigned)a.sections) * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0);
    if (FROM == Normaliser::Sums && a.loss.out && blockIdx.x == gridDim.x - 1) return join_pair_loss(a.loss);   // (a workgroup more than the rows need)
    if (ROWS > 1 && in >= a.rows) return;
    const int64_t t = a.first + (a.rows - 1 - in), y = a.l.targets[t];
    const char* row = row_of(a, t, E::BYTES);
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const float d = a.dlogp[t], lse = FROM == Normaliser::Lse ? a.lse_in[t] : 0.f, k = a.l.k;
    const int first = section * NT * C;
    if (!counts(a.l, t, y) || d == 0.f) {
        zero_row<E, NT>(out, V, tid, first, section + 1 == a.sections ? 0x7fffffff : first + NT * C);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    const float c = d * a.l.inv_t;
    if (FROM == Normaliser::Lse && !(fabsf(lse) <= kMostLse<E>)) {
        if (section > 0) return;
        const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
        const MaxSum all = join_group<NT>(with_element(scan_chunks<E, NT, Reading::Again>(row, sp, k, tid), edge, k), k, shared);
        const Slope p = slope_of(k, all, c, y);
        store_again<E, NT>(row, out, sp, p, tid);
        if (tid < sp.edge) store_slope<E>(edge, out, sp, p, tid);
        return;
    }
    u32x4 x[C];
    load_chunks<E, NT>(x, row, sp, first + tid);
    const float edge = section == 0 && tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    Slope p;
    if constexpr (FROM == Normaliser::Sums) {
        p = slope_of(k, a.sums_in[t], c, y);
    } else {
        // p_j = 2^((l_j - m) k - rest log2 e) with an m near lse times the temperature, and what lse is more than m / temperature: only differences
        // are multiplied with the rounded k
        const float m = lse / a.l.inv_t, rest = __builtin_fmaf(-m, a.l.inv_t, lse) - m * a.l.inv_t_low, e = rintf(m * k);
        p = Slope{k, e, m, -c * __builtin_amdgcn_exp2f(-(__builtin_fmaf(m, k, -e) + rest * kLog2e)), c, (int)y, false};
    }
    store_slopes<E, NT>(x, out, sp, p, first + tid);
    if (section == 0 && tid < sp.edge) store_slope<E>(edge, out, sp, p, tid);
}

// Workspace of the sums: a ticket, then four doubles a workgroup.
constexpr int kStatsGroups = 64;

// (a token's ratio comes from the same two numbers as in the launch that made its gradient, so that both say the same of the clip's border)
__global__ __launch_bounds__(kSumThreads) void policy_stats_kernel(const Logits l, const PolicyArgs a, const float* logp, const float* logp_low,
                                                                   float* stats, unsigned int* ticket, double* sums) {
    __shared__ double shared[kSumThreads / 64][4];
    __shared__ bool last;
    double sum[4] = {0, 0, 0, 0};
    for (int64_t t = (int64_t)blockIdx.x * kSumThreads + threadIdx.x; t < l.tokens; t += (int64_t)gridDim.x * kSumThreads)
        if (counts(l, t, l.targets[t])) add_policy_term(sum, policy_term(a, t, Two{logp[t], logp_low[t]}), l.weights ? (double)l.weights[t] : 1.0);
    group_sums<kSumThreads>(sum, shared);
    if (gridDim.x > 1) {
        // the workgroup that comes last joins all of them, in their own order
        if (threadIdx.x == 0) {
            for (int i = 0; i < 4; ++i) __hip_atomic_store(sums + 4 * blockIdx.x + i, sum[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
        }
        __syncthreads();
        if (!last) return;
        for (int i = 0; i < 4; ++i)
            sum[i] = threadIdx.x < gridDim.x ? __hip_atomic_load(sums + 4 * threadIdx.x + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        group_sums<kSumThreads>(sum, shared);
    }
    if (threadIdx.x == 0)
        for (int i = 0; i < 4; ++i) stats[i] = (float)(sum[i] * a.scale);
}

// A workgroup a pair.
__global__ __launch_bounds__(kBlock) void pair_kernel(const Logits l, const PreferenceArgs a, const PairOffsets offsets, const float* logp,
                                                      const float* logp_low, float* dlogp, float* margins, double* terms) {
    __shared__ double shared[kBlock / 64][1];
    __shared__ double all;
    const int b = blockIdx.x;
    const int64_t from = offsets.at[2 * b], mid = offsets.at[2 * b + 1], to = offsets.at[2 * b + 2];
    double sum[1] = {0.0};
    for (int64_t t = from + threadIdx.x; t < to; t += kBlock) {
        if (!counts(l, t, l.targets[t])) continue;
        const double d = (((double)logp[t] - (double)a.ref_logp[t]) + (double)logp_low[t]) * (l.weights ? (double)l.weights[t] : 1.0);
        sum[0] += t < mid ? d : -d;
    }
    group_sums<kBlock>(sum, shared);
    if (threadIdx.x == 0) all = a.beta * sum[0];
    __syncthreads();
    const double s = all;
    // -log sigmoid(s) = max(-s, 0) + log(1 + e^-|s|); the two shares are 1 together, and one of 0 costs nothing, also of an infinite margin
    const double tail = log1p(exp(-fabs(s))), share = s >= 0.0 ? (double)a.smooth : 1.0 - (double)a.smooth;
    if (threadIdx.x == 0) {
        if (margins) margins[b] = (float)s;
        terms[b] = tail + (share != 0.0 ? share * fabs(s) : 0.0);
    }
    const double sig = s >= 0 ? 1.0 / (1.0 + exp(-s)) : exp(s) / (1.0 + exp(s));
    // dl/ds = sigmoid(s) - (1 - smooth); for large s that is smooth - sigmoid(-s), without the cancellation
    const double inv = s >= 0 ? exp(-s) / (1.0 + exp(-s)) : 1.0 / (1.0 + exp(s));
    const double slope = a.scale * (double)a.beta * (s >= 0 ? (double)a.smooth - inv : sig - (1.0 - (double)a.smooth));
    if (dlogp)
        for (int64_t t = from + threadIdx.x; t < to; t += kBlock) {
            const double w = l.weights ? (double)l.weights[t] : 1.0;
            dlogp[t] = (float)((t < mid ? slope : -slope) * w);
        }
}

__global__ __launch_bounds__(kBlock) void pair_loss_kernel(const PairLoss p) { join_pair_loss(p); }

// ---------------------------------------------------------------- launches
template <class E>
int64_t chunks_of(const Logits& l) {
    return (l.vocab + E::VEC - 1) / E::VEC;
}
int64_t chunks_of(int dtype, int64_t vocab) { return dtype == STAR_F32 ? (vocab + 3) / 4 : (vocab + 7) / 8; }

// Few rows are cut into sections, of the largest size that still makes two workgroups a compute unit of them.
struct Sections {
    int chunks_a_thread, count;   // 0: rows are not cut
};
Sections sections_of(int dtype, int64_t tokens, int64_t vocab, int64_t least) {
    const int64_t chunks = chunks_of(dtype, vocab);
    if (tokens > kFewTokens || chunks < least) return Sections{0, 0};
    int c = 8;
    while (c > 1 && tokens * ((chunks + kSectionThreads * c - 1) / (kSectionThreads * c)) < 512) c /= 2;
    return Sections{c, (int)((chunks + kSectionThreads * c - 1) / (kSectionThreads * c))};
}

// Lanes that join the sections of a row, where one workgroup joins all rows (kFewTokens at most).
static_assert(kFewTokens <= kSectionThreads);
int join_lanes(int64_t rows) {
    int lanes = 64;
    while (lanes > 1 && rows * lanes > kSectionThreads) lanes /= 2;
    return lanes;
}

template <class F>
void for_section(const Sections& s, F&& launch) {
    if (s.chunks_a_thread == 8) launch(std::integral_constant<int, 8>{});
    else if (s.chunks_a_thread == 4) launch(std::integral_constant<int, 4>{});
    else if (s.chunks_a_thread == 2) launch(std::integral_constant<int, 2>{});
    else launch(std::integral_constant<int, 1>{});
}

template <class E, RowWork WORK>
void launch_rows_of(const RowArgs& a, hipStream_t stream) {
    const int64_t chunks = chunks_of<E>(a.l);
    const unsigned rows = (unsigned)a.rows, fours = (rows + 3) / 4;
    if (chunks <= 64) return logits_held_kernel<E, 64, 1, 4, WORK><<<fours, 256, 0, stream>>>(a);
    if (chunks <= 128) return logits_held_kernel<E, 64, 2, 4, WORK><<<fours, 256, 0, stream>>>(a);
    if (chunks <= 256) return logits_held_kernel<E, 64, 4, 4, WORK><<<fours, 256, 0, stream>>>(a);
    if (chunks <= 512) return logits_held_kernel<E, 64, 8, 4, WORK><<<fours, 256, 0, stream>>>(a);
    if (chunks <= 1024) return logits_held_kernel<E, 256, 4, 1, WORK><<<rows, 256, 0, stream>>>(a);
    if (chunks <= 2048) return logits_held_kernel<E, 256, 8, 1, WORK><<<rows, 256, 0, stream>>>(a);
    if (chunks <= 4096) return logits_held_kernel<E, 1024, 4, 1, WORK><<<rows, 1024, 0, stream>>>(a);
    if (chunks <= 8192) return logits_held_kernel<E, 1024, 8, 1, WORK><<<rows, 1024, 0, stream>>>(a);
    if constexpr (WORK == RowWork::Policy) {
        // two workgroups of 512 threads a unit, of which one reads while the other writes, against one of 1024 (us, two / one): 4096 x 72000, bf16:
        // 211 / 270, 4096 x 100000: 300 / 346; fp32, 1500 x 36000: 85 / 89.  Rows of fp32 beyond 10240 chunks gain while there are few rounds of them,
        // 512 in each: 777 x 50021 61.9 / 67.6, 1024 x 41001 62.6 / 69.3, x 45056 67.9 / 74.6, x 53248 82.6 / 85.8, 1500 x 41001 94.4 / 99.7, x 50021 116.4 /
        // 117.5, x 53248 122.3 / 121.7, 1536 x 45056 108.0 / 107.7, 2000 x 50021 151.5 / 150.2, 3000 x 50021 221 / 218
        if (chunks <= 10240) return logits_held_kernel<E, 512, 20, 1, WORK><<<rows, 512, 0, stream>>>(a);
        if (chunks <= 13312 && (E::VEC == 8 || rows < 1536)) return logits_held_kernel<E, 512, 26, 1, WORK><<<rows, 512, 0, stream>>>(a);
        if (chunks <= 16384) return logits_held_kernel<E, 1024, 16, 1, WORK><<<rows, 1024, 0, stream>>>(a);
        logits_scan_kernel<E, 1024, 18, WORK><<<rows, 1024, 0, stream>>>(a);
    } else {
        logits_scan_kernel<E, 512, 0, WORK><<<rows, 512, 0, stream>>>(a);
    }
}

template <class E, Normaliser FROM>
void launch_grad_of(RowArgs a, hipStream_t stream) {
    const int64_t chunks = chunks_of<E>(a.l);
    const unsigned rows = (unsigned)a.rows;
    a.sections = 1;
    const unsigned fours = (rows + 3) / 4, more = a.loss.out ? 1 : 0;
    if (chunks <= 128) return logits_grad_kernel<E, 64, 2, 4, FROM><<<fours + more, 256, 0, stream>>>(a);
    if (chunks <= 512) return logits_grad_kernel<E, 64, 8, 4, FROM><<<fours + more, 256, 0, stream>>>(a);
    const bool few = a.rows * chunks < 512 * 2048;   // (fewer than two workgroups a unit with sections of 2048 chunks)
    a.sections = (int)(few ? (chunks + 511) / 512 : (chunks + 2047) / 2048);
    const unsigned grid = rows * (unsigned)a.sections + more;
    if (few) logits_grad_kernel<E, 256, 2, 1, FROM><<<grid, 256, 0, stream>>>(a);
    else logits_grad_kernel<E, 256, 8, 1, FROM><<<grid, 256, 0, stream>>>(a);
}

// Workspace of rows in sections: their results, then the targets' logits.
size_t round16(size_t n) { return (n + 15) / 16 * 16; }
size_t parts_bytes(const Sections& s, int64_t tokens) { return round16(sizeof(MaxSum) * (size_t)tokens * (size_t)s.count); }
size_t section_bytes(const Sections& s, int64_t tokens) { return s.count ? parts_bytes(s, tokens) + round16(sizeof(float) * (size_t)tokens) : 0; }

// Workspace of the policy loss: ticket | sums of the workgroups | sections | log-probabilities, their lower parts.
struct PolicySpace {
    size_t sums, parts, logp, logp_low, total;
};
PolicySpace policy_space(int dtype, int64_t tokens, int64_t vocab) {
    PolicySpace s;
    s.sums = 16;
    s.parts = s.sums + sizeof(double) * 4 * kStatsGroups;
    s.logp = s.parts + section_bytes(sections_of(dtype, tokens, vocab, kPolicySections), tokens);
    s.logp_low = s.logp + round16(sizeof(float) * (size_t)tokens);
    s.total = s.logp_low + round16(sizeof(float) * (size_t)tokens);
    return s;
}
template <class T>
T* at(void* workspace, size_t offset) {
    return reinterpret_cast<T*>(reinterpret_cast<char*>(workspace) + offset);
}

// Launches hold at most this many rows (sections of a row are workgroups of their own).
template <class F>
hipError_t in_launches(RowArgs a, int64_t first, int64_t count, F&& launch) {
    constexpr int64_t kRows = (int64_t)1 << 21;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kRows, ((int64_t)1 << 23) / std::max<int64_t>(1, chunks_of(a.l.dtype, a.l.vocab) / 512)));
    for (a.first = first; count > 0; a.first += a.rows, count -= a.rows) {
        a.rows = std::min(count, most);
        launch(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t logprobs_workspace(int dtype, int64_t tokens, int64_t vocab) {
    return section_bytes(sections_of(dtype, tokens, vocab, kLogprobsSections), tokens);
}
size_t policy_workspace(int dtype, int64_t tokens, int64_t vocab) { return policy_space(dtype, tokens, vocab).total; }

hipError_t launch_logprobs(const Logits& l, int64_t first, int64_t count, float* logp, float* logp_low, float* lse, MaxSum* sums, bool again,
                           void* workspace, hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.logp = logp;
    a.logp_low = logp_low;
    a.lse = lse;
    a.sums = sums;
    a.again = again;
    const Sections s = workspace ? sections_of(l.dtype, count, l.vocab, kLogprobsSections) : Sections{0, 0};
    if (s.count > 1) {
        a.first = first;
        a.rows = count;
        a.parts = at<MaxSum>(workspace, 0);
        a.picked = at<float>(workspace, parts_bytes(s, count));
        a.sections = s.count;
        a.lanes = join_lanes(count);
        const unsigned grid = (unsigned)(count * s.count);
        auto both = [&](auto elem) {
            typedef decltype(elem) E;
            for_section(s, [&](auto C) { logits_part_kernel<E, decltype(C)::value><<<grid, kSectionThreads, 0, stream>>>(a); });
            logits_join_kernel<<<1, kSectionThreads, 0, stream>>>(a);
        };
        if (l.dtype == STAR_F32) both(ElemF32{});
        else both(ElemBf16{});
        return hipGetLastError();
    }
    return in_launches(a, first, count, [&](const RowArgs& r) {
        if (l.dtype == STAR_F32) launch_rows_of<ElemF32, RowWork::Logprobs>(r, stream);
        else launch_rows_of<ElemBf16, RowWork::Logprobs>(r, stream);
    });
}

hipError_t launch_logprobs_grad(const Logits& l, int64_t first, int64_t count, const float* lse, const MaxSum* sums, const float* dlogp,
                                void* dlogits, int64_t ld_out, const PairLoss& loss, hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.lse_in = lse;
    a.sums_in = sums;
    a.dlogp = dlogp;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    return in_launches(a, first, count, [&](RowArgs r) {
        if (r.first + r.rows == first + count) r.loss = loss;   // the last one
        auto of = [&](auto elem) {
            typedef decltype(elem) E;
            if (sums) launch_grad_of<E, Normaliser::Sums>(r, stream);
            else launch_grad_of<E, Normaliser::Lse>(r, stream);
        };
        if (l.dtype == STAR_F32) of(ElemF32{});
        else of(ElemBf16{});
    });
}

hipError_t launch_policy(const Logits& l, const PolicyArgs& p, float* logp, void* dlogits, int64_t ld_out, float* stats, void* workspace,
                         hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.policy = p;
    a.logp = logp;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    const PolicySpace space = policy_space(l.dtype, l.tokens, l.vocab);
    if (!a.logp && l.tokens > 0) a.logp = at<float>(workspace, space.logp);
    const Sections s = sections_of(l.dtype, l.tokens, l.vocab, kPolicySections);
    if (s.count > 1 && l.tokens > 0 && dlogits) {
        a.rows = l.tokens;
        a.parts = at<MaxSum>(workspace, space.parts);
        a.picked = at<float>(workspace, space.parts + parts_bytes(s, l.tokens));
        a.sections = s.count;
        a.lanes = join_lanes(l.tokens);
        a.stats = stats;
        const unsigned grid = (unsigned)(l.tokens * s.count);
        auto both = [&](auto elem) {
            typedef decltype(elem) E;
            for_section(s, [&](auto C) { logits_part_kernel<E, decltype(C)::value><<<grid, kSectionThreads, 0, stream>>>(a); });
            for_section(s, [&](auto C) { policy_section_kernel<E, decltype(C)::value><<<grid + 1, kSectionThreads, 0, stream>>>(a); });
        };
        if (l.dtype == STAR_F32) both(ElemF32{});
        else both(ElemBf16{});
        return hipGetLastError();
    }
    // (a token a thread while workgroups last: 8192 tokens 14.2 us, 16.1 with four a thread in fewer workgroups; up to 4096 it is the same)
    const int64_t groups = std::min<int64_t>(kStatsGroups, (l.tokens + kSumThreads - 1) / kSumThreads);
    a.ticket = groups > 1 ? at<unsigned int>(workspace, 0) : nullptr;
    if (l.tokens > 0) a.logp_low = at<float>(workspace, space.logp_low);
    const hipError_t e = in_launches(a, 0, l.tokens, [&](const RowArgs& r) {
        if (!dlogits) l.dtype == STAR_F32 ? launch_rows_of<ElemF32, RowWork::Logprobs>(r, stream) : launch_rows_of<ElemBf16, RowWork::Logprobs>(r, stream);
        else l.dtype == STAR_F32 ? launch_rows_of<ElemF32, RowWork::Policy>(r, stream) : launch_rows_of<ElemBf16, RowWork::Policy>(r, stream);
    });
    if (e != hipSuccess) return e;
    policy_stats_kernel<<<dim3((unsigned)std::max<int64_t>(1, groups)), kSumThreads, 0, stream>>>(l, p, a.logp, a.logp_low, stats, a.ticket,
                                                                                                 groups > 1 ? at<double>(workspace, space.sums) : nullptr);
    return hipGetLastError();
}

hipError_t launch_pairs(const Logits& l, const PreferenceArgs& a, const PairOffsets& offsets, int pairs, const float* logp,
                        const float* logp_low, float* dlogp, float* margins, double* terms, hipStream_t stream) {
    if (pairs <= 0) return hipSuccess;
    pair_kernel<<<dim3((unsigned)pairs), kBlock, 0, stream>>>(l, a, offsets, logp, logp_low, dlogp, margins, terms);
    return hipGetLastError();
}

hipError_t launch_pair_loss(const PairLoss& loss, hipStream_t stream) {
    pair_loss_kernel<<<dim3(1), kBlock, 0, stream>>>(loss);
    return hipGetLastError();
}

}  // namespace star
