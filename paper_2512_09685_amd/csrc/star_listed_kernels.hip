// Gradients of losses that name some words of a row: the distillation loss on a teacher's alternatives, and any function of the log-probabilities
// of a row's alternatives, its taken token and its entropy.
//
// Both are dense functions of the row, dl_j = e_j (a - b x_j) with x_j = (l_j - m) k and e_j = 2^x_j, but at the named words, at most 129 of them.
// These have numbers of their own, which a wave forms in 64 bits beside the row: a list in LDS, and for every thread the chain of its entries
// among the words that the thread itself reads and writes.  So a thread leaves the words that the loss keeps apart out of its sums, and writes
// the named words behind its own chunks: no two threads write one word, and nobody waits.
//
// Distillation.  With q_i the teacher's share of word i, p_i the student's, q_r and p_r what either gives to all words not named, Q = sum q_i + q_r:
//     KL = sum q_i log(q_i / p_i) + q_r log(q_r / p_r),    dKL/dz_j = Q p_j - q_j  (named),   Q p_j - q_r p_j / p_r  (not named).
// p_r comes from a sum over the words that are not named, relative to their own maximum: 1 - sum p_i would lose it for a student that is sure of
// its words.  As sum p_i + p_r = 1, KL = sum q f(log p - log q) + Q - 1 with f(d) = e^d - d - 1, whose terms are never negative: where student and
// teacher agree, errors enter squared.
//
// Alternatives.  With D the sum of all derivatives by log-probabilities, H' that by the entropy and E = sum e_j x_j / s:
//     dz_j = sum_i d_i [j = i] - D p_j - H' p_j log 2 (x_j - E).
#include <hip/hip_runtime.h>

#include "star_logits.h"

namespace star {

namespace {

enum class Listed { Distill, Alternatives };

struct ListedArgs {
    Logits l;                              // its targets may be null: all rows count, and no token is taken
    ListedWords words;
    DistillArgs distill;
    const float *dlogp, *dentropy, *dtop;  // of the alternatives; each may be null
    char* dlogits;                         // null: the loss alone
    int64_t ld_out, first, rows;
    float* kl;                             // may be null
    double* terms;                         // [tokens][2]: KL, -log p of the taken token
    unsigned int* ticket;                  // cleared for the launch behind this one; null: it needs none
};

constexpr int kEntries = kMostAlternatives + 1;   // the taken token is the last

// The named words of a row, which its first wave puts together.  An entry that names no word, or one that an earlier entry names, is dead: its id
// is -1.
template <int NT>
struct WordList {
    int id[kEntries], next[kEntries], head[NT];
    float logit[kEntries], value[kEntries];       // value: what is written there
    float q[kMostAlternatives], log_q[kMostAlternatives];
};

// The wave's own LDS accesses before and behind this keep their order, also for the compiler; the hardware takes them in order.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Who reads and writes a word: a thread, and the thread's chunk that holds it (-1: its element outside the chunks).
struct Owner {
    int thread, chunk;
};
template <class E, int NT>
__device__ __forceinline__ Owner owner_of(const RowSpan& sp, int id) {
    const int in = id - sp.head;
    if (in < 0) return Owner{id, -1};
    const int c = in / E::VEC;
    return c < sp.chunks ? Owner{c % NT, c} : Owner{id - (sp.V - sp.edge), -1};
}

// The first entry that names the word of entry e.
template <class E, int NT>
__device__ __forceinline__ int first_of(const WordList<NT>& w, const RowSpan& sp, int e) {
    const int id = w.id[e];
    if (id < 0) return -1;
    int least = e;
    for (int f = w.head[owner_of<E, NT>(sp, id).thread]; f >= 0; f = w.next[f])
        if (w.id[f] == id) least = min(least, f);
    return least;
}

// A thread's words that its sums leave out, from its first chunk on: `at` is the next chunk that holds any.
template <class E, int NT>
struct LeftOut {
    const WordList<NT>& w;
    const RowSpan& sp;
    int tid, at;
    bool edge;
    __device__ __forceinline__ LeftOut(const WordList<NT>& words, const RowSpan& span, int thread) : w(words), sp(span), tid(thread), at(0x7fffffff), edge(false) {
        for (int e = w.head[tid]; e >= 0; e = w.next[e]) {
            if (e == kMostAlternatives || w.id[e] < 0) continue;       // (the taken token is no word of the teacher's)
            const int c = owner_of<E, NT>(sp, w.id[e]).chunk;
            edge |= c < 0;
            if (c >= 0) at = min(at, c);
        }
    }
    // Takes the words of chunk c, which is `at`, out of x.
    __device__ __forceinline__ void take(u32x4& x, int c) {
        uint32_t mask = 0;
        at = 0x7fffffff;
        for (int e = w.head[tid]; e >= 0; e = w.next[e]) {
            if (e == kMostAlternatives || w.id[e] < 0) continue;
            const int chunk = owner_of<E, NT>(sp, w.id[e]).chunk;
            if (chunk == c) mask |= 1u << (w.id[e] - sp.head - c * E::VEC);
            if (chunk > c) at = min(at, chunk);
        }
        static_for<0, 4>([&](auto I) {
            constexpr int i = decltype(I)::value;
            if constexpr (E::VEC == 4) {
                if (mask >> i & 1) x[i] = E::NOTHING;
            } else {
                if (mask >> (2 * i) & 1) x[i] = (x[i] & 0xffff0000u) | (E::NOTHING & 0xffffu);
                if (mask >> (2 * i + 1) & 1) x[i] = (x[i] & 0xffffu) | (E::NOTHING & 0xffff0000u);
            }
        });
    }
};

// Dense part of the gradient: e (a - b (x - mean)), with x = (l - m) k and e = 2^x.
struct Dense {
    float m, k, a, b, mean;
    template <bool ENTROPY>
    __device__ __forceinline__ float of(float l) const {
        const float x = (l - m) * k, e = __builtin_amdgcn_exp2f(x);
        if (!ENTROPY) return e * a;
        return e * (a - b * (fmaxf(x, kNoExponent) - mean));
    }
};
template <class E, int NT, bool ENTROPY, int C>
__device__ __forceinline__ void store_dense(const u32x4 (&x)[C], char* out, const RowSpan& sp, const Dense& d, int first) {
    u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        const int at = first + i * NT;
        if (at < sp.chunks) {
            float v[E::VEC];
            static_for<0, E::VEC>([&](auto J) { v[decltype(J)::value] = d.of<ENTROPY>(E::template get<decltype(J)::value>(x[i])); });
            __builtin_nontemporal_store(E::pack(v), to + at);
        }
    });
}

__device__ __forceinline__ double sum_wave(double x) {
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// What the first wave hands to the others.
struct RowNumbers {
    float a, b, mean;
};

// What the first wave knows of its row before the row's sums do: sum of the teacher's shares, of the derivatives, and the entry that stands for the
// taken token (-1: none is taken).
struct Prelude {
    double sum;
    int taken;
};

// Puts the list together: entries `lane`, 64 + lane and the taken token.
template <class E, int NT, Listed WORK>
__device__ __forceinline__ Prelude list_words(const ListedArgs& a, WordList<NT>& w, const RowSpan& sp, const char* row, int64_t t, int64_t y) {
    const int lane = threadIdx.x, n = a.words.k;
    for (int i = lane; i < NT; i += 64) w.head[i] = -1;
#pragma unroll
    for (int e = lane; e < kEntries; e += 64) {
        const int64_t id = e < n ? a.words.ids[t * n + e] : (e == kMostAlternatives ? y : -1);
        const bool there = id >= 0 && id < sp.V;
        w.id[e] = there ? (int)id : -1;
        if (there) w.logit[e] = E::one(row, id);
    }
    wave_order();
    for (int e = lane; e < kEntries; e += 64)
        if (w.id[e] >= 0) w.next[e] = atomicExch(&w.head[owner_of<E, NT>(sp, w.id[e]).thread], e);
    wave_order();
    const int first = first_of<E, NT>(w, sp, lane), second = first_of<E, NT>(w, sp, 64 + lane), taken = first_of<E, NT>(w, sp, kMostAlternatives);
    wave_order();
    const bool again[2] = {first >= 0 && first != lane, second >= 0 && second != 64 + lane};
    if (again[0]) w.id[lane] = -1;
    if (again[1]) w.id[64 + lane] = -1;
    if (taken != kMostAlternatives && lane == 0) w.id[kMostAlternatives] = -1;
    Prelude p{0.0, taken};
    if constexpr (WORK == Listed::Distill) {
#pragma unroll 1
        for (int e = lane; e < kMostAlternatives; e += 64) {
            const bool live = e < 64 ? first == e : second == e;
            const float log_q = live ? a.words.logp[t * n + e] : -INFINITY;
            const double q = exp((double)log_q);
            w.log_q[e] = log_q;
            w.q[e] = (float)q;
            p.sum += q;
        }
        p.sum = sum_wave(p.sum);
    } else {
        // derivatives by the words' log-probabilities, equal words' added in the order of the entries, to `q`
        const float inv_t = a.l.inv_t;
        double mine[2] = {0.0, 0.0};
        if (first >= 0) mine[0] = (double)a.dtop[t * n + lane];
        if (second >= 0) mine[1] = (double)a.dtop[t * n + 64 + lane];
        p.sum = sum_wave(mine[0] + mine[1]);
        if (__any(again[0] || again[1])) {
            for (int f = 1; f < n; ++f) {
                const int same = f < 64 ? __shfl(first, f) : __shfl(second, f - 64);
                const double d = f < 64 ? __shfl(mine[0], f) : __shfl(mine[1], f - 64);
                if (same != f && same == lane) mine[0] += d;
                if (same != f && same == 64 + lane) mine[1] += d;
            }
        }
        const double dy = taken >= 0 && a.dlogp ? (double)a.dlogp[t] : 0.0;
        p.sum += dy;
        w.q[lane] = (float)((mine[0] + (taken == lane ? dy : 0.0)) * inv_t);
        w.q[64 + lane] = (float)((mine[1] + (taken == 64 + lane ? dy : 0.0)) * inv_t);
    }
    return p;
}

// e^x to the accuracy of fp32, of any x.
__device__ __forceinline__ double near_exp(double x) {
    const double z = fmax(x * 1.4426950408889634, -2000.0), n = rint(z);   // (NaN is dropped: whoever sums these sums the row's own as well)
    return ldexp((double)__builtin_amdgcn_exp2f((float)(z - n)), (int)n);
}

// q f(log p - log q), f(d) = e^d - d - 1, with d = log p - log q.
__device__ __forceinline__ double divergence_term(double q, double d, double p) {
    if (q == 0.0) return p;
    return fabs(d) < 0.25 ? q * (double)kl_of((float)d, 0.f) : p - q - q * d;
}

// Numbers of the distillation loss, from the maximum m and sum s of the words that are not named.
template <int NT>
__device__ __forceinline__ RowNumbers distill_words(const ListedArgs& a, WordList<NT>& w, const Prelude& given, int64_t t, float m, float s) {
    const int lane = threadIdx.x, taken = given.taken;
    const double weight = a.l.weights ? (double)a.l.weights[t] : 1.0, inv_t = (double)a.l.inv_t + a.l.inv_t_low, base = m == -INFINITY ? 0.f : m;
    float most = m;
    for (int e = lane; e < kMostAlternatives; e += 64)
        if (w.id[e] >= 0) most = fmaxf(most, w.logit[e]);
    most = fold_wave<64>(most, [](float p, float q) { return fmaxf(p, q); });
    const double whole_base = most == -INFINITY ? 0.f : most;
    // the sum over all words, relative to the largest: of the named ones, and of the rest (which without any word is 0)
    double named = 0.0;
    float sure = 0.f;   // NaN if a named word's logit is
    for (int e = lane; e < kMostAlternatives; e += 64)
        if (w.id[e] >= 0) {
            named += near_exp(((double)w.logit[e] - whole_base) * inv_t);
            sure += w.logit[e] - w.logit[e] == 0.f || w.logit[e] == -INFINITY ? 0.f : NAN;
        }
    named = sum_wave(named + (double)sure);
    const bool rest = !(s == 0.f);
    const double down = rest ? near_exp((base - whole_base) * inv_t) : 0.0, all = named + (rest ? s * down : 0.0);
    const double none = all > 0.0 && all < INFINITY ? 0.0 : NAN;   // NaN: a row without probabilities
    double share = given.sum, left = 0.0, divide = 1.0;
    if (a.distill.renormalise) {
        divide = share;
        share = share == 0.0 ? 0.0 : share / share;
    } else if (rest) {
        left = share < 1.0 ? 1.0 - share : share - share;   // (0, or NaN)
    }
    const double logs = log(lane == 0 ? all : lane == 1 ? (double)s : lane == 2 ? left : divide);
    const double log_all = __shfl(logs, 0), log_s = __shfl(logs, 1), log_left = __shfl(logs, 2), shift = a.distill.renormalise ? __shfl(logs, 3) : 0.0;
    // the row's loss, and at the named words c ((Q + ce) p - q - ce [taken])
    const double whole = share + left, ce = a.distill.ce, c = (double)a.distill.scale * weight * inv_t + none;
    double kl = 0.0;
#pragma unroll 1
    for (int e = lane; e < kMostAlternatives; e += 64) {
        if (w.id[e] < 0) continue;
        const double log_p = ((double)w.logit[e] - whole_base) * inv_t - log_all, p = exp(log_p);
        const double q = w.q[e] == 0.f ? 0.0 : w.q[e] / divide;
        kl += divergence_term(q, log_p - (w.log_q[e] - shift), p);
        w.value[e] = (float)(c * ((whole + ce) * p - q - (taken == e ? ce : 0.0)));
    }
    kl = sum_wave(kl);
    if (rest) kl += divergence_term(left, log_s + (base - whole_base) * inv_t - log_all - log_left, s * down / all);
    kl = (whole == 0.0 ? 0.0 : kl + (whole - 1.0)) + none;     // (a teacher that says nothing costs nothing)
    // of the rest e (c (Q + ce) / sum of all - c q_r / sum of the rest)
    const double slope = rest ? c * ((whole + ce) * down / all - left / s) : none;
    const double ly = taken >= 0 ? (double)w.logit[kMostAlternatives] : 0.0, nll = taken >= 0 ? log_all - (ly - whole_base) * inv_t : 0.0;
    if (lane == 0) {
        w.value[kMostAlternatives] = (float)(slope * (rest ? exp((ly - base) * inv_t) : 0.0) - c * ce);
        if (a.kl) a.kl[t] = (float)kl;
        a.terms[2 * t] = kl;
        a.terms[2 * t + 1] = nll;
    }
    return RowNumbers{(float)slope, 0.f, 0.f};
}

// Numbers of a function of the alternatives, from the maximum m, sum s and sum of e_j x_j of all words.
template <int NT, bool ENTROPY>
__device__ __forceinline__ RowNumbers alternatives_words(const ListedArgs& a, WordList<NT>& w, const Prelude& given, int64_t t, float m, float s, float sx) {
    const int lane = threadIdx.x;
    const double inv_t = (double)a.l.inv_t + a.l.inv_t_low;
    const double slope = ENTROPY ? (double)a.dentropy[t] * 0.693147180559945309 * inv_t / s : 0.0;
    const Dense dense{m == -INFINITY ? 0.f : m, a.l.k, (float)(-given.sum * inv_t / s), (float)slope, ENTROPY ? sx / s : 0.f};
    for (int e = lane; e < kMostAlternatives; e += 64)
        if (w.id[e] >= 0) w.value[e] = dense.of<ENTROPY>(w.logit[e]) + w.q[e];
    if (lane == 0 && w.id[kMostAlternatives] >= 0)
        w.value[kMostAlternatives] = dense.of<ENTROPY>(w.logit[kMostAlternatives]) + (a.dlogp ? a.dlogp[t] * a.l.inv_t : 0.f);
    return RowNumbers{dense.a, dense.b, dense.mean};
}

// A workgroup a row; the last H chunks a thread stay in registers, those before are read a second time, from their end.
template <class E, int NT, int H, Listed WORK, bool ENTROPY>
__global__ __launch_bounds__(NT, NT >= 512 ? 4 : 5) void listed_kernel(const ListedArgs a) {
    __shared__ WordList<NT> w;
    __shared__ float shared[3][NT / 64];
    __shared__ RowNumbers numbers;
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    if (a.ticket && blockIdx.x == 0 && tid == 0) *a.ticket = 0u;
    const int64_t t = a.first + (NT >= 512 ? die_run(blockIdx.x) : (int64_t)blockIdx.x), y = a.l.targets ? a.l.targets[t] : -1;
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    char* out = a.dlogits ? a.dlogits + t * a.ld_out * E::BYTES : nullptr;
    const float k = a.l.k;
    if ((a.l.targets && (y < 0 || y >= V)) || (a.l.weights && a.l.weights[t] == 0.f)) {
        if (WORK == Listed::Distill && tid == 0) {
            if (a.kl) a.kl[t] = 0.f;
            a.terms[2 * t] = a.terms[2 * t + 1] = 0.0;
        }
        if (out) zero_row<E, NT>(out, V, tid);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    const int rest = (max(sp.chunks - H * NT, 0) + NT - 1) / NT * NT;   // (whole turns of the threads: chunk c is thread c % NT's)
    u32x4 x[H];
    load_chunks<E, NT>(x, row, sp, rest + tid);
    const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    Prelude given{0.0, -1};
    if (tid < 64) given = list_words<E, NT, WORK>(a, w, sp, row, t, y);
    __syncthreads();

    Seen seen{-INFINITY, 0.f, 0.f};
    float edge_left = edge;
    RowSpan before = sp;
    before.chunks = rest;
    {
        LeftOut<E, NT> left(w, sp, tid);
        if (WORK == Listed::Alternatives) left.at = 0x7fffffff;
        else if (left.edge) edge_left = -INFINITY;
        for (int c = tid; c < rest; c += 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT, Reading::Again>(z, row, before, c);
            static_for<0, 4>([&](auto I) {
                constexpr int i = decltype(I)::value;
                if (WORK == Listed::Distill && c + i * NT == left.at && c + i * NT < rest) left.take(z[i], c + i * NT);
            });
            see_chunks<E, ENTROPY>(seen, z, k);
        }
        static_for<0, H>([&](auto I) {
            constexpr int i = decltype(I)::value;
            if (WORK == Listed::Distill && rest + tid + i * NT == left.at) left.take(x[i], rest + tid + i * NT);
        });
    }
    const float most = max_of<E>(x, fmaxf(seen.m, edge_left));
    keep_packed(x);
    const float m = fold_row<NT>(most, shared[0], [](float p, float q) { return fmaxf(p, q); });
    see_max<ENTROPY>(seen, m, k);
    see<ENTROPY>(seen, edge_left, k);
    static_for<0, H>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { see<ENTROPY>(seen, E::template get<decltype(J)::value>(x[decltype(I)::value]), k); });
        // (a chunk after the other: the compiler would put a sum off to where it is used, and keep all of its terms till then)
        asm volatile("" : "+v"(seen.s), "+v"(seen.w));
    });
    keep_packed(x);
    auto plus = [](float p, float q) { return p + q; };
    const float s = fold_row<NT>(seen.s, shared[1], plus);
    const float sx = ENTROPY ? fold_row<NT>(seen.w, shared[2], plus) : 0.f;

    if (tid < 64) {
        RowNumbers r;
        if constexpr (WORK == Listed::Distill) r = distill_words<NT>(a, w, given, t, m, s);
        else r = alternatives_words<NT, ENTROPY>(a, w, given, t, m, s, sx);
        if (tid == 0) numbers = r;
    }
    __syncthreads();
    if (!out) return;
    keep_packed(x);
    int mine = tid;
    asm volatile("" : "+v"(mine));   // (the addresses are formed again: kept since the loads, they would not fit the registers)
    const Dense dense{m == -INFINITY ? 0.f : m, k, numbers.a, numbers.b, numbers.mean};
    store_dense<E, NT, ENTROPY>(x, out, sp, dense, rest + mine);
    for (int first = (rest - 1) / (4 * NT) * (4 * NT); rest > 0 && first >= 0; first -= 4 * NT) {
        u32x4 z[4];
        load_chunks<E, NT>(z, row, before, first + tid);
        store_dense<E, NT, ENTROPY>(z, out, before, dense, first + tid);
    }
    if (tid < sp.edge) E::put(out, sp.edge_element(tid), dense.of<ENTROPY>(edge));
    // (a wave's own stores to one word keep their order)
    for (int e = w.head[tid]; e >= 0; e = w.next[e])
        if (w.id[e] >= 0) E::put(out, w.id[e], w.value[e]);
}

constexpr int kSumThreads = 1024, kSumGroups = 64;

// loss, KL, -log p of the taken tokens, weight: sums over the tokens in 64 bits, in a fixed order.
__global__ __launch_bounds__(kSumThreads) void distill_stats_kernel(const Logits l, const DistillArgs a, const double* terms, float* stats,
                                                                    unsigned int* ticket, double* sums) {
    __shared__ double shared[kSumThreads / 64][3];
    __shared__ bool last;
    double sum[3] = {0, 0, 0};
    for (int64_t t = (int64_t)blockIdx.x * kSumThreads + threadIdx.x; t < l.tokens; t += (int64_t)gridDim.x * kSumThreads) {
        const int64_t y = l.targets ? l.targets[t] : 0;
        const double w = l.weights ? (double)l.weights[t] : 1.0;
        if (y < 0 || y >= l.vocab || w == 0.0) continue;
        sum[0] += w * terms[2 * t];
        sum[1] += w * terms[2 * t + 1];
        sum[2] += w;
    }
    group_sums<kSumThreads>(sum, shared);
    if (gridDim.x > 1) {
        // the workgroup that comes last joins all of them, in their own order
        if (threadIdx.x == 0) {
            for (int i = 0; i < 3; ++i) __hip_atomic_store(sums + 3 * blockIdx.x + i, sum[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
        }
        __syncthreads();
        if (!last) return;
        for (int i = 0; i < 3; ++i)
            sum[i] = threadIdx.x < gridDim.x ? __hip_atomic_load(sums + 3 * threadIdx.x + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        group_sums<kSumThreads>(sum, shared);
    }
    if (threadIdx.x == 0) {
        const double scale = a.scale, ce = a.ce;
        stats[0] = (float)(scale * (ce == 0.0 ? sum[0] : sum[0] + ce * sum[1]));
        stats[1] = (float)(scale * sum[0]);
        stats[2] = (float)(scale * sum[1]);
        stats[3] = (float)(scale * sum[2]);
    }
}

template <class E, Listed WORK, bool ENTROPY>
void launch_listed_of(const ListedArgs& a, hipStream_t stream) {
    const int64_t chunks = (a.l.vocab + E::VEC - 1) / E::VEC;
    const unsigned rows = (unsigned)a.rows;
    if (chunks <= 512) return listed_kernel<E, 256, 2, WORK, ENTROPY><<<rows, 256, 0, stream>>>(a);
    if (chunks <= 2048) return listed_kernel<E, 256, 8, WORK, ENTROPY><<<rows, 256, 0, stream>>>(a);
    listed_kernel<E, 512, 16, WORK, ENTROPY><<<rows, 512, 0, stream>>>(a);
}

template <Listed WORK>
hipError_t launch_listed(ListedArgs a, bool entropy, hipStream_t stream) {
    constexpr int64_t kRows = (int64_t)1 << 21;
    for (a.first = 0; a.first < a.l.tokens; a.first += kRows) {
        a.rows = std::min(kRows, a.l.tokens - a.first);
        auto of = [&](auto elem) {
            typedef decltype(elem) E;
            if constexpr (WORK == Listed::Alternatives)
                if (entropy) return launch_listed_of<E, WORK, true>(a, stream);
            launch_listed_of<E, WORK, false>(a, stream);
        };
        if (a.l.dtype == STAR_F32) of(ElemF32{});
        else of(ElemBf16{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Workspace of the distillation loss: ticket | sums of the workgroups | terms.
constexpr size_t kTermsAt = 16 + sizeof(double) * 4 * kSumGroups;

}  // namespace

size_t distill_workspace(int64_t tokens) { return kTermsAt + 2 * sizeof(double) * (size_t)tokens; }

hipError_t launch_distill(const Logits& l, const ListedWords& words, const DistillArgs& d, void* dlogits, int64_t ld_out, float* kl, float* stats,
                          void* workspace, hipStream_t stream) {
    ListedArgs a{};
    a.l = l;
    a.words = words;
    a.distill = d;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    a.kl = kl;
    a.terms = reinterpret_cast<double*>(reinterpret_cast<char*>(workspace) + kTermsAt);
    const int64_t groups = std::min<int64_t>(kSumGroups, std::max<int64_t>(1, (l.tokens + kSumThreads - 1) / kSumThreads));
    a.ticket = groups > 1 ? reinterpret_cast<unsigned int*>(workspace) : nullptr;
    const hipError_t e = launch_listed<Listed::Distill>(a, false, stream);
    if (e != hipSuccess) return e;
    distill_stats_kernel<<<dim3((unsigned)groups), kSumThreads, 0, stream>>>(l, d, a.terms, stats, a.ticket,
                                                                            reinterpret_cast<double*>(reinterpret_cast<char*>(workspace) + 16));
    return hipGetLastError();
}

hipError_t launch_top_grad(const Logits& l, const ListedWords& words, const float* dlogp, const float* dentropy, const float* dtop, void* dlogits,
                           int64_t ld_out, hipStream_t stream) {
    ListedArgs a{};
    a.l = l;
    a.words = words;
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.dtop = dtop;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    return launch_listed<Listed::Alternatives>(a, dentropy != nullptr, stream);
}

}  // namespace star
