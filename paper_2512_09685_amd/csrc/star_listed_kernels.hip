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
// Bound by memory, a row read once and written once where it is held (8192 x 65536, bf16, 64 words, a quarter of the rows written as zeros and not read: 360
// us, 5.2 TB/s; without the list 346); short rows by the list, which one wave puts together (16384 x 1000, 20 words, all rows counting: 41 us, and 7 % more
// with ids and numbers asked for after the row and equal words looked for by every entry's own chain).
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

// What the first wave knows of its row before the row's sums do: sum of the teacher's shares, relative to exp(likeliest), its largest, or of the
// derivatives; what such a share is to be multiplied with; the entry that stands for the taken token (-1: none is taken); of the teacher's words
// the largest logit, and the sum of exp(z - that one's).
struct Prelude {
    double sum, named, part;
    float most, likeliest;
    int taken;
};

// The named words of a row, which its first wave puts together.  An entry that names no word, or one that an earlier entry names, is dead: its id
// is -1.  Words that the sums leave out are marked, a byte for each of a thread's held chunks.
template <int NT, int H>
struct WordList {
    static constexpr int MARKS = (H + 3) / 4;
    int id[kEntries], next[kEntries], head[NT];
    __align__(16) uint32_t marks[NT * MARKS];
    uint32_t edge_marks[4];                       // (fewer than 128 elements lie outside the chunks)
    float logit[kEntries], value[kEntries];       // value: what is written there
    float q[kMostAlternatives], log_q[kMostAlternatives];   // (in fp32, as the sums behind p are: neither leaves p - q more digits than the other)
    Prelude given;
    float slope;                                  // of the words that are not named
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
template <class E, int NT, class Words>
__device__ __forceinline__ int first_of(const Words& w, const RowSpan& sp, int e) {
    const int id = w.id[e];
    if (id < 0) return -1;
    int least = e;
    for (int f = w.head[owner_of<E, NT>(sp, id).thread]; f >= 0; f = w.next[f])
        if (w.id[f] == id) least = min(least, f);
    return least;
}

// Takes the words that `mask` names out of a chunk.
template <class E>
__device__ __forceinline__ void take_out(u32x4& x, uint32_t mask) {
    static_for<0, 4>([&](auto I) {
        constexpr int i = decltype(I)::value;
        uint32_t out;
        if constexpr (E::VEC == 4) out = (uint32_t)__builtin_amdgcn_sbfe((int)mask, i, 1);
        else out = ((uint32_t)__builtin_amdgcn_sbfe((int)mask, 2 * i, 1) & 0xffffu) | ((uint32_t)__builtin_amdgcn_sbfe((int)mask, 2 * i + 1, 1) & 0xffff0000u);
        x[i] = (x[i] & ~out) | (E::NOTHING & out);
    });
}

// A thread's words in the chunks that are not held: `at` is the next chunk that holds any.
template <class E, int NT, class Words>
struct LeftOut {
    const Words& w;
    const RowSpan& sp;
    int tid, rest, at;
    __device__ __forceinline__ LeftOut(const Words& words, const RowSpan& span, int thread, int not_held) : w(words), sp(span), tid(thread), rest(not_held) {
        find(-1);
    }
    __device__ __forceinline__ uint32_t find(int c) {   // the words of chunk c; `at` becomes the one behind it
        uint32_t mask = 0;
        at = 0x7fffffff;
        for (int e = rest > 0 ? w.head[tid] : -1; e >= 0; e = w.next[e]) {
            if (e == kMostAlternatives || w.id[e] < 0) continue;   // (the taken token is no word of the teacher's)
            const int chunk = owner_of<E, NT>(sp, w.id[e]).chunk;
            if (chunk == c && chunk >= 0) mask |= 1u << (w.id[e] - sp.head - c * E::VEC);
            if (chunk > c && chunk < rest) at = min(at, chunk);
        }
        return mask;
    }
};

// Dense part of the gradient: e (a - b x), with x = (l - m) k and e = 2^x.
struct Dense {
    double a, b;
    struct At {
        float a, b;
        template <bool ENTROPY>
        __device__ __forceinline__ float at(float x) const {
            const float e = __builtin_amdgcn_exp2f(x);
            return ENTROPY ? e * __builtin_fmaf(-b, fmaxf(x, kNoExponent), a) : e * a;
        }
    };
    // The same of an x that is `off` too large.
    __device__ __forceinline__ At with(float off) const {
        const float f = __builtin_amdgcn_exp2f(-off);
        return At{(float)(a + b * off) * f, (float)b * f};
    }
};
// Its chunks; `p` as they were summed.
template <class E, int NT, bool ENTROPY, int C>
__device__ __forceinline__ void store_dense(u32x4 (&x)[C], char* out, const RowSpan& sp, const Dense& d, const Exponent& p, int first) {
    u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
    const Dense::At here = d.with(p.off);
    auto all = [&](auto far) {
        keep_packed(x);
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int at = first + i * NT;
            if (at < sp.chunks) {
                float v[E::VEC];
                static_for<0, E::VEC>([&](auto J) {
                    v[decltype(J)::value] = here.template at<ENTROPY>(p.of<decltype(far)::value>(E::template get<decltype(J)::value>(x[i])));
                });
                __builtin_nontemporal_store(E::pack(v), to + at);
            }
        });
    };
    if (p.far) all(std::true_type{});
    else all(std::false_type{});
}

// One lane's number, and the sum over a wave, in every lane.
__device__ __forceinline__ double lane_of(double x, int lane) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), high = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __longlong_as_double((long long)((unsigned long long)high << 32 | low));
}
__device__ __forceinline__ double sum_wave(double x) { return lane_of(wave_sum_to_lane63(x), 63); }

// e^x in 64 bits: n log 2 taken out, then the series up to the twelfth power, which at most log 2 / 2 leaves 2e-16 of.
__device__ __forceinline__ double exp_of(double x) {
    x = x < -760.0 ? -760.0 : x > 760.0 ? 760.0 : x;
    const double n = rint(x * 1.4426950408889634), y = __builtin_fma(-n, 0.69314718055994531, x);
    double r = 1.0 / 479001600.0;
    constexpr double c[12] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880, 1.0 / 3628800, 1.0 / 39916800};
#pragma unroll
    for (int i = 11; i >= 0; --i) r = __builtin_fma(r, y, c[i]);
    return ldexp(r, (int)n);
}
// log v: of the mantissa in fp32, then one step of Newton's, which squares its error.
__device__ __forceinline__ double log_of(double v) {
    int n;
    const double f = frexp(v, &n), near = (double)logf((float)f) + n * 0.69314718055994531;
    return v > 0.0 && v < INFINITY ? near + (v * exp_of(-near) - 1.0) : near;
}

// What the first wave asks for before the row itself is asked for: it comes in the order it was asked for.  Entries `lane` and 64 + lane.
struct Asked {
    int64_t id[2];
    float number[2];
};
template <Listed WORK>
__device__ __forceinline__ Asked ask_words(const ListedArgs& a, int64_t t) {
    Asked w{{-1, -1}, {0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = (int)threadIdx.x + 64 * i, n = a.words.k;
        if (e < n) {
            w.id[i] = a.words.ids[t * n + e];
            w.number[i] = WORK == Listed::Distill ? a.words.logp[t * n + e] : a.dtop[t * n + e];
        }
    }
    return w;
}

// Puts the list together: entries `lane`, 64 + lane and the taken token.
template <class E, int NT, Listed WORK, class Words>
__device__ __forceinline__ void list_words(const ListedArgs& a, Words& w, const Asked& asked, const RowSpan& sp, const char* row, int64_t t, int64_t y, int rest) {
    const int lane = threadIdx.x, n = a.words.k;
    const bool takes = y >= 0 && y < sp.V;
    float logit[2] = {-INFINITY, -INFINITY}, number[2] = {asked.number[0], asked.number[1]}, y_logit = 0.f;
    int id[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool there = asked.id[i] >= 0 && asked.id[i] < sp.V;
        id[i] = there ? (int)asked.id[i] : -1;
        if (there) logit[i] = E::one(row, id[i]);
        w.id[lane + 64 * i] = id[i];
    }
    if (takes) y_logit = E::one(row, y);
    // (what does not need the logits comes first, while they are on their way)
    const double dy = WORK == Listed::Alternatives && takes && a.dlogp ? (double)a.dlogp[t] : 0.0;
    for (int i = lane; i < NT; i += 64) w.head[i] = -1;
    if (WORK == Listed::Distill) {
        for (int i = lane; i < NT * Words::MARKS / 4; i += 64) reinterpret_cast<u32x4*>(w.marks)[i] = u32x4{0, 0, 0, 0};
        if (lane < 4) w.edge_marks[lane] = 0;
    }
    // the entry that stands for the taken token: the first that names it, or its own
    const unsigned long long named[2] = {__ballot(takes && id[0] == (int)y), __ballot(takes && id[1] == (int)y)};
    const int taken = !takes ? -1 : named[0] ? __ffsll(named[0]) - 1 : named[1] ? 63 + __ffsll(named[1]) : kMostAlternatives;
    if (lane == 0) w.id[kMostAlternatives] = taken == kMostAlternatives ? (int)y : -1;
    wave_order();
    bool again = false;   // a word that an entry of the chain below names too
    auto link = [&](int e, int word) {
        const Owner o = owner_of<E, NT>(sp, word);
        int below = atomicExch(&w.head[o.thread], e);
        w.next[e] = below;
        if (WORK == Listed::Distill && e != kMostAlternatives) {
            const int turn = (o.chunk - rest) / NT;
            if (o.chunk >= rest)
                atomicOr(&w.marks[o.thread * Words::MARKS + turn / 4], 1u << (8 * (turn % 4) + (word - sp.head) % E::VEC));
            else if (o.chunk < 0)
                atomicOr(&w.edge_marks[o.thread / 32], 1u << (o.thread % 32));
        }
    };
    if (id[0] >= 0) link(lane, id[0]);
    if (id[1] >= 0) link(64 + lane, id[1]);
    if (lane == 0 && taken == kMostAlternatives) link(kMostAlternatives, (int)y);
    wave_order();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        for (int e = id[i] >= 0 ? w.next[lane + 64 * i] : -1; e >= 0; e = w.next[e]) again |= w.id[e] == id[i];
    bool live[2] = {id[0] >= 0, id[1] >= 0};
    const bool repeats = __any(again);
    int first[2] = {lane, 64 + lane};
    if (repeats) {
        if (live[0]) first[0] = first_of<E, NT>(w, sp, lane);
        if (live[1]) first[1] = first_of<E, NT>(w, sp, 64 + lane);
        wave_order();
        for (int i = 0; i < 2; ++i)
            if (live[i] && first[i] != lane + 64 * i) {
                live[i] = false;
                w.id[lane + 64 * i] = -1;
            }
    }
    Prelude p{0.0, 0.0, 1.0, -INFINITY, 0.f, taken};
    if constexpr (WORK == Listed::Distill) {
        for (int i = 0; i < 2; ++i)
            if (!live[i]) number[i] = -INFINITY;
        const float likeliest = wave_max(fmaxf(number[0], number[1]));
        p.likeliest = likeliest == -INFINITY ? 0.f : likeliest;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = lane + 64 * i;
            const double q = number[i] == -INFINITY ? 0.0 : exp_of((double)number[i] - p.likeliest);
            w.log_q[e] = number[i];
            w.q[e] = (float)q;
            p.sum += q;
            if (n <= 64) {
                w.log_q[64 + e] = -INFINITY;
                w.q[64 + e] = 0.f;
                break;
            }
        }
        p.sum = sum_wave(p.sum);
        p.part = a.distill.renormalise ? 1.0 / p.sum : exp_of(p.likeliest);
        const double inv_t = (double)a.l.inv_t + a.l.inv_t_low;
        p.most = wave_max(fmaxf(live[0] ? logit[0] : -INFINITY, live[1] ? logit[1] : -INFINITY));
        const double base = p.most == -INFINITY ? 0.0 : (double)p.most;
        for (int i = 0; i < (n <= 64 ? 1 : 2); ++i)
            if (live[i] && logit[i] != -INFINITY) p.named += exp_of(((double)logit[i] - base) * inv_t);   // (+inf, NaN: NaN)
        p.named = sum_wave(p.named);
    } else {
        // derivatives by the words' log-probabilities, equal words' added in the order of the entries, to `q`
        const float inv_t = a.l.inv_t;
        double mine[2] = {id[0] >= 0 ? (double)number[0] : 0.0, id[1] >= 0 ? (double)number[1] : 0.0};
        p.sum = sum_wave(mine[0] + mine[1]) + dy;
        if (repeats) {
            for (int f = 1; f < n; ++f) {
                const int same = f < 64 ? __shfl(id[0] >= 0 ? first[0] : -1, f) : __shfl(id[1] >= 0 ? first[1] : -1, f - 64);
                const double d = (double)(f < 64 ? __shfl(number[0], f) : __shfl(number[1], f - 64));
                if (same != f && same == lane) mine[0] += d;
                if (same != f && same == 64 + lane) mine[1] += d;
            }
        }
        w.q[lane] = (float)((mine[0] + (taken == lane ? dy : 0.0)) * inv_t);
        w.q[64 + lane] = (float)((mine[1] + (taken == 64 + lane ? dy : 0.0)) * inv_t);
    }
    w.logit[lane] = logit[0];
    w.logit[64 + lane] = logit[1];
    if (lane == 0) {
        w.logit[kMostAlternatives] = y_logit;
        w.given = p;
    }
}

// q f(log p - log q), f(d) = e^d - d - 1, with d = log p - log q.
__device__ __forceinline__ double divergence_term(double q, double d, double p) {
    if (q == 0.0) return p;
    const float near = (float)d;   // (as kl_of sees it: what rounds to 0.25 is not of its series either)
    return fabsf(near) < 0.25f ? q * (double)kl_of(near, 0.f) : p - q - q * d;
}

// A row of the distillation loss, from the maximum m and sum s of the words that are not named.
struct Distilled {
    double base, all;         // the largest logit, and the sum over all words of exp(z - that one's)
    double down;              // exp of m's distance from it
    double part, whole, left, c, slope;   // part: of a share, what it is taken as
    bool rest;                // whether there are words that are not named
    __device__ __forceinline__ void form(const ListedArgs& a, const Prelude& given, double weight, float m, float s) {
        const double inv_t = (double)a.l.inv_t + a.l.inv_t_low, most = given.most;
        const bool named_lead = given.most > m;
        rest = !(s == 0.f);
        base = named_lead ? most : m == -INFINITY ? 0.0 : (double)m;
        const double apart = rest && given.named != 0.0 ? exp_of((named_lead ? (double)m - most : most - (double)m) * inv_t) : 0.0;
        down = !rest ? 0.0 : named_lead ? apart : 1.0;
        all = given.named * (named_lead ? 1.0 : rest ? apart : 1.0) + (rest ? s * down : 0.0);
        const double none = all > 0.0 && all < INFINITY ? 0.0 : NAN;   // NaN: a row without probabilities
        left = 0.0, part = given.part;
        const double share = given.sum == 0.0 ? 0.0 : given.sum * part;
        if (!a.distill.renormalise && rest) left = share < 1.0 ? 1.0 - share : share - share;   // (0, or NaN)
        whole = share + left;
        c = (double)a.distill.scale * weight * inv_t + none;
        // of the rest e (c (Q + ce) / sum of all - c q_r / sum of the rest)
        slope = rest ? c * (((whole + a.distill.ce) * down * s - left * all) / (all * s)) : none;
    }
};

// The named words' numbers, c ((Q + ce) p - q - ce [taken]), and the row's loss, by the first wave.
template <class Words>
__device__ __forceinline__ void distill_words(const ListedArgs& a, Words& w, const Distilled& d, int64_t t, float m, float s) {
    const int lane = threadIdx.x, taken = w.given.taken;
    const double inv_t = (double)a.l.inv_t + a.l.inv_t_low, ce = a.distill.ce;
    const double logs = log_of(lane == 0 ? d.all : lane == 1 ? (double)s : lane == 2 ? d.left : d.part);
    const double log_all = lane_of(logs, 0), log_s = lane_of(logs, 1), log_left = lane_of(logs, 2);
    const double shift = a.distill.renormalise ? lane_of(logs, 3) - w.given.likeliest : 0.0;
    double kl = 0.0;
#pragma unroll 1
    for (int e = lane; e < kMostAlternatives; e += 64) {
        if (w.id[e] < 0) continue;
        const double log_p = ((double)w.logit[e] - d.base) * inv_t - log_all, p = w.logit[e] == -INFINITY ? 0.0 : exp_of(log_p);
        const double q = w.q[e] == 0.f ? 0.0 : w.q[e] * d.part;
        kl += divergence_term(q, log_p - (w.log_q[e] + shift), p);
        w.value[e] = (float)(d.c * ((d.whole + ce) * p - q - (taken == e ? ce : 0.0)));
    }
    kl = sum_wave(kl);
    const double base = m == -INFINITY ? 0.0 : (double)m, none = d.all > 0.0 && d.all < INFINITY ? 0.0 : NAN;
    if (d.rest) kl += divergence_term(d.left, log_s + (base - d.base) * inv_t - log_all - log_left, s * d.down / d.all);
    kl = (d.whole == 0.0 ? 0.0 : kl + (d.whole - 1.0)) + none;     // (a teacher that says nothing costs nothing)
    if (lane == 0) {
        const double ly = taken >= 0 ? (double)w.logit[kMostAlternatives] : 0.0;
        w.value[kMostAlternatives] = (float)(d.slope * (d.rest ? exp_of((ly - base) * inv_t) : 0.0) - d.c * ce);
        if (a.kl) a.kl[t] = (float)kl;
        a.terms[2 * t] = kl;
        a.terms[2 * t + 1] = taken >= 0 ? log_all - (ly - d.base) * inv_t : 0.0;
    }
}

// The same of a function of the alternatives.
template <bool ENTROPY, class Words>
__device__ __forceinline__ void alternatives_words(const ListedArgs& a, Words& w, const Dense& dense, int64_t t, const Exponent& p) {
    const int lane = threadIdx.x;
    const Dense::At of = dense.with(0.f);
    for (int e = lane; e < kMostAlternatives; e += 64)
        if (w.id[e] >= 0) w.value[e] = of.at<ENTROPY>((w.logit[e] - p.m) * p.k) + w.q[e];
    if (lane == 0 && w.id[kMostAlternatives] >= 0)
        w.value[kMostAlternatives] = of.at<ENTROPY>((w.logit[kMostAlternatives] - p.m) * p.k) + (a.dlogp ? a.dlogp[t] * a.l.inv_t : 0.f);
}

// A workgroup a row; the last H chunks a thread stay in registers, those before are read a second time, from their end.
template <class E, int NT, int H, Listed WORK, bool ENTROPY>
__global__ __launch_bounds__(NT, H == 16 ? 4 : H == 8 ? 6 : 7) void listed_kernel(const ListedArgs a) {
    typedef WordList<NT, H> Words;
    __shared__ Words w;
    __shared__ float shared[3][NT / 64];
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    if (a.ticket && blockIdx.x == 0 && tid == 0) *a.ticket = 0u;
    const int64_t t = a.first + (NT >= 512 ? die_run(blockIdx.x) : (int64_t)blockIdx.x), y = a.l.targets ? a.l.targets[t] : -1;
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    char* out = a.dlogits ? a.dlogits + t * a.ld_out * E::BYTES : nullptr;
    const float k = a.l.k;
    const float weight = a.l.weights ? a.l.weights[t] : 1.f;
    Asked asked{};
    if (tid < 64) asked = ask_words<WORK>(a, t);
    if ((a.l.targets && (y < 0 || y >= V)) || weight == 0.f) {
        if (WORK == Listed::Distill && tid == 0) {
            if (a.kl) a.kl[t] = 0.f;
            a.terms[2 * t] = a.terms[2 * t + 1] = 0.0;
        }
        if (out) zero_row<E, NT>(out, V, tid);
        return;
    }
    const RowSpan sp = row_span<E, NT>(row, V);
    // (16 chunks a thread: the rows that are longer, too)
    const int rest = H == 16 ? (max(sp.chunks - H * NT, 0) + NT - 1) / NT * NT : 0;   // (whole turns of the threads: chunk c is thread c % NT's)
    u32x4 x[H];
    load_chunks<E, NT>(x, row, sp, rest + tid);
    const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    if (tid < 64) list_words<E, NT, WORK>(a, w, asked, sp, row, t, y, rest);
    __syncthreads();

    Seen seen{-INFINITY, 0.f, 0.f};
    float edge_left = edge;
    RowSpan before = sp;
    before.chunks = rest;
    if constexpr (WORK == Listed::Distill) {
        LeftOut<E, NT, Words> left(w, sp, tid, rest);
        if (tid < sp.edge && (w.edge_marks[tid / 32] >> (tid % 32) & 1)) edge_left = -INFINITY;
        for (int c = tid; c < rest; c += 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT, Reading::Again>(z, row, before, c);
            static_for<0, 4>([&](auto I) {
                constexpr int i = decltype(I)::value;
                if (c + i * NT == left.at) take_out<E>(z[i], left.find(c + i * NT));
            });
            see_chunks<E, ENTROPY>(seen, z, k);
        }
        static_for<0, Words::MARKS>([&](auto G) {
            constexpr int g = decltype(G)::value;
            const uint32_t marks = w.marks[tid * Words::MARKS + g];
            if (__any(marks != 0))
                static_for<0, (H - 4 * g < 4 ? H - 4 * g : 4)>([&](auto I) {
                    constexpr int i = decltype(I)::value;
                    const uint32_t mask = marks >> (8 * i) & 255;
                    if (__any(mask != 0)) take_out<E>(x[4 * g + i], mask);
                });
        });
    } else {
        for (int c = tid; c < rest; c += 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT, Reading::Again>(z, row, before, c);
            see_chunks<E, ENTROPY>(seen, z, k);
        }
    }
    const float most = max_of_many<E>(x, fmaxf(seen.m, edge_left));
    keep_packed(x);
    float m = max_group<NT / 64>(most, shared[0]);
    asm volatile("" : "+v"(m));   // (known to be one number for all threads, it would have the whole rest compiled once for rows that are far and once not)
    see_max<ENTROPY>(seen, m, k);
    const Exponent p = exponent_of(m, k);
    see_held<E, ENTROPY>(seen, x, edge_left, p);
    keep_packed(x);
    const float s = sum_group<NT / 64>(seen.s, shared[1]), sx = ENTROPY ? sum_group<NT / 64>(seen.w, shared[2]) : 0.f;

    auto finish = [&](const Dense& dense) {
        keep_packed(x);
        int mine = tid;
        asm volatile("" : "+v"(mine));   // (the addresses are formed again: kept since the loads, they would not fit the registers)
        store_dense<E, NT, ENTROPY>(x, out, sp, dense, p, rest + mine);
        for (int first = (rest - 1) / (4 * NT) * (4 * NT); rest > 0 && first >= 0; first -= 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT>(z, row, before, first + tid);
            store_dense<E, NT, ENTROPY>(z, out, before, dense, p, first + tid);
        }
        if (tid < sp.edge) E::put(out, sp.edge_element(tid), dense.with(0.f).template at<ENTROPY>((edge - p.m) * k));
    };
    // (the list's numbers come behind the row's: the other waves write while the first one forms them)
    if constexpr (WORK == Listed::Distill) {
        Distilled d;
        if (tid < 64) {
            d.form(a, w.given, weight, m, s);
            if (tid == 0) w.slope = (float)d.slope;
        }
        __syncthreads();
        if (out) finish(Dense{w.slope, 0.0});
        if (tid < 64) distill_words(a, w, d, t, m, s);
    } else {
        const double inv_t = (double)a.l.inv_t + a.l.inv_t_low, slope = ENTROPY ? (double)a.dentropy[t] * 0.693147180559945309 * inv_t / s : 0.0;
        const Dense dense{-w.given.sum * inv_t / s + (ENTROPY ? slope * (sx / s) : 0.0), slope};
        finish(dense);
        if (tid < 64) alternatives_words<ENTROPY>(a, w, dense, t, p);
    }
    if (!out) return;
    __syncthreads();
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

// Threads a row, by its chunks (us, this way / the other; bf16, distillation): one and two waves up to 128 and 512 chunks against four: 16384 x 1000, 20
// words: 41 / 89, 16384 x 4000: 74 / 100; 4 chunks a thread up to 1024 against 8: 8192 x 8000, 64 words: 72 / 78; 8 up to 4096 against 16: 2048 x
// 32000: 66 / 74; beyond, two rows a unit of 512 threads against one of 1024: 2000 x 131075: 212 / 230, 777 x 50021, fp32: 66 / 74.  More than 16 chunks a
// thread held of long rows: 2048 x 40000, fp32, 16 / 18 / 20: 126 / 128 / 130, 2000 x 131075: 213 / 216 / 212.
template <class E, Listed WORK, bool ENTROPY>
void launch_listed_of(const ListedArgs& a, hipStream_t stream) {
    const int64_t chunks = (a.l.vocab + E::VEC - 1) / E::VEC;
    const unsigned rows = (unsigned)a.rows;
    if (chunks <= 128) return listed_kernel<E, 64, 2, WORK, ENTROPY><<<rows, 64, 0, stream>>>(a);
    if (chunks <= 512) return listed_kernel<E, 128, 4, WORK, ENTROPY><<<rows, 128, 0, stream>>>(a);
    if (chunks <= 1024) return listed_kernel<E, 256, 4, WORK, ENTROPY><<<rows, 256, 0, stream>>>(a);
    if (chunks <= 2048) return listed_kernel<E, 256, 8, WORK, ENTROPY><<<rows, 256, 0, stream>>>(a);
    if (chunks <= 4096) return listed_kernel<E, 512, 8, WORK, ENTROPY><<<rows, 512, 0, stream>>>(a);
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
