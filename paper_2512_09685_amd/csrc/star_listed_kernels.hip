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

// The named words of a row.  An entry that names no word, or one that an earlier entry has named, is dead: its id is -1.
template <int NT>
struct WordList {
    int n;
    int id[kEntries], next[kEntries], head[NT];
    float value[kEntries];                        // what is written there
};

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

// Chains of the first `n` entries by their owners.  Ends with a barrier.
template <class E, int NT>
__device__ __forceinline__ void chain_words(WordList<NT>& w, const RowSpan& sp, int n, int tid) {
    for (int i = tid; i < NT; i += NT) w.head[i] = -1;
    __syncthreads();
    if (tid < n && w.id[tid] >= 0) w.next[tid] = atomicExch(&w.head[owner_of<E, NT>(sp, w.id[tid]).thread], tid);
    __syncthreads();
}
// The first entry that names the word of entry i.
template <class E, int NT>
__device__ __forceinline__ int first_of(const WordList<NT>& w, const RowSpan& sp, int i) {
    int least = i;
    for (int e = w.head[owner_of<E, NT>(sp, w.id[i]).thread]; e >= 0; e = w.next[e])
        if (w.id[e] == w.id[i]) least = min(least, e);
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
            if (e == kMostAlternatives) continue;       // (the taken token is no word of the teacher's)
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
            if (e == kMostAlternatives) continue;
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

// What the wave that holds the list hands to the others.
struct RowNumbers {
    float a, b, mean;
};

// A workgroup a row; the last H chunks a thread stay in registers, those before are read a second time, from their end.
template <class E, int NT, int H, Listed WORK, bool ENTROPY>
__global__ __launch_bounds__(NT, H <= 8 ? 8 : 4) void listed_kernel(const ListedArgs a) {
    __shared__ WordList<NT> w;
    __shared__ float shared[3][NT / 64];
    __shared__ RowNumbers numbers;
    const int V = (int)a.l.vocab, tid = threadIdx.x, n = a.words.k;
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
    u32x4 x[H > 0 ? H : 1];
    if constexpr (H > 0) load_chunks<E, NT>(x, row, sp, rest + tid);
    float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;

    // the list: the words of entries 0 .. n - 1, then the taken token
    float logit = 0.f;
    if (tid < kEntries) {
        const int64_t id = tid < n ? a.words.ids[t * n + tid] : (tid == kMostAlternatives ? y : -1);
        const bool there = id >= 0 && id < V;
        w.id[tid] = there ? (int)id : -1;
        if (there) logit = E::one(row, id);
    }
    chain_words<E, NT>(w, sp, kEntries, tid);
    int same = -1;   // the entry that stands for this one's word
    if (tid < kEntries && w.id[tid] >= 0) same = first_of<E, NT>(w, sp, tid);

    Seen seen{-INFINITY, 0.f, 0.f};
    float edge_left = edge;
    RowSpan before = sp;
    before.chunks = rest;
    if constexpr (WORK == Listed::Distill) {
        LeftOut<E, NT> left(w, sp, tid);
        if (left.edge) edge_left = -INFINITY;
        for (int c = tid; c < rest; c += 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT, Reading::Again>(z, row, before, c);
            static_for<0, 4>([&](auto I) {
                constexpr int i = decltype(I)::value;
                if (c + i * NT == left.at && c + i * NT < rest) left.take(z[i], c + i * NT);
            });
            see_chunks<E, false>(seen, z, k);
        }
        if constexpr (H > 0)
            static_for<0, H>([&](auto I) {
                constexpr int i = decltype(I)::value;
                if (rest + tid + i * NT == left.at) left.take(x[i], rest + tid + i * NT);
            });
    } else {
        for (int c = tid; c < rest; c += 4 * NT) {
            u32x4 z[4];
            load_chunks<E, NT, Reading::Again>(z, row, before, c);
            see_chunks<E, ENTROPY>(seen, z, k);
        }
    }
    see_max<ENTROPY>(seen, fmaxf(seen.m, edge_left), k);
    see<ENTROPY>(seen, edge_left, k);
    if constexpr (H > 0) see_chunks<E, ENTROPY>(seen, x, k);
    const float m = fold_row<NT>(seen.m, shared[0], [](float p, float q) { return fmaxf(p, q); }), base = m == -INFINITY ? 0.f : m;
    see_max<ENTROPY>(seen, m, k);
    auto plus = [](float p, float q) { return p + q; };
    const float s = fold_row<NT>(seen.s, shared[1], plus);
    const float sx = ENTROPY ? fold_row<NT>(seen.w, shared[2], plus) : 0.f;

    // the list's numbers, by the first wave: entries `lane`, 64 + lane, and the taken token by all of it
    // (the logits lie with the threads that read them: they go through LDS)
    if (tid < kEntries) w.value[tid] = logit;
    __shared__ int stands[kEntries];
    if (tid < kEntries) stands[tid] = same;
    __syncthreads();
    if (tid < 64) {
        const double weight = a.l.weights ? (double)a.l.weights[t] : 1.0, inv_t = (double)a.l.inv_t + a.l.inv_t_low;
        const int ye = stands[kMostAlternatives];   // entry that stands for the taken token, or -1
        const double ly = ye >= 0 ? (double)w.value[kMostAlternatives] : 0.0;
        float value[2] = {0.f, 0.f}, y_value = 0.f;
        bool live[2];
        float l[2];
        for (int i = 0; i < 2; ++i) {
            const int e = tid + 64 * i;
            live[i] = e < n && stands[e] == e;
            l[i] = w.value[e];
        }
        if constexpr (WORK == Listed::Distill) {
            double logq[2], q[2], share = 0.0;
            float lm = -INFINITY;
            for (int i = 0; i < 2; ++i) {
                logq[i] = live[i] ? (double)a.words.logp[t * n + tid + 64 * i] : -INFINITY;
                q[i] = exp(logq[i]);
                share += q[i];
                if (live[i]) lm = fmaxf(lm, l[i]);
            }
            share = sum_wave(share);
            lm = fold_wave<64>(lm, [](float p, float r) { return fmaxf(p, r); });
            const float whole_m = fmaxf(m, lm), whole_base = whole_m == -INFINITY ? 0.f : whole_m;
            // sum over all words, relative to the largest: that of the rest, that of the named
            double named = 0.0;
            for (int i = 0; i < 2; ++i)
                if (live[i]) named += exp(((double)l[i] - whole_base) * inv_t);
            named = sum_wave(named);
            const double down = exp(((double)base - whole_base) * inv_t);   // (a rest without any word has s = 0)
            const double all = named + (s == 0.f ? 0.0 : s * down), log_all = log(all);
            double left = 0.0, shift = 0.0;
            if (a.distill.renormalise) {
                shift = log(share);
                for (int i = 0; i < 2; ++i) q[i] /= share;
                if (share == 0.0) q[0] = q[1] = 0.0;
                share = share == 0.0 ? 0.0 : 1.0;
            } else if (!(s == 0.f)) {
                left = fmax(0.0, 1.0 - share);
                if (share != share) left = share;
            }
            const double whole = share + left, none = all > 0.0 && all < INFINITY ? 0.0 : NAN;   // (NAN: a row without probabilities)
            // KL = sum q f(log p - log q) + Q - 1
            auto term = [](double q_, double log_q, double log_p) -> double {
                const double p = exp(log_p);
                if (q_ == 0.0) return p;
                const double d = log_p - log_q;
                if (!(d < 1.0)) return p - q_ - q_ * d;
                const float df = (float)d;
                return q_ * (double)kl_of(df, expm1f(df));
            };
            double kl = 0.0, log_p[2];
            for (int i = 0; i < 2; ++i) {
                log_p[i] = ((double)l[i] - whole_base) * inv_t - log_all;
                if (live[i]) kl += term(q[i], logq[i] - shift, log_p[i]);
            }
            kl = sum_wave(kl);
            const double log_rest = s == 0.f ? -INFINITY : log((double)s) + ((double)base - whole_base) * inv_t - log_all;
            kl += term(left, log(left), log_rest) + (whole - 1.0);
            if (whole == 0.0) kl = 0.0;     // (a teacher that says nothing)
            kl += none;
            const double ce = a.distill.ce, ly_p = (ly - whole_base) * inv_t - log_all;
            const double nll = ye >= 0 ? -ly_p : 0.0;
            const double c = (double)a.distill.scale * weight * inv_t + none;
            // at named words c ((Q + ce) p - q - ce [taken]), of the rest e (c (Q + ce) / sum - c q_r / sum of the rest)
            for (int i = 0; i < 2; ++i)
                value[i] = (float)(c * ((whole + ce) * exp(log_p[i]) - q[i] - (ye == tid + 64 * i ? ce : 0.0)));
            const double slope = s == 0.f ? none : c * ((whole + ce) * down / all - left / s);
            y_value = (float)(slope * exp((ly - base) * inv_t) - c * ce);
            if (tid == 0) {
                numbers = RowNumbers{(float)slope, 0.f, 0.f};
                if (a.kl) a.kl[t] = (float)kl;
                a.terms[2 * t] = kl;
                a.terms[2 * t + 1] = nll;
            }
        } else {
            // derivatives by the words' log-probabilities, equal words' added in the order of the entries
            double d[2] = {0.0, 0.0}, all_d = 0.0, yd = 0.0;
            const double dy = ye >= 0 && a.dlogp ? (double)a.dlogp[t] : 0.0;
            bool again = false;
            for (int i = 0; i < 2; ++i) {
                const int e = tid + 64 * i;
                if (e < n && stands[e] >= 0) all_d += d[i] = (double)a.dtop[t * n + e];
                again |= e < n && stands[e] >= 0 && !live[i];
            }
            if (__any(again))
                for (int i = 0; i < 2; ++i)
                    for (int f = tid + 64 * i + 1; live[i] && f < n; ++f)
                        if (stands[f] == tid + 64 * i) d[i] += (double)a.dtop[t * n + f];
            for (int i = 0; i < 2; ++i)
                if (ye == tid + 64 * i) d[i] += dy;
            all_d = sum_wave(all_d) + dy;
            if (ye == kMostAlternatives) yd = dy;
            const double dH = a.dentropy ? (double)a.dentropy[t] * 0.693147180559945309 : 0.0, mean = ENTROPY ? (double)sx / s : 0.0;
            const Dense dense{base, k, (float)(-all_d * inv_t / s), (float)(dH * inv_t / s), (float)mean};
            for (int i = 0; i < 2; ++i) value[i] = dense.of<ENTROPY>(l[i]) + (float)(d[i] * inv_t);
            y_value = dense.of<ENTROPY>((float)ly) + (float)(yd * inv_t);
            if (tid == 0) numbers = RowNumbers{dense.a, dense.b, dense.mean};
        }
        for (int i = 0; i < 2; ++i) w.value[tid + 64 * i] = value[i];
        if (tid == 0) w.value[kMostAlternatives] = y_value;
    }
    __syncthreads();
    if (!out) return;
    const Dense dense{base, k, numbers.a, numbers.b, numbers.mean};
    if constexpr (H > 0) store_dense<E, NT, ENTROPY>(x, out, sp, dense, rest + tid);
    for (int first = (rest - 1) / (4 * NT) * (4 * NT); rest > 0 && first >= 0; first -= 4 * NT) {
        u32x4 z[4];
        load_chunks<E, NT>(z, row, before, first + tid);
        store_dense<E, NT, ENTROPY>(z, out, before, dense, first + tid);
    }
    if (tid < sp.edge) E::put(out, sp.edge_element(tid), dense.of<ENTROPY>(edge));
    // (a wave's own stores to one word keep their order)
    for (int e = w.head[tid]; e >= 0; e = w.next[e])
        if (stands[e] == e) E::put(out, w.id[e], w.value[e]);
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
    if (chunks <= 8192) return listed_kernel<E, 1024, 8, WORK, ENTROPY><<<rows, 1024, 0, stream>>>(a);
    listed_kernel<E, 1024, 16, WORK, ENTROPY><<<rows, 1024, 0, stream>>>(a);
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
