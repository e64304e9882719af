// Losses on the logits of the taken tokens, and their gradients.
//
// A row of logits l_0 .. l_{V-1} gives, with k = log2(e) / temperature and m = max l,
//     e_j = 2^((l_j - m) k),   s = sum e_j,   logp = (l_y - m) / temperature - log s,   p_j = e_j / s
// and every loss here is a function of the rows' logp, so that its gradient is one number c a row:
//     dl_j = c / temperature ([j = y] - p_j).
// All of it is bound by memory: 2 or 4 bytes an element in, as many out, against about 4 operations.
#include <hip/hip_runtime.h>

#include "star_device.h"
#include "star_worker.h"

namespace star {

namespace {

typedef u32x4 u32x4_any __attribute__((aligned(2)));   // (see f32x4_any)

constexpr float kLog2e = 1.44269504088896340736f;

// 16 bytes of a row as VEC numbers, and back.
struct ElemF32 {
    static constexpr int VEC = 4, BYTES = 4;
    static constexpr uint32_t NOTHING = 0xff800000u;   // -inf, in every element of 4 bytes
    template <int K>
    static __device__ __forceinline__ float get(const u32x4& x) { return __uint_as_float(x[K]); }
    static __device__ __forceinline__ float one(const void* row, int64_t j) { return reinterpret_cast<const float*>(row)[j]; }
    static __device__ __forceinline__ u32x4 pack(const float* v) {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ void put(void* row, int64_t j, float v) { reinterpret_cast<float*>(row)[j] = v; }
};
struct ElemBf16 {
    static constexpr int VEC = 8, BYTES = 2;
    static constexpr uint32_t NOTHING = 0xff80ff80u;
    template <int K>
    static __device__ __forceinline__ float get(const u32x4& x) { return bf16_of<K>(x[K >> 1]); }
    static __device__ __forceinline__ float one(const void* row, int64_t j) {
        return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(row)[j] << 16);
    }
    static __device__ __forceinline__ u32x4 pack(const float* v) {   // (one instruction a pair, to nearest even, NaN stays NaN)
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        union {
            bf16x2 pair[4];
            u32x4 all;
        } r;
        static_for<0, 4>([&](auto I) {
            constexpr int i = decltype(I)::value;
            r.pair[i] = bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
        });
        return r.all;
    }
    static __device__ __forceinline__ void put(void* row, int64_t j, float v) { reinterpret_cast<uint16_t*>(row)[j] = (uint16_t)bf16_bits_rne(v); }
};

// A row as whole 16-byte chunks at aligned addresses, and what is before and behind them: fewer than 2 VEC elements,
// one a thread.  (An odd vocabulary puts every other row off 16 bytes.)
struct RowSpan {
    int head, chunks, edge;   // elements before the chunks, chunks, elements outside them
    int V;
    __device__ __forceinline__ int edge_element(int tid) const { return tid < head ? tid : V - edge + tid; }
};
template <class E>
__device__ __forceinline__ RowSpan row_span(const char* row, int V) {
    RowSpan r;
    r.V = V;
    const int off = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / E::BYTES;
    r.head = off < V ? off : V;
    r.chunks = (V - r.head) / E::VEC;
    r.edge = V - r.chunks * E::VEC;
    return r;
}

// Running maximum and sum of 2^((l - m) k).
struct MaxSum {
    float m, s;
};
__device__ __forceinline__ MaxSum join(const MaxSum a, const MaxSum b, float k) {
    const float m = fmaxf(a.m, b.m);
    // (a side that has seen nothing but -inf adds nothing; two such sides make NaN, as a row of nothing else has to)
    const float fa = __builtin_amdgcn_exp2f((a.m - m) * k), fb = __builtin_amdgcn_exp2f((b.m - m) * k);
    return MaxSum{m, a.s * fa + b.s * fb};
}

// Whether token t counts.
__device__ __forceinline__ bool counts(const Logits& l, int64_t t, int64_t y) {
    return y >= 0 && y < l.vocab && (!l.weights || l.weights[t] != 0.f);
}

// One token's loss, KL estimate, whether it is clipped, and its derivative by logp (unweighted).
struct PolicyTerm {
    float loss, kl, clipped, slope;
};
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& a, int64_t t, float logp) {
    const float A = a.advantages[t], r = expf(logp - a.old_logp[t]);
    const float held = fminf(fmaxf(r, a.low), a.high);
    // (an advantage of 0 costs nothing, also where the ratio has run over)
    const float free_cost = A == 0.f ? 0.f : -A * r, held_cost = A == 0.f ? 0.f : -A * held;
    PolicyTerm p;
    p.clipped = free_cost < held_cost ? 1.f : 0.f;
    p.loss = free_cost < held_cost ? held_cost : free_cost;
    p.slope = free_cost < held_cost ? 0.f : free_cost;
    p.kl = 0.f;
    if (a.kl != 0.f) {
        const float d = a.ref_logp[t] - logp, q = expm1f(d);
        p.kl = q - d;
        p.loss += a.kl * p.kl;
        p.slope -= a.kl * q;
    }
    return p;
}

template <class E, int NT>
__device__ __forceinline__ MaxSum scan_row(const char* row, const RowSpan sp, float k) {
    MaxSum a{-INFINITY, 0.f};
    const int tid = threadIdx.x;
    for (int c = tid; c < sp.chunks; c += NT) {
        const u32x4 x = *(reinterpret_cast<const u32x4*>(row + sp.head * E::BYTES) + c);
        float m = a.m;
        static_for<0, E::VEC>([&](auto I) { m = fmaxf(m, E::template get<decltype(I)::value>(x)); });
        const float base = m == -INFINITY ? 0.f : m;
        float s = a.s * __builtin_amdgcn_exp2f((a.m - base) * k);
        static_for<0, E::VEC>([&](auto I) { s += __builtin_amdgcn_exp2f((E::template get<decltype(I)::value>(x) - base) * k); });
        a = MaxSum{m, s};
    }
    if (tid < sp.edge) {
        const float v = E::one(row, sp.edge_element(tid));
        const float m = fmaxf(a.m, v), base = m == -INFINITY ? 0.f : m;
        a = MaxSum{m, a.s * __builtin_amdgcn_exp2f((a.m - base) * k) + __builtin_amdgcn_exp2f((v - base) * k)};
    }
    return a;
}

// Over the workgroup, in a fixed order; every thread gets the whole.
template <int NT>
__device__ __forceinline__ MaxSum join_group(MaxSum a, float k, MaxSum* shared) {
    float m = a.m;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.f : m;
    float s = a.s * __builtin_amdgcn_exp2f((a.m - base) * k);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    constexpr int WAVES = NT / 64;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = MaxSum{m, s};
    __syncthreads();
    // (every wave joins the waves' results for itself, one a lane)
    const MaxSum w = shared[threadIdx.x % WAVES];
    MaxSum all{w.m, 0.f};
    for (int d = WAVES / 2; d; d >>= 1) all.m = fmaxf(all.m, __shfl_xor(all.m, d));
    all.s = w.s * __builtin_amdgcn_exp2f((w.m - (all.m == -INFINITY ? 0.f : all.m)) * k);
    for (int d = WAVES / 2; d; d >>= 1) all.s += __shfl_xor(all.s, d);
    return all;
}

// dl_j = scaled * 2^((l_j - m) k), plus `c` at the target: one chunk, one element.
struct Slope {
    float k, m, scaled, c;
    int y;
};
template <class E>
__device__ __forceinline__ u32x4 slope_chunk(const u32x4& x, const Slope& p, int first) {
    float v[E::VEC];
    static_for<0, E::VEC>([&](auto I) {
        constexpr int n = decltype(I)::value;
        v[n] = p.scaled * __builtin_amdgcn_exp2f((E::template get<n>(x) - p.m) * p.k);
    });
    const int at = p.y - first;
    if (at >= 0 && at < E::VEC)
        static_for<0, E::VEC>([&](auto I) { v[decltype(I)::value] += at == decltype(I)::value ? p.c : 0.f; });
    return E::pack(v);
}
template <class E>
__device__ __forceinline__ void slope_edge(const char* row, char* out, const RowSpan& sp, const Slope& p) {
    if ((int)threadIdx.x >= sp.edge) return;
    const int j = sp.edge_element(threadIdx.x);
    const float v = p.scaled * __builtin_amdgcn_exp2f((E::one(row, j) - p.m) * p.k);
    E::put(out, j, j == p.y ? v + p.c : v);
}
template <class E, int NT>
__device__ __forceinline__ void write_row(const char* row, char* out, const RowSpan sp, const Slope& p) {
    const u32x4* from = reinterpret_cast<const u32x4*>(row + sp.head * E::BYTES);
    u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
    for (int i = threadIdx.x; i < sp.chunks; i += NT) to[i] = slope_chunk<E>(from[i], p, sp.head + i * E::VEC);
    slope_edge<E>(row, out, sp, p);
}

template <class E, int NT>
__device__ __forceinline__ void zero_row(char* out, int V) {
    const RowSpan sp = row_span<E>(out, V);
    for (int i = threadIdx.x; i < sp.chunks; i += NT) *(reinterpret_cast<u32x4*>(out + sp.head * E::BYTES) + i) = u32x4{0, 0, 0, 0};
    if ((int)threadIdx.x < sp.edge) E::put(out, sp.edge_element(threadIdx.x), 0.f);
}

enum class RowWork { Logprobs, Policy, Grad };

struct RowArgs {
    Logits l;
    PolicyArgs policy;
    float *logp, *lse;
    const float *lse_in, *dlogp;
    char* dlogits;
    int64_t ld_out, first;
};

// A workgroup a row; the row is read a second time for its gradient.
template <class E, int NT, RowWork WORK>
__global__ __launch_bounds__(NT) void logits_row_kernel(const RowArgs a) {
    __shared__ MaxSum shared[NT / 64];
    const int64_t t = a.first + blockIdx.x;
    const int V = (int)a.l.vocab;
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const int64_t y = a.l.targets[t];
    const float k = kLog2e * a.l.inv_t;
    bool live = counts(a.l, t, y);
    if (WORK == RowWork::Grad && live) live = a.dlogp[t] != 0.f;
    if (!live) {
        if (WORK != RowWork::Grad && threadIdx.x == 0) {
            a.logp[t] = 0.f;
            if (WORK == RowWork::Logprobs && a.lse) a.lse[t] = 0.f;
        }
        if (WORK != RowWork::Logprobs) zero_row<E, NT>(out, V);
        return;
    }
    const RowSpan sp = row_span<E>(row, V);
    if constexpr (WORK == RowWork::Grad) {
        // p_j = 2^((l_j - lse temperature) k): the row's maximum is not known here, nor needed
        const float c = a.dlogp[t] * a.l.inv_t, m = a.lse_in[t] / a.l.inv_t;
        write_row<E, NT>(row, out, sp, Slope{k, m, -c, c, (int)y});
    } else {
        const float ly = E::one(row, y);
        const MaxSum all = join_group<NT>(scan_row<E, NT>(row, sp, k), k, shared);
        const float log_s = logf(all.s), logp = (ly - all.m) * a.l.inv_t - log_s;
        if (threadIdx.x == 0) {
            a.logp[t] = logp;
            if (WORK == RowWork::Logprobs && a.lse) a.lse[t] = all.m * a.l.inv_t + log_s;
        }
        if constexpr (WORK == RowWork::Policy) {
            const float w = a.policy.scale * (a.l.weights ? a.l.weights[t] : 1.f);
            const float c = w * policy_term(a.policy, t, logp).slope * a.l.inv_t;
            write_row<E, NT>(row, out, sp, Slope{k, all.m, -c / all.s, c, (int)y});
        }
    }
}

// The chunks as they were loaded, for all that the compiler knows: it would keep every element of a bf16 row widened from one use to the
// next, in twice the registers, for the sake of one instruction an element.
template <int C>
__device__ __forceinline__ void keep_packed(u32x4 (&x)[C]) {
#pragma unroll
    for (int i = 0; i < C; ++i) asm volatile("" : "+v"(x[i]));
}

// The same with the whole row in registers, C chunks a thread: read once.
template <class E, int NT, int C, RowWork WORK>
__global__ __launch_bounds__(NT, C <= 8 ? 8 : 4) void logits_held_kernel(const RowArgs a) {
    __shared__ MaxSum shared[NT / 64];
    const int64_t t = a.first + blockIdx.x;
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    char* out = a.dlogits + t * a.ld_out * E::BYTES;
    const int64_t y = a.l.targets[t];
    const float k = kLog2e * a.l.inv_t;
    if (!counts(a.l, t, y)) {
        if (tid == 0) {
            a.logp[t] = 0.f;
            if (WORK == RowWork::Logprobs && a.lse) a.lse[t] = 0.f;
        }
        if (WORK == RowWork::Policy) zero_row<E, NT>(out, V);
        return;
    }
    const RowSpan sp = row_span<E>(row, V);
    const u32x4* from = reinterpret_cast<const u32x4*>(row + sp.head * E::BYTES);
    u32x4 x[C];
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        x[i] = u32x4{E::NOTHING, E::NOTHING, E::NOTHING, E::NOTHING};
        if (tid + i * NT < sp.chunks) x[i] = __builtin_nontemporal_load(from + tid + i * NT);
    });
    const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    const float ly = E::one(row, y);
    MaxSum mine{edge, 0.f};
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { mine.m = fmaxf(mine.m, E::template get<decltype(J)::value>(x[decltype(I)::value])); });
    });
    const float base = mine.m == -INFINITY ? 0.f : mine.m;
    mine.s = __builtin_amdgcn_exp2f((edge - base) * k);
    keep_packed(x);
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) {
            mine.s += __builtin_amdgcn_exp2f((E::template get<decltype(J)::value>(x[decltype(I)::value]) - base) * k);
        });
    });
    const MaxSum all = join_group<NT>(mine, k, shared);
    const float log_s = logf(all.s), logp = (ly - all.m) * a.l.inv_t - log_s;
    if (tid == 0) {
        a.logp[t] = logp;
        if (WORK == RowWork::Logprobs && a.lse) a.lse[t] = all.m * a.l.inv_t + log_s;
    }
    if constexpr (WORK == RowWork::Policy) {
        const float w = a.policy.scale * (a.l.weights ? a.l.weights[t] : 1.f);
        const float c = w * policy_term(a.policy, t, logp).slope * a.l.inv_t;
        const Slope p{k, all.m, -c / all.s, c, (int)y};
        keep_packed(x);
        u32x4_any* to = reinterpret_cast<u32x4_any*>(out + sp.head * E::BYTES);
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int at = tid + i * NT;
            if (at < sp.chunks) __builtin_nontemporal_store(slope_chunk<E>(x[i], p, sp.head + at * E::VEC), to + at);
        });
        if (tid < sp.edge) {
            const int j = sp.edge_element(tid);
            const float v = p.scaled * __builtin_amdgcn_exp2f((edge - p.m) * p.k);
            E::put(out, j, j == p.y ? v + p.c : v);
        }
    }
}

template <class E, RowWork WORK>
void launch_rows_of(const RowArgs& a, unsigned count, hipStream_t stream) {
    const int64_t chunks = (a.l.vocab + E::VEC - 1) / E::VEC;
    if constexpr (WORK != RowWork::Grad) {
        if (chunks <= 256) return logits_held_kernel<E, 256, 1, WORK><<<count, 256, 0, stream>>>(a);
        if (chunks <= 512) return logits_held_kernel<E, 256, 2, WORK><<<count, 256, 0, stream>>>(a);
        if (chunks <= 1024) return logits_held_kernel<E, 256, 4, WORK><<<count, 256, 0, stream>>>(a);
        if (chunks <= 2048) return logits_held_kernel<E, 512, 4, WORK><<<count, 512, 0, stream>>>(a);
        if (chunks <= 4096) return logits_held_kernel<E, 512, 8, WORK><<<count, 512, 0, stream>>>(a);
        if (chunks <= 8192) return logits_held_kernel<E, 1024, 8, WORK><<<count, 1024, 0, stream>>>(a);
        if (chunks <= 16384) return logits_held_kernel<E, 1024, 16, WORK><<<count, 1024, 0, stream>>>(a);
    }
    logits_row_kernel<E, 512, WORK><<<count, 512, 0, stream>>>(a);
}

template <RowWork WORK>
hipError_t launch_rows(const RowArgs& a, int64_t count, hipStream_t stream) {
    if (count <= 0) return hipSuccess;
    if (a.l.dtype == STAR_F32) launch_rows_of<ElemF32, WORK>(a, (unsigned)count, stream);
    else launch_rows_of<ElemBf16, WORK>(a, (unsigned)count, stream);
    return hipGetLastError();
}

// ---------------------------------------------------------------- sums over tokens
constexpr int kSumThreads = 1024;

// Sum over the workgroup in a fixed order, valid in thread 0.
__device__ __forceinline__ double group_sum(double x, double* shared) {
    x = wave_sum_to_lane63(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)blockDim.x / 64; ++w) s += shared[w];
    return s;
}

__global__ __launch_bounds__(kSumThreads) void policy_stats_kernel(const Logits l, const PolicyArgs a, const float* logp, float* stats) {
    __shared__ double shared[kSumThreads / 64];
    double sum[4] = {0, 0, 0, 0};
    for (int64_t t = threadIdx.x; t < l.tokens; t += kSumThreads) {
        if (!counts(l, t, l.targets[t])) continue;
        const PolicyTerm p = policy_term(a, t, logp[t]);
        const double w = l.weights ? (double)l.weights[t] : 1.0;
        sum[0] += w * p.loss;
        sum[1] += w * p.kl;
        sum[2] += w * p.clipped;
        sum[3] += w;
    }
    for (int i = 0; i < 4; ++i) {
        const double s = group_sum(sum[i], shared);
        if (threadIdx.x == 0) stats[i] = (float)(s * a.scale);
    }
}

// A workgroup a pair.
__global__ __launch_bounds__(kBlock) void pair_kernel(const Logits l, const PreferenceArgs a, const PairOffsets offsets, const float* logp,
                                                      float* dlogp, float* margins, double* terms) {
    __shared__ double shared[kBlock / 64];
    __shared__ double all;
    const int b = blockIdx.x;
    const int64_t from = offsets.at[2 * b], mid = offsets.at[2 * b + 1], to = offsets.at[2 * b + 2];
    double sum = 0.0;
    for (int64_t t = from + threadIdx.x; t < to; t += kBlock) {
        if (!counts(l, t, l.targets[t])) continue;
        const double d = ((double)logp[t] - (double)a.ref_logp[t]) * (l.weights ? (double)l.weights[t] : 1.0);
        sum += t < mid ? d : -d;
    }
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) all = a.beta * sum;
    __syncthreads();
    const double s = all;
    // -log sigmoid(s) = max(-s, 0) + log(1 + e^-|s|)
    const double tail = log1p(exp(-fabs(s)));
    if (threadIdx.x == 0) {
        if (margins) margins[b] = (float)s;
        terms[b] = (1.0 - a.smooth) * (fmax(-s, 0.0) + tail) + a.smooth * (fmax(s, 0.0) + tail);
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

__global__ __launch_bounds__(kBlock) void pair_loss_kernel(const double* terms, const int pairs, const float scale, float* loss) {
    __shared__ double shared[kBlock / 64];
    double sum = 0.0;
    for (int b = threadIdx.x; b < pairs; b += kBlock) sum += terms[b];
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) *loss = (float)(sum * scale);
}

}  // namespace

hipError_t launch_logprobs(const Logits& l, int64_t first, int64_t count, float* logp, float* lse, void*, hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.logp = logp;
    a.lse = lse;
    a.first = first;
    return launch_rows<RowWork::Logprobs>(a, count, stream);
}

hipError_t launch_logprobs_grad(const Logits& l, int64_t first, int64_t count, const float* lse, const float* dlogp, void* dlogits,
                                int64_t ld_out, hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.lse_in = lse;
    a.dlogp = dlogp;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    a.first = first;
    return launch_rows<RowWork::Grad>(a, count, stream);
}

hipError_t launch_policy(const Logits& l, const PolicyArgs& p, float* logp, void* dlogits, int64_t ld_out, void*, hipStream_t stream) {
    RowArgs a{};
    a.l = l;
    a.policy = p;
    a.logp = logp;
    a.dlogits = reinterpret_cast<char*>(dlogits);
    a.ld_out = ld_out;
    return launch_rows<RowWork::Policy>(a, l.tokens, stream);
}

hipError_t launch_policy_stats(const Logits& l, const PolicyArgs& a, const float* logp, float* stats, void*, hipStream_t stream) {
    policy_stats_kernel<<<dim3(1), kSumThreads, 0, stream>>>(l, a, logp, stats);
    return hipGetLastError();
}

hipError_t launch_pairs(const Logits& l, const PreferenceArgs& a, const PairOffsets& offsets, int pairs, const float* logp, float* dlogp,
                        float* margins, double* terms, hipStream_t stream) {
    if (pairs <= 0) return hipSuccess;
    pair_kernel<<<dim3((unsigned)pairs), kBlock, 0, stream>>>(l, a, offsets, logp, dlogp, margins, terms);
    return hipGetLastError();
}

hipError_t launch_pair_loss(const double* terms, int pairs, float scale, float* loss, hipStream_t stream) {
    pair_loss_kernel<<<dim3(1), kBlock, 0, stream>>>(terms, pairs, scale, loss);
    return hipGetLastError();
}

}  // namespace star
