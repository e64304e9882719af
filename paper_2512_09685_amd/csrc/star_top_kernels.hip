// Log-probabilities of the taken tokens with the entropy and the most likely alternatives.
//
// With x_j = (l_j - m) k, m = max l, k = log2(e) / temperature, e_j = 2^x_j, s = sum e_j and w = sum e_j x_j (none of it above 0):
//     log p_j = (l_j - m) / temperature - log s,   H = -sum p_j log p_j = log s - log 2 w / s.
// Alternatives are ordered by their logits, which no rounding has touched yet, ties by the lower id: a word's key is its value's order in 32 bits,
// then the complement of its id, so that no two are alike.
#include <hip/hip_runtime.h>

#include "star_logits.h"

namespace star {

namespace {

struct TopArgs {
    Logits l;                            // its targets may be null: all rows count
    int k;                               // 0 to kMostAlternatives
    float *logp, *entropy, *lse, *top;   // each may be null
    int64_t* ids;
    int64_t first;
};

// Order of a value among others as an unsigned number (0 and -0 alike).  -inf, and what is below it, is no alternative.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
constexpr uint32_t kBanned = 0x007fffffu;   // order_of(-inf)
__device__ __forceinline__ uint64_t key_of(uint32_t order, int j) { return (uint64_t)order << 32 | (uint32_t)~j; }

// A row's maximum, sum and sum of e_j x_j.
struct Moments {
    float m, s, w;
};
// The same relative to a larger maximum.  (A side that has seen nothing but -inf adds nothing.)
__device__ __forceinline__ Moments rebased(const Moments& a, float base, float k) {
    const float x = (a.m - base) * k, f = __builtin_amdgcn_exp2f(x);
    return Moments{base, a.s * f, a.s == 0.f ? 0.f : (a.w + a.s * x) * f};
}
__device__ __forceinline__ void add_element(Moments& a, float l, float k) {   // (a.m is finite, or all so far is -inf)
    const float x = (l - a.m) * k, e = __builtin_amdgcn_exp2f(x);
    a.s += e;
    a.w = __builtin_fmaf(e, fmaxf(x, -1e30f), a.w);   // (0 of a value of -inf; NaN comes through e)
}

// f(value, id) for a thread's elements of a row.
template <class E, int NT, class F>
__device__ __forceinline__ void for_elements(const char* row, const RowSpan& sp, int tid, F&& f) {
    const u32x4* chunk = reinterpret_cast<const u32x4*>(row + sp.head * E::BYTES);
    for (int c = tid; c < sp.chunks; c += NT) {
        const u32x4 x = chunk[c];
        static_for<0, E::VEC>([&](auto J) { f(E::template get<decltype(J)::value>(x), sp.head + c * E::VEC + decltype(J)::value); });
    }
    if (tid < sp.edge) f(E::one(row, sp.edge_element(tid)), sp.edge_element(tid));
}

// Keys that a workgroup has put together, and the count of them.
struct KeyList {
    int count;
    uint64_t key[kMostAlternatives];
};

// The k largest keys of the row, one digit of 8 bits at a time: a histogram of the keys that agree with the digits found so far, then the digit in
// which the k-th lies.  Reads the row once a digit, and once more; ends where a digit leaves no choice.  Fewer than k if the row holds fewer.
template <class E, int NT>
__device__ void select_by_digits(const char* row, const RowSpan& sp, int k, KeyList& list, int (&bins)[256], int (&found)[2]) {
    const int tid = threadIdx.x;
    uint64_t prefix = 0;   // digits found, the rest 0: in the end the k-th key
    int need = k;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += NT) bins[i] = 0;
        __syncthreads();
        for_elements<E, NT>(row, sp, tid, [&](float v, int j) {
            const uint64_t key = key_of(order_of(v), j);
            if (order_of(v) > kBanned && (shift == 56 || (key ^ prefix) >> (shift + 8) == 0)) atomicAdd(&bins[key >> shift & 255], 1);
        });
        __syncthreads();
        if (tid == 0) {
            int more = 0, b = 255;   // keys in the digits above b
            for (; b > 0 && more + bins[b] < need; --b) more += bins[b];
            found[0] = b;
            found[1] = need - more;   // wanted of digit b, which may hold fewer: all of them then
        }
        __syncthreads();
        const int b = found[0];
        need = found[1];
        prefix |= (uint64_t)b << shift;
        const bool all = bins[b] <= need;
        __syncthreads();
        if (all) break;
    }
    if (tid == 0) list.count = 0;
    __syncthreads();
    for_elements<E, NT>(row, sp, tid, [&](float v, int j) {
        const uint64_t key = key_of(order_of(v), j);
        if (order_of(v) > kBanned && key >= prefix) list.key[atomicAdd(&list.count, 1)] = key;
    });
    __syncthreads();
}

template <class E, int NT>
__global__ __launch_bounds__(NT) void top_kernel(const TopArgs a) {
    __shared__ float shared[3][NT / 64];
    __shared__ KeyList list;
    __shared__ int bins[256], found[2];
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    const int64_t t = a.first + blockIdx.x, y = a.l.targets ? a.l.targets[t] : 0;
    int64_t* ids = a.ids + t * a.k;
    float* top = a.top + t * a.k;
    if (a.l.targets && (y < 0 || y >= V)) {
        if (tid == 0) {
            if (a.logp) a.logp[t] = 0.f;
            if (a.entropy) a.entropy[t] = 0.f;
            if (a.lse) a.lse[t] = 0.f;
        }
        if (tid < a.k) {
            ids[tid] = -1;
            top[tid] = 0.f;
        }
        return;
    }
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    const RowSpan sp = row_span<E, NT>(row, V);
    const float k = a.l.k;
    float most = -INFINITY;
    for_elements<E, NT>(row, sp, tid, [&](float v, int) { most = fmaxf(most, v); });
    const float m = fold_row<NT>(most, shared[0], [](float p, float q) { return fmaxf(p, q); });
    Moments mine{m == -INFINITY ? 0.f : m, 0.f, 0.f};
    for_elements<E, NT>(row, sp, tid, [&](float v, int) { add_element(mine, v, k); });
    const float s = fold_row<NT>(mine.s, shared[1], [](float p, float q) { return p + q; });
    const float w = fold_row<NT>(mine.w, shared[2], [](float p, float q) { return p + q; });
    const Two log_s = two_log(s);
    if (tid == 0) {
        if (a.logp) a.logp[t] = add(scaled_difference(a.l, E::one(row, y), m), log_s, -1.f).high;
        if (a.lse) a.lse[t] = add(scaled_difference(a.l, m, 0.f), log_s, 1.f).high;
        if (a.entropy) a.entropy[t] = (log_s.high - kLn2 * (w / s)) + log_s.low;
    }
    if (a.k == 0) return;
    const bool there = s > 0.f && s < INFINITY;   // (a row of NaN, +inf or nothing but -inf has no alternatives)
    if (there) select_by_digits<E, NT>(row, sp, a.k, list, bins, found);
    const int n = there ? min(list.count, a.k) : 0;
    if (tid < n) {
        const uint64_t key = list.key[tid];
        int rank = 0;
        for (int i = 0; i < n; ++i) rank += list.key[i] > key;
        ids[rank] = (int64_t)(uint32_t)~(uint32_t)key;
        top[rank] = add(scaled_difference(a.l, value_of((uint32_t)(key >> 32)), m), log_s, -1.f).high;
    }
    if (tid >= n && tid < a.k) {
        ids[tid] = -1;
        top[tid] = there ? -INFINITY : NAN;
    }
}

template <class E>
void launch_top_of(const TopArgs& a, unsigned rows, hipStream_t stream) {
    if (a.l.vocab <= 2048 * E::VEC) top_kernel<E, 256><<<rows, 256, 0, stream>>>(a);
    else top_kernel<E, 1024><<<rows, 1024, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_top(const Logits& l, int k, float* logp, float* entropy, float* lse, int64_t* ids, float* top, hipStream_t stream) {
    TopArgs a{l, k, logp, entropy, lse, top, ids, 0};
    constexpr int64_t kRows = (int64_t)1 << 21;
    for (a.first = 0; a.first < l.tokens; a.first += kRows) {
        const unsigned rows = (unsigned)std::min(kRows, l.tokens - a.first);
        if (l.dtype == STAR_F32) launch_top_of<ElemF32>(a, rows, stream);
        else launch_top_of<ElemBf16>(a, rows, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace star
