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

// Keys that a workgroup has put together, and the count of them (which may be more than there is room for).
constexpr int kListed = 1024;
struct KeyList {
    int count;
    uint64_t key[kListed];
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

// Over a wave, without LDS: the maximum, in every lane.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_max(float x) {   // (lanes without a source keep their own)
    const int b = __float_as_int(x);
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(b, b, CTRL, ROW_MASK, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float x) {
    x = dpp_max<0xB1, 0xf>(x);    // within pairs, quads, 8, 16 lanes, then the rows of 16 (see wave_sum_to_lane63)
    x = dpp_max<0x4E, 0xf>(x);
    x = dpp_max<0x141, 0xf>(x);
    x = dpp_max<0x140, 0xf>(x);
    x = dpp_max<0x142, 0xa>(x);
    x = dpp_max<0x143, 0xc>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// The r-th largest of the lanes' values.
__device__ __forceinline__ float wave_rth(float x, int r) {
    float m = wave_max(x);
    for (; r > 1 && m > -INFINITY; --r) {
        if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)__ballot(x == m)) - 1) x = -INFINITY;
        m = wave_max(x);
    }
    return m;
}

// Puts the values of x that are no less than `least` on the list.  (A lane's largest value of a chunk tells first whether any is.)
template <class E>
__device__ __forceinline__ void list_chunk(KeyList& list, const u32x4& x, float least, int id) {
    u32x4 one[1] = {x};
    if (max_of<E>(one, -INFINITY) < least) return;
    static_for<0, E::VEC>([&](auto J) {
        const float v = E::template get<decltype(J)::value>(x);
        if (v >= least) {
            const int at = atomicAdd(&list.count, 1);
            if (at < kListed) list.key[at] = key_of(order_of(v), id + decltype(J)::value);
        }
    });
}

// A workgroup a row.  Its first H chunks a thread are held in registers until their largest values are known, one a thread: of these the
// `rank`-th of every wave, and of those the least, is no more than the k-th largest value of the row.  Words that reach it go on a list, which
// holds the alternatives and little else (about 1.3 k words of a row held whole, more in proportion of one that is not), and a word's place among them is the
// number of larger keys.  The rest of the row goes by once.  A row that has more such words than the list holds -- of equal values, or
// rising ones -- is searched digit by digit.
template <class E, int NT, int H, bool ENTROPY>
__global__ __launch_bounds__(NT, 8) void top_kernel(const TopArgs a) {
    __shared__ float shared[4][NT / 64];
    __shared__ KeyList list;
    __shared__ int bins[256], found[2];
    const int V = (int)a.l.vocab, tid = threadIdx.x;
    const int64_t t = a.first + (NT >= 512 ? die_run(blockIdx.x) : (int64_t)blockIdx.x), y = a.l.targets ? a.l.targets[t] : 0;
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
    u32x4 x[H];
    load_chunks<E, NT>(x, row, sp, tid);
    const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    const float ly = E::one(row, y);
    if (tid == 0) list.count = 0;
    const float mine = max_of<E>(x, edge);
    keep_packed(x);
    const float rth = a.k ? wave_rth(mine, (a.k + NT / 64 - 1) / (NT / 64)) : INFINITY, most = wave_max(mine);
    if ((tid & 63) == 0) {
        shared[0][tid >> 6] = most;
        shared[1][tid >> 6] = rth;
    }
    __syncthreads();
    Seen seen{-INFINITY, 0.f, 0.f};
    float least = shared[1][0];
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        seen.m = fmaxf(seen.m, shared[0][i]);
        least = fminf(least, shared[1][i]);
    }
    least = fmaxf(least, -3.402823466e38f);   // (banned words are no alternatives)
    static_for<0, H>([&](auto I) {
        constexpr int i = decltype(I)::value;
        list_chunk<E>(list, x[i], least, sp.head + (tid + i * NT) * E::VEC);
    });
    if (edge >= least) {
        const int at = atomicAdd(&list.count, 1);
        if (at < kListed) list.key[at] = key_of(order_of(edge), sp.edge_element(tid));
    }
    keep_packed(x);
    see<ENTROPY>(seen, edge, k);
    static_for<0, H>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { see<ENTROPY>(seen, E::template get<decltype(J)::value>(x[decltype(I)::value]), k); });
    });
    for (int c = tid + H * NT; c < sp.chunks; c += 4 * NT) {
        u32x4 z[4];
        load_chunks<E, NT>(z, row, sp, c);
        const float m = max_of<E>(z, -INFINITY);
        if (m >= least)
            static_for<0, 4>([&](auto I) {
                constexpr int i = decltype(I)::value;
                list_chunk<E>(list, z[i], least, sp.head + (c + i * NT) * E::VEC);
            });
        if (m > seen.m) see_max<ENTROPY>(seen, m, k);
        static_for<0, 4>([&](auto I) {
            static_for<0, E::VEC>([&](auto J) { see<ENTROPY>(seen, E::template get<decltype(J)::value>(z[decltype(I)::value]), k); });
        });
    }
    float m = seen.m;
    if (sp.chunks > H * NT) {
        m = wave_max(m);
        __syncthreads();
        if ((tid & 63) == 0) shared[0][tid >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) m = fmaxf(m, shared[0][i]);
        see_max<ENTROPY>(seen, m, k);
    }
    auto plus = [](float p, float q) { return p + q; };
    const float s = fold_row<NT>(seen.s, shared[2], plus), w = ENTROPY ? fold_row<NT>(seen.w, shared[3], plus) : 0.f;
    const Two log_s = two_log(s);
    if (tid == 0) {
        if (a.logp) a.logp[t] = add(scaled_difference(a.l, ly, m), log_s, -1.f).high;
        if (a.lse) a.lse[t] = add(scaled_difference(a.l, m, 0.f), log_s, 1.f).high;
        if (ENTROPY) a.entropy[t] = (log_s.high - kLn2 * (w / s)) + log_s.low;
    }
    if (a.k == 0) return;
    const bool there = s > 0.f && s < INFINITY;   // (a row of NaN, +inf or nothing but -inf has no alternatives)
    if (there && list.count > kListed) {
        __syncthreads();
        select_by_digits<E, NT>(row, sp, a.k, list, bins, found);
    }
    const int listed = there ? list.count : 0, n = min(listed, a.k);
    for (int e = tid; e < listed; e += NT) {
        const uint64_t key = list.key[e];
        int rank = 0;
        for (int i = 0; i < listed; ++i) rank += list.key[i] > key;
        if (rank >= a.k) continue;
        ids[rank] = (int64_t)(uint32_t)~(uint32_t)key;
        top[rank] = add(scaled_difference(a.l, value_of((uint32_t)(key >> 32)), m), log_s, -1.f).high;
    }
    if (tid >= n && tid < a.k) {
        ids[tid] = -1;
        top[tid] = there ? -INFINITY : NAN;
    }
}

template <class E, bool ENTROPY>
void launch_top_of(const TopArgs& a, unsigned rows, hipStream_t stream) {
    const int64_t chunks = (a.l.vocab + E::VEC - 1) / E::VEC;
    if (chunks <= 512) top_kernel<E, 256, 2, ENTROPY><<<rows, 256, 0, stream>>>(a);
    else if (chunks <= 2048) top_kernel<E, 256, 8, ENTROPY><<<rows, 256, 0, stream>>>(a);
    else if (chunks <= 4096) top_kernel<E, 1024, 4, ENTROPY><<<rows, 1024, 0, stream>>>(a);
    else top_kernel<E, 1024, 8, ENTROPY><<<rows, 1024, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_top(const Logits& l, int k, float* logp, float* entropy, float* lse, int64_t* ids, float* top, hipStream_t stream) {
    TopArgs a{l, k, logp, entropy, lse, top, ids, 0};
    constexpr int64_t kRows = (int64_t)1 << 21;
    for (a.first = 0; a.first < l.tokens; a.first += kRows) {
        const unsigned rows = (unsigned)std::min(kRows, l.tokens - a.first);
        if (l.dtype == STAR_F32) entropy ? launch_top_of<ElemF32, true>(a, rows, stream) : launch_top_of<ElemF32, false>(a, rows, stream);
        else entropy ? launch_top_of<ElemBf16, true>(a, rows, stream) : launch_top_of<ElemBf16, false>(a, rows, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace star
