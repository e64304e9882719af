// Log-probabilities of the taken tokens with the entropy and the most likely alternatives.
//
// With x_j = (l_j - m) k, m = max l, k = log2(e) / temperature, e_j = 2^x_j, s = sum e_j and w = sum e_j x_j (none of it above 0):
//     log p_j = (l_j - m) / temperature - log s,   H = -sum p_j log p_j = log s - log 2 w / s.
// Alternatives are ordered by their logits, which no rounding has touched yet, ties by the lower id: a word's key is its value's order in 32 bits,
// then the complement of its id, so that no two are alike.
//
// One reading of the logits is all that it cannot do without.  Beside the memory it is the vector instructions that count: nine an element of a bf16
// row (widen, multiply-add, exponential of two turns, two sums, the entropy's product and its guard, half a maximum), and what the lists cost a row.
// 4096 x 131072, bf16, k = 64, a tenth of the rows without a target: 197 us, 4.9 TB/s, vector pipes busy 86 % (without the entropy 187, without
// alternatives 168, without both 152; the scan for log-probabilities alone 148).  All rows counting: 210, 201, 180, 167 and 159.  1023 x 50021, fp32, k =
// 5, all counting: 37 us, 5.5 TB/s.
#include <hip/hip_runtime.h>

#include "star_logits.h"

namespace star {

namespace {

struct TopArgs {
    Logits l;                            // its targets may be null: all rows count
    int k;                               // 0 to kMostAlternatives
    float *logp, *entropy, *lse, *top;   // each may be null
    int64_t* ids;
    bool again;                          // the rows may be read again by the gradient's launch
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
template <int ROOM>
struct KeyList {
    int count;
    uint64_t key[ROOM];
    __device__ __forceinline__ void put(uint64_t k) {
        const int at = atomicAdd(&count, 1);
        if (at < ROOM) key[at] = k;
    }
};

// The k largest keys of the row, one digit of 8 bits at a time: a histogram of the keys that agree with the digits found so far, then the digit in
// which the k-th lies.  Reads the row once a digit, and once more; ends where a digit leaves no choice.  Fewer than k if the row holds fewer.
template <class E, int NT, int ROOM>
__device__ void select_by_digits(const char* row, const RowSpan& sp, int k, KeyList<ROOM>& list, int (&bins)[256], int (&found)[2]) {
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
        if (order_of(v) > kBanned && key >= prefix) list.put(key);
    });
    __syncthreads();
}

// A wave's chunks that hold a value that may be an alternative, as they were read, and the ids of their first words; `count` is the wave's, and may
// be more than there is room for.  (A list a wave needs no atomics; one list of the workgroup took 6 % more for 4096 x 131072, k = 64.)
constexpr int kHot = 128;
struct HotChunks {
    u32x4 chunk[kHot];
    int id[kHot];
    __device__ __forceinline__ void put(int& count, bool hot, const u32x4& x, int first) {
        const unsigned long long lanes = __ballot(hot);
        if (lanes == 0) return;
        const int at = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0u));
        if (hot && at < kHot) {
            chunk[at] = x;
            id[at] = first;
        }
        count += __popcll(lanes);
    }
};

// How far values lie below the row's largest one, in steps of 1/32 of an octave from 2^-14 to 2^18 (what lies nearer or further: the first, the
// last).  In such steps the k-th value's distance is found to 3 % at any scale of the logits.
constexpr int kSteps = 1024;
__device__ __forceinline__ int step_of(float distance) {
    return min(max((int)(__float_as_uint(distance) >> 18) - ((127 - 14) << 5), 0), kSteps - 1);   // (NaN: the last)
}
// A little more than any distance of that step.
__device__ __forceinline__ float beyond_step(int step) {
    return step == kSteps - 1 ? INFINITY : __uint_as_float((uint32_t)(step + 1 + ((127 - 14) << 5)) << 18) * (1.f + 0x1p-20f);
}

// A bound that at least k values of the row reach: the least of about the k largest of what the threads have seen at most, one value a thread (or
// of what `count` counts), by a histogram of their distances from the largest.  `most` becomes the workgroup's.  Without alternatives nothing
// but that is formed, and no barrier stands behind the reading of `shared`: it is this function's alone.
template <int NT, class F>
__device__ __forceinline__ float bound_of(float& most, int k, float* shared, int (&steps)[kSteps], float& least, F&& count) {
    constexpr int WAVES = NT / 64;
    const int tid = threadIdx.x;
    const float mine = most, m = wave_max(mine);
    if ((tid & 63) == 0) shared[tid >> 6] = m;
    for (int i = tid; i < kSteps / 4; i += NT) reinterpret_cast<u32x4*>(steps)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) most = fmaxf(most, shared[i]);
    if (k == 0) return INFINITY;
    count(mine, [&](float v) { atomicAdd(&steps[step_of(most - v)], 1); });
    __syncthreads();
    if (tid < 64) {
        // 16 steps a lane, then the lane in which the k-th value lies, then the step
        u32x4 n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = reinterpret_cast<const u32x4*>(steps)[4 * tid + i];
        int own = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) own += (int)n[i / 4][i % 4];
        int up_to = own;
        for (int d = 1; d < 64; d *= 2) {
            const int below = __shfl_up(up_to, d);
            if (tid >= d) up_to += below;
        }
        if (tid == 63 && up_to < k) least = -3.402823466e38f;   // (fewer words than alternatives)
        if (up_to >= k && up_to - own < k) {                    // (one lane)
            int sum = up_to - own, step = -1;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (step < 0 && sum + (int)n[i / 4][i % 4] >= k) step = i;
                sum += (int)n[i / 4][i % 4];
            }
            least = fmaxf(most - beyond_step(16 * tid + step), -3.402823466e38f);   // (banned words are no alternatives)
        }
    }
    __syncthreads();
    return least;
}

// A workgroup a row.  Its first H chunks a thread are held in registers until their largest values are known, one a thread: the k-th largest
// of these (or a little less) is no more than that of the row.  Chunks with a value that reaches it go on a list, their words that do on a second one, which holds the
// alternatives and little else (about 1.1 k words of a row held whole, more in proportion of one that is not), and a word's place among
// them is the number of larger keys.  The rest of the row goes by once.  A row that has more such words than the lists hold -- of equal
// values, or rising ones -- is searched digit by digit.
template <class E, int NT, int H, bool ENTROPY>
__global__ __launch_bounds__(NT, H == 16 || NT == 64 ? 4 : 6) void top_kernel(const TopArgs a) {
    constexpr int WAVES = NT / 64, KEYS = NT >= 512 ? 1024 : NT == 256 ? 512 : 256, AHEAD = H == 16 && E::VEC == 8 ? 8 : 4;
    constexpr bool LONG = H == 16;   // rows that are not held whole; the others' registers are not to pay for them (8192 x 8000, k = 20: 35 / 38 us)
    __shared__ float shared[4][WAVES];   // sum of the exponentials, that of the entropy, the whole row's maximum, the bound's: each written once
    __shared__ __align__(16) int steps[kSteps];
    __shared__ float bound;
    __shared__ KeyList<KEYS> list;
    __shared__ HotChunks hots[WAVES];
    __shared__ uint64_t sorted[kMostAlternatives];
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
        for (int i = tid; i < a.k; i += NT) {
            ids[i] = -1;
            top[i] = 0.f;
        }
        return;
    }
    const char* row = reinterpret_cast<const char*>(a.l.x) + t * a.l.ld * E::BYTES;
    const RowSpan sp = row_span<E, NT>(row, V);
    const float k = a.l.k;
    u32x4 x[H];
    if (a.again) load_chunks<E, NT, Reading::Again>(x, row, sp, tid);
    else load_chunks<E, NT>(x, row, sp, tid);
    const float edge = tid < sp.edge ? E::one(row, sp.edge_element(tid)) : -INFINITY;
    const float ly = E::one(row, y);
    if (tid == 0) list.count = 0;
    HotChunks& hot = hots[tid >> 6];
    int chunks = 0;   // of the wave's
    float most_of[H], most = edge;
    static_for<0, H>([&](auto I) {
        constexpr int i = decltype(I)::value;
        const u32x4 one[1] = {x[i]};
        most_of[i] = max_of<E>(one, -INFINITY);
        most = fmaxf(most, most_of[i]);
    });
    keep_packed(x);
    // (few threads have a value for so many alternatives: all words are counted then)
    const bool all = H <= 4 && min(sp.chunks, NT) < 2 * a.k;
    const float least = bound_of<NT>(most, a.k, shared[3], steps, bound, [&](float mine, auto&& add_one) {
        if (all) {
            static_for<0, H>([&](auto I) {
                static_for<0, E::VEC>([&](auto J) {
                    const float v = E::template get<decltype(J)::value>(x[decltype(I)::value]);
                    if (v > -INFINITY) add_one(v);
                });
            });
            if (edge > -INFINITY) add_one(edge);
        } else {
            add_one(mine);
        }
    });
    static_for<0, H>([&](auto I) {
        constexpr int i = decltype(I)::value;
        hot.put(chunks, most_of[i] >= least, x[i], sp.head + (tid + i * NT) * E::VEC);
    });
    Seen seen{most, 0.f, 0.f};
    see_held<E, ENTROPY>(seen, x, edge, exponent_of(most, k));
    if constexpr (LONG) for (int c = tid + H * NT; c - tid < sp.chunks; c += AHEAD * NT) {   // (all of a wave, for its list)
        u32x4 z[AHEAD];
        if (a.again) load_chunks<E, NT, Reading::Again>(z, row, sp, c);
        else load_chunks<E, NT>(z, row, sp, c);
        float m[AHEAD], of_all = -INFINITY;
        static_for<0, AHEAD>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const u32x4 one[1] = {z[i]};
            m[i] = max_of<E>(one, -INFINITY);
            of_all = fmaxf(of_all, m[i]);
        });
        if (__any(of_all >= least))
            static_for<0, AHEAD>([&](auto I) {
                constexpr int i = decltype(I)::value;
                hot.put(chunks, m[i] >= least, z[i], sp.head + (c + i * NT) * E::VEC);
            });
        if (of_all > seen.m) see_max<ENTROPY>(seen, of_all, k);
        static_for<0, AHEAD>([&](auto I) {
            static_for<0, E::VEC>([&](auto J) { see<ENTROPY>(seen, E::template get<decltype(J)::value>(z[decltype(I)::value]), k); });
        });
    }
    float m = most;
    if (LONG && sp.chunks > H * NT) {
        m = max_group<WAVES>(seen.m, shared[2]);
        see_max<ENTROPY>(seen, m, k);
    }
    float s = sum_group<WAVES>(seen.s, shared[0]), w = ENTROPY ? sum_group<WAVES>(seen.w, shared[1]) : 0.f;
    // (the largest term is 1 and its x 0, which two exponentials that undo each other need not give: no log-probability is above 0, no entropy below)
    s = s > 0.f && s < 1.f ? 1.f : s;
    w = fminf(w, 0.f);
    Two log_s{0.f, 0.f};
    if (tid < kMostAlternatives) log_s = two_log(s);   // (the threads that write)
    if (tid == 0) {
        if (a.logp) a.logp[t] = add(scaled_difference(a.l, ly, m), log_s, -1.f).high;
        if (a.lse) a.lse[t] = add(scaled_difference(a.l, m, 0.f), log_s, 1.f).high;
        if (ENTROPY) a.entropy[t] = (log_s.high - kLn2 * (w / s)) + log_s.low;
    }
    if (a.k == 0) return;
    const bool there = s > 0.f && s < INFINITY;   // (a row of NaN, +inf or nothing but -inf has no alternatives)
    int n = 0;
    if (there) {
        // every wave's own list; one that has run over leaves too many keys
        if (chunks > kHot) {
            if ((tid & 63) == 0) atomicAdd(&list.count, KEYS + 1);
            chunks = 0;
        }
        for (int first = 0; first < chunks * E::VEC; first += 64) {
            const int i = first + (tid & 63), in = min(i / E::VEC, kHot - 1);
            const float v = i < chunks * E::VEC ? E::one(&hot.chunk[in], i % E::VEC) : -INFINITY;
            const unsigned long long lanes = __ballot(v >= least);
            int at = 0;
            if ((tid & 63) == 0) at = atomicAdd(&list.count, __popcll(lanes));
            at = __builtin_amdgcn_readlane(at, 0) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0u));
            if (v >= least && at < KEYS) list.key[at] = key_of(order_of(v), hot.id[in] + i % E::VEC);
        }
        if (edge >= least) list.put(key_of(order_of(edge), sp.edge_element(tid)));
        __syncthreads();
        n = list.count;
        if (n > KEYS) {
            __syncthreads();
            select_by_digits<E, NT>(row, sp, a.k, list, *reinterpret_cast<int(*)[256]>(steps), *reinterpret_cast<int(*)[2]>(steps + 256));
            n = list.count;
        }
        // four threads a key, a quarter of the others each
        for (int first = (tid & ~63) / 4; first < n; first += NT / 4) {
            const int e = first + (tid & 63) / 4;
            const uint64_t key = e < n ? list.key[e] : ~0ull;
            int place = 0;
#pragma unroll 8
            for (int i = tid % 4; i < n; i += 4) place += list.key[i] > key;
            place += __builtin_amdgcn_update_dpp(0, place, 0xB1, 0xf, 0xf, false);
            place += __builtin_amdgcn_update_dpp(0, place, 0x4E, 0xf, 0xf, false);
            if (e < n && place < a.k && tid % 4 == 0) sorted[place] = key;
        }
        n = min(n, a.k);
    }
    __syncthreads();
    for (int i = tid; i < a.k; i += NT) {
        const uint64_t key = i < n ? sorted[i] : 0;
        ids[i] = i < n ? (int64_t)(uint32_t)~(uint32_t)key : -1;
        top[i] = i < n ? add(scaled_difference(a.l, value_of((uint32_t)(key >> 32)), m), log_s, -1.f).high : there ? -INFINITY : NAN;
    }
}

// Threads a row, by its chunks: as few as hold it in registers up to 8192 chunks, two rows a unit at least (us, this way / the other; bf16):
// one and two waves up to 128 and 512 chunks against four: 16384 x 1000, k = 20: 27 / 58, 16384 x 4000: 41 / 54; 4 chunks a thread up to 1024
// against 8: 8192 x 8000: 34 / 46; 512 threads up to 4096 against 1024: 4096 x 32000: 58 / 70; beyond, 16 chunks a thread against 8 of 1024:
// 4096 x 131072, k = 64: 217 / 277.  Against 8 of 512, which leave room for a third row on a unit, but hold half as much and list twice as many words:
// k = 64: 4096 x 131072: 217 / 224, 2048 x 65536: 63 / 64; k = 8: 194 / 173, 2048 x 65536 with the gradient 152 / 148; 1023 x 50021, fp32, k = 5: 37.3 /
// 35.4.  (So the few alternatives of a server would do better with 8: the rule does not look at k.)
template <class E, bool ENTROPY>
void launch_top_of(const TopArgs& a, unsigned rows, hipStream_t stream) {
    const int64_t chunks = (a.l.vocab + E::VEC - 1) / E::VEC;
    if (chunks <= 128) top_kernel<E, 64, 2, ENTROPY><<<rows, 64, 0, stream>>>(a);
    else if (chunks <= 512) top_kernel<E, 128, 4, ENTROPY><<<rows, 128, 0, stream>>>(a);
    else if (chunks <= 1024) top_kernel<E, 256, 4, ENTROPY><<<rows, 256, 0, stream>>>(a);
    else if (chunks <= 2048) top_kernel<E, 256, 8, ENTROPY><<<rows, 256, 0, stream>>>(a);
    else if (chunks <= 4096) top_kernel<E, 512, 8, ENTROPY><<<rows, 512, 0, stream>>>(a);
    else top_kernel<E, 512, 16, ENTROPY><<<rows, 512, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_top(const Logits& l, int k, float* logp, float* entropy, float* lse, int64_t* ids, float* top, bool again, hipStream_t stream) {
    TopArgs a{l, k, logp, entropy, lse, top, ids, again, 0};
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
