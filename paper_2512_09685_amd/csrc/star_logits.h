// Rows of logits in a kernel: access in 16-byte chunks at any address, numbers in two parts, sums over a wave and a workgroup.
#pragma once

#include "star_device.h"
#include "star_worker.h"

namespace star {

typedef u32x4 u32x4_any __attribute__((aligned(2)));   // (see f32x4_any)

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

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

// A row as whole 16-byte chunks at aligned addresses, and what is before and behind them, one element a thread.  (An odd
// vocabulary puts the rows at any address.)  Workgroups of a row begin their chunks on whole cache lines, so that no two waves write
// parts of one; single waves, with 64 threads for the rest, on 16 bytes.
struct RowSpan {
    int head, chunks, edge;   // elements before the chunks, chunks, elements outside them
    int V;
    __device__ __forceinline__ int edge_element(int tid) const { return tid < head ? tid : V - edge + tid; }
};
template <class E, int NT>
__device__ __forceinline__ RowSpan row_span(const char* row, int V) {
    constexpr int ALIGN = NT > 64 ? 128 : 16;
    RowSpan r;
    r.V = V;
    r.head = min((int)(-reinterpret_cast<uintptr_t>(row) & (ALIGN - 1)) / E::BYTES, V);
    r.chunks = (V - r.head) / E::VEC;
    r.edge = V - r.chunks * E::VEC;
    return r;
}

// A value and what rounding it to fp32 left.  Log-probabilities of size 10 are rounded by up to 5e-7, which ratios of policies and differences of
// sums over tokens would show.
struct Two {
    float high, low;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = a + b, t = s - a;
    return Two{s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Two normal(float high, float low) {
    if (!(fabsf(high) < INFINITY)) return Two{high, 0.f};
    const float s = high + low;
    return Two{s, low - (s - high)};
}
// (a - b) / temperature
__device__ __forceinline__ Two scaled_difference(const Logits& l, float a, float b) {
    const Two d = two_sum(a, -b);
    const float z = d.high * l.inv_t;
    return Two{z, __builtin_fmaf(d.high, l.inv_t, -z) + (d.high * l.inv_t_low + d.low * l.inv_t)};
}
// log s, for s >= 1/2: n log 2 + log f, 1 <= f < 2, with log 2 in two parts of which the first times n is exact.
__device__ __forceinline__ Two two_log(float s) {
    if (!(s < INFINITY)) return Two{s, 0.f};
    const uint32_t b = __float_as_uint(s);
    const float n = (float)((int)(b >> 23) - 127), f = __uint_as_float((b & 0x7fffffu) | 0x3f800000u);
    return Two{n * 0x1.62ep-1f, n * 3.194618494528623e-5f + logf(f)};
}
__device__ __forceinline__ Two add(const Two& a, const Two& b, float sign) {
    const Two s = two_sum(a.high, sign * b.high);
    return normal(s.high, s.low + (a.low + sign * b.low));
}

// e^d - d - 1, `q` = e^d - 1: of small d from its series, where q - d would leave few digits and, of policies close to each other, the wrong sign.
__device__ __forceinline__ float kl_of(float d, float q) {
    if (!(fabsf(d) < 0.25f)) return q - d;
    const float more = __builtin_fmaf(d, __builtin_fmaf(d, __builtin_fmaf(d, __builtin_fmaf(d, 1.f / 5040.f, 1.f / 720.f), 1.f / 120.f), 1.f / 24.f), 1.f / 6.f);
    return d * d * __builtin_fmaf(d, more, 0.5f);
}

// What one thread sees of a row: C chunks in registers (those that it does not have hold -inf) and at most one element more.
template <class E, int C>
__device__ __forceinline__ float max_of(const u32x4 (&x)[C], float more) {
    float m = more;
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { m = fmaxf(m, E::template get<decltype(J)::value>(x[decltype(I)::value])); });
    });
    return m;
}
template <class E, int C>
__device__ __forceinline__ float sum_from(const u32x4 (&x)[C], float more, float m, float k) {
    const float base = m == -INFINITY ? 0.f : m;
    float s = __builtin_amdgcn_exp2f((more - base) * k);
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { s += __builtin_amdgcn_exp2f((E::template get<decltype(J)::value>(x[decltype(I)::value]) - base) * k); });
    });
    return s;
}

// The chunks as they were loaded, for all that the compiler knows: it would keep every element of a bf16 row widened from one use to the
// next, in twice the registers, for the sake of one instruction an element.
template <int C>
__device__ __forceinline__ void keep_packed(u32x4 (&x)[C]) {
#pragma unroll
    for (int i = 0; i < C; ++i) asm volatile("" : "+v"(x[i]));
}

// C chunks a thread from chunk `first` on, NT apart; what is beyond the row holds -inf.  What is read for the last time goes past the
// memory-side cache, which is faster (4096 x 131072, bf16: 157 against 180 us); what is read again is left in it, which the second
// reading gains more from (preference loss of 4096 x 32000, bf16: 107 against 126 us, of 12288 x 32768: 341 against 373; rows of the
// logits_scan_kernel, policy loss of 2048 x 131072, fp32: 345 against 402).
enum class Reading { Last, Again };
template <class E, int NT, Reading HOW = Reading::Last, int C>
__device__ __forceinline__ void load_chunks(u32x4 (&x)[C], const char* row, const RowSpan& sp, int first) {
    const u32x4* from = reinterpret_cast<const u32x4*>(row + sp.head * E::BYTES);
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        x[i] = u32x4{E::NOTHING, E::NOTHING, E::NOTHING, E::NOTHING};
        if (first + i * NT < sp.chunks) x[i] = HOW == Reading::Again ? from[first + i * NT] : __builtin_nontemporal_load(from + first + i * NT);
    });
}

// Over a wave; every lane gets the whole.  (Sides that have seen nothing but -inf add nothing.  A row of nothing else ends here with a sum of 0 and gets its
// NaN from the difference of the taken logit, or of any other, with its maximum.)
template <int LANES = 64>
__device__ __forceinline__ MaxSum join_wave(const MaxSum a, float k) {
    float m = a.m;
    for (int d = LANES / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    float s = a.s * __builtin_amdgcn_exp2f((a.m - (m == -INFINITY ? 0.f : m)) * k);
    for (int d = LANES / 2; d; d >>= 1) s += __shfl_xor(s, d);
    return MaxSum{m, s};
}
// Over the workgroup, in a fixed order; every thread gets the whole.
template <int NT>
__device__ __forceinline__ MaxSum join_group(const MaxSum a, float k, MaxSum* shared) {
    const MaxSum w = join_wave(a, k);
    if constexpr (NT == 64) return w;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = w;
    __syncthreads();
    return join_wave<NT / 64>(shared[threadIdx.x % (NT / 64)], k);   // (every wave for itself, one result a lane)
}

// A long row, chunk by chunk, four of them under way at a time, by NT threads.
template <class E, int NT, Reading HOW = Reading::Last>
__device__ __forceinline__ MaxSum scan_chunks(const char* row, const RowSpan& sp, float k, int tid) {
    MaxSum a{-INFINITY, 0.f};
    for (int c = tid; c < sp.chunks; c += 4 * NT) {
        u32x4 x[4];
        load_chunks<E, NT, HOW>(x, row, sp, c);
        const float m = max_of<E>(x, a.m), base = m == -INFINITY ? 0.f : m;
        a = MaxSum{m, a.s * __builtin_amdgcn_exp2f((a.m - base) * k) + sum_from<E>(x, -INFINITY, m, k)};
    }
    return a;
}

// One element more.
__device__ __forceinline__ MaxSum with_element(const MaxSum& a, float l, float k) {
    const float m = fmaxf(a.m, l), base = m == -INFINITY ? 0.f : m;
    return MaxSum{m, a.s * __builtin_amdgcn_exp2f((a.m - base) * k) + __builtin_amdgcn_exp2f((l - base) * k)};
}

// Whether a row's exponents have to be formed from differences with its maximum, `z` the maximum times k: round(z) is off by up to
// |z| 2^-24 from m k, which up to 2^22 adds nothing to what rounding to a whole number leaves, and from 2^31 on would leave an exponent
// that fp32 does not hold for the maximum itself.  (True also for infinities and NaN.)
__device__ __forceinline__ bool is_far(float z) { return !(fabsf(z) <= 0x1p22f); }

// Zeros to the chunks of [from, to) by NT threads, and to the rest of the row if they begin it.
template <class E, int NT>
__device__ __forceinline__ void zero_row(char* out, int V, int tid, int from = 0, int to = 0x7fffffff) {
    const RowSpan sp = row_span<E, NT>(out, V);
    u32x4* chunk = reinterpret_cast<u32x4*>(out + sp.head * E::BYTES);
    for (int i = from + tid; i < min(to, sp.chunks); i += NT) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, chunk + i);
    if (from == 0 && tid < sp.edge) E::put(out, sp.edge_element(tid), 0.f);
}

// N sums over a workgroup of NT threads in a fixed order, valid in thread 0.
template <int NT, int N>
__device__ __forceinline__ void group_sums(double (&x)[N], double (*shared)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_sum_to_lane63(x[i]);
    __syncthreads();
    if ((threadIdx.x & 63) == 63)
#pragma unroll
        for (int i = 0; i < N; ++i) shared[threadIdx.x >> 6][i] = x[i];
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = 0.0;
            for (int w = 0; w < NT / 64; ++w) x[i] += shared[w][i];
        }
    }
}

// Maximum and sum over the threads of a row, in a fixed order; every thread gets them.
template <int LANES, class Op>
__device__ __forceinline__ float fold_wave(float x, Op&& op) {
    for (int d = LANES / 2; d; d >>= 1) x = op(x, __shfl_xor(x, d));
    return x;
}
template <int NT, class Op>
__device__ __forceinline__ float fold_row(float x, float* shared, Op&& op) {
    x = fold_wave<64>(x, op);
    if constexpr (NT == 64) return x;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    return fold_wave<NT / 64>(shared[threadIdx.x % (NT / 64)], op);
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

// Maximum and sum over the workgroup, in a fixed order; every thread gets them.
template <int WAVES>
__device__ __forceinline__ float max_group(float x, float* shared) {
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) x = fmaxf(x, shared[i]);
    return x;
}
template <int WAVES>
__device__ __forceinline__ float sum_group(float x, float* shared) {
    x = wave_sum_to_lane63(x);
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) x += shared[i];
    return x;
}

// 2^x is 0 from here on down; products of it with x are formed with no less, so that they are 0 too.
constexpr float kNoExponent = -1e4f;

// Maximum, sum, and (where asked) sum of e_j x_j of what a thread has seen.
struct Seen {
    float m, s, w;
};
template <bool ENTROPY>
__device__ __forceinline__ void see_max(Seen& a, float m, float k) {
    const float base = m == -INFINITY ? 0.f : m, x = (a.m - base) * k, f = __builtin_amdgcn_exp2f(x);
    if (ENTROPY) a.w = (a.w + a.s * fmaxf(x, kNoExponent)) * f;
    a.s *= f;
    a.m = m;
}
template <bool ENTROPY>
__device__ __forceinline__ void see(Seen& a, float l, float k) {   // a.m is no less
    const float x = (l - (a.m == -INFINITY ? 0.f : a.m)) * k, e = __builtin_amdgcn_exp2f(x);
    a.s += e;
    if (ENTROPY) a.w = __builtin_fmaf(e, fmaxf(x, kNoExponent), a.w);   // (0 of a value of -inf; NaN comes through e)
}
template <class E, bool ENTROPY, int C>
__device__ __forceinline__ void see_chunks(Seen& a, u32x4 (&x)[C], float k) {
    see_max<ENTROPY>(a, max_of<E>(x, a.m), k);
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) { see<ENTROPY>(a, E::template get<decltype(J)::value>(x[decltype(I)::value]), k); });
    });
}

// x = (l - m) k as one multiply-add, l k - e with the whole number e = round(m k), where that loses nothing (is_far); it is `off` too large.
struct Exponent {
    float m, k, e, off;
    bool far;
    template <bool FAR>
    __device__ __forceinline__ float of(float l) const {
        return FAR ? (l - m) * k : __builtin_fmaf(l, k, -e);
    }
};
__device__ __forceinline__ Exponent exponent_of(float m, float k) {
    const bool far = is_far(m * k);
    const float e = far ? 0.f : rintf(m * k);
    return Exponent{m == -INFINITY ? 0.f : m, k, e, far ? 0.f : __builtin_fmaf(m, k, -e), far};
}
// Both have been formed here, for all that the compiler knows: it would put a sum off to where it is used, and keep all of its terms till then.
__device__ __forceinline__ void pinned(float& s, float& w) { asm volatile("" : "+v"(s), "+v"(w)); }
// max_of many values: those that are not negative are ordered as their bits are, two bf16 to an instruction and none widened; a wave with a thread that
// has nothing but negative values looks at all of them again.  (A NaN comes out, or the largest of the others.  Distillation, 8192 x 65536, bf16:
// 359.4 us, with max_of 361.4; alternatives and their gradient, 2048 x 65536: 136 either way.)
template <class E, int C>
__device__ __forceinline__ float max_of_many(const u32x4 (&x)[C], float more) {
    if constexpr (E::VEC == 4) {
        return max_of<E>(x, more);
    } else {
        typedef short __attribute__((ext_vector_type(2))) s16x2;
        s16x2 m{-32768, -32768};
        static_for<0, C>([&](auto I) {
            static_for<0, 4>([&](auto J) {
                const uint32_t pair = x[decltype(I)::value][decltype(J)::value];   // (of a vector's element itself, a bit cast takes the first)
                m = __builtin_elementwise_max(m, __builtin_bit_cast(s16x2, pair));
            });
        });
        const int most = max((int)m[0], (int)m[1]);
        float f = __uint_as_float((uint32_t)most << 16);
        if (__any(most < 0)) f = max_of<E>(x, -INFINITY);
        return fmaxf(f, more);
    }
}
// Adds C chunks a thread and one element more, none of them above a.m.
template <class E, bool ENTROPY, int C>
__device__ __forceinline__ void see_held(Seen& a, u32x4 (&x)[C], float more, const Exponent& p) {
    float s = 0.f, w = 0.f;
    auto all = [&](auto far) {
        keep_packed(x);   // (or elements would be widened for both ways at once)
        auto one = [&](float l) {
            const float z = p.of<decltype(far)::value>(l), e = __builtin_amdgcn_exp2f(z);
            s += e;
            if (ENTROPY) w = __builtin_fmaf(e, fmaxf(z, kNoExponent), w);
        };
        one(more);
        static_for<0, C>([&](auto I) {
            static_for<0, E::VEC>([&](auto J) { one(E::template get<decltype(J)::value>(x[decltype(I)::value])); });
            pinned(s, w);
        });
    };
    if (p.far) all(std::true_type{});
    else all(std::false_type{});
    const float f = __builtin_amdgcn_exp2f(-p.off);
    a.s += s * f;
    if (ENTROPY) a.w += (w - p.off * s) * f;
}

// Workgroups go round the 8 dies; this gives each die a run of long rows of its own (8192 x 65536, bf16: 4 % faster, 16384 x
// 32768: 7 %; rows of 16 KB and less are up to 5 % slower that way and stay in the order of the workgroups, as do rows whose number is no
// multiple of 8).
__device__ __forceinline__ int64_t die_run(unsigned id) {
    return gridDim.x % 8 == 0 ? (id % 8) * (gridDim.x / 8) + id / 8 : id;
}

}  // namespace star
