// Root-mean-square norm with the residual's addition, and its gradient.
//
//     h = x + residual (as it is stored),   rstd = 1 / sqrt(mean h^2 + eps),   y = h rstd g
//     dh = rstd (g dy - h' mean(g dy h')) + dresidual,   dg = sum over the rows of dy h',   h' = h rstd
// Bound by memory: a row stays in registers between its sum and what is made of it, so that every tensor is read or written once.  Sums are taken
// in 64 bits, which costs two instructions an element of the fifty that there is time for, and leaves squares of any size in range.
// (16381 x 4096, bf16, with residual: 86 us, 6.2 TB/s; the gradient of 8192 x 8192, bf16: 94 us, 5.7 TB/s, and 4 us for the join of the gain's sums.)
#include <hip/hip_runtime.h>

#include "star_logits.h"

namespace star {

namespace {

// Rows as chunks of 16 bytes from their first element on, at any address; the elements behind the last chunk are one a thread.
struct Span {
    int chunks, tail;
};
template <class E>
__device__ __forceinline__ Span span_of(int width) {
    return Span{width / E::VEC, width % E::VEC};
}
__device__ __forceinline__ const char* at_row(const Rows& r, int64_t t, int bytes) { return reinterpret_cast<const char*>(r.x) + t * r.ld * bytes; }

template <class E, int NT, int C>
__device__ __forceinline__ void load_row(u32x4 (&x)[C], const char* row, const Span& sp, int tid) {
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        x[i] = u32x4{0, 0, 0, 0};
        if (tid + i * NT < sp.chunks) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row) + tid + i * NT);
    });
}

// VEC gains from column j on.
template <int VEC>
__device__ __forceinline__ void load_gain(float (&g)[VEC], const void* gain, int dtype, int j) {
    if (!gain) {
        static_for<0, VEC>([&](auto I) { g[decltype(I)::value] = 1.f; });
    } else if (dtype == STAR_F32) {
        static_for<0, VEC / 4>([&](auto I) {
            const f32x4 v = reinterpret_cast<const f32x4_any*>(reinterpret_cast<const float*>(gain) + j)[decltype(I)::value];
            static_for<0, 4>([&](auto J) { g[4 * decltype(I)::value + decltype(J)::value] = v[decltype(J)::value]; });
        });
    } else {
        static_for<0, VEC / 4>([&](auto I) {
            const u32x2 v = reinterpret_cast<const u32x2_any*>(reinterpret_cast<const uint16_t*>(gain) + j)[decltype(I)::value];
            static_for<0, 4>([&](auto J) {
                constexpr int jj = decltype(J)::value;
                g[4 * decltype(I)::value + jj] = bf16_of<jj>(v[jj >> 1]);
            });
        });
    }
}
__device__ __forceinline__ float one_gain(const void* gain, int dtype, int j) {
    return !gain ? 1.f : dtype == STAR_F32 ? ElemF32::one(gain, j) : ElemBf16::one(gain, j);
}

// Sum over the NT threads of a row, in a fixed order; every thread gets it.  `shared`: NT / 64 numbers of the row's own.
template <int NT>
__device__ __forceinline__ double sum_row(double x, double* shared) {
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    if constexpr (NT == 64) return x;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) x += shared[i];
    return x;
}

struct NormArgs {
    Norm n;
    Rows x, residual;
    char *sum, *y;
    int64_t ld_sum, ld_y;
    float* rstd;
    float eps;
    int64_t first;
};

// NT threads a row of C chunks each, 256 / NT rows a workgroup (one, of more threads).
template <class E, int NT, int C>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_kernel(const NormArgs a) {
    constexpr int ROWS = NT < 256 ? 256 / NT : 1;
    __shared__ double shared[NT / 64];
    const int tid = threadIdx.x % NT, width = (int)a.n.width;
    const int64_t t = a.first + (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0);
    if (ROWS > 1 && t >= a.n.tokens) return;
    const Span sp = span_of<E>(width);
    const int last = width - sp.tail + tid;   // the thread's element behind the chunks, if tid < sp.tail
    const char* row = at_row(a.x, t, E::BYTES);
    u32x4 x[C];
    load_row<E, NT>(x, row, sp, tid);
    float more = tid < sp.tail ? E::one(row, last) : 0.f;
    if (a.residual.x) {
        const char* other = at_row(a.residual, t, E::BYTES);
        u32x4 r[C];
        load_row<E, NT>(r, other, sp, tid);
        u32x4_any* to = reinterpret_cast<u32x4_any*>(a.sum + t * a.ld_sum * E::BYTES);
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            float v[E::VEC];
            static_for<0, E::VEC>([&](auto J) {
                constexpr int j = decltype(J)::value;
                v[j] = E::template get<j>(x[i]) + E::template get<j>(r[i]);
            });
            x[i] = E::pack(v);   // the norm is that of the sum as it is stored
            if (tid + i * NT < sp.chunks) __builtin_nontemporal_store(x[i], to + tid + i * NT);
        });
        if (tid < sp.tail) {
            more += E::one(other, last);
            E::put(to, last, more);
            if (E::BYTES == 2) more = __uint_as_float(bf16_bits_rne(more) << 16);
        }
    }
    double s = (double)more * more;
    static_for<0, C>([&](auto I) {
        static_for<0, E::VEC>([&](auto J) {
            const double v = (double)E::template get<decltype(J)::value>(x[decltype(I)::value]);
            s = __builtin_fma(v, v, s);
        });
    });
    keep_packed(x);
    s = sum_row<NT>(s, shared);
    const float rstd = (float)(1.0 / sqrt(s / width + (double)a.eps));
    if (tid == 0 && a.rstd) a.rstd[t] = rstd;
    char* out = a.y + t * a.ld_y * E::BYTES;
    static_for<0, C>([&](auto I) {
        constexpr int i = decltype(I)::value;
        const int c = tid + i * NT;
        if (c < sp.chunks) {
            float v[E::VEC], g[E::VEC];
            load_gain(g, a.n.gain, a.n.gain_dtype, c * E::VEC);
            static_for<0, E::VEC>([&](auto J) { v[decltype(J)::value] = (E::template get<decltype(J)::value>(x[i]) * rstd) * g[decltype(J)::value]; });
            reinterpret_cast<u32x4_any*>(out)[c] = E::pack(v);
        }
    });
    if (tid < sp.tail) E::put(out, last, (more * rstd) * one_gain(a.n.gain, a.n.gain_dtype, last));
}

// ---------------------------------------------------------------- gradient
struct NormGradArgs {
    Norm n;
    Rows dy, h, dresidual;
    const float* rstd;
    char* dx;
    int64_t ld_dx;
    float* partial;   // [workgroups][width]: sums of the gain's gradient; null: not wanted
};

// Workgroups take rows in turn and keep the gains of their columns, and the sums of dy h', in registers.
template <class E, int NT, int C, bool GAIN>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_grad_kernel(const NormGradArgs a) {
    constexpr int ROWS = NT < 256 ? 256 / NT : 1;
    constexpr bool HELD = NT < 1024 || C <= 2;   // (gains and dresidual: of longer rows they do not fit, and are read where they are used)
    __shared__ double shared[2][NT / 64];
    __shared__ float joined[GAIN && ROWS > 1 ? (ROWS - 1) * NT * (C * E::VEC + 1) : 1];
    const int tid = threadIdx.x % NT, in = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0, width = (int)a.n.width;
    const Span sp = span_of<E>(width);
    const int last = width - sp.tail + tid;
    float sum[C][E::VEC] = {}, sum_more = 0.f, held[HELD ? C : 1][E::VEC] = {};
    auto gains_of = [&](auto I, float (&g)[E::VEC]) {
        constexpr int i = decltype(I)::value;
        load_gain(g, a.n.gain, a.n.gain_dtype, (tid + i * NT) * E::VEC);
    };
    if constexpr (HELD)
        static_for<0, C>([&](auto I) {
            if (tid + decltype(I)::value * NT < sp.chunks) gains_of(I, held[decltype(I)::value]);
        });
    const float g_more = tid < sp.tail ? one_gain(a.n.gain, a.n.gain_dtype, last) : 0.f;
    int turn = 0;
    for (int64_t t = (int64_t)blockIdx.x * ROWS + in; t < a.n.tokens; t += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const char *dy_row = at_row(a.dy, t, E::BYTES), *h_row = at_row(a.h, t, E::BYTES);
        const char* more_row = a.dresidual.x ? at_row(a.dresidual, t, E::BYTES) : nullptr;
        u32x4 d[C], h[C], r[HELD ? C : 1];
        load_row<E, NT>(d, dy_row, sp, tid);
        load_row<E, NT>(h, h_row, sp, tid);
        if constexpr (HELD) {
            if (more_row) load_row<E, NT>(r, more_row, sp, tid);
            else static_for<0, C>([&](auto I) { r[decltype(I)::value] = u32x4{0, 0, 0, 0}; });
        }
        const float rstd = a.rstd[t];
        float d_more = 0.f, h_more = 0.f, r_more = 0.f;
        if (tid < sp.tail) {
            d_more = E::one(dy_row, last);
            h_more = E::one(h_row, last) * rstd;
            if (more_row) r_more = E::one(more_row, last);
        }
        double s = (double)(d_more * g_more) * h_more;
        if (GAIN) sum_more += d_more * h_more;
        static_for<0, C>([&](auto I) {   // (what a row does not have holds 0)
            constexpr int i = decltype(I)::value;
            if (!HELD && tid + i * NT >= sp.chunks) return;   // (a branch a chunk keeps the compiler from having all chunks' gains under way)
            float g[E::VEC];
            if constexpr (!HELD) gains_of(I, g);
            static_for<0, E::VEC>([&](auto J) {
                constexpr int j = decltype(J)::value;
                const float dj = E::template get<j>(d[i]), hj = E::template get<j>(h[i]) * rstd, gj = HELD ? held[HELD ? i : 0][j] : g[j];
                if (GAIN) sum[i][j] += dj * hj;
                s = __builtin_fma((double)(dj * gj), (double)hj, s);
            });
        });
        keep_packed(d);
        keep_packed(h);
        const float mean = (float)(sum_row<NT>(s, shared[turn]) / width);   // (two turns' numbers lie apart: one barrier a row is enough)
        u32x4_any* out = reinterpret_cast<u32x4_any*>(a.dx + t * a.ld_dx * E::BYTES);
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int c = tid + i * NT;
            if (c < sp.chunks) {
                float v[E::VEC], g[E::VEC];
                u32x4 more{0, 0, 0, 0};
                if constexpr (HELD) {
                    more = r[i];
                } else {
                    gains_of(I, g);
                    if (more_row) more = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(more_row) + c);
                }
                static_for<0, E::VEC>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    const float hj = E::template get<j>(h[i]) * rstd, gj = HELD ? held[HELD ? i : 0][j] : g[j];
                    v[j] = rstd * (E::template get<j>(d[i]) * gj - hj * mean) + E::template get<j>(more);
                });
                __builtin_nontemporal_store(E::pack(v), out + c);
            }
        });
        if (tid < sp.tail) E::put(out, last, rstd * (d_more * g_more - h_more * mean) + r_more);
    }
    if constexpr (GAIN) {
        if constexpr (ROWS > 1) {
            // the waves' sums, in their order
            if (in > 0) {
                float* mine = joined + (in - 1) * NT * (C * E::VEC + 1) + tid;
                static_for<0, C>([&](auto I) {
                    static_for<0, E::VEC>([&](auto J) { mine[(decltype(I)::value * E::VEC + decltype(J)::value) * NT] = sum[decltype(I)::value][decltype(J)::value]; });
                });
                mine[C * E::VEC * NT] = sum_more;
            }
            __syncthreads();
            if (in > 0) return;
            for (int w = 0; w < ROWS - 1; ++w) {
                const float* other = joined + w * NT * (C * E::VEC + 1) + tid;
                static_for<0, C>([&](auto I) {
                    static_for<0, E::VEC>([&](auto J) { sum[decltype(I)::value][decltype(J)::value] += other[(decltype(I)::value * E::VEC + decltype(J)::value) * NT]; });
                });
                sum_more += other[C * E::VEC * NT];
            }
        }
        float* to = a.partial + (int64_t)blockIdx.x * width;
        static_for<0, C>([&](auto I) {
            constexpr int i = decltype(I)::value;
            const int c = tid + i * NT;
            if (c < sp.chunks)
                static_for<0, E::VEC / 4>([&](auto J) {
                    constexpr int j = 4 * decltype(J)::value;
                    reinterpret_cast<f32x4_any*>(to + c * E::VEC)[decltype(J)::value] = f32x4{sum[i][j], sum[i][j + 1], sum[i][j + 2], sum[i][j + 3]};
                });
        });
        if (tid < sp.tail) to[last] = sum_more;
    }
}

// The workgroups' sums joined: 32 columns a workgroup, 32 threads a column.
constexpr int kJoinThreads = 1024, kJoinColumns = 32;
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const float* partial, int groups, int width, void* dgain, int dtype, bool accumulate) {
    constexpr int PARTS = kJoinThreads / kJoinColumns;
    __shared__ double shared[PARTS][kJoinColumns + 1];
    const int in = threadIdx.x % kJoinColumns, c = (int)blockIdx.x * kJoinColumns + in, part = threadIdx.x / kJoinColumns;
    double s = 0.0;
    if (c < width)
#pragma unroll 8
        for (int g = part; g < groups; g += PARTS) s += (double)partial[(int64_t)g * width + c];
    shared[part][in] = s;
    __syncthreads();
    // (a column's 32 sums lie with the lanes of half a wave)
    s = shared[in][part];
    for (int d = 16; d; d >>= 1) s += __shfl_xor(s, d);
    const int column = (int)blockIdx.x * kJoinColumns + part;
    if (in != 0 || column >= width) return;
    if (dtype == STAR_F32) {
        float* to = reinterpret_cast<float*>(dgain) + column;
        *to = (float)(accumulate ? (double)*to + s : s);
    } else {
        uint16_t* to = reinterpret_cast<uint16_t*>(dgain) + column;
        const double held = accumulate ? (double)__uint_as_float((uint32_t)*to << 16) : 0.0;
        *to = (uint16_t)bf16_bits_rne((float)(held + s));
    }
}

// Threads a row and chunks a thread, by the chunks of a row (8 a thread: fp32 alone, the widest rows).  Measured (us, this way / the other; bf16, both
// directions but where said): a wave a row up to 256 chunks against 256 threads: 16384 x 1024: 58 / 86; 256 threads up to 512 against 512: 16384 x
// 4096: 178.5 / 181; 512 up to 1024 against 256: 8192 x 8192, the norm alone: 82.7 / 85.9; 1024 up to 2048 against 512: 8192 x 16384: 378 / 395, 1000 x
// 5003, fp32: 32 / 30.
static_assert(kMostNormWidth / ElemBf16::VEC <= 4096 && kMostNormWidth / ElemF32::VEC <= 8192);
template <class F>
void for_width(int64_t chunks, F&& f) {
    if (chunks <= 64) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    else if (chunks <= 256) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
    else if (chunks <= 512) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    else if (chunks <= 1024) f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    else if (chunks <= 2048) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    else if (chunks <= 4096) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
}
int64_t chunks_of(int dtype, int64_t width) { return dtype == STAR_F32 ? (width + 3) / 4 : (width + 7) / 8; }
int rows_a_group(int64_t chunks) { return chunks <= 256 ? 4 : 1; }

}  // namespace

hipError_t launch_norm(const Norm& n, const Rows& x, const Rows& residual, float eps, void* sum, int64_t ld_sum, void* y, int64_t ld_y, float* rstd,
                       hipStream_t stream) {
    const int64_t chunks = chunks_of(n.dtype, n.width), rows = rows_a_group(chunks);
    NormArgs a{n, x, residual, reinterpret_cast<char*>(sum), reinterpret_cast<char*>(y), ld_sum, ld_y, rstd, eps, 0};
    constexpr int64_t kGroups = (int64_t)1 << 21;
    for (a.first = 0; a.first < n.tokens; a.first += kGroups * rows) {
        const unsigned grid = (unsigned)std::min(kGroups, (n.tokens - a.first + rows - 1) / rows);
        for_width(chunks, [&](auto nt, auto c) {
            constexpr int NT = decltype(nt)::value, C = decltype(c)::value;
            if (n.dtype == STAR_F32) norm_kernel<ElemF32, NT, C><<<grid, NT < 256 ? 256 : NT, 0, stream>>>(a);
            else if constexpr (C < 8) norm_kernel<ElemBf16, NT, C><<<grid, NT < 256 ? 256 : NT, 0, stream>>>(a);
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int norm_grad_groups(int dtype, int64_t tokens, int64_t width) {
    // Two a unit, which hold the row, its gains and their sums in registers (us, 512 / 256 / 1024 groups: 8192 x 8192 and 16384 x 4096, bf16: 192 / 213 /
    // 199 and 180 / 220 / 195), one where that leaves them fewer than four turns, whose sums cost as much as their rows (1000 x 5003, fp32:
    // 34.3 / 31.5 / 39.1).
    const int64_t rows = rows_a_group(chunks_of(dtype, width)), turns = (tokens + rows - 1) / rows;
    return (int)std::max<int64_t>(1, std::min<int64_t>({turns, 512, std::max<int64_t>(256, turns / 4)}));
}

hipError_t launch_norm_grad(const Norm& n, const Rows& dy, const Rows& h, const float* rstd, const Rows& dresidual, void* dx, int64_t ld_dx, void* dgain,
                            int dgain_dtype, bool accumulate, void* workspace, hipStream_t stream) {
    NormGradArgs a{n, dy, h, dresidual, rstd, reinterpret_cast<char*>(dx), ld_dx, dgain ? reinterpret_cast<float*>(workspace) : nullptr};
    const int groups = norm_grad_groups(n.dtype, n.tokens, n.width);
    if (n.tokens > 0) {
        for_width(chunks_of(n.dtype, n.width), [&](auto nt, auto c) {
            constexpr int NT = decltype(nt)::value, C = decltype(c)::value;
            auto of = [&](auto elem) {
                typedef decltype(elem) E;
                if (dgain) norm_grad_kernel<E, NT, C, true><<<groups, NT < 256 ? 256 : NT, 0, stream>>>(a);
                else norm_grad_kernel<E, NT, C, false><<<groups, NT < 256 ? 256 : NT, 0, stream>>>(a);
            };
            if (n.dtype == STAR_F32) of(ElemF32{});
            else if constexpr (C < 8) of(ElemBf16{});
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!dgain) return hipSuccess;
    norm_join_kernel<<<dim3((unsigned)((n.width + kJoinColumns - 1) / kJoinColumns)), kJoinThreads, 0, stream>>>(a.partial, n.tokens > 0 ? groups : 0, (int)n.width, dgain,
                                                                                         dgain_dtype, accumulate);
    return hipGetLastError();
}

}  // namespace star
