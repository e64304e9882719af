// Weight gradient from activations kept in 8 bits: dw[n][k] = sum_t dy[t][n] x[t][k].
//
// The kept values are e4m3 * 2^e and with that bf16 numbers, so the matrix instructions for bf16 take them without a rounding;
// one conversion instruction makes two of them, scale and all.  dy in fp32 is cut into three bf16 parts of 8 bits each, whose
// products are all exact: the sums, in fp32, are the only place where anything is rounded before the result.
#include <hip/hip_runtime.h>

#include <cmath>

#include "star_device.h"
#include "star_worker.h"

namespace star {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // (see f32x4_any)
typedef __attribute__((address_space(3))) char lds_char;

struct GradArgs {
    const char* dy;
    const uint8_t *kept, *exponents;
    void* dw;
    float* partial;      // sums of this launch's parts, [parts][out][width]; null: one part, straight to dw
    int64_t tokens, out, ld, width, columns;
    int tiles_n, tiles_k, parts;
    int dw_bf16, accumulate, near;   // near: a stage's offsets into dy fit 31 bits
};

// How dy comes into LDS.  Direct: 16 bytes a lane straight from memory, past the registers, for bf16 rows on 16-byte
// addresses.  Bf16, F32: through registers, from any address; fp32 is cut into its three bf16 parts on the way.
enum class Dy { Direct, Bf16, F32 };

// A tile of dw that a workgroup makes, WAVES_N by WAVES_K waves of NI by NJ results of the 32x32x16 instruction each, in
// steps of STEP tokens.
template <int WAVES_N, int WAVES_K, int NI_, int NJ_, Dy DY>
struct Tile {
    static constexpr int NI = NI_, NJ = NJ_, WAVES_OF_K = WAVES_K, WAVES = WAVES_N * WAVES_K, THREADS = 64 * WAVES;
    static constexpr int N = WAVES_N * NI * 32, K = WAVES_K * NJ * 32;
    static constexpr int PLANES = DY == Dy::F32 ? 3 : 1;
    static constexpr int STEP = DY == Dy::F32 ? 32 : 64, BLOCKS = STEP / kActBlock;
    // One stage in LDS: dy as [plane][token][column] bf16, 32-byte chunks of a token's row in another order
    // (dy_chunk); x as [block][column][32 tokens] bytes; the exponents as [block][column].
    static constexpr int ROW = N * 2, PLANE = STEP * ROW, X_AT = PLANES * PLANE, E_AT = X_AT + STEP * K;
    static constexpr int BYTES = E_AT + (BLOCKS * K + 255) / 256 * 256;
    // Loads of one wave for a stage, 1024 bytes each (256 of exponents).
    static constexpr int DY_LOADS = PLANE / 1024 / WAVES;
    static constexpr int X_ALL = STEP * K / 1024, X_LOADS = (X_ALL + WAVES - 1) / WAVES;
    static constexpr int E_ALL = (BLOCKS * K + 255) / 256;
    // Registers of one thread that dy passes through, 16 bytes each.
    static constexpr int ELEM = DY == Dy::F32 ? 4 : 2, VEC = 16 / ELEM, LANES = N / VEC, ROWS = THREADS / LANES, PASSES = STEP / ROWS;
    static constexpr int GROUPS = BLOCKS * 2 * NJ;   // of products, a column of NI results each
};

// Where chunk c (16 columns, 32 bytes) of token t's row lies: a transposing read takes chunks c and c + 1 of four tokens
// in a row, and the same of the tokens 16 further on; the order puts any 8 of them that one half of a wave asks for
// on different banks (a row is a whole number of turns of all 64 banks, or half of one).
template <int N>
__device__ __forceinline__ int dy_chunk(int t, int c) {
    const int f = N >= 128 ? ((t & 3) << 1) | ((t >> 4) & 1) : (t & 2) | ((t >> 4) & 1);
    return c ^ f;
}

// A buffer of `bytes` bytes (none: 0 or fewer): loads beyond them give 0, stores beyond them do nothing.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, max(bytes, 0), 0x00020000);
}

// What a thread asks for in every stage: offsets from the stage's first token, block and column.
template <class T, Dy DY>
struct Sources {
    int dy[DY == Dy::Direct ? T::DY_LOADS : 1], x[T::X_LOADS], e;
    __device__ __forceinline__ Sources(const GradArgs& a, int wave, int lane) {
        if constexpr (DY == Dy::Direct) {
#pragma unroll
            for (int i = 0; i < T::DY_LOADS; ++i) {
                const int at = (i * T::WAVES + wave) * 1024 + lane * 16, t = at / T::ROW, unit = at % T::ROW / 16;
                dy[i] = t * (int)a.ld * 2 + dy_chunk<T::N>(t, unit >> 1) * 32 + (unit & 1) * 16;
            }
        }
#pragma unroll
        for (int i = 0; i < T::X_LOADS; ++i) {
            const int at = (i * T::WAVES + wave) % T::X_ALL * 1024 + lane * 16, b = at / (T::K * kActBlock);
            x[i] = b * (int)a.columns * kActBlock + at % (T::K * kActBlock);
        }
        const int at = wave % T::E_ALL * 256 + lane * 4, b = at / T::K;
        e = b < T::BLOCKS ? b * (int)a.columns + at % T::K : 0x7fffffff;   // (beyond every buffer: reads 0)
    }
};

// Where the next stage begins.  Sizes within a stage fit 31 bits (launch_choice), addresses move on in 64.
struct Cursor {
    const char* dy;
    const uint8_t *kept, *exponents;
    int tokens;   // still to come, held to 31 bits
};

// Starts the loads of x and its exponents, and of dy where it comes straight, for the next stage.  What lies beyond the last token or
// element is not read and comes as 0; waves in excess load again what another one loads.
template <class T, Dy DY>
__device__ __forceinline__ void load_stage(lds_char* lds, const GradArgs& a, const Sources<T, DY>& s, Cursor& c, int64_t n0, int64_t k0, int wave) {
    if constexpr (DY == Dy::Direct) {
        const int left = min(c.tokens, T::STEP) * (int)a.ld - (int)(a.ld - a.out + n0);   // elements
        // (to the end of the last element's 4-byte word: a word that lies only half in range comes as 0 all of it.  Its other half, of an odd `out`,
        // makes a column that is not written)
        const __amdgpu_buffer_rsrc_t dy = buffer(c.dy, (left * 2 + 3) & ~3);
#pragma unroll
        for (int i = 0; i < T::DY_LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(dy, lds + (i * T::WAVES + wave) * 1024, 16, s.dy[i], 0, 0, 0);
        c.dy += (int64_t)T::STEP * a.ld * 2;
    }
    const int blocks = min((c.tokens + kActBlock - 1) / kActBlock, T::BLOCKS), left = blocks * (int)a.columns - (int)k0;
    const __amdgpu_buffer_rsrc_t x = buffer(c.kept, left * kActBlock), e = buffer(c.exponents, left);
#pragma unroll
    for (int i = 0; i < T::X_LOADS; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(x, lds + T::X_AT + (i * T::WAVES + wave) % T::X_ALL * 1024, 16, s.x[i], 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(e, lds + T::E_AT + wave % T::E_ALL * 256, 4, s.e, 0, 0, 0);
    c.kept += T::BLOCKS * a.columns * kActBlock;
    c.exponents += T::BLOCKS * a.columns;
    c.tokens = max(c.tokens - T::STEP, 0);
}

// dy on its way through registers: VEC columns of PASSES tokens.
template <class T>
struct InRegisters {
    u32x4 v[T::PASSES];
};
// Where a stage's rows of dy lie.  Whole: all of its tokens are there, and nothing that a thread reads is beyond the last row's end (what is
// beyond a row's own end makes columns that are not written).
struct Rows {
    const char* from;
    int first, next;
    bool whole;
};
template <class T>
__device__ __forceinline__ Rows rows_at(const GradArgs& a, int64_t t0, int64_t end, int64_t n0) {
    const int n = (int)(threadIdx.x % T::LANES) * T::VEC, row = (int)(threadIdx.x / T::LANES);
    const int64_t all = (a.tokens - 1) * a.ld + a.out;   // elements up to the last one
    return Rows{a.dy + (t0 * a.ld + n0) * T::ELEM, (int)((row * a.ld + n) * T::ELEM), (int)(T::ROWS * a.ld * T::ELEM),
                a.near && t0 + T::STEP <= end && (t0 + T::STEP - 1) * a.ld + n0 + T::N <= all};
}
template <class T, int P>
__device__ __forceinline__ void fetch_pass(InRegisters<T>& r, const Rows& rows) {
    r.v[P] = *reinterpret_cast<const u32x4_any*>(rows.from + (rows.first + P * rows.next));
}
// A stage that is not whole.
template <class T>
__device__ __forceinline__ void fetch_part(InRegisters<T>& r, const GradArgs& a, int64_t t0, int64_t end, int64_t n0) {
    const int n = (int)(threadIdx.x % T::LANES) * T::VEC, row = (int)(threadIdx.x / T::LANES);
    const int64_t all = (a.tokens - 1) * a.ld + a.out;
    for (int p = 0; p < T::PASSES; ++p) {
        const int64_t t = t0 + p * T::ROWS + row, at = t * a.ld + n0 + n;
        u32x4 v = u32x4{0, 0, 0, 0};
        if (t < end && n0 + n < a.out) {
            const char* from = a.dy + at * T::ELEM;
            const int here = (int)min(all - at, (int64_t)T::VEC);   // fewer than VEC in the last row
            if (here == T::VEC) {
                v = *reinterpret_cast<const u32x4_any*>(from);
            } else {
#pragma unroll
                for (int i = 0; i < T::VEC; ++i) {
                    if (i >= here) continue;
                    if constexpr (T::ELEM == 4) v[i] = reinterpret_cast<const uint32_t*>(from)[i];
                    else v[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(from)[i] << (i % 2 * 16);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < T::PASSES; ++q)
            if (q == p) r.v[q] = v;
    }
}

// The bf16 parts of four fp32 values, highest first, two in a word: each is what the ones before leave, cut off (not rounded) to its
// upper 8 bits, so that nothing is lost in three.
struct Parts {
    u32x2 part[3];
};
__device__ __forceinline__ uint32_t upper_halves(uint32_t low, uint32_t high) { return __builtin_amdgcn_perm(high, low, 0x07060302u); }
__device__ __forceinline__ Parts parts_of(const u32x4& v) {
    u32x4 mid, last;
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = __uint_as_float(v[i]), rest = x - __uint_as_float(v[i] & 0xffff0000u);
        mid[i] = __float_as_uint(rest);
        last[i] = __float_as_uint(rest - __uint_as_float(mid[i] & 0xffff0000u));
        odd = __builtin_fmaf(x, 0.f, odd);
    }
    u32x4 high = v;
    if (__any(odd != odd)) {   // inf and NaN are all in the first part; a NaN whose upper half would read as infinity stays a NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __uint_as_float(v[i]);
            if (!(fabsf(x) < INFINITY)) mid[i] = last[i] = 0u;
            if (x != x) high[i] = 0x7fc00000u;
        }
    }
    return Parts{{u32x2{upper_halves(high[0], high[1]), upper_halves(high[2], high[3])}, u32x2{upper_halves(mid[0], mid[1]), upper_halves(mid[2], mid[3])},
                  u32x2{upper_halves(last[0], last[1]), upper_halves(last[2], last[3])}}};
}

template <class T, int P>
__device__ __forceinline__ void put_pass(lds_char* lds, const InRegisters<T>& r) {
    const int n = (int)(threadIdx.x % T::LANES) * T::VEC, t = P * T::ROWS + (int)(threadIdx.x / T::LANES);
    lds_char* to = lds + t * T::ROW + dy_chunk<T::N>(t, n >> 4) * 32 + (n & 15) * 2;
    if constexpr (T::ELEM == 2) {
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(to) = r.v[P];
    } else {
        const Parts w = parts_of(r.v[P]);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(to + q * T::PLANE) = w.part[q];
    }
}

// 8 kept values as the matrix instruction takes them.
__device__ __forceinline__ bf16x8 widen8(uint32_t low, uint32_t high, float scale) {
    union {
        bf16x2 pair[4];
        bf16x8 all;
    } r;
    r.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false);
    r.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true);
    r.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false);
    r.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true);
    return r.all;
}

// One stage's products.  The instruction sums over 16 tokens, 8 in each half of the wave; which 8 is free as long as both operands agree.
// A lane reads 16 tokens of its column of x at once, tokens 16 o .. 16 o + 15 in half o, and gives the first and then the last
// 8 of them; dy, whose rows are tokens, is read through the transposing load, 4 tokens of 16 columns a time.  `beside(i)` is called with
// i = 0 .. T::GROUPS - 1 among the products.
template <class T, class F>
__device__ __forceinline__ void multiply(lds_char* lds, f32x16 (&sum)[T::NI][T::NJ], int wn, int wk, int lane, F&& beside) {
    const int o = lane >> 5, row = (lane & 15) >> 2, column = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    static_for<0, T::BLOCKS>([&](auto B) {
        constexpr int b = decltype(B)::value;
        u32x4 q[T::NJ];
        float scale[T::NJ];
#pragma unroll
        for (int j = 0; j < T::NJ; ++j) {
            const int k = b * T::K + wk + j * 32 + (lane & 31);
            q[j] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(lds + T::X_AT + k * kActBlock + o * 16);
            scale[j] = __uint_as_float((uint32_t) * reinterpret_cast<const __attribute__((address_space(3))) uint8_t*>(lds + T::E_AT + k) << 23);
        }
        static_for<0, 2>([&](auto H) {
            constexpr int h = decltype(H)::value;
            bf16x8 d[T::PLANES][T::NI];
#pragma unroll
            for (int p = 0; p < T::PLANES; ++p)
#pragma unroll
                for (int i = 0; i < T::NI; ++i) {
                    union {
                        s16x4 half[2];
                        bf16x8 all;
                    } r;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int t = b * kActBlock + o * 16 + h * 8 + e * 4 + row, n = wn + i * 32 + column;
                        r.half[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4*>(
                            lds + p * T::PLANE + t * T::ROW + dy_chunk<T::N>(t, n >> 4) * 32 + (n & 15) * 2));
                    }
                    d[p][i] = r.all;
                }
            static_for<0, T::NJ>([&](auto J) {
                constexpr int j = decltype(J)::value;
                const bf16x8 x = widen8(q[j][2 * h], q[j][2 * h + 1], scale[j]);
#pragma unroll
                for (int p = T::PLANES - 1; p >= 0; --p)   // (the small parts first)
#pragma unroll
                    for (int i = 0; i < T::NI; ++i) sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d[p][i], x, sum[i][j], 0, 0, 0);
                beside(std::integral_constant<int, (b * 2 + h) * T::NJ + j>{});
            });
        });
    });
}

// A wave's results.  Lane -> column (lane & 31), rows 8 (e / 4) + 4 (lane >> 5) + e % 4 of each 32 by 32.  What lies outside of
// dw is beyond the buffer's end, and not written.
enum class Out { F32, AddF32, Bf16, AddBf16 };
template <class T, Out OUT>
__device__ __forceinline__ void write_tile(void* dw, const GradArgs& a, const f32x16 (&sum)[T::NI][T::NJ], int64_t n, int64_t k, int lane) {
    constexpr int BYTES = OUT == Out::F32 || OUT == Out::AddF32 ? 4 : 2;
    const int width = (int)a.width;
#pragma unroll
    for (int x = 0; x < T::NI; ++x)
#pragma unroll
        for (int j = 0; j < T::NJ; ++j) {
            const int64_t base = (n + x * 32) * a.width + k + j * 32;
            const __amdgpu_buffer_rsrc_t to = buffer(reinterpret_cast<char*>(dw) + base * BYTES, block_range(a.out * a.width, base, BYTES));
            const int at = k + j * 32 + (lane & 31) < a.width ? ((lane >> 5) * 4 * width + (lane & 31)) * BYTES : kBlockRange;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int where = at + (8 * (e / 4) + e % 4) * width * BYTES;
                float v = sum[x][j][e];
                if constexpr (OUT == Out::AddF32) v += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(to, where, 0, 0));
                if constexpr (OUT == Out::AddBf16) v += __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b16(to, where, 0, 0) << 16);
                if constexpr (BYTES == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), to, where, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bf16_bits_rne(v), to, where, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);   // (a part at a time: all addresses at once do not fit the registers)
        }
}

// One result of the joining launch.
__device__ __forceinline__ void write_dw(const GradArgs& a, int64_t i, float v) {
    if (a.dw_bf16) {
        uint16_t* dw = reinterpret_cast<uint16_t*>(a.dw);
        if (a.accumulate) v += __uint_as_float((uint32_t)dw[i] << 16);
        dw[i] = (uint16_t)bf16_bits_rne(v);
    } else {
        float* dw = reinterpret_cast<float*>(a.dw);
        dw[i] = a.accumulate ? dw[i] + v : v;
    }
}

// Waits for the loads of this wave but the last `LEFT`, and for its reads of LDS; then for the other waves.
template <int LEFT>
__device__ __forceinline__ void stage_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

template <class T, Dy DY>
__global__ __launch_bounds__(T::THREADS, T::WAVES == 8 ? 2 : (T::NI == 1 ? 4 : 2)) void weight_grad_kernel(const GradArgs a) {
    // (arrays of their own and not one: only so does the compiler know that a stage's loads and another one's reads never meet)
    __shared__ __align__(1024) char stage0[T::BYTES];
    __shared__ __align__(1024) char stage1[T::BYTES];
    __shared__ __align__(1024) char stage2[DY == Dy::Direct ? T::BYTES : 16];
    lds_char *const s0 = (lds_char*)stage0, *const s1 = (lds_char*)stage1, *const s2 = (lds_char*)stage2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go round the 8 dies: each die gets a run of tiles of its own, which go through 8 rows of tiles at a
    // time, so that what its workgroups read together fits its cache.
    const int tiles = a.tiles_n * a.tiles_k, all = tiles * a.parts;
    int id = blockIdx.x;
    if (all % 8 == 0) id = (id & 7) * (all / 8) + (id >> 3);
    const int part = id / tiles;
    id -= part * tiles;
    constexpr int GROUP = 8;
    const int first = id / (GROUP * a.tiles_k) * GROUP, rows = min(GROUP, a.tiles_n - first);
    id -= first * a.tiles_k;
    const int64_t n0 = (int64_t)(first + id % rows) * T::N, k0 = (int64_t)(id / rows) * T::K;
    const int wn = wave / T::WAVES_OF_K * T::NI * 32, wk = wave % T::WAVES_OF_K * T::NJ * 32;

    const int all_steps = (int)((a.tokens + T::STEP - 1) / T::STEP);
    const int from = (int)((int64_t)all_steps * part / a.parts), to = (int)((int64_t)all_steps * (part + 1) / a.parts);
    int steps = to - from;
    f32x16 sum[T::NI][T::NJ] = {};
    if (steps > 0) {
        const Sources<T, DY> sources(a, wave, lane);
        const int64_t t0 = (int64_t)from * T::STEP, end = min((int64_t)to * T::STEP, a.tokens);
        Cursor cursor{a.dy + (t0 * a.ld + n0) * T::ELEM, a.kept + (t0 / kActBlock * a.columns + k0) * kActBlock,
                      a.exponents + t0 / kActBlock * a.columns + k0, (int)(end - t0)};
        auto load = [&](lds_char* s) { load_stage<T, DY>(s, a, sources, cursor, n0, k0, wave); };
        if constexpr (DY == Dy::Direct) {
            // Three stages: while one is worked on the loads of the next are under way and those of the one after it start.
            constexpr int LOADS = T::DY_LOADS + T::X_LOADS + 1;
            load(s0);
            load(s1);
            auto step = [&](lds_char* now, lds_char* after) {
                stage_barrier<LOADS>();
                load(after);
                multiply<T>(now, sum, wn, wk, lane, [](auto) {});
            };
            for (; steps >= 3; steps -= 3) {
                step(s0, s2);
                step(s1, s0);
                step(s2, s1);
            }
            if (steps > 0) step(s0, s2);
            if (steps > 1) step(s1, s0);
        } else {
            // Two stages: dy of the next one lies in registers when a stage begins.  A pass of it is put away, and the stage after it
            // asked for, behind each of the first groups of products: the vector instructions that cut fp32 into parts then run beside the
            // matrix instructions and not in front of them (16384 x 4096 x 4096, fp32: 1378 -> 1231 us, 1.34 PFLOP/s of bf16 products).
            InRegisters<T> r;
            int64_t t = t0;
            auto fetch = [&] {
                const Rows rows = rows_at<T>(a, t, end, n0);
                if (rows.whole) static_for<0, T::PASSES>([&](auto P) { fetch_pass<T, decltype(P)::value>(r, rows); });
                else fetch_part<T>(r, a, t, end, n0);
            };
            fetch();
            load(s0);
            static_for<0, T::PASSES>([&](auto P) { put_pass<T, decltype(P)::value>(s0, r); });
            t += T::STEP;
            fetch();
            constexpr int EACH = (T::PASSES + T::GROUPS - 1) / T::GROUPS;   // passes behind a group
            auto step = [&](lds_char* now, lds_char* next) {
                stage_barrier<0>();
                load(next);
                t += T::STEP;
                const Rows rows = rows_at<T>(a, t, end, n0);
                multiply<T>(now, sum, wn, wk, lane, [&](auto I) {
                    constexpr int from = std::min(decltype(I)::value * EACH, T::PASSES), to = std::min(from + EACH, T::PASSES);
                    static_for<from, to>([&](auto P) {
                        __builtin_amdgcn_sched_barrier(0);
                        put_pass<T, decltype(P)::value>(next, r);
                        if (rows.whole) fetch_pass<T, decltype(P)::value>(r, rows);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                });
                if (!rows.whole) fetch_part<T>(r, a, t, end, n0);
            };
            for (; steps >= 2; steps -= 2) {
                step(s0, s1);
                step(s1, s0);
            }
            if (steps > 0) step(s0, s1);
        }
    }
    if (a.partial) write_tile<T, Out::F32>(a.partial + part * a.out * a.width, a, sum, n0 + wn, k0 + wk, lane);
    else if (a.dw_bf16 && a.accumulate) write_tile<T, Out::AddBf16>(a.dw, a, sum, n0 + wn, k0 + wk, lane);
    else if (a.dw_bf16) write_tile<T, Out::Bf16>(a.dw, a, sum, n0 + wn, k0 + wk, lane);
    else if (a.accumulate) write_tile<T, Out::AddF32>(a.dw, a, sum, n0 + wn, k0 + wk, lane);
    else write_tile<T, Out::F32>(a.dw, a, sum, n0 + wn, k0 + wk, lane);
}

// The parts' sums, joined in order.
__global__ __launch_bounds__(kBlock) void weight_grad_join_kernel(const GradArgs a) {
    const int64_t total = a.out * a.width;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < total; i += (int64_t)gridDim.x * kBlock) {
        float v = 0.f;
        for (int p = 0; p < a.parts; ++p) v += a.partial[p * total + i];
        write_dw(a, i, v);
    }
}

template <int WAVES_N, int WAVES_K, int NI, int NJ>
hipError_t launch_tile(GradArgs a, Dy dy, hipStream_t stream) {
    typedef Tile<WAVES_N, WAVES_K, NI, NJ, Dy::Direct> Direct;
    typedef Tile<WAVES_N, WAVES_K, NI, NJ, Dy::Bf16> Bf16;
    typedef Tile<WAVES_N, WAVES_K, NI, NJ, Dy::F32> F32;
    a.tiles_n = (int)((a.out + Direct::N - 1) / Direct::N);
    a.tiles_k = (int)((a.width + Direct::K - 1) / Direct::K);
    const unsigned grid = (unsigned)(a.tiles_n * a.tiles_k * a.parts);
    if (dy == Dy::Direct) weight_grad_kernel<Direct, Dy::Direct><<<grid, Direct::THREADS, 0, stream>>>(a);
    else if (dy == Dy::Bf16) weight_grad_kernel<Bf16, Dy::Bf16><<<grid, Bf16::THREADS, 0, stream>>>(a);
    else weight_grad_kernel<F32, Dy::F32><<<grid, F32::THREADS, 0, stream>>>(a);
    return hipGetLastError();
}

// The tile of a call (its edge) and the parts that its tokens are cut into: whichever is the least by this account of what a
// launch takes.  A workgroup alone on its compute unit takes `alone` microseconds for 64 tokens, a unit full of them
// `full` for each of them; the two differ most for the small tiles, whose steps are latency, and least for the large
// one, of which a unit holds one.  Joining parts costs a launch and two passes over their sums.  The figures, of launches
// with 1 to 16 parts on 11 shapes of 1 to 32768 tokens, predict the best of them or one within 15 % of it; bf16 rows that do
// not lie on 16-byte addresses take longer (1.3 to 1.9 times) in much the same proportions.
// (16384 x 8192 x 8192, tiles of 256 / 128: 1700 / 1992 us; 4096 x 2048 x 4096, 256 / 128 / 64: 82 / 68 / 100 us; 16000 x
// 1024 x 1024, 128 with 1 / 4 / 8 / 16 parts: 121 / 46 / 42 / 49 us; dy in fp32, 4096 x 2048 x 4096, 256 with 1 / 2 / 4 parts: 288 / 188 /
// 213 us, 128: 207 / 225 / 239, 64 with 1: 298; 1000 x 1024 x 1000, 64 with 1 / 2 parts: 23 / 23, 128 with 1 / 2 / 4: 45 / 28 / 25.)
struct Choice {
    int tile, parts;
};
Choice choose(int dy_dtype, int64_t tokens, int64_t out, int64_t width) {
    struct Cost {
        int tile, held;   // workgroups that a unit holds
        double alone, full;
    };
    static constexpr Cost bf16[3] = {{256, 1, 1.16, 1.66}, {128, 2, 0.48, 0.47}, {64, 4, 0.54, 0.18}};
    static constexpr Cost f32[3] = {{256, 1, 4.5, 4.8}, {128, 2, 2.6, 1.65}, {64, 4, 1.35, 0.57}};
    constexpr double kUnits = 256, kJoin = 5.0, kBytesPerUs = 5e6;
    const int64_t steps = (tokens + 63) / 64;
    Choice best{64, 1};
    double least = 1e300;
    for (const Cost& c : dy_dtype == STAR_F32 ? f32 : bf16) {
        const double tiles = (double)((out + c.tile - 1) / c.tile) * (double)((width + c.tile - 1) / c.tile);
        for (int parts = 1; parts <= 64 && (parts == 1 || 2 * parts <= steps); parts *= 2) {
            const double sums = (double)parts * (double)out * (double)width * sizeof(float);
            if (parts > 1 && sums > (double)(1 << 29)) break;
            const double n = tiles * parts / kUnits, load = c.held == 1 ? std::ceil(n) * (n > 0.5 ? c.full : c.alone) : n * c.full;
            const double took = (double)((steps + parts - 1) / parts) * std::max(c.alone, load) + (parts > 1 ? kJoin + 2 * sums / kBytesPerUs : 0.0);
            if (took < least) {
                least = took;
                best = Choice{c.tile, parts};
            }
        }
    }
    return best;
}

hipError_t launch_choice(const WeightGrad& g, const Choice& c, void* workspace, hipStream_t stream) {
    GradArgs a{};
    a.dy = reinterpret_cast<const char*>(g.dy);
    a.columns = act_columns(g.width);
    a.kept = reinterpret_cast<const uint8_t*>(g.packed);
    a.exponents = a.kept + act_blocks(g.tokens) * a.columns * kActBlock;
    a.dw = g.dw;
    a.tokens = g.tokens;
    a.out = g.out;
    a.ld = g.ld;
    a.width = g.width;
    a.parts = c.parts;
    a.partial = c.parts > 1 ? reinterpret_cast<float*>(workspace) : nullptr;
    a.dw_bf16 = g.dw_dtype == STAR_BF16;
    a.accumulate = g.accumulate;
    a.near = g.ld < (1 << 23);
    // straight to LDS: whole 16 bytes at addresses of 16
    const bool direct = g.dy_dtype == STAR_BF16 && reinterpret_cast<uintptr_t>(g.dy) % 16 == 0 && g.ld % 8 == 0 && a.near;
    const Dy dy = g.dy_dtype == STAR_F32 ? Dy::F32 : (direct ? Dy::Direct : Dy::Bf16);
    hipError_t e = c.tile == 256 ? launch_tile<4, 2, 2, 4>(a, dy, stream)
                                 : (c.tile == 128 ? launch_tile<2, 2, 2, 2>(a, dy, stream) : launch_tile<2, 2, 1, 1>(a, dy, stream));
    if (e == hipSuccess && a.partial) {
        weight_grad_join_kernel<<<(unsigned)std::min<int64_t>(2048, (g.out * g.width + kBlock - 1) / kBlock), kBlock, 0, stream>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int weight_grad_parts(int dy_dtype, int64_t tokens, int64_t out, int64_t width) { return choose(dy_dtype, tokens, out, width).parts; }

hipError_t launch_weight_grad(const WeightGrad& g, void* workspace, hipStream_t stream) {
    return launch_choice(g, choose(g.dy_dtype, g.tokens, g.out, g.width), workspace, stream);
}

}  // namespace star
