// Activations kept in 8 bits for the backward pass: blocks of 32 tokens of one column share a power of two.
//
// The block runs along the tokens because the weight gradient sums over them: one lane of a matrix instruction holds
// 8 tokens of one column, so that a block has one scale a lane, and the 32 bytes of a column lie together, in the order in
// which the instruction takes them (star_act_grad_kernels.hip).  A power of two leaves the mantissa as it is: every kept value
// is a bf16 number, and outlier columns, the usual shape of activations, spoil no neighbour.
#include <hip/hip_runtime.h>

#include "star_device.h"
#include "star_worker.h"

namespace star {

namespace {

constexpr float kE4m3Max = 448.f;
constexpr int kLeastExponent = -117;   // 2^-9 * 2^-117, the least kept value, is still a normal number of bf16
constexpr float kMostKept = 0x1.ep127f;   // 240 * 2^120: the next kept value would be 2^128

// Smallest e >= kLeastExponent with most <= 448 * 2^e (most finite, not negative).
__device__ __forceinline__ int block_exponent(float most) {
    // 448 = 1.75 * 2^8: with most = f * 2^x, 1 <= f < 2, it is x - 8, one more if f > 1.75
    const uint32_t b = __float_as_uint(most);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kLeastExponent ? kLeastExponent : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

__device__ __forceinline__ float load_x(const float* x, int64_t i) { return x[i]; }
__device__ __forceinline__ float load_x(const uint16_t* x, int64_t i) { return __uint_as_float((uint32_t)x[i] << 16); }
__device__ __forceinline__ void store_x(float* x, int64_t i, float v) { x[i] = v; }
__device__ __forceinline__ void store_x(uint16_t* x, int64_t i, float v) { x[i] = (uint16_t)(__float_as_uint(v) >> 16); }   // (exact)

// 4 kept values of scale 1 / inverse; |x| <= 448 / inverse, or not finite.
__device__ __forceinline__ uint32_t keep4(const float* x, float inverse) {
    float v[4];
    for (int i = 0; i < 4; ++i) {
        const float bounded = fminf(fmaxf(x[i], -kMostKept), kMostKept);
        v[i] = fabsf(x[i]) < INFINITY ? bounded * inverse : NAN;
    }
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], low, true);
}

struct ActShape {
    int64_t tokens, width, ld, columns, items, first;   // items: blocks * columns, what a launch begins with
};

// A wave makes one block of 64 columns: it reads rows, 16 bytes a lane, turns them through LDS (which no other wave touches, so that nobody
// waits), and every lane keeps one column, whose 32 bytes lie beside its neighbour's.  Bound by memory; a thread a column, without LDS, read
// 2 bytes a lane and took three times as long (16381 x 4096, bf16: 109 us, now 37 -- 5.5 TB/s).
constexpr int kPackColumns = 64;
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void act_pack_kernel(const T* x, uint8_t* packed, const ActShape s) {
    constexpr int VEC = 16 / sizeof(T), LANES = kPackColumns / VEC, ROWS = 64 / LANES, LOADS = kActBlock / ROWS;
    __shared__ __align__(16) T rows[THREADS / 64][kActBlock][kPackColumns];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t groups = (s.columns + kPackColumns - 1) / kPackColumns, blocks = s.items / s.columns;
    const int64_t item = s.first + (int64_t)blockIdx.x * (THREADS / 64) + wave, b = item / groups, c0 = (item - b * groups) * kPackColumns;
    if (b >= blocks) return;
    typedef u32x4 u32x4_any __attribute__((aligned(2)));
    const int64_t all = (s.tokens - 1) * s.ld + s.width;   // elements up to the last one
    u32x4 v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int64_t t = b * kActBlock + i * ROWS + lane / LANES, c = c0 + lane % LANES * VEC, at = t * s.ld + c;
        v[i] = u32x4{0, 0, 0, 0};
        if (t < s.tokens && c < s.width) {
            if (at + VEC <= all) {   // (what is beyond the row's end is dropped below)
                v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(x + at));
            } else {
                union {
                    T e[VEC];
                    u32x4 all;
                } part = {};
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (at + j < all) part.e[j] = x[at + j];
                v[i] = part.all;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) *reinterpret_cast<u32x4*>(&rows[wave][i * ROWS + lane / LANES][lane % LANES * VEC]) = v[i];
    // (the wave's own reads follow its writes, also for the compiler; the hardware takes one wave's LDS accesses in order)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int64_t c = c0 + lane;
    float column[kActBlock], most = 0.f;
#pragma unroll
    for (int i = 0; i < kActBlock; ++i) {
        column[i] = c < s.width ? load_x(&rows[wave][i][0], lane) : 0.f;
        const float size = fabsf(column[i]);
        most = fmaxf(most, size < INFINITY ? size : 0.f);
    }
    if (c >= s.columns) return;
    const int e = block_exponent(most);
    const float inverse = power_of_two(-e);
    u32x4* to = reinterpret_cast<u32x4*>(packed + (b * s.columns + c) * kActBlock);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        to[h] = u32x4{keep4(column + 16 * h, inverse), keep4(column + 16 * h + 4, inverse), keep4(column + 16 * h + 8, inverse),
                      keep4(column + 16 * h + 12, inverse)};
    packed[s.items * kActBlock + b * s.columns + c] = c < s.width ? (uint8_t)(e + 127) : 0;
}

// Columns of blocks are numbered through, [B][C] as they lie in the packed form: a thread each, from `first` on.
template <class T>
__global__ __launch_bounds__(kBlock) void act_unpack_kernel(const uint8_t* packed, T* out, const ActShape s) {
    const int64_t item = s.first + (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (item >= s.items) return;
    const int64_t b = item / s.columns, c = item - b * s.columns;
    if (c >= s.width) return;
    const u32x4* from = reinterpret_cast<const u32x4*>(packed + item * kActBlock);
    const u32x4 q[2] = {from[0], from[1]};
    const float scale = power_of_two((int)packed[s.items * kActBlock + item] - 127);
    static_for<0, kActBlock>([&](auto I) {
        constexpr int i = decltype(I)::value;
        const int64_t t = b * kActBlock + i;
        if (t < s.tokens) store_x(out, t * s.ld + c, __builtin_amdgcn_cvt_f32_fp8((int)q[i / 16][i / 4 % 4], i % 4) * scale);
    });
}

// A launch holds fewer than 2^32 threads: what is beyond goes into further ones.  `launch(shape, workgroups)` for runs of `a_group` items of
// `items`.
template <class F>
hipError_t in_launches(ActShape s, int64_t items, int a_group, F&& launch) {
    constexpr int64_t kGroups = (int64_t)1 << 22;
    for (s.first = 0; s.first < items; s.first += kGroups * a_group) {
        launch(s, (unsigned)std::min(kGroups, (items - s.first + a_group - 1) / a_group));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

ActShape act_shape(int64_t tokens, int64_t width, int64_t ld) {
    return ActShape{tokens, width, ld, act_columns(width), act_blocks(tokens) * act_columns(width), 0};
}

template <class T>
hipError_t pack(const T* x, uint8_t* to, const ActShape& s, hipStream_t stream) {
    const int64_t waves = s.items / s.columns * ((s.columns + kPackColumns - 1) / kPackColumns);
    // (a wave a workgroup while there are few: they then spread over all units)
    if (waves <= 2048)
        return in_launches(s, waves, 1, [&](const ActShape& r, unsigned grid) { act_pack_kernel<T, 64><<<grid, 64, 0, stream>>>(x, to, r); });
    return in_launches(s, waves, 4, [&](const ActShape& r, unsigned grid) { act_pack_kernel<T, 256><<<grid, 256, 0, stream>>>(x, to, r); });
}

}  // namespace

hipError_t launch_act_pack(const void* x, int dtype, int64_t tokens, int64_t width, int64_t ld, void* packed, hipStream_t stream) {
    const ActShape s = act_shape(tokens, width, ld);
    uint8_t* to = reinterpret_cast<uint8_t*>(packed);
    return dtype == STAR_F32 ? pack(reinterpret_cast<const float*>(x), to, s, stream) : pack(reinterpret_cast<const uint16_t*>(x), to, s, stream);
}

hipError_t launch_act_unpack(const void* packed, int64_t tokens, int64_t width, void* out, int dtype, int64_t ld, hipStream_t stream) {
    const uint8_t* from = reinterpret_cast<const uint8_t*>(packed);
    const ActShape shape = act_shape(tokens, width, ld);
    return in_launches(shape, shape.items, kBlock, [&](const ActShape& s, unsigned grid) {
        if (dtype == STAR_F32)
            act_unpack_kernel<float><<<grid, kBlock, 0, stream>>>(from, reinterpret_cast<float*>(out), s);
        else
            act_unpack_kernel<uint16_t><<<grid, kBlock, 0, stream>>>(from, reinterpret_cast<uint16_t*>(out), s);
    });
}

}  // namespace star
