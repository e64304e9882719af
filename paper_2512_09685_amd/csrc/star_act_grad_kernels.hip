// Weight gradient from activations kept in 8 bits: dw[n][k] = sum_t dy[t][n] x[t][k].
//
// The kept values are e4m3 * 2^e and with that bf16 numbers, so the matrix instructions for bf16 take them without a rounding;
// one conversion instruction makes two of them, scale and all.  dy in fp32 is cut into three bf16 parts of 8 bits each, whose
// products are all exact: the sums, in fp32, are the only place where anything is rounded before the result.
#include <hip/hip_runtime.h>

#include "star_device.h"
#include "star_worker.h"

namespace star {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Tile of dw that a workgroup makes: kTileN rows (columns of dy) by kTileK columns (of x), in steps of 32 tokens -- one scale
// block, and the depth of one matrix instruction.
constexpr int kTileN = 128, kTileK = 128;
// Bytes from one column of dy to the next in LDS: 32 tokens and 16 bytes, so that the 16 columns that one read takes start on
// different banks.
constexpr int kColumnBytes = 32 * 2 + 16;

struct GradArgs {
    const void* dy;
    const uint8_t* packed;
    void* dw;
    float* partial;      // sums of this launch's parts, [parts][out][width]; null: one part, straight to dw
    int64_t tokens, out, ld, width, columns, blocks;
    int parts;
    int dw_bf16, accumulate;
};

// 8 kept values as the matrix instruction takes them.
__device__ __forceinline__ bf16x8 widen8(const u32x2 q, float scale) {
    union {
        bf16x2 pair[4];
        bf16x8 all;
    } r;
    r.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[0], scale, false);
    r.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[0], scale, true);
    r.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[1], scale, false);
    r.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[1], scale, true);
    return r.all;
}

// The bf16 parts of a value of dy, highest first.  fp32: each part is what the ones before leave, cut off (not rounded) to
// its 8 upper bits; inf and NaN are all in the first.
template <int PARTS>
struct DyParts {
    uint32_t part[PARTS];
};
__device__ __forceinline__ DyParts<1> dy_parts(const uint16_t* dy, int64_t i) { return DyParts<1>{{dy[i]}}; }
__device__ __forceinline__ DyParts<3> dy_parts(const float* dy, int64_t i) {
    const float v = dy[i];
    const uint32_t high = __float_as_uint(v) & 0xffff0000u;
    const bool finite = fabsf(v) < INFINITY;
    const float rest = finite ? v - __uint_as_float(high) : 0.f;
    const uint32_t mid = __float_as_uint(rest) & 0xffff0000u;
    const float last = rest - __uint_as_float(mid);
    // (a NaN whose upper half reads as infinity stays a NaN)
    const uint32_t first = v != v ? 0x7fc0u : high >> 16;
    return DyParts<3>{{first, mid >> 16, __float_as_uint(last) >> 16}};
}

__device__ __forceinline__ void write_dw(const GradArgs& a, int64_t n, int64_t k, float v) {
    const int64_t i = n * a.width + k;
    if (a.dw_bf16) {
        uint16_t* dw = reinterpret_cast<uint16_t*>(a.dw);
        if (a.accumulate) v += __uint_as_float((uint32_t)dw[i] << 16);
        dw[i] = (uint16_t)bf16_bits_rne(v);
    } else {
        float* dw = reinterpret_cast<float*>(a.dw);
        dw[i] = a.accumulate ? dw[i] + v : v;
    }
}

// 4 waves, each 64 by 64 of the tile.  Any address, any size: dy goes through registers, every element of it checked.
template <class T>
__global__ __launch_bounds__(kBlock) void weight_grad_kernel(const GradArgs a) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    __shared__ __align__(16) char columns_lds[PARTS][kTileN * kColumnBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tiles_k = (a.width + kTileK - 1) / kTileK, tiles_n = (a.out + kTileN - 1) / kTileN;
    const int64_t tile = blockIdx.x % (tiles_k * tiles_n), part = blockIdx.x / (tiles_k * tiles_n);
    const int64_t n0 = tile / tiles_k * kTileN, k0 = tile % tiles_k * kTileK;
    const int wn = (wave >> 1) * 64, wk = (wave & 1) * 64;
    const int64_t b_from = a.blocks * part / a.parts, b_to = a.blocks * (part + 1) / a.parts;
    const T* dy = reinterpret_cast<const T*>(a.dy);
    f32x4 sum[4][4] = {};

    // staging: thread -> two tokens (2 p, 2 p + 1) of 8 columns
    const int pair = tid >> 4, column8 = (tid & 15) * 8;
    for (int64_t b = b_from; b < b_to; ++b) {
        __syncthreads();
        const int64_t t = b * kActBlock + 2 * pair;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t n = n0 + column8 + i;
            DyParts<PARTS> even{}, odd{};
            if (n < a.out) {
                if (t < a.tokens) even = dy_parts(dy, t * a.ld + n);
                if (t + 1 < a.tokens) odd = dy_parts(dy, (t + 1) * a.ld + n);
            }
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
                *reinterpret_cast<uint32_t*>(columns_lds[p] + (column8 + i) * kColumnBytes + pair * 4) = even.part[p] | (odd.part[p] << 16);
        }
        // x: lane -> column (lane & 15) of each 16, tokens 8 (lane >> 4) .. + 7
        bf16x8 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int64_t k = k0 + wk + j * 16 + (lane & 15);
            if (k >= a.columns) k = a.columns - 1;   // (what it makes is not written)
            const int64_t item = b * a.columns + k;
            const u32x2 q = *reinterpret_cast<const u32x2*>(a.packed + item * kActBlock + (lane >> 4) * 8);
            const uint32_t e = a.packed[a.blocks * a.columns * kActBlock + item];
            x[j] = widen8(q, __uint_as_float(e << 23));
        }
        __syncthreads();
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 d = *reinterpret_cast<const bf16x8*>(columns_lds[p] + (wn + i * 16 + (lane & 15)) * kColumnBytes + (lane >> 4) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(d, x[j], sum[i][j], 0, 0, 0);
            }
    }
    // lane -> column (lane & 15), rows 4 (lane >> 4) .. + 3 of each 16 by 16
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + wn + i * 16 + (lane >> 4) * 4 + r, k = k0 + wk + j * 16 + (lane & 15);
                if (n >= a.out || k >= a.width) continue;
                if (a.partial) a.partial[(part * a.out + n) * a.width + k] = sum[i][j][r];
                else write_dw(a, n, k, sum[i][j][r]);
            }
}

// The parts' sums, joined in order.
__global__ __launch_bounds__(kBlock) void weight_grad_join_kernel(const GradArgs a) {
    const int64_t total = a.out * a.width;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < total; i += (int64_t)gridDim.x * kBlock) {
        float v = 0.f;
        for (int p = 0; p < a.parts; ++p) v += a.partial[p * total + i];
        write_dw(a, 0, i, v);
    }
}

}  // namespace

int weight_grad_parts(int, int64_t tokens, int64_t out, int64_t width) {
    const int64_t tiles = ((out + kTileN - 1) / kTileN) * ((width + kTileK - 1) / kTileK), blocks = act_blocks(tokens);
    if (tiles == 0 || blocks == 0) return 1;
    // two workgroups a compute unit, at least 8 blocks each
    return (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, blocks / 8));
}

hipError_t launch_weight_grad(const WeightGrad& g, void* workspace, hipStream_t stream) {
    GradArgs a{};
    a.dy = g.dy;
    a.packed = reinterpret_cast<const uint8_t*>(g.packed);
    a.dw = g.dw;
    a.tokens = g.tokens;
    a.out = g.out;
    a.ld = g.ld;
    a.width = g.width;
    a.columns = act_columns(g.width);
    a.blocks = act_blocks(g.tokens);
    a.parts = weight_grad_parts(g.dy_dtype, g.tokens, g.out, g.width);
    a.partial = a.parts > 1 ? reinterpret_cast<float*>(workspace) : nullptr;
    a.dw_bf16 = g.dw_dtype == STAR_BF16;
    a.accumulate = g.accumulate;
    const int64_t tiles = ((g.out + kTileN - 1) / kTileN) * ((g.width + kTileK - 1) / kTileK);
    const unsigned grid = (unsigned)(tiles * a.parts);
    if (g.dy_dtype == STAR_F32) weight_grad_kernel<float><<<grid, kBlock, 0, stream>>>(a);
    else weight_grad_kernel<uint16_t><<<grid, kBlock, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.partial) {
        weight_grad_join_kernel<<<(unsigned)std::min<int64_t>(2048, (g.out * g.width + kBlock - 1) / kBlock), kBlock, 0, stream>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace star
