// Launch interface of the worker-side operators: loss on logits, activations in 8 bits, weight gradient.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "star.h"

namespace star {

// What the C-ABI layer of these operators shares with that of the group update.
star_status set_error(star_status s, const char* text);
star_status hip_error(hipError_t e, const char* what);

// ---------------------------------------------------------------- logits
struct Logits {
    const void* x;
    int dtype;             // star_dtype
    int64_t tokens, vocab, ld;
    const int64_t* targets;
    const float* weights;  // null: all 1; a token of weight 0 does not count
    float inv_t, inv_t_low;   // 1 / temperature, and what rounding it left
    float k;                  // log2(e) / temperature
};

struct PolicyArgs {
    const float *old_logp, *ref_logp, *advantages;
    float scale, low, high, kl;   // ratio held within [low, high]
};

// Workspace bytes of the launches below.
size_t logprobs_workspace(int dtype, int64_t tokens, int64_t vocab);
size_t policy_workspace(int dtype, int64_t tokens, int64_t vocab);

// A row's maximum m and sum of 2^((l_j - m) k).
struct MaxSum {
    float m, s;
};
// logp, lse (may be null) of rows [first, first + count).  Without a workspace a row is one workgroup's.
// `logp_low`, if not null: what rounding the log-probabilities to `logp` left.  `sums`, if not null: the rows' maxima and sums, for the gradient.
// `again`: the gradient will read the logits once more soon.
hipError_t launch_logprobs(const Logits& l, int64_t first, int64_t count, float* logp, float* logp_low, float* lse, MaxSum* sums, bool again,
                           void* workspace, hipStream_t stream);
// The loss of pairs from their terms (one double each).
struct PairLoss {
    const double* terms;
    int pairs;
    float scale;
    float* out;
};
// dlogits of rows [first, first + count) from dlogp and the rows' maxima and sums or, where there are none, lse; with a loss whose `out` is not
// null, that too.
hipError_t launch_logprobs_grad(const Logits& l, int64_t first, int64_t count, const float* lse, const MaxSum* sums, const float* dlogp,
                                void* dlogits, int64_t ld_out, const PairLoss& loss, hipStream_t stream);
// logp (may be null), dlogits (may be null) and the four sums of the policy loss.
hipError_t launch_policy(const Logits& l, const PolicyArgs& a, float* logp, void* dlogits, int64_t ld_out, float* stats, void* workspace,
                         hipStream_t stream);

// Pairs of one launch: their offsets travel in the kernel arguments.
constexpr int kPairsPerLaunch = 128;
struct PairOffsets {
    int64_t at[2 * kPairsPerLaunch + 1];
};
struct PreferenceArgs {
    const float* ref_logp;
    float scale, beta, smooth;
};
// Margins of `pairs` pairs, their tokens' derivatives and the terms of the loss (one double a pair).
hipError_t launch_pairs(const Logits& l, const PreferenceArgs& a, const PairOffsets& offsets, int pairs, const float* logp,
                        const float* logp_low, float* dlogp, float* margins, double* terms, hipStream_t stream);
hipError_t launch_pair_loss(const PairLoss& loss, hipStream_t stream);

// ---------------------------------------------------------------- saved activations
constexpr int kActBlock = 32;    // tokens that share a scale
constexpr int kActPad = 16;      // columns of the packed form come in multiples of this
inline int64_t act_blocks(int64_t tokens) { return (tokens + kActBlock - 1) / kActBlock; }
inline int64_t act_columns(int64_t width) { return (width + kActPad - 1) / kActPad * kActPad; }

hipError_t launch_act_pack(const void* x, int dtype, int64_t tokens, int64_t width, int64_t ld, void* packed, hipStream_t stream);
hipError_t launch_act_unpack(const void* packed, int64_t tokens, int64_t width, void* out, int dtype, int64_t ld, hipStream_t stream);

// ---------------------------------------------------------------- weight gradient
struct WeightGrad {
    const void* dy;
    int dy_dtype;
    int64_t tokens, out, ld;
    const void* packed;
    int64_t width;
    void* dw;
    int dw_dtype;
    bool accumulate;
};
// What a 32 by 32 block of results, whose first element is `base`, may write of a matrix of `elements`: bytes from there to the end, none for a
// block that begins behind it (by up to 223 rows, which at the widest do not fit 31 bits), and no more than a block can reach.  What a block must
// not write lies at kBlockRange or beyond.
constexpr int kBlockRange = 0x40000000;
constexpr int block_range(int64_t elements, int64_t base, int bytes) {
    const int64_t left = elements - base;
    return left <= 0 ? 0 : (left >= kBlockRange / bytes ? kBlockRange : (int)left * bytes);
}

// Parts that the tokens are cut into (each part's sums are written apart and joined by a second launch; 1: none).
int weight_grad_parts(int dy_dtype, int64_t tokens, int64_t out, int64_t width);
hipError_t launch_weight_grad(const WeightGrad& g, void* workspace, hipStream_t stream);

}  // namespace star
