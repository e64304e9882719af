// C-ABI layer of the worker-side operators: argument checks and launches.  Nothing here allocates or throws.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "star.h"
#include "star_worker.h"

namespace {

using star::set_error;

constexpr int64_t kMostRows = (int64_t)1 << 22;     // rows of one launch: fewer than 2^32 threads
constexpr int64_t kMostVocab = (int64_t)1 << 30;
constexpr int64_t kMostElements = (int64_t)1 << 42;   // of one tensor: no byte offset leaves 63 bits
constexpr int64_t kMostTiles = (int64_t)1 << 22;      // of dw, 64 by 64 each
constexpr int64_t kMostSummed = (int64_t)1 << 30;     // tokens that one weight gradient sums over
constexpr int64_t kMostWidth = (int64_t)1 << 22;      // columns of a weight gradient: 32 rows of it stay within kBlockRange
constexpr int64_t kCacheBytes = (int64_t)1 << 28;     // of the memory-side cache

bool known(int dtype) { return dtype == STAR_F32 || dtype == STAR_BF16; }
size_t bytes_of(int dtype) { return dtype == STAR_F32 ? 4 : 2; }
bool on_grid(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Whether log-probabilities written to `out` would be written over `in`, both `tokens` floats: inputs are read again behind them.
bool over(const float* out, const float* in, int64_t tokens) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(in), bytes = sizeof(float) * (uintptr_t)tokens;
    return out && in && (a < b ? b - a : a - b) < bytes;
}

// `rows` rows of `length` values, `ld` apart: no size negative, no offset beyond 63 bits.
bool rows_fit(int64_t rows, int64_t length, int64_t ld) {
    return rows >= 0 && length >= 0 && ld >= length && ld <= kMostElements && (rows == 0 || ld == 0 || rows <= kMostElements / ld);
}

star_status check_workspace(const void* workspace, size_t have, size_t need) {
    if (need == 0) return STAR_OK;
    if (!workspace) return set_error(STAR_ERR_NULL, "workspace is NULL");
    if (have < need) return set_error(STAR_ERR_SHAPE, "workspace is too small");
    if (!on_grid(workspace, 16)) return set_error(STAR_ERR_SHAPE, "workspace is not aligned to 16 bytes");
    return STAR_OK;
}

// The checks that all calls on logits share.
star_status check_logits(const void* logits, int dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets, float temperature,
                         const void* dlogits, int64_t ld_out) {
    if (!known(dtype)) return set_error(STAR_ERR_DTYPE, "unknown dtype of the logits");
    if (tokens < 0 || tokens > kMostRows) return set_error(STAR_ERR_SHAPE, "tokens is negative or above 2^22");
    if (vocab < 1 || vocab > kMostVocab) return set_error(STAR_ERR_SHAPE, "vocab is below 1 or above 2^30");
    if (!rows_fit(tokens, vocab, ld)) return set_error(STAR_ERR_SHAPE, "ld is below vocab, or the logits are too large");
    if (dlogits && !rows_fit(tokens, vocab, ld_out)) return set_error(STAR_ERR_SHAPE, "ld_out is below vocab, or the gradient is too large");
    if (!(temperature >= 1e-4f && temperature <= 1e4f)) return set_error(STAR_ERR_HPARAM, "temperature must lie in 1e-4 to 1e4");
    if (tokens == 0) return STAR_OK;
    if (!logits || !targets) return set_error(STAR_ERR_NULL, "logits or targets is NULL");
    if (!on_grid(logits, bytes_of(dtype)) || !on_grid(dlogits, bytes_of(dtype)) || !on_grid(targets, 8))
        return set_error(STAR_ERR_SHAPE, "an address is not a multiple of its element's size");
    if (dlogits == logits && dlogits && ld != ld_out) return set_error(STAR_ERR_SHAPE, "a gradient in place needs ld_out == ld");
    return STAR_OK;
}

star::Logits make_logits(const void* x, int dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets, const float* weights,
                         float temperature) {
    const double inverse = 1.0 / (double)temperature;
    const float rounded = (float)inverse;
    return star::Logits{x, dtype, tokens, vocab, ld, targets, weights, rounded, (float)(inverse - rounded), (float)(1.4426950408889634 * inverse)};
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// Workspace of the preference loss: terms [pairs] double, then sums [tokens] MaxSum, dlogp, logp, logp_low [tokens] float, then that of the
// log-probabilities.
struct PreferenceSpace {
    size_t terms, sums, dlogp, logp, logp_low, rows, total;
};
PreferenceSpace preference_space(int dtype, int64_t tokens, int64_t vocab, int32_t pairs) {
    PreferenceSpace s;
    const size_t each = round16(sizeof(float) * (size_t)tokens);
    s.terms = 0;
    s.sums = round16(sizeof(double) * (size_t)pairs);
    s.dlogp = s.sums + round16(sizeof(star::MaxSum) * (size_t)tokens);
    s.logp = s.dlogp + each;
    s.logp_low = s.logp + each;
    s.rows = s.logp_low + each;
    s.total = s.rows + round16(star::logprobs_workspace(dtype, tokens, vocab));
    return s;
}

template <class T>
T* at(void* workspace, size_t offset) {
    return reinterpret_cast<T*>(reinterpret_cast<char*>(workspace) + offset);
}

#define STAR_CHECK(call)                    \
    do {                                    \
        const star_status s_ = (call);      \
        if (s_ != STAR_OK) return s_;       \
    } while (0)
#define STAR_LAUNCH(call)                                                    \
    do {                                                                     \
        const hipError_t e_ = (call);                                        \
        if (e_ != hipSuccess) return star::hip_error(e_, #call);             \
    } while (0)

}  // namespace

extern "C" {

static bool logits_fit(int dtype, int64_t tokens, int64_t vocab) {
    return known(dtype) && tokens > 0 && tokens <= kMostRows && vocab > 0 && vocab <= kMostVocab;
}

size_t star_token_logprobs_workspace(star_dtype dtype, int64_t tokens, int64_t vocab) {
    return logits_fit(dtype, tokens, vocab) ? star::logprobs_workspace(dtype, tokens, vocab) : 0;
}

size_t star_policy_loss_workspace(star_dtype dtype, int64_t tokens, int64_t vocab) {
    return logits_fit(dtype, tokens, vocab) ? star::policy_workspace(dtype, tokens, vocab) : 0;
}

size_t star_preference_loss_workspace(star_dtype dtype, int64_t tokens, int64_t vocab, int32_t pairs) {
    if ((tokens != 0 && !logits_fit(dtype, tokens, vocab)) || pairs < 0) return 0;
    return preference_space(dtype, tokens, vocab, pairs).total;
}

star_status star_token_logprobs(const void* logits, star_dtype dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets,
                                float temperature, float* logp_out, float* lse_out, void* workspace, size_t workspace_bytes,
                                void* hip_stream) {
    set_error(STAR_OK, "");
    STAR_CHECK(check_logits(logits, dtype, tokens, vocab, ld, targets, temperature, nullptr, 0));
    if (tokens == 0) return STAR_OK;
    if (!logp_out) return set_error(STAR_ERR_NULL, "logp_out is NULL");
    STAR_CHECK(check_workspace(workspace, workspace_bytes, star_token_logprobs_workspace(dtype, tokens, vocab)));
    const star::Logits l = make_logits(logits, dtype, tokens, vocab, ld, targets, nullptr, temperature);
    // A normaliser is asked for where a gradient is to follow: logits that the memory-side cache holds stay in it (1023 x 50021, fp32, both
    // calls: 97 against 102 us).  Larger ones are mostly gone by then.
    const bool again = lse_out && tokens * vocab <= kCacheBytes / (int64_t)bytes_of(dtype);
    STAR_LAUNCH(star::launch_logprobs(l, 0, tokens, logp_out, nullptr, lse_out, nullptr, again, workspace, static_cast<hipStream_t>(hip_stream)));
    return STAR_OK;
}

star_status star_token_logprobs_grad(const void* logits, star_dtype dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets,
                                     float temperature, const float* lse, const float* dlogp, void* dlogits, int64_t ld_out,
                                     void* hip_stream) {
    set_error(STAR_OK, "");
    STAR_CHECK(check_logits(logits, dtype, tokens, vocab, ld, targets, temperature, dlogits, ld_out));
    if (tokens == 0) return STAR_OK;
    if (!lse || !dlogp || !dlogits) return set_error(STAR_ERR_NULL, "lse, dlogp or dlogits is NULL");
    const star::Logits l = make_logits(logits, dtype, tokens, vocab, ld, targets, nullptr, temperature);
    STAR_LAUNCH(star::launch_logprobs_grad(l, 0, tokens, lse, nullptr, dlogp, dlogits, ld_out, star::PairLoss{}, static_cast<hipStream_t>(hip_stream)));
    return STAR_OK;
}

star_status star_policy_loss(const void* logits, star_dtype dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets,
                             const float* old_logp, const float* ref_logp, const float* advantages, const float* weights,
                             const star_policy_params* params, void* dlogits, int64_t ld_out, float* logp_out, float* stats_out,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
    set_error(STAR_OK, "");
    if (!params) return set_error(STAR_ERR_NULL, "params is NULL");
    if (!std::isfinite(params->scale)) return set_error(STAR_ERR_HPARAM, "scale must be finite");
    if (!(params->clip_low >= 0.f) || !(params->clip_high >= 0.f)) return set_error(STAR_ERR_HPARAM, "a clip range must not be negative");
    if (!(params->kl_coef >= 0.f) || !std::isfinite(params->kl_coef)) return set_error(STAR_ERR_HPARAM, "kl_coef must be finite and not negative");
    STAR_CHECK(check_logits(logits, dtype, tokens, vocab, ld, targets, params->temperature, dlogits, ld_out));
    if (!stats_out) return set_error(STAR_ERR_NULL, "stats_out is NULL");
    if (tokens > 0) {
        if (!old_logp || !advantages) return set_error(STAR_ERR_NULL, "old_logp or advantages is NULL");
        if (!ref_logp && params->kl_coef != 0.f) return set_error(STAR_ERR_NULL, "ref_logp is NULL and kl_coef is not 0");
        if (over(logp_out, old_logp, tokens) || over(logp_out, ref_logp, tokens) || over(logp_out, advantages, tokens) || over(logp_out, weights, tokens))
            return set_error(STAR_ERR_SHAPE, "logp_out overlaps an input");
        STAR_CHECK(check_workspace(workspace, workspace_bytes, star_policy_loss_workspace(dtype, tokens, vocab)));
    }
    const star::Logits l = make_logits(logits, dtype, tokens, vocab, ld, targets, weights, params->temperature);
    const star::PolicyArgs a{old_logp, ref_logp, advantages, params->scale, 1.f - params->clip_low, 1.f + params->clip_high, params->kl_coef};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    STAR_LAUNCH(star::launch_policy(l, a, logp_out, dlogits, ld_out, stats_out, workspace, stream));
    return STAR_OK;
}

star_status star_preference_loss(const void* logits, star_dtype dtype, int64_t tokens, int64_t vocab, int64_t ld, const int64_t* targets,
                                 const float* ref_logp, const float* weights, int32_t pairs, const int64_t* offsets,
                                 const star_preference_params* params, void* dlogits, int64_t ld_out, float* logp_out, float* margins_out,
                                 float* loss_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
    set_error(STAR_OK, "");
    if (!params) return set_error(STAR_ERR_NULL, "params is NULL");
    if (!std::isfinite(params->scale) || !std::isfinite(params->beta)) return set_error(STAR_ERR_HPARAM, "scale and beta must be finite");
    if (!(params->label_smoothing >= 0.f && params->label_smoothing <= 1.f)) return set_error(STAR_ERR_HPARAM, "label_smoothing must lie in 0 to 1");
    STAR_CHECK(check_logits(logits, dtype, tokens, vocab, ld, targets, params->temperature, dlogits, ld_out));
    if (pairs < 0 || pairs > (1 << 22)) return set_error(STAR_ERR_SHAPE, "pairs is negative or above 2^22");
    if (!loss_out || !offsets) return set_error(STAR_ERR_NULL, "loss_out or offsets is NULL");
    if (tokens > 0 && !ref_logp) return set_error(STAR_ERR_NULL, "ref_logp is NULL");
    if (offsets[0] != 0 || offsets[2 * (int64_t)pairs] != tokens) return set_error(STAR_ERR_GROUP, "offsets must run from 0 to tokens");
    for (int64_t i = 0; i < 2 * (int64_t)pairs; ++i)
        if (offsets[i + 1] < offsets[i]) return set_error(STAR_ERR_GROUP, "offsets decrease");
    if (over(logp_out, ref_logp, tokens) || over(logp_out, weights, tokens)) return set_error(STAR_ERR_SHAPE, "logp_out overlaps an input");
    const PreferenceSpace space = preference_space(dtype, tokens, vocab, pairs);
    STAR_CHECK(check_workspace(workspace, workspace_bytes, space.total));
    const star::Logits l = make_logits(logits, dtype, tokens, vocab, ld, targets, weights, params->temperature);
    const star::PreferenceArgs a{ref_logp, params->scale, params->beta, params->label_smoothing};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    double* terms = at<double>(workspace, space.terms);
    star::MaxSum* sums = dlogits ? at<star::MaxSum>(workspace, space.sums) : nullptr;
    float* dlogp = at<float>(workspace, space.dlogp);
    float *logp = logp_out ? logp_out : at<float>(workspace, space.logp), *logp_low = at<float>(workspace, space.logp_low);
    const star::PairLoss loss{terms, pairs, params->scale, loss_out};
    bool joined = false;
    void* rows = space.total > space.rows ? at<char>(workspace, space.rows) : nullptr;
    for (int32_t first = 0; first < pairs; first += star::kPairsPerLaunch) {
        const int n = std::min<int32_t>(star::kPairsPerLaunch, pairs - first);
        star::PairOffsets o{};
        for (int i = 0; i <= 2 * n; ++i) o.at[i] = offsets[2 * (int64_t)first + i];
        const int64_t from = o.at[0], count = o.at[2 * n] - from;
        STAR_LAUNCH(star::launch_logprobs(l, from, count, logp, logp_low, nullptr, sums, dlogits != nullptr,
                                          count == tokens ? rows : nullptr, stream));
        STAR_LAUNCH(star::launch_pairs(l, a, o, n, logp, logp_low, dlogits ? dlogp : nullptr, margins_out ? margins_out + first : nullptr, terms + first,
                                       stream));
        const bool last = first + n == pairs && count > 0;   // the loss is joined beside the last gradient
        if (dlogits) STAR_LAUNCH(star::launch_logprobs_grad(l, from, count, nullptr, sums, dlogp, dlogits, ld_out, last ? loss : star::PairLoss{}, stream));
        joined = dlogits && last;
    }
    if (!joined) STAR_LAUNCH(star::launch_pair_loss(loss, stream));
    return STAR_OK;
}

size_t star_act_bytes(int64_t tokens, int64_t width) {
    if (!rows_fit(tokens, width, width)) return 0;
    return (size_t)(star::act_blocks(tokens) * star::act_columns(width) * (star::kActBlock + 1));
}

static star_status check_act(const void* x, int dtype, int64_t tokens, int64_t width, int64_t ld, const void* packed) {
    if (!known(dtype)) return set_error(STAR_ERR_DTYPE, "unknown dtype of the activations");
    if (!rows_fit(tokens, width, ld)) return set_error(STAR_ERR_SHAPE, "a size is negative, ld is below width, or the activations are too large");
    if (tokens == 0 || width == 0) return STAR_OK;
    if (!x || !packed) return set_error(STAR_ERR_NULL, "the activations or their packed form is NULL");
    if (!on_grid(x, bytes_of(dtype))) return set_error(STAR_ERR_SHAPE, "an address is not a multiple of its element's size");
    if (!on_grid(packed, 16)) return set_error(STAR_ERR_SHAPE, "packed is not aligned to 16 bytes");
    return STAR_OK;
}

star_status star_act_pack(const void* x, star_dtype dtype, int64_t tokens, int64_t width, int64_t ld, void* packed, void* hip_stream) {
    set_error(STAR_OK, "");
    STAR_CHECK(check_act(x, dtype, tokens, width, ld, packed));
    if (tokens == 0 || width == 0) return STAR_OK;
    STAR_LAUNCH(star::launch_act_pack(x, dtype, tokens, width, ld, packed, static_cast<hipStream_t>(hip_stream)));
    return STAR_OK;
}

star_status star_act_unpack(const void* packed, int64_t tokens, int64_t width, void* out, star_dtype dtype, int64_t ld, void* hip_stream) {
    set_error(STAR_OK, "");
    STAR_CHECK(check_act(out, dtype, tokens, width, ld, packed));
    if (tokens == 0 || width == 0) return STAR_OK;
    STAR_LAUNCH(star::launch_act_unpack(packed, tokens, width, out, dtype, ld, static_cast<hipStream_t>(hip_stream)));
    return STAR_OK;
}

size_t star_act_weight_grad_workspace(star_dtype dy_dtype, int64_t tokens, int64_t out, int64_t width) {
    if (!rows_fit(tokens, width, width) || !rows_fit(out, width, width) || tokens < 0) return 0;
    const int parts = star::weight_grad_parts(dy_dtype, tokens, out, width);
    return parts > 1 ? round16(sizeof(float) * (size_t)parts * (size_t)out * (size_t)width) : 0;
}

star_status star_act_weight_grad(const void* dy, star_dtype dy_dtype, int64_t tokens, int64_t out, int64_t ld, const void* packed,
                                 int64_t width, void* dw, star_dtype dw_dtype, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
    set_error(STAR_OK, "");
    if (!known(dy_dtype)) return set_error(STAR_ERR_DTYPE, "unknown dtype of dy");
    if (!known(dw_dtype)) return set_error(STAR_ERR_DTYPE, "unknown dtype of dw");
    if (!rows_fit(tokens, out, ld) || !rows_fit(tokens, width, width) || !rows_fit(out, width, width))
        return set_error(STAR_ERR_SHAPE, "a size is negative, ld is below out, or a matrix is too large");
    if (out == 0 || width == 0) return STAR_OK;
    if (!dw) return set_error(STAR_ERR_NULL, "dw is NULL");
    if (!on_grid(dw, bytes_of(dw_dtype))) return set_error(STAR_ERR_SHAPE, "an address is not a multiple of its element's size");
    if (tokens > 0) {
        if (!dy || !packed) return set_error(STAR_ERR_NULL, "dy or packed is NULL");
        if (!on_grid(dy, bytes_of(dy_dtype))) return set_error(STAR_ERR_SHAPE, "an address is not a multiple of its element's size");
        if (!on_grid(packed, 16)) return set_error(STAR_ERR_SHAPE, "packed is not aligned to 16 bytes");
    }
    if (tokens > kMostSummed || width > kMostWidth || (out + 63) / 64 * ((width + 63) / 64) > kMostTiles)
        return set_error(STAR_ERR_SHAPE, "tokens is above 2^30, width above 2^22, or dw is too large");
    STAR_CHECK(check_workspace(workspace, workspace_bytes, star_act_weight_grad_workspace(dy_dtype, tokens, out, width)));
    const star::WeightGrad g{dy, dy_dtype, tokens, out, ld, packed, width, dw, dw_dtype, accumulate != 0};
    STAR_LAUNCH(star::launch_weight_grad(g, workspace, static_cast<hipStream_t>(hip_stream)));
    return STAR_OK;
}

}  // extern "C"
