// train.cpp -- entry points of the training stage: argument checks and kernel
// sequencing on the caller's stream.  No context, no allocation, no state.
#include "rl_decode.h"
#include "rl_internal.h"

#include <hip/hip_runtime.h>

#include <cmath>

using namespace rl;

namespace {

constexpr int kMaxRows = 1 << 20, kMaxVocab = 1 << 24, kMaxTokens = 1 << 24, kMaxSeqs = 1 << 20, kMaxPairs = 1 << 19;

constexpr double kMinTemperature = 1e-30, kMaxTemperature = 1e30;   // 1 / T and log2(e) / T are normal fp32 numbers

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
size_t elem_bytes(int dtype) { return dtype == RL_DTYPE_FP32 ? 4 : 2; }
rl_status status_of(hipError_t e) { return e == hipSuccess ? RL_OK : RL_ERR_HIP; }

bool rows_ok(int32_t n, int32_t vocab, int32_t dtype, int64_t ld, double T) {
    return n >= 0 && n <= kMaxRows && vocab >= 1 && vocab <= kMaxVocab && (dtype == RL_DTYPE_FP32 || dtype == RL_DTYPE_BF16) &&
           ld >= vocab && ld <= (int64_t(1) << 40) / (n > 0 ? n : 1) && (T == 0.0 || (T >= kMinTemperature && T <= kMaxTemperature));
}

// bytes from the first to past the last entry of a matrix of rows
size_t span_bytes(int32_t n, int32_t vocab, int64_t ld, size_t es) { return es * (static_cast<size_t>(n - 1) * ld + vocab); }

// d_logits is the logits themselves, or apart from them
bool place_ok(const void* z, int64_t ld, const void* d, int64_t ldd, int32_t n, int32_t vocab, size_t es) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(z), b = reinterpret_cast<uintptr_t>(d);
    if (a == b) return ld == ldd;
    return a + span_bytes(n, vocab, ld, es) <= b || b + span_bytes(n, vocab, ldd, es) <= a;
}

rl_status workspace_ok(const void* ws, size_t have, size_t need) {
    if (need == 0) return RL_OK;
    if (!ws || !aligned(ws, 256)) return RL_ERR_INVALID_ARG;
    return have < need ? RL_ERR_CAPACITY : RL_OK;
}

size_t logprob_ws(int n, int V) { return align256(logprob_parts(n, V) * sizeof(RowPart)); }

// What rl_policy_loss_logits keeps between its kernels: the loss's own, d_logp
// and d_entropy, what logp lost by rounding, the rows' statistics, the vocabulary chunks' sums.
struct LogitsWs {
    size_t off_g, off_ge, off_rest, off_stats, off_parts, bytes;
};
LogitsWs logits_ws(int n, int n_seqs, int V) {
    LogitsWs w;
    size_t at = policy_ws_bytes(n, n_seqs);
    w.off_g = at;
    at += align256(sizeof(float) * n);
    w.off_ge = at;
    at += align256(sizeof(float) * n);
    w.off_rest = at;
    at += align256(sizeof(float) * n);
    w.off_stats = at;
    at += align256(2 * sizeof(float) * n);
    w.off_parts = at;
    w.bytes = at + logprob_ws(n, V);
    return w;
}

bool policy_ok(const rl_policy_batch* b, const rl_policy_params* q, PolicyArgs* p) {
    if (!b || !q || q->reserved != 0) return false;
    if (b->n < 0 || b->n > kMaxTokens || b->n_seqs < 1 || b->n_seqs > kMaxSeqs || (!b->seq_offsets && b->n_seqs != 1)) return false;
    if (!(q->clip_low >= 0.0 && q->clip_low < 1.0) || !(q->clip_high >= 0.0) || !std::isfinite(q->clip_high)) return false;
    if (!(q->dual_clip == 0.0 || q->dual_clip > 1.0) || !std::isfinite(q->dual_clip)) return false;
    if (!std::isfinite(q->kl_coef) || !std::isfinite(q->entropy_coef) || !std::isfinite(q->scale)) return false;
    if (q->kl < RL_KL_K1 || q->kl > RL_KL_K3 || q->aggregate < RL_AGG_TOKEN_MEAN || q->aggregate > RL_AGG_SUM) return false;
    if (q->token_advantages != 0 && q->token_advantages != 1) return false;
    if (!b->ref_logp && q->kl_coef != 0.0) return false;
    if (b->n > 0 && (!b->old_logp || !b->advantages)) return false;
    *p = PolicyArgs{b->n, b->n_seqs, b->seq_offsets, b->old_logp, b->ref_logp, b->advantages, b->mask, 1.0 - q->clip_low,
                    1.0 + q->clip_high, q->dual_clip, q->kl_coef, q->entropy_coef, q->scale, q->kl, q->aggregate,
                    q->token_advantages, nullptr};
    return true;
}

}  // namespace

extern "C" {

size_t rl_logprob_workspace_bytes(int32_t n, int32_t vocab) {
    return n < 1 || n > kMaxRows || vocab < 1 || vocab > kMaxVocab ? 0 : logprob_ws(n, vocab);
}

rl_status rl_token_logprobs(int32_t n, int32_t vocab, int32_t dtype, const void* logits, int64_t ld, const int32_t* targets,
                            double temperature, float* out_logp, float* out_entropy, float* out_stats, void* workspace,
                            size_t ws_bytes, void* stream) {
    if (!rows_ok(n, vocab, dtype, ld, temperature)) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    if (!logits || !targets || !out_logp || !aligned(logits, elem_bytes(dtype))) return RL_ERR_INVALID_ARG;
    if (const rl_status st = workspace_ok(workspace, ws_bytes, logprob_ws(n, vocab)); st != RL_OK) return st;
    const LogprobArgs a{logits, ld, n, vocab, targets, temperature == 0.0 ? 1.0 : temperature, out_logp, out_entropy,
                        out_stats, nullptr};
    return status_of(launch_token_logprobs(dtype, a, static_cast<RowPart*>(workspace), static_cast<hipStream_t>(stream)));
}

rl_status rl_token_logprobs_backward(int32_t n, int32_t vocab, int32_t dtype, const void* logits, int64_t ld,
                                     const int32_t* targets, double temperature, const float* stats, const float* entropy,
                                     const float* d_logp, const float* d_entropy, void* d_logits, int64_t ldd, void* stream) {
    if (!rows_ok(n, vocab, dtype, ld, temperature) || !rows_ok(n, vocab, dtype, ldd, temperature)) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    const size_t es = elem_bytes(dtype);
    if (!logits || !targets || !stats || !d_logp || !d_logits || (d_entropy && !entropy)) return RL_ERR_INVALID_ARG;
    if (!aligned(logits, es) || !aligned(d_logits, es) || !place_ok(logits, ld, d_logits, ldd, n, vocab, es))
        return RL_ERR_INVALID_ARG;
    return status_of(launch_token_logprobs_backward(dtype, logits, ld, n, vocab, targets, temperature == 0.0 ? 1.0 : temperature,
                                                    stats, entropy, d_logp, d_entropy, d_logits, ldd,
                                                    static_cast<hipStream_t>(stream)));
}

size_t rl_policy_workspace_bytes(int32_t n, int32_t n_seqs) {
    return n < 0 || n > kMaxTokens || n_seqs < 1 || n_seqs > kMaxSeqs ? 0 : policy_loss_ws_bytes(n, n_seqs);
}

rl_status rl_policy_loss(const rl_policy_batch* batch, const rl_policy_params* params, const float* logp, const float* entropy,
                         float* out_loss, float* d_logp, float* d_entropy, void* workspace, size_t ws_bytes, void* stream) {
    PolicyArgs p;
    if (!policy_ok(batch, params, &p) || !out_loss) return RL_ERR_INVALID_ARG;
    if (p.n > 0 && (!logp || !d_logp)) return RL_ERR_INVALID_ARG;
    if (!entropy && p.ent_coef != 0.0) return RL_ERR_INVALID_ARG;
    if (const rl_status st = workspace_ok(workspace, ws_bytes, policy_loss_ws_bytes(p.n, p.n_seqs)); st != RL_OK) return st;
    return status_of(launch_policy_loss(p, logp, entropy, out_loss, d_logp, d_entropy, workspace, static_cast<hipStream_t>(stream)));
}

size_t rl_policy_logits_workspace_bytes(int32_t n, int32_t n_seqs, int32_t vocab) {
    if (n < 0 || n > kMaxRows || n_seqs < 1 || n_seqs > kMaxSeqs || vocab < 1 || vocab > kMaxVocab) return 0;
    return logits_ws(n, n_seqs, vocab).bytes;
}

rl_status rl_policy_loss_logits(const rl_policy_batch* batch, const rl_policy_params* params, int32_t vocab, int32_t dtype,
                                const void* logits, int64_t ld, const int32_t* targets, double temperature, float* out_loss,
                                float* out_logp, float* out_entropy, void* d_logits, int64_t ldd, void* workspace,
                                size_t ws_bytes, void* stream) {
    PolicyArgs p;
    if (!policy_ok(batch, params, &p) || !out_loss) return RL_ERR_INVALID_ARG;
    if (!rows_ok(p.n, vocab, dtype, ld, temperature) || !rows_ok(p.n, vocab, dtype, ldd, temperature)) return RL_ERR_INVALID_ARG;
    if (!out_entropy && p.ent_coef != 0.0) return RL_ERR_INVALID_ARG;
    const size_t es = elem_bytes(dtype);
    if (p.n > 0) {
        if (!logits || !targets || !out_logp || !d_logits || !aligned(logits, es) || !aligned(d_logits, es)) return RL_ERR_INVALID_ARG;
        if (!place_ok(logits, ld, d_logits, ldd, p.n, vocab, es)) return RL_ERR_INVALID_ARG;
    }
    const LogitsWs w = logits_ws(p.n, p.n_seqs, vocab);
    if (const rl_status st = workspace_ok(workspace, ws_bytes, w.bytes); st != RL_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(workspace);
    float* g = reinterpret_cast<float*>(base + w.off_g);
    float* ge = p.ent_coef != 0.0 ? reinterpret_cast<float*>(base + w.off_ge) : nullptr;
    float* stats = reinterpret_cast<float*>(base + w.off_stats);
    const double T = temperature == 0.0 ? 1.0 : temperature;
    const LogprobArgs a{logits, ld, p.n, vocab, targets, T, out_logp, out_entropy, stats, &p};
    if (policy_rows_fit(dtype, p.n, vocab)) {
        const PolicyWs pw = policy_ws(p, base);
        hipError_t e = launch_policy_counts(p, pw, s);
        int n_parts = 0;
        if (e == hipSuccess) e = launch_policy_rows(dtype, p, pw, a, d_logits, ldd, &n_parts, s);
        if (e == hipSuccess) e = launch_policy_final(p, pw, n_parts, out_loss, s);
        return status_of(e);
    }
    p.rest = reinterpret_cast<float*>(base + w.off_rest);
    hipError_t e = launch_token_logprobs(dtype, a, reinterpret_cast<RowPart*>(base + w.off_parts), s);
    if (e == hipSuccess) e = launch_policy_loss(p, out_logp, out_entropy, out_loss, g, ge, base, s);
    if (e == hipSuccess)
        e = launch_token_logprobs_backward(dtype, logits, ld, p.n, vocab, targets, T, stats, out_entropy, g, ge, d_logits, ldd, s);
    return status_of(e);
}

size_t rl_preference_workspace_bytes(int32_t n, int32_t n_pairs) {
    return n < 0 || n > kMaxTokens || n_pairs < 1 || n_pairs > kMaxPairs ? 0 : preference_ws_bytes(n, n_pairs);
}

rl_status rl_preference_loss(int32_t n, int32_t n_pairs, const int32_t* seq_offsets, const float* logp, const float* ref_logp,
                             const uint8_t* mask, const rl_preference_params* q, float* out_loss, float* out_rewards,
                             float* d_logp, void* workspace, size_t ws_bytes, void* stream) {
    if (n < 0 || n > kMaxTokens || n_pairs < 1 || n_pairs > kMaxPairs || !seq_offsets || !q || !out_loss) return RL_ERR_INVALID_ARG;
    if (n > 0 && (!logp || !d_logp)) return RL_ERR_INVALID_ARG;
    if (!(q->beta > 0.0) || !std::isfinite(q->beta) || !std::isfinite(q->margin) || !std::isfinite(q->scale)) return RL_ERR_INVALID_ARG;
    if (q->form < RL_PREF_SIGMOID || q->form > RL_PREF_SQUARED || (q->average != 0 && q->average != 1)) return RL_ERR_INVALID_ARG;
    if (!(q->label_smoothing >= 0.0 && q->label_smoothing <= 0.5)) return RL_ERR_INVALID_ARG;
    if (q->label_smoothing != 0.0 && q->form != RL_PREF_SIGMOID) return RL_ERR_INVALID_ARG;
    if (const rl_status st = workspace_ok(workspace, ws_bytes, preference_ws_bytes(n, n_pairs)); st != RL_OK) return st;
    const PrefArgs p{n, n_pairs, seq_offsets, logp, ref_logp, mask, q->beta, q->label_smoothing, q->margin, q->scale, q->form,
                     q->average, out_rewards, d_logp};
    return status_of(launch_preference_loss(p, out_loss, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
