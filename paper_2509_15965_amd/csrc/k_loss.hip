// k_loss.hip -- the RL losses on packed per-token log-probabilities, with
// their gradients: the clipped policy loss with a KL term, and the loss of
// paired log ratios.  Tokens are 10-30 bytes each and a batch a few MB, so
// these are bound by launches and memory latency; all arithmetic on tokens
// and every sum is fp64, in a fixed order.
#include "rl_device.h"
#include "rl_internal.h"
#include "train.h"

namespace rl {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Counted tokens of each sequence (one wave a sequence), and per workgroup
// the counted tokens and the sequences that have some.
constexpr int kMaxCountBlocks = 256;

__global__ void __launch_bounds__(kThreads) policy_count_kernel(int n, int n_seqs, const int32_t* __restrict__ offs,
                                                                const uint8_t* __restrict__ mask,
                                                                int32_t* __restrict__ counts, CountPart* __restrict__ parts) {
    __shared__ CountPart sp[kWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    CountPart mine{0, 0};
    for (int s = blockIdx.x * kWaves + wave; s < n_seqs; s += gridDim.x * kWaves) {
        int a, b;
        seq_range(offs, n, s, &a, &b);
        int k = b - a;
        if (mask) {
            k = 0;
            for (int i = a + lane; i < b; i += 64) k += mask[i] != 0;
            k = wave_sum(k);
        }
        if (lane == 0) counts[s] = k;
        mine.tokens += k;
        mine.seqs += k > 0;
    }
    if (lane == 0) sp[wave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) { mine.tokens += sp[w].tokens; mine.seqs += sp[w].seqs; }
        parts[blockIdx.x] = mine;
    }
}

constexpr int kSums = kPolicySums;

template <int N> __device__ void block_sums(double* v, double* out) {
    __shared__ double sh[kWaves][N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if ((threadIdx.x & 63) == 0)
        for (int k = 0; k < N; ++k) sh[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
    if (threadIdx.x < N) {
        double t = 0.0;
        for (int w = 0; w < kWaves; ++w) t += sh[w][threadIdx.x];
        out[threadIdx.x] = t;
    }
}

constexpr int kTokensPerBlock = 1024;

__global__ void __launch_bounds__(kThreads) policy_loss_kernel(PolicyArgs p, const float* __restrict__ logp,
        const float* __restrict__ ent, const int32_t* __restrict__ counts, const CountPart* __restrict__ cparts,
        int n_cparts, float* __restrict__ d_logp, float* __restrict__ d_ent, double* __restrict__ parts) {
    __shared__ int total[2];
    if (threadIdx.x < 64) {
        int tok = 0, seqs = 0;
        for (int k = threadIdx.x; k < n_cparts; k += 64) { tok += cparts[k].tokens; seqs += cparts[k].seqs; }
        tok = wave_sum(tok);
        seqs = wave_sum(seqs);
        if (threadIdx.x == 0) { total[0] = tok; total[1] = seqs; }
    }
    __syncthreads();
    double v[kSums] = {};
    const int end = min(p.n, (static_cast<int>(blockIdx.x) + 1) * kTokensPerBlock);
    for (int i = blockIdx.x * kTokensPerBlock + threadIdx.x; i < end; i += kThreads) {
        double g = 0.0, ge = 0.0;
        const int s = seq_of(p.offs, p.n_seqs, i);
        if (s >= 0 && !(p.mask && !p.mask[i])) {
            const double w = p.agg == 0 ? 1.0 / total[0] : p.agg == 1 ? 1.0 / (static_cast<double>(counts[s]) * total[1]) : 1.0;
            const TokenLoss t = policy_token(p, logp[i], p.old_logp[i], p.ref ? p.ref[i] : 0.0f, p.adv[p.token_adv ? i : s]);
            v[0] += w * t.pg;
            v[1] += w * t.kl;
            if (ent) v[2] += w * ent[i];
            v[3] += t.clipped;
            v[4] += t.dual;
            v[5] -= t.lr;
            v[6] += 1.0;
            g = p.scale * w * t.g;
            ge = -p.scale * w * p.ent_coef;
        }
        if (d_logp) d_logp[i] = static_cast<float>(g);
        if (d_ent) d_ent[i] = static_cast<float>(ge);
    }
    block_sums<kSums>(v, parts + static_cast<size_t>(blockIdx.x) * kSums);
}

__global__ void __launch_bounds__(kThreads) policy_final_kernel(const double* __restrict__ parts, int n_parts, double kl_coef,
                                                                double ent_coef, double scale, float* __restrict__ out) {
    __shared__ double t[kSums];
    double v[kSums] = {};
    for (int b = threadIdx.x; b < n_parts; b += kThreads)
        for (int k = 0; k < kSums; ++k) v[k] += parts[static_cast<size_t>(b) * kSums + k];
    block_sums<kSums>(v, t);
    __syncthreads();
    if (threadIdx.x != 0) return;
    const double n = t[6] > 0.0 ? t[6] : 1.0;
    out[0] = static_cast<float>(scale * (t[0] + (kl_coef != 0.0 ? kl_coef * t[1] : 0.0) - (ent_coef != 0.0 ? ent_coef * t[2] : 0.0)));
    for (int k = 0; k < 3; ++k) out[1 + k] = static_cast<float>(t[k]);
    for (int k = 3; k < 6; ++k) out[1 + k] = static_cast<float>(t[k] / n);
    out[7] = static_cast<float>(t[6]);
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }
int blocks_of(int n) { return (n + kTokensPerBlock - 1) / kTokensPerBlock; }

// ---- preference loss -------------------------------------------------------

// Sums of a pair: loss, rewards chosen and rejected, chosen above rejected,
// logp chosen and rejected.
constexpr int kPairSums = 6;

__global__ void __launch_bounds__(kThreads) preference_kernel(PrefArgs p, double* __restrict__ parts) {
    __shared__ double sums[6];   // log ratio, logp, counted tokens: chosen, rejected
    const int pair = blockIdx.x;
    if (pair == p.n_pairs) {     // tokens that no sequence holds
        int a, b;
        seq_range(p.offs, p.n, 0, &a, &b);
        for (int i = threadIdx.x; i < a; i += kThreads) p.d_logp[i] = 0.0f;
        seq_range(p.offs, p.n, 2 * p.n_pairs - 1, &a, &b);
        for (int i = b + threadIdx.x; i < p.n; i += kThreads) p.d_logp[i] = 0.0f;
        return;
    }
    int a[2], b[2];
    double v[6] = {};
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        seq_range(p.offs, p.n, 2 * pair + side, &a[side], &b[side]);
        for (int i = a[side] + threadIdx.x; i < b[side]; i += kThreads) {
            if (p.mask && !p.mask[i]) continue;
            const double lp = p.logp[i];
            v[3 * side] += p.ref ? lp - p.ref[i] : lp;
            v[3 * side + 1] += lp;
            v[3 * side + 2] += 1.0;
        }
    }
    block_sums<6>(v, sums);
    __syncthreads();
    double per[2], R[2];
    for (int side = 0; side < 2; ++side) {
        const double cnt = sums[3 * side + 2];
        per[side] = p.average && cnt > 0.0 ? 1.0 / cnt : 1.0;
        R[side] = p.beta * (sums[3 * side] * per[side]);
    }
    const double h = R[0] - R[1] - p.margin;
    double loss, dh;
    if (p.form == 0) {
        // ln sigmoid(x) = min(x, 0) - ln(1 + exp(-|x|))
        const double tail = log1p(exp(-fabs(h)));
        const double lp = (h < 0.0 ? h : 0.0) - tail, ln = (h > 0.0 ? -h : 0.0) - tail;
        loss = -(1.0 - p.smooth) * lp - p.smooth * ln;
        dh = h != h ? h : p.smooth - exp(ln);   // s sigmoid(h) - (1 - s) sigmoid(-h)
    } else if (p.form == 1) {
        loss = h >= 1.0 ? 0.0 : 1.0 - h;
        dh = h >= 1.0 ? 0.0 : -1.0;
    } else {
        const double x = (h - 0.5) / p.beta;
        loss = x * x;
        dh = 2.0 * x / p.beta;
    }
    if (threadIdx.x == 0) {
        double* o = parts + static_cast<size_t>(pair) * kPairSums;
        o[0] = loss;
        o[1] = R[0];
        o[2] = R[1];
        o[3] = R[0] > R[1];
        o[4] = sums[1] * per[0];
        o[5] = sums[4] * per[1];
        if (p.rewards) {
            p.rewards[2 * pair] = static_cast<float>(R[0]);
            p.rewards[2 * pair + 1] = static_cast<float>(R[1]);
        }
    }
    const double coef = p.scale * p.beta * dh / p.n_pairs;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const float g = static_cast<float>((side ? -coef : coef) * per[side]);
        for (int i = a[side] + threadIdx.x; i < b[side]; i += kThreads) p.d_logp[i] = p.mask && !p.mask[i] ? 0.0f : g;
    }
}

__global__ void __launch_bounds__(kThreads) preference_final_kernel(const double* __restrict__ parts, int n_pairs,
                                                                    double scale, float* __restrict__ out) {
    __shared__ double t[kPairSums];
    double v[kPairSums] = {};
    for (int b = threadIdx.x; b < n_pairs; b += kThreads)
        for (int k = 0; k < kPairSums; ++k) v[k] += parts[static_cast<size_t>(b) * kPairSums + k];
    block_sums<kPairSums>(v, t);
    __syncthreads();
    if (threadIdx.x != 0) return;
    const double i = 1.0 / n_pairs;
    out[0] = static_cast<float>(scale * t[0] * i);
    out[1] = static_cast<float>(t[1] * i);
    out[2] = static_cast<float>(t[2] * i);
    out[3] = static_cast<float>((t[1] - t[2]) * i);
    out[4] = static_cast<float>(t[3] * i);
    out[5] = static_cast<float>(t[4] * i);
    out[6] = static_cast<float>(t[5] * i);
    out[7] = static_cast<float>(n_pairs);
}

}  // namespace

// counts, count partials, loss partials
PolicyWs policy_ws(const PolicyArgs& p, void* ws) {
    char* w = static_cast<char*>(ws);
    PolicyWs r;
    r.counts = reinterpret_cast<int32_t*>(w);
    w += align256(static_cast<size_t>(p.n_seqs) * sizeof(int32_t));
    r.cparts = reinterpret_cast<CountPart*>(w);
    w += align256(kMaxCountBlocks * sizeof(CountPart));
    r.parts = reinterpret_cast<double*>(w);
    const int nc = (p.n_seqs + kWaves - 1) / kWaves;
    r.n_cparts = nc < kMaxCountBlocks ? nc : kMaxCountBlocks;
    return r;
}

static size_t ws_bytes(int n_parts, int n_seqs) {
    return align256(static_cast<size_t>(n_seqs) * sizeof(int32_t)) + align256(kMaxCountBlocks * sizeof(CountPart)) +
           align256(static_cast<size_t>(n_parts) * kSums * sizeof(double));
}
size_t policy_ws_bytes(int n, int n_seqs) { return ws_bytes(blocks_of(n), n_seqs); }
size_t policy_rows_ws_bytes(int n, int n_seqs) { return ws_bytes(n, n_seqs); }

hipError_t launch_policy_counts(const PolicyArgs& p, const PolicyWs& w, hipStream_t s) {
    hipLaunchKernelGGL(policy_count_kernel, dim3(w.n_cparts), dim3(kThreads), 0, s, p.n, p.n_seqs, p.offs, p.mask, w.counts, w.cparts);
    return hipGetLastError();
}

hipError_t launch_policy_final(const PolicyArgs& p, const PolicyWs& w, int n_parts, float* out, hipStream_t s) {
    hipLaunchKernelGGL(policy_final_kernel, dim3(1), dim3(kThreads), 0, s, w.parts, n_parts, p.kl_coef, p.ent_coef, p.scale, out);
    return hipGetLastError();
}

hipError_t launch_policy_loss(const PolicyArgs& p, const float* logp, const float* ent, float* out, float* d_logp,
                              float* d_ent, void* ws, hipStream_t s) {
    const PolicyWs w = policy_ws(p, ws);
    hipError_t e = launch_policy_counts(p, w, s);
    const int nb = blocks_of(p.n);
    if (nb)
        hipLaunchKernelGGL(policy_loss_kernel, dim3(nb), dim3(kThreads), 0, s, p, logp, ent, w.counts, w.cparts, w.n_cparts,
                           d_logp, d_ent, w.parts);
    if (e == hipSuccess) e = launch_policy_final(p, w, nb, out, s);
    return e;
}

size_t preference_ws_bytes(int, int n_pairs) {
    return align256(static_cast<size_t>(n_pairs) * kPairSums * sizeof(double));
}

hipError_t launch_preference_loss(const PrefArgs& p, float* out, void* ws, hipStream_t s) {
    double* parts = static_cast<double*>(ws);
    hipLaunchKernelGGL(preference_kernel, dim3(p.n_pairs + 1), dim3(kThreads), 0, s, p, parts);
    hipLaunchKernelGGL(preference_final_kernel, dim3(1), dim3(kThreads), 0, s, parts, p.n_pairs, p.scale, out);
    return hipGetLastError();
}

}  // namespace rl
