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

// Bytes of x that are not 0.
__device__ __forceinline__ int nonzero_bytes(uint32_t x) {
    return __popc((((x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | x) & 0x80808080u);
}
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));

// Counted tokens of each sequence, and per workgroup the counted tokens and
// the sequences that have some.  LANES lanes a sequence: a wave reads 1024
// mask bytes at once, a workgroup 4096.
constexpr int kMaxCountBlocks = 1024;

template <int LANES>
__global__ void __launch_bounds__(kThreads) policy_count_kernel(int n, int n_seqs, const int32_t* __restrict__ offs,
                                                                const uint8_t* __restrict__ mask,
                                                                int32_t* __restrict__ counts, CountPart* __restrict__ parts) {
    constexpr int GROUPS = kThreads / LANES, W = LANES / 64;
    __shared__ int32_t part[kWaves];
    __shared__ CountPart sp[kWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int group = threadIdx.x / LANES, at = threadIdx.x % LANES;
    CountPart mine{0, 0};
    // every wave runs the same number of turns (a workgroup's share of a sequence meets at barriers)
    for (int s0 = blockIdx.x * GROUPS; s0 < n_seqs; s0 += gridDim.x * GROUPS) {
        const int s = s0 + group;
        int a = 0, b = 0, k = 0;
        if (s < n_seqs) seq_range(offs, n, s, &a, &b);
        if (!mask) {
            k = b - a;
        } else {
            for (int i = a + 16 * at; i < b; i += 16 * LANES) {
                if (i + 16 <= b) {
                    const u32x4 x = *reinterpret_cast<const u32x4_any*>(mask + i);
                    k += nonzero_bytes(x[0]) + nonzero_bytes(x[1]) + nonzero_bytes(x[2]) + nonzero_bytes(x[3]);
                } else {
                    for (int q = i; q < b; ++q) k += mask[q] != 0;
                }
            }
            k = wave_sum(k);
            if (W > 1) {
                if (lane == 0) part[wave] = k;
                __syncthreads();
                k = 0;
                for (int w = 0; w < W; ++w) k += part[w];
                __syncthreads();
            }
        }
        if (at == 0 && s < n_seqs) {
            counts[s] = k;
            mine.tokens += k;
            mine.seqs += k > 0;
        }
    }
    if (lane == 0) sp[wave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) { mine.tokens += sp[w].tokens; mine.seqs += sp[w].seqs; }
        parts[blockIdx.x] = mine;
    }
}

constexpr int kSums = kPolicySums;

// Sums over a workgroup of N values a lane; lane k < N of the first wave writes out[k].
template <int N, int THREADS> __device__ void block_sums(double* v, double* out) {
    __shared__ double sh[THREADS / 64][N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if ((threadIdx.x & 63) == 0)
        for (int k = 0; k < N; ++k) sh[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
    if (threadIdx.x < N) {
        double t = 0.0;
        for (int w = 0; w < THREADS / 64; ++w) t += sh[w][threadIdx.x];
        out[threadIdx.x] = t;
    }
}

__device__ __forceinline__ void policy_outputs(const double* t, double kl_coef, double ent_coef, double scale, float* out) {
    const double n = t[6] > 0.0 ? t[6] : 1.0;
    out[0] = static_cast<float>(scale * (t[0] + (kl_coef != 0.0 ? kl_coef * t[1] : 0.0) - (ent_coef != 0.0 ? ent_coef * t[2] : 0.0)));
    for (int k = 0; k < 3; ++k) out[1 + k] = static_cast<float>(t[k]);
    for (int k = 3; k < 6; ++k) out[1 + k] = static_cast<float>(t[k] / n);
    out[7] = static_cast<float>(t[6]);
}

// One token: its terms into v, its gradients out.  s: its sequence, or -1.
struct TokenIn { float logp, old_logp, ref, ent; };
__device__ __forceinline__ TokenIn load_token(const PolicyArgs& p, const float* logp, const float* ent, int i) {
    return TokenIn{logp[i], p.old_logp[i], p.ref ? p.ref[i] : 0.0f, ent ? ent[i] : 0.0f};
}
__device__ __forceinline__ void one_token(const PolicyArgs& p, const TokenIn& in, bool live, float adv, double w, double* v,
                                          float* d_logp, float* d_ent, int i) {
    double g = 0.0, ge = 0.0;
    if (live) {
        const TokenLoss t = policy_token(p, in.logp, in.old_logp, in.ref, adv);
        v[0] += w * t.pg;
        v[1] += w * t.kl;
        v[2] += w * in.ent;
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

// Tokens of a workgroup, four a lane.  The sequences they lie in are found
// once for the workgroup, then by each lane among those in LDS.
constexpr int kTokensPerLane = 4, kTokensPerBlock = kThreads * kTokensPerLane, kSpan = 512;

__global__ void __launch_bounds__(kThreads) policy_loss_kernel(PolicyArgs p, const float* __restrict__ logp,
        const float* __restrict__ ent, const int32_t* __restrict__ counts, const CountPart* __restrict__ cparts,
        int n_cparts, float* __restrict__ d_logp, float* __restrict__ d_ent, double* __restrict__ parts) {
    __shared__ int32_t span[kSpan];
    __shared__ int32_t ends[2];
    const int tid = threadIdx.x, first = blockIdx.x * kTokensPerBlock;
    const int last = min(p.n, first + kTokensPerBlock) - 1;
    TokenIn in[kTokensPerLane];
    bool live[kTokensPerLane];
#pragma unroll
    for (int k = 0; k < kTokensPerLane; ++k) {
        const int i = min(first + k * kThreads + tid, last);
        in[k] = load_token(p, logp, ent, i);
        live[k] = !p.mask || p.mask[i];
    }
    const PolicyTotals totals = policy_totals(p, cparts, n_cparts);
    int s_lo = 0, s_hi = 0;
    if (p.offs) {
        // entries at most the first token, and at most the last
        if (tid < 128) {
            const int s = seq_of_wave(p.offs, p.n_seqs, tid < 64 ? first : last);
            const int i = tid < 64 ? first : last;
            if ((tid & 63) == 0) ends[tid >> 6] = s >= 0 ? s + 1 : i < p.offs[0] ? 0 : p.n_seqs + 1;
        }
        __syncthreads();
        s_lo = min(ends[0], ends[1]);
        s_hi = max(ends[0], ends[1]);
        if (s_hi - s_lo <= kSpan) {
            for (int k = tid; k < s_hi - s_lo; k += kThreads) span[k] = p.offs[s_lo + k];
            __syncthreads();
        }
    }
    double v[kSums] = {};
#pragma unroll
    for (int k = 0; k < kTokensPerLane; ++k) {
        const int i = first + k * kThreads + tid;
        if (i > last) break;
        int s = 0;
        if (p.offs) {
            const int c = s_hi - s_lo <= kSpan ? s_lo + count_upto(span, 0, s_hi - s_lo, i) : count_upto(p.offs, s_lo, s_hi, i);
            s = c - 1 < p.n_seqs ? c - 1 : -1;
        }
        const bool on = live[k] && s >= 0;
        one_token(p, in[k], on, on ? p.adv[p.token_adv ? i : s] : 0.0f, on ? policy_weight(p, totals, s, counts) : 0.0, v,
                  d_logp, d_ent, i);
    }
    block_sums<kSums, kThreads>(v, parts + static_cast<size_t>(blockIdx.x) * kSums);
}

constexpr int kFinalThreads = 1024;

__global__ void __launch_bounds__(kFinalThreads) policy_final_kernel(const double* __restrict__ parts, int n_parts,
        double kl_coef, double ent_coef, double scale, float* __restrict__ out) {
    __shared__ double t[kSums];
    double v[kSums] = {};
    for (int b = threadIdx.x; b < n_parts; b += kFinalThreads)
#pragma unroll
        for (int k = 0; k < kSums; ++k) v[k] += parts[static_cast<size_t>(b) * kSums + k];
    block_sums<kSums, kFinalThreads>(v, t);
    __syncthreads();
    if (threadIdx.x == 0) policy_outputs(t, kl_coef, ent_coef, scale, out);
}

// The whole loss of few tokens in one workgroup and one launch: counts by
// integer atomics in LDS, tokens, sums.
constexpr int kSmallThreads = 1024, kSmallTokens = 4096, kSmallSeqs = 1024;

__global__ void __launch_bounds__(kSmallThreads) policy_small_kernel(PolicyArgs p, const float* __restrict__ logp,
        const float* __restrict__ ent, float* __restrict__ d_logp, float* __restrict__ d_ent, float* __restrict__ out) {
    constexpr int PER = kSmallTokens / kSmallThreads;
    __shared__ int32_t offs[kSmallSeqs + 1], counts[kSmallSeqs];
    __shared__ int32_t total[2];
    __shared__ double t[kSums];
    const int tid = threadIdx.x;
    TokenIn in[PER];
    bool live[PER];
    int seq[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = k * kSmallThreads + tid;
        live[k] = i < p.n && (!p.mask || p.mask[i]);
        if (live[k]) in[k] = load_token(p, logp, ent, i);
    }
    for (int s = tid; s <= p.n_seqs; s += kSmallThreads) offs[s] = p.offs ? p.offs[s] : s * p.n;
    for (int s = tid; s < p.n_seqs; s += kSmallThreads) counts[s] = 0;
    if (tid < 2) total[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = count_upto(offs, 0, p.n_seqs + 1, k * kSmallThreads + tid);
        seq[k] = live[k] && c - 1 < p.n_seqs ? c - 1 : -1;
        if (seq[k] >= 0) atomicAdd(&counts[seq[k]], 1);
    }
    __syncthreads();
    int tokens = 0, seqs = 0;
    for (int s = tid; s < p.n_seqs; s += kSmallThreads) {
        tokens += counts[s];
        seqs += counts[s] > 0;
    }
    tokens = wave_sum(tokens);
    seqs = wave_sum(seqs);
    if ((tid & 63) == 0 && tokens) {
        atomicAdd(&total[0], tokens);
        atomicAdd(&total[1], seqs);
    }
    __syncthreads();
    const PolicyTotals totals{total[0], total[1]};
    double v[kSums] = {};
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = k * kSmallThreads + tid, s = seq[k];
        if (i < p.n)
            one_token(p, in[k], s >= 0, s >= 0 ? p.adv[p.token_adv ? i : s] : 0.0f,
                      s >= 0 ? policy_weight(p, totals, s, counts) : 0.0, v, d_logp, d_ent, i);
    }
    block_sums<kSums, kSmallThreads>(v, t);
    __syncthreads();
    if (tid == 0) policy_outputs(t, p.kl_coef, p.ent_coef, p.scale, out);
}

bool policy_small(int n, int n_seqs) { return n <= kSmallTokens && n_seqs <= kSmallSeqs; }

// The counts need a kernel of their own where a mask takes tokens out, or many offsets would be read by every workgroup.
bool policy_needs_counts(const PolicyArgs& p) { return p.agg != 2 && (p.mask || (p.agg == 1 && p.n_seqs > 1024)); }

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
    block_sums<6, kThreads>(v, sums);
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
    block_sums<kPairSums, kThreads>(v, t);
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


// Sequences of more than 1024 tokens on average take a workgroup each, shorter ones a wave.
bool count_by_workgroup(const PolicyArgs& p) { return p.n / p.n_seqs > 1024; }

}  // namespace

// counts, count partials, loss partials
PolicyWs policy_ws(const PolicyArgs& p, void* ws) {
    char* w = static_cast<char*>(ws);
    PolicyWs r{nullptr, nullptr, 0, nullptr};
    if (policy_needs_counts(p)) {
        r.counts = reinterpret_cast<int32_t*>(w);
        r.cparts = reinterpret_cast<CountPart*>(w + align256(static_cast<size_t>(p.n_seqs) * sizeof(int32_t)));
        const int nc = count_by_workgroup(p) ? p.n_seqs : (p.n_seqs + kWaves - 1) / kWaves;
        r.n_cparts = nc < kMaxCountBlocks ? nc : kMaxCountBlocks;
    }
    w += align256(static_cast<size_t>(p.n_seqs) * sizeof(int32_t)) + align256(kMaxCountBlocks * sizeof(CountPart));
    r.parts = reinterpret_cast<double*>(w);
    return r;
}

size_t policy_loss_ws_bytes(int n, int n_seqs) { return policy_small(n, n_seqs) ? 0 : policy_ws_bytes(n, n_seqs); }

size_t policy_ws_bytes(int n, int n_seqs) {
    const int parts = blocks_of(n) > kPolicyMaxRowParts ? blocks_of(n) : kPolicyMaxRowParts;
    return align256(static_cast<size_t>(n_seqs) * sizeof(int32_t)) + align256(kMaxCountBlocks * sizeof(CountPart)) +
           align256(static_cast<size_t>(parts) * kSums * sizeof(double));
}

hipError_t launch_policy_counts(const PolicyArgs& p, const PolicyWs& w, hipStream_t s) {
    if (!w.counts) return hipSuccess;
    const auto kernel = count_by_workgroup(p) ? policy_count_kernel<kThreads> : policy_count_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3(w.n_cparts), dim3(kThreads), 0, s, p.n, p.n_seqs, p.offs, p.mask, w.counts, w.cparts);
    return hipGetLastError();
}

hipError_t launch_policy_final(const PolicyArgs& p, const PolicyWs& w, int n_parts, float* out, hipStream_t s) {
    hipLaunchKernelGGL(policy_final_kernel, dim3(1), dim3(kFinalThreads), 0, s, w.parts, n_parts, p.kl_coef, p.ent_coef,
                       p.scale, out);
    return hipGetLastError();
}

hipError_t launch_policy_loss(const PolicyArgs& p, const float* logp, const float* ent, float* out, float* d_logp,
                              float* d_ent, void* ws, hipStream_t s) {
    if (policy_small(p.n, p.n_seqs)) {
        hipLaunchKernelGGL(policy_small_kernel, dim3(1), dim3(kSmallThreads), 0, s, p, logp, ent, d_logp, d_ent, out);
        return hipGetLastError();
    }
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
