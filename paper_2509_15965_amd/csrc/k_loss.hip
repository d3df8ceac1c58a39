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
// the sequences that have some.  LANES lanes a sequence, 16 mask bytes a lane
// at once.
constexpr int kMaxCountBlocks = 1024;

template <int LANES> constexpr int kCountThreads = LANES > kThreads ? LANES : kThreads;

template <int LANES>
__global__ void __launch_bounds__(kCountThreads<LANES>) policy_count_kernel(int n, int n_seqs, const int32_t* __restrict__ offs,
                                                                const uint8_t* __restrict__ mask,
                                                                int32_t* __restrict__ counts, CountPart* __restrict__ parts) {
    constexpr int THREADS = kCountThreads<LANES>, WAVES = THREADS / 64, GROUPS = THREADS / LANES, W = LANES / 64;
    __shared__ int32_t part[WAVES];
    __shared__ CountPart sp[WAVES];
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
        for (int w = 1; w < WAVES; ++w) { mine.tokens += sp[w].tokens; mine.seqs += sp[w].seqs; }
        parts[blockIdx.x] = mine;
    }
}

constexpr int kSums = kPolicySums;

// Adds the lane that a DPP control names (nothing where it names none or the row is masked).
template <int CTRL, int ROWS> __device__ __forceinline__ double add_dpp(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(b), CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(b >> 32), CTRL, ROWS, 0xF, false);
    return v + __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
// Sums over a wave; lane 63 has them.  Within rows of 16 lanes, then row to
// row: register moves, where shuffles would go through LDS twelve times a value.
template <int N> __device__ __forceinline__ void wave_sums(double* v) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = add_dpp<0x111, 0xF>(v[k]);   // row_shr 1, 2, 4, 8
        v[k] = add_dpp<0x112, 0xF>(v[k]);
        v[k] = add_dpp<0x114, 0xF>(v[k]);
        v[k] = add_dpp<0x118, 0xF>(v[k]);
        v[k] = add_dpp<0x142, 0xA>(v[k]);   // lane 15 of rows 0 and 2 to rows 1 and 3
        v[k] = add_dpp<0x143, 0xC>(v[k]);   // lane 31 to rows 2 and 3
    }
}

// Sums over a workgroup of N values a lane; lane k < N of the first wave writes out[k].
template <int N, int THREADS> __device__ __forceinline__ void block_sums(double* v, double* out) {
    __shared__ double sh[THREADS / 64][N];
    wave_sums<N>(v);
    if ((threadIdx.x & 63) == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) sh[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
    if (threadIdx.x < N) {
        double t = 0.0;
#pragma unroll 1
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

// One token: its terms into v, its gradients out.
struct TokenIn { float logp, old_logp, ref, ent, rest; };
__device__ __forceinline__ TokenIn load_token(const PolicyArgs& p, const float* logp, const float* ent, int i) {
    TokenIn t{*nth(logp, i), *nth(p.old_logp, i), 0.0f, 0.0f, 0.0f};
    if (p.rest) t.rest = *nth(p.rest, i);
    if (p.ref) t.ref = *nth(p.ref, i);
    if (ent) t.ent = *nth(ent, i);
    return t;
}
__device__ __forceinline__ void one_token(const PolicyArgs& p, const TokenIn& in, bool live, float adv, double w, double* v,
                                          float* d_logp, float* d_ent, int i) {
    double g = 0.0, ge = 0.0;
    if (live) {
        const TokenLoss t = policy_token(p, static_cast<double>(in.logp) + in.rest, in.old_logp, in.ref, adv);
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
    *nth(d_logp, i) = static_cast<float>(g);
    if (d_ent) *nth(d_ent, i) = static_cast<float>(ge);
}

// K tokens a lane, loaded before anything else.  The sequences they lie in are found once for the workgroup, then by each
// lane among those in LDS.  512 sequences of 1500 tokens: 14.8 us with the last kernel, 19.2 with a mask's count before
// it, where 21 MB are 4 us of the memory: bound by one workgroup's chain of loads, search, fp64 exponentials and sums.
constexpr int kSpan = 512;

template <int K>
__global__ void __launch_bounds__(kThreads) policy_loss_kernel(PolicyArgs p, const float* __restrict__ logp,
        const float* __restrict__ ent, const int32_t* __restrict__ counts, const CountPart* __restrict__ cparts,
        int n_cparts, float* __restrict__ d_logp, float* __restrict__ d_ent, double* __restrict__ parts) {
    __shared__ int32_t span[kSpan];
    __shared__ double weight[kSpan + 1];
    __shared__ float adv[kSpan + 1];
    __shared__ int32_t ends[2];
    __shared__ PolicyTotals total;
    const int tid = threadIdx.x, first = blockIdx.x * (K * kThreads);
    const int last = min(p.n, first + K * kThreads) - 1;
    TokenIn in[K];
    uint8_t m[K];
    float own_adv[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int at = min(first + k * kThreads + tid, last);
        in[k] = load_token(p, logp, ent, at);
        m[k] = 1;
        own_adv[k] = 0.0f;
        if (p.mask) m[k] = *nth(p.mask, at);
        if (p.token_adv) own_adv[k] = *nth(p.adv, at);
    }
    // two waves: offsets at most the first token, and at most the last; another: the totals
    if (tid < 128) {
        const int t = tid < 64 ? first : last;
        const int s = seq_of_wave(p.offs, p.n_seqs, t);
        if ((tid & 63) == 0) ends[tid >> 6] = !p.offs ? 1 : s >= 0 ? s + 1 : t < p.offs[0] ? 0 : p.n_seqs + 1;
    } else if (tid < 192) {
        const PolicyTotals t = policy_totals(p, cparts, n_cparts);
        if (tid == 128) total = t;
    }
    __syncthreads();
    const int s_lo = min(ends[0], ends[1]), s_hi = max(ends[0], ends[1]);
    const PolicyTotals totals = total;
    const bool held = s_hi - s_lo <= kSpan;
    if (held) {   // entry k: offset s_lo + k, sequence s_lo - 1 + k
        for (int k = tid; k <= s_hi - s_lo; k += kThreads) {
            if (k < s_hi - s_lo) span[k] = p.offs[s_lo + k];
            const int s = s_lo - 1 + k;
            if (s < 0 || s >= p.n_seqs) continue;
            weight[k] = policy_weight(p, totals, s, counts);
            if (!p.token_adv) adv[k] = p.adv[s];
        }
        __syncthreads();
    }
    double v[kSums] = {};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = first + k * kThreads + tid;
        if (i > last) break;
        const int c = held ? s_lo + count_upto(span, 0, s_hi - s_lo, i) : count_upto(p.offs, s_lo, s_hi, i);
        const int s = c - 1 < p.n_seqs ? c - 1 : -1;
        const bool on = m[k] && s >= 0;
        float A = own_adv[k];
        double w = 0.0;
        if (on) {
            if (!p.token_adv) A = held ? adv[c - s_lo] : p.adv[s];
            w = held ? weight[c - s_lo] : policy_weight(p, totals, s, counts);
        }
        one_token(p, in[k], on, A, w, v, d_logp, d_ent, i);
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
// integer atomics in LDS, tokens, sums.  Bound by one CU's fp64: 256 tokens
// 5.6 us where two or three launches take 9 and 11, 2048 9.6 (8.5 and 11.2),
// 4096 14.7 (8.5 and 11.2).
constexpr int kSmallThreads = 1024, kSmallTokens = 2048, kSmallSeqs = 1024;

__global__ void __launch_bounds__(kSmallThreads) policy_small_kernel(PolicyArgs p, const float* __restrict__ logp,
        const float* __restrict__ ent, float* __restrict__ d_logp, float* __restrict__ d_ent, float* __restrict__ out) {
    __shared__ int32_t offs[kSmallSeqs + 1], counts[kSmallSeqs];
    __shared__ int16_t seq[kSmallTokens];
    __shared__ int32_t total[2];
    __shared__ double t[kSums];
    const int tid = threadIdx.x;
    TokenIn next{};
    if (tid < p.n) next = load_token(p, logp, ent, tid);
    for (int s = tid; s <= p.n_seqs; s += kSmallThreads) {
        offs[s] = p.offs ? p.offs[s] : s * p.n;
        if (s < kSmallSeqs) counts[s] = 0;
    }
    if (tid < 2) total[tid] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < p.n; i += kSmallThreads) {
        const uint8_t m = p.mask ? *nth(p.mask, i) : 1;
        const int c = count_upto(offs, 0, p.n_seqs + 1, i);
        const int s = m && c - 1 < p.n_seqs ? c - 1 : -1;
        seq[i] = static_cast<int16_t>(s);
        if (s >= 0) atomicAdd(&counts[s], 1);
    }
    __syncthreads();
    if (tid < p.n_seqs && counts[tid]) {   // kSmallSeqs lanes
        atomicAdd(&total[0], counts[tid]);
        atomicAdd(&total[1], 1);
    }
    __syncthreads();
    const PolicyTotals totals{total[0], total[1]};
    double v[kSums] = {};
#pragma unroll 1
    for (int i = tid; i < p.n; i += kSmallThreads) {
        const TokenIn in = next;
        if (i + kSmallThreads < p.n) next = load_token(p, logp, ent, i + kSmallThreads);
        const int s = seq[i];
        one_token(p, in, s >= 0, s >= 0 ? *nth(p.adv, p.token_adv ? i : s) : 0.0f,
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
// Two tokens a lane (768000 tokens: 14.8 us, with one 17.1, with four 15.0), and one where two workgroups a CU hold all
// that way (51200 tokens: 9.4 us, with two 10.7; 120000: 9.3 and 10.1).
int tokens_per_lane(int n) { return n <= 2 * kCUs * kThreads ? 1 : 2; }
int blocks_of(int n) {
    const int each = kThreads * tokens_per_lane(n);
    return (n + each - 1) / each;
}

// ---- preference loss -------------------------------------------------------

// Sums of a pair: loss, rewards chosen and rejected, chosen above rejected,
// logp chosen and rejected.
constexpr int kPairSums = 6;

// A sequence's sums: log ratio, logp, counted tokens.
struct SeqSums { double ratio, logp, count; };

// Lane `at` of `lanes` adds its share of tokens [a, b), the same lane the same token of every sequence:
// equal sequences have equal sums wherever they lie.
template <int U> __device__ __forceinline__ SeqSums seq_sums(const PrefArgs& p, int a, int b, int at, int lanes) {
    SeqSums t{0.0, 0.0, 0.0};
#pragma unroll 1
    for (int i = a + at; i < b; i += U * lanes) {
        float lp[U], ref[U] = {};
        uint8_t m[U];
        int q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {   // every load before any sum, none of them behind a lane's branch
            q[u] = i + u * lanes < b ? i + u * lanes : i;
            lp[u] = *nth(p.logp, q[u]);
            m[u] = 1;
        }
        if (p.ref)
#pragma unroll
            for (int u = 0; u < U; ++u) ref[u] = *nth(p.ref, q[u]);
        if (p.mask)
#pragma unroll
            for (int u = 0; u < U; ++u) m[u] = *nth(p.mask, q[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!m[u] || i + u * lanes >= b) continue;
            t.ratio += static_cast<double>(lp[u]) - ref[u];
            t.logp += lp[u];
            t.count += 1.0;
        }
    }
    return t;
}

// Loss of a pair and the factors of its tokens' gradients, chosen and rejected.
struct PairLoss { double loss, reward[2], logp[2], grad[2]; };
__device__ __forceinline__ PairLoss pair_loss(const PrefArgs& p, const SeqSums* s) {
    PairLoss r;
    double per[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        per[k] = p.average && s[k].count > 0.0 ? 1.0 / s[k].count : 1.0;
        r.reward[k] = p.beta * (s[k].ratio * per[k]);
        r.logp[k] = s[k].logp * per[k];
    }
    const double h = r.reward[0] - r.reward[1] - p.margin;
    double dh;
    if (p.form == 0) {
        // e = exp(-|h|): ln sigmoid(x) = min(x, 0) - ln(1 + e), and sigmoid(-|h|) = e / (1 + e)
        const double e = exp_below(h < 0.0 ? h : -h), tail = log1p_unit(e), q = 1.0 / (1.0 + e);
        const double lp = (h < 0.0 ? h : 0.0) - tail, ln = (h > 0.0 ? -h : 0.0) - tail;
        r.loss = -(1.0 - p.smooth) * lp - (p.smooth != 0.0 ? p.smooth * ln : 0.0);   // ln is -inf at h = inf
        dh = p.smooth - (h < 0.0 ? q : e * q);   // s sigmoid(h) - (1 - s) sigmoid(-h)
    } else if (p.form == 1) {
        r.loss = h >= 1.0 ? 0.0 : 1.0 - h;
        dh = h >= 1.0 ? 0.0 : h < 1.0 ? -1.0 : h;
    } else {
        const double x = (h - 0.5) / p.beta;
        r.loss = x * x;
        dh = 2.0 * x / p.beta;
    }
    const double coef = p.scale * p.beta * dh / p.n_pairs;
    r.grad[0] = coef * per[0];
    r.grad[1] = -coef * per[1];
    return r;
}

__device__ __forceinline__ void pair_outputs(const double* t, int n_pairs, double scale, float* out) {
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

template <int U>
__device__ __forceinline__ void write_grads(const PrefArgs& p, int a, int b, int at, int lanes, double grad) {
    const float g = static_cast<float>(grad);
#pragma unroll 1
    for (int i = a + at; i < b; i += U * lanes) {
        uint8_t m[U];
#pragma unroll
        for (int u = 0; u < U; ++u) m[u] = 1;
        if (p.mask)
#pragma unroll
            for (int u = 0; u < U; ++u) m[u] = *nth(p.mask, i + u * lanes < b ? i + u * lanes : i);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * lanes < b) *nth(p.d_logp, i + u * lanes) = m[u] ? g : 0.0f;
    }
}

__device__ __forceinline__ void write_pair(const PrefArgs& p, int pair, const PairLoss& r, double* o) {
    o[0] = r.loss;
    o[1] = r.reward[0];
    o[2] = r.reward[1];
    o[3] = r.reward[0] > r.reward[1];
    o[4] = r.logp[0];
    o[5] = r.logp[1];
    if (p.rewards) {
        p.rewards[2 * pair] = static_cast<float>(r.reward[0]);
        p.rewards[2 * pair + 1] = static_cast<float>(r.reward[1]);
    }
}

// Tokens before the first sequence and behind the last.
template <int LANES> __device__ __forceinline__ void write_outside(const PrefArgs& p, int at) {
    int a, b;
    seq_range(p.offs, p.n, 0, &a, &b);
#pragma unroll 1
    for (int i = at; i < a; i += LANES) p.d_logp[i] = 0.0f;
    seq_range(p.offs, p.n, 2 * p.n_pairs - 1, &a, &b);
#pragma unroll 1
    for (int i = b + at; i < p.n; i += LANES) p.d_logp[i] = 0.0f;
}

// One workgroup a pair, half of it a sequence (256 pairs of 2 x 1500 tokens 9.9 us with the last kernel; bound by latency:
// loads, sums, the pair's loss, stores, 9 MB in and out); one more for the tokens that no sequence holds.
constexpr int kPairThreads = 1024, kSide = kPairThreads / 2;

__global__ void __launch_bounds__(kPairThreads) preference_kernel(PrefArgs p, double* __restrict__ parts) {
    __shared__ SeqSums sums[2];
    const int pair = blockIdx.x, tid = threadIdx.x, side = tid / kSide, at = tid % kSide;
    if (pair == p.n_pairs) return write_outside<kPairThreads>(p, tid);
    int a, b;
    seq_range(p.offs, p.n, 2 * pair + side, &a, &b);
    const SeqSums t = seq_sums<4>(p, a, b, at, kSide);
    double v[6];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[3 * k] = side == k ? t.ratio : 0.0;
        v[3 * k + 1] = side == k ? t.logp : 0.0;
        v[3 * k + 2] = side == k ? t.count : 0.0;
    }
    block_sums<6, kPairThreads>(v, &sums[0].ratio);
    __syncthreads();
    const PairLoss r = pair_loss(p, sums);
    write_grads<4>(p, a, b, at, kSide, side ? r.grad[1] : r.grad[0]);   // an index would put r into LDS
    if (tid == 0) write_pair(p, pair, r, parts + static_cast<size_t>(pair) * kPairSums);
}

// Few pairs of many tokens: `cuts` workgroups a sequence.  Each adds up its
// share; after that each adds up its pair's shares and writes its tokens.
constexpr int kCutThreads = 256, kMaxCuts = kCutThreads;

__device__ __forceinline__ void cut_range(const PrefArgs& p, int seq, int cut, int cuts, int* a, int* b) {
    int lo, hi;
    seq_range(p.offs, p.n, seq, &lo, &hi);
    const int each = (hi - lo + cuts - 1) / cuts;
    *a = min(hi, lo + cut * each);
    *b = min(hi, *a + each);
}

__global__ void __launch_bounds__(kCutThreads) preference_sums_kernel(PrefArgs p, SeqSums* __restrict__ shares) {
    if (static_cast<int>(blockIdx.y) == 2 * p.n_pairs) {
        if (blockIdx.x == 0) write_outside<kCutThreads>(p, threadIdx.x);
        return;
    }
    int a, b;
    cut_range(p, blockIdx.y, blockIdx.x, gridDim.x, &a, &b);
    const SeqSums t = seq_sums<4>(p, a, b, threadIdx.x, kCutThreads);
    double v[3] = {t.ratio, t.logp, t.count};
    block_sums<3, kCutThreads>(v, &shares[blockIdx.y * gridDim.x + blockIdx.x].ratio);
}

__global__ void __launch_bounds__(kCutThreads) preference_cut_kernel(PrefArgs p, const SeqSums* __restrict__ shares,
                                                                     double* __restrict__ parts) {
    __shared__ SeqSums sums[2];
    const int tid = threadIdx.x, seq = blockIdx.y, pair = seq / 2, cuts = gridDim.x;
    int a, b;
    cut_range(p, seq, blockIdx.x, cuts, &a, &b);
    double v[6] = {};
    if (tid < cuts) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const SeqSums t = shares[(2 * pair + k) * cuts + tid];
            v[3 * k] = t.ratio;
            v[3 * k + 1] = t.logp;
            v[3 * k + 2] = t.count;
        }
    }
    block_sums<6, kCutThreads>(v, &sums[0].ratio);
    __syncthreads();
    const PairLoss r = pair_loss(p, sums);
    write_grads<4>(p, a, b, tid, kCutThreads, seq & 1 ? r.grad[1] : r.grad[0]);
    if (tid == 0 && blockIdx.x == 0 && !(seq & 1)) write_pair(p, pair, r, parts + static_cast<size_t>(pair) * kPairSums);
}

__global__ void __launch_bounds__(kFinalThreads) preference_final_kernel(const double* __restrict__ parts, int n_pairs,
                                                                         double scale, float* __restrict__ out) {
    __shared__ double t[kPairSums];
    double v[kPairSums] = {};
    for (int b = threadIdx.x; b < n_pairs; b += kFinalThreads)
#pragma unroll
        for (int k = 0; k < kPairSums; ++k) v[k] += parts[static_cast<size_t>(b) * kPairSums + k];
    block_sums<kPairSums, kFinalThreads>(v, t);
    __syncthreads();
    if (threadIdx.x == 0) pair_outputs(t, n_pairs, scale, out);
}

// Few pairs of few tokens: one workgroup and one launch, its 16 waves shared out over the sequences.  4 pairs of 2 x 200
// tokens 5.4 us (8.7 by a workgroup a pair and a last one), 16 of 2 x 512 8.8 (9.0), 32 of 2 x 200 10.7 (8.7); one of 2 x
// 8192 8.5 (10.4), of 2 x 20000 14.1 (10.7 cut).
constexpr int kSmallPairs = 16, kSmallPairTokens = 16384, kSmallWaves = kSmallThreads / 64;
bool preference_small(int n, int n_pairs) { return n_pairs <= kSmallPairs && n <= kSmallPairTokens; }

__global__ void __launch_bounds__(kSmallThreads) preference_small_kernel(PrefArgs p, float* __restrict__ out) {
    __shared__ SeqSums share[2 * kSmallPairs > kSmallWaves ? 2 * kSmallPairs : kSmallWaves];
    __shared__ double grad[2 * kSmallPairs];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, seqs = 2 * p.n_pairs;
    const int each = seqs < kSmallWaves ? kSmallWaves / seqs : 1;   // waves a sequence
    const int lanes = 64 * each, at = (wave % each) * 64 + lane, turn = kSmallWaves / each;
    write_outside<kSmallThreads>(p, tid);
#pragma unroll 1
    for (int s = wave / each; s < seqs; s += turn) {
        int a, b;
        seq_range(p.offs, p.n, s, &a, &b);
        const SeqSums t = seq_sums<4>(p, a, b, at, lanes);
        double w[3] = {t.ratio, t.logp, t.count};
        wave_sums<3>(w);
        if (lane == 63) share[s * each + wave % each] = SeqSums{w[0], w[1], w[2]};
    }
    __syncthreads();
    if (wave == 0) {   // a lane a pair
        double v[kPairSums] = {};
        if (lane < p.n_pairs) {
            SeqSums sums[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                sums[k] = SeqSums{0.0, 0.0, 0.0};
#pragma unroll 1
                for (int e = 0; e < each; ++e) {
                    const SeqSums t = share[(2 * lane + k) * each + e];
                    sums[k].ratio += t.ratio;
                    sums[k].logp += t.logp;
                    sums[k].count += t.count;
                }
            }
            const PairLoss r = pair_loss(p, sums);
            grad[2 * lane] = r.grad[0];
            grad[2 * lane + 1] = r.grad[1];
            write_pair(p, lane, r, v);
        }
        wave_sums<kPairSums>(v);
        if (lane == 63) pair_outputs(v, p.n_pairs, p.scale, out);
    }
    __syncthreads();
#pragma unroll 1
    for (int s = wave / each; s < seqs; s += turn) {
        int a, b;
        seq_range(p.offs, p.n, s, &a, &b);
        write_grads<4>(p, a, b, at, lanes, grad[s]);
    }
}

// Workgroups a sequence where pairs alone do not fill the chip and are long
// enough to cut (0: a workgroup a pair): one pair of 2 x 20000 10.7 us (uncut
// 17.2), 8 of them 12.1 (17.6), 128 20.2 (21.0), 200 25.5 (23.0); 8 of 2 x 8192
// 11.9 (12.4).
int preference_cuts(int n, int n_pairs) {
    if (n_pairs > 128 || n / n_pairs < 16384) return 0;
    const int want = 1024 / (2 * n_pairs);
    return want < kMaxCuts ? want : kMaxCuts;
}

// Lanes that count a sequence: a mask of one sequence of 2^20 tokens takes 17
// us more than none with 1024, 53 with 256; of 8 x 131072 4.5 and 9; of 512 x
// 1500 with 256 lanes 5.
int count_lanes(const PolicyArgs& p) {
    const int mean = p.n / p.n_seqs;
    return mean > 16384 ? 1024 : mean > 1024 ? 256 : 64;
}

}  // namespace

// counts, count partials, loss partials
PolicyWs policy_ws(const PolicyArgs& p, void* ws) {
    char* w = static_cast<char*>(ws);
    PolicyWs r{nullptr, nullptr, 0, nullptr};
    if (policy_needs_counts(p)) {
        r.counts = reinterpret_cast<int32_t*>(w);
        r.cparts = reinterpret_cast<CountPart*>(w + align256(static_cast<size_t>(p.n_seqs) * sizeof(int32_t)));
        const int nc = count_lanes(p) > 64 ? p.n_seqs : (p.n_seqs + kWaves - 1) / kWaves;
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
    const int lanes = count_lanes(p);
    const auto kernel = lanes == 1024 ? policy_count_kernel<1024> : lanes == 256 ? policy_count_kernel<256> : policy_count_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3(w.n_cparts), dim3(lanes > kThreads ? lanes : kThreads), 0, s, p.n, p.n_seqs, p.offs, p.mask,
                       w.counts, w.cparts);
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
        hipLaunchKernelGGL((tokens_per_lane(p.n) == 1 ? policy_loss_kernel<1> : policy_loss_kernel<2>), dim3(nb), dim3(kThreads), 0, s, p, logp, ent, w.counts, w.cparts, w.n_cparts,
                           d_logp, d_ent, w.parts);
    if (e == hipSuccess) e = launch_policy_final(p, w, nb, out, s);
    return e;
}

size_t preference_ws_bytes(int n, int n_pairs) {
    if (preference_small(n, n_pairs)) return 0;
    return align256(static_cast<size_t>(n_pairs) * kPairSums * sizeof(double)) +
           align256(static_cast<size_t>(preference_cuts(n, n_pairs)) * 2 * n_pairs * sizeof(SeqSums));
}

hipError_t launch_preference_loss(const PrefArgs& p, float* out, void* ws, hipStream_t s) {
    if (preference_small(p.n, p.n_pairs)) {
        hipLaunchKernelGGL(preference_small_kernel, dim3(1), dim3(kSmallThreads), 0, s, p, out);
        return hipGetLastError();
    }
    double* parts = static_cast<double*>(ws);
    if (const int cuts = preference_cuts(p.n, p.n_pairs); cuts > 0) {
        SeqSums* shares = reinterpret_cast<SeqSums*>(static_cast<char*>(ws) +
                                                     align256(static_cast<size_t>(p.n_pairs) * kPairSums * sizeof(double)));
        hipLaunchKernelGGL(preference_sums_kernel, dim3(cuts, 2 * p.n_pairs + 1), dim3(kCutThreads), 0, s, p, shares);
        hipLaunchKernelGGL(preference_cut_kernel, dim3(cuts, 2 * p.n_pairs), dim3(kCutThreads), 0, s, p, shares, parts);
    } else {
        hipLaunchKernelGGL(preference_kernel, dim3(p.n_pairs + 1), dim3(kPairThreads), 0, s, p, parts);
    }
    hipLaunchKernelGGL(preference_final_kernel, dim3(1), dim3(kFinalThreads), 0, s, parts, p.n_pairs, p.scale, out);
    return hipGetLastError();
}

}  // namespace rl
