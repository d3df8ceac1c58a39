// train.h -- device-side pieces that the training-stage kernels share: which
// tokens count and with what weight, and the clipped policy loss of one token.
#pragma once

#include "rl_device.h"
#include "rl_internal.h"

namespace rl {

// First and one-past-last token of sequence s, inside [0, n] whatever the offsets hold.
__device__ __forceinline__ void seq_range(const int32_t* offs, int n, int s, int* a, int* b) {
    const int lo = offs ? offs[s] : 0, hi = offs ? offs[s + 1] : n;
    *a = lo < 0 ? 0 : lo > n ? n : lo;
    *b = hi < *a ? *a : hi > n ? n : hi;
}

// Entries of offs[lo .. hi) that are at most i (the entries do not decrease).
__device__ __forceinline__ int count_upto(const int32_t* offs, int lo, int hi, int i) {
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (offs[mid] <= i) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Sequence of token i, or -1, by a whole wave (i the same in every lane): 64
// probes a round, two rounds up to 4095 sequences.
__device__ __forceinline__ int seq_of_wave(const int32_t* offs, int n_seqs, int i) {
    if (!offs) return 0;
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n_seqs + 1;   // the first entry above i is in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6;
        const int at = lo + (lane + 1) * step - 1;
        const int c = __popcll(__ballot(at < hi && offs[at < hi ? at : hi - 1] <= i));
        lo += c * step;
        hi = lo + step - 1 < hi ? lo + step - 1 : hi;
        lo = lo < hi ? lo : hi;
    }
    return lo - 1 < n_seqs ? lo - 1 : -1;
}

// Sequence of row i when its token counts, else -1 (the whole wave asks for one row).
__device__ __forceinline__ int counted_seq(const PolicyArgs& p, int i) {
    return p.mask && !p.mask[i] ? -1 : seq_of_wave(p.offs, p.n_seqs, i);
}

// The policy and KL terms of one counted token and their derivatives by its
// log-probability.  fp64 throughout: a ratio next to a clip border falls on
// the side that its inputs say, and a few hundred fp64 operations a token
// cost less than reading it.  NaN passes every comparison and clamp below.
struct TokenLoss {
    double pg, kl, g, lr;
    bool clipped, dual;
};
// exp(x) - 1 for |x| <= 20 in fp64: with e = exp(x / 2^14) - 1 from its series
// (x / 2^14 is at most 1.3e-3: the term after the fifth is 4e-21), fourteen
// times e <- e (2 + e), each of which doubles the argument.  Within 2e-14 of
// the value, with five constants where the library's exp and expm1 have some
// fifty: beside a row in registers those do not fit.
__device__ __forceinline__ double expm1_20(double x) {
    const double r = x * (1.0 / 16384.0);
    double e = r * (1.0 + r * (0.5 + r * (1.0 / 6.0 + r * (1.0 / 24.0 + r * (1.0 / 120.0)))));
#pragma unroll 1
    for (int i = 0; i < 14; ++i) e = e * (2.0 + e);
    return e;
}

// exp(x) for any x <= 0: x = k ln 2 + r.  ln 2 in two parts: rounded to 40 bits behind the point, so that k times it is
// exact (k has 11 bits here), and what is left.
__device__ __forceinline__ double exp_below(double x) {
    const double lim = x < -1100.0 ? -1100.0 : x;
    const double k = rint(lim * 1.4426950408889634);
    const double r = (lim - k * (762123384786.0 / 1099511627776.0)) + k * 1.7239444525614835e-13;
    return ldexp(1.0 + expm1_20(r), static_cast<int>(k));
}

// ln(1 + e) for 0 <= e <= 1 in fp64: with y near it, ln(1 + e) = y + ln(1 + d), d = (e - E) / (1 + E), E = exp(y) - 1.
__device__ __forceinline__ double log1p_unit(double e) {
    const double y = e < 1e-3 ? e : static_cast<double>(__builtin_amdgcn_logf(static_cast<float>(1.0 + e))) * 0.69314718055994530942;
    const double E = expm1_20(y), d = (e - E) / (1.0 + E);
    return y + d * (1.0 - 0.5 * d);
}

// ln s in fp64 for a positive fp32 sum: the exponent, the hardware's logarithm
// of the mantissa in [1, 2) and one Newton step; 0 for 1, NaN for 0 and NaN.
__device__ __forceinline__ double ln_sum(float s) {
    const float m = 2.0f * __builtin_amdgcn_frexp_mantf(s);
    const double y = static_cast<double>(__builtin_amdgcn_logf(m)) * 0.69314718055994530942;
    const double d = m * (1.0 + expm1_20(-y)) - 1.0;
    return (__builtin_amdgcn_frexp_expf(s) - 1) * 0.69314718055994530942 + (y + d * (1.0 - 0.5 * d));
}

__device__ __forceinline__ double clamp20(double x) { return x < -20.0 ? -20.0 : x > 20.0 ? 20.0 : x; }
__device__ __forceinline__ TokenLoss policy_token(const PolicyArgs& p, double logp, double old_logp, double ref, double A) {
    TokenLoss t;
    t.lr = logp - old_logp;
    const double lr = clamp20(t.lr);
    const double r = 1.0 + expm1_20(lr);
    t.clipped = (A > 0.0 && r > p.hi) || (A < 0.0 && r < p.lo);
    t.dual = p.dual > 0.0 && A < 0.0 && r > p.dual;
    const double bound = A > 0.0 ? p.hi : p.lo;
    t.pg = -A * (t.dual ? p.dual : t.clipped ? bound : r);
    t.g = t.clipped || t.dual || lr != t.lr ? 0.0 : -A * r;
    if (t.lr != t.lr) t.g = t.lr;
    t.kl = 0.0;
    if (p.ref) {
        const double raw = ref - logp, d = clamp20(raw);
        double dk;
        if (p.kl == 1) {
            t.kl = -d;
            dk = 1.0;
        } else if (p.kl == 2) {
            t.kl = 0.5 * d * d;
            dk = -d;
        } else {
            const double e = expm1_20(d);
            t.kl = e - d;
            dk = -e;
        }
        if (p.kl_coef != 0.0 && (d == raw || d != d)) t.g += p.kl_coef * dk;
    }
    return t;
}

// Entry i of an array of fewer than 2^30 entries: scalar base, 32-bit offset.
template <typename T> __device__ __forceinline__ T* nth(T* p, int i) {
    return reinterpret_cast<T*>(reinterpret_cast<char*>(p) + static_cast<uint32_t>(i) * static_cast<uint32_t>(sizeof(T)));
}
template <typename T> __device__ __forceinline__ const T* nth(const T* p, int i) {
    return reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) +
                                      static_cast<uint32_t>(i) * static_cast<uint32_t>(sizeof(T)));
}

__device__ __forceinline__ int wave_sum(int v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// What the weights divide by: counted tokens, sequences that have some.
struct PolicyTotals { int tokens, seqs; };

// Called by every lane of every wave; each wave sums for itself.  Without
// counts (cparts null) no mask takes a token out, and they come from the offsets.
__device__ __forceinline__ PolicyTotals policy_totals(const PolicyArgs& p, const CountPart* cparts, int n_cparts) {
    const int lane = threadIdx.x & 63;
    PolicyTotals t{0, 0};
    if (p.agg == 2) return t;
    if (cparts) {
        for (int k = lane; k < n_cparts; k += 64) { t.tokens += cparts[k].tokens; t.seqs += cparts[k].seqs; }
    } else if (p.agg == 1) {
        for (int s = lane; s < p.n_seqs; s += 64) {
            int a, b;
            seq_range(p.offs, p.n, s, &a, &b);
            t.tokens += b - a;
            t.seqs += b > a;
        }
    } else {
        int a, b, e;
        seq_range(p.offs, p.n, 0, &a, &b);
        seq_range(p.offs, p.n, p.n_seqs - 1, &e, &b);
        return PolicyTotals{b - a, 0};
    }
    return PolicyTotals{wave_sum(t.tokens), wave_sum(t.seqs)};
}

// Weight of a counted token of sequence s.
__device__ __forceinline__ double policy_weight(const PolicyArgs& p, const PolicyTotals& t, int s, const int32_t* counts) {
    double by = p.agg == 0 ? t.tokens : 1.0;
    if (p.agg == 1) {
        int a, b;
        if (counts) {
            b = counts[s];
        } else {
            seq_range(p.offs, p.n, s, &a, &b);
            b -= a;
        }
        by = static_cast<double>(b) * t.seqs;
    }
    return 1.0 / by;
}

}  // namespace rl
