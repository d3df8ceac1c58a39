// k_logprob.hip -- token log-probabilities and entropies from logits, and the
// gradient of both to the logits.
//
// With c = log2(e) / T, t_v = (z_v - m) c, m the row's largest logit,
// s = sum 2^t_v and u = sum 2^t_v t_v:
//   log p_y = (z_y - m) / T - ln s        H = ln s - ln 2 u / s
//   d z_v   = (g (1[v = y] - p_v) - ge p_v (ln p_v + H)) / T
// Exponents are one fma, z c - R: R stands for m c, and what rounding it costs
// cancels (sums carry the R they are relative to; a gradient's factor takes
// 2^(R rounded - R)).  A row with m c past 2^28, where that rounding is more
// than 8, or without a sum (logits of the type's lowest value and nothing
// else) is summed again with the difference before the product; a gradient
// takes it first from 2^24 on.
#include "rl_device.h"
#include "rl_internal.h"
#include "train.h"

#include <cfloat>

namespace rl {

namespace {

// 16 bytes of logits at any element boundary.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> constexpr int kVec = 16 / sizeof(T);

template <typename T> __device__ __forceinline__ void unpack(u32x4 w, float* v);
template <> __device__ __forceinline__ void unpack<float>(u32x4 w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void unpack<uint16_t>(u32x4 w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
template <typename T> __device__ __forceinline__ u32x4 pack(const float* v);
template <> __device__ __forceinline__ u32x4 pack<float>(const float* v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
    return w;
}
template <> __device__ __forceinline__ u32x4 pack<uint16_t>(const float* v) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)   // one v_cvt_pk_bf16_f32 (round to nearest even)
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * i], v[2 * i + 1]}, bf16x2));
    return w;
}
// A vector of -inf.
template <typename T> __device__ __forceinline__ u32x4 nothing();
template <> __device__ __forceinline__ u32x4 nothing<float>() { return u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u}; }
template <> __device__ __forceinline__ u32x4 nothing<uint16_t>() { return u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}; }

// Vector `first` of a row plus a lane's byte offset: scalar base, 32-bit lane offset.
template <typename T> __device__ __forceinline__ T* vec_at(T* row, int first, uint32_t at) {
    return reinterpret_cast<T*>(reinterpret_cast<char*>(row) + static_cast<size_t>(first) * 16 + at);
}
template <typename T> __device__ __forceinline__ const T* vec_at(const T* row, int first, uint32_t at) {
    return reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + static_cast<size_t>(first) * 16 + at);
}

// Logits are streamed: non-temporal loads where nothing reads them again soon
// (8192 x 152064 bf16 log-probabilities in 364 us, 6.8 TB/s; plain loads 410),
// plain ones where the backward pass will, which then finds part of them in
// the memory-side cache (both passes over 437 MB in 218 us and 230, over 1.2
// GB in 582 and 596; gradients stored plainly and read plainly 262 and 689).
// The gradient is stored non-temporally: 1792 x 32000 rows to gradients in 63
// us, plainly 70, and with a reader of the gradient behind it 84 and 85.
template <bool KEEP, typename T> __device__ __forceinline__ u32x4 load_row(const T* p) {
    const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p);
    return KEEP ? *q : __builtin_nontemporal_load(q);
}
template <typename T> __device__ __forceinline__ void store_row(T* p, u32x4 w) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any*>(p));
}

// Smallest exponent that enters a product: 2^kFloor is 0 in fp32, so an entry
// of probability 0 adds 0 instead of 0 x inf.
constexpr float kFloor = -200.0f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The sums of a part of a row relative to another m.
__device__ __forceinline__ void rebase(RowPart& a, float m, float c) {
    const float d = fmaxf((a.m - m) * c, -1e4f), f = exp2_hw(d);
    a.u = f * (a.u + d * a.s);
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ RowPart merge(RowPart a, RowPart b, float c) {
    const float m = fmaxf(a.m, b.m);
    rebase(a, m, c);
    rebase(b, m, c);
    return RowPart{m, a.s + b.s, a.u + b.u};
}

// A lane's running sums, relative to 2^R.  R stays until an entry lies more
// than 2^64 above it: moving it to every new maximum would cost an exponential
// in nearly every vector of a wave (some lane always has one).
struct LaneSum { float R, s, u, top; };   // top: the largest entry
constexpr float kAhead = 64.0f, kNowhere = -1e30f;
__device__ __forceinline__ LaneSum empty_sum() { return LaneSum{kNowhere, 0.0f, 0.0f, -FLT_MAX}; }

template <int N, bool ENT> __device__ __forceinline__ void add_entries(LaneSum& a, const float* v, float c) {
    float x = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) x = fmaxf(x, v[i]);
    a.top = fmaxf(a.top, x);
    if (__builtin_fmaf(x, c, -a.R) > kAhead) {
        const float R = x * c, d = fmaxf(a.R - R, -1e4f), f = exp2_hw(d);
        if (ENT) a.u = f * (a.u + d * a.s);
        a.s *= f;
        a.R = R;
    }
    // The vector's own sums first: a small entry leaves no trace in a sum of hundreds (log-probabilities under 152064
    // logits at T = 0.6 were 6.4e-7 too high on average, 7.4e-7 off in the mean square; now 5e-8 and 3.0e-7, of which
    // rounding them to fp32 is 2.8e-7).
    float s = 0.0f, u = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = __builtin_fmaf(v[i], c, -a.R), e = exp2_hw(t);
        s += e;
        if (ENT) u += e * fmaxf(t, kFloor);
    }
    a.s += s;
    if (ENT) a.u += u;
}
// The same relative to the lane's largest entry.  Without ENT, u is for straight() alone: every entry counts as the
// lane's largest.
template <bool ENT> __device__ __forceinline__ RowPart close_sum(const LaneSum& a, float c) {
    const float d = a.s == 0.0f ? 0.0f : fmaxf(__builtin_fmaf(-a.top, c, a.R), -1e4f), f = exp2_hw(d);
    return RowPart{a.top, f * a.s, ENT ? f * (a.u + d * a.s) : 0.0f};
}

// A lane's value moved by register (`old` where the control names no lane or the row of 16 is masked).
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float old, float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(v), CTRL, ROWS, 0xF, false));
}
template <int LANE> __device__ __forceinline__ float of_lane(float v) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), LANE));
}
// Over the first N lanes, 16 or 64: to the right within rows of 16, then row to row.
template <int N> __device__ __forceinline__ float max_of(float v) {
    v = fmaxf(v, moved<0x111, 0xF>(v, v));
    v = fmaxf(v, moved<0x112, 0xF>(v, v));
    v = fmaxf(v, moved<0x114, 0xF>(v, v));
    v = fmaxf(v, moved<0x118, 0xF>(v, v));
    if (N == 64) {
        v = fmaxf(v, moved<0x142, 0xA>(v, v));
        v = fmaxf(v, moved<0x143, 0xC>(v, v));
    }
    return of_lane<N - 1>(v);
}
template <int N> __device__ __forceinline__ float sum_of(float v) {
    v += moved<0x111, 0xF>(0.0f, v);
    v += moved<0x112, 0xF>(0.0f, v);
    v += moved<0x114, 0xF>(0.0f, v);
    v += moved<0x118, 0xF>(0.0f, v);
    if (N == 64) {
        v += moved<0x142, 0xA>(0.0f, v);
        v += moved<0x143, 0xC>(0.0f, v);
    }
    return of_lane<N - 1>(v);
}
// The sums of the first N lanes' parts, the same bits in every lane.
template <int N> __device__ __forceinline__ RowPart merge_of(RowPart a, float c) {
    const float m = max_of<N>(a.m);
    rebase(a, m, c);
    return RowPart{m, sum_of<N>(a.s), sum_of<N>(a.u)};
}

// Over a workgroup, the same bits in every lane.
template <int WAVES> __device__ __forceinline__ RowPart merge_workgroup(RowPart a, RowPart* sp, float c) {
    static_assert(WAVES <= 16);
    a = merge_of<64>(a, c);
    const int lane = threadIdx.x & 63;
    if (lane == 0) sp[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lane < WAVES ? sp[lane] : RowPart{-FLT_MAX, 0.0f, 0.0f};
    return merge_of<16>(a, c);
}

// Whether the sums stand: at least the largest entry's 1, no NaN, and an R whose rounding (half a step of fp32 at m c: 8 at
// 2^28) stays far from kAhead and from what an exponential can hold.  One rounded by more than kAhead would move again at
// every entry, by what its rounding was, and take the sums before it away.  (Entries that far below m end as 0, but for a u
// that they made infinite.)
constexpr float kFarSum = 268435456.0f;
__device__ __forceinline__ bool stands(const RowPart& a, float c) {
    return a.s > 0.5f && a.s < FLT_MAX && fabsf(a.u) < FLT_MAX && fabsf(a.m * c) < kFarSum;
}

// Entries [0, n) again, with the difference to m before the product.
template <typename T, int WAVES> __device__ __forceinline__ RowPart sums_again(const T* z, int n, float m, float c, RowPart* sp) {
    RowPart a{m, 0.0f, 0.0f};
    for (int v = threadIdx.x; v < n; v += 64 * WAVES) {
        const float t = (Elem<T>::load(z, v) - m) * c, e = exp2_hw(t);
        a.s += e;
        a.u += e * fmaxf(t, kFloor);
    }
    __syncthreads();   // sp is free
    return merge_workgroup<WAVES>(a, sp, c);
}

// ln sum exp((z - m) / T): of the sum with c in fp32, ln s, plus what c's rounding did to it, (log2(e) / T - c) / c =
// bend / ln 2 times the mean of ln 2 t.  Near 1e-8 times 5 to 20, but the same way for every row.
__device__ __forceinline__ double straight(double ln_c, const RowPart& a, float bend) {
    return a.s > 1.0f ? ln_c + bend * (a.u / a.s) : ln_c;
}

template <typename T>
__device__ __forceinline__ void finish_row(RowPart a, const T* z, int V, int y, double inv_T, float bend, int row, float* logp,
                                           float* ent, float* stats, float* rest) {
    const double ln_c = ln_sum(a.s), ln_s = straight(ln_c, a, bend);
    double lp = __builtin_nan("");
    if (y >= 0 && y < V) lp = (static_cast<double>(Elem<T>::load(z, y)) - a.m) * inv_T - ln_s;
    lp = lp > 0.0 ? 0.0 : lp;
    const float lp32 = static_cast<float>(lp);
    logp[row] = lp32;
    if (rest) rest[row] = lp32 < -FLT_MAX ? 0.0f : static_cast<float>(lp - lp32);
    if (ent) {
        const double h = ln_c - 0.69314718055994530942 * static_cast<double>(a.u / a.s);
        ent[row] = static_cast<float>(h < 0.0 ? 0.0 : h);
    }
    if (stats) {
        stats[2 * static_cast<size_t>(row)] = a.m;
        stats[2 * static_cast<size_t>(row) + 1] = static_cast<float>(ln_s);
    }
}

__device__ __forceinline__ void finish_dead(int row, float* logp, float* ent, float* stats) {
    logp[row] = 0.0f;
    if (ent) ent[row] = 0.0f;
    if (stats) stats[2 * static_cast<size_t>(row)] = stats[2 * static_cast<size_t>(row) + 1] = 0.0f;
}

constexpr int kRowThreads = 256;

// One workgroup per (row, vocabulary chunk), four vectors a lane in flight;
// chunks of a row are merged in order by token_logprobs_join_kernel.  One
// read of the logits and one exponential an entry: bound by memory (8192 x
// 152064 bf16, 2.5 GB, 366 us, 6.8 TB/s; 1792 x 32000 21 us, 24 with nothing
// of them in the caches, 4.8 TB/s), few rows by a row's own latency.
template <typename T, int THREADS, bool ENT, bool KEEP>
__global__ void __launch_bounds__(THREADS) token_logprobs_kernel(const T* __restrict__ logits, int64_t ld, int V,
        const int32_t* __restrict__ targets, double inv_T, float c, float bend, int chunk, bool check, PolicyArgs live,
        RowPart* __restrict__ parts, float* __restrict__ logp, float* __restrict__ ent, float* __restrict__ stats) {
    constexpr int E = kVec<T>, U = 4, WAVES = THREADS / 64;
    __shared__ RowPart sp[WAVES];
    const int row = blockIdx.x, nchunks = gridDim.y, tid = threadIdx.x;
    if (check && counted_seq(live, row) < 0) {
        if (tid == 0 && nchunks == 1) finish_dead(row, logp, ent, stats);
        return;
    }
    const int beg = blockIdx.y * chunk, end = min(V, beg + chunk);
    const T* z = logits + row * ld + beg;
    LaneSum acc = empty_sum();
    const int nvec = (end - beg) / E, tail = end - beg - nvec * E;
    const float last = tid < tail ? Elem<T>::load(z, nvec * E + tid) : -INFINITY;
    int v = tid;
#pragma unroll 1
    for (; v + (U - 1) * THREADS < nvec; v += U * THREADS) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_row<KEEP>(z + static_cast<size_t>(v + u * THREADS) * E);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[E];
            unpack<T>(w[u], x);
            add_entries<E, ENT>(acc, x, c);
        }
    }
    if (v < nvec) {   // up to U - 1 vectors more; what is not there is -inf
        u32x4 w[U - 1];
#pragma unroll
        for (int u = 0; u < U - 1; ++u) {
            w[u] = nothing<T>();
            if (v + u * THREADS < nvec) w[u] = load_row<KEEP>(z + static_cast<size_t>(v + u * THREADS) * E);
        }
#pragma unroll
        for (int u = 0; u < U - 1; ++u) {
            float x[E];
            unpack<T>(w[u], x);
            add_entries<E, ENT>(acc, x, c);
        }
    }
    add_entries<1, ENT>(acc, &last, c);
    RowPart a = merge_workgroup<WAVES>(close_sum<ENT>(acc, c), sp, c);
    if (!stands(a, c)) a = sums_again<T, WAVES>(z, end - beg, a.m, c, sp);
    if (tid != 0) return;
    if (nchunks > 1)
        parts[static_cast<size_t>(row) * nchunks + blockIdx.y] = a;
    else
        finish_row(a, z, V, targets[row], inv_T, bend, row, logp, ent, stats, live.rest);
}

// One wave per row.
template <typename T>
__global__ void __launch_bounds__(64) token_logprobs_join_kernel(const RowPart* __restrict__ parts, int nchunks,
        const T* __restrict__ logits, int64_t ld, int V, const int32_t* __restrict__ targets, double inv_T, float c, float bend,
        bool check, PolicyArgs live, float* __restrict__ logp, float* __restrict__ ent, float* __restrict__ stats) {
    const int row = blockIdx.x;
    if (check && counted_seq(live, row) < 0) {
        if (threadIdx.x == 0) finish_dead(row, logp, ent, stats);
        return;
    }
    RowPart a{-FLT_MAX, 0.0f, 0.0f};
    for (int k = threadIdx.x; k < nchunks; k += 64) a = merge(a, parts[static_cast<size_t>(row) * nchunks + k], c);
    a = merge_of<64>(a, c);
    if (threadIdx.x == 0) finish_row(a, logits + row * ld, V, targets[row], inv_T, bend, row, logp, ent, stats, live.rest);
}

// Gradients of a row's entries (the same row in every lane): with q = z c - K, 2^q (A + B q); K = m c + log2 s
// rounded to fp32, and A and B make up for that.  `top` is the target's own, with 1 - p_y as -(exp(log p_y) - 1): a token
// that is certain has none where its lane's sum is relative to it, else a few 2^-23 of g (its term is 2^t 2^-t then).
struct RowGrad {
    float K, A, B, top;
    float m, l2;
    bool zero, far;   // far: K is past kFar, q = (z - m) c - l2
};
// Rounding K to fp32 moves it by half a step, 1/2 up to here; past 2^32 the factor that makes up for it would not be finite.
constexpr double kFar = 16777216.0;
// ln_s: ln s; lp: log p_y; i: 1 / T
__device__ __forceinline__ RowGrad row_grad(float g, float ge, float H, float i, float m, double ln_s, double lp, float c) {
    RowGrad k;
    const double l2 = ln_s * 1.4426950408889634, K = static_cast<double>(m) * c + l2;
    k.K = static_cast<float>(K);
    k.m = m;
    k.l2 = static_cast<float>(l2);
    k.far = __builtin_amdgcn_readfirstlane(!(fabs(K) < kFar));
    const float off = k.far ? 0.0f : static_cast<float>(static_cast<double>(k.K) - K), f = exp2_hw(off);
    k.B = -ge * 0.69314718f * i;
    k.A = f * (-(g + ge * H) * i + k.B * off);
    k.B *= f;
    const double q = lp < -140.0 ? -140.0 : lp;
    const float p = exp2_hw(static_cast<float>(q * 1.4426950408889634));
    k.top = i * (static_cast<float>(-g * expm1_20(clamp20(lp))) - ge * p * (static_cast<float>(q) + H));
    k.zero = __builtin_amdgcn_readfirstlane(g == 0.0f && ge == 0.0f);
    return k;
}
template <bool ENT> __device__ __forceinline__ float grad_of(const RowGrad& k, float q) {
    return exp2_hw(q) * (ENT ? k.A + k.B * fmaxf(q, kFloor) : k.A);
}
// Of N entries; y: the target's place among them.
template <int N, bool ENT> __device__ __forceinline__ void grad_entries(const RowGrad& k, float* x, float c, int y) {
    if (k.far) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = (x[j] - k.m) * c - k.l2;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = __builtin_fmaf(x[j], c, -k.K);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = grad_of<ENT>(k, x[j]);
    if (static_cast<uint32_t>(y) < static_cast<uint32_t>(N)) {   // one lane of a row
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = j == y ? k.top : x[j];
    }
}

// A workgroup a chunk of a row, two 16-byte vectors a lane: the row's logarithm, the target's gradient and the factors are
// worked out once a lane, in fp64, and then each vector is a load, an exponential an entry and a store.  Bound by memory:
// 4096 x 151936 bf16, 2.5 GB in and out, 406 us (6.1 TB/s, part of the logits from the cache that the forward pass has
// filled), with one vector a lane 428, with four 412, eight 457; 24 rows 5.5 us (5.7, 5.7 and 6.8); 2048 x 20000 fp32 53
// (four 56, eight 61).
template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowThreads) token_logprobs_backward_kernel(const T* logits, int64_t ld, int V,
        const int32_t* __restrict__ targets, double inv_T, float c, const float* __restrict__ stats,
        const float* __restrict__ ent, const float* __restrict__ d_logp, const float* __restrict__ d_ent, int chunk, T* dz,
        int64_t ldd) {
    const int row = blockIdx.y;
    const int beg = blockIdx.x * chunk, n = min(V, beg + chunk) - beg, tid = threadIdx.x;
    const T* z = logits + row * ld + beg;
    T* d = dz + row * ldd + beg;
    int y = targets[row];
    const float g = y >= 0 && y < V ? d_logp[row] : 0.0f, ge = ENT ? d_ent[row] : 0.0f;
    y -= beg;
    const float m = stats[2 * static_cast<size_t>(row)];
    const double ln_s = stats[2 * static_cast<size_t>(row) + 1];
    double lp = y >= 0 && y < n ? (static_cast<double>(Elem<T>::load(z, y)) - m) * inv_T - ln_s : 0.0;
    lp = lp > 0.0 ? 0.0 : lp;
    const RowGrad k = row_grad(g, ge, ENT ? ent[row] : 0.0f, static_cast<float>(inv_T), m, ln_s, lp, c);
    constexpr int E = kVec<T>;
    const int whole = n / E * E;
    for (int v = E * tid; v < whole; v += E * kRowThreads) {
        float x[E] = {};
        if (!k.zero) {
            unpack<T>(load_row<false>(z + v), x);
            grad_entries<E, ENT>(k, x, c, y - v);
        }
        store_row(d + v, pack<T>(x));
    }
    const int v = whole + tid;
    if (v < n) {
        float x = 0.0f;
        if (!k.zero) {
            x = Elem<T>::load(z, v);
            grad_entries<1, ENT>(k, &x, c, y - v);
        }
        Elem<T>::store(d, v, x);
    }
}

// ---- the policy loss of a row and the gradient of its logits, the row read once ----

// The row's 16-byte vectors stay in registers (NV a lane, vector i * THREADS +
// lane) from the load to the gradient: sums as the loads arrive, one barrier,
// the token's loss, then each vector's gradient is stored.  HBM traffic is one
// read and one write of the logits where the forward and backward kernels need
// two reads.  A lane's entries behind the row's last vector are -inf.
// Workgroups stay and take rows in turn; the next row's vectors are loaded as
// this row's gradients leave the registers.  Bound by memory: 8192 x 152064
// bf16 with a tenth of the tokens masked, 2.24 GB in and 2.49 GB out, 990 us
// (4.8 TB/s, where a copy of 2 GiB reaches 4.95); 1792 x 32000, 229 MB, 49 us
// (4.7).  Loads pause while a row is summed.  Of 128 registers a lane, 20
// vectors leave too few for the rest: by the compiler's report those forms keep
// 10 (bf16) or 27-28 (fp32) registers in scratch, 28 and 96-100 bytes a lane,
// those of 16 vectors 2 (bf16, 12 bytes) or 9-10 (fp32, 24-28), others none.
template <typename T, int THREADS, int NV, bool ENT>
__global__ void __launch_bounds__(THREADS, 4) policy_rows_kernel(PolicyArgs p, const int32_t* __restrict__ counts,
        const CountPart* __restrict__ cparts, int n_cparts, const T* logits, int64_t ld, int V,
        const int32_t* __restrict__ targets, double inv_T, float c, float bend, T* dz, int64_t ldd, float* __restrict__ logp,
        float* __restrict__ ent, double* __restrict__ parts) {
    constexpr int E = kVec<T>, WAVES = THREADS / 64;
    __shared__ RowPart sp[2][WAVES];
    __shared__ double sums[kPolicySums];   // of this workgroup's rows, the first lane's
    const int tid = threadIdx.x;
    const int nvec = V / E, tail = V - nvec * E;
    const uint32_t at = tid * 16;
    u32x4 w[NV];
    float last = -INFINITY;
    if (tid == 0)
        for (int q = 0; q < kPolicySums; ++q) sums[q] = 0.0;
    int row = blockIdx.x;
    int seq = counted_seq(p, row);
    const PolicyTotals totals = policy_totals(p, cparts, n_cparts);
#pragma unroll
    for (int i = 0; i < NV; ++i) w[i] = nothing<T>();
    if (seq >= 0) {
        const T* z = logits + row * ld;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (tid < nvec - i * THREADS) w[i] = load_row<false>(vec_at(z, i * THREADS, at));
        if (tid < tail) last = Elem<T>::load(z, nvec * E + tid);
    }
    int turn = 0;   // half of sp: of two rows in a row that use it, the second has a barrier behind the first's reads
    while (row < p.n) {
        const int next = row + gridDim.x;
        const int next_seq = next < p.n ? counted_seq(p, next) : -1;
        const T* zn = logits + next * ld;
        T* d = dz + row * ldd;
        RowGrad k{};
        k.zero = true;
        int y = -1;
        if (seq < 0) {
            if (tid == 0) {
                logp[row] = 0.0f;
                if (ent) ent[row] = 0.0f;
            }
        } else {
            y = targets[row];
            const bool held = y >= 0 && y < V;
            const float zy = held ? Elem<T>::load(logits + row * ld, y) : __builtin_nanf("");
            const double weight = policy_weight(p, totals, seq, counts);
            const float adv = p.adv[p.token_adv ? row : seq], old_logp = p.old_logp[row], ref = p.ref ? p.ref[row] : 0.0f;
            LaneSum acc = empty_sum();
            int nv = nvec;
            asm volatile("" : "+s"(nv));   // or the comparisons of every turn are kept in registers
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i * THREADS < nv) {
                    float x[E];
                    unpack<T>(w[i], x);
                    add_entries<E, ENT>(acc, x, c);
                }
                __builtin_amdgcn_sched_barrier(0);   // a vector at a time: unpacked ones would not fit beside the row
            }
            add_entries<1, ENT>(acc, &last, c);
            RowPart a = merge_workgroup<WAVES>(close_sum<ENT>(acc, c), sp[turn], c);
            if (!stands(a, c)) a = sums_again<T, WAVES>(logits + row * ld, V, a.m, c, sp[turn]);
            turn ^= 1;
            const double ln_c = ln_sum(a.s), ln_s = straight(ln_c, a, bend);
            double lp = (static_cast<double>(zy) - a.m) * inv_T - ln_s;
            lp = lp > 0.0 ? 0.0 : lp;
            const float lp32 = static_cast<float>(lp);
            float H = 0.0f;
            if (ENT) {
                const double h = ln_c - 0.69314718055994530942 * static_cast<double>(a.u / a.s);
                H = static_cast<float>(h < 0.0 ? 0.0 : h);
            }
            const TokenLoss t = policy_token(p, lp, old_logp, ref, adv);
            const float g = held ? static_cast<float>(p.scale * weight * t.g) : 0.0f;
            const float ge = ENT ? static_cast<float>(-p.scale * weight * p.ent_coef) : 0.0f;
            if (tid == 0) {
                logp[row] = lp32;
                if (ent) ent[row] = H;
                sums[0] += weight * t.pg;
                sums[1] += weight * t.kl;
                sums[2] += weight * H;
                sums[3] += t.clipped;
                sums[4] += t.dual;
                sums[5] -= t.lr;
                sums[6] += 1.0;
            }
            k = row_grad(g, ge, H, static_cast<float>(inv_T), a.m, ln_s, lp, c);
            if (!held) y = -1;
        }
        int nv = nvec;
        asm volatile("" : "+s"(nv));
        const int y_lane = y - tid * E;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            asm volatile("" : "+v"(w[i]));   // unpacked again: the values of the first pass would not fit beside the row
            if (tid < nv - i * THREADS) {
                float x[E] = {};
                if (!k.zero) {
                    unpack<T>(w[i], x);
                    grad_entries<E, ENT>(k, x, c, y_lane - i * THREADS * E);
                }
                store_row(vec_at(d, i * THREADS, at), pack<T>(x));
            }
            __builtin_amdgcn_sched_barrier(0);
            // Four stores, then four loads.  Compared in one sitting (the merge of a row's parts took 15 us more then: now
            // 990): 8192 rows of 152064 bf16 logits 1006 us, one by one 1019, in twos 1023, in eights 1013; a whole row of
            // stores first 992, and then 59 us for 1792 rows of 32000 where fours took 56 (now 50).
            if (next_seq >= 0 && (i % 4 == 3 || i == NV - 1)) {
#pragma unroll
                for (int j = i / 4 * 4; j <= i; ++j)
                    if (tid < nv - j * THREADS) w[j] = load_row<false>(vec_at(zn, j * THREADS, at));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (tid < tail) {
            float x = 0.0f;
            if (!k.zero) {
                x = last;
                grad_entries<1, ENT>(k, &x, c, y - nvec * E - tid);
            }
            Elem<T>::store(d, nvec * E + tid, x);
            if (next_seq >= 0) last = Elem<T>::load(zn, nvec * E + tid);
        }
        row = next;
        seq = next_seq;
    }
    if (tid == 0)
        for (int q = 0; q < kPolicySums; ++q) parts[static_cast<size_t>(blockIdx.x) * kPolicySums + q] = sums[q];
}

// How a row is cut.  A workgroup of 1024 lanes takes 7 us for 32000 bf16
// logits, 13 for 152064; cut into chunks of 256 lanes and joined by a second
// kernel 24 rows of 152064 take 8.3 (uncut 13.6), 128 rows 15.3 (16.3), 200
// rows 20 (17).  At 50000 entries the cut would save 1 us of the GPU's time and
// cost a launch.  Past 512 rows workgroups of 256 lanes fill the chip (600 rows
// of 32000: 13 us, with 1024 lanes 15; 400 rows 11.6 and 11.4; 256 rows of
// 152064: 30 and 18).
struct RowCut { int chunk, nchunks, threads; };
RowCut cut_rows(int n, int V) {
    if (n < 160 && V > 65536) {
        const int want = (512 + n - 1) / n, each = ((V + want - 1) / want + 2047) / 2048 * 2048;
        const int chunk = each < 4096 ? 4096 : each;
        return RowCut{chunk, (V + chunk - 1) / chunk, kRowThreads};
    }
    return RowCut{V, 1, n <= 512 && V > 8192 ? 1024 : kRowThreads};
}

float log2_scale(double T) { return static_cast<float>(1.4426950408889634 / T); }
float bend_of(double T) {
    return static_cast<float>((1.4426950408889634 / T / log2_scale(T) - 1.0) * 0.69314718055994530942);
}

template <typename T, int THREADS>
void launch_forward(const LogprobArgs& a, const RowCut& r, RowPart* parts, hipStream_t s) {
    const PolicyArgs live = a.live ? *a.live : PolicyArgs{};
    const bool keep = a.stats != nullptr;   // the backward pass follows
    const auto kernel = a.ent ? (keep ? token_logprobs_kernel<T, THREADS, true, true> : token_logprobs_kernel<T, THREADS, true, false>)
                              : (keep ? token_logprobs_kernel<T, THREADS, false, true> : token_logprobs_kernel<T, THREADS, false, false>);
    hipLaunchKernelGGL(kernel, dim3(a.n, r.nchunks), dim3(THREADS), 0, s, static_cast<const T*>(a.logits), a.ld, a.V, a.targets,
                       1.0 / a.T, log2_scale(a.T), bend_of(a.T), r.chunk, a.live != nullptr, live, parts, a.logp, a.ent, a.stats);
    if (r.nchunks > 1)
        hipLaunchKernelGGL(token_logprobs_join_kernel<T>, dim3(a.n), dim3(64), 0, s, parts, r.nchunks,
                           static_cast<const T*>(a.logits), a.ld, a.V, a.targets, 1.0 / a.T, log2_scale(a.T), bend_of(a.T),
                           a.live != nullptr, live, a.logp, a.ent, a.stats);
}

template <typename T> hipError_t forward(const LogprobArgs& a, RowPart* parts, hipStream_t s) {
    const RowCut r = cut_rows(a.n, a.V);
    if (r.threads == 1024) launch_forward<T, 1024>(a, r, parts, s);
    else launch_forward<T, kRowThreads>(a, r, parts, s);
    return hipGetLastError();
}

// Vectors a lane holds at most: 20 take 80 of the 128 registers that 16 waves
// a CU leave each lane.
constexpr int kRowVecs = 20;

template <typename T, int THREADS, int NV>
int rows(const PolicyArgs& p, const PolicyWs& w, const LogprobArgs& a, void* dz, int64_t ldd, hipStream_t s) {
    static_assert(kCUs * (1024 / THREADS) <= kPolicyMaxRowParts, "a workgroup's sums need a place in the workspace");
    const auto kernel = a.ent ? policy_rows_kernel<T, THREADS, NV, true> : policy_rows_kernel<T, THREADS, NV, false>;
    const int fit = kCUs * (1024 / THREADS), grid = a.n < fit ? a.n : fit;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(THREADS), 0, s, p, w.counts, w.cparts, w.n_cparts,
                       static_cast<const T*>(a.logits), a.ld, a.V, a.targets, 1.0 / a.T, log2_scale(a.T), bend_of(a.T),
                       static_cast<T*>(dz), ldd, a.logp, a.ent, w.parts);
    return grid;
}

// The narrowest workgroup that holds a row, so that a CU has up to four rows in different phases (1792 x 32000 bf16: 256
// lanes 49 us, 512 50, 1024 63; 8192 x 8000: 68, 98, 170); up to two rows a CU twice that (192 rows of 32000: 13.6 us, with
// 256 lanes 15.6; 500 of 40000: 20.2 and 22.1; 600 of 32000: 24.2 and 22.2).
template <typename T>
int rows_of(const PolicyArgs& p, const PolicyWs& w, const LogprobArgs& a, void* dz, int64_t ldd, hipStream_t s) {
    const int nvec = a.V / kVec<T>;
    if (nvec <= 4 * 256) return rows<T, 256, 4>(p, w, a, dz, ldd, s);
    if (nvec <= 8 * 256) return rows<T, 256, 8>(p, w, a, dz, ldd, s);
    const bool few = a.n <= 2 * kCUs;
    if (nvec <= 16 * 256 && !few) return rows<T, 256, 16>(p, w, a, dz, ldd, s);
    if (nvec <= 20 * 256 && !few) return rows<T, 256, 20>(p, w, a, dz, ldd, s);
    if (nvec <= 10 * 512) return rows<T, 512, 10>(p, w, a, dz, ldd, s);
    if (nvec <= 16 * 512) return rows<T, 512, 16>(p, w, a, dz, ldd, s);
    if (nvec <= 20 * 512) return rows<T, 512, 20>(p, w, a, dz, ldd, s);
    if (nvec <= 16 * 1024) return rows<T, 1024, 16>(p, w, a, dz, ldd, s);
    return rows<T, 1024, kRowVecs>(p, w, a, dz, ldd, s);
}

}  // namespace

// One kernel beside the forward, loss and backward kernels, whose times stand in brackets: one row of 4096 fp32 logits 9.5
// us (11.3), 32 of 32000 bf16 12.8 (14.4), one of 50000 14.6 (14.8).  Fewer than 96 wider rows are cut over the chip by
// those: one of 65536 15.9 (14.9), 32 of 152064 25.1 (19.1), 64 of 80000 18.9 (19.2), 96 of 152064 26.9 (29.1), 1024 of
// 152064 133 (162).
bool policy_rows_fit(int dt, int n, int V) {
    const int nvec = V / (dt == DT_F32 ? 4 : 8);
    return n >= (nvec <= 6 * 1024 ? 1 : 96) && nvec <= kRowVecs * 1024;
}

hipError_t launch_policy_rows(int dt, const PolicyArgs& p, const PolicyWs& w, const LogprobArgs& a, void* dz, int64_t ldd,
                              int* n_parts, hipStream_t s) {
    *n_parts = dt == DT_F32 ? rows_of<float>(p, w, a, dz, ldd, s) : rows_of<uint16_t>(p, w, a, dz, ldd, s);
    return hipGetLastError();
}

size_t logprob_parts(int n, int V) {
    if (n <= 0) return 0;
    const RowCut r = cut_rows(n, V);
    return r.nchunks > 1 ? static_cast<size_t>(n) * r.nchunks : 0;
}

hipError_t launch_token_logprobs(int dt, const LogprobArgs& a, RowPart* parts, hipStream_t s) {
    if (a.n <= 0) return hipSuccess;
    return dt == DT_F32 ? forward<float>(a, parts, s) : forward<uint16_t>(a, parts, s);
}

hipError_t launch_token_logprobs_backward(int dt, const void* logits, int64_t ld, int n, int V, const int32_t* targets,
                                          double T, const float* stats, const float* ent, const float* g,
                                          const float* ge, void* dz, int64_t ldd, hipStream_t s) {
    // rows in y, at most 65535 a launch
    constexpr int kRows = 32768;
    const size_t es = dt == DT_F32 ? 4 : 2;
    const int chunk = 2 * kRowThreads * static_cast<int>(16 / es), nchunks = (V + chunk - 1) / chunk;
    for (int r = 0; r < n; r += kRows) {
        const int m = n - r < kRows ? n - r : kRows;
        const char* z = static_cast<const char*>(logits) + es * ld * r;
        char* d = static_cast<char*>(dz) + es * ldd * r;
        const float* e = ent ? ent + r : nullptr;
        const float* h = ge ? ge + r : nullptr;
        if (dt == DT_F32)
            hipLaunchKernelGGL((h ? token_logprobs_backward_kernel<float, true> : token_logprobs_backward_kernel<float, false>),
                               dim3(nchunks, m), dim3(kRowThreads), 0, s, reinterpret_cast<const float*>(z), ld, V, targets + r,
                               1.0 / T, log2_scale(T), stats + 2 * r, e, g + r, h, chunk, reinterpret_cast<float*>(d), ldd);
        else
            hipLaunchKernelGGL((h ? token_logprobs_backward_kernel<uint16_t, true> : token_logprobs_backward_kernel<uint16_t, false>),
                               dim3(nchunks, m), dim3(kRowThreads), 0, s, reinterpret_cast<const uint16_t*>(z), ld, V,
                               targets + r, 1.0 / T, log2_scale(T), stats + 2 * r, e, g + r, h, chunk,
                               reinterpret_cast<uint16_t*>(d), ldd);
    }
    return hipGetLastError();
}

}  // namespace rl
