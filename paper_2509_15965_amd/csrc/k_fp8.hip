// k_fp8.hip -- numbers to 8 bits and back: RMS norm with the residual's addition,
// rows, SwiGLU's product, weight tiles, and the tokens of a paged K/V cache.
#include "fp8.h"
#include "rl_decode.h"

namespace rl {

namespace {

// ---------------------------------------------------------------------------
// RMS norm.  s = x + add (as stored), y = s w / sqrt(mean s^2 + eps), y in blocks of
// 128.  LANES lanes a row, a row in registers from its one read to its codes: NV
// times 16 bytes of x a lane.  Bound by memory: 8192 x 3584 in fp32 with a bf16
// branch, 323 MB, 64.9 us (5.0 TB/s, a copy's rate); 32 bytes of x a lane at a time, so that
// an instruction takes every other 16: a third more.  The arithmetic has room: sums,
// root and products are in 64 bits, so that a code is off only where 64 bits
// are (in fp32 20 of the 29 M codes round to a neighbour, in 62.8 us).
// ---------------------------------------------------------------------------
// 1 / sqrt(a) of a positive a: the hardware's, and two steps of Newton's method, which double its digits each
__device__ __forceinline__ double inverse_root(double a) {
    double y = __builtin_amdgcn_rsq(a);
    if (a < 1e300) {   // an infinite one stays 0
#pragma unroll
        for (int i = 0; i < 2; ++i) y = __builtin_fma(y, __builtin_fma(-0.5 * a * y, y, 0.5), y);
    }
    return y;
}

// x cut to 24 bits, the last of which is set where something was cut off: rounded once more, to fewer bits, that is x rounded
__device__ __forceinline__ float to_odd(double x) {
    const int lo = __double2loint(x), kept = lo & ~0x1FFFFFFF;
    return static_cast<float>(__hiloint2double(__double2hiint(x), lo & 0x1FFFFFFF ? kept | 0x20000000 : kept));
}

template <typename T, int LANES, int NV>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES, NV <= 2 ? 8 : 4) rmsnorm_fp8_kernel(NormArgs p) {
    constexpr int E = kEntries<T>, ROWS = LANES < 256 ? 256 / LANES : 1, WAVES = LANES / 64;
    static_assert(LANES >= kFp8Block / E && (LANES <= 64 || LANES >= 256), "a block within a row's lanes; rows of whole workgroups or waves");
    const int row = blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / LANES : 0);
    const int lane = threadIdx.x % LANES;
    if (row >= p.n) return;   // all lanes of a row; with several waves a row every workgroup has its row
    const int H = p.hidden, kb = fp8_blocks(H);
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    float v[NV][E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = E * (lane + LANES * i);
        load_row<E>(x + at, H - at, v[i]);
    }
    if (p.add) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = E * (lane + LANES * i);
            float b[E];
            if (p.add_dt == RL_DTYPE_FP32) load_row<E>(static_cast<const float*>(p.add) + row * p.ld_add + at, H - at, b);
            else load_row<E>(static_cast<const uint16_t*>(p.add) + row * p.ld_add + at, H - at, b);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[i][e] += b[e];
                if (sizeof(T) == 2) v[i][e] = bf16_to_f32(f32_to_bf16(v[i][e]));   // the norm is of what is stored
            }
        }
    }
    if (p.sum) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = E * (lane + LANES * i);
            store_row<E>(static_cast<T*>(p.sum) + row * p.ld_sum + at, H - at, v[i]);
        }
    }
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            ss = __builtin_fma(static_cast<double>(v[i][e]), static_cast<double>(v[i][e]), ss);
            asm("" : "+v"(v[i][e]));   // converted again below: its 64 bits are not kept in registers
        }
    ss = lanes_sum<LANES < 64 ? LANES : 64>(ss);
    if constexpr (WAVES > 1) {
        __shared__ double part[WAVES];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
        __syncthreads();
        ss = 0.0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ss += part[w];
    }
    const double r = inverse_root(ss * p.per_entry + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = E * (lane + LANES * i);
        float g[E];
        if (p.w_dt == RL_DTYPE_FP32) load_row<E>(static_cast<const float*>(p.w) + at, H - at, g);
        else load_row<E>(static_cast<const uint16_t*>(p.w) + at, H - at, g);
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = to_odd(v[i][e] * (r * g[e]));
        if (at + E > H) {   // nothing behind the row, whatever r is
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (at + e >= H) v[i][e] = 0.0f;
        }
        uint32_t c[E / 4];
        const int b = fp8_encode<E, kFp8Block / E>(v[i], c);
        if (at < kb * kFp8Block) {
            store_codes<E>(p.out.codes + row * p.out.ld + at, c);
            if (at % kFp8Block == 0) p.out.scales[row * p.out.lds + at / kFp8Block] = static_cast<uint8_t>(b);
        }
    }
}

// ---------------------------------------------------------------------------
// Rows: 128 / E lanes a block, U blocks a lane group.  Bound by memory: SwiGLU of 8192 x
// 18944 bf16, 0.78 GB, 152 us (5.1 TB/s; 149 with the exponential of the rounded argument, whose error
// grows with the gate, (2 |g| + 10) 2^-24); of 512 x 18944, 49 MB, 12.6 (15 where nothing is in the caches).  With division and
// the library's exponential and one block a lane group the latter took 15.6, bound by arithmetic.
// ---------------------------------------------------------------------------
// log2(e) as the nearest fp32 number and what it leaves
constexpr float kLog2eHi = 1.44269502e+0f, kLog2eLo = 1.92596303e-8f, kLn2 = 0.693147182f;

constexpr float kFarGate = 80.0f;
// silu(g) u = g u / (1 + e^-g) for |g| <= 80, within 8 2^-24: the exponential is the hardware's of g log2(e) rounded, times
// 1 + ln(2) of what the rounding left, the reciprocal the hardware's.
__device__ __forceinline__ float swiglu_near(float g, float u) {
    const float h = g * kLog2eHi, left = __builtin_fmaf(g, kLog2eLo, __builtin_fmaf(g, kLog2eHi, -h));
    const float e = __builtin_amdgcn_exp2f(-h);
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_fmaf(e, -kLn2 * left, e)) * u;
}
// The same beyond, where 1 + e^-|g| is 1.  For a negative gate e^g = f 2^i may pass fp32 where g e^g u does not: 2^i is shared by
// the gate, which takes up to 2^-120 of it and stays a normal number, and u.
__device__ __forceinline__ float swiglu_far(float g, float u) {
    const float c = fminf(fmaxf(g, -700.0f), 0.0f), i = __builtin_rintf(c * kLog2eHi);
    const float f = __builtin_amdgcn_exp2f(__builtin_fmaf(c, kLog2eLo, __builtin_fmaf(c, kLog2eHi, -i)));
    const int n = static_cast<int>(i), gate = max(n, -120);
    return __builtin_ldexpf(g * f, gate) * __builtin_ldexpf(u, n - gate);
}

template <typename T, bool SWIGLU, int U>
__global__ void __launch_bounds__(256) quantise_rows_kernel(int n, int k, const T* __restrict__ x, int64_t ldx, Fp8Out out) {
    constexpr int E = kEntries<T>, LANES = kFp8Block / E, GROUPS = 256 / LANES;
    const int kb = fp8_blocks(k);
    const int lane = threadIdx.x % LANES;
    float v[U][E], u[U][SWIGLU ? E : 1];
    int row[U], blk[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int unit = (blockIdx.x * U + i) * GROUPS + threadIdx.x / LANES;
        row[i] = unit / kb;
        blk[i] = unit - row[i] * kb;
        const int at = blk[i] * kFp8Block + E * lane;
        const T* xr = x + static_cast<int64_t>(row[i]) * ldx + at;
        const int left = row[i] < n ? k - at : 0;
        load_row<E>(xr, left, v[i]);
        if constexpr (SWIGLU) load_row<E>(xr + k, left, u[i]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if constexpr (SWIGLU) {
            bool far = false;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                far |= !(fabsf(v[i][e]) <= kFarGate);
                y[e] = swiglu_near(v[i][e], u[i][e]);
            }
            if (far) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (!(fabsf(v[i][e]) <= kFarGate)) y[e] = swiglu_far(v[i][e], u[i][e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) v[i][e] = y[e];
        }
        uint32_t c[E / 4];
        const int b = fp8_encode<E, LANES>(v[i], c);
        if (row[i] >= n) continue;   // whole groups
        store_codes<E>(out.codes + row[i] * out.ld + blk[i] * kFp8Block + E * lane, c);
        if (lane == 0) out.scales[row[i] * out.lds + blk[i]] = static_cast<uint8_t>(b);
    }
}

// ---------------------------------------------------------------------------
// Weight tiles of 128 x 128 under one scale: a workgroup a tile, the tile in
// registers.  Bound by memory: 37888 x 3584 bf16, 407 MB, 80 us (5.1 TB/s).
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) quantise_tiles_kernel(int n, int k, const T* __restrict__ x, int64_t ldx, Fp8Out out) {
    constexpr int E = kEntries<T>, LANES = kFp8Block / E, ROWS = 256 / LANES, U = kFp8Block / ROWS;
    __shared__ float part[4];
    const int kb = fp8_blocks(k);
    const int tr = blockIdx.x / kb, tc = blockIdx.x - tr * kb;
    const int at = tc * kFp8Block + E * (threadIdx.x % LANES), r0 = tr * kFp8Block + threadIdx.x / LANES;
    float v[U][E];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int row = r0 + ROWS * i;
        load_row<E>(x + static_cast<int64_t>(row) * ldx + at, row < n ? k - at : 0, v[i]);
    }
    auto of_tile = [&](float a) {
        a = lanes_max<64>(a);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
        __syncthreads();
        return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    };
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i) a = fmaxf(a, largest<E>(v[i]));
    a = of_tile(a);
    if (a > kLargestFloat) {   // the same in the whole workgroup
        a = 0.0f;
#pragma unroll
        for (int i = 0; i < U; ++i) a = fmaxf(a, drop_infinities<E>(v[i]));
        __syncthreads();
        a = of_tile(a);
    }
    const int b = fp8_scale_byte(a);
    const float inv = fp8_inverse(b);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int row = r0 + ROWS * i;
        uint32_t c[E / 4];
        fp8_pack<E>(v[i], inv, c);
        if (row < n) store_codes<E>(out.codes + static_cast<int64_t>(row) * out.ld + at, c);
    }
    if (threadIdx.x == 0) out.scales[tr * out.lds + tc] = static_cast<uint8_t>(b);
}

// ---------------------------------------------------------------------------
// The cache.  One scale for a head's entries of one position; D / 8 lanes a
// head, 8 entries a lane.  Bound by chains of three loads (place, page, data): 512 single tokens of 4 heads of 128 in bf16 take
// 5.1 us to write and 4.2 to read.  Many tokens go eight a lane group, so that there is one chain for eight rows: 21162 of
// them, 65 MB each way, 17.3 and 17.4 us (3.8 TB/s; a lane group a token and eights found together 22.4 and 20.7, values
// byte by byte 62 and 27).
// ---------------------------------------------------------------------------
// Page block of (token i, head h) and the position in it; null where the token has no place.
__device__ __forceinline__ uint8_t* kv_place(const KvFp8& c, const KvTokens& t, int i, int h, int* local) {
    const int s = t.seqs[i], pos = t.pos[i];
    const int j = pos / c.page;
    if (s < 0 || s >= c.n_seqs || pos < 0 || j >= c.max_pages) return nullptr;
    const int pg = c.table[static_cast<int64_t>(s) * c.max_pages + j];
    if (pg < 0 || pg >= c.n_pages) return nullptr;
    *local = pos - j * c.page;
    return c.pool + (static_cast<int64_t>(pg) * c.heads + h) * c.block;
}

// Token and head of this lane group, of LANES lanes.
template <int LANES> __device__ __forceinline__ int kv_unit(const KvFp8& c, int* h) {
    const uint32_t unit = static_cast<uint32_t>((static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x) / LANES);
    const uint32_t i = unit / static_cast<uint32_t>(c.heads);
    *h = static_cast<int>(unit - i * c.heads);
    return static_cast<int>(i);
}

// 8 x 8 bytes turned: byte e of o[j] (as 64 bits) is byte j of a[e].
__device__ __forceinline__ void turn8(const uint32_t (&a)[8][2], uint32_t (&o)[8][2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int sh = 8 * (j & 3);
            o[j][q] = (a[4 * q][j / 4] >> sh & 255u) | (a[4 * q + 1][j / 4] >> sh & 255u) << 8 | (a[4 * q + 2][j / 4] >> sh & 255u) << 16 |
                      (a[4 * q + 3][j / 4] >> sh & 255u) << 24;
        }
}

// One token and head's entries v of a lane, at its page block.
template <int LANES> __device__ __forceinline__ void kv_put(const KvFp8& c, uint8_t* blk, int local, bool values, int lane, float* v) {
    constexpr int D = 8 * LANES;
    uint32_t w[2];
    const int b = fp8_encode<8, LANES>(v, w);
    if (!blk) return;
    if (lane == 0) blk[2 * c.page * D + (values ? c.page : 0) + local] = static_cast<uint8_t>(b);
    if (!values) {
        store_codes<8>(blk + local * D + 8 * lane, w);
        return;
    }
    uint8_t* dst = blk + c.page * D + (local / 8 * D + 8 * lane) * 8 + local % 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) dst[8 * e] = static_cast<uint8_t>(w[e / 4] >> (8 * (e & 3)));
}

// eight codes as numbers; the hardware's conversion takes the scale's exponent along
__device__ __forceinline__ void fp8_decode8(const uint32_t* w, float scale, float* v) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e], scale, false);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e], scale, true);
        v[4 * e] = a[0];
        v[4 * e + 1] = a[1];
        v[4 * e + 2] = b[0];
        v[4 * e + 3] = b[1];
    }
}

// The same read: codes and scale byte, of the pool's first place where there is no block (no branch: the loads of several
// tokens are under way together).
struct KvRead { uint32_t w[2]; int scale; };
template <int LANES> __device__ __forceinline__ KvRead kv_get(const KvFp8& c, const uint8_t* blk, int local, bool values, int lane) {
    constexpr int D = 8 * LANES;
    const uint8_t* p = blk ? blk : c.pool;
    KvRead r{{0u, 0u}, 0};
    r.scale = p[2 * c.page * D + (values ? c.page : 0) + local];
    if (!values) {
        const uint2 q = *reinterpret_cast<const uint2*>(p + local * D + 8 * lane);
        r.w[0] = q.x;
        r.w[1] = q.y;
    } else {
        const uint8_t* src = p + c.page * D + (local / 8 * D + 8 * lane) * 8 + local % 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e / 4] |= static_cast<uint32_t>(src[8 * e]) << (8 * (e & 3));
    }
    return r;
}
// Its numbers; zeros where there is no block.
__device__ __forceinline__ void kv_numbers(const uint8_t* blk, const KvRead& r, float* v) {
    const uint32_t w[2] = {blk ? r.w[0] : 0u, blk ? r.w[1] : 0u};
    fp8_decode8(w, fp8_scale(blk ? r.scale : 127), v);
}

// Few tokens: a lane group a (token, head); blockIdx.y 0: keys, 1: values.
template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_append_kernel(KvFp8 c, KvTokens t) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const bool values = blockIdx.y != 0;
    int h, local = 0;
    const int i = kv_unit<LANES>(c, &h);
    if (i >= t.n) return;   // whole groups of LANES lanes
    float v[8];
    load_row<8>((values ? static_cast<const T*>(t.v) + i * t.ldv : static_cast<const T*>(t.k) + i * t.ldk) + h * D + 8 * lane, 8, v);
    uint8_t* blk = kv_place(c, t, i, h, &local);   // under the load
    kv_put<LANES>(c, blk, local, values, lane, v);
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_read_kernel(KvFp8 c, KvTokens t) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const bool values = blockIdx.y != 0;
    int h, local = 0;
    const int i = kv_unit<LANES>(c, &h);
    if (i >= t.n) return;
    const uint8_t* blk = kv_place(c, t, i, h, &local);
    float v[8];
    kv_numbers(blk, kv_get<LANES>(c, blk, local, values, lane), v);
    store_row<8>((values ? static_cast<T*>(t.out_v) + i * t.ld_ov : static_cast<T*>(t.out_k) + i * t.ld_ok) + h * D + 8 * lane, 8, v);
}

// Many tokens: a lane group a head of the window of tokens i0 .. i0 + 7, whose rows are all under way at once.  Values of eight
// tokens that follow one another in the call and fill positions 8 j .. 8 j + 7 of their sequence are one 64-bit word an
// entry: the window in which those start takes them whole, and each takes its tokens that are of no such eight one by one.
struct KvWindow {
    int start;        // token at which an eight starts, or -1: at most one in a window
    uint32_t alone;   // bit e: token i0 + e is there, and of no eight
};
template <int LANES> __device__ __forceinline__ KvWindow kv_window(const KvTokens& t, int i0, int lane) {
    constexpr int LOADS = (24 + LANES - 1) / LANES;   // tokens i0 - 8 .. i0 + 15 at least: bit b is token i0 - 8 + b
    uint32_t there = 0u, first = 0u, next = 0u;       // a token; at a position of 8 j; the one after the token before
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
        const int j = i0 - 8 + u * LANES + lane;
        const bool in = j >= 0 && j < t.n;
        const uint32_t pos = in ? static_cast<uint32_t>(t.pos[j]) : 1u;
        const bool follows = in && j > 0 && t.seqs[j - 1] == t.seqs[j] && static_cast<uint32_t>(t.pos[j - 1]) == pos - 1u;
        const int sh = (threadIdx.x & 63) / LANES * LANES;
        constexpr uint64_t kMine = (uint64_t(1) << LANES) - 1;
        there |= static_cast<uint32_t>(__ballot(in) >> sh & kMine) << (u * LANES);
        first |= static_cast<uint32_t>(__ballot(pos % 8 == 0) >> sh & kMine) << (u * LANES);
        next |= static_cast<uint32_t>(__ballot(follows) >> sh & kMine) << (u * LANES);
    }
    uint32_t eights = first, of = 0u;
#pragma unroll
    for (int e = 1; e < 8; ++e) eights &= next >> e;
#pragma unroll
    for (int e = 0; e < 8; ++e) of |= eights << e;
    const uint32_t here = eights >> 8 & 255u;
    return KvWindow{here ? i0 + __ffs(static_cast<int>(here)) - 1 : -1, (there & ~of) >> 8 & 255u};
}

// A token's place from the lane of its group that looked it up.
template <int LANES> __device__ __forceinline__ uint8_t* kv_from(uint8_t* blk, int e) {
    return reinterpret_cast<uint8_t*>(__shfl(reinterpret_cast<unsigned long long>(blk), e, LANES));
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_append_window_kernel(KvFp8 c, KvTokens t) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    int h, local = 0;
    const int i0 = 8 * kv_unit<LANES>(c, &h);
    if (i0 >= t.n) return;   // whole groups of LANES lanes
    const int at = h * D + 8 * lane;
    float x[8][8];
    uint32_t w[8][2];
    int b[8];
    if (blockIdx.y == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) load_row<8>(static_cast<const T*>(t.k) + min(i0 + e, t.n - 1) * t.ldk + at, 8, x[e]);
        uint8_t* mine = i0 + (lane & 7) < t.n ? kv_place(c, t, i0 + (lane & 7), h, &local) : nullptr;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = fp8_encode<8, LANES>(x[e], w[e]);
        int scale = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint8_t* blk = kv_from<LANES>(mine, e);
            const int l = __shfl(local, e, LANES);
            if (blk) store_codes<8>(blk + l * D + 8 * lane, w[e]);
            scale = lane == e ? b[e] : scale;
        }
        if (lane < 8 && mine) mine[2 * c.page * D + local] = static_cast<uint8_t>(scale);
        return;
    }
    const KvWindow win = kv_window<LANES>(t, i0, lane);
    if (win.start >= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) load_row<8>(static_cast<const T*>(t.v) + (win.start + e) * t.ldv + at, 8, x[e]);
        uint8_t* blk = kv_place(c, t, win.start, h, &local);
        uint32_t o[8][2], sb[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) sb[e / 4] |= static_cast<uint32_t>(fp8_encode<8, LANES>(x[e], w[e])) << (8 * (e & 3));
        turn8(w, o);
        if (blk) {
            uint8_t* dst = blk + c.page * D + (local * D + 64 * lane);
#pragma unroll
            for (int j = 0; j < 8; j += 2) *reinterpret_cast<u32x4*>(dst + 8 * j) = u32x4{o[j][0], o[j][1], o[j + 1][0], o[j + 1][1]};
            if (lane == 0) *reinterpret_cast<uint2*>(blk + 2 * c.page * D + c.page + local) = make_uint2(sb[0], sb[1]);
        }
    }
    if (!win.alone) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) load_row<8>(static_cast<const T*>(t.v) + min(i0 + e, t.n - 1) * t.ldv + at, 8, x[e]);
    uint8_t* mine = win.alone >> (lane & 7) & 1u ? kv_place(c, t, i0 + (lane & 7), h, &local) : nullptr;
#pragma unroll
    for (int e = 0; e < 8; ++e) kv_put<LANES>(c, kv_from<LANES>(mine, e), __shfl(local, e, LANES), true, lane, x[e]);
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_read_window_kernel(KvFp8 c, KvTokens t) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    int h, local = 0;
    const int i0 = 8 * kv_unit<LANES>(c, &h);
    if (i0 >= t.n) return;
    const int at = h * D + 8 * lane;
    float v[8];
    if (blockIdx.y == 0) {
        uint8_t* mine = i0 + (lane & 7) < t.n ? kv_place(c, t, i0 + (lane & 7), h, &local) : nullptr;
        KvRead r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = kv_get<LANES>(c, kv_from<LANES>(mine, e), __shfl(local, e, LANES), false, lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            kv_numbers(kv_from<LANES>(mine, e), r[e], v);
            if (i0 + e < t.n) store_row<8>(static_cast<T*>(t.out_k) + (i0 + e) * t.ld_ok + at, 8, v);
        }
        return;
    }
    const KvWindow win = kv_window<LANES>(t, i0, lane);
    if (win.start >= 0) {
        const uint8_t* blk = kv_place(c, t, win.start, h, &local);
        uint32_t all[8][2] = {}, o[8][2];
        uint2 s8 = make_uint2(0u, 0u);
        if (blk) {
            const uint8_t* src = blk + c.page * D + (local * D + 64 * lane);
            s8 = *reinterpret_cast<const uint2*>(blk + 2 * c.page * D + c.page + local);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const u32x4 q = ld16(src + 8 * j);
                all[j][0] = q[0];
                all[j][1] = q[1];
                all[j + 1][0] = q[2];
                all[j + 1][1] = q[3];
            }
        }
        turn8(all, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            fp8_decode8(o[e], fp8_scale((e < 4 ? s8.x : s8.y) >> (8 * (e & 3)) & 255u), v);
            store_row<8>(static_cast<T*>(t.out_v) + (win.start + e) * t.ld_ov + at, 8, v);
        }
    }
    if (!win.alone) return;
    uint8_t* mine = win.alone >> (lane & 7) & 1u ? kv_place(c, t, i0 + (lane & 7), h, &local) : nullptr;
    KvRead r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = kv_get<LANES>(c, kv_from<LANES>(mine, e), __shfl(local, e, LANES), true, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        kv_numbers(kv_from<LANES>(mine, e), r[e], v);
        if (win.alone >> e & 1u) store_row<8>(static_cast<T*>(t.out_v) + (i0 + e) * t.ld_ov + at, 8, v);
    }
}

template <typename T, int LANES, int NV> hipError_t norm_launch(const NormArgs& a, hipStream_t s) {
    constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;
    rmsnorm_fp8_kernel<T, LANES, NV><<<(a.n + ROWS - 1) / ROWS, LANES < 256 ? 256 : LANES, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t norm_for(const NormArgs& a, hipStream_t s) {
    // 16-byte vectors of a row.  Two to a lane, so that many waves fit a SIMD; a wave takes a short row alone, in fp32 up to four to
    // a lane, and no barrier.  67 M entries, a bf16 branch, the sum stored: fp32 rows of 128 take 154 us, of 3584 141, of 8192 140, of
    // 16384 158; bf16 rows of 128 95, of 2048 94 (64 lanes: 111), of 4096 89, of 5120 113, of 12288 111.  Compared with sums in 32
    // bits, which were up to a fifth faster: fp32 rows of 128 145 (64 lanes: 258), of 640 148 (256: 216), of 3584 137 (256: 146), of
    // 8192 137 (512: 142, 256: 159), of 16384 144 (256: 220); bf16 rows of 128 87 (64: 284), of 4096 86 (64: 128), of 12288 92
    // (512: 98, 256: 138).
    const int vecs = fp8_blocks(a.hidden) * (kFp8Block / kEntries<T>);
    if constexpr (sizeof(T) == 2)
        if (vecs <= 16) return norm_launch<T, 16, 1>(a, s);
    if (vecs <= 32) return norm_launch<T, 32, 1>(a, s);
    if (vecs <= 64) return norm_launch<T, 64, 1>(a, s);
    if (vecs <= 128) return norm_launch<T, 64, 2>(a, s);
    if constexpr (sizeof(T) == 4) {
        if (vecs <= 256) return norm_launch<T, 64, 4>(a, s);
    } else {
        if (vecs <= 256) return norm_launch<T, 256, 1>(a, s);
    }
    if (vecs <= 512) return norm_launch<T, 256, 2>(a, s);
    if (vecs <= 1024) return norm_launch<T, 512, 2>(a, s);
    if (vecs <= 2048) return norm_launch<T, 1024, 2>(a, s);
    if constexpr (sizeof(T) == 4)
        if (vecs > 4096) return norm_launch<T, 1024, 8>(a, s);
    return norm_launch<T, 1024, 4>(a, s);
}

template <typename T> hipError_t quantise_for(int form, int n, int k, const void* x, int64_t ldx, const Fp8Out& out, hipStream_t s) {
    const T* p = static_cast<const T*>(x);
    const int kb = fp8_blocks(k);
    constexpr int U = 2;
    const int groups = 256 / (kFp8Block / kEntries<T>) * U, grid = (n * kb + groups - 1) / groups;
    if (form == 2) quantise_tiles_kernel<T><<<fp8_blocks(n) * kb, 256, 0, s>>>(n, k, p, ldx, out);
    else if (form == 1) quantise_rows_kernel<T, true, U><<<grid, 256, 0, s>>>(n, k, p, ldx, out);
    else quantise_rows_kernel<T, false, U><<<grid, 256, 0, s>>>(n, k, p, ldx, out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm_fp8(const NormArgs& a, hipStream_t s) {
    return a.x_dt == RL_DTYPE_FP32 ? norm_for<float>(a, s) : norm_for<uint16_t>(a, s);
}

hipError_t launch_quantise_fp8(int form, int n, int k, int dt, const void* x, int64_t ldx, const Fp8Out& out, hipStream_t s) {
    return dt == RL_DTYPE_FP32 ? quantise_for<float>(form, n, k, x, ldx, out, s) : quantise_for<uint16_t>(form, n, k, x, ldx, out, s);
}

namespace {

// Pairs of a token and a head from which on windows are taken, whose one round costs 4 to 12 us whatever the tokens.  4096
// tokens of 4 heads of 128, written and read: of prompts 5.7 + 5.4 us (a lane group a token 15.0 + 8.1), single ones 19.3
// + 13.4 (16.4 + 8.2); half as many: 5.2 + 4.7 (8.5 + 5.2) and 14.4 + 12.5 (9.8 + 5.1); 32768 single ones: 104 + 54 (98 + 49).
constexpr int64_t kManyTokens = 1 << 14;

template <typename T, int D> void kv_append(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    const int64_t units = static_cast<int64_t>(t.n) * c.heads, windows = (t.n + 7) / 8 * static_cast<int64_t>(c.heads);
    constexpr int GROUPS = 256 / (D / 8);
    if (units >= kManyTokens) kv_fp8_append_window_kernel<T, D><<<dim3((windows + GROUPS - 1) / GROUPS, 2), 256, 0, s>>>(c, t);
    else kv_fp8_append_kernel<T, D><<<dim3((units + GROUPS - 1) / GROUPS, 2), 256, 0, s>>>(c, t);
}
template <typename T, int D> void kv_read(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    const int64_t units = static_cast<int64_t>(t.n) * c.heads, windows = (t.n + 7) / 8 * static_cast<int64_t>(c.heads);
    constexpr int GROUPS = 256 / (D / 8);
    if (units >= kManyTokens) kv_fp8_read_window_kernel<T, D><<<dim3((windows + GROUPS - 1) / GROUPS, 2), 256, 0, s>>>(c, t);
    else kv_fp8_read_kernel<T, D><<<dim3((units + GROUPS - 1) / GROUPS, 2), 256, 0, s>>>(c, t);
}

}  // namespace

hipError_t launch_kv_fp8_append(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    if (t.dt == RL_DTYPE_FP32) c.dim == 128 ? kv_append<float, 128>(c, t, s) : kv_append<float, 64>(c, t, s);
    else c.dim == 128 ? kv_append<uint16_t, 128>(c, t, s) : kv_append<uint16_t, 64>(c, t, s);
    return hipGetLastError();
}

hipError_t launch_kv_fp8_read(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    if (t.dt == RL_DTYPE_FP32) c.dim == 128 ? kv_read<float, 128>(c, t, s) : kv_read<float, 64>(c, t, s);
    else c.dim == 128 ? kv_read<uint16_t, 128>(c, t, s) : kv_read<uint16_t, 64>(c, t, s);
    return hipGetLastError();
}

}  // namespace rl
