// k_fp8.hip -- numbers to 8 bits and back: RMS norm with the residual's addition,
// rows, SwiGLU's product, weight tiles, and the tokens of a paged K/V cache.
#include "fp8.h"
#include "rl_decode.h"

namespace rl {

namespace {

// ---------------------------------------------------------------------------
// RMS norm.  s = x + add (as stored), y = s w / sqrt(mean s^2 + eps), y in blocks of
// 128.  ROWS rows a workgroup, WAVES waves a row, a row in registers from its one
// read to its codes: 8 NV entries a lane, 16 lanes a block.
// ---------------------------------------------------------------------------
template <typename T, int WAVES, int NV>
__global__ void __launch_bounds__(256) rmsnorm_fp8_kernel(NormArgs p, bool xvec, bool avec, bool svec, bool wvec) {
    constexpr int ROWS = 4 / WAVES, LANES = 64 * WAVES;
    const int row = blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / LANES : 0);
    const int lane = threadIdx.x % LANES;
    if (row >= p.n) return;   // whole waves; with several waves a row every workgroup has its row
    const int H = p.hidden, kb = fp8_blocks(H);
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    float v[NV][8];
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (lane + LANES * i);
        load8(x + at, xvec, H - at, v[i]);
    }
    if (p.add) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (lane + LANES * i);
            float b[8];
            if (p.add_dt == RL_DTYPE_FP32) load8(static_cast<const float*>(p.add) + row * p.ld_add + at, avec, H - at, b);
            else load8(static_cast<const uint16_t*>(p.add) + row * p.ld_add + at, avec, H - at, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] += b[e];
                if (sizeof(T) == 2) v[i][e] = bf16_to_f32(f32_to_bf16(v[i][e]));   // the norm is of what is stored
            }
        }
    }
    if (p.sum) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (lane + LANES * i);
            store8(static_cast<T*>(p.sum) + row * p.ld_sum + at, svec, H - at, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += v[i][e] * v[i][e];
    ss = wave_sum(ss);
    if constexpr (WAVES > 1) {
        __shared__ float part[WAVES];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
        __syncthreads();
        ss = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ss += part[w];
    }
    const float r = 1.0f / sqrtf(ss / static_cast<float>(H) + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (lane + LANES * i);
        float g[8];
        if (p.w_dt == RL_DTYPE_FP32) load8(static_cast<const float*>(p.w) + at, wvec, H - at, g);
        else load8(static_cast<const uint16_t*>(p.w) + at, wvec, H - at, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * r * g[e];
        if (at + 8 > H) {   // nothing behind the row, whatever r is
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e >= H) v[i][e] = 0.0f;
        }
        uint2 c;
        const int b = fp8_encode8<16>(v[i], &c);
        if (at < kb * kFp8Block) {
            *reinterpret_cast<uint2*>(p.out.codes + row * p.out.ld + at) = c;
            if ((lane & 15) == 0) p.out.scales[row * p.out.lds + at / kFp8Block] = static_cast<uint8_t>(b);
        }
    }
}

// ---------------------------------------------------------------------------
// Rows: 16 lanes a block of 128 entries, 8 a lane.
// ---------------------------------------------------------------------------
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(256) quantise_rows_kernel(int n, int k, const T* __restrict__ x, int64_t ldx, bool vec,
                                                            bool uvec, Fp8Out out) {
    const int kb = fp8_blocks(k);
    const int unit = blockIdx.x * 16 + (threadIdx.x >> 4);
    if (unit >= n * kb) return;   // whole groups of 16 lanes
    const int row = unit / kb, blk = unit - row * kb;
    const int at = blk * kFp8Block + 8 * (threadIdx.x & 15);
    const T* xr = x + row * ldx;
    float v[8];
    load8(xr + at, vec, k - at, v);
    if (SWIGLU) {
        float u[8];
        load8(xr + k + at, uvec, k - at, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] / (1.0f + expf(-v[e])) * u[e];
    }
    uint2 c;
    const int b = fp8_encode8<16>(v, &c);
    *reinterpret_cast<uint2*>(out.codes + row * out.ld + at) = c;
    if ((threadIdx.x & 15) == 0) out.scales[row * out.lds + blk] = static_cast<uint8_t>(b);
}

// ---------------------------------------------------------------------------
// Weight tiles of 128 x 128 under one scale: a workgroup a tile, the tile in
// registers (16 lanes a row, 8 rows a lane).
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) quantise_tiles_kernel(int n, int k, const T* __restrict__ x, int64_t ldx, bool vec,
                                                             Fp8Out out) {
    __shared__ float part[4];
    const int kb = fp8_blocks(k);
    const int tr = blockIdx.x / kb, tc = blockIdx.x - tr * kb;
    const int at = tc * kFp8Block + 8 * (threadIdx.x & 15);
    float v[8][8];
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = tr * kFp8Block + 16 * i + (threadIdx.x >> 4);
        load8(x + static_cast<int64_t>(row) * ldx + at, vec, row < n ? k - at : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) a = fmaxf(a, finite_abs(v[i][e]));
    a = wave_max(a);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
    __syncthreads();
    const int b = fp8_scale_byte(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    const float inv = fp8_inverse(b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = tr * kFp8Block + 16 * i + (threadIdx.x >> 4);
        if (row < n)
            *reinterpret_cast<uint2*>(out.codes + static_cast<int64_t>(row) * out.ld + at) =
                make_uint2(fp8_pack4(v[i], inv), fp8_pack4(v[i] + 4, inv));
    }
    if (threadIdx.x == 0) out.scales[tr * out.lds + tc] = static_cast<uint8_t>(b);
}

// ---------------------------------------------------------------------------
// The cache.  One scale for a head's entries of one position; D / 8 lanes a
// head, 8 entries a lane.
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

template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_append_kernel(KvFp8 c, KvTokens t, bool kvec, bool vvec) {
    constexpr int LANES = D / 8;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / LANES;
    const int lane = threadIdx.x % LANES;
    const int i = static_cast<int>(unit / c.heads), h = static_cast<int>(unit - static_cast<int64_t>(i) * c.heads);
    if (i >= t.n) return;   // whole groups of LANES lanes
    int local = 0;
    uint8_t* blk = kv_place(c, t, i, h, &local);
    if (!blk) return;
    const int at = h * D + 8 * lane;
    float v[8];
    uint2 w;
    load8(static_cast<const T*>(t.k) + i * t.ldk + at, kvec, 8, v);
    int b = fp8_encode8<LANES>(v, &w);
    *reinterpret_cast<uint2*>(blk + local * D + 8 * lane) = w;
    if (lane == 0) blk[2 * c.page * D + local] = static_cast<uint8_t>(b);
    load8(static_cast<const T*>(t.v) + i * t.ldv + at, vvec, 8, v);
    b = fp8_encode8<LANES>(v, &w);
    uint8_t* dst = blk + c.page * D + (local / 8 * D + 8 * lane) * 8 + local % 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) dst[8 * e] = static_cast<uint8_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    if (lane == 0) blk[2 * c.page * D + c.page + local] = static_cast<uint8_t>(b);
}

// eight codes as numbers; the hardware's conversion takes the scale's exponent along
__device__ __forceinline__ void fp8_decode8(uint2 w, float scale, float* v) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t q = e ? w.y : w.x;
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q, scale, false);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q, scale, true);
        v[4 * e] = a[0];
        v[4 * e + 1] = a[1];
        v[4 * e + 2] = b[0];
        v[4 * e + 3] = b[1];
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv_fp8_read_kernel(KvFp8 c, KvTokens t, bool kvec, bool vvec) {
    constexpr int LANES = D / 8;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / LANES;
    const int lane = threadIdx.x % LANES;
    const int i = static_cast<int>(unit / c.heads), h = static_cast<int>(unit - static_cast<int64_t>(i) * c.heads);
    if (i >= t.n) return;
    int local = 0;
    const uint8_t* blk = kv_place(c, t, i, h, &local);
    const int at = h * D + 8 * lane;
    float k[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = v[e] = 0.0f;
    if (blk) {
        fp8_decode8(*reinterpret_cast<const uint2*>(blk + local * D + 8 * lane), fp8_scale(blk[2 * c.page * D + local]), k);
        const uint8_t* src = blk + c.page * D + (local / 8 * D + 8 * lane) * 8 + local % 8;
        uint2 w = make_uint2(0u, 0u);
#pragma unroll
        for (int e = 0; e < 8; ++e) (e < 4 ? w.x : w.y) |= static_cast<uint32_t>(src[8 * e]) << (8 * (e & 3));
        fp8_decode8(w, fp8_scale(blk[2 * c.page * D + c.page + local]), v);
    }
    store8(static_cast<T*>(t.out_k) + i * t.ld_ok + at, kvec, 8, k);
    store8(static_cast<T*>(t.out_v) + i * t.ld_ov + at, vvec, 8, v);
}

size_t es_of(int dt) { return dt == RL_DTYPE_FP32 ? 4 : 2; }

template <typename T, int WAVES, int NV> hipError_t norm_launch(const NormArgs& a, hipStream_t s) {
    constexpr int ROWS = 4 / WAVES;
    rmsnorm_fp8_kernel<T, WAVES, NV><<<(a.n + ROWS - 1) / ROWS, 256, 0, s>>>(
        a, rows_on_16(a.x, a.ldx, sizeof(T)), a.add && rows_on_16(a.add, a.ld_add, es_of(a.add_dt)),
        a.sum && rows_on_16(a.sum, a.ld_sum, sizeof(T)), rows_on_16(a.w, 0, es_of(a.w_dt)));
    return hipGetLastError();
}
template <typename T> hipError_t norm_for(const NormArgs& a, hipStream_t s) {
    const int vecs = fp8_blocks(a.hidden) * 16;   // lanes' vectors of a row
    if (vecs <= 64) return norm_launch<T, 1, 1>(a, s);
    if (vecs <= 128) return norm_launch<T, 1, 2>(a, s);
    if (vecs <= 256) return norm_launch<T, 1, 4>(a, s);
    if (vecs <= 512) return norm_launch<T, 1, 8>(a, s);
    if (vecs <= 1024) return norm_launch<T, 4, 4>(a, s);
    return norm_launch<T, 4, 16>(a, s);
}

template <typename T> hipError_t quantise_for(int form, int n, int k, const void* x, int64_t ldx, const Fp8Out& out, hipStream_t s) {
    const T* p = static_cast<const T*>(x);
    const bool vec = rows_on_16(p, ldx, sizeof(T));
    const int kb = fp8_blocks(k);
    if (form == 2) quantise_tiles_kernel<T><<<fp8_blocks(n) * kb, 256, 0, s>>>(n, k, p, ldx, vec, out);
    else if (form == 1)
        quantise_rows_kernel<T, true><<<(n * kb + 15) / 16, 256, 0, s>>>(n, k, p, ldx, vec, rows_on_16(p + k, ldx, sizeof(T)), out);
    else quantise_rows_kernel<T, false><<<(n * kb + 15) / 16, 256, 0, s>>>(n, k, p, ldx, vec, false, out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm_fp8(const NormArgs& a, hipStream_t s) {
    return a.x_dt == RL_DTYPE_FP32 ? norm_for<float>(a, s) : norm_for<uint16_t>(a, s);
}

hipError_t launch_quantise_fp8(int form, int n, int k, int dt, const void* x, int64_t ldx, const Fp8Out& out, hipStream_t s) {
    return dt == RL_DTYPE_FP32 ? quantise_for<float>(form, n, k, x, ldx, out, s) : quantise_for<uint16_t>(form, n, k, x, ldx, out, s);
}

hipError_t launch_kv_fp8_append(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    const size_t es = es_of(t.dt);
    const bool kv = rows_on_16(t.k, t.ldk, es), vv = rows_on_16(t.v, t.ldv, es);
    const int64_t threads = static_cast<int64_t>(t.n) * c.heads * (c.dim / 8);
    const int grid = static_cast<int>((threads + 255) / 256);
    if (t.dt == RL_DTYPE_FP32) {
        if (c.dim == 128) kv_fp8_append_kernel<float, 128><<<grid, 256, 0, s>>>(c, t, kv, vv);
        else kv_fp8_append_kernel<float, 64><<<grid, 256, 0, s>>>(c, t, kv, vv);
    } else {
        if (c.dim == 128) kv_fp8_append_kernel<uint16_t, 128><<<grid, 256, 0, s>>>(c, t, kv, vv);
        else kv_fp8_append_kernel<uint16_t, 64><<<grid, 256, 0, s>>>(c, t, kv, vv);
    }
    return hipGetLastError();
}

hipError_t launch_kv_fp8_read(const KvFp8& c, const KvTokens& t, hipStream_t s) {
    const size_t es = es_of(t.dt);
    const bool kv = rows_on_16(t.out_k, t.ld_ok, es), vv = rows_on_16(t.out_v, t.ld_ov, es);
    const int64_t threads = static_cast<int64_t>(t.n) * c.heads * (c.dim / 8);
    const int grid = static_cast<int>((threads + 255) / 256);
    if (t.dt == RL_DTYPE_FP32) {
        if (c.dim == 128) kv_fp8_read_kernel<float, 128><<<grid, 256, 0, s>>>(c, t, kv, vv);
        else kv_fp8_read_kernel<float, 64><<<grid, 256, 0, s>>>(c, t, kv, vv);
    } else {
        if (c.dim == 128) kv_fp8_read_kernel<uint16_t, 128><<<grid, 256, 0, s>>>(c, t, kv, vv);
        else kv_fp8_read_kernel<uint16_t, 64><<<grid, 256, 0, s>>>(c, t, kv, vv);
    }
    return hipGetLastError();
}

}  // namespace rl
