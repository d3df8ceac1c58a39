// k_fp8_attention.hip -- decode attention over a paged K/V cache in 8 bits: each row
// is one query token whose heads attend over positions 0 .. length - 1 of its
// sequence; the heads that share a kv-head are the columns of one wave's tiles.
//
// Per 32 positions a wave computes S^T = K q^T and adds V^T P^T to its sums with
// 16x16x32 bf16 matrix instructions: e4m3 codes and their power-of-two scales
// are bf16 numbers exactly, and the layout of the S tiles is that of the P operand
// when the rows of K are taken in the order of row_of below, so nothing crosses lanes
// but two maxima.  P and fp32 queries enter as sums of bf16 numbers (TERMS).
#include "fp8.h"
#include "rl_decode.h"

namespace rl {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;
constexpr int kStep = 32;   // positions a wave takes at a time

// v as a sum of N bf16 numbers: the rest after each is exact
template <int N> __device__ __forceinline__ void split_bf16(const float* v, bf16x8* out) {
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            out[t][j] = static_cast<__bf16>(r[j]);
            r[j] -= static_cast<float>(out[t][j]);
        }
}

// Partial results of one (row, kv-head, chunk): sums [16][D], then maxima [16] and totals [16].
template <int D> constexpr int kPartFloats = 16 * D + 32;

template <typename T, int D, int QT, int PT>
__global__ void __launch_bounds__(64 * kWaves) attention_fp8_kernel(AttnFp8 p, int chunk, int n_chunks) {
    constexpr int NQ = D / 64;          // 16-byte K loads a row, of 4 lane groups
    constexpr int NV = D / 32;          // 16-byte V loads a lane: two entries each
    const int c = blockIdx.x % n_chunks, pair = blockIdx.x / n_chunks;
    const int row = pair / p.c.heads, kvh = pair - row * p.c.heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int G = p.heads / p.c.heads;
    const int seq = p.seqs ? p.seqs[row] : row;
    int len = p.lengths[row];
    len = len < 0 || seq < 0 || seq >= p.c.n_seqs ? 0 : len > p.max_length ? p.max_length : len;
    const int lo = c * chunk, hi = len - lo < chunk ? len : lo + chunk;

    __shared__ __attribute__((aligned(16))) float sums[kWaves][16 * D];
    __shared__ float maxs[kWaves][16], tots[kWaves][16];

    // the queries: lane (r, g) holds head r, entries 64 u + 16 g + 8 v .. + 7 for (u, v)
    bf16x8 q[NQ][2][QT];
    {
        const T* src = static_cast<const T*>(p.q) + row * p.ldq + (kvh * G + r) * D;
#pragma unroll
        for (int u = 0; u < NQ; ++u)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = r < G ? Elem<T>::load(src, 64 * u + 16 * g + 8 * v + j) : 0.0f;
                split_bf16<QT>(x, q[u][v]);
            }
    }
    const float to_log2 = p.scale * kLog2e;
    f32x4 acc[NV][2];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v) acc[i][v] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.0f;

    const int32_t* table = p.c.table + static_cast<int64_t>(seq) * p.c.max_pages;
    for (int at = lo + kStep * wave; at < hi; at += kStep * kWaves) {
        const int j = at / p.c.page, local = at - j * p.c.page;
        const int pg = table[j];
        if (pg < 0 || pg >= p.c.n_pages) continue;   // no such page: nothing there to attend to
        const uint8_t* blk = p.c.pool + (static_cast<int64_t>(pg) * p.c.heads + kvh) * p.c.block;
        const uint8_t* vb = blk + p.c.page * D;
        const uint8_t* sb = vb + p.c.page * D;
        // K row r of tile t is position 8 (r / 4) + r % 4 + 4 t of the step
        const int pos = local + 8 * (r >> 2) + (r & 3);
        u32x4 kw[2][NQ], vw[NV];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < NQ; ++u) kw[t][u] = ld16(blk + (pos + 4 * t) * D + 64 * u + 16 * g);
#pragma unroll
        for (int i = 0; i < NV; ++i) vw[i] = ld16(vb + ((local / 8 + g) * D + 32 * i + 2 * r) * 8);
        const float ks0 = fp8_scale(sb[pos]), ks1 = fp8_scale(sb[pos + 4]);
        const uint2 vsb = *reinterpret_cast<const uint2*>(sb + p.c.page + local + 8 * g);
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < NQ; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const bf16x8 k = codes_bf16(kw[t][u][2 * v], kw[t][u][2 * v + 1], t ? ks1 : ks0);
#pragma unroll
                    for (int w = 0; w < QT; ++w) s[t] = mfma16x16x32(k, q[u][v][w], s[t]);
                }
        }
        // this lane's positions are 8 g .. 8 g + 7 of the step: tile 0 has the first four
        float x[8];
        const int left = hi - at - 8 * g;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < left ? s[e >> 2][e & 3] * to_log2 : -INFINITY;
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx);
        const float base = m_new == -INFINITY ? 0.0f : m_new;
        const float keep = __builtin_amdgcn_exp2f(m - base);
        float pv[8], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = __builtin_amdgcn_exp2f(x[e] - base);
            sum += w;
            // nothing of what stands behind the last position may enter the products
            pv[e] = e < left ? w * fp8_scale(((e < 4 ? vsb.x : vsb.y) >> (8 * (e & 3))) & 255u) : 0.0f;
        }
        if (left < 8) {
            const int n = left < 0 ? 0 : left;   // bytes kept of each entry's eight
            const uint32_t lom = n >= 4 ? ~0u : (1u << (8 * n)) - 1u, him = n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1u;
#pragma unroll
            for (int i = 0; i < NV; ++i) vw[i] = u32x4{vw[i][0] & lom, vw[i][1] & him, vw[i][2] & lom, vw[i][3] & him};
        }
        l = l * keep + sum;
        m = m_new;
        bf16x8 pt[PT];
        split_bf16<PT>(pv, pt);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                acc[i][v] *= keep;
                const bf16x8 w = codes_bf16(vw[i][2 * v], vw[i][2 * v + 1], 1.0f);
#pragma unroll
                for (int t = 0; t < PT; ++t) acc[i][v] = mfma16x16x32(w, pt[t], acc[i][v]);
            }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
        maxs[wave][r] = m;
        tots[wave][r] = l;
    }
    // acc[i][v][e] is entry 32 i + 8 g + 2 e + v of head r
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int v = 0; v < 2; ++v) sums[wave][r * D + 32 * i + 8 * g + 2 * e + v] = acc[i][v][e];
    __syncthreads();
    float* part = n_chunks > 1 ? p.part + (static_cast<int64_t>(pair) * n_chunks + c) * kPartFloats<D> : nullptr;
    T* out = static_cast<T*>(p.out) + row * p.ldo + kvh * G * D;
    for (int at = tid; at < G * D; at += 64 * kWaves) {
        const int h = at / D;
        float M = -INFINITY, L = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, maxs[w][h]);
        const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(maxs[w][h] - base);
            L += f * tots[w][h];
            o += f * sums[w][at];
        }
        if (part) {
            part[at] = o;
            if (at - h * D == 0) {
                part[16 * D + h] = M;
                part[16 * D + 16 + h] = L;
            }
        } else {
            Elem<T>::store(out, at, L == 0.0f ? 0.0f : o / L);   // nothing to attend to: zeros
        }
    }
}

// The chunks of one (row, kv-head), joined in their order.
template <typename T, int D>
__global__ void __launch_bounds__(256) attention_fp8_join_kernel(AttnFp8 p, int n_chunks) {
    const int row = blockIdx.x / p.c.heads, kvh = blockIdx.x - row * p.c.heads;
    const int G = p.heads / p.c.heads;
    const float* part = p.part + static_cast<int64_t>(blockIdx.x) * n_chunks * kPartFloats<D>;
    T* out = static_cast<T*>(p.out) + row * p.ldo + kvh * G * D;
    for (int at = threadIdx.x; at < G * D; at += 256) {
        const int h = at / D;
        float M = -INFINITY;
        for (int c = 0; c < n_chunks; ++c) M = fmaxf(M, part[c * kPartFloats<D> + 16 * D + h]);
        const float base = M == -INFINITY ? 0.0f : M;
        float L = 0.0f, o = 0.0f;
        for (int c = 0; c < n_chunks; ++c) {
            const float* q = part + c * kPartFloats<D>;
            const float f = __builtin_amdgcn_exp2f(q[16 * D + h] - base);
            L += f * q[16 * D + 16 + h];
            o += f * q[at];
        }
        Elem<T>::store(out, at, L == 0.0f ? 0.0f : o / L);
    }
}

// Positions a workgroup takes, a multiple of 128.
int chunk_of(int n, int kv_heads, int max_length) {
    int chunk = 1024;
    while (chunk > 256 && static_cast<int64_t>(n) * kv_heads * ((max_length + chunk - 1) / chunk) < 1024) chunk /= 2;
    return chunk;
}
int chunks_of(int n, int kv_heads, int max_length) {
    const int c = chunk_of(n, kv_heads, max_length);
    const int k = (max_length + c - 1) / c;
    return k < 1 ? 1 : k;
}

template <typename T, int D, int QT, int PT> hipError_t attend(const AttnFp8& a, hipStream_t s) {
    const int chunk = chunk_of(a.n, a.c.heads, a.max_length), n_chunks = chunks_of(a.n, a.c.heads, a.max_length);
    attention_fp8_kernel<T, D, QT, PT><<<a.n * a.c.heads * n_chunks, 64 * kWaves, 0, s>>>(a, chunk, n_chunks);
    if (n_chunks > 1) attention_fp8_join_kernel<T, D><<<a.n * a.c.heads, 256, 0, s>>>(a, n_chunks);
    return hipGetLastError();
}

}  // namespace

bool attention_fp8_fits(int n, int kv_heads, int max_length) {
    return static_cast<int64_t>(n) * kv_heads * chunks_of(n, kv_heads, max_length) < (int64_t(1) << 31);
}
size_t attention_fp8_ws_bytes(int n, int kv_heads, int dim, int max_length) {
    const int c = chunks_of(n, kv_heads, max_length);
    return c > 1 ? sizeof(float) * static_cast<size_t>(n) * kv_heads * c * (16 * dim + 32) : 0;
}

hipError_t launch_attention_fp8(const AttnFp8& a, hipStream_t s) {
    // bf16 queries are one bf16 number; the weights keep 16 bits for bf16 outputs, 24 for fp32
    if (a.dt == RL_DTYPE_FP32) return a.c.dim == 128 ? attend<float, 128, 3, 3>(a, s) : attend<float, 64, 3, 3>(a, s);
    return a.c.dim == 128 ? attend<uint16_t, 128, 1, 2>(a, s) : attend<uint16_t, 64, 1, 2>(a, s);
}

}  // namespace rl
