// k_fp8_attention.hip -- decode attention over a paged K/V cache in 8 bits: each row
// is one query token whose heads attend over positions 0 .. length - 1 of its
// sequence; the heads that share a kv-head are the columns of one wave's tiles.
//
// Per 32 positions a wave computes S^T = K q^T and adds V^T P^T to its sums with
// 16x16x32 bf16 matrix instructions: e4m3 codes and their power-of-two scales
// are bf16 numbers exactly, and the layout of the S tiles is that of the P operand
// when the rows of K are taken in the order that Step says, so nothing crosses lanes but
// two maxima.  P and fp32 queries enter as sums of three bf16 numbers, 24 bits (PT, QT).
// Bound by the cache's bytes: 512 sequences of 2000 positions, 28 q-heads on 4 kv-heads
// of 128, 1.2 GB, take 247 us (4.9 TB/s); three of 8000, 40 on 8, 52 MB, 15.
#include "fp8.h"
#include "rl_decode.h"

#include <algorithm>

namespace rl {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStep = 32;   // positions a wave takes at a time
// bf16 numbers whose sum is a weight.  With two, 16 bits, weights that cancel lose what is left of them; the third costs at most
// 5% (512 x 4 x 2000: 216 us and 215; 8 x 32 x 4000: 50 and 48).
constexpr int PT = 3;

// Chunks of a row of `len` positions; len + chunk may pass 31 bits.
__host__ __device__ constexpr int chunks_in(int len, int chunk) { return len / chunk + (len % chunk != 0); }

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

// Four entries of a row; nothing to attend to: zeros.
template <typename T> __device__ __forceinline__ void write_out(T* out, int at, f32x4 o, float L) {
#pragma unroll
    for (int e = 0; e < 4; ++e) Elem<T>::store(out, at + e, L == 0.0f ? 0.0f : o[e] / L);
}

// Sums o, total L and maximum M of one part of a row's positions, joined with another's.
__device__ __forceinline__ void add_part(float& M, float& L, f32x4& o, float m, float l, f32x4 v) {
    const float m_new = fmaxf(M, m), base = m_new == -INFINITY ? 0.0f : m_new;
    const float f = __builtin_amdgcn_exp2f(M - base), g = __builtin_amdgcn_exp2f(m - base);
    L = f * L + g * l;
    o = f * o + g * v;
    M = m_new;
}

// Partial results of one (row, kv-head, chunk): sums [G][D], then maxima [G] and totals [G].
__host__ __device__ constexpr int part_floats(int G, int D) { return G * (D + 2); }

// A workgroup takes one chunk of one row's positions for one kv-head, its waves every
// kWaves-th step of 32, the next step's loads under this one's arithmetic.
template <typename T, int D, int QT, int kWaves>
__global__ void __launch_bounds__(64 * kWaves, 2) attention_fp8_kernel(AttnFp8 p, int chunk, int n_chunks) {
    constexpr int NQ = D / 64;          // 16-byte K loads a row, of 4 lane groups
    constexpr int NV = D / 32;          // 16-byte V loads a lane: two entries each
    const int c = blockIdx.x % n_chunks, pair = blockIdx.x / n_chunks;
    const int row = pair / p.c.heads, kvh = pair - row * p.c.heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int G = p.heads / p.c.heads;
    const int seq = p.seqs ? p.seqs[row] : row;
    int len = p.lengths[row];
    len = len < 0 || seq < 0 || seq >= p.c.n_seqs ? 0 : len > p.max_length ? p.max_length : len;
    const int lo = c * chunk, hi = len - lo < chunk ? len : lo + chunk;
    float* part = n_chunks > 1 ? p.part + (static_cast<int64_t>(pair) * n_chunks + c) * part_floats(G, D) : nullptr;
    if (part && lo >= hi) return;       // the join goes by the length

    const int first = lo + kStep * wave;
    const int steps = first < hi ? (hi - first + kStep * kWaves - 1) / (kStep * kWaves) : 0;
    // page of step i in lane i (at most 64 steps: kMaxChunk)
    int pages = -1;
    if (lane < steps) pages = p.c.table[static_cast<int64_t>(seq) * p.c.max_pages + (first + kStep * kWaves * lane) / p.c.page];

    // K row r of tile t is position 8 (r / 4) + r % 4 + 4 t of the step
    struct Step { u32x4 k[2][NQ], v[NV]; uint2 ks, vs; bool there; };
    auto load = [&](int i, Step& s) {
        const int pg = __builtin_amdgcn_readlane(pages, i);
        s.there = pg >= 0 && pg < p.c.n_pages;
        if (!s.there) return;           // no such page: nothing there to attend to
        const int local = (first + kStep * kWaves * i) % p.c.page;
        const uint8_t* blk = p.c.pool + (static_cast<int64_t>(pg) * p.c.heads + kvh) * p.c.block;
        const uint8_t* vb = blk + p.c.page * D;
        const uint8_t* sb = vb + p.c.page * D;
        const int pos = local + 8 * (r >> 2) + (r & 3);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < NQ; ++u) s.k[t][u] = ld16(blk + (pos + 4 * t) * D + 64 * u + 16 * g);
        s.ks = *reinterpret_cast<const uint2*>(sb + local + 8 * (r >> 2));
        s.vs = *reinterpret_cast<const uint2*>(sb + p.c.page + local + 8 * g);
#pragma unroll
        for (int i2 = 0; i2 < NV; ++i2) s.v[i2] = ld16(vb + ((local / 8 + g) * D + 32 * i2 + 2 * r) * 8);
    };
    Step s0, s1;
    if (steps > 0) load(0, s0);

    // the queries: lane (r, g) holds head r, entries 64 u + 16 g + 8 v .. + 7 for (u, v)
    bf16x8 q[NQ][2][QT];
    {
        const T* src = static_cast<const T*>(p.q) + row * p.ldq + (kvh * G + (r < G ? r : 0)) * D + 16 * g;
#pragma unroll
        for (int u = 0; u < NQ; ++u)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                float x[8];
                load_row<8>(src + 64 * u + 8 * v, r < G ? 8 : 0, x);
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

    auto take = [&](int i, Step& st) {
        if (!st.there) return;
        const uint32_t kw = (r & 3) * 8;
        const float ks0 = fp8_scale((st.ks.x >> kw) & 255u), ks1 = fp8_scale((st.ks.y >> kw) & 255u);
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < NQ; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const bf16x8 k = codes_bf16(st.k[t][u][2 * v], st.k[t][u][2 * v + 1], t ? ks1 : ks0);
#pragma unroll
                    for (int w = 0; w < QT; ++w) s[t] = mfma16x16x32(k, q[u][v][w], s[t]);
                }
        }
        // this lane's positions are 8 g .. 8 g + 7 of the step: tile 0 has the first four
        float x[8];
        const int at = first + kStep * kWaves * i;
        const int left = hi - at - 8 * g;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * to_log2;
        if (hi - at < kStep) {
            // nothing of what stands behind the last position may enter the sums or the products
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= left) x[e] = -INFINITY;
            const int n = left < 0 ? 0 : left > 8 ? 8 : left;   // bytes kept of each entry's eight
            const uint32_t lom = n >= 4 ? ~0u : (1u << (8 * n)) - 1u, him = n >= 8 ? ~0u : n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1u;
#pragma unroll
            for (int j = 0; j < NV; ++j) st.v[j] = u32x4{st.v[j][0] & lom, st.v[j][1] & him, st.v[j][2] & lom, st.v[j][3] & him};
            st.vs = make_uint2(st.vs.x & lom, st.vs.y & him);
        }
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
            pv[e] = w * fp8_scale(((e < 4 ? st.vs.x : st.vs.y) >> (8 * (e & 3))) & 255u);
        }
        l = l * keep + sum;
        m = m_new;
        bf16x8 pt[PT];
        split_bf16<PT>(pv, pt);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                acc[j][v] *= keep;
                const bf16x8 w = codes_bf16(st.v[j][2 * v], st.v[j][2 * v + 1], 1.0f);
#pragma unroll
                for (int t = 0; t < PT; ++t) acc[j][v] = mfma16x16x32(w, pt[t], acc[j][v]);
            }
    };
    for (int i = 0; i < steps; i += 2) {
        if (i + 1 < steps) load(i + 1, s1);
        take(i, s0);
        if (i + 1 >= steps) break;
        if (i + 2 < steps) load(i + 2, s0);
        take(i + 1, s1);
    }

    extern __shared__ __attribute__((aligned(16))) float sums[];   // [kWaves][G * D]
    __shared__ float maxs[kWaves][16], tots[kWaves][16];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
        maxs[wave][r] = m;
        tots[wave][r] = l;
    }
    // acc[j][v][e] is entry 32 j + 8 g + 2 e + v of head r
    if (r < G) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float* to = sums + (wave * G + r) * D + 32 * j + 8 * g;
            *reinterpret_cast<f32x4*>(to) = f32x4{acc[j][0][0], acc[j][1][0], acc[j][0][1], acc[j][1][1]};
            *reinterpret_cast<f32x4*>(to + 4) = f32x4{acc[j][0][2], acc[j][1][2], acc[j][0][3], acc[j][1][3]};
        }
    }
    __syncthreads();
    T* out = static_cast<T*>(p.out) + row * p.ldo + kvh * G * D;
    for (int at = 4 * tid; at < G * D; at += 4 * 64 * kWaves) {
        const int h = at / D;
        float M = -INFINITY, L = 0.0f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, maxs[w][h]);
        const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(maxs[w][h] - base);
            L += f * tots[w][h];
            o += f * *reinterpret_cast<const f32x4*>(sums + w * G * D + at);
        }
        if (part) {
            *reinterpret_cast<float2*>(part + at) = make_float2(o[0], o[1]);
            *reinterpret_cast<float2*>(part + at + 2) = make_float2(o[2], o[3]);
            if (at - h * D == 0) {
                part[G * D + h] = M;
                part[G * D + G + h] = L;
            }
        } else {
            write_out(out, at, o, L);
        }
    }
}

// The chunks of one (row, kv-head), joined in their order; four entries a thread, eight chunks' loads at once.  8 us
// for 512 x 4 of at most five chunks.
template <typename T, int D>
__global__ void __launch_bounds__(256) attention_fp8_join_kernel(AttnFp8 p, int chunk, int n_chunks) {
    constexpr int U = 8;   // chunks whose loads are in flight together
    const int row = blockIdx.x / p.c.heads, kvh = blockIdx.x - row * p.c.heads;
    const int G = p.heads / p.c.heads, step = part_floats(G, D);
    const int seq = p.seqs ? p.seqs[row] : row;
    int len = p.lengths[row];
    len = len < 0 || seq < 0 || seq >= p.c.n_seqs ? 0 : len > p.max_length ? p.max_length : len;
    const int n = chunks_in(len, chunk);   // chunks with a position
    const float* part = p.part + static_cast<int64_t>(blockIdx.x) * n_chunks * step;
    T* out = static_cast<T*>(p.out) + row * p.ldo + kvh * G * D;
    for (int at = 4 * threadIdx.x; at < G * D; at += 4 * 256) {
        const int h = at / D;
        float M = -INFINITY, L = 0.0f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < n; c0 += U) {
            float cm[U], cl[U];
            float2 a[U], b[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float* q = part + static_cast<int64_t>(c0 + u < n ? c0 + u : c0) * step;
                cm[u] = q[G * D + h];
                cl[u] = q[G * D + G + h];
                a[u] = *reinterpret_cast<const float2*>(q + at);
                b[u] = *reinterpret_cast<const float2*>(q + at + 2);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u < n) add_part(M, L, o, cm[u], cl[u], f32x4{a[u].x, a[u].y, b[u].x, b[u].y});
        }
        write_out(out, at, o, L);
    }
}

// The same for many chunks: a workgroup a query head, its lane groups every GROUPS-th chunk, joined in LDS in their order.
// 24 x 34 chunks of 5 heads take 4.2 us, 7 the other way, where a thread reads them all.
template <typename T, int D>
__global__ void __launch_bounds__(256) attention_fp8_join_head_kernel(AttnFp8 p, int chunk, int n_chunks) {
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, U = 4;
    __shared__ f32x4 os[GROUPS][LANES];
    __shared__ float ms[GROUPS], ls[GROUPS];
    const int row = blockIdx.x / p.heads, head = blockIdx.x - row * p.heads;
    const int G = p.heads / p.c.heads, step = part_floats(G, D), kvh = head / G, h = head - kvh * G;
    const int seq = p.seqs ? p.seqs[row] : row;
    int len = p.lengths[row];
    len = len < 0 || seq < 0 || seq >= p.c.n_seqs ? 0 : len > p.max_length ? p.max_length : len;
    const int n = chunks_in(len, chunk);
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const float* part = p.part + (static_cast<int64_t>(row) * p.c.heads + kvh) * n_chunks * step;
    float M = -INFINITY, L = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = group; c0 < n; c0 += GROUPS * U) {
        float cm[U], cl[U];
        float2 a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + GROUPS * u;
            const float* q = part + static_cast<int64_t>(c < n ? c : c0) * step;
            cm[u] = q[G * D + h];
            cl[u] = q[G * D + G + h];
            a[u] = *reinterpret_cast<const float2*>(q + h * D + 4 * lane);
            b[u] = *reinterpret_cast<const float2*>(q + h * D + 4 * lane + 2);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + GROUPS * u >= n) break;
            add_part(M, L, o, cm[u], cl[u], f32x4{a[u].x, a[u].y, b[u].x, b[u].y});
        }
    }
    os[group][lane] = o;
    if (lane == 0) {
        ms[group] = M;
        ls[group] = L;
    }
    __syncthreads();
    if (group > 0) return;
    for (int q = 1; q < GROUPS; ++q) add_part(M, L, o, ms[q], ls[q], os[q][lane]);
    write_out(static_cast<T*>(p.out) + row * p.ldo + head * D, 4 * lane, o, L);
}

// Positions a workgroup takes, a multiple of 128: 1024 (512 x 4 x 2000: 248 us; with 512 278, with 2048 247), fewer where
// that leaves fewer than 1024 workgroups.
constexpr int kMaxChunk = 64 * kStep;
int chunk_of(int n, int kv_heads, int max_length) {
    int chunk = 1024;
    while (chunk > 256 && static_cast<int64_t>(n) * kv_heads * chunks_in(max_length, chunk) < 1024) chunk /= 2;
    return chunk;
}
static_assert(1024 <= kMaxChunk, "a step's page in a lane");
int chunks_of(int n, int kv_heads, int max_length) {
    return std::max(1, chunks_in(max_length, chunk_of(n, kv_heads, max_length)));
}

template <typename T, int D, int QT, int WAVES> void start(const AttnFp8& a, int chunk, int n_chunks, hipStream_t s) {
    const int lds = WAVES * (a.heads / a.c.heads) * D * sizeof(float);
    attention_fp8_kernel<T, D, QT, WAVES><<<a.n * a.c.heads * n_chunks, 64 * WAVES, lds, s>>>(a, chunk, n_chunks);
}

template <typename T, int D, int QT> hipError_t attend(const AttnFp8& a, hipStream_t s) {
    const int chunk = chunk_of(a.n, a.c.heads, a.max_length), n_chunks = chunks_of(a.n, a.c.heads, a.max_length);
    // Waves a workgroup: one where rows are short and many (11968 pairs of 105 positions: 92 us, with two 96, four 119), four where
    // workgroups are few (304 of them: 18 us, with two 20, one 23), else two (512 x 4 x 2000: 252, four 249; 24 x 8000: 23 and 25;
    // 1732 x 820 in fp32: 130 and 135).
    const int64_t pairs = static_cast<int64_t>(a.n) * a.c.heads;
    if (pairs * n_chunks < 512) start<T, D, QT, 4>(a, chunk, n_chunks, s);
    else if (a.max_length <= 128 && pairs >= 2048) start<T, D, QT, 1>(a, chunk, n_chunks, s);
    else start<T, D, QT, 2>(a, chunk, n_chunks, s);
    if (n_chunks > 8) attention_fp8_join_head_kernel<T, D><<<a.n * a.heads, 256, 0, s>>>(a, chunk, n_chunks);
    else if (n_chunks > 1) attention_fp8_join_kernel<T, D><<<a.n * a.c.heads, 256, 0, s>>>(a, chunk, n_chunks);
    return hipGetLastError();
}

}  // namespace

bool attention_fp8_fits(int n, int kv_heads, int heads, int max_length) {
    const int64_t chunks = chunks_of(n, kv_heads, max_length), pairs = static_cast<int64_t>(n) * kv_heads;
    const int64_t threads = pairs * chunks * 128, join = chunks > 8 ? 256ll * n * heads : chunks > 1 ? 256 * pairs : 0;   // at most
    return std::max(threads, join) < (int64_t(1) << 32);
}
size_t attention_fp8_ws_bytes(int n, int kv_heads, int heads, int dim, int max_length) {
    const int c = chunks_of(n, kv_heads, max_length);
    return c > 1 ? sizeof(float) * static_cast<size_t>(n) * kv_heads * c * part_floats(heads / kv_heads, dim) : 0;
}

hipError_t launch_attention_fp8(const AttnFp8& a, hipStream_t s) {
    // a bf16 query is one bf16 number, an fp32 one the sum of three
    if (a.dt == RL_DTYPE_FP32) return a.c.dim == 128 ? attend<float, 128, 3>(a, s) : attend<float, 64, 3>(a, s);
    return a.c.dim == 128 ? attend<uint16_t, 128, 1>(a, s) : attend<uint16_t, 64, 1>(a, s);
}

}  // namespace rl
