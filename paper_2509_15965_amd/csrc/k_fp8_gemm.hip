// k_fp8_gemm.hip -- out = A W^T of matrices in 8 bits: e4m3 codes, a power-of-two
// scale for each row's 128 entries of A and each 128 x 128 tile of W.
//
// Codes and their scales are bf16 numbers exactly, and go as such through bf16
// instructions, which add in fp32: 24 bits throughout, whatever the output's type.
// The 8-bit instructions, at twice the rate, add eight products with 14 bits, counted
// from the leading bit of the largest (measured, of either form of them: with one
// product of 2^16 among the eight, 2^3 still counts and 2^2 does not), so that
// large products which cancel take the small ones beside them along; they are
// not used.  Which entries of the block a lane group holds is free, as long as A
// and W agree.
#include "fp8.h"
#include "rl_decode.h"

#include <algorithm>
#include <type_traits>

namespace rl {

namespace {

struct Codes32 { uint32_t c[8]; };   // 32 codes

__device__ __forceinline__ Codes32 join(u32x4 a, u32x4 b) { return Codes32{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}}; }

typedef __attribute__((address_space(3))) void lds_void_t;

// Rows of memory that lanes load from to LDS.  `there` 0: nothing is there, and a load reads nothing (the
// hardware compares each offset with the number of bytes).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const uint8_t* p, bool there) {
    constexpr int kFormat32 = 4 << 15;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, there ? 0x7FFFFFFF : 0, kFormat32);
}
// BYTES a lane, off + more past the first row, straight to LDS: lane i to BYTES i past lds.
template <int BYTES> __device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t rows, uint32_t off, int more, uint8_t* lds) {
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void_t*)(lds), 16, off, more, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void_t*)(lds), 4, off, more, 0, 0);
}

// s_waitcnt vmcnt(N), the other counters left alone
template <int N> __device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// Barrier of the workgroup behind which the wave's loads to LDS but the last N, and its reads of LDS, are done.
template <int N> __device__ __forceinline__ void barrier_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// ---------------------------------------------------------------------------
// Few tokens: a workgroup takes 16 RW weights, its eight waves every eighth block of
// its K slice, straight from memory to registers, and the waves' sums meet in LDS
// in wave order.  MT x 16 tokens.  Bound by the weights' bytes, read at 5.6 TB/s
// (one token, 152064 x 3584): the conversions cost nothing here.  Two
// blocks in flight a wave, or non-temporal loads, are 4 to 14% and 14 to 26% slower:
// more waves do better than more registers each.
// ---------------------------------------------------------------------------
constexpr int kGemvWaves = 8;
template <typename TO, int RW, int MT, bool SPLIT>
__global__ void __launch_bounds__(64 * kGemvWaves, 4) gemv_fp8_kernel(Fp8Gemm p, int per) {
    constexpr int WV = kGemvWaves;
    __shared__ f32x4 red[WV][RW * MT][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * RW;
    const int k0 = blockIdx.y * per, k1 = min(p.kb, k0 + per);
    const uint8_t* wp[RW];
    const uint8_t* ap[MT];
    const uint8_t* sp[MT];
    const uint8_t* swp[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) {
        const int n = min(n0 + 16 * i + r16, p.n - 1);
        wp[i] = p.w.codes + n * p.w.ld + 16 * g;
        swp[i] = p.w.scales + static_cast<int64_t>(min(n0 + 16 * i, p.n - 1) / 128) * p.w.lds;
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int m = min(16 * j + r16, p.m - 1);
        ap[j] = p.a.codes + m * p.a.ld + 16 * g;
        sp[j] = p.a.scales + m * p.a.lds;
    }
    f32x4 acc[RW][MT];
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = k0 + wave; k < k1; k += WV) {
        u32x4 w[RW][2], a[MT][2];
        float sw[RW], sa[MT];
#pragma unroll
        for (int i = 0; i < RW; ++i) {
            w[i][0] = ld16(wp[i] + k * 128);
            w[i][1] = ld16(wp[i] + k * 128 + 64);
            sw[i] = fp8_scale(swp[i][k]);
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            a[j][0] = ld16(ap[j] + k * 128);
            a[j][1] = ld16(ap[j] + k * 128 + 64);
            sa[j] = fp8_scale(sp[j][k]);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            bf16x8 wf[RW];
#pragma unroll
            for (int i = 0; i < RW; ++i) wf[i] = codes_bf16(w[i][h / 2][2 * (h & 1)], w[i][h / 2][2 * (h & 1) + 1], sw[i]);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const bf16x8 af = codes_bf16(a[j][h / 2][2 * (h & 1)], a[j][h / 2][2 * (h & 1) + 1], sa[j]);
#pragma unroll
                for (int i = 0; i < RW; ++i) acc[i][j] = mfma16x16x32(wf[i], af, acc[i][j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) red[wave][i * MT + j][lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int x0 = 0; x0 < RW * MT; x0 += WV) {
        const int x = x0 + wave;
        if (x >= RW * MT) break;
        f32x4 v = red[0][x][lane];
#pragma unroll
        for (int q = 1; q < WV; ++q) v += red[q][x][lane];
        const int m = 16 * (x % MT) + r16, n = n0 + 16 * (x / MT) + 4 * g;
        if (m >= p.m) continue;
        const float f[4] = {v[0], v[1], v[2], v[3]};
        if constexpr (SPLIT) store_row<4>(p.part + (static_cast<int64_t>(blockIdx.y) * p.m + m) * p.n + n, p.n - n, f);
        else store_row<4>(static_cast<TO*>(p.out) + m * p.ldo + n, p.n - n, f);
    }
}

// ---------------------------------------------------------------------------
// Tiles of 128 tokens x 128 weights, 2 x 2 waves, four 32x32x16 instructions for half
// a block's 64 entries, over the nk blocks of K from k0 on, a multiple of four.
//
// A block of K of either operand is a slot of 128-byte rows in LDS, moved
// there from memory without passing through registers, eight whole lines an
// instruction; two slots.  Chunk c (16 bytes) of row r sits at c ^ (r / 2 % 8), which
// frees the fragment reads of bank conflicts.  A wave holds a block's weights in
// registers and multiplies them with the first half of its tokens, then with the
// second; the fragments of the half that follows are read under each half's
// instructions.  So a block's weights and first tokens have left their slot when its first
// half begins and the second tokens when that ends: behind a barrier there, the slot
// takes what the block after the next needs, and all of it has a block and a half's
// time to arrive.
//
// Bound by the matrix unit and the power that it draws: 8192 x 3584 x 18944 takes 836 to
// 868 us, 1.3 PFLOP/s, with the unit busy 73% of the cycles at 1.7 GHz, beside four conversions an
// instruction; such instructions alone, on codes in registers, reach 1.8 to 2.0.
//
// LDS row 32 t + 8 q + 4 h + e of a wave's weights (t tile, 4 q + e register and h lane half
// of the instruction's output) holds weight h TN / 2 + q TN / 8 + 4 t + e: a lane's outputs
// of one token are runs of TN / 8 weights, stored 16 bytes at a time.
// Rows past the last token or weight are the last one again, and are not stored.
// ---------------------------------------------------------------------------
struct TileMap { int m_tiles, n_tiles, gm; };

constexpr int kTile = 128;
constexpr int kTileLds = 2 * (2 * kTile * 128 + 2048);

template <typename TO>
__device__ __forceinline__ void tile_fp8(const Fp8Gemm& p, int m0, int n0, int k0, int nk, uint8_t* smem, float* part) {
    constexpr int TM = kTile / 2, TN = kTile / 2, MT = TM / 32, NT = TN / 32;
    constexpr int AQ = kTile / 64, WQ = kTile / 32;                // line instructions a wave issues for half of the tokens, for the weights
    constexpr int Q1 = WQ + AQ, Q2 = AQ;                     // a block's first refill and its second
    constexpr int ASLOT = kTile * 128, WSLOT = kTile * 128, SSLOT = 2048;   // SSLOT: scale words, of four blocks each
    uint8_t* const aslots = smem;
    uint8_t* const wslots = smem + 2 * ASLOT;
    uint8_t* const sslots = smem + 2 * (ASLOT + WSLOT);

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, r32 = lane & 31, kh = lane >> 5;

    const uint8_t* abase = p.a.codes + m0 * p.a.ld + k0 * 128;
    const uint8_t* wbase = p.w.codes + n0 * p.w.ld + k0 * 128;
    uint32_t aoff[2][AQ], woff[WQ];
    auto arow = [&](int half, int q) {   // first LDS row of the eight that an instruction moves: halves of each wave row's tokens
        const int r = 8 * (wave * AQ + q);
        return r / (TM / 2) * TM + half * (TM / 2) + r % (TM / 2);
    };
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int q = 0; q < AQ; ++q) {
            const int r = arow(f, q) + (lane >> 3);
            aoff[f][q] = min(r, p.m - 1 - m0) * static_cast<uint32_t>(p.a.ld) + 16u * ((lane & 7) ^ ((r >> 1) & 7));
        }
#pragma unroll
    for (int q = 0; q < WQ; ++q) {
        const int r = 8 * (wave * WQ + q) + (lane >> 3), b = r % TN;   // b = 32 t + 8 q + 4 h + e
        const int n = r - b + ((b >> 2) & 1) * (TN / 2) + ((b >> 3) & 3) * (TN / 8) + 4 * (b >> 5) + (b & 3);
        woff[q] = min(n, p.n - 1 - n0) * static_cast<uint32_t>(p.w.ld) + 16u * ((lane & 7) ^ ((r >> 1) & 7));
    }
    const uint32_t soff = min((64 * wave + lane) % kTile, p.m - 1 - m0) * static_cast<uint32_t>(p.a.lds);
    const uint8_t* sabase = p.a.scales + m0 * p.a.lds + k0;
    const uint8_t* swbase = p.w.scales + static_cast<int64_t>(min((n0 + wn * TN) / 128, (p.n - 1) / 128)) * p.w.lds + k0;

    struct Source { __amdgpu_buffer_rsrc_t a, w, sa, sw; };
    auto source = [&](bool there) { return Source{rows_at(abase, there), rows_at(wbase, there), rows_at(sabase, there), rows_at(swbase, there)}; };
    auto issue = [&](const Source& from, int kt, int slot, int part, int q) {   // instruction q of block kt's first or second refill
        uint8_t* as = aslots + slot * ASLOT;
        if (part == 1) to_lds<16>(from.a, aoff[1][q < AQ ? q : 0], kt * 128, as + arow(1, q) * 128);
        else if (q < WQ) to_lds<16>(from.w, woff[q < WQ ? q : 0], kt * 128, wslots + slot * WSLOT + (wave * WQ + q) * 1024);
        else to_lds<16>(from.a, aoff[0][q >= WQ ? q - WQ : 0], kt * 128, as + arow(0, q - WQ) * 128);
    };
    // The scales of four blocks are one word of each row, 64 lines an instruction: they come with every second block's first
    // refill and serve both.
    auto issue_scales = [&](const Source& from, int kt) {
        uint8_t* to = sslots + (kt >> 1 & 1) * SSLOT + wave * 256;
        to_lds<4>(from.sa, soff, kt & ~3, to);
        to_lds<4>(from.sw, 0u, kt & ~3, to + 1024);
    };

    f32x16 acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][i][e] = 0.f;

    // the swizzle of a fragment's row goes by r32 alone: rows of tiles are multiples of 32 apart
    const int swz = (r32 >> 1) & 7;
    const uint32_t la = (wm * TM + r32) * 128, lw = (wn * TN + r32) * 128;
    const uint32_t lsa = (wm * TM + r32) * 4, lsw = 1024 + wave * 256;
    uint32_t ch[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) ch[c] = ((2 * c + kh) ^ swz) << 4;
    struct Weights { Codes32 w[NT][2]; };        // [tile][half of the block]
    struct Tokens { Codes32 a[2]; };
    auto frag = [&](const uint8_t* row, int k) {
        return join(*reinterpret_cast<const u32x4*>(row + ch[2 * k]), *reinterpret_cast<const u32x4*>(row + ch[2 * k + 1]));
    };
    auto read_w = [&](int slot, Weights& f, int t, int k) { f.w[t][k] = frag(wslots + slot * WSLOT + lw + 4096 * t, k); };
    auto read_a = [&](int slot, Tokens& f, int i, int k) { f.a[k] = frag(aslots + slot * ASLOT + la + 4096 * i, k); };
    struct Scales { uint32_t w, a[MT]; };
    auto read_scales = [&](int kt, Scales& f) {
        const uint8_t* from = sslots + (kt >> 1 & 1) * SSLOT;
        f.w = *reinterpret_cast<const uint32_t*>(from + lsw);
#pragma unroll
        for (int i = 0; i < MT; ++i) f.a[i] = *reinterpret_cast<const uint32_t*>(from + lsa + 128 * i);
    };
    // a block's products in two groups: every weight tile with half of the token tiles
    constexpr int GA = MT / 2, G = NT * 2 * GA;
    Weights w;
    Tokens at[2][GA];
    Scales sc, sc_next{};
    // Barriers stand B products into the halves, where the reads of the half before have long arrived.
    constexpr int B = 2 * GA, B0 = B, B1 = G + B;
    // Block kt, in slots SLOT = kt % 2.  Past the last block the same instructions run: their loads bring nothing, what they read is
    // not used, and where the blocks are odd in number the one behind the last multiplies codes that were there, of one
    // of the blocks, under scales of 2^-127 each, which leaves every sum as it is.  (An end of its own for each number of
    // blocks costs registers: the accumulators of several ways meet, and are spilled.)
    auto block = [&](int kt, auto slot) {
        constexpr int SLOT = decltype(slot)::value;
        const Source from = source(kt + 2 < nk);
        const int sh = 8 * (kt & 3);
        const bool real = SLOT == 0 || kt < nk;
        const int sw = static_cast<int>(real ? sc.w >> sh : 0u);
        int sa[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = static_cast<int>(real ? sc.a[i] >> sh : 0u);
#pragma unroll
        for (int y = 0; y < 2 * G; ++y) {
            // at B0: this block's second tokens are there, and every wave has read its weights and first tokens;
            // at B1: the next block's weights and first tokens are there, and the second tokens are read
            // (where scale words are among those under way, the wait is for two more than it need be)
            if (y == B0 || y == B1) barrier_vm<Q1 + Q2>();
            const int h = y / G, x = y % G, t = x / (2 * GA), k = x / GA % 2, u = x % GA;
            f32x16& c = acc[t][h * GA + u];
            const float fw = fp8_scale(sw & 255), fa = fp8_scale(sa[h * GA + u] & 255);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c = mfma32x32x16(codes_bf16(w.w[t][k].c[2 * j], w.w[t][k].c[2 * j + 1], fw),
                                 codes_bf16(at[h][u].a[k].c[2 * j], at[h][u].a[k].c[2 * j + 1], fa), c);
            if (y >= B0 && y < B0 + 2 * GA) read_a(SLOT, at[1][(y - B0) / 2], GA + (y - B0) / 2, (y - B0) % 2);
            if (y >= B1 && y < B1 + 2 * GA) read_a(SLOT ^ 1, at[0][(y - B1) / 2], (y - B1) / 2, (y - B1) % 2);
            if (SLOT == 1 && y == B1 + 1) read_scales(kt + 1, sc_next);
#pragma unroll
            for (int j = 0; j < 2 * NT; ++j) {   // the next block's weights, GA products behind the last of those that they replace
                const int at_y = B1 + j * GA + GA - 1;
                if (at_y == y) read_w(SLOT ^ 1, w, j / 2, j % 2);
                if (at_y == y + 2 * G) read_w(SLOT, w, j / 2, j % 2);
            }
            constexpr int EACH = Q1 > G ? 2 : 1;   // instructions a product
            if (SLOT == 0 && y == B0) issue_scales(from, kt + 2);
            const int since = y >= B1 ? y - B1 : y - B0, n = y >= B1 ? Q2 : Q1;   // the first refill has ended when the second begins
#pragma unroll
            for (int q = EACH * since; q < EACH * (since + 1); ++q)
                if (q >= 0 && q < n) issue(from, kt + 2, SLOT, y >= B1, q);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (SLOT == 1) sc = sc_next;
    };
    static_assert(2 * G >= Q1 && G >= Q2, "a refill within half a block");

#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const Source from = source(true);
        if (b == 0) issue_scales(from, 0);
#pragma unroll
        for (int q = 0; q < Q1; ++q) issue(from, min(b, nk - 1), b, 0, q);
#pragma unroll
        for (int q = 0; q < Q2; ++q) issue(from, min(b, nk - 1), b, 1, q);
    }
    barrier_vm<Q1 + 2 * Q2>();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int t = 0; t < NT; ++t) read_w(0, w, t, k);
#pragma unroll
        for (int u = 0; u < GA; ++u) read_a(0, at[0][u], u, k);
    }
    read_scales(0, sc);
    for (int kt = 0; kt < nk; kt += 2) {
        block(kt, std::integral_constant<int, 0>{});
        block(kt + 1, std::integral_constant<int, 1>{});
    }
    wait_vm<0>();   // nothing may come to LDS behind the workgroup's end

    TO* out = static_cast<TO*>(p.out);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + wm * TM + 32 * i + r32;
        if (m >= p.m) continue;
        TO* row = out + m * p.ldo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n0 + wn * TN + kh * (TN / 2) + q * (TN / 8);
#pragma unroll
            for (int t = 0; t < NT; t += 2) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = acc[t][i][4 * q + e];
                    v[4 + e] = acc[t + 1][i][4 * q + e];
                }
                if (part) store_row<8>(part + static_cast<int64_t>(m) * p.n + n + 4 * t, p.n - n - 4 * t, v);
                else store_row<8>(row + n + 4 * t, p.n - n - 4 * t, v);
            }
        }
    }
}

// Tile number `tile` of tm: tokens fastest inside groups of gm.
__device__ __forceinline__ void tile_of(const TileMap& tm, int tile, int* m_tile, int* n_tile) {
    const int grp = tile / (tm.gm * tm.n_tiles);
    const int rem = tile - grp * tm.gm * tm.n_tiles;
    const int gsz = min(tm.gm, tm.m_tiles - grp * tm.gm);
    *m_tile = grp * tm.gm + rem % gsz;
    *n_tile = rem / gsz;
}

// Workgroup 8 j + x runs on XCD x, which takes an eighth of the tiles: those that it runs together share operands in its L2.
// -1: none.
__device__ __forceinline__ int tile_of_workgroup(int w, int tiles) {
    const int per = (tiles + 7) >> 3, j = w >> 3, tile = (w & 7) * per + j;
    return j < per && tile < tiles ? tile : -1;
}

// Two workgroups a CU; blockIdx.y: the K slice of `per` blocks.
template <typename TO>
__global__ void __launch_bounds__(256, 2) gemm_fp8_tiles_kernel(Fp8Gemm p, TileMap tm, int per) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kTileLds];
    const int tile = tile_of_workgroup(blockIdx.x, tm.m_tiles * tm.n_tiles);
    if (tile < 0) return;
    int mt, nt;
    tile_of(tm, tile, &mt, &nt);
    const int k0 = blockIdx.y * per;
    float* part = p.part ? p.part + static_cast<int64_t>(blockIdx.y) * p.m * p.n : nullptr;
    tile_fp8<TO>(p, mt * kTile, nt * kTile, k0, min(per, p.kb - k0), smem, part);
}

// Sum of the K slices, in their order; bound by their bytes and its launch (4 us).
template <typename TO>
__global__ void __launch_bounds__(256) gemm_fp8_join_kernel(Fp8Gemm p, int slices) {
    const int per_row = (p.n + 3) / 4;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int m = static_cast<int>(at / per_row), n = 4 * static_cast<int>(at - static_cast<int64_t>(m) * per_row);
    if (m >= p.m) return;
    const float* src = p.part + static_cast<int64_t>(m) * p.n + n;
    const int64_t step = static_cast<int64_t>(p.m) * p.n;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < slices; ++s) {
        float x[4];
        load_row<4>(src + s * step, p.n - n, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += x[e];
    }
    store_row<4>(static_cast<TO*>(p.out) + m * p.ldo + n, p.n - n, v);
}

// ---------------------------------------------------------------------------
// Which kernel, and how many K slices.
// ---------------------------------------------------------------------------
enum Kind { GEMV, TILES };
struct Plan {
    Kind kind;
    int slices, per;   // K slices of `per` blocks
    int rw;            // GEMV: 16 rw weights a workgroup
};

constexpr int kCus = 256;

int up(int a, int b) { return (a + b - 1) / b; }

// Slices that give every CU a workgroup, with two blocks a wave at least.
int gemv_slices(int workgroups, int kb) {
    return workgroups >= kCus / 2 ? 1 : std::max(1, std::min(kCus / workgroups, kb / (2 * kGemvWaves)));
}

Plan plan_of(int m, int n, int kb) {
    Plan q{TILES, 1, kb, 1};
    if (m <= 32) {
        // From 33 tokens on tiles are faster (64 x 3584 x 18944: 28 us, 58 here).  Past 16 tokens their re-reading shows: 64
        // weights a workgroup where those fill the chip (32 x 37888 x 3584: 39 us, with 32 weights 41, with 16 54; 24 x
        // 152064: 127, 138, 174), else 32 (20 x 4608 x 3584: 10.1, with 64 12.7, with 16 11.1).  Up to 16 tokens 16 weights
        // (8 x 2048 x 1536: 3.9, with 32 4.7, with 64 6.4; 4096 x 4096: 6.5 and 8.1; 8960 x 1536: 6.4 and 6.7), or 32 where their
        // workgroups are half the rounds (8 x 4608 x 3584: 7.2, with 16 8.2, with 64 11.2; 16 x 37888 x 3584: 33, 38, 35; one
        // token: 26.9 and 26.3).
        q.kind = GEMV;
        if (m <= 16) q.rw = 2 * up(up(n, 32), kCus) <= up(up(n, 16), kCus) ? 2 : 1;
        else q.rw = up(n, 64) * gemv_slices(up(n, 64), kb) >= kCus * 7 / 8 ? 4 : 2;
        q.slices = gemv_slices(up(n, 16 * q.rw), kb);
    } else {
        const int tiles = up(m, kTile) * up(n, kTile);
        if (tiles <= kCus) {
            // K slices.  A block of K takes a tile 0.75 us alone on its CU and 1.4 beside another, from the 257th workgroup of
            // the launch on (whose tiles are rounded up to eights: 84 of them in three slices are 264); slices cost a launch of
            // 3 us more and their sums, written and read at 3.5 TB/s.  33 x 4608 x 3584 in four: 14.7 us, whole 25.3, in
            // seven 16.4; 257 x 3584 x 18944 in six: 56.7, whole 111, in three 71.5; 512 x 4608 x 3584 whole: 27.1, in two 34.
            // Of 58 such sizes, each cut in all ways, the rule's choice is 8% behind the fastest at worst.
            auto time_of = [&](int s) {
                const int per = s > 1 ? up(up(kb, s), 4) * 4 : kb, slices = up(kb, per), wg = up(tiles, 8) * 8 * slices;
                return per * (wg <= kCus ? 0.75 : 1.4 * std::max(1.0, wg / (2.0 * kCus))) + (slices > 1 ? 3.0 + 8e-6 * slices * m * n / 3.5 : 0.0);
            };
            for (int s = 2; s <= 16 && s <= kb; ++s)
                if (time_of(s) < time_of(q.slices)) q.slices = s;
        }
    }
    q.per = up(kb, q.slices);
    if (q.kind == TILES) q.per = up(q.per, 4) * 4;   // whole scale words
    q.slices = up(kb, q.per);
    return q;
}

template <typename TO, int RW, int MT> void gemv(const Fp8Gemm& g, const Plan& q, hipStream_t s) {
    const dim3 grid(up(g.n, 16 * RW), q.slices);
    constexpr bool MANY = RW == 2 && MT == 1;   // taken from 129 workgroups on, so never in K slices
    if constexpr (!MANY)
        if (q.slices > 1) {
            gemv_fp8_kernel<TO, RW, MT, true><<<grid, 64 * kGemvWaves, 0, s>>>(g, q.per);
            return;
        }
    gemv_fp8_kernel<TO, RW, MT, false><<<grid, 64 * kGemvWaves, 0, s>>>(g, q.per);
}

template <typename TO> void run_plan(const Fp8Gemm& a, const Plan& q, hipStream_t s) {
    Fp8Gemm g = a;
    if (q.slices == 1) g.part = nullptr;
    if (q.kind == GEMV) {
        if (g.m <= 16 && q.rw == 1) gemv<TO, 1, 1>(g, q, s);
        else if (g.m <= 16) gemv<TO, 2, 1>(g, q, s);
        else if (q.rw == 2) gemv<TO, 2, 2>(g, q, s);
        else gemv<TO, 4, 2>(g, q, s);
    } else {
        TileMap tm{up(g.m, kTile), up(g.n, kTile), 0};
        tm.gm = std::min(tm.m_tiles, 8);
        gemm_fp8_tiles_kernel<TO><<<dim3(up(tm.m_tiles * tm.n_tiles, 8) * 8, q.slices), 256, 0, s>>>(g, tm, q.per);
    }
    if (q.slices > 1)
        gemm_fp8_join_kernel<TO><<<static_cast<int>((static_cast<int64_t>(g.m) * up(g.n, 4) + 255) / 256), 256, 0, s>>>(g, q.slices);
}

}  // namespace

size_t gemm_fp8_ws_bytes(int m, int n, int kb) {
    const int s = plan_of(m, n, kb).slices;
    return s > 1 ? sizeof(float) * static_cast<size_t>(s) * m * n : 0;
}

hipError_t launch_gemm_fp8(const Fp8Gemm& g, hipStream_t s) {
    const Plan q = plan_of(g.m, g.n, g.kb);
    if (g.out_dt == RL_DTYPE_FP32) run_plan<float>(g, q, s);
    else run_plan<uint16_t>(g, q, s);
    return hipGetLastError();
}

}  // namespace rl
