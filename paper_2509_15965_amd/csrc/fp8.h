// fp8.h -- what the 8-bit operators share: e4m3 codes under power-of-two block
// scales, wide loads of either element type, the arguments of their launches.
#pragma once

#include "rl_device.h"

namespace rl {

constexpr int kFp8Block = 128;   // entries of a row under one scale
__host__ __device__ constexpr int fp8_blocks(int k) { return (k + kFp8Block - 1) / kFp8Block; }

// [rows][ld] codes and [rows or rows / 128][lds] scale bytes
struct Fp8Out { uint8_t* codes; int64_t ld; uint8_t* scales; int64_t lds; };
struct Fp8In { const uint8_t* codes; int64_t ld; const uint8_t* scales; int64_t lds; };

struct NormArgs {
    int n, hidden;
    const void* x; int64_t ldx; int x_dt;
    const void* add; int64_t ld_add; int add_dt;   // or null
    const void* w; int w_dt;
    double eps, per_entry;                         // 1 / hidden
    void* sum; int64_t ld_sum;                     // x_dt; or null
    Fp8Out out;
};
hipError_t launch_rmsnorm_fp8(const NormArgs& a, hipStream_t s);

// form: 0 rows, 1 SwiGLU of the row's two halves of k entries, 2 tiles of 128 x 128
hipError_t launch_quantise_fp8(int form, int n, int k, int dt, const void* x, int64_t ldx, const Fp8Out& out, hipStream_t s);

struct Fp8Gemm {
    int m, n, kb;                  // kb blocks of 128 codes
    Fp8In a, w;
    void* out; int64_t ldo; int out_dt;
    float* part;                   // fp32 sums of the K slices, [slice][m][n]
};
size_t gemm_fp8_ws_bytes(int m, int n, int kb);
hipError_t launch_gemm_fp8(const Fp8Gemm& g, hipStream_t s);

// The cache: page p, kv-head h is `block` bytes at (p * heads + h) * block.
struct KvFp8 {
    uint8_t* pool;
    const int32_t* table;          // [n_seqs][max_pages]
    int n_seqs, max_pages, n_pages, page, heads, dim;
    int64_t block;
};
struct KvTokens {
    int n;
    const int32_t *seqs, *pos;
    const void *k, *v; int64_t ldk, ldv;       // append
    void *out_k, *out_v; int64_t ld_ok, ld_ov; // read
    int dt;
};
hipError_t launch_kv_fp8_append(const KvFp8& c, const KvTokens& t, hipStream_t s);
hipError_t launch_kv_fp8_read(const KvFp8& c, const KvTokens& t, hipStream_t s);

struct AttnFp8 {
    KvFp8 c;
    int n, max_length;
    const int32_t *seqs, *lengths;             // seqs null: row i is sequence i
    const void* q; int64_t ldq;
    void* out; int64_t ldo;
    int dt, heads;                             // query heads
    float scale;
    float* part;
};
bool attention_fp8_fits(int n, int kv_heads, int heads, int max_length);   // its launches' threads can be counted in 32 bits
size_t attention_fp8_ws_bytes(int n, int kv_heads, int heads, int dim, int max_length);
hipError_t launch_attention_fp8(const AttnFp8& a, hipStream_t s);

// Scale byte b of a block whose largest finite magnitude is a: 2^(b - 127) is the
// smallest power of two with a / 2^(b - 127) <= 448 = 1.75 x 2^8, and b >= 1 so
// that it and its reciprocal are normal fp32 numbers; 127 for a = 0.  From the
// bits of a: exponent - 8, one more where the significand is above 1.75.
__device__ __forceinline__ int fp8_scale_byte(float a) {
    const uint32_t u = __float_as_uint(a);
    const int b = static_cast<int>(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return u == 0u ? 127 : b < 1 ? 1 : b;
}
__device__ __forceinline__ float fp8_scale(int b) { return __uint_as_float(static_cast<uint32_t>(b) << 23); }
__device__ __forceinline__ float fp8_inverse(int b) { return __uint_as_float(static_cast<uint32_t>(254 - b) << 23); }

// four codes of four numbers, the first in the lowest byte (round to nearest even; NaN stays)
__device__ __forceinline__ uint32_t fp8_pack4(const float* v, float inv) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w, true));
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// eight codes as bf16 numbers, times the scale
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Entries of a row that a lane moves at once: 16 bytes of its type.
template <typename T> constexpr int kEntries = 16 / sizeof(T);

// Vectors at any address that their elements' alignment allows: the hardware takes unaligned global accesses.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// E entries of a row, of which `left` are there (the others are 0).
template <int E, typename T> __device__ __forceinline__ void load_row(const T* p, int left, float* v) {
    if (left >= E) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int q = 0; q < E; q += 4) {
                const u32x4 a = *reinterpret_cast<const u32x4_any*>(p + q);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[q + e] = __uint_as_float(a[e]);
            }
        } else {
            uint32_t a[E / 2];
            if constexpr (E == 8) {
                const u32x4 w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = w[e];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2_any*>(p);
                a[0] = w[0];
                a[1] = w[1];
            }
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                v[2 * e] = __uint_as_float(a[e] << 16);
                v[2 * e + 1] = __uint_as_float(a[e] & 0xFFFF0000u);
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < left ? Elem<T>::load(p, e) : 0.0f;
}
template <int E, typename T> __device__ __forceinline__ void store_row(T* p, int left, const float* v) {
    if (left >= E) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int q = 0; q < E; q += 4)
                *reinterpret_cast<u32x4_any*>(p + q) = u32x4{__float_as_uint(v[q]), __float_as_uint(v[q + 1]), __float_as_uint(v[q + 2]),
                                                             __float_as_uint(v[q + 3])};
        } else {
            uint32_t w[E / 2];
#pragma unroll
            for (int e = 0; e < E / 2; ++e) w[e] = f32_to_bf16(v[2 * e]) | static_cast<uint32_t>(f32_to_bf16(v[2 * e + 1])) << 16;
            if constexpr (E == 8) *reinterpret_cast<u32x4_any*>(p) = u32x4{w[0], w[1], w[2], w[3]};
            else *reinterpret_cast<u32x2_any*>(p) = u32x2{w[0], w[1]};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < left) Elem<T>::store(p, e, v[e]);
}

// v of the lane N places on in its row of 16 (cyclic)
template <int N> __device__ __forceinline__ float row_rotated(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + N, 0xF, 0xF, true));
}
// largest of LANES neighbouring lanes (8 .. 64); NaN counts only where there is nothing else
template <int LANES> __device__ __forceinline__ float lanes_max(float v) {
    if constexpr (LANES == 8) {
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
        return v;
    }
    v = fmaxf(v, row_rotated<8>(v));
    v = fmaxf(v, row_rotated<4>(v));
    v = fmaxf(v, row_rotated<2>(v));
    v = fmaxf(v, row_rotated<1>(v));
#pragma unroll
    for (int o = 16; o < LANES; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
template <int N> __device__ __forceinline__ double row_rotated(double v) {
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), 0x120 + N, 0xF, 0xF, true);
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), 0x120 + N, 0xF, 0xF, true), lo);
}
// sum of LANES neighbouring lanes (16 .. 64)
template <int LANES> __device__ __forceinline__ double lanes_sum(double v) {
    v += row_rotated<8>(v);
    v += row_rotated<4>(v);
    v += row_rotated<2>(v);
    v += row_rotated<1>(v);
#pragma unroll
    for (int o = 16; o < LANES; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

constexpr float kLargestFloat = 3.402823466e38f;
// Infinities in v become NaN; the largest magnitude of the finite ones.
template <int E> __device__ __forceinline__ float drop_infinities(float* v) {
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const bool fine = fabsf(v[e]) <= kLargestFloat;
        a = fine ? fmaxf(a, fabsf(v[e])) : a;
        v[e] = fine ? v[e] : __uint_as_float(0x7FC00000u);
    }
    return a;
}
template <int E> __device__ __forceinline__ float largest(const float* v) {
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) a = fmaxf(a, fabsf(v[e]));
    return a;
}

template <int E> __device__ __forceinline__ void fp8_pack(const float* v, float inv, uint32_t* codes) {
#pragma unroll
    for (int q = 0; q < E / 4; ++q) codes[q] = fp8_pack4(v + 4 * q, inv);
}
template <int E> __device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t* codes) {
    if constexpr (E == 4) *reinterpret_cast<uint32_t*>(p) = codes[0];
    else *reinterpret_cast<uint2*>(p) = make_uint2(codes[0], codes[1]);
}

// The E numbers of a lane, LANES lanes a block, as codes; the block's scale byte.
template <int E, int LANES> __device__ __forceinline__ int fp8_encode(float* v, uint32_t* codes) {
    float a = lanes_max<LANES>(largest<E>(v));
    if (a > kLargestFloat) a = lanes_max<LANES>(drop_infinities<E>(v));   // the same in all lanes of the block
    const int b = fp8_scale_byte(a);
    fp8_pack<E>(v, fp8_inverse(b), codes);
    return b;
}

}  // namespace rl
