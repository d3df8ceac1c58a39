// fp8.cpp -- entry points of the 8-bit operators: argument checks and launches
// on the caller's stream.  No context, no allocation, no state.
#include "fp8.h"
#include "rl_decode.h"

#include <cmath>

using namespace rl;

namespace {

constexpr int kMaxRows = 1 << 20, kMaxWidth = 1 << 17, kMaxHidden = 1 << 15, kMaxTokens = 1 << 24, kMaxSeqs = 1 << 20;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool dtype_ok(int32_t dt) { return dt == RL_DTYPE_FP32 || dt == RL_DTYPE_BF16; }
size_t elem_bytes(int dt) { return dt == RL_DTYPE_FP32 ? 4 : 2; }
rl_status status_of(hipError_t e) { return e == hipSuccess ? RL_OK : RL_ERR_HIP; }

bool numbers_ok(const int32_t* p) { return p && aligned(p, 4); }

// rows of `width` entries, ld apart, at p; below 2^40 entries in all
bool rows_ok(int32_t dt, const void* p, int32_t n, int64_t width, int64_t ld) {
    return dtype_ok(dt) && p && aligned(p, elem_bytes(dt)) && ld >= width && ld <= (int64_t(1) << 40) / (n > 0 ? n : 1);
}
bool matrix_ok(const rl_fp8_matrix* m, int32_t k) {
    return m && m->codes && m->scales && aligned(m->codes, 16) && aligned(m->scales, 4) && m->ld % 16 == 0 && m->ld_scales % 4 == 0 &&
           m->ld >= 128 * static_cast<int64_t>(fp8_blocks(k)) && m->ld <= (1 << 20) && m->ld_scales >= fp8_blocks(k) &&
           m->ld_scales <= (1 << 20);
}
Fp8Out out_of(const rl_fp8_matrix* m) { return Fp8Out{m->codes, m->ld, m->scales, m->ld_scales}; }
Fp8In in_of(const rl_fp8_matrix* m) { return Fp8In{m->codes, m->ld, m->scales, m->ld_scales}; }

rl_status workspace_ok(const void* ws, size_t have, size_t need) {
    if (need == 0) return RL_OK;
    if (!ws || !aligned(ws, 256)) return RL_ERR_INVALID_ARG;
    return have < need ? RL_ERR_CAPACITY : RL_OK;
}

// bytes of one page of one kv-head, 0 for what is not supported
int64_t page_bytes(int32_t page_size, int32_t head_dim) {
    if (page_size < 32 || page_size > 65536 || page_size % 32 != 0 || (head_dim != 64 && head_dim != 128)) return 0;
    return (2 * static_cast<int64_t>(page_size) * (head_dim + 1) + 255) / 256 * 256;
}

// Pools end below 2^48 bytes: every offset in them, and their size, is a 64-bit number.
bool pool_ok(int32_t n_pages, int32_t n_kv_heads, int64_t block) {
    return n_pages > 0 && n_kv_heads > 0 && n_kv_heads <= 1024 && block > 0 && n_pages <= (int64_t(1) << 48) / (block * n_kv_heads);
}

// The runtime counts a launch's threads in 32 bits.  A workgroup of 256 takes 16 blocks of an fp32 matrix, so that the last 16
// below 2^28 would need 2^32; 16 threads take one token's head.
constexpr int64_t kMaxBlocks = (int64_t(1) << 28) - 16, kMaxHeads = (int64_t(1) << 28) - 1;
constexpr int64_t kMaxTiles = (int64_t(1) << 24) - 8;   // of 128 x 128, a workgroup each, rounded up to eights

bool cache_ok(const rl_kv_fp8* c, KvFp8* o) {
    if (!c || !c->pool || !aligned(c->pool, 256) || !c->page_table || !aligned(c->page_table, 4)) return false;
    if (c->n_seqs < 1 || c->n_seqs > kMaxSeqs || c->max_pages < 1) return false;
    const int64_t block = page_bytes(c->page_size, c->head_dim);
    if (!pool_ok(c->n_pages, c->n_kv_heads, block) || static_cast<int64_t>(c->max_pages) * c->page_size > INT32_MAX) return false;
    *o = KvFp8{static_cast<uint8_t*>(c->pool), c->page_table, c->n_seqs, c->max_pages, c->n_pages, c->page_size, c->n_kv_heads,
               c->head_dim, block};
    return true;
}

}  // namespace

extern "C" {

rl_status rl_rmsnorm_quant(int32_t n, int32_t hidden, int32_t dtype, const void* x, int64_t ldx, int32_t add_dtype, const void* add,
                         int64_t ld_add, int32_t w_dtype, const void* weight, double eps, void* out_sum, int64_t ld_sum,
                         const rl_fp8_matrix* out, void* stream) {
    if (n < 0 || n > kMaxRows || hidden < 1 || hidden > kMaxHidden || !dtype_ok(dtype) || !dtype_ok(w_dtype)) return RL_ERR_INVALID_ARG;
    if (!(eps > 0.0) || !(eps <= 1.0) || static_cast<float>(eps) == 0.0f) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    if (!rows_ok(dtype, x, n, hidden, ldx) || !rows_ok(w_dtype, weight, 1, hidden, hidden) || !matrix_ok(out, hidden)) return RL_ERR_INVALID_ARG;
    if (add && !rows_ok(add_dtype, add, n, hidden, ld_add)) return RL_ERR_INVALID_ARG;
    if (out_sum && !rows_ok(dtype, out_sum, n, hidden, ld_sum)) return RL_ERR_INVALID_ARG;
    const NormArgs a{n, hidden, x, ldx, dtype, add, ld_add, add_dtype, weight, w_dtype, eps, 1.0 / hidden, out_sum, ld_sum,
                     out_of(out)};
    return status_of(launch_rmsnorm_fp8(a, static_cast<hipStream_t>(stream)));
}

rl_status rl_quantise(int32_t form, int32_t n, int32_t k, int32_t dtype, const void* x, int64_t ldx, const rl_fp8_matrix* out,
                          void* stream) {
    if (form < RL_FP8_ROWS || form > RL_FP8_TILES || n < 0 || n > kMaxRows || k < 1 || k > kMaxWidth) return RL_ERR_INVALID_ARG;
    if (n == 0) return dtype_ok(dtype) ? RL_OK : RL_ERR_INVALID_ARG;
    if (!rows_ok(dtype, x, n, form == RL_FP8_SWIGLU ? 2 * static_cast<int64_t>(k) : k, ldx) || !matrix_ok(out, k)) return RL_ERR_INVALID_ARG;
    if (static_cast<int64_t>(n) * fp8_blocks(k) > kMaxBlocks) return RL_ERR_UNSUPPORTED;
    return status_of(launch_quantise_fp8(form, n, k, dtype, x, ldx, out_of(out), static_cast<hipStream_t>(stream)));
}

size_t rl_gemm_quant_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    return m < 1 || m > kMaxRows || n < 1 || n > kMaxRows || k < 1 || k > kMaxWidth ? 0 : gemm_fp8_ws_bytes(m, n, fp8_blocks(k));
}

rl_status rl_gemm_quant(int32_t m, int32_t n, int32_t k, const rl_fp8_matrix* a, const rl_fp8_matrix* w, int32_t out_dtype, void* out,
                      int64_t ldo, void* workspace, size_t ws_bytes, void* stream) {
    if (m < 0 || m > kMaxRows || n < 1 || n > kMaxRows || k < 1 || k > kMaxWidth || !dtype_ok(out_dtype)) return RL_ERR_INVALID_ARG;
    if (m == 0) return RL_OK;
    if (!matrix_ok(a, k) || !matrix_ok(w, k) || !rows_ok(out_dtype, out, m, n, ldo)) return RL_ERR_INVALID_ARG;
    const int kb = fp8_blocks(k);
    if (static_cast<int64_t>(fp8_blocks(m)) * fp8_blocks(n) > kMaxTiles) return RL_ERR_UNSUPPORTED;
    if (const rl_status st = workspace_ok(workspace, ws_bytes, gemm_fp8_ws_bytes(m, n, kb)); st != RL_OK) return st;
    const Fp8Gemm g{m, n, kb, in_of(a), in_of(w), out, ldo, out_dtype, static_cast<float*>(workspace)};
    return status_of(launch_gemm_fp8(g, static_cast<hipStream_t>(stream)));
}

size_t rl_kv_quant_bytes(int32_t n_pages, int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
    const int64_t block = page_bytes(page_size, head_dim);
    return pool_ok(n_pages, n_kv_heads, block) ? static_cast<size_t>(block) * n_pages * n_kv_heads : 0;
}

rl_status rl_kv_quant_append(const rl_kv_fp8* cache, int32_t n, const int32_t* seqs, const int32_t* positions, int32_t dtype,
                           const void* k, int64_t ldk, const void* v, int64_t ldv, void* stream) {
    KvFp8 c;
    if (!cache_ok(cache, &c) || n < 0 || n > kMaxTokens || !dtype_ok(dtype)) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    if (static_cast<int64_t>(n) * c.heads > kMaxHeads) return RL_ERR_UNSUPPORTED;
    const int64_t width = static_cast<int64_t>(c.heads) * c.dim;
    if (!numbers_ok(seqs) || !numbers_ok(positions)) return RL_ERR_INVALID_ARG;
    if (!rows_ok(dtype, k, n, width, ldk) || !rows_ok(dtype, v, n, width, ldv)) return RL_ERR_INVALID_ARG;
    const KvTokens t{n, seqs, positions, k, v, ldk, ldv, nullptr, nullptr, 0, 0, dtype};
    return status_of(launch_kv_fp8_append(c, t, static_cast<hipStream_t>(stream)));
}

rl_status rl_kv_quant_read(const rl_kv_fp8* cache, int32_t n, const int32_t* seqs, const int32_t* positions, int32_t dtype,
                         void* out_k, int64_t ldk, void* out_v, int64_t ldv, void* stream) {
    KvFp8 c;
    if (!cache_ok(cache, &c) || n < 0 || n > kMaxTokens || !dtype_ok(dtype)) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    if (static_cast<int64_t>(n) * c.heads > kMaxHeads) return RL_ERR_UNSUPPORTED;
    const int64_t width = static_cast<int64_t>(c.heads) * c.dim;
    if (!numbers_ok(seqs) || !numbers_ok(positions)) return RL_ERR_INVALID_ARG;
    if (!rows_ok(dtype, out_k, n, width, ldk) || !rows_ok(dtype, out_v, n, width, ldv)) return RL_ERR_INVALID_ARG;
    const KvTokens t{n, seqs, positions, nullptr, nullptr, 0, 0, out_k, out_v, ldk, ldv, dtype};
    return status_of(launch_kv_fp8_read(c, t, static_cast<hipStream_t>(stream)));
}

size_t rl_attention_quant_workspace_bytes(int32_t n, int32_t n_kv_heads, int32_t n_q_heads, int32_t head_dim, int32_t max_length) {
    if (n < 1 || n > kMaxSeqs || n_kv_heads < 1 || n_kv_heads > 1024 || n_q_heads < n_kv_heads || n_q_heads % n_kv_heads != 0 ||
        n_q_heads / n_kv_heads > 16 || (head_dim != 64 && head_dim != 128) || max_length < 0 ||
        !attention_fp8_fits(n, n_kv_heads, n_q_heads, max_length))
        return 0;
    return attention_fp8_ws_bytes(n, n_kv_heads, n_q_heads, head_dim, max_length);
}

rl_status rl_attention_quant(const rl_kv_fp8* cache, int32_t n, const int32_t* seqs, const int32_t* lengths, int32_t max_length,
                           int32_t dtype, const void* q, int64_t ldq, int32_t n_q_heads, double scale, void* out, int64_t ldo,
                           void* workspace, size_t ws_bytes, void* stream) {
    KvFp8 c;
    if (!cache_ok(cache, &c) || n < 0 || n > kMaxSeqs || !dtype_ok(dtype) || !std::isfinite(static_cast<float>(scale))) return RL_ERR_INVALID_ARG;
    if (n_q_heads < c.heads || n_q_heads % c.heads != 0 || n_q_heads / c.heads > 16) return RL_ERR_INVALID_ARG;
    if (max_length < 0 || max_length > static_cast<int64_t>(c.max_pages) * c.page || (!seqs && n > c.n_seqs)) return RL_ERR_INVALID_ARG;
    if (n == 0) return RL_OK;
    if (!attention_fp8_fits(n, c.heads, n_q_heads, max_length)) return RL_ERR_UNSUPPORTED;
    const int64_t width = static_cast<int64_t>(n_q_heads) * c.dim;
    if (!numbers_ok(lengths) || !aligned(seqs, 4)) return RL_ERR_INVALID_ARG;
    if (!rows_ok(dtype, q, n, width, ldq) || !rows_ok(dtype, out, n, width, ldo)) return RL_ERR_INVALID_ARG;
    if (const rl_status st = workspace_ok(workspace, ws_bytes, attention_fp8_ws_bytes(n, c.heads, n_q_heads, c.dim, max_length)); st != RL_OK)
        return st;
    const AttnFp8 a{c, n, max_length, seqs, lengths, q, ldq, out, ldo, dtype, n_q_heads, static_cast<float>(scale),
                    static_cast<float*>(workspace)};
    return status_of(launch_attention_fp8(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
