// The entry points of attention over latent rows: checks of arguments, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include <cuda_runtime.h>

#include "head_product.cuh"
#include "kv_checks.h"
#include "latent_attend.cuh"
#include "latent_expand.cuh"
#include "latent_prompts.cuh"
#include "latent_write.cuh"
#include "tma_maps.h"

using namespace spm;

namespace {

constexpr int kMaxSmem = 232448;

int check_latent_shape(const char* call, const spm_latent_cache* kv) {
    if (!kv) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (kv->latent_dim < 128 || kv->latent_dim > 512 || kv->latent_dim % 128)
        return fail(call, SPM_ERR_CONFIG, "latent_dim " + std::to_string(kv->latent_dim) + " not supported: 128, 256, 384 or 512");
    if (kv->rope_dim < 16 || kv->rope_dim > 64 || kv->rope_dim % 16)
        return fail(call, SPM_ERR_CONFIG, "rope_dim " + std::to_string(kv->rope_dim) + " not supported: 16, 32, 48 or 64");
    if (kv->page_size < 16 || kv->page_size % 16 || kv->page_size > 65536)
        return fail(call, SPM_ERR_CONFIG, "page_size " + std::to_string(kv->page_size) + " is not a multiple of 16 up to 65536");
    if (kv->n_pages < 0) return fail(call, SPM_ERR_INVALID_ARG, "n_pages is negative");
    if (static_cast<long long>(kv->n_pages) * kv->page_size > INT32_MAX) return fail(call, SPM_ERR_CONFIG, "n_pages * page_size is over 2^31 - 1 tokens");
    return SPM_OK;
}
int check_latent_cache(const char* call, const spm_latent_cache* kv) {
    if (int rc = check_latent_shape(call, kv)) return rc;
    if (!kv->rows && kv->n_pages > 0) return fail(call, SPM_ERR_INVALID_ARG, "rows is null");
    if (!aligned(kv->rows, 16) || !aligned(kv->status, 4))
        return fail(call, SPM_ERR_INVALID_ARG, "rows must be 16-byte aligned, status 4-byte aligned");
    return SPM_OK;
}
int check_heads(const char* call, int n) { return n >= 1 && n <= 1024 ? SPM_OK : fail(call, SPM_ERR_CONFIG, "heads outside 1..1024"); }

LatentPool pool_of(const spm_latent_cache* kv) {
    return {static_cast<__nv_bfloat16*>(kv->rows), kv->status, kv->n_pages, kv->page_size, kv->latent_dim, kv->rope_dim};
}

// ---- absorbed attention ----
// Columns of a CTA: what a sequence has, in equal blocks of at most 64 (fp32, three parts each: 16). max_rows may be a guess: any choice is right.
int columns_of(const spm_kv_batch* b, int n_heads, int dtype) {
    if (dtype == SPM_DTYPE_FP32) return 16;
    long long rows = 1;
    if (b->row_start && b->n_seq > 0) rows = b->max_rows > 0 ? b->max_rows : (b->n_rows + b->n_seq - 1) / b->n_seq;
    const long long columns = std::max(1ll, std::min<long long>(rows, b->n_rows) * n_heads), blocks = (columns + 63) / 64;
    return int(((columns + blocks - 1) / blocks + 15) / 16 * 16);
}
constexpr size_t kLaJoinBytes = (kLaMaxCtas * sizeof(int4) + 255) / 256 * 256;
size_t attend_bytes(int cols, int latent) { return kLaJoinBytes + kLaMaxCtas * 2 * size_t(cols) * (latent + 2) * sizeof(float); }

template <typename T, int COLS>
cudaError_t launch_attend(LatentAttendArgs a, int dev, int sms, cudaStream_t st) {
    const int page_size = a.kv.page_size;
    using S = LaShape<T, COLS>;
    cudaError_t e = allow_smem<latent_attend_kernel<T, COLS>>(dev, kMaxSmem);
    if (e != cudaSuccess) return e;
    const int fixed = kLaOwnBytes + S::fixed(a.chunks), stage = a.chunks * kLaChunkBytes;
    a.stages = std::min(kLaMaxStages, (kMaxSmem - fixed) / stage);
    a.box = page_size % 64 == 0 ? 64 : page_size % 32 == 0 ? 32 : 16;
    CUtensorMap map{};                           // (a pool without pages: no copy is made)
    if (a.kv.n_pages > 0 && !make_token_map(&map, a.kv.rows, a.kv.latent + a.kv.rope, uint64_t(a.kv.n_pages) * page_size, a.box)) return cudaErrorInvalidValue;
    const int ctas = std::min(sms, kLaMaxCtas);
    e = launch_early(latent_attend_kernel<T, COLS>, ctas, kLaThreads, fixed + a.stages * stage, st, a, map);
    return e == cudaSuccess ? launch_early(latent_join_kernel<T, COLS>, kLaJoinBlocks, kLaJoinThreads, 0, st, a, ctas) : e;
}

// ---- expanded attention ----
// The workspace: keys and values of a round's heads, [heads][tokens][head_dim] each, the shared parts of keys, [heads][tokens][64] (written where a
// head's differ) and [tokens][64], a bit a token, powers of two of keys and of values for each 32 tokens, and the attention's items
struct Expanded { int tokens, heads, rounds; size_t values, own, shared, there, key_exps, value_exps, items, bytes; int n_items; };
constexpr size_t kLxMost = size_t(512) << 20;    // of keys and values together, where more than one head is more
Expanded expanded_of(const spm_kv_batch* b, int n_heads, int head_dim, int n_tokens) {
    Expanded e{};
    e.tokens = int(std::max(1ll, (n_tokens + 127ll * b->n_seq) / 128) * 128);
    const size_t head = size_t(e.tokens) * (2 * head_dim + 64) * 2;
    e.rounds = int((n_heads + std::max<size_t>(1, kLxMost / head) - 1) / std::max<size_t>(1, kLxMost / head));
    e.heads = (n_heads + e.rounds - 1) / e.rounds;
    e.rounds = (n_heads + e.heads - 1) / e.heads;
    const size_t rows = size_t(e.heads) * e.tokens;
    e.values = rows * head_dim * 2;
    e.own = 2 * e.values;
    e.shared = e.own + rows * 128;
    e.there = e.shared + size_t(e.tokens) * 128;
    e.key_exps = e.there + size_t(e.tokens) / 8;
    e.value_exps = e.key_exps + size_t(e.heads) * e.tokens / 16;
    e.items = (e.value_exps + size_t(e.heads) * e.tokens / 16 + 15) / 16 * 16;
    e.n_items = b->n_rows / kPfCols + b->n_seq;
    e.bytes = e.items + size_t(e.n_items) * sizeof(LxItem);
    return e;
}
int check_expanded(const char* call, const spm_kv_batch* b, int n_heads, int head_dim, int n_tokens, int dtype) {
    if (int rc = check_dtype(call, dtype)) return rc;
    if (dtype != SPM_DTYPE_BF16) return fail(call, SPM_ERR_CONFIG, "the expanded form is for bf16 rows; fp32 rows have the absorbed form");
    if (int rc = check_heads(call, n_heads)) return rc;
    if (head_dim != 64 && head_dim != 128) return fail(call, SPM_ERR_CONFIG, "head_dim " + std::to_string(head_dim) + " not supported: 64 or 128");
    // (rows of the workspace are counted in 32 bits, the shared parts of keys behind one head's; more heads a round are 512 MB at most)
    if (n_tokens < 0 || n_tokens + 127ll * b->n_seq >= 1ll << 30) return fail(call, SPM_ERR_INVALID_ARG, "n_tokens outside 0..2^30 - 127 n_seq - 1");
    if (static_cast<long long>(b->n_rows) * n_heads > INT32_MAX - 64) return fail(call, SPM_ERR_INVALID_ARG, "n_rows * n_heads is over 2^31 - 65");
    return SPM_OK;
}
int check_matrices(const char* call, const char* name, const spm_matrices* w, int rows) {
    if (!w || !w->p) return fail(call, SPM_ERR_INVALID_ARG, std::string(name) + " is null");
    if (!aligned(w->p, 16) || w->row_stride % 8 || w->head_stride % 8 || w->row_stride < rows || w->head_stride < rows)
        return fail(call, SPM_ERR_INVALID_ARG, std::string(name) + ": rows of weights must start on 16-byte boundaries and not overlap");
    return SPM_OK;
}

template <int HD>
cudaError_t launch_expanded(LatentExpandArgs x, LatentPromptArgs a, const Expanded& e, int n_heads, const CUtensorMap& rows, const CUtensorMap& wk, const CUtensorMap& wv,
                            const CUtensorMap& keys, const CUtensorMap& ropes, const CUtensorMap& ropes32, const CUtensorMap& values, int dev, int sms, cudaStream_t st) {
    cudaError_t err = allow_smem<latent_expand_kernel<HD>>(dev, kMaxSmem);
    if (err == cudaSuccess) err = allow_smem<latent_prompt_kernel<HD>>(dev, LpShape<HD>::smem);
    const int fixed = kLxOwnBytes + 1024 + x.kv.latent / 64 * kLxChunkBytes, stage = 2 * HD * 128;
    x.stages = std::min(8, (kMaxSmem - fixed) / stage);
    const int tiles = e.tokens / kLxTile;
    for (int h0 = 0; err == cudaSuccess && h0 < n_heads; h0 += e.heads) {
        x.h0 = a.h0 = h0;
        x.heads = a.heads = std::min(e.heads, n_heads - h0);
        const long long units = static_cast<long long>(tiles) * x.heads;
        err = launch_early(latent_expand_kernel<HD>, unsigned(std::min<long long>(units, sms)), kLxThreads, fixed + x.stages * stage, st, x, rows, wk, wv);
        if (err != cudaSuccess) break;
        const long long items = static_cast<long long>(e.n_items) * a.heads;
        if (items > INT32_MAX) return cudaErrorInvalidValue;
        err = launch_early(latent_prompt_kernel<HD>, unsigned(items), kLpThreads, LpShape<HD>::smem, st, a, keys, ropes, ropes32, values);
    }
    return err;
}

template <typename T, bool TRANSPOSED>
cudaError_t launch_product(HeadProductArgs a, int n_heads, int out, int dev, cudaStream_t st) {
    // CTAs of 64 rows and 128 outputs read everything once, and pay where there are rows that fill them and enough of them for most SMs. Kernel times in us,
    // these / the others, heads x in to out, transposed (T) or not:
    //   bf16  128 x 512 to 128 T: 32 rows 10.1 / 9.3, 48 10.6 / 13.3, 64 10.6 / 13.8, 128 18.4 / 22.5;  128 x 128 to 512: 32 rows 13.9 / 10.9, 48 14.3 / 17.5, 128 24.9 / 30.8
    //   fp32  128 x 512 to 128 T: 32 rows 17.0 / 14.7, 48 17.7 / 17.1, 49 17.5 / 20.8, 64 18.1 / 21.4;  128 x 128 to 512: 32 rows 21.3 / 16.7, 48 22.6 / 22.9, 128 40.3 / 51.6
    //   few tiles, bf16 / fp32  16 x 128 to 512, 64 rows, 64 tiles: 5.6 / 5.7, 7.3 / 6.3;  16 x 512 to 128 T, 400 rows, 112 tiles: 10.2 / 11.9, 17.4 / 16.9;
    //   20 x 384 to 128 T, 400 rows, 140 tiles: 8.6 / 11.0, 14.2 / 17.6;  33 x 64 to 128, 128 rows, 66 tiles: 4.9 / 4.9, 6.2 / 5.5
    const long long tiles = (a.n_rows + kHtRows - 1ll) / kHtRows * ((out + kHtOut - 1) / kHtOut);
    if (a.n_rows > (sizeof(T) == 4 ? 48 : 32) && tiles * n_heads >= 96) {
        const cudaError_t e = allow_smem<head_product_tile_kernel<T, TRANSPOSED>>(dev, HtShape<T>::smem);
        if (e != cudaSuccess) return e;
        a.out_tiles = (out + kHtOut - 1) / kHtOut;
        return launch_early(head_product_tile_kernel<T, TRANSPOSED>, dim3(unsigned(tiles), n_heads), kHtThreads, HtShape<T>::smem, st, a, out);
    }
    // fp32 rows take registers threefold: 16 of them a CTA. Eight warps wait less long for one another than four, but where these are more CTAs than the
    // SMs hold of them (two of 16 bf16 rows, else one) four are better. Kernel times in us, four warps / eight: bf16 16 x 512 to 128 T, 16 rows, 32 CTAs 6.1 / 5.1;
    // 128 x 512 to 128 T, 256 CTAs: 8 rows 7.9 / 7.5, 16 rows 7.9 / 8.1, 32 rows 9.3 / 11.9; 20 x 384 to 128 T, 128 rows, 160 CTAs 6.7 / 9.8;
    // fp32 16 x 512 to 128 T: 64 rows, 128 CTAs 7.7 / 6.5, 128 rows, 256 CTAs 8.4 / 11.0; 128 x 512 to 128 T, 16 rows, 256 CTAs 9.9 / 12.2
    const bool one = a.n_rows <= 16 || sizeof(T) == 4;
    a.out_tiles = out / kHpOut;
    const dim3 grid(unsigned((a.n_rows + (one ? 15 : 31)) / (one ? 16 : 32)) * a.out_tiles, n_heads);
    const bool many = static_cast<long long>(grid.x) * n_heads > (one && sizeof(T) == 2 ? 2 : 1) * 148;
    if constexpr (sizeof(T) == 2)
        if (!one) return many ? launch_early(head_product_kernel<T, TRANSPOSED, 2, 4>, grid, 128, 0, st, a) : launch_early(head_product_kernel<T, TRANSPOSED, 2, 8>, grid, 256, 0, st, a);
    return many ? launch_early(head_product_kernel<T, TRANSPOSED, 1, 4>, grid, 128, 0, st, a) : launch_early(head_product_kernel<T, TRANSPOSED, 1, 8>, grid, 256, 0, st, a);
}

}  // namespace

extern "C" {

int spm_latent_write(const spm_latent_cache* kv, const spm_kv_batch* batch, const spm_rope* rope, const int32_t* positions, int64_t pos_stride,
                     const spm_rows* q, const spm_rows* q_out, int n_q_heads, const spm_rows* latent, const spm_rows* key, int dtype, void* stream) {
    const char* call = "spm_latent_write";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_latent_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (n_q_heads < 0 || n_q_heads > 1024) return fail(call, SPM_ERR_INVALID_ARG, "n_q_heads outside 0..1024");
    if (q && !rope) return fail(call, SPM_ERR_INVALID_ARG, "q without rope: there is nothing to do to it");
    if (rope && rope->q_gamma) return fail(call, SPM_ERR_INVALID_ARG, "q_gamma: queries have no norm here");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    if (rope)
        if (int rc = check_rope(call, rope, positions, pos_stride, batch->n_rows, kv->rope_dim)) return rc;
    if (int rc = check_rows(call, "latent", latent, dtype)) return rc;
    if (int rc = check_rows(call, "key", key, dtype)) return rc;
    if (q) {
        if (int rc = check_rows(call, "q", q, dtype)) return rc;
        if (int rc = check_rows(call, "q_out", q_out, dtype)) return rc;
        if (q->p == q_out->p && other_strides(q, q_out)) return fail(call, SPM_ERR_INVALID_ARG, "q_out in q's place has other strides");
    }
    LatentWriteArgs a{};
    a.kv = pool_of(kv);
    a.batch = batch_of(batch);
    if (rope) { a.rope = rope_of(rope, positions, pos_stride); a.turn = 1; }
    if (q) { a.q = rows_of(q); a.q_out = rows_of(q_out); a.q_heads = n_q_heads; }
    a.latent = rows_of(latent); a.key = rows_of(key);
    a.n_rows = batch->n_rows;
    // a row a warp, or where these are few its query heads shared out
    constexpr int kWarps = 592 * kKvWarps;       // that the GPU has room for
    const int parts = std::max(1, std::min((a.q_heads + 7) / 8, kWarps / a.n_rows));
    const dim3 grid(unsigned((a.n_rows + kKvWarps - 1ll) / kKvWarps), parts);
    const auto st = static_cast<cudaStream_t>(stream);
    return launched(call, dtype == SPM_DTYPE_BF16 ? launch_early(latent_write_kernel<__nv_bfloat16>, grid, kKvWarps * 32, 0, st, a)
                                                  : launch_early(latent_write_kernel<float>, grid, kKvWarps * 32, 0, st, a));
}

int spm_latent_attend_workspace(const spm_latent_cache* kv, const spm_kv_batch* batch, int n_heads, int dtype, size_t* bytes) {
    const char* call = "spm_latent_attend_workspace";
    if (!bytes) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_latent_shape(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (int rc = check_heads(call, n_heads)) return rc;
    *bytes = attend_bytes(columns_of(batch, n_heads, dtype), kv->latent_dim);
    return SPM_OK;
}

int spm_latent_attend(const spm_latent_cache* kv, const spm_kv_batch* batch, const spm_rows* q, int n_heads, const spm_rows* out, float scale,
                      int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const char* call = "spm_latent_attend";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_latent_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (int rc = check_heads(call, n_heads)) return rc;
    const float factor = scale * 1.4426950408889634f;
    if (!std::isfinite(factor)) return fail(call, SPM_ERR_INVALID_ARG, "scale is not finite, or not below 2^127");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    if (int rc = check_rows(call, "q", q, dtype)) return rc;
    if (int rc = check_rows(call, "out", out, dtype)) return rc;
    if (q->p == out->p) return fail(call, SPM_ERR_INVALID_ARG, "out is in the place of q, which is read until the end");
    if (static_cast<long long>(batch->n_rows) * n_heads > INT32_MAX - 64) return fail(call, SPM_ERR_INVALID_ARG, "n_rows * n_heads is over 2^31 - 65");
    const int cols = columns_of(batch, n_heads, dtype);
    const size_t need = attend_bytes(cols, kv->latent_dim);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
        return fail(call, SPM_ERR_INVALID_ARG, "workspace must be 16-byte aligned and hold " + std::to_string(need) + " bytes");
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return fail(call, SPM_ERR_CUDA, cudaGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(call, SPM_ERR_CONFIG, "device ordinal out of range");
    LatentAttendArgs a{};
    a.kv = pool_of(kv);
    a.batch = batch_of(batch);
    a.q = rows_of(q); a.out = rows_of(out);
    a.heads = n_heads;
    int bits = 0;                                // x / d = x * ceil(2^(31 + bits) / d) >> (31 + bits), 2^bits >= d, for x below 2^31
    while (1 << bits < n_heads) ++bits;
    a.heads_shift = 31 + bits;
    a.heads_times = uint32_t(((1ull << a.heads_shift) + n_heads - 1) / n_heads);
    a.chunks = kv->latent_dim / 64 + 1;
    a.factor = factor;
    a.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    a.withhold = g_withhold.load(std::memory_order_relaxed);
    a.joins = static_cast<int4*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kLaJoinBytes);
    const auto st = static_cast<cudaStream_t>(stream);
    if (dtype == SPM_DTYPE_FP32) e = launch_attend<float, 16>(a, dev, sms, st);
    else if (cols == 16) e = launch_attend<__nv_bfloat16, 16>(a, dev, sms, st);
    else if (cols == 32) e = launch_attend<__nv_bfloat16, 32>(a, dev, sms, st);
    else if (cols == 48) e = launch_attend<__nv_bfloat16, 48>(a, dev, sms, st);
    else e = launch_attend<__nv_bfloat16, 64>(a, dev, sms, st);
    return launched(call, e);
}

int spm_latent_attend_expanded_workspace(const spm_latent_cache* kv, const spm_kv_batch* batch, int n_heads, int head_dim, int n_tokens, int dtype,
                                         size_t* bytes) {
    const char* call = "spm_latent_attend_expanded_workspace";
    if (!bytes) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (int rc = check_latent_shape(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (int rc = check_expanded(call, batch, n_heads, head_dim, n_tokens, dtype)) return rc;
    *bytes = expanded_of(batch, n_heads, head_dim, n_tokens).bytes;
    return SPM_OK;
}

int spm_latent_attend_expanded(const spm_latent_cache* kv, const spm_kv_batch* batch, const spm_rows* q, const spm_matrices* w_k, const spm_matrices* w_v,
                               int n_heads, int head_dim, const spm_rows* out, float scale, int n_tokens, int dtype, void* workspace, size_t workspace_bytes,
                               void* stream) {
    const char* call = "spm_latent_attend_expanded";
    if (int rc = check_latent_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (int rc = check_expanded(call, batch, n_heads, head_dim, n_tokens, dtype)) return rc;
    const float factor = scale * 1.4426950408889634f;
    if (!std::isfinite(factor)) return fail(call, SPM_ERR_INVALID_ARG, "scale is not finite, or not below 2^127");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    if (int rc = check_rows(call, "q", q, dtype)) return rc;
    if (int rc = check_rows(call, "out", out, dtype)) return rc;
    if (q->p == out->p) return fail(call, SPM_ERR_INVALID_ARG, "out is in the place of q, which is read until the end");
    if (int rc = check_matrices(call, "w_k", w_k, kv->latent_dim)) return rc;
    if (int rc = check_matrices(call, "w_v", w_v, kv->latent_dim)) return rc;
    const Expanded e = expanded_of(batch, n_heads, head_dim, n_tokens);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < e.bytes)
        return fail(call, SPM_ERR_INVALID_ARG, "workspace must be 256-byte aligned and hold " + std::to_string(e.bytes) + " bytes");
    int dev = 0, sms = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (err != cudaSuccess) return fail(call, SPM_ERR_CUDA, cudaGetErrorString(err));
    if (dev < 0 || dev >= kMaxDevices) return fail(call, SPM_ERR_CONFIG, "device ordinal out of range");
    char* work = static_cast<char*>(workspace);
    LatentExpandArgs x{};
    x.kv = pool_of(kv);
    x.batch = batch_of(batch);
    x.box = kv->page_size % 128 == 0 ? 128 : kv->page_size % 64 == 0 ? 64 : kv->page_size % 32 == 0 ? 32 : 16;
    x.tokens = e.tokens;
    x.keys = reinterpret_cast<__half*>(work);
    x.values = reinterpret_cast<__half*>(work + e.values);
    x.own = reinterpret_cast<__half*>(work + e.own);
    x.shared = reinterpret_cast<__half*>(work + e.shared);
    x.key_exps = reinterpret_cast<short*>(work + e.key_exps);
    x.value_exps = reinterpret_cast<short*>(work + e.value_exps);
    x.there = reinterpret_cast<uint32_t*>(work + e.there);
    x.items = reinterpret_cast<LxItem*>(work + e.items);
    x.n_items = e.n_items;
    x.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    x.withhold = g_withhold.load(std::memory_order_relaxed);
    LatentPromptArgs a{};
    a.kv = x.kv;
    a.batch = x.batch;
    a.q = rows_of(q); a.out = rows_of(out);
    a.tokens = e.tokens;
    a.shared_row = e.heads * e.tokens;
    a.there = x.there;
    a.items = x.items;
    a.key_exps = x.key_exps;
    a.value_exps = x.value_exps;
    a.factor = factor;
    a.wait_ns = x.wait_ns;
    a.withhold = x.withhold;
    CUtensorMap rows{}, wk, wv, keys, ropes, ropes32, values;         // (a pool without pages: no copy is made of it)
    const uint64_t made = uint64_t(e.heads) * e.tokens;
    if ((kv->n_pages > 0 && !make_token_map(&rows, kv->rows, kv->latent_dim + kv->rope_dim, uint64_t(kv->n_pages) * kv->page_size, x.box)) ||
        !make_matrix_map(&wk, w_k->p, kv->latent_dim, head_dim, n_heads, w_k->row_stride, w_k->head_stride) ||
        !make_matrix_map(&wv, w_v->p, kv->latent_dim, head_dim, n_heads, w_v->row_stride, w_v->head_stride) ||
        !make_token_map(&keys, x.keys, head_dim, made, kLpTile) || !make_token_map(&values, x.values, head_dim, made, kLpTile) ||
        !make_token_map(&ropes, x.own, 64, made + e.tokens, kLpTile) || !make_token_map(&ropes32, x.own, 64, made + e.tokens, 32))
        return fail(call, SPM_ERR_CUDA, "no tensor map of the cache's rows, the matrices or the workspace");
    const auto st = static_cast<cudaStream_t>(stream);
    return launched(call, head_dim == 64 ? launch_expanded<64>(x, a, e, n_heads, rows, wk, wv, keys, ropes, ropes32, values, dev, sms, st)
                                         : launch_expanded<128>(x, a, e, n_heads, rows, wk, wv, keys, ropes, ropes32, values, dev, sms, st));
}

int spm_head_product(const spm_rows* x, const void* w, int64_t w_head_stride, int64_t w_row_stride, int transposed, const spm_rows* y, int n_rows,
                     int n_heads, int in_dim, int out_dim, int dtype, void* stream) {
    const char* call = "spm_head_product";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_heads(call, n_heads)) return rc;
    if (in_dim < 64 || in_dim > 8192 || in_dim % 64 || out_dim < 64 || out_dim > 8192 || out_dim % 64)
        return fail(call, SPM_ERR_CONFIG, "in_dim and out_dim are multiples of 64 up to 8192");
    if (n_rows < 0) return fail(call, SPM_ERR_INVALID_ARG, "a negative size");
    if (n_rows > INT32_MAX / 128 - 32) return fail(call, SPM_ERR_INVALID_ARG, "too many rows");          // (tiles of rows times tiles of outputs are a number)
    if (n_rows == 0) return SPM_OK;
    if (int rc = check_rows(call, "x", x, dtype)) return rc;
    if (int rc = check_rows(call, "y", y, dtype)) return rc;
    if (x->p == y->p) return fail(call, SPM_ERR_INVALID_ARG, "y is in the place of x, which is read until the end");
    if (!w || !aligned(w, 16) || w_head_stride % 8 || w_row_stride % 8)
        return fail(call, SPM_ERR_INVALID_ARG, "w: rows of weights must start on 16-byte boundaries");
    HeadProductArgs a{};
    a.x = rows_of(x); a.y = rows_of(y);
    a.w = static_cast<const __nv_bfloat16*>(w);
    a.w_head = w_head_stride; a.w_row = w_row_stride;
    a.n_rows = n_rows; a.in = in_dim;
    const auto st = static_cast<cudaStream_t>(stream);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail(call, SPM_ERR_CUDA, cudaGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(call, SPM_ERR_CONFIG, "device ordinal out of range");
    if (dtype == SPM_DTYPE_BF16)
        e = transposed ? launch_product<__nv_bfloat16, true>(a, n_heads, out_dim, dev, st) : launch_product<__nv_bfloat16, false>(a, n_heads, out_dim, dev, st);
    else e = transposed ? launch_product<float, true>(a, n_heads, out_dim, dev, st) : launch_product<float, false>(a, n_heads, out_dim, dev, st);
    return launched(call, e);
}

}  // extern "C"
