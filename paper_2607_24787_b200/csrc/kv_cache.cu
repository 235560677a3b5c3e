// The entry points of the attention block: checks of arguments, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include <cuda_runtime.h>

#include "kv_attend.cuh"
#include "kv_checks.h"
#include "kv_prefill.cuh"
#include "kv_write.cuh"

using namespace spm;

namespace {

int check_head_dim(const char* call, int hd) {
    if (hd == 64 || hd == 128 || hd == 256) return SPM_OK;
    return fail(call, SPM_ERR_CONFIG, "head_dim " + std::to_string(hd) + " not supported: 64, 128 or 256");
}
int check_cache_shape(const char* call, const spm_kv_cache* kv) {
    if (!kv) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (int rc = check_head_dim(call, kv->head_dim)) return rc;
    if (kv->page_size < kKvBlock || kv->page_size % kKvBlock || kv->page_size > 65536)
        return fail(call, SPM_ERR_CONFIG, "page_size " + std::to_string(kv->page_size) + " is not a multiple of 16 up to 65536");
    if (kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return fail(call, SPM_ERR_CONFIG, "n_kv_heads outside 1..1024");
    if (kv->n_pages < 0) return fail(call, SPM_ERR_INVALID_ARG, "n_pages is negative");
    return SPM_OK;
}
int check_cache(const char* call, const spm_kv_cache* kv) {
    if (int rc = check_cache_shape(call, kv)) return rc;
    if (!kv->pages && kv->n_pages > 0) return fail(call, SPM_ERR_INVALID_ARG, "pages is null");
    if (!aligned(kv->pages, 16) || !aligned(kv->status, 4))
        return fail(call, SPM_ERR_INVALID_ARG, "pages must be 16-byte aligned, status 4-byte aligned");
    return SPM_OK;
}
KvPool pool_of(const spm_kv_cache* kv) { return {static_cast<unsigned char*>(kv->pages), kv->status, kv->n_pages, kv->page_size, kv->n_kv_heads}; }

// calls f with a null pointer of the row type and the head size as a constant
template <typename F>
void by_type(int dtype, int hd, F f) {
    auto size = [&](auto* t) {
        if (hd == 64) f(t, std::integral_constant<int, 64>{});
        else if (hd == 128) f(t, std::integral_constant<int, 128>{});
        else f(t, std::integral_constant<int, 256>{});
    };
    if (dtype == SPM_DTYPE_BF16) size(static_cast<__nv_bfloat16*>(nullptr));
    else size(static_cast<float*>(nullptr));
}

int launch_write(const char* call, const WriteArgs& a, int hd, int dtype, cudaStream_t st) {
    const int heads = 2 * a.kv_heads + a.q_heads;
    if (a.n_rows == 0 || heads == 0) return SPM_OK;
    // a row a warp, or where these are few a row's turns shared out, up to a turn a warp
    const int at_once = 256 / hd, turns = 2 * ((a.kv_heads + at_once - 1) / at_once) + (a.q_heads + at_once - 1) / at_once;
    constexpr int kWarps = 592 * kKvWarps;       // that the GPU has room for
    const int parts = std::max(1, std::min(turns, kWarps / a.n_rows));
    const unsigned grid = unsigned((static_cast<long long>(a.n_rows) * parts + kKvWarps - 1) / kKvWarps);
    cudaError_t e = cudaSuccess;
    by_type(dtype, hd, [&](auto* t, auto size) {
        e = launch_early(kv_write_kernel<std::remove_pointer_t<decltype(t)>, size.value>, grid, kKvWarps * 32, 0, st, a, parts);
    });
    return launched(call, e);
}

// joins, the rows that each of two kernels takes, parts
constexpr size_t kAtJoinBytes = kAtMaxCtas * 32, kAtRowsBytes = 2 * SPM_KV_MAX_SEQS * sizeof(int);
size_t attend_bytes(int hd) { return kAtJoinBytes + kAtRowsBytes + kAtMaxCtas * 2 * size_t(8) * (hd + 2) * 4; }

template <typename T, int HD>
cudaError_t launch_attend(const AttendArgs& a, int dev, int sms, cudaStream_t st) {
    using S = AtShape<T, HD>;
    cudaError_t e = allow_smem<kv_attend_kernel<T, HD>>(dev, S::smem(SPM_KV_MAX_SEQS));
    if (e != cudaSuccess) return e;
    const int ctas = std::min(sms, kAtMaxCtas);
    e = launch_early(kv_attend_kernel<T, HD>, ctas, S::warps * 32, S::smem(a.batch.n_seq), st, a);
    return e == cudaSuccess ? launch_early(kv_attend_join_kernel<T, HD>, dim3(ctas, S::cols), kAtJoinThreads, 0, st, a) : e;
}

// Which of the two kernels a call's rows are for. Per token of context the tensor-core kernel takes 19 ns a round of CTAs (an SM does 256
// columns of a head, and an item's tokens are not shared out), the other 4.5 ps a column of a head on all SMs together, whatever the rows
// are; lengths cancel where sequences are alike, and long ones of few rows are taken out (kv_split_kernel). Measured with 4 heads of 128 over
// 4096 tokens, columns times heads (tensor cores / other, us): 3200: 80 / 64, 4096: 79 / 79, 8192: 79 / 140, 37888: 87 / 594; in two rounds,
// 10240: 159 / 177.
constexpr int kPfColumns = 4000;                 // a round
bool prefill_pays(const spm_kv_cache* kv, const spm_kv_batch* b, int n_q_heads, int dtype) {
    if (dtype != SPM_DTYPE_BF16 || kv->head_dim > 128 || !b->row_start) return false;
    const long long columns = static_cast<long long>(b->n_rows) * (n_q_heads / kv->n_kv_heads), each = (columns + b->n_seq - 1) / b->n_seq;
    const long long items = (each + kPfCols - 1) / kPfCols * b->n_seq * kv->n_kv_heads;
    return columns * kv->n_kv_heads > kPfColumns * ((items + kAtMaxCtas - 1) / kAtMaxCtas);
}
template <int HD>
cudaError_t launch_prefill(AttendArgs a, void* workspace, int dev, int sms, cudaStream_t st) {
    cudaError_t e = allow_smem<kv_prefill_kernel<HD>>(dev, PfShape<HD>::smem);
    if (e != cudaSuccess) return e;
    if (a.batch.n_seq > 1 && a.batch.stride * a.kv.page_size > kPfLongTokens) {       // there may be sequences that are not for it
        int* rows = reinterpret_cast<int*>(static_cast<char*>(workspace) + kAtJoinBytes);
        e = launch_early(kv_split_kernel, 1, SPM_KV_MAX_SEQS, 0, st, a, kPfColumns, rows, rows + SPM_KV_MAX_SEQS);
        a.rows = rows;
        if (e == cudaSuccess) e = launch_attend<__nv_bfloat16, HD>(a, dev, sms, st);
        if (e != cudaSuccess) return e;
        a.rows = rows + SPM_KV_MAX_SEQS;
    }
    // as many CTAs as there can be items: full ones of all rows, and one a sequence that is not full
    const long long items = (static_cast<long long>(a.batch.n_rows) * a.group / kPfCols + a.batch.n_seq) * a.kv.heads;
    if (items > INT32_MAX) return cudaErrorInvalidValue;
    return launch_early(kv_prefill_kernel<HD>, unsigned(items), kPfThreads, PfShape<HD>::smem, st, a);
}

}  // namespace

extern "C" {

int spm_kv_cache_bytes(const spm_kv_cache* kv, size_t* bytes) {
    if (!bytes) return fail("spm_kv_cache_bytes", SPM_ERR_INVALID_ARG, "null argument");
    if (int rc = check_cache_shape("spm_kv_cache_bytes", kv)) return rc;
    *bytes = size_t(kv->n_pages) * kv->n_kv_heads * (kv->page_size / kKvBlock) * kv_block_bytes(kv->head_dim);
    return SPM_OK;
}

int spm_rotate_heads(const spm_rope* rope, const int32_t* positions, int64_t pos_stride, const spm_rows* x, const spm_rows* y,
                     int n_rows, int n_heads, int head_dim, int dtype, void* stream) {
    const char* call = "spm_rotate_heads";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_head_dim(call, head_dim)) return rc;
    if (n_rows < 0 || n_heads < 0) return fail(call, SPM_ERR_INVALID_ARG, "a negative size");
    if (n_rows == 0 || n_heads == 0) return SPM_OK;
    if (int rc = check_rope(call, rope, positions, pos_stride, n_rows, head_dim)) return rc;
    if (int rc = check_rows(call, "x", x, dtype)) return rc;
    if (int rc = check_rows(call, "y", y, dtype)) return rc;
    if (x->p == y->p && other_strides(x, y)) return fail(call, SPM_ERR_INVALID_ARG, "y in x's place has other strides");
    WriteArgs a{};
    a.kv.page_size = kKvBlock;
    a.batch.n_seq = -1;
    a.rope = rope_of(rope, positions, pos_stride);
    a.q = rows_of(x); a.q_out = rows_of(y);
    a.q_heads = n_heads; a.n_rows = n_rows;
    return launch_write(call, a, head_dim, dtype, static_cast<cudaStream_t>(stream));
}

int spm_kv_write(const spm_kv_cache* kv, const spm_kv_batch* batch, const spm_rope* rope, const int32_t* positions, int64_t pos_stride,
                 const spm_rows* q, const spm_rows* q_out, int n_q_heads, const spm_rows* k, const spm_rows* v, int dtype, void* stream) {
    const char* call = "spm_kv_write";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (n_q_heads < 0) return fail(call, SPM_ERR_INVALID_ARG, "a negative size");
    if (q && !rope) return fail(call, SPM_ERR_INVALID_ARG, "q without rope: there is nothing to do to it");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    if (rope)
        if (int rc = check_rope(call, rope, positions, pos_stride, batch->n_rows, kv->head_dim)) return rc;
    if (int rc = check_rows(call, "k", k, dtype)) return rc;
    if (int rc = check_rows(call, "v", v, dtype)) return rc;
    if (q) {
        if (int rc = check_rows(call, "q", q, dtype)) return rc;
        if (int rc = check_rows(call, "q_out", q_out, dtype)) return rc;
        if (q->p == q_out->p && other_strides(q, q_out)) return fail(call, SPM_ERR_INVALID_ARG, "q_out in q's place has other strides");
    }
    WriteArgs a{};
    a.kv = pool_of(kv);
    a.batch = batch_of(batch);
    if (rope) a.rope = rope_of(rope, positions, pos_stride);
    if (q) { a.q = rows_of(q); a.q_out = rows_of(q_out); a.q_heads = n_q_heads; }
    a.k = rows_of(k); a.v = rows_of(v);
    a.kv_heads = kv->n_kv_heads; a.n_rows = batch->n_rows;
    return launch_write(call, a, kv->head_dim, dtype, static_cast<cudaStream_t>(stream));
}

int spm_kv_read(const spm_kv_cache* kv, const spm_kv_batch* batch, const spm_rows* k_out, const spm_rows* v_out, int dtype, void* stream) {
    const char* call = "spm_kv_read";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (!k_out && !v_out) return fail(call, SPM_ERR_INVALID_ARG, "neither k_out nor v_out");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    ReadArgs a{};
    a.kv = pool_of(kv);
    a.batch = batch_of(batch);
    if (k_out) { if (int rc = check_rows(call, "k_out", k_out, dtype)) return rc; a.k = rows_of(k_out); }
    if (v_out) { if (int rc = check_rows(call, "v_out", v_out, dtype)) return rc; a.v = rows_of(v_out); }
    const int each = kKvWarps * 32 / (kv->head_dim / 8);
    const unsigned grid = unsigned((static_cast<long long>(batch->n_rows) + each - 1) / each);
    cudaError_t e = cudaSuccess;
    by_type(dtype, kv->head_dim, [&](auto* t, auto size) {
        e = launch_early(kv_read_kernel<std::remove_pointer_t<decltype(t)>, size.value>, grid, kKvWarps * 32, 0, static_cast<cudaStream_t>(stream), a);
    });
    return launched(call, e);
}

int spm_kv_attend_workspace(const spm_kv_cache* kv, const spm_kv_batch* batch, int n_q_heads, int dtype, size_t* bytes) {
    const char* call = "spm_kv_attend_workspace";
    if (!bytes) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_cache_shape(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return fail(call, SPM_ERR_CONFIG, "n_q_heads is not a multiple of n_kv_heads");
    *bytes = attend_bytes(kv->head_dim);
    return SPM_OK;
}

int spm_kv_attend(const spm_kv_cache* kv, const spm_kv_batch* batch, const spm_rows* q, int n_q_heads, const spm_rows* out, float scale,
                  int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const char* call = "spm_kv_attend";
    if (int rc = check_dtype(call, dtype)) return rc;
    if (int rc = check_cache(call, kv)) return rc;
    if (int rc = check_batch(call, kv->page_size, batch)) return rc;
    if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return fail(call, SPM_ERR_CONFIG, "n_q_heads is not a multiple of n_kv_heads");
    if (!std::isfinite(scale)) return fail(call, SPM_ERR_INVALID_ARG, "scale is not finite");
    if (batch->n_rows == 0 || batch->n_seq == 0) return SPM_OK;
    if (int rc = check_rows(call, "q", q, dtype)) return rc;
    if (int rc = check_rows(call, "out", out, dtype)) return rc;
    if (q->p == out->p) return fail(call, SPM_ERR_INVALID_ARG, "out is in the place of q, which is read until the end");
    if (static_cast<long long>(batch->n_rows) * n_q_heads > INT32_MAX) return fail(call, SPM_ERR_INVALID_ARG, "n_rows * n_q_heads is over 2^31 - 1");
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < attend_bytes(kv->head_dim))
        return fail(call, SPM_ERR_INVALID_ARG, "workspace must be 16-byte aligned and hold " + std::to_string(attend_bytes(kv->head_dim)) + " bytes");
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return fail(call, SPM_ERR_CUDA, cudaGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(call, SPM_ERR_CONFIG, "device ordinal out of range");
    AttendArgs a{};
    a.kv = pool_of(kv);
    a.batch = batch_of(batch);
    a.q = rows_of(q); a.out = rows_of(out);
    a.group = n_q_heads / kv->n_kv_heads;
    const int per_page = kv->page_size / kKvBlock;
    a.page_shift = a.group_shift = -1;
    for (int i = 0; i < 16; ++i) {
        if (per_page == 1 << i) a.page_shift = i;
        if (a.group == 1 << i) a.group_shift = i;
    }
    // one block of columns a sequence (a guess where max_rows is one: it only says what to keep in L2)
    a.once = (batch->row_start ? std::max(batch->max_rows, 1) : 1ll) * a.group <= 8;
    a.scale = scale;
    a.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    a.withhold = g_withhold.load(std::memory_order_relaxed);
    a.joins = static_cast<int*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kAtJoinBytes + kAtRowsBytes);
    if (prefill_pays(kv, batch, n_q_heads, dtype))
        e = (kv->head_dim == 64 ? launch_prefill<64> : launch_prefill<128>)(a, workspace, dev, sms, static_cast<cudaStream_t>(stream));
    else by_type(dtype, kv->head_dim, [&](auto* t, auto size) {
        using T = std::remove_pointer_t<decltype(t)>;
        e = launch_attend<T, size.value>(a, dev, sms, static_cast<cudaStream_t>(stream));
    });
    return launched(call, e);
}

int spm_test_kv_waits(int withhold, int limit_us) {
    // (copies that a kernel gives up on have to land within the limit again before it ends)
    if (limit_us != 0 && limit_us < 1000) return fail("spm_test_kv_waits", SPM_ERR_INVALID_ARG, "limit_us is less than a millisecond");
    g_withhold.store(withhold != 0, std::memory_order_relaxed);
    g_wait_ns.store(limit_us ? static_cast<unsigned long long>(limit_us) * 1000ull : 2'000'000'000ull, std::memory_order_relaxed);
    return SPM_OK;
}

}  // extern "C"
