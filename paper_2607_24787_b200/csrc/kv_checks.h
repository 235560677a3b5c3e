// Checks of arguments and conversions that the attention block's entry points share.
#pragma once

#include <atomic>
#include <cstdint>
#include <string>

#include <cuda_runtime.h>

#include "kv_cache.cuh"
#include "kv_write.cuh"

namespace spm {

void set_thread_error(const std::string& msg);   // defined next to spm_last_error

inline int fail(const char* call, int code, const std::string& msg) {
    set_thread_error(std::string(call) + ": " + msg);
    return code;
}
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline int check_dtype(const char* call, int dtype) {
    return dtype == SPM_DTYPE_FP32 || dtype == SPM_DTYPE_BF16 ? SPM_OK : fail(call, SPM_ERR_CONFIG, "rows are fp32 or bf16");
}
inline int check_batch(const char* call, int page_size, const spm_kv_batch* b) {
    if (!b) return fail(call, SPM_ERR_INVALID_ARG, "null argument");
    if (b->n_seq < 0 || b->n_seq > SPM_KV_MAX_SEQS)
        return fail(call, SPM_ERR_INVALID_ARG, "n_seq " + std::to_string(b->n_seq) + " outside 0.." + std::to_string(SPM_KV_MAX_SEQS));
    if (b->n_rows < 0 || b->max_rows < 0 || b->table_stride < 0) return fail(call, SPM_ERR_INVALID_ARG, "a negative size");
    // (a tile's tokens more than a sequence's are still a number)
    if (static_cast<long long>(b->table_stride) * page_size > INT32_MAX - 4095ll)
        return fail(call, SPM_ERR_INVALID_ARG, "table_stride * page_size is over 2^31 - 4096 tokens");
    if (b->n_seq > 0 && (!b->lengths || (!b->page_table && b->table_stride > 0)))
        return fail(call, SPM_ERR_INVALID_ARG, "page_table or lengths is null");
    if (!aligned(b->page_table, 4) || !aligned(b->lengths, 4) || !aligned(b->row_start, 4))
        return fail(call, SPM_ERR_INVALID_ARG, "page_table, lengths and row_start must be 4-byte aligned");
    if (!b->row_start && b->n_rows < b->n_seq) return fail(call, SPM_ERR_INVALID_ARG, "fewer rows than sequences, and no row_start");
    return SPM_OK;
}
inline int check_rows(const char* call, const char* name, const spm_rows* r, int dtype) {
    const long long e = dtype == SPM_DTYPE_BF16 ? 2 : 4;
    if (!r || !r->p) return fail(call, SPM_ERR_INVALID_ARG, std::string(name) + " is null");
    if (!aligned(r->p, 16) || r->row_stride * e % 16 || r->head_stride * e % 16)
        return fail(call, SPM_ERR_INVALID_ARG, std::string(name) + ": rows of heads must start on 16-byte boundaries");
    return SPM_OK;
}
inline bool other_strides(const spm_rows* x, const spm_rows* y) { return x->row_stride != y->row_stride || x->head_stride != y->head_stride; }
inline int check_rope(const char* call, const spm_rope* r, const int32_t* positions, int64_t pos_stride, int n_rows, int hd) {
    if (!r) return fail(call, SPM_ERR_INVALID_ARG, "rope is null");
    if (r->rot_dim < 0 || r->rot_dim > hd || r->rot_dim % 16)
        return fail(call, SPM_ERR_CONFIG, "rot_dim " + std::to_string(r->rot_dim) + " is not a multiple of 16 up to head_dim");
    if (r->n_axes < 1 || r->n_axes > SPM_KV_MAX_AXES) return fail(call, SPM_ERR_INVALID_ARG, "n_axes outside 1.." + std::to_string(SPM_KV_MAX_AXES));
    if (r->rot_dim > 0 && (!r->inv_freq || !positions)) return fail(call, SPM_ERR_INVALID_ARG, "inv_freq or positions is null");
    if (r->rot_dim > 0 && r->n_axes > 1 && pos_stride < n_rows) return fail(call, SPM_ERR_INVALID_ARG, "pos_stride is less than the rows");
    if (!aligned(r->inv_freq, 4) || !aligned(positions, 4) || !aligned(r->q_gamma, 16) || !aligned(r->k_gamma, 16))
        return fail(call, SPM_ERR_INVALID_ARG, "gammas must be 16-byte aligned, inv_freq and positions 4-byte aligned");
    return SPM_OK;
}

inline KvBatch batch_of(const spm_kv_batch* b) { return {b->page_table, b->lengths, b->row_start, b->n_seq, b->table_stride, b->n_rows}; }
inline HeadRows rows_of(const spm_rows* r) { return {r->p, r->row_stride, r->head_stride}; }
inline RopeArgs rope_of(const spm_rope* r, const int32_t* positions, int64_t pos_stride) {
    return {r->inv_freq, r->axis_of, r->q_gamma, r->k_gamma, positions, pos_stride, r->n_axes, r->rot_dim, r->neighbours, r->eps};
}

inline int launched(const char* call, cudaError_t e) {
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess ? SPM_OK : fail(call, SPM_ERR_CUDA, std::string("launch: ") + cudaGetErrorString(e));
}

// What spm_test_kv_waits sets: the limit of a kernel's waits, arrivals that barriers wait for and nobody makes
inline std::atomic<unsigned long long> g_wait_ns{2'000'000'000ull};
inline std::atomic<int> g_withhold{0};

constexpr int kMaxDevices = 64;
// Once a kernel and device: shared memory beyond 48 KB
template <auto KERNEL>
cudaError_t allow_smem(int dev, int bytes) {
    static std::atomic<bool> done[kMaxDevices];
    if (done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done[dev].store(true, std::memory_order_release);
    return e;
}

}  // namespace spm
