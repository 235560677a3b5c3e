// The cache of latent rows: where a token's row is.
#pragma once

#include "kv_cache.cuh"
#include "mma_ops.cuh"

namespace spm {

struct LatentPool {
    __nv_bfloat16* rows;       // [n_pages][page_size][latent + rope]
    int* status;
    int n_pages, page_size, latent, rope;
};
__device__ __forceinline__ void kv_note(const LatentPool& kv, int bit) {
    if (kv.status) atomicOr(kv.status, bit);
}
// The row of token `pos` of a sequence, counted in the pool; -1: there is none, and the status says why
__device__ __forceinline__ long long latent_row_at(const LatentPool& kv, const KvBatch& b, int seq, int pos, bool note) {
    const int slot = pos / kv.page_size;
    const int page = slot < b.stride ? b.table[size_t(seq) * b.stride + slot] : -1;
    if (page >= 0 && page < kv.n_pages) return static_cast<long long>(page) * kv.page_size + (pos - slot * kv.page_size);
    if (note) kv_note(kv, slot >= b.stride ? SPM_KV_TOO_LONG : SPM_KV_BAD_PAGE);
    return -1;
}

// bf16 parts of two numbers: cut off, so that the sum is exact (an infinity's are itself and zeros, a NaN's first is one whatever its bits)
__device__ __forceinline__ void cut_parts(float a, float b, uint32_t (&p)[3]) {
    const Split3 s = split3(a + 0.f, b + 0.f);
#pragma unroll
    for (int i = 0; i < 3; ++i) p[i] = s.part[i];
}
__device__ __forceinline__ void cut_parts(uint32_t v, uint32_t (&p)[1]) { p[0] = v; }

}  // namespace spm
