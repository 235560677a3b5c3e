// The 4-bit key/value cache: where a token's bytes are, and which token a row of a batch is.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/spm.h"

namespace spm {

constexpr int kKvBlock = 16;           // tokens of a block: the rows of one mma tile
__host__ __device__ constexpr int kv_block_bytes(int hd) { return 18 * hd; }
__host__ __device__ constexpr int kv_v_codes(int hd) { return 8 * hd; }        // offsets in a block; key codes are at 0
__host__ __device__ constexpr int kv_k_scales(int hd) { return 16 * hd; }
__host__ __device__ constexpr int kv_v_scales(int hd) { return 17 * hd; }

struct KvPool {
    unsigned char* pages;
    int* status;
    int n_pages, page_size, heads;
};
struct KvBatch {
    const int* table;
    const int* lengths;
    const int* row_start;
    int n_seq, stride, n_rows;
};
struct HeadRows { void* p; long long row, head; };

__device__ __forceinline__ void kv_note(const KvPool& kv, int bit) {
    if (kv.status) atomicOr(kv.status, bit);
}

// Byte offset of the block that holds token `pos` of `head`, -1 where there is none
template <int HD>
__device__ __forceinline__ long long kv_block_at(const KvPool& kv, const KvBatch& b, int seq, int pos, int head) {
    const int slot = pos / kv.page_size;
    if (slot >= b.stride) return -1;
    const int page = b.table[size_t(seq) * b.stride + slot];
    if (page < 0 || page >= kv.n_pages) return -1;
    const int blocks = kv.page_size / kKvBlock;
    return ((static_cast<long long>(page) * kv.heads + head) * blocks + (pos - slot * kv.page_size) / kKvBlock) * kv_block_bytes(HD);
}

// Sequence of a row, by a warp together (n_seq: no sequence's), and the row's position there
struct RowAt { int seq, pos, len; };
__device__ __forceinline__ RowAt kv_row_at(const KvBatch& b, int row) {
    const int lane = threadIdx.x & 31;
    RowAt r{row, 0, 0};
    int first = row, n = 1;
    if (b.row_start) {
        r.seq = 0;
        for (int i = 0; i < b.n_seq; i += 32) {
            const int ended = __popc(__ballot_sync(0xffffffffu, i + lane < b.n_seq && b.row_start[i + lane + 1] <= row));
            r.seq += ended;
            if (ended < 32) break;
        }
        if (r.seq < b.n_seq) {
            first = b.row_start[r.seq];
            n = b.row_start[r.seq + 1] - first;
        }
        if (row < first) r.seq = b.n_seq;
    }
    if (r.seq < b.n_seq) {
        r.len = b.lengths[r.seq];
        r.pos = r.len - n + (row - first);
    }
    return r;
}

// two fp32 numbers in one register pair
__device__ __forceinline__ unsigned long long two_words(uint32_t a, uint32_t b) {
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b));
    return v;
}
__device__ __forceinline__ unsigned long long two_floats(float a, float b) { return two_words(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ void floats_of(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}

// E consecutive elements in 32 bits
template <int E>
__device__ __forceinline__ void load_row(const float* p, float (&f)[E]) {
    if constexpr (E == 2) { const float2 v = *reinterpret_cast<const float2*>(p); f[0] = v.x; f[1] = v.y; }
    else
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + i);
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
}
__device__ __forceinline__ void two_bf16(uint32_t v, float& a, float& b) { a = __uint_as_float(v << 16); b = __uint_as_float(v & 0xffff0000u); }
template <int E>
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, float (&f)[E]) {
    if constexpr (E == 2) two_bf16(*reinterpret_cast<const uint32_t*>(p), f[0], f[1]);
    else if constexpr (E == 4) { const uint2 v = *reinterpret_cast<const uint2*>(p); two_bf16(v.x, f[0], f[1]); two_bf16(v.y, f[2], f[3]); }
    else {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        two_bf16(v.x, f[0], f[1]); two_bf16(v.y, f[2], f[3]); two_bf16(v.z, f[4], f[5]); two_bf16(v.w, f[6], f[7]);
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int E>
__device__ __forceinline__ void store_row(float* p, const float (&f)[E]) {
    if constexpr (E == 2) *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]);
    else
#pragma unroll
        for (int i = 0; i < E; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}
template <int E>
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&f)[E]) {
    if constexpr (E == 2) *reinterpret_cast<uint32_t*>(p) = pack_bf16(f[0], f[1]);
    else if constexpr (E == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    else *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// Launched so that its CTAs may be in place before the stream's kernel before it has ended: every kernel launched so waits for that
// one before it reads or writes anything but weights, and then lets its own successor do the same.
template <typename... A, typename... B>
cudaError_t launch_early(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t st, const B&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, A(args)...);
}

}  // namespace spm
