// Attention of new rows over the 4-bit cache.
#pragma once

#include "kv_write.cuh"
#include "ptx.cuh"

namespace spm {

struct AttendArgs {
    KvPool kv;
    KvBatch batch;
    HeadRows q, out;
    int q_heads;
    float scale;
};

// A block takes a row and a head, a warp every eighth token: softmax by its running maximum and sum
template <typename T, int HD>
__global__ void __launch_bounds__(kKvWarps * 32) kv_attend_kernel(const AttendArgs a) {
    constexpr int E = HD / 32;
    __shared__ float part[kKvWarps][HD + 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x, head = blockIdx.y;
    const RowAt r = kv_row_at(a.batch, row);
    if (r.seq >= a.batch.n_seq) return;
    const int kv_head = head / (a.q_heads / a.kv.heads);
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    load_row<E>(static_cast<const T*>(a.q.p) + row * a.q.row + head * a.q.head + lane * E, q);
    const int g = lane * E / 32, in = lane * E % 32;
    const long long cap = static_cast<long long>(a.batch.stride) * a.kv.page_size;
    if (r.pos >= cap && threadIdx.x == 0) kv_note(a.kv, SPM_KV_TOO_LONG);
    const int n = int(min(static_cast<long long>(r.pos) + 1, cap));
    for (int t = warp; t < n; t += kKvWarps) {
        const long long block = kv_block_at<HD>(a.kv, a.batch, r.seq, t, kv_head);
        if (block < 0) { if (lane == 0) kv_note(a.kv, SPM_KV_BAD_PAGE); continue; }
        const unsigned char* at = a.kv.pages + block;
        const int tok = t % kKvBlock;
        float x[2][E];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const unsigned char* c = at + p * kv_v_codes(HD) + (g * kKvBlock + tok) * 16 + in / 2;
            const float d = __half2float(*reinterpret_cast<const __half*>(at + kv_k_scales(HD) + p * HD + (tok * (HD / 32) + g) * 2));
#pragma unroll
            for (int e = 0; e < E; ++e) x[p][e] = (float(c[e / 2] >> (4 * (e % 2)) & 15) - 8.f) * d;
        }
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += q[e] * x[0][e];
        s = warp_sum(s) * a.scale;
        const float top = fmaxf(m, s), keep = __expf(m - top), p = __expf(s - top);
        l = l * keep + p;
        m = top;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * keep + p * x[1][e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) part[warp][lane * E + e] = o[e];
    if (lane == 0) { part[warp][HD] = m; part[warp][HD + 1] = l; }
    __syncthreads();
    for (int d = threadIdx.x * 8; d < HD; d += blockDim.x * 8) {
        float top = -INFINITY, sum = 0.f, y[8] = {};
        for (int w = 0; w < kKvWarps; ++w) top = fmaxf(top, part[w][HD]);
        if (top > -INFINITY)
            for (int w = 0; w < kKvWarps; ++w) {
                const float f = __expf(part[w][HD] - top);
                sum += part[w][HD + 1] * f;
                for (int e = 0; e < 8; ++e) y[e] += part[w][d + e] * f;
            }
        for (int e = 0; e < 8; ++e) y[e] = sum > 0.f ? y[e] / sum : 0.f;
        store_row<8>(static_cast<T*>(a.out.p) + row * a.out.row + head * a.out.head + d, y);
    }
}

}  // namespace spm
