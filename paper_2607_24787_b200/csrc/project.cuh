// Projections of the attention block for the few rows of a decode step: y = W x, x fp32 rows (normed or not), up to 64 of them.
//
// Bound by reading W once. Each row x is normed and split by a block of its own first (three bf16 parts, so that activations stay fp32 as
// everywhere in a step), laid out as the B operand wants it; then a CTA takes 16 or 32 rows of W, its warps every eighth 32 columns, and
// their sums meet in shared memory in a fixed order.
// 5120 rows of 2048: 9.0 us for one row x (2.3 TB/s; launches, first words and the sums' joining are most of it), 37 for 64 rows, which read
// x's parts from L2 once a CTA; 2048 rows of 4096: 12.7 and 27. (Each kernel alone and from a cold cache.)
#pragma once

#include <cstdint>

#include "kv_cache.cuh"
#include "mma_ops.cuh"
#include "ptx.cuh"

namespace spm {

constexpr int kPrWarps = 8;

// Row blockIdx.x of x [rows][K]: times gamma / rms (gamma NULL: as it is). parts: [row block of 8][K / 32][3][32 lanes] of 16 bytes, lane 4 r + c
// holding elements 8 c .. 8 c + 7 of row r; or, plain != NULL, fp32 [rows][K].
__global__ void __launch_bounds__(256) project_rows_kernel(const float* x, int K, const float* gamma, float eps, uint4* parts, float* plain) {
    __shared__ float sums[8];
    const int row = blockIdx.x, tid = threadIdx.x;
    const float* from = x + static_cast<size_t>(row) * K;
    float by = 1.f;
    grid_dep_wait();
    grid_dep_launch();
    if (gamma) {
        float sum = 0.f;
        for (int i = tid * 4; i < K; i += 1024) {
            const float4 v = *reinterpret_cast<const float4*>(from + i);
            sum += v.x * v.x + v.y * v.y + v.z * v.z + v.w * v.w;
        }
        sum = warp_sum(sum);
        if ((tid & 31) == 0) sums[tid >> 5] = sum;
        __syncthreads();
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += sums[i];
        by = rsqrtf(sum / float(K) + eps);
    }
    for (int i = tid * 8; i < K; i += 2048) {
        float v[8];
        load_row<8>(from + i, v);
        if (gamma) {
            float g[8];
            load_row<8>(gamma + i, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] * by * g[e];
        }
        if (plain) {
            store_row<8>(plain + static_cast<size_t>(row) * K + i, v);
            continue;
        }
        const int kb = i / 32, lane = (row & 7) * 4 + i % 32 / 8;
        Split3 s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = split3(v[2 * j], v[2 * j + 1]);
        uint4* to = parts + ((static_cast<size_t>(row / 8) * (K / 32) + kb) * 3) * 32 + lane;
#pragma unroll
        for (int p = 0; p < 3; ++p) to[p * 32] = make_uint4(s[0].part[p], s[1].part[p], s[2].part[p], s[3].part[p]);
    }
}

// y[t * stride + n] (+)= sum over k of W[n][k] x[t][k]; N a multiple of 16 * MT, K of 32
// U: turns of W that a warp has in registers ahead of their use (0: with many rows there are no registers for that)
template <int NT, int MT, int U>
__global__ void __launch_bounds__(kPrWarps * 32, U == 4 ? 4 : 1) project_kernel(const __nv_bfloat16* W, const uint4* parts, int rows, int K, float* y,
                                                                                long long stride, int add) {
    __shared__ float red[kPrWarps / 2][MT * 16][8 * NT + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const int n0 = blockIdx.x * (16 * MT), KB = K / 32;
    const __nv_bfloat16* at = W + static_cast<size_t>(n0 + r) * K + 8 * c;
    float acc[NT][MT][4] = {};
    int from[NT];                                // columns behind the rows take the last row's numbers: they go nowhere
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = min(8 * nt + r, rows - 1);
        from[nt] = row / 8 * KB * 96 + row % 8 * 4 + c;
    }
    auto take = [&](int kb, const uint4 (&w)[MT][2]) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const uint4* b = parts + from[nt] + kb * 96;
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const uint4 x = b[p * 32];
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    mma_k16(acc[nt][m], w[m][0].x, w[m][1].x, w[m][0].y, w[m][1].y, x.x, x.y);
                    mma_k16(acc[nt][m], w[m][0].z, w[m][1].z, w[m][0].w, w[m][1].w, x.z, x.w);
                }
            }
        }
    };
    auto bring = [&](int kb, uint4 (&w)[MT][2]) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) w[m][e] = *reinterpret_cast<const uint4*>(at + static_cast<size_t>(16 * m + 8 * e) * K + kb * 32);
    };
    if constexpr (U > 0) {                       // U turns' words of W ahead; the first ones do not wait for the kernel before this one
        uint4 w[U][MT][2];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (warp + i * kPrWarps < KB) bring(warp + i * kPrWarps, w[i]);
        grid_dep_wait();
        grid_dep_launch();
        for (int kb0 = warp; kb0 < KB; kb0 += U * kPrWarps) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int kb = kb0 + i * kPrWarps;
                if (kb >= KB) break;
                take(kb, w[i]);
                if (kb + U * kPrWarps < KB) bring(kb + U * kPrWarps, w[i]);
            }
        }
    } else {
        grid_dep_wait();
        grid_dep_launch();
#pragma unroll 2
        for (int kb = warp; kb < KB; kb += kPrWarps) {
            uint4 w[MT][2];
            bring(kb, w);
            take(kb, w);
        }
    }
    // the upper four warps' sums, then the lower four's onto them
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        if ((warp < kPrWarps / 2) == (turn == 1)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float& to = red[warp % (kPrWarps / 2)][16 * m + r + (j & 2 ? 8 : 0)][8 * nt + 2 * c + (j & 1)];
                        to = turn ? to + acc[nt][m][j] : acc[nt][m][j];
                    }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < MT * 16 * 8 * NT; i += kPrWarps * 32) {
        const int n = i % (MT * 16), t = i / (MT * 16);
        if (t >= rows) continue;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kPrWarps / 2; ++w) sum += red[w][n][t];
        float* to = y + t * stride + n0 + n;
        *to = add ? *to + sum : sum;
    }
}

// The same for fp32 weights (parity models): a warp takes a row of W and eight rows of x at a time
__global__ void __launch_bounds__(kPrWarps * 32) project_fp32_kernel(const float* W, const float* x, int rows, int K, int N, float* y,
                                                                     long long stride, int add) {
    const int lane = threadIdx.x & 31, n = blockIdx.x * kPrWarps + (threadIdx.x >> 5), t0 = blockIdx.y * 8;
    grid_dep_wait();
    grid_dep_launch();
    if (n >= N) return;
    const float* w = W + static_cast<size_t>(n) * K;
    float acc[8] = {};
    for (int k = lane * 4; k < K; k += 128) {
        const float4 a = *reinterpret_cast<const float4*>(w + k);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (t0 + t >= rows) break;
            const float4 b = *reinterpret_cast<const float4*>(x + static_cast<size_t>(t0 + t) * K + k);
            acc[t] += a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w;
        }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const float sum = warp_sum(acc[t]);
        if (lane == 0 && t0 + t < rows) {
            float* to = y + (t0 + t) * stride + n;
            *to = add ? *to + sum : sum;
        }
    }
}

}  // namespace spm
