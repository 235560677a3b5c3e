// The rows of a batch on their way into the latent cache, and the queries' rotation beside it.
//
// row = [latent * rsqrt(mean(latent^2) + eps) * gamma | R(position) key], rounded to bf16 once; a query's last elements are turned alike.
#pragma once

#include "kv_write.cuh"
#include "latent_cache.cuh"
#include "ptx.cuh"

namespace spm {

struct LatentWriteArgs {
    LatentPool kv;
    KvBatch batch;
    RopeArgs rope;
    int turn;                          // there is a rotation
    HeadRows q, q_out, latent, key;
    int q_heads, n_rows;
};

// Two elements a lane, turned: where they stand in a row of `rope` elements
__device__ __forceinline__ void pair_of(const RopeArgs& r, int lane, int& e0, int& e1) {
    const int half = r.rot_dim / 2;
    const bool apart = !r.neighbours && lane < half;
    e0 = apart ? lane : 2 * lane;
    e1 = apart ? lane + half : 2 * lane + 1;
}
__device__ __forceinline__ float2 load_pair(const float* p, int e0, int e1) {
    return e1 == e0 + 1 ? *reinterpret_cast<const float2*>(p + e0) : make_float2(p[e0], p[e1]);
}
__device__ __forceinline__ float2 load_pair(const __nv_bfloat16* p, int e0, int e1) {
    return e1 == e0 + 1 ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p + e0)) : make_float2(__bfloat162float(p[e0]), __bfloat162float(p[e1]));
}
__device__ __forceinline__ void store_pair(float* p, int e0, int e1, float2 v) {
    if (e1 == e0 + 1) *reinterpret_cast<float2*>(p + e0) = v;
    else { p[e0] = v.x; p[e1] = v.y; }
}
__device__ __forceinline__ void store_pair(__nv_bfloat16* p, int e0, int e1, float2 v) {
    if (e1 == e0 + 1) *reinterpret_cast<__nv_bfloat162*>(p + e0) = __floats2bfloat162_rn(v.x, v.y);
    else { p[e0] = __float2bfloat16_rn(v.x); p[e1] = __float2bfloat16_rn(v.y); }
}

// A warp takes a row, or one of gridDim.y parts of its query heads (the first part the cache's row too). A lane turns one pair of a head: at most 64
// elements turn, so a row's angles, taken in 64 bits (far positions), are one a lane and stay in two registers. The norm's sum is fp32: what
// it scales is rounded to bf16's 8 bits.
template <typename T>
__global__ void __launch_bounds__(kKvWarps * 32, 4) latent_write_kernel(const LatentWriteArgs a) {
    constexpr int AHEAD = 8;                   // query heads in flight
    const int lane = threadIdx.x & 31, pairs = a.kv.rope / 2;
    grid_dep_wait();
    grid_dep_launch();
    int e0, e1;
    pair_of(a.rope, lane, e0, e1);
    const int part = blockIdx.y, row = blockIdx.x * kKvWarps + (threadIdx.x >> 5);
    if (row >= a.n_rows) return;
    int h = a.q_heads * part / int(gridDim.y);
    const int h_end = a.q_heads * (part + 1) / int(gridDim.y);
    // loads that need not know where the row goes
    float2 q[AHEAD];
    const T* q_at = static_cast<const T*>(a.q.p) + row * a.q.row;
    T* q_to = static_cast<T*>(a.q_out.p) + row * a.q_out.row;
    auto take = [&] {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (h + u < h_end && lane < pairs) q[u] = load_pair(q_at + (h + u) * a.q.head, e0, e1);
    };
    take();
    float x[2][8] = {};
    float2 key = make_float2(0.f, 0.f);
    if (part == 0) {
        const T* from = static_cast<const T*>(a.latent.p) + row * a.latent.row;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i * 256 + lane * 8 < a.kv.latent) unpack8<T>(raw8(from + i * 256 + lane * 8), x[i]);
        if (lane < pairs) key = load_pair(static_cast<const T*>(a.key.p) + row * a.key.row, e0, e1);
    }
    const RowAt r = kv_row_at(a.batch, row);
    if (r.seq >= a.batch.n_seq) return;
    float c = 1.f, s = 0.f;
    const bool turns = a.turn && lane < a.rope.rot_dim / 2;
    if (turns) {
        const int axis = a.rope.axis_of ? min(int(a.rope.axis_of[lane]), a.rope.n_axes - 1) : 0;
        double ds, dc;
        sincos(double(a.rope.positions[axis * a.rope.pos_stride + row]) * double(a.rope.inv_freq[lane]), &ds, &dc);
        c = float(dc);
        s = float(ds);
    }
    auto turned = [&](float2 v) { return turns ? make_float2(v.x * c - v.y * s, v.y * c + v.x * s) : v; };
    if (part == 0 && r.pos >= 0) {
        const long long at = latent_row_at(a.kv, a.batch, r.seq, r.pos, lane == 0);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[i][e], x[i][e], sum);
        const float inv = rsqrtf(warp_sum(sum) / float(a.kv.latent) + a.rope.eps);
        if (at >= 0) {
            __nv_bfloat16* to = a.kv.rows + at * (a.kv.latent + a.kv.rope);
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = i * 256 + lane * 8;
                if (e >= a.kv.latent) continue;
                if (a.rope.k_gamma) {
                    float g[8];
                    load_row<8>(a.rope.k_gamma + e, g);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[i][k] = x[i][k] * inv * g[k];
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) odd |= !(fabsf(x[i][k]) < 0x1.ffp127f);      // (what rounds to an infinity too)
                store_row<8>(to + e, x[i]);
            }
            if (lane < pairs) {
                const float2 v = turned(key);
                odd |= !(fabsf(v.x) < 0x1.ffp127f) || !(fabsf(v.y) < 0x1.ffp127f);
                store_pair(to + a.kv.latent, e0, e1, v);
            }
            if (__any_sync(0xffffffffu, odd) && lane == 0) kv_note(a.kv, SPM_KV_NONFINITE);
        }
    }
    while (h < h_end) {
        float2 now[AHEAD];
        const int h_now = h;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) now[u] = q[u];
        h += AHEAD;
        take();
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (h_now + u < h_end && lane < pairs) store_pair(q_to + (h_now + u) * a.q_out.head, e0, e1, turned(now[u]));
    }
}

}  // namespace spm
