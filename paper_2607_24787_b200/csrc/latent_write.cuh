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

// A warp takes a row, or one of gridDim.y parts of its query heads (the first part the cache's row too). A lane holds eight elements of a head,
// rope / 8 lanes a head, so a warp takes several heads at once. A row's angles, taken in 64 bits (far positions), are one a lane (at most 64
// elements turn) and pass through shared memory to the lanes that need them. The norm's sum is fp32, what it scales being rounded to bf16's 8 bits.
// With a head at a time, an element pair a lane, 18124 prompt rows of 16 heads took 76 us, 33.5 now (135 MB); 1271
// instructions a row fill two thirds of the issue slots, the rest waits for loads, with 44 % of the warps that an SM holds.
template <typename T>
__global__ void __launch_bounds__(kKvWarps * 32, 4) latent_write_kernel(const LatentWriteArgs a) {
    constexpr int AHEAD = 2;           // vectors in flight (four: registers spill, 41 us for 38 with nothing in L2)
    __shared__ float2 angles_of[kKvWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lanes = a.kv.rope / 8, per = 32 / lanes, sub = lane % lanes, place = lane / lanes;
    grid_dep_wait();
    grid_dep_launch();
    const int part = blockIdx.y, row = blockIdx.x * kKvWarps + warp;
    if (row >= a.n_rows) return;
    // loads that need not know where the row goes
    const int h_end = a.q_heads * (part + 1) / int(gridDim.y);
    int h = a.q_heads * part / int(gridDim.y) + (place < per ? place : h_end);
    Raw8 raw[AHEAD];
    const T* q_at = static_cast<const T*>(a.q.p) + row * a.q.row + sub * 8;
    T* q_to = static_cast<T*>(a.q_out.p) + row * a.q_out.row + sub * 8;
    auto take = [&] {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (h + u * per < h_end) raw[u] = raw8(q_at + (h + u * per) * a.q.head);
    };
    take();
    Raw8 latent[2] = {}, key = {};
    if (part == 0) {
        const T* from = static_cast<const T*>(a.latent.p) + row * a.latent.row;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i * 256 + lane * 8 < a.kv.latent) latent[i] = raw8(from + i * 256 + lane * 8);
        if (lane < lanes) key = raw8(static_cast<const T*>(a.key.p) + row * a.key.row + lane * 8);
    }
    const RowAt r = kv_row_at(a.batch, row);
    if (r.seq >= a.batch.n_seq) return;
    const int half = a.turn ? a.rope.rot_dim / 2 : 0;
    if (lane < half) {
        const int axis = a.rope.axis_of ? min(int(a.rope.axis_of[lane]), a.rope.n_axes - 1) : 0;
        double s, c;
        sincos(double(a.rope.positions[axis * a.rope.pos_stride + row]) * double(a.rope.inv_freq[lane]), &s, &c);
        angles_of[warp][lane] = make_float2(float(c), float(s));
    }
    __syncwarp();
    // element e turns with element e ^ 1 (neighbours), or with the same one of the lane half / 8 on: cosine, and sine with its sign
    const bool turns = sub * 8 < 2 * half, first = sub < half / 8;
    const int partner = !turns || a.rope.neighbours ? lane : first ? lane + half / 8 : lane - half / 8;
    float c[8], s[8];
    if (turns)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 v = angles_of[warp][a.rope.neighbours ? sub * 4 + e / 2 : (first ? sub : sub - half / 8) * 8 + e];
            c[e] = v.x;
            s[e] = (a.rope.neighbours ? e % 2 == 0 : first) ? -v.y : v.y;
        }
    auto turn = [&](float (&x)[8]) {
        float o[8];
        if (a.rope.neighbours || half == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = x[e ^ 1];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = __shfl_sync(0xffffffffu, x[e], partner);
        }
        if (turns)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * c[e] + o[e] * s[e];
    };
    if (part == 0 && r.pos >= 0) {
        const long long at = latent_row_at(a.kv, a.batch, r.seq, r.pos, lane == 0);
        __nv_bfloat16* to = a.kv.rows + (at >= 0 ? at : 0) * (a.kv.latent + a.kv.rope);
        bool odd = false;
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) unpack8<T>(latent[i], x[i]);
        auto mean_of_squares = [&] {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(x[i][e], x[i][e], sum);
            return warp_sum(sum) / float(a.kv.latent);
        };
        float mean = mean_of_squares() + a.rope.eps;
        if (a.rope.k_gamma && !(mean > 0x1p-80f && mean < 0x1p110f)) {         // squares that fp32 does not hold, or not all of: of the row times a power of two
            const float by = mean < 1.f ? 0x1p100f : 0x1p-70f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= by;
            mean = mean_of_squares() + a.rope.eps * by * by;
        }
        const float inv = rsqrtf(mean);
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
            for (int k = 0; k < 8; ++k) odd |= !(fabsf(x[i][k]) < 0x1.ffp127f);          // (what rounds to an infinity too)
            if (at >= 0) store_row<8>(to + e, x[i]);
        }
        unpack8<T>(key, x[0]);
        turn(x[0]);
        if (lane < lanes) {
#pragma unroll
            for (int k = 0; k < 8; ++k) odd |= !(fabsf(x[0][k]) < 0x1.ffp127f);
            if (at >= 0) store_row<8>(to + a.kv.latent + lane * 8, x[0]);
        }
        if (__any_sync(0xffffffffu, odd) && at >= 0 && lane == 0) kv_note(a.kv, SPM_KV_NONFINITE);
    }
    while (__any_sync(0xffffffffu, h < h_end)) {
        Raw8 now[AHEAD];
        const int h_now = h;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) now[u] = raw[u];
        h += AHEAD * per;
        take();
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            float x[8];
            unpack8<T>(now[u], x);
            turn(x);
            if (h_now + u * per < h_end) store_row<8>(q_to + (h_now + u * per) * a.q_out.head, x);
        }
    }
}

}  // namespace spm
