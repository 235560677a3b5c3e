// Rotation of heads, and the rows of a batch on their way into the 4-bit cache and out of it.
#pragma once

#include "kv_cache.cuh"

namespace spm {

constexpr int kKvWarps = 8;            // of a block of the kernels here

struct RopeArgs {
    const float* inv_freq;
    const unsigned char* axis_of;
    const float *q_gamma, *k_gamma;
    const int* positions;
    long long pos_stride;
    int n_axes, rot_dim, neighbours;
    float eps;
};
struct WriteArgs {
    KvPool kv;
    KvBatch batch;                     // n_seq < 0: rotation alone, every row
    RopeArgs rope;
    HeadRows q, q_out, k, v;
    int q_heads, kv_heads, n_rows;
};

// What a lane turns of a head row: its elements' cosines and sines, and the lane that holds their partners
template <int E>
struct Turn {
    float c[E], s[E];
    int partner;                       // -1: not turned
};

// x: E elements a lane of one head row. Products and sums are rounded one by one and the norm's sum is taken in 64 bits, so that the
// 4-bit codes do not depend on how the compiler contracts or on the order of a sum.
template <int E>
__device__ __forceinline__ void norm_and_turn(const RopeArgs& a, const Turn<E>& t, const float* gamma, int lane, float (&x)[E]) {
    if (gamma) {
        double sum = 0.;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += double(x[e]) * double(x[e]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float inv = float(1. / sqrt(sum / (32 * E) + double(a.eps)));
        float g[E];
        load_row<E>(gamma + lane * E, g);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __fmul_rn(__fmul_rn(x[e], inv), g[e]);
    }
    if (a.rot_dim == 0) return;
    if (a.neighbours) {
        if (t.partner < 0) return;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float p = x[e], q = x[e + 1];
            x[e] = __fsub_rn(__fmul_rn(p, t.c[e]), __fmul_rn(q, t.s[e]));
            x[e + 1] = __fadd_rn(__fmul_rn(q, t.c[e]), __fmul_rn(p, t.s[e]));
        }
        return;
    }
    const int from = t.partner < 0 ? lane : t.partner;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float o = __shfl_sync(0xffffffffu, x[e], from);
        if (t.partner < 0) continue;
        const float xc = __fmul_rn(x[e], t.c[e]), os = __fmul_rn(o, t.s[e]);
        x[e] = t.partner > lane ? __fsub_rn(xc, os) : __fadd_rn(xc, os);
    }
}

// One head row into the cache: `at` is its block, tok its place there, part 0 / 1 keys / values
template <int HD>
__device__ __forceinline__ void quantise_row(const KvPool& kv, unsigned char* at, int tok, int part, int lane, float (&x)[HD / 32]) {
    constexpr int E = HD / 32;
    bool odd = false;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        odd |= !(fabsf(x[e]) < INFINITY);
        if (x[e] != x[e]) x[e] = 0.f;
        if (fabsf(x[e]) > fabsf(m)) m = x[e];
    }
    if (__any_sync(0xffffffffu, odd) && lane == 0) kv_note(kv, SPM_KV_NONFINITE);
#pragma unroll
    for (int o = 1; o < 32 / E; o <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, m, o);
        if (fabsf(other) > fabsf(m) || (fabsf(other) == fabsf(m) && (lane & o))) m = other;
    }
    const __half scale = __float2half_rn(fminf(fmaxf(m * -0.125f, -65504.f), 65504.f));
    const float d = __half2float(scale), inv = d == 0.f ? 0.f : __frcp_rn(d);
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float r = fminf(fmaxf(rintf(__fmul_rn(x[e], inv)), -8.f), 7.f);
        codes |= uint32_t(int(r) + 8) << (4 * e);
    }
    const int g = lane * E / 32, in = lane * E % 32;
    unsigned char* to = at + part * kv_v_codes(HD) + (g * kKvBlock + tok) * 16 + in / 2;
    if constexpr (E == 2) *to = (unsigned char)codes;
    else if constexpr (E == 4) *reinterpret_cast<unsigned short*>(to) = (unsigned short)codes;
    else *reinterpret_cast<uint32_t*>(to) = codes;
    if (in == 0) *reinterpret_cast<__half*>(at + kv_k_scales(HD) + part * HD + (tok * (HD / 32) + g) * 2) = scale;
}

// A block takes a row and, of its heads (keys, values, queries), every gridDim.y-th eight; a warp takes a head.
template <typename T, int HD>
__global__ void __launch_bounds__(kKvWarps * 32) kv_write_kernel(const WriteArgs a) {
    constexpr int E = HD / 32;
    __shared__ float2 turn[HD / 2];
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long block = -1;
    int tok = 0;
    if (a.batch.n_seq >= 0) {
        const RowAt r = kv_row_at(a.batch, row);
        if (r.seq >= a.batch.n_seq) return;
        if (r.pos >= 0 && a.kv_heads) {
            block = kv_block_at<HD>(a.kv, a.batch, r.seq, r.pos, 0);
            tok = r.pos % kKvBlock;
            if (block < 0 && lane == 0) kv_note(a.kv, r.pos / a.kv.page_size >= a.batch.stride ? SPM_KV_TOO_LONG : SPM_KV_BAD_PAGE);
        }
    }
    const int half = a.rope.rot_dim / 2;
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        const int axis = a.rope.axis_of ? min(int(a.rope.axis_of[i]), a.rope.n_axes - 1) : 0;
        double s, c;
        sincos(double(a.rope.positions[axis * a.rope.pos_stride + row]) * double(a.rope.inv_freq[i]), &s, &c);
        turn[i] = make_float2(float(c), float(s));
    }
    __syncthreads();
    Turn<E> t;
    const int lanes = a.rope.rot_dim / E;            // that hold turned elements
    t.partner = lane >= lanes ? -1 : lane < lanes / 2 ? lane + lanes / 2 : lane - lanes / 2;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int pair = a.rope.neighbours ? (lane * E + e) / 2 : (t.partner < lane ? t.partner : lane) * E + e;
        const float2 cs = t.partner < 0 ? make_float2(1.f, 0.f) : turn[pair];
        t.c[e] = cs.x; t.s[e] = cs.y;
    }
    const long long head_bytes = static_cast<long long>(a.kv.page_size / kKvBlock) * kv_block_bytes(HD);
    const int heads = 2 * a.kv_heads + a.q_heads;
    for (int h = blockIdx.y * kKvWarps + warp; h < heads; h += gridDim.y * kKvWarps) {
        const int kind = h < a.kv_heads ? 0 : h < 2 * a.kv_heads ? 1 : 2;       // key, value, query
        const int in = h - kind * a.kv_heads;
        const HeadRows& src = kind == 0 ? a.k : kind == 1 ? a.v : a.q;
        if (kind < 2 && block < 0) continue;
        float x[E];
        load_row<E>(static_cast<const T*>(src.p) + row * src.row + in * src.head + lane * E, x);
        if (kind != 1) norm_and_turn<E>(a.rope, t, kind == 0 ? a.rope.k_gamma : a.rope.q_gamma, lane, x);
        if (kind == 2) store_row<E>(static_cast<T*>(a.q_out.p) + row * a.q_out.row + in * a.q_out.head + lane * E, x);
        else quantise_row<HD>(a.kv, a.kv.pages + block + in * head_bytes, tok, kind, lane, x);
    }
}

struct ReadArgs {
    KvPool kv;
    KvBatch batch;
    HeadRows k, v;
};

// A warp takes a row; HD / 8 lanes a head's keys or values, eight elements each
template <typename T, int HD>
__global__ void __launch_bounds__(kKvWarps * 32) kv_read_kernel(const ReadArgs a) {
    constexpr int LANES = HD / 8;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const long long row = static_cast<long long>(blockIdx.x) * kKvWarps + (threadIdx.x >> 5);
    if (row >= a.batch.n_rows) return;
    const RowAt r = kv_row_at(a.batch, int(row));
    if (r.seq >= a.batch.n_seq) return;
    long long block = -1;
    if (r.pos >= 0) {
        block = kv_block_at<HD>(a.kv, a.batch, r.seq, r.pos, 0);
        if (block < 0 && lane == 0) kv_note(a.kv, r.pos / a.kv.page_size >= a.batch.stride ? SPM_KV_TOO_LONG : SPM_KV_BAD_PAGE);
    }
    const int tok = r.pos % kKvBlock;
    const long long head_bytes = static_cast<long long>(a.kv.page_size / kKvBlock) * kv_block_bytes(HD);
    for (int i = lane / LANES; i < 2 * a.kv.heads; i += 32 / LANES) {
        const int part = i >= a.kv.heads, head = i - part * a.kv.heads;
        const HeadRows& out = part ? a.v : a.k;
        if (!out.p) continue;
        float x[8] = {};
        if (block >= 0) {
            const unsigned char* at = a.kv.pages + block + head * head_bytes;
            const uint32_t w = *reinterpret_cast<const uint32_t*>(at + part * kv_v_codes(HD) + (sub / 4 * kKvBlock + tok) * 16 + sub % 4 * 4);
            const float d = __half2float(*reinterpret_cast<const __half*>(at + kv_k_scales(HD) + part * HD + (tok * (HD / 32) + sub / 4) * 2));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float(w >> (4 * e) & 15) - 8.f) * d;
        }
        store_row<8>(static_cast<T*>(out.p) + row * out.row + head * out.head + sub * 8, x);
    }
}

}  // namespace spm
