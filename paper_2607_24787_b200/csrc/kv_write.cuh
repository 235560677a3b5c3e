// Rotation of heads, and the rows of a batch on their way into the 4-bit cache and out of it.
#pragma once

#include "kv_cache.cuh"
#include "ptx.cuh"

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

// A lane holds eight consecutive elements of a head, HD / 8 lanes a head, so a warp takes 32 / (HD / 8) heads at once.
//
// The norm and the rotation decide between 4-bit codes, so their roundings are spelled out: every product and sum is rounded by itself
// (in pairs, nothing is contracted), the norm's sum is taken in 64 bits, and so are the angles.

// 1 / sqrt(v): Newton's step from the fp32 instruction's 22 bits leaves more than 40 (with the double root and division 107 MB of image
// patches take 40.9 us for 39.9)
__device__ __forceinline__ float rsqrt_of(double v) {
    if (!(v > 1e-30 && v < 1e30)) return float(1. / sqrt(v));
    const double y = rsqrtf(float(v));
    return float(fma(0.5 * y, fma(-v * y, y, 1.0), y));
}

// Cosines and sines of a row's pairs. Lane `sub` of the first halves turns pairs 8 sub .. 8 sub + 7 (with neighbours: pairs 4 sub .. 4 sub + 3),
// lane sub + rot_dim / 16 their second halves; entry [j][i] holds the cosines, then the sines, of pairs
// 8 i + 2 j and 8 i + 2 j + 1, so that lanes read side by side. The
// second table has the sines' signs turned: a first half is a cos + b (-sin), rounded as a cos - b sin is.
template <int HD>
struct Angles { float4 at[2][4][HD / 16]; };
template <int HD>
__device__ __forceinline__ void set_angle(Angles<HD>& t, int pair, float c, float s) {
    const int j = pair % 8 / 2, i = pair / 8, odd = pair & 1;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float* to = reinterpret_cast<float*>(&t.at[k][j][i]) + odd;
        to[0] = c;
        to[2] = k ? -s : s;
    }
}

// Norm (with gammas g) and rotation of eight elements a lane
template <int HD>
__device__ __forceinline__ void norm_and_turn(const RopeArgs& a, const Angles<HD>& t, bool norm, const float (&g)[8], int sub, float (&x)[8]) {
    constexpr int LANES = HD / 8;
    if (norm) {
        double sum = 0.;
#pragma unroll
        for (int e = 0; e < 8; ++e) { const double v = x[e]; sum = fma(v, v, sum); }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float inv = rsqrt_of(sum * (1. / HD) + double(a.eps));
        const unsigned long long inv2 = two_floats(inv, inv);
#pragma unroll
        for (int e = 0; e < 8; e += 2) floats_of(mul2(mul2(two_floats(x[e], x[e + 1]), inv2), two_floats(g[e], g[e + 1])), x[e], x[e + 1]);
    }
    if (a.rot_dim == 0) return;
    if (a.neighbours) {
        if (sub * 8 >= a.rot_dim) return;
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const float4 v = t.at[0][2 * (sub & 1) + e / 4][sub / 2];
            const float p0 = x[e], q0 = x[e + 1], p1 = x[e + 2], q1 = x[e + 3];
            x[e] = __fsub_rn(__fmul_rn(p0, v.x), __fmul_rn(q0, v.z));
            x[e + 1] = __fadd_rn(__fmul_rn(q0, v.x), __fmul_rn(p0, v.z));
            x[e + 2] = __fsub_rn(__fmul_rn(p1, v.y), __fmul_rn(q1, v.w));
            x[e + 3] = __fadd_rn(__fmul_rn(q1, v.y), __fmul_rn(p1, v.w));
        }
        return;
    }
    const int half = a.rot_dim / 16;             // lanes of the first halves
    const bool low = sub < half, in = sub < 2 * half;
    const int from = (threadIdx.x & 31) + (!in ? 0 : low ? half : -half);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = __shfl_sync(0xffffffffu, x[e], from);
    if (!in) return;
    const float4* at = &t.at[low][0][low ? sub : sub - half];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float4 v = at[e / 2 * (HD / 16)];
        const unsigned long long own = mul2(two_floats(x[e], x[e + 1]), two_floats(v.x, v.y)), theirs = mul2(two_floats(o[e], o[e + 1]), two_floats(v.z, v.w));
        floats_of(add2(own, theirs), x[e], x[e + 1]);
    }
}

// A lane's eight elements into the cache (lanes with `write`): `at` is the head's block and part, tok the row's place there. Four lanes hold
// a group.
template <int HD>
__device__ __forceinline__ void quantise_row(const KvPool& kv, unsigned char* codes_at, unsigned char* scales_at, int tok, bool write, int sub,
                                             float (&x)[8]) {
    bool odd = false;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        odd |= !(fabsf(x[e]) < INFINITY);
        if (x[e] != x[e]) x[e] = 0.f;
        if (fabsf(x[e]) > fabsf(m)) m = x[e];
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, m, o);
        if (fabsf(other) > fabsf(m) || (fabsf(other) == fabsf(m) && (sub & o))) m = other;
    }
    if (!write) return;
    if (odd) kv_note(kv, SPM_KV_NONFINITE);
    const __half scale = __float2half_rn(fminf(fmaxf(m * -0.125f, -65504.f), 65504.f));
    const float d = __half2float(scale), inv = d == 0.f ? 0.f : __frcp_rn(d);
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = fminf(fmaxf(rintf(__fmul_rn(x[e], inv)), -8.f), 7.f);
        codes |= uint32_t(int(r) + 8) << (4 * e);
    }
    const int g = sub / 4;
    *reinterpret_cast<uint32_t*>(codes_at + (g * kKvBlock + tok) * 16 + sub % 4 * 4) = codes;
    if (sub % 4 == 0) *reinterpret_cast<__half*>(scales_at + (tok * (HD / 32) + g) * 2) = scale;
}

// Eight elements as they are in memory
struct Raw8 { uint4 a, b; };
__device__ __forceinline__ Raw8 raw8(const float* p) { return {reinterpret_cast<const uint4*>(p)[0], reinterpret_cast<const uint4*>(p)[1]}; }
__device__ __forceinline__ Raw8 raw8(const __nv_bfloat16* p) { return {*reinterpret_cast<const uint4*>(p), make_uint4(0, 0, 0, 0)}; }
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8& r, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        two_bf16(r.a.x, x[0], x[1]); two_bf16(r.a.y, x[2], x[3]); two_bf16(r.a.z, x[4], x[5]); two_bf16(r.a.w, x[6], x[7]);
    } else {
        x[0] = __uint_as_float(r.a.x); x[1] = __uint_as_float(r.a.y); x[2] = __uint_as_float(r.a.z); x[3] = __uint_as_float(r.a.w);
        x[4] = __uint_as_float(r.b.x); x[5] = __uint_as_float(r.b.y); x[6] = __uint_as_float(r.b.z); x[7] = __uint_as_float(r.b.w);
    }
}

// A warp takes a row, or one of `parts` of its heads: its angles first, then a few heads of one kind at a time (a turn), the next ones loaded
// meanwhile. Warps share nothing, so that one's angles go along with another's heads.
// Bound by instruction issue (74 % of the slots): some 240 a turn of two heads of 128, of which norm, rotation and finding the code are two
// thirds, and a row's angles in 64 bits. 18124 prompt rows with 32 query heads: 121 us for 344 MB, 2.8 TB/s; a block of four warps a row
// with barriers between angles and heads took 139. One row: 4 us, the chain from row number to page to codes.
template <typename T, int HD>
__global__ void __launch_bounds__(kKvWarps * 32, 4) kv_write_kernel(const WriteArgs a, int parts) {
    constexpr int LANES = HD / 8, HEADS = 32 / LANES;
    __shared__ Angles<HD> angles_of[kKvWarps];
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    Angles<HD>& angles = angles_of[threadIdx.x >> 5];
    grid_dep_wait();
    grid_dep_launch();
    // turns: keys, values, queries
    const int kv_turns = (a.kv_heads + HEADS - 1) / HEADS, turns = 2 * kv_turns + (a.q_heads + HEADS - 1) / HEADS;
    const int half = a.rope.rot_dim / 2;
    float gk[8] = {}, gq[8] = {};
    if (a.rope.k_gamma && a.kv_heads) load_row<8>(a.rope.k_gamma + sub * 8, gk);
    if (a.rope.q_gamma && a.q_heads) load_row<8>(a.rope.q_gamma + sub * 8, gq);
    for (long long task = static_cast<long long>(blockIdx.x) * kKvWarps + (threadIdx.x >> 5); task < static_cast<long long>(a.n_rows) * parts;
         task += static_cast<long long>(gridDim.x) * kKvWarps) {
        const int row = int(task / parts), part = int(task - static_cast<long long>(row) * parts);
        int turn = turns * part / parts;
        const int end = turns * (part + 1) / parts;
        int kind = 0, head = 0;
        bool is = false;
        Raw8 raw{};
        auto take = [&] {
            kind = turn < kv_turns ? 0 : turn < 2 * kv_turns ? 1 : 2;
            head = (turn - kind * kv_turns) * HEADS + lane / LANES;
            const HeadRows& from = kind == 0 ? a.k : kind == 1 ? a.v : a.q;
            is = turn < end && head < (kind == 2 ? a.q_heads : a.kv_heads);
            if (is) raw = raw8(static_cast<const T*>(from.p) + row * from.row + head * from.head + sub * 8);
        };
        take();
        long long block = -1;                    // of the row's head 0 in the cache; -1: nowhere
        int tok = 0;
        if (a.batch.n_seq >= 0) {
            const RowAt r = kv_row_at(a.batch, row);
            if (r.seq >= a.batch.n_seq) continue;
            if (r.pos >= 0) {
                block = kv_block_at<HD>(a.kv, a.batch, r.seq, r.pos, 0);
                tok = r.pos % kKvBlock;
                if (block < 0 && lane == 0) kv_note(a.kv, r.pos / a.kv.page_size >= a.batch.stride ? SPM_KV_TOO_LONG : SPM_KV_BAD_PAGE);
            }
        }
        __syncwarp();
        for (int p = lane; p < half; p += 32) {
            const int axis = a.rope.axis_of ? min(int(a.rope.axis_of[p]), a.rope.n_axes - 1) : 0;
            double s, c;
            sincos(double(a.rope.positions[axis * a.rope.pos_stride + row]) * double(a.rope.inv_freq[p]), &s, &c);
            set_angle(angles, p, float(c), float(s));
        }
        __syncwarp();
        while (turn < end) {
            float x[8];
            unpack8<T>(raw, x);
            const int kind_now = kind, head_now = head;
            const bool is_now = is;
            ++turn;
            take();
            if (kind_now == 2) {
                norm_and_turn<HD>(a.rope, angles, a.rope.q_gamma != nullptr, gq, sub, x);
                if (is_now) store_row<8>(static_cast<T*>(a.q_out.p) + row * a.q_out.row + head_now * a.q_out.head + sub * 8, x);
            } else {
                if (kind_now == 0) norm_and_turn<HD>(a.rope, angles, a.rope.k_gamma != nullptr, gk, sub, x);
                unsigned char* at = a.kv.pages + block + head_now * static_cast<long long>(a.kv.page_size / kKvBlock) * kv_block_bytes(HD);
                quantise_row<HD>(a.kv, at + kind_now * kv_v_codes(HD), at + kv_k_scales(HD) + kind_now * HD, tok, is_now && block >= 0, sub, x);
            }
        }
    }
}

struct ReadArgs {
    KvPool kv;
    KvBatch batch;
    HeadRows k, v;
};

// A thread takes eight elements of a row, of every head's keys and values, four of them in flight. Neighbouring tokens, whose codes stand
// side by side, are in one warp. 16 sequences of up to 8190 tokens, 197 MB: 46 us, 4.3 TB/s, nearly all of it written, 16 bytes a thread.
template <typename T, int HD>
__global__ void __launch_bounds__(kKvWarps * 32, 6) kv_read_kernel(const ReadArgs a) {
    constexpr int LANES = HD / 8, ROWS = kKvWarps * 32 / LANES, AHEAD = 4;
    __shared__ long long blocks[ROWS];           // of the row's head 0; -1: nowhere (zeros), -2: no sequence's row
    __shared__ int toks[ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row0 = static_cast<long long>(blockIdx.x) * ROWS;
    grid_dep_wait();
    grid_dep_launch();
    const int rows = int(min(static_cast<long long>(ROWS), a.batch.n_rows - row0));
    for (int i = warp; i < rows; i += kKvWarps) {
        const RowAt r = kv_row_at(a.batch, int(row0) + i);
        long long block = r.seq >= a.batch.n_seq ? -2 : -1;
        if (block == -1 && r.pos >= 0) {
            block = kv_block_at<HD>(a.kv, a.batch, r.seq, r.pos, 0);
            if (block < 0 && lane == 0) kv_note(a.kv, r.pos / a.kv.page_size >= a.batch.stride ? SPM_KV_TOO_LONG : SPM_KV_BAD_PAGE);
        }
        if (lane == 0) { blocks[i] = block; toks[i] = r.pos % kKvBlock; }
    }
    __syncthreads();
    const int sub = threadIdx.x % LANES, rr = threadIdx.x / LANES;
    if (rr >= rows || blocks[rr] == -2) return;
    const bool there = blocks[rr] >= 0;
    const int tok = there ? toks[rr] : 0;
    const long long head_bytes = static_cast<long long>(a.kv.page_size / kKvBlock) * kv_block_bytes(HD);
    const unsigned char* at = a.kv.pages + (there ? blocks[rr] : 0) + (sub / 4 * kKvBlock + tok) * 16 + sub % 4 * 4;
    const unsigned char* scales = a.kv.pages + (there ? blocks[rr] : 0) + kv_k_scales(HD) + (tok * (HD / 32) + sub / 4) * 2;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const HeadRows& out = part ? a.v : a.k;
        if (!out.p) continue;
        T* to = static_cast<T*>(out.p) + (row0 + rr) * out.row + sub * 8;
        for (int h0 = 0; h0 < a.kv.heads; h0 += AHEAD) {
            uint32_t w[AHEAD];
            __half d[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (!there || h0 + u >= a.kv.heads) continue;
                w[u] = *reinterpret_cast<const uint32_t*>(at + part * kv_v_codes(HD) + (h0 + u) * head_bytes);
                d[u] = *reinterpret_cast<const __half*>(scales + part * HD + (h0 + u) * head_bytes);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (h0 + u >= a.kv.heads) continue;
                float x[8] = {};
                if (there) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = (float(w[u] >> (4 * e) & 15) - 8.f) * __half2float(d[u]);
                }
                store_row<8>(to + (h0 + u) * out.head, x);
            }
        }
    }
}

}  // namespace spm
