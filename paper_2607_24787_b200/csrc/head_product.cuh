// y_h = x_h W_h or x_h W_h^T for every head h of every row: what stands before and behind attention over latent rows.
//
// A CTA takes 64 outputs of a head for 16 MT rows; its warps share the contracted axis out and add up in shared memory. Weights go
// from global memory into mma.sync's B fragments without a stop: the contracted elements and the outputs may be numbered as one likes as
// long as both operands and the result agree. Output g * 8 + j is column g of the j-th 8-wide product, so a thread reads eight neighbouring
// weights of a row and writes sixteen neighbouring outputs; contracted element 4 c + i (or 8 c + i, where these are the neighbours) is
// thread c's i-th of a step.
//
// Rows in fp32 are three bf16 parts, cut off and not rounded (their sum is the number, 24 bits, and none overflows), so that products are
// exact and sums fp32. mma.sync cuts sums off where it does not round them, some 2^-23 of a sum a product, which adds up where terms are of one sign (8192
// elements in one sum: 343 * 2^-24 too small). So fp32 calls' sums leave the products every few elements and are added up outside: here a step's, the
// lower parts first, so that the first parts' bits are all there and only the lower ones' last are cut off.
#pragma once

#include "latent_cache.cuh"
#include "mma_ops.cuh"
#include "ptx.cuh"
#include "tc_ops.cuh"

namespace spm {

struct HeadProductArgs {
    HeadRows x, y;
    const __nv_bfloat16* w;
    long long w_head, w_row;       // strides in elements
    int n_rows, in, out_tiles;
};

constexpr int kHpOut = 64;

__device__ __forceinline__ void hp_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// N pairs of neighbouring elements of a row of x: as they are in memory, and as PARTS bf16 words each
template <typename T, int N> struct Pairs;
template <int N>
struct Pairs<float, N> {
    float4 v[N / 2];
    __device__ __forceinline__ void load(const float* p, bool there) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = there ? reinterpret_cast<const float4*>(p)[i] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void parts(uint32_t (&w)[N][3]) const {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { cut_parts(v[i].x, v[i].y, w[2 * i]); cut_parts(v[i].z, v[i].w, w[2 * i + 1]); }
    }
};
template <int N>
struct Pairs<__nv_bfloat16, N> {
    uint32_t v[N];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool there) {
        if constexpr (N == 2) {
            const uint2 u = there ? *reinterpret_cast<const uint2*>(p) : make_uint2(0, 0);
            v[0] = u.x; v[1] = u.y;
        } else {
            const uint4 u = there ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
            v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
        }
    }
    __device__ __forceinline__ void parts(uint32_t (&w)[N][1]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i][0] = v[i];
    }
};

// TRANSPOSED: W is [out][in], else [in][out]
template <typename T, bool TRANSPOSED, int MT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) head_product_kernel(const HeadProductArgs a) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int STEP = TRANSPOSED ? 32 : 16, PAIRS = TRANSPOSED ? 4 : 2;       // contracted elements of a step, of them pairs of a thread
    __shared__ float sums[WARPS / 2][MT * 16][kHpOut];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int head = blockIdx.y, o0 = blockIdx.x % a.out_tiles * kHpOut, row0 = blockIdx.x / a.out_tiles * (16 * MT);
    const __nv_bfloat16* w = a.w + head * a.w_head;
    const T* x = static_cast<const T*>(a.x.p) + head * a.x.head;
    const int steps = a.in / STEP, from = steps * warp / WARPS, to = steps * (warp + 1) / WARPS;
    float acc[MT][8][4] = {};
    grid_dep_wait();
    grid_dep_launch();
    // a step's weights and rows as they are in memory, one step ahead
    uint4 w_raw[TRANSPOSED ? 8 : 4];
    Pairs<T, PAIRS> x_raw[MT][2];
    auto load = [&](int s) {
        if (s >= to) return;
#pragma unroll
        for (int j = 0; j < (TRANSPOSED ? 8 : 4); ++j)
            w_raw[j] = *reinterpret_cast<const uint4*>(TRANSPOSED ? w + (o0 + g * 8 + j) * a.w_row + s * 32 + c * 8 : w + (s * 16 + c * 4 + j) * a.w_row + o0 + g * 8);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = row0 + t * 16 + i * 8 + g;
                x_raw[t][i].load(x + r * a.x.row + s * STEP + c * 2 * PAIRS, r < a.n_rows);
            }
    };
    load(from);
    for (int s = from; s < to; ++s) {
        uint32_t b[8][TRANSPOSED ? 4 : 2], rows[MT][2][PAIRS][PARTS];
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { b[j][0] = w_raw[j].x; b[j][1] = w_raw[j].y; b[j][2] = w_raw[j].z; b[j][3] = w_raw[j].w; }
        } else {
            const uint32_t v[4][4] = {{w_raw[0].x, w_raw[0].y, w_raw[0].z, w_raw[0].w}, {w_raw[1].x, w_raw[1].y, w_raw[1].z, w_raw[1].w},
                                      {w_raw[2].x, w_raw[2].y, w_raw[2].z, w_raw[2].w}, {w_raw[3].x, w_raw[3].y, w_raw[3].z, w_raw[3].w}};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t pick = j & 1 ? 0x7632 : 0x5410;
                b[j][0] = __byte_perm(v[0][j / 2], v[1][j / 2], pick);
                b[j][1] = __byte_perm(v[2][j / 2], v[3][j / 2], pick);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) x_raw[t][i].parts(rows[t][i]);
        load(s + 1);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            auto product = [&](float (&d)[4], int j, int k, int p) {
                const uint32_t frag[4] = {rows[t][0][k][p], rows[t][1][k][p], rows[t][0][k + 1][p], rows[t][1][k + 1][p]};
                hp_mma(d, frag, b[j][k], b[j][k + 1]);
            };
            if constexpr (PARTS == 3) {
                float step[8][4] = {};
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                    for (int k = 0; k < PAIRS; k += 2)
#pragma unroll
                        for (int j = 0; j < 8; ++j) product(step[j], j, k, p);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][j][e] += step[j][e];
            } else
#pragma unroll
                for (int k = 0; k < PAIRS; k += 2)
#pragma unroll
                    for (int j = 0; j < 8; ++j) product(acc[t][j], j, k, 0);
        }
    }
    // ---- the warps' sums: the upper half hands over, the lower half adds, twice in turn; always in the same order ----
#pragma unroll
    for (int n = WARPS / 2; n > 0; n /= 2) {
        if (n < WARPS / 2) __syncthreads();
        if (warp >= n && warp < 2 * n)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums[warp - n][t * 16 + j * 2 + (e >> 1)][(e & 1) * 32 + lane] = acc[t][j][e];
        __syncthreads();
        if (warp < n)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][j][e] += sums[warp][t * 16 + j * 2 + (e >> 1)][(e & 1) * 32 + lane];
    }
    if (warp > 0) return;
    // thread (g, c): rows g and g + 8, outputs 16 c .. 16 c + 15
    T* y = static_cast<T*>(a.y.p) + head * a.y.head + o0 + 16 * c;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = row0 + t * 16 + half * 8 + g;
            if (r >= a.n_rows) continue;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = acc[t][j][half * 2 + k];
                store_row<8>(y + r * a.y.row + 8 * k, v);
            }
        }
}

// The same for more rows: a CTA takes 128 outputs of a head for 64 rows, four warps' rows by two warps' outputs, and chunks of 64 contracted
// elements come into shared memory by asynchronous copies, several ahead, so that every weight and every element comes from memory once.
// Elements and outputs are numbered as above. 16-byte units of a row are moved by the row's number so that what eight (or, of 8 bytes, 16)
// threads read together lies in different banks. What bounds it with fp32 rows, whose parts make three products of one, is mma.sync, some 16 cycles
// a product and scheduler (64 rows, 128 heads from 512 to 128: 18 us, the kernel above 21, both with cold caches).
constexpr int kHtRows = 64, kHtOut = 128, kHtChunk = 64, kHtStages = 5, kHtThreads = 256;
template <typename T>
struct HtShape {
    static constexpr int w_bytes = kHtOut * kHtChunk * 2, x_bytes = kHtRows * kHtChunk * int(sizeof(T)), stage = w_bytes + x_bytes;
    static constexpr int smem = kHtStages * stage;
};
template <typename T, bool TRANSPOSED>
__global__ void __launch_bounds__(kHtThreads) head_product_tile_kernel(const HeadProductArgs a, int out) {
    using S = HtShape<T>;
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, STEP = TRANSPOSED ? 32 : 16, PAIRS = TRANSPOSED ? 4 : 2;
    extern __shared__ __align__(128) unsigned char ht_smem[];
    const uint32_t base = smem_u32(ht_smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3, wr = warp & 3, wn = warp >> 2;
    const int head = blockIdx.y, o0 = blockIdx.x % a.out_tiles * kHtOut, row0 = blockIdx.x / a.out_tiles * kHtRows;
    const __nv_bfloat16* w = a.w + head * a.w_head;
    const T* x = static_cast<const T*>(a.x.p) + head * a.x.head;
    grid_dep_wait();
    grid_dep_launch();
    // where unit u of a row lies: W by rows of outputs (transposed) or of contracted elements, x by rows
    auto w_unit = [](int r, int u) { return TRANSPOSED ? uint32_t(r * 128 + ((u ^ ((r >> 3 & 1) << 2)) << 4)) : uint32_t(r * 256 + ((u ^ ((r >> 2 & 3) << 1)) << 4)); };
    auto x_unit = [](int r, int u) {
        const int by = sizeof(T) == 4 ? (TRANSPOSED ? r & 1 : (r & 1) << 2) : (TRANSPOSED ? (r & 1) << 2 : (r & 3) << 1);
        return uint32_t(r * (kHtChunk * int(sizeof(T))) + ((u ^ by) << 4));
    };
    const int chunks = a.in / kHtChunk;
    auto copy = [&](int k) {
        if (k < chunks) {
            const uint32_t to = base + k % kHtStages * S::stage;
#pragma unroll
            for (int i = tid; i < S::w_bytes / 16; i += kHtThreads) {
                constexpr int UNITS = TRANSPOSED ? kHtChunk / 8 : kHtOut / 8;
                const int r = i / UNITS, u = i % UNITS, o = o0 + (TRANSPOSED ? r : u * 8);
                const bool is = o < out;
                copy16_or_zero(to + w_unit(r, u), is ? (TRANSPOSED ? w + o * a.w_row + k * kHtChunk + u * 8 : w + (k * kHtChunk + r) * a.w_row + o) : w, is);
            }
#pragma unroll
            for (int i = tid; i < S::x_bytes / 16; i += kHtThreads) {
                constexpr int EACH = 16 / int(sizeof(T)), UNITS = kHtChunk / EACH;
                const int r = i / UNITS, u = i % UNITS;
                const bool is = row0 + r < a.n_rows;
                copy16_or_zero(to + S::w_bytes + x_unit(r, u), is ? x + (row0 + r) * a.x.row + k * kHtChunk + u * EACH : x, is);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kHtStages - 1; ++k) copy(k);
    float acc[8][4] = {}, low[8][4] = {};
    const bool idle = o0 + wn * 64 >= out;       // (the last 64 of an odd number of them)
    for (int k = 0; k < chunks; ++k) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kHtStages - 2) : "memory");
        __syncthreads();
        copy(k + kHtStages - 1);
        if (idle) continue;
        const uint32_t w_at = base + k % kHtStages * S::stage, x_at = w_at + S::w_bytes;
        float part[8][4] = {};                   // fp32: the first parts' sums of a chunk; the others' are 2^-7 of them at most and stay in the products
        float (&sum)[8][4] = sizeof(T) == 4 ? part : acc;
#pragma unroll
        for (int s = 0; s < kHtChunk / STEP; ++s) {
            uint32_t rows[2][PAIRS][PARTS], b[8][TRANSPOSED ? 4 : 2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = wr * 16 + i * 8 + g;
                if constexpr (sizeof(T) == 4) {
                    Pairs<float, PAIRS> p;
#pragma unroll
                    for (int u = 0; u < PAIRS / 2; ++u) {
                        const uint4 v = lds128(x_at + x_unit(r, s * (STEP / 4) + c * (PAIRS / 2) + u));
                        p.v[u] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
                    }
                    p.parts(rows[i]);
                } else if constexpr (TRANSPOSED) {
                    const uint4 v = lds128(x_at + x_unit(r, s * 4 + c));
                    rows[i][0][0] = v.x; rows[i][1][0] = v.y; rows[i][2][0] = v.z; rows[i][3][0] = v.w;
                } else
                    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(rows[i][0][0]), "=r"(rows[i][1][0]) : "r"(x_at + x_unit(r, s * 2 + (c >> 1)) + (c & 1) * 8));
            }
            if constexpr (TRANSPOSED) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 v = lds128(w_at + w_unit(wn * 64 + g * 8 + j, s * 4 + c));
                    b[j][0] = v.x; b[j][1] = v.y; b[j][2] = v.z; b[j][3] = v.w;
                }
            } else {
                uint32_t v[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 u = lds128(w_at + w_unit(s * 16 + c * 4 + i, wn * 8 + g));
                    v[i][0] = u.x; v[i][1] = u.y; v[i][2] = u.z; v[i][3] = u.w;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t pick = j & 1 ? 0x7632 : 0x5410;
                    b[j][0] = __byte_perm(v[0][j / 2], v[1][j / 2], pick);
                    b[j][1] = __byte_perm(v[2][j / 2], v[3][j / 2], pick);
                }
            }
#pragma unroll
            for (int e = 0; e < PAIRS; e += 2)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const uint32_t frag[4] = {rows[0][e][p], rows[1][e][p], rows[0][e + 1][p], rows[1][e + 1][p]};
#pragma unroll
                    for (int j = 0; j < 8; ++j) hp_mma(p == 0 ? sum[j] : low[j], frag, b[j][e], b[j][e + 1]);
                }
        }
        if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] += part[j][e];
    }
    if (idle) return;
    if constexpr (sizeof(T) == 4)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] += low[j][e];
    T* y = static_cast<T*>(a.y.p) + head * a.y.head + o0 + wn * 64 + 16 * c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = row0 + wr * 16 + i * 8 + g;
        if (r >= a.n_rows) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = acc[j][i * 2 + k];
            store_row<8>(y + r * a.y.row + 8 * k, v);
        }
    }
}

}  // namespace spm
