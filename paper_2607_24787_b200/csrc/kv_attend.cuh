// Attention of new rows over the 4-bit cache, for a few rows a sequence (and for many fp32 ones).
//
// For a cache head, the new rows' query heads that read it are columns: column x is head x % group of row x / group, and eight columns are
// the N of an m16n8k16. Keys are its A operand (16 tokens by 16 elements) straight from their nibbles, and the scale of a group is put on
// the sum of the group's 32 products. Values are the A operand of the second product, transposed by ldmatrix (32 elements by 16 tokens);
// their scale goes onto the probability, which is the B operand, so no value is ever rounded. fp32 queries and scaled probabilities are two
// fp16 parts each, the number's rounding and the rounding of what that leaves: 23 bits at least, down to 2^-40 of a head's largest query
// element and 2^-34 of the largest product (three bf16 parts, 24 bits and six products for four, took 72.7 us where these take 69.2: 64
// sequences of 4096 tokens, 32 heads on 4).
// Nibbles are exact operands as they are masked out of their word, as bf16 subnormals (q4_mma.cuh): five instructions for eight of them.
// bf16 calls leave them so. Keys: the query is scaled up to them, and -8 times the sum of a group's queries is what the group's sum starts
// with. Values: the same words are fp16 subnormals, and probabilities times scales are fp16 numbers, of 11 bits and not bf16's 8: with bf16
// the result's error was 1.5 times that of its own rounding, now it is 1.02 times that, for 2 % of the time.
// For their range a group's scales are taken to 2 by a power of two that is above all of them so far, kept like the running
// maximum, and probabilities to 2^8: fp16's 11 bits hold for a probability down to 2^-22 of the largest, a scale down to 2^-15 of its
// group's largest and their product down to 2^-23, and no product is above 65504. One more product with -8 in the codes' place goes into the
// running sum before theirs, so that what is left to round is a tile's and not the whole context's sum of codes. fp32 calls subtract the 8
// from each code, nine instructions for eight, and lose nothing to it; a tile's sums are added to the running ones outside of the products,
// which cut sums off where they do not round them.
//
// All (sequence, columns, head) items together are a line of tiles of 32 tokens that is cut evenly between CTAs, and a CTA's piece
// evenly between its warps, whatever the lengths are: a warp walks its tiles with the running maximum and sum of each column, fed by its
// own ring of bulk copies. Where a cut falls into an item the parts meet in shared memory (cuts between warps) or, for cuts between
// CTAs, in the workspace, where kv_attend_join_kernel adds them in order.
//
// What bounds it: instructions and their latencies, some 670 a tile for eight columns or one, 49 % of the issue slots with four warps a
// scheduler (which is what 128 registers leave); not memory. 64 sequences of up to 16001 tokens, 268 MB: 72 us, 3.7 TB/s, of it 2.2 us a
// tile and warp, and 11 us at the ends (the kernel before, counting and finding the tiles 4, the parts' joining 4). More column tiles a warp
// (16, 32 columns) were slower a column, and so were 12 warps with deeper rings, and loops rolled up against the size of the code.
#pragma once

#include "kv_cache.cuh"
#include "ptx.cuh"
#include "q4_mma.cuh"

namespace spm {

struct AttendArgs {
    KvPool kv;
    KvBatch batch;
    HeadRows q, out;
    int group;                  // query heads a cache head
    int page_shift, group_shift;        // blocks a page, query heads a cache head are 1 << this, or -1
    float scale;
    float* parts;               // [2 * CTAs][part floats]
    int* joins;                 // [CTAs][8], of the item that begins in this CTA and goes on behind it: CTAs that share it (0: none), columns,
                                // head, first row, rows
    const int* rows;            // new rows of each sequence that this kernel takes; NULL: all of them
    int once;                   // every block is read by one warp alone
    unsigned long long wait_ns; // a wait in a kernel gives up after this long
    int withhold;               // (tests) arrivals that barriers wait for and nobody makes
};

// Row of column x (eight sequences of five drafted rows, 8 heads a cache head: 26.1 us with the division alone, 24.9)
__device__ __forceinline__ int column_row(const AttendArgs& a, int x) { return a.group_shift >= 0 ? x >> a.group_shift : x / a.group; }

constexpr int kAtTile = 32;     // tokens
constexpr int kAtMaxCtas = 148;
constexpr int kAtMinTiles = 4;  // of a CTA, before another one starts: a tile a scheduler (16, one a warp: 1025 tokens 11.8 us, 9.7 with 4)
constexpr int kAtFewBlocks = 8; // column blocks of a sequence that a lane counts by itself

template <typename T, int HD>
struct AtShape {
    static constexpr int cols = 8;
    static constexpr int tile_bytes = kAtTile / kKvBlock * kv_block_bytes(HD);
    static constexpr int part_floats = cols * (HD + 2);      // sums, then maxima, then sums of probabilities
    static constexpr int part_bytes = (part_floats * 4 + 15) / 16 * 16;
    // warps and stages of a warp's ring: what registers (the sums of HD x cols numbers, the queries) and shared memory leave
    static constexpr int warps = HD == 256 ? 8 : sizeof(T) == 4 ? 12 : 16;
    static constexpr int stages = HD == 64 ? 4 : HD == 256 || warps == 16 ? 2 : 3;
    static constexpr bool raw = sizeof(T) == 2;              // codes as they are masked out
    static constexpr float up = 8.f;                       // probabilities are taken to 2^8 then, so that none is above 2^14
    static constexpr float unscale = raw ? 0x1p23f : 0.5f;   // of sums of codes times probabilities
    // a sum of an odd element, beside that of the even one before it
    __device__ static float odd(float both, float low) { return raw ? (both - low) * (1.f / 16.f) : both; }
    static constexpr int ring_bytes = stages * tile_bytes;
    static_assert(ring_bytes >= part_bytes, "a warp's last part takes the place of its ring");
    static constexpr int smem(int n_seq) { return warps * (ring_bytes + part_bytes + stages * 8) + (n_seq > 64 ? n_seq * 8 : 0); }
    static_assert(warps * (ring_bytes + part_bytes + stages * 8) + SPM_KV_MAX_SEQS * 8 + (raw ? 9728 : 4608) <= 232448,
                  "227 KB, the last of it for the kernel's own arrays");
};

// A walk along the line of tiles. nk: tokens that the last of the item's columns sees, nt: tiles (one at least, so that rows that see
// nothing are written too).
template <int COLS>
struct Walk {
    int seq, ct, head, t, nt, first, n, len, nk;

    __device__ __forceinline__ void load(const AttendArgs& a) {      // of `seq`
        len = a.batch.lengths[seq];
        first = seq; n = 1;
        if (a.batch.row_start) {
            first = a.batch.row_start[seq];
            n = a.rows ? a.rows[seq] : min(a.batch.row_start[seq + 1] - first, a.batch.n_rows);
        }
    }
    __device__ __forceinline__ int blocks(const AttendArgs& a) const { return n > 0 ? (n * a.group + COLS - 1) / COLS : 0; }
    __device__ __forceinline__ void columns(const AttendArgs& a) {
        const int last = n == 1 ? 0 : min(n - 1, column_row(a, (ct + 1) * COLS - 1));
        nk = max(0, min(len - n + last + 1, a.batch.stride * a.kv.page_size));
        nt = max(1, (nk + kAtTile - 1) / kAtTile);
    }
    // tiles of all heads of column blocks `from`, `from` + `step`, ...
    __device__ __forceinline__ long long tiles_of_sequence(const AttendArgs& a, int from, int step) {
        long long sum = 0;
        const int m = blocks(a);
        for (ct = from; ct < m; ct += step) { columns(a); sum += nt; }
        return sum * a.kv.heads;
    }
    // to tile `rest` of the sequence, by a warp: lanes look at 32 column blocks at a time
    __device__ __forceinline__ void seek(const AttendArgs& a, long long rest) {
        const int lane = threadIdx.x & 31;
        const int m = blocks(a);
        for (int ct0 = 0; m > 1; ct0 += 32) {
            ct = ct0 + lane;
            columns(a);
            const long long own = ct < m ? static_cast<long long>(nt) * a.kv.heads : 0;
            long long upto = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            const int behind = __popc(__ballot_sync(0xffffffffu, upto <= rest));
            if (behind < 32) {
                rest -= __shfl_sync(0xffffffffu, upto - own, behind);
                ct = ct0 + behind;
                break;
            }
            rest -= __shfl_sync(0xffffffffu, upto, 31);
        }
        if (m <= 1) ct = 0;
        columns(a);
        head = int(rest / nt);
        t = int(rest - static_cast<long long>(head) * nt);
    }
    __device__ __forceinline__ void next(const AttendArgs& a) {
        if (++t < nt) return;
        t = 0;
        if (++head < a.kv.heads) return;
        head = 0;
        if (++ct >= blocks(a)) {
            ct = 0;
            do {
                if (++seq >= a.batch.n_seq) return;
                load(a);
            } while (n <= 0);
        }
        columns(a);
    }
};

// Where a column's result goes: its row, -1 where the item has no such column
template <int COLS>
__device__ __forceinline__ int row_of_column(const AttendArgs& a, int first, int n, int ct, int col, int& g) {
    const int x = ct * COLS + col, i = n == 1 ? (x >= a.group) : column_row(a, x);
    g = x - i * a.group;
    return i < n && first + i >= 0 && first + i < a.batch.n_rows ? first + i : -1;
}

// tiles [from, to) of nt; id: the item's first tile on the line, -1: none
struct PartMeta { long long id; int ct, head, from, to, nt, first, n; };

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// D = A B + C
__device__ __forceinline__ void mma_k16_from(float (&d)[4], const float4& c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c.x), "f"(c.y), "f"(c.z), "f"(c.w));
}
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }
__device__ __forceinline__ uint32_t bits_of(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ uint32_t pack_half(float a, float b) { return bits_of(__floats2half2_rn(a, b)); }
// D += A B of fp16
__device__ __forceinline__ void mma_half_k16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_half_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// A word's codes less 8 as fp16, exact: 1024 + code and 1024 + 16 code are numbers
__device__ __forceinline__ Nib4 q4_halves(uint32_t w) {
    const __half2 off = as_half2(0xe408e408u), sixteenth = as_half2(0x2c002c00u), off72 = as_half2(0xd480d480u);       // -1032, 1 / 16, -72
    const uint32_t v = w >> 8;
    return Nib4{{bits_of(__hadd2(as_half2((w & 0x000f000fu) | 0x64006400u), off)), bits_of(__hfma2(as_half2((w & 0x00f000f0u) | 0x64006400u), sixteenth, off72)),
                 bits_of(__hadd2(as_half2((v & 0x000f000fu) | 0x64006400u), off)), bits_of(__hfma2(as_half2((v & 0x00f000f0u) | 0x64006400u), sixteenth, off72))}};
}
// Two numbers as fp16, and what that leaves of them
__device__ __forceinline__ void two_parts(float x0, float x1, uint32_t& high, uint32_t& low) {
    const __half2 h = __floats2half2_rn(x0, x1);
    const float2 f = __half22float2(h);
    high = bits_of(h);
    low = pack_half(x0 - f.x, x1 - f.y);
}
// HD / 32 scales of a token, two a word; as numbers
template <int G>
__device__ __forceinline__ void scale_words(uint32_t addr, uint32_t (&w)[G / 2]) {
    if constexpr (G == 2) w[0] = lds32(addr);
    else if constexpr (G == 4) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
    else { const uint4 v = lds128(addr); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
}
template <int G>
__device__ __forceinline__ void token_scales(uint32_t addr, float (&s)[G]) {
    uint32_t w[G / 2];
    scale_words<G>(addr, w);
#pragma unroll
    for (int i = 0; i < G / 2; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        s[2 * i] = f.x; s[2 * i + 1] = f.y;
    }
}

// One column's group of queries as the B operand: pairs (i, i + 4) of the eight elements 8 c .. 8 c + 7. bf16 columns are taken by a power of
// two to a largest element in [1, 2), times 2^64 for codes of 2^-133 and 2^60 for 16 times those; sums then stand at 2^-69.
constexpr float kAtUp69 = 0x1p69f;
constexpr uint32_t kAtNarrowest = 0x04000400u, kAtWidest = 0x78007800u;     // 2^-14, 2^15
// Of a column's factor of scores. So small a one makes all alike, and yet a masked score stays one; so large a one makes all differ.
constexpr float kAtLeast = 1e-35f, kAtMost = 0x1p80f;
__device__ __forceinline__ uint32_t bf16_power(int e) { return uint32_t(127 + e << 7) * 0x10001u; }
// A word's bytes as operands: the low nibble of bytes 0, 2 and both nibbles of them (low + 16 high, also linear), the same of bytes 1, 3:
// four instructions. Values' elements are rows of the product, so the high nibble's sum is had from the two.
constexpr uint32_t kAtMinus8 = 0x80088008u, kAtMinus136 = 0x80888088u;      // -8 and -8 - 16 * 8 as codes
__device__ __forceinline__ Nib4 q4_bytes(uint32_t w) {
    const uint32_t even = w & 0x00ff00ffu, odd = __byte_perm(w, 0u, 0x4341);
    return Nib4{{even & 0x000f000fu, even, odd & 0x000f000fu, odd}};
}
__device__ __forceinline__ void query_words(uint32_t (&w)[1][4], uint32_t up64, uint32_t up60, bool flip) {         // in: eight bf16 numbers as they were loaded
    const uint32_t x = w[0][0], y = w[0][1], z = w[0][2], u = w[0][3], sign = flip ? 0x80008000u : 0u;
    w[0][0] = __byte_perm(x, z, 0x5410) ^ sign; w[0][1] = __byte_perm(x, z, 0x7632) ^ sign;
    w[0][2] = __byte_perm(y, u, 0x5410) ^ sign; w[0][3] = __byte_perm(y, u, 0x7632) ^ sign;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[0][i] = bits2(__hmul2(bf2(w[0][i]), bf2(i & 1 ? up60 : up64)));
}
__device__ __forceinline__ void query_parts(uint32_t (&w)[2][4], float by) {           // in: eight fp32 numbers
#pragma unroll
    for (int i = 0; i < 4; ++i) two_parts(__uint_as_float(w[0][i]) * by, __uint_as_float(w[1][i]) * by, w[0][i], w[1][i]);
}

template <typename T, int HD>
__global__ void __launch_bounds__(AtShape<T, HD>::warps * 32, 1) kv_attend_kernel(const AttendArgs a) {
    using S = AtShape<T, HD>;
    constexpr int G = HD / 32, COLS = S::cols, W = S::warps, STAGES = S::stages, BB = kv_block_bytes(HD);
    constexpr bool RAW = S::raw;
    constexpr int QP = sizeof(T) / 2;                          // parts of a query
    extern __shared__ __align__(128) unsigned char smem[];
    // pieces of a line go round the SM's four schedulers a quarter of the warps apart, so that a CTA of a few tiles uses all four
    const int tid = threadIdx.x, lane = tid & 31, place = tid >> 5, warp = (place & 3) * (W / 4) + (place >> 2), r = lane >> 2, c = lane & 3;
    unsigned char* ring = smem + warp * S::ring_bytes;
    float* own_part = reinterpret_cast<float*>(smem + W * S::ring_bytes + warp * S::part_bytes);
    unsigned char* rest = smem + W * (S::ring_bytes + S::part_bytes);
    const uint32_t bars = smem_u32(rest) + warp * STAGES * 8;
    long long* before = reinterpret_cast<long long*>(rest + W * STAGES * 8);      // tiles before each sequence, where there are many of these
    __shared__ PartMeta meta[2 * W];
    __shared__ Walk<COLS> copied[W], used[W];      // the items that a warp's copies and its sums are at
    __shared__ float4 starts[RAW ? W : 1][G][4];   // -8 times the sum of a group's queries, as the product's C for columns 2 c, 2 c + 1
    __shared__ long long warp_sum_of[W];

    if (lane == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(bars + 8 * i, 1 + a.withhold);
        fence_barrier_init();
        meta[2 * warp].id = meta[2 * warp + 1].id = -1;
    }
    __syncwarp();
    grid_dep_wait();
    grid_dep_launch();
    // ---- the line of tiles: how many there are, and before each sequence. Up to 64 sequences are two a lane, in every warp for itself ----
    const int n_seq = a.batch.n_seq;
    long long all = 0, before0 = 0, before1 = 0;
    int len0 = 0, len1 = 0, n0 = 0, n1 = 0, first0 = 0, first1 = 0;
    auto loaded = [&](int s) {
        Walk<COLS> w;
        w.seq = s; w.n = 0; w.first = 0; w.len = 0;
        if (s < n_seq) w.load(a);
        return w;
    };
    auto count_tiles = [&](Walk<COLS> w) {
        if (w.n > 0 && w.len > a.batch.stride * a.kv.page_size && blockIdx.x == 0) kv_note(a.kv, SPM_KV_TOO_LONG);
        return w.blocks(a) <= kAtFewBlocks ? w.tiles_of_sequence(a, 0, 1) : -1ll;
    };
    // sequences of many column blocks: their lanes' counts come back as -1, and the warp counts together
    auto count_many = [&](long long k, int s) {
        for (uint32_t left = __ballot_sync(0xffffffffu, k < 0); left; left &= left - 1) {
            const int owner = __ffs(left) - 1;
            Walk<COLS> w;
            w.seq = __shfl_sync(0xffffffffu, s, owner);
            w.load(a);
            long long sum = w.tiles_of_sequence(a, lane, 32);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == owner) k = sum;
        }
        return k;
    };
    if (n_seq <= 64) {
        const Walk<COLS> w0 = loaded(2 * lane), w1 = loaded(2 * lane + 1);
        const long long k0 = count_many(count_tiles(w0), 2 * lane), k1 = count_many(count_tiles(w1), 2 * lane + 1);
        len0 = w0.len; len1 = w1.len; n0 = w0.n; n1 = w1.n; first0 = w0.first; first1 = w1.first;
        long long upto = k0 + k1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        all = __shfl_sync(0xffffffffu, upto, 31);
        before0 = upto - k0 - k1;
        before1 = upto - k1;
    } else {
        const int each = (n_seq + W * 32 - 1) / (W * 32);
        long long mine = 0;
        for (int i = 0; i < each; ++i) {
            const int s = tid * each + i;
            const long long k = count_many(count_tiles(loaded(s)), s);
            if (s < n_seq) before[s] = mine;
            mine += k;
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warp_sum_of[place] = upto;
        __syncthreads();
        long long off = upto - mine;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < place) off += warp_sum_of[w];
            all += warp_sum_of[w];
        }
        for (int i = 0; i < each; ++i)
            if (tid * each + i < n_seq) before[tid * each + i] += off;
        __syncthreads();
    }

    const bool full = all >= static_cast<long long>(gridDim.x) * kAtMinTiles;
    const int ctas = full ? int(gridDim.x) : max(1, (int(all) + kAtMinTiles - 1) / kAtMinTiles), cta = blockIdx.x;
    const long long cta_lo = cta < ctas ? all * cta / ctas : all, cta_hi = cta < ctas ? all * (cta + 1) / ctas : all;
    const long long lo = cta_lo + (cta_hi - cta_lo) * warp / W;
    const int count = int(cta_lo + (cta_hi - cta_lo) * (warp + 1) / W - lo);

    float m[2], l[2], y[G][2][4];
    uint32_t wide[G / 2];                        // (bf16) a power of two per group that no value's scale so far is above, as fp16, as far as these go
    uint32_t qf[QP][G][4];
    if (count > 0) {
        {
            Walk<COLS> at;
            if (n_seq <= 64) {
                const int s = __popc(__ballot_sync(0xffffffffu, 2 * lane < n_seq && before0 <= lo)) +
                              __popc(__ballot_sync(0xffffffffu, 2 * lane + 1 < n_seq && before1 <= lo)) - 1;
                const long long b0 = __shfl_sync(0xffffffffu, before0, s / 2), b1 = __shfl_sync(0xffffffffu, before1, s / 2);
                auto of = [&](int x0, int x1) { return __shfl_sync(0xffffffffu, s & 1 ? x1 : x0, s / 2); };
                at.seq = s; at.len = of(len0, len1); at.n = of(n0, n1); at.first = of(first0, first1);
                at.seek(a, lo - (s & 1 ? b1 : b0));
            } else {
                int s = 0, end = n_seq;          // the last sequence with before[s] <= lo
                while (end - s > 1) {
                    const int mid = (s + end) / 2;
                    if (before[mid] <= lo) s = mid; else end = mid;
                }
                at.seq = s;
                at.load(a);
                at.seek(a, lo - before[s]);
            }
            if (lane == 0) copied[warp] = used[warp] = at;
            __syncwarp();
        }
        const Walk<COLS>& use = used[warp];
        int t = use.t, left_there = use.nt - t;     // tile of its item, tiles left there
        // an item's queries, as they are in memory
        auto fetch = [&] {
            int g;
            const int row = row_of_column<COLS>(a, use.first, use.n, use.ct, r, g);
            const T* p = static_cast<const T*>(a.q.p) + row * a.q.row + (use.head * a.group + g) * a.q.head + 8 * c;
#pragma unroll
            for (int k = 0; k < G; ++k)
#pragma unroll
                for (int q = 0; q < QP; ++q) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (row >= 0) v = *reinterpret_cast<const uint4*>(p + 32 * k + 4 * q);
                    qf[q][k][0] = v.x; qf[q][k][1] = v.y; qf[q][k][2] = v.z; qf[q][k][3] = v.w;
                }
        };
        fetch();
        // ---- copies: lanes 0 and 1 walk ahead and look up a block's page each, a tile before its use. A page of an even number of
        // blocks holds both ----
        const int per_page = a.kv.page_size / kKvBlock;
        const bool even = per_page % 2 == 0;
        const long long page_bytes = static_cast<long long>(a.kv.heads) * per_page * BB;
        const uint32_t ring_at = smem_u32(ring);
        uint32_t present = 0;                    // two bits a stage: which blocks are there
        int issued = 0, page = -1, in_page = 0;
        int to_t, to_left, to_nk, to_head;
        const int* to_table;
        auto copies_at = [&](const Walk<COLS>& w) {
            to_t = w.t; to_left = w.nt - w.t; to_nk = w.nk; to_head = w.head * per_page;
            to_table = a.batch.table + size_t(w.seq) * a.batch.stride;
        };
        auto look_up = [&] {
            const int block = to_t * 2 + lane;
            const int slot = a.page_shift >= 0 ? block >> a.page_shift : block / per_page;
            in_page = to_head + block - slot * per_page;
            page = block * kKvBlock < to_nk ? to_table[slot] : -2;       // -2: not wanted
        };
        auto issue = [&](int stage) {
            uint32_t have = 0;
            if (lane < 2) {
                const bool ok = page >= 0 && page < a.kv.n_pages;
                if (!ok && page != -2) kv_note(a.kv, SPM_KV_BAD_PAGE);
                const unsigned char* from = a.kv.pages + (page * page_bytes + static_cast<long long>(in_page) * BB);
                have = __ballot_sync(3u, ok);
                const uint32_t bar = bars + 8 * stage, dst = ring_at + stage * S::tile_bytes, bytes = __popc(have) * BB;
                if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
                __syncwarp(3u);
                if (ok && (lane == 0 || !even)) {        // (what nobody reads again leaves tables, queries and code in L2)
                    if (a.once) bulk_g2s(dst + lane * BB, from, even ? bytes : BB, bar, policy_evict_first());
                    else bulk_g2s_plain(dst + lane * BB, from, even ? bytes : BB, bar);
                }
                if (issued + 1 < count) {
                    ++to_t;
                    if (--to_left == 0) {
                        Walk<COLS> w = copied[warp];
                        w.t = w.nt - 1;
                        w.next(a);
                        __syncwarp(3u);
                        if (lane == 0) copied[warp] = w;
                        __syncwarp(3u);
                        copies_at(w);
                    }
                    look_up();
                }
            }
            ++issued;
            present = (present & ~(3u << (2 * stage))) | __shfl_sync(0xffffffffu, have, 0) << (2 * stage);
        };
        copies_at(use);
        if (lane < 2) look_up();
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
            if (i < count) issue(i);
        // scores are kept as the products give them; f > 0 takes them to powers of two (a negative scale turns the queries' signs, and
        // with a scale of 0 a masked score still counts as one)
        float f[2], slack[2];                    // of columns 2 c, 2 c + 1
        const bool flip = a.scale < 0.f;
        int whole_tiles = 0;
        int began = 0;                           // the item's tile with which this warp's part of it begins
        auto begin = [&] {
            uint32_t tops[4] = {};               // a column's largest query element, of which the exponent counts
#pragma unroll
            for (int k = 0; k < G; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (RAW) tops[j] = __vmaxu2(tops[j], qf[0][k][j] & 0x7fff7fffu);
                    else tops[j] = max(tops[j], max(qf[0][k][j] & 0x7fffffffu, qf[1][k][j] & 0x7fffffffu));
                }
            uint32_t top = RAW ? __vmaxu2(__vmaxu2(tops[0], tops[1]), __vmaxu2(tops[2], tops[3])) : max(max(tops[0], tops[1]), max(tops[2], tops[3]));
            top = RAW ? max(top & 0xffffu, top >> 16) >> 7 : top >> 23;
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = top == 0 ? -126 : top == 255 ? 0 : int(top) - 127;
            const int up = RAW ? -e : min(126, 14 - e);          // fp32 columns go to [2^14, 2^15)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float down = __int_as_float((127 - __shfl_sync(0xffffffffu, up, (2 * c + i) * 4)) << 23);
                f[i] = fminf(fmaxf(fabsf(a.scale) * 1.4426950408889634f * down * (RAW ? kAtUp69 : 1.f), kAtLeast), RAW ? kAtMost * 0x1p40f : kAtMost);
                slack[i] = __fdividef(6.f, f[i]);
            }
            const bool tiny = RAW && e < -60;    // 2^(64 - e) is no number then: in two steps
            if (__any_sync(0xffffffffu, tiny))
#pragma unroll
                for (int k = 0; k < G; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) qf[0][k][j] = bits2(__hmul2(bf2(qf[0][k][j]), bf2(bf16_power(tiny ? 100 : 0))));
            const uint32_t up64 = RAW ? bf16_power(64 - (tiny ? e + 100 : e)) : 0, up60 = up64 - 0x02000200u;      // 2^-4 of it
#pragma unroll
            for (int k = 0; k < G; ++k) {
                uint32_t w[QP][4];
#pragma unroll
                for (int q = 0; q < QP; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[q][j] = qf[q][k][j];
                if constexpr (RAW) query_words(w, up64, up60, flip);
                else query_parts(w, __int_as_float((127 + up) << 23 | (flip ? int(0x80000000u) : 0)));
#pragma unroll
                for (int q = 0; q < QP; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) qf[q][k][j] = w[q][j];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[k][0][j] = y[k][1][j] = 0.f;
                if constexpr (RAW) {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x0, x1;
                        two_bf16(w[0][j], x0, x1);
                        sum += (x0 + x1) * (j & 1 ? 16.f : 1.f);
                    }
                    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                    sum *= -8.f * 0x1p-133f;       // to where a code's 1 stands
                    if (c == 0) {
                        float* to = reinterpret_cast<float*>(&starts[warp][k][r / 2]) + r % 2;
                        to[0] = to[2] = sum;
                    }
                }
            }
            m[0] = m[1] = -INFINITY;
            l[0] = l[1] = 0.f;
#pragma unroll
            for (int k = 0; k < G / 2; ++k) wide[k] = kAtNarrowest;
            if constexpr (RAW) __syncwarp();
            began = t;
            whole_tiles = min(use.nk, use.len - use.n + column_row(a, use.ct * COLS) + 1) / kAtTile;
        };
        begin();
        int stage = 0;
        uint32_t phase = 0;
        for (int i = 0; i < count; ++i) {
            if (!__all_sync(0xffffffffu, mbar_wait_bounded(bars + 8 * stage, phase, a.wait_ns))) {       // give up, but not with copies in flight
                if (lane == 0) kv_note(a.kv, SPM_KV_TIMEOUT);
                for (int j = i; j < issued; ++j) mbar_wait_bounded(bars + 8 * (j % STAGES), j / STAGES & 1, a.wait_ns);
                break;
            }
            const uint32_t at = ring_at + stage * S::tile_bytes, have = present >> (2 * stage) & 3;
            // ---- scores: tokens r, r + 8 of each block for columns 2 c, 2 c + 1 ----
            float s[2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t block = at + b * BB;
                float s0[G], s1[G];
                token_scales<G>(block + kv_k_scales(HD) + r * (2 * G), s0);
                token_scales<G>(block + kv_k_scales(HD) + (r + 8) * (2 * G), s1);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[b][j] = 0.f;
#pragma unroll
                for (int k = 0; k < G; k += 2) {
                    const uint4 w = ldsm4(block + (k + (lane >> 4)) * (kKvBlock * 16) + (lane & 15) * 16);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t low = h ? w.z : w.x, high = h ? w.w : w.y;
                        const Nib4 u = RAW ? q4_unpack(low) : q4_halves(low), v = RAW ? q4_unpack(high) : q4_halves(high);
                        float d[4];
                        if constexpr (RAW) {
                            mma_k16_from(d, starts[warp][k + h][c], u.p[0], v.p[0], u.p[1], v.p[1], qf[0][k + h][0], qf[0][k + h][1]);
                            mma_k16(d, u.p[2], v.p[2], u.p[3], v.p[3], qf[0][k + h][2], qf[0][k + h][3]);
                        } else {
                            mma_half_first(d, u.p[0], v.p[0], u.p[1], v.p[1], qf[1][k + h][0], qf[1][k + h][1]);
                            mma_half_k16(d, u.p[2], v.p[2], u.p[3], v.p[3], qf[1][k + h][2], qf[1][k + h][3]);
                            mma_half_k16(d, u.p[0], v.p[0], u.p[1], v.p[1], qf[0][k + h][0], qf[0][k + h][1]);
                            mma_half_k16(d, u.p[2], v.p[2], u.p[3], v.p[3], qf[0][k + h][2], qf[0][k + h][3]);
                        }
                        s[b][0] += s0[k + h] * d[0]; s[b][1] += s0[k + h] * d[1];
                        s[b][2] += s1[k + h] * d[2]; s[b][3] += s1[k + h] * d[3];
                    }
                }
            }
            // ---- tokens that are not there, or behind a column's row ----
            const bool whole = have == 3 && t < whole_tiles;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i2 = column_row(a, use.ct * COLS + 2 * c + e);
                    const int sees = min(use.nk, use.len - use.n + i2 + 1) - t * kAtTile;      // tokens of this tile
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (!(have >> b & 1) || 16 * b + 8 * j + r >= sees) s[b][2 * j + e] = -INFINITY;
                }
            }
            // ---- running maximum: moved only where a score is above it by a factor of 2^6 ----
            bool raise = false;
            float top[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v = fmaxf(fmaxf(s[0][e], s[0][2 + e]), fmaxf(s[1][e], s[1][2 + e]));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
                top[e] = v;
                raise |= v - m[e] > slack[e];         // (two of -infinity leave NaN, which is not above)
            }
            // ---- the values' scales, and whether one is above its group's power of two (what has never been written may be anything) ----
            uint32_t vs[2][2][G / 2], widest[G / 2];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    scale_words<G>(at + b * BB + kv_v_scales(HD) + (8 * j + r) * (2 * G), vs[b][j]);
                    if (!whole && (!(have >> b & 1) || t * kAtTile + 16 * b + 8 * j + r >= use.nk))
#pragma unroll
                        for (int k = 0; k < G / 2; ++k) vs[b][j][k] = 0;
                }
#pragma unroll
            for (int k = 0; k < G / 2; ++k) {
                auto of = [&](int b, int j) { return __habs2(as_half2(vs[b][j][k])); };
                widest[k] = bits_of(__hmax2(__hmax2(__hmax2(of(0, 0), of(0, 1)), __hmax2(of(1, 0), of(1, 1))), as_half2(wide[k])));
                raise |= widest[k] != wide[k];
            }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int k = 0; k < G / 2; ++k) {
                    uint32_t w = widest[k];
                    w = __vmaxu2(w, __shfl_xor_sync(0xffffffffu, w, 4));
                    w = __vmaxu2(w, __shfl_xor_sync(0xffffffffu, w, 8));
                    w = __vmaxu2(w, __shfl_xor_sync(0xffffffffu, w, 16));
                    w = __vminu2(w, kAtWidest) + 0x03ff03ffu & 0x7c007c00u;
                    const float2 was = __half22float2(as_half2(wide[k])), is = __half22float2(as_half2(w));
                    const float by0 = was.x / is.x, by1 = was.y / is.y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        y[2 * k][0][j] *= by0; y[2 * k][1][j] *= by0;
                        y[2 * k + 1][0][j] *= by1; y[2 * k + 1][1][j] *= by1;
                    }
                    wide[k] = w;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float to = fmaxf(m[e], top[e]), by = to == -INFINITY ? 1.f : ex2((m[e] - to) * f[e]);
                    m[e] = to;
                    l[e] *= by;
#pragma unroll
                    for (int k = 0; k < G; ++k) { y[k][0][e] *= by; y[k][0][2 + e] *= by; y[k][1][e] *= by; y[k][1][2 + e] *= by; }
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // (the difference first: of large scores times f the maximum's rounding alone is more than the range of fp16's exponents)
                const float base = m[e] == -INFINITY ? 0.f : m[e];
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float p = ex2(fmaf(s[b][2 * j + e] - base, f[e], S::up));
                        s[b][2 * j + e] = p;
                        l[e] += p;
                    }
            }
            // ---- y += V^T p, the values' scales on p ----
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t block = at + b * BB;
                if constexpr (RAW) {
                    const __half2 p0 = as_half2(pack_half(s[b][0], s[b][1])), p1 = as_half2(pack_half(s[b][2], s[b][3]));
#pragma unroll
                    for (int k = 0; k < G; k += 2) {
                        const uint4 w = ldsm4t(block + kv_v_codes(HD) + (k + (lane >> 4)) * (kKvBlock * 16) + (lane & 15) * 16);
                        const __half2 down = as_half2(0x7c007c00u - wide[k / 2]);          // 2 / wide
                        const __half2 s0 = __hmul2(as_half2(vs[b][0][k / 2]), down), s1 = __hmul2(as_half2(vs[b][1][k / 2]), down);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const Nib4 u = q4_bytes(h ? w.z : w.x), v = q4_bytes(h ? w.w : w.y);
                            const uint32_t b0 = transpose8(bits_of(__hmul2(p0, h ? __high2half2(s0) : __low2half2(s0))));
                            const uint32_t b1 = transpose8(bits_of(__hmul2(p1, h ? __high2half2(s1) : __low2half2(s1))));
                            mma_half_k16(y[k + h][0], kAtMinus8, kAtMinus136, kAtMinus8, kAtMinus136, b0, b1);
                            mma_half_k16(y[k + h][1], kAtMinus8, kAtMinus136, kAtMinus8, kAtMinus136, b0, b1);
                            mma_half_k16(y[k + h][0], u.p[0], u.p[1], v.p[0], v.p[1], b0, b1);
                            mma_half_k16(y[k + h][1], u.p[2], u.p[3], v.p[2], v.p[3], b0, b1);
                        }
                    }
                } else {
                    float s0[G], s1[G];
#pragma unroll
                    for (int k = 0; k < G / 2; ++k) {
                        const float2 down = __half22float2(as_half2(0x7c007c00u - wide[k]));     // 2 / wide
                        const float2 f0 = __half22float2(as_half2(vs[b][0][k])), f1 = __half22float2(as_half2(vs[b][1][k]));
                        s0[2 * k] = f0.x * down.x; s0[2 * k + 1] = f0.y * down.y; s1[2 * k] = f1.x * down.x; s1[2 * k + 1] = f1.y * down.y;
                    }
#pragma unroll
                    for (int k = 0; k < G; k += 2) {
                        const uint4 w = ldsm4t(block + kv_v_codes(HD) + (k + (lane >> 4)) * (kKvBlock * 16) + (lane & 15) * 16);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const Nib4 u = q4_halves(h ? w.z : w.x), v = q4_halves(h ? w.w : w.y);
                            uint32_t b0, b1, low0, low1;
                            two_parts(s[b][0] * s0[k + h], s[b][1] * s0[k + h], b0, low0);
                            two_parts(s[b][2] * s1[k + h], s[b][3] * s1[k + h], b1, low1);
                            b0 = transpose8(b0); b1 = transpose8(b1); low0 = transpose8(low0); low1 = transpose8(low1);
                            float d[2][4];
                            mma_half_first(d[0], u.p[0], u.p[1], v.p[0], v.p[1], low0, low1);
                            mma_half_first(d[1], u.p[2], u.p[3], v.p[2], v.p[3], low0, low1);
                            mma_half_k16(d[0], u.p[0], u.p[1], v.p[0], v.p[1], b0, b1);
                            mma_half_k16(d[1], u.p[2], u.p[3], v.p[2], v.p[3], b0, b1);
#pragma unroll
                            for (int j = 0; j < 4; ++j) { y[k + h][0][j] += d[0][j]; y[k + h][1][j] += d[1][j]; }
                        }
                    }
                }
            }
            __syncwarp();
            if (i + STAGES < count) issue(stage);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }

            // ---- the item ends, or the warp's piece ----
            const bool ends = left_there == 1;
            if (ends || i + 1 == count) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float v = l[e];
                    v += __shfl_xor_sync(0xffffffffu, v, 4);
                    v += __shfl_xor_sync(0xffffffffu, v, 8);
                    v += __shfl_xor_sync(0xffffffffu, v, 16);
                    l[e] = v;
                }
#pragma unroll
                for (int k = 0; k < G / 2; ++k) {
                    const float2 by = __half22float2(as_half2(wide[k]));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        y[2 * k][0][j] *= by.x; y[2 * k][1][j] *= by.x;
                        y[2 * k + 1][0][j] *= by.y; y[2 * k + 1][1][j] *= by.y;
                    }
                }
                if (ends && began == 0) {        // all of it is this warp's
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        int g;
                        const int row = row_of_column<COLS>(a, use.first, use.n, use.ct, 2 * c + e, g);
                        if (row < 0) continue;
                        const float by = l[e] > 0.f ? S::unscale / l[e] : 0.f;
                        T* p = static_cast<T*>(a.out.p) + row * a.out.row + (use.head * a.group + g) * a.out.head + 4 * r;
#pragma unroll
                        for (int k = 0; k < G; ++k) {
                            float o[4] = {y[k][0][e] * by, S::odd(y[k][0][2 + e], y[k][0][e]) * by,
                                          y[k][1][e] * by, S::odd(y[k][1][2 + e], y[k][1][e]) * by};
                            store_row<4>(p + 32 * k, o);
                        }
                    }
                } else {
                    // an item that ends here began in another warp: the warp's first part. One that goes on is its last part, and the ring is free
                    float* part = ends ? own_part : reinterpret_cast<float*>(ring);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int col = 2 * c + e;
#pragma unroll
                        for (int k = 0; k < G; ++k)
                            *reinterpret_cast<float4*>(part + col * HD + 32 * k + 4 * r) =
                                make_float4(y[k][0][e], S::odd(y[k][0][2 + e], y[k][0][e]), y[k][1][e], S::odd(y[k][1][2 + e], y[k][1][e]));
                        if (r == 0) { part[COLS * HD + col] = m[e] == -INFINITY ? -INFINITY : m[e] * f[e]; part[COLS * HD + COLS + col] = l[e]; }
                    }
                    if (lane == 0) meta[2 * warp + !ends] = PartMeta{lo + i - t, use.ct, use.head, began, t + 1, use.nt, use.first, use.n};
                }
            }
            ++t;
            if (--left_there == 0 && i + 1 < count) {
                Walk<COLS> w = use;
                w.t = w.nt - 1;
                w.next(a);
                __syncwarp();
                if (lane == 0) used[warp] = w;
                __syncwarp();
                t = 0;
                left_there = w.nt;
                fetch();
                begin();
            }
        }
    }
    __syncthreads();

    // ---- parts of one item in this CTA meet: they stand one after another, and every warp sees which belong together (lane j: part j).
    // A warp takes a column of an item, whatever the number of items: the parts' weights, a lane each, then their sums ----
    const long long id = lane < 2 * W ? meta[lane].id : -1;
    const uint32_t mates = __match_any_sync(0xffffffffu, id);
    const bool leads = id >= 0 && (mates & ((1u << lane) - 1)) == 0;
    const uint32_t leaders = __ballot_sync(0xffffffffu, leads);
    const int rank = __popc(leaders & ((1u << lane) - 1)), columns = __popc(leaders) * COLS;
    auto part_of = [&](int j) {
        return reinterpret_cast<const float*>(j & 1 ? smem + (j >> 1) * S::ring_bytes : smem + W * S::ring_bytes + (j >> 1) * S::part_bytes);
    };
    if (warp == 0) {                             // an item that begins here and goes on: up to the CTA of its last tile
        const PartMeta first = meta[leads ? lane : 0];
        const bool open = leads && first.from == 0 && meta[leads ? 31 - __clz(mates) : 0].to < first.nt;
        const uint32_t any = __ballot_sync(0xffffffffu, open);
        if (open || (any == 0 && lane == 0)) {
            int4 join = make_int4(0, 0, 0, 0);
            if (open) join = make_int4(int(((first.id + first.nt) * ctas - 1) / all) - cta + 1, first.ct, first.head, first.first);
            *reinterpret_cast<int4*>(a.joins + 8 * cta) = join;
            a.joins[8 * cta + 4] = open ? first.n : 0;
        }
    }
    for (int x = warp; x < columns; x += W) {
        const int col = x % COLS;
        const int at = __ffs(__ballot_sync(0xffffffffu, leads && rank == x / COLS)) - 1;
        const uint32_t group = __shfl_sync(0xffffffffu, mates, at);
        const PartMeta& first = meta[at];
        const bool in = group >> lane & 1;
        const float v = in ? part_of(lane)[COLS * HD + col] : -INFINITY;
        float top = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float weight = top == -INFINITY ? 0.f : ex2(v - top);
        const float total = warp_sum(in ? weight * part_of(lane)[COLS * HD + COLS + col] : 0.f);
        constexpr int N = HD / 32 < 4 ? HD / 32 : 4, RUNS = HD / (32 * N);       // N numbers side by side
        float o[RUNS][N] = {};
        for (uint32_t left = group; left;) {     // four parts' loads at a time
            float y4[4][RUNS][N], by[4];
            bool one[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                one[i] = left != 0;
                const int j = one[i] ? __ffs(left) - 1 : at;
                left &= left - 1;
                by[i] = __shfl_sync(0xffffffffu, weight, j);
                const float* part = part_of(j) + col * HD + lane * N;
#pragma unroll
                for (int k = 0; k < RUNS; ++k)
                    if constexpr (N == 4) {
                        const float4 f = *reinterpret_cast<const float4*>(part + k * 128);
                        y4[i][k][0] = f.x; y4[i][k][1] = f.y; y4[i][k][2] = f.z; y4[i][k][3] = f.w;
                    } else {
                        const float2 f = *reinterpret_cast<const float2*>(part);
                        y4[i][k][0] = f.x; y4[i][k][1] = f.y;
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (one[i])
#pragma unroll
                    for (int k = 0; k < RUNS; ++k)
#pragma unroll
                        for (int e = 0; e < N; ++e) o[k][e] += by[i] * y4[i][k][e];
        }
        if (first.from == 0 && meta[31 - __clz(group)].to == first.nt) {
            int g;
            const int row = row_of_column<COLS>(a, first.first, first.n, first.ct, col, g);
            const float by = total > 0.f ? S::unscale / total : 0.f;
            if (row < 0) continue;
            T* to = static_cast<T*>(a.out.p) + row * a.out.row + (first.head * a.group + g) * a.out.head + lane * N;
#pragma unroll
            for (int k = 0; k < RUNS; ++k) {
#pragma unroll
                for (int e = 0; e < N; ++e) o[k][e] *= by;
                store_row<N>(to + k * 128, o[k]);
            }
        } else {                                 // slot 0: an item that began before this CTA
            float* to = a.parts + (size_t(cta) * 2 + (first.from == 0)) * S::part_floats;
#pragma unroll
            for (int k = 0; k < RUNS; ++k)
#pragma unroll
                for (int e = 0; e < N; e += 2) *reinterpret_cast<float2*>(to + col * HD + k * 128 + lane * N + e) = make_float2(o[k][e], o[k][e + 1]);
            // (a part whose scores are NaN is not to be taken for one that sees nothing: its maximum is above all, and the item becomes NaN)
            if (lane == 0) { to[COLS * HD + col] = total == total ? top : INFINITY; to[COLS * HD + COLS + col] = total; }
        }
    }
}

// Adds the parts of items that were cut between CTAs: block (x, column) takes the item that begins in CTA x and goes on behind it. Its
// 256 threads take the parts in turn by HD-wide groups, eight parts at a time with their loads ahead of their use.
constexpr int kAtJoinThreads = 256;
template <typename T, int HD>
__global__ void __launch_bounds__(kAtJoinThreads) kv_attend_join_kernel(const AttendArgs a) {
    using S = AtShape<T, HD>;
    constexpr int COLS = S::cols, FLOATS = S::part_floats, SETS = kAtJoinThreads / HD;
    __shared__ float tops[SETS], sums[SETS], rows[SETS][HD];
    grid_dep_wait();
    grid_dep_launch();
    const int cta = blockIdx.x, col = blockIdx.y, d = threadIdx.x % HD, set = threadIdx.x / HD;
    const int4 join = *reinterpret_cast<const int4*>(a.joins + 8 * cta);
    const int n = a.joins[8 * cta + 4];
    if (join.x == 0) return;
    int g;
    const int row = row_of_column<COLS>(a, join.w, n, join.y, col, g);
    if (row < 0) return;
    // part 0 is the second slot of its CTA, the others are the first slots of theirs
    const float* part = a.parts + size_t(cta) * 2 * FLOATS;
    float top = -INFINITY, sum = 0.f, o = 0.f;
    for (int j0 = set; j0 < join.x; j0 += 8 * SETS) {
        float m[8], l[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + i * SETS;
            const float* p = part + size_t(j == 0 ? 1 : 2 * j) * FLOATS;
            m[i] = j < join.x ? p[COLS * HD + col] : -INFINITY;
            l[i] = j < join.x ? p[COLS * HD + COLS + col] : 0.f;
            y[i] = j < join.x ? p[col * HD + d] : 0.f;
        }
        float to = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) to = fmaxf(to, m[i]);
        if (to == -INFINITY) continue;
        const float keep = ex2(top - to);
        sum *= keep; o *= keep; top = to;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float by = ex2(m[i] - to);
            sum += by * l[i]; o += by * y[i];
        }
    }
    if constexpr (SETS > 1) {
        rows[set][d] = o;
        if (d == 0) { tops[set] = top; sums[set] = sum; }
        __syncthreads();
        if (set > 0) return;
        float to = top;
#pragma unroll
        for (int i = 1; i < SETS; ++i) to = fmaxf(to, tops[i]);
        o = sum = 0.f;
        if (to > -INFINITY)
#pragma unroll
            for (int i = 0; i < SETS; ++i) {
                const float by = ex2(tops[i] - to);
                sum += by * sums[i]; o += by * rows[i][d];
            }
    }
    o = sum == 0.f ? 0.f : o * (S::unscale / sum);
    T* to = static_cast<T*>(a.out.p) + row * a.out.row + (join.z * a.group + g) * a.out.head + d;
    if constexpr (sizeof(T) == 2) *to = __float2bfloat16_rn(o);
    else *to = o;
}

}  // namespace spm
