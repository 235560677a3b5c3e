// Attention of new rows over latent rows, which are keys and values of all heads at once (the absorbed form), on tcgen05.
//
// A column is a head of a new row: column x of a sequence is head x % heads of row x / heads. A CTA takes COLS columns and walks their
// tokens 64 at a time. Both products have the cache's rows as their A operand, where they lie, and columns as N, so that few columns cost
// few cycles: scores S^T [tokens][columns] = C q^T, the rows K-major, and sums O^T [latent][columns] += C^T P^T, the same bytes M-major.
// S^T, in two buffers, and O^T, latent / 128 tiles, are in tensor memory. Every byte of a row comes to the SM once, for both.
//
// A warp brings tiles by TMA (64 elements of a page's rows a copy, swizzled) into a ring of as many stages as there is room for; one issues
// the products, of a tile's scores as soon as it has landed, of its sums as soon as its probabilities are there; four turn scores into
// probabilities, 16 tokens each, and write results. A probability is 2^(s - m), m not the running maximum but one that was it: it is moved
// only when a score is above it by more than 8, which it seldom is after a tile (P is bf16, which has fp32's range, and loses nothing above 1; sums of
// values up to 2^100 stay in fp32's range over 2^18 tokens of a CTA). So a tile needs no maximum over its tokens, only a vote that none is that far above.
//
// fp32 queries and probabilities are three bf16 parts each, cut off and not rounded: three columns side by side in one product, added up
// as scores and results are read. Their sums leave the products every kLaAside tiles, which cut sums off where they do not round them: with 63 tiles of
// one sign in them results were 1.1e-5 too small, now they are as near as plain fp32 ones. bf16 calls' probabilities are two such parts (results then differ
// from plain fp32 arithmetic's by their own rounding alone; 64 sequences 103 -> 107 us), but with 64 columns, whose second parts neither shared memory nor
// tensor memory has room for: one, of 8 bits (0.0020 of a result where its own rounding is 0.0017).
//
// All (sequence, columns) items together are a line of tiles that is cut evenly between CTAs, whatever the lengths are. An item's parts
// in several CTAs go to the workspace and latent_join_kernel adds them in order. (Items count with all of a sequence's tokens; columns that
// see fewer, as a prompt's do, leave their CTA idle for the others. Such calls are few: prompts have the expanded form.)
//
// What bounds it: DRAM, with 16 columns (64 sequences, 536 MB of rows of 512 + 64: 100.5 us, 5.4 TB/s); with 64, of whose queries beside shared memory
// has room for two tiles only, a tile's copy, scores, softmax and sums waiting for one another (3700 cycles a tile, 2300 of them products; 32 sequences, 145 MB,
// 128 heads: 80 us). A few tiles a CTA: the way to the first scores and from the last sums.
#pragma once

#include <type_traits>

#include <cuda.h>

#include "kv_cache.cuh"
#include "latent_cache.cuh"
#include "mma_ops.cuh"
#include "ptx.cuh"
#include "tc_ops.cuh"

namespace spm {

struct LatentAttendArgs {
    LatentPool kv;
    KvBatch batch;
    HeadRows q, out;
    int heads, heads_shift;     // x / heads is x * heads_times >> heads_shift for x below 2^31
    uint32_t heads_times;
    int chunks, stages;         // 64-element chunks of a row, tiles of the ring
    int box;                    // tokens of a copy: 16, 32 or 64, all of one page
    float factor;               // of scores: scale times log2(e)
    float* parts;               // [2 * CTAs][LaPart floats]
    int4* joins;                // [CTAs], of the item that begins in this CTA and goes on behind it: CTAs that share it (0: none), its
                                // sequence's first row and rows, block of columns
    unsigned long long wait_ns; // a wait in a kernel gives up after this long
    int withhold;               // (tests) arrivals that barriers wait for and nobody makes
};

// Row of column x
__device__ __forceinline__ int la_row(const LatentAttendArgs& a, int x) { return int(static_cast<unsigned long long>(uint32_t(x)) * a.heads_times >> a.heads_shift); }

constexpr int kLaTile = 64, kLaMaxCtas = 148, kLaMaxStages = 8, kLaThreads = 192;
constexpr int kLaChunkBytes = kLaTile * 128;
constexpr float kLaSlack = 8.f;
constexpr int kLaAside = 4;                      // tiles whose sums an fp32 call's products hold, the others' stand behind O

template <typename T, int COLS>
struct LaShape {
    static constexpr int parts = sizeof(T) == 4 ? 3 : 1;                             // of a query's number
    static constexpr int p_parts = sizeof(T) == 4 ? 3 : COLS <= 48 ? 2 : 1;          // of a probability (64 columns: shared memory has room for one)
    static constexpr int n = COLS * parts, n_o = COLS * p_parts;                     // N of the products
    static_assert(2 * n + 4 * n_o + (parts == 3 ? 4 * COLS : 0) <= 512 && n % 16 == 0, "O^T of 512 elements, two buffers of S^T, and sums aside fit tensor memory");
    static constexpr int q_bytes(int chunks) { return chunks * n * 128; }
    static constexpr int p_bytes = n_o * 128;
    static constexpr int fixed(int chunks) { return 1024 + q_bytes(chunks) + p_bytes; }
    static constexpr int part_floats(int latent) { return COLS * (latent + 2); }     // sums, then maxima, then sums of probabilities
};
constexpr int kLaOwnBytes = 2048;                            // LaShared below


__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int element, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(element), "r"(row), "r"(bar) : "memory");
}
// the same for rows that nobody else reads
__device__ __forceinline__ void tma_rows_once(uint32_t dst, const CUtensorMap* map, int element, int row, uint32_t bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
        ::"r"(dst), "l"(map), "r"(element), "r"(row), "r"(bar), "l"(policy) : "memory");
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        " .reg .pred p;\n"
        " mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// bf16 x bf16 -> fp32
__host__ __device__ constexpr uint32_t la_idesc(int m, int n, bool a_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(a_mn_major) << 15) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}
// D[tmem] (+)= A * B by the descriptors' words
template <bool MORE>
__device__ __forceinline__ void tc_mma_lo(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        ".reg .b64 x, y;\n\t"
        "mov.b64 x, {%1, %2};\n\t"
        "mov.b64 y, {%3, %4};\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %5, p;\n\t"
        "}\n"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "n"(int(MORE)) : "memory");
}
// 16 lanes, 16 columns, in the layout of mma.sync's accumulators: r[4 i + 2 h + e] is row lane / 4 + 8 h, column 8 i + 2 (lane % 4) + e
__device__ __forceinline__ void tmem_ld_frag(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : SPM_R8(r, 0) : "r"(at) : "memory");
}
// a word of two bf16 numbers, one of them not finite
__device__ __forceinline__ bool odd_word(uint32_t v) { return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u; }
// four 8 x 8 matrices, each stored by columns
__device__ __forceinline__ void st_matrix_trans(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A sequence's items on the line: blocks of columns, tiles of each (one at least, so that rows that see nothing are written too)
struct LaSequence { int first, n, len, cap_len, blocks, tiles; };
// An item counts so many tiles more than it has: what its queries and its result cost beside them. Kernel times in us with 1, this, twice this and four times:
// bf16, latent 512: 64 sequences of up to 16000 tokens, 16 heads 112, 108, 110, 112; 300 of up to 500 tokens 40, 39.5, 38, 40; 32 of up to 8190, 128 heads
// 97, 84, 87, 94; 64 of up to 500, 128 heads 45, 34, 32, 32; 8 of up to 8193, 5 rows of 16 heads 41, 36, 38, 39; 64 of up to 400, 4 rows of 16 heads 23.5, 27.7, 29,
// 31.5. fp32: 16 of up to 4099, 10 heads, latent 256 22, 16.7, 17, 17; 64 of up to 600, 20 heads, latent 384 31, 30, 25, 26; 64 of up to 4000, 16 heads 49, 47.3, 47, 51
template <int COLS> constexpr int kLaItemCost = 1 + COLS / 16;
struct LaShared {
    unsigned long long full[kLaMaxStages], empty[kLaMaxStages], s_full[2], p_full, q_full, drained;
    uint32_t tmem;
    int quit;                                                // a wait has run out: everybody leaves
    int ctas;                                                // that have a piece
    int seq, group, tile;                                    // where this CTA's piece of the line begins
    LaSequence first;                                        // that sequence
    long long left, all, at;                                 // its tiles, all tiles, its first one
    int absent[kLaMaxStages];                                // a tile's copies (`box` tokens each) that there are not
    int limit[2][64];                                        // tokens that a column sees; of one item and the next
};
static_assert(sizeof(LaShared) <= kLaOwnBytes, "what shared memory has beside the ring");

template <int COLS>
__device__ __forceinline__ LaSequence la_sequence(const LatentAttendArgs& a, int s) {
    LaSequence q;
    q.first = s;
    q.n = 1;
    if (a.batch.row_start) {
        q.first = a.batch.row_start[s];
        q.n = max(0, min(a.batch.row_start[s + 1] - q.first, a.batch.n_rows));
    }
    q.len = a.batch.lengths[s];
    q.cap_len = max(0, min(q.len, a.batch.stride * a.kv.page_size));
    q.blocks = (q.n * a.heads + COLS - 1) / COLS;
    q.tiles = max(1, (q.cap_len + kLaTile - 1) / kLaTile);
    return q;
}

// A CTA's walk over its items. [begin, end): its units of the item's cost; from: its first tile; tiles: how many of its tiles the item's
// columns see a token in.
template <int COLS>
struct LaWalk {
    static constexpr int kCost = kLaItemCost<COLS>;
    LaSequence s;
    int seq, group, begin, end, from, sees, tiles;
    long long left;
    __device__ __forceinline__ void start(const LatentAttendArgs& a, const LaShared& sh) {
        seq = sh.seq; group = sh.group; begin = sh.tile; left = sh.left;
        if (left > 0) { s = sh.first; piece(a); }
    }
    __device__ __forceinline__ void piece(const LatentAttendArgs& a) {
        end = int(min(static_cast<long long>(s.tiles + kCost), begin + left));
        from = max(0, begin - kCost);
        const int last = min(s.n - 1, la_row(a, (group + 1) * COLS - 1));
        sees = max(0, min(s.len - s.n + last + 1, s.cap_len));
        tiles = max(0, min(end - kCost, (sees + kLaTile - 1) / kLaTile) - from);
    }
    __device__ __forceinline__ bool begins() const { return begin == 0; }
    __device__ __forceinline__ bool ends() const { return end == s.tiles + kCost; }
    __device__ __forceinline__ void next(const LatentAttendArgs& a) {
        left -= end - begin;
        if (left <= 0) return;
        begin = 0;
        if (++group >= s.blocks) {
            group = 0;
            do {
                if (++seq >= a.batch.n_seq) { left = 0; return; }
                s = la_sequence<COLS>(a, seq);
            } while (s.n <= 0);
        }
        piece(a);
    }
};

template <typename T, int COLS>
__global__ void __launch_bounds__(kLaThreads, 1) latent_attend_kernel(const LatentAttendArgs a, const __grid_constant__ CUtensorMap rows_map) {
    using S = LaShape<T, COLS>;
    constexpr int N = S::n, NO = S::n_o, PARTS = S::parts, P_PARTS = S::p_parts, BLOCKS = COLS / 8;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    // (the kernel's own arrays first: they take the room that aligning the rest would)
    LaShared& sh = *reinterpret_cast<LaShared*>(raw_smem);
    const uint32_t base = (smem_u32(raw_smem) + kLaOwnBytes + 1023) & ~1023u;
    const int chunks = a.chunks, stages = a.stages, latent = a.kv.latent;
    const uint32_t stage_bytes = chunks * kLaChunkBytes, q_at = base + stages * stage_bytes, p_at = q_at + S::q_bytes(chunks);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 128 && a.kv.n_pages > 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&rows_map) : "memory");
    grid_dep_wait();
    grid_dep_launch();
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) { mbar_init(smem_u32(&sh.full[i]), 1 + a.withhold); mbar_init(smem_u32(&sh.empty[i]), 1); }
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sh.s_full[i]), 1);
        mbar_init(smem_u32(&sh.p_full), 128);
        mbar_init(smem_u32(&sh.q_full), 128);
        mbar_init(smem_u32(&sh.drained), 1);
        sh.quit = 0;
        fence_barrier_init();
    }
    if (warp == 5) tmem_alloc(smem_u32(&sh.tmem), 512);
    if (warp == 4) {
        // ---- this CTA's piece of the line: a lane counts sequences side by side ----
        const int each = (a.batch.n_seq + 31) / 32, s0 = lane * each, s1 = min(s0 + each, a.batch.n_seq);
        long long mine = 0;
        LaSequence q{};                          // (up to 32 sequences: loaded once)
        for (int s = s0; s < s1; ++s) {
            q = la_sequence<COLS>(a, s);
            mine += static_cast<long long>(q.blocks) * (q.tiles + kLaItemCost<COLS>);
            if (q.n > 0 && q.len > q.cap_len && blockIdx.x == 0) kv_note(a.kv, SPM_KV_TOO_LONG);
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const long long all = __shfl_sync(0xffffffffu, upto, 31);
        // (no more CTAs than tiles: those that share an item are neighbours)
        const long long ctas = max(1ll, min(all, static_cast<long long>(gridDim.x))), cta = min(static_cast<long long>(blockIdx.x), ctas);
        const bool narrow = all < 1 << 24;       // (divisions of 64 bits are slow)
        const long long at = narrow ? uint32_t(all * cta) / uint32_t(ctas) : all * cta / ctas;
        const long long end = cta == ctas ? at : narrow ? uint32_t(all * (cta + 1)) / uint32_t(ctas) : all * (cta + 1) / ctas;
        if (lane == 0) { sh.left = end - at; sh.all = all; sh.at = at; sh.ctas = int(ctas); }
        long long rest = at - (upto - mine);
        if (end > at && rest >= 0 && rest < mine)
            for (int s = s0; s < s1; ++s) {
                if (each > 1) q = la_sequence<COLS>(a, s);
                const int cost = q.tiles + kLaItemCost<COLS>;
                const long long own = static_cast<long long>(q.blocks) * cost;
                if (rest < own) {
                    sh.seq = s;
                    sh.first = q;
                    sh.group = narrow ? int(uint32_t(rest) / uint32_t(cost)) : int(rest / cost);
                    sh.tile = int(rest - static_cast<long long>(sh.group) * cost);
                    break;
                }
                rest -= own;
            }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t t_s = sh.tmem, t_o = t_s + 2 * N, aside_at = t_o + latent / 128 * NO;

    // a warp goes on, or gives up, as one
    auto wait = [&](const unsigned long long& bar, int parity) {
        const uint32_t at = smem_u32(&bar);
        if (__all_sync(0xffffffffu, mbar_try_wait(at, parity))) return true;
        const unsigned long long t0 = global_timer_ns();
        for (;;) {
#pragma unroll 1
            for (int i = 0; i < 32; ++i)
                if (__all_sync(0xffffffffu, mbar_try_wait(at, parity))) return true;
            const bool late = global_timer_ns() - t0 > a.wait_ns;
            if (late) {
                *reinterpret_cast<volatile int*>(&sh.quit) = 1;
                kv_note(a.kv, SPM_KV_TIMEOUT);
            }
            if (__any_sync(0xffffffffu, late || *reinterpret_cast<volatile int*>(&sh.quit))) return false;
        }
    };

    LaWalk<COLS> w;
    w.start(a, sh);
    bool ok = true;
    if (warp < 4) {
        // ---- queries, softmax, results ----
        int item = 0, st = 0, turn = 0;          // items with a token in them; stage of the tile, and its barriers' phase
        unsigned it = 0;                         // tiles
        const int r0 = lane >> 2, c2 = (lane & 3) * 2;
        auto together = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
        auto vote = [](bool yes) {
            int any;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
                         : "=r"(any) : "r"(int(yes)) : "memory");
            return any != 0;
        };
        // This item's queries, eight lanes a column, all of a warp's loads in flight together
        auto bring_queries = [&](int half) {
            const int unit = lane & 7, last_units = a.kv.rope / 8;
#pragma unroll
            for (int c0 = 0; c0 < COLS; c0 += 16) {
                const int col = c0 + warp * 4 + (lane >> 3), x = w.group * COLS + col, i = la_row(a, x), row = w.s.first + i;
                const bool is = i < w.s.n && row >= 0 && row < a.batch.n_rows;
                const T* from = static_cast<const T*>(a.q.p) + (is ? row * a.q.row + (x - i * a.heads) * a.q.head + unit * 8 : 0);
                if (unit == 0) sh.limit[half][col] = is ? max(0, min(w.s.len - w.s.n + i + 1, w.s.cap_len)) : 0;
                const uint32_t to = q_at + col * 128 + ((unit ^ col & 7) << 4);
                if constexpr (PARTS == 1) {
#pragma unroll 3
                    for (int k = 0; k + 1 < chunks; ++k) copy16_or_zero(to + k * (N * 128), from + (is ? k * 64 : 0), is);
                    if (unit < last_units) copy16_or_zero(to + (chunks - 1) * (N * 128), from + (is ? (chunks - 1) * 64 : 0), is);
                } else {
                    Raw8 v[9];
#pragma unroll
                    for (int k = 0; k < 9; ++k) v[k] = is && (k + 1 < chunks || (k + 1 == chunks && unit < last_units)) ? raw8(from + k * 64) : Raw8{};
#pragma unroll
                    for (int k = 0; k < 9; ++k) {
                        if (k >= chunks) continue;
                        float f[8];
                        unpack8<T>(v[k], f);
                        uint32_t p[4][3];
#pragma unroll
                        for (int u = 0; u < 4; ++u) cut_parts(f[2 * u], f[2 * u + 1], p[u]);
#pragma unroll
                        for (int u = 0; u < 3; ++u) st_shared16(to + k * (N * 128) + u * (COLS * 128), make_uint4(p[0][u], p[1][u], p[2][u], p[3][u]));
                    }
                }
            }
            if constexpr (PARTS == 1) copies_arrived();
        };
        float* red = reinterpret_cast<float*>(raw_smem + (p_at - smem_u32(raw_smem)));       // [4 warps][COLS], in the probabilities' place
        long long* to_of = reinterpret_cast<long long*>(red + 4 * COLS);         // [COLS]
        while (w.left > 0 && ok) {
            const int half = item & 1;
            // ---- this item's columns: a warp brings every fourth ----
            if (w.tiles > 0) {
                bring_queries(half);
                fence_proxy_async();
                mbar_arrive(smem_u32(&sh.q_full));
            }
            bool first = true;                   // no token so far
            float m[BLOCKS][2], l[BLOCKS][2] = {};
            bool aside = false;                  // fp32 calls: there are sums of tiles before, behind O
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) m[i][0] = m[i][1] = 0.f;
            // tokens that all columns see: behind them are masks to look at
            const int all_see = w.s.n == 1 ? w.sees : max(0, min(w.s.len - w.s.n + la_row(a, w.group * COLS) + 1, w.s.cap_len));
            for (int j = 0; j < w.tiles; ++j, ++it) {
                const int t0 = (w.from + j) * kLaTile;
                // (a warp that gives up still comes to the others' barriers; they leave together)
                ok = ok && wait(sh.s_full[it & 1], (it >> 1) & 1) && wait(sh.full[st], turn);
                tc_fence_after();
                uint32_t r[N / 16][8];
#pragma unroll
                for (int i = 0; i < N / 16; ++i) tmem_ld_frag(t_s + (it & 1) * N + 16 * i + (uint32_t(warp) << 21), r[i]);
                tmem_wait_ld();
                const int absent = *reinterpret_cast<volatile int*>(&sh.absent[st]);
                const bool masks = t0 + kLaTile > all_see || absent != 0;
                float s[BLOCKS][4];              // (s - m): [8-wide block][row half * 2 + column]
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = __uint_as_float(r[i / 2][(i & 1) * 4 + e]);
                        if constexpr (PARTS == 3) v = v + __uint_as_float(r[i / 2 + 1][(i & 1) * 4 + e]) + __uint_as_float(r[i / 2 + 2][(i & 1) * 4 + e]);
                        s[i][e] = fmaf(v, a.factor, -m[i][e & 1]);
                    }
                auto highest = [&] {
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = fmaxf(top, s[i][e]);
                    return top;
                };
                auto lowest = [&] {
                    float low = INFINITY;
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) low = fminf(low, s[i][e]);
                    return low;
                };
                // the sums of the tile before are done (and the item before's, at its end): P and O may be touched
                auto sums_done = [&] { ok = ok && (j == 0 || wait(sh.empty[(st == 0 ? stages : st) - 1], st == 0 ? turn ^ 1 : turn)); };
                if (vote(highest() > kLaSlack || lowest() == -INFINITY || first || masks || !ok)) {
                    if (vote(!ok)) { ok = false; break; }
                    sums_done();
                    // A score of -infinity comes of an infinity in the query or the row, as one of +infinity does, which becomes NaN by itself. From
                    // here on it is what masks put in place of a score
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (s[i][e] == -INFINITY) s[i][e] = __int_as_float(0x7fffffff);
                    if (masks) {
                        // a thread looks at half of a token's row. What no column may see becomes zeros, so that 0 * NaN does not come up, and so
                        // does a row that is not finite where some columns see it and some do not
                        uint32_t* odd = reinterpret_cast<uint32_t*>(red);
                        if (tid < 2) odd[tid] = 0;
                        together();
                        const int t = tid >> 1, token = t0 + t;
                        const bool there = token < w.sees && !(absent >> (t / a.box) & 1);
                        const uint32_t at = base + st * stage_bytes + t * 128;
                        const int units = latent / 8;
                        bool bad = false;
                        if (there && token >= all_see)
                            for (int u = tid & 1; u < units; u += 2) {
                                const uint4 v = lds128(at + (u >> 3) * kLaChunkBytes + (((u & 7) ^ (t & 7)) << 4));
                                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int k = 0; k < 4; ++k) bad |= odd_word(x[k]);
                            }
                        const bool either = __shfl_xor_sync(0xffffffffu, bad, 1) | bad;
                        if (!there || either)
                            for (int u = tid & 1; u < units; u += 2)
                                st_shared16(at + (u >> 3) * kLaChunkBytes + (((u & 7) ^ (t & 7)) << 4), make_uint4(0, 0, 0, 0));
                        if (either) atomicOr(&odd[t >> 5], 1u << (t & 31));
                        together();
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int mine = warp * 16 + r0 + 8 * k;
                            const bool gone = absent >> (mine / a.box) & 1, poison = odd[mine >> 5] >> (mine & 31) & 1;
#pragma unroll
                            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    if (gone || t0 + mine >= sh.limit[half][8 * i + c2 + e]) s[i][2 * k + e] = -INFINITY;
                                    else if (poison) s[i][2 * k + e] = __int_as_float(0x7fffffff);
                                }
                        }
                    }
                    if (vote(highest() > kLaSlack || first)) {
                        tc_fence_after();
#pragma unroll
                        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float top = fmaxf(s[i][e], s[i][e + 2]);
#pragma unroll
                                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                                if (lane < 4) red[warp * COLS + 8 * i + c2 + e] = top;
                            }
                        together();
                        float by[BLOCKS][2];
#pragma unroll
                        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int col = 8 * i + c2 + e;
                                float top = fmaxf(fmaxf(red[col], red[COLS + col]), fmaxf(red[2 * COLS + col], red[3 * COLS + col]));
                                // (nothing seen, or no reason to move but that another column has one: stays. The first tile's may be below zero)
                                if (top == -INFINITY || (!first && top <= kLaSlack)) top = 0.f;
                                m[i][e] += top;
                                by[i][e] = first ? 1.f : ex2(-top);
                                l[i][e] *= by[i][e];
                                s[i][e] -= top;
                                s[i][e + 2] -= top;
                            }
                        together();
                        if (!first) {                // seldom: the sums so far go down
                            if (warp == 0 && lane < 4)
#pragma unroll
                                for (int i = 0; i < BLOCKS; ++i) { red[8 * i + c2] = by[i][0]; red[8 * i + c2 + 1] = by[i][1]; }
                            together();
#pragma unroll 1
                            for (int mt = 0; mt < latent / 128; ++mt)
#pragma unroll 1
                                for (int ch = 0; ch < NO / 16 + aside; ++ch) {
                                    uint32_t o[16];
                                    const uint32_t at = (ch < NO / 16 ? t_o + mt * NO + ch * 16 : aside_at + mt * 16) + (uint32_t(warp) << 21);
                                    tmem_ld16_raw(at, o);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * red[(ch * 16 + i) % COLS]);
                                    tmem_st16(at, o);
                                }
                            tmem_wait_st();
                            together();
                        }
                        first &= absent == (1 << kLaTile / a.box) - 1;
                    }
                } else sums_done();
                if constexpr (PARTS == 3)
                    if (j > 0 && j % kLaAside == 0) {        // the products begin anew
                        tc_fence_after();
#pragma unroll 1
                        for (int mt = 0; mt < latent / 128; ++mt) {
                            const uint32_t to = aside_at + mt * 16 + (uint32_t(warp) << 21);
                            uint32_t o[PARTS][16], v[16] = {};
#pragma unroll
                            for (int u = 0; u < PARTS; ++u) tmem_ld16_raw(t_o + mt * NO + u * COLS + (uint32_t(warp) << 21), o[u]);
                            if (aside) tmem_ld16_raw(to, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                v[i] = __float_as_uint(__uint_as_float(o[2][i]) + __uint_as_float(o[1][i]) + __uint_as_float(o[0][i]) + __uint_as_float(v[i]));
                            tmem_st16(to, v);
                        }
                        tmem_wait_st();
                        aside = true;
                    }
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[i][e] = ex2(s[i][e]);
                        l[i][e & 1] += s[i][e];
                    }
                // [column][token]: 16-byte unit 2 warp + (row half) of a column's 128 bytes
                const uint32_t to = p_at + ((lane >> 4) * 8 + (lane & 7)) * 128 + ((2 * warp + (lane >> 3 & 1) ^ (lane & 7)) << 4);
#pragma unroll
                for (int i = 0; i < BLOCKS; i += 2) {
                    uint32_t p[4][3];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float x = s[i + k / 2][(k & 1) * 2], y = s[i + k / 2][(k & 1) * 2 + 1];
                        if constexpr (PARTS == 3) cut_parts(x, y, p[k]);
                        else p[k][0] = pack_bf16(x, y);
                        if constexpr (P_PARTS == 2) {
                            float x0, y0;
                            two_bf16(p[k][0], x0, y0);
                            p[k][1] = pack_bf16(x - x0, y - y0);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < P_PARTS; ++u) st_matrix_trans(to + (u * COLS + 8 * i) * 128, p[0][u], p[1][u], p[2][u], p[3][u]);
                }
                fence_proxy_async();
                tc_fence_before();
                mbar_arrive(smem_u32(&sh.p_full));
                if (++st == stages) { st = 0; turn ^= 1; }
            }
            // ---- the item's result, or this CTA's part of it ----
            const bool whole = w.begins() && w.ends();
            if (w.tiles > 0) {
                ok = ok && wait(sh.empty[(st == 0 ? stages : st) - 1], st == 0 ? turn ^ 1 : turn);
                if (vote(!ok)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) l[i][e] += __shfl_xor_sync(0xffffffffu, l[i][e], o);
                        if (lane < 4) red[warp * COLS + 8 * i + c2 + e] = l[i][e];
                    }
                together();
            }
            float* part = a.parts + (size_t(blockIdx.x) * 2 + w.begins()) * S::part_floats(latent);       // slot 0: an item that began before this CTA
            float total = 0.f;
            if (w.tiles > 0 && tid < COLS) total = red[tid] + red[COLS + tid] + red[2 * COLS + tid] + red[3 * COLS + tid];
            together();
            if (!whole) {
                // (NaN is no part that sees nothing: its maximum is above all, and the item becomes NaN)
                if (warp == 0 && lane < 4)
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i) { red[8 * i + c2] = m[i][0]; red[8 * i + c2 + 1] = m[i][1]; }
                together();
                if (tid < COLS) {
                    part[COLS * latent + tid] = total == 0.f ? -INFINITY : total == total ? red[tid] : INFINITY;
                    part[COLS * latent + COLS + tid] = total;
                }
            } else if (tid < COLS) {             // where the column's result goes (-1: nowhere), and what it is scaled by
                const int x = w.group * COLS + tid, row_in = la_row(a, x), row = w.s.first + row_in;
                const bool is = row_in < w.s.n && row >= 0 && row < a.batch.n_rows;
                red[tid] = total == 0.f ? 0.f : 1.f / total;
                to_of[tid] = is ? row * a.out.row + (x - row_in * a.heads) * a.out.head : -1;
            }
            together();
            // a part: four columns of an element side by side, elements behind each other. A result: an element a thread, in bf16 two of one column of
            // each two
            if (w.tiles > 0 || whole) {
#pragma unroll 1
                for (int ch = 0; ch < COLS / 16; ++ch) {
                    float by[16];
                    long long at[16];            // of the column in bf16 of every other one: of this lane's
                    if (whole)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            by[i] = red[ch * 16 + i];
                            at[i] = to_of[ch * 16 + (sizeof(T) == 2 ? i / 2 * 2 + (lane & 1) : i)];
                        }
#pragma unroll 1
                    for (int mt = 0; mt < latent / 128; ++mt) {
                        const int d = mt * 128 + tid;
                        uint32_t o[P_PARTS][16] = {}, before[16] = {};
                        if (w.tiles > 0) {
                            if (PARTS == 3 && aside) tmem_ld16_raw(aside_at + mt * 16 + (uint32_t(warp) << 21), before);
#pragma unroll
                            for (int u = 0; u < P_PARTS; ++u) tmem_ld16_raw(t_o + mt * NO + u * COLS + ch * 16 + (uint32_t(warp) << 21), o[u]);
                            tmem_wait_ld();
                        }
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            v[i] = __uint_as_float(o[0][i]);
                            if constexpr (P_PARTS == 2) v[i] += __uint_as_float(o[1][i]);
                            if constexpr (PARTS == 3) v[i] = __uint_as_float(o[2][i]) + __uint_as_float(o[1][i]) + v[i] + __uint_as_float(before[i]);
                        }
                        if (!whole) {
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                *reinterpret_cast<float4*>(part + ((mt * (COLS / 4) + ch * 4 + i / 4) * 128 + tid) * 4) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        } else if constexpr (sizeof(T) == 2) {
                            const bool odd = lane & 1;
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                const float x = v[i] * by[i], y = v[i + 1] * by[i + 1], got = __shfl_xor_sync(0xffffffffu, odd ? x : y, 1);
                                if (at[i] >= 0) *reinterpret_cast<uint32_t*>(static_cast<T*>(a.out.p) + at[i] + (d & ~1)) = odd ? pack_bf16(got, y) : pack_bf16(x, got);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (at[i] >= 0) static_cast<T*>(a.out.p)[at[i] + d] = v[i] * by[i];
                        }
                    }
                }
            }
            tc_fence_before();
            together();                          // (`red` has been read)
            item += w.tiles > 0;
            w.next(a);
        }
    } else if (warp == 4) {
        // ---- tiles on their way in ----
        int st = 0, turn = 0;
        unsigned it = 0;
        const uint64_t once = policy_evict_first();          // (262145 tokens of 16 heads: 72 us without, 64)
        int4 join = make_int4(0, 0, 0, 0);
        long long joined = 0;
        while (w.left > 0 && ok) {
            if (w.begins() && !w.ends()) {       // goes on behind this CTA, up to there
                joined = sh.at + (sh.left - w.left) + w.s.tiles + w.kCost;
                join = make_int4(0, w.s.first, w.s.n, w.group);
            }
            // pages are asked for two tiles ahead, and looked at one tile ahead
            const int copies = kLaTile / a.box, copy = lane & (copies - 1);
            const int* table = a.batch.table + size_t(w.seq) * a.batch.stride;
            auto token_of = [&](int j) { return (w.from + j) * kLaTile + copy * a.box; };
            auto page_of = [&](int j) { return j < w.tiles && token_of(j) < w.sees ? table[token_of(j) / a.kv.page_size] : -1; };
            auto row_of = [&](int j, int page) { // of this lane's copy in the pool; -1: there is none, or nobody sees it
                if (page >= 0 && page < a.kv.n_pages) return page * a.kv.page_size + token_of(j) % a.kv.page_size;
                if (j < w.tiles && token_of(j) < w.sees) kv_note(a.kv, SPM_KV_BAD_PAGE);
                return -1;
            };
            const int first_page = page_of(0);
            int page = page_of(1), row = row_of(0, first_page);
            for (int j = 0; j < w.tiles; ++j, ++it) {
                const int page_then = page_of(j + 2);
                if (it >= unsigned(stages) && !(ok = wait(sh.empty[st], turn ^ 1))) break;
                const uint32_t there = __ballot_sync(0xffffffffu, row >= 0) & ((1u << copies) - 1);
                const uint32_t bar = smem_u32(&sh.full[st]), to = base + st * stage_bytes;
                if (lane == 0) {
                    sh.absent[st] = int(~there & ((1u << copies) - 1));
                    mbar_arrive_expect_tx(bar, __popc(there) * a.box * 128 * chunks);
                }
                __syncwarp();
                if (row >= 0)                    // (a lane's copy is the same for each of its chunks)
                    for (int c = lane / copies; c < chunks; c += 32 / copies) {
                        const uint32_t at = to + c * kLaChunkBytes + copy * a.box * 128;
                        if (w.s.blocks == 1) tma_rows_once(at, &rows_map, c * 64, row, bar, once);
                        else tma_rows(at, &rows_map, c * 64, row, bar);
                    }
                __syncwarp();
                row = row_of(j + 1, page);
                page = page_then;
                if (++st == stages) { st = 0; turn ^= 1; }
            }
            if (ok) w.next(a);
        }
        // copies under way end before shared memory is given back, whoever has given up
        for (unsigned k = it > unsigned(stages) ? it - stages : 0; k < it; ++k) mbar_wait_bounded(smem_u32(&sh.full[k % stages]), (k / stages) & 1, a.wait_ns);
        if (joined > 0) join.x = int((joined * sh.ctas - 1) / sh.all) - int(blockIdx.x) + 1;             // up to the CTA that has its last tile
        if (lane == 0) a.joins[blockIdx.x] = join;
        __syncwarp();
    } else {
        // ---- products. The warp walks as one, so that the elected lane is one lane throughout ----
        const uint32_t idesc_s = la_idesc(kLaTile, N, false), idesc_o = la_idesc(128, NO, true);
        const int rope_steps = a.kv.rope / 16, m_tiles = latent / 128;
        int st = 0, turn = 0, item = 0;
        unsigned it = 0;
        bool any = false;
        // Descriptors differ in their address alone, the low word. One instruction or two a product, or the issuing thread is slower than they are
        const uint64_t rows_k = smem_desc_sw128(base, 16, 1024), rows_m = smem_desc_sw128(base, kLaChunkBytes, 1024);
        const uint64_t q_k = smem_desc_sw128(q_at, 16, 1024), p_k = smem_desc_sw128(p_at, 16, 1024);
        const uint32_t hi_k = uint32_t(rows_k >> 32), hi_m = uint32_t(rows_m >> 32), lo_p = uint32_t(p_k);
        auto scores = [&](unsigned tile, int stage) {
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = t_s + (tile & 1) * N;
                uint32_t lo_a = uint32_t(rows_k) + stage * (stage_bytes >> 4), lo_b = uint32_t(q_k);
                tc_mma_lo<false>(d, lo_a, hi_k, lo_b, hi_k, idesc_s);
                tc_mma_lo<true>(d, lo_a + 2, hi_k, lo_b + 2, hi_k, idesc_s);
                tc_mma_lo<true>(d, lo_a + 4, hi_k, lo_b + 4, hi_k, idesc_s);
                tc_mma_lo<true>(d, lo_a + 6, hi_k, lo_b + 6, hi_k, idesc_s);
#pragma unroll 2
                for (int c = 2; c < chunks; ++c) {
                    lo_a += kLaChunkBytes >> 4;
                    lo_b += N * 8;
                    tc_mma_lo<true>(d, lo_a, hi_k, lo_b, hi_k, idesc_s);
                    tc_mma_lo<true>(d, lo_a + 2, hi_k, lo_b + 2, hi_k, idesc_s);
                    tc_mma_lo<true>(d, lo_a + 4, hi_k, lo_b + 4, hi_k, idesc_s);
                    tc_mma_lo<true>(d, lo_a + 6, hi_k, lo_b + 6, hi_k, idesc_s);
                }
                lo_a += kLaChunkBytes >> 4;
                lo_b += N * 8;
                for (int k = 0; k < rope_steps; ++k) tc_mma_lo<true>(d, lo_a + 2 * k, hi_k, lo_b + 2 * k, hi_k, idesc_s);
                tc_commit(smem_u32(&sh.s_full[tile & 1]));
            }
            any = true;
            __syncwarp();
        };
        auto sums = [&](int stage, bool more) {
            if (elect_one()) {
                uint32_t lo_a = uint32_t(rows_m) + stage * (stage_bytes >> 4), d = t_o;
                for (int mt = 0; mt < m_tiles; ++mt) {
                    if (more) tc_mma_lo<true>(d, lo_a, hi_m, lo_p, hi_k, idesc_o);
                    else tc_mma_lo<false>(d, lo_a, hi_m, lo_p, hi_k, idesc_o);
                    tc_mma_lo<true>(d, lo_a + 128, hi_m, lo_p + 2, hi_k, idesc_o);
                    tc_mma_lo<true>(d, lo_a + 256, hi_m, lo_p + 4, hi_k, idesc_o);
                    tc_mma_lo<true>(d, lo_a + 384, hi_m, lo_p + 6, hi_k, idesc_o);
                    lo_a += 2 * kLaChunkBytes >> 4;
                    d += NO;
                }
                tc_commit(smem_u32(&sh.empty[stage]));
            }
            __syncwarp();
        };
        while (w.left > 0 && ok) {
            if (w.tiles > 0) {
                if (!(ok = wait(sh.q_full, item & 1))) break;
                if (!(ok = wait(sh.full[st], turn))) break;
                scores(it, st);
                for (int j = 0; j < w.tiles; ++j, ++it) {
                    const int next = st + 1 == stages ? 0 : st + 1, next_turn = next == 0 ? turn ^ 1 : turn;
                    bool more = j + 1 < w.tiles;
                    // the next tile's scores, should it land before this one's probabilities are there
                    const unsigned long long t0 = global_timer_ns();
                    for (int i = 1;; ++i) {
                        if (more && __all_sync(0xffffffffu, mbar_test(smem_u32(&sh.full[next]), next_turn))) { scores(it + 1, next); more = false; }
                        if (!more) { ok = wait(sh.p_full, it & 1); break; }
                        if (__all_sync(0xffffffffu, mbar_test(smem_u32(&sh.p_full), it & 1))) break;
                        if (i % 64 == 0 && __any_sync(0xffffffffu, global_timer_ns() - t0 > a.wait_ns)) { ok = wait(sh.p_full, it & 1); break; }
                    }
                    if (!ok) break;
                    tc_fence_after();
                    sums(st, PARTS == 3 ? j % kLaAside != 0 : j > 0);
                    if (more) {
                        if (!(ok = wait(sh.full[next], next_turn))) break;
                        scores(it + 1, next);
                    }
                    st = next; turn = next_turn;
                }
                ++item;
            }
            if (ok) w.next(a);
        }
        if (any) {                               // products under way end before tensor memory is given back, whoever has given up
            if (elect_one()) tc_commit(smem_u32(&sh.drained));
            __syncwarp();
            mbar_wait_bounded(smem_u32(&sh.drained), 0, 2'000'000'000ull);
            __syncwarp();
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_dealloc(t_s, 512);
}

// Adds the parts of items that were cut between CTAs. A task is four columns of one such item and 128 of their elements, a warp's; where these
// are fewer than warps, 32 elements; where these are no more than blocks, a block's, whose eight warps take the parts in turn. Parts are
// added in the same order each time.
constexpr int kLaJoinThreads = 256, kLaJoinBlocks = 592, kLaJoinWarps = kLaJoinThreads / 32;
struct LaJoinShared {
    float weights[kLaJoinWarps][kLaMaxCtas][4];
    float4 sums[kLaJoinWarps][32];
    float tops[kLaJoinWarps][4], totals[kLaJoinWarps][4];
};
// WIDE: runs of 32 elements a lane has four columns of. BLOCK: all warps of a block together
template <typename T, int COLS, int WIDE, bool BLOCK>
__device__ __forceinline__ void la_join(const LatentAttendArgs& a, LaJoinShared& sh, int owner, int quad, int d0) {
    using S = LaShape<T, COLS>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, latent = a.kv.latent, from = BLOCK ? warp : 0, step = BLOCK ? kLaJoinWarps : 1;
    const int4 join = a.joins[owner];
    // part 0 is the second slot of its CTA, the others are the first slots of theirs
    const size_t each = S::part_floats(latent);
    const float* parts = a.parts + size_t(owner) * 2 * each;
    auto part = [&](int j) { return parts + (j == 0 ? 1 : 2 * j) * each; };
    const int mine = from < join.x ? (join.x - from + step - 1) / step : 0;
    // lane (i, k): maxima and sums of column k
    const int k = lane & 3, end_at = COLS * latent + quad * 4 + k;
    float top = -INFINITY, sum = 0.f;
    for (int i0 = lane >> 2; i0 < mine; i0 += 32) {
        float m[4], l[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool is = i0 + 8 * u < mine;
            const float* at = part(from + (is ? i0 + 8 * u : 0) * step) + end_at;
            m[u] = is ? at[0] : -INFINITY;
            l[u] = is ? at[COLS] : 0.f;
        }
        float to = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) to = fmaxf(to, m[u]);
        if (sum != 0.f) sum *= ex2(top - to);
        top = to;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (m[u] != -INFINITY) sum += l[u] * ex2(m[u] - to);
            if (i0 + 8 * u < mine) sh.weights[warp][i0 + 8 * u][k] = m[u];
        }
    }
    const float own = top;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (sum != 0.f) sum *= ex2(own - top);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    for (int i = lane >> 2; i < mine; i += 8) {
        const float m = sh.weights[warp][i][k];
        sh.weights[warp][i][k] = m == -INFINITY ? 0.f : ex2(m - top);
    }
    __syncwarp();
    float o[WIDE][4] = {};
    const size_t at = ((d0 / 128 * (COLS / 4) + quad) * 128 + d0 % 128 + lane) * 4;
#pragma unroll 8 / WIDE
    for (int i = 0; i < mine; ++i) {
        const float4 by = *reinterpret_cast<const float4*>(sh.weights[warp][i]);
        float4 v[WIDE];
#pragma unroll
        for (int u = 0; u < WIDE; ++u) v[u] = *reinterpret_cast<const float4*>(part(from + i * step) + at + u * 128);
        // (a part that saw nothing has written no sums)
#pragma unroll
        for (int u = 0; u < WIDE; ++u) {
            o[u][0] += by.x == 0.f ? 0.f : by.x * v[u].x; o[u][1] += by.y == 0.f ? 0.f : by.y * v[u].y;
            o[u][2] += by.z == 0.f ? 0.f : by.z * v[u].z; o[u][3] += by.w == 0.f ? 0.f : by.w * v[u].w;
        }
    }
    if constexpr (BLOCK) {                       // the warps' sums, by their maxima
        if (lane < 4) { sh.tops[warp][lane] = top; sh.totals[warp][lane] = sum; }
        sh.sums[warp][lane] = make_float4(o[0][0], o[0][1], o[0][2], o[0][3]);
        __syncthreads();
        if (warp == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float most = -INFINITY, total = 0.f, y = 0.f;
#pragma unroll
                for (int u = 0; u < kLaJoinWarps; ++u) most = fmaxf(most, sh.tops[u][i]);
#pragma unroll
                for (int u = 0; u < kLaJoinWarps; ++u) {
                    const float by = sh.tops[u][i] == -INFINITY ? 0.f : ex2(sh.tops[u][i] - most);
                    if (by != 0.f) { total += by * sh.totals[u][i]; y += by * reinterpret_cast<const float*>(&sh.sums[u][lane])[i]; }
                }
                o[0][i] = y;
                if (k == i) sum = total;
            }
        __syncthreads();
        if (warp > 0) return;
    }
    const float norm = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int x = join.w * COLS + quad * 4 + i, row_in = la_row(a, x), h = x - row_in * a.heads, row = join.y + row_in;
        const float by = __shfl_sync(0xffffffffu, norm, i);
        if (row_in >= join.z || row < 0 || row >= a.batch.n_rows) continue;
        T* to = static_cast<T*>(a.out.p) + row * a.out.row + h * a.out.head + d0 + lane;
#pragma unroll
        for (int u = 0; u < WIDE; ++u) {
            const float y = o[u][i] * by;
            if constexpr (sizeof(T) == 2) to[u * 32] = __float2bfloat16_rn(y);
            else to[u * 32] = y;
        }
    }
    __syncwarp();
}
template <typename T, int COLS>
__global__ void __launch_bounds__(kLaJoinThreads) latent_join_kernel(const LatentAttendArgs a, int ctas) {
    __shared__ int owners[kLaMaxCtas], n_owners;
    __shared__ __align__(16) LaJoinShared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dep_wait();
    grid_dep_launch();
    if (warp == 0) {
        int count = 0;
#pragma unroll
        for (int i = 0; i < kLaMaxCtas; i += 32) {
            const bool is = i + lane < ctas && a.joins[i + lane].x > 0;
            const uint32_t who = __ballot_sync(0xffffffffu, is);
            if (is) owners[count + __popc(who & ((1u << lane) - 1))] = i + lane;
            count += __popc(who);
        }
        if (lane == 0) n_owners = count;
    }
    __syncthreads();
    constexpr int QUADS = COLS / 4;
    const int runs = a.kv.latent / 32, narrow = n_owners * QUADS * runs, wide = narrow / 4;
    const auto narrow_task = [&](int task, auto block) {
        const int item = task / (QUADS * runs), in = task % (QUADS * runs);
        la_join<T, COLS, 1, block.value>(a, sh, owners[item], in / runs, in % runs * 32);
    };
    if (narrow <= int(gridDim.x)) {
        if (int(blockIdx.x) < narrow) narrow_task(blockIdx.x, std::integral_constant<bool, true>{});
    } else if (wide < int(gridDim.x) * kLaJoinWarps / 2)
        for (int task = blockIdx.x * kLaJoinWarps + warp; task < narrow; task += gridDim.x * kLaJoinWarps) narrow_task(task, std::integral_constant<bool, false>{});
    else
        for (int task = blockIdx.x * kLaJoinWarps + warp; task < wide; task += gridDim.x * kLaJoinWarps) {
            const int item = task / (QUADS * runs / 4), in = task % (QUADS * runs / 4);
            la_join<T, COLS, 4, false>(a, sh, owners[item], in / (runs / 4), in % (runs / 4) * 128);
        }
}

}  // namespace spm
