// Keys and values of a batch's tokens, made from their latent vectors for one head after another, on tcgen05.
//
// [key | value] of a head = C [W_k ; W_v]^T: 128 tokens of one sequence, all of their latent vectors in shared memory, against the head's
// matrices, whose rows come by in chunks of 64 elements. Sums of two heads are in tensor memory, so that one is rounded to fp16 and
// written while the next is made. All (tile of tokens, head) pairs are a line that is cut evenly between CTAs, so that a CTA brings the latent
// vectors of two or three tiles and not of many: four prompts' 10563 tokens of 16 heads take 56 us, 0.80 PFLOP/s (54 with the cut before there were powers of
// two, 59 with a CTA for each tile and a third of the heads). What bounds it: the products of a tile and head, some 4500 cycles, and the results' way
// out of tensor memory and the SM, which is longer than these and only partly beside them. Sequences stand behind each other in the workspace, each
// from a multiple of 128 tokens on.
//
// Both are fp16, times a power of two for each 32 tokens of a head: bf16's roundings of keys, values and probabilities were together 1.4 times that
// of the result. A key's power is 1 where the largest of its 32 tokens is in fp16's range as it is, which it is but for odd models, and the part
// that all heads share is there once; elsewhere each head has a copy of that too, times its own power of two.
//
// A token that does not exist becomes zeros, and its bit in `there` too. A token whose keys are not finite, or have an element of 2^109 or more, gets
// NaN as its key's first element and finite values: scores of rows that see it are NaN, and 0 * NaN does not come up for those that do not.
#pragma once

#include <cuda.h>

#include "kv_cache.cuh"
#include "latent_attend.cuh"
#include "latent_cache.cuh"
#include "prompt_items.cuh"
#include "ptx.cuh"
#include "tc_ops.cuh"

namespace spm {

constexpr int kLxLeast = -110;                   // E of values that are all zero, or nearly
// Where keys end, as fp32 bits: 2^109. A score is less than 192 products of 2^10 by 2^10, times 2^E, E at most 108 - 9: 2^127, and so is a difference of two
constexpr uint32_t kLxKeyEnd = (127 + 109) << 23;
__device__ __forceinline__ uint32_t pack_fp16(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
constexpr int kLxTile = 128, kLxThreads = 320, kLxChunkBytes = kLxTile * 128;

// What a CTA of the attention takes (its rows, and where their tokens stand in the workspace), found here, where it is beside other work
struct alignas(16) LxItem { PfItem item; int at, tokens, unused; };
static_assert(sizeof(LxItem) == 32, "two 16-byte words");

struct LatentExpandArgs {
    LatentPool kv;
    KvBatch batch;
    int heads, h0;              // of this round, the first one's number
    int box;                    // tokens of a copy, all of one page
    int stages;                 // of the matrices' ring
    int tokens;                 // that the workspace has room for, a multiple of 128
    __half *keys, *values;                      // [heads][tokens][HD] twice, times 2^-E
    __half *shared, *own;                       // the shared parts of keys: [tokens][64], and [heads][tokens][64] times 2^-E, where that is not 1
    short *key_exps, *value_exps;               // [heads][tokens / 32]: E
    uint32_t* there;            // [tokens / 32]
    LxItem* items;              // [n_items]
    int n_items;
    unsigned long long wait_ns;
    int withhold;
};

// Where a sequence's tokens stand in the workspace, and how many of them
struct LxPlace { int seq, at, tokens, tile; };

// Of a sequence (all lanes of a warp together): tokens that count, and rows
__device__ __forceinline__ int lx_tokens(const KvBatch& b, int cap, int s) {
    if (s >= b.n_seq) return 0;
    if (b.row_start && min(b.row_start[s + 1] - b.row_start[s], b.n_rows) <= 0) return 0;     // (no rows look at them)
    return max(0, min(b.lengths[s], cap));
}
// Tiles of all sequences, as far as there is room, by a warp
__device__ __forceinline__ int lx_tiles(const KvBatch& b, int cap, int room) {
    long long sum = 0;
    for (int s0 = 0; s0 < b.n_seq; s0 += 32) sum += (lx_tokens(b, cap, s0 + (threadIdx.x & 31)) + kLxTile - 1) / kLxTile;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return int(min(sum, static_cast<long long>(room / kLxTile)));
}
// Tile `tile` of the workspace (tile < 0: sequence `seq`'s first), by a warp
__device__ __forceinline__ LxPlace lx_find(const KvBatch& b, int cap, int room, int seq, int tile) {
    const int lane = threadIdx.x & 31;
    LxPlace p{-1, 0, 0, 0};
    long long before = 0;                        // tiles
    for (int s0 = 0; s0 < b.n_seq; s0 += 32) {
        const int tokens = lx_tokens(b, cap, s0 + lane);
        const long long own = (tokens + kLxTile - 1) / kLxTile;
        long long upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const long long first = before + upto - own;
        const bool here = tile >= 0 ? first <= tile && tile < first + own : s0 + lane == seq;
        const uint32_t who = __ballot_sync(0xffffffffu, here);
        if (who) {
            const int from = __ffs(who) - 1;
            const long long at = min(__shfl_sync(0xffffffffu, first, from) * kLxTile, static_cast<long long>(room));
            p.seq = s0 + from;
            p.at = int(at);
            p.tokens = min(__shfl_sync(0xffffffffu, tokens, from), room - p.at);
            p.tile = tile - p.at / kLxTile;
            return p;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return p;
}

struct LxShared {
    unsigned long long a_full, a_empty, b_full[8], b_empty[8], d_full[2], d_empty[2], drained;
    uint32_t tmem;
    int quit, tiles;
    PfItem items[8];                             // a warp's
};
// A CTA's piece of the line, tile by tile
struct LxWalk {
    long long at, end;
    int heads, tile, h0, h1;
    __device__ __forceinline__ LxWalk(int tiles, int n) : heads(n) {
        const long long all = static_cast<long long>(tiles) * n;
        at = all * blockIdx.x / gridDim.x;
        end = all * (blockIdx.x + 1) / gridDim.x;
        piece();
    }
    __device__ __forceinline__ void piece() {
        tile = int(at / heads);
        h0 = int(at - static_cast<long long>(tile) * heads);
        h1 = int(min(static_cast<long long>(heads), h0 + end - at));
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void next() { at += h1 - h0; if (more()) piece(); }
};
constexpr int kLxOwnBytes = 1024;
static_assert(sizeof(LxShared) <= kLxOwnBytes, "what shared memory has beside the operands");

__device__ __forceinline__ void tma_matrix(uint32_t dst, const CUtensorMap* map, int element, int row, int head, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(element), "r"(row), "r"(head), "r"(bar) : "memory");
}
// a sector of 32 bytes a thread
__device__ __forceinline__ void st_global32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), SPM_W8(v, 0) : "memory");
}
__device__ __forceinline__ bool not_finite(uint32_t bits) { return (bits & 0x7f800000u) == 0x7f800000u; }

template <int HD>
__global__ void __launch_bounds__(kLxThreads, 1) latent_expand_kernel(const LatentExpandArgs a, const __grid_constant__ CUtensorMap rows_map,
                                                                      const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    constexpr int N = 2 * HD, STAGE = N * 128;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    LxShared& sh = *reinterpret_cast<LxShared*>(raw_smem);
    const uint32_t a_at = (smem_u32(raw_smem) + kLxOwnBytes + 1023) & ~1023u;
    const int chunks = a.kv.latent / 64, cap = a.batch.stride * a.kv.page_size;
    const uint32_t b_at = a_at + chunks * kLxChunkBytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    grid_dep_wait();
    grid_dep_launch();
    if (tid == 0) {
        mbar_init(smem_u32(&sh.a_full), 1 + a.withhold);
        mbar_init(smem_u32(&sh.a_empty), 1);
        for (int i = 0; i < a.stages; ++i) { mbar_init(smem_u32(&sh.b_full[i]), 1); mbar_init(smem_u32(&sh.b_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&sh.d_full[i]), 1); mbar_init(smem_u32(&sh.d_empty[i]), 256); }
        mbar_init(smem_u32(&sh.drained), 1);
        sh.quit = 0;
        fence_barrier_init();
    }
    if (warp == 9) tmem_alloc(smem_u32(&sh.tmem), 2 * N);
    if (warp == 8) {
        const int tiles = lx_tiles(a.batch, cap, a.tokens);
        if (lane == 0) sh.tiles = tiles;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    LxWalk w(sh.tiles, a.heads);
    // where a token of the place's tile stands in the pool, -1: nowhere
    auto row_of = [&](const LxPlace& place, int in, bool note) {
        const int token = place.tile * kLxTile + in;
        if (place.seq < 0 || token >= place.tokens) return -1;
        const int page = a.batch.table[size_t(place.seq) * a.batch.stride + token / a.kv.page_size];
        if (page >= 0 && page < a.kv.n_pages) return page * a.kv.page_size + token % a.kv.page_size;
        if (note) kv_note(a.kv, SPM_KV_BAD_PAGE);
        return -1;
    };

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
    bool ok = true;

    if (warp < 8) {
        // ---- rows out: a token a thread, four warps its keys and four its values ----
        const int part = warp >> 2, in = tid & 127;
        const uint32_t lanes = uint32_t(warp & 3) << 21;
        for (int x = blockIdx.x * 8 + warp; x < a.n_items; x += gridDim.x * 8) {
            PfItem& item = sh.items[warp];
            pf_find(a.batch, nullptr, 1, cap, x, item);
            __syncwarp();
            const LxPlace p = lx_find(a.batch, cap, a.tokens, item.n > 0 ? item.seq : 0, -1);
            if (lane == 0) a.items[x] = LxItem{item, p.at, p.tokens, 0};
            __syncwarp();
        }
        int i = 0;                               // heads so far
        for (; w.more() && ok; w.next()) {
            const LxPlace place = lx_find(a.batch, cap, a.tokens, 0, w.tile);
            const int row = row_of(place, in, false);
            const bool there = row >= 0;
            const size_t to = size_t(w.tile) * kLxTile + in;
            // the shared key, as it is in the cache
            const uint4* from = reinterpret_cast<const uint4*>(a.kv.rows + static_cast<long long>(there ? row : 0) * (a.kv.latent + a.kv.rope) + a.kv.latent);
            auto rope = [&](int k) { return there && k < a.kv.rope / 8 ? from[k] : make_uint4(0, 0, 0, 0); };
            auto shared_key = [&](__half* out, float by) {
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const uint4 u = rope(k), v = rope(k + 1);
                    const uint32_t x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
                    uint32_t y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float lo, hi;
                        two_bf16(x[e], lo, hi);
                        y[e] = pack_fp16(lo * by, hi * by);
                    }
                    st_global32(out + k * 8, y);
                }
            };
            if (w.h0 == 0 && part == 0) {
                const uint32_t bits = __ballot_sync(0xffffffffu, there);
                if (lane == 0) a.there[to / 32] = bits;
                shared_key(a.shared + to * 64, 1.f);
            }
            uint32_t rope_top = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint4 v = rope(k);
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) rope_top = max(rope_top, max(x[e] << 16 & 0x7fffffffu, x[e] & 0x7fff0000u));
            }
            for (int h = w.h0; h < w.h1; ++h, ++i) {
                const int buf = i & 1, turn = i >> 1 & 1;
                if (!(ok = wait(sh.d_full[buf], turn))) break;
                tc_fence_after();
                uint32_t r[HD], word[HD / 2];
                auto take = [&](int which) {
#pragma unroll
                    for (int ch = 0; ch < HD / 32; ++ch)
                        tmem_ld32(tmem + buf * N + which * HD + ch * 32 + lanes, *reinterpret_cast<uint32_t(*)[32]>(r + ch * 32));
                    tmem_wait_ld();
                };
                auto largest = [&] {             // as fp32 bits; what is not finite is above all else
                    uint32_t v = 0;
#pragma unroll
                    for (int e = 0; e < HD; ++e) v = max(v, r[e] & 0x7fffffffu);
                    return there ? v : 0u;
                };
                take(part);
                uint32_t top = part == 0 ? max(rope_top, largest()) : largest();
                const bool odd = top >= (part == 0 ? kLxKeyEnd : 0x7f800000u);
                if (part == 1 && __any_sync(0xffffffffu, odd)) {             // values: is it the token, or the matrix?
                    take(0);
                    const bool token = max(rope_top, largest()) >= kLxKeyEnd;
                    take(1);
                    if (token)
#pragma unroll
                        for (int e = 0; e < HD; ++e) r[e] = not_finite(r[e]) ? 0u : r[e];
                    top = largest();
                }
                tc_fence_before();
                mbar_arrive(smem_u32(&sh.d_empty[buf]));
                if (!there)
#pragma unroll
                    for (int e = 0; e < HD; ++e) r[e] = 0u;
                // the largest of a warp's tokens is brought to [2^9, 2^10); of keys if it is below 2^-4 or not below 2^15
                top = __reduce_max_sync(0xffffffffu, part == 0 && odd ? 0u : top);
                const int power = part == 0 && (top == 0 || (top >= 0x3d800000u && top < 0x47000000u)) ? 0 : top == 0 ? kLxLeast : max(kLxLeast, min(int(top >> 23) - 127 - 9, 118));
                const float by = __int_as_float((127 - power) << 23);
#pragma unroll
                for (int e = 0; e < HD; e += 2) word[e / 2] = pack_fp16(__uint_as_float(r[e]) * by, __uint_as_float(r[e + 1]) * by);
                if (lane == 0) (part == 0 ? a.key_exps : a.value_exps)[(size_t(h) * a.tokens + to) / 32] = short(power);
                if (part == 0 && odd) word[0] = 0x7fff7fffu;
                __half* out = (part == 0 ? a.keys : a.values) + (size_t(h) * a.tokens + to) * HD;
#pragma unroll
                for (int e = 0; e < HD / 2; e += 8) st_global32(out + 2 * e, word + e);
                if (part == 0 && power != 0) shared_key(a.own + (size_t(h) * a.tokens + to) * 64, by);
            }
        }
    } else if (warp == 8) {
        // ---- latent vectors, then matrices, on their way in ----
        const int copies = kLxTile / a.box;
        const uint32_t a_bar = smem_u32(&sh.a_full);
        int st = 0, turn = 0, it = 0, tile = 0;
        for (; w.more() && ok; w.next(), ++tile) {
            const LxPlace place = lx_find(a.batch, cap, a.tokens, 0, w.tile);
            const int row = lane < copies ? row_of(place, lane * a.box, true) : -1, n = __popc(__ballot_sync(0xffffffffu, row >= 0));
            if (tile > 0 && !(ok = wait(sh.a_empty, (tile - 1) & 1))) break;
            if (lane == 0) mbar_arrive_expect_tx(a_bar, n * a.box * 128 * chunks);
            __syncwarp();
            if (row >= 0)
                for (int c = 0; c < chunks; ++c) tma_rows(a_at + c * kLxChunkBytes + lane * a.box * 128, &rows_map, c * 64, row, a_bar);
            __syncwarp();
            for (int h = w.h0; h < w.h1 && ok; ++h)
                for (int c = 0; c < chunks; ++c, ++it) {
                    if (it >= a.stages && !(ok = wait(sh.b_empty[st], turn ^ 1))) break;
                    if (elect_one()) {
                        const uint32_t bar = smem_u32(&sh.b_full[st]), to = b_at + st * STAGE;
                        mbar_arrive_expect_tx(bar, STAGE);
                        tma_matrix(to, &k_map, c * 64, 0, a.h0 + h, bar);
                        tma_matrix(to + HD * 128, &v_map, c * 64, 0, a.h0 + h, bar);
                    }
                    __syncwarp();
                    if (++st == a.stages) { st = 0; turn ^= 1; }
                }
        }
        // copies under way end before shared memory is given back, whoever has given up
        if (tile > 0 || !ok) mbar_wait_bounded(a_bar, (max(tile, 1) - 1) & 1, a.wait_ns);
        for (int k = it > a.stages ? it - a.stages : 0; k < it; ++k) mbar_wait_bounded(smem_u32(&sh.b_full[k % a.stages]), (k / a.stages) & 1, a.wait_ns);
        __syncwarp();
    } else {
        // ---- products ----
        const uint32_t idesc = la_idesc(kLxTile, N, false);
        const uint64_t a_desc = smem_desc_sw128(a_at, 16, 1024), b_desc = smem_desc_sw128(b_at, 16, 1024);
        const uint32_t hi = uint32_t(a_desc >> 32);
        int st = 0, turn = 0;
        bool any = false;
        int i = 0, tile = 0;
        for (; w.more() && ok; w.next(), ++tile) {
            ok = wait(sh.a_full, tile & 1);
            for (int h = w.h0; h < w.h1 && ok; ++h, ++i) {
                const int buf = i & 1;
                if (i >= 2 && !(ok = wait(sh.d_empty[buf], (i / 2 - 1) & 1))) break;
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = wait(sh.b_full[st], turn))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t d = tmem + buf * N, lo_a = uint32_t(a_desc) + c * (kLxChunkBytes >> 4), lo_b = uint32_t(b_desc) + st * (STAGE >> 4);
                        if (c == 0) tc_mma_lo<false>(d, lo_a, hi, lo_b, hi, idesc);
                        else tc_mma_lo<true>(d, lo_a, hi, lo_b, hi, idesc);
                        tc_mma_lo<true>(d, lo_a + 2, hi, lo_b + 2, hi, idesc);
                        tc_mma_lo<true>(d, lo_a + 4, hi, lo_b + 4, hi, idesc);
                        tc_mma_lo<true>(d, lo_a + 6, hi, lo_b + 6, hi, idesc);
                        tc_commit(smem_u32(&sh.b_empty[st]));
                        if (c + 1 == chunks) {
                            tc_commit(smem_u32(&sh.d_full[buf]));
                            if (h + 1 == w.h1) tc_commit(smem_u32(&sh.a_empty));
                        }
                    }
                    any = true;
                    __syncwarp();
                    if (++st == a.stages) { st = 0; turn ^= 1; }
                }
            }
        }
        if (any) {                               // products under way end before tensor memory is given back, whoever has given up
            if (elect_one()) tc_commit(smem_u32(&sh.drained));
            __syncwarp();
            mbar_wait_bounded(smem_u32(&sh.drained), 0, 2'000'000'000ull);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 2 * N);
}

}  // namespace spm
