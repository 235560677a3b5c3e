// Attention of prompts over keys and values that latent_expand_kernel has made, on tcgen05.
//
// A CTA takes 256 rows of a head of one sequence, two M = 128 halves, and walks the tokens in tiles of 128. A key is HD elements of its
// head and a chunk of up to 64 that all heads share; keys and values come by TMA. One warp issues the products; four warps a half turn scores
// into probabilities, one row a thread, while the tensor cores are at the other half: S(j) of one half, then P V(j) and S(j + 1) of the
// other. Scores, probabilities (fp16, in the scores' place, as the A operand of the second product) and sums stay in tensor memory.
//
// Keys and values stand at 2^-E, E for each 32 tokens, and a row's queries are brought to [2^9, 2^10) by its largest, all in fp16. A row's maximum is
// moved, and its sums scaled, only where a score is above it by more than 2^6. Probabilities are fp16, times 2^4 and 2^(E - R), R the largest
// E of values so far but for 5, which moves, and the sums with it, where an E is above that. So no probability is above 2^15, and 11 bits
// hold for those down to 2^-18 of the largest and values down to 2^-18 of their head's largest.
//
// What bounds it: a half's chain, 3300 cycles a tile, while the other's runs beside it: scores out of tensor memory and maxima 550, exponentials 1300 (the
// special function units' 16 a cycle, so that a quarter of them are a polynomial: 148 us without, 144), products and their hand-over 1400, of which 20
// products at 60 cycles are all but 200. With two threads a row it took 161 us: registers for 512 threads spill, and the units are the same. Values in two
// stages of 64 tokens: 152. Four prompts of up to 2049 rows over up to 4097 tokens, 16 heads of 128 + 64: 144 us, 0.87 PFLOP/s at 1.72 GHz; a CTA's
// queries and first keys are 5 us of that, its results 2, three times.
#pragma once

#include <cuda.h>

#include "latent_expand.cuh"
#include "mma_ops.cuh"
#include "prompt_items.cuh"

namespace spm {

struct LatentPromptArgs {
    LatentPool kv;              // (its status, sizes)
    KvBatch batch;
    HeadRows q, out;
    int heads, h0;              // of this round, the first one's number
    int tokens, shared_row;     // of the workspace; where, behind the heads' copies, the shared parts of keys begin
    const uint32_t* there;
    const LxItem* items;
    const short *key_exps, *value_exps;
    float factor;               // of scores: scale times log2(e)
    unsigned long long wait_ns;
    int withhold;
};

constexpr int kLpTile = 128;
constexpr int kLpAtOnce = 4;                      // times four rows of queries, that a warp has under way
constexpr float kLpSlack = 6.f, kLpUp = 4.f;     // scores above the maximum that was, and probabilities' scale, as powers of two
constexpr int kLpRoom = 5;                       // of E above R
// two halves' softmax warps, then the copying warp, the issuing warp and two that only make its four whole. Registers a thread: 168 at the launch,
// of which the last four give some to the softmax warps
constexpr int kLpThreads = 12 * 32, kLpSoftmaxRegs = 208, kLpOtherRegs = 88;
static_assert(2 * kLpSoftmaxRegs + kLpOtherRegs <= 3 * 168, "the split is what the launch has");
__device__ __forceinline__ float two_to(int e) { return __int_as_float((127 + e) << 23); }
template <int HD>
struct LpShape {
    static constexpr int chunk = kLpTile * 128;                          // 64 elements of 128 rows
    static constexpr int k_chunks = HD / 64 + 1, v_chunks = HD / 64;
    static constexpr int k_bytes = k_chunks * chunk, v_bytes = v_chunks * chunk;
    static constexpr int v_stages = HD == 64 ? 2 : 1;                    // (what shared memory has room for)
    static constexpr int smem = 1024 + 2 * k_bytes + 2 * k_bytes + v_stages * v_bytes;       // queries of two halves, two stages of keys, values
};

struct LpShared {
    unsigned long long k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2][2], o_full[2], drained;
    uint32_t tmem;
    int quit;
};

// 2^x of two numbers below 2^7 by the pipes that ex2 leaves idle: 2^n (1 + f (c1 + f (c2 + f c3))), n the next integer, |f| <= 1/2, where the cubic of least
// relative error that is 1 at 0 is off by 1.02e-4, less than half of fp16's rounding. Below -127 it is 0; NaN stays.
__device__ __forceinline__ unsigned long long two_to2(unsigned long long x) {
    float x0, x1;
    floats_of(x, x0, x1);
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x0));             // -127
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x1));
    x = two_floats(x0, x1);
    const float round = 12582912.f;              // 1.5 * 2^23: the sum's lowest bits are n
    const unsigned long long t = add2(x, two_floats(round, round)), n = add2(t, two_floats(-round, -round)), f = fma2(n, two_floats(-1.f, -1.f), x);
    unsigned long long y = fma2(f, two_floats(0.05500893f, 0.05500893f), two_floats(0.24221096f, 0.24221096f));
    y = fma2(y, f, two_floats(0.69328293f, 0.69328293f));
    y = fma2(y, f, two_floats(1.f, 1.f));
    float t0, t1;
    floats_of(t, t0, t1);
    const unsigned long long by = two_words((__float_as_uint(t0) << 23) + 0x3f800000u, (__float_as_uint(t1) << 23) + 0x3f800000u);
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(y) : "l"(by));
    return y;
}
template <int HD>
__global__ void __launch_bounds__(kLpThreads, 1) latent_prompt_kernel(const LatentPromptArgs a, const __grid_constant__ CUtensorMap k_map,
                                                                      const __grid_constant__ CUtensorMap rope_map, const __grid_constant__ CUtensorMap rope32_map,
                                                                      const __grid_constant__ CUtensorMap v_map) {
    using S = LpShape<HD>;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    const uint32_t q_at = (smem_u32(raw_smem) + 1023) & ~1023u, k_at = q_at + 2 * S::k_bytes, v_at = k_at + 2 * S::k_bytes;
    __shared__ LpShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvBatch& b = a.batch;

    grid_dep_wait();
    grid_dep_launch();
    const int head = blockIdx.x % a.heads, cap = b.stride * a.kv.page_size;
    const LxItem mine = a.items[blockIdx.x / a.heads];
    if (mine.item.n == 0) return;                // more CTAs than items
    if (warp == 9 && lane == 0) {                // (the warp that copies, which need not wait for others then)
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 1 + a.withhold); mbar_init(smem_u32(&sh.v_full[i]), 1);
            mbar_init(smem_u32(&sh.k_empty[i]), 1); mbar_init(smem_u32(&sh.v_empty[i]), 1);
            mbar_init(smem_u32(&sh.s_full[i]), 1); mbar_init(smem_u32(&sh.p_full[i][0]), 128); mbar_init(smem_u32(&sh.p_full[i][1]), 128); mbar_init(smem_u32(&sh.o_full[i]), 1);
        }
        mbar_init(smem_u32(&sh.drained), 1);
        sh.quit = 0;
        fence_barrier_init();
    }
    __syncwarp();
    if (warp == 8) tmem_alloc(smem_u32(&sh.tmem), 512);
    const int rb = mine.item.rb, first = mine.item.first, n = mine.item.n, len = mine.item.len;
    const int at = mine.at, there_are = max(0, min(min(len, cap), mine.tokens));     // tokens in the workspace
    if (len > there_are && rb == 0 && head == 0 && tid == 0) kv_note(a.kv, SPM_KV_TOO_LONG);
    // tiles of a half: up to the token that its last row sees
    auto sees = [&](int x) { return max(0, min(len - n + min(n - 1, x) + 1, there_are)); };
    const bool used1 = rb * kPfCols + kLpTile < n;
    const int tiles0 = (sees(rb * kPfCols + kLpTile - 1) + kLpTile - 1) / kLpTile;
    const int tiles1 = used1 ? (sees(rb * kPfCols + kPfCols - 1) + kLpTile - 1) / kLpTile : 0;
    const int tiles = max(tiles0, tiles1);

    // a warp goes on, or gives up, as one
    auto wait = [&](const unsigned long long& bar, int parity) {
        const uint32_t w = smem_u32(&bar);
        if (__all_sync(0xffffffffu, mbar_try_wait(w, parity))) return true;
        const unsigned long long t0 = global_timer_ns();
        for (;;) {
#pragma unroll 1
            for (int i = 0; i < 32; ++i)
                if (__all_sync(0xffffffffu, mbar_try_wait(w, parity))) return true;
            const bool late = global_timer_ns() - t0 > a.wait_ns;
            if (late) {
                *reinterpret_cast<volatile int*>(&sh.quit) = 1;
                kv_note(a.kv, SPM_KV_TIMEOUT);
            }
            if (__any_sync(0xffffffffu, late || *reinterpret_cast<volatile int*>(&sh.quit))) return false;
        }
    };
    uint32_t tmem = 0, t_s = 0, t_o = 0;
    auto together = [&] {                        // queries, barriers and tensor memory are there
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        tmem = t_s = sh.tmem;
        t_o = tmem + 256;
    };

    if (warp < 8) {
        more_registers<kLpSoftmaxRegs>();
        // ---- queries: a warp brings its 32 rows ----
        const int half = warp >> 2, row_in = tid & 127, i_row = rb * kPfCols + tid;
        const int row = i_row < n && first + i_row >= 0 && first + i_row < b.n_rows ? first + i_row : -1;
        const int limit = i_row < n ? sees(i_row) : 0;
        // (eight lanes a row, so that a row's largest magnitude is three exchanges away and nothing but the result goes through shared memory)
        const int oct = lane >> 3, unit = lane & 7, i0 = i_row - lane, there_to = min(n, b.n_rows - first);
        const bool tail = unit < a.kv.rope / 8;  // of the last chunk's units
        const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(a.q.p) + (first + static_cast<long long>(i0 + oct)) * a.q.row + (a.h0 + head) * a.q.head + unit * 8;
        const uint32_t to_at = q_at + half * S::k_bytes + ((row_in & ~31) + oct) * 128;
        float up = 1.f;                          // 2^e of this lane's row
#pragma unroll 1
        for (int g = 0; g < 8; g += kLpAtOnce) {
            uint4 v[kLpAtOnce][S::k_chunks];
#pragma unroll
            for (int k = 0; k < kLpAtOnce; ++k) {
                const int i = i0 + (g + k) * 4 + oct;
                const bool is = i < there_to && first + i >= 0;
#pragma unroll
                for (int c = 0; c < S::k_chunks; ++c) {
                    v[k][c] = make_uint4(0, 0, 0, 0);
                    if (is && (c + 1 < S::k_chunks || tail)) v[k][c] = *reinterpret_cast<const uint4*>(from + (g + k) * 4 * a.q.row + c * 64);
                }
            }
#pragma unroll
            for (int k = 0; k < kLpAtOnce; ++k) {
                uint32_t top = 0;                // as bf16 bits
#pragma unroll
                for (int c = 0; c < S::k_chunks; ++c) {
                    const uint32_t w[4] = {v[k][c].x, v[k][c].y, v[k][c].z, v[k][c].w};
#pragma unroll
                    for (int u = 0; u < 4; ++u) top = max(top, max(w[u] & 0x7fffu, w[u] >> 16 & 0x7fffu));
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float by = two_to(top == 0 || top >= 0x7f80u ? 0 : min(9 - (int(top >> 7) - 127), 120)), signed_by = a.factor < 0.f ? -by : by;
                const float of_row = __shfl_sync(0xffffffffu, by, (lane & 3) * 8);
                if (lane >> 2 == g + k) up = of_row;
#pragma unroll
                for (int c = 0; c < S::k_chunks; ++c) {
                    float x[8];
                    two_bf16(v[k][c].x, x[0], x[1]); two_bf16(v[k][c].y, x[2], x[3]); two_bf16(v[k][c].z, x[4], x[5]); two_bf16(v[k][c].w, x[6], x[7]);
                    st_shared16(to_at + c * S::chunk + (g + k) * 512 + ((unit ^ ((g + k) * 4 + oct & 7)) << 4),
                                make_uint4(pack_fp16(x[0] * signed_by, x[1] * signed_by), pack_fp16(x[2] * signed_by, x[3] * signed_by),
                                           pack_fp16(x[4] * signed_by, x[5] * signed_by), pack_fp16(x[6] * signed_by, x[7] * signed_by)));
                }
            }
        }
        fence_proxy_async();
        together();
        // ---- softmax: this thread's row is lane 32 (warp % 4) + lane of tensor memory ----
        const int own_tiles = half == 0 ? tiles0 : tiles1;
        const uint32_t lanes = uint32_t(warp & 3) << 21, s_at = t_s + half * 128 + lanes, o_at = t_o + half * HD + lanes;
        const float f = fmaxf(fabsf(a.factor) / up, 0x1p-149f);                // (not zero: masked scores are -infinity)
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        const uint4* bits = reinterpret_cast<const uint4*>(a.there + at / 32);
        const size_t first_32 = (size_t(head) * a.tokens + at) / 32;
        const short4 *powers_of = reinterpret_cast<const short4*>(a.value_exps + first_32), *units_of = reinterpret_cast<const short4*>(a.key_exps + first_32);
        uint4 bits_then = own_tiles > 0 ? bits[0] : make_uint4(0, 0, 0, 0);
        short4 powers_then = own_tiles > 0 ? powers_of[0] : make_short4(0, 0, 0, 0), units_then = own_tiles > 0 ? units_of[0] : powers_then;
        int run = -1000;                         // R
        for (int j = 0; j < own_tiles && ok; ++j) {
            uint32_t there[4] = {bits_then.x, bits_then.y, bits_then.z, bits_then.w};
            const int power[4] = {powers_then.x, powers_then.y, powers_then.z, powers_then.w};
            float unit[4] = {two_to(units_then.x), two_to(units_then.y), two_to(units_then.z), two_to(units_then.w)};
            if (j + 1 < own_tiles) { bits_then = bits[j + 1]; powers_then = powers_of[j + 1]; units_then = units_of[j + 1]; }
            bool whole = (j + 1) * kLpTile <= limit && (there[0] & there[1] & there[2] & there[3]) == 0xffffffffu;
            whole = __all_sync(0xffffffffu, whole);
            if (!(ok = wait(sh.s_full[half], j & 1))) break;
            tc_fence_after();
            if (!whole)                          // tokens that this row sees
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int left = limit - j * kLpTile - 32 * i;
                    if (left < 32) there[i] &= left <= 0 ? 0u : (1u << left) - 1;
                }
            uint32_t r[4][32];
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_at + 32 * ch, r[ch]);
            tmem_wait_ld();
            if (!whole)
#pragma unroll
                for (int ch = 0; ch < 4; ++ch)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(there[ch] >> i & 1)) r[ch][i] = 0xff800000u;
            float tops[4];
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) {
                tops[ch] = __uint_as_float(r[ch][0]);
#pragma unroll
                for (int i = 1; i < 32; ++i) tops[ch] = fmaxf(tops[ch], __uint_as_float(r[ch][i]));
            }
            const float peak = fmaxf(fmaxf(tops[0] * unit[0], tops[1] * unit[1]), fmaxf(tops[2] * unit[2], tops[3] * unit[3]));
            int power_top = -1000;               // of values that this row sees
#pragma unroll
            for (int ch = 0; ch < 4; ++ch)
                if (whole || there[ch] != 0) power_top = max(power_top, power[ch]);
            const bool any = (there[0] | there[1] | there[2] | there[3]) != 0;      // (rows that there are not would scale sums at every tile)
            // (a row moves its maximum when it has to and not with the warp's others, so that its bits are its own; one that is NaN already need not)
            const bool moves = (any && m == -INFINITY && l == l) || (peak - m) * f > kLpSlack;
            if (__any_sync(0xffffffffu, moves || power_top > run + kLpRoom)) {
                // (scores of a query with an infinity may all be -infinity, as those of tokens that it does not see are: NaN)
                if (any && m == -INFINITY && peak == -INFINITY) l = __int_as_float(0x7fffffff);
                const float to = moves ? fmaxf(m, peak) : m, by = m == -INFINITY ? 1.f : ex2((m - to) * f);
                m = to;
                l *= by;
                const int run_then = power_top > run + kLpRoom ? power_top : run;
                const float down = by * exp2f(float(max(run - run_then, -200)));
                run = run_then;
                if (j > 0) {                     // (before that the sums hold nothing)
#pragma unroll 1
                    for (int ch = 0; ch < HD / 16; ++ch) {
                        uint32_t o[16];
                        tmem_ld16_raw(o_at + 16 * ch, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * down);
                        tmem_st16(o_at + 16 * ch, o);
                    }
                }
            }
            float base = m == -INFINITY ? 0.f : -m * f;
            // Of large scores the rounding of this and of their own products is more than the range of fp16's exponents: rows that have such take the
            // differences from the maximum first, in its unit (below 2^8 the rounding is 2^-16 at most)
            const bool far = !(fabsf(base) < 256.f);
            if (__any_sync(0xffffffffu, far)) {
                const float from = far ? -m : 0.f;
                const unsigned long long from2 = two_floats(from, from);
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    const float by = far ? unit[ch] : 1.f;
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x0, x1;
                        floats_of(fma2(two_words(r[ch][i], r[ch][i + 1]), two_floats(by, by), from2), x0, x1);
                        r[ch][i] = __float_as_uint(x0);
                        r[ch][i + 1] = __float_as_uint(x1);
                    }
                    if (far) unit[ch] = 1.f;
                }
                if (far) base = 0.f;
            }
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) {
                // (values 2^60 below the largest are as good as zero, and yet their tokens' probabilities count)
                const float f_of = fmaxf(f * unit[ch], 0x1p-149f);
                const float shift = float(max(power[ch] - run, -60)), from = base + (kLpUp + shift);
                const unsigned long long from2 = two_floats(from, from), f2 = two_floats(f_of, f_of);
                unsigned long long sum0 = 0, sum1 = 0;
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    const unsigned long long x = fma2(two_words(r[ch][i], r[ch][i + 1]), f2, from2);
                    float p0, p1;
                    if (i % 8 == 2) floats_of(two_to2(x), p0, p1);             // two of eight
                    else {
                        floats_of(x, p0, p1);
                        p0 = ex2(p0); p1 = ex2(p1);
                    }
                    unsigned long long& sum = i & 2 ? sum1 : sum0;
                    sum = add2(sum, two_floats(p0, p1));
                    p[i / 2] = pack_fp16(p0, p1);
                }
                tmem_st16(s_at + 16 * ch, p);
                float x0, x1;
                floats_of(add2(sum0, sum1), x0, x1);
                l = fmaf(x0 + x1, ex2(-shift), l);
                if (ch & 1) {                    // 64 tokens' probabilities: their product need not wait for the others'
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(smem_u32(&sh.p_full[half][ch / 2]));
                }
            }
        }
        if (own_tiles > 0 && ok) ok = wait(sh.o_full[half], 0);
        tc_fence_after();
        if (ok) {
            // the rows go out by way of the half's queries' place, HD / 8 lanes a row
            constexpr int LANES = HD / 8, AT_ONCE = 32 / LANES;
            const float by = l == 0.f ? 0.f : exp2f(float(run)) / l;
            const uint32_t rows_at = q_at + half * S::k_bytes + (row_in & ~31) * (HD * 2);
#pragma unroll 1
            for (int ch = 0; ch < HD / 32; ++ch) {
                uint32_t r[32];
                if (own_tiles > 0) {
                    tmem_ld32(o_at + 32 * ch, r);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = 0u;
                }
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = __uint_as_float(r[i + k]) * by;
                    st_shared16(rows_at + lane * (HD * 2) + ((ch * 4 + i / 8 ^ lane & LANES - 1) << 4),
                                make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])));
                }
            }
            __syncwarp();
            __nv_bfloat16* to = row < 0 ? nullptr : static_cast<__nv_bfloat16*>(a.out.p) + row * a.out.row + (a.h0 + head) * a.out.head;
#pragma unroll 4
            for (int k = 0; k < LANES; ++k) {
                const int i = k * AT_ONCE + lane / LANES;
                auto* dst = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), i));
                const uint4 v = lds128(rows_at + i * (HD * 2) + ((lane % LANES ^ i & LANES - 1) << 4));
                if (dst) *reinterpret_cast<uint4*>(dst + lane % LANES * 8) = v;
            }
        }
    } else {
        fewer_registers<kLpOtherRegs>();
        bool ok = true;
        if (warp == 9) {
            // ---- keys and values on their way in (they need no queries: begun before the others are ready) ----
            const int row0 = head * a.tokens + at;
            const short4* units_of = reinterpret_cast<const short4*>(a.key_exps + (size_t(head) * a.tokens + at) / 32);
            short4 units = tiles > 0 ? units_of[0] : make_short4(0, 0, 0, 0);      // of the next tile's keys
            auto keys = [&](int j) {
                const int own[4] = {units.x, units.y, units.z, units.w};
                if (j + 1 < tiles) units = units_of[j + 1];
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&sh.k_full[j & 1]), to = k_at + (j & 1) * S::k_bytes, rope_to = to + HD / 64 * S::chunk;
                    const int own_row = row0 + j * kLpTile, shared = a.shared_row + at + j * kLpTile;
                    mbar_arrive_expect_tx(bar, S::k_bytes);
                    for (int c = 0; c < HD / 64; ++c) tma_rows(to + c * S::chunk, &k_map, c * 64, own_row, bar);
                    if ((own[0] | own[1] | own[2] | own[3]) == 0) tma_rows(rope_to, &rope_map, 0, shared, bar);
                    else                         // this head's copy where there is one
#pragma unroll
                        for (int k = 0; k < 4; ++k) tma_rows(rope_to + k * 32 * 128, &rope32_map, 0, (own[k] != 0 ? own_row : shared) + k * 32, bar);
                }
                __syncwarp();
            };
            auto values = [&](int j) {
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&sh.v_full[j % S::v_stages]), to = v_at + j % S::v_stages * S::v_bytes;
                    mbar_arrive_expect_tx(bar, S::v_bytes);
                    for (int c = 0; c < HD / 64; ++c) tma_rows(to + c * S::chunk, &v_map, c * 64, row0 + j * kLpTile, bar);
                }
                __syncwarp();
            };
            int k_sent = 0, v_sent = 0;
            if (tiles > 0) { keys(0); k_sent = 1; }
            together();                          // (values are not wanted before, and would be in the queries' way)
            if (tiles > 0) { values(0); v_sent = 1; }
            for (int j = 0; j < tiles; ++j) {
                if (j + 1 < tiles) {             // (their place is free before that of the values is)
                    if (j + 1 >= 2 && !(ok = wait(sh.k_empty[(j + 1) & 1], ((j + 1) / 2 - 1) & 1))) break;
                    keys(j + 1);
                    ++k_sent;
                }
                if (j > 0) {
                    if (j >= S::v_stages && !(ok = wait(sh.v_empty[j % S::v_stages], (j / S::v_stages - 1) & 1))) break;
                    values(j);
                    ++v_sent;
                }
            }
            // copies under way end before shared memory is given back, whoever has given up
            for (int j = max(0, k_sent - 2); j < k_sent; ++j) mbar_wait_bounded(smem_u32(&sh.k_full[j & 1]), j / 2 & 1, a.wait_ns);
            for (int j = max(0, v_sent - S::v_stages); j < v_sent; ++j) mbar_wait_bounded(smem_u32(&sh.v_full[j % S::v_stages]), j / S::v_stages & 1, a.wait_ns);
        } else {
            together();
            // ---- products. The warp walks as one, so that the elected lane is one lane throughout ----
            if (warp == 8) {
                constexpr uint32_t idesc_s = (1u << 4) | (uint32_t(kLpTile >> 3) << 17) | (uint32_t(kLpTile >> 4) << 24);        // fp16 x fp16 -> fp32
                constexpr uint32_t idesc_o = (1u << 4) | (1u << 16) | (uint32_t(HD >> 3) << 17) | (uint32_t(128 >> 4) << 24);
                const int rope_steps = a.kv.rope / 16;
                const uint64_t q_desc = smem_desc_sw128(q_at, 16, 1024), k_desc = smem_desc_sw128(k_at, 16, 1024), v_desc = smem_desc_sw128(v_at, S::chunk, 1024);
                const uint32_t hi = uint32_t(q_desc >> 32);
                auto scores = [&](int h, int j) {
                    if (elect_one()) {
                        const uint32_t d = t_s + h * 128, lo_q = uint32_t(q_desc) + h * (S::k_bytes >> 4), lo_k = uint32_t(k_desc) + (j & 1) * (S::k_bytes >> 4);
#pragma unroll
                        for (int k = 0; k < HD / 16; ++k) {
                            const uint32_t off = (k / 4) * (S::chunk >> 4) + (k % 4) * 2;
                            if (k == 0) tc_mma_lo<false>(d, lo_q, hi, lo_k, hi, idesc_s);
                            else tc_mma_lo<true>(d, lo_q + off, hi, lo_k + off, hi, idesc_s);
                        }
                        for (int k = 0; k < rope_steps; ++k) {
                            const uint32_t off = HD / 64 * (S::chunk >> 4) + k * 2;
                            tc_mma_lo<true>(d, lo_q + off, hi, lo_k + off, hi, idesc_s);
                        }
                        tc_commit(smem_u32(&sh.s_full[h]));
                    }
                    __syncwarp();
                };
                auto sums = [&](int h, int j, int part) {
                    if (elect_one()) {
                        const uint64_t v = v_desc + uint64_t(j % S::v_stages * (S::v_bytes >> 4));
#pragma unroll
                        for (int i = 0; i < kLpTile / 32; ++i) {
                            const int k = part * (kLpTile / 32) + i;
                            tc_mma_f16_ts(t_o + h * HD, t_s + h * 128 + 8 * k, v + uint64_t(k * 128), idesc_o, j > 0 || k > 0);
                        }
                    }
                    __syncwarp();
                };
                auto signal = [&](unsigned long long& bar) {
                    if (elect_one()) tc_commit(smem_u32(&bar));
                    __syncwarp();
                };
                const int count[2] = {tiles0, tiles1};
                bool any = false;
                ok = tiles == 0 || wait(sh.k_full[0], 0);
                tc_fence_after();
                if (ok && tiles > 0) {
                    any = true;
                    for (int h = 0; h < 2; ++h)
                        if (count[h] > 0) scores(h, 0);
                    signal(sh.k_empty[0]);
                }
                for (int j = 0; ok && j < tiles; ++j) {
                    const int vs = j % S::v_stages;
                    // (ahead of the probabilities, which come last)
                    if (j + 1 < tiles && !(ok = wait(sh.k_full[(j + 1) & 1], (j + 1) / 2 & 1))) break;
                    if (!(ok = wait(sh.v_full[vs], j / S::v_stages & 1))) break;
                    tc_fence_after();
                    for (int h = 0; h < 2; ++h) {
                        if (j < count[h]) {
                            for (int part = 0; part < 2 && ok; ++part) {
                                if (!(ok = wait(sh.p_full[h][part], j & 1))) break;
                                tc_fence_after();
                                sums(h, j, part);
                            }
                            if (!ok) break;
                            if (j + 1 == count[h]) signal(sh.o_full[h]);
                        }
                        if (h == 1) signal(sh.v_empty[vs]);      // (ahead of the next scores)
                        if (j + 1 < count[h]) {
                            scores(h, j + 1);
                        }
                    }
                    if (!ok) break;
                    if (j + 1 < tiles) signal(sh.k_empty[(j + 1) & 1]);
                }
                if (any) {                       // products under way end before tensor memory is given back, whoever has given up
                    signal(sh.drained);
                    mbar_wait_bounded(smem_u32(&sh.drained), 0, 2'000'000'000ull);
                    __syncwarp();
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
}

}  // namespace spm
