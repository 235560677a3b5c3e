// Attention of many bf16 rows a sequence (prompts) over the 4-bit cache, on tcgen05.
//
// A CTA takes 256 columns (column x: head x % group of row x / group) of one cache head, two M = 128 halves, and walks the tokens in tiles
// of 128. Four warps bring a tile's codes to fp16 operands in shared memory, once for both halves; one warp issues the products; four
// warps a half turn scores into probabilities, one row a thread, while the tensor cores are at the other half: S(j) of one half, then
// P V(j) and S(j + 1) of the other. Scores, probabilities (fp16, in the scores' place, as the A operand of the second product) and sums
// stay in tensor memory: 2 x 128 + 2 x HD columns.
//
// fp16 and not bf16 operands, since a bf16 rounding of probabilities and values would each cost as much as that of the result. Ranges are
// kept by powers of two, which round nothing: a row's queries are brought to [2^9, 2^10) by its largest, keys of a tile in which one would
// not fit are taken times 2^-4, a probability times 2^8 (it is at most 2^6 above the running maximum, see below), and values times 2^-E, E
// from the largest scale so far (a tile whose values would not fit raises E, and the sums so far are scaled down).
//
// A row's maximum is moved, and its sums scaled, only where a score is above it by more than 2^6.
//
// What bounds it, a CTA's tile of 128 tokens for 256 columns: 4017 cycles. The halves take turns, 2250 cycles of softmax and 1770 of products
// with their hand-over; the exponentials (128 x 256 at 16 a cycle), the products and the shared memory that these read are 2050 each. Four
// prompts of up to 2049 rows after up to 2048 tokens, 32 heads: 236 us, 0.78 PFLOP/s (the cycles are of 228 us, before exponents were taken from
// differences and waits by whole warps), of which an item's start and end (search 2 us, queries 3, first scores 1.6, rows out 2.5) are a fifth.
// Slower: waits with a time hint (262 us for 245 then), steps of 64 tokens with two score buffers a half (262), probabilities against the old
// maximum held in registers (311, spills).
#pragma once

#include "kv_attend.cuh"
#include "tc_ops.cuh"

namespace spm {

constexpr int kPfTile = 128;                     // tokens of a tile, rows of a half
constexpr int kPfCols = 256;
// two halves' softmax warps, operand warps, the issuing warp and three that only make its four whole. Registers a thread: 128 at the launch,
// of which the last two fours give some to the softmax warps (2 x 176 + 104 + 56 = 4 x 128).
constexpr int kPfThreads = 16 * 32;
constexpr int kPfSoftmaxRegs = 176, kPfOperandRegs = 104, kPfIssueRegs = 56;
static_assert(2 * kPfSoftmaxRegs + kPfOperandRegs + kPfIssueRegs == 4 * 128, "the split is what the launch has");
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int HD>
struct PfShape {
    static constexpr int block_bytes = kPfTile * 128;                    // 64 elements of 128 rows
    static constexpr int op_bytes = HD / 64 * block_bytes;               // one operand tile
    static constexpr int smem = 6 * op_bytes + 1024;                     // queries of two halves, two stages of keys and values
};

// A in tensor memory
__device__ __forceinline__ void pf_mma_ts(uint32_t d, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}\n"
        ::"r"(d), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// fp16 x fp16 -> fp32, M = 128
__host__ __device__ constexpr uint32_t pf_idesc(int n, bool b_mn_major) {
    return (1u << 4) | (uint32_t(b_mn_major) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(128 >> 4) << 24);
}
#define PF_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define PF_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
        "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : PF_R8(r, 0), PF_R8(r, 8), PF_R8(r, 16), PF_R8(r, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_ld16_raw(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : PF_R8(r, 0), PF_R8(r, 8) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::PF_W8(r, 0), PF_W8(r, 8), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }


// Eight codes of a word as fp16 elements times a scale, in the order (0, 4, 1, 5, 2, 6, 3, 7): 1024 + q (low nibbles of the masked halves)
// less 1032, 1024 + 16 q over 16 less 72, both exact, then one rounding
__device__ __forceinline__ uint4 pf_expand(uint32_t w, __half2 s) {
    const __half2 off = as_half2(0xe408e408u), sixteenth = as_half2(0x2c002c00u), off72 = as_half2(0xd480d480u);       // -1032, 1 / 16, -72
    const uint32_t h = w >> 8;
    return make_uint4(bits_of(__hmul2(__hadd2(as_half2((w & 0x000f000fu) | 0x64006400u), off), s)),
                      bits_of(__hmul2(__hfma2(as_half2((w & 0x00f000f0u) | 0x64006400u), sixteenth, off72), s)),
                      bits_of(__hmul2(__hadd2(as_half2((h & 0x000f000fu) | 0x64006400u), off), s)),
                      bits_of(__hmul2(__hfma2(as_half2((h & 0x00f000f0u) | 0x64006400u), sixteenth, off72), s)));
}
__device__ __forceinline__ void st_shared16(uint32_t at, const uint4& v) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// 16-byte chunk `ch` (eight elements) of a row of an operand tile: 128-byte rows of 64 elements, swizzled
__device__ __forceinline__ uint32_t pf_chunk(int row, int ch) {
    return uint32_t((ch >> 3) * (kPfTile * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
}

struct PfShared {
    unsigned long long k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2], drained;
    uint32_t tmem;
    int quit;                                    // a wait has run out: everybody leaves
    int rb, seq, first, n, len;                  // the item: its columns, its sequence's rows and tokens
    int exps[4];                                 // E of a tile, and whether its keys are times 2^-4 (bit 16)
    int widest[4], widest_key[4];                // an operand warp's largest scale of a tile's values and keys, as fp32 bits
    uint32_t there[4][4];                        // which tokens of a tile exist
};

// 16 bytes to shared memory, or zeros, without a register on the way; then: this thread's have arrived.
__device__ __forceinline__ void copy16_or_zero(uint32_t at, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Sequences of a batch of prompts that are not for the kernel below: it walks an item's tokens one after another, so a few of few columns over
// many tokens are better shared out between all SMs. They are those of over twice the tokens that the batch's columns see in the mean, if
// all of them together are less than a round of CTAs has of columns times heads over the longest one's tokens (`few`, from where on the kernel
// below is the faster one). One block, a thread a sequence; rows_few, rows_many: each sequence's rows in the one place, 0 in the other.
// A prompt of 2048 rows and seven sequences of 100 000 tokens: 172 us, 1911 without; a batch without such sequences takes 6 us more.
constexpr int kPfLongTokens = 8192;              // an item of no more tokens than that ends soon enough wherever it is
__global__ void __launch_bounds__(SPM_KV_MAX_SEQS) kv_split_kernel(const AttendArgs a, int few, int* rows_few, int* rows_many) {
    __shared__ unsigned long long sums[3][32];
    __shared__ int tops[32];
    grid_dep_wait();
    grid_dep_launch();
    const int s = threadIdx.x, lane = s & 31, warp = s >> 5;
    int n = 0, len = 0;
    if (s < a.batch.n_seq) {
        n = max(0, min(a.batch.row_start[s + 1] - a.batch.row_start[s], a.batch.n_rows));
        len = max(0, min(a.batch.lengths[s], a.batch.stride * a.kv.page_size));
    }
    auto over_all = [&](unsigned long long v, unsigned long long (&at)[32]) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) at[warp] = v;
    };
    auto sum_of = [](const unsigned long long (&at)[32]) {
        unsigned long long v = 0;
#pragma unroll
        for (int w = 0; w < 32; ++w) v += at[w];
        return v;
    };
    const unsigned long long columns = static_cast<unsigned long long>(n) * a.group, seen = columns * len;
    over_all(columns, sums[0]);
    over_all(seen, sums[1]);
    __syncthreads();
    const bool out = len > kPfLongTokens && n > 0 && len * sum_of(sums[0]) > 2 * sum_of(sums[1]);
    over_all(out ? seen : 0, sums[2]);
    const int top = __reduce_max_sync(0xffffffffu, out ? len : 0);
    if (lane == 0) tops[warp] = top;
    __syncthreads();
    const int longest = __reduce_max_sync(0xffffffffu, tops[lane]);
    const bool all_out = sum_of(sums[2]) * a.kv.heads <= static_cast<unsigned long long>(few) * longest;
    if (s >= a.batch.n_seq) return;
    rows_few[s] = out && all_out ? n : 0;
    rows_many[s] = out && all_out ? 0 : n;
}

template <int HD>
__global__ void __launch_bounds__(kPfThreads, 1) kv_prefill_kernel(const AttendArgs a) {
    using S = PfShape<HD>;
    constexpr int G = HD / 32;
    extern __shared__ unsigned char raw_smem[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem), q_at = base, k_at = base + 2 * S::op_bytes, v_at = base + 4 * S::op_bytes;
    __shared__ PfShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvBatch& b = a.batch;

    grid_dep_wait();
    grid_dep_launch();
    // ---- which item, heads together. Up to 32 sequences: those of the most tokens first, so that what is left at the end is short; more:
    // one sequence after another, its last (longest) columns first. A warp searches, others prepare what all items need ----
    const int head = blockIdx.x % a.kv.heads, cap = b.stride * a.kv.page_size;
    if (warp == 13) {
        int block = blockIdx.x / a.kv.heads;
        if (lane == 0) sh.n = 0;
        __syncwarp();
        for (int s0 = 0; s0 < b.n_seq; s0 += 32) {
            const int s = s0 + lane;
            int f = s, m = s < b.n_seq ? 1 : 0;
            if (b.row_start && s < b.n_seq) {
                f = b.row_start[s];
                m = a.rows ? a.rows[s] : max(0, min(b.row_start[s + 1] - f, b.n_rows));
            }
            const int len = s < b.n_seq ? b.lengths[s] : 0, tokens = max(0, min(len, cap));
            const int own = (m * a.group + kPfCols - 1) / kPfCols;               // (a call's rows times heads fit)
            auto running = [&](int v) {
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int w = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += w;
                }
                return v;
            };
            int before = running(own) - own;
            const int all = __shfl_sync(0xffffffffu, before + own, 31);
            if (block >= all) { block -= all; continue; }
            int ours = own, skip = 0;            // of this sequence's items, longest first: `ours` after `skip`
            if (b.n_seq <= 32) {
                // items whose first row sees `t` tokens and more
                auto at_least = [&](int t) {
                    if (t <= 0) return own;
                    if (t > tokens) return 0;
                    return max(0, own - int(unsigned(max(0, min(t - 1 - (len - m), m)) * a.group + kPfCols - 1) / kPfCols));
                };
                int low = 0, high = __reduce_max_sync(0xffffffffu, tokens) + 1;  // `low`: the most tokens that more than `block` items have
                while (high - low > 1) {         // (eight parts at a time: seven sums that do not wait for one another)
                    const int step = (high - low + 7) / 8;
                    int above = 0;
#pragma unroll
                    for (int i = 1; i < 8; ++i) above += int(__reduce_add_sync(0xffffffffu, at_least(low + i * step))) > block;
                    low += above * step;
                    high = min(high, low + step);
                }
                skip = at_least(low + 1);
                ours = at_least(low) - skip;
                block -= __reduce_add_sync(0xffffffffu, skip);
                before = running(ours) - ours;
            }
            if (before <= block && block < before + ours) {
                sh.rb = own - 1 - skip - (block - before);
                sh.seq = s; sh.first = f; sh.n = m; sh.len = len;
            }
            break;
        }
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 128); mbar_init(smem_u32(&sh.v_full[i]), 128);
            mbar_init(smem_u32(&sh.k_empty[i]), 1); mbar_init(smem_u32(&sh.v_empty[i]), 1);
            mbar_init(smem_u32(&sh.s_full[i]), 1); mbar_init(smem_u32(&sh.p_full[i]), 128 + a.withhold); mbar_init(smem_u32(&sh.o_full[i]), 1);
        }
        mbar_init(smem_u32(&sh.drained), 1);
        sh.quit = 0;
        fence_barrier_init();
    }
    if (warp == 12) tmem_alloc(smem_u32(&sh.tmem), 512);
    __syncthreads();
    const int rb = sh.rb, seq = sh.seq, first = sh.first, n = sh.n, len = sh.len;
    if (n == 0) {                                // more CTAs than items
        tc_fence_before();
        if (warp == 12) tmem_dealloc(sh.tmem, 512);
        return;
    }
    if (len > cap && rb == 0 && head == 0 && tid == 0) kv_note(a.kv, SPM_KV_TOO_LONG);
    // tiles of a half: up to the token that its last row sees
    auto sees = [&](int x) { return max(0, min(len - n + min(n - 1, column_row(a, x)) + 1, cap)); };
    const bool used1 = rb * kPfCols + kPfTile < n * a.group;
    const int tiles0 = (sees(rb * kPfCols + kPfTile - 1) + kPfTile - 1) / kPfTile;
    const int tiles1 = used1 ? (sees(rb * kPfCols + kPfCols - 1) + kPfTile - 1) / kPfTile : 0;
    const int tiles = max(tiles0, tiles1);

    // a warp goes on, or gives up, as one: what follows is for all of its lanes together
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

    // ---- queries: a softmax warp brings its 32 rows, HD / 8 lanes a row; then a lane has a row (swizzled as the operand is: no two lanes
    // of a quarter meet in a bank) ----
    constexpr int LANES = HD / 8, AT_ONCE = 32 / LANES;
    const int half = warp >> 2, row_in = tid & 127;             // (softmax warps: 0 - 3, 4 - 7)
    int row = -1, g = 0, limit = 0;
    float f = 1.f;
    if (warp < 8) {
        const int x = rb * kPfCols + tid, i = column_row(a, x);
        g = x - i * a.group;
        if (i < n && first + i >= 0 && first + i < b.n_rows) row = first + i;
        limit = sees(x);
        if (i >= n) limit = 0;
        const __nv_bfloat16* src = row < 0 ? nullptr : static_cast<const __nv_bfloat16*>(a.q.p) + row * a.q.row + (head * a.group + g) * a.q.head;
        const uint32_t to = q_at + half * S::op_bytes;
#pragma unroll 4
        for (int k = 0; k < LANES; ++k) {
            const int i = k * AT_ONCE + lane / LANES;
            const auto* from = reinterpret_cast<const __nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(src), i));
            copy16_or_zero(to + pf_chunk((row_in & ~31) + i, lane % LANES), from ? from + lane % LANES * 8 : a.q.p, from != nullptr);
        }
        copies_arrived();
        __syncwarp();
        uint32_t top = 0;                        // this lane's row: its largest magnitude, as bf16 bits
#pragma unroll 4
        for (int ch = 0; ch < LANES; ++ch) {
            const uint4 v = lds128(to + pf_chunk(row_in, ch));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7fffu, w[j] >> 16 & 0x7fffu));
        }
        // to [2^9, 2^10). A row with a NaN or an infinity becomes NaN as a whole: infinite scores could all be -infinity, as those of tokens
        // that it does not see are
        const int e = top == 0 || top >= 0x7f80u ? 0 : 9 - (int(top >> 7) - 127);
        const float up = top < 0x80u ? 0x1p100f : exp2f(float(min(e, 120))), sign = top >= 0x7f80u ? __int_as_float(0x7fffffff) : a.scale < 0.f ? -up : up;
        f = fminf(fmaxf(fabsf(a.scale) * 1.4426950408889634f / up, kAtLeast), kAtMost);
#pragma unroll 4
        for (int ch = 0; ch < LANES; ++ch) {
            const uint32_t at = to + pf_chunk(row_in, ch);
            const uint4 v = lds128(at);
            float q[8];
            two_bf16(v.x, q[0], q[1]); two_bf16(v.y, q[2], q[3]); two_bf16(v.z, q[4], q[5]); two_bf16(v.w, q[6], q[7]);
            st_shared16(at, make_uint4(pack_half(q[0] * sign, q[4] * sign), pack_half(q[1] * sign, q[5] * sign),
                                       pack_half(q[2] * sign, q[6] * sign), pack_half(q[3] * sign, q[7] * sign)));
        }
        fence_proxy_async();
    }
    uint32_t tmem = 0, t_s = 0, t_o = 0;
    auto together = [&] {                        // queries, barriers and tensor memory are there; each role has begun what needs none of them
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        tmem = t_s = sh.tmem;
        t_o = tmem + 256;
    };
    const int own_tiles = half == 0 ? tiles0 : tiles1;

    if (warp < 8) {
        more_registers<kPfSoftmaxRegs>();
        together();
        // ---- softmax: this thread's row is lane 32 (warp % 4) + lane of tensor memory ----
        const uint32_t lanes = uint32_t(warp & 3) << 21, s_at = t_s + half * 128 + lanes, o_at = t_o + half * HD + lanes;
        float m = -INFINITY, l = 0.f;
        const float slack = 6.f / f;
        int e_now = 0;
        bool ok = true;
        for (int j = 0; j < own_tiles && ok; ++j) {
            if (!(ok = wait(sh.s_full[half], j & 1))) break;
            tc_fence_after();
            const int packed = *reinterpret_cast<volatile int*>(&sh.exps[j & 3]), e = int(short(packed & 0xffff));
            const float units = packed >> 16 & 1 ? 16.f : 1.f;
            uint32_t there[4];
            bool whole = (j + 1) * kPfTile <= limit;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                there[i] = *reinterpret_cast<volatile uint32_t*>(&sh.there[j & 3][i]);
                whole &= there[i] == 0xffffffffu;
            }
            whole = __all_sync(0xffffffffu, whole);
            if (!whole)                          // tokens that this row sees
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int left = limit - j * kPfTile - 32 * i;
                    if (left < 32) there[i] &= left <= 0 ? 0u : (1u << left) - 1;
                }
            uint32_t r[4][32];
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_at + 32 * ch, r[ch]);
            tmem_wait_ld();
            if (!whole) {
#pragma unroll
                for (int ch = 0; ch < 4; ++ch)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(there[ch] >> i & 1)) r[ch][i] = 0xff800000u;
            }
            float tops[4];
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) {
                tops[ch] = __uint_as_float(r[ch][0]);
#pragma unroll
                for (int i = 1; i < 32; ++i) tops[ch] = fmaxf(tops[ch], __uint_as_float(r[ch][i]));
            }
            // m is in scores of whole keys
            const float peak = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * units;
            if (__any_sync(0xffffffffu, peak - m > slack || e != e_now)) {
                const float to = fmaxf(m, peak), by = m == -INFINITY ? 0.f : ex2((m - to) * f);
                m = to;
                l *= by;
                if (j > 0) {                     // (before that the sums hold nothing)
                    const float scale = by * exp2f(float(e_now - e));
#pragma unroll 1
                    for (int ch = 0; ch < HD / 16; ++ch) {
                        uint32_t o[16];
                        tmem_ld16_raw(o_at + 16 * ch, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * scale);
                        tmem_st16(o_at + 16 * ch, o);
                    }
                }
                e_now = e;
            }
            // the difference from the maximum first: of large scores times f the rounding alone is more than the range of fp16's exponents
            const float base = m == -INFINITY ? 0.f : -m;
            const unsigned long long units2 = two_floats(units, units), base2 = two_floats(base, base), f2 = two_floats(f, f), eight2 = two_floats(8.f, 8.f);
            unsigned long long sum0 = 0, sum1 = 0;
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    float x0, x1;
                    floats_of(fma2(fma2(two_words(r[ch][i], r[ch][i + 1]), units2, base2), f2, eight2), x0, x1);
                    const float p0 = ex2(x0), p1 = ex2(x1);
                    unsigned long long& sum = i & 2 ? sum1 : sum0;
                    sum = add2(sum, two_floats(p0, p1));
                    p[i / 2] = pack_half(p0, p1);
                }
                tmem_st16(s_at + 16 * ch, p);
            }
            {
                float x0, x1;
                floats_of(add2(sum0, sum1), x0, x1);
                l += x0 + x1;
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&sh.p_full[half]));
        }
        if (own_tiles > 0 && ok) ok = wait(sh.o_full[half], 0);
        tc_fence_after();
        if (ok) {
            // values stand at 2^-E, probabilities and their sum at 2^8. The rows go out by way of the half's queries' place, HD / 8 lanes a row
            const float by = l == 0.f ? 0.f : exp2f(float(e_now)) / l;
            const uint32_t rows_at = q_at + half * S::op_bytes + (row_in & ~31) * (HD * 2);
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
                    for (int k = 0; k < 4; ++k) {                // (0, 4, 1, 5, 2, 6, 3, 7)
                        y[k] = __uint_as_float(r[i + 2 * k]) * by;
                        y[k + 4] = __uint_as_float(r[i + 2 * k + 1]) * by;
                    }
                    st_shared16(rows_at + lane * (HD * 2) + ((ch * 4 + i / 8 ^ lane & LANES - 1) << 4),
                                make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])));
                }
            }
            __syncwarp();
            __nv_bfloat16* to = row < 0 ? nullptr : static_cast<__nv_bfloat16*>(a.out.p) + row * a.out.row + (head * a.group + g) * a.out.head;
#pragma unroll 4
            for (int k = 0; k < LANES; ++k) {
                const int i = k * AT_ONCE + lane / LANES;
                auto* dst = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), i));
                const uint4 v = lds128(rows_at + i * (HD * 2) + ((lane % LANES ^ i & LANES - 1) << 4));
                if (dst) *reinterpret_cast<uint4*>(dst + lane % LANES * 8) = v;
            }
        }
    } else if (warp < 12) {
        fewer_registers<kPfOperandRegs>();
        // ---- operands: a thread takes a token of each tile, its codes a tile ahead ----
        const int t = tid - 256, w = warp - 8;
        const int nk = max(sees(rb * kPfCols + kPfTile - 1), used1 ? sees(rb * kPfCols + kPfCols - 1) : 0);
        const int per_page = a.kv.page_size / kKvBlock;
        const int* table = b.table + static_cast<size_t>(seq) * b.stride;
        const int tok = t % kKvBlock;
        uint4 kc[G], vc[G];
        uint32_t ks[G / 2], vs[G / 2], ks_then[G / 2], vs_then[G / 2];
        // where this thread's token of tile j is; its page has been loaded a tile before (-2: there is no such token)
        auto slot_of = [&](int j) {
            const int block = (j * kPfTile + t) / kKvBlock;
            return a.page_shift >= 0 ? block >> a.page_shift : block / per_page;
        };
        auto page_of = [&](int j) { return j * kPfTile + t < nk ? table[slot_of(j)] : -2; };
        const unsigned char* at = nullptr;
        bool exists = false;
        auto locate = [&](int j, int page) {
            exists = page >= 0 && page < a.kv.n_pages;
            if (!exists && page != -2) kv_note(a.kv, SPM_KV_BAD_PAGE);
            const int block = (j * kPfTile + t) / kKvBlock - slot_of(j) * per_page;
            at = a.kv.pages + ((static_cast<long long>(exists ? page : 0) * a.kv.heads + head) * per_page + block) * kv_block_bytes(HD) + tok * 16;
        };
        auto scales = [&](uint32_t (&s)[G / 2], int part) {
            const unsigned char* p = at + kv_k_scales(HD) + part * HD + tok * (2 * G - 16);
#pragma unroll
            for (int i = 0; i < G / 2; ++i) s[i] = exists ? *reinterpret_cast<const uint32_t*>(p + 4 * i) : 0u;
        };
        auto codes = [&](uint4 (&x)[G], int part) {
#pragma unroll
            for (int k = 0; k < G; ++k)
                x[k] = exists ? *reinterpret_cast<const uint4*>(at + part * kv_v_codes(HD) + k * (kKvBlock * 16)) : make_uint4(0, 0, 0, 0);
        };
        auto expand = [&](uint32_t to, const uint4 (&x)[G], const uint32_t (&s)[G / 2], float by) {
            const uint32_t row_at = to + t * 128 + ((t & 7) << 4);               // (tiles start on 1024 bytes)
#pragma unroll
            for (int k = 0; k < G; ++k) {
                const float2 pair = __half22float2(as_half2(s[k / 2]));
                const __half2 d = __float2half2_rn((k & 1 ? pair.y : pair.x) * by);
                const uint32_t word[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) st_shared16((row_at ^ ((4 * k + i & 7) << 4)) + (k >> 1) * S::block_bytes, pf_expand(word[i], d));
            }
        };
        auto largest = [&](const uint32_t (&s)[G / 2]) {
            __half2 m = __habs2(as_half2(s[0]));
#pragma unroll
            for (int i = 1; i < G / 2; ++i) m = __hmax2_nan(m, __habs2(as_half2(s[i])));
            return __half2float(__hmax_nan(__low2half(m), __high2half(m)));
        };
        int page = -2;
        if (tiles > 0) {
            const int first_page = page_of(0);
            if (tiles > 1) page = page_of(1);
            locate(0, first_page);
            scales(ks, 0); scales(vs, 1);
            codes(kc, 0); codes(vc, 1);
        }
        together();
        int e = -1000;                           // E keeps eight times the largest scale of values so far, times 2^-E, below 2^15
        float v_limit = -1.f, by_v = 1.f;        // the largest scale that E allows, 2^-E
        bool ok = true;                          // (a warp that has given up still comes to the others' barrier)
        for (int j = 0; j < tiles; ++j) {
            const uint32_t have = __ballot_sync(0xffffffffu, exists);
            if (lane == 0) sh.there[j & 3][w] = have;
            const float wide = largest(vs), wide_key = largest(ks);
            const bool keys_fit = wide_key < 8192.f;                             // eight times it is below 2^16
            int any;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
                         : "=r"(any) : "r"(int(!(wide <= v_limit) || !keys_fit)) : "memory");
            bool down = false;
            if (any) {                           // (seldom, but for the first tile)
                if (lane == 0) sh.widest[w] = sh.widest_key[w] = 0;
                __syncwarp();
                atomicMax(&sh.widest[w], __float_as_int(wide < INFINITY ? wide : 0.f));
                atomicMax(&sh.widest_key[w], __float_as_int(wide_key));
                asm volatile("bar.sync 1, 128;" ::: "memory");
                float widest = 0.f, widest_key = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    widest = fmaxf(widest, __int_as_float(*reinterpret_cast<volatile int*>(&sh.widest[i])));
                    widest_key = fmaxf(widest_key, __int_as_float(*reinterpret_cast<volatile int*>(&sh.widest_key[i])));
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                down = !(widest_key < 8192.f);
                if (widest > v_limit || e == -1000) {
                    const int need = widest > 0.f ? ilogbf(widest) + 4 : 0;      // eight times it is below 2^need
                    e = need - 8;                // (a little room, so that E is raised seldom)
                    v_limit = exp2f(float(e + 15 - 3)) * 0.999f;
                    by_v = exp2f(float(-e));
                }
            }
            if (t == 0) sh.exps[j & 3] = (e & 0xffff) | int(down) << 16;
            const int st = j & 1;
            if (ok && j >= 2) ok = wait(sh.k_empty[st], (j / 2 - 1) & 1);
            const bool more = j + 1 < tiles;
            if (ok) {
                expand(k_at + st * S::op_bytes, kc, ks, down ? 1.f / 16.f : 1.f);
                fence_proxy_async();
                mbar_arrive(smem_u32(&sh.k_full[st]));
                if (more) {
                    locate(j + 1, page);
                    scales(ks_then, 0); scales(vs_then, 1);
                    codes(kc, 0);
                }
                if (j + 2 < tiles) page = page_of(j + 2);
                if (j >= 2) ok = wait(sh.v_empty[st], (j / 2 - 1) & 1);
            }
            if (ok) {
                expand(v_at + st * S::op_bytes, vc, vs, by_v);
                fence_proxy_async();
                mbar_arrive(smem_u32(&sh.v_full[st]));
                if (more) codes(vc, 1);
            }
#pragma unroll
            for (int i = 0; i < G / 2; ++i) { ks[i] = ks_then[i]; vs[i] = vs_then[i]; }
        }
    } else {
        fewer_registers<kPfIssueRegs>();
        together();
        // ---- products. The warp walks as one, so that the elected lane is one lane throughout, and what it commits at the end covers all that it
        // has issued (a lane by itself, which computes its descriptors: 260 us for 236) ----
        if (warp == 12) {
            constexpr uint32_t idesc_s = pf_idesc(kPfTile, false), idesc_o = pf_idesc(HD, true);
            auto scores = [&](int h, int st) {
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < HD / 16; ++k) {
                        const uint32_t off = (k / 4) * S::block_bytes + (k % 4) * 32;
                        tc_mma_f16(t_s + h * 128, smem_desc_sw128(q_at + h * S::op_bytes + off, 16, 1024),
                                   smem_desc_sw128(k_at + st * S::op_bytes + off, 16, 1024), idesc_s, k > 0);
                    }
                    tc_commit(smem_u32(&sh.s_full[h]));
                }
                __syncwarp();
            };
            auto sums = [&](int h, int st, bool more) {
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kPfTile / 16; ++k)
                        pf_mma_ts(t_o + h * HD, t_s + h * 128 + 8 * k, smem_desc_sw128(v_at + st * S::op_bytes + k * 2048, S::block_bytes, 1024),
                                  idesc_o, more || k > 0);
                }
                __syncwarp();
            };
            auto signal = [&](unsigned long long& bar) {
                if (elect_one()) tc_commit(smem_u32(&bar));
                __syncwarp();
            };
            const int count[2] = {tiles0, tiles1};
            bool ok = tiles == 0 || wait(sh.k_full[0], 0);
            tc_fence_after();
            if (ok && tiles > 0) {
                for (int h = 0; h < 2; ++h)
                    if (count[h] > 0) scores(h, 0);
                signal(sh.k_empty[0]);
            }
            for (int j = 0; ok && j < tiles; ++j) {
                const int st = j & 1, next = (j + 1) & 1;
                bool keys = false;                   // of the next tile have been waited for
                if (!(ok = wait(sh.v_full[st], (j / 2) & 1))) break;
                for (int h = 0; h < 2; ++h) {
                    if (j < count[h]) {
                        if (!(ok = wait(sh.p_full[h], j & 1))) break;
                        tc_fence_after();
                        sums(h, st, j > 0);
                        if (j + 1 == count[h]) signal(sh.o_full[h]);
                    }
                    if (j + 1 < count[h]) {
                        if (!keys && !(ok = wait(sh.k_full[next], ((j + 1) / 2) & 1))) break;
                        keys = true;
                        tc_fence_after();
                        scores(h, next);
                    }
                }
                if (!ok) break;
                signal(sh.v_empty[st]);
                if (j + 1 < tiles) signal(sh.k_empty[next]);
            }
            if (tiles > 0) {                         // products under way end before tensor memory is given back, whoever has given up
                signal(sh.drained);
                mbar_wait_bounded(smem_u32(&sh.drained), 0, 2'000'000'000ull);
                __syncwarp();
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 12) tmem_dealloc(tmem, 512);
}

}  // namespace spm
