// Which rows of which sequence a block of attention over prompts takes.
#pragma once

#include "kv_cache.cuh"

namespace spm {

constexpr int kPfCols = 256;                     // columns of a block: heads that share a cache head, times rows

struct PfItem { int rb, seq, first, n, len; };   // its columns from rb * kPfCols on; its sequence's first row, rows (0: there is no such item) and tokens

// Item `block`, by a warp. Up to 32 sequences: those of the most tokens first, so that what is left at the end is short; more:
// one sequence after another, its last (longest) columns first. rows: each sequence's rows that count; NULL: all of them.
__device__ __forceinline__ void pf_find(const KvBatch& b, const int* rows, int group, int cap, int block, PfItem& item) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) item.n = 0;
    __syncwarp();
    for (int s0 = 0; s0 < b.n_seq; s0 += 32) {
        const int s = s0 + lane;
        int f = s, m = s < b.n_seq ? 1 : 0;
        if (b.row_start && s < b.n_seq) {
            f = b.row_start[s];
            m = rows ? rows[s] : max(0, min(b.row_start[s + 1] - f, b.n_rows));
        }
        const int len = s < b.n_seq ? b.lengths[s] : 0, tokens = max(0, min(len, cap));
        const int own = (m * group + kPfCols - 1) / kPfCols;               // (a call's rows times heads fit)
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
                return max(0, own - int(unsigned(max(0, min(t - 1 - (len - m), m)) * group + kPfCols - 1) / kPfCols));
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
            item.rb = own - 1 - skip - (block - before);
            item.seq = s; item.first = f; item.n = m; item.len = len;
        }
        break;
    }
}

}  // namespace spm
