// The attention block of a decode step, as spm.cu keeps and enqueues it (attention_block.cu).
#pragma once

#include <string>
#include <vector>

#include <cuda_runtime.h>

#include "../../include/spm.h"

namespace spm {

struct AttentionBlock {
    spm_attention a{};
    std::vector<spm_kv_cache> caches;
    bool on = false;
};
// Kernels that one layer's block is
constexpr int kAttentionLaunches = 7;

size_t attention_bytes(const spm_model_cfg& m, const spm_attention& a);
// SPM_OK or the status of what is wrong, with a message
int check_attention(const spm_model_cfg& m, const spm_attention* a, std::string* why);
// `timed`: for its time alone. The cache and its status word stay as they are (k and v are cut to codes that go nowhere).
int enqueue_attention(const AttentionBlock& block, const spm_model_cfg& m, int layer, float* h, int nb, cudaStream_t stream, std::string* why,
                      bool timed = false);

}  // namespace spm
