// The attention block of a decode step: projections, and the calls of the key/value cache between them.
#include "attention_block.h"

#include <algorithm>
#include <cmath>

#include "project.cuh"

namespace spm {

namespace {

bool fp32_model(const spm_model_cfg& m) { return m.dtype == SPM_DTYPE_FP32; }
int q_width(const spm_attention& a) { return a.n_q_heads * a.caches[0].head_dim; }
int qkv_width(const spm_attention& a) { return (a.n_q_heads + 2 * a.caches[0].n_kv_heads) * a.caches[0].head_dim; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// a layer's work memory, in this order
struct Work { size_t rows, qkv, out, attend; };
Work work_of(const spm_model_cfg& m, const spm_attention& a) {
    const size_t nb = m.max_batch, k = std::max(m.hidden, q_width(a));
    spm_kv_batch b = a.batch;
    b.row_start = nullptr;
    b.n_rows = b.n_seq;
    size_t attend = 0;
    spm_kv_attend_workspace(&a.caches[0], &b, a.n_q_heads, SPM_DTYPE_FP32, &attend);
    return {up256((nb + 7) / 8 * 8 * k * 6), up256(nb * qkv_width(a) * 4), up256(nb * q_width(a) * 4), up256(attend)};
}

template <int NT, int MT, int U>
cudaError_t launch_project(const __nv_bfloat16* W, const uint4* parts, int rows, int K, int N, float* y, int add, cudaStream_t st) {
    return launch_early(project_kernel<NT, MT, U>, N / (16 * MT), kPrWarps * 32, 0, st, W, parts, rows, K, y, N, add);
}

// y [rows][N] (+)= W [N][K] x [rows][K] (normed with gamma)
cudaError_t project(bool fp32, const void* W, const float* x, const float* gamma, float eps, int rows, int K, int N, void* work, float* y, int add,
                    cudaStream_t st) {
    uint4* parts = fp32 ? nullptr : static_cast<uint4*>(work);
    float* plain = fp32 ? static_cast<float*>(work) : nullptr;
    const cudaError_t e = launch_early(project_rows_kernel, rows, 256, 0, st, x, K, gamma, eps, parts, plain);
    if (e != cudaSuccess) return e;
    if (fp32)
        return launch_early(project_fp32_kernel, dim3((N + kPrWarps - 1) / kPrWarps, (rows + 7) / 8), kPrWarps * 32, 0, st, static_cast<const float*>(W),
                            plain, rows, K, N, y, N, add);
    // one round of CTAs: more of W in flight. With many rows a CTA takes 32 rows of W where that still makes a CTA an SM: what it reads of x
    // from L2 is what it then waits for
    const auto* w = static_cast<const __nv_bfloat16*>(W);
    const bool few = N / 16 <= 148;
    if (rows <= 8 && few) return launch_project<1, 1, 8>(w, parts, rows, K, N, y, add, st);
    if (rows <= 8) return launch_project<1, 1, 4>(w, parts, rows, K, N, y, add, st);
    if (rows <= 16) return launch_project<2, 1, 0>(w, parts, rows, K, N, y, add, st);
    if (rows <= 32) return few ? launch_project<4, 1, 0>(w, parts, rows, K, N, y, add, st) : launch_project<4, 2, 0>(w, parts, rows, K, N, y, add, st);
    return few ? launch_project<8, 1, 0>(w, parts, rows, K, N, y, add, st) : launch_project<8, 2, 0>(w, parts, rows, K, N, y, add, st);
}

}  // namespace

size_t attention_bytes(const spm_model_cfg& m, const spm_attention& a) {
    const Work w = work_of(m, a);
    return w.rows + w.qkv + w.out + w.attend;
}

int check_attention(const spm_model_cfg& m, const spm_attention* a, std::string* why) {
    auto no = [&](int code, const char* what) { *why = what; return code; };
    if (!a || !a->caches) return no(SPM_ERR_INVALID_ARG, "attention: null argument");
    if (a->n_q_heads < 1 || a->n_q_heads > 1024) return no(SPM_ERR_CONFIG, "attention: n_q_heads outside 1..1024");
    spm_kv_batch b = a->batch;
    b.row_start = nullptr;
    b.n_rows = b.n_seq;
    for (int l = 0; l < m.n_layers; ++l) {
        const spm_kv_cache &c = a->caches[l], &first = a->caches[0];
        size_t bytes = 0;
        if (int rc = spm_kv_attend_workspace(&c, &b, a->n_q_heads, SPM_DTYPE_FP32, &bytes)) return no(rc, spm_last_error(nullptr));
        if (c.page_size != first.page_size || c.n_kv_heads != first.n_kv_heads || c.head_dim != first.head_dim || c.n_pages != first.n_pages)
            return no(SPM_ERR_CONFIG, "attention: the layers' caches differ in shape");
        if (!c.pages || reinterpret_cast<uintptr_t>(c.pages) % 16 || reinterpret_cast<uintptr_t>(c.status) % 4)
            return no(SPM_ERR_INVALID_ARG, "attention: pages must be 16-byte aligned, status 4-byte aligned");
    }
    if (!std::isfinite(a->scale)) return no(SPM_ERR_INVALID_ARG, "attention: scale is not finite");
    if (b.n_seq < 1) return no(SPM_ERR_INVALID_ARG, "attention: no sequences");
    return SPM_OK;
}

int enqueue_attention(const AttentionBlock& block, const spm_model_cfg& m, int layer, float* h, int nb, cudaStream_t stream, std::string* why,
                      bool timed) {
    const spm_attention& a = block.a;
    spm_kv_cache kv = block.caches[layer], into = kv;
    if (timed) {
        kv.status = into.status = nullptr;
        into.n_pages = 0;                        // (a page number outside the pool: not written)
    }
    if (nb > a.batch.n_seq) { *why = "attention: more rows than sequences"; return SPM_ERR_INVALID_ARG; }
    const bool fp32 = fp32_model(m);
    const size_t e = fp32 ? 4 : 2, D = m.hidden, NQ = q_width(a), N = qkv_width(a), hd = kv.head_dim;
    const Work w = work_of(m, a);
    char* at = static_cast<char*>(a.workspace);
    void* rows = at;
    float* qkv = reinterpret_cast<float*>(at + w.rows);
    float* out = reinterpret_cast<float*>(at + w.rows + w.qkv);
    void* attend = at + w.rows + w.qkv + w.out;
    auto cuda = [&](cudaError_t ce) { *why = std::string("attention: ") + cudaGetErrorString(ce); return SPM_ERR_CUDA; };
    cudaError_t ce = project(fp32, static_cast<const char*>(a.w_qkv) + layer * N * D * e, h, a.rms_gamma + layer * D, m.rms_eps, nb, int(D), int(N), rows,
                             qkv, 0, stream);
    if (ce != cudaSuccess) return cuda(ce);
    spm_kv_batch b = a.batch;
    b.row_start = nullptr;
    b.n_seq = b.n_rows = nb;
    b.max_rows = 1;
    spm_rope rope = a.rope;
    if (rope.q_gamma) rope.q_gamma += layer * hd;
    if (rope.k_gamma) rope.k_gamma += layer * hd;
    const int64_t row = int64_t(N), head = int64_t(hd);
    const spm_rows q{qkv, row, head}, k{qkv + NQ, row, head}, v{qkv + NQ + hd * kv.n_kv_heads, row, head}, o{out, int64_t(NQ), head};
    int rc = spm_kv_write(&into, &b, &rope, a.positions, a.pos_stride, &q, &q, a.n_q_heads, &k, &v, SPM_DTYPE_FP32, stream);
    if (rc == SPM_OK) rc = spm_kv_attend(&kv, &b, &q, a.n_q_heads, &o, a.scale, SPM_DTYPE_FP32, attend, w.attend, stream);
    if (rc != SPM_OK) { *why = spm_last_error(nullptr); return rc; }
    ce = project(fp32, static_cast<const char*>(a.w_o) + layer * D * NQ * e, out, nullptr, 0.f, nb, int(NQ), int(D), rows, h, 1, stream);
    return ce == cudaSuccess ? SPM_OK : cuda(ce);
}

}  // namespace spm
