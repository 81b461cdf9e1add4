// Host side of choosing tokens (ee_sample of ee.h): argument checks.
#include "ee_internal.h"
#include "ee_sample.h"

using namespace ee;

extern "C" {

static int workspace_of(int rows, int vocab, bool cuts, size_t* workspace_bytes) {
    if (!workspace_bytes || rows < 0 || rows > (1 << 20)) return EE_ERR_ARG;
    if (vocab < 1 || vocab > (1 << 18)) return EE_ERR_CONFIG;
    *workspace_bytes = sample_workspace(rows, vocab, cuts);
    return EE_OK;
}

int ee_sample_bytes(int rows, int vocab, size_t* workspace_bytes) { return workspace_of(rows, vocab, true, workspace_bytes); }
int ee_sample_uncut_bytes(int rows, int vocab, size_t* workspace_bytes) { return workspace_of(rows, vocab, false, workspace_bytes); }

int ee_sample(int rows, int vocab, int dtype, const void* dev_logits, int64_t row_stride, const float* dev_u, const float* dev_temperature,
                         const int32_t* dev_top_k, const float* dev_top_p, const float* dev_min_p, float temperature, int32_t top_k, float top_p,
                         float min_p, int32_t* dev_token, float* dev_logprob, float* dev_confidence, void* dev_workspace,
              size_t workspace_bytes, void* stream) {
    if (rows < 0 || rows > (1 << 20)) return EE_ERR_ARG;
    if (vocab < 1 || vocab > (1 << 18) || (dtype != EE_F32 && dtype != EE_BF16)) return EE_ERR_CONFIG;
    if (!dev_temperature && !(temperature >= 0.f && temperature <= 3.4028235e38f)) return EE_ERR_ARG;
    if ((!dev_top_k && top_k < 0) || (!dev_top_p && !(top_p >= 0.f && top_p <= 1.f)) || (!dev_min_p && !(min_p >= 0.f && min_p <= 1.f))) return EE_ERR_ARG;
    if (rows == 0) return EE_OK;
    const int64_t es = dtype == EE_BF16 ? 2 : 4;
    if (!dev_logits || !dev_u || !dev_token || (uintptr_t)dev_logits & (es - 1)) return EE_ERR_ARG;
    if (((uintptr_t)dev_u | (uintptr_t)dev_temperature | (uintptr_t)dev_top_k | (uintptr_t)dev_top_p | (uintptr_t)dev_min_p | (uintptr_t)dev_token |
         (uintptr_t)dev_logprob | (uintptr_t)dev_confidence) & 3)
        return EE_ERR_ARG;
    if (!dev_workspace || (uintptr_t)dev_workspace & 255) return EE_ERR_ARG;
    Sampling p;
    p.rows = rows, p.vocab = vocab, p.dtype = dtype;
    p.logits = dev_logits, p.row_stride = row_stride;
    p.u = dev_u, p.temperature = dev_temperature, p.top_k = dev_top_k, p.top_p = dev_top_p, p.min_p = dev_min_p;
    p.one_temperature = temperature, p.one_top_k = top_k, p.one_top_p = top_p, p.one_min_p = min_p;
    p.token = dev_token, p.logprob = dev_logprob, p.confidence = dev_confidence;
    p.workspace = (char*)dev_workspace;
    p.vec = ((uintptr_t)dev_logits & (4 * es - 1)) == 0 && row_stride % 4 == 0;
    const size_t need = sample_workspace(rows, vocab, p.cuts());
    if (workspace_bytes < need) return EE_ERR_NOMEM;
    // rows are read while others' results are already written
    const int64_t span = (int64_t)(rows - 1) * row_stride * es;
    const uintptr_t lo = (uintptr_t)dev_logits + (uintptr_t)(span < 0 ? span : 0), hi = (uintptr_t)dev_logits + (uintptr_t)((span < 0 ? 0 : span) + vocab * es);
    const void* out[3] = {dev_token, dev_logprob, dev_confidence};
    const void* in[5] = {dev_u, dev_temperature, dev_top_k, dev_top_p, dev_min_p};
    const uintptr_t bytes = (uintptr_t)rows * 4;
    auto meet = [](const void* a, uintptr_t b_lo, uintptr_t b_hi, uintptr_t n) { return a && (uintptr_t)a < b_hi && b_lo < (uintptr_t)a + n; };
    if (meet(dev_workspace, lo, hi, need)) return EE_ERR_ARG;
    for (int j = 0; j < 5; ++j)
        if (in[j] && meet(dev_workspace, (uintptr_t)in[j], (uintptr_t)in[j] + bytes, need)) return EE_ERR_ARG;
    for (int i = 0; i < 3; ++i) {
        if (out[i] && meet(dev_workspace, (uintptr_t)out[i], (uintptr_t)out[i] + bytes, need)) return EE_ERR_ARG;
        if (meet(out[i], lo, hi, bytes)) return EE_ERR_ARG;
        for (int j = 0; j < 5; ++j)
            if (in[j] && meet(out[i], (uintptr_t)in[j], (uintptr_t)in[j] + bytes, bytes)) return EE_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (out[j] && meet(out[i], (uintptr_t)out[j], (uintptr_t)out[j] + bytes, bytes)) return EE_ERR_ARG;
    }
    const hipError_t e = launch_sample(p, (hipStream_t)stream);
    return e == hipSuccess ? EE_OK : note_hip_error((int)e);
}

}  // extern "C"
