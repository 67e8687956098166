// Arguments of the sampler (gdn_sample.cu).
#pragma once

#include "gdn_internal.cuh"

namespace gdn {

constexpr int GDN_MAX_VOCAB = GDN_SAMPLE_MAX_VOCAB;

struct SampleParams {
    int n_rows, vocab;
    long long row_stride;
    const void *logits;
    const float *temperature;   // these four may be null: 1, off, off, off
    const int32_t *top_k;
    const float *top_p, *min_p;
    const float *uniform;
    int32_t *token;
    float *prob;                // may be null
};

cudaError_t launch_sample(const SampleParams &p, bool bf16, cudaStream_t stream);

}  // namespace gdn
