// Choosing tokens (ee_sample of ee.h): the launch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ee.h"

namespace ee {

struct Sampling {
    int rows, vocab, dtype;
    const void* logits;
    int64_t row_stride;
    const float *u, *temperature;
    const int32_t* top_k;
    const float *top_p, *min_p;
    float one_temperature;  // of all rows, where there is no array
    int32_t one_top_k;
    float one_top_p, one_min_p;
    int32_t* token;
    float *logprob, *confidence;
    char* workspace;
    int vec;  // rows can be read four elements at a time
};

// What the first kernel leaves of a row for the second, by index alone: the largest logit of each run of 64 tokens, and of each run of 1024
// the sum of the weights, in 2^-44 of the run's largest, and the sum of exp(z - largest).
constexpr int SAMPLE_RUN = 1024, SAMPLE_CHUNK = 64;
struct SampleRow {
    int runs;
    constexpr explicit SampleRow(int vocab) : runs((vocab + SAMPLE_RUN - 1) / SAMPLE_RUN) {}
    constexpr size_t sums() const { return (size_t)runs * (SAMPLE_RUN / SAMPLE_CHUNK) * 4; }
    constexpr size_t raws() const { return sums() + (size_t)runs * 8; }
    constexpr size_t bytes() const { return (raws() + (size_t)runs * 4 + 15) / 16 * 16; }
};

hipError_t launch_sample(const Sampling& p, hipStream_t st);

}  // namespace ee
