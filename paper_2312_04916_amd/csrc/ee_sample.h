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
    int vec;  // rows can be read 16 bytes at a time
};

hipError_t launch_sample(const Sampling& p, hipStream_t st);

}  // namespace ee
