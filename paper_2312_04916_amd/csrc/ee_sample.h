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
    // whether the settings can cut anything, as far as the host knows
    bool cuts() const { return top_k || top_p || min_p || (one_top_k > 0 && one_top_k < vocab) || one_top_p < 1.f || one_min_p > 0.f; }
};

// The workspace of a row.  The first kernel leaves, by index alone, the largest logit of each run of 64 tokens, and of each run of 1024 the
// sum of the weights, in 2^-44 of the run's largest, and the sum of exp(z - largest).  The second one leaves a note for the third where
// a row has too many tokens that may be kept.
constexpr int SAMPLE_RUN = 1024, SAMPLE_CHUNK = 64, SAMPLE_BINS = 1024;
struct SampleNote {
    uint32_t wide;               // for the third kernel
    uint32_t top_key, least;     // keys of the largest logit, of the floor
    uint32_t arrived;            // workgroups of the row that have left their bins
    unsigned long long total;    // of all weights, where it is asked for
    double log_raw, raw;         // sum of exp(z - top)
};
struct SampleRow {
    int runs;
    constexpr explicit SampleRow(int vocab) : runs((vocab + SAMPLE_RUN - 1) / SAMPLE_RUN) {}
    constexpr size_t sums() const { return (size_t)runs * (SAMPLE_RUN / SAMPLE_CHUNK) * 4; }
    constexpr size_t raws() const { return sums() + (size_t)runs * 8; }
    constexpr size_t note() const { return (raws() + (size_t)runs * 4 + 15) / 16 * 16; }
    constexpr size_t bytes() const { return note() + (sizeof(SampleNote) + 15) / 16 * 16; }
};
// For the third kernel, for each row that several of its workgroups share: a weight and a count for each bin, to which they add; and what each of these leaves, for
// each bin a weight and where its elements begin, and the part's elements.
constexpr size_t SAMPLE_ROW_BINS = (size_t)SAMPLE_BINS * 12;
constexpr size_t sample_part_bytes(int part_length) { return (size_t)SAMPLE_BINS * 12 + 16 + (size_t)part_length * 2; }
int sample_parts(int rows, int vocab);
size_t sample_workspace(int rows, int vocab, bool cuts);

hipError_t launch_sample(const Sampling& p, hipStream_t st);

}  // namespace ee
