// Internal interface between the translation units of libdscores (not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dtree_scores.h"

namespace dscores {

// Rows of few classes are worked on by one lane each, others by teams of 1, 4, 8 or 16 wavefronts.
constexpr int kLaneClasses = 64;

// Long rows (times of top_scores on rows of 131,072 bf16, k = 64).  Where there are no more rows
// than compute units, each has one to itself, for 16 wavefronts (1 row: 20 us, 28 with 8; 256
// rows: 25 and 35).  Of teams of 4 wavefronts a compute unit holds four, whose phases overlap: they pay from
// as many rows on (2,048 rows: 126 us, 142 with 8 wavefronts; 257 rows: 35 and 29).
constexpr int64_t kFewRows = 256, kManyRows = 1024;
// 256 threads find no good bound for many classes (2,048 rows, k = 96: 132 us, 138 with 8
// wavefronts; k = 128: 154 and 150).
constexpr int kQuarter = 96;
// The same for one wavefront, on rows of at most 1,024 classes (60,000 rows of 1,000 bf16, k = 48:
// 305 us, 429 with 4 wavefronts; k = 60: 502 and 476; fp32, k = 200: 1,725 and 953).
constexpr int kSixteenth = 48;
// The sampler's teams are chosen by the same numbers, but without one of 8 where most classes stay:
// 64 rows of 5,000 bf16 by top-p in 25 us with 4 wavefronts and 27 with 16, of 9,000 in 33 and 31;
// 256 of 131,072 in 298 and 149, 512 of 32,768 in 91 and 103, 1,024 in 126 and 191.  Just above 256
// rows 16 would still be faster on the longest (300 of 131,072: 328 and 242).

struct RowArgs {
    const void *x;
    int64_t n, ld;
    int32_t classes;
    int32_t align;        // every row starts at a multiple of this many bytes (1 .. 16)
};

struct TopArgs {
    RowArgs in;
    int32_t k;
    float *values;
    int32_t *index;
    float *lse;
};

struct SampleArgs {
    RowArgs in;
    const float *u;
    ds_sampling set;
    int32_t *labels;
};

struct DistillArgs {
    RowArgs in;
    const float *values;
    const int32_t *index;
    int32_t k;
    float temperature;
    const float *g;
    float *loss;
    float2 *stats;        // (largest score, sum of e^((x - largest) / temperature)) of each row
    void *grad;
    int64_t ld_grad;
    float2 *part;         // the same of each part of each row
    int32_t parts;        // of a row
};

hipError_t launch_top(const TopArgs &a, dt_dtype type, hipStream_t stream);
hipError_t launch_sample(const SampleArgs &a, dt_dtype type, hipStream_t stream);
hipError_t launch_distill(const DistillArgs &a, dt_dtype type, hipStream_t stream);
hipError_t launch_distill_backward(const DistillArgs &a, dt_dtype type, hipStream_t stream);
int distill_parts(int64_t n, int32_t classes);

}  // namespace dscores
