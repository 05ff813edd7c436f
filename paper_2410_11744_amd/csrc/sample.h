// Arguments and launcher of dyspec_sample and dyspec_filter_logits (sample.hip).
#pragma once
#include "dyspec_device.h"

namespace dyspec {

// Settings of a sequence's rows.
struct Filter {                                  // top_k 0, top_p 1, min_p 0: no such filter
    float temperature, top_p, min_p;
    int top_k;
    double per_nat, least;                       // log2(e) / temperature, log2(min_p)
};

struct SampleHead {
    const void* logits;
    void* out;                                   // the filtered logits, or nullptr: a token is drawn
    const float* uniform;
    int* token;
    float* prob;
    int* n_kept;
    long long stride, out_stride;                // elements between rows
    int V, rows, n_seq;
};
template <int S> struct SampleArgs : SampleHead { int row0[S]; Filter filter[S]; };

hipError_t launch_sample(const SampleHead& a, const int* row0, const Filter* filter, int dtype, hipStream_t stream);
hipError_t prepare_sample();

}  // namespace dyspec
