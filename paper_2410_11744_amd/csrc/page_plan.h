// Arguments and launcher of dyspec_page_plan (page_plan.hip).
#pragma once
#include "dyspec_device.h"

namespace dyspec {

struct PlanArgs {
    int *ring, *state, *table, *granted;
    const int *held, *wanted, *slots_from;       // slots_from: or nullptr
    long long* slots;                            // or nullptr
    long long n_slots;
    int n_pages, page_shift, max_pages, table_stride, n_seq;
};
hipError_t launch_page_plan(const PlanArgs& a, hipStream_t stream);
hipError_t prepare_page_plan();

}  // namespace dyspec
