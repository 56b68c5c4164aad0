// Page tables: what host code and paged_plan.hip share.
#pragma once
#include "path_common.h"

namespace path {

struct PlanArgs {
    const int *cached, *fresh;       // [nseq] tokens that stay, new ones behind them
    int *table, *free_pages, *count; // [nseq, per_seq], [num_pages], [1]
    int* cu;                         // [nseq + 1]
    long long* slots;                // [T]
    int* missing;                    // [nseq]
    int nseq, per_seq, num_pages, shift, T;
    int* scratch;                    // the first count, then [nseq] pages that go back and [nseq] that are wanted
};
hipError_t launch_plan(const PlanArgs& a, hipStream_t stream);

}  // namespace path
