// glu_stage.hpp -- which values a thread lays out when rows are made operands of the
// tiled products (kernels_glu_point.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace exemcl {

constexpr int kStageThreads = 256;

// Up to three arrays in one launch.
struct StageJobs {
    DenseStageJob job[3];
    int64_t blocks[3];  // workgroups up to and with each
};

// The jobs' workgroups; returns their number.
inline int64_t stage_jobs(const DenseStageJob *jobs, int count, StageJobs *s) {
    int64_t blocks = 0;
    for (int i = 0; i < 3; ++i) {
        if (i < count) {
            s->job[i] = jobs[i];
            blocks += (jobs[i].n * ((jobs[i].d + 7) / 8) + kStageThreads - 1) / kStageThreads;
        }
        s->blocks[i] = blocks;
    }
    return blocks;
}

// Eight values of a row of a job, from column c on.  job -1: none, for the last threads of
// a job and for workgroups past the last one's (a grid of whole rows has some).
struct StagePlace {
    int job;
    int64_t row, c, ld;  // ld: elements of a row as it is laid out
};
__host__ __device__ inline StagePlace stage_place(const StageJobs &jobs, int64_t block, int thread) {
    if (block >= jobs.blocks[2]) return {-1, 0, 0, 0};
    const int which = block < jobs.blocks[0] ? 0 : block < jobs.blocks[1] ? 1 : 2;
    if (which) block -= jobs.blocks[which - 1];
    const int64_t per = (jobs.job[which].d + 7) / 8, i = block * kStageThreads + thread, row = i / per;
    if (row >= jobs.job[which].n) return {-1, 0, 0, 0};
    return {which, row, (i - row * per) * 8, per * 8};
}

}  // namespace exemcl
