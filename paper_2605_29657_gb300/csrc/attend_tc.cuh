// attend_tc.cuh -- launcher of the tensor-core attention kernel (internal header).
#pragma once

#include "attend.cuh"

namespace occam {

// Sequences with p.row_lo < rows * G <= p.row_hi; at most kAttendTcCtas CTAs.
int launch_attend_tc(const AttendParams& p, int dim, cudaStream_t st);

}  // namespace occam
