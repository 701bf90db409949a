// attend_tc.cuh -- launcher of the tensor-core attention kernel (internal header).
#pragma once

#include <cuda.h>

#include "attend.cuh"

namespace occam {

// Sequences with p.row_lo < rows * G <= p.row_hi; at most kAttendTcCtas CTAs.
template <int MODE>
int launch_attend_tc(const AttendCall<MODE>& p, int dim, cudaStream_t st);

// Tensor map of the codes as [layers * pages][heads * page_tokens][dim] bytes, boxes of
// `box_rows` rows of one page (swizzled by the row's bytes, 128 or 64, if asked).
bool encode_blocks(CUtensorMap* m, const CacheDev& c, const void* codes, int dim, int box_rows, bool swizzle);

}  // namespace occam
