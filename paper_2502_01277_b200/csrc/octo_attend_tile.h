// The attention kernel for many query rows (octo_attend_tile.cu), as the plan of a call uses it.
#pragma once

#include "octo_attend.cuh"

namespace octo {

constexpr int kTileRows = 256;  // rows (query row, head) of a work item
constexpr int kTileKeys = 128;  // keys per turn; splits are multiples of it

// grid: CTAs (at most one per SM); tiles_per_segment: used where every segment has the same number of rows.
cudaError_t launch_attend_tile(const AttendArgs& a, int bf16, int grid, int tiles_per_segment, cudaStream_t stream);

}  // namespace octo
