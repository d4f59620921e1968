// Host side of the kernels on rows of logits: argument checks, how a row is
// split over a cluster, and the launch.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/epic.h"
#include "mass_parts.h"

namespace epic {

constexpr int kRowCtasMax = 8;  // the portable limit of a cluster

struct RowShape {
  int ctas;     // CTAs of a row: one cluster
  int threads;  // of a CTA
  int per;      // chunks of 16 bytes per CTA
};

// A row of V elements of `size` bytes, `rows` of them in the call; CTAs of at least `least` and at most `most` threads.
RowShape row_shape(long long rows, int V, int size, int least, int most);

// EPIC_OK, or the error of a bad description of rows
epic_status check_rows(const void* logits, int dtype, int B, int n, int V, int64_t stride_b, int64_t stride_n,
                       const int32_t* pos, int k);

// rows * shape.ctas CTAs in clusters of shape.ctas; `args` points at the kernel's one argument
epic_status launch_rows(const void* kernel, const RowShape& shape, long long rows, void* args, cudaStream_t st);

}  // namespace epic
