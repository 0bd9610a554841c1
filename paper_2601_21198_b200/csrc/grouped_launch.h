// The kernels behind zipmoe_grouped_matmul, as its checks hand them a call.
#pragma once
#include <cuda_runtime.h>

#include "grouped.cuh"

namespace zipmoe_host {

// Any group sizes; made for few tokens per group.
zipmoe_status launch_grouped_few(int dev, bool int8, bool pair, const zipmoe_dev::GroupedMaps &maps, const zipmoe_dev::GroupedArgs &a,
                                 cudaStream_t stream);
// Any group sizes; made for many.  packed: a.R rows of a.Kb bytes, where a.order names the rows of x.
zipmoe_status launch_grouped_wide(int dev, bool int8, bool pair, const zipmoe_dev::GroupedMaps &maps, const zipmoe_dev::GroupedArgs &a,
                                  void *packed, cudaStream_t stream);

}  // namespace zipmoe_host
