// Launch interface between the C ABI layer and the expert-layer kernels
// (norm.hip, route.hip, exchange.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "taccl.h"

namespace taccl {

constexpr int kNormMaxCols = 16384;
constexpr int kNormMaxBlocks = 1024;  // partial rows of dweight in the workspace
constexpr int kMaxExperts = 1024;
constexpr int kMaxChoices = 16;
constexpr int kRouteMaxBlocks = 256;  // partial counts and sums in the workspace
// a grid has fewer than 2^32 threads, up to 1024 of them per row
constexpr int64_t kMaxRows = 1 << 21;
constexpr int kExchangeMaxCols = 1 << 20;

// Arguments are the C ABI's, checked; each launch takes the current device's
// CU count where its grid depends on it.
hipError_t launch_norm(const taccl_norm_t &a, hipStream_t stream);
hipError_t launch_norm_backward(const taccl_norm_backward_t &a, int cus, hipStream_t stream);
hipError_t launch_route(const taccl_route_t &a, hipStream_t stream);
hipError_t launch_route_backward(const taccl_route_backward_t &a, int cus, hipStream_t stream);
hipError_t launch_dispatch(const taccl_dispatch_t &a, int cus, hipStream_t stream);
hipError_t launch_combine(const taccl_combine_t &a, hipStream_t stream);
hipError_t launch_combine_backward(const taccl_combine_backward_t &a, int cus, hipStream_t stream);

}  // namespace taccl
