// The router's kernels for scores of fp32 (route.h).
#include "route.h"

template <>
void ds_route_rows<float>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<float>(*(const RouteArgs*)args, blocks, stream);
}
template <>
void ds_route_rows_backward<float>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<float>(*(const RouteGradArgs*)args, blocks, stream);
}
