// The router's kernels for scores of fp16 (route.h).
#include "route.h"

template <>
void ds_route_rows<_Float16>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<_Float16>(*(const RouteArgs*)args, blocks, stream);
}
template <>
void ds_route_rows_backward<_Float16>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<_Float16>(*(const RouteGradArgs*)args, blocks, stream);
}
