// The router's kernels for scores of bf16 (route.h).
#include "route.h"

template <>
void ds_route_rows<__bf16>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<__bf16>(*(const RouteArgs*)args, blocks, stream);
}
template <>
void ds_route_rows_backward<__bf16>(const void* args, unsigned blocks, hipStream_t stream) {
  launch_for<__bf16>(*(const RouteGradArgs*)args, blocks, stream);
}
