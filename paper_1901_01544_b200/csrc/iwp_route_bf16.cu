// The router's kernels for logits of one type.
#define IWP_ROUTE_TYPE IWP_BF16
#include "iwp_route_launch.hpp"

template int iwp_router::launch_route<IWP_ROUTE_TYPE>(const Args&, int, cudaStream_t);
template int iwp_router::launch_route_grad<IWP_ROUTE_TYPE>(const GradArgs&, int, cudaStream_t);
