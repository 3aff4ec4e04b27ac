// Waits that ran out (include/ebrl_pages.h: ebrl_pages_check).
#include "pages_internal.h"

namespace ebrl {
namespace pg {

__device__ int wait_status;       // EBRL_ERR_TIMEOUT once a wait ran out; one on each device

cudaError_t take_status(int *status)
{
    const int zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status, wait_status, sizeof(int));
    if (e == cudaSuccess && *status) e = cudaMemcpyToSymbol(wait_status, &zero, sizeof(int));
    return e;
}

}  // namespace pg
}  // namespace ebrl
