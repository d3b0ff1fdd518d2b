// Helpers of the sequence-layer operators' entry points (layer.hpp).
#include <cstdio>

#include "layer.hpp"

namespace la {

__global__ __launch_bounds__(256) void k_zero(uint16_t *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
        p[i] = 0;
}

la_status zero_bytes(void *p, size_t bytes, hipStream_t st)
{
    const size_t n = bytes / 2;
    if (!p || !n)
        return LA_OK;
    const size_t blocks = (n + 255) / 256;
    LA_LAUNCH(k_zero, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, (uint16_t *)p, n);
    return launch_check("zero");
}

la_status check_workspace(const void *ws, size_t given, size_t need, const char *asked)
{
    if (!need)
        return LA_OK;
    if (!ws || given < need) {
        char text[160];
        snprintf(text, sizeof(text), "this call needs a workspace of %s bytes: %zu, %zu given", asked, need, ws ? given : (size_t)0);
        set_error_text(text);
        return LA_ERR_WORKSPACE;
    }
    return (uintptr_t)ws & 255 ? LA_ERR_INVALID_ARG : LA_OK;
}

}  // namespace la
