// Causal attention to the last W keys: forward.  A wave per row.
#include "window.h"

namespace moba {

template <typename T, int D>
__global__ __launch_bounds__(256) void window_forward_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                             const T* __restrict__ V, T* __restrict__ O,
                                                             float* __restrict__ lse)
{
    const int r = blockIdx.x * 4 + threadIdx.x / kWave;
    if (r < a.q) plain_forward_row<T, D>(a, Q, K, V, O, lse, blockIdx.y, r, threadIdx.x % kWave);
}

size_t window_forward_ws_bytes(const WindowDims&) { return 0; }

template <typename T, int D>
static hipError_t forward_t(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                            void* O, float* lse, hipStream_t st)
{
    hipLaunchKernelGGL((window_forward_kernel<T, D>), dim3((s.q + 3) / 4, s.bh), dim3(256), 0, st, window_args(s, first),
                       (const T*)Q, (const T*)K, (const T*)V, (T*)O, lse);
    return hipGetLastError();
}

hipError_t launch_window_forward(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                                 void* O, float* lse, void*, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? forward_t<bf16_t, 64>(s, Q, K, V, first, O, lse, st)
                         : forward_t<bf16_t, 128>(s, Q, K, V, first, O, lse, st);
    return s.D == 64 ? forward_t<float, 64>(s, Q, K, V, first, O, lse, st)
                     : forward_t<float, 128>(s, Q, K, V, first, O, lse, st);
}

}  // namespace moba
