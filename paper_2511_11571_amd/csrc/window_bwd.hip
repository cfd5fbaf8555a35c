// Causal attention to the last W keys: backward.  D = rowsum(dO o O), then a wave per row for dQ and a
// wave per key for dK and dV.
#include "window.h"

namespace moba {

template <typename T, int D>
__global__ __launch_bounds__(256) void window_rowdot_kernel(const T* __restrict__ O, const T* __restrict__ dO,
                                                            float* __restrict__ Dv, int64_t rows)
{
    constexpr int L = D / 8;                                 // lanes of a row
    const int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if (row >= rows) return;
    float x[8], y[8], a = 0.f;
    Vec8<T>::load(O + row * D + 8 * (threadIdx.x % L), x);
    Vec8<T>::load(dO + row * D + 8 * (threadIdx.x % L), y);
#pragma unroll
    for (int e = 0; e < 8; ++e) a = fmaf(x[e], y[e], a);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) a += __shfl_xor(a, o, L);
    if (threadIdx.x % L == 0) Dv[row] = a;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void window_dq_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                        const T* __restrict__ V, const T* __restrict__ dO,
                                                        const float* __restrict__ lse, const float* __restrict__ Dv,
                                                        T* __restrict__ dQ)
{
    const int r = blockIdx.x * 4 + threadIdx.x / kWave;
    if (r < a.q) plain_dq_row<T, D>(a, Q, K, V, dO, lse, Dv, dQ, blockIdx.y, r, threadIdx.x % kWave);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void window_dkdv_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                          const T* __restrict__ V, const T* __restrict__ dO,
                                                          const float* __restrict__ lse, const float* __restrict__ Dv,
                                                          T* __restrict__ dK, T* __restrict__ dV)
{
    const int u = blockIdx.x * 4 + threadIdx.x / kWave;
    if (u < a.N) plain_dkdv_key<T, D>(a, Q, K, V, dO, lse, Dv, dK, dV, blockIdx.y, u, threadIdx.x % kWave);
}

size_t window_backward_ws_bytes(const WindowDims& s) { return a256(sizeof(float) * (size_t)s.bh * s.q); }

template <typename T, int D>
static hipError_t backward_t(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O,
                             const float* lse, const void* dO, const int32_t* first, void* dQ, void* dK, void* dV,
                             void* ws, hipStream_t st)
{
    const WindowArgs a = window_args(s, first);
    float* Dv = static_cast<float*>(ws);
    const int64_t rows = (int64_t)s.bh * s.q, per = 256 / (D / 8);
    hipLaunchKernelGGL((window_rowdot_kernel<T, D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st,
                       (const T*)O, (const T*)dO, Dv, rows);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dq_kernel<T, D>), dim3((s.q + 3) / 4, s.bh), dim3(256), 0, st, a, (const T*)Q, (const T*)K,
                       (const T*)V, (const T*)dO, lse, Dv, (T*)dQ);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dkdv_kernel<T, D>), dim3((s.N + 3) / 4, s.bhk), dim3(256), 0, st, a, (const T*)Q,
                       (const T*)K, (const T*)V, (const T*)dO, lse, Dv, (T*)dK, (T*)dV);
    return hipGetLastError();
}

hipError_t launch_window_backward(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O,
                                  const float* lse, const void* dO, const int32_t* first, void* dQ, void* dK, void* dV,
                                  void* ws, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? backward_t<bf16_t, 64>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st)
                         : backward_t<bf16_t, 128>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st);
    return s.D == 64 ? backward_t<float, 64>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st)
                     : backward_t<float, 128>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st);
}

}  // namespace moba
