// Causal attention to the last W keys (W = N: dense) and its backward: what the kernels share.
//
// The query in row r stands at position t = N - q_len + r and attends the keys from
// max(0, t - W + 1, first_key[row]) to t.  Query slices are [batch * heads], key/value slices
// [batch * kv_heads] of `rows` rows each; G query heads share a key/value head.
#pragma once
#include "mfma.h"

namespace moba {

struct WindowDims {
    int batch, heads, hkv, G;
    int bh, bhk;                // query and key/value slices
    int q, N, rows, D, W;       // W <= N
    int dtype;
    float scale;
};

// dynamic LDS of a kernel, beyond what every launch may have
inline hipError_t window_lds(const void* kernel, size_t bytes) { return bytes > 64 * 1024 ? ensure_dynamic_lds(kernel, bytes) : hipSuccess; }

// what a kernel needs of it
struct WindowArgs {
    int q, N, rows, W, G, heads, bhk;
    float scale;
    const int32_t* first;       // [batch, q] or nullptr
};
inline WindowArgs window_args(const WindowDims& s, const int32_t* first)
{
    return {s.q, s.N, s.rows, s.W, s.G, s.heads, s.bhk, s.scale, first};
}

// first key that row r of query slice s attends; behind its position where it attends none
__device__ __forceinline__ int window_first(const WindowArgs& a, int s, int r)
{
    const int t = a.N - a.q + r;
    int lo = t - a.W + 1;
    if (a.first) lo = max(lo, a.first[(int64_t)(s / a.heads) * a.q + r]);
    return max(lo, 0);
}

// ---- one row, or one key, by a wave: plain loops over its pairs alone ---------------------------
// They touch nothing but the row's own pairs, so what stands elsewhere cannot reach the result: the tiled
// kernels, where a weight of zero meets every key and value of a tile, come here with rows and keys
// whose sums are not finite.  A sum that is NaN stays so: once every channel's is, the loops end, so that a call whose
// inputs are NaN throughout does not do all its pairs twice.
template <typename T, int D>
__device__ __forceinline__ float row_dot(const T* __restrict__ x, const T* __restrict__ y)
{
    float a = 0.f;
#pragma unroll 2
    for (int c = 0; c < D; c += 8) {
        float u[8], v[8];
        Vec8<T>::load(x + c, u);
        Vec8<T>::load(y + c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) a = fmaf(u[e], v[e], a);
    }
    return a;
}

// acc (channel lane + 64 c) += sum over the lanes j < n of w_j * row(j)
template <typename T, int D, typename F>
__device__ __forceinline__ void add_rows(float (&acc)[D / 64], float w, int n, int lane, F row)
{
    for (int j = 0; j < n; ++j) {
        const float x = __shfl(w, j, kWave);
        const T* p = row(j);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) acc[c] = fmaf(x, to_f32<T>(p[lane + 64 * c]), acc[c]);
    }
}

// every channel's sum is NaN
template <int C>
__device__ __forceinline__ bool all_nan(const float (&acc)[C])
{
    bool x = true;
#pragma unroll
    for (int c = 0; c < C; ++c) x = x && acc[c] != acc[c];
    return __ballot(!x) == 0;
}

template <typename T, int D>
__device__ __forceinline__ void plain_forward_row(const WindowArgs& a, const T* __restrict__ Q, const T* __restrict__ K,
                                                  const T* __restrict__ V, T* __restrict__ O, float* __restrict__ lse,
                                                  int s, int r, int lane)
{
    const int t = a.N - a.q + r, lo = window_first(a, s, r);
    const int64_t row = (int64_t)s * a.q + r;
    const T* q = Q + row * D;
    const T* Ks = K + (int64_t)(s / a.G) * a.rows * D;
    const T* Vs = V + (int64_t)(s / a.G) * a.rows * D;
    float m = -INFINITY, l = 0.f, acc[D / 64] = {};
    for (int u0 = lo; u0 <= t; u0 += kWave) {
        const int n = min(kWave, t - u0 + 1);
        const float z = lane < n ? row_dot<T, D>(q, Ks + (int64_t)(u0 + lane) * D) * (a.scale * kLog2e) : -INFINITY;
        const float top = fmaxf(m, wave_max(z));
        const float ref = fmaxf(top, -3.402823466e+38f);             // (no finite logit yet: exponents stay -inf)
        const float alpha = fast_exp2(m - ref), p = lane < n ? fast_exp2(z - ref) : 0.f;
        m = top;
        l = fmaf(l, alpha, wave_sum(p));
#pragma unroll
        for (int c = 0; c < D / 64; ++c) acc[c] *= alpha;
        add_rows<T, D>(acc, p, n, lane, [&](int j) { return Vs + (int64_t)(u0 + j) * D; });
        if (l != l) break;                                   // (the same in every lane)
    }
    const bool empty = lo > t;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) O[row * D + lane + 64 * c] = from_f32<T>(empty ? 0.f : acc[c] / l);
    if (lane == 0) lse[row] = empty ? -INFINITY : (m + fast_log2(l)) * kLn2;
}

// The gradient with respect to the one logit of a row that attends one key is zero, and dO . v - D only as far as sums in
// different orders agree.  So dS of such a row is multiplied by zero, which leaves a NaN one; for dQ its sum is.
__device__ __forceinline__ float ds_factor(int lo, int t) { return lo < t ? 1.f : 0.f; }
__device__ __forceinline__ float dq_factor(const WindowArgs& a, int lo, int t) { return a.scale * ds_factor(lo, t); }

template <typename T, int D>
__device__ __forceinline__ void plain_dq_row(const WindowArgs& a, const T* __restrict__ Q, const T* __restrict__ K,
                                             const T* __restrict__ V, const T* __restrict__ dO,
                                             const float* __restrict__ lse, const float* __restrict__ Dv,
                                             T* __restrict__ dQ, int s, int r, int lane)
{
    const int t = a.N - a.q + r, lo = window_first(a, s, r);
    const int64_t row = (int64_t)s * a.q + r;
    const T* Ks = K + (int64_t)(s / a.G) * a.rows * D;
    const T* Vs = V + (int64_t)(s / a.G) * a.rows * D;
    const float z = lse[row] * kLog2e, Dr = Dv[row];
    float acc[D / 64] = {};
    for (int u0 = lo; u0 <= t; u0 += kWave) {
        const int n = min(kWave, t - u0 + 1);
        float ds = 0.f;
        if (lane < n) {
            const int64_t key = (int64_t)(u0 + lane) * D;
            const float p = fast_exp2(fmaf(row_dot<T, D>(Q + row * D, Ks + key), a.scale * kLog2e, -z));
            ds = p * (row_dot<T, D>(dO + row * D, Vs + key) - Dr);
        }
        add_rows<T, D>(acc, ds, n, lane, [&](int j) { return Ks + (int64_t)(u0 + j) * D; });
        if (all_nan(acc)) break;
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) dQ[row * D + lane + 64 * c] = from_f32<T>(acc[c] * dq_factor(a, lo, t));
}

// dK and dV of key u of key/value slice sk; D of the rows from Dv or (OWN) from O
template <typename T, int D, bool OWN>
__device__ __forceinline__ void plain_dkdv_key(const WindowArgs& a, const T* __restrict__ Q, const T* __restrict__ K,
                                               const T* __restrict__ V, const T* __restrict__ O, const T* __restrict__ dO,
                                               const float* __restrict__ lse, const float* __restrict__ Dv,
                                               T* __restrict__ dK, T* __restrict__ dV, int sk, int u, int lane)
{
    const int64_t key = ((int64_t)sk * a.rows + u) * D;
    const int r_lo = max(0, u - (a.N - a.q)), r_hi = (int)min((int64_t)a.q, (int64_t)u - (a.N - a.q) + a.W);
    float ak[D / 64] = {}, av[D / 64] = {};
    for (int g = 0; g < a.G; ++g) {
        const int s = sk * a.G + g;
        const int64_t base = (int64_t)s * a.q;
        for (int r0 = r_lo; r0 < r_hi && !(all_nan(ak) && all_nan(av)); r0 += kWave) {
            const int r = r0 + lane;
            const int lo = r < r_hi ? window_first(a, s, r) : 0;
            const bool on = r < r_hi && lo <= u;
            float p = 0.f, ds = 0.f;
            if (on) {
                p = fast_exp2(fmaf(row_dot<T, D>(Q + (base + r) * D, K + key), a.scale * kLog2e, -lse[base + r] * kLog2e));
                const float Dr = OWN ? row_dot<T, D>(dO + (base + r) * D, O + (base + r) * D) : Dv[base + r];
                ds = p * (row_dot<T, D>(dO + (base + r) * D, V + key) - Dr) * ds_factor(lo, a.N - a.q + r);
            }
            for (uint64_t left = __ballot(on); left; left &= left - 1) {
                const int j = __builtin_ctzll(left);
                const float pj = __shfl(p, j, kWave), dj = __shfl(ds, j, kWave);
                const int64_t row = (base + r0 + j) * D + lane;
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    av[c] = fmaf(pj, to_f32<T>(dO[row + 64 * c]), av[c]);
                    ak[c] = fmaf(dj, to_f32<T>(Q[row + 64 * c]), ak[c]);
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        dK[key + lane + 64 * c] = from_f32<T>(ak[c] * a.scale);
        dV[key + lane + 64 * c] = from_f32<T>(av[c]);
    }
}

size_t window_forward_ws_bytes(const WindowDims& s);
hipError_t launch_window_forward(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                                 void* O, float* lse, void* ws, hipStream_t st);
// few tiles of queries (window_few.hip)
bool window_few(const WindowDims& s);
size_t window_few_ws_bytes(const WindowDims& s);
hipError_t launch_window_few(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                             void* O, float* lse, void* ws, hipStream_t st);
bool window_few_dq(const WindowDims& s);
bool window_few_dkdv(const WindowDims& s);
hipError_t launch_window_few_dq(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse,
                                const void* dO, const int32_t* first, void* dQ, float* Dv, hipStream_t st);
hipError_t launch_window_few_dkdv(const WindowDims& s, const void* Q, const void* K, const void* V, const float* lse, const void* dO,
                                  const int32_t* first, void* dK, void* dV, float* Dv, hipStream_t st);
// both in one launch
bool window_few_both(const WindowDims& s);
hipError_t launch_window_few_backward(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse,
                                      const void* dO, const int32_t* first, void* dQ, void* dK, void* dV, float* Dv, hipStream_t st);
size_t window_backward_ws_bytes(const WindowDims& s);
hipError_t launch_window_backward(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O,
                                  const float* lse, const void* dO, const int32_t* first, void* dQ, void* dK, void* dV,
                                  void* ws, hipStream_t st);

}  // namespace moba
