// Causal attention to the last W keys: forward, O = softmax(scale Q K^T) V over max(0, t - W + 1, first key) .. t.
//
// A workgroup takes a tile of 128 neighbouring queries of one head, a wave 32 of them, and walks the keys that some of
// them attend in tiles of KT rows through LDS (two tiles, the next one on its way through registers).  Scores are computed
// transposed, S^T = K Q^T, so that a lane holds a query's scores of half the keys and the softmax's maximum and sum cost
// one exchange of halves; O^T = V^T P^T takes P as it comes out.  Statistics and sums are fp32; P enters its product in the
// I/O type (half a step, 2^-9 of it, which the sum over the keys averages), its sum is taken before that.
//
// The reference m of a row's exponents follows its maximum only when that has grown by more than 2^8: P stays
// below 2^8, and most tiles scale nothing.
//
// What bounds it: instruction issue, products and vector units by turns.  A lot of 32 keys x 32 queries at d = 64 is 256 cycles of
// products and some 400 of exponentials, multiply-adds, maxima, sums and roundings (counters, dense: matrix units 41 %, vector
// units 72 % busy, LDS 31 %), at d = 128 512 and 450 (44 %, 47 %); the chip's clock goes down to 1.8 GHz meanwhile.  Measured: 16
// heads on 4 of 16384, d = 128, dense 1.13 ms, 970 TFLOP/s (a library product of 8192^3 1330); 32 of 8192, d = 64, dense 0.38 ms, 725;
// W = 256, 16 of 32768, d = 64 78 us: 3.4 TB/s of Q, K, V and O, a wave has 9 lots and as much again to begin and end.
// Slower, us at W = 256, 16 heads of 8192 (25 as it is): 64 queries to a wave 31, two waves to a workgroup 35, eight 26, tiles
// of 32 keys 26, two lots at once 29; priorities for the products, dense 16384: 1.11 -> 1.21 ms; without operands read
// ahead of their products 1 to 2 % at each size.  Slower there and faster for long walks: weights by the old reference first and a
// maximum only where they come out large, at three waves a SIMD (four spill): 16 of 32768, W = 256 76 -> 83, 32 of 8192, dense 371 ->
// 352; tiles straight into LDS, 23 -> 24 and 379 -> 358.
#include "window_tiles.h"

namespace moba {

template <typename M, int D, int NW, int KT, int OCC, int KA, int VA, typename T = in_memory_t<M>>
__global__ __launch_bounds__(NW* kWave, OCC) void window_forward_kernel(WindowArgs a, const T* __restrict__ Q,
                                                                   const T* __restrict__ K, const T* __restrict__ V,
                                                                   T* __restrict__ O, float* __restrict__ lse, int ntiles)
{
    constexpr int NT = NW * kWave, QT = 32 * NW, STEPS = D / 16, MT = D / 32;
    using KV = Tile<M, D, KT>;
    extern __shared__ __align__(16) unsigned char smem[];    // K, V | K, V
    __shared__ int2 wg_keys[NW];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int skv, pos;
    if (!schedule(blockIdx.x, a.bhk, a.G * ntiles, skv, pos)) return;
    const int tile = ntiles - 1 - pos / a.G, s = skv * a.G + pos % a.G;      // the longest rows first
    const T* Ks = K + (int64_t)skv * a.rows * D;
    const T* Vs = V + (int64_t)skv * a.rows * D;
    const int t0 = a.N - a.q, r0 = tile * QT + wave * 32;
    const int r = min(r0 + m32, a.q - 1), t = t0 + r, lo = window_first(a, s, r);            // (rows past the end: the last one again, not stored)
    const int64_t row = (int64_t)s * a.q + r;
    Opnd<M> q[STEPS];
#pragma unroll
    for (int e = 0; e < STEPS; ++e) load_opnd(q[e], Q + row * D + 16 * e + 8 * h);
    const WaveKeys k = wave_keys<NW>(a, t0, tile * QT, r0, t, lo, wave, lane, wg_keys);
    const int begin = k.begin, end = min(t0 + min((tile + 1) * QT, a.q), k.high + 1);        // (begin beyond it: nobody attends anything)

    const float c2 = a.scale * kLog2e;
    f32x16_t acc[MT];
    float ref = kLowest, l = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16_t{};
    auto keys32 = [&](const unsigned char* kt, const unsigned char* vt, int row0, int u, bool late, bool early) __attribute__((always_inline)) {
        f32x16_t S = f32x16_t{};
        {
            Opnd<M> k[KA + 1];
            read_ahead<STEPS, KA>([&](int e, int i) __attribute__((always_inline)) { KV::rows(k[i], kt, row0, e, h, m32); },
                                  [&](int e, int i) __attribute__((always_inline)) { S = mma(k[i], q[e], S); });
        }
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = S[i];
        if (late) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = result_row(i) <= t - u - 4 * h ? x[i] : -INFINITY;
        }
        if (early) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = result_row(i) >= lo - u - 4 * h ? x[i] : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = max_nan(top, x[i]);
        top = max_halves(top) * c2;
        if (__ballot(top > ref + 8.f)) {
            const float now = fmaxf(ref, top), alpha = fast_exp2(ref - now);
            ref = now;
            l *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[mt] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fast_exp2(fmaf(x[i], c2, -ref));
        l += sum16(x);
        Opnd<M> p[2];
        pack_opnd(p[0], x);
        pack_opnd(p[1], x + 8);
        {
            Opnd<M> v[VA + 1];
            read_ahead<2 * MT, VA>(
                [&](int e, int i) __attribute__((always_inline)) { KV::cols(v[i], vt, row0 + 16 * (e / MT), e % MT, lane); },
                [&](int e, int i) __attribute__((always_inline)) { acc[e % MT] = mma(v[i], p[e / MT], acc[e % MT]); });
        }
    };
    if (begin < end) {
        Coming<KV, T, NT, false> next;
        next.start(smem, Ks, Vs, begin, k.low, k.high, tid);
        next.finish(smem, tid);
        __syncthreads();
        // (the two buffers by turns, each with its own code: places in LDS are constants)
        auto step = [&](int u0, auto buf) __attribute__((always_inline)) {
            const unsigned char* kt = smem + decltype(buf)::value * 2 * KV::BYTES;
            unsigned char* to = smem + (decltype(buf)::value ^ 1) * 2 * KV::BYTES;
            if (u0 + KT < end) next.start(to, Ks, Vs, u0 + KT, k.low, k.high, tid);
#pragma unroll
            for (int x = 0; x < KT / 32; ++x) {
                const int u = u0 + 32 * x;
                if (u > k.t_max || u + 31 < k.lo_min) continue;
                keys32(kt, kt + KV::BYTES, 32 * x, u, u + 31 > k.t_min, u < k.lo_max);
            }
            if (u0 + KT < end) next.finish(to, tid);
            __syncthreads();
        };
        for (int u0 = begin; u0 < end; u0 += 2 * KT) {
            step(u0, std::integral_constant<int, 0>());
            if (u0 + KT < end) step(u0 + KT, std::integral_constant<int, 1>());
        }
    }
    const bool empty = lo > t;
    const float L = sum_halves(l), inv = empty ? 0.f : 1.f / L;
    float most = 0.f;
    if (r0 + m32 < a.q) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float o[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                o[i] = acc[mt][i] * inv;
                most = max_nan(most, fabsf(o[i]));
            }
            store_result(O + row * D + 32 * mt, o, h);
        }
        if (h == 0) lse[row] = empty ? -INFINITY : (ref + fast_log2(L)) * kLn2;
    }
    // A weight of zero does not hide an infinity or a NaN: such rows are done once more, from their own pairs alone
    uint64_t bad = __ballot(!(most < INFINITY));
    bad = (bad | bad >> 32) & 0xffffffffu;
    for (; bad; bad &= bad - 1) plain_forward_row<T, D>(a, Q, K, V, O, lse, s, r0 + __builtin_ctzll(bad), lane);
}

size_t window_forward_ws_bytes(const WindowDims& s) { return window_few(s) ? window_few_ws_bytes(s) : 0; }

template <typename M, int D, int NW, int KT, int OCC, int KA, int VA>
static hipError_t tiles_t(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                          void* O, float* lse, hipStream_t st)
{
    using T = in_memory_t<M>;
    auto* kernel = window_forward_kernel<M, D, NW, KT, OCC, KA, VA>;
    constexpr size_t lds = 4 * Tile<M, D, KT>::BYTES;
    const hipError_t e = window_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    constexpr int QT = 32 * NW;
    const int ntiles = (s.q + QT - 1) / QT;
    hipLaunchKernelGGL(kernel, dim3((unsigned)schedule_grid(s.bhk, s.G * ntiles)), dim3(NW * kWave), lds, st,
                       window_args(s, first), (const T*)Q, (const T*)K, (const T*)V, (T*)O, lse, ntiles);
    return hipGetLastError();
}

hipError_t launch_window_forward(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first,
                                 void* O, float* lse, void* ws, hipStream_t st)
{
    if (window_few(s)) return launch_window_few(s, Q, K, V, first, O, lse, ws, st);
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? tiles_t<bf16_t, 64, 4, 64, 4, 0, 1>(s, Q, K, V, first, O, lse, st)
                         : tiles_t<bf16_t, 128, 4, 64, 2, 2, 3>(s, Q, K, V, first, O, lse, st);
    return s.D == 64 ? tiles_t<Split, 64, 4, 32, 3, 0, 0>(s, Q, K, V, first, O, lse, st)
                     : tiles_t<Split, 128, 4, 32, 1, 0, 0>(s, Q, K, V, first, O, lse, st);
}

}  // namespace moba
