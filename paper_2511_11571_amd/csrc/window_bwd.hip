// Causal attention to the last W keys: backward, which recomputes the probabilities P = exp(S - lse).
//
// Two kernels, no atomics, the same sums in every run:
//   dQ by tiles of queries, as the forward walks: S^T = K Q^T and dP^T = V dO^T, dS = P o (dP - D), dQ^T += K^T dS^T.
//     The rows' D = rowsum(dO o O) is taken here, from the operands at hand, and left for the other kernel;
//   dK and dV by tiles of keys, a wave 32 of them, walking the queries that see them, all heads that share the
//     keys one after the other: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
// Seven products for the five that are needed; one kernel for both would add dQ up by atomics or write partial
// sums of it.  D enters as the start value of the dP product.
//
// Roundings, bf16: P and dS enter their products in bf16, D comes from O as it is stored.  Against 64 bits dQ and dK are 2.8e-3
// (dense) to 3.2e-3 (W = 256) off in the 2-norm: 1.7e-3 is the rounding of the results, 1.7e-3 D, 2e-3 dS.  Without either of
// the last two it would be 2.4e-3: dS in two halves would cost two products of seven, D from the probabilities a product more
// for dQ (a quarter of its time) and at d = 128 more registers than two waves have.
//
// What bounds them: issue and latency with two or three waves a SIMD (counters, d = 64 dense: dQ matrix units 51 %, vector units 53 %
// busy; dK and dV 43 % and 43 %; d = 128, W = 2048: 53 % and 36 %, 45 % and 33 %; LDS 28 to 38 %, no bank conflicts).  Measured, dQ | dK and dV:
// 32 heads of 8192, d = 64, dense 0.44 | 0.60 ms (940 | 920 TFLOP/s of the products made); 16 heads on 4 of 32768, d = 128, W = 2048
// 0.78 | 1.15 ms (1030 | 930); 16 of 32768, d = 64, W = 256 102 | 150 us.  Slower for dK and dV at d = 64: three waves a SIMD by tiles of 32
// queries 640, of 64 (10 registers spilled) 680; two or eight waves to a workgroup 655 and 605, at W = 256 158 and 200.
// Operands are asked for one product ahead of their use where registers allow, which gains 1 to 2 %, for dQ at d = 128 5 %; two or three ahead
// the same, or as many registers spilled as to cost 15 to 60 %.  Spilled as it is: dQ at d = 64 and dK and dV at d = 128 five registers each, fp32
// dK and dV at d = 64 one.  fp32 at d = 128: three parts of a wave's own Q and dO, or K and V, are 192 registers, and dQ takes 414, dK and
// dV 437 of them in all, which leaves one wave a SIMD: 16 heads of 8192, W = 256 0.54 ms, 2.8 times what its products take.
#include "window_tiles.h"

namespace moba {

// what the kernel for dK and dV finds: D of every row and, with first keys, for 32 rows each (x, y) the smallest and largest of
// them and (z, w) the first and last row that attends something.  Rows that attend nothing count as INT_MAX in x.
struct WindowLeft {
    const float* D;             // [bh][q]
    const int4* lo;             // [batch][ceil(q / 32)]
};

// those, where the kernel for dQ by tiles has not left them: a wave per two lots of 32 rows
__global__ __launch_bounds__(256) void window_lo_kernel(WindowArgs a, int4* __restrict__ lo, int lots)
{
    const int i = blockIdx.x * 8 + threadIdx.x / 32, b = blockIdx.y;
    const int r = min(i * 32 + (int)threadIdx.x % 32, a.q - 1);
    const int first = window_first(a, b * a.heads, r);
    const bool live = first <= a.N - a.q + r;
    int least = live ? first : 0x7fffffff, most = first, live_min = live ? r : 0x7fffffff, live_max = live ? r : -1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        least = min(least, __shfl_xor(least, o, 32));
        most = max(most, __shfl_xor(most, o, 32));
        live_min = min(live_min, __shfl_xor(live_min, o, 32));
        live_max = max(live_max, __shfl_xor(live_max, o, 32));
    }
    if (i < lots && threadIdx.x % 32 == 0) lo[(int64_t)b * lots + i] = make_int4(least, most, live_min, live_max);
}

template <typename M, int D, int NW, int KT, int OCC, int QA, int QB, typename T = in_memory_t<M>>
__global__ __launch_bounds__(NW* kWave, OCC) void window_dq_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                              const T* __restrict__ V, const T* __restrict__ O,
                                                              const float* __restrict__ lse, const T* __restrict__ dO,
                                                              T* __restrict__ dQ, float* __restrict__ Dv,
                                                              int4* __restrict__ lo_out, int ntiles)
{
    constexpr int NT = NW * kWave, QT = 32 * NW, STEPS = D / 16, MT = D / 32;
    using KV = Tile<M, D, KT>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int2 wg_keys[NW];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int skv, pos;
    if (!schedule(blockIdx.x, a.bhk, a.G * ntiles, skv, pos)) return;
    const int tile = ntiles - 1 - pos / a.G, s = skv * a.G + pos % a.G;
    const T* Ks = K + (int64_t)skv * a.rows * D;
    const T* Vs = V + (int64_t)skv * a.rows * D;
    const int t0 = a.N - a.q, r0 = tile * QT + wave * 32;
    const int r = min(r0 + m32, a.q - 1), t = t0 + r, lo = window_first(a, s, r);
    const int64_t row = (int64_t)s * a.q + r;
    Opnd<M> q[STEPS], g[STEPS];
    float Dr = 0.f;
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
        const int64_t at = row * D + 16 * e + 8 * h;
        load_opnd(q[e], Q + at);
        load_opnd(g[e], dO + at);
        float x[8], y[8];
        Vec8<T>::load(dO + at, x);
        Vec8<T>::load(O + at, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) Dr = fmaf(x[i], y[i], Dr);
    }
    Dr = sum_halves(Dr);
    const bool mine = r0 + m32 < a.q;
    if (mine && h == 0) Dv[row] = Dr;
    const float z = lse[row] * kLog2e, c2 = a.scale * kLog2e;
    const WaveKeys w = wave_keys<NW>(a, t0, tile * QT, r0, t, lo, wave, lane, wg_keys);
    if (lo_out && lane == 0 && s % a.heads == 0 && r0 < a.q)
        lo_out[(int64_t)(s / a.heads) * ((a.q + 31) / 32) + r0 / 32] = make_int4(w.lo_min, w.lo_max, w.live_min - t0, w.live_max - t0);
    const int begin = w.begin, end = min(t0 + min((tile + 1) * QT, a.q), w.high + 1);

    f32x16_t acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16_t{};
    auto keys32 = [&](const unsigned char* kt, const unsigned char* vt, int row0, int u, bool late, bool early) __attribute__((always_inline)) {
        f32x16_t S = f32x16_t{}, dP;
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] = -Dr;
        {
            Opnd<M> k[QA + 1], v[QA + 1];
            read_ahead<STEPS, QA>(
                [&](int e, int i) __attribute__((always_inline)) {
                    KV::rows(k[i], kt, row0, e, h, m32);
                    KV::rows(v[i], vt, row0, e, h, m32);
                },
                [&](int e, int i) __attribute__((always_inline)) {
                    S = mma(k[i], q[e], S);
                    dP = mma(v[i], g[e], dP);
                });
        }
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fast_exp2(fmaf(S[i], c2, -z)) * dP[i];
        if (late) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = result_row(i) <= t - u - 4 * h ? x[i] : 0.f;
        }
        if (early) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = result_row(i) >= lo - u - 4 * h ? x[i] : 0.f;
        }
        Opnd<M> p[2];
        pack_opnd(p[0], x);
        pack_opnd(p[1], x + 8);
        {
            Opnd<M> k[QB + 1];
            read_ahead<2 * MT, QB>(
                [&](int e, int i) __attribute__((always_inline)) { KV::cols(k[i], kt, row0 + 16 * (e / MT), e % MT, lane); },
                [&](int e, int i) __attribute__((always_inline)) { acc[e % MT] = mma(k[i], p[e / MT], acc[e % MT]); });
        }
    };
    if (begin < end) {
        Coming<KV, T, NT, false> next;
        next.start(smem, Ks, Vs, begin, w.low, w.high, tid);
        next.finish(smem, tid);
        __syncthreads();
        // (the two buffers by turns, each with its own code: places in LDS are constants)
        auto step = [&](int u0, auto buf) __attribute__((always_inline)) {
            const unsigned char* kt = smem + decltype(buf)::value * 2 * KV::BYTES;
            unsigned char* to = smem + (decltype(buf)::value ^ 1) * 2 * KV::BYTES;
            if (u0 + KT < end) next.start(to, Ks, Vs, u0 + KT, w.low, w.high, tid);
#pragma unroll
            for (int x = 0; x < KT / 32; ++x) {
                const int u = u0 + 32 * x;
                if (u > w.t_max || u + 31 < w.lo_min) continue;
                keys32(kt, kt + KV::BYTES, 32 * x, u, u + 31 > w.t_min, u < w.lo_max);
            }
            if (u0 + KT < end) next.finish(to, tid);
            __syncthreads();
        };
        for (int u0 = begin; u0 < end; u0 += 2 * KT) {
            step(u0, std::integral_constant<int, 0>());
            if (u0 + KT < end) step(u0 + KT, std::integral_constant<int, 1>());
        }
    }
    const float factor = dq_factor(a, lo, t);
    float most = 0.f;
    if (mine) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float o[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                o[i] = acc[mt][i] * factor;
                most = max_nan(most, fabsf(o[i]));
            }
            store_result(dQ + row * D + 32 * mt, o, h);
        }
    }
    // rows with a sum that is not finite once more, from their own pairs alone
    uint64_t bad = __ballot(!(most < INFINITY));
    bad = (bad | bad >> 32) & 0xffffffffu;
    for (; bad; bad &= bad - 1) plain_dq_row<T, D>(a, Q, K, V, dO, lse, Dv, dQ, s, r0 + __builtin_ctzll(bad), lane);
}

// KA, KB: how many products ahead the operands of the first two and of the last two are read
template <typename M, int D, int NW, int QT, int OCC, bool DIRECT, int KA, int KB, typename T = in_memory_t<M>>
__global__ __launch_bounds__(NW* kWave, OCC) void window_dkdv_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                                const T* __restrict__ V, const float* __restrict__ lse,
                                                                const T* __restrict__ dO, T* __restrict__ dK,
                                                                T* __restrict__ dV, WindowLeft left, int ntiles)
{
    constexpr int NT = NW * kWave, KTILE = 32 * NW, STEPS = D / 16, MT = D / 32;
    static_assert(QT <= kWave, "a lane per row of a tile");
    using QG = Tile<M, D, QT>;
    extern __shared__ __align__(16) unsigned char smem[];    // Q, dO | Q, dO
    __shared__ __align__(16) float stat_z[2][QT], stat_d[2][QT];             // -lse (log2 units), -D
    __shared__ __align__(16) int stat_lo[2][QT];
    __shared__ int2 range[NW];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int skv, tile;
    if (!schedule(blockIdx.x, a.bhk, ntiles, skv, tile)) return;             // (the first keys have the most queries)
    const int t0 = a.N - a.q, k0 = tile * KTILE, ku = k0 + wave * 32, key = ku + m32;
    Opnd<M> k[STEPS], v[STEPS];
    {
        const int64_t at = ((int64_t)skv * a.rows + min(key, a.N - 1)) * D;  // (keys past the end: the last one, not stored)
#pragma unroll
        for (int e = 0; e < STEPS; ++e) {
            load_opnd(k[e], K + at + 16 * e + 8 * h);
            load_opnd(v[e], V + at + 16 * e + 8 * h);
        }
    }
    const float c2 = a.scale * kLog2e;
    // rows that may see a key of the workgroup: from the first key's own on, to the last key's last one
    int begin = max(0, k0 - t0) & ~31, low = 0, high = a.q - 1;
    const int last = min(k0 + KTILE, a.N) - 1;
    int end = (int)min((int64_t)a.q, (int64_t)last - t0 + a.W);
    const int4* lo_of = left.lo ? left.lo + (int64_t)(skv * a.G / a.heads) * ((a.q + 31) / 32) : nullptr;
    if (lo_of) {                                             // ... that belong to the same sequence, and no row of padding at either end
        low = 0x7fffffff;
        high = -1;
        for (int i = begin / 32 + tid; i < (end + 31) / 32; i += NT) {
            const int4 x = lo_of[i];
            if (x.x <= last) {
                low = min(low, x.z);
                high = max(high, x.w);
            }
        }
        low = wave_min_i(low);
        high = wave_max_i(high);
        if (lane == 0) range[wave] = make_int2(low, high);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            low = min(low, range[w].x);
            high = max(high, range[w].y);
        }
        low = __builtin_amdgcn_readfirstlane(low);
        high = __builtin_amdgcn_readfirstlane(high);
        begin = max(begin, low & ~31);
        end = min(end, high + 1);
    }
    f32x16_t ak[MT], av[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) ak[mt] = av[mt] = f32x16_t{};

    // rows r .. r + 31 of the tile in LDS (from its row row0 on) against the wave's keys; late: some key is a row's own or lies
    // behind it; alone: some row may attend its own key and no other
    auto rows32 = [&](const unsigned char* qt, const unsigned char* gt, const float* sz, const float* sd, const int* sl, int row0, int r,
                      bool late, bool early, bool alone) __attribute__((always_inline)) {
        f32x16_t S = f32x16_t{}, dP;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 x = *reinterpret_cast<const float4*>(sd + row0 + result_row(i) + 4 * h);
            dP[i] = x.x; dP[i + 1] = x.y; dP[i + 2] = x.z; dP[i + 3] = x.w;
        }
        {
            Opnd<M> x[KA + 1], y[KA + 1];
            read_ahead<STEPS, KA>(
                [&](int e, int i) __attribute__((always_inline)) {
                    QG::rows(x[i], qt, row0, e, h, m32);
                    QG::rows(y[i], gt, row0, e, h, m32);
                },
                [&](int e, int i) __attribute__((always_inline)) {
                    S = mma(x[i], k[e], S);
                    dP = mma(y[i], v[e], dP);
                });
        }
        float p[16], ds[16];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 x = *reinterpret_cast<const float4*>(sz + row0 + result_row(i) + 4 * h);
            const float z[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[i + e] = fast_exp2(fmaf(S[i + e], c2, z[e]));
                ds[i + e] = p[i + e] * dP[i + e];
            }
        }
        // rows from the key's own on ...
        auto only = [&](int i, bool on) __attribute__((always_inline)) {
            p[i] = on ? p[i] : 0.f;
            ds[i] = on ? ds[i] : 0.f;
        };
        if (late) {
            const int least = key - t0 - r - 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i) only(i, result_row(i) >= least);
            if (alone) {
                const uint32_t rows = (uint32_t)__ballot(ds_factor(sl[row0 + m32], t0 + r + m32) == 0.f) >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] *= rows >> result_row(i) & 1 ? 0.f : 1.f;
            }
        }
        if (early) {
            // ... up to the last that exists and whose window still holds it; with first keys, by each row's own
            const int most = min(a.q - 1 - r, key - t0 - r + a.W - 1) - 4 * h;               // (sums of numbers up to 2^24)
#pragma unroll
            for (int i = 0; i < 16; ++i) only(i, result_row(i) <= most);
            if (lo_of) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int4 x = *reinterpret_cast<const int4*>(sl + row0 + result_row(i) + 4 * h);
                    only(i, key >= x.x);
                    only(i + 1, key >= x.y);
                    only(i + 2, key >= x.z);
                    only(i + 3, key >= x.w);
                }
            }
        }
        Opnd<M> pp[2], pd[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            pack_opnd(pp[j], p + 8 * j);
            pack_opnd(pd[j], ds + 8 * j);
        }
        {
            Opnd<M> x[KB + 1], y[KB + 1];
            read_ahead<2 * MT, KB>(
                [&](int e, int i) __attribute__((always_inline)) {
                    QG::cols(x[i], gt, row0 + 16 * (e / MT), e % MT, lane);
                    QG::cols(y[i], qt, row0 + 16 * (e / MT), e % MT, lane);
                },
                [&](int e, int i) __attribute__((always_inline)) {
                    av[e % MT] = mma(x[i], pp[e / MT], av[e % MT]);
                    ak[e % MT] = mma(y[i], pd[e / MT], ak[e % MT]);
                });
        }
    };
    float nz = 0.f, nd = 0.f;
    int nl = 0;
    Coming<QG, T, NT, DIRECT> next;
    int2 lo_next[QT / 32], lo_here[QT / 32];
    auto fetch = [&](int g, int r, int buf) __attribute__((always_inline)) {
        const int s = skv * a.G + g;
        const int64_t base = (int64_t)s * a.q;
        if (tid < QT) {
            const int rr = min(r + tid, a.q - 1);
            nz = -lse[base + rr] * kLog2e;
            nd = -left.D[base + rr];
            nl = window_first(a, s, rr);
        }
#pragma unroll
        for (int x = 0; x < QT / 32; ++x) {
            const int rx = min(r + 32 * x, a.q - 1);
            lo_next[x] = lo_of ? *reinterpret_cast<const int2*>(lo_of + rx / 32) : make_int2(max(0, t0 + rx - a.W + 1), max(0, t0 + rx + 31 - a.W + 1));
        }
        next.start(smem + buf * 2 * QG::BYTES, Q + base * D, dO + base * D, r, low, high, tid);
    };
    // the tile is there: its rows' statistics go to LDS, too
    auto arrived = [&](int buf) __attribute__((always_inline)) {
        next.finish(smem + buf * 2 * QG::BYTES, tid);
        if (tid < QT) {
            stat_z[buf][tid] = nz;
            stat_d[buf][tid] = nd;
            stat_lo[buf][tid] = nl;
        }
#pragma unroll
        for (int x = 0; x < QT / 32; ++x)
            lo_here[x] = make_int2(__builtin_amdgcn_readfirstlane(lo_next[x].x), __builtin_amdgcn_readfirstlane(lo_next[x].y));
        __syncthreads();
    };
    if (begin < end) {
        fetch(0, begin, 0);
        arrived(0);
        int g = 0, r0 = begin, buf = 0;
        for (bool more = true; more; buf ^= 1) {
            const int r_here = r0;
            r0 += QT;
            if (r0 >= end) { r0 = begin; ++g; }
            more = g < a.G;
            if (more) fetch(g, r0, buf ^ 1);
            const unsigned char* qt = smem + buf * 2 * QG::BYTES;
#pragma unroll
            for (int x = 0; x < QT / 32; ++x) {
                const int r = r_here + 32 * x;
                if (r >= a.q || t0 + min(r + 31, a.q - 1) < ku || ku >= a.N || lo_here[x].x > ku + 31) continue;
                rows32(qt, qt + QG::BYTES, stat_z[buf], stat_d[buf], stat_lo[buf], 32 * x, r, t0 + r <= ku + 31, r + 31 >= a.q || lo_here[x].y > ku,
                       lo_here[x].y >= t0 + r);
            }
            if (more) arrived(buf ^ 1);
        }
    }
    float most = 0.f;
    if (key < a.N) {
        const int64_t at = ((int64_t)skv * a.rows + key) * D;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float x[16], y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = ak[mt][i] * a.scale;
                y[i] = av[mt][i];
                most = max_nan(max_nan(most, fabsf(x[i])), fabsf(y[i]));
            }
            store_result(dK + at + 32 * mt, x, h);
            store_result(dV + at + 32 * mt, y, h);
        }
    }
    // keys with a sum that is not finite once more, from their own pairs alone
    uint64_t bad = __ballot(!(most < INFINITY));
    bad = (bad | bad >> 32) & 0xffffffffu;
    for (; bad; bad &= bad - 1) plain_dkdv_key<T, D, false>(a, Q, K, V, nullptr, dO, lse, left.D, dK, dV, skv, ku + __builtin_ctzll(bad), lane);
}

// [D of every row][first keys of 32 rows each]
static size_t rows_bytes(const WindowDims& s) { return a256(sizeof(float) * (size_t)s.bh * s.q); }
size_t window_backward_ws_bytes(const WindowDims& s) { return rows_bytes(s) + a256(sizeof(int4) * (size_t)s.batch * ((s.q + 31) / 32)); }

template <typename M, int D, int NW, int KT, int QT, int OCCQ, int OCCK, bool DIRECT, int KA, int KB, int QA, int QB>
static hipError_t backward_t(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O,
                             const float* lse, const void* dO, const int32_t* first, void* dQ, void* dK, void* dV,
                             void* ws, hipStream_t st)
{
    using T = in_memory_t<M>;
    const WindowArgs a = window_args(s, first);
    float* Dv = static_cast<float*>(ws);
    const bool few_q = window_few_dq(s), few_k = window_few_dkdv(s);
    if (window_few_both(s)) return launch_window_few_backward(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, Dv, st);
    int4* lo = first && !few_k ? reinterpret_cast<int4*>(static_cast<char*>(ws) + rows_bytes(s)) : nullptr;
    hipError_t e;
    if (few_q) {
        e = launch_window_few_dq(s, Q, K, V, O, lse, dO, first, dQ, Dv, st);
        if (e != hipSuccess) return e;
    } else {
        constexpr size_t lds = 4 * Tile<M, D, KT>::BYTES;
        auto* kernel = window_dq_kernel<M, D, NW, KT, OCCQ, QA, QB>;
        e = window_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        const int tiles = (s.q + 32 * NW - 1) / (32 * NW);
        hipLaunchKernelGGL(kernel, dim3((unsigned)schedule_grid(s.bhk, s.G * tiles)), dim3(NW * kWave), lds, st, a, (const T*)Q,
                           (const T*)K, (const T*)V, (const T*)O, lse, (const T*)dO, (T*)dQ, Dv, lo, tiles);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (few_k) return launch_window_few_dkdv(s, Q, K, V, lse, dO, first, dK, dV, Dv, st);
    if (lo && few_q) {
        const int lots = (s.q + 31) / 32;
        hipLaunchKernelGGL(window_lo_kernel, dim3((lots + 7) / 8, s.batch), dim3(256), 0, st, a, lo, lots);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    constexpr size_t lds = 4 * Tile<M, D, QT>::BYTES;
    auto* kernel = window_dkdv_kernel<M, D, NW, QT, OCCK, DIRECT, KA, KB>;
    e = window_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    const int tiles = (s.N + 32 * NW - 1) / (32 * NW);
    hipLaunchKernelGGL(kernel, dim3((unsigned)schedule_grid(s.bhk, tiles)), dim3(NW * kWave), lds, st, a, (const T*)Q, (const T*)K,
                       (const T*)V, lse, (const T*)dO, (T*)dK, (T*)dV, WindowLeft{Dv, lo}, tiles);
    return hipGetLastError();
}

hipError_t launch_window_backward(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O,
                                  const float* lse, const void* dO, const int32_t* first, void* dQ, void* dK, void* dV,
                                  void* ws, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? backward_t<bf16_t, 64, 4, 64, 64, 3, 2, false, 1, 1, 0, 1>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st)
                         : backward_t<bf16_t, 128, 4, 32, 32, 2, 2, true, 0, 1, 1, 1>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st);
    return s.D == 64 ? backward_t<Split, 64, 4, 32, 32, 2, 2, false, 0, 0, 0, 0>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st)
                     : backward_t<Split, 128, 4, 32, 32, 1, 1, false, 0, 0, 0, 0>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, ws, st);
}

}  // namespace moba
