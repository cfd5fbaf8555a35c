// Causal attention to the last W keys where there are few tiles of queries -- the tokens of a serving step against
// a cache, short calls -- forward and backward.
//
// The G q_len queries of a key/value head count as one sequence of rows, position by position, 32 of which are the
// columns of every product: keys and values are read once for all heads that share them.  The waves of a workgroup
// take 32 keys at a time in turn, each through LDS of its own (the next 32 on their way in registers), without a
// barrier, and are merged at the end; where rows are few and keys many, workgroups share a row's keys and a second
// kernel merges their parts, in their order.  The backward's waves share the walk of dQ's rows, and of dK's and dV's keys, alike.
//
// What bounds it: with many keys, how fast they come in -- 4 positions of 16 heads on 4 against 131109 keys, d = 128 50 us, 5.4 TB/s (a copy of
// that size runs at 5.4), 6 of them the second kernel, fp32 107 us, 5.0 TB/s; with few, the chain of steps: a position against 256 keys 4.5 us,
// fp32, 2 heads of 2048, W = 256 11 us forward and 20 backward.
//
// Roundings are those of the tiled kernels: bf16 P and dS enter their products in bf16, half a step of 2^-9 each, after the sums of P and
// with D in fp32; everything else is fp32.  A token's O is 2.0e-3 off 64 bits in the 2-norm where its own rounding is 1.7e-3; P in two parts
// would take that off for 2 to 6 % of a token's time (5.3 -> 5.6 us against 256 keys, 20.1 -> 21.1 for 16 positions of 16 heads on 4
// against 32768) and 6 to 20 % of a short prompt's (16 of 2048, dense 21.4 -> 24.7).
//
// fp32 at d = 128, backward, takes fp32 products and more registers than there are: both directions in one launch spill 88, dK and dV alone 25.
#include <algorithm>

#include "window_tiles.h"

namespace moba {

constexpr int kFewWaves = 4;
constexpr int kFewKeys = 32;            // keys a wave takes at a time

// fp32 products by bf16 parts where four waves' tiles of them fit (98 KB at d = 64)
template <typename T, int D>
using FewOperand = std::conditional_t<sizeof(T) == 4 && D == 64, Split, T>;
// the forward at d = 128 has them as well: values follow the keys into the same place
template <typename T>
using FewForward = std::conditional_t<sizeof(T) == 4, Split, T>;
template <typename T, int D>
constexpr bool few_one = sizeof(T) == 4 && D == 128;
template <typename M, int D, bool ONE>
constexpr int few_wave_bytes()
{
    return std::max((ONE ? 1 : 2) * Tile<M, D, kFewKeys>::BYTES, 32 * D * 4);
}

// parts of rows shared by workgroups: [slice][32 rows each][share][row][m (log2 units), l, O]
template <int D>
constexpr int kPartWords = D + 2;

// position of the last of a wave's rows, in order in its lanes 0 .. 31 and again 32 .. 63, that attends something; -1: of none
__device__ __forceinline__ int last_live(int lo, int t)
{
    const uint32_t live = (uint32_t)__ballot(lo <= t);
    return live ? __builtin_amdgcn_readlane(t, 31 - __builtin_clz(live)) : -1;
}

// O of 32 rows of every wave through LDS, 16-byte pieces of row m exchanged by m & 7; then every thread takes CH
// channels ch0 .. of row c
template <int D>
struct WaveSums {
    static constexpr int NW = kFewWaves, TPR = NW * kWave / 32, CH = D / TPR;
    static __device__ __forceinline__ void put(unsigned char* mine, const f32x16_t (&acc)[D / 32], int h, int m32)
    {
        wave_lds_order();
#pragma unroll
        for (int mt = 0; mt < D / 32; ++mt)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int piece = (32 * mt + result_row(i) + 4 * h) / 4;
                *reinterpret_cast<float4*>(mine + m32 * D * 4 + 16 * (piece ^ (m32 & 7))) =
                    make_float4(acc[mt][i], acc[mt][i + 1], acc[mt][i + 2], acc[mt][i + 3]);
            }
    }
    // o += w_wave * what the waves put
    template <typename F>
    static __device__ __forceinline__ void add(float (&o)[CH], const unsigned char* smem, int wave_bytes, int c, int ch0, F weight)
    {
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float wt = weight(w);
#pragma unroll
            for (int e = 0; e < CH; e += 4) {
                const float4 x = *reinterpret_cast<const float4*>(smem + w * wave_bytes + c * D * 4 + 16 * (((ch0 + e) / 4) ^ (c & 7)));
                o[e] = fmaf(wt, x.x, o[e]);
                o[e + 1] = fmaf(wt, x.y, o[e + 1]);
                o[e + 2] = fmaf(wt, x.z, o[e + 2]);
                o[e + 3] = fmaf(wt, x.w, o[e + 3]);
            }
        }
    }
};

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, sizeof(T) == 2 ? 2 : 1) void window_few_kernel(WindowArgs a, const T* __restrict__ Q,
                                                                      const T* __restrict__ K, const T* __restrict__ V,
                                                                      T* __restrict__ O, float* __restrict__ lse,
                                                                      float* __restrict__ part, int groups, int shares, int each)
{
    constexpr int NW = kFewWaves, STEPS = D / 16, MT = D / 32;
    using M = FewForward<T>;
    using KV = Tile<M, D, kFewKeys>;
    constexpr bool ONE = few_one<T, D>;
    constexpr int WAVE_BYTES = few_wave_bytes<M, D, ONE>();
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float wave_ref[NW][32], wave_l[NW][32];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int skv, pos;
    if (!schedule(blockIdx.x, a.bhk, groups * shares, skv, pos)) return;
    const int group = groups - 1 - pos / shares, share = pos % shares;          // (the longest rows first)
    const int rows = a.G * a.q, t0 = a.N - a.q;
    const T* Ks = K + (int64_t)skv * a.rows * D;
    const T* Vs = V + (int64_t)skv * a.rows * D;
    const int idx = min(32 * group + m32, rows - 1);         // (rows past the end: the last one again, not stored)
    const int r = idx / a.G, s = skv * a.G + idx % a.G, t = t0 + r, lo = window_first(a, s, r);
    Opnd<M> q[STEPS];
#pragma unroll
    for (int e = 0; e < STEPS; ++e) load_opnd(q[e], Q + ((int64_t)s * a.q + r) * D + 16 * e + 8 * h);
    const int t_min = t0 + 32 * group / a.G, t_max = t0 + min(32 * group + 31, rows - 1) / a.G;
    const int lo_min = a.first ? wave_min_i(lo <= t ? lo : 0x7fffffff) : max(0, t_min - a.W + 1);
    const int lo_max = a.first ? wave_max_i(lo) : max(0, t_max - a.W + 1);
    const int low = a.first ? lo_min : 0, high = a.first ? last_live(lo, t) : a.N - 1;           // (no other keys are read)
    // the share's keys: a stretch of those that the group's rows can see by their positions
    const int from = max(0, t_min - a.W + 1) / kFewKeys * kFewKeys;
    const int first = max(from + share * each, lo_min == 0x7fffffff ? t_max + 1 : lo_min / kFewKeys * kFewKeys);
    const int end = min(from + (share + 1) * each, min(t_max, high) + 1);

    unsigned char* mine = smem + wave * WAVE_BYTES;
    const float c2 = a.scale * kLog2e;
    f32x16_t acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16_t{};
    float ref = kLowest, l = 0.f;
    u32x4_t mk[KV::template pieces<kWave>], mv[KV::template pieces<kWave>];
    auto keys32 = [&](int u, bool late, bool early) __attribute__((always_inline)) {
        f32x16_t S = f32x16_t{};
#pragma unroll
        for (int e = 0; e < STEPS; ++e) {
            Opnd<M> k;
            KV::rows(k, mine, 0, e, h, m32);
            S = mma(k, q[e], S);
        }
        if constexpr (ONE) {
            wave_lds_order();
            KV::template store<kWave>(mv, mine, lane);
            wave_lds_order();
            if (u + NW * kFewKeys < end) KV::template load<kWave>(mv, Vs, u + NW * kFewKeys, low, high, lane);
        }
        float x[16], top = -INFINITY;
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
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max_nan(top, x[i]);
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
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                Opnd<M> v;
                KV::cols(v, mine + (ONE ? 0 : KV::BYTES), 16 * j, mt, lane);
                acc[mt] = mma(v, p[j], acc[mt]);
            }
    };
    {
        int u = first + wave * kFewKeys;
        if (u < end) {
            KV::template load<kWave>(mk, Ks, u, low, high, lane);
            KV::template load<kWave>(mv, Vs, u, low, high, lane);
        }
        for (; u < end; u += NW * kFewKeys) {
            wave_lds_order();                                // (the wave's own LDS: no other wave has to be waited for)
            KV::template store<kWave>(mk, mine, lane);
            if constexpr (!ONE) KV::template store<kWave>(mv, mine + KV::BYTES, lane);
            wave_lds_order();
            if (u + NW * kFewKeys < end) {
                KV::template load<kWave>(mk, Ks, u + NW * kFewKeys, low, high, lane);
                if constexpr (!ONE) KV::template load<kWave>(mv, Vs, u + NW * kFewKeys, low, high, lane);
            }
            keys32(u, u + kFewKeys - 1 > t_min, u < lo_max);
        }
    }
    // ---- merge the waves
    l = sum_halves(l);
    if (h == 0) { wave_ref[wave][m32] = ref; wave_l[wave][m32] = l; }
    using Sums = WaveSums<D>;
    constexpr int TPR = Sums::TPR, CH = Sums::CH;
    Sums::put(mine, acc, h, m32);
    __syncthreads();
    const int c = tid / TPR, ch0 = tid % TPR * CH;
    float top = kLowest, L = 0.f, o[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, wave_ref[w][c]);
#pragma unroll
    for (int w = 0; w < NW; ++w) L = fmaf(fast_exp2(wave_ref[w][c] - top), wave_l[w][c], L);
    Sums::add(o, smem, WAVE_BYTES, c, ch0, [&](int w) { return fast_exp2(wave_ref[w][c] - top); });
    const int cidx = 32 * group + c;
    if (shares > 1) {
        if (cidx < rows) {
            float* to = part + ((((int64_t)skv * groups + group) * shares + share) * 32 + c) * kPartWords<D>;
            if (ch0 == 0) { to[0] = top; to[1] = L; }
#pragma unroll
            for (int e = 0; e < CH; e += 2) *reinterpret_cast<float2*>(to + 2 + ch0 + e) = make_float2(o[e], o[e + 1]);
        }
        return;
    }
    bool odd = false;
    int cr = 0, cs = 0;
    if (cidx < rows) {
        cr = cidx / a.G;
        cs = skv * a.G + cidx % a.G;
        const int64_t row = (int64_t)cs * a.q + cr;
        const bool empty = window_first(a, cs, cr) > t0 + cr;
        const float inv = empty ? 0.f : 1.f / L;
#pragma unroll
        for (int e = 0; e < CH; e += 8) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = empty ? 0.f : o[e + i] * inv;
                odd |= !(fabsf(x[i]) < INFINITY);
            }
            Vec8<T>::store(O + row * D + ch0 + e, x);
        }
        if (ch0 == 0) lse[row] = empty ? -INFINITY : (top + fast_log2(L)) * kLn2;
    }
    // rows that are not finite once more, from their own pairs alone
    for (uint64_t bad = __ballot(odd); bad;) {
        const int x = __builtin_ctzll(bad) / TPR;
        bad &= ~(((1ull << TPR) - 1) << (x * TPR));
        plain_forward_row<T, D>(a, Q, K, V, O, lse, __shfl(cs, x * TPR, kWave), __shfl(cr, x * TPR, kWave), lane);
    }
}

// A workgroup per row: its waves take the row's parts in turn, sixteen on their way at a time, and are added up in order
template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave) void window_merge_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                                        const T* __restrict__ V, T* __restrict__ O, float* __restrict__ lse,
                                                                        const float* __restrict__ part, int groups, int shares)
{
    __shared__ float wave_sum[kFewWaves][D + 2];
    const int lane = threadIdx.x % kWave, rows = a.G * a.q;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int skv = blockIdx.x / rows, idx = blockIdx.x % rows, r = idx / a.G, s = skv * a.G + idx % a.G;
    const float* p = part + (((int64_t)skv * groups + idx / 32) * shares * 32 + idx % 32) * kPartWords<D>;
    const int64_t step = 32 * kPartWords<D>;
    float top = kLowest, L = 0.f, o[D / 64] = {};
    constexpr int U = 16;
    for (int x0 = wave; x0 < shares; x0 += U * kFewWaves) {
        float m[U], l[U], y[U][D / 64], now = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {                        // (past the end: the last one again, weight 0)
            const float* at = p + min(x0 + u * kFewWaves, shares - 1) * step;
            m[u] = at[0];
            l[u] = at[1];
#pragma unroll
            for (int c = 0; c < D / 64; ++c) y[u][c] = at[2 + lane + 64 * c];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) now = fmaxf(now, m[u]);
        const float alpha = fast_exp2(top - now);
        top = now;
        L *= alpha;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) o[c] *= alpha;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * kFewWaves >= shares) break;
            const float w = fast_exp2(m[u] - top);
            L = fmaf(w, l[u], L);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) o[c] = fmaf(w, y[u][c], o[c]);
        }
    }
    if (lane == 0) { wave_sum[wave][0] = top; wave_sum[wave][1] = L; }
#pragma unroll
    for (int c = 0; c < D / 64; ++c) wave_sum[wave][2 + lane + 64 * c] = o[c];
    __syncthreads();
    if (wave > 0) return;
    L = 0.f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) o[c] = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, wave_sum[w][0]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        const float wt = fast_exp2(wave_sum[w][0] - top);
        L = fmaf(wt, wave_sum[w][1], L);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) o[c] = fmaf(wt, wave_sum[w][2 + lane + 64 * c], o[c]);
    }
    const bool empty = window_first(a, s, r) > a.N - a.q + r;
    const int64_t row = (int64_t)s * a.q + r;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        const float x = empty ? 0.f : o[c] / L;
        odd |= !(fabsf(x) < INFINITY);
        O[row * D + lane + 64 * c] = from_f32<T>(x);
    }
    if (lane == 0) lse[row] = empty ? -INFINITY : (top + fast_log2(L)) * kLn2;
    if (__ballot(odd)) plain_forward_row<T, D>(a, Q, K, V, O, lse, s, r, lane);
}

// dQ: as the forward, the waves' sums added up at the end.  D of every row is left for dK and dV.
template <typename T, int D>
__device__ __forceinline__ void few_dq(const WindowArgs& a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                       const T* __restrict__ O, const float* __restrict__ lse, const T* __restrict__ dO,
                                       T* __restrict__ dQ, float* __restrict__ Dv, int skv, int group, unsigned char* smem)
{
    constexpr int NW = kFewWaves, STEPS = D / 16, MT = D / 32;
    using M = FewOperand<T, D>;
    using KV = Tile<M, D, kFewKeys>;
    constexpr int WAVE_BYTES = few_wave_bytes<M, D, false>();
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int rows = a.G * a.q, t0 = a.N - a.q;
    const T* Ks = K + (int64_t)skv * a.rows * D;
    const T* Vs = V + (int64_t)skv * a.rows * D;
    const int idx = min(32 * group + m32, rows - 1);
    const int r = idx / a.G, s = skv * a.G + idx % a.G, t = t0 + r, lo = window_first(a, s, r);
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
    if (wave == 0 && h == 0 && 32 * group + m32 < rows) Dv[row] = Dr;
    const float z = lse[row] * kLog2e, c2 = a.scale * kLog2e;
    const int t_min = t0 + 32 * group / a.G, t_max = t0 + min(32 * group + 31, rows - 1) / a.G;
    const int lo_min = a.first ? wave_min_i(lo <= t ? lo : 0x7fffffff) : max(0, t_min - a.W + 1);
    const int lo_max = a.first ? wave_max_i(lo) : max(0, t_max - a.W + 1);
    const int low = a.first ? lo_min : 0, high = a.first ? last_live(lo, t) : a.N - 1;
    const int u_last = min(t_max, high);
    unsigned char* mine = smem + wave * WAVE_BYTES;
    f32x16_t acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16_t{};
    {
        u32x4_t mk[KV::template pieces<kWave>], mv[KV::template pieces<kWave>];
        int u = (lo_min == 0x7fffffff ? t_max + 1 : lo_min / kFewKeys * kFewKeys) + wave * kFewKeys;
        if (u <= u_last) {
            KV::template load<kWave>(mk, Ks, u, low, high, lane);
            KV::template load<kWave>(mv, Vs, u, low, high, lane);
        }
        for (; u <= u_last; u += NW * kFewKeys) {
            wave_lds_order();
            KV::template store<kWave>(mk, mine, lane);
            KV::template store<kWave>(mv, mine + KV::BYTES, lane);
            wave_lds_order();
            if (u + NW * kFewKeys <= u_last) {
                KV::template load<kWave>(mk, Ks, u + NW * kFewKeys, low, high, lane);
                KV::template load<kWave>(mv, Vs, u + NW * kFewKeys, low, high, lane);
            }
            f32x16_t S = f32x16_t{}, dP;
#pragma unroll
            for (int i = 0; i < 16; ++i) dP[i] = -Dr;
#pragma unroll
            for (int e = 0; e < STEPS; ++e) {
                Opnd<M> k, v;
                KV::rows(k, mine, 0, e, h, m32);
                S = mma(k, q[e], S);
                KV::rows(v, mine + KV::BYTES, 0, e, h, m32);
                dP = mma(v, g[e], dP);
            }
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = fast_exp2(fmaf(S[i], c2, -z)) * dP[i];
            if (u + kFewKeys - 1 > t_min) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = result_row(i) <= t - u - 4 * h ? x[i] : 0.f;
            }
            if (u < lo_max) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = result_row(i) >= lo - u - 4 * h ? x[i] : 0.f;
            }
            Opnd<M> p[2];
            pack_opnd(p[0], x);
            pack_opnd(p[1], x + 8);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    Opnd<M> k;
                    KV::cols(k, mine, 16 * j, mt, lane);
                    acc[mt] = mma(k, p[j], acc[mt]);
                }
        }
    }
    using Sums = WaveSums<D>;
    constexpr int TPR = Sums::TPR, CH = Sums::CH;
    Sums::put(mine, acc, h, m32);
    __syncthreads();
    const int c = tid / TPR, ch0 = tid % TPR * CH;
    float o[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) o[e] = 0.f;
    Sums::add(o, smem, WAVE_BYTES, c, ch0, [](int) { return 1.f; });
    bool odd = false;
    int cr = 0, cs = 0;
    if (32 * group + c < rows) {
        cr = (32 * group + c) / a.G;
        cs = skv * a.G + (32 * group + c) % a.G;
        const float factor = dq_factor(a, window_first(a, cs, cr), t0 + cr);
#pragma unroll
        for (int e = 0; e < CH; e += 8) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = o[e + i] * factor;
                odd |= !(fabsf(x[i]) < INFINITY);
            }
            Vec8<T>::store(dQ + ((int64_t)cs * a.q + cr) * D + ch0 + e, x);
        }
    }
    // rows that are not finite once more, from their own pairs alone (their D, the first wave's stores, is there since the barrier)
    for (uint64_t bad = __ballot(odd); bad;) {
        const int x = __builtin_ctzll(bad) / TPR;
        bad &= ~(((1ull << TPR) - 1) << (x * TPR));
        plain_dq_row<T, D>(a, Q, K, V, dO, lse, Dv, dQ, __shfl(cs, x * TPR, kWave), __shfl(cr, x * TPR, kWave), lane);
    }
}

// sum over the L neighbouring lanes of a row
template <int L>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = 1; o < L; o <<= 1) x += __shfl_xor(x, o, kWave);
    return x;
}
__device__ __forceinline__ float piece_dot(const u32x4_t& x, const u32x4_t& y, bf16_t)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
        s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
    return s;
}
__device__ __forceinline__ float piece_dot(const u32x4_t& x, const u32x4_t& y, float)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(__uint_as_float(x[i]), __uint_as_float(y[i]), s);
    return s;
}

// dK and dV of 32 keys: the waves take 32 rows at a time in turn, of all heads that share the keys.  D of the rows is found
// in Dv, or (OWN) taken from O on the way, so that nothing has to be done before.
template <typename T, int D, bool OWN>
__device__ __forceinline__ void few_dkdv(const WindowArgs& a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                         const T* __restrict__ O, const float* __restrict__ lse, const T* __restrict__ dO,
                                         T* __restrict__ dK, T* __restrict__ dV, float* __restrict__ Dv, int skv, int tile,
                                         unsigned char* smem)
{
    constexpr int NW = kFewWaves, STEPS = D / 16, MT = D / 32;
    using M = FewOperand<T, D>;
    using QG = Tile<M, D, 32>;
    constexpr int WAVE_BYTES = few_wave_bytes<M, D, false>();
    __shared__ __align__(16) float stat_z[NW][32], stat_d[NW][32];
    __shared__ __align__(16) int stat_lo[NW][32];
    __shared__ int2 range[NW];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int t0 = a.N - a.q, ku = 32 * tile, key = ku + m32;
    Opnd<M> k[STEPS], v[STEPS];
    const int64_t own = ((int64_t)skv * a.rows + min(key, a.N - 1)) * D;
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
        load_opnd(k[e], K + own + 16 * e + 8 * h);
        load_opnd(v[e], V + own + 16 * e + 8 * h);
    }
    const float c2 = a.scale * kLog2e;
    int begin = max(0, ku - t0) & ~31, low = 0, high = a.q - 1;
    const int last = min(ku + 32, a.N) - 1;
    int end = (int)min((int64_t)a.q, (int64_t)last - t0 + a.W);
    if (a.first) {                                           // from the first to the last row that sees a key; no other is read
        low = 0x7fffffff;
        high = -1;
        for (int r = begin + tid; r < end; r += NW * kWave) {
            const int lo = window_first(a, skv * a.G, r);
            if (lo <= min(last, t0 + r)) {
                low = min(low, r);
                high = r;
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
    const int per = begin < end ? (end - begin + 31) / 32 : 0, total = per * a.G;
    unsigned char* mine = smem + wave * WAVE_BYTES;
    float *sz = stat_z[wave], *sd = stat_d[wave];
    int* sl = stat_lo[wave];
    f32x16_t ak[MT], av[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) ak[mt] = av[mt] = f32x16_t{};
    {
        constexpr int P = QG::template pieces<kWave>, LANES = QG::PIECES, LOADS = QG::LOADS;
        u32x4_t mq[P], mg[P], mo[OWN ? P : 1];
        float nz = 0.f, nd = 0.f;
        int nl = 0;
        auto fetch = [&](int i) __attribute__((always_inline)) {
            const int s = skv * a.G + i / per, r = begin + i % per * 32;
            const int64_t base = (int64_t)s * a.q;
            QG::template load<kWave>(mq, Q + base * D, r, low, high, lane);
            QG::template load<kWave>(mg, dO + base * D, r, low, high, lane);
            const int rr = min(r + m32, a.q - 1);
            nz = -lse[base + rr] * kLog2e;
            if constexpr (OWN) QG::template load<kWave>(mo, O + base * D, r, low, high, lane);
            else nd = -Dv[base + rr];
            nl = window_first(a, s, rr);
        };
        if (wave < total) fetch(wave);
        for (int i = wave; i < total; i += NW) {
            const int r = begin + i % per * 32;
            wave_lds_order();
            QG::template store<kWave>(mq, mine, lane);
            QG::template store<kWave>(mg, mine + QG::BYTES, lane);
            if (h == 0) { sz[m32] = nz; sl[m32] = nl; }
            if constexpr (OWN) {
#pragma unroll
                for (int j = 0; j < P / LOADS; ++j) {
                    float x = 0.f;
#pragma unroll
                    for (int e = 0; e < LOADS; ++e) x += piece_dot(mo[LOADS * j + e], mg[LOADS * j + e], T());
                    x = lanes_sum<LANES>(x);
                    if (lane % LANES == 0) sd[lane / LANES + j * (kWave / LANES)] = -x;
                }
            } else if (h == 0) {
                sd[m32] = nd;
            }
            wave_lds_order();
            // late: some key is a row's own or lies behind it; alone: the rows that attend their own key and no other
            const bool late = t0 + r <= ku + 31, early = r + 31 >= a.q || __ballot(nl > ku) != 0;
            const uint32_t alone = (uint32_t)__ballot(ds_factor(nl, t0 + r + m32) == 0.f);
            if (i + NW < total) fetch(i + NW);
            f32x16_t S = f32x16_t{}, dP;
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 x = *reinterpret_cast<const float4*>(sd + result_row(j) + 4 * h);
                dP[j] = x.x; dP[j + 1] = x.y; dP[j + 2] = x.z; dP[j + 3] = x.w;
            }
#pragma unroll
            for (int e = 0; e < STEPS; ++e) {
                Opnd<M> x;
                QG::rows(x, mine, 0, e, h, m32);
                S = mma(x, k[e], S);
                QG::rows(x, mine + QG::BYTES, 0, e, h, m32);
                dP = mma(x, v[e], dP);
            }
            float p[16], ds[16];
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 x = *reinterpret_cast<const float4*>(sz + result_row(j) + 4 * h);
                const float z[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[j + e] = fast_exp2(fmaf(S[j + e], c2, z[e]));
                    ds[j + e] = p[j + e] * dP[j + e];
                }
            }
            auto only = [&](int j, bool on) __attribute__((always_inline)) {
                p[j] = on ? p[j] : 0.f;
                ds[j] = on ? ds[j] : 0.f;
            };
            if (late) {
                const int least = key - t0 - r - 4 * h;
#pragma unroll
                for (int j = 0; j < 16; ++j) only(j, result_row(j) >= least);
                if (alone) {
                    const uint32_t rows = alone >> (4 * h);
#pragma unroll
                    for (int j = 0; j < 16; ++j) ds[j] *= rows >> result_row(j) & 1 ? 0.f : 1.f;
                }
            }
            if (early) {
                const int most = a.q - 1 - r - 4 * h;
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const int4 x = *reinterpret_cast<const int4*>(sl + result_row(j) + 4 * h);
                    only(j, (key >= x.x) & (result_row(j) <= most));
                    only(j + 1, (key >= x.y) & (result_row(j + 1) <= most));
                    only(j + 2, (key >= x.z) & (result_row(j + 2) <= most));
                    only(j + 3, (key >= x.w) & (result_row(j + 3) <= most));
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Opnd<M> pp, pd;
                pack_opnd(pp, p + 8 * j);
                pack_opnd(pd, ds + 8 * j);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    Opnd<M> x;
                    QG::cols(x, mine + QG::BYTES, 16 * j, mt, lane);
                    av[mt] = mma(x, pp, av[mt]);
                    QG::cols(x, mine, 16 * j, mt, lane);
                    ak[mt] = mma(x, pd, ak[mt]);
                }
            }
        }
    }
    using Sums = WaveSums<D>;
    constexpr int TPR = Sums::TPR, CH = Sums::CH;
    const int c = tid / TPR, ch0 = tid % TPR * CH;
    bool odd = false;
    auto out = [&](const f32x16_t(&acc)[MT], T* to, float factor) __attribute__((always_inline)) {
        Sums::put(mine, acc, h, m32);
        __syncthreads();
        float o[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) o[e] = 0.f;
        Sums::add(o, smem, WAVE_BYTES, c, ch0, [](int) { return 1.f; });
        if (ku + c >= a.N) return;
#pragma unroll
        for (int e = 0; e < CH; e += 8) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = o[e + i] * factor;
                odd |= !(fabsf(x[i]) < INFINITY);
            }
            Vec8<T>::store(to + ((int64_t)skv * a.rows + ku + c) * D + ch0 + e, x);
        }
    };
    out(ak, dK, a.scale);
    __syncthreads();
    out(av, dV, 1.f);
    // keys that are not finite once more, from their own pairs alone
    for (uint64_t bad = __ballot(odd); bad;) {
        const int x = __builtin_ctzll(bad) / TPR;
        bad &= ~(((1ull << TPR) - 1) << (x * TPR));
        const int u = ku + __shfl(c, x * TPR, kWave);
        plain_dkdv_key<T, D, OWN>(a, Q, K, V, O, dO, lse, Dv, dK, dV, skv, u, lane);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, 1) void window_few_dq_kernel(WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K,
                                                                            const T* __restrict__ V, const T* __restrict__ O,
                                                                            const float* __restrict__ lse, const T* __restrict__ dO,
                                                                            T* __restrict__ dQ, float* __restrict__ Dv, int groups)
{
    extern __shared__ __align__(16) unsigned char smem[];
    int skv, pos;
    if (schedule(blockIdx.x, a.bhk, groups, skv, pos)) few_dq<T, D>(a, Q, K, V, O, lse, dO, dQ, Dv, skv, groups - 1 - pos, smem);
}

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, 1) void window_few_dkdv_kernel(WindowArgs a, const T* __restrict__ Q,
                                                                              const T* __restrict__ K, const T* __restrict__ V,
                                                                              const float* __restrict__ lse, const T* __restrict__ dO,
                                                                              T* __restrict__ dK, T* __restrict__ dV,
                                                                              float* __restrict__ Dv, int ktiles)
{
    extern __shared__ __align__(16) unsigned char smem[];
    int skv, tile;
    if (schedule(blockIdx.x, a.bhk, ktiles, skv, tile)) few_dkdv<T, D, false>(a, Q, K, V, nullptr, lse, dO, dK, dV, Dv, skv, tile, smem);
}

// Both at once, the first `first_k` workgroups (a multiple of eight) for dQ: short calls leave half the chip to either alone
template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, 1) void window_few_backward_kernel(
    WindowArgs a, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
    const float* __restrict__ lse, const T* __restrict__ dO, T* __restrict__ dQ, T* __restrict__ dK, T* __restrict__ dV,
    float* __restrict__ Dv, int groups, int grid_q, int first_k, int ktiles)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const int b = blockIdx.x;
    int skv, pos;
    if (b < first_k) {
        if (b < grid_q && schedule(b, a.bhk, groups, skv, pos)) few_dq<T, D>(a, Q, K, V, O, lse, dO, dQ, Dv, skv, groups - 1 - pos, smem);
    } else if (schedule(b - first_k, a.bhk, ktiles, skv, pos)) {
        few_dkdv<T, D, true>(a, Q, K, V, O, lse, dO, dK, dV, Dv, skv, pos, smem);
    }
}

static int few_groups(const WindowDims& s) { return (s.G * s.q + 31) / 32; }
// keys that 32 rows can see between them
static int few_keys(const WindowDims& s)
{
    const int64_t positions = std::min<int64_t>(s.q, (31 + s.G - 1) / s.G + 1);
    return (int)std::min<int64_t>(s.N, s.W + positions - 1);
}
// Workgroups that share a group's keys: one for every compute unit in all, with two turns of every wave at least; rows of
// less than 1024 keys are not shared, for the second kernel takes 5 us.  us with at least 256 | 512 | 1024 | 2048 keys each, up to 512
// workgroups: 1 token, 16 heads on 4, d = 128, N = 4096 10.5 | 11.8 | 14.8 | 21.4; 16384 14.2 | 13.7 | 16.0 | 22.4; 131109
// 53.6 | 53.3 | 53.2 | 48.8 (the last is the one with 256 workgroups); unshared 31.7, 111, 844.
constexpr int kShareKeys = 256, kSharedKeys = 1024;
static int few_shares(const WindowDims& s)
{
    if (few_keys(s) < kSharedKeys) return 1;
    const int64_t items = (int64_t)s.bhk * few_groups(s);
    return (int)std::max<int64_t>(1, std::min<int64_t>(256 / items, few_keys(s) / kShareKeys));
}
// Calls of up to 32 positions: always, for all heads that share keys read them once (1 position of 2047 x 32 heads on 8, 512 keys,
// d = 128: 1676 -> 707 us).  Otherwise: few tiles?  The tiled kernels take as long as their longest walk where the chip is not full, the ones here cut it in four but
// take about 1.3 times as long where it is: few, where tiles x average walk < c x longest walk - x.  us, tiled | here, 16 heads,
// bf16, d = 64: forward N = 1024, W = 256 11.1 | 7.1; 2048 11.6 | 13.0; 2048 dense 40.0 | 26.0; 8192 dense 235 | 241; 4 heads of
// 8192, W = 2048 42.9 | 35.2; 4096 (16) 51.8 | 53.3.  Backward: N = 1024, W = 256 26.5 | 19.2; 2048 28.3 | 34.2; dense 4096
// 236 | 194; 8192 567 | 668; d = 128, W = 256: N = 1024 46.1 | 42.5; 2048 50.1 | 80.1; dense 2048 176 | 162, 4096 412 | 502.
// fp32, dense: d = 64 forward 4096 294 | 301, on 4 heads 240 | 303; 2048 106 | 86; 4 heads of 8192 400 | 293; d = 128 2048 189 | 170, 4096 421 | 604;
// backward 2048 562 | 633, 1024 293 | 188.
// The last positions of a longer sequence, forward, dense, bf16: against 131072 keys, 16 heads on 4, d = 128: 64 2760 | 153, 1024 2872 | 1729, 2048
// 3052 | 3278, 4096 4616 | 6373; 16 heads, d = 64: 1024 2390 | 1020, 2048 2416 | 1878, 4096 3049 | 3547; 4 heads: 4096 2342 | 990.  Against 32768, 16 on 4,
// d = 128: 1024 745 | 440, 2048 750 | 789; 16, d = 64: 2048 571 | 451, 4096 678 | 816.  The rule takes the faster one of each pair.  First keys it does not
// know: a packed batch counts as one sequence, of its window's length where that is given.
static bool few_tiles(const WindowDims& s, double tiles, double walk, double longest, double c)
{
    return tiles * walk < c * longest - (s.D == 64 ? 24000 : 12000);
}
static double few_factor(const WindowDims& s, bool backward)
{
    if (s.dtype == MOBA_F32) return s.D == 64 ? 250 : backward ? 130 : 180;
    return s.D == 64 ? 325 : backward ? 170 : 230;
}
static double all_pairs(const WindowDims& s)                 // of one head
{
    const double first = s.N - s.q, ramp = std::max<double>(0, std::min<double>(s.W, s.N) - first);
    return (2 * first + ramp + 1) * ramp / 2 + (s.q - ramp) * s.W;
}
bool window_few(const WindowDims& s)
{
    const double tiles = (double)s.bh * s.q / 128;
    return s.q <= 32 || tiles <= 128 || few_tiles(s, tiles, all_pairs(s) / s.q, s.W, few_factor(s, false));
}
size_t window_few_ws_bytes(const WindowDims& s)
{
    const int n = few_shares(s);
    return n == 1 ? 0 : a256(sizeof(float) * (size_t)s.bhk * few_groups(s) * n * 32 * (s.D + 2));
}

template <typename T, int D>
constexpr size_t few_lds = kFewWaves * few_wave_bytes<FewOperand<T, D>, D, false>();
template <typename T, int D>
static hipError_t few_t(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first, void* O,
                        float* lse, void* ws, hipStream_t st)
{
    const WindowArgs a = window_args(s, first);
    const int groups = few_groups(s), shares = few_shares(s);
    // keys of a share: whole turns of 32 (the first keys of a group start at a multiple of 32 up to 31 before its own)
    const int each = ((few_keys(s) + 31 + shares - 1) / shares + kFewKeys - 1) / kFewKeys * kFewKeys;
    constexpr size_t lds = kFewWaves * few_wave_bytes<FewForward<T>, D, few_one<T, D>>();
    auto* kernel = window_few_kernel<T, D>;
    const hipError_t g = window_lds((const void*)kernel, lds);
    if (g != hipSuccess) return g;
    hipLaunchKernelGGL(kernel, dim3((unsigned)schedule_grid(s.bhk, groups * shares)), dim3(kFewWaves * kWave), lds, st, a,
                       (const T*)Q, (const T*)K, (const T*)V, (T*)O, lse, (float*)ws, groups, shares, each);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || shares == 1) return e;
    hipLaunchKernelGGL((window_merge_kernel<T, D>), dim3((unsigned)(s.bh * s.q)), dim3(kFewWaves * kWave), 0, st, a, (const T*)Q,
                       (const T*)K, (const T*)V, (T*)O, lse, (const float*)ws, groups, shares);
    return hipGetLastError();
}

template <typename T, int D>
static hipError_t few_dq_t(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse, const void* dO,
                           const int32_t* first, void* dQ, float* Dv, hipStream_t st)
{
    const hipError_t e = window_lds((const void*)window_few_dq_kernel<T, D>, few_lds<T, D>);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_few_dq_kernel<T, D>), dim3((unsigned)schedule_grid(s.bhk, few_groups(s))), dim3(kFewWaves * kWave),
                       (few_lds<T, D>), st, window_args(s, first), (const T*)Q, (const T*)K, (const T*)V, (const T*)O, lse, (const T*)dO,
                       (T*)dQ, Dv, few_groups(s));
    return hipGetLastError();
}
template <typename T, int D>
static hipError_t few_dkdv_t(const WindowDims& s, const void* Q, const void* K, const void* V, const float* lse, const void* dO,
                             const int32_t* first, void* dK, void* dV, float* Dv, hipStream_t st)
{
    const hipError_t e = window_lds((const void*)window_few_dkdv_kernel<T, D>, few_lds<T, D>);
    if (e != hipSuccess) return e;
    const int ktiles = (s.N + 31) / 32;
    hipLaunchKernelGGL((window_few_dkdv_kernel<T, D>), dim3((unsigned)schedule_grid(s.bhk, ktiles)), dim3(kFewWaves * kWave),
                       (few_lds<T, D>), st, window_args(s, first), (const T*)Q, (const T*)K, (const T*)V, lse, (const T*)dO, (T*)dK, (T*)dV,
                       Dv, ktiles);
    return hipGetLastError();
}

template <typename T, int D>
static hipError_t few_backward_t(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse,
                                 const void* dO, const int32_t* first, void* dQ, void* dK, void* dV, float* Dv, hipStream_t st)
{
    const hipError_t e = window_lds((const void*)window_few_backward_kernel<T, D>, few_lds<T, D>);
    if (e != hipSuccess) return e;
    const int groups = few_groups(s), ktiles = (s.N + 31) / 32;
    const int grid_q = schedule_grid(s.bhk, groups), first_k = (grid_q + kXcds - 1) / kXcds * kXcds;
    hipLaunchKernelGGL((window_few_backward_kernel<T, D>), dim3((unsigned)(first_k + schedule_grid(s.bhk, ktiles))),
                       dim3(kFewWaves * kWave), (few_lds<T, D>), st, window_args(s, first), (const T*)Q, (const T*)K, (const T*)V,
                       (const T*)O, lse, (const T*)dO, (T*)dQ, (T*)dK, (T*)dV, Dv, groups, grid_q, first_k, ktiles);
    return hipGetLastError();
}

bool window_few_dq(const WindowDims& s)
{
    const double tiles = (double)s.bh * s.q / 128;
    return tiles <= 128 || few_tiles(s, tiles, all_pairs(s) / s.q, s.W, few_factor(s, true));
}
bool window_few_dkdv(const WindowDims& s)
{
    const double tiles = (double)s.bhk * s.N / 128;
    return tiles <= 128 || few_tiles(s, tiles, all_pairs(s) / s.N, std::min(s.q, s.W), few_factor(s, true));
}

hipError_t launch_window_few_dq(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse,
                                const void* dO, const int32_t* first, void* dQ, float* Dv, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? few_dq_t<bf16_t, 64>(s, Q, K, V, O, lse, dO, first, dQ, Dv, st)
                         : few_dq_t<bf16_t, 128>(s, Q, K, V, O, lse, dO, first, dQ, Dv, st);
    return s.D == 64 ? few_dq_t<float, 64>(s, Q, K, V, O, lse, dO, first, dQ, Dv, st)
                     : few_dq_t<float, 128>(s, Q, K, V, O, lse, dO, first, dQ, Dv, st);
}

// One launch for both directions' kernels gains where together they do not fill the chip and loses elsewhere, for dK and dV read O
// for every 32 keys again.  us, two launches | one, bf16: 16 heads of 100, d = 64 9.9 | 6.2; 16 of 512, W = 256 13.6 | 12.0, d = 128
// 22.1 | 26.2; 1 of 4096 22.5 | 19.3, of 8192 27.0 | 30.4; 16 on 4 of 512 33.5 | 44.8.  fp32, d = 128: 4 of 1024 70.8 | 59.6,
// of 2048 75.3 | 92.9; d = 64, W = 256: 5 of 1000 (320 workgroups) 31.9 | 29.4, 6 of 1000 31.6 | 31.5; 512 workgroups gain where the
// window is half of the keys or more, for the longest walks of either kernel then begin early: dense 16 of 512 37.1 | 35.2, 8 of 1024 61.0 | 46.7, 4 of
// 2048 109 | 82, 1 of 8192 400 | 295; 8 of 1024, W = 512 43.3 | 41.8, W = 256 31.2 | 31.2; 4 of 2048, W = 1024 68.0 | 68.8, W = 512
// 43.9 | 44.8; 2 of 4096, W = 1024 69.0 | 72.2, W = 256 32.1 | 33.5.  Dense 4 of 4096 (1024 workgroups) 249 | 268.
bool window_few_both(const WindowDims& s)
{
    const int64_t groups = (int64_t)s.bhk * (few_groups(s) + (s.N + 31) / 32);
    const int most = s.D != 64 || s.G != 1 ? 256 : s.dtype == MOBA_BF16 || s.W >= s.N / 2 ? 512 : 384;
    return window_few_dq(s) && window_few_dkdv(s) && groups <= most;
}

hipError_t launch_window_few_backward(const WindowDims& s, const void* Q, const void* K, const void* V, const void* O, const float* lse,
                                      const void* dO, const int32_t* first, void* dQ, void* dK, void* dV, float* Dv, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? few_backward_t<bf16_t, 64>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, Dv, st)
                         : few_backward_t<bf16_t, 128>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, Dv, st);
    return s.D == 64 ? few_backward_t<float, 64>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, Dv, st)
                     : few_backward_t<float, 128>(s, Q, K, V, O, lse, dO, first, dQ, dK, dV, Dv, st);
}

hipError_t launch_window_few_dkdv(const WindowDims& s, const void* Q, const void* K, const void* V, const float* lse, const void* dO,
                                  const int32_t* first, void* dK, void* dV, float* Dv, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? few_dkdv_t<bf16_t, 64>(s, Q, K, V, lse, dO, first, dK, dV, Dv, st)
                         : few_dkdv_t<bf16_t, 128>(s, Q, K, V, lse, dO, first, dK, dV, Dv, st);
    return s.D == 64 ? few_dkdv_t<float, 64>(s, Q, K, V, lse, dO, first, dK, dV, Dv, st)
                     : few_dkdv_t<float, 128>(s, Q, K, V, lse, dO, first, dK, dV, Dv, st);
}

hipError_t launch_window_few(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first, void* O,
                             float* lse, void* ws, hipStream_t st)
{
    if (s.dtype == MOBA_BF16)
        return s.D == 64 ? few_t<bf16_t, 64>(s, Q, K, V, first, O, lse, ws, st)
                         : few_t<bf16_t, 128>(s, Q, K, V, first, O, lse, ws, st);
    return s.D == 64 ? few_t<float, 64>(s, Q, K, V, first, O, lse, ws, st)
                     : few_t<float, 128>(s, Q, K, V, first, O, lse, ws, st);
}

}  // namespace moba
