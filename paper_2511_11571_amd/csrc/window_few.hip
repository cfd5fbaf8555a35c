// Causal attention to the last W keys: forward where there are few tiles of queries -- the tokens of a serving
// step against a cache, short calls.
//
// The G q_len queries of a key/value head count as one sequence of rows, position by position, 32 of which are the
// columns of every product: keys and values are read once for all heads that share them.  The waves of a workgroup
// take 32 keys at a time in turn, each through LDS of its own (the next 32 on their way in registers), without a
// barrier, and are merged at the end; where rows are few and keys many, workgroups share a row's keys and a second
// kernel merges their parts, in their order.  Bound by how fast the keys and values come in.
#include <algorithm>

#include "window_tiles.h"

namespace moba {

constexpr int kFewWaves = 4;
constexpr int kFewKeys = 32;            // keys a wave takes at a time

// parts of rows shared by workgroups: [slice][32 rows each][share][row][m (log2 units), l, O]
template <int D>
constexpr int kPartWords = D + 2;

template <typename T, int D>
__global__ __launch_bounds__(kFewWaves* kWave, sizeof(T) == 2 ? 2 : 1) void window_few_kernel(WindowArgs a, const T* __restrict__ Q,
                                                                      const T* __restrict__ K, const T* __restrict__ V,
                                                                      T* __restrict__ O, float* __restrict__ lse,
                                                                      float* __restrict__ part, int groups, int shares, int each)
{
    constexpr int NW = kFewWaves, STEPS = D / 16, MT = D / 32;
    using KV = Tile<T, D, kFewKeys>;
    constexpr int WAVE_BYTES = 2 * KV::BYTES > 32 * D * 4 ? 2 * KV::BYTES : 32 * D * 4;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float wave_ref[NW][32], wave_l[NW][32];
    const int tid = threadIdx.x, lane = tid % kWave, h = lane >> 5, m32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int skv, pos;
    if (!schedule(blockIdx.x, a.bhk, groups * shares, skv, pos)) return;
    const int group = pos / shares, share = pos % shares;
    const int rows = a.G * a.q, t0 = a.N - a.q;
    const T* Ks = K + (int64_t)skv * a.rows * D;
    const T* Vs = V + (int64_t)skv * a.rows * D;
    const int idx = min(32 * group + m32, rows - 1);         // (rows past the end: the last one again, not stored)
    const int r = idx / a.G, s = skv * a.G + idx % a.G, t = t0 + r, lo = window_first(a, s, r);
    Opnd<T> q[STEPS];
#pragma unroll
    for (int e = 0; e < STEPS; ++e) load_opnd(q[e], Q + ((int64_t)s * a.q + r) * D + 16 * e + 8 * h);
    const int lo_min = wave_min_i(lo <= t ? lo : 0x7fffffff), lo_max = wave_max_i(lo);
    const int t_min = t0 + 32 * group / a.G, t_max = t0 + min(32 * group + 31, rows - 1) / a.G;
    // the share's keys: a stretch of those that the group's rows can see by their positions
    const int from = max(0, t_min - a.W + 1) / kFewKeys * kFewKeys;
    const int first = max(from + share * each, lo_min == 0x7fffffff ? t_max + 1 : lo_min / kFewKeys * kFewKeys);
    const int end = min(from + (share + 1) * each, t_max + 1);

    unsigned char* mine = smem + wave * WAVE_BYTES;
    const float c2 = a.scale * kLog2e;
    f32x16_t acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16_t{};
    float ref = kLowest, l = 0.f;
    auto keys32 = [&](int u, bool late, bool early) __attribute__((always_inline)) {
        f32x16_t S = f32x16_t{};
#pragma unroll
        for (int e = 0; e < STEPS; ++e) {
            Opnd<T> k;
            KV::rows(k, mine, 0, e, h, m32);
            S = mma(k, q[e], S);
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
        Opnd<T> p[2];
        pack_opnd(p[0], x);
        pack_opnd(p[1], x + 8);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                Opnd<T> v;
                KV::cols(v, mine + KV::BYTES, 16 * j, mt, lane);
                acc[mt] = mma(v, p[j], acc[mt]);
            }
    };
    {
        u32x4_t mk[KV::template pieces<kWave>], mv[KV::template pieces<kWave>];
        int u = first + wave * kFewKeys;
        if (u < end) {
            KV::template load<kWave>(mk, Ks, u, a.N - 1, lane);
            KV::template load<kWave>(mv, Vs, u, a.N - 1, lane);
        }
        for (; u < end; u += NW * kFewKeys) {
            // (the wave's own LDS: its reads of the keys before are done before these stores, in order)
            KV::template store<kWave>(mk, mine, lane);
            KV::template store<kWave>(mv, mine + KV::BYTES, lane);
            if (u + NW * kFewKeys < end) {
                KV::template load<kWave>(mk, Ks, u + NW * kFewKeys, a.N - 1, lane);
                KV::template load<kWave>(mv, Vs, u + NW * kFewKeys, a.N - 1, lane);
            }
            keys32(u, u + kFewKeys - 1 > t_min, u < lo_max);
        }
    }
    // ---- merge the waves: O of every wave to LDS, 16-byte pieces of row m exchanged by m & 7
    l = sum_halves(l);
    if (h == 0) { wave_ref[wave][m32] = ref; wave_l[wave][m32] = l; }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int piece = (32 * mt + result_row(i) + 4 * h) / 4;
            *reinterpret_cast<float4*>(mine + m32 * D * 4 + 16 * (piece ^ (m32 & 7))) =
                make_float4(acc[mt][i], acc[mt][i + 1], acc[mt][i + 2], acc[mt][i + 3]);
        }
    __syncthreads();
    constexpr int TPR = NW * kWave / 32, CH = D / TPR;       // threads of a row, channels of a thread
    const int c = tid / TPR, ch0 = tid % TPR * CH;
    float top = kLowest, L = 0.f, o[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, wave_ref[w][c]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float wt = fast_exp2(wave_ref[w][c] - top);
        L = fmaf(wt, wave_l[w][c], L);
#pragma unroll
        for (int e = 0; e < CH; e += 4) {
            const float4 x = *reinterpret_cast<const float4*>(smem + w * WAVE_BYTES + c * D * 4 + 16 * (((ch0 + e) / 4) ^ (c & 7)));
            o[e] = fmaf(wt, x.x, o[e]);
            o[e + 1] = fmaf(wt, x.y, o[e + 1]);
            o[e + 2] = fmaf(wt, x.z, o[e + 2]);
            o[e + 3] = fmaf(wt, x.w, o[e + 3]);
        }
    }
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

// A workgroup per row: its waves take the row's parts in turn, eight on their way at a time, and are added up in order
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
    float top = kLowest;
    for (int x = lane; x < shares; x += kWave) top = fmaxf(top, p[x * step]);
    top = wave_max(top);
    float L = 0.f, o[D / 64] = {};
    constexpr int U = 8;
    for (int x0 = wave; x0 < shares; x0 += U * kFewWaves) {
        float m[U], l[U], y[U][D / 64];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float* at = p + min(x0 + u * kFewWaves, shares - 1) * step;
            m[u] = at[0];
            l[u] = at[1];
#pragma unroll
            for (int c = 0; c < D / 64; ++c) y[u][c] = at[2 + lane + 64 * c];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * kFewWaves >= shares) break;
            const float w = fast_exp2(m[u] - top);
            L = fmaf(w, l[u], L);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) o[c] = fmaf(w, y[u][c], o[c]);
        }
    }
    if (lane == 0) wave_sum[wave][0] = L;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) wave_sum[wave][2 + lane + 64 * c] = o[c];
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kFewWaves; ++w) {
        L += wave_sum[w][0];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) o[c] += wave_sum[w][2 + lane + 64 * c];
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

static int few_groups(const WindowDims& s) { return (s.G * s.q + 31) / 32; }
// keys that 32 rows can see between them
static int few_keys(const WindowDims& s)
{
    const int64_t positions = std::min<int64_t>(s.q, (31 + s.G - 1) / s.G + 1);
    return (int)std::min<int64_t>(s.N, s.W + positions - 1);
}
// workgroups that share a group's keys: two for every compute unit in all, and no less than two turns of every wave
static int few_shares(const WindowDims& s)
{
    const int64_t items = (int64_t)s.bhk * few_groups(s);
    const int64_t most = (few_keys(s) + 2 * kFewWaves * kFewKeys - 1) / (2 * kFewWaves * kFewKeys);
    return (int)std::max<int64_t>(1, std::min(512 / items, most));
}
bool window_few(const WindowDims& s) { return (int64_t)s.bh * ((s.q + 127) / 128) < 256; }
size_t window_few_ws_bytes(const WindowDims& s)
{
    const int n = few_shares(s);
    return n == 1 ? 0 : a256(sizeof(float) * (size_t)s.bhk * few_groups(s) * n * 32 * (s.D + 2));
}

template <typename T, int D>
static hipError_t few_t(const WindowDims& s, const void* Q, const void* K, const void* V, const int32_t* first, void* O,
                        float* lse, void* ws, hipStream_t st)
{
    const WindowArgs a = window_args(s, first);
    const int groups = few_groups(s), shares = few_shares(s);
    // keys of a share: whole turns of 32 (the first keys of a group start at a multiple of 32 up to 31 before its own)
    const int each = ((few_keys(s) + 31 + shares - 1) / shares + kFewKeys - 1) / kFewKeys * kFewKeys;
    constexpr size_t lds = kFewWaves * std::max<size_t>(2 * Tile<T, D, kFewKeys>::BYTES, 32 * D * 4);
    auto* kernel = window_few_kernel<T, D>;
    const hipError_t g = ensure_dynamic_lds((const void*)kernel, lds);
    if (g != hipSuccess) return g;
    hipLaunchKernelGGL(kernel, dim3((unsigned)schedule_grid(s.bhk, groups * shares)), dim3(kFewWaves * kWave), lds, st, a,
                       (const T*)Q, (const T*)K, (const T*)V, (T*)O, lse, (float*)ws, groups, shares, each);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || shares == 1) return e;
    hipLaunchKernelGGL((window_merge_kernel<T, D>), dim3((unsigned)(s.bh * s.q)), dim3(kFewWaves * kWave), 0, st, a, (const T*)Q,
                       (const T*)K, (const T*)V, (T*)O, lse, (const float*)ws, groups, shares);
    return hipGetLastError();
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
