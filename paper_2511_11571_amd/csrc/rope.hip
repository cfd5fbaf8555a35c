// Rotary positions of queries and keys in one launch, and their gradient (the turn backwards).
//
// A pair of channels (x, y) at position p becomes a (x cos - y sin, y cos + x sin), angle = p f.  The
// angle is taken in turns and in 64 bits, of which only the fraction counts: at position 10^6 a product
// in 32 bits is off by a sixteenth of a radian.
//
// A thread owns VEC pairs of one position -- two runs of VEC channels, half the turned part apart, or one
// of 2 VEC where pairs are neighbours -- and walks a stretch of the heads with their cosines and sines in
// registers.  The operator reads and writes every element once and is bound by that.  Measured, beside a library copy of the same
// tensors: 32 heads of 32768, d = 64 44 us, 6.1 TB/s (copy 6.6); 16 on 4 of 131072, d = 128, 96 channels turned 270 us, 5.0 TB/s (5.3); fp32,
// 32 of 16384, d = 128 104 us, 5.2 TB/s (5.2); a token of 8 sequences 3 us.  Two and four heads on their way at a time were no faster (44, 46; 263,
// 264; 108, 112 us) and slower for few tokens.  The turned part's width decides how wide all accesses are: 16 on 4 of 131072, d = 128, bf16,
// with 32 channels turned 271 us (8 pairs to an access), 20 284 (2), 2 390 (1); in place the same as elsewhere (128 channels 259 | 266, 32
// 271 | 273).
#include <algorithm>

#include "rope.h"

namespace moba {

// cos and sin of 2 pi f, f in [-1/2, 1/2]
template <typename T>
__device__ __forceinline__ void turn(double f, float& c, float& s)
{
    const float h = (float)f;
    if constexpr (sizeof(T) == 2) {
        // 2^-20 or so absolute, against the 2^-9 of the result's own rounding: it turns the last bit of 6 results in 100000, which
        // leaves the error against 64 bits as it is (1.6587e-3 in the 2-norm either way).  As for fp32: a call of few tokens
        // 3.3 -> 4.1 us, 16 + 16 heads of 8192, d = 64 13.0 -> 14.4.
        c = __builtin_amdgcn_cosf(h);
        s = __builtin_amdgcn_sinf(h);
    } else {
        // the fraction's rounding to 32 bits is made good to first order
        float c0, s0;
        sincospif(2.f * h, &s0, &c0);
        const float lo = (float)(f - (double)h) * 6.283185307179586f;
        c = fmaf(-lo, s0, c0);
        s = fmaf(lo, c0, s0);
    }
}

template <typename T, int VEC>
struct RopeVec;                          // VEC elements by one access
template <> struct RopeVec<bf16_t, 8> { using type = uint4; };
template <> struct RopeVec<bf16_t, 4> { using type = uint2; };
template <> struct RopeVec<bf16_t, 2> { using type = uint32_t; };
template <> struct RopeVec<bf16_t, 1> { using type = uint16_t; };
template <> struct RopeVec<float, 4> { using type = uint4; };
template <> struct RopeVec<float, 2> { using type = uint2; };
template <> struct RopeVec<float, 1> { using type = uint32_t; };

template <typename T, int VEC>
union RopeRun {
    typename RopeVec<T, VEC>::type v;
    T e[VEC];
};

template <typename T, int VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int per_row, int heads_each)
{
    using V = typename RopeVec<T, VEC>::type;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t n_all = (int64_t)a.N * per_row;
    if (i >= n_all) return;
    const int b = blockIdx.y, piece = (int)(i % per_row), n = (int)(i / per_row);
    // first channels of the thread's two runs, and of its pairs
    const int half = a.rot / 2, pair = piece * VEC;
    const bool turned = pair < half;
    int c0, c1;
    if (!turned) { c0 = 2 * pair; c1 = c0 + VEC; }           // (rot_dim .. head_dim: copied)
    else if (a.interleaved) { c0 = 2 * pair; c1 = c0 + VEC; }
    else { c0 = pair; c1 = half + pair; }
    float cs[VEC], sn[VEC];
    if (turned) {
        const double p = a.pos ? (double)a.pos[(int64_t)b * a.N + n] : (double)(a.pos0 + n);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const double t = p * a.freq[pair + e];
            turn<T>(t - rint(t), cs[e], sn[e]);
            cs[e] *= a.amp;
            sn[e] *= a.amp * a.sign;
        }
    }
    const int h_end = min(a.heads[0] + a.heads[1], (int)(blockIdx.z + 1) * heads_each);
    for (int h = blockIdx.z * heads_each; h < h_end; ++h) {
        const int w = h >= a.heads[0], hh = w ? h - a.heads[0] : h;
        const int64_t slice = (int64_t)b * a.heads[w] + hh;
        const T* x = (const T*)a.x[w] + (slice * a.xrows[w] + n) * a.D;
        T* y = (T*)a.y[w] + (slice * a.yrows[w] + n) * a.D;
        RopeRun<T, VEC> u, v;
        u.v = *reinterpret_cast<const V*>(x + c0);
        v.v = *reinterpret_cast<const V*>(x + c1);
        if (turned) {
            float f[2 * VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) { f[e] = to_f32<T>(u.e[e]); f[VEC + e] = to_f32<T>(v.e[e]); }
            float r[2 * VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float p = a.interleaved ? f[2 * e] : f[e], q = a.interleaved ? f[2 * e + 1] : f[VEC + e];
                // (written out: the same roundings whatever the width of the accesses)
                const float rp = fmaf(p, cs[e], -(q * sn[e])), rq = fmaf(q, cs[e], p * sn[e]);
                r[a.interleaved ? 2 * e : e] = rp;
                r[a.interleaved ? 2 * e + 1 : VEC + e] = rq;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) { u.e[e] = from_f32<T>(r[e]); v.e[e] = from_f32<T>(r[VEC + e]); }
        }
        *reinterpret_cast<V*>(y + c0) = u.v;
        *reinterpret_cast<V*>(y + c1) = v.v;
    }
}

template <typename T, int VEC>
static hipError_t rope_t(const RopeArgs& a, hipStream_t st)
{
    const int per_row = a.D / (2 * VEC), heads = a.heads[0] + a.heads[1];
    const int64_t groups = ((int64_t)a.N * per_row + 255) / 256;
    // heads of a thread: as many as leave the chip 2048 workgroups
    const int64_t shares = std::min<int64_t>(heads, std::max<int64_t>(1, 2048 / (groups * a.batch)));
    const int each = (int)((heads + shares - 1) / shares);
    hipLaunchKernelGGL((rope_kernel<T, VEC>), dim3((unsigned)groups, a.batch, (heads + each - 1) / each), dim3(256), 0, st,
                       a, per_row, each);
    return hipGetLastError();
}

// elements that one access may take: runs start at multiples of it, in channels and in memory
static int rope_vec(const RopeArgs& a, int es)
{
    uintptr_t at = (uintptr_t)a.x[0] | (uintptr_t)a.y[0] | (uintptr_t)a.x[1] | (uintptr_t)a.y[1];
    int v = 16 / es;
    while (v > 1 && (a.rot / 2 % v != 0 || at % ((uintptr_t)v * es) != 0)) v /= 2;
    return v;
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t st)
{
    if (a.dtype == MOBA_BF16) {
        switch (rope_vec(a, 2)) {
            case 8: return rope_t<bf16_t, 8>(a, st);
            case 4: return rope_t<bf16_t, 4>(a, st);
            case 2: return rope_t<bf16_t, 2>(a, st);
            default: return rope_t<bf16_t, 1>(a, st);
        }
    }
    switch (rope_vec(a, 4)) {
        case 4: return rope_t<float, 4>(a, st);
        case 2: return rope_t<float, 2>(a, st);
        default: return rope_t<float, 1>(a, st);
    }
}

}  // namespace moba
