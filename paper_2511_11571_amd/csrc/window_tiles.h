// Operands of the 32 x 32 matrix products of the window-attention kernels, for bf16 and fp32 alike.
//
// A step of a product contracts 16 slots.  With lane = 32 h + m, an operand holds row (or column) m, slots
// 8 h .. 8 h + 7: one v_mfma_f32_32x32x16_bf16, or eight v_mfma_f32_32x32x2_f32 of which the s-th contracts
// slots s and 8 + s.  Result element i of a lane is row 8 (i >> 2) + 4 h + (i & 3) of column m.  Elements
// 8 j .. 8 j + 7 of a result are therefore the second operand of step j of a product over its rows, whose slot
// 8 h + s is row 16 j + 8 (s >> 2) + 4 h + (s & 3): probabilities never change lanes.
//
// Tiles of rows lie in LDS row by row, the 16-byte pieces of a row at places exchanged by place(row): sixteen rows
// read at one piece (operands of rows) and four rows at four neighbouring pieces (columns) both cover the 64
// banks, 256 bytes, once.  Exchanged by row & 7, both met banks two and four times: d = 128, W = 2048, a third of the time.
#pragma once
#include "window.h"

namespace moba {

template <typename T> struct Opnd;
template <> struct Opnd<bf16_t> { Frag f; };
template <> struct Opnd<float> { float v[8]; };
// fp32 as three bf16 numbers, x = f0 + f1 + f2 exactly (24 bits; below 2^-108 the last of them may be lost): six of
// the nine products stand for one in fp32, for the others are below 2^-26 of it.  Six v_mfma_f32_32x32x16_bf16 take 192 cycles, the
// eight fp32 products 512.  us, fp32 products -> these: 16 heads of 8192, W = 256, d = 64 forward 123 -> 71, backward 367 -> 221, d = 128
// 215 -> 173, 823 -> 530; of 4096, dense, d = 128 1025 -> 444, 2190 -> 1300.  An infinity (or what rounds to one) becomes a NaN
// in two of the parts, which the second pass over sums that are not finite clears up.
struct Split {};
template <> struct Opnd<Split> { Frag f[3]; };

// type in memory
template <typename M> struct InMemory { using type = M; };
template <> struct InMemory<Split> { using type = float; };
template <typename M> using in_memory_t = typename InMemory<M>::type;

__device__ __forceinline__ f32x16_t mma(const Opnd<bf16_t>& a, const Opnd<bf16_t>& b, f32x16_t c) { return mfma32(a.f, b.f, c); }
__device__ __forceinline__ f32x16_t mma(const Opnd<float>& a, const Opnd<float>& b, f32x16_t c)
{
#pragma unroll
    for (int s = 0; s < 8; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[s], b.v[s], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ f32x16_t mma(const Opnd<Split>& a, const Opnd<Split>& b, f32x16_t c)
{
    c = mfma32(a.f[2], b.f[0], c);
    c = mfma32(a.f[0], b.f[2], c);
    c = mfma32(a.f[1], b.f[1], c);
    c = mfma32(a.f[1], b.f[0], c);
    c = mfma32(a.f[0], b.f[1], c);
    return mfma32(a.f[0], b.f[0], c);
}
__device__ __forceinline__ void split(Frag (&f)[3], const float* v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = v[2 * e], b = v[2 * e + 1];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t x = pack2(a, b);
            f[i].u[e] = x;
            a -= __uint_as_float(x << 16);
            b -= __uint_as_float(x & 0xffff0000u);
        }
    }
}

// eight neighbouring elements of a row in memory
__device__ __forceinline__ void load_opnd(Opnd<bf16_t>& o, const bf16_t* p) { o.f.q = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load_opnd(Opnd<float>& o, const float* p) { Vec8<float>::load(p, o.v); }
__device__ __forceinline__ void load_opnd(Opnd<Split>& o, const float* p)
{
    float v[8];
    Vec8<float>::load(p, v);
    split(o.f, v);
}

// eight elements of a result
__device__ __forceinline__ void pack_opnd(Opnd<bf16_t>& o, const float* p)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) o.f.u[e] = pack2(p[2 * e], p[2 * e + 1]);
}
__device__ __forceinline__ void pack_opnd(Opnd<float>& o, const float* p)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = p[e];
}
__device__ __forceinline__ void pack_opnd(Opnd<Split>& o, const float* p) { split(o.f, p); }

// a result's sixteen channels of column m to the 32 channels of row m that `to` points at.  bf16: the two lanes of a row swap
// four channels each, so that both write eight neighbouring ones.
__device__ __forceinline__ void store_result(bf16_t* to, const float (&o)[16], int h)
{
#pragma unroll
    for (int j = 0; j < 16; j += 8) {
        const auto x = __builtin_amdgcn_permlane32_swap(pack2(o[j], o[j + 1]), pack2(o[j + 4], o[j + 5]), false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(pack2(o[j + 2], o[j + 3]), pack2(o[j + 6], o[j + 7]), false, false);
        *reinterpret_cast<uint4*>(to + 2 * j + 8 * h) = make_uint4(x[0], y[0], x[1], y[1]);
    }
}
__device__ __forceinline__ void store_result(float* to, const float (&o)[16], int h)
{
#pragma unroll
    for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(to + 2 * i + 4 * h) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
}

// sum of sixteen probabilities as they are before they are rounded (in pairs: short chains)
__device__ __forceinline__ float sum16(const float (&x)[16])
{
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (x[i] + x[4 + i]) + (x[8 + i] + x[12 + i]);
    return (y[0] + y[1]) + (y[2] + y[3]);
}

// A tile of ROWS rows of D channels in LDS
template <typename T, int D, int ROWS>
struct Tile {
    static constexpr int RB = D * (int)sizeof(T), PIECES = RB / 16, LOADS = 1, BYTES = ROWS * RB;      // a piece takes LOADS loads
    static __device__ __forceinline__ constexpr int place(int row)
    {
        return PIECES == 8 ? ((row >> 1) & 1) << 2 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3);
    }

    // what NT threads move from memory to LDS: `pieces` of every thread
    template <int NT>
    static constexpr int pieces = ROWS * PIECES / NT;
    // rows first .. first + ROWS of a slice, those outside low .. high replaced by the nearer of the two
    template <int NT>
    static __device__ __forceinline__ void load(u32x4_t (&x)[ROWS * PIECES / NT], const T* __restrict__ slice, int first, int low, int high, int tid)
    {
        static_assert(ROWS * PIECES % NT == 0 && (NT % PIECES == 0), "whole pieces");
        constexpr int STEP = NT / PIECES;
        if (first >= low && first + ROWS - 1 <= high) {                      // (one offset for all lanes' pieces, the rest is scalar)
            const char* from = reinterpret_cast<const char*>(slice) + (int64_t)first * RB;
            const uint32_t at = 16u * (uint32_t)tid;
#pragma unroll
            for (int i = 0; i < ROWS * PIECES / NT; ++i) x[i] = *reinterpret_cast<const u32x4_t*>(from + i * (STEP * RB) + at);
        } else {
            const int row = first + tid / PIECES;
#pragma unroll
            for (int i = 0; i < ROWS * PIECES / NT; ++i)
                x[i] = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(slice) + (int64_t)min(max(row + i * STEP, low), high) * RB + 16 * (tid % PIECES));
        }
    }
    template <int NT>
    static __device__ __forceinline__ void store(const u32x4_t (&x)[ROWS * PIECES / NT], unsigned char* tile, int tid)
    {
#pragma unroll
        for (int i = 0; i < ROWS * PIECES / NT; ++i) {
            const int row = tid / PIECES + i * (NT / PIECES);
            *reinterpret_cast<u32x4_t*>(tile + row * RB + 16 * ((tid % PIECES) ^ place(row))) = x[i];
        }
    }

    // The same straight into LDS: a wave's instruction fills 1 KB, so a lane fetches the piece that belongs at its place.
    // The caller waits (fetched()) before the barrier after which the tile is read.
    template <int NT>
    static __device__ __forceinline__ void fetch(unsigned char* tile, const T* __restrict__ slice, int first, int low, int high, int tid)
    {
        static_assert(ROWS * PIECES % NT == 0 && NT % PIECES == 0, "whole pieces");
        const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
#pragma unroll
        for (int i = 0; i < ROWS * PIECES / NT; ++i) {
            const int row = tid / PIECES + i * (NT / PIECES);
            const char* at = reinterpret_cast<const char*>(slice) + (int64_t)min(max(first + row, low), high) * RB + 16 * ((tid % PIECES) ^ place(row));
            const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(tile + 16 * (i * NT + wave * kWave));
            // (by hand: the compiler would wait for the builtin's loads before the next read of any LDS)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(at) : "memory", "m0");
        }
    }

    // rows row0 + m, channels 16 c + 8 h .. + 7 (row0 a multiple of 16)
    static __device__ __forceinline__ void rows(Opnd<T>& o, const unsigned char* tile, int row0, int c, int h, int m)
    {
        const unsigned char* p = tile + (row0 + m) * RB;
        if constexpr (sizeof(T) == 2) {
            o.f.q = *reinterpret_cast<const uint4*>(p + ((32 * c) ^ (16 * (h ^ place(m)))));
        } else {
            const float4 a = *reinterpret_cast<const float4*>(p + ((64 * c) ^ (16 * ((2 * h) ^ place(m)))));
            const float4 b = *reinterpret_cast<const float4*>(p + ((64 * c) ^ (16 * ((2 * h + 1) ^ place(m)))));
            o.v[0] = a.x; o.v[1] = a.y; o.v[2] = a.z; o.v[3] = a.w;
            o.v[4] = b.x; o.v[5] = b.y; o.v[6] = b.z; o.v[7] = b.w;
        }
    }
    // the transpose: channel 32 mt + m, slots in the order of a result's rows, of rows row0 .. row0 + 15
    // (row0 a multiple of 16; rows eight apart have places that differ by 2)
    static __device__ __forceinline__ void cols(Opnd<T>& o, const unsigned char* tile, int row0, int mt, int lane)
    {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            const int row = 4 * h + ((lane & 15) >> 2), q = lane & 3;
            const int at = (64 * mt) ^ (16 * ((2 * ((lane >> 4) & 1) + (q >> 1)) ^ place(row)));
            const unsigned char* p = tile + (row0 + row) * RB + 8 * (q & 1);
            const uint2 a = lds_read_tr16(p + at), b = lds_read_tr16(p + 8 * RB + (at ^ 32));
            o.f.u[0] = a.x; o.f.u[1] = a.y; o.f.u[2] = b.x; o.f.u[3] = b.y;
        } else {
            const int m = lane & 31;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int r = 8 * (s >> 2) + 4 * h + (s & 3);
                o.v[s] = *reinterpret_cast<const float*>(tile + (row0 + r) * RB + ((128 * mt) ^ (16 * ((m >> 2) ^ place(r)))) + 4 * (m & 3));
            }
        }
    }
};

// fp32 rows as three tiles of bf16, split on their way into LDS: once for all waves that read them
template <int D, int ROWS>
struct Tile<Split, D, ROWS> {
    using Part = Tile<bf16_t, D, ROWS>;
    static constexpr int PIECES = Part::PIECES, LOADS = 2, BYTES = 3 * Part::BYTES;
    template <int NT>
    static constexpr int pieces = 2 * ROWS * PIECES / NT;    // (eight fp32 elements make a piece of each part)
    template <int NT>
    static __device__ __forceinline__ void load(u32x4_t (&x)[2 * ROWS * PIECES / NT], const float* __restrict__ slice, int first, int low, int high, int tid)
    {
        static_assert(ROWS * PIECES % NT == 0 && NT % PIECES == 0, "whole pieces");
#pragma unroll
        for (int i = 0; i < ROWS * PIECES / NT; ++i) {
            const int row = min(max(first + tid / PIECES + i * (NT / PIECES), low), high);
            const u32x4_t* p = reinterpret_cast<const u32x4_t*>(slice + (int64_t)row * D + 8 * (tid % PIECES));
            x[2 * i] = p[0];
            x[2 * i + 1] = p[1];
        }
    }
    template <int NT>
    static __device__ __forceinline__ void store(const u32x4_t (&x)[2 * ROWS * PIECES / NT], unsigned char* tile, int tid)
    {
#pragma unroll
        for (int i = 0; i < ROWS * PIECES / NT; ++i) {
            const int row = tid / PIECES + i * (NT / PIECES);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x[2 * i + e / 4][e % 4]);
            Frag f[3];
            split(f, v);
#pragma unroll
            for (int j = 0; j < 3; ++j)
                *reinterpret_cast<u32x4_t*>(tile + j * Part::BYTES + row * Part::RB + 16 * ((tid % PIECES) ^ Part::place(row))) = f[j].n;
        }
    }
    static __device__ __forceinline__ void rows(Opnd<Split>& o, const unsigned char* tile, int row0, int c, int h, int m)
    {
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            Opnd<bf16_t> x;
            Part::rows(x, tile + j * Part::BYTES, row0, c, h, m);
            o.f[j] = x.f;
        }
    }
    static __device__ __forceinline__ void cols(Opnd<Split>& o, const unsigned char* tile, int row0, int mt, int lane)
    {
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            Opnd<bf16_t> x;
            Part::cols(x, tile + j * Part::BYTES, row0, mt, lane);
            o.f[j] = x.f;
        }
    }
};

// Between a wave's accesses to LDS of which one lane's writes meet another lane's reads, or the other way round.  The hardware
// keeps a wave's LDS accesses in order; this says so to the compiler, and costs no instruction.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ void fetched() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Two tiles, one behind the other in LDS, on their way while a workgroup of NT threads works on two others: through
// registers, or (DIRECT) straight into LDS, which takes fewer registers.  us through registers | direct, d = 64: forward, 16 heads of
// 8192, W = 256 22.9 | 24.1, 2 x 16 of 8192, dense 379 | 358, both backward kernels 1045 | 1031 (dQ direct), 1042 | 1035 (dK and dV); d = 128, 16
// heads on 4 of 32768, W = 2048: forward 592 | 573, backward 1969 | 1953 (dQ), 2485 | 1930 (dK and dV; 26 registers spilled | 5).  Taken
// where it saves spilled registers, in dK and dV at d = 128; the forward keeps to the side of short windows.
template <class TILE, typename T, int NT, bool DIRECT>
struct Coming {
    static constexpr int P = DIRECT ? 1 : TILE::template pieces<NT>;
    u32x4_t x[P], y[P];
    __device__ __forceinline__ void start(unsigned char* to, const T* __restrict__ a, const T* __restrict__ b, int first, int low, int high, int tid)
    {
        if constexpr (DIRECT) {
            TILE::template fetch<NT>(to, a, first, low, high, tid);
            TILE::template fetch<NT>(to + TILE::BYTES, b, first, low, high, tid);
        } else {
            TILE::template load<NT>(x, a, first, low, high, tid);
            TILE::template load<NT>(y, b, first, low, high, tid);
        }
    }
    // (a barrier has to follow)
    __device__ __forceinline__ void finish(unsigned char* to, int tid)
    {
        if constexpr (DIRECT) {
            fetched();
        } else {
            TILE::template store<NT>(x, to, tid);
            TILE::template store<NT>(y, to + TILE::BYTES, tid);
        }
    }
};

// use(i, slot) for i = 0 .. N - 1, what load(i + AHEAD, slot) asks for on its way meanwhile (AHEAD + 1 slots).  Left to itself the
// compiler reads an operand, waits and multiplies.
template <int N, int AHEAD, typename L, typename U>
__device__ __forceinline__ void read_ahead(L load, U use)
{
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) load(i, i % (AHEAD + 1));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + AHEAD < N) load(i + AHEAD, (i + AHEAD) % (AHEAD + 1));
        if (AHEAD > 0) __builtin_amdgcn_sched_barrier(0);
        use(i, i % (AHEAD + 1));
    }
}

__device__ __forceinline__ int wave_min_i(int x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o, kWave));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max_i(int x) { return -wave_min_i(-x); }

// Keys that a wave's 32 rows from r0 on attend: some of them those from lo_min to t_max, all of them those from lo_max to
// t_min.  begin: a multiple of 32 that is not behind the first key of the workgroup, whose rows start at wg_r0.  With first keys
// low .. high hold all that some row of the workgroup attends, and no other row is read: padding may hold anything.
// live_min, live_max: positions of the wave's first and last row that attend something.
struct WaveKeys {
    int lo_min, lo_max, t_min, t_max, begin, low, high, live_min, live_max;
};
template <int NW>
__device__ __forceinline__ WaveKeys wave_keys(const WindowArgs& a, int t0, int wg_r0, int r0, int t, int lo, int wave, int lane, int2* wg_keys)
{
    WaveKeys k;
    k.t_min = t0 + min(r0, a.q - 1);
    k.t_max = t0 + min(r0 + 31, a.q - 1);
    if (!a.first) {                                          // first keys rise with the rows
        k.lo_min = r0 < a.q ? max(0, k.t_min - a.W + 1) : 0x7fffffff;
        k.lo_max = max(0, k.t_max - a.W + 1);
        k.begin = max(0, t0 + wg_r0 - a.W + 1) & ~31;
        k.low = 0;
        k.high = a.N - 1;
        return k;
    }
    const bool mine = r0 + (lane & 31) < a.q && lo <= t;
    const uint32_t live = (uint32_t)__ballot(mine);          // (lanes 32 .. 63 hold the same rows)
    k.lo_min = wave_min_i(mine ? lo : 0x7fffffff);
    k.lo_max = wave_max_i(lo);
    k.live_min = live ? t0 + r0 + __builtin_ctz(live) : 0x7fffffff;
    k.live_max = live ? t0 + r0 + 31 - __builtin_clz(live) : -1;
    if (lane == 0) wg_keys[wave] = make_int2(k.lo_min, k.live_max);
    __syncthreads();
    int low = wg_keys[0].x, high = wg_keys[0].y;
#pragma unroll
    for (int w = 1; w < NW; ++w) {
        low = min(low, wg_keys[w].x);
        high = max(high, wg_keys[w].y);
    }
    k.low = __builtin_amdgcn_readfirstlane(low);
    k.high = __builtin_amdgcn_readfirstlane(high);
    k.begin = k.low & ~31;
    return k;
}

// row of a result's element i
__device__ __forceinline__ constexpr int result_row(int i) { return 8 * (i >> 2) + (i & 3); }

constexpr float kLowest = -3.402823466e+38f;

}  // namespace moba
