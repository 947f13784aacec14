// Codes in 8-bit floating point with a scale per block of 128 values:
//   top = max |x| of the block (at least 2^-100),  s = top / max,  code = nearest value of the format to x max / top
// or, with scales as powers of two, s = the smallest 2^e >= top / max.  Blocks lie along a row (rows), down a column (cols, codes
// transposed) or are 128 x 128 tiles (tiles, tiles_t).  Every value is read once and its code written once; memory bounds all four.
#include <algorithm>

#include "fp8_common.h"

namespace trdq {
namespace {

using namespace fp8;

constexpr int kThreads = 256;

struct QuantArgs {
    const void *X;
    uint8_t *Q;
    void *S;
    int64_t ldx, ldq, lds;
    int rows, c;               // of X
    int nkb;                   // blocks along the codes' rows
    int groups;                // rows: groups of KT blocks; turned forms: column tiles
    int first;                 // rows: the launch's first row
};

// ---- the nearest code -----------------------------------------------------------------------------
// A value's code is the nearest to the exact quotient x max / top, ties to even.  Both are brought next to 1 by a power of two (no step
// overflows, and none of those that decide about a code underflows): with t = 0.875 x and top2 = top / 2^TopExp, q0 = t rc is within
// two steps of t / top2 and one step of the residual, fma(t - q0 top2, rc, q0), gives the nearest float.
//   x of bf16: t is exact, and quotients that are no border between two codes are further from it than a float's rounding (x max and
//   top have 11 and 8 bits): the nearest float is on a border where the quotient is, which many are.
//   x of float32: t leaves a remainder tl, which joins the residual, and a quotient may be that near to a border without being on
//   it.  So a float that is not the quotient gives its place to the one of its two neighbours around the quotient that is odd: borders
//   have few bits, are even, and none lies between it and the quotient.  (The sign of what is left is right: where the fma
//   has more than 24 bits, tl is at most half of it.)  Most values need none of that: x k (1 - 2^-20) and x k (1 + 2^-20), with k within
//   2^-21 of max / top, lie on both sides of the quotient, and where they have the same code so has it; one value in 2^15 does not
//   (by rows, us, all steps for every value / so: 16384 x 1152 19.2 / 16.4, 1003 x 771 5.9 / 5.1; bf16 values, many on borders, 5.4 / 6.1
//   at 4096 x 1152).
struct Divisor {
    float rc, top2, pre;       // 1 / top2, top2 and 0.875, the latter two times the power; e8m0: the factor 2^-e, 0, 0

    template <int FMT, bool POW2>
    __device__ __forceinline__ static Divisor of(uint32_t top_bits, const BlockScale &b)
    {
        if constexpr (POW2) return {b.rc, 0.0f, 0.0f};
        const float nan = __uint_as_float(0x7FC00000u);
        const bool bad = top_bits >= 0x7F800000u;
        top_bits = umax(top_bits, (uint32_t)(127 - 100) << 23);
        const float power = __uint_as_float((256u - (top_bits >> 23)) << 23);                     // top power lies in [4, 8)
        const float top2 = __uint_as_float(top_bits) * power * (TopExp<FMT>::value == 9 ? 0x1p-9f : 0x1p-16f);
        const float r = __builtin_amdgcn_rcpf(top2);
        return {bad ? nan : __builtin_fmaf(__builtin_fmaf(-top2, r, 1.0f), r, r), top2, 0.875f * power};
    }

    template <bool POW2, bool F32>
    __device__ __forceinline__ float quotient(float x) const
    {
        if constexpr (POW2) return x * rc;
        const float t = x * pre, q0 = t * rc, r = __builtin_fmaf(-q0, top2, t);
        if constexpr (!F32) return __builtin_fmaf(r, rc, q0);
        const float tl = __builtin_fmaf(x, pre, -t);
        const float q = __builtin_fmaf(r + tl, rc, q0);
        const uint32_t bits = __float_as_uint(q), rest = __float_as_uint(__builtin_fmaf(-q, top2, t) + tl);      // (+0 where nothing is left)
        const uint32_t some = rest < 1u ? rest : 1u, beyond = (uint32_t)((int32_t)(bits ^ rest) >> 31) & some;
        return __uint_as_float((bits - beyond) | some);
    }
    __device__ __forceinline__ float about() const { return rc * pre; }      // max / top, float32 scales
};

// The codes of eight values of a block.  about: of its divisor, for float32 values and scales; divisor(): itself, where it is needed.
template <int FMT, bool POW2, bool F32, class F>
__device__ __forceinline__ u32x2_t codes8(const float (&x)[8], float about, F &&divisor)
{
    float v[8];
    auto all = [&](auto &&f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = f(x[j]);
        return u32x2_t{pack4<FMT>(v[0], v[1], v[2], v[3]), pack4<FMT>(v[4], v[5], v[6], v[7])};
    };
    auto in_steps = [&] {
        const Divisor d = divisor();
        return all([&](float f) { return d.quotient<POW2, F32>(f); });
    };
    if constexpr (POW2 || !F32) return in_steps();
    const float below = about * (1.0f - 0x1p-20f), above = about * (1.0f + 0x1p-20f);
    const u32x2_t w = all([&](float f) { return f * below; }), u = all([&](float f) { return f * above; });
    if ((w[0] ^ u[0]) | (w[1] ^ u[1])) return in_steps();
    return w;
}

// A workgroup takes 32 rows x KT blocks of 128, 16 lanes to a block: a wave's load covers four blocks' 256 (bf16) bytes, and all of a
// lane's 2 KT pieces are in flight before the first is used.  Scales of one block column and 32 rows leave together (128 bytes):
// written by each block's own lanes they are single values, a row stride apart.
template <class T, int FMT, bool POW2, int KT>
__global__ __launch_bounds__(kThreads) void quant_rows_kernel(QuantArgs a)
{
    __shared__ uint32_t scales[KT * 32];
    const int group = blockIdx.x % a.groups, row0 = a.first + (int)(blockIdx.x / a.groups) * 32;
    const int kb0 = group * KT, p = threadIdx.x & 15, g = threadIdx.x >> 4;
    Piece<T> in[2 * KT];
#pragma unroll
    for (int i = 0; i < 2 * KT; ++i) {
        const int item = i * 16 + g, row = row0 + item / KT, kb = kb0 + item % KT;
        const int col = kb * 128 + p * 8;
        in[i] = load8(static_cast<const T *>(a.X) + (int64_t)min(row, a.rows - 1) * a.ldx, col, a.c);
    }
#pragma unroll
    for (int i = 0; i < 2 * KT; ++i) {
        const int item = i * 16 + g, r = item / KT, kb = kb0 + item % KT;
        settle(in[i], row0 + r < a.rows ? a.c - kb * 128 - p * 8 : 0, a.c);
        float v[8];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) { v[j] = piece_get(in[i], j); top = umax(top, mag_bits(v[j])); }
        top = row16_umax(top);
        const BlockScale b = BlockScale::of<FMT, POW2>(top);
        const Divisor d = Divisor::of<FMT, POW2>(top, b);
        if (row0 + r < a.rows && kb < a.nkb) {
            const u32x2_t w = codes8<FMT, POW2, sizeof(T) == 4>(v, d.about(), [&] { return d; });
            *reinterpret_cast<u32x2_t *>(a.Q + (int64_t)(row0 + r) * a.ldq + kb * 128 + p * 8) = w;
        }
        if (p == 0) scales[(item % KT) * 32 + r] = POW2 ? b.code : __float_as_uint(b.s);
    }
    __syncthreads();
    if (threadIdx.x < KT * 32) {
        const int r = threadIdx.x & 31, kb = kb0 + (threadIdx.x >> 5);
        if (row0 + r < a.rows && kb < a.nkb) {
            const int64_t at = (int64_t)kb * a.lds + row0 + r;
            if constexpr (POW2) static_cast<uint8_t *>(a.S)[at] = (uint8_t)scales[threadIdx.x];
            else static_cast<float *>(a.S)[at] = __uint_as_float(scales[threadIdx.x]);
        }
    }
}

__device__ __forceinline__ uint32_t wave_umax(uint32_t x)
{
    x = row16_umax(x);
    const uint32_t a = umax(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16));
    return umax(a, umax(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}

// A workgroup takes a tile of 128 x 128 values, 8 pieces of 8 to a thread.
template <class T, int FMT, bool POW2>
__global__ __launch_bounds__(kThreads) void quant_tiles_kernel(QuantArgs a)
{
    __shared__ uint32_t tops[kThreads / 64];
    const int kb = blockIdx.x % a.nkb, rt = blockIdx.x / a.nkb;
    const int col = kb * 128 + (threadIdx.x & 15) * 8, r0 = rt * 128 + (threadIdx.x >> 4);
    Piece<T> in[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        in[i] = load8(static_cast<const T *>(a.X) + (int64_t)min(r0 + 16 * i, a.rows - 1) * a.ldx, col, a.c);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        settle(in[i], r0 + 16 * i < a.rows ? a.c - col : 0, a.c);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = umax(top, mag_bits(piece_get(in[i], j)));
    }
    top = wave_umax(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = umax(umax(tops[0], tops[1]), umax(tops[2], tops[3]));
    const BlockScale b = BlockScale::of<FMT, POW2>(top);
    const Divisor d = Divisor::of<FMT, POW2>(top, b);
    if (threadIdx.x == 0) store_scale<POW2>(a.S, (int64_t)kb * a.lds + rt, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + 16 * i >= a.rows) break;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = piece_get(in[i], j);
        const u32x2_t w = codes8<FMT, POW2, sizeof(T) == 4>(v, d.about(), [&] { return d; });
        *reinterpret_cast<u32x2_t *>(a.Q + (int64_t)(r0 + 16 * i) * a.ldq + col) = w;
    }
}

// Transposed codes: a workgroup takes 128 rows x 128 columns, a thread 8 rows x 8 columns, so that the 8 codes of a column that
// a thread holds are a piece of the code row as they are packed; the pieces pass through shared memory (rotated by the thread's
// column group: its 16 lanes of a store would otherwise meet in the same banks), and each code row leaves as 128 bytes.
template <class T, int FMT, bool POW2, bool TILE>
__global__ __launch_bounds__(kThreads) void quant_turned_kernel(QuantArgs a)
{
    __shared__ __align__(16) uint32_t maxima[TILE ? 4 : 16 * 128];
    // of the columns, float32 scales: for float32 values the factor about right and the maximum, else the divisor in two parts; e8m0: the
    // factor
    constexpr bool F32 = sizeof(T) == 4 && !POW2;
    __shared__ __align__(16) uint2 factors[TILE ? 1 : 128];
    __shared__ __align__(16) float pres[TILE || POW2 || F32 ? 1 : 128];
    __shared__ __align__(16) uint2 codes[128 * 16];
    const int ct = blockIdx.x % a.groups, kb = blockIdx.x / a.groups;
    const int cc = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int col = ct * 128 + cc * 8, r0 = kb * 128 + rg * 8;
    Piece<T> in[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        in[i] = load8(static_cast<const T *>(a.X) + (int64_t)min(r0 + i, a.rows - 1) * a.ldx, col, a.c);
#pragma unroll
    for (int i = 0; i < 8; ++i) settle(in[i], r0 + i < a.rows ? a.c - col : 0, a.c);
    Divisor one{};
    if constexpr (TILE) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = umax(top, mag_bits(piece_get(in[i], j)));
        top = wave_umax(top);
        if ((threadIdx.x & 63) == 0) maxima[threadIdx.x >> 6] = top;
        __syncthreads();
        top = umax(umax(maxima[0], maxima[1]), umax(maxima[2], maxima[3]));
        const BlockScale b = BlockScale::of<FMT, POW2>(top);
        one = Divisor::of<FMT, POW2>(top, b);
        if (threadIdx.x == 0) store_scale<POW2>(a.S, (int64_t)kb * a.lds + ct, b);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = umax(top, mag_bits(piece_get(in[i], j)));
            maxima[rg * 128 + cc * 8 + j] = top;
        }
        __syncthreads();
        if (threadIdx.x < 128) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = umax(top, maxima[i * 128 + threadIdx.x]);
            const BlockScale b = BlockScale::of<FMT, POW2>(top);
            const Divisor d = Divisor::of<FMT, POW2>(top, b);
            factors[threadIdx.x] = F32 ? make_uint2(__float_as_uint(d.about()), top) : make_uint2(__float_as_uint(d.rc), __float_as_uint(d.top2));
            if constexpr (!POW2 && !F32) pres[threadIdx.x] = d.pre;
            const int n = ct * 128 + (int)threadIdx.x;
            if (n < a.c) store_scale<POW2>(a.S, (int64_t)kb * a.lds + n, b);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = piece_get(in[i], j);
        u32x2_t w;
        if constexpr (TILE) {
            w = codes8<FMT, POW2, F32>(v, one.about(), [&] { return one; });
        } else {
            const uint2 f = factors[cc * 8 + j];
            w = codes8<FMT, POW2, F32>(v, __uint_as_float(f.x), [&] {
                if constexpr (F32) return Divisor::of<FMT, false>(f.y, BlockScale{});
                return Divisor{__uint_as_float(f.x), __uint_as_float(f.y), POW2 ? 0.0f : pres[cc * 8 + j]};
            });
        }
        codes[(cc * 8 + j) * 16 + (rg ^ cc)] = make_uint2(w[0], w[1]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = i * 32 + (threadIdx.x >> 3), q = threadIdx.x & 7, f = n >> 3;
        if (ct * 128 + n >= a.c) continue;
        const uint2 lo = codes[n * 16 + ((2 * q) ^ f)], hi = codes[n * 16 + ((2 * q + 1) ^ f)];
        *reinterpret_cast<uint4 *>(a.Q + (int64_t)(ct * 128 + n) * a.ldq + kb * 128 + q * 16) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
}

template <class T, int FMT, bool POW2>
hipError_t launch(QuantArgs a, int blocks, hipStream_t st)
{
    const int row_tiles = (a.rows + 127) / 128, col_tiles = (a.c + 127) / 128;
    switch (blocks) {
        case TRDQ_BLOCKS_ROWS: {
            // the blocks of a row in groups of up to four, of equal size (9 = 3 x 3: a group of one would leave lanes idle)
            a.groups = (a.nkb + 3) / 4;
            const int kt = (a.nkb + a.groups - 1) / a.groups;
            const int64_t at_once = kMostThreads / kThreads / a.groups * 32;
            for (int64_t first = 0; first < a.rows; first += at_once) {
                a.first = (int)first;
                const int64_t n = std::min(a.rows - first, at_once);
                const dim3 g((unsigned)(a.groups * ((n + 31) / 32))), t(kThreads);
                if (kt == 1) quant_rows_kernel<T, FMT, POW2, 1><<<g, t, 0, st>>>(a);
                else if (kt == 2) quant_rows_kernel<T, FMT, POW2, 2><<<g, t, 0, st>>>(a);
                else if (kt == 3) quant_rows_kernel<T, FMT, POW2, 3><<<g, t, 0, st>>>(a);
                else quant_rows_kernel<T, FMT, POW2, 4><<<g, t, 0, st>>>(a);
                if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            }
            return hipSuccess;
        }
        case TRDQ_BLOCKS_TILES:
            quant_tiles_kernel<T, FMT, POW2><<<dim3((unsigned)((int64_t)row_tiles * col_tiles)), dim3(kThreads), 0, st>>>(a);
            break;
        case TRDQ_BLOCKS_COLS:
            a.groups = col_tiles;
            quant_turned_kernel<T, FMT, POW2, false><<<dim3((unsigned)((int64_t)row_tiles * col_tiles)), dim3(kThreads), 0, st>>>(a);
            break;
        default:
            a.groups = col_tiles;
            quant_turned_kernel<T, FMT, POW2, true><<<dim3((unsigned)((int64_t)row_tiles * col_tiles)), dim3(kThreads), 0, st>>>(a);
    }
    return hipGetLastError();
}

template <class T>
hipError_t launch_from(const QuantArgs &a, int blocks, bool e5m2, bool pow2, hipStream_t st)
{
    if (e5m2) return pow2 ? launch<T, kE5M2, true>(a, blocks, st) : launch<T, kE5M2, false>(a, blocks, st);
    return pow2 ? launch<T, kE4M3, true>(a, blocks, st) : launch<T, kE4M3, false>(a, blocks, st);
}

}  // namespace

hipError_t launch_fp8_quant(const void *X, bool f32, int rows, int c, int64_t ldx, int blocks, bool e5m2, uint8_t *Q, int64_t ldq,
                            void *S, int64_t lds, bool pow2, hipStream_t st)
{
    const bool turned = blocks == TRDQ_BLOCKS_COLS || blocks == TRDQ_BLOCKS_TILES_T;
    QuantArgs a{X, Q, S, ldx, ldq, lds, rows, c, ((turned ? rows : c) + 127) / 128, 0, 0};
    return f32 ? launch_from<float>(a, blocks, e5m2, pow2, st) : launch_from<Bf16>(a, blocks, e5m2, pow2, st);
}

}  // namespace trdq
