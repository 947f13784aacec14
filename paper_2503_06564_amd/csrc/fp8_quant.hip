// Codes in 8-bit floating point with a scale per block of 128 values:
//   top = max |x| of the block (at least 2^-100),  s = top / max,  code = nearest value of the format to x / s
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
        const BlockScale b = BlockScale::of<FMT, POW2>(row16_umax(top));
        if (row0 + r < a.rows && kb < a.nkb) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = b.scaled<POW2>(v[j]);
            const u32x2_t w = {pack4<FMT>(v[0], v[1], v[2], v[3]), pack4<FMT>(v[4], v[5], v[6], v[7])};
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
    const BlockScale b = BlockScale::of<FMT, POW2>(umax(umax(tops[0], tops[1]), umax(tops[2], tops[3])));
    if (threadIdx.x == 0) store_scale<POW2>(a.S, (int64_t)kb * a.lds + rt, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + 16 * i >= a.rows) break;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = b.scaled<POW2>(piece_get(in[i], j));
        const u32x2_t w = {pack4<FMT>(v[0], v[1], v[2], v[3]), pack4<FMT>(v[4], v[5], v[6], v[7])};
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
    __shared__ __align__(16) uint2 factors[TILE ? 1 : 128];
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
    BlockScale one{};
    if constexpr (TILE) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = umax(top, mag_bits(piece_get(in[i], j)));
        top = wave_umax(top);
        if ((threadIdx.x & 63) == 0) maxima[threadIdx.x >> 6] = top;
        __syncthreads();
        one = BlockScale::of<FMT, POW2>(umax(umax(maxima[0], maxima[1]), umax(maxima[2], maxima[3])));
        if (threadIdx.x == 0) store_scale<POW2>(a.S, (int64_t)kb * a.lds + ct, one);
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
            factors[threadIdx.x] = make_uint2(__float_as_uint(b.rc), __float_as_uint(b.top2));
            const int n = ct * 128 + (int)threadIdx.x;
            if (n < a.c) store_scale<POW2>(a.S, (int64_t)kb * a.lds + n, b);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        BlockScale b = one;
        if constexpr (!TILE) {
            const uint2 f = factors[cc * 8 + j];
            b.rc = __uint_as_float(f.x);
            b.top2 = __uint_as_float(f.y);
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = b.scaled<POW2>(piece_get(in[i], j));
        codes[(cc * 8 + j) * 16 + (rg ^ cc)] = make_uint2(pack4<FMT>(v[0], v[1], v[2], v[3]), pack4<FMT>(v[4], v[5], v[6], v[7]));
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
