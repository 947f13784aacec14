// Device pieces shared by the 8-bit floating-point quantiser, the product of such codes and the norms that write them:
// 8-element pieces of rows at any alignment, scales of 128-value blocks, rounding to the OCP formats e4m3 and e5m2.
#pragma once

#include "device_utils.h"
#include "trdq_internal.h"

namespace trdq {
namespace fp8 {

// ---- pieces of a row ------------------------------------------------------------------------------
// Rows begin anywhere a value may lie (a row stride that is no multiple of 8 values): 16-byte loads and stores need the
// alignment of their type only here, the memory pipe splits what crosses a line.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

struct Bf16 { uint16_t bits; };

// 8 values as loaded: a row piece that waits for its use takes 4 (bf16) or 8 (float) registers
template <class T> struct Piece;
template <> struct Piece<Bf16> { uint32_t w[4]; };
template <> struct Piece<float> { float f[8]; };

__device__ __forceinline__ float piece_get(const Piece<Bf16> &p, int j) { return j & 1 ? bf16_hi(p.w[j >> 1]) : bf16_lo(p.w[j >> 1]); }
__device__ __forceinline__ float piece_get(const Piece<float> &p, int j) { return p.f[j]; }

// Values at .. at + 7 of a row of c values (any at), in two steps, so that many loads can be in flight: load8, one load in every
// lane (a piece that ends early reads the row's last eight values, one behind the end reads them for nothing), and settle, which
// moves what was read into place; n: how many of the piece's values exist (c - at; at most 0: none), the others become zeros.
// Loads under conditions, one a value, each wait for the one before (1003 rows of 771 values with nine vectors 8.2 / 7.3 us, gradients
// of 1721 x 4672 99 / 55).
__device__ __forceinline__ Piece<Bf16> load8(const Bf16 *row, int at, int c)
{
    Piece<Bf16> r;
    if (c < 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[j] = 0;
#pragma unroll 1
        for (int k = 0; k < c - at; ++k) {
            const uint32_t v = row[at + k].bits;
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[j] |= j == k >> 1 ? v << (16 * (k & 1)) : 0u;
        }
        return r;
    }
    const u32x4_a2 v = *reinterpret_cast<const u32x4_a2 *>(reinterpret_cast<const char *>(row) + (uint32_t)(min(at, c - 8) * 2));
#pragma unroll
    for (int j = 0; j < 4; ++j) r.w[j] = v[j];
    return r;
}

__device__ __forceinline__ void settle(Piece<Bf16> &r, int n, int c)
{
    if (n < 8) {
        const uint32_t v[4] = {r.w[0], r.w[1], r.w[2], r.w[3]};
        const int by = c < 8 ? 0 : 8 - n;                    // (rows of fewer than eight values are read in place)
        const bool one = by & 1, two = by & 2, four = by & 4, all = n <= 0;
        // (named values: an array here ends in scratch memory)
        const uint32_t a0 = four ? v[2] : v[0], a1 = four ? v[3] : v[1], a2 = four ? 0u : v[2], a3 = four ? 0u : v[3];
        const uint32_t b0 = two ? a1 : a0, b1 = two ? a2 : a1, b2 = two ? a3 : a2, b3 = two ? 0u : a3;
        r.w[0] = all ? 0u : one ? (b0 >> 16 | b1 << 16) : b0;
        r.w[1] = all ? 0u : one ? (b1 >> 16 | b2 << 16) : b1;
        r.w[2] = all ? 0u : one ? (b2 >> 16 | b3 << 16) : b2;
        r.w[3] = all ? 0u : one ? b3 >> 16 : b3;
    }
}

__device__ __forceinline__ Piece<float> load8(const float *row, int at, int c)
{
    Piece<float> r;
    if (c < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.f[j] = 0.0f;
#pragma unroll 1
        for (int k = 0; k < c - at; ++k) {
            const float v = row[at + k];
#pragma unroll
            for (int j = 0; j < 8; ++j) r.f[j] = j == k ? v : r.f[j];
        }
        return r;
    }
    const u32x4_a4 *const p = reinterpret_cast<const u32x4_a4 *>(reinterpret_cast<const char *>(row) + (uint32_t)(min(at, c - 8) * 4));
    const u32x4_a4 a = p[0], b = p[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) { r.f[j] = __uint_as_float(a[j]); r.f[4 + j] = __uint_as_float(b[j]); }
    return r;
}

__device__ __forceinline__ void settle(Piece<float> &r, int n, int c)
{
    if (n < 8) {
        const uint32_t a[4] = {__float_as_uint(r.f[0]), __float_as_uint(r.f[1]), __float_as_uint(r.f[2]), __float_as_uint(r.f[3])};
        const uint32_t b[4] = {__float_as_uint(r.f[4]), __float_as_uint(r.f[5]), __float_as_uint(r.f[6]), __float_as_uint(r.f[7])};
        const int by = c < 8 ? 0 : 8 - n;                    // (rows of fewer than eight values are read in place)
        const bool one = by & 1, two = by & 2, four = by & 4, all = n <= 0;
        const uint32_t c0 = four ? b[0] : a[0], c1 = four ? b[1] : a[1], c2 = four ? b[2] : a[2], c3 = four ? b[3] : a[3];
        const uint32_t c4 = four ? 0u : b[0], c5 = four ? 0u : b[1], c6 = four ? 0u : b[2], c7 = four ? 0u : b[3];
        const uint32_t d0 = two ? c2 : c0, d1 = two ? c3 : c1, d2 = two ? c4 : c2, d3 = two ? c5 : c3, d4 = two ? c6 : c4, d5 = two ? c7 : c5;
        const uint32_t d6 = two ? 0u : c6, d7 = two ? 0u : c7;
        r.f[0] = __uint_as_float(all ? 0u : one ? d1 : d0);
        r.f[1] = __uint_as_float(all ? 0u : one ? d2 : d1);
        r.f[2] = __uint_as_float(all ? 0u : one ? d3 : d2);
        r.f[3] = __uint_as_float(all ? 0u : one ? d4 : d3);
        r.f[4] = __uint_as_float(all ? 0u : one ? d5 : d4);
        r.f[5] = __uint_as_float(all ? 0u : one ? d6 : d5);
        r.f[6] = __uint_as_float(all ? 0u : one ? d7 : d6);
        r.f[7] = __uint_as_float(all || one ? 0u : d7);
    }
}

__device__ __forceinline__ void store8(Bf16 *p, int n, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
    if (n >= 8) {
        *reinterpret_cast<u32x4_a2 *>(p) = u32x4_a2{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j].bits = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}

__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        u32x4_a4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) { a[j] = __float_as_uint(v[j]); b[j] = __float_as_uint(v[4 + j]); }
        *reinterpret_cast<u32x4_a4 *>(p) = a;
        *reinterpret_cast<u32x4_a4 *>(p + 4) = b;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = v[j];
    }
}

// the value as the row will hold it
__device__ __forceinline__ float as_stored(const Bf16 *, float v) { return bf16_lo(pack_bf16x2(v, 0.0f)); }
__device__ __forceinline__ float as_stored(const float *, float v) { return v; }

// ---- scales of a block -----------------------------------------------------------------------------
enum { kE4M3 = 0, kE5M2 = 1 };
// largest magnitude = 0.875 * 2^kTopExp (448, 57344)
template <int FMT> struct TopExp { static constexpr int value = FMT == kE4M3 ? 9 : 16; };

// Magnitudes are compared by their bits, so that a NaN is the largest of all and reaches the scale.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// largest over the 16 lanes of a row, in all of them
__device__ __forceinline__ uint32_t row16_umax(uint32_t x)
{
    x = umax(x, dpp_u<kDppXor1>(x));
    x = umax(x, dpp_u<kDppXor2>(x));
    x = umax(x, dpp_u<kDppHalfMirror>(x));          // every four lanes agree by now: the mirrors reach the other four, the other eight
    x = umax(x, dpp_u<0x140>(x));
    return x;
}

// What a block's largest magnitude makes of it.  Scales in float32: s = top / max; a value is divided by it as x max / top: with t =
// 0.875 x (no overflow) and top2 = top / 2^TopExp, q0 = t rc is within two steps of t / top2, and one step of the residual,
// fma(t - q0 top2, rc, q0), leaves a float32 rounding or two (2^-22) of the quotient.  That is for values that carry such roundings
// themselves, as a norm's; the quantiser has to give the nearest code (fp8_quant.hip).  Scales as powers of two (e8m0): the smallest
// that is at least top / max, undone exactly.  A block whose largest magnitude is Inf or NaN gets a NaN as its scale and as its codes;
// one of zeros (or of values below 2^-100) the scale of 2^-100.
struct BlockScale {
    float rc, top2;            // float32 scales: 1 / top2 and top2; e8m0: the factor 2^-e, and 0
    float s;                   // float32 scale
    uint32_t code;             // e8m0 scale

    template <int FMT, bool POW2>
    __device__ __forceinline__ static BlockScale of(uint32_t top_bits)
    {
        constexpr int E = TopExp<FMT>::value;
        BlockScale b;
        const bool bad = top_bits >= 0x7F800000u;
        top_bits = umax(top_bits, (uint32_t)(127 - 100) << 23);
        const float nan = __uint_as_float(0x7FC00000u);
        if constexpr (POW2) {
            const uint32_t code = (top_bits >> 23) + 1 - E + ((top_bits & 0x7FFFFFu) > 0x600000u ? 1u : 0u);
            b.code = bad ? 255u : code;
            b.rc = bad ? nan : __uint_as_float((254u - code) << 23);
            b.top2 = 0.0f;
            b.s = 0.0f;
        } else {
            constexpr float kMax = E == 9 ? 448.0f : 57344.0f;
            const float top = __uint_as_float(top_bits);
            const float q = top * (1.0f / kMax);
            b.s = bad ? nan : __builtin_fmaf(__builtin_fmaf(-kMax, q, top), 1.0f / kMax, q);      // the nearest float to top / max
            b.top2 = top * (E == 9 ? 0x1p-9f : 0x1p-16f);
            const float r = __builtin_amdgcn_rcpf(b.top2);
            b.rc = bad ? nan : __builtin_fmaf(__builtin_fmaf(-b.top2, r, 1.0f), r, r);
            b.code = 0;
        }
        return b;
    }

    template <bool POW2>
    __device__ __forceinline__ float scaled(float x) const
    {
        if constexpr (POW2) return x * rc;
        const float t = 0.875f * x, q0 = t * rc;
        return __builtin_fmaf(__builtin_fmaf(-q0, top2, t), rc, q0);
    }
};

// four values in the format's range -> four codes, nearest, ties to even (the conversion instructions take bf8 = e5m2)
template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d)
{
    int w = 0;
    if constexpr (FMT == kE4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}

template <bool POW2>
__device__ __forceinline__ void store_scale(void *S, int64_t i, const BlockScale &b)
{
    if constexpr (POW2) static_cast<uint8_t *>(S)[i] = (uint8_t)b.code;
    else static_cast<float *>(S)[i] = b.s;
}

}  // namespace fp8
}  // namespace trdq
