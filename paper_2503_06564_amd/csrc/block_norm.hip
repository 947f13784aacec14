// The operator between two branches of a transformer block, and its gradient:
//   p  = y, or norm(y) w2 + b2           (a norm behind the branch)
//   x' = x + gate p                      (rounded to the stream's type and stored)
//   h  = (norm(x') w + b)(1 + scale) + shift
// norm(v) = (v - mean v) / sqrt(mean (v - mean v)^2 + eps) (layer) or v / sqrt(mean v^2 + eps) (rms); gate, scale and shift belong to the
// row's segment (the gate may be one vector for all).  A row stays in registers from its one read to its one write, sums are
// float32, a mean is taken off before squares are summed (a stream with a large mean or massive channels loses its variance in
// mean v^2 - (mean v)^2).  Memory bounds both directions from a few thousand rows on, the chain of a row's reductions below that.
#include <algorithm>
#include <type_traits>

#include "fp8_common.h"

namespace trdq {
namespace {

using namespace fp8;

// ---- what both directions need of a row ------------------------------------------------------------------
// A row of c values is shared by W waves, 8 values to a lane at a time, NCH pieces a lane: piece i of the row is at 8 i.
template <int W, int NCH>
struct Row {
    static constexpr int kLanes = 64 * W;
    int lane;                  // in the row
    int c;
    __device__ __forceinline__ int at(int n) const { return 8 * (lane + kLanes * n); }
    __device__ __forceinline__ int left(int n) const { return c - at(n); }       // values of piece n that exist: <= 0 none, >= 8 all
};

__device__ __forceinline__ float wave_sum(float x)
{
    x += row_xor<1>(x);
    x += row_xor<2>(x);
    x += dpp_f<kDppHalfMirror>(x);
    x += dpp_f<0x140>(x);
    const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 0)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 16));
    const float b = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 32)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 48));
    return a + b;
}

// Sums over a row's W waves; two areas of shared memory in turn, so that one barrier a sum is enough.
template <int W>
struct RowSums {
    float (*area)[2 * W];      // [2][2 W]
    int turn = 0;
    __device__ __forceinline__ void two(float &a, float &b)
    {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (W > 1) {
            float *const s = area[turn & 1];
            ++turn;
            const int w = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) { s[w] = a; s[W + w] = b; }
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) { a += s[i]; b += s[W + i]; }
        }
    }
    __device__ __forceinline__ float one(float a)
    {
        float b = 0.0f;
        if constexpr (W > 1) two(a, b);
        else a = wave_sum(a);
        return a;
    }
};

// mean (0 for rms) and 1 / root of the mean square of v - mean; get(n, j): value j of the lane's piece n, zero behind the row's end
template <int W, int NCH, class Get>
__device__ __forceinline__ void stats(const Row<W, NCH> &row, Get &&get, bool layer, float inv_c, float eps, RowSums<W> &sums, float &mean, float &r)
{
    mean = 0.0f;
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int n = 0; n < NCH; ++n) s += ((get(n, 0) + get(n, 1)) + (get(n, 2) + get(n, 3))) + ((get(n, 4) + get(n, 5)) + (get(n, 6) + get(n, 7)));
        mean = sums.one(s) * inv_c;
    }
    float s = 0.0f;
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        const int left = row.left(n);
        if (left >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float d = get(n, j) - mean; s = __builtin_fmaf(d, d, s); }
        } else if (left > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float d = j < left ? get(n, j) - mean : 0.0f; s = __builtin_fmaf(d, d, s); }
        }
    }
    r = __builtin_amdgcn_rsqf(__builtin_fmaf(sums.one(s), inv_c, eps));
}

// Segment of a row: seg_len rows each, or by borders, off[0] .. off[n_seg]: the borders behind the first that are not above the row.
__device__ __forceinline__ int segment_of(const NormArgs &a, int row)
{
    if (!a.seg_off) return min((int)((uint32_t)row / (uint32_t)a.seg_len), a.n_seg - 1);
    int seg = 0;
    for (int i = 0; i < a.n_seg; i += 64) {
        const int k = i + (int)(threadIdx.x & 63);
        const uint64_t below = __ballot(k + 1 < a.n_seg && a.seg_off[k + 1 < a.n_seg ? k + 1 : 0] <= row);
        seg += __popcll(below);
        if (below != ~0ull) break;
    }
    return __builtin_amdgcn_readfirstlane(seg);
}

// Piece of a matrix' row: the row's address is the same in all lanes (scalar registers), a lane adds 32 bits.
template <class T>
__device__ __forceinline__ T *piece_of(void *base, int64_t row_at, int at)
{
    return reinterpret_cast<T *>(reinterpret_cast<char *>(static_cast<T *>(base) + row_at) + (uint32_t)(at * (int)sizeof(T)));
}
template <class P>
__device__ __forceinline__ Piece<P> param(const void *base, int64_t row_at, int at, int c)
{
    return load8(static_cast<const P *>(base) + row_at, at, c);
}
template <class P>
__device__ __forceinline__ Piece<P> param_now(const void *base, int64_t row_at, int at, int c)
{
    Piece<P> v = load8(static_cast<const P *>(base) + row_at, at, c);
    settle(v, c - at, c);
    return v;
}

// ---- forward --------------------------------------------------------------------------------------------------
// Rows and threads of a workgroup; workgroups along x (more rows go on along y: an argument for the first row of several launches, which
// moves the others or stands behind them, cost 4096 x 1152 11.0 / 11.3 us).
template <int W>
struct Forward {
    static constexpr uint32_t kRows = W == 1 ? 4 : 1, kThreads = W == 1 ? 256 : 64 * W, kAcross = kMostThreads / kThreads;
};

template <class T, class P, int W, int NCH>
__global__ __launch_bounds__(Forward<W>::kThreads) void block_norm_kernel(NormArgs a)
{
    using F = Forward<W>;
    __shared__ float area[2][2 * W];
    const int r_in = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const uint32_t row_u = (blockIdx.y * F::kAcross + blockIdx.x) * F::kRows + r_in;
    if (row_u >= (uint32_t)a.rows) return;
    const int row_i = (int)row_u;
    const Row<W, NCH> row{(int)threadIdx.x - 64 * r_in, a.c};
    RowSums<W> sums{area};

    Piece<T> px[NCH];
    Piece<Bf16> py[NCH];
#pragma unroll
    for (int n = 0; n < NCH; ++n) px[n] = load8(static_cast<const T *>(a.X) + (int64_t)row_i * a.ldx, row.at(n), a.c);
    if (a.Y)
#pragma unroll
        for (int n = 0; n < NCH; ++n) py[n] = load8(static_cast<const Bf16 *>(a.Y) + (int64_t)row_i * a.ldy, row.at(n), a.c);
    const int seg = a.by_segment ? segment_of(a, row_i) : 0;

    // Parameters are loaded ahead of the reduction before their use: one after the other, each at its use, they cost a row six trips to
    // the L2 (1003 x 771 with all of them 9.5 / 8.2 us; all of them at the start instead cost occupancy, 4096 x 1152 10.9 / 12.1).
    Piece<P> gate[NCH], post_w[NCH], post_b[NCH], pre_w[NCH], pre_b[NCH], scale[NCH], shift[NCH];
    auto fetch = [&](const void *p, int64_t at, Piece<P> (&v)[NCH]) {
        if (p)
#pragma unroll
            for (int n = 0; n < NCH; ++n) v[n] = param<P>(p, at, row.at(n), a.c);
    };
    auto times = [&](const void *p, Piece<P> (&v)[NCH], float (&x)[NCH][8]) {
        if (p)
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                settle(v[n], row.left(n), a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] *= piece_get(v[n], j);
            }
    };
    auto plus = [&](const void *p, Piece<P> (&v)[NCH], float (&x)[NCH][8]) {
        if (p)
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                settle(v[n], row.left(n), a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] += piece_get(v[n], j);
            }
    };
    if (a.Y) {
        fetch(a.post_w, 0, post_w);
        fetch(a.post_b, 0, post_b);
        fetch(a.gate, (int64_t)seg * a.ld_gate, gate);
    }
    float x[NCH][8];
    float mean, r;
    if (a.Y) {
        float y[NCH][8];
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            settle(py[n], row.left(n), a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[n][j] = piece_get(py[n], j);
        }
        if (a.post) {
            stats(row, [&](int n, int j) { return y[n][j]; }, a.post == TRDQ_NORM_LAYER, a.inv_c, a.eps, sums, mean, r);
#pragma unroll
            for (int n = 0; n < NCH; ++n)
#pragma unroll
                for (int j = 0; j < 8; ++j) y[n][j] = (y[n][j] - mean) * r;
            times(a.post_w, post_w, y);
            plus(a.post_b, post_b, y);
        }
        times(a.gate, gate, y);
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            const int left = row.left(n);
            T *const to = piece_of<T>(a.Xout, (int64_t)row_i * a.ldxo, row.at(n));
            settle(px[n], left, a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[n][j] = piece_get(px[n], j) + y[n][j];
            store8(to, left, x[n]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[n][j] = as_stored(to, j < left ? x[n][j] : 0.0f);
        }
    } else {
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            settle(px[n], row.left(n), a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[n][j] = piece_get(px[n], j);
        }
    }
    fetch(a.pre_w, 0, pre_w);
    fetch(a.pre_b, 0, pre_b);
    fetch(a.scale, (int64_t)seg * a.ld_scale, scale);
    fetch(a.shift, (int64_t)seg * a.ld_shift, shift);
    stats(row, [&](int n, int j) { return x[n][j]; }, a.pre == TRDQ_NORM_LAYER, a.inv_c, a.eps, sums, mean, r);
#pragma unroll
    for (int n = 0; n < NCH; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[n][j] = (x[n][j] - mean) * r;
    times(a.pre_w, pre_w, x);
    plus(a.pre_b, pre_b, x);
    if (a.scale)
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            settle(scale[n], row.left(n), a.c);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[n][j] = __builtin_fmaf(x[n][j], piece_get(scale[n], j), x[n][j]);
        }
    plus(a.shift, shift, x);
#pragma unroll
    for (int n = 0; n < NCH; ++n) {
        const int left = row.left(n), at = row.at(n);
        if (a.out == TRDQ_E4M3) {
            // a block of 128 lies in 16 lanes; values behind the row's end are zeros to it, codes there are written as zeros
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= left) x[n][j] = 0.0f;
                top = umax(top, mag_bits(x[n][j]));
            }
            top = row16_umax(top);
            const int kb = at >> 7;
            if (kb >= a.nkb) continue;
            u32x2_t w;
            if (a.pow2) {
                const BlockScale b = BlockScale::of<kE4M3, true>(top);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] = b.scaled<true>(x[n][j]);
                if ((threadIdx.x & 15) == 0) store_scale<true>(a.S, (int64_t)kb * a.lds + row_i, b);
            } else {
                const BlockScale b = BlockScale::of<kE4M3, false>(top);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] = b.scaled<false>(x[n][j]);
                if ((threadIdx.x & 15) == 0) store_scale<false>(a.S, (int64_t)kb * a.lds + row_i, b);
            }
            w[0] = pack4<kE4M3>(x[n][0], x[n][1], x[n][2], x[n][3]);
            w[1] = pack4<kE4M3>(x[n][4], x[n][5], x[n][6], x[n][7]);
            *reinterpret_cast<u32x2_t *>(a.Q + (int64_t)row_i * a.ldq + at) = w;
        } else if (a.out == TRDQ_BF16) {
            store8(piece_of<Bf16>(a.H, (int64_t)row_i * a.ldh, at), left, x[n]);
        } else {
            store8(piece_of<float>(a.H, (int64_t)row_i * a.ldh, at), left, x[n]);
        }
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------
// With n = norm(x'), u = dh (1 + scale) w and t = d loss / d x' (all that reaches the stream):
//   t  = dx' + r (u - n mean(u n) - [layer] mean u)                       -> dx
//   dp = gate t,  u2 = dp w2,  dy = r2 (u2 - n2 mean(u2 n2) - [layer] mean u2)   (dy = dp without the norm)
// Every parameter's gradient is made of four sums over a segment's rows, S1 = sum dh n, S0 = sum dh, T1 = sum t n2, T0 = sum t
// (n2 = y without the norm):
//   dscale = w S1 + b S0, dshift = S0, dw = sum over segments (1 + scale) S1, db the same of S0,
//   dgate = w2 T1 + b2 T0, dw2 = sum over segments gate T1, db2 the same of T0.
// First kernel: a workgroup walks a run of rows, keeps the sums in registers and writes them out whenever a segment ends; the
// second adds what belongs to a segment.  No atomics: the same inputs give the same bits.
// Slot of workgroup g's sums of segment s: g + s.  Neither ever decreases along the rows, so no two pairs meet, and a segment's
// slots lie together.
// All of a row's loads go out before its first reduction.  The factors (1 + scale) w and gate w2 are formed once a segment and wait in
// shared memory: in registers, beside the sums and a row, they spill.  What spills still: at three pieces a lane (1025 to 1536 values)
// up to 46 registers with all four sums, up to 10 with three; at 16 waves (above 8192 values, 128 registers a lane) 35 to 178, in every
// form: 4096 rows of 8192 bf16 values take 104 us, of 8704 567, of 16384 635.
constexpr int kBwdWaves = 8;                          // of a workgroup whose waves have a row each
template <int W, int NCH>
constexpr size_t bwd_factor_bytes() { return 2 * (size_t)(64 * W) * NCH * 8 * sizeof(float); }
template <class T, class P, int W, int NCH, int SUMS>
__global__ __launch_bounds__(W == 1 ? 64 * kBwdWaves : 64 * W) void block_norm_bwd_kernel(NormArgs a)
{
    constexpr int kRows = W == 1 ? kBwdWaves : 1;
    constexpr bool kS0 = SUMS & 1, kT1 = SUMS & 2, kT0 = SUMS & 4;
    __shared__ float area[2][2 * W];
    __shared__ float joined[W == 1 ? kBwdWaves / 2 * 512 * NCH : 1];
    extern __shared__ __align__(16) v4f factors[];           // [pre, post][NCH][two halves][lanes of a row]
    const int r_in = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const Row<W, NCH> row{(int)threadIdx.x - 64 * r_in, a.c};
    RowSums<W> sums{area};
    const int begin = (int)blockIdx.x * a.rows_per_group, end = begin + min(a.rows - begin, a.rows_per_group);
    const bool pre_layer = a.pre == TRDQ_NORM_LAYER, post_layer = a.post == TRDQ_NORM_LAYER;

    int seg = a.by_segment ? segment_of(a, begin) : 0;
    for (int first = begin; first < end; ++seg) {
        int last = end;
        if (a.by_segment && seg + 1 < a.n_seg) {
            const int64_t border = a.seg_off ? (int64_t)a.seg_off[seg + 1] : (int64_t)(seg + 1) * a.seg_len;
            last = border < end ? max((int)border, first) : end;
        }
        const bool is_last = !a.by_segment || seg + 1 >= a.n_seg;
        if (last <= first) {
            if (is_last) break;
            continue;
        }
        float s1[NCH][8] = {}, s0[NCH][8] = {}, t1[NCH][8] = {}, t0[NCH][8] = {};
        if (W == 1) __syncthreads();                         // nobody reads the segment before any more
#pragma unroll
        for (int n = 0; n < NCH; ++n) {
            const int left = row.left(n), at = row.at(n);
            if (W > 1 || r_in == n) {
                float f[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
                if (a.scale) {
                    const Piece<P> v = param_now<P>(a.scale, (int64_t)seg * a.ld_scale, at, a.c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] += piece_get(v, j);
                }
                if (a.pre_w) {
                    const Piece<P> v = param_now<P>(a.pre_w, 0, at, a.c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] *= piece_get(v, j);
                }
                factors[(2 * n) * 64 * W + row.lane] = v4f{f[0], f[1], f[2], f[3]};
                factors[(2 * n + 1) * 64 * W + row.lane] = v4f{f[4], f[5], f[6], f[7]};
            }
            if (kT1 && (W > 1 || r_in == kBwdWaves / 2 + n)) {
                float f[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
                if (a.gate) {
                    const Piece<P> v = param_now<P>(a.gate, (int64_t)seg * a.ld_gate, at, a.c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = piece_get(v, j);
                }
                if (a.post_w) {
                    const Piece<P> v = param_now<P>(a.post_w, 0, at, a.c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] *= piece_get(v, j);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = j < left ? f[j] : 0.0f;
                factors[(2 * (NCH + n)) * 64 * W + row.lane] = v4f{f[0], f[1], f[2], f[3]};
                factors[(2 * (NCH + n) + 1) * 64 * W + row.lane] = v4f{f[4], f[5], f[6], f[7]};
            }
        }
        if (W == 1) __syncthreads();
        auto factor = [&](int which, int n, float (&f)[8]) {
            const v4f lo = factors[(2 * (which * NCH + n)) * 64 * W + row.lane], hi = factors[(2 * (which * NCH + n) + 1) * 64 * W + row.lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[j] = lo[j]; f[4 + j] = hi[j]; }
        };
        for (int row_i = first + r_in; row_i < last; row_i += kRows) {
            Piece<T> px[NCH], pt[NCH];
            Piece<Bf16> pd[NCH], py[NCH];
#pragma unroll
            for (int n = 0; n < NCH; ++n) px[n] = load8(static_cast<const T *>(a.X) + (int64_t)row_i * a.ldx, row.at(n), a.c);
#pragma unroll
            for (int n = 0; n < NCH; ++n) pd[n] = load8(static_cast<const Bf16 *>(a.dH) + (int64_t)row_i * a.lddh, row.at(n), a.c);
#pragma unroll
            for (int n = 0; n < NCH; ++n) pt[n] = load8(static_cast<const T *>(a.dXout ? a.dXout : a.X) + (int64_t)row_i * (a.dXout ? a.lddxo : a.ldx), row.at(n), a.c);
            if constexpr (kT1)
#pragma unroll
                for (int n = 0; n < NCH; ++n) py[n] = load8(static_cast<const Bf16 *>(a.Y) + (int64_t)row_i * a.ldy, row.at(n), a.c);
            float x[NCH][8], t[NCH][8];
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                settle(px[n], row.left(n), a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[n][j] = piece_get(px[n], j);
            }
            float mean, r;
            stats(row, [&](int n, int j) { return x[n][j]; }, pre_layer, a.inv_c, a.eps, sums, mean, r);
            __builtin_amdgcn_sched_barrier(0);               // (one phase after the other: mixed, the schedule takes a third more registers)
            float un = 0.0f, us = 0.0f;
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                float f[8];
                factor(0, n, f);
                settle(pd[n], row.left(n), a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) {                // dh is zero behind the row's end
                    const float d = piece_get(pd[n], j), u = d * f[j];
                    x[n][j] = (x[n][j] - mean) * r;
                    s1[n][j] = __builtin_fmaf(d, x[n][j], s1[n][j]);
                    if constexpr (kS0) s0[n][j] += d;
                    un = __builtin_fmaf(u, x[n][j], un);
                    us += u;
                }
            }
            sums.two(un, us);
            un *= a.inv_c;
            us = pre_layer ? us * a.inv_c : 0.0f;
#pragma unroll
            for (int n = 0; n < NCH; ++n) {
                float f[8];
                factor(0, n, f);
                settle(pt[n], row.left(n), a.c);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    t[n][j] = __builtin_fmaf(r, __builtin_fmaf(-un, x[n][j], __builtin_fmaf(piece_get(pd[n], j), f[j], -us)),
                                             a.dXout ? piece_get(pt[n], j) : 0.0f);
                store8(piece_of<T>(a.dX, (int64_t)row_i * a.lddx, row.at(n)), row.left(n), t[n]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kT1) {
                float y[NCH][8];
#pragma unroll
                for (int n = 0; n < NCH; ++n) {
                    settle(py[n], row.left(n), a.c);
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[n][j] = piece_get(py[n], j);
                }
                float mean2 = 0.0f, r2 = 1.0f;
                if (a.post) stats(row, [&](int n, int j) { return y[n][j]; }, post_layer, a.inv_c, a.eps, sums, mean2, r2);
                __builtin_amdgcn_sched_barrier(0);
                float tn = 0.0f, ts = 0.0f;
#pragma unroll
                for (int n = 0; n < NCH; ++n) {
                    float f[8];
                    factor(1, n, f);                         // zero behind the row's end
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        y[n][j] = (y[n][j] - mean2) * r2;
                        t1[n][j] = __builtin_fmaf(t[n][j], y[n][j], t1[n][j]);
                        if constexpr (kT0) t0[n][j] += t[n][j];
                        t[n][j] *= f[j];
                        tn = __builtin_fmaf(t[n][j], y[n][j], tn);
                        ts += t[n][j];
                    }
                }
                if (a.post) {
                    sums.two(tn, ts);
                    tn *= a.inv_c;
                    ts = post_layer ? ts * a.inv_c : 0.0f;
#pragma unroll
                    for (int n = 0; n < NCH; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j) t[n][j] = r2 * __builtin_fmaf(-tn, y[n][j], t[n][j] - ts);
                }
#pragma unroll
                for (int n = 0; n < NCH; ++n) store8(piece_of<Bf16>(a.dY, (int64_t)row_i * a.lddy, row.at(n)), row.left(n), t[n]);
            }
        }
        // the sums of this workgroup's rows of the segment
        if (a.part) {
            float *const to = a.part + ((int64_t)blockIdx.x + seg) * kNormSums * a.c;
            auto put = [&](int which, float (&v)[NCH][8]) {
                if constexpr (W == 1) {
                    // the upper half of the waves hands its sums to the lower half, whose sums are then added
                    constexpr int kHalf = kBwdWaves / 2, kPlace = 512 * NCH;
                    float *const mine = joined + r_in % kHalf * kPlace + row.lane;
                    __syncthreads();
#pragma unroll
                    for (int n = 0; n < NCH; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (r_in >= kHalf) mine[n * 512 + j * 64] = v[n][j];
                    __syncthreads();
#pragma unroll
                    for (int n = 0; n < NCH; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (r_in < kHalf) mine[n * 512 + j * 64] += v[n][j];
                    __syncthreads();
                    for (int i = threadIdx.x; i < kPlace; i += 64 * kBwdWaves) {
                        const int k = 512 * (i / 512) + 8 * (i % 64) + i % 512 / 64;          // the column that place i holds
                        float s = 0.0f;
#pragma unroll
                        for (int w = 0; w < kHalf; ++w) s += joined[w * kPlace + i];
                        if (k < a.c) to[(int64_t)which * a.c + k] = s;
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < NCH; ++n)
                        if (row.left(n) > 0) store8(to + (int64_t)which * a.c + row.at(n), row.left(n), v[n]);
                }
            };
            put(0, s1);
            if constexpr (kS0) put(1, s0);
            if constexpr (kT1) put(2, t1);
            if constexpr (kT0) put(3, t0);
        }
        first = last;
        if (is_last) break;
    }
}

// Second kernel: COLS columns to a workgroup, 256 / COLS threads to a column and sum.  The threads take segments side by side, `per`
// threads to a segment when there are fewer segments than threads; what they add is joined in a fixed order.  Eight slots' loads
// are in flight at a time (one after the other the kernel took as long as the first one: 18 us for 512 runs of 1152 columns, 16
// segments).  Few columns give narrow rows their workgroups, many columns wide ones whole lines of the sums (us, 8 / 16 / 32 columns: 19056 x
// 384 in 30 segments 11.1 / 15.7 / 22.0, 4096 x 1152 in 16 6.0 / 5.2 / 7.1, 1721 x 4672 in 50 35.0 / 31.7 / 24.8).  Where nothing is added over
// segments, segments that are not done at once go to other workgroups.
constexpr int kJoinThreads = kNormSums * 256;

template <class P>
__device__ __forceinline__ float value_of(const void *p, int64_t i, float without)
{
    if (!p) return without;
    if constexpr (sizeof(P) == 2) return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
    else return static_cast<const float *>(p)[i];
}

template <class P, int COLS>
__global__ __launch_bounds__(kJoinThreads) void block_norm_join_kernel(NormArgs a, int per)
{
    constexpr int kJoinCols = COLS, kJoinLanes = 256 / COLS;
    __shared__ float area[kNormSums][kJoinLanes][kJoinCols];
    const int cc = threadIdx.x % kJoinCols, lane = threadIdx.x / kJoinCols % kJoinLanes;
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x / (kJoinCols * kJoinLanes));          // the thread's sum
    const int k = (int)blockIdx.x * kJoinCols + cc;
    const bool in = k < a.c;
    const int at_once = kJoinLanes / per, mine = lane / per, part = lane % per;
    const int n_seg = a.by_segment ? a.n_seg : 1;
    const float w = in ? value_of<P>(a.pre_w, k, 1.0f) : 0.0f, b = in ? value_of<P>(a.pre_b, k, 0.0f) : 0.0f;
    const float w2 = in ? value_of<P>(a.post_w, k, 1.0f) : 0.0f, b2 = in ? value_of<P>(a.post_b, k, 0.0f) : 0.0f;
    float all[4] = {};                                         // dw, db, dw2, db2 (per thread: of its segments)
    for (int base = (int)blockIdx.y * at_once; base < n_seg; base += (int)gridDim.y * at_once) {
        const int seg = base + mine;
        const bool there = seg < n_seg && in;
        int lo = 0, hi = a.rows;
        if (there && a.by_segment) {
            if (seg > 0) lo = a.seg_off ? a.seg_off[seg] : (int)min((int64_t)seg * a.seg_len, (int64_t)a.rows);
            if (seg + 1 < n_seg) hi = a.seg_off ? a.seg_off[seg + 1] : (int)min((int64_t)(seg + 1) * a.seg_len, (int64_t)a.rows);
            lo = max(0, min(lo, a.rows));
            hi = max(0, min(hi, a.rows));
        }
        // (read here, ahead of the sums, which wait for memory too)
        const bool writes = which == 0 && part == 0 && there, some = hi > lo;
        const float scale = writes ? value_of<P>(a.scale, (int64_t)seg * a.ld_scale + k, 0.0f) : 0.0f;
        const float gate = writes ? value_of<P>(a.gate, (int64_t)seg * a.ld_gate + k, 1.0f) : 1.0f;
        const int g0 = lo / a.rows_per_group, g1 = there && hi > lo ? (hi - 1) / a.rows_per_group : -1;
        float add = 0.0f;
        if (a.sums >> which & 1)
            for (int g = g0 + part; g <= g1; g += 8 * per) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = a.part[(((int64_t)min(g + u * per, g1) + seg) * kNormSums + which) * a.c + k];
#pragma unroll
                for (int u = 0; u < 8; ++u) add += g + u * per <= g1 ? v[u] : 0.0f;
            }
        __syncthreads();
        area[which][lane][cc] = add;
        __syncthreads();
        for (int h = per / 2; h > 0; h /= 2) {
            if (part < h) area[which][lane][cc] += area[which][lane + h][cc];
            __syncthreads();
        }
        const float sum[kNormSums] = {area[0][lane][cc], area[1][lane][cc], area[2][lane][cc], area[3][lane][cc]};
        if (writes) {
            // (a segment without rows: zeros, whatever its parameters and the weights are: nothing was computed with them)
            const int64_t to = (int64_t)seg * a.c + k;
            if (a.dscale) a.dscale[to] = some ? __builtin_fmaf(w, sum[0], b * sum[1]) : 0.0f;
            if (a.dshift) a.dshift[to] = sum[1];
            if (a.dgate && a.gate_by_segment) a.dgate[to] = some ? __builtin_fmaf(w2, sum[2], b2 * sum[3]) : 0.0f;
            if (some) {
                all[0] += (1.0f + scale) * sum[0];
                all[1] += (1.0f + scale) * sum[1];
                if (a.gate_by_segment) {
                    all[2] += gate * sum[2];
                    all[3] += gate * sum[3];
                } else {
                    all[2] += sum[2];
                    all[3] += sum[3];
                }
            }
        }
    }
    __syncthreads();
    if (which == 0)
#pragma unroll
        for (int i = 0; i < kNormSums; ++i) area[i][lane][cc] = all[i];
    __syncthreads();
    for (int h = kJoinLanes / 2; h > 0; h /= 2) {
        if (lane < h) area[which][lane][cc] += area[which][lane + h][cc];
        __syncthreads();
    }
    if (which > 0 || lane > 0 || !in || gridDim.y > 1) return;     // (more than one: nothing is added over segments)
#pragma unroll
    for (int i = 0; i < kNormSums; ++i) all[i] = area[i][0][cc];
    const float gate = a.gate_by_segment ? 1.0f : value_of<P>(a.gate, k, 1.0f);
    if (a.dpre_w) a.dpre_w[k] = all[0];
    if (a.dpre_b) a.dpre_b[k] = all[1];
    if (a.dgate && !a.gate_by_segment) a.dgate[k] = __builtin_fmaf(w2, all[2], b2 * all[3]);
    if (a.dpost_w) a.dpost_w[k] = gate * all[2];
    if (a.dpost_b) a.dpost_b[k] = gate * all[3];
}

// Gradients of a call without rows: sums over nothing.
struct ZeroArgs {
    float *to[7];
    int64_t n[7];
};
__global__ __launch_bounds__(256) void block_norm_zero_kernel(ZeroArgs a)
{
    float *const to = a.to[blockIdx.y];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.n[blockIdx.y]; i += (int64_t)gridDim.x * 256) to[i] = 0.0f;
}

// Waves of a row and pieces of a lane.  Up to 1024 values one wave.  Up to 1536 the gradient keeps one wave (three waves a row, each with its
// sums to write: 4096 x 1152 26 us in place of 21); forward three waves with one piece a lane take 43 to 49 registers in place of 94 to 147, eight
// waves a SIMD in place of three to five (us, one wave / three: 4096 x 1152 bf16 13.3 / 11.8, float32 to codes 32768 x 1152 98.1 / 98.2, one
// row 3.0 / 2.6).  Wider rows: a workgroup each.
template <bool FORWARD, class F>
hipError_t by_width(int c, F &&f)
{
    const int pieces = (c + 7) / 8;
    if (pieces <= 64) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    if (pieces <= 128) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
    if (pieces <= 192) {
        if constexpr (FORWARD) return f(std::integral_constant<int, 3>{}, std::integral_constant<int, 1>{});
        else return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 3>{});
    }
    if (pieces <= 256) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    if (pieces <= 512) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    if (pieces <= 1024) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
}

template <class T, class P>
hipError_t forward(const NormArgs &a, hipStream_t st)
{
    // (codes are written up to the end of the last block)
    return by_width<true>(a.out == TRDQ_E4M3 ? a.nkb * 128 : a.c, [&](auto w, auto nch) {
        constexpr int W = decltype(w)::value, NCH = decltype(nch)::value;
        using F = Forward<W>;
        const uint32_t groups = ((uint32_t)a.rows + F::kRows - 1) / F::kRows;
        block_norm_kernel<T, P, W, NCH><<<dim3(std::min(groups, F::kAcross), (groups + F::kAcross - 1) / F::kAcross), dim3(F::kThreads), 0, st>>>(a);
        return hipGetLastError();
    });
}

template <class T, class P>
hipError_t backward(const NormArgs &a, hipStream_t st)
{
    hipError_t e = by_width<false>(a.c, [&](auto w, auto nch) {
        constexpr int W = decltype(w)::value, NCH = decltype(nch)::value;
        const dim3 grid((unsigned)norm_bwd_groups(a.rows, a.c, a.n_seg)), threads(W == 1 ? 64 * kBwdWaves : 64 * W);
        const bool s0 = a.sums & 2, t0 = a.sums & 8;
        constexpr size_t lds = bwd_factor_bytes<W, NCH>();
        auto go = [&](auto sums) {
            const auto kernel = block_norm_bwd_kernel<T, P, W, NCH, decltype(sums)::value>;
            if (hipError_t f = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), lds); f != hipSuccess) return f;
            kernel<<<grid, threads, lds, st>>>(a);
            return hipGetLastError();
        };
        if (!a.Y) return s0 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 0>{});
        if (t0) return s0 ? go(std::integral_constant<int, 7>{}) : go(std::integral_constant<int, 6>{});
        return s0 ? go(std::integral_constant<int, 3>{}) : go(std::integral_constant<int, 2>{});
    });
    if (e != hipSuccess || !a.part) return e;
    const int n_seg = a.by_segment ? a.n_seg : 1;
    const bool over_segments = a.dpre_w || a.dpre_b || a.dpost_w || a.dpost_b || (a.dgate && !a.gate_by_segment);
    auto join = [&](auto cols) {
        constexpr int COLS = decltype(cols)::value;
        int per = 1;
        while (per * 2 * n_seg <= 256 / COLS) per *= 2;
        const int at_once = 256 / COLS / per;
        const unsigned turns = over_segments ? 1u : (unsigned)std::min((n_seg + at_once - 1) / at_once, 65535);
        block_norm_join_kernel<P, COLS><<<dim3((unsigned)((a.c + COLS - 1) / COLS), turns), dim3(kJoinThreads), 0, st>>>(a, per);
        return hipGetLastError();
    };
    if (a.c <= 1024) return join(std::integral_constant<int, 8>{});
    if (a.c <= 2048) return join(std::integral_constant<int, 16>{});
    return join(std::integral_constant<int, 32>{});
}

}  // namespace

// Rows of a workgroup's run: enough for one workgroup (two or three pieces a lane) or two a compute unit, as many as fit the
// registers, whose sums the second kernel then adds (one piece, 19056 x 384: 32.7 us with 256 runs, 25.1 with 512; 1721 x 4672 in
// float32, its join too: 76 with 512, 65 with 256); but no more than a segment has, on average, while there are few: a run that crosses segments does them one after the other
// (16 rows in 16 segments in two runs of eight: 67 us).
int norm_bwd_rows_per_group(int rows, int c, int64_t segments)
{
    const bool waves = c <= 1536;
    // (in 64 bits: rows may be all but 2^31)
    const int64_t most = (c > 512 && waves) || c > 4096 ? 256 : 512, least = (rows + most - 1) / most;
    const int64_t segment = (rows + segments - 1) / segments;
    const int64_t per = std::max<int64_t>(least, waves ? std::min<int64_t>(segment, kBwdWaves) : 1);
    return (int)(per < kBwdWaves || !waves ? per : (per + kBwdWaves - 1) / kBwdWaves * kBwdWaves);
}

int norm_bwd_groups(int rows, int c, int64_t segments)
{
    const int64_t per = norm_bwd_rows_per_group(rows, c, segments);
    return (int)((rows + per - 1) / per);
}

hipError_t launch_block_norm(const NormArgs &a, bool stream_f32, bool params_f32, hipStream_t st)
{
    if (stream_f32) return params_f32 ? forward<float, float>(a, st) : forward<float, Bf16>(a, st);
    return params_f32 ? forward<Bf16, float>(a, st) : forward<Bf16, Bf16>(a, st);
}

hipError_t launch_zero_gradients(float *const (&grads)[7], const int64_t (&sizes)[7], hipStream_t st)
{
    ZeroArgs a{};
    int64_t most = 0;
    for (int i = 0; i < 7; ++i) {
        a.to[i] = grads[i];
        a.n[i] = grads[i] ? sizes[i] : 0;
        most = std::max(most, a.n[i]);
    }
    if (most == 0) return hipSuccess;
    block_norm_zero_kernel<<<dim3((unsigned)std::min<int64_t>((most + 255) / 256, 1024), 7), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_block_norm_bwd(const NormArgs &a, bool stream_f32, bool params_f32, hipStream_t st)
{
    if (stream_f32) return params_f32 ? backward<float, float>(a, st) : backward<float, Bf16>(a, st);
    return params_f32 ? backward<Bf16, float>(a, st) : backward<Bf16, Bf16>(a, st);
}

}  // namespace trdq
