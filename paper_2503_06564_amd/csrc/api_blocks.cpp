// Entry points around a block's linears: argument checks (all before the first HIP call) and launches.
#include <cmath>

#include "trdq_internal.h"

namespace {

constexpr int64_t kMostRows = 0x80000000 - 256;           // refused from here on: rows of a tile behind the last still count in 31 bits
constexpr int kMostNormChannels = 16384;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline trdq_status hip_status(hipError_t e) { return e == hipSuccess ? TRDQ_OK : TRDQ_ERR_HIP; }
inline int64_t up(int64_t k) { return (k + 127) / 128 * 128; }
inline bool is_float(int t) { return t == TRDQ_BF16 || t == TRDQ_F32; }
inline size_t size_of(int t) { return t == TRDQ_F32 ? 4 : t == TRDQ_BF16 ? 2 : 1; }

// a matrix of c values a row: there, aligned to its values, rows that do not overlap (a single row's stride does not matter)
trdq_status check_matrix(const void *p, int64_t rows, int64_t c, int64_t ld, size_t size)
{
    if (!p) return TRDQ_ERR_NULL;
    if ((rows > 1 && ld < c) || !aligned(p, size)) return TRDQ_ERR_SHAPE;
    return TRDQ_OK;
}

// rows of codes: written and read 16 bytes at a time
trdq_status check_codes(const void *p, int64_t rows, int64_t k, int64_t ld)
{
    if (!p) return TRDQ_ERR_NULL;
    if ((rows > 1 && (ld < k || ld % 16 != 0)) || !aligned(p, 16)) return TRDQ_ERR_SHAPE;
    return TRDQ_OK;
}

#define TRDQ_TRY(call) do { if (trdq_status rc_ = (call); rc_ != TRDQ_OK) return rc_; } while (0)

// what both directions of the block norm check of the description; segments_out: rows of scale, shift and gate
trdq_status check_norm(const trdq_norm *n, int64_t *segments_out)
{
    if (!n) return TRDQ_ERR_NULL;
    if (n->rows < 0 || n->c <= 0) return TRDQ_ERR_SHAPE;
    if (!is_float(n->x_dtype) || !is_float(n->param_dtype) || n->c > kMostNormChannels || n->rows >= kMostRows) return TRDQ_ERR_UNSUPPORTED;
    if ((n->pre != TRDQ_NORM_LAYER && n->pre != TRDQ_NORM_RMS) || n->post < TRDQ_NORM_NONE || n->post > TRDQ_NORM_RMS) return TRDQ_ERR_RANGE;
    if (!(n->eps >= 0.0f) || std::isinf(n->eps) || n->seg_len < 0 || (n->seg_len == 0 && n->seg_off && n->n_seg <= 0)) return TRDQ_ERR_RANGE;
    if (n->seg_len == 0 && n->seg_off && !aligned(n->seg_off, 4)) return TRDQ_ERR_SHAPE;
    // (rows + seg_len may not fit 64 bits)
    const int64_t segments = n->seg_len > 0 ? n->rows / n->seg_len + (n->rows % n->seg_len != 0) : n->seg_off ? n->n_seg : 1;
    const size_t size = size_of(n->param_dtype);
    const void *const vectors[] = {n->pre_weight, n->pre_bias, n->post_weight, n->post_bias, n->scale, n->shift, n->gate};
    for (const void *v : vectors)
        if (!aligned(v, size)) return TRDQ_ERR_SHAPE;
    if (segments > 1 && ((n->scale && n->ld_scale < n->c) || (n->shift && n->ld_shift < n->c) || (n->gate && n->ld_gate != 0 && n->ld_gate < n->c)))
        return TRDQ_ERR_SHAPE;
    if (n->ld_scale < 0 || n->ld_shift < 0 || n->ld_gate < 0) return TRDQ_ERR_SHAPE;
    if (n->post == TRDQ_NORM_NONE && (n->post_weight || n->post_bias)) return TRDQ_ERR_RANGE;
    *segments_out = segments;
    return TRDQ_OK;
}

trdq::NormArgs norm_args(const trdq_norm &n, int64_t segments)
{
    trdq::NormArgs a{};
    a.rows = (int)n.rows; a.c = n.c; a.nkb = (int)(up(n.c) / 128);
    a.pre = n.pre; a.post = n.post; a.eps = n.eps; a.inv_c = 1.0f / (float)n.c;
    a.pre_w = n.pre_weight; a.pre_b = n.pre_bias; a.post_w = n.post_weight; a.post_b = n.post_bias;
    a.scale = n.scale; a.shift = n.shift; a.gate = n.gate;
    a.ld_scale = n.ld_scale; a.ld_shift = n.ld_shift; a.ld_gate = n.ld_gate;
    a.n_seg = (int)segments;
    a.seg_len = n.seg_len > 0 ? (int)(n.seg_len < n.rows ? n.seg_len : n.rows) : 0;
    a.seg_off = n.seg_len > 0 ? nullptr : n.seg_off;
    a.gate_by_segment = n.gate && n.ld_gate != 0;
    // one segment has nothing to look up
    a.by_segment = segments > 1 && (n.scale || n.shift || a.gate_by_segment);
    return a;
}

}  // namespace

extern "C" {

trdq_status trdq_fp8_quant(const void *X_dev, int x_dtype, int64_t rows, int c, int64_t ldx, int blocks,
                           int q_dtype, void *Q_dev, int64_t ldq, int s_dtype, void *S_dev, int64_t lds, void *stream)
{
    if (rows < 0 || c <= 0) return TRDQ_ERR_SHAPE;
    if (blocks < TRDQ_BLOCKS_ROWS || blocks > TRDQ_BLOCKS_TILES_T) return TRDQ_ERR_RANGE;
    if (!is_float(x_dtype) || (q_dtype != TRDQ_E4M3 && q_dtype != TRDQ_E5M2) || (s_dtype != TRDQ_F32 && s_dtype != TRDQ_E8M0) ||
        rows >= kMostRows || c > (1 << 24))
        return TRDQ_ERR_UNSUPPORTED;
    if (rows == 0) return TRDQ_OK;
    const bool turned = blocks == TRDQ_BLOCKS_COLS || blocks == TRDQ_BLOCKS_TILES_T, tiles = blocks >= TRDQ_BLOCKS_TILES;
    const int64_t r = turned ? c : rows, k = up(turned ? rows : c);
    TRDQ_TRY(check_matrix(X_dev, rows, c, ldx, size_of(x_dtype)));
    TRDQ_TRY(check_codes(Q_dev, r, k, ldq));
    TRDQ_TRY(check_matrix(S_dev, k / 128, tiles ? (r + 127) / 128 : r, lds, size_of(s_dtype)));
    return hip_status(trdq::launch_fp8_quant(X_dev, x_dtype == TRDQ_F32, (int)rows, c, ldx, blocks, q_dtype == TRDQ_E5M2,
                                             static_cast<uint8_t *>(Q_dev), ldq, S_dev, lds, s_dtype == TRDQ_E8M0,
                                             static_cast<hipStream_t>(stream)));
}

size_t trdq_fp8_gemm_ws_nbytes(int64_t M, int N, int K)
{
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    return trdq::fp8_gemm_workspace_bytes(M, N, K);
}

size_t trdq_fp8_gemm_ws_nbytes_upto(int64_t M, int N, int K)
{
    if (M <= 0 || M >= kMostRows || N <= 0 || K <= 0) return 0;
    return trdq::fp8_gemm_workspace_bytes_upto(M, N, K);
}

trdq_status trdq_fp8_gemm(int64_t M, int N, int K, const void *A_dev, int a_dtype, int64_t lda, const void *sa_dev, int64_t ldsa,
                          const void *B_dev, int b_dtype, int64_t ldb, const void *sb_dev, int64_t ldsb, int b_tiles, int s_dtype,
                          const float *bias_dev, void *Y_dev, int y_dtype, int64_t ldy, void *ws_dev, size_t ws_bytes, void *stream)
{
    if (M < 0 || N <= 0 || K <= 0 || K % 128 != 0) return TRDQ_ERR_SHAPE;
    if ((a_dtype != TRDQ_E4M3 && a_dtype != TRDQ_E5M2) || b_dtype != TRDQ_E4M3 || (s_dtype != TRDQ_F32 && s_dtype != TRDQ_E8M0) ||
        !is_float(y_dtype) || M >= kMostRows || N >= kMostRows)
        return TRDQ_ERR_UNSUPPORTED;
    if (M == 0) return TRDQ_OK;
    TRDQ_TRY(check_codes(A_dev, M, K, lda));
    TRDQ_TRY(check_codes(B_dev, N, K, ldb));
    if ((M > 1 && lda > (1 << 22)) || (N > 1 && ldb > (1 << 22))) return TRDQ_ERR_SHAPE;
    TRDQ_TRY(check_matrix(sa_dev, K / 128, M, ldsa, size_of(s_dtype)));
    TRDQ_TRY(check_matrix(sb_dev, K / 128, b_tiles ? (N + 127) / 128 : N, ldsb, size_of(s_dtype)));
    TRDQ_TRY(check_matrix(Y_dev, M, N, ldy, size_of(y_dtype)));
    if (!aligned(bias_dev, 4)) return TRDQ_ERR_SHAPE;
    if (const size_t need = trdq::fp8_gemm_workspace_bytes(M, N, K)) {
        if (!ws_dev) return TRDQ_ERR_NULL;
        if (ws_bytes < need || !aligned(ws_dev, 16)) return TRDQ_ERR_SHAPE;
    }
    trdq::Fp8GemmArgs a{};
    a.A = static_cast<const uint8_t *>(A_dev); a.B = static_cast<const uint8_t *>(B_dev);
    a.sa = sa_dev; a.sb = sb_dev; a.bias = bias_dev; a.Y = Y_dev; a.ws = static_cast<float *>(ws_dev);
    a.lda = lda; a.ldb = ldb; a.ldsa = ldsa; a.ldsb = ldsb; a.ldy = ldy;
    a.M = (int)M; a.N = N; a.nkb = K / 128;
    a.out_f32 = y_dtype == TRDQ_F32;
    a.b_tiles = b_tiles != 0;
    return hip_status(trdq::launch_fp8_gemm(a, a_dtype == TRDQ_E5M2, s_dtype == TRDQ_E8M0, b_tiles != 0, static_cast<hipStream_t>(stream)));
}

trdq_status trdq_block_norm(const trdq_norm *n, const void *X_dev, int64_t ldx, const void *Y_dev, int64_t ldy,
                            void *Xout_dev, int64_t ldxo, int h_dtype, void *H_dev, int64_t ldh, int s_dtype, void *S_dev, int64_t lds,
                            void *stream)
{
    int64_t segments = 0;
    TRDQ_TRY(check_norm(n, &segments));
    const bool codes = h_dtype == TRDQ_E4M3;
    if (!is_float(h_dtype) && !codes) return TRDQ_ERR_UNSUPPORTED;
    if (codes && s_dtype != TRDQ_F32 && s_dtype != TRDQ_E8M0) return TRDQ_ERR_UNSUPPORTED;
    if (n->rows == 0) return TRDQ_OK;
    const size_t xs = size_of(n->x_dtype);
    TRDQ_TRY(check_matrix(X_dev, n->rows, n->c, ldx, xs));
    if (!Y_dev != !Xout_dev) return TRDQ_ERR_SHAPE;
    if (Y_dev) {
        TRDQ_TRY(check_matrix(Y_dev, n->rows, n->c, ldy, 2));
        TRDQ_TRY(check_matrix(Xout_dev, n->rows, n->c, ldxo, xs));
    }
    if (codes) {
        TRDQ_TRY(check_codes(H_dev, n->rows, up(n->c), ldh));
        TRDQ_TRY(check_matrix(S_dev, up(n->c) / 128, n->rows, lds, size_of(s_dtype)));
    } else {
        TRDQ_TRY(check_matrix(H_dev, n->rows, n->c, ldh, size_of(h_dtype)));
    }
    trdq::NormArgs a = norm_args(*n, segments);
    a.X = X_dev; a.ldx = ldx; a.Y = Y_dev; a.ldy = ldy; a.Xout = Xout_dev; a.ldxo = ldxo;
    a.out = h_dtype;
    if (codes) { a.Q = static_cast<uint8_t *>(H_dev); a.ldq = ldh; a.S = S_dev; a.lds = lds; a.pow2 = s_dtype == TRDQ_E8M0; }
    else { a.H = H_dev; a.ldh = ldh; }
    return hip_status(trdq::launch_block_norm(a, n->x_dtype == TRDQ_F32, n->param_dtype == TRDQ_F32, static_cast<hipStream_t>(stream)));
}

size_t trdq_block_norm_bwd_ws_nbytes(int64_t rows, int c, int64_t segments)
{
    if (rows <= 0 || rows >= kMostRows || c <= 0 || c > kMostNormChannels || segments <= 0 || segments > 0x7FFFFFFF) return 0;
    return (size_t)(trdq::norm_bwd_groups((int)rows, c, segments) + segments) * trdq::kNormSums * c * sizeof(float);
}

trdq_status trdq_block_norm_bwd(const trdq_norm *n, const trdq_norm_grads *g, void *ws_dev, size_t ws_bytes, void *stream)
{
    int64_t segments = 0;
    TRDQ_TRY(check_norm(n, &segments));
    if (!g) return TRDQ_ERR_NULL;
    const bool none = n->rows == 0;                    // no row to read or write, but parameters' gradients, which are zeros
    if (!none) {
        const size_t xs = size_of(n->x_dtype);
        TRDQ_TRY(check_matrix(g->Xout_dev, n->rows, n->c, g->ldxo, xs));
        TRDQ_TRY(check_matrix(g->dH_dev, n->rows, n->c, g->lddh, 2));
        TRDQ_TRY(check_matrix(g->dX_dev, n->rows, n->c, g->lddx, xs));
        if (g->dXout_dev) TRDQ_TRY(check_matrix(g->dXout_dev, n->rows, n->c, g->lddxo, xs));
        if (!g->Y_dev != !g->dY_dev) return TRDQ_ERR_SHAPE;
        if (g->Y_dev) {
            TRDQ_TRY(check_matrix(g->Y_dev, n->rows, n->c, g->ldy, 2));
            TRDQ_TRY(check_matrix(g->dY_dev, n->rows, n->c, g->lddy, 2));
        }
    }
    const bool branch = none || g->Y_dev;              // (a branch of no rows need not have an address)
    const void *const params[] = {n->scale, n->shift, branch ? n->gate : nullptr, n->pre_weight, n->pre_bias,
                                  branch ? n->post_weight : nullptr, branch ? n->post_bias : nullptr};
    float *const grads[] = {g->dscale_dev, g->dshift_dev, g->dgate_dev, g->dpre_weight_dev, g->dpre_bias_dev, g->dpost_weight_dev, g->dpost_bias_dev};
    bool any = false;
    for (int i = 0; i < 7; ++i) {
        if (grads[i] && !params[i]) return TRDQ_ERR_NULL;
        if (!aligned(grads[i], 4)) return TRDQ_ERR_SHAPE;
        any = any || grads[i];
    }
    if (none) {
        const int64_t per_segment = segments * n->c, vector = n->c;
        const int64_t sizes[] = {per_segment, per_segment, n->ld_gate != 0 ? per_segment : vector, vector, vector, vector, vector};
        return hip_status(trdq::launch_zero_gradients(grads, sizes, static_cast<hipStream_t>(stream)));
    }
    trdq::NormArgs a = norm_args(*n, segments);
    if (any) {
        if (!ws_dev) return TRDQ_ERR_NULL;
        if (ws_bytes < trdq_block_norm_bwd_ws_nbytes(n->rows, n->c, segments) || !aligned(ws_dev, 16)) return TRDQ_ERR_SHAPE;
        a.part = static_cast<float *>(ws_dev);
    }
    a.X = g->Xout_dev; a.ldx = g->ldxo; a.Y = g->Y_dev; a.ldy = g->ldy;
    a.dXout = g->dXout_dev; a.lddxo = g->lddxo; a.dH = g->dH_dev; a.lddh = g->lddh;
    a.dX = g->dX_dev; a.lddx = g->lddx; a.dY = g->dY_dev; a.lddy = g->lddy;
    a.dscale = g->dscale_dev; a.dshift = g->dshift_dev; a.dgate = g->dgate_dev;
    a.dpre_w = g->dpre_weight_dev; a.dpre_b = g->dpre_bias_dev; a.dpost_w = g->dpost_weight_dev; a.dpost_b = g->dpost_bias_dev;
    a.rows_per_group = trdq::norm_bwd_rows_per_group(a.rows, a.c, segments);
    a.sums = 1 | (a.dshift || a.dpre_b || (a.dscale && a.pre_b) ? 2 : 0) | (a.Y ? 4 : 0) |
             (a.Y && (a.dpost_b || (a.dgate && a.post_b)) ? 8 : 0);
    return hip_status(trdq::launch_block_norm_bwd(a, n->x_dtype == TRDQ_F32, n->param_dtype == TRDQ_F32, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
