// C-ABI layer of the operators around the quantized linears (norms, nonlinearities, 8-bit checkpoints, products of single tokens):
// host-side validation before the first HIP call, then one launcher each.
#include "../../include/tjnvfp4.h"
#include "block_ops.h"

namespace tj {

namespace {

constexpr int64_t kMaxElems = (int64_t)1 << 33;      // of an array
constexpr int64_t kMaxSpan = (int64_t)1 << 46;       // elements from its first to its last, with the strides
constexpr int64_t kMaxRow = (int64_t)1 << 22;        // of a norm, and of a reduction
constexpr int64_t kMaxCols = (int64_t)1 << 30;       // of any other row

bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_sizes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxElems || cols > kMaxCols) return NVFP4_ERR_SHAPE;
    return rows > 0 && cols > kMaxElems / rows ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

int check_span(int64_t rows, int64_t cols, int64_t ld)
{
    if (ld < cols) return NVFP4_ERR_SHAPE;
    return rows > 0 && ld > kMaxSpan / rows ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

int check_ckpt(const nvfp4_ckpt8 *c)
{
    return !c || !c->codes || !c->exps ? NVFP4_ERR_NULL : NVFP4_OK;
}

int64_t groups_of(int64_t cols) { return (cols + kCkptGroup - 1) / kCkptGroup; }

// a strided source of rows x cols, or a checkpoint of ckpt_rows x ckpt_cols (ckpt_rows < 0: none is taken)
int make_src(const void *p, int kind, int64_t ld, int64_t rows, int64_t cols, int64_t ckpt_rows, int64_t ckpt_cols, RowSrc *s)
{
    if (!p) return NVFP4_ERR_NULL;
    if (kind == NVFP4_SRC_CKPT8 && ckpt_rows >= 0) {
        const nvfp4_ckpt8 *c = static_cast<const nvfp4_ckpt8 *>(p);
        const int rc = check_ckpt(c);
        if (rc) return rc;
        if (c->rows != ckpt_rows || c->K != ckpt_cols) return NVFP4_ERR_MISMATCH;
        *s = RowSrc{c->codes, c->exps, ckpt_cols, groups_of(ckpt_cols), kCkpt8};
        return NVFP4_OK;
    }
    if (kind != NVFP4_SRC_BF16 && kind != NVFP4_SRC_F32) return NVFP4_ERR_ENUM;
    const int rc = check_span(rows, cols, ld);
    if (rc) return rc;
    if (!aligned(p, kind == NVFP4_SRC_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
    *s = RowSrc{p, nullptr, ld, 0, kind == NVFP4_SRC_F32 ? kF32 : kBf16};
    return NVFP4_OK;
}

int make_dst(void *p, int out_dtype, int64_t ld, int64_t rows, int64_t cols, RowDst *d)
{
    if (!p) return NVFP4_ERR_NULL;
    if (out_dtype != NVFP4_OUT_BF16 && out_dtype != NVFP4_OUT_F32) return NVFP4_ERR_ENUM;
    const int rc = check_span(rows, cols, ld);
    if (rc) return rc;
    if (!aligned(p, out_dtype == NVFP4_OUT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
    *d = RowDst{p, ld, out_dtype == NVFP4_OUT_F32};
    return NVFP4_OK;
}

// where a checkpoint goes; `optional`: a null one is none
int make_ckpt(nvfp4_ckpt8 *c, bool optional, int64_t cols, CkptOut *o)
{
    *o = CkptOut{nullptr, nullptr, 0};
    if (!c && optional) return NVFP4_OK;
    const int rc = check_ckpt(c);
    if (rc) return rc;
    *o = CkptOut{c->codes, c->exps, groups_of(cols)};
    return NVFP4_OK;
}

void stamp(nvfp4_ckpt8 *c, int64_t rows, int64_t cols)
{
    if (!c) return;
    c->rows = rows;
    c->K = cols;
}

int status(hipError_t e) { return e == hipSuccess ? NVFP4_OK : NVFP4_ERR_HIP; }

}  // namespace

}  // namespace tj

using namespace tj;

extern "C" {

int nvfp4_norm_fwd(const void *X, int src_kind, int64_t ldx, int64_t N, int64_t D, const float *gamma, const float *beta, float eps,
                   int norm, void *Y, int out_dtype, int64_t ldy, float *stats, nvfp4_ckpt8 *ckpt, void *stream)
{
    int rc = check_sizes(N, D);
    if (rc) return rc;
    if (D > kMaxRow) return NVFP4_ERR_SHAPE;
    RowSrc x;
    RowDst y;
    CkptOut c;
    rc = make_src(X, src_kind, ldx, N, D, -1, 0, &x);
    if (rc) return rc;
    rc = make_dst(Y, out_dtype, ldy, N, D, &y);
    if (rc) return rc;
    rc = make_ckpt(ckpt, true, D, &c);
    if (rc) return rc;
    if (norm != NVFP4_NORM_LAYER && norm != NVFP4_NORM_RMS) return NVFP4_ERR_ENUM;
    if (!(eps >= 0.0f)) return NVFP4_ERR_ENUM;
    if (!aligned(gamma, 16) || !aligned(beta, 16) || !aligned(stats, 8)) return NVFP4_ERR_ALIGN;
    stamp(ckpt, N, D);
    if (N == 0 || D == 0) return NVFP4_OK;
    return status(launch_norm_fwd(x, N, D, gamma, beta, eps, norm == NVFP4_NORM_LAYER, y, stats, c, static_cast<hipStream_t>(stream)));
}

size_t nvfp4_norm_workspace_bytes(int64_t N, int64_t D)
{
    if (check_sizes(N, D) || D > kMaxRow || N == 0 || D == 0) return 0;
    return norm_bwd_workspace_bytes(N, D);
}

int nvfp4_norm_bwd(const void *dY, int dy_kind, int64_t lddy, const void *X, int src_kind, int64_t ldx, const float *stats,
                   const float *gamma, int64_t N, int64_t D, int norm, void *dX, int out_dtype, int64_t lddx, float *dgamma,
                   float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_sizes(N, D);
    if (rc) return rc;
    if (D > kMaxRow) return NVFP4_ERR_SHAPE;
    RowSrc dy, x;
    RowDst dx;
    rc = make_src(dY, dy_kind, lddy, N, D, -1, 0, &dy);
    if (rc) return rc;
    rc = make_src(X, src_kind, ldx, N, D, N, D, &x);
    if (rc) return rc;
    if (!stats) return NVFP4_ERR_NULL;
    rc = make_dst(dX, out_dtype, lddx, N, D, &dx);
    if (rc) return rc;
    if (norm != NVFP4_NORM_LAYER && norm != NVFP4_NORM_RMS) return NVFP4_ERR_ENUM;
    if (!aligned(stats, 8) || !aligned(gamma, 16) || !aligned(dgamma, 16) || !aligned(dbeta, 16)) return NVFP4_ERR_ALIGN;
    const size_t need = dgamma || dbeta ? nvfp4_norm_workspace_bytes(N, D) : 0;
    if (need && (!ws || ws_bytes < need)) return NVFP4_ERR_WORKSPACE;
    if (need && !aligned(ws, 16)) return NVFP4_ERR_ALIGN;
    if (D == 0) return NVFP4_OK;
    return status(launch_norm_bwd(dy, x, stats, gamma, N, D, norm == NVFP4_NORM_LAYER, dx, dgamma, dbeta, ws, static_cast<hipStream_t>(stream)));
}

int nvfp4_act_fwd(const void *H, int src_kind, int64_t ldh, int64_t N, int64_t F, int act, void *A, int out_dtype, int64_t lda,
                  nvfp4_ckpt8 *ckpt, void *stream)
{
    if (act != NVFP4_ACT_SWIGLU && act != NVFP4_ACT_GELU) return NVFP4_ERR_ENUM;
    const int64_t parts = act == NVFP4_ACT_SWIGLU ? 2 : 1;
    int rc = F < 0 || F > kMaxCols ? NVFP4_ERR_SHAPE : check_sizes(N, parts * F);      // within these, 2 F does not overflow
    if (rc) return rc;
    RowSrc h;
    RowDst a;
    CkptOut c;
    rc = make_src(H, src_kind, ldh, N, parts * F, -1, 0, &h);
    if (rc) return rc;
    rc = make_dst(A, out_dtype, lda, N, F, &a);
    if (rc) return rc;
    rc = make_ckpt(ckpt, true, F, &c);
    if (rc) return rc;
    stamp(ckpt, parts * N, F);
    if (N == 0 || F == 0) return NVFP4_OK;
    return status(launch_act_fwd(h, N, F, act, a, c, static_cast<hipStream_t>(stream)));
}

int nvfp4_act_bwd(const void *dA, int da_kind, int64_t ldda, const void *H, int src_kind, int64_t ldh, int64_t N, int64_t F, int act,
                  void *dH, int out_dtype, int64_t lddh, void *stream)
{
    if (act != NVFP4_ACT_SWIGLU && act != NVFP4_ACT_GELU) return NVFP4_ERR_ENUM;
    const int64_t parts = act == NVFP4_ACT_SWIGLU ? 2 : 1;
    int rc = F < 0 || F > kMaxCols ? NVFP4_ERR_SHAPE : check_sizes(N, parts * F);      // within these, 2 F does not overflow
    if (rc) return rc;
    RowSrc da, h;
    RowDst dh;
    rc = make_src(dA, da_kind, ldda, N, F, -1, 0, &da);
    if (rc) return rc;
    rc = make_src(H, src_kind, ldh, N, parts * F, parts * N, F, &h);
    if (rc) return rc;
    rc = make_dst(dH, out_dtype, lddh, N, parts * F, &dh);
    if (rc) return rc;
    if (N == 0 || F == 0) return NVFP4_OK;
    return status(launch_act_bwd(da, h, N, F, act, dh, static_cast<hipStream_t>(stream)));
}

int nvfp4_ckpt8_save(const void *X, int src_kind, int64_t ldx, int64_t N, int64_t D, nvfp4_ckpt8 *out, void *stream)
{
    int rc = check_sizes(N, D);
    if (rc) return rc;
    RowSrc x;
    CkptOut c;
    rc = make_src(X, src_kind, ldx, N, D, -1, 0, &x);
    if (rc) return rc;
    rc = make_ckpt(out, false, D, &c);
    if (rc) return rc;
    stamp(out, N, D);
    if (N == 0 || D == 0) return NVFP4_OK;
    return status(launch_ckpt8_save(x, N, D, c, static_cast<hipStream_t>(stream)));
}

int nvfp4_ckpt8_load(const nvfp4_ckpt8 *src, void *Y, int out_dtype, int64_t ldy, void *stream)
{
    int rc = check_ckpt(src);
    if (rc) return rc;
    const int64_t N = src->rows, D = src->K;
    rc = check_sizes(N, D);
    if (rc) return rc;
    RowSrc x;
    RowDst y;
    rc = make_src(src, NVFP4_SRC_CKPT8, 0, N, D, N, D, &x);
    if (rc) return rc;
    rc = make_dst(Y, out_dtype, ldy, N, D, &y);
    if (rc) return rc;
    if (N == 0 || D == 0) return NVFP4_OK;
    return status(launch_ckpt8_load(x, N, D, y, static_cast<hipStream_t>(stream)));
}

int nvfp4_gemv(const void *X, int64_t ldx, int64_t M, const nvfp4_tensor *W, void *Y, int out_dtype, int64_t ldy, void *stream)
{
    if (!X || !W || !W->codes || !W->scales || !W->gscale) return NVFP4_ERR_NULL;
    if (W->outer_mode != NVFP4_OUTER_TENSOR && W->outer_mode != NVFP4_OUTER_BLOCK128) return NVFP4_ERR_ENUM;
    const int64_t C = W->rows, K = W->K;
    if (K % (W->outer_mode == NVFP4_OUTER_BLOCK128 ? 128 : 16) != 0 || K > kMaxRow) return NVFP4_ERR_SHAPE;
    if (M > kMaxGemvTokens || C > kMaxGemvRows) return NVFP4_ERR_SHAPE;
    int rc = check_sizes(C, K);
    if (rc) return rc;
    rc = check_sizes(M, K);
    if (rc) return rc;
    rc = check_sizes(M, C);
    if (rc) return rc;
    if (!aligned(W->codes, 16) || !aligned(W->scales, 16) || !aligned(W->gscale, 4)) return NVFP4_ERR_ALIGN;
    RowSrc x;
    RowDst y;
    rc = make_src(X, NVFP4_SRC_BF16, ldx, M, K, -1, 0, &x);
    if (rc) return rc;
    rc = make_dst(Y, out_dtype, ldy, M, C, &y);
    if (rc) return rc;
    if (M == 0 || C == 0) return NVFP4_OK;
    const GemmOperand w{W->codes, W->scales, W->gscale, C, W->outer_mode == NVFP4_OUTER_BLOCK128, 0};
    return status(launch_gemv(X, ldx, M, w, K, y, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
