// Host-side checks of strided row arrays and 8-bit checkpoints, shared by the C-ABI layers of the operators that take them.
#pragma once
#include "../../include/tjnvfp4.h"
#include "block_ops.h"

namespace tj {

namespace {

constexpr int64_t kMaxElems = (int64_t)1 << 33;      // of an array
constexpr int64_t kMaxSpan = (int64_t)1 << 46;       // elements from its first to its last, with the strides
constexpr int64_t kMaxCols = (int64_t)1 << 30;       // of a row

inline bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline int check_sizes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > kMaxElems || cols > kMaxCols) return NVFP4_ERR_SHAPE;
    return rows > 0 && cols > kMaxElems / rows ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

inline int check_span(int64_t rows, int64_t cols, int64_t ld)
{
    if (ld < cols) return NVFP4_ERR_SHAPE;
    return rows > 0 && ld > kMaxSpan / rows ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

inline int check_ckpt(const nvfp4_ckpt8 *c)
{
    return !c || !c->codes || !c->exps ? NVFP4_ERR_NULL : NVFP4_OK;
}

inline int64_t groups_of(int64_t cols) { return (cols + kCkptGroup - 1) / kCkptGroup; }

// a strided source of rows x cols, or a checkpoint of ckpt_rows x ckpt_cols (ckpt_rows < 0: none is taken)
inline int make_src(const void *p, int kind, int64_t ld, int64_t rows, int64_t cols, int64_t ckpt_rows, int64_t ckpt_cols, RowSrc *s)
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

inline int make_dst(void *p, int out_dtype, int64_t ld, int64_t rows, int64_t cols, RowDst *d)
{
    if (!p) return NVFP4_ERR_NULL;
    if (out_dtype != NVFP4_OUT_BF16 && out_dtype != NVFP4_OUT_F32) return NVFP4_ERR_ENUM;
    const int rc = check_span(rows, cols, ld);
    if (rc) return rc;
    if (!aligned(p, out_dtype == NVFP4_OUT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
    *d = RowDst{p, ld, out_dtype == NVFP4_OUT_F32};
    return NVFP4_OK;
}

inline int status(hipError_t e) { return e == hipSuccess ? NVFP4_OK : NVFP4_ERR_HIP; }

}  // namespace

}  // namespace tj
