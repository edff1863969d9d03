// Launchers of the operators around the quantized linears: norms, nonlinearities, 8-bit checkpoints, products of single tokens.
#pragma once
#include "internal.h"

namespace tj {

constexpr int kCkptGroup = 128;          // elements of a row that share a power of two in an 8-bit checkpoint
enum { kBf16 = 0, kF32 = 1, kCkpt8 = 2 };   // kinds of a source

struct RowSrc {
    const void *p;           // elements, or the codes of a checkpoint
    const uint8_t *exps;     // of a checkpoint: [rows][groups]
    int64_t ld;              // elements from row to row
    int64_t groups;          // of a checkpoint: groups of a row
    int kind;
};
struct RowDst {
    void *p;
    int64_t ld;
    int f32;
};
struct CkptOut {
    uint8_t *codes;          // [rows][n], null where none is wanted
    uint8_t *exps;           // [rows][groups]: 127 + e
    int64_t groups;
};

// Calls that move more than half of the 256 MB last-level cache read their arrays past it: what the reads would leave there displaces what the call
// writes, which is read next.  A kernel of its own: asked at each access, the question costs more than it gives.  us, through the caches /
// past them: SwiGLU 16384 x 4096 (537 MB) forward 95.5 / 91.5, backward 91 / 82, norm backward 4096 x 16384 (336 MB) 78 / 66, checkpoint 8192 x 8192
// saved (201 MB) 39.5 / 34.7; and under it the other way: GELU 4099 x 2752 (56 MB) forward 11.8 / 13.2, backward 12.2 / 13.5.  (The norm's
// forward pass gains nothing: 4096 x 16384 67.9 / 68.7; writes past the caches make the next reader pay: the same checkpoint loaded 31 / 40.)
inline bool streams(double bytes) { return bytes > (double)(128 << 20); }

// norm of N rows of D (layer: with the mean taken off); gamma, beta, stats ([N] pairs of mean and 1 / deviation) and the checkpoint are optional
hipError_t launch_norm_fwd(const RowSrc &x, int64_t N, int64_t D, const float *gamma, const float *beta, float eps, int layer, const RowDst &y,
                           float *stats, const CkptOut &ckpt, hipStream_t st);
// its gradients; dgamma and dbeta are optional.  ws: norm_bwd_workspace_bytes, not read where both are null
size_t norm_bwd_workspace_bytes(int64_t N, int64_t D);
hipError_t launch_norm_bwd(const RowSrc &dy, const RowSrc &x, const float *stats, const float *gamma, int64_t N, int64_t D, int layer,
                           const RowDst &dx, float *dgamma, float *dbeta, void *ws, hipStream_t st);

// the nonlinearity on N rows: act 0 SwiGLU (rows of H and dH: F gates, then F up values; a checkpoint has them as two rows), 1 GELU
hipError_t launch_act_fwd(const RowSrc &h, int64_t N, int64_t F, int act, const RowDst &out, const CkptOut &ckpt, hipStream_t st);
hipError_t launch_act_bwd(const RowSrc &da, const RowSrc &h, int64_t N, int64_t F, int act, const RowDst &out, hipStream_t st);
hipError_t launch_ckpt8_save(const RowSrc &src, int64_t N, int64_t D, const CkptOut &ckpt, hipStream_t st);
hipError_t launch_ckpt8_load(const RowSrc &src, int64_t N, int64_t D, const RowDst &out, hipStream_t st);

// Y[M x W.rows] = X[M x K] (bf16) * W^T; at most kMaxGemvTokens rows of X and kMaxGemvRows rows of W (the launch's grid)
constexpr int64_t kMaxGemvTokens = 1 << 20, kMaxGemvRows = 1 << 26;
hipError_t launch_gemv(const void *X, int64_t ldx, int64_t M, const GemmOperand &W, int64_t K, const RowDst &y, hipStream_t st);

}  // namespace tj
