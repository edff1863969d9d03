// Layer norm and RMS norm of the rows of an [N x D] array, forward and backward.
//
//   forward    mu = sum x / D (RMS norm: 0), r = 1 / sqrt(sum (x - mu)^2 / D + eps), y = (x - mu) r gamma + beta
//   backward   h = (x - mu) r, g = dy gamma:  dx = r (g - mean(g) - h mean(g h))  (RMS norm: without mean(g)),
//              dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// A row is read once and stays in the registers of the TPR threads that hold it (a wave, or a workgroup for longer rows), so
// that the variance is taken about the mean without a second read.  All sums are binary32.  Bound: HBM (a copy of 1 GB reaches 5.1 TB/s here,
// one of 64 MB, which the last-level cache holds, 6.9); calls of a few rows: the launch, 2.2 us.
//
// Figures: bf16 rows where nothing else stands, layer norm, us of a kernel in a kernel trace and TB/s over the bytes that a call has to read and write; calls on three sets of
// arrays in turn (the comparisons of two forms: on one set).
#include "rowwise.h"

namespace tj {

namespace {

struct NormFwdArgs {
    RowSrc x;
    int64_t N;
    int D;
    const float *gamma, *beta;
    float eps;
    int layer;
    RowDst y;
    float2_t *stats;
    CkptOut ckpt;
};

struct NormBwdArgs {
    RowSrc dy, x;
    const float2_t *stats;
    const float *gamma;
    int64_t N;
    int D, layer;
    RowDst dx;
    float *part_g, *part_b;      // sums of a workgroup's rows: workgroup w writes D floats at part + w * part_ld; null where not wanted
    int64_t part_ld;
};

// eight parameters of the columns from col on, `fill` where there are none
__device__ __forceinline__ void param8(const float *p, int col, int D, float fill, float (&v)[8])
{
    if (p && col + kChunk <= D) {
        const float4_t lo = *reinterpret_cast<const float4_t *>(p + col), hi = *reinterpret_cast<const float4_t *>(p + col + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = lo[i];
            v[4 + i] = hi[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p && col + i < D ? p[col + i] : fill;
    }
}

// The parameters of the columns of a row of at least eight to LDS, [halves of a chunk][V TPR chunks], by the TPR threads of a row; `fill` without parameters.  All
// loads are on their way at once: no lane is asked whether it has columns, one that has none gets zeros in the end.
template <int TPR, int V> __device__ __forceinline__ void params_to_lds(const float *p, int D, float fill, float4_t *to)
{
    const int t = threadIdx.x % TPR;
    Raw<kF32> w[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        w[v].lo = w[v].hi = float4_t{fill, fill, fill, fill};
        if (p) {
            const int col = (t + v * TPR) * kChunk, at = col + kChunk > D ? D - kChunk : col;
            w[v].lo = load_as<f32x4_at4, false>(p + at);
            w[v].hi = load_as<f32x4_at4, false>(p + at + 4);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = (t + v * TPR) * kChunk;
        if (p) w[v] = settle8(w[v], col, D);
        to[t + v * TPR] = col < D ? w[v].lo : float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        to[V * TPR + t + v * TPR] = col < D ? w[v].hi : float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
}

// A row lies in the registers of TPR threads, V chunks of eight each; the parameters of a thread's columns stay there for all of its rows,
// and the next row is on its way while a row is summed and written.
//                      8192 x 768    16384 x 1024   16384 x 2048   16384 x 4096   8192 x 8192   4096 x 16384
//   with a checkpoint   10.4  3.0      15.0  5.6      34.8  4.8      67.8  5.0      64.3  5.2      63.3  5.3
//   without              8.2  3.1      11.8  5.7      25.7  5.2      51.6  5.2      49.0  5.5      49.4  5.4
// RMS norm with a checkpoint 8192 x 768 9.4, 8192 x 4096 33.0, 5.1; binary32 with one 16384 x 1024 32.7, 4.6, 8192 x 4096 58.0, 5.2, 4096 x 16384 112, 5.4.
template <int KIND, bool OF32, int TPR, int V>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_fwd_kernel(const NormFwdArgs a)
{
    constexpr int ROWS = TPR < 256 ? 256 / TPR : 1, CHUNKS = V * TPR;
    constexpr bool LDS = TPR == 64 && V > 2;        // parameters there: registers for more waves (V = 2 without: 16384 x 1024 15.1 us, with 16.6)
    __shared__ float2_t red[2][ROWS * TPR / 64];
    __shared__ float4_t weight[LDS ? 4 * CHUNKS : 1];      // [gamma, beta][halves of a chunk][chunks]
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inv_d = 1.0f / (float)a.D;
    float g[V][8], b[V][8];
    Raw<KIND> next[V];
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            next[v] = col < a.D ? load8<KIND, true, false>(a.x, row, col, a.D) : zero8<KIND>();
        }
    };
    int64_t row = (int64_t)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);     // the same in all lanes of a wave
    int turn = 0;              // half of red that the next sum takes: every sum the other one, of whichever row
    if constexpr (LDS) {
        if (row < a.N) load(row);
        const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
        if (slot == 0) params_to_lds<TPR, V>(a.gamma, a.D, 1.0f, weight);
        if (slot == 1) params_to_lds<TPR, V>(a.beta, a.D, 0.0f, weight + 2 * CHUNKS);
        __syncthreads();
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            param8(a.gamma, (t + v * TPR) * kChunk, a.D, 1.0f, g[v]);
            param8(a.beta, (t + v * TPR) * kChunk, a.D, 0.0f, b[v]);
        }
        if (row < a.N) load(row);
    }
    for (; row < a.N; row += step) {       // one row a workgroup where TPR > 64: all of its threads are here
        float x[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) widen8(next[v], (t + v * TPR) * kChunk, a.D, x[v]);
        if (row + step < a.N) load(row + step);
        float mean = 0.0f, none = 0.0f;
        if (a.layer) {
            float sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[v][i];
            row_sum2<TPR>(sum, none, red[turn]);
            turn ^= 1;
            mean = sum * inv_d;
        }
        if (a.ckpt.codes) {
#pragma unroll
            for (int v = 0; v < V; ++v) ckpt_store8<true>(a.ckpt, row, (t + v * TPR) * kChunk, a.D, x[v]);
        }
        float sq = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[v][i] -= mean;
                if ((t + v * TPR) * kChunk + i < a.D) sq = fmaf(x[v][i], x[v][i], sq);
            }
        row_sum2<TPR>(sq, none, red[turn]);
        turn ^= 1;
        const float rstd = 1.0f / sqrtf(sq * inv_d + a.eps);
        if (a.stats && t == 0) a.stats[row] = float2_t{mean, rstd};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D) continue;
            if constexpr (LDS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    g[v][i] = weight[i / 4 * CHUNKS + t + v * TPR][i & 3];
                    b[v][i] = weight[(2 + i / 4) * CHUNKS + t + v * TPR][i & 3];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] = fmaf(x[v][i] * rstd, g[v][i], b[v][i]);
            store8<OF32, true>(a.y.p, a.y.ld, row, col, a.D, x[v]);
        }
    }
}

// rows that no workgroup's registers hold, and rows shorter than a chunk: three sweeps over the row, the later ones from the caches
// (2048 x 32768 88 us, 3.1 TB/s, with a checkpoint 102, 3.3)
template <int KIND, bool OF32>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(const NormFwdArgs a)
{
    constexpr int TPR = 1024;
    __shared__ float2_t red[2][TPR / 64];
    const int t = threadIdx.x;
    const float inv_d = 1.0f / (float)a.D;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        float x[8];
        float none = 0.0f, mean = 0.0f, sq = 0.0f;
        if (a.layer) {
            float sum = 0.0f;
            for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
                widen8(load8<KIND, false, false>(a.x, row, col, a.D), col, a.D, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i];
            }
            row_sum2<TPR>(sum, none, red[turn]);
            turn ^= 1;
            mean = sum * inv_d;
        }
        for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
            widen8(load8<KIND, false, false>(a.x, row, col, a.D), col, a.D, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = x[i] - mean;
                if (col + i < a.D) sq = fmaf(d, d, sq);
            }
        }
        row_sum2<TPR>(sq, none, red[turn]);
        turn ^= 1;
        const float rstd = 1.0f / sqrtf(sq * inv_d + a.eps);
        if (a.stats && t == 0) a.stats[row] = float2_t{mean, rstd};
        for (int base = 0; base < a.D; base += TPR * kChunk) {     // all lanes of a group stay for the checkpoint
            const int col = base + t * kChunk;
            const Raw<KIND> raw = col < a.D ? load8<KIND, false, false>(a.x, row, col, a.D) : zero8<KIND>();
            widen8(raw, col, a.D, x);
            if (a.ckpt.codes) ckpt_store8<false>(a.ckpt, row, col, a.D, x);
            if (col >= a.D) continue;
            float g[8], b[8];
            param8(a.gamma, col, a.D, 1.0f, g);
            param8(a.beta, col, a.D, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf((x[i] - mean) * rstd, g[i], b[i]);
            store8<OF32, false>(a.y.p, a.y.ld, row, col, a.D, x);
        }
    }
}

// As the forward kernel, with blockDim.x / TPR rows at once; a thread also keeps the sums of its columns over all of its rows.  In the
// end those of the workgroup's rows are added through LDS, in their order: one partial sum a workgroup, one workgroup a CU, no atomics.
//                        8192 x 768    16384 x 1024   16384 x 2048   16384 x 4096   8192 x 8192   4096 x 16384
//   from a checkpoint     12.0  2.6      18.8  4.5      34.1  4.9      62.6  5.4      65.7  5.1      68.6  4.9
//   from the input        12.2  3.1      19.8  5.1      37.5  5.4      72.6  5.5      74.4  5.4      78.4  5.1
//   checkpoint, dx alone   9.8  3.2      16.5  5.1      32.6  5.2      60.0  5.6      63.6  5.3      64.3  5.2
// Binary32 from the input 16384 x 1024 54.2, 3.7, 8192 x 4096 104, 3.9, 4096 x 16384 160, 5.0: with 128 registers a thread, as 1024 threads leave it, these forms (V = 2, binary32
// arrays) keep up to 28 of a thread's numbers in scratch memory; from a checkpoint 36.5, 4.1, 60.7, 5.0, 120, 5.1.
template <int KIND, bool GF32, bool OF32, bool STREAM, int TPR, int V>
__global__ __launch_bounds__(TPR == 64 && V > 2 ? 512 : 1024) void norm_bwd_kernel(const NormBwdArgs a)
{
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    constexpr int CHUNKS = V * TPR;
    __shared__ float2_t red[2][16];
    extern __shared__ float all[];                  // first the weights, then the sums
    float4_t *const weight = reinterpret_cast<float4_t *>(all);      // [halves of a chunk][chunks]: not in registers, which the sums need
    const int rows = blockDim.x / TPR, slot = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * rows;
    const float inv_d = 1.0f / (float)a.D;
    float sum_g[V][8], sum_b[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_g[v][i] = sum_b[v][i] = 0.0f;
    }
    Raw<KIND> next_x[V];
    Raw<GKIND> next_g[V];
    float2_t next_st = {0.0f, 0.0f};
    const auto load = [&](int64_t row) {             // a row past the end, its statistics too, and columns past the row's: zeros, which add nothing
        const int D = row < a.N ? a.D : 0;
        next_st = D ? a.stats[row] : float2_t{0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            next_x[v] = col < D ? load8<KIND, true, STREAM>(a.x, row, col, a.D) : zero8<KIND>();
            next_g[v] = col < D ? load8<GKIND, true, STREAM>(a.dy, row, col, a.D) : zero8<GKIND>();
        }
    };
    int turn = 0;
    int64_t base = (int64_t)blockIdx.x * rows;      // of the workgroup: all of its threads stay together for the sums
    load(base + slot);
    if (slot == 0) params_to_lds<TPR, V>(a.gamma, a.D, 1.0f, weight);
    __syncthreads();
    for (; base < a.N; base += step) {
        const int64_t row = base + slot;
        if (TPR == 64 && row >= a.N) break;
        const float2_t st = next_st;
        float h[V][8];
        Raw<GKIND> dy[V];                            // widened twice: registers
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            widen8(next_x[v], (t + v * TPR) * kChunk, a.D, h[v]);
            dy[v] = settle8(next_g[v], (t + v * TPR) * kChunk, a.D);
        }
        load(row + step);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float4_t w[2] = {weight[t + v * TPR], weight[CHUNKS + t + v * TPR]};
            float g[8];
            widen(dy[v], g);
            // Past the row's end (0 - mean) r may overflow, which dy = 0 there would not cancel: h is zero.  The question costs 0.1 to 1.2 us in 21 to 71,
            // and less than a branch around it for rows that fill their threads, which spills registers.
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[v][i] = (t + v * TPR) * kChunk + i < a.D ? (h[v][i] - st.x) * st.y : 0.0f;
                sum_g[v][i] = fmaf(g[i], h[v][i], sum_g[v][i]);
                sum_b[v][i] += g[i];
                g[i] *= w[i / 4][i & 3];
                s1 += g[i];
                s2 = fmaf(g[i], h[v][i], s2);
            }
        }
        row_sum2<TPR>(s1, s2, red[turn]);
        turn ^= 1;
        const float m1 = a.layer ? s1 * inv_d : 0.0f, m2 = s2 * inv_d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D || row >= a.N) continue;
            const float4_t w[2] = {weight[t + v * TPR], weight[CHUNKS + t + v * TPR]};
            float o[8];
            widen(dy[v], o);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = st.y * (fmaf(-h[v][i], m2, o[i] * w[i / 4][i & 3]) - m1);
            store8<OF32, true>(a.dx.p, a.dx.ld, row, col, a.D, o);
        }
    }
    if (!a.part_g && !a.part_b) return;
    if (rows > 1) {
        float4_t *const both = reinterpret_cast<float4_t *>(all);      // [sums][rows at once][halves of a chunk][chunks]
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float4_t *const mine = both + slot * 2 * CHUNKS + t + v * TPR;
            mine[0] = float4_t{sum_g[v][0], sum_g[v][1], sum_g[v][2], sum_g[v][3]};
            mine[CHUNKS] = float4_t{sum_g[v][4], sum_g[v][5], sum_g[v][6], sum_g[v][7]};
            mine[rows * 2 * CHUNKS] = float4_t{sum_b[v][0], sum_b[v][1], sum_b[v][2], sum_b[v][3]};
            mine[(rows * 2 + 1) * CHUNKS] = float4_t{sum_b[v][4], sum_b[v][5], sum_b[v][6], sum_b[v][7]};
        }
        __syncthreads();
        for (int u = threadIdx.x; u < 4 * CHUNKS; u += blockDim.x) {
            const int which = u / (2 * CHUNKS), at = u % (2 * CHUNKS), col = at % CHUNKS * kChunk + at / CHUNKS * 4;
            float *const part = which ? a.part_b : a.part_g;
            if (!part || col >= a.D) continue;
            const float4_t *const from = both + which * rows * 2 * CHUNKS + at;
            float4_t s = from[0];
            for (int r = 1; r < rows; ++r) s += from[r * 2 * CHUNKS];
            float *const to = part + blockIdx.x * a.part_ld + col;
            if (col + 4 <= a.D) {
                *reinterpret_cast<f32x4_at4 *>(to) = s;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (col + i < a.D) to[i] = s[i];
            }
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D) continue;
            if (a.part_g) store8<true, true>(a.part_g, a.part_ld, blockIdx.x, col, a.D, sum_g[v]);
            if (a.part_b) store8<true, true>(a.part_b, a.part_ld, blockIdx.x, col, a.D, sum_b[v]);
        }
    }
}

// rows longer than that or shorter than a chunk: the gradient of the input by two sweeps over a row (2048 x 32768 108 us, 3.7 TB/s) ...
template <int KIND, bool GF32, bool OF32>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(const NormBwdArgs a)
{
    constexpr int TPR = 1024, GKIND = GF32 ? kF32 : kBf16;
    __shared__ float2_t red[2][TPR / 64];
    const int t = threadIdx.x;
    const float inv_d = 1.0f / (float)a.D;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const float2_t st = a.stats[row];
        float h[8], g[8], w[8];
        float s1 = 0.0f, s2 = 0.0f;
        for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
            widen8(load8<KIND, false, false>(a.x, row, col, a.D), col, a.D, h);
            widen8(load8<GKIND, false, false>(a.dy, row, col, a.D), col, a.D, g);
            param8(a.gamma, col, a.D, 1.0f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gw = g[i] * w[i];
                s1 += gw;
                if (col + i < a.D) s2 = fmaf(gw, (h[i] - st.x) * st.y, s2);
            }
        }
        row_sum2<TPR>(s1, s2, red[turn]);
        turn ^= 1;
        const float m1 = a.layer ? s1 * inv_d : 0.0f, m2 = s2 * inv_d;
        for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
            widen8(load8<KIND, false, false>(a.x, row, col, a.D), col, a.D, h);
            widen8(load8<GKIND, false, false>(a.dy, row, col, a.D), col, a.D, g);
            param8(a.gamma, col, a.D, 1.0f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = st.y * (fmaf(-((h[i] - st.x) * st.y), m2, g[i] * w[i]) - m1);
            store8<OF32, false>(a.dx.p, a.dx.ld, row, col, a.D, g);
        }
    }
}

// ... and the sums over rows by threads that own eight columns of every gridDim.y-th row (58.4 us, 4.6 TB/s)
template <int KIND, bool GF32>
__global__ __launch_bounds__(256) void norm_params_long_kernel(const NormBwdArgs a)
{
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    const int col = (blockIdx.x * 256 + threadIdx.x) * kChunk;
    if (col >= a.D) return;
    float sum_g[8] = {}, sum_b[8] = {};
    for (int64_t row = blockIdx.y; row < a.N; row += gridDim.y) {
        const float2_t st = a.stats[row];
        float h[8], g[8];
        widen8(load8<KIND, false, false>(a.x, row, col, a.D), col, a.D, h);
        widen8(load8<GKIND, false, false>(a.dy, row, col, a.D), col, a.D, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum_g[i] = fmaf(g[i], (h[i] - st.x) * st.y, sum_g[i]);
            sum_b[i] += g[i];
        }
    }
    if (a.part_g) store8<true, false>(a.part_g, a.part_ld, blockIdx.y, col, a.D, sum_g);
    if (a.part_b) store8<true, false>(a.part_b, a.part_ld, blockIdx.y, col, a.D, sum_b);
}

// The partial sums of G <= 256 workgroups, in an order of their own: a workgroup takes 32 columns (a cache line), four neighbouring ones a thread; of
// the 32 threads of a column each adds every 32nd partial sum (all of its loads are on their way at once), then eight lanes the threads' sums.
// 256 partial sums of D = 1024 3.9 us, of which the launch and one trip to memory are all but 0.5; 16384 6.9, 32768 13.0.
constexpr int kMostPartials = 256;
__global__ __launch_bounds__(256) void norm_params_reduce_kernel(const float *part_g, const float *part_b, int64_t part_ld, int G, int D, float *dgamma, float *dbeta)
{
    __shared__ float4_t red[32][8];
    const int quad = threadIdx.x & 7, first = threadIdx.x >> 3;
    const int c = blockIdx.x * 32 + quad * 4;
    const float *const part = blockIdx.y ? part_b : part_g;
    float *const out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    // Threads without a partial sum, or without columns, load another's: under a condition the loads would be waited for one by one.
    float4_t v[kMostPartials / 32];
    const int at = c < D ? c : 0;
    if (G > 0) {
#pragma unroll
        for (int i = 0; i < kMostPartials / 32; ++i) {
            const int g = first + 32 * i;
            v[i] = *reinterpret_cast<const float4_t *>(part + (g < G ? g : G - 1) * part_ld + at);      // rows are padded to whole quads
        }
    }
#pragma unroll
    for (int i = 0; i < kMostPartials / 32; ++i)
        if (first + 32 * i >= G) v[i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 1; i < kMostPartials / 32; ++i) v[0] += v[i];
    red[first][quad] = v[0];
    __syncthreads();
    const int lane = threadIdx.x & 7, column = threadIdx.x >> 3;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s += red[lane + 8 * i][column >> 2][column & 3];
    s += u2f(dpp<DPP_QUAD_XOR1>(f2u(s)));
    s += u2f(dpp<DPP_QUAD_XOR2>(f2u(s)));
    s += u2f(dpp<DPP_ROW_HALF_MIRROR>(f2u(s)));
    if (lane == 0 && blockIdx.x * 32 + column < D) out[blockIdx.x * 32 + column] = s;
}

constexpr int kMaxHeldRow = 16384;      // longest row that a workgroup's registers hold
constexpr int kLongBlocks = 8192;       // most workgroups where a row is longer

bool held(int64_t D) { return D >= kChunk && D <= kMaxHeldRow; }
// Threads that hold a row.  A wave as long as its registers last: no barrier, and no wave of a workgroup without columns.  us, a wave / 256 threads: with a checkpoint
// forward 12000 x 1280 17.3 / 22.5, 16384 x 2048 28.7 / 30.2, 1000 x 2048 6.2 / 5.8, 4 x 1280 3.8 / 3.5; backward 19.1 / 24.4, 33.7 / 38.8, 8.7 / 7.4, 4.6 / 3.6.  Few rows
// keep the wave all the same, so that what a row gives does not depend on the rows around it.
int threads_of_row(int64_t D) { return D <= 2048 ? 64 : D <= 4096 ? 256 : D <= 8192 ? 512 : 1024; }

// rows that a workgroup of the backward kernel takes at once, as many as give every CU a workgroup and at most 1024 threads (512 where a wave holds over
// 1024 elements, for the registers), and its workgroups: each leaves a partial sum of D columns, so there is one a CU
int64_t bwd_rows(int64_t N, int64_t D)
{
    const int64_t most = !held(D) ? 1 : D > 1024 && D <= 2048 ? 8 : 1024 / threads_of_row(D), want = (N + kMostPartials - 1) / kMostPartials;
    return want < 1 ? 1 : want < most ? want : most;
}
int64_t bwd_blocks(int64_t N, int64_t D)
{
    const int64_t rows = bwd_rows(N, D), want = (N + rows - 1) / rows;
    return want < kMostPartials ? want : kMostPartials;
}

template <int KIND, bool OF32, int TPR, int V> void run_norm_fwd(const NormFwdArgs &a, hipStream_t st)
{
    constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
    // 16 waves a CU, which then walk over their rows; with half the registers twice as many are there at once, and two rounds are faster still
    // (32768 x 512 17.3 us with 16 waves a CU, 16.2 with 64; 16384 x 1024, which has the registers for 20, 15.2, 16.9)
    constexpr int MOST = 256 * (1024 / THREADS) * (V == 1 ? 4 : 1);
    const int64_t want = (a.N + ROWS - 1) / ROWS;
    norm_fwd_kernel<KIND, OF32, TPR, V><<<(unsigned)(want < MOST ? want : MOST), THREADS, 0, st>>>(a);
}

template <int KIND, bool OF32> void run_norm_fwd(const NormFwdArgs &a, hipStream_t st)
{
    if (!held(a.D)) norm_fwd_long_kernel<KIND, OF32><<<(unsigned)(a.N < kLongBlocks ? a.N : kLongBlocks), 1024, 0, st>>>(a);
    else if (a.D <= 512) run_norm_fwd<KIND, OF32, 64, 1>(a, st);
    else if (a.D <= 1024) run_norm_fwd<KIND, OF32, 64, 2>(a, st);
    else if (a.D <= 1536) run_norm_fwd<KIND, OF32, 64, 3>(a, st);
    else if (a.D <= 2048) run_norm_fwd<KIND, OF32, 64, 4>(a, st);
    else if (a.D <= 4096) run_norm_fwd<KIND, OF32, 256, 2>(a, st);
    else if (a.D <= 8192) run_norm_fwd<KIND, OF32, 512, 2>(a, st);
    else run_norm_fwd<KIND, OF32, 1024, 2>(a, st);
}

template <int KIND, bool GF32, bool OF32, int TPR, int V> void run_norm_bwd(const NormBwdArgs &a, unsigned blocks, hipStream_t st)
{
    const unsigned rows = (unsigned)bwd_rows(a.N, a.D);
    const size_t weights = (size_t)V * TPR * kChunk, sums = rows > 1 && (a.part_g || a.part_b) ? 2 * rows * weights : 0;
    const size_t lds = (weights > sums ? weights : sums) * sizeof(float);
    const double each = (GF32 ? 4 : 2) + (KIND == kF32 ? 4 : KIND == kBf16 ? 2 : 1) + (OF32 ? 4 : 2);
    // From a checkpoint past the caches from half that size on, us of a forward and a backward pass, through / past: 16384 x 1024 (80 MB) 38.0 / 35.2, 4096 x 4096 40.0 / 37.7,
    // 20000 x 768 38.3 / 36.1, 16384 x 768 (60 MB) 30.5 / 30.3; not so from the input: 16384 x 1024 (96 MB) 33.8 / 34.5, 20000 x 768 32.5 / 34.5
    if (streams((double)a.N * a.D * each * (KIND == kCkpt8 ? 2 : 1))) norm_bwd_kernel<KIND, GF32, OF32, true, TPR, V><<<blocks, rows * TPR, lds, st>>>(a);
    else norm_bwd_kernel<KIND, GF32, OF32, false, TPR, V><<<blocks, rows * TPR, lds, st>>>(a);
}

template <int KIND, bool GF32, bool OF32> void run_norm_bwd(const NormBwdArgs &a, unsigned blocks, hipStream_t st)
{
    if (!held(a.D)) {
        norm_bwd_long_kernel<KIND, GF32, OF32><<<(unsigned)(a.N < kLongBlocks ? a.N : kLongBlocks), 1024, 0, st>>>(a);
        if (a.part_g || a.part_b)
            norm_params_long_kernel<KIND, GF32><<<dim3((unsigned)((a.D + 2047) / 2048), blocks), 256, 0, st>>>(a);
    }
    else if (a.D <= 512) run_norm_bwd<KIND, GF32, OF32, 64, 1>(a, blocks, st);
    else if (a.D <= 1024) run_norm_bwd<KIND, GF32, OF32, 64, 2>(a, blocks, st);
    else if (a.D <= 1536) run_norm_bwd<KIND, GF32, OF32, 64, 3>(a, blocks, st);
    else if (a.D <= 2048) run_norm_bwd<KIND, GF32, OF32, 64, 4>(a, blocks, st);
    else if (a.D <= 4096) run_norm_bwd<KIND, GF32, OF32, 256, 2>(a, blocks, st);
    else if (a.D <= 8192) run_norm_bwd<KIND, GF32, OF32, 512, 2>(a, blocks, st);
    else run_norm_bwd<KIND, GF32, OF32, 1024, 2>(a, blocks, st);
}

}  // namespace

hipError_t launch_norm_fwd(const RowSrc &x, int64_t N, int64_t D, const float *gamma, const float *beta, float eps, int layer, const RowDst &y,
                           float *stats, const CkptOut &ckpt, hipStream_t st)
{
    const NormFwdArgs a{x, N, (int)D, gamma, beta, eps, layer, y, reinterpret_cast<float2_t *>(stats), ckpt};
    if (x.kind == kF32) y.f32 ? run_norm_fwd<kF32, true>(a, st) : run_norm_fwd<kF32, false>(a, st);
    else y.f32 ? run_norm_fwd<kBf16, true>(a, st) : run_norm_fwd<kBf16, false>(a, st);
    return hipGetLastError();
}

// columns of a row of partial sums: whole quads, on 16 bytes (D = 1023: 8.9 us of the kernel that adds them without)
static int64_t padded(int64_t D) { return (D + 3) / 4 * 4; }

// for the most workgroups that N rows have at any width: their number itself falls where a workgroup takes another row (D = 1024: 256 of one row at
// N = 256, 129 of two at N = 257), and what a large call needs has to do for a small one
size_t norm_bwd_workspace_bytes(int64_t N, int64_t D)
{
    const int64_t most = N < kMostPartials ? N : kMostPartials;
    return most > 1 ? (size_t)(most * 2 * padded(D)) * sizeof(float) : 0;
}

hipError_t launch_norm_bwd(const RowSrc &dy, const RowSrc &x, const float *stats, const float *gamma, int64_t N, int64_t D, int layer,
                           const RowDst &dx, float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    const int64_t G = bwd_blocks(N, D);
    const dim3 params((unsigned)((D + 31) / 32), dbeta ? 2 : 1);
    if (N == 0) {                        // sums over no rows
        if (dgamma || dbeta) norm_params_reduce_kernel<<<params, 256, 0, st>>>(nullptr, nullptr, 0, 0, (int)D, dgamma, dbeta);
        return hipGetLastError();
    }
    NormBwdArgs a{dy, x, reinterpret_cast<const float2_t *>(stats), gamma, N, (int)D, layer, dx, dgamma, dbeta, 0};
    if (G > 1) {
        float *const part = static_cast<float *>(ws);
        a.part_g = dgamma ? part : nullptr;
        a.part_b = dbeta ? part + padded(D) : nullptr;
        a.part_ld = 2 * padded(D);
    }
    const unsigned b = (unsigned)G;
    auto by_out = [&](auto kind, auto gf32) {
        constexpr int K = decltype(kind)::value;
        constexpr bool GF = decltype(gf32)::value;
        dx.f32 ? run_norm_bwd<K, GF, true>(a, b, st) : run_norm_bwd<K, GF, false>(a, b, st);
    };
    auto by_dy = [&](auto kind) {
        dy.kind == kF32 ? by_out(kind, std::true_type{}) : by_out(kind, std::false_type{});
    };
    if (x.kind == kCkpt8) by_dy(std::integral_constant<int, kCkpt8>{});
    else if (x.kind == kF32) by_dy(std::integral_constant<int, kF32>{});
    else by_dy(std::integral_constant<int, kBf16>{});
    if (G > 1 && (dgamma || dbeta))
        norm_params_reduce_kernel<<<params, 256, 0, st>>>(a.part_g, a.part_b, a.part_ld, (int)G, (int)D, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace tj
