// Layer norm and RMS norm of the rows of an [N x D] array, forward and backward.
//
//   forward    mu = sum x / D (RMS norm: 0), r = 1 / sqrt(sum (x - mu)^2 / D + eps), y = (x - mu) r gamma + beta
//   backward   h = (x - mu) r, g = dy gamma:  dx = r (g - mean(g) - h mean(g h))  (RMS norm: without mean(g)),
//              dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// A row is read once and stays in the registers of the TPR threads that hold it (a wave, or a workgroup for longer rows), so
// that the variance is taken about the mean without a second read.  All sums are binary32.  Bound: HBM.
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

constexpr int rows_at_once(int TPR) { return TPR == 64 ? 4 : 1; }

template <int KIND, bool OF32, int TPR, int V>
__global__ __launch_bounds__(TPR *rows_at_once(TPR)) void norm_fwd_kernel(const NormFwdArgs a)
{
    constexpr int ROWS = rows_at_once(TPR);
    __shared__ float red[2][2 * (TPR / 64)];
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inv_d = 1.0f / (float)a.D;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < a.N; row += step) {
        float x[V][8];
        float sum = 0.0f, none = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            const Raw<KIND> raw = col < a.D ? load8<KIND>(a.x, row, col, a.D) : zero8<KIND>();
            widen8(raw, x[v]);
        }
        if (a.ckpt.codes) {
#pragma unroll
            for (int v = 0; v < V; ++v) ckpt_store8(a.ckpt, row, (t + v * TPR) * kChunk, a.D, x[v]);
        }
        float mean = 0.0f;
        if (a.layer) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[v][i];
            row_sum2<TPR>(sum, none, red[0]);
            mean = sum * inv_d;
        }
        float sq = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = x[v][i] - mean;
                if ((t + v * TPR) * kChunk + i < a.D) sq = fmaf(d, d, sq);
            }
        row_sum2<TPR>(sq, none, red[1]);
        const float rstd = 1.0f / sqrtf(sq * inv_d + a.eps);
        if (a.stats && t == 0) a.stats[row] = float2_t{mean, rstd};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D) continue;
            float g[8], b[8];
            param8(a.gamma, col, a.D, 1.0f, g);
            param8(a.beta, col, a.D, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] = fmaf((x[v][i] - mean) * rstd, g[i], b[i]);
            store8<OF32>(a.y.p, a.y.ld, row, col, a.D, x[v]);
        }
    }
}

// rows that no workgroup's registers hold: three sweeps over the row, the later ones from the caches
template <int KIND, bool OF32>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(const NormFwdArgs a)
{
    constexpr int TPR = 1024;
    __shared__ float red[2][2 * (TPR / 64)];
    const int t = threadIdx.x;
    const float inv_d = 1.0f / (float)a.D;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        float x[8];
        float none = 0.0f, mean = 0.0f, sq = 0.0f;
        if (a.layer) {
            float sum = 0.0f;
            for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
                widen8(load8<KIND>(a.x, row, col, a.D), x);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i];
            }
            row_sum2<TPR>(sum, none, red[0]);
            mean = sum * inv_d;
        }
        for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
            widen8(load8<KIND>(a.x, row, col, a.D), x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = x[i] - mean;
                if (col + i < a.D) sq = fmaf(d, d, sq);
            }
        }
        row_sum2<TPR>(sq, none, red[1]);
        const float rstd = 1.0f / sqrtf(sq * inv_d + a.eps);
        if (a.stats && t == 0) a.stats[row] = float2_t{mean, rstd};
        for (int base = 0; base < a.D; base += TPR * kChunk) {     // all lanes of a group stay for the checkpoint
            const int col = base + t * kChunk;
            const Raw<KIND> raw = col < a.D ? load8<KIND>(a.x, row, col, a.D) : zero8<KIND>();
            widen8(raw, x);
            if (a.ckpt.codes) ckpt_store8(a.ckpt, row, col, a.D, x);
            if (col >= a.D) continue;
            float g[8], b[8];
            param8(a.gamma, col, a.D, 1.0f, g);
            param8(a.beta, col, a.D, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf((x[i] - mean) * rstd, g[i], b[i]);
            store8<OF32>(a.y.p, a.y.ld, row, col, a.D, x);
        }
    }
}

template <int KIND, bool GF32, bool OF32, int TPR, int V>
__global__ __launch_bounds__(TPR *rows_at_once(TPR)) void norm_bwd_kernel(const NormBwdArgs a)
{
    constexpr int ROWS = rows_at_once(TPR);
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    __shared__ float red[2][2 * (TPR / 64)];
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inv_d = 1.0f / (float)a.D;
    float sum_g[V][8], sum_b[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_g[v][i] = sum_b[v][i] = 0.0f;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row < a.N; row += step) {
        const float2_t st = a.stats[row];
        float h[V][8], g[V][8];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            const Raw<KIND> rx = col < a.D ? load8<KIND>(a.x, row, col, a.D) : zero8<KIND>();
            const Raw<GKIND> rg = col < a.D ? load8<GKIND>(a.dy, row, col, a.D) : zero8<GKIND>();
            widen8(rx, h[v]);
            widen8(rg, g[v]);
            float w[8];
            param8(a.gamma, col, a.D, 1.0f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[v][i] = (h[v][i] - st.x) * st.y;
                if (col + i >= a.D) h[v][i] = 0.0f;
                sum_g[v][i] = fmaf(g[v][i], h[v][i], sum_g[v][i]);
                sum_b[v][i] += g[v][i];
                g[v][i] *= w[i];
                s1 += g[v][i];
                s2 = fmaf(g[v][i], h[v][i], s2);
            }
        }
        row_sum2<TPR>(s1, s2, red[turn]);
        turn ^= 1;
        const float m1 = a.layer ? s1 * inv_d : 0.0f, m2 = s2 * inv_d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = st.y * (fmaf(-h[v][i], m2, g[v][i]) - m1);
            store8<OF32>(a.dx.p, a.dx.ld, row, col, a.D, o);
        }
    }
    if (!a.part_g && !a.part_b) return;
    if constexpr (ROWS > 1) {      // the waves' sums, in the order of the waves
        __shared__ float all[ROWS][V * TPR * kChunk];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float *const part = which ? a.part_b : a.part_g;
            if (which) __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) all[threadIdx.x / TPR][(t + v * TPR) * kChunk + i] = which ? sum_b[v][i] : sum_g[v][i];
            __syncthreads();
            if (part)
                for (int c = threadIdx.x; c < a.D; c += TPR * ROWS) {
                    float s = all[0][c];
#pragma unroll
                    for (int r = 1; r < ROWS; ++r) s += all[r][c];
                    part[blockIdx.x * a.part_ld + c] = s;
                }
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (t + v * TPR) * kChunk;
            if (col >= a.D) continue;
            if (a.part_g) store8<true>(a.part_g, a.part_ld, blockIdx.x, col, a.D, sum_g[v]);
            if (a.part_b) store8<true>(a.part_b, a.part_ld, blockIdx.x, col, a.D, sum_b[v]);
        }
    }
}

// longer rows: the gradient of the input by two sweeps over a row ...
template <int KIND, bool GF32, bool OF32>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(const NormBwdArgs a)
{
    constexpr int TPR = 1024, GKIND = GF32 ? kF32 : kBf16;
    __shared__ float red[2][2 * (TPR / 64)];
    const int t = threadIdx.x;
    const float inv_d = 1.0f / (float)a.D;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const float2_t st = a.stats[row];
        float h[8], g[8], w[8];
        float s1 = 0.0f, s2 = 0.0f;
        for (int col = t * kChunk; col < a.D; col += TPR * kChunk) {
            widen8(load8<KIND>(a.x, row, col, a.D), h);
            widen8(load8<GKIND>(a.dy, row, col, a.D), g);
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
            widen8(load8<KIND>(a.x, row, col, a.D), h);
            widen8(load8<GKIND>(a.dy, row, col, a.D), g);
            param8(a.gamma, col, a.D, 1.0f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = st.y * (fmaf(-((h[i] - st.x) * st.y), m2, g[i] * w[i]) - m1);
            store8<OF32>(a.dx.p, a.dx.ld, row, col, a.D, g);
        }
    }
}

// ... and the sums over rows by threads that own eight columns of every gridDim.y-th row
template <int KIND, bool GF32>
__global__ __launch_bounds__(256) void norm_params_long_kernel(const NormBwdArgs a)
{
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kChunk;
    if (col >= a.D) return;
    float sum_g[8] = {}, sum_b[8] = {};
    for (int64_t row = blockIdx.y; row < a.N; row += gridDim.y) {
        const float2_t st = a.stats[row];
        float h[8], g[8];
        widen8(load8<KIND>(a.x, row, col, a.D), h);
        widen8(load8<GKIND>(a.dy, row, col, a.D), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum_g[i] = fmaf(g[i], (h[i] - st.x) * st.y, sum_g[i]);
            sum_b[i] += g[i];
        }
    }
    if (a.part_g) store8<true>(a.part_g, a.part_ld, blockIdx.y, col, a.D, sum_g);
    if (a.part_b) store8<true>(a.part_b, a.part_ld, blockIdx.y, col, a.D, sum_b);
}

// The partial sums of G workgroups, in their order: a workgroup takes 64 columns, each of its 16 waves every sixteenth partial sum.
__global__ __launch_bounds__(1024) void norm_params_reduce_kernel(const float *part_g, const float *part_b, int64_t part_ld, int G, int D, float *dgamma, float *dbeta)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    const float *const part = blockIdx.y ? part_b : part_g;
    float *const out = blockIdx.y ? dbeta : dgamma;
    float s = 0.0f;
    if (out && c < D)
        for (int g = w; g < G; g += 16) s += part[g * part_ld + c];
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && out && c < D) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += red[i][lane];
        out[c] = s;
    }
}

constexpr int kMaxHeldRow = 16384;      // longest row that a workgroup's registers hold
constexpr int kFwdBlocks = 8192;        // most workgroups of a forward launch
constexpr int kBwdBlocks = 512;         // most workgroups, and partial sums, of a backward launch

int64_t bwd_blocks(int64_t N, int64_t D)
{
    const int64_t rows = D <= 1024 ? 4 : 1;
    const int64_t want = (N + rows - 1) / rows;
    const int64_t most = D <= 8192 ? kBwdBlocks : kBwdBlocks / 2;
    return want < most ? want : most;
}

template <int KIND, bool OF32> void run_norm_fwd(const NormFwdArgs &a, hipStream_t st)
{
    const int64_t want4 = (a.N + 3) / 4;
    const unsigned waves = (unsigned)(want4 < kFwdBlocks ? want4 : kFwdBlocks), rows = (unsigned)(a.N < kFwdBlocks ? a.N : kFwdBlocks);
    if (a.D <= 512) norm_fwd_kernel<KIND, OF32, 64, 1><<<waves, 256, 0, st>>>(a);
    else if (a.D <= 1024) norm_fwd_kernel<KIND, OF32, 64, 2><<<waves, 256, 0, st>>>(a);
    else if (a.D <= 2048) norm_fwd_kernel<KIND, OF32, 64, 4><<<waves, 256, 0, st>>>(a);
    else if (a.D <= 4096) norm_fwd_kernel<KIND, OF32, 256, 2><<<rows, 256, 0, st>>>(a);
    else if (a.D <= 8192) norm_fwd_kernel<KIND, OF32, 256, 4><<<rows, 256, 0, st>>>(a);
    else if (a.D <= kMaxHeldRow) norm_fwd_kernel<KIND, OF32, 1024, 2><<<rows, 1024, 0, st>>>(a);
    else norm_fwd_long_kernel<KIND, OF32><<<rows, 1024, 0, st>>>(a);
}

template <int KIND, bool GF32, bool OF32> void run_norm_bwd(const NormBwdArgs &a, unsigned blocks, hipStream_t st)
{
    if (a.D <= 512) norm_bwd_kernel<KIND, GF32, OF32, 64, 1><<<blocks, 256, 0, st>>>(a);
    else if (a.D <= 1024) norm_bwd_kernel<KIND, GF32, OF32, 64, 2><<<blocks, 256, 0, st>>>(a);
    else if (a.D <= 2048) norm_bwd_kernel<KIND, GF32, OF32, 256, 1><<<blocks, 256, 0, st>>>(a);
    else if (a.D <= 4096) norm_bwd_kernel<KIND, GF32, OF32, 256, 2><<<blocks, 256, 0, st>>>(a);
    else if (a.D <= 8192) norm_bwd_kernel<KIND, GF32, OF32, 256, 4><<<blocks, 256, 0, st>>>(a);
    else if (a.D <= kMaxHeldRow) norm_bwd_kernel<KIND, GF32, OF32, 1024, 2><<<blocks, 1024, 0, st>>>(a);
    else {
        norm_bwd_long_kernel<KIND, GF32, OF32><<<(unsigned)(a.N < kFwdBlocks ? a.N : kFwdBlocks), 1024, 0, st>>>(a);
        if (a.part_g || a.part_b)
            norm_params_long_kernel<KIND, GF32><<<dim3((unsigned)((a.D + 2047) / 2048), blocks), 256, 0, st>>>(a);
    }
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

size_t norm_bwd_workspace_bytes(int64_t N, int64_t D)
{
    const int64_t G = bwd_blocks(N, D);
    return G > 1 ? (size_t)(G * 2 * D) * sizeof(float) : 0;
}

hipError_t launch_norm_bwd(const RowSrc &dy, const RowSrc &x, const float *stats, const float *gamma, int64_t N, int64_t D, int layer,
                           const RowDst &dx, float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    const int64_t G = bwd_blocks(N, D);
    const dim3 params((unsigned)((D + 63) / 64), dbeta ? 2 : 1);
    if (N == 0) {                        // sums over no rows
        if (dgamma || dbeta) norm_params_reduce_kernel<<<params, 1024, 0, st>>>(nullptr, nullptr, 0, 0, (int)D, dgamma, dbeta);
        return hipGetLastError();
    }
    NormBwdArgs a{dy, x, reinterpret_cast<const float2_t *>(stats), gamma, N, (int)D, layer, dx, dgamma, dbeta, 0};
    if (G > 1) {
        float *const part = static_cast<float *>(ws);
        a.part_g = dgamma ? part : nullptr;
        a.part_b = dbeta ? part + D : nullptr;
        a.part_ld = 2 * D;
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
        norm_params_reduce_kernel<<<params, 1024, 0, st>>>(a.part_g, a.part_b, a.part_ld, (int)G, (int)D, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace tj
