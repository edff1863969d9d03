// The nonlinearity between the linears of an MLP, forward and backward, and 8-bit checkpoints by themselves.
//
//   SwiGLU  a = g s(g) u         dg = da u s(g) (1 + g s(-g)),  du = da g s(g)        gate g, up u: the halves of a row of H
//   GELU    a = x s(z(x))        dx = da (s(z) + x s(z) s(-z) z'(x)),  z = 2 sqrt(2 / pi) (x + 0.044715 x^3)   (the tanh form)
//   with s(z) = 1 / (1 + exp(-z)); s(-z) comes from the same exponential, without the cancellation of 1 - s(z).
//
// Element by element but for the maxima of a checkpoint's groups, which the 16 lanes of a group exchange in registers.  Bound: HBM.
#include "rowwise.h"

namespace tj {

namespace {

constexpr int kSwiglu = 0, kGelu = 1;
constexpr int kThreads = 256;
constexpr int kMaxBlocks = 1 << 16;     // workgroups of a launch; beyond that each walks over several runs of chunks

// the chunks of all rows in one sequence, each row padded to whole groups
struct Chunks {
    int64_t rows;
    int64_t per_row;                     // a multiple of 16
    int64_t cols;
};

struct ActArgs {
    RowSrc da, h;
    Chunks n;                            // of the output of the forward pass: cols = F
    RowDst out;
    CkptOut ckpt;                        // of [N x F] (GELU) or [2 N x F] (SwiGLU: row 2n the gate, 2n + 1 the up part of token n)
};

struct CopyArgs {
    RowSrc src;
    Chunks n;
    RowDst out;
    CkptOut ckpt;
};

struct Sigmoid { float pos, neg; };      // s(z) and s(-z)
__device__ __forceinline__ Sigmoid sigmoid(float z)
{
    const float e = __expf(-fabsf(z));   // never overflows
    const float r = 1.0f / (1.0f + e), q = e * r;
    return z >= 0.0f ? Sigmoid{r, q} : Sigmoid{q, r};
}

constexpr float kGeluC = 1.5957691216057308f, kGeluA = 0.044715f;
// beyond |x| = 16 both s(z) and x s(z) s(-z) z'(x) have reached their limits in binary32, and x^3 overflows far out; a NaN stays
__device__ __forceinline__ float gelu_in(float x) { return x > 16.0f ? 16.0f : x < -16.0f ? -16.0f : x; }
__device__ __forceinline__ float gelu_z(float c) { return kGeluC * fmaf(kGeluA * c * c, c, c); }

// f(row, column) for every chunk of the launch; the lanes of a group come together, those past the end of a row with col >= cols
template <typename F>
__device__ __forceinline__ void for_chunks(const Chunks &n, const F &f)
{
    const int64_t total = n.rows * n.per_row;
    for (int64_t base = (int64_t)blockIdx.x * kThreads; base < total; base += (int64_t)gridDim.x * kThreads) {
        const int64_t row0 = base / n.per_row;
        const int64_t c = base - row0 * n.per_row + threadIdx.x;          // under per_row + 256
        const int64_t over = (uint64_t)c < (uint64_t)n.per_row ? 0 : (int64_t)((uint32_t)c / (uint32_t)n.per_row);
        if (row0 + over < n.rows) f(row0 + over, (c - over * n.per_row) * kChunk);   // whole groups: total and the runs are multiples of 16
    }
}

template <int KIND>
__device__ __forceinline__ Raw<KIND> load8_or_0(const RowSrc &s, int64_t row, int64_t col, int64_t n, int64_t at)
{
    return col < n ? load8<KIND>(s, row, at + col, at + n) : zero8<KIND>();
}

template <int KIND, bool OF32, int ACT>
__global__ __launch_bounds__(kThreads) void act_fwd_kernel(const ActArgs a)
{
    for_chunks(a.n, [&](int64_t row, int64_t col) {
        const int64_t F = a.n.cols;
        float x[8], o[8];
        widen8(load8_or_0<KIND>(a.h, row, col, F, 0), x);
        if constexpr (ACT == kSwiglu) {
            float u[8];
            widen8(load8_or_0<KIND>(a.h, row, col, F, F), u);
            if (a.ckpt.codes) {
                ckpt_store8(a.ckpt, 2 * row, col, F, x);
                ckpt_store8(a.ckpt, 2 * row + 1, col, F, u);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = x[i] * sigmoid(x[i]).pos * u[i];
        } else {
            if (a.ckpt.codes) ckpt_store8(a.ckpt, row, col, F, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = x[i] * sigmoid(gelu_z(gelu_in(x[i]))).pos;
        }
        if (col < F) store8<OF32>(a.out.p, a.out.ld, row, col, F, o);
    });
}

template <int KIND, bool GF32, bool OF32, int ACT>
__global__ __launch_bounds__(kThreads) void act_bwd_kernel(const ActArgs a)
{
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    for_chunks(a.n, [&](int64_t row, int64_t col) {
        const int64_t F = a.n.cols;
        if (col >= F) return;
        float x[8], da[8];
        widen8(load8<GKIND>(a.da, row, col, F), da);
        if constexpr (ACT == kSwiglu) {
            float u[8];
            if constexpr (KIND == kCkpt8) {
                widen8(load8<KIND>(a.h, 2 * row, col, F), x);
                widen8(load8<KIND>(a.h, 2 * row + 1, col, F), u);
            } else {
                widen8(load8<KIND>(a.h, row, col, F), x);
                widen8(load8<KIND>(a.h, row, F + col, 2 * F), u);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Sigmoid s = sigmoid(x[i]);
                const float du = da[i] * x[i] * s.pos;
                x[i] = da[i] * u[i] * s.pos * fmaf(x[i], s.neg, 1.0f);
                u[i] = du;
            }
            store8<OF32>(a.out.p, a.out.ld, row, col, F, x);
            store8<OF32>(static_cast<char *>(a.out.p) + F * (OF32 ? 4 : 2), a.out.ld, row, col, F, u);
        } else {
            widen8(load8<KIND>(a.h, row, col, F), x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = gelu_in(x[i]);
                const Sigmoid s = sigmoid(gelu_z(c));
                const float slope = kGeluC * fmaf(3.0f * kGeluA * c, c, 1.0f);
                x[i] = da[i] * fmaf(c * s.pos * s.neg, slope, s.pos);
            }
            store8<OF32>(a.out.p, a.out.ld, row, col, F, x);
        }
    });
}

template <int KIND>
__global__ __launch_bounds__(kThreads) void ckpt8_save_kernel(const CopyArgs a)
{
    for_chunks(a.n, [&](int64_t row, int64_t col) {
        float x[8];
        widen8(load8_or_0<KIND>(a.src, row, col, a.n.cols, 0), x);
        ckpt_store8(a.ckpt, row, col, a.n.cols, x);
    });
}

template <bool OF32>
__global__ __launch_bounds__(kThreads) void ckpt8_load_kernel(const CopyArgs a)
{
    for_chunks(a.n, [&](int64_t row, int64_t col) {
        if (col >= a.n.cols) return;
        float x[8];
        widen8(load8<kCkpt8>(a.src, row, col, a.n.cols), x);
        store8<OF32>(a.out.p, a.out.ld, row, col, a.n.cols, x);
    });
}

Chunks chunks_of(int64_t rows, int64_t cols)
{
    const int64_t groups = (cols + kCkptGroup - 1) / kCkptGroup;
    return Chunks{rows, groups * kGroupLanes, cols};
}

unsigned blocks_of(const Chunks &n)
{
    const int64_t want = (n.rows * n.per_row + kThreads - 1) / kThreads;
    return (unsigned)(want < kMaxBlocks ? want : kMaxBlocks);
}

template <int KIND, bool OF32> void run_act_fwd(const ActArgs &a, int act, hipStream_t st)
{
    if (act == kSwiglu) act_fwd_kernel<KIND, OF32, kSwiglu><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    else act_fwd_kernel<KIND, OF32, kGelu><<<blocks_of(a.n), kThreads, 0, st>>>(a);
}

template <int KIND, bool GF32, bool OF32> void run_act_bwd(const ActArgs &a, int act, hipStream_t st)
{
    if (act == kSwiglu) act_bwd_kernel<KIND, GF32, OF32, kSwiglu><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    else act_bwd_kernel<KIND, GF32, OF32, kGelu><<<blocks_of(a.n), kThreads, 0, st>>>(a);
}

template <int KIND> void run_act_bwd(const ActArgs &a, int act, hipStream_t st)
{
    if (a.da.kind == kF32) a.out.f32 ? run_act_bwd<KIND, true, true>(a, act, st) : run_act_bwd<KIND, true, false>(a, act, st);
    else a.out.f32 ? run_act_bwd<KIND, false, true>(a, act, st) : run_act_bwd<KIND, false, false>(a, act, st);
}

}  // namespace

hipError_t launch_act_fwd(const RowSrc &h, int64_t N, int64_t F, int act, const RowDst &out, const CkptOut &ckpt, hipStream_t st)
{
    const ActArgs a{RowSrc{}, h, chunks_of(N, F), out, ckpt};
    if (h.kind == kF32) out.f32 ? run_act_fwd<kF32, true>(a, act, st) : run_act_fwd<kF32, false>(a, act, st);
    else out.f32 ? run_act_fwd<kBf16, true>(a, act, st) : run_act_fwd<kBf16, false>(a, act, st);
    return hipGetLastError();
}

hipError_t launch_act_bwd(const RowSrc &da, const RowSrc &h, int64_t N, int64_t F, int act, const RowDst &out, hipStream_t st)
{
    const ActArgs a{da, h, chunks_of(N, F), out, CkptOut{}};
    if (h.kind == kCkpt8) run_act_bwd<kCkpt8>(a, act, st);
    else if (h.kind == kF32) run_act_bwd<kF32>(a, act, st);
    else run_act_bwd<kBf16>(a, act, st);
    return hipGetLastError();
}

hipError_t launch_ckpt8_save(const RowSrc &src, int64_t N, int64_t D, const CkptOut &ckpt, hipStream_t st)
{
    const CopyArgs a{src, chunks_of(N, D), RowDst{}, ckpt};
    if (src.kind == kF32) ckpt8_save_kernel<kF32><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    else ckpt8_save_kernel<kBf16><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_ckpt8_load(const RowSrc &src, int64_t N, int64_t D, const RowDst &out, hipStream_t st)
{
    const CopyArgs a{src, chunks_of(N, D), out, CkptOut{}};
    if (out.f32) ckpt8_load_kernel<true><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    else ckpt8_load_kernel<false><<<blocks_of(a.n), kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace tj
