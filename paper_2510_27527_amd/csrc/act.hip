// The nonlinearity between the linears of an MLP, forward and backward, and 8-bit checkpoints by themselves.
//
//   SwiGLU  a = g s(g) u         dg = da u s(g) (1 + g s(-g)),  du = da g s(g)        gate g, up u: the halves of a row of H
//   GELU    a = x s(z(x))        dx = da (s(z) + x s(z) s(-z) z'(x)),  z = 2 sqrt(2 / pi) (x + 0.044715 x^3)   (the tanh form)
//   with s(z) = 1 / (1 + exp(-z)); s(-z) comes from the same exponential, without the cancellation of 1 - s(z).
//
// Element by element but for the maxima of a checkpoint's groups, which the 16 lanes of a group exchange in registers.  Bound: HBM (a copy of
// 1 GB reaches 5.1 TB/s here, one of 64 MB, which the last-level cache holds, 6.9); small calls: the launch.
//
// Figures: bf16 arrays where nothing else stands, us of a kernel in a kernel trace and TB/s over the bytes that a call has to read and write; calls on three sets of arrays in turn
// (the comparisons of two forms below: on one set).
#include <type_traits>

#include "rowwise.h"

namespace tj {

namespace {

constexpr int kSwiglu = 0, kGelu = 1;
constexpr int kThreads = 256;
// Calls by the bytes that they move: large ones read past the caches (see streams()).
enum { kSmall = 0, kMiddle = 1, kLarge = 2 };
constexpr double kMiddleBytes = 8 << 20;
// Rows of a thread whose loads are on their way together: two keep more bytes in flight, one starts and ends sooner and leaves registers for more waves.
// us of one / two, bf16 source where nothing else stands:
//   SwiGLU forward with checkpoint   16384 x 4096  92 / 96      2000 x 2752  10.6 / 11.4    64 x 8192  3.9 / 4.8      always one
//   SwiGLU backward from one         16384 x 4096  81 / 90                                                            always one
//   GELU backward                    8192 x 8192   62 / 63      4099 x 2752  12.3 / 13.8    64 x 8192  3.0 / 3.6      always one
//   GELU backward, checkpoint        8192 x 8192   58 / 55      4099 x 2752  11.7 / 12.1    64 x 8192  3.1 / 3.7      two if large
//   GELU forward with checkpoint     8192 x 8192   57 / 52      4099 x 2752  11.7 / 11.5    64 x 8192  3.1 / 3.8      two from the middle on
//   checkpoint saved                 8192 x 8192   41 / 36      4099 x 2752   8.2 /  7.8    64 x 8192  2.9 / 3.3      two from the middle on
//   checkpoint loaded                8192 x 8192   42 / 38      4099 x 2752   7.9 /  7.3    64 x 8192  2.6 / 2.9      two from the middle on
constexpr int rows_fwd(int act, int size) { return act == kSwiglu || size == kSmall ? 1 : 2; }
constexpr int rows_bwd(int act, int kind, int size) { return act == kGelu && kind == kCkpt8 && size == kLarge ? 2 : 1; }
constexpr int rows_copy(int size) { return size == kSmall ? 1 : 2; }
constexpr int kMaxRowBlocks = 65535;    // of a launch's grid; beyond that a workgroup walks over several

// rows x cols in chunks of eight; a workgroup takes 2^shift chunks of 256 / 2^shift rows, whole groups of 16 chunks
struct Chunks {
    int64_t rows;
    int cols, shift;
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

// s(z) and s(-z) with w = -z log2(e); the exponential never overflows, and the two are exact to a few units in the last place however far z is out
struct Sigmoid { float pos, neg; };
__device__ __forceinline__ Sigmoid sigmoid(float w)
{
    const float e = __builtin_amdgcn_exp2f(-fabsf(w));
    const float r = __builtin_amdgcn_rcpf(1.0f + e), q = e * r;      // reciprocal: within one unit in the last place
    return w <= 0.0f ? Sigmoid{r, q} : Sigmoid{q, r};
}
// s(z) alone: an exponential that overflows gives 0
__device__ __forceinline__ float sigmoid_pos(float w) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w)); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kGeluC = 1.5957691216057308, kGeluA = 0.044715;     // z(x) = C (x + A x^3)
// -z log2(e) = x (k0 + k1 x^2)
__device__ __forceinline__ float gelu_w(float x)
{
    return x * fmaf(x * x, (float)(-kGeluC * kGeluA * 1.4426950408889634), (float)(-kGeluC * 1.4426950408889634));
}
__device__ __forceinline__ float gelu(float x) { return x * sigmoid_pos(gelu_w(x)); }
// z and its slope are taken at most at |x| = 16, beyond which s(z) s(-z) is zero in binary32 (x^2 times it would overflow far out)
__device__ __forceinline__ float gelu_slope(float x)
{
    const float c = __builtin_amdgcn_fmed3f(x, -16.0f, 16.0f);
    const Sigmoid s = sigmoid(gelu_w(c));
    return fmaf(x * (s.pos * s.neg), fmaf(c * c, (float)(3.0 * kGeluC * kGeluA), (float)kGeluC), s.pos);
}

// For every chunk of the launch use(row, column, load(row, column)), R rows of a thread loaded before the first is used.  The lanes of a
// group come together, those past the end of a row with col >= cols.
template <int R, typename Load, typename Use>
__device__ __forceinline__ void for_chunks(const Chunks &n, const Load &load, const Use &use)
{
    const int col = (int)((blockIdx.x << n.shift) | (threadIdx.x & ((1u << n.shift) - 1))) * kChunk;
    const int step = kThreads >> n.shift;                          // rows that the workgroup takes at once, R times in succession
    for (int64_t row = (int64_t)blockIdx.y * (R * step) + (threadIdx.x >> n.shift); row < n.rows; row += (int64_t)gridDim.y * (R * step)) {
        decltype(load(row, col)) in[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (row + r * step < n.rows) in[r] = load(row + r * step, col);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (row + r * step < n.rows) use(row + r * step, col, in[r]);
    }
}

// chunk of a row's part that starts at `at` and has n elements
template <int KIND, bool STREAM>
__device__ __forceinline__ Raw<KIND> load8_at(const RowSrc &s, int64_t row, int col, int n, int at)
{
    const int size = KIND == kF32 ? 4 : 2;
    return load8<KIND, false, STREAM>(RowSrc{static_cast<const char *>(s.p) + (int64_t)at * size, nullptr, s.ld, 0, s.kind}, row, col, n);
}
template <int KIND, bool STREAM>
__device__ __forceinline__ Raw<KIND> load8_or_0(const RowSrc &s, int64_t row, int col, int n, int at)
{
    return col < n ? load8_at<KIND, STREAM>(s, row, col, n, at) : zero8<KIND>();
}

template <int KIND> struct Pair { Raw<KIND> a, b; };
template <int KIND, int GKIND> struct Triple { Raw<KIND> a, b; Raw<GKIND> da; };

// SwiGLU with a checkpoint 16384 x 4096 90 us, 6.0 TB/s, without 66, 6.1; GELU with a checkpoint 4099 x 2752 11.3, 5.0, 8192 x 8192 58, 5.8; 64 x 8192 3.3.
// Binary32: SwiGLU with a checkpoint 8192 x 4096 89, 5.3, GELU 8192 x 8192 115, 5.3.
template <int KIND, bool OF32, int SIZE, int ACT>
__global__ __launch_bounds__(kThreads) void act_fwd_kernel(const ActArgs a)
{
    constexpr bool STREAM = SIZE == kLarge;
    const int F = a.n.cols;
    const auto load = [&](int64_t row, int col) {
        Pair<KIND> in;
        in.a = load8_or_0<KIND, STREAM>(a.h, row, col, F, 0);
        if constexpr (ACT == kSwiglu) in.b = load8_or_0<KIND, STREAM>(a.h, row, col, F, F);
        return in;
    };
    for_chunks<rows_fwd(ACT, SIZE)>(a.n, load, [&](int64_t row, int col, const Pair<KIND> &in) {
        float x[8], o[8];
        widen8(in.a, col, F, x);
        if constexpr (ACT == kSwiglu) {
            float u[8];
            widen8(in.b, col, F, u);
            if (a.ckpt.codes) {
                ckpt_store8<false>(a.ckpt, 2 * row, col, F, x);
                ckpt_store8<false>(a.ckpt, 2 * row + 1, col, F, u);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = x[i] * sigmoid_pos(-kLog2e * x[i]) * u[i];
        } else {
            if (a.ckpt.codes) ckpt_store8<false>(a.ckpt, row, col, F, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = gelu(x[i]);
        }
        if (col < F) store8<OF32, false>(a.out.p, a.out.ld, row, col, F, o);
    });
}

// SwiGLU 16384 x 4096 from a checkpoint 89 us, 6.1 TB/s, from H 114, 5.9; GELU from a checkpoint 4099 x 2752 11.6, 4.9, 8192 x 8192 60, 5.6, from the input 69, 5.9.
// Binary32 from a checkpoint: SwiGLU 8192 x 4096 91, 5.2, GELU 8192 x 8192 117, 5.2.
template <int KIND, bool GF32, bool OF32, int SIZE, int ACT>
__global__ __launch_bounds__(kThreads) void act_bwd_kernel(const ActArgs a)
{
    constexpr bool STREAM = SIZE == kLarge;
    constexpr int GKIND = GF32 ? kF32 : kBf16;
    using In = Triple<KIND, GKIND>;
    const int F = a.n.cols;
    const auto load = [&](int64_t row, int col) {
        In in;
        if (col >= F) return in;
        in.da = load8<GKIND, false, STREAM>(a.da, row, col, F);
        if constexpr (ACT == kGelu) {
            in.a = load8<KIND, false, STREAM>(a.h, row, col, F);
        } else if constexpr (KIND == kCkpt8) {
            in.a = load8<KIND, false, STREAM>(a.h, 2 * row, col, F);
            in.b = load8<KIND, false, STREAM>(a.h, 2 * row + 1, col, F);
        } else {
            in.a = load8<KIND, false, STREAM>(a.h, row, col, F);
            in.b = load8_at<KIND, STREAM>(a.h, row, col, F, F);
        }
        return in;
    };
    for_chunks<rows_bwd(ACT, KIND, SIZE)>(a.n, load, [&](int64_t row, int col, const In &in) {
        if (col >= F) return;
        float x[8], da[8];
        widen8(in.da, col, F, da);
        widen8(in.a, col, F, x);
        if constexpr (ACT == kSwiglu) {
            float u[8];
            widen8(in.b, col, F, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Sigmoid s = sigmoid(-kLog2e * x[i]);
                // the bounded factors first: da x and da u may overflow where s(x) makes the product small or zero
                const float du = x[i] * s.pos * da[i];
                x[i] = s.pos * fmaf(x[i], s.neg, 1.0f) * u[i] * da[i];
                u[i] = du;
            }
            store8<OF32, false>(a.out.p, a.out.ld, row, col, F, x);
            store8<OF32, false>(static_cast<char *>(a.out.p) + (int64_t)F * (OF32 ? 4 : 2), a.out.ld, row, col, F, u);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = da[i] * gelu_slope(x[i]);
            store8<OF32, false>(a.out.p, a.out.ld, row, col, F, x);
        }
    });
}

// 8192 x 8192 35 us, 5.8 TB/s; binary32 60, 5.6
template <int KIND, int SIZE>
__global__ __launch_bounds__(kThreads) void ckpt8_save_kernel(const CopyArgs a)
{
    constexpr bool STREAM = SIZE == kLarge;
    for_chunks<rows_copy(SIZE)>(a.n, [&](int64_t row, int col) { return load8_or_0<KIND, STREAM>(a.src, row, col, a.n.cols, 0); },
                      [&](int64_t row, int col, const Raw<KIND> &in) {
        float x[8];
        widen8(in, col, a.n.cols, x);
        ckpt_store8<false>(a.ckpt, row, col, a.n.cols, x);
    });
}

// 8192 x 8192 37 us, 5.5 TB/s, right after it was saved 31, 6.5; to binary32 79, 4.2
template <bool OF32, int SIZE>
__global__ __launch_bounds__(kThreads) void ckpt8_load_kernel(const CopyArgs a)
{
    constexpr bool STREAM = SIZE == kLarge;
    for_chunks<rows_copy(SIZE)>(a.n, [&](int64_t row, int col) { return col < a.n.cols ? load8<kCkpt8, false, STREAM>(a.src, row, col, a.n.cols) : zero8<kCkpt8>(); },
                      [&](int64_t row, int col, const Raw<kCkpt8> &in) {
        if (col >= a.n.cols) return;
        float x[8];
        widen8(in, col, a.n.cols, x);
        store8<OF32, false>(a.out.p, a.out.ld, row, col, a.n.cols, x);
    });
}

// As many chunks of a row as leave at most an eighth of the workgroups' threads without work (sixteen leave none but in the last group)
Chunks chunks_of(int64_t rows, int64_t cols)
{
    const int64_t per_row = (cols + kCkptGroup - 1) / kCkptGroup * kGroupLanes;
    int shift = 8;
    const auto padded = [&](int sh) { return (((per_row - 1) >> sh) + 1) << sh; };
    while (shift > 4 && padded(shift) * 8 > per_row * 9) --shift;
    return Chunks{rows, (int)cols, shift};
}

dim3 grid_of(const Chunks &n, int rows)      // of a thread
{
    const int64_t wide = (int64_t)kChunk << n.shift, tall = kThreads >> n.shift, blocks = (n.rows + rows * tall - 1) / (rows * tall);
    return dim3((unsigned)((n.cols + wide - 1) / wide), (unsigned)(blocks < kMaxRowBlocks ? blocks : kMaxRowBlocks));
}

// f(size) for a call of so many bytes per element, the size as a constant
template <typename F> void by_size(const Chunks &n, double bytes, const F &f)
{
    const double all = (double)n.rows * n.cols * bytes;
    if (streams(all)) f(std::integral_constant<int, kLarge>{});
    else if (all > kMiddleBytes) f(std::integral_constant<int, kMiddle>{});
    else f(std::integral_constant<int, kSmall>{});
}
constexpr double bytes_of(int kind) { return kind == kF32 ? 4.0 : kind == kBf16 ? 2.0 : 1.0; }

template <int KIND, bool OF32, int SIZE, int ACT> void run_act_fwd(const ActArgs &a, hipStream_t st)
{
    constexpr int R = rows_fwd(ACT, SIZE), S = R == 1 && SIZE == kMiddle ? kSmall : SIZE;     // what differs in nothing is one kernel
    act_fwd_kernel<KIND, OF32, S, ACT><<<grid_of(a.n, R), kThreads, 0, st>>>(a);
}
template <int KIND, bool OF32> void run_act_fwd(const ActArgs &a, int act, hipStream_t st)
{
    const double parts = act == kSwiglu ? 2.0 : 1.0;
    by_size(a.n, parts * (bytes_of(KIND) + (a.ckpt.codes ? 1.0 : 0.0)) + (OF32 ? 4.0 : 2.0), [&](auto size) {
        constexpr int S = decltype(size)::value;
        act == kSwiglu ? run_act_fwd<KIND, OF32, S, kSwiglu>(a, st) : run_act_fwd<KIND, OF32, S, kGelu>(a, st);
    });
}

template <int KIND, bool GF32, bool OF32, int SIZE, int ACT> void run_act_bwd(const ActArgs &a, hipStream_t st)
{
    constexpr int S = SIZE == kMiddle ? kSmall : SIZE;
    act_bwd_kernel<KIND, GF32, OF32, S, ACT><<<grid_of(a.n, rows_bwd(ACT, KIND, S)), kThreads, 0, st>>>(a);
}
template <int KIND, bool GF32, bool OF32> void run_act_bwd(const ActArgs &a, int act, hipStream_t st)
{
    const double parts = act == kSwiglu ? 2.0 : 1.0;
    by_size(a.n, parts * (bytes_of(KIND) + (OF32 ? 4.0 : 2.0)) + (GF32 ? 4.0 : 2.0), [&](auto size) {
        constexpr int S = decltype(size)::value;
        act == kSwiglu ? run_act_bwd<KIND, GF32, OF32, S, kSwiglu>(a, st) : run_act_bwd<KIND, GF32, OF32, S, kGelu>(a, st);
    });
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
    by_size(a.n, bytes_of(src.kind) + 1.0, [&](auto size) {
        constexpr int S = decltype(size)::value;
        if (src.kind == kF32) ckpt8_save_kernel<kF32, S><<<grid_of(a.n, rows_copy(S)), kThreads, 0, st>>>(a);
        else ckpt8_save_kernel<kBf16, S><<<grid_of(a.n, rows_copy(S)), kThreads, 0, st>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_ckpt8_load(const RowSrc &src, int64_t N, int64_t D, const RowDst &out, hipStream_t st)
{
    const CopyArgs a{src, chunks_of(N, D), out, CkptOut{}};
    by_size(a.n, 1.0 + (out.f32 ? 4.0 : 2.0), [&](auto size) {
        constexpr int S = decltype(size)::value;
        if (out.f32) ckpt8_load_kernel<true, S><<<grid_of(a.n, rows_copy(S)), kThreads, 0, st>>>(a);
        else ckpt8_load_kernel<false, S><<<grid_of(a.n, rows_copy(S)), kThreads, 0, st>>>(a);
    });
    return hipGetLastError();
}

}  // namespace tj
