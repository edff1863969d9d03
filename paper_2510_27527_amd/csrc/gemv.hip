// Products of packed weights with the bf16 activations of a few tokens: Y[M x C] = X[M x K] * W[C x K]^T, W in NVFP4.
//
//   y(m, c) = sum over k of x(m, k) * E2M1(code(c, k)) * E4M3(scale(c, k / 16)) * gscale
//
// E2M1 * E4M3 has six significant bits and is exact in bf16, so the weights go to the matrix cores as bf16 next to the activations as they
// are: every product is exact and the sums are binary32.  Bound: reading the weights, 0.5625 B each.
#include "device_fmt.h"
#include "block_ops.h"

namespace tj {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at8 __attribute__((ext_vector_type(4), aligned(8)));     // codes of a row whose length is a multiple of 16
typedef uint32_t u32x2_at8 __attribute__((ext_vector_type(2), aligned(8)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));     // eight bf16 that start at any bf16

struct GemvArgs {
    const uint16_t *x;
    int64_t ldx, M;
    const uint8_t *codes, *scales;
    const float *gscale;
    int64_t C;
    int K;
    void *y;
    int64_t ldy;
    int f32;
};

// eight codes of one scale -> eight bf16 (element 2j in the low half of dword j)
__device__ __forceinline__ u32x4 weights8(uint32_t codes, float scale)
{
    u32x4 r;
    const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0);
    const float2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    const float2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2);
    const float2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    const auto pack = [&](float2_t v) { return __builtin_amdgcn_perm(f2u(v.y * scale), f2u(v.x * scale), 0x07060302u); };   // exact: the low halves are zero
    r[0] = pack(a);
    r[1] = pack(b);
    r[2] = pack(c);
    r[3] = pack(d);
    return r;
}

// A workgroup computes 16 outputs (rows of W) of up to 16 NT tokens; its four waves split the reduction in turns of 128 k and join their sums
// through LDS.  A lane holds 32 consecutive k of one row and of one token per block of 128; with outer blocks the sum over a block is
// multiplied by the row's outer scale before it joins the total.
template <int NT, bool OUTER>
__global__ __launch_bounds__(256) void gemv_kernel(const GemvArgs a)
{
    __shared__ float4_t red[4][NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, q = lane >> 4;
    const int64_t c0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * NT);
    const int64_t row = c0 + r < a.C ? c0 + r : a.C - 1;                     // rows and tokens past the end repeat the last one, and are not stored
    const uint8_t *const codes = a.codes + row * (a.K / 2), *const scales = a.scales + row * (a.K / 16);
    const uint16_t *x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t m = m0 + 16 * n + r;
        x[n] = a.x + (m < a.M ? m : a.M - 1) * a.ldx;
    }
    float4_t acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = wave * 128; k0 < a.K; k0 += 4 * 128) {
        const int k = k0 + 32 * q;
        u32x4 w = {0, 0, 0, 0};
        float s0 = 0.0f, s1 = 0.0f;
        if (k + 32 <= a.K) {
            w = *reinterpret_cast<const u32x4_at8 *>(codes + k / 2);
            s0 = e4m3_value(scales[k / 16]);
            s1 = e4m3_value(scales[k / 16 + 1]);
        } else if (k < a.K) {
            const u32x2_at8 h = *reinterpret_cast<const u32x2_at8 *>(codes + k / 2);
            w[0] = h[0];
            w[1] = h[1];
            s0 = e4m3_value(scales[k / 16]);
        }
        float4_t block[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) block[n] = OUTER ? float4_t{0.0f, 0.0f, 0.0f, 0.0f} : acc[n];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x4 wj = weights8(w[j], j < 2 ? s0 : s1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                u32x4 xj = {0, 0, 0, 0};
                if (k + 8 * j < a.K) xj = *reinterpret_cast<const u32x4_at2 *>(x[n] + k + 8 * j);
                block[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wj), __builtin_bit_cast(bf16x8_t, xj), block[n], 0, 0, 0);
            }
        }
        if constexpr (OUTER) {
            float4_t g;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t c = c0 + 4 * q + i;
                g[i] = a.gscale[(c < a.C ? c : a.C - 1) * (a.K / 128) + k0 / 128];
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = fmaf(block[n][i], g[i], acc[n][i]);
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] = block[n];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) red[wave][n][lane] = acc[n];
    __syncthreads();
    const float g = OUTER || a.K == 0 ? 1.0f : a.gscale[0];
    for (int n = wave; n < NT; n += 4) {
        float4_t s = red[0][n][lane];
#pragma unroll
        for (int i = 1; i < 4; ++i) s += red[i][n][lane];
        const int64_t m = m0 + 16 * n + r, c = c0 + 4 * q;                  // lane: token m, outputs c .. c + 3
        if (m >= a.M) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < a.C) {
                if (a.f32) static_cast<float *>(a.y)[m * a.ldy + c + i] = s[i] * g;
                else static_cast<__bf16 *>(a.y)[m * a.ldy + c + i] = (__bf16)(s[i] * g);
            }
    }
}

template <int NT> void run_gemv(const GemvArgs &a, int outer, hipStream_t st)
{
    const int64_t tiles = (a.M + 16 * NT - 1) / (16 * NT);
    const dim3 grid((unsigned)((a.C + 15) / 16), (unsigned)tiles);
    if (outer) gemv_kernel<NT, true><<<grid, 256, 0, st>>>(a);
    else gemv_kernel<NT, false><<<grid, 256, 0, st>>>(a);
}

}  // namespace

hipError_t launch_gemv(const void *X, int64_t ldx, int64_t M, const GemmOperand &W, int64_t K, const RowDst &y, hipStream_t st)
{
    const GemvArgs a{static_cast<const uint16_t *>(X), ldx, M, W.codes, W.scales, W.gscale, W.rows, (int)K, y.p, y.ld, y.f32};
    if (M <= 16) run_gemv<1>(a, W.outer, st);
    else if (M <= 32) run_gemv<2>(a, W.outer, st);
    else run_gemv<4>(a, W.outer, st);
    return hipGetLastError();
}

}  // namespace tj
