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

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t uint32_at1 __attribute__((aligned(1)));
typedef uint16_t uint16_at1 __attribute__((aligned(1)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at8 __attribute__((ext_vector_type(4), aligned(8)));     // codes of a row whose length is a multiple of 16
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_at1 __attribute__((ext_vector_type(2), aligned(1)));
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

// LDS accesses of one wave on either side stay in their order (the hardware keeps it; this binds the compiler)
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// one E4M3 byte of a pair
template <int SEL> __device__ __forceinline__ float scale_of(uint32_t pair) { return __builtin_amdgcn_cvt_f32_fp8((int)pair, SEL); }

// sum of v over the LR neighbouring lanes of a row, in every one of them
template <int LR> __device__ __forceinline__ float lanes_sum(float v)
{
    v += u2f(dpp<DPP_QUAD_XOR1>(f2u(v)));
    v += u2f(dpp<DPP_QUAD_XOR2>(f2u(v)));
    v += u2f(dpp<DPP_ROW_HALF_MIRROR>(f2u(v)));
    v += u2f(dpp<DPP_ROW_MIRROR>(f2u(v)));
    if constexpr (LR > 16) v += __shfl_xor(v, 16, 64);
    if constexpr (LR > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

// One or two tokens: LR lanes lie along a row, each with 32 consecutive k of it (16 bytes of codes, two scale bytes) per step of 32 LR
// k, so a wave's loads are contiguous runs of a row, 64 / LR rows at once and R of them in turn against the same activations in
// registers.  Codes become bf16 pairs unscaled and meet the activations in two-term dot products (exact products, binary32 sums);
// the sum of a group of 16 is then multiplied by its scale.  `parts` waves share the reduction of their rows.
// us and TB/s of weights (rows x reduction), one token: 8192 x 1024 3.8, 4096 x 4096 with outer blocks 5.1 (mostly the launch and one trip to memory), 8192 x 8192
// 9.0, 4.2 out of the last-level cache and 10.6, 3.6 out of memory, with outer blocks 13.2, 3.0, 16384 x 16384 27.5, 5.5; two tokens 8192 x 8192 13.3.
template <int M, int LR, int R, bool OUTER>
__global__ __launch_bounds__(256) void gemv_few_kernel(const GemvArgs a, int parts)
{
    constexpr int P = 64 / LR;
    __shared__ float red[4][R * P][M];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l = lane % LR, part = wave % parts;
    const int64_t row0 = ((int64_t)blockIdx.x * (4 / parts) + wave / parts) * (R * P) + lane / LR;      // and row0 + P, + 2 P ...
    const uint8_t *codes[R], *scales[R];
    const float *gs[R];
    float acc[R][M];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t row = row0 + r * P < a.C ? row0 + r * P : a.C - 1;     // rows past the end repeat the last one, and are not stored
        codes[r] = a.codes + row * (a.K / 2);
        scales[r] = a.scales + row * (a.K / 16);
        gs[r] = a.gscale + row * (a.K / 128);
#pragma unroll
        for (int m = 0; m < M; ++m) acc[r][m] = 0.0f;
    }
    for (int k = (part * LR + l) * 32; k < a.K; k += parts * LR * 32) {
        const bool whole = k + 32 <= a.K;                                    // else 16 are left
        u32x4 x[M][4], w[R];
        uint32_t s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (whole) {
                w[r] = *reinterpret_cast<const u32x4_at8 *>(codes[r] + k / 2);
                s[r] = *reinterpret_cast<const uint16_at1 *>(scales[r] + k / 16);
            } else {
                const u32x2_at8 h = *reinterpret_cast<const u32x2_at8 *>(codes[r] + k / 2);
                w[r] = u32x4{h[0], h[1], 0, 0};
                s[r] = scales[r][k / 16];
            }
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[m][j] = u32x4{0, 0, 0, 0};
                if (j < 2 || whole) x[m][j] = *reinterpret_cast<const u32x4_at2 *>(a.x + m * a.ldx + k + 8 * j);
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s0 = scale_of<0>(s[r]), s1 = scale_of<1>(s[r]);
            if constexpr (OUTER) {
                const float g = gs[r][k / 128];
                s0 *= g;
                s1 *= g;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float d[M];
#pragma unroll
                for (int m = 0; m < M; ++m) d[m] = 0.0f;
#pragma unroll
                for (int j = 2 * half; j < 2 * half + 2; ++j) {
                    const bf16x2_t p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][j], 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][j], 1.0f, 1),
                                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][j], 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][j], 1.0f, 3)};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int m = 0; m < M; ++m) d[m] = __builtin_amdgcn_fdot2_f32_bf16(p[i], __builtin_bit_cast(bf16x2_t, (uint32_t)x[m][j][i]), d[m], false);
                }
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] = fmaf(d[m], half ? s1 : s0, acc[r][m]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) acc[r][m] = lanes_sum<LR>(acc[r][m]);
    if (parts > 1) {
        if (l == 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m) red[wave][r * P + lane / LR][m] = acc[r][m];
        __syncthreads();
        if (part) return;
        for (int i = 1; i < parts; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] += red[wave + i][r * P + lane / LR][m];
    }
    const float g = OUTER || a.K == 0 ? 1.0f : a.gscale[0];
    if (l != 0) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t c = row0 + r * P;
        if (c >= a.C) continue;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (a.f32) static_cast<float *>(a.y)[m * a.ldy + c] = acc[r][m] * g;
            else static_cast<__bf16 *>(a.y)[m * a.ldy + c] = (__bf16)(acc[r][m] * g);
        }
    }
}

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

// More tokens: a workgroup computes 16 RT outputs (rows of W) of up to 16 NT tokens; its waves split the reduction into consecutive runs of
// whole 256-k pieces and join their sums through LDS.  The matrix instruction wants 16 rows (16 tokens) in 16 neighbouring lanes; loaded so, neighbouring
// lanes would be a row apart and the address unit would take a load lane by lane.  So a wave loads pieces in the order of memory - 128 bytes of codes and
// 512 bytes of activations of a row in neighbouring lanes - and turns them in an LDS area of its own (16-byte places, exclusive-or with the row
// against bank conflicts), while the loads of the next piece are on their way.  With outer blocks the sum over 128 k is multiplied by the
// row's outer scale before it joins the total.
// us out of memory: 5 tokens, 5003 x 2064 7.2; 16 tokens, 4096 x 4096 with outer blocks 7.0, 6144 x 4096 8.6, 8192 x 8192 15.0, 16384 x 16384 42 (3.6 TB/s); 8192 x 8192
// with 32 tokens 23.1, with 64 39.  Between the launch and the join a wave's pieces follow each other: a trip to memory each, whose time the two waves a SIMD cover in part, and
// 3.4 vector instructions a weight (6.7 us of all SIMDs' time at 8192 x 8192), most of which make the weights bf16.
constexpr int kPiece = 256;                                                  // k
template <int NT, int RT> struct GemvStage {
    u32x4 x[NT][16][32];                                                     // [token][place of 8 k]
    u32x4 codes[RT][16][8];                                                  // [row][place of 32 k]
    uint32_t scales[RT][16][4];                                              // [row][64 k]
    float outer[RT][16][2];                                                  // [row][128 k]
};

template <int NT, int RT, bool OUTER>
__global__ __launch_bounds__(512) void gemv_kernel(const GemvArgs a)
{
    extern __shared__ u32x4 lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    GemvStage<NT, RT> &stage = reinterpret_cast<GemvStage<NT, RT> *>(lds)[wave];
    const int r = lane & 15, q = lane >> 4;
    const int64_t c0 = (int64_t)blockIdx.x * (16 * RT), m0 = (int64_t)blockIdx.y * (16 * NT);
    const int pieces = (a.K + kPiece - 1) / kPiece;
    const int k_first = (int)((int64_t)pieces * wave / waves) * kPiece;
    const int k_last = (int)((int64_t)pieces * (wave + 1) / waves) * kPiece;
    const int k_end = k_last < a.K ? k_last : a.K;

    // where this lane's loads start: rows past the end repeat the last one and are not stored, tokens past the end are zeros
    const auto row_of = [&](int t, int i) { const int64_t c = c0 + 16 * t + i; return c < a.C ? c : a.C - 1; };
    const uint8_t *codes[RT][2], *scales[RT];
    const float *outer[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) codes[t][i] = a.codes + row_of(t, 8 * i + (lane >> 3)) * (a.K / 2) + 16 * (lane & 7);
        scales[t] = a.scales + row_of(t, lane >> 2) * (a.K / 16) + 4 * (lane & 3);
        outer[t] = a.gscale + row_of(t, (lane & 31) >> 1) * (a.K / 128) + (lane & 1);
    }
    const int64_t token = m0 + (lane >> 5);
    const uint16_t *const x = a.x + token * a.ldx + 8 * (lane & 31);

    u32x4 vx[NT][8], vc[RT][2];
    uint32_t vs[RT];
    float vo[RT];
    const auto load = [&](int k0) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int k = k0 + 32 * (lane & 7);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                vc[t][i] = u32x4{0, 0, 0, 0};
                if (k + 32 <= k_end) {
                    vc[t][i] = *reinterpret_cast<const u32x4_at8 *>(codes[t][i] + k0 / 2);
                } else if (k < k_end) {
                    const u32x2_at8 h = *reinterpret_cast<const u32x2_at8 *>(codes[t][i] + k0 / 2);
                    vc[t][i][0] = h[0];
                    vc[t][i][1] = h[1];
                }
            }
            const int ks = k0 + 64 * (lane & 3);
            vs[t] = 0;
            if (ks + 64 <= k_end) {
                vs[t] = *reinterpret_cast<const uint32_at1 *>(scales[t] + k0 / 16);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (ks + 16 * i < k_end) vs[t] |= (uint32_t)scales[t][k0 / 16 + i] << (8 * i);
            }
            if constexpr (OUTER) vo[t] = k0 + 128 * (lane & 1) < k_end ? outer[t][k0 / 128] : 0.0f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                vx[n][i] = u32x4{0, 0, 0, 0};
                const int ahead = 16 * n + 2 * i;
                if (token + ahead < a.M && k0 + 8 * (lane & 31) < k_end) vx[n][i] = *reinterpret_cast<const u32x4_at2 *>(x + ahead * a.ldx + k0);
            }
    };
    const auto turn = [&]() {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
            for (int i = 0; i < 2; ++i) stage.codes[t][8 * i + (lane >> 3)][(lane ^ (lane >> 3)) & 7] = vc[t][i];
            stage.scales[t][lane >> 2][lane & 3] = vs[t];
            if constexpr (OUTER)
                if (lane < 32) stage.outer[t][lane >> 1][lane & 1] = vo[t];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) stage.x[n][2 * i + (lane >> 5)][(lane & 31) ^ (2 * i + (lane >> 5))] = vx[n][i];
    };

    float4_t acc[RT][NT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (k_first < k_end) load(k_first);
    for (int k0 = k_first; k0 < k_end; k0 += kPiece) {
        wave_lds_order();            // the last piece has been read
        turn();
        if (k0 + kPiece < k_end) load(k0 + kPiece);
        wave_lds_order();            // this one has been written
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 w[RT];
            float s0[RT], s1[RT];
            float4_t block[RT][NT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                w[t] = stage.codes[t][r][(4 * h + q) ^ (r & 7)];
                const uint32_t s = stage.scales[t][r][2 * h + (q >> 1)] >> (16 * (q & 1));
                s0[t] = scale_of<0>(s);
                s1[t] = scale_of<1>(s);
#pragma unroll
                for (int n = 0; n < NT; ++n) block[t][n] = OUTER ? float4_t{0.0f, 0.0f, 0.0f, 0.0f} : acc[t][n];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8_t v[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) v[n] = __builtin_bit_cast(bf16x8_t, stage.x[n][r][(16 * h + 4 * q + j) ^ r]);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const bf16x8_t wj = __builtin_bit_cast(bf16x8_t, weights8(w[t][j], j < 2 ? s0[t] : s1[t]));
#pragma unroll
                    for (int n = 0; n < NT; ++n) block[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wj, v[n], block[t][n], 0, 0, 0);
                }
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (OUTER) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[t][n][i] = fmaf(block[t][n][i], stage.outer[t][4 * q + i][h], acc[t][n][i]);
                    } else {
                        acc[t][n] = block[t][n];
                    }
                }
        }
    }
    __syncthreads();
    float4_t *const red = reinterpret_cast<float4_t *>(lds);                 // [waves][RT NT][64]
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) red[(wave * RT * NT + t * NT + n) * 64 + lane] = acc[t][n];
    __syncthreads();
    const float g = OUTER || a.K == 0 ? 1.0f : a.gscale[0];
    for (int i = wave; i < RT * NT; i += waves) {
        float4_t sum = red[i * 64 + lane];
        for (int o = 1; o < waves; ++o) sum += red[(o * RT * NT + i) * 64 + lane];
        const int64_t m = m0 + 16 * (i % NT) + r, c = c0 + 16 * (i / NT) + 4 * q;      // lane: token m, outputs c .. c + 3
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < a.C) {
                if (a.f32) static_cast<float *>(a.y)[m * a.ldy + c + j] = sum[j] * g;
                else static_cast<__bf16 *>(a.y)[m * a.ldy + c + j] = (__bf16)(sum[j] * g);
            }
    }
}

template <int NT, int RT> void run_gemv(const GemvArgs &a, int outer, int most_waves, hipStream_t st)
{
    const dim3 grid((unsigned)((a.C + 16 * RT - 1) / (16 * RT)), (unsigned)((a.M + 16 * NT - 1) / (16 * NT)));
    const int pieces = (a.K + kPiece - 1) / kPiece, waves = pieces < 1 ? 1 : pieces < most_waves ? pieces : most_waves;
    const size_t lds = waves * sizeof(GemvStage<NT, RT>);
    if (outer) gemv_kernel<NT, RT, true><<<grid, waves * 64, lds, st>>>(a);
    else gemv_kernel<NT, RT, false><<<grid, waves * 64, lds, st>>>(a);
}

// Tiles of 16 rows and how they are dealt, us of a call in a replayed graph, out of memory, by rows x waves of a workgroup (0.2 to 4 us less where the last-level cache
// has the weights):
//   up to one a CU      a workgroup each, whose eight waves split the reduction (85 KB of LDS)
//   up to two a CU      a workgroup takes two, which share the activations, and is still alone on its CU with eight waves (six for 32 tokens: 127 KB of LDS)
//   up to three a CU    one each with four waves: three workgroups (two for 32 tokens) fit on a CU and all run at once
//   more                two each with four waves
//                                  M = 5                       M = 16                      M = 32
//   outputs x reduction    16x4   32x8   32x4          16x4   32x8   32x4          16x4   32x6   32x4
//    4112 x 2048            5.2    5.3    5.8           5.9    5.9    6.3           7.9    8.3    7.8
//    5120 x 4096            8.7    8.0    8.9          10.0    9.3   10.3          14.4   13.0   13.2
//    8000 x 2048            6.1    6.2    6.3           7.2    7.1    7.2           9.4    9.3    8.8
//    8000 x 8192           14.8   13.8   15.8          17.1   15.7   18.6          25.8   21.7   24.6
//    8208 x 4096            9.8   13.8   11.5          12.5   15.6   12.2          21.1   22.7   23.4
//   12288 x 4096           10.8   14.7   12.7          13.7   17.2   14.5          22.6   24.6   25.2
//   12304 x 4096           13.2   14.7   12.7          16.4   17.3   14.6          25.3   24.7   25.3
//   16384 x 8192           25.1   25.4   22.5          33.6   29.0   25.9          47.3   40.6   45.7
// (at its worst the rule gives 7.8 for 7.1: 4112 x 2816, 16 tokens.)  A reduction of few pieces has no work for the waves that two tiles would add: up to two
// a CU, 5120 x 1024 4.3 / 4.5 (5 tokens, 16 / 32 rows), 4.8 / 4.8 (16), 6.2 / 5.8 (32); 5003 x 768 4.1 / 4.4 (3), 4.6 / 4.6 (16), 5.7 / 5.7 (32).  Three waves a workgroup leave two tiles of 32 tokens room for a second workgroup: 11264 x 768
// 9.0 / 7.0.
template <int NT> void run_gemv(const GemvArgs &a, int outer, hipStream_t st)
{
    const int64_t tiles = (a.C + 15) / 16;
    const int pieces = (a.K + kPiece - 1) / kPiece;
    if (tiles <= 256) run_gemv<NT, 1>(a, outer, 8, st);
    else if (tiles <= 512 && pieces >= (NT == 1 ? 5 : 4)) run_gemv<NT, 2>(a, outer, NT == 1 ? 8 : 6, st);
    else if (tiles <= 512 || (tiles <= 768 && (NT == 1 || pieces >= 4))) run_gemv<NT, 1>(a, outer, 4, st);
    else run_gemv<NT, 2>(a, outer, 4, st);
}

template <int M, int LR, int R> void run_few(const GemvArgs &a, int outer, hipStream_t st)
{
    constexpr int ROWS = R * (64 / LR);                       // of a wave
    const int64_t waves = (a.C + ROWS - 1) / ROWS;
    int parts = 1;
    while (parts < 4 && waves * parts < 4096 && LR * 32 * parts < a.K) parts *= 2;
    const unsigned blocks = (unsigned)((waves * parts + 3) / 4);
    if (outer) gemv_few_kernel<M, LR, R, true><<<blocks, 256, 0, st>>>(a, parts);
    else gemv_few_kernel<M, LR, R, false><<<blocks, 256, 0, st>>>(a, parts);
}

// Four rows a lane read the activations half as often as two, two rows give twice the waves: two where four would leave under 2048 waves.
// us, one token, two rows / four: 2304 x 768 3.3 / 3.8, 4096 x 4096 4.6 / 4.9, 8192 x 8192 11.0 / 10.4, 16384 x 16384 35 / 27.6.  The reduction
// is split until there are 4096 waves (8192 x 8192 with 2048: 12.3).
template <int M, int LR> void run_few(const GemvArgs &a, int outer, hipStream_t st)
{
    if (a.C >= 2048 * 4 * (64 / LR)) run_few<M, LR, 4>(a, outer, st);
    else run_few<M, LR, 2>(a, outer, st);
}

template <int M> void run_few(const GemvArgs &a, int outer, hipStream_t st)
{
    if (a.K <= 512) run_few<M, 16>(a, outer, st);
    else if (a.K <= 1024) run_few<M, 32>(a, outer, st);
    else run_few<M, 64>(a, outer, st);
}

}  // namespace

hipError_t launch_gemv(const void *X, int64_t ldx, int64_t M, const GemmOperand &W, int64_t K, const RowDst &y, hipStream_t st)
{
    const GemvArgs a{static_cast<const uint16_t *>(X), ldx, M, W.codes, W.scales, W.gscale, W.rows, (int)K, y.p, y.ld, y.f32};
    // us of a call in a replayed graph, out of memory, dot products / matrix instructions:
    //                    1 token        2 tokens       3 tokens       4 tokens
    //    1024 x 1024    2.5 /  3.6     2.9 /  3.6     3.3 /  3.6     3.9 /  3.7
    //    4096 x 4096    4.7 /  6.1     5.9 /  6.2     7.1 /  6.2     8.4 /  6.2
    //    8192 x 8192   10.4 / 13.4    12.9 / 13.4    16.6 / 13.7    18.7 / 13.5
    //   16384 x 16384  30.4 / 37.2    37.5 / 36.2    47.1 / 36.7    57.3 / 37.1
    // (1 x 128 outer blocks 0.1 to 5 us more on either side, the same order).  Three tokens gain 0.4 us at most by dot products, on weights of up to 2 MB, and are left to the others.
    if (M == 1) run_few<1>(a, W.outer, st);
    else if (M == 2) run_few<2>(a, W.outer, st);
    else if (M <= 16) run_gemv<1>(a, W.outer, st);
    else run_gemv<2>(a, W.outer, st);
    return hipGetLastError();
}

}  // namespace tj
