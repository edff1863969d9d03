// What the row-wise kernels (norms, nonlinearities, 8-bit checkpoints) share: chunks of eight consecutive elements of a
// row, sums over the threads of a row, and the 8-bit checkpoint format.
//
// Rows may start at any element: the vector accesses below ask for the alignment of one element only, which the hardware's global
// loads and stores take (a row whose start is not on 16 bytes costs an access that touches one cache line more).  The last
// chunk of a row whose length is not a multiple of eight goes element by element.
#pragma once
#include "block_ops.h"
#include "device_fmt.h"

namespace tj {

typedef uint32_t bf16x8_at2 __attribute__((ext_vector_type(4), aligned(2)));     // eight bf16 that start at any bf16
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));         // four binary32 that start at any of them
typedef uint32_t code8_at1 __attribute__((ext_vector_type(2), aligned(1)));      // eight E4M3 codes that start at any byte
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kChunk = 8;                             // elements of a chunk
constexpr int kGroupLanes = kCkptGroup / kChunk;       // a checkpoint's group is the chunks of 16 neighbouring lanes

// two binary32 -> two bf16, nearest even
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const float2_t f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

// ---- eight elements of a row, as they lie in memory ------------------------------------------

template <int KIND> struct Raw;
template <> struct Raw<kBf16> { u32x4 q; };
template <> struct Raw<kF32> { float4_t lo, hi; };
template <> struct Raw<kCkpt8> { u32x2 q; uint32_t e; };

// elements [col, col + 8) of a row; those at or past n are zeros (n > col: at least one is there)
template <int KIND>
__device__ __forceinline__ Raw<KIND> load8(const RowSrc &s, int64_t row, int64_t col, int64_t n)
{
    Raw<KIND> r;
    if constexpr (KIND == kBf16) {
        const uint16_t *p = static_cast<const uint16_t *>(s.p) + row * s.ld + col;
        if (col + kChunk <= n) {
            r.q = *reinterpret_cast<const bf16x8_at2 *>(p);
        } else {
            r.q = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) r.q[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
        }
    } else if constexpr (KIND == kF32) {
        const float *p = static_cast<const float *>(s.p) + row * s.ld + col;
        if (col + kChunk <= n) {
            r.lo = *reinterpret_cast<const f32x4_at4 *>(p);
            r.hi = *reinterpret_cast<const f32x4_at4 *>(p + 4);
        } else {
            r.lo = r.hi = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) (i < 4 ? r.lo : r.hi)[i & 3] = p[i];
        }
    } else {
        const uint8_t *p = static_cast<const uint8_t *>(s.p) + row * s.ld + col;
        if (col + kChunk <= n) {
            r.q = *reinterpret_cast<const code8_at1 *>(p);
        } else {
            r.q = u32x2{0, 0};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) r.q[i / 4] |= (uint32_t)p[i] << (8 * (i & 3));
        }
        r.e = s.exps[row * s.groups + col / kCkptGroup];
    }
    return r;
}

template <int KIND> __device__ __forceinline__ Raw<KIND> zero8()
{
    Raw<KIND> r;
    if constexpr (KIND == kBf16) r.q = u32x4{0, 0, 0, 0};
    else if constexpr (KIND == kF32) r.lo = r.hi = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    else { r.q = u32x2{0, 0}; r.e = 127; }
    return r;
}

__device__ __forceinline__ void widen8(const Raw<kBf16> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(r.q[i]);
        v[2 * i + 1] = bf16_hi(r.q[i]);
    }
}
__device__ __forceinline__ void widen8(const Raw<kF32> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = r.lo[i];
        v[4 + i] = r.hi[i];
    }
}
// code * 2^e: exact but for results below 2^-126
__device__ __forceinline__ void widen8(const Raw<kCkpt8> &r, float (&v)[8])
{
    const float scale = u2f(r.e << 23);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.q[i], false);
        const float2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.q[i], true);
        v[4 * i] = a.x * scale;
        v[4 * i + 1] = a.y * scale;
        v[4 * i + 2] = b.x * scale;
        v[4 * i + 3] = b.y * scale;
    }
}

// ---- stores -----------------------------------------------------------------------------------

template <bool F32>
__device__ __forceinline__ void store8(void *out, int64_t ld, int64_t row, int64_t col, int64_t n, const float (&v)[8])
{
    if constexpr (F32) {
        float *p = static_cast<float *>(out) + row * ld + col;
        if (col + kChunk <= n) {
            *reinterpret_cast<f32x4_at4 *>(p) = f32x4_at4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_at4 *>(p + 4) = f32x4_at4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) p[i] = v[i];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(out) + row * ld + col;
        const u32x4 q = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        if (col + kChunk <= n) {
            *reinterpret_cast<bf16x8_at2 *>(p) = q;
        } else {
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
        }
    }
}

// ---- 8-bit checkpoints ------------------------------------------------------------------------

// Stores the codes of eight values of a row, and the group's exponent once.  The group's 16 lanes call it together (lanes past the
// row's end with zeros).  a = max |v| over the finite values, e the least integer with a <= 1.75 * 2^(8 + e) = 448 * 2^e within
// [-126, 120]: both 2^e and 2^-e are then ordinary binary32 numbers, the product v * 2^-e is exact (rounded below 2^-126, far
// under half of the smallest code) and the conversion's rounding is the only one.  Values that are not finite become the NaN 0x7F.
__device__ __forceinline__ void ckpt_store8(const CkptOut &o, int64_t row, int64_t col, int64_t n, const float (&v)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, f2u(v[i]) & 0x7FFFFFFFu);
    const bool odd = a >= 0x7F800000u;                  // some value here is not finite
    if (odd) {
        a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = f2u(v[i]) & 0x7FFFFFFFu;
            a = b < 0x7F800000u ? max(a, b) : a;
        }
    }
    a = max(a, dpp<DPP_QUAD_XOR1>(a));
    a = max(a, dpp<DPP_QUAD_XOR2>(a));
    a = max(a, dpp<DPP_ROW_HALF_MIRROR>(a));
    a = max(a, dpp<DPP_ROW_MIRROR>(a));
    int e = (int)((a + 0x1FFFFFu) >> 23) - (127 + 8);
    e = e < -126 ? -126 : e;
    const float inv = u2f((uint32_t)(127 - e) << 23);
    u32x2 q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
        q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, w, true);
    }
    if (odd) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((f2u(v[i]) & 0x7FFFFFFFu) >= 0x7F800000u) q[i / 4] = (q[i / 4] & ~(0xFFu << (8 * (i & 3)))) | (0x7Fu << (8 * (i & 3)));
    }
    if (col >= n) return;
    uint8_t *p = o.codes + row * n + col;
    if (col + kChunk <= n) {
        *reinterpret_cast<code8_at1 *>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < kChunk - 1; ++i)
            if (col + i < n) p[i] = (uint8_t)(q[i / 4] >> (8 * (i & 3)));
    }
    if (col % kCkptGroup == 0) o.exps[row * o.groups + col / kCkptGroup] = (uint8_t)(e + 127);
}

// ---- sums over the threads of a row -----------------------------------------------------------

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Sums of two numbers over the TPR threads that hold a row; every one of them gets both.  red: 2 floats per wave of the workgroup;
// a workgroup that sums again passes the other half of a doubled array, so that no barrier is needed before the next sum.
template <int TPR>
__device__ __forceinline__ void row_sum2(float &a, float &b, float *red)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            red[2 * w] = a;
            red[2 * w + 1] = b;
        }
        __syncthreads();
        a = red[0];
        b = red[1];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            a += red[2 * i];
            b += red[2 * i + 1];
        }
    }
}

}  // namespace tj
