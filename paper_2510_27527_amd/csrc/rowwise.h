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

// Start of a row that all lanes of a wave share, in scalar registers: a lane's addresses are then this and a 32-bit offset, not a pair of registers
// each (which the loops over rows would hold for every array).
template <typename T> __device__ __forceinline__ T *shared_row(T *p)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return reinterpret_cast<T *>((uint64_t)hi << 32 | lo);
}
// SHARED: the lanes of a wave share the row, whose elements 32-bit numbers count
template <bool SHARED, typename T, typename I> __device__ __forceinline__ T *row_at(T *p, int64_t row, int64_t ld, I at)
{
    if constexpr (SHARED) return shared_row(p + row * ld) + (uint32_t)at;
    else return p + row * ld + at;
}

// STREAM: past the caches (see streams())
template <typename T, bool STREAM> __device__ __forceinline__ T load_as(const void *p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const T *>(p));
    else return *static_cast<const T *>(p);
}

// Elements [col, col + 8) of a row (n > col: at least one is there), for widen8 of the same place.  A chunk that the row's end cuts is read as
// the row's last eight elements, where there are eight (one load, few registers), else element by element.
// HELD: rows have at least eight elements, and the lanes of a wave share them.
template <int KIND, bool HELD, bool STREAM, typename I>
__device__ __forceinline__ Raw<KIND> load8(const RowSrc &s, int64_t row, I col, I n)
{
    Raw<KIND> r;
    const I at = col + kChunk > n ? n - kChunk : col;     // below zero in a row of fewer than eight
    if constexpr (KIND == kBf16) {
        const uint16_t *const p = static_cast<const uint16_t *>(s.p);
        if (HELD || n >= kChunk) {
            r.q = load_as<bf16x8_at2, STREAM>(row_at<HELD>(p, row, s.ld, at));
        } else {
            r.q = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (i < n) r.q[i / 2] |= (uint32_t)p[row * s.ld + i] << (16 * (i & 1));
        }
    } else if constexpr (KIND == kF32) {
        const float *const p = static_cast<const float *>(s.p);
        if (HELD || n >= kChunk) {
            r.lo = load_as<f32x4_at4, STREAM>(row_at<HELD>(p, row, s.ld, at));
            r.hi = load_as<f32x4_at4, STREAM>(row_at<HELD>(p, row, s.ld, at) + 4);
        } else {
            r.lo = r.hi = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (i < n) (i < 4 ? r.lo : r.hi)[i & 3] = p[row * s.ld + i];
        }
    } else {
        const uint8_t *const p = static_cast<const uint8_t *>(s.p);
        if (HELD || n >= kChunk) {
            r.q = load_as<code8_at1, STREAM>(row_at<HELD>(p, row, s.ld, at));
        } else {
            r.q = u32x2{0, 0};
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (i < n) r.q[i / 4] |= (uint32_t)p[row * s.ld + i] << (8 * (i & 3));
        }
        r.e = *row_at<HELD>(s.exps, row, s.groups, col / kCkptGroup);
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

// v moved down by `by` elements (0 to 7), zeros above
__device__ __forceinline__ u32x4 move_down(u32x4 v, uint32_t by)      // bf16
{
    const uint32_t half = (by & 1) * 16;
    v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], half), __builtin_amdgcn_alignbit(v[2], v[1], half), __builtin_amdgcn_alignbit(v[3], v[2], half), v[3] >> half};
    if (by & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (by & 4) v = u32x4{v[2], v[3], 0, 0};
    return v;
}
__device__ __forceinline__ u32x2 move_down(u32x2 v, uint32_t by)      // bytes
{
    const uint64_t u = (((uint64_t)v[1] << 32) | v[0]) >> (8 * by);
    return u32x2{(uint32_t)u, (uint32_t)(u >> 32)};
}
__device__ __forceinline__ void move_down(float4_t &lo, float4_t &hi, uint32_t by)
{
    if (by & 1) lo = float4_t{lo[1], lo[2], lo[3], hi[0]}, hi = float4_t{hi[1], hi[2], hi[3], 0.0f};
    if (by & 2) lo = float4_t{lo[2], lo[3], hi[0], hi[1]}, hi = float4_t{hi[2], hi[3], 0.0f, 0.0f};
    if (by & 4) lo = hi, hi = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
}

__device__ __forceinline__ void widen(const Raw<kBf16> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(r.q[i]);
        v[2 * i + 1] = bf16_hi(r.q[i]);
    }
}
__device__ __forceinline__ void widen(const Raw<kF32> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = r.lo[i];
        v[4 + i] = r.hi[i];
    }
}
// code * 2^e: exact but for results below 2^-126
__device__ __forceinline__ void widen(const Raw<kCkpt8> &r, float (&v)[8])
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

// A chunk that load8 or zero8 gave for this place, in its place: one that the row's end cuts was read further up and is moved down here, where the
// loads after it are on their way.  Whether rows have such a chunk is asked of the row length, the same for all lanes: a question to each
// lane would be passed with the lanes masked, the wait for the load included.
template <int KIND, typename I> __device__ __forceinline__ Raw<KIND> settle8(Raw<KIND> r, I col, I n)
{
    if (n % kChunk != 0 && n > kChunk) {
        const I over = col + kChunk - n;
        const uint32_t by = over > 0 && over < kChunk ? (uint32_t)over : 0;      // past the end altogether: zeros already
        if constexpr (KIND == kF32) move_down(r.lo, r.hi, by);
        else r.q = move_down(r.q, by);
    }
    return r;
}
// its values; those at or past n are zeros
template <int KIND, typename I> __device__ __forceinline__ void widen8(const Raw<KIND> &r, I col, I n, float (&v)[8])
{
    widen(settle8(r, col, n), v);
}

// ---- stores -----------------------------------------------------------------------------------

template <bool F32, bool SHARED, typename I>
__device__ __forceinline__ void store8(void *out, int64_t ld, int64_t row, I col, I n, const float (&v)[8])
{
    if constexpr (F32) {
        float *const p = row_at<SHARED>(static_cast<float *>(out), row, ld, col);
        if (col + kChunk <= n) {
            *reinterpret_cast<f32x4_at4 *>(p) = f32x4_at4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_at4 *>(p + 4) = f32x4_at4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < kChunk - 1; ++i)
                if (col + i < n) p[i] = v[i];
        }
    } else {
        uint16_t *const p = row_at<SHARED>(static_cast<uint16_t *>(out), row, ld, col);
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
template <bool SHARED, typename I>
__device__ __forceinline__ void ckpt_store8(const CkptOut &o, int64_t row, I col, I n, const float (&v)[8])
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
    uint8_t *const p = row_at<SHARED>(o.codes, row, n, col);
    if (col + kChunk <= n) {
        *reinterpret_cast<code8_at1 *>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < kChunk - 1; ++i)
            if (col + i < n) p[i] = (uint8_t)(q[i / 4] >> (8 * (i & 3)));
    }
    if (col % kCkptGroup == 0) *row_at<SHARED>(o.exps, row, o.groups, col / kCkptGroup) = (uint8_t)(e + 127);
}

// ---- sums over the threads of a row -----------------------------------------------------------

// over the 64 lanes of a wave, the same bits in each: four exchanges inside rows of 16 lanes, then between the rows
__device__ __forceinline__ float wave_sum(float v)
{
    v += u2f(dpp<DPP_QUAD_XOR1>(f2u(v)));
    v += u2f(dpp<DPP_QUAD_XOR2>(f2u(v)));
    v += u2f(dpp<DPP_ROW_HALF_MIRROR>(f2u(v)));
    v += u2f(dpp<DPP_ROW_MIRROR>(f2u(v)));
    const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
    v = u2f(a[0]) + u2f(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
    return u2f(b[0]) + u2f(b[1]);
}

// Sums of two numbers over the TPR threads that hold a row; every one of them gets both.  red: two floats per wave of the workgroup, all of whose
// threads call this together where TPR > 64.  No barrier follows the last read of red: a workgroup's next sum, of the same row or of the next, has to
// take the other half of a doubled array (the one after it may take this half again, since the barrier between lies behind all reads of it).
template <int TPR>
__device__ __forceinline__ void row_sum2(float &a, float &b, float2_t *red)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[w] = float2_t{a, b};
        __syncthreads();
        const float2_t m = red[w / W * W + (threadIdx.x & (W - 1))];     // W lanes add what the row's W waves left
        a = m.x;
        b = m.y;
        const auto both = [&](auto step) {
            a += u2f(step(f2u(a)));
            b += u2f(step(f2u(b)));
        };
        static_assert(W == 4 || W == 8 || W == 16);
        both([](uint32_t v) { return dpp<DPP_QUAD_XOR1>(v); });
        both([](uint32_t v) { return dpp<DPP_QUAD_XOR2>(v); });
        if constexpr (W >= 8) both([](uint32_t v) { return dpp<DPP_ROW_HALF_MIRROR>(v); });
        if constexpr (W >= 16) both([](uint32_t v) { return dpp<DPP_ROW_MIRROR>(v); });
    }
}

}  // namespace tj
