// Rotary positions, and the paged cache of keys and values: appending (with the rotation on the way) and reading back.
//
//   pair (a, b) of a head, angle t = position * frequency:  (a cos t - b sin t, b cos t + a sin t), and with -t on the way back
//
// Bound by memory: every element is read once and written once.  A unit of work is eight pairs (16 elements, two 16-byte accesses each way)
// or eight elements that stay as they are; cosines and sines are computed once per token and pair, in LDS, for all of the token's heads.
// Medians: 16384 rows of 32 heads of 64 (bf16, 134 MB) 24.5 us, 5.5 TB/s; 1001 x 5 heads of 80 in binary32 3.7; appending one token 2.8, 256 tokens 4.9 (32 query heads, 8 key heads of 128);
// 6253 tokens into 8 bits 38, and read back as bf16 11.5; into bf16 42 (3.6 TB/s), read back 12 (4.2).  In 8 bits several tokens a workgroup (47 to 75 us, where one took 42 to 46) and two units a thread at once (59 to 62) were slower.
#include "rowwise.h"
#include "seq_ops.h"

namespace tj {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;               // of a workgroup
constexpr int kTurnTable = 2048;             // cosines and sines that a workgroup's LDS holds
constexpr int kSliceElems = 2048;            // elements of the key heads that a workgroup of an 8-bit cache takes: 8 KB of LDS

// i / by for i * by < 2^32, by a product
struct Quotient {
    int by;
    uint32_t magic;
    __device__ __forceinline__ int operator()(int i) const { return magic ? (int)__umulhi((uint32_t)i, magic) : i; }
};
Quotient quotient(int by) { return Quotient{by, by == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + by - 1) / by)}; }

// Cosine and sine of position * freq.  The product of a 31-bit integer and a 24-bit significand has up to 55 bits: in 64 bits it is off by half a unit of
// the last place at most.  Its turns less the nearest quarter turn leave |x| <= pi / 4 for binary32, where the Taylor series to x^9 and x^10 are off by 2e-9.
__device__ __forceinline__ float2_t cos_sin(int pos, float freq)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189533577;
    const double quarters = rint(4.0 * turns);
    const float x = (float)(fma(-0.25, quarters, turns)) * 6.28318530717958647692f;
    const int q = (int)(long long)quarters & 3;
    const float z = x * x;
    const float s = x + x * z * fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;
    return float2_t{q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b};
}

// The same in 64 bits, for keys that are rounded to E4M3: an error of 2^-23 moves one in a million of them to a neighbouring code.  The series to x^17 and x^16 are off by 2^-55.
struct Turn64 {
    double x, y;
};
__device__ __forceinline__ Turn64 cos_sin64(int pos, float freq)
{
    const double turns = (double)pos * (double)freq * 0.15915494309189533577;
    const double quarters = rint(4.0 * turns);
    const double x = fma(-0.25, quarters, turns) * 6.28318530717958647692, z = x * x;
    const int q = (int)(long long)quarters & 3;
    double s = 1.0 / 355687428096000, c = 1.0 / 20922789888000;
    s = fma(s, z, -1.0 / 1307674368000);
    s = fma(s, z, 1.0 / 6227020800);
    s = fma(s, z, -1.0 / 39916800);
    s = fma(s, z, 1.0 / 362880);
    s = fma(s, z, -1.0 / 5040);
    s = fma(s, z, 1.0 / 120);
    s = fma(s, z, -1.0 / 6);
    s = fma(s * z, x, x);
    c = fma(c, z, -1.0 / 87178291200);
    c = fma(c, z, 1.0 / 479001600);
    c = fma(c, z, -1.0 / 3628800);
    c = fma(c, z, 1.0 / 40320);
    c = fma(c, z, -1.0 / 720);
    c = fma(c, z, 1.0 / 24);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const double a = q & 1 ? s : c, b = q & 1 ? c : s;
    return Turn64{q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b};
}
// to binary32 for a second rounding to few bits: toward zero, with the last bit set where that left something off, so that the second rounding is that of the number itself
__device__ __forceinline__ float round_to_odd(double v)
{
    const float f = __double2float_rz(v);
    return (double)f != v && fabsf(f) < INFINITY ? u2f(f2u(f) | 1u) : f;
}

// Up to eight consecutive elements as they lie in memory; those from n on are zeros.
template <typename T> using RawOf = Raw<sizeof(T) == 2 ? kBf16 : kF32>;
template <typename T> __device__ __forceinline__ RawOf<T> raw8(const T *p, int n)
{
    RawOf<T> r = zero8<sizeof(T) == 2 ? kBf16 : kF32>();
    if (n >= 8) {
        if constexpr (sizeof(T) == 2) r.q = *reinterpret_cast<const bf16x8_at2 *>(p);
        else r.lo = *reinterpret_cast<const f32x4_at4 *>(p), r.hi = *reinterpret_cast<const f32x4_at4 *>(p + 4);
        return r;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) {
            if constexpr (sizeof(T) == 2) r.q[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
            else (i < 4 ? r.lo : r.hi)[i & 3] = p[i];
        }
    return r;
}
template <typename T> __device__ __forceinline__ void put8(T *p, int n, const float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        const u32x4 q = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        if (n >= 8) {
            *reinterpret_cast<bf16x8_at2 *>(p) = q;
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
    } else {
        if (n >= 8) {
            *reinterpret_cast<f32x4_at4 *>(p) = f32x4_at4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_at4 *>(p + 4) = f32x4_at4{v[4], v[5], v[6], v[7]};
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = v[i];
    }
}

// units of a head: runs of eight pairs, then runs of eight elements that are not turned
__host__ __device__ __forceinline__ int units_of(int D, int half) { return (half + 7) / 8 + (D - 2 * half + 7) / 8; }

// Unit u of a head: two runs of up to eight elements, the second one of turned units alone.
template <typename S> struct Unit { RawOf<S> x, y; };
template <typename S> __device__ __forceinline__ Unit<S> read_unit(const S *src, int D, int half, int pairs, int u)
{
    const int runs = (half + 7) >> 3, j = 8 * u, n = half - j;
    Unit<S> r;
    r.y = zero8<sizeof(S) == 2 ? kBf16 : kF32>();
    if (u >= runs) {
        const int at = 2 * half + 8 * (u - runs);
        r.x = raw8(src + at, D - at);
    } else if (pairs) {
        r.x = raw8(src + 2 * j, 2 * n);
        r.y = raw8(src + 2 * j + 8, 2 * n - 8);
    } else {
        r.x = raw8(src + j, n);
        r.y = raw8(src + half + j, n);
    }
    return r;
}
__device__ __forceinline__ void turn_pair(float &a, float &b, float2_t t)
{
    const float c = fmaf(a, t.x, -(b * t.y));
    b = fmaf(b, t.x, a * t.y);
    a = c;
}
__device__ __forceinline__ void turn_pair(float &a, float &b, const Turn64 &t)
{
    const double c = fma((double)a, t.x, -((double)b * t.y));
    b = round_to_odd(fma((double)b, t.x, (double)a * t.y));
    a = round_to_odd(c);
}

// The unit turned, in its place.  cs: the token's cosines and sines.  All of a unit has been read before any of it is written: src may be dst.
template <typename S, typename T>
__device__ __forceinline__ void write_unit(const Unit<S> &r, T *dst, int D, int half, int pairs, int u, const float2_t *cs)
{
    const int runs = (half + 7) >> 3, j = 8 * u, n = half - j;
    float x[8], y[8];
    widen(r.x, x);
    if (u >= runs) {
        const int at = 2 * half + 8 * (u - runs);
        put8(dst + at, D - at, x);
        return;
    }
    widen(r.y, y);
    if (pairs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turn_pair(x[2 * i], x[2 * i + 1], cs[min(j + i, half - 1)]);
            turn_pair(y[2 * i], y[2 * i + 1], cs[min(j + 4 + i, half - 1)]);
        }
        put8(dst + 2 * j, 2 * n, x);
        put8(dst + 2 * j + 8, 2 * n - 8, y);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn_pair(x[i], y[i], cs[min(j + i, half - 1)]);
        put8(dst + j, n, x);
        put8(dst + half + j, n, y);
    }
}

__device__ __forceinline__ float2_t turn_of(const Rotation &r, int pos, int j, int inverse)
{
    float2_t t = cos_sin(pos, r.freqs[j]);
    t.x *= r.scale;
    t.y *= inverse ? -r.scale : r.scale;
    return t;
}

// ---- rotary positions of whole rows ------------------------------------------------------------

template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void rope_kernel(const S *x, int64_t ldx, const int *pos, int N, int D, int units, int row_units, int tokens, Rotation r, int inverse,
                                                       T *y, int64_t ldy)
{
    __shared__ float2_t cs[kTurnTable];
    const int n0 = blockIdx.x * tokens, count = min(tokens, N - n0);
    for (int i = threadIdx.x; i < count * r.half; i += kThreads) {
        const int t = i / r.half;
        cs[i] = turn_of(r, pos[n0 + t], i - t * r.half, inverse);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count * row_units; i += kThreads) {
        const int t = i / row_units, w = i - t * row_units, h = w / units;
        const int64_t n = n0 + t;
        const int u = w - h * units;
        write_unit(read_unit(x + n * ldx + (int64_t)h * D, D, r.half, r.pairs, u), y + n * ldy + (int64_t)h * D, D, r.half, r.pairs, u, cs + t * r.half);
    }
}

// tokens of a workgroup: enough units for its threads, as long as their cosines fit
int tokens_of_group(int64_t row_units, int half)
{
    int t = (int)(kThreads / row_units);
    if (half > 0 && t > kTurnTable / half) t = kTurnTable / half;
    return t < 1 ? 1 : t > kMaxTokens ? kMaxTokens : t;
}

// ---- appending --------------------------------------------------------------------------------

// The queries of all heads, the keys and values of a token: bf16 cache.
template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const S *q, int64_t ldq, int Hq, const S *k, int64_t ldk, const S *v, int64_t ldv, int N, KvCache c, KvBatch b,
                                                            Rotation r, T *qo, int64_t ldqo, int tokens)
{
    __shared__ float2_t cs[kTurnTable];
    __shared__ int64_t base[kMaxTokens];        // of the token in its page, head 0; -1: no place
    __shared__ int seen[kMaxTokens];            // whether the row has a place in a sequence
    __shared__ int position[kMaxTokens];
    const int n0 = blockIdx.x * tokens, count = min(tokens, N - n0);
    const int units = units_of(c.D, r.half), plain = c.D >> 3;
    const int uq = Hq * units, uk = c.heads * units, row = uq + uk + c.heads * plain;
    if ((int)threadIdx.x < count) {
        int seq;
        const int place = place_of(b, c, n0 + threadIdx.x, N, seq);
        const int page = place < 0 ? -1 : page_of(b, c, seq, place);
        seen[threadIdx.x] = place >= 0;
        position[threadIdx.x] = place + b.prefix;
        base[threadIdx.x] = page < 0 ? -1 : ((((int64_t)page * c.heads) << c.page_log2) + (place & ((1 << c.page_log2) - 1))) * c.D;
    }
    __syncthreads();
    if (r.half > 0) {
        for (int i = threadIdx.x; i < count * r.half; i += kThreads) {
            const int t = i / r.half;
            cs[i] = turn_of(r, position[t], i - t * r.half, 0);
        }
        __syncthreads();
    }
    const int64_t head_stride = (int64_t)c.D << c.page_log2;
    uint16_t *const ck = static_cast<uint16_t *>(c.k), *const cv = static_cast<uint16_t *>(c.v);
    for (int i = threadIdx.x; i < count * row; i += kThreads) {
        const int t = i / row;
        int w = i - t * row;
        const int64_t n = n0 + t;
        if (!seen[t]) continue;
        if (w < uq) {
            const int h = w / units, u = w - h * units;
            write_unit(read_unit(q + n * ldq + (int64_t)h * c.D, c.D, r.half, r.pairs, u), qo + n * ldqo + (int64_t)h * c.D, c.D, r.half, r.pairs, u, cs + t * r.half);
            continue;
        }
        if (base[t] < 0) continue;
        w -= uq;
        if (w < uk) {
            const int h = w / units, u = w - h * units;
            write_unit(read_unit(k + n * ldk + (int64_t)h * c.D, c.D, r.half, r.pairs, u), ck + base[t] + h * head_stride, c.D, r.half, r.pairs, u, cs + t * r.half);
        } else {
            w -= uk;
            const int h = w / plain, at = 8 * (w - h * plain);
            float e[8];
            widen(raw8(v + n * ldv + (int64_t)h * c.D + at, 8), e);
            put8(cv + base[t] + h * head_stride + at, 8, e);
        }
    }
}

// Keys and values of a token into an 8-bit cache.  Keys lie in LDS in binary32 and are turned there, a thread a pair; then 16 lanes take the up to 128 elements that share a power of
// two.  blockIdx.y: which key heads, `slice` of them; the query heads in as many parts.
template <typename S, typename T>
__global__ __launch_bounds__(kThreads) void kv_append8_kernel(const S *q, int64_t ldq, int Hq, const S *k, int64_t ldk, const S *v, int64_t ldv, int N, KvCache c, KvBatch b,
                                                             Rotation r, T *qo, int64_t ldqo, int slice, Quotient units, Quotient half)
{
    __shared__ float2_t cs[kMaxHeadDim / 2];
    __shared__ Turn64 cs64[kMaxHeadDim / 2];
    __shared__ __align__(16) float keys[kSliceElems];
    const int n = blockIdx.x, t = threadIdx.x;
    const int h0 = blockIdx.y * slice, heads = min(slice, c.heads - h0);
    const int q0 = (int)((int64_t)Hq * blockIdx.y / gridDim.y), q1 = (int)((int64_t)Hq * (blockIdx.y + 1) / gridDim.y);
    const int uq = (q1 - q0) * units.by, shift = c.groups == 1 ? 4 : 5;        // 16 or 32 lanes a head where its elements are rounded
    const S *const qn = q + n * ldq + (int64_t)q0 * c.D, *const kn = k + n * ldk + (int64_t)h0 * c.D, *const vn = v + n * ldv + (int64_t)h0 * c.D;
    const auto read_query = [&](int i) {
        const int h = units(i);
        return read_unit(qn + (int64_t)h * c.D, c.D, r.half, r.pairs, i - h * units.by);
    };
    const auto read_value = [&](int i) {
        const int h = i >> shift, at = 8 * (i - (h << shift));
        return raw8(vn + (int64_t)h * c.D + at, c.D - at);
    };
    // what the thread loads first is on its way while the place is looked up
    Unit<S> qu;
    RawOf<S> vu;
    if (t < heads << shift) vu = read_value(t);
    if (t < uq) qu = read_query(t);
    for (int i = t; i < heads * (c.D / 8); i += kThreads) {
        float e[8];
        widen(raw8(kn + 8 * i, 8), e);
        put8(keys + 8 * i, 8, e);
    }
    int seq;
    const int place = place_of(b, c, n, N, seq);
    if (place < 0) return;
    const int page = page_of(b, c, seq, place);
    for (int j = t; j < r.half; j += kThreads) {
        Turn64 x = cos_sin64(place + b.prefix, r.freqs[j]);
        x.x *= (double)r.scale, x.y *= (double)r.scale;
        cs64[j] = x;
        cs[j] = float2_t{(float)x.x, (float)x.y};
    }
    __syncthreads();
    for (int i = t; i < heads * r.half; i += kThreads) {
        const int h = half(i), j = i - h * r.half;
        float *const a = keys + h * c.D + (r.pairs ? 2 * j : j), *const z = a + (r.pairs ? 1 : r.half);
        float x = *a, y = *z;
        turn_pair(x, y, cs64[j]);
        *a = x, *z = y;
    }
    for (int i = t; i < uq; i += kThreads) {
        const int h = units(i);
        if (i >= kThreads) qu = read_query(i);
        write_unit(qu, qo + n * ldqo + (int64_t)(q0 + h) * c.D, c.D, r.half, r.pairs, i - h * units.by, cs);
    }
    if (page < 0) return;
    __syncthreads();
    const int slot = place & ((1 << c.page_log2) - 1);
    // Every lane of 16 that share a group come by together: the count is a multiple of 16.
    for (int i = t; i < heads << shift; i += kThreads) {
        const int h = i >> shift, at = 8 * (i - (h << shift));
        const int64_t row = (((int64_t)page * c.heads + h0 + h) << c.page_log2) + slot;
        float e[8] = {};
        if (at < c.D) widen(raw8(keys + h * c.D + at, 8), e);
        ckpt_store8<false>(CkptOut{static_cast<uint8_t *>(c.k), c.k_exps, c.groups}, row, at, c.D, e);
        if (i >= kThreads) vu = read_value(i);
        widen(vu, e);
        ckpt_store8<false>(CkptOut{static_cast<uint8_t *>(c.v), c.v_exps, c.groups}, row, at, c.D, e);
    }
}

// ---- reading back -----------------------------------------------------------------------------

template <int KIND, bool F32>
__global__ __launch_bounds__(kThreads) void kv_load_kernel(KvCache c, KvBatch b, int N, RowDst k, RowDst v)
{
    const int n = blockIdx.x;
    int seq;
    const int place = place_of(b, c, n, N, seq);
    if (place < 0) return;
    const int page = page_of(b, c, seq, place);
    const int chunks = c.D >> 3, slot = place & ((1 << c.page_log2) - 1);
    for (int i = threadIdx.x; i < 2 * c.heads * chunks; i += kThreads) {
        const int value = i >= c.heads * chunks;
        const int w = i - value * c.heads * chunks, h = w / chunks, at = 8 * (w - h * chunks);
        float e[8] = {};
        if (page >= 0) {
            const RowSrc s{value ? c.v : c.k, value ? c.v_exps : c.k_exps, c.D, c.groups, KIND};
            widen(load8<KIND, false, false>(s, (((int64_t)page * c.heads + h) << c.page_log2) + slot, at, c.D), e);
        }
        const RowDst &o = value ? v : k;
        store8<F32, false>(o.p, o.ld, n, h * c.D + at, c.heads * c.D, e);
    }
}

template <typename S, typename T>
hipError_t run_rope(const RowSrc &x, const int *pos, int64_t N, int64_t H, int64_t D, const Rotation &r, int inverse, const RowDst &y, hipStream_t st)
{
    const int units = units_of((int)D, r.half);
    const int64_t row_units = H * units;
    const int tokens = tokens_of_group(row_units, r.half);
    rope_kernel<S, T><<<(unsigned)((N + tokens - 1) / tokens), kThreads, 0, st>>>(static_cast<const S *>(x.p), x.ld, pos, (int)N, (int)D, units, (int)row_units, tokens, r,
                                                                                  inverse, static_cast<T *>(y.p), y.ld);
    return hipGetLastError();
}

template <typename S, typename T>
hipError_t run_append(const RowSrc &q, int Hq, const RowSrc &k, const RowSrc &v, int64_t N, const KvCache &c, const KvBatch &b, const Rotation &r, const RowDst &qo,
                      hipStream_t st)
{
    const S *const qp = static_cast<const S *>(q.p), *const kp = static_cast<const S *>(k.p), *const vp = static_cast<const S *>(v.p);
    T *const op = static_cast<T *>(qo.p);
    if (c.bits8) {
        const int fit = kSliceElems / c.D, slice = fit < c.heads ? fit : c.heads;
        const dim3 grid((unsigned)N, (unsigned)((c.heads + slice - 1) / slice));
        kv_append8_kernel<S, T><<<grid, kThreads, 0, st>>>(qp, q.ld, Hq, kp, k.ld, vp, v.ld, (int)N, c, b, r, op, qo.ld, slice, quotient(units_of(c.D, r.half)),
                                                          quotient(r.half > 0 ? r.half : 1));
    } else {
        const int64_t row_units = (int64_t)(Hq + c.heads) * units_of(c.D, r.half) + (int64_t)c.heads * (c.D / 8);
        const int tokens = tokens_of_group(row_units, r.half);
        kv_append_kernel<S, T><<<(unsigned)((N + tokens - 1) / tokens), kThreads, 0, st>>>(qp, q.ld, Hq, kp, k.ld, vp, v.ld, (int)N, c, b, r, op, qo.ld, tokens);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RowSrc &x, const int *pos, int64_t N, int64_t H, int64_t D, const Rotation &r, int inverse, const RowDst &y, hipStream_t st)
{
    if (x.kind == kF32) return y.f32 ? run_rope<float, float>(x, pos, N, H, D, r, inverse, y, st) : run_rope<float, uint16_t>(x, pos, N, H, D, r, inverse, y, st);
    return y.f32 ? run_rope<uint16_t, float>(x, pos, N, H, D, r, inverse, y, st) : run_rope<uint16_t, uint16_t>(x, pos, N, H, D, r, inverse, y, st);
}

hipError_t launch_kv_append(const RowSrc &q, int Hq, const RowSrc &k, const RowSrc &v, int64_t N, const KvCache &c, const KvBatch &b, const Rotation &r,
                            const RowDst &qo, hipStream_t st)
{
    if (k.kind == kF32) return qo.f32 ? run_append<float, float>(q, Hq, k, v, N, c, b, r, qo, st) : run_append<float, uint16_t>(q, Hq, k, v, N, c, b, r, qo, st);
    return qo.f32 ? run_append<uint16_t, float>(q, Hq, k, v, N, c, b, r, qo, st) : run_append<uint16_t, uint16_t>(q, Hq, k, v, N, c, b, r, qo, st);
}

hipError_t launch_kv_load(const KvCache &c, const KvBatch &b, int64_t N, const RowDst &k, const RowDst &v, hipStream_t st)
{
    const unsigned grid = (unsigned)N;
    if (c.bits8) {
        if (k.f32) kv_load_kernel<kCkpt8, true><<<grid, kThreads, 0, st>>>(c, b, (int)N, k, v);
        else kv_load_kernel<kCkpt8, false><<<grid, kThreads, 0, st>>>(c, b, (int)N, k, v);
    } else {
        if (k.f32) kv_load_kernel<kBf16, true><<<grid, kThreads, 0, st>>>(c, b, (int)N, k, v);
        else kv_load_kernel<kBf16, false><<<grid, kThreads, 0, st>>>(c, b, (int)N, k, v);
    }
    return hipGetLastError();
}

}  // namespace tj
