// The choice of one token per row of logits x [N x V] from a given number u.
//
//   w = exp((x - max) / T);  order: by x from the largest down, equal ones by index;  kept: a run of the order from its first token on, as long as top_k,
//   top_p and min_p let it be;  W = sum of the kept w;  the token is the first whose sum of w with those before it exceeds u W.
//
// Nothing is sorted.  The order is cut into bins 1/32 of a unit of x / T wide (a function of x that never falls as x grows, whatever it is rounded to), and a bin's weight and number of tokens say which bin a
// border lies in: one kernel makes the bins of slices of a row, a second joins them and takes from the row the tokens of the few bins that matter, a third finds the places inside these
// bins by further cuts, of the number (x, index) of 52 bits that the order goes by.
//
// Medians of the three kernels: one row of 50021 logits 8.8 + 10.1 + 11.9 us, 64 rows of 131072 in binary32 (33.6 MB) 18.4 + 16.8 + 10.2, of which 64-bit exponentials take 8.
//
// Weights are fixed-point numbers, 2^43 for the largest: their sums do not depend on the order of the additions, which LDS atomics leave open.
#include "rowwise.h"
#include "seq_ops.h"

namespace tj {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 1024;                   // the last one: 31.9 and more below the largest, where weights are 0
constexpr int kChoose = 512;                  // threads that draw from a row's list
constexpr int kCuts = kChoose;                // cuts of a bin
constexpr int kCutBits = 9;
constexpr int kIndexBits = 20;                // of a token in a row: V is at most 2^20
constexpr int kFew = 64;                      // tokens among which a wave finds the place
constexpr int kList = 8192;                   // tokens that are taken out of a row; where there are more, they stay in it
constexpr int kSliceList = 4096;              // and out of a slice
constexpr int kMaxSlices = 8;
constexpr int kKept = 2;                      // runs of eight logits that a thread keeps between its two walks over them
constexpr double kOne = 8796093022208.0;      // 2^43

// what a slice leaves
struct Slice {
    float top;                // its largest logit
    int index;                // where that is first
};

struct Weight {
    double top, step;         // largest logit, log2 e / T
    // round(2^43 * 2^(-(top - x) step)).  The Taylor series of 2^-f about f = 1/2 to degree 11 is off by 2^-47 of it: the largest weight comes out as 2^43.
    __device__ __forceinline__ uint64_t operator()(float x) const
    {
        const double y = fmin((top - (double)x) * step, 46.0);                  // 46 and more, and no number (of -infinity): 0
        const double n = floor(y), z = (0.5 - (y - n)) * 0.69314718055994530942;
        double p = 1.0 / 39916800;
        p = fma(p, z, 1.0 / 3628800);
        p = fma(p, z, 1.0 / 362880);
        p = fma(p, z, 1.0 / 40320);
        p = fma(p, z, 1.0 / 5040);
        p = fma(p, z, 1.0 / 720);
        p = fma(p, z, 1.0 / 120);
        p = fma(p, z, 1.0 / 24);
        p = fma(p, z, 1.0 / 6);
        p = fma(p, z, 0.5);
        p = fma(p, z, 1.0);
        p = fma(p, z, 1.0);
        // times 2^(43 - n) / sqrt 2, and rounded to an integer in the low bits of a number from 2^52 on
        const double scale = __longlong_as_double((long long)(1023 + 43 - (int)n) << 52) * 0.70710678118654752440;
        return (uint64_t)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
    }
};

// Bin number of a logit, counted from the row's own zero upwards.  NaN and -infinity have the lowest, which is also that of logits far below zero: who counts tokens leaves them out by
// their value.
__device__ __forceinline__ float bin_of(float x, float per_unit)
{
    return floorf(fminf(fmaxf(x * per_unit, -0x1p30f), 0x1p30f));
}
__device__ __forceinline__ int bin_below(float anchor, float x, float per_unit)
{
    return (int)fminf(anchor - bin_of(x, per_unit), (float)(kBins - 1));
}
// bins per unit of x: 32 / T, and no more than 2^20, with which the last bin's weights are 0 still
__device__ __forceinline__ float bins_per_unit(float T) { return fminf(32.0f / T, 0x1p20f); }

__device__ __forceinline__ float temperature_of(const SampleArgs &a, int64_t n) { return a.temperature ? a.temperature[n] : 1.0f; }
__device__ __forceinline__ bool is_greedy(float T) { return !(T > 0.0f); }
__device__ __forceinline__ double share_of(float u) { return u > 0.0f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0; }

// A logit as the order sees it: NaN as -infinity, -0 as 0; where the largest is +infinity, 0 for it and -infinity for everything else.
__device__ __forceinline__ float seen(float x, bool infinite)
{
    if (infinite) return x == INFINITY ? 0.0f : -INFINITY;
    return x != x ? -INFINITY : x + 0.0f;
}

// eight logits from `at` on, -infinity behind the end
template <bool F32> __device__ __forceinline__ void logits8(const SampleArgs &a, int64_t row, int at, int end, float (&v)[8])
{
    const RowSrc s{a.logits, nullptr, a.ld, 0, F32 ? kF32 : kBf16};
    if (at + 8 <= end) {
        widen(load8<F32 ? kF32 : kBf16, true, false>(s, row, at, at + 8), v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = -INFINITY;
        if (at + i < end) {
            if constexpr (F32) v[i] = static_cast<const float *>(a.logits)[row * a.ld + at + i];
            else v[i] = u2f((uint32_t) static_cast<const uint16_t *>(a.logits)[row * a.ld + at + i] << 16);
        }
    }
}

// the larger logit, of equal ones the one that comes first
__device__ __forceinline__ void larger(float &x, int &at, float y, int where)
{
    if (y > x || (y == x && where < at)) x = y, at = where;
}

// What the second kernel says of a row: its bins joined, which of them hold a border, and their tokens.
struct RowBins {
    double ends[kBins];        // weight of the row's tokens up to and with each bin
    uint32_t count_ends[kBins];
    uint32_t keys[kList], index[kList];
    uint32_t listed;           // tokens in the list; more than kList: some were left out
    int by_k, by_p, by_m;
    int k0, p0, p1, m0, m1, u0, u1;       // first and last bin in which the border can lie
};

// ws: what is said of each row, then of each row its slices, their bins' weights and numbers of tokens
struct Space {
    RowBins *rows;
    uint64_t *sums;            // [N][slices][kBins]
    uint32_t *counts;
    Slice *slices;             // [N][slices]
};
Space space_of(void *ws, int64_t N, int slices)
{
    Space s;
    s.rows = static_cast<RowBins *>(ws);
    s.sums = reinterpret_cast<uint64_t *>(s.rows + N);
    s.counts = reinterpret_cast<uint32_t *>(s.sums + N * slices * kBins);
    s.slices = reinterpret_cast<Slice *>(s.counts + N * slices * kBins);
    return s;
}
size_t space_bytes(int64_t N, int slices) { return (size_t)N * (sizeof(RowBins) + (size_t)slices * (kBins * 12 + sizeof(Slice))); }

template <bool F32> __global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a, Space ws, int slices, int slice_len)
{
    __shared__ uint64_t sums[kBins];
    __shared__ uint32_t counts[kBins];
    __shared__ float tops[kWaves];
    __shared__ int where[kWaves];
    const int64_t row = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, begin = slice * slice_len, end = min((int)a.V, begin + slice_len);
    float top = -INFINITY;
    int at = 0x7FFFFFFF;
    float kept[kKept][8];                         // a thread's first logits, for the second walk
#pragma unroll
    for (int c = 0; c < kKept; ++c) {
        const int i = begin + 8 * (threadIdx.x + c * kThreads);
        if (i < end) logits8<F32>(a, row, i, end, kept[c]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) kept[c][j] = -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (kept[c][j] > top) top = kept[c][j], at = i + j;
    }
    for (int i = begin + 8 * (threadIdx.x + kKept * kThreads); i < end; i += 8 * kThreads) {
        float v[8];
        logits8<F32>(a, row, i, end, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (v[j] > top) top = v[j], at = i + j;
    }
    for (int o = 1; o < 64; o <<= 1) larger(top, at, __shfl_xor(top, o, 64), __shfl_xor(at, o, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top, where[threadIdx.x >> 6] = at;
    sums[threadIdx.x] = 0;
    counts[threadIdx.x] = 0;
    __syncthreads();
    top = tops[0], at = where[0];
    for (int w = 1; w < kWaves; ++w) larger(top, at, tops[w], where[w]);
    if (threadIdx.x == 0) {
        ws.slices[blockIdx.x] = Slice{top, at};
        if (slice == 0) ws.rows[row].listed = 0;
    }
    const float T = temperature_of(a, row);
    if (is_greedy(T) || top == -INFINITY) return;
    const bool infinite = top == INFINITY, count = a.top_k != nullptr;
    if (infinite) top = 0.0f;
    const Weight weight{(double)top, 1.44269504088896340736 / (double)T};
    const float per_unit = bins_per_unit(T), anchor = bin_of(top, per_unit);
    const auto add = [&](float (&v)[8]) {
        if (infinite) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = seen(v[j], true);
        }
        uint64_t w[8];
        int b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = weight(v[j]);
            b[j] = bin_below(anchor, v[j], per_unit);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (b[j] < kBins - 1 && v[j] > -INFINITY) {
                atomicAdd(reinterpret_cast<unsigned long long *>(&sums[b[j]]), (unsigned long long)w[j]);
                if (count) atomicAdd(&counts[b[j]], 1u);
            }
    };
#pragma unroll
    for (int c = 0; c < kKept; ++c)
        if (begin + 8 * c * kThreads < end) add(kept[c]);
    for (int i = begin + 8 * (threadIdx.x + kKept * kThreads); i < end; i += 8 * kThreads) {
        float v[8];
        logits8<F32>(a, row, i, end, v);
        add(v);
    }
    __syncthreads();
    ws.sums[(int64_t)blockIdx.x * kBins + threadIdx.x] = sums[threadIdx.x];
    if (count) ws.counts[(int64_t)blockIdx.x * kBins + threadIdx.x] = counts[threadIdx.x];
}

// (Weight, number of tokens) up to and with each thread's; all threads of the workgroup call it.  In integers: a thread without tokens has the sum of the one in front of it, however the
// additions are grouped, so that no sum is between the two and a place looked up by one always holds a token.
template <int WAVES> __device__ __forceinline__ void scan(uint64_t &w, uint32_t &c, uint64_t *lw, uint32_t *lc)
{
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up((unsigned long long)w, o, 64);
        const uint32_t y = __shfl_up(c, o, 64);
        const bool in = (int)(threadIdx.x & 63) >= o;
        w += in ? x : 0, c += in ? y : 0;
    }
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lw[wave] = w, lc[wave] = c;
    __syncthreads();
    uint64_t x = 0;
    uint32_t y = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i)
        if (i < wave) x += lw[i], y += lc[i];
    w += x, c += y;
}

// A row as its second kernel sees it.
struct Row {
    Weight weight;
    float per_unit, anchor;
    bool infinite;
    int64_t row;
    int listed;                // tokens in the list; -1: there were more than it holds, and they are looked up in the row
};

struct Shared {
    double ends[kBins];        // of RowBins
    uint32_t count_ends[kBins];
    uint32_t keys[kList], index[kList];
    uint64_t weights[kList];
    uint64_t sums[kCuts];
    uint32_t counts[kCuts];
    uint64_t lw[kWaves];
    uint32_t lc[kWaves];
    uint64_t few[kFew], few_weight[kFew];
    double found[2];
    int cut, bin;
    uint32_t n;
    int token;
};

// The row's largest logit, its temperature and what follows from them; false: the token is `token`, without a draw.
__device__ __forceinline__ bool row_of(const SampleArgs &a, const Space &ws, int64_t row, int slices, Row &r, float (&tops)[kMaxSlices], int64_t &token)
{
    float top = -INFINITY;
    int at = 0x7FFFFFFF;
    Slice s[kMaxSlices];
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i) s[i] = i < slices ? ws.slices[row * slices + i] : Slice{-INFINITY, 0x7FFFFFFF};
    const float T = temperature_of(a, row);
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i) {
        larger(top, at, s[i].top, s[i].index);
        tops[i] = s[i].top;
    }
    token = top == -INFINITY ? -1 : at;
    if (top == -INFINITY || is_greedy(T)) return false;
    r.infinite = top == INFINITY;
    if (r.infinite) {
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kMaxSlices; ++i) tops[i] = tops[i] == INFINITY ? 0.0f : -INFINITY;
    }
    r.weight = Weight{(double)top, 1.44269504088896340736 / (double)T};
    r.per_unit = bins_per_unit(T);
    r.anchor = bin_of(top, r.per_unit);
    r.row = row;
    r.listed = -1;
    return true;
}

// ascending with the order: larger logits have smaller numbers
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = f2u(x);
    return b & 0x80000000u ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t index) { return (uint64_t)key << kIndexBits | index; }
__device__ __forceinline__ float logit_of(uint32_t k) { return u2f(k & 0x80000000u ? k : ~k & 0x7FFFFFFFu); }

// what(place in the order as a number, logit, weight) for every token of bin `bin`
template <bool F32, typename Do> __device__ __forceinline__ void each(const SampleArgs &a, const Row &r, Shared &s, int bin, Do &&what)
{
    if (r.listed >= 0) {
        for (int i = threadIdx.x; i < r.listed; i += kChoose) {
            const float x = logit_of(s.keys[i]);
            if (bin_below(r.anchor, x, r.per_unit) == bin) what(place_of(s.keys[i], s.index[i]), x, s.weights[i]);
        }
    } else {
        // many of these logits are equal, and their weight is made once
        float last = INFINITY;
        uint64_t weight = 0;
        for (int i = 8 * threadIdx.x; i < (int)a.V; i += 8 * kChoose) {
            float v[8];
            logits8<F32>(a, r.row, i, (int)a.V, v);
            for (int j = 0; j < 8; ++j) {
                const float x = seen(v[j], r.infinite);
                if (x == -INFINITY || bin_below(r.anchor, x, r.per_unit) != bin) continue;
                if (x != last) last = x, weight = r.weight(x);
                what(place_of(key_of(x), (uint32_t)(i + j)), x, weight);
            }
        }
    }
}

// The token of bin `bin` that `target` falls on: by weight the first with which the sum of weights exceeds it, by rank the target-th of the order (counted from 0).  s.found: the
// weight of what comes before it, and with it; s.token: which it is.  All threads of the workgroup call it.
template <bool F32, bool RANK> __device__ void locate(const SampleArgs &a, const Row &r, Shared &s, int bin, double target)
{
    double before = bin ? s.ends[bin - 1] : 0.0;
    uint32_t rank = bin ? s.count_ends[bin - 1] : 0;
    // The numbers that the bin's tokens can have, from its edges (a little wider, for the product's rounding); everything where the bin's number was limited, or has no edges.
    uint64_t low = 0, high = (1ull << (32 + kIndexBits)) - 1;
    {
        const double f = (double)r.anchor - bin, per = (double)r.per_unit, up = (f + 1.0) / per, down = f / per;
        if (fabs(f) < 0x1p29 && fabs(up) < 0x1p126 && fabs(down) < 0x1p126) {
            low = place_of(key_of((float)(up + fabs(up) * 0x1p-20 + 0x1p-126)), 0);
            high = place_of(key_of((float)(down - fabs(down) * 0x1p-20 - 0x1p-126)), (1u << kIndexBits) - 1);
        }
    }
    const uint64_t span = high - low;
    int shift = span >> kCutBits ? 64 - kCutBits - __clzll((long long)span) : 0;           // span >> shift < kCuts
    __syncthreads();
    for (;;) {
        s.sums[threadIdx.x] = 0;
        s.counts[threadIdx.x] = 0;
        if (threadIdx.x == 0) s.cut = -1;
        __syncthreads();
        // What a thread has for one cut is held back until it meets another: where a row is searched whole most tokens fall into the same one, and additions to it follow each other
        // (131072 equal logits: a quarter of the time, with weights of equal logits made once; 0.58 ms with top_p).
        uint64_t held = 0;
        uint32_t many = 0;
        int held_cut = 0;
        const auto give = [&] {
            if (!many) return;
            atomicAdd(reinterpret_cast<unsigned long long *>(&s.sums[held_cut]), (unsigned long long)held);
            atomicAdd(&s.counts[held_cut], many);
        };
        each<F32>(a, r, s, bin, [&](uint64_t k, float, uint64_t weight) {
            const uint64_t c = (k - low) >> shift;
            if (k < low || c >= kCuts) return;
            if (r.listed >= 0) {
                atomicAdd(reinterpret_cast<unsigned long long *>(&s.sums[c]), (unsigned long long)weight);
                atomicAdd(&s.counts[c], 1u);
                return;
            }
            if ((int)c != held_cut) {
                give();
                held = 0, many = 0, held_cut = (int)c;
            }
            held += weight, ++many;
        });
        give();
        __syncthreads();
        const uint32_t here = s.counts[threadIdx.x];
        const uint64_t own = s.sums[threadIdx.x];
        uint64_t sum = own;
        uint32_t c = here;
        scan<kChoose / 64>(sum, c, s.lw, s.lc);
        c += rank;
        // The first cut with which the sum passes the target; the last one that weighs anything where none does.
        const bool some = RANK ? here > 0 : own > 0;
        const uint64_t any = __ballot(some), passes = __ballot(some && (RANK ? (double)c > target : before + (double)sum > target));
        if ((threadIdx.x & 63) == 0) {
            if (passes) atomicMax(&s.cut, 2 * kCuts - ((int)threadIdx.x + __ffsll((unsigned long long)passes) - 1));
            else if (any) atomicMax(&s.cut, (int)threadIdx.x + 63 - __clzll((long long)any));
        }
        __syncthreads();
        const int cut = s.cut >= kCuts ? 2 * kCuts - s.cut : s.cut;
        if ((int)threadIdx.x == cut) s.found[0] = before + (double)(sum - own), s.n = c - here;
        __syncthreads();
        before = s.found[0];
        rank = s.n;
        low += (uint64_t)cut << shift;
        const uint32_t tokens = s.counts[cut];
        __syncthreads();
        if (tokens <= kFew) break;                           // with shift = 0 there is one
        shift = shift > kCutBits ? shift - kCutBits : 0;
    }
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    each<F32>(a, r, s, bin, [&](uint64_t k, float, uint64_t weight) {
        if (k < low || (k - low) >> shift) return;
        const uint32_t i = atomicAdd(&s.n, 1u);
        s.few[i] = k;
        s.few_weight[i] = weight;
    });
    __syncthreads();
    if (threadIdx.x < 64) {
        const int n = (int)s.n, i = threadIdx.x;
        uint64_t sum = 0, behind = 0;
        uint32_t at = 0;
        if (i < n) {
            for (int j = 0; j < n; ++j) {
                if (s.few[j] < s.few[i]) sum += s.few_weight[j], ++at;
                else behind += s.few_weight[j];
            }
            const double b = before + (double)sum, e = before + (double)(sum + s.few_weight[i]);
            // the first that passes the target; if none does, the last that weighs anything
            const bool passes = RANK ? (double)(rank + at) == target : e > target && !(b > target && at > 0);
            const bool last = !RANK && e <= target && s.few_weight[i] > 0 && behind == s.few_weight[i];
            if (passes || last) s.found[0] = b, s.found[1] = e, s.token = (int)(s.few[i] & ((1u << kIndexBits) - 1));
        }
    }
    __syncthreads();
}

// Joins the bins of a row's slices, says which of them hold the borders, and lists the slice's tokens in them.
template <bool F32> __global__ __launch_bounds__(kThreads) void sample_list_kernel(SampleArgs a, Space ws, int slices, int slice_len)
{
    __shared__ double ends[kBins];
    __shared__ uint32_t count_ends[kBins];
    __shared__ uint32_t keys[kSliceList], index[kSliceList];
    __shared__ double factors[kMaxSlices];
    __shared__ uint64_t lw[kWaves];
    __shared__ uint32_t lc[kWaves], n, base;
    __shared__ int bins[8];
    const int64_t row = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, t = threadIdx.x;
    const int begin_at = slice * slice_len, end = min((int)a.V, begin_at + slice_len);
    float ahead[8];                               // the thread's first logits, on their way while the bins are joined
    if (begin_at + 8 * t < end) logits8<F32>(a, row, begin_at + 8 * t, end, ahead);
    Row r;
    float tops[kMaxSlices];
    int64_t token;
    if (!row_of(a, ws, row, slices, r, tops, token)) return;
    const int k = a.top_k ? a.top_k[row] : 0;
    float p = a.top_p ? a.top_p[row] : 1.0f, m = a.min_p ? a.min_p[row] : 0.0f;
    const double u = share_of(a.u[row]);
    if (t < kMaxSlices) {
        float top = tops[0];
#pragma unroll
        for (int i = 1; i < kMaxSlices; ++i) top = t == i ? tops[i] : top;
        factors[t] = exp2(-(r.weight.top - (double)top) * r.weight.step);
    }
    if (t < 8) bins[t] = -1;
    if (t == 0) n = 0;
    // The slices' bins, moved to where they lie below the row's largest logit and scaled by their own.
    uint64_t sums[kMaxSlices];
    uint32_t counts[kMaxSlices];
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i) {
        const float off = tops[i] == -INFINITY ? (float)kBins : r.anchor - bin_of(tops[i], r.per_unit);
        const int b = t - (int)fminf(off, (float)kBins);
        const bool some = b >= 0 && t < kBins - 1;
        const int64_t at = (row * slices + i) * kBins + b;
        sums[i] = some ? ws.sums[at] : 0;
        counts[i] = some && a.top_k ? ws.counts[at] : 0;
    }
    __syncthreads();
    uint64_t own = 0;
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i) {
        if (sums[i]) own += (uint64_t)((double)sums[i] * factors[i]);
        c += counts[i];
    }
    uint64_t sum = own;
    const uint32_t own_count = c;
    scan<kWaves>(sum, c, lw, lc);
    const double w = (double)sum;
    ends[t] = w;
    count_ends[t] = c;
    __syncthreads();
    const double total = ends[kBins - 1], begin = t ? ends[t - 1] : 0.0;
    const uint32_t tokens = count_ends[kBins - 1];
    // bins[i]: the bin that a sum falls in, the last one with weight where it is beyond all
    const auto bin_at = [&](int i, double sum) {
        if (own > 0 && begin <= sum && (sum < w || w >= total)) bins[i] = t;
    };
    const bool by_k = k >= 1 && (uint32_t)k < tokens, by_p = p < 1.0f, by_m = m > 0.0f;
    p = p > 0.0f ? p : 0.0f;
    m = fminf(m, 1.0f);
    if (by_k && own_count && c - own_count < (uint32_t)k && (uint32_t)k <= c) bins[0] = t;
    __syncthreads();
    const int k0 = bins[0];
    const double least_k = by_k ? (k0 ? ends[k0 - 1] : 0.0) : total, most_k = by_k ? ends[k0] : total;
    if (by_p) bin_at(1, (double)p * least_k), bin_at(2, (double)p * most_k);
    // the border of min_p is at log2(1 / m) / step below the largest logit; one bin more on either side, for the roundings
    int m0 = kBins - 2, m1 = kBins - 2;
    if (by_m) {
        const float edge = (float)(r.weight.top + log2((double)m) / r.weight.step);
        const int e = edge == edge ? bin_below(r.anchor, edge, r.per_unit) : 0;
        m0 = max(0, min(e - 1, kBins - 2)), m1 = max(0, min(e + 1, kBins - 2));
    }
    __syncthreads();
    const int p0 = bins[1], p1 = bins[2];
    double least = least_k, most = most_k;
    if (by_p) least = fmin(least, p0 ? ends[p0 - 1] : 0.0), most = fmin(most, ends[p1]);
    if (by_m) least = fmin(least, m0 ? ends[m0 - 1] : 0.0), most = fmin(most, ends[m1]);
    least = fmax(least, kOne), most = fmax(most, kOne);
    bin_at(3, u * least * (1.0 - 0x1p-40));
    bin_at(4, u * most * (1.0 + 0x1p-40));
    __syncthreads();
    const int u0 = bins[3], u1 = bins[4];
    RowBins &out = ws.rows[row];
    if (slice == 0) {
        out.ends[t] = w;
        out.count_ends[t] = c;
        if (t == 0) {
            out.by_k = by_k, out.by_p = by_p, out.by_m = by_m;
            out.k0 = k0, out.p0 = p0, out.p1 = p1, out.m0 = m0, out.m1 = m1, out.u0 = u0, out.u1 = u1;
        }
    }
    // lengths of the runs of bins, less one; without a border a run that no bin is in
    const uint32_t uk = u1 - u0, pk = p1 - p0, mk = m1 - m0;
    const int ks = by_k ? k0 : kBins, ps = by_p ? p0 : kBins, ms = by_m ? m0 : kBins;
    for (int i0 = begin_at; i0 < end; i0 += 8 * kThreads) {
        const int i = i0 + 8 * t;
        float v[8];
        uint32_t mine = 0;
        if (i < end) {
            if (i0 == begin_at) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = ahead[j];
            } else {
                logits8<F32>(a, row, i, end, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = seen(v[j], r.infinite);
                const int b = bin_below(r.anchor, v[j], r.per_unit);
                const bool wanted = (uint32_t)(b - u0) <= uk || b == ks || (uint32_t)(b - ps) <= pk || (uint32_t)(b - ms) <= mk;
                mine |= (uint32_t)(wanted && v[j] != -INFINITY) << j;
            }
        }
        if (!__any(mine)) continue;
        // places in the list: the lanes' numbers of tokens summed over the wave, one addition for all
        uint32_t at = __popc(mine);
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(at, o, 64);
            if ((t & 63) >= o) at += x;
        }
        uint32_t from = 0;
        if ((t & 63) == 63) from = atomicAdd(&n, at);
        at += __shfl(from, 63, 64) - __popc(mine);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (mine >> j & 1) {
                if (at < kSliceList) keys[at] = key_of(v[j]), index[at] = (uint32_t)(i + j);
                ++at;
            }
    }
    __syncthreads();
    const uint32_t many = n;
    if (many == 0) return;
    if (t == 0) base = atomicAdd(&out.listed, many > kSliceList ? kList + 1u : many);
    __syncthreads();
    const uint32_t to = base;
    for (uint32_t i = t; i < min(many, (uint32_t)kSliceList); i += kThreads)
        if (to + i < kList) out.keys[to + i] = keys[i], out.index[to + i] = index[i];
}

// The draw, from the joined bins and the listed tokens.
template <bool F32> __global__ __launch_bounds__(kChoose) void sample_choose_kernel(SampleArgs a, Space ws, int slices)
{
    __shared__ Shared s;
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    Row r;
    float tops[kMaxSlices];
    int64_t token;
    if (!row_of(a, ws, row, slices, r, tops, token)) {
        if (t == 0) a.tokens[row] = token;
        return;
    }
    const RowBins &in = ws.rows[row];
    const int k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? fmaxf(a.top_p[row], 0.0f) : 1.0f, m = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.0f;
    const double u = share_of(a.u[row]);
    const uint32_t listed = in.listed;
    for (int i = t; i < kBins; i += kChoose) s.ends[i] = in.ends[i], s.count_ends[i] = in.count_ends[i];
    for (uint32_t i = t; i < min(listed, (uint32_t)kList); i += kChoose) {
        const uint32_t key = in.keys[i];
        s.keys[i] = key, s.index[i] = in.index[i], s.weights[i] = r.weight(logit_of(key));
    }
    if (listed <= kList) r.listed = (int)listed;
    __syncthreads();
    const double total = s.ends[kBins - 1];
    // the bin in which a sum falls, from `first` to `last`
    const auto bin_of_sum = [&](double sum, int first, int last) {
        if (t == 0) s.bin = last;
        __syncthreads();
        for (int i = first + t; i < last; i += kChoose)
            if (sum < s.ends[i]) atomicMin(&s.bin, i);
        __syncthreads();
        return s.bin;
    };
    // what the filters leave, as a sum of weights
    double kept = total;
    if (in.by_k) {
        locate<F32, true>(a, r, s, in.k0, (double)(k - 1));
        kept = s.found[1];
    }
    if (in.by_p) {
        const double target = (double)p * kept;
        locate<F32, false>(a, r, s, bin_of_sum(target, in.p0, in.p1), target);
        kept = fmin(kept, s.found[0] == target ? s.found[0] : s.found[1]);
    }
    if (in.by_m) {
        // the tokens of the bins around the border that are heavy enough, after all those in front of them
        uint64_t sum = 0;
        for (int b = in.m0; b <= in.m1; ++b)
            each<F32>(a, r, s, b, [&](uint64_t, float x, uint64_t weight) {
                if (exp2(-(r.weight.top - (double)x) * r.weight.step) >= (double)m) sum += weight;
            });
        uint32_t none = 0;
        scan<kChoose / 64>(sum, none, s.lw, s.lc);
        if (t == kChoose - 1) s.found[0] = (double)sum + (in.m0 ? s.ends[in.m0 - 1] : 0.0);
        __syncthreads();
        kept = fmin(kept, s.found[0]);
    }
    kept = fmax(kept, kOne);                                 // the first token stays
    const double target = u * kept;
    locate<F32, false>(a, r, s, bin_of_sum(target, in.u0, in.u1), target);
    if (t == 0) a.tokens[row] = s.token;
}

// Slices of a row: enough workgroups for two a CU, as long as a slice gives each thread eight logits.
int slices_of(int64_t N, int64_t V)
{
    int64_t s = 512 / N;
    const int64_t most = V / (8 * kThreads);
    s = s < most ? s : most;
    return (int)(s < 1 ? 1 : s > kMaxSlices ? kMaxSlices : s);
}

template <bool F32> hipError_t run(const SampleArgs &a, void *ws, hipStream_t st)
{
    const int slices = slices_of(a.N, a.V);
    const int len = (int)(((a.V + slices - 1) / slices + 7) / 8 * 8);
    const Space space = space_of(ws, a.N, slices);
    sample_bins_kernel<F32><<<(unsigned)(a.N * slices), kThreads, 0, st>>>(a, space, slices, len);
    sample_list_kernel<F32><<<(unsigned)(a.N * slices), kThreads, 0, st>>>(a, space, slices, len);
    sample_choose_kernel<F32><<<(unsigned)a.N, kChoose, 0, st>>>(a, space, slices);
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int64_t N, int64_t V) { return space_bytes(N, slices_of(N, V)); }

hipError_t launch_sample(const SampleArgs &a, void *ws, hipStream_t st)
{
    return a.f32 ? run<true>(a, ws, st) : run<false>(a, ws, st);
}

}  // namespace tj
