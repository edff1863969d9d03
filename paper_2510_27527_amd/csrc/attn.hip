// Attention of a batch's rows over the paged cache of keys and values: tiles of 16 rows, and what joins the parts of all tiles.  (Formulas: attn_common.h.)
#include "attn_common.h"

namespace tj {

namespace {

constexpr int kTile = 16;                 // rows of a tile
constexpr int kBlock = 32;                // tokens that a wave takes at once

// Bound by memory where there is enough of it: 64 sequences of 1024 to 8192 tokens (8 key heads of 128, bf16) 220 us, 5.5 TB/s; one of 200000 tokens in 8 bits 76 us, 5.4 TB/s.  One of 1000 tokens
// takes 6.7 us, trips to memory that follow each other.  The join: 6.3 us for the 64, 5.6 for the one of 200000, 4.1 for the one of 1000.

__device__ __forceinline__ float max16_32(float v)             // over the four lanes that hold a row
{
    const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
    v = fmaxf(u2f(a[0]), u2f(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
    return fmaxf(u2f(b[0]), u2f(b[1]));
}
__device__ __forceinline__ float sum16_32(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
    v = u2f(a[0]) + u2f(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
    return u2f(b[0]) + u2f(b[1]);
}

// ---- a block of 32 tokens in registers ---------------------------------------------------------
// Products: scores^T [tokens x rows] = K Q^T and out^T [D x rows] += V^T P^T, 16 x 16 x 32 each.  The tokens of a block are dealt to the rows of the two score tiles so that lane
// (g, row) (g = lane / 16) ends up with tokens 8g .. 8g + 7 of its row, which is what the second product takes from it.  Values come as rows of tokens
// and are turned in registers: eight tokens x D / 16 elements a lane.
template <int DP, bool BITS8> struct Keys {
    static constexpr int STEPS = BITS8 ? DP / 64 : DP / 32;
    u32x4 k[2][STEPS];                                   // [tile][step]: eight elements a step of the product (8 bits: sixteen, two steps)
    uint32_t e[2];                                       // 8 bits: exponents of the lane's token of each tile, a byte a group
};
template <int DP, bool BITS8> struct Values {
    static constexpr int WORDS = BITS8 ? DP / 64 : DP / 32;
    uint32_t v[8][WORDS];                                // [token][elements]
    uint32_t e[4];                                       // 8 bits: exponents of the eight tokens
};
// Where the two halves of a block lie: first byte of the head's tokens 0 .. 15 and, less 16 tokens, 16 .. 31, counted in tokens; bit h of ok: half h lies in a page of the cache.
struct Spot {
    int64_t s0, s1;
    uint32_t ok;
};

__device__ __forceinline__ Spot spot_of(const KvCache &c, int head, int t0, int p0, int p1)
{
    const int mask = (1 << c.page_log2) - 1;
    return Spot{(((int64_t)(p0 < 0 ? 0 : p0) * c.heads + head) << c.page_log2) + (t0 & mask), (((int64_t)(p1 < 0 ? 0 : p1) * c.heads + head) << c.page_log2) + ((t0 + 16) & mask) - 16,
                (uint32_t)(p0 >= 0) | (uint32_t)(p1 >= 0) << 1};
}

template <int DP, bool BITS8> __device__ __forceinline__ void load_keys(const KvCache &c, Spot s, int lane, Keys<DP, BITS8> &r)
{
    constexpr int E = BITS8 ? 1 : 2, STEP = 64 / E;      // elements that four lanes take with 16 bytes each
    const int m = lane & 15, g = lane >> 4;
    const int64_t near = s.s0, far = s.s1;
    const int64_t token = (m < 8 ? near : far) + (m >> 2) * 8 + (m & 3);        // of the first tile's row m; the second has the one four further on
    const char *const p = static_cast<const char *>(c.k) + token * (c.D * E);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < Keys<DP, BITS8>::STEPS; ++i) {
            const int d = STEP * i + (16 / E) * g;
            r.k[t][i] = u32x4{0, 0, 0, 0};
            if (d < c.D) r.k[t][i] = *reinterpret_cast<const u32x4 *>(p + (4 * t * c.D + d) * E);
        }
    if constexpr (BITS8) {
        const uint8_t *const e = c.k_exps + token * c.groups;
        if constexpr (DP <= 128) r.e[0] = e[0], r.e[1] = e[4];
        else r.e[0] = *reinterpret_cast<const uint16_t *>(e), r.e[1] = *reinterpret_cast<const uint16_t *>(e + 8);
    }
}

template <int DP, bool BITS8> __device__ __forceinline__ void load_values(const KvCache &c, Spot s, int lane, Values<DP, BITS8> &r)
{
    constexpr int E = BITS8 ? 1 : 2, DV = DP / 16, W = Values<DP, BITS8>::WORDS;
    const int m = lane & 15, g = lane >> 4;
    const int64_t near = s.s0, far = s.s1;
    const int64_t token = (g < 2 ? near : far) + 8 * g;
    const char *const p = static_cast<const char *>(c.v) + token * (c.D * E) + DV * m * E;
    const bool there = DV * m < c.D;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t *const x = reinterpret_cast<const uint32_t *>(p + i * c.D * E);
#pragma unroll
        for (int w = 0; w < W; ++w) r.v[i][w] = 0;
        if (there) {
            if constexpr (W % 4 == 0) {
#pragma unroll
                for (int w = 0; w < W; w += 4) {
                    const u32x4 y = *reinterpret_cast<const u32x4 *>(x + w);
                    r.v[i][w] = y[0], r.v[i][w + 1] = y[1], r.v[i][w + 2] = y[2], r.v[i][w + 3] = y[3];
                }
            } else if constexpr (W == 2) {
                const u32x2 y = *reinterpret_cast<const u32x2 *>(x);
                r.v[i][0] = y[0], r.v[i][1] = y[1];
            } else {
                r.v[i][0] = x[0];
            }
        }
    }
    if constexpr (BITS8) {
        const uint8_t *const e = c.v_exps + token * c.groups;
        if constexpr (DP <= 128) {
            const u32x2 y = *reinterpret_cast<const u32x2 *>(e);
            r.e[0] = y[0], r.e[1] = y[1];
        } else {
            const u32x4 y = *reinterpret_cast<const u32x4 *>(e);
            r.e[0] = y[0], r.e[1] = y[1], r.e[2] = y[2], r.e[3] = y[3];
        }
    }
}

__device__ __forceinline__ float4_t mfma(u32x4 a, u32x4 b, float4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// state of 16 rows: lane (g, row) holds m and a part of l of its row, and out[j][i] = element DV (4g + i) + j of the row
template <int DP> struct Rows {
    float m, l;
    float4_t o[DP / 16];
};

template <int DP, bool BITS8>
__device__ __forceinline__ void score(const Keys<DP, BITS8> &r, const u32x4 (&q)[DP / 32], float4_t (&sc)[2])
{
    sc[0] = sc[1] = float4_t{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
            if constexpr (BITS8) {
                const uint32_t w0 = r.k[t][c / 2][2 * (c & 1)], w1 = r.k[t][c / 2][2 * (c & 1) + 1];
                const float power = power_of(r.e[t], c / 4);
                sc[t] = mfma(u32x4{bf16_of_codes(w0, false, power), bf16_of_codes(w0, true, power), bf16_of_codes(w1, false, power), bf16_of_codes(w1, true, power)}, q[c], sc[t]);
            } else {
                sc[t] = mfma(r.k[t][c], q[c], sc[t]);
            }
        }
}

// Weights of the lane's eight tokens in bf16 from their scores; the running maximum and sum, and what was summed under an older maximum scaled to the new one.
// whole: every row sees the whole block, else the lane's row sees its tokens below `sees`.
template <int DP> __device__ __forceinline__ u32x4 weigh(const float4_t (&sc)[2], float scale2, bool whole, int sees, Rows<DP> &s)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = sc[i >> 2][i & 3] * scale2;
    if (!whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= sees) x[i] = -INFINITY;
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = max16_32(top);
    if (__any(top > s.m)) {
        const float m = fmaxf(s.m, top);
        const float by = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s.m - m);
        s.l *= by;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) s.o[j] *= by;
        s.m = m;
    }
    const float m = s.m == -INFINITY ? 0.0f : s.m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_exp2f(x[i] - m);
    const u32x4 p = {bf16_pair(w[0], w[1]), bf16_pair(w[2], w[3]), bf16_pair(w[4], w[5]), bf16_pair(w[6], w[7])};
#pragma unroll
    for (int i = 0; i < 4; ++i) s.l = add_pair(p[i], s.l);
    return p;
}

// element j of the lane's DV for its eight tokens
template <int DP, bool BITS8> __device__ __forceinline__ u32x4 turned(const Values<DP, BITS8> &r, int j, int lane)
{
    u32x4 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BITS8) {
            // heads of more than 128 elements have two groups; the second begins with lane 8's elements
            const auto wide = [&](int t) {
                const float power = DP > 128 ? power_of(r.e[t / 2], 2 * (t & 1) + ((lane & 15) >> 3)) : power_of(r.e[t / 4], t & 3);
                return bf16_of_codes(r.v[t][j / 4], (j & 2) != 0, power);
            };
            f[i] = __builtin_amdgcn_perm(wide(2 * i + 1), wide(2 * i), j & 1 ? 0x07060302u : 0x05040100u);
        } else {
            f[i] = __builtin_amdgcn_perm(r.v[2 * i + 1][j / 2], r.v[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        }
    }
    return f;
}

// out += values^T x weights.  Tokens that no row of the tile sees (from `there` on, of the lane's eight) may hold anything: zeros in their place.  Values that are not finite
// reach the rows that see them (tokens below `sees`, the lane's own row's) and no others: a product of each row's own then.
template <int DP, bool BITS8> __device__ __forceinline__ void add_values(const Values<DP, BITS8> &r, u32x4 p, bool whole, int there, int sees, int lane, Rows<DP> &s)
{
    if (whole) {
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) s.o[j] = mfma(turned<DP, BITS8>(r, j, lane), p, s.o[j]);
        return;
    }
#pragma unroll
    for (int j = 0; j < DP / 16; ++j) {
        const u32x4 f = first_tokens(turned<DP, BITS8>(r, j, lane), there);
        bool fine = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) fine &= bf16_pair_finite(f[i]);
        if (__all(fine)) {
            s.o[j] = mfma(f, p, s.o[j]);
        } else {
#pragma unroll 1
            for (int n = 0; n < kTile; ++n) {
                const int row_sees = __shfl(sees, (lane & 48) + n, 64);       // this lane's tokens that row n sees
                const float4_t o = mfma(first_tokens(f, row_sees), p, float4_t{0, 0, 0, 0});
                if ((lane & 15) == n) s.o[j] += o;
            }
        }
    }
}

// PREFIX: tiles of all rows against the shared tokens; else of a sequence's rows against its own
template <int DP, bool BITS8, bool PREFIX>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void attn_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, LD = DP + 4;
    __shared__ __align__(16) float part[kWaves][kTile][LD];
    __shared__ float2_t part_ml[kWaves][kTile];
    const int head = blockIdx.x % a.c.heads, item = blockIdx.x / a.c.heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    Work w;
    if (!work_of<PREFIX>(a, item, w)) return;
    const int first = w.first, r = w.tile * kTile + row, rows = w.count * a.G;
    int high = sees_of<PREFIX>(a, w, w.tile * kTile + kTile - 1);
    const int begin = w.begin, end = min(w.end, high);
    high = end;
    const int limit = min(sees_of<PREFIX>(a, w, r), end), low = min(sees_of<PREFIX>(a, w, w.tile * kTile), end);
    const bool valid = r < rows;
    // queries of the tile's rows: elements 32c + 8g .. of step c (8 bits: as the codes' sixteen elements are dealt)
    u32x4 q[DP / 32];
    {
        const uint16_t *const p = a.q + (int64_t)(first + (valid ? r / a.G : 0)) * a.ldq + (int64_t)(head * a.G + (valid ? r % a.G : 0)) * a.c.D;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
            const int d = BITS8 ? 64 * (c / 2) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
            q[c] = u32x4{0, 0, 0, 0};
            if (valid && d < a.c.D) q[c] = *reinterpret_cast<const bf16x8_at2 *>(p + d);
        }
    }
    Rows<DP> s;
    s.m = -INFINITY, s.l = 0.0f;
#pragma unroll
    for (int j = 0; j < DV; ++j) s.o[j] = float4_t{0, 0, 0, 0};
    // The waves take blocks in turn.  The keys of the next block are on their way from the moment that the scores have taken this one's, its values from when the products have.
    // Page numbers come 64 at once: lane 2i + h has half h of the wave's i-th block from now.
    constexpr int STRIDE = kWaves * kBlock, AHEAD = 32;
    const int t0 = begin + wave * kBlock;
    const int blocks = end > t0 ? (end - t0 + STRIDE - 1) / STRIDE : 0;
    int pages = -1, held = AHEAD;
    const auto next_spot = [&](int t) {
        if (held == AHEAD) {
            const int i = (t + (lane >> 1) * STRIDE + (lane & 1) * 16) >> a.c.page_log2;
            pages = i < w.table_len ? w.table[i] : -1;
            pages = pages < a.c.pages ? pages : -1;
            held = 0;
        }
        const int p0 = __builtin_amdgcn_readlane(pages, 2 * held), p1 = __builtin_amdgcn_readlane(pages, 2 * held + 1);
        ++held;
        return spot_of(a.c, head, t, p0, p1);
    };
    Keys<DP, BITS8> k;
    Values<DP, BITS8> v;
    Spot now = {0, 0, 0};
    if (blocks > 0) {
        now = next_spot(t0);
        load_keys<DP, BITS8>(a.c, now, lane, k);
        load_values<DP, BITS8>(a.c, now, lane, v);
    }
    for (int i = 0; i < blocks; ++i) {
        const int t = t0 + i * STRIDE;
        float4_t sc[2];
        score<DP, BITS8>(k, q, sc);
        const uint32_t ok = now.ok;
        if (i + 1 < blocks) {
            now = next_spot(t + STRIDE);
            load_keys<DP, BITS8>(a.c, now, lane, k);
        }
        const bool whole = t + kBlock <= low && ok == 3, mine = ok >> (g >> 1) & 1;
        const int sees = mine ? limit - t - 8 * g : 0, there = mine ? high - t - 8 * g : 0;
        const u32x4 p = weigh<DP>(sc, a.scale2, whole, sees, s);
        add_values<DP, BITS8>(v, p, whole, there, sees, lane, s);
        if (i + 1 < blocks) load_values<DP, BITS8>(a.c, now, lane, v);
    }
    // the four waves' shares: out = sum 2^(m_w - m) out_w
    s.l = sum16_32(s.l);
    if (s.l != s.l) s.m = INFINITY;                          // no part that has seen a NaN counts as empty, or is outweighed
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DV; ++j) part[wave][row][DV * (4 * g + i) + j] = s.o[j][i];
    if (g == 0) part_ml[wave][row] = float2_t{s.m, s.l};
    __syncthreads();
    const int orow = threadIdx.x >> 4, od = (threadIdx.x & 15) * DV;
    float m = -INFINITY, l = 0.0f, o[DV] = {};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = fmaxf(m, part_ml[i][orow].x);
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const float2_t ml = part_ml[i][orow];
        const float by = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
        l += ml.y * by;
#pragma unroll
        for (int j = 0; j < DV; ++j) o[j] += ml.x == -INFINITY ? 0.0f : part[i][orow][od + j] * by;
    }
    const int at = w.tile * kTile + orow;
    if (at >= rows || od >= a.c.D) return;
    if (w.parts == 1) {
        const float by = over(l);
        uint16_t *const p = a.out + (int64_t)(first + at / a.G) * a.ldo + (int64_t)(head * a.G + at % a.G) * a.c.D + od;
#pragma unroll
        for (int j = 0; j < DV; j += 2) {
            const uint32_t w = bf16_pair(o[j] * by, o[j + 1] * by);
            p[j] = (uint16_t)w, p[j + 1] = (uint16_t)(w >> 16);
        }
    } else {
        const int64_t slot = (w.slot * a.c.heads + head) * kTile + orow;
        float *const p = (PREFIX ? a.prefix_o : a.own_o) + slot * a.c.D + od;
#pragma unroll
        for (int j = 0; j < DV; j += 4) *reinterpret_cast<float4_t *>(p + j) = float4_t{o[j], o[j + 1], o[j + 2], o[j + 3]};
        if (od == 0) (PREFIX ? a.prefix_ml : a.own_ml)[slot] = float2_t{m, l};
    }
}

// Joins the parts of a row and query head: D / 4 lanes a part, the parts dealt to the lane groups, their shares added through LDS.
template <int DP>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs a)
{
    constexpr int L = DP / 4, GROUPS = kThreads / L;          // lanes of a part; parts at once
    __shared__ float4_t sums[GROUPS][L];
    __shared__ float2_t mls[GROUPS];
    const int head = blockIdx.x % a.Hq, n = blockIdx.x / a.Hq;
    const int b = sequence_of(a.b, n);
    if (b < 0) return;
    int first, count;
    rows_of(a.b, b, a.N, first, count);
    if (n < first || n >= first + count) return;
    const int64_t base = a.lie[2 * b], parts64 = a.lie[2 * b + 1];
    if (parts64 == 1 && !a.b.prefix) return;                  // written already
    // starts that name rows twice can leave sequences without parts: what the workspace says of them then is no place in it
    if (base < 0 || parts64 < 1 || parts64 > a.slots || base > a.slots - (int64_t)tiles_of(count, a.G, a.own_rows) * parts64) return;
    const int parts = (int)parts64;
    const int kv = head / a.G, in_seq = (n - first) * a.G + head % a.G, in_all = n * a.G + head % a.G;
    const int total = parts + a.prefix_parts;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    // the row's place among the parts of its tile: own parts, parts of the prefix
    const int64_t own = ((base + (int64_t)(in_seq / a.own_rows) * parts) * a.c.heads + kv) * a.own_rows + in_seq % a.own_rows;
    const int64_t pre = a.prefix_parts ? ((int64_t)(in_all / a.prefix_rows) * a.prefix_parts * a.c.heads + kv) * a.prefix_rows + in_all % a.prefix_rows : 0;
    float m = -INFINITY, l = 0.0f;
    float4_t o = {0, 0, 0, 0};
    constexpr int AT_ONCE = 4;                                // parts whose loads a group has on their way together
    for (int i0 = group; i0 < total; i0 += AT_ONCE * GROUPS) {
        float2_t ml[AT_ONCE];
        float4_t v[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int i = i0 + j * GROUPS;
            const bool mine = i < parts;
            const int64_t slot = mine ? own + (int64_t)i * a.c.heads * a.own_rows : pre + (int64_t)(i - parts) * a.c.heads * a.prefix_rows;
            ml[j] = i < total ? (mine ? a.own_ml : a.prefix_ml)[slot] : float2_t{-INFINITY, 0.0f};
            v[j] = i < total && 4 * lane < a.c.D ? *reinterpret_cast<const float4_t *>((mine ? a.own_o : a.prefix_o) + slot * a.c.D + 4 * lane) : float4_t{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const float top = fmaxf(m, ml[j].x);
            if (top == -INFINITY) continue;
            const float old = __builtin_amdgcn_exp2f(m - top), by = __builtin_amdgcn_exp2f(ml[j].x - top);
            l = l * old + ml[j].y * by;
            o = ml[j].x == -INFINITY ? o * old : o * old + v[j] * by;
            m = top;
        }
    }
    sums[group][lane] = o;
    if (lane == 0) mls[group] = float2_t{m, l};
    __syncthreads();
    if (group != 0 || 4 * lane >= a.c.D) return;
    for (int i = 0; i < GROUPS; ++i) m = fmaxf(m, mls[i].x);
    l = 0.0f;
    o = float4_t{0, 0, 0, 0};
    for (int i = 0; i < GROUPS; ++i) {
        const float2_t ml = mls[i];
        if (ml.x == -INFINITY) continue;
        const float by = __builtin_amdgcn_exp2f(ml.x - m);
        l += ml.y * by;
        o += sums[i][lane] * by;
    }
    const float by = over(l);
    uint16_t *const out = a.out + (int64_t)n * a.ldo + (int64_t)head * a.c.D + 4 * lane;
    const uint32_t w0 = bf16_pair(o[0] * by, o[1] * by), w1 = bf16_pair(o[2] * by, o[3] * by);
    out[0] = (uint16_t)w0, out[1] = (uint16_t)(w0 >> 16), out[2] = (uint16_t)w1, out[3] = (uint16_t)(w1 >> 16);
}

// ---- how a call is cut -------------------------------------------------------------------------

struct Cut {
    int target, min_units, own_rows, prefix_rows, through, prefix_units, prefix_parts;
    int64_t slots, items, prefix_items;        // of a key head
};

// Workgroups that a batch's own tokens are spread over: where there are few tiles, all at once, two a CU; where there are many, whose lengths differ, four times as many, so that
// none is left behind with much.  us, 512 / 1024 / 2048 workgroups: one sequence of 200000 tokens in 8 bits 77 / 85 / 98, 64 of 1024 to 8192 tokens 248 / 237 / 226.
constexpr int kGroups = 512, kManyGroups = 2048;
constexpr int kManyTiles = 256;

// us, tiles of 16 / of 128 rows, four query heads a key head, heads of 128: 32 sequences up to 2000 tokens long, 32 rows each 61.3 / 57.6, 48 rows 77.5 / 63.0, 64 rows 84.2 / 68.5; one of 8000 tokens
// 20.1 / 20.6, 22.0 / 21.7, 23.7 / 22.4; eight up to 1000 in 8 bits 19.5 / 20.9, 20.6 / 22.1, 26.1 / 23.6.
int rows_of_tile(int64_t rows) { return rows < 48 ? kTile : kWideRows; }

// Sequences of whole tiles that nobody cuts can take the prefix themselves: no partial results, no join.  A tile's workgroup then walks the whole prefix alone, which is short against the partial
// results, or there are workgroups enough to fill the GPU; else parts of the prefix are shared out.  Partial results of `groups` workgroups take the time of 300 + 9 groups tokens of a walk, and parts
// need groups / 384 of the walk; with heads of more than 128 elements, one workgroup a CU, half of either.
// us, through / in parts, four query heads a key head, 8 key heads of 128, a table of 256 own tokens.  50 new tokens of one sequence (16 workgroups) after 300 shared ones 21 / 29, 1000 40 / 31,
// 64000 1768 / 124.  Two of 200 (112): 1000 44 / 68, 4000 122 / 102, 64000 1733 / 815.  Four of 256 (256): 4000 126 / 168, 16000 437 / 392.  Eight of 256 (512): 64000 2343 / 2538.  Heads of 256, one of
// 200 (56): 600 66 / 75, 1200 108 / 97; four (224): 20000 1194 / 1699.
bool parts_pay(int64_t groups, int D, int64_t prefix)
{
    const int64_t by = D > 128 ? 2 : 1;
    return by * prefix * (384 - by * groups) > 384 * (300 + 9 * groups);
}

Cut cut_of(int64_t N, int Hq, int heads, int D, int B, int64_t tokens, int64_t prefix)
{
    Cut p;
    const int64_t G = Hq / heads;
    p.own_rows = rows_of_tile((N + B - 1) / B * G);
    p.min_units = p.own_rows == kTile ? 2 : 4;
    const int64_t tiles = N * G / p.own_rows + B, units = (tokens + kUnit - 1) / kUnit;
    // Enough tiles of several rows: nothing is cut.  Else the own tokens are cut, also where there are many sequences: their lengths differ.  us, 32 query heads, 8 key heads of 128, uncut / cut: four
    // prompts up to 4096 tokens 342 / 518, 16 up to 1000 127 / 363, 32 of up to 100 new tokens after up to 2000 107 / 162, 128 of up to four after up to 4000 241 / 241.  The rule does not see lengths:
    // a prompt of 2048 tokens beside 63 single tokens, one of which comes after 100000, 3160 / 508, and in two calls 271 + 74.
    const int64_t groups = p.own_rows == kTile && tiles * heads > kManyTiles ? kManyGroups : kGroups;
    const bool cut = (N <= 2 * B || tiles * heads < groups) && units > p.min_units;
    p.target = cut ? (int)((groups + heads - 1) / heads) : 0;
    const int64_t most = cut ? (units + p.min_units - 1) / p.min_units : 1;                // parts of a tile
    p.items = tiles * most < tiles + p.target ? tiles * most : tiles + p.target;           // every tile at least once, and the cuts
    p.through = prefix > 0 && !cut && N * G >= (int64_t)B * kWideRows && !parts_pay(B * ((N * G / B + kWideRows - 1) / kWideRows) * heads, D, prefix);
    if (p.through) prefix = 0;
    p.slots = cut || prefix ? p.items : 0;
    p.prefix_rows = p.prefix_units = p.prefix_parts = 0;
    p.prefix_items = 0;
    if (prefix > 0) {
        p.prefix_rows = rows_of_tile(N * G);
        const int64_t tiles = (N * G + p.prefix_rows - 1) / p.prefix_rows;
        const int64_t units = (prefix + kUnit - 1) / kUnit, want = (kGroups + tiles * heads - 1) / (tiles * heads);
        int64_t part = (units + want - 1) / want;
        const int least = p.prefix_rows == kTile ? 2 : 4;
        part = part < least ? least : part;
        p.prefix_units = (int)part;
        p.prefix_parts = (int)((units + part - 1) / part);
        p.prefix_items = tiles * p.prefix_parts;
    }
    return p;
}

int64_t own_parts(const Cut &p, int heads) { return p.slots * heads * p.own_rows; }              // rows of them
int64_t prefix_parts(const Cut &p, int heads) { return p.prefix_items * heads * p.prefix_rows; }

template <int DP, bool BITS8> hipError_t run(const AttnArgs &a, const Cut &p, hipStream_t st)
{
    if (p.prefix_items > 0) {
        if (p.prefix_rows > kTile) {
            const hipError_t e = launch_attn_wide(a, true, p.prefix_items, st);
            if (e != hipSuccess) return e;
        } else {
            attn_kernel<DP, BITS8, true><<<(unsigned)(p.prefix_items * a.c.heads), kThreads, 0, st>>>(a);
        }
    }
    if (p.own_rows > kTile) {
        const hipError_t e = launch_attn_wide(a, false, p.items, st);
        if (e != hipSuccess) return e;
    } else {
        attn_kernel<DP, BITS8, false><<<(unsigned)(p.items * a.c.heads), kThreads, 0, st>>>(a);
    }
    if (p.slots > 0) attn_join_kernel<DP><<<(unsigned)((int64_t)a.N * a.Hq), kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_workspace_bytes(int64_t N, int Hq, int heads, int D, int B, int64_t tokens, int64_t prefix)
{
    const Cut p = cut_of(N, Hq, heads, D, B, tokens, prefix);
    if (p.items > kMaxGroups / heads || p.prefix_items > kMaxGroups / heads || (p.slots > 0 && N * Hq > kMaxGroups)) return -1;
    return (own_parts(p, heads) + prefix_parts(p, heads)) * (D * 4 + 8) + (p.slots > 0 ? (int64_t)B * 16 : 0);
}

hipError_t launch_attn(const uint16_t *q, int64_t ldq, int64_t N, int Hq, const KvCache &c, const KvBatch &b, float scale, uint16_t *out, int64_t ldo, void *ws,
                       hipStream_t st)
{
    const Cut p = cut_of(N, Hq, c.heads, c.D, b.B, (int64_t)b.width << c.page_log2, b.prefix);
    const int64_t own = own_parts(p, c.heads), pre = prefix_parts(p, c.heads);
    float *const o = static_cast<float *>(ws);
    float2_t *const ml = reinterpret_cast<float2_t *>(o + (own + pre) * c.D);
    const AttnArgs a{q, ldq, out, ldo, (int)N, Hq, Hq / c.heads, c, b, scale * 1.44269504088896340736f, p.target, p.min_units, p.own_rows, p.prefix_rows, p.through, p.slots, p.prefix_units,
                     p.prefix_parts, o, o + own * c.D, ml, ml + own, reinterpret_cast<int64_t *>(ml + own + pre)};
    if (c.D <= 64) return c.bits8 ? run<64, true>(a, p, st) : run<64, false>(a, p, st);
    if (c.D <= 128) return c.bits8 ? run<128, true>(a, p, st) : run<128, false>(a, p, st);
    return c.bits8 ? run<256, true>(a, p, st) : run<256, false>(a, p, st);
}

}  // namespace tj
