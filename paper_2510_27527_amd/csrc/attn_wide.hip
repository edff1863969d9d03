// Attention on tiles of 128 rows: prompts, and many sequences' rows against a shared prefix.  (Formulas: attn_common.h.)
//
// 4 D flops and one exponential a (row, token) pair.  Four prompts up to 4096 tokens long (32 query heads, 8 key heads of 128): 331 us, 755 TFLOP/s (385 and more in the first 30 ms after the
// GPU was idle); matrix instructions are busy 35 % of the time, the vector ALU 44 %, waves wait 27 % of theirs.  Without the exponentials it takes 316 us.  The four waves of a workgroup have 32 rows
// each and share tiles of 64 tokens in LDS, the next tile on its way in registers.  Products: scores^T [tokens x rows] = K Q^T and out^T [D x rows] += V^T P^T, 32 x 32 x 16
// each; the tokens are dealt to the rows of a score tile so that a lane ends up with the weights that the second product takes from it.  Values lie in LDS as rows of tokens and are turned by the
// transposing LDS reads.  8-bit caches become bf16 on their way into LDS, once for all four waves.
#include <type_traits>

#include "attn_common.h"

namespace tj {

namespace {

typedef short short4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float16_t mfma(u32x4 a, u32x4 b, float16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ float max32(float v)             // over the two lanes that hold a row
{
    const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
    return fmaxf(u2f(b[0]), u2f(b[1]));
}
__device__ __forceinline__ float sum32(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
    return u2f(b[0]) + u2f(b[1]);
}

// Rows of a tile lie in LDS one after the other, their 16-byte chunks exchanged by the token: chunk c of token t is at c ^ bank(t).  The lanes that read at once then meet all
// banks alike, whether 128 or 256 bytes are read in a step: 8 or 16 tokens' same chunk of keys (tokens that differ in bits 0, 1, 3 and 2), or 32 or 64 bytes of each of
// four tokens' values (bits 0 and 1).
template <int DP> __device__ __forceinline__ int bank(int t)
{
    return DP > 64 ? (t & 1) * 10 ^ (t & 2) * 2 ^ (t >> 3 & 1) ^ (t & 4) * 2 : (t & 1) * 2 ^ (t & 2) * 2 ^ (t >> 3 & 1) ^ (t >> 1 & 2);
}
// byte of chunk c of token t
template <int DP> __device__ __forceinline__ int place(int t, int c) { return t * 2 * DP + 16 * (c ^ bank<DP>(t)); }

template <int DP> struct Shape {
    static constexpr int TOK = DP > 128 ? 32 : 64;           // tokens of a tile
    static constexpr int BYTES = 2 * DP;                     // of a token
    static constexpr int CHUNKS = DP / 8;                    // of 16 bytes
    static constexpr int PER = kThreads / CHUNKS;            // tokens that the workgroup moves at once
    static constexpr int MOVES = TOK / PER;
    static constexpr int GROUPS = TOK / 16;                  // runs of 16 tokens, each in one page
};

// a tile on its way: what a thread moves of keys and values
template <int DP, bool BITS8> struct Moved {
    u32x4 k[Shape<DP>::MOVES], v[Shape<DP>::MOVES];          // 8 bits: codes in the first two words, the exponent in the third
};

// EXACT: heads of DP elements, else of fewer
template <int DP, bool EXACT, bool BITS8, bool PREFIX>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void attn_wide_kernel(AttnArgs a)
{
    using S = Shape<DP>;
    constexpr int ROWS = kWideRows, TT = S::TOK / 32, DT = DP / 32;
    __shared__ int odd[2][kWaves];                            // of a tile that not every row sees: whether a wave has put a value that is not finite
    __shared__ __align__(16) char keys[2 * S::TOK * S::BYTES];
    __shared__ __align__(16) char values[2 * S::TOK * S::BYTES];
    const int head = blockIdx.x % a.c.heads, item = blockIdx.x / a.c.heads;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int row = lane & 31, h = lane >> 5;
    Work w;
    if (!work_of<PREFIX>(a, item, w)) return;
    const int rows = w.count * a.G, r0 = w.tile * ROWS + wave * 32;
    const int r = r0 + row;
    const bool valid = r < rows;
    u32x4 q[DP / 16];
    const uint16_t *const qp = a.q + (int64_t)(w.first + (valid ? r / a.G : 0)) * a.ldq + (int64_t)(head * a.G + (valid ? r % a.G : 0)) * a.c.D;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int d = 16 * c + 8 * h;
        q[c] = u32x4{0, 0, 0, 0};
        if (valid && (EXACT || d < a.c.D)) q[c] = *reinterpret_cast<const bf16x8_at2 *>(qp + d);
    }
    // What is walked over: tokens begin .. end of a table; how many of them the lane's row sees, the least that a row of the workgroup sees, the least and the most of a row of the wave.
    // THROUGH: first the prefix, which every row sees, then the sequence's own tokens.
    const int *table = w.table;
    int table_len = w.table_len, begin = w.begin, end, limit, least, low, high;
    const auto own_tokens = [&]() {
        end = min(w.end, sees_of<PREFIX>(a, w, w.tile * ROWS + ROWS - 1));
        limit = min(sees_of<PREFIX>(a, w, r), end);
        least = min(sees_of<PREFIX>(a, w, w.tile * ROWS), end);
        low = min(sees_of<PREFIX>(a, w, r0), end), high = min(sees_of<PREFIX>(a, w, r0 + 31), end);
    };
    const bool through = !PREFIX && a.through;
    if (through) {
        table = a.b.prefix_table;
        table_len = (a.b.prefix + (1 << a.c.page_log2) - 1) >> a.c.page_log2;
        begin = 0, end = limit = least = low = high = a.b.prefix;
    } else {
        own_tokens();
    }

    float m = -INFINITY, l = 0.0f;
    float16_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    // ---- tiles on their way ----
    // A wave's loads of a move are of one run of 16 tokens, in one page: its start is in scalar registers, a lane's place in the run is always the same.
    const int mt = threadIdx.x / S::CHUNKS, mc = threadIdx.x % S::CHUNKS;      // the thread's token (of PER) and chunk
    const bool there = 8 * mc < a.c.D;                                         // else zeros, whatever was loaded
    const uint32_t in_run = (mt & 15) * a.c.D + (there ? 8 * mc : 0), e_in_run = (mt & 15) * a.c.groups + (there ? mc / 16 : 0);
    int pages = -1, held = 64 / S::GROUPS;                                     // page numbers of the next tiles, lane GROUPS i + g: run g of the i-th
    Moved<DP, BITS8> x;
    uint32_t ok_next = 0;
    const auto fetch = [&](int t0) {
        if (held == 64 / S::GROUPS) {
            const int i = (t0 + 16 * lane) >> a.c.page_log2;
            pages = i < table_len ? table[i] : -1;
            pages = pages < a.c.pages ? pages : -1;
            held = 0;
        }
        ok_next = 0;
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g) ok_next |= (uint32_t)(__builtin_amdgcn_readlane(pages, S::GROUPS * held + g) >= 0) << g;
#pragma unroll
        for (int i = 0; i < S::MOVES; ++i) {
            const int run = uniform((i * S::PER + mt) >> 4);
            const int page = __builtin_amdgcn_readlane(pages, S::GROUPS * held + run);
            const int64_t token = (((int64_t)(page < 0 ? 0 : page) * a.c.heads + head) << a.c.page_log2) + ((t0 + 16 * run) & ((1 << a.c.page_log2) - 1)) +
                                  (i * S::PER & 15);
            if constexpr (BITS8) {
                const u32x2 k = *reinterpret_cast<const u32x2 *>(shared_row(static_cast<const char *>(a.c.k) + token * a.c.D) + in_run);
                const u32x2 v = *reinterpret_cast<const u32x2 *>(shared_row(static_cast<const char *>(a.c.v) + token * a.c.D) + in_run);
                x.k[i] = u32x4{k[0], k[1], shared_row(a.c.k_exps + token * a.c.groups)[e_in_run], 0};
                x.v[i] = u32x4{v[0], v[1], shared_row(a.c.v_exps + token * a.c.groups)[e_in_run], 0};
            } else {
                x.k[i] = *reinterpret_cast<const u32x4 *>(shared_row(static_cast<const uint16_t *>(a.c.k) + token * a.c.D) + in_run);
                x.v[i] = *reinterpret_cast<const u32x4 *>(shared_row(static_cast<const uint16_t *>(a.c.v) + token * a.c.D) + in_run);
            }
        }
        ++held;
    };
    // whether some row does not see some token of the tile
    const auto edge = [&](int t0, uint32_t ok) { return t0 + S::TOK > least || ok != (1u << S::GROUPS) - 1; };
    const auto put = [&](int t0, int buffer) {
        if constexpr (BITS8) {
#pragma unroll
            for (int i = 0; i < S::MOVES; ++i) {
                const u32x4 k = x.k[i], v = x.v[i];
                const float ke = power_of(k[2], 0), ve = power_of(v[2], 0);
                x.k[i] = u32x4{bf16_of_codes(k[0], false, ke), bf16_of_codes(k[0], true, ke), bf16_of_codes(k[1], false, ke), bf16_of_codes(k[1], true, ke)};
                x.v[i] = u32x4{bf16_of_codes(v[0], false, ve), bf16_of_codes(v[0], true, ve), bf16_of_codes(v[1], false, ve), bf16_of_codes(v[1], true, ve)};
            }
        }
        if (!EXACT && !there) {
#pragma unroll
            for (int i = 0; i < S::MOVES; ++i) x.k[i] = x.v[i] = u32x4{0, 0, 0, 0};
        }
        if (edge(t0, ok_next)) {
            bool fine = true;
#pragma unroll
            for (int i = 0; i < S::MOVES; ++i) {
                const int t = i * S::PER + mt;
                // tokens that no row of the workgroup sees may hold anything
                if (t0 + t >= end || !(ok_next >> (t >> 4) & 1)) x.v[i] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j) fine &= bf16_pair_finite(x.v[i][j]);
            }
            const int any = !__all(fine);
            if (lane == 0) odd[buffer][wave] = any;
        }
#pragma unroll
        for (int i = 0; i < S::MOVES; ++i) {
            const int at = buffer * S::TOK * S::BYTES + place<DP>(i * S::PER + mt, mc);
            *reinterpret_cast<u32x4 *>(keys + at) = x.k[i];
            *reinterpret_cast<u32x4 *>(values + at) = x.v[i];
        }
    };

    // ---- the lane's places in a tile ----
    // keys: row i of a score tile is the token that has bits 2 and 3 exchanged; chunk 2c + h
    const int kt = (row & 0x13) | (row & 4) << 1 | (row & 8) >> 1;
    int kat[DP / 16];
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) kat[c] = place<DP>(kt, 2 * c + h);
    // values: 16 lanes turn 4 tokens x 16 elements; tokens 8h + 4i + (lane / 4 mod 4), elements 16 (lane / 16 mod 2) + 4 (lane mod 4) of 32
    int vat[2][DT];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int d = 0; d < DT; ++d) vat[i][d] = place<DP>(8 * h + 4 * i + (lane >> 2 & 3), 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) + 8 * (lane & 1);

    // One tile.  ODD: it has values that are not finite: they reach the rows that see them and no others, by a product of each row's own.
    const auto take = [&](int t0, int buffer, uint32_t ok, auto is_odd) {
        constexpr bool ODD = decltype(is_odd)::value;
        const int in = buffer * S::TOK * S::BYTES;
        float16_t sc[TT];
#pragma unroll
        for (int i = 0; i < TT * (DP / 16); ++i) {
            const int t = i % TT, c = i / TT;
            const u32x4 k = *reinterpret_cast<const u32x4 *>(keys + (kat[c] + in) + t * 32 * S::BYTES);
            if (c == 0) sc[t] = mfma(k, q[c], float16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0});
            else sc[t] = mfma(k, q[c], sc[t]);
        }
        const bool whole = t0 + S::TOK <= low && ok == (1u << S::GROUPS) - 1;
        if (!whole) {
            const int sees = limit - t0 - 8 * h;
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int run = 2 * t + (i >> 3);
                    if (16 * run + (i & 7) >= (ok >> run & 1 ? sees : 0)) sc[t][i] = -INFINITY;
                }
        }
        float tops[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            tops[j] = sc[0][j];
#pragma unroll
            for (int i = 1; i < 4 * TT; ++i) tops[j] = fmaxf(tops[j], sc[i / 4][4 * (i & 3) + j]);
        }
        float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        top = max32(top) * a.scale2;
        // Moved whenever it is exceeded: a row's largest weight is then 1, which bf16 holds exactly.  (Moved from 2^8 on only: 322 us instead of 332 for four prompts up to 4096 tokens, and
        // outputs 0.0022 off instead of 0.0018, where rounding the exact ones to bf16 gives 0.0016.)
        if (__any(top > m)) {
            const float to = fmaxf(m, top), old = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
            l *= old;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= old;
            m = to;
        }
        // score * scale - maximum in one operation: the product is not rounded, and the largest one not taken from itself exactly.  Scores that the difference then matters for are
        // scaled first.
        float mm = m == -INFINITY ? 0.0f : m, by = a.scale2;
        if (__any(fabsf(mm) > 0x1p20f)) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = sc[t][i] * a.scale2 - mm;
            mm = 0.0f, by = 1.0f;
        }
        // weights of the lane's eight tokens of run g
        const auto weights = [&](int g) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(sc[g / 2][8 * (g & 1) + i], by, -mm));
            const u32x4 w = {bf16_pair(e[0], e[1]), bf16_pair(e[2], e[3]), bf16_pair(e[4], e[5]), bf16_pair(e[6], e[7])};
#pragma unroll
            for (int i = 0; i < 4; ++i) l = add_pair(w[i], l);
            return w;
        };
        const auto turned = [&](int g, int d) {
            u32x4 f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                typedef __attribute__((address_space(3))) short4_t *lds4;
                const u32x2 part = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4)(values + (vat[i][d] + in) + 16 * g * S::BYTES)));
                f[2 * i] = part[0], f[2 * i + 1] = part[1];
            }
            return f;
        };
        if constexpr (!ODD) {
            // the next run's weights and values while the products take this one's
            u32x4 p = weights(0), f[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d) f[d] = turned(0, d);
#pragma unroll
            for (int g = 0; g < S::GROUPS; ++g) {
                u32x4 next[DT], pn;
                if (g + 1 < S::GROUPS) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) next[d] = turned(g + 1, d);
                    pn = weights(g + 1);
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = mfma(f[d], p, o[d]);
                if (g + 1 < S::GROUPS) {
                    p = pn;
#pragma unroll
                    for (int d = 0; d < DT; ++d) f[d] = next[d];
                }
            }
        } else {
            // values that are not finite reach the rows that see them and no others: a product of each row's own
            u32x4 p[S::GROUPS];
#pragma unroll
            for (int g = 0; g < S::GROUPS; ++g) p[g] = weights(g);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
#pragma unroll 1
                for (int j = 0; j < 32; ++j) {
                    const int sees = __shfl(limit, j, 64) - t0 - 8 * h;
                    float16_t own;
#pragma unroll
                    for (int i = 0; i < 16; ++i) own[i] = 0.0f;
#pragma unroll
                    for (int g = 0; g < S::GROUPS; ++g) own = mfma(first_tokens(turned(g, d), sees - 16 * g), p[g], own);
                    if (row == j) o[d] += own;
                }
            }
        }
    };

    // The tile after the next is on its way from the moment that the next one is in LDS.
    int buffer = 0, t0 = begin;
    uint32_t ok = 0;
    const auto put_next = [&](int t, int to) {
        put(t, to);
        ok = ok_next;
        if (t + S::TOK < end) fetch(t + S::TOK);
    };
    const auto walk = [&](auto is_odd) {
        for (; t0 < end; t0 += S::TOK, buffer ^= 1) {
            __syncthreads();
            if constexpr (!decltype(is_odd)::value)
                if (edge(t0, ok) && (odd[buffer][0] | odd[buffer][1] | odd[buffer][2] | odd[buffer][3])) break;
            if (t0 < high) take(t0, buffer, ok, is_odd);
            if (t0 + S::TOK < end) put_next(t0 + S::TOK, buffer ^ 1);
        }
    };
    for (int pass = through ? 0 : 1; pass < 2; ++pass) {
        if (t0 < end) {
            held = 64 / S::GROUPS;
            fetch(t0);
            put_next(t0, buffer);
        }
        // From the first tile with values that are not finite and that not every row sees, a second loop: the first one's registers stay where they are.
        walk(std::false_type());
        walk(std::true_type());
        if (pass == 0) {
            table = w.table, table_len = w.table_len;
            t0 = w.begin;
            own_tokens();
            __syncthreads();                                  // the last tile of the prefix has been read
        }
    }

    float sum = sum32(l);
    if (sum != sum) m = INFINITY;                             // no part that has seen a NaN counts as empty, or is outweighed
    if (!valid) return;
    if (w.parts == 1) {
        const float by = over(sum);
        uint16_t *const p = a.out + (int64_t)(w.first + r / a.G) * a.ldo + (int64_t)(head * a.G + r % a.G) * a.c.D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = 32 * d + 8 * j + 4 * h;
                typedef uint32_t bf16x4_at2 __attribute__((ext_vector_type(2), aligned(2)));
                if (EXACT || at < a.c.D)
                    *reinterpret_cast<bf16x4_at2 *>(p + at) = bf16x4_at2{bf16_pair(o[d][4 * j] * by, o[d][4 * j + 1] * by), bf16_pair(o[d][4 * j + 2] * by, o[d][4 * j + 3] * by)};
            }
    } else {
        const int64_t slot = (w.slot * a.c.heads + head) * ROWS + wave * 32 + row;
        float *const p = (PREFIX ? a.prefix_o : a.own_o) + slot * a.c.D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = 32 * d + 8 * j + 4 * h;
                if (EXACT || at < a.c.D) *reinterpret_cast<float4_t *>(p + at) = float4_t{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
            }
        if (h == 0) (PREFIX ? a.prefix_ml : a.own_ml)[slot] = float2_t{m, sum};
    }
}

template <int DP, bool EXACT, bool BITS8> void run(const AttnArgs &a, bool prefix, int64_t items, hipStream_t st)
{
    const unsigned grid = (unsigned)(items * a.c.heads);
    if (prefix) attn_wide_kernel<DP, EXACT, BITS8, true><<<grid, kThreads, 0, st>>>(a);
    else attn_wide_kernel<DP, EXACT, BITS8, false><<<grid, kThreads, 0, st>>>(a);
}
template <int DP> void run(const AttnArgs &a, bool prefix, int64_t items, hipStream_t st)
{
    if (a.c.D == DP) a.c.bits8 ? run<DP, true, true>(a, prefix, items, st) : run<DP, true, false>(a, prefix, items, st);
    else a.c.bits8 ? run<DP, false, true>(a, prefix, items, st) : run<DP, false, false>(a, prefix, items, st);
}

}  // namespace

hipError_t launch_attn_wide(const AttnArgs &a, bool prefix, int64_t items, hipStream_t st)
{
    if (a.c.D <= 64) run<64>(a, prefix, items, st);
    else if (a.c.D <= 128) run<128>(a, prefix, items, st);
    else run<256>(a, prefix, items, st);
    return hipGetLastError();
}

}  // namespace tj
