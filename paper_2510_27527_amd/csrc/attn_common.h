// What the kernels of attention share: how a call is cut into tiles and parts, and where a workgroup lies in it.
//
//   s_t = scale q . k_t,  m = max s,  l = sum 2^(s_t - m),  out = sum 2^(s_t - m) v_t / l       (s in units of log2)
//
// A tile is a number of rows of one key head: (new token, query head) pairs of one sequence, or of the whole batch against the shared prefix.  The tokens that a tile sees are cut into
// parts, so that few rows fill the GPU as well; a part leaves (m, l, unnormalised out) and a last kernel joins them:
//   out = sum_p 2^(m_p - m) out_p / sum_p 2^(m_p - m) l_p.
// Where a tile has one part only, and there is no prefix, the first kernel writes the output itself.
#pragma once
#include "rowwise.h"
#include "seq_ops.h"

namespace tj {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kUnit = 64;                 // tokens in which the parts' lengths are counted

struct AttnArgs {
    const uint16_t *q;
    int64_t ldq;
    uint16_t *out;
    int64_t ldo;
    int N, Hq, G;                         // rows, query heads, query heads of a key head
    KvCache c;
    KvBatch b;
    float scale2;                         // scale * log2 e
    int target;                           // parts that a key head's own tokens are to be cut into; 0: none are cut
    int min_units;                        // of a part, at least
    int own_rows, prefix_rows;            // rows of a tile of the own tokens, and of the prefix
    int through;                          // 1: a sequence's tiles take the prefix themselves, in front of their own tokens
    int64_t slots;                        // own parts of a key head, at most
    int prefix_units, prefix_parts;       // units of a part of the prefix, and how many there are
    float *own_o, *prefix_o;              // [slot][key head][rows of a tile][D]
    float2_t *own_ml, *prefix_ml;         // [slot][key head][rows of a tile]: maximum (of log2), sum
    int64_t *lie;                         // [B][2]: first slot of a sequence, parts of its tiles
};

// What a workgroup has to know of the batch: how many units a part has, and where a part lies.
struct Place {
    int b, tile, part, parts;             // sequence; tile and part in it; parts of its tiles
    int64_t base;                         // first slot of the sequence
};

__device__ __forceinline__ int units(int tokens) { return (tokens + kUnit - 1) / kUnit; }
__device__ __forceinline__ int tiles_of(int rows, int G, int of) { return (rows * G + of - 1) / of; }

// v of another lane by a DPP control, 0 where there is none or the row is masked.  Counts are doubles here: exact, and two words a move.
template <int CTRL, int ROWS> __device__ __forceinline__ double lane_in_front(double v)
{
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Sum over the workgroup; before: over the threads in front.  No barrier follows the last read of lds: the next call takes another array.
__device__ __forceinline__ double block_sum_scan(double v, double *lds, double &before)
{
    double incl = v;
    incl += lane_in_front<0x111, 0xF>(incl);                   // from 1, 2, 4 and 8 lanes in front, within rows of 16
    incl += lane_in_front<0x112, 0xF>(incl);
    incl += lane_in_front<0x114, 0xF>(incl);
    incl += lane_in_front<0x118, 0xF>(incl);
    incl += lane_in_front<0x142, 0xA>(incl);                   // the row in front's last lane, into rows 1 and 3
    incl += lane_in_front<0x143, 0xC>(incl);                   // lane 31, into rows 2 and 3
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) lds[w] = incl;
    __syncthreads();
    double total = 0.0;
    before = incl - v;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) before += lds[i];
        total += lds[i];
    }
    return total;
}

// Units of a part of the own tokens: all tiles' units over the parts wanted.  Then where slot `slot` lies.
// Every thread of the workgroup calls it, once; false: there is no such slot.
__device__ inline bool find(const AttnArgs &a, int slot, Place &p, int &part_units)
{
    __shared__ Place found;
    __shared__ double lds[2][kWaves];
    const int per = (a.b.B + kThreads - 1) / kThreads, b0 = threadIdx.x * per, b1 = min(b0 + per, a.b.B);
    if (threadIdx.x == 0) found.b = -1;
    // tiles and units of a sequence; those of the thread's first are kept
    const auto size_of = [&](int b, int &tiles, int &length) {
        int first, count;
        rows_of(a.b, b, a.N, first, count);
        tiles = tiles_of(count, a.G, a.own_rows);
        length = units(tokens_of(a.b, a.c, b));
    };
    int tiles0 = 0, length0 = 0;
    if (b0 < b1) size_of(b0, tiles0, length0);
    const auto sized = [&](int b, int &tiles, int &length) {
        if (b == b0) tiles = tiles0, length = length0;
        else size_of(b, tiles, length);
    };
    part_units = 1 << 25;                                      // more than any sequence has
    double at;
    if (a.target > 0) {
        double sum = 0.0;
        for (int b = b0; b < b1; ++b) {
            int tiles, length;
            sized(b, tiles, length);
            sum += (double)tiles * (double)length;
        }
        const double wanted = ceil(block_sum_scan(sum, lds[0], at) / (double)a.target);
        part_units = wanted < (double)a.min_units ? a.min_units : wanted < (double)part_units ? (int)wanted : part_units;
    }
    double sum = 0.0;
    for (int b = b0; b < b1; ++b) {
        int tiles, length;
        sized(b, tiles, length);
        sum += (double)tiles * (double)max(1, (length + part_units - 1) / part_units);
    }
    block_sum_scan(sum, lds[1], at);
    for (int b = b0; b < b1; ++b) {
        int tiles, length;
        sized(b, tiles, length);
        const int parts = max(1, (length + part_units - 1) / part_units);
        const double next = at + (double)tiles * (double)parts;
        if ((double)slot >= at && (double)slot < next) {
            const int in = (int)((double)slot - at);
            found = Place{b, in / parts, in % parts, parts, (int64_t)at};
            break;
        }
        at = next;
    }
    __syncthreads();
    p = found;
    return p.b >= 0;
}


// The tile of a workgroup: rows first .. of the call, tokens begin .. end of the table.
struct Work {
    int first, count, tile, parts, begin, end, table_len;
    int len;                              // own tokens of the sequence; the prefix: its length
    int64_t slot;
    const int *table;
};

// Tile and part number `item` of a key head; false: there is none.  PREFIX: of all rows against the prefix; else of a sequence's against its own.  Every thread of the workgroup calls it.
template <bool PREFIX> __device__ __forceinline__ bool work_of(const AttnArgs &a, int item, Work &w)
{
    if constexpr (PREFIX) {
        w.first = 0, w.count = a.N;
        w.tile = item / a.prefix_parts;
        w.parts = 2;                                         // never alone: the own tokens follow
        w.begin = item % a.prefix_parts * a.prefix_units * kUnit;
        w.len = a.b.prefix;
        w.end = min(w.begin + a.prefix_units * kUnit, w.len);
        w.slot = item;
        w.table = a.b.prefix_table;
        w.table_len = (a.b.prefix + (1 << a.c.page_log2) - 1) >> a.c.page_log2;
        return true;
    } else {
        Place p;
        int part_units;
        if (!find(a, item, p, part_units)) return false;
        rows_of(a.b, p.b, a.N, w.first, w.count);
        // the tiles that see most come first
        w.tile = tiles_of(w.count, a.G, a.own_rows) - 1 - p.tile;
        w.slot = p.base + (int64_t)w.tile * p.parts + p.part;
        if (a.slots > 0 && w.slot >= a.slots) return false;  // starts that name rows twice make more tiles than the workspace has room for
        w.parts = a.b.prefix && !a.through ? 2 : p.parts;
        if (a.slots > 0 && blockIdx.x % a.c.heads == 0 && p.tile == 0 && p.part == 0 && threadIdx.x == 0) a.lie[2 * p.b] = p.base, a.lie[2 * p.b + 1] = p.parts;
        w.len = tokens_of(a.b, a.c, p.b);
        w.begin = p.part * part_units * kUnit;
        w.end = p.part == p.parts - 1 ? w.len : min(w.len, w.begin + part_units * kUnit);
        w.table = a.b.table + (int64_t)p.b * a.b.width;
        w.table_len = a.b.width;
        return true;
    }
}

// tokens that row r of the tile's sequence (new token r / G) sees
template <bool PREFIX> __device__ __forceinline__ int sees_of(const AttnArgs &a, const Work &w, int r)
{
    if constexpr (PREFIX) return w.len;
    else return max(0, w.len - w.count + min(r / a.G, w.count - 1) + 1);
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ bool bf16_pair_finite(uint32_t w) { return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u; }

// zeros for the tokens from `keep` on of a lane's eight, in pairs
__device__ __forceinline__ u32x4 first_tokens(u32x4 f, int keep)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = keep >= 2 * i + 2 ? f[i] : keep == 2 * i + 1 ? f[i] & 0xFFFFu : 0;
    return f;
}

// two of a word's four E4M3 codes times a power of two as bf16: exact
__device__ __forceinline__ uint32_t bf16_of_codes(uint32_t w, bool high, float power)
{
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false));
}
__device__ __forceinline__ float power_of(uint32_t bytes, int at) { return u2f(((bytes >> (8 * at)) & 0xFF) << 23); }

// l + the two bf16 of w.  A row's sum is that of its weights as the matrix instructions take them, rounded: where few tokens have most of the weight their roundings cancel.
__device__ __forceinline__ float add_pair(uint32_t w, float l)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), l, false);
}

// what a sum of weights divides by: nothing seen gives zeros, NaN stays
__device__ __forceinline__ float over(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }

// tiles of many rows (attn_wide.hip); items: of a key head
constexpr int kWideRows = 128;
hipError_t launch_attn_wide(const AttnArgs &a, bool prefix, int64_t items, hipStream_t st);

}  // namespace tj
