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

// The maximum that a row's weights are taken from is moved when scores exceed it by more than this (of log2): weights are up to 2^8 then, which loses nothing, and what was summed
// is rarely scaled.
constexpr float kSlack = 8.0f;

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
    int64_t slots;                        // own parts of a key head, at most
    int prefix_units, prefix_parts;       // units of a part of the prefix, and how many there are
    float *own_o, *prefix_o;              // [slot][key head][rows of a tile][D]
    float2_t *own_ml, *prefix_ml;         // [slot][key head][rows of a tile]: maximum (of log2), sum
};

// What a workgroup has to know of the batch: how many units a part has, and where a part lies.
struct Place {
    int b, tile, part, parts;             // sequence; tile and part in it; parts of its tiles
    int64_t base;                         // first slot of the sequence
};

__device__ __forceinline__ int units(int tokens) { return (tokens + kUnit - 1) / kUnit; }
__device__ __forceinline__ int tiles_of(int rows, int G, int of) { return (rows * G + of - 1) / of; }

__device__ __forceinline__ int64_t block_sum_scan(int64_t v, int64_t *lds, int64_t &before)      // sum over the workgroup; before: over the threads in front
{
    int64_t incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t t = __shfl_up((long long)incl, o, 64);
        if ((int)(threadIdx.x & 63) >= o) incl += t;
    }
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[w] = incl;
    __syncthreads();
    int64_t total = 0;
    before = incl - v;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) before += lds[i];
        total += lds[i];
    }
    return total;
}

// Units of a part of the own tokens: all tiles' units over the parts wanted.  Then where slot `slot` lies (slot >= 0), or where sequence `seq` starts.
// Every thread of the workgroup calls it; false: there is no such slot.
__device__ inline bool find(const AttnArgs &a, int slot, int seq, Place &p, int &part_units, int64_t *lds)
{
    __shared__ Place found;
    const int per = (a.b.B + kThreads - 1) / kThreads, b0 = threadIdx.x * per, b1 = min(b0 + per, a.b.B);
    if (threadIdx.x == 0) found.b = -1;
    part_units = 1 << 25;                                      // more than any sequence has
    if (a.target > 0) {
        int64_t sum = 0;
        for (int b = b0; b < b1; ++b) {
            int first, count;
            rows_of(a.b, b, a.N, first, count);
            sum += (int64_t)tiles_of(count, a.G, a.own_rows) * units(tokens_of(a.b, a.c, b));
        }
        int64_t before;
        const int64_t total = block_sum_scan(sum, lds, before), wanted = (total + a.target - 1) / a.target;
        part_units = wanted < a.min_units ? a.min_units : wanted < part_units ? (int)wanted : part_units;
    }
    int64_t sum = 0, at;
    for (int b = b0; b < b1; ++b) {
        int first, count;
        rows_of(a.b, b, a.N, first, count);
        sum += (int64_t)tiles_of(count, a.G, a.own_rows) * max(1, (units(tokens_of(a.b, a.c, b)) + part_units - 1) / part_units);
    }
    block_sum_scan(sum, lds, at);
    for (int b = b0; b < b1; ++b) {
        int first, count;
        rows_of(a.b, b, a.N, first, count);
        const int parts = max(1, (units(tokens_of(a.b, a.c, b)) + part_units - 1) / part_units);
        const int64_t n = (int64_t)tiles_of(count, a.G, a.own_rows) * parts;
        if (slot >= 0 ? slot >= at && slot < at + n : b == seq) {
            const int in = slot >= 0 ? (int)(slot - at) : 0;
            found = Place{b, in / parts, in % parts, parts, at};
            break;
        }
        at += n;
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
template <bool PREFIX> __device__ __forceinline__ bool work_of(const AttnArgs &a, int item, int64_t *lds, Work &w)
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
        if (!find(a, item, -1, p, part_units, lds)) return false;
        rows_of(a.b, p.b, a.N, w.first, w.count);
        // the tiles that see most come first
        w.tile = tiles_of(w.count, a.G, a.own_rows) - 1 - p.tile;
        w.slot = p.base + (int64_t)w.tile * p.parts + p.part;
        w.parts = a.b.prefix ? 2 : p.parts;
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

// what a sum of weights divides by: nothing seen gives zeros, NaN stays
__device__ __forceinline__ float over(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }

// tiles of many rows (attn_wide.hip); items: of a key head
constexpr int kWideRows = 128;
hipError_t launch_attn_wide(const AttnArgs &a, bool prefix, int64_t items, hipStream_t st);

}  // namespace tj
