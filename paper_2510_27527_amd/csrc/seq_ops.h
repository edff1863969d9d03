// Launchers of the operators on sequences of tokens: rotary positions, the paged cache of keys and values, attention over it, sampling.
#pragma once
#include "block_ops.h"

namespace tj {

constexpr int kMaxHeadDim = 256;
constexpr int64_t kMaxSequences = 1 << 16;      // of a batch
constexpr int64_t kMaxGroups = (1 << 24) - 1;   // workgroups of 256 threads: a launch has less than 2^32 threads
constexpr int64_t kMaxRows = kMaxGroups;        // tokens of a call
constexpr int64_t kMaxDraws = (1 << 22) - 1;    // rows to draw from: their workgroups have 1024 threads
constexpr int kMinPage = 16, kMaxPage = 1 << 16;

struct Rotation {
    const float *freqs;      // [half]
    int half;                // turned pairs of a head; 0: nothing is turned
    int pairs;               // 1: neighbours (2j, 2j + 1), 0: (j, half + j)
    float scale;             // of cosine and sine
};

struct KvCache {
    void *k, *v;                       // [pages][heads][page][D]: bf16, or E4M3 codes
    uint8_t *k_exps, *v_exps;          // [pages][heads][page][groups] of an 8-bit cache
    int pages, heads, D, page_log2, groups, bits8;
};

struct KvBatch {
    const int *table;        // [B][width]
    const int *lens;         // [B]
    const int *starts;       // [B + 1]; null: a token each
    const int *prefix_table; // pages of the prefix
    int B, width, prefix;
};

hipError_t launch_rope(const RowSrc &x, const int *pos, int64_t N, int64_t H, int64_t D, const Rotation &r, int inverse, const RowDst &y, hipStream_t st);

// k, v [N x heads * D] and, where q.p is not null, q [N x Hq * D], which is turned into qo
hipError_t launch_kv_append(const RowSrc &q, int Hq, const RowSrc &k, const RowSrc &v, int64_t N, const KvCache &c, const KvBatch &b, const Rotation &r,
                            const RowDst &qo, hipStream_t st);
hipError_t launch_kv_load(const KvCache &c, const KvBatch &b, int64_t N, const RowDst &k, const RowDst &v, hipStream_t st);

// tokens: the most that a sequence can have of its own; below 0: more workgroups than a launch can have
int64_t attn_workspace_bytes(int64_t N, int Hq, int heads, int D, int B, int64_t tokens, int64_t prefix);
hipError_t launch_attn(const uint16_t *q, int64_t ldq, int64_t N, int Hq, const KvCache &c, const KvBatch &b, float scale, uint16_t *out, int64_t ldo,
                       void *ws, hipStream_t st);

struct SampleArgs {
    const void *logits;
    int64_t ld;
    int f32;
    int64_t N, V;
    const float *temperature, *top_p, *min_p, *u;     // [N]; all but u may be null
    const int *top_k;                                 // [N] or null
    int64_t *tokens;                                  // [N]
};
size_t sample_workspace_bytes(int64_t N, int64_t V);
hipError_t launch_sample(const SampleArgs &a, void *ws, hipStream_t st);

// ---- which sequence a row belongs to -----------------------------------------------------------
// Lengths and starts are device memory that no host check has seen: whatever they hold, the values below lie within the call's arrays.

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// first row and number of rows of sequence b
__device__ __forceinline__ void rows_of(const KvBatch &t, int b, int N, int &first, int &count)
{
    if (!t.starts) {
        first = b;
        count = 1;
        return;
    }
    first = clamp_int(t.starts[b], 0, N);
    count = clamp_int(t.starts[b + 1], first, N) - first;
}
// own tokens of sequence b, those of the call among them
__device__ __forceinline__ int tokens_of(const KvBatch &t, const KvCache &c, int b)
{
    const int64_t room = (int64_t)t.width << c.page_log2;
    const int len = t.lens[b];
    return len < 0 ? 0 : len < room ? len : (int)room;
}

// the sequence of row n, or -1: the last b whose start is not behind n
__device__ __forceinline__ int sequence_of(const KvBatch &t, int n)
{
    if (!t.starts) return n;
    if (n < t.starts[0] || n >= t.starts[t.B]) return -1;
    int lo = 0, hi = t.B;                      // starts[lo] <= n < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.starts[mid] <= n) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Where row n lies in its sequence (-1: nowhere: the row belongs to no sequence, or the sequence has fewer tokens than rows)
__device__ __forceinline__ int place_of(const KvBatch &t, const KvCache &c, int n, int N, int &b)
{
    b = sequence_of(t, n);
    if (b < 0) return -1;
    int first, count;
    rows_of(t, b, N, first, count);
    if (n < first || n >= first + count) return -1;       // starts that are no ascending list
    return tokens_of(t, c, b) - count + (n - first);
}

// the page of an own token, -1 where the table names none of the cache's
__device__ __forceinline__ int page_of(const KvBatch &t, const KvCache &c, int b, int place)
{
    const int at = place >> c.page_log2;
    if (place < 0 || at >= t.width) return -1;
    const int p = t.table[(int64_t)b * t.width + at];
    return p >= 0 && p < c.pages ? p : -1;
}

}  // namespace tj
