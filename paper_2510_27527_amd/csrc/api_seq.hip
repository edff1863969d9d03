// C-ABI layer of the operators on sequences of tokens (rotary positions, the paged cache, attention over it, sampling): host-side
// validation before the first HIP call, then one launcher each.
#include <math.h>

#include "../../include/tjnvfp4.h"
#include "api_rows.h"
#include "seq_ops.h"

namespace tj {

namespace {

constexpr int64_t kMaxWidth = (int64_t)1 << 22;          // elements of a row of heads
constexpr int64_t kMaxTurned = 4096;                     // elements of a head that nvfp4_rope takes
constexpr int64_t kMaxCache = (int64_t)1 << 40;          // elements
constexpr int64_t kMaxVocabulary = (int64_t)1 << 20;
constexpr int64_t kMaxHeadRows = (int64_t)1 << 30;       // rows times query heads of an attention call

int check_rotation(const nvfp4_rotation *r, int64_t D, Rotation *o)
{
    *o = Rotation{nullptr, 0, 0, 1.0f};
    if (!r) return NVFP4_OK;
    if (r->form != NVFP4_ROPE_HALF && r->form != NVFP4_ROPE_PAIRS) return NVFP4_ERR_ENUM;
    if (r->R < 0 || r->R > D || r->R % 2 != 0) return NVFP4_ERR_SHAPE;
    if (r->R > 0 && !r->freqs) return NVFP4_ERR_NULL;
    if (!aligned(r->freqs, 4)) return NVFP4_ERR_ALIGN;
    *o = Rotation{r->freqs, (int)(r->R / 2), r->form == NVFP4_ROPE_PAIRS, r->scale};
    return NVFP4_OK;
}

bool is_page(int64_t page) { return page >= kMinPage && page <= kMaxPage && (page & (page - 1)) == 0; }
bool is_head_dim(int64_t D) { return D >= 16 && D <= kMaxHeadDim && D % 16 == 0; }

int check_cache(const nvfp4_kvcache *c, KvCache *o)
{
    if (!c || !c->k || !c->v) return NVFP4_ERR_NULL;
    if (c->kind != NVFP4_KV_BF16 && c->kind != NVFP4_KV_8) return NVFP4_ERR_ENUM;
    const bool bits8 = c->kind == NVFP4_KV_8;
    if (bits8 && (!c->k_exps || !c->v_exps)) return NVFP4_ERR_NULL;
    if (!is_page(c->page) || !is_head_dim(c->D) || c->H < 1 || c->H * c->D > kMaxWidth || c->H > kMaxWidth) return NVFP4_ERR_SHAPE;
    if (c->pages < 0 || c->pages > 0x7FFFFFFF || c->pages > kMaxCache / (c->H * c->page * c->D)) return NVFP4_ERR_SHAPE;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || (bits8 && (!aligned(c->k_exps, 16) || !aligned(c->v_exps, 16)))) return NVFP4_ERR_ALIGN;
    int log2 = 0;
    while (((int64_t)1 << log2) < c->page) ++log2;
    *o = KvCache{c->k, c->v, c->k_exps, c->v_exps, (int)c->pages, (int)c->H, (int)c->D, log2, (int)((c->D + kCkptGroup - 1) / kCkptGroup), bits8};
    return NVFP4_OK;
}

int check_counts(int64_t B, int64_t width, int64_t prefix, int64_t page)
{
    const int64_t most = 0x7FFFFFFF - kMaxPage;
    if (B < 0 || B > kMaxSequences || width < 0 || prefix < 0 || prefix >= most || width > most / page || width * page + prefix >= most) return NVFP4_ERR_SHAPE;
    return NVFP4_OK;
}

int check_batch(const nvfp4_kvbatch *b, const KvCache &c, int64_t N, KvBatch *o)
{
    if (!b || !b->table || !b->lens || (b->prefix > 0 && !b->prefix_table)) return NVFP4_ERR_NULL;
    const int rc = check_counts(b->B, b->width, b->prefix, (int64_t)1 << c.page_log2);
    if (rc) return rc;
    if (!aligned(b->table, 4) || !aligned(b->lens, 4) || !aligned(b->starts, 4) || !aligned(b->prefix_table, 4)) return NVFP4_ERR_ALIGN;
    if (!b->starts && N != b->B) return NVFP4_ERR_MISMATCH;
    *o = KvBatch{b->table, b->lens, b->starts, b->prefix_table, (int)b->B, (int)b->width, (int)b->prefix};
    return NVFP4_OK;
}

}  // namespace

}  // namespace tj

using namespace tj;

extern "C" {

int nvfp4_rope_frequencies(int64_t R, double base, int scaling, double factor, double trained, double low, double high, float *freqs)
{
    if (R < 0 || R % 2 != 0 || R > (1 << 20)) return NVFP4_ERR_SHAPE;
    if (R > 0 && !freqs) return NVFP4_ERR_NULL;
    if (scaling < NVFP4_ROPE_PLAIN || scaling > NVFP4_ROPE_PARTS || !(base > 0.0) || !isfinite(base) || !(factor > 0.0) || !isfinite(factor)) return NVFP4_ERR_ENUM;
    if (scaling == NVFP4_ROPE_PARTS && (!(trained > 0.0) || !isfinite(trained) || !(low >= 0.0) || !(low < high) || !isfinite(high))) return NVFP4_ERR_ENUM;
    if (scaling == NVFP4_ROPE_BASE && R <= 2) return R == 0 ? NVFP4_OK : NVFP4_ERR_SHAPE;
    if (scaling == NVFP4_ROPE_BASE) base *= pow(factor, (double)R / (double)(R - 2));
    for (int64_t j = 0; j < R / 2; ++j) {
        double f = pow(base, -2.0 * (double)j / (double)R);
        if (scaling == NVFP4_ROPE_LINEAR) f /= factor;
        if (scaling == NVFP4_ROPE_PARTS) {
            const double turns = trained * f * 0.15915494309189533577, share = fmin(1.0, fmax(0.0, (turns - low) / (high - low)));
            f = f * share + f / factor * (1.0 - share);
        }
        freqs[j] = (float)f;
    }
    return NVFP4_OK;
}

int nvfp4_rope(const void *X, int src_kind, int64_t ldx, const int32_t *pos, int64_t N, int64_t H, int64_t D, const nvfp4_rotation *rotation, int inverse,
               void *Y, int out_dtype, int64_t ldy, void *stream)
{
    if (!rotation || !pos) return NVFP4_ERR_NULL;
    if (N < 0 || N > kMaxRows || H < 0 || D < 0 || D > kMaxTurned || H > kMaxWidth || H * D > kMaxWidth) return NVFP4_ERR_SHAPE;
    RowSrc x;
    RowDst y;
    Rotation r;
    int rc = check_sizes(N, H * D);
    if (rc) return rc;
    rc = make_src(X, src_kind, ldx, N, H * D, -1, 0, &x);
    if (rc) return rc;
    rc = make_dst(Y, out_dtype, ldy, N, H * D, &y);
    if (rc) return rc;
    rc = check_rotation(rotation, D, &r);
    if (rc) return rc;
    if (!aligned(pos, 4)) return NVFP4_ERR_ALIGN;
    if (N == 0 || H == 0 || D == 0) return NVFP4_OK;
    return status(launch_rope(x, pos, N, H, D, r, inverse != 0, y, static_cast<hipStream_t>(stream)));
}

int nvfp4_kv_append(const void *Q, int64_t ldq, int64_t Hq, const void *K, int64_t ldk, const void *V, int64_t ldv, int src_kind, int64_t N,
                    const nvfp4_kvcache *cache, const nvfp4_kvbatch *batch, const nvfp4_rotation *rotation, void *Qo, int out_dtype, int64_t ldqo,
                    void *stream)
{
    KvCache c;
    KvBatch b;
    Rotation r;
    int rc = check_cache(cache, &c);
    if (rc) return rc;
    if (N < 0 || N > kMaxRows) return NVFP4_ERR_SHAPE;
    rc = check_batch(batch, c, N, &b);
    if (rc) return rc;
    rc = check_rotation(rotation, c.D, &r);
    if (rc) return rc;
    const int64_t width = (int64_t)c.heads * c.D;
    RowSrc q{nullptr, nullptr, 0, 0, src_kind == NVFP4_SRC_F32 ? kF32 : kBf16}, k, v;
    RowDst qo{nullptr, 0, 0};
    rc = check_sizes(N, width);
    if (rc) return rc;
    rc = make_src(K, src_kind, ldk, N, width, -1, 0, &k);
    if (rc) return rc;
    rc = make_src(V, src_kind, ldv, N, width, -1, 0, &v);
    if (rc) return rc;
    if (!Q) Hq = 0;
    if (Q) {
        if (Hq < 0 || Hq > kMaxWidth || Hq * c.D > kMaxWidth) return NVFP4_ERR_SHAPE;
        rc = check_sizes(N, Hq * c.D);
        if (rc) return rc;
        rc = make_src(Q, src_kind, ldq, N, Hq * c.D, -1, 0, &q);
        if (rc) return rc;
        rc = make_dst(Qo, out_dtype, ldqo, N, Hq * c.D, &qo);
        if (rc) return rc;
    }
    if (N == 0 || b.B == 0) return NVFP4_OK;
    return status(launch_kv_append(q, (int)Hq, k, v, N, c, b, r, qo, static_cast<hipStream_t>(stream)));
}

int nvfp4_kv_load(const nvfp4_kvcache *cache, const nvfp4_kvbatch *batch, int64_t N, void *K, int64_t ldk, void *V, int64_t ldv, int out_dtype, void *stream)
{
    KvCache c;
    KvBatch b;
    int rc = check_cache(cache, &c);
    if (rc) return rc;
    if (N < 0 || N > kMaxRows) return NVFP4_ERR_SHAPE;
    rc = check_batch(batch, c, N, &b);
    if (rc) return rc;
    const int64_t width = (int64_t)c.heads * c.D;
    RowDst k, v;
    rc = check_sizes(N, width);
    if (rc) return rc;
    rc = make_dst(K, out_dtype, ldk, N, width, &k);
    if (rc) return rc;
    rc = make_dst(V, out_dtype, ldv, N, width, &v);
    if (rc) return rc;
    if (N == 0 || b.B == 0) return NVFP4_OK;
    return status(launch_kv_load(c, b, N, k, v, static_cast<hipStream_t>(stream)));
}

size_t nvfp4_attn_workspace_bytes(int64_t N, int64_t Hq, int64_t H, int64_t D, int64_t page, int64_t B, int64_t width, int64_t prefix)
{
    if (N <= 0 || N > kMaxRows || H < 1 || H > kMaxWidth || Hq < 1 || Hq % H != 0 || Hq > kMaxHeadRows / N || !is_head_dim(D) || !is_page(page) || B <= 0 ||
        check_counts(B, width, prefix, page))
        return 0;
    const int64_t need = attn_workspace_bytes(N, (int)Hq, (int)H, (int)D, (int)B, width * page, prefix);
    return need > 0 ? (size_t)need : 0;
}

int nvfp4_attn(const void *Q, int64_t ldq, int64_t N, int64_t Hq, const nvfp4_kvcache *cache, const nvfp4_kvbatch *batch, float scale, void *Out, int64_t ldo,
               void *ws, size_t ws_bytes, void *stream)
{
    KvCache c;
    KvBatch b;
    int rc = check_cache(cache, &c);
    if (rc) return rc;
    if (N < 0 || N > kMaxRows || Hq < 1 || Hq % c.heads != 0 || Hq > kMaxWidth / c.D || (N > 0 && Hq > kMaxHeadRows / N)) return NVFP4_ERR_SHAPE;
    rc = check_batch(batch, c, N, &b);
    if (rc) return rc;
    RowSrc q;
    RowDst out;
    rc = check_sizes(N, Hq * c.D);
    if (rc) return rc;
    rc = make_src(Q, NVFP4_SRC_BF16, ldq, N, Hq * c.D, -1, 0, &q);
    if (rc) return rc;
    rc = make_dst(Out, NVFP4_OUT_BF16, ldo, N, Hq * c.D, &out);
    if (rc) return rc;
    if (!isfinite(scale) || !(scale > 0.0f)) return NVFP4_ERR_ENUM;
    // The kernels load page 0 in the place of one that the cache does not have.  Where it has none at all there are no tokens either, whatever the tables say.
    if (c.pages == 0) b.width = 0, b.prefix = 0;
    const int64_t need = N == 0 || b.B == 0 ? 0 : attn_workspace_bytes(N, (int)Hq, c.heads, c.D, b.B, (int64_t)b.width << c.page_log2, b.prefix);
    if (need < 0) return NVFP4_ERR_SHAPE;
    if (need && (!ws || ws_bytes < (size_t)need)) return NVFP4_ERR_WORKSPACE;
    if (need && !aligned(ws, 16)) return NVFP4_ERR_ALIGN;
    if (N == 0 || b.B == 0) return NVFP4_OK;
    return status(launch_attn(static_cast<const uint16_t *>(Q), q.ld, N, (int)Hq, c, b, scale, static_cast<uint16_t *>(Out), out.ld, ws, static_cast<hipStream_t>(stream)));
}

size_t nvfp4_sample_workspace_bytes(int64_t N, int64_t V)
{
    if (N <= 0 || N > kMaxDraws || V < 1 || V > kMaxVocabulary) return 0;
    return sample_workspace_bytes(N, V);
}

int nvfp4_sample(const void *logits, int src_kind, int64_t ld, int64_t N, int64_t V, const float *u, const float *temperature, const int32_t *top_k,
                 const float *top_p, const float *min_p, int64_t *tokens, void *ws, size_t ws_bytes, void *stream)
{
    if (!u || !tokens) return NVFP4_ERR_NULL;
    if (N < 0 || N > kMaxDraws || V < 1 || V > kMaxVocabulary) return NVFP4_ERR_SHAPE;
    int rc = check_sizes(N, V);
    if (rc) return rc;
    RowSrc x;
    rc = make_src(logits, src_kind, ld, N, V, -1, 0, &x);
    if (rc) return rc;
    if (!aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(tokens, 8)) return NVFP4_ERR_ALIGN;
    const size_t need = nvfp4_sample_workspace_bytes(N, V);
    if (need && (!ws || ws_bytes < need)) return NVFP4_ERR_WORKSPACE;
    if (need && !aligned(ws, 16)) return NVFP4_ERR_ALIGN;
    if (N == 0) return NVFP4_OK;
    const SampleArgs a{x.p, x.ld, x.kind == kF32, N, V, temperature, top_p, min_p, u, top_k, tokens};
    return status(launch_sample(a, ws, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
