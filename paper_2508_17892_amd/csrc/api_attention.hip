// C ABI of libilre, the operators around a recall: rotary positions, fill of a paged cache, attention.  Host code only; the kernels live in rope.hip and
// attention.hip.
#include <math.h>

#include "ilre_internal.h"

namespace {

using ilre::fail;
using ilre::hip_fail;

int check_common(const ilre_opts *o, int32_t T, int32_t Hq, int32_t d)
{
    const int rc = ilre::check_opts(o);
    if (rc) return rc;
    if (T < 0 || Hq < 1) return fail(ILRE_EINVAL, "T must be non-negative, the number of heads positive");
    if (d != ILRE_HEAD_DIM) return fail(ILRE_EUNSUPPORTED, "head_dim %d unsupported (only %d)", d, ILRE_HEAD_DIM);
    if (o->dtype != ILRE_F32 && o->dtype != ILRE_BF16) return fail(ILRE_EUNSUPPORTED, "unknown dtype %d", o->dtype);
    if ((int64_t)Hq * T > 0x3FFFFFFF || T > 4 * ilre::kMaxUnits) return fail(ILRE_EUNSUPPORTED, "too many query rows");
    return ILRE_OK;
}

// Byte strides of a tensor [tokens, heads, d].
int bytes_of(const char *what, const void *p, int64_t token, int64_t head, int heads, int es, int64_t *token_bytes, int64_t *head_bytes)
{
    if ((uintptr_t)p & 15) return fail(ILRE_EINVAL, "%s must be 16-byte aligned", what);
    const int64_t t = token ? token : (int64_t)heads * ILRE_HEAD_DIM, h = head ? head : ILRE_HEAD_DIM;
    if (t < ILRE_HEAD_DIM || h < ILRE_HEAD_DIM) return fail(ILRE_EINVAL, "%s: strides must be >= d (rows may not overlap)", what);
    if (t * es % 16 != 0 || h * es % 16 != 0) return fail(ILRE_EINVAL, "%s: strides must be multiples of 16 bytes", what);
    // tile copies address the 16 tokens of a page's part with 32-bit offsets
    if (t > (int64_t)0x7FFFFFF / es) return fail(ILRE_EUNSUPPORTED, "%s: token stride %lld too large", what, (long long)t);
    *token_bytes = t * es;
    *head_bytes = h * es;
    return ILRE_OK;
}

int check_freqs(const ilre_rope_freqs *f, int32_t d, int32_t pairing)
{
    if (!f) return fail(ILRE_EINVAL, "freqs is null");
    if (f->struct_size != (int32_t)sizeof(ilre_rope_freqs)) return fail(ILRE_EINVAL, "freqs->struct_size %d != %zu", f->struct_size, sizeof(ilre_rope_freqs));
    if (f->rotary < 2 || f->rotary > d) return fail(ILRE_EINVAL, "rotary must be in [2, d]");
    if (f->rotary % 16 != 0) return fail(ILRE_EUNSUPPORTED, "rotary %d unsupported (multiples of 16 only)", f->rotary);
    if (!isfinite(f->magnitude)) return fail(ILRE_EINVAL, "magnitude is not finite");
    for (int j = 0; j < f->rotary / 2; ++j)
        if (!isfinite(f->inv_freq[j])) return fail(ILRE_EINVAL, "inv_freq[%d] is not finite", j);
    if (pairing != ILRE_ROPE_HALF && pairing != ILRE_ROPE_INTERLEAVED) return fail(ILRE_EUNSUPPORTED, "unknown pairing %d", pairing);
    return ILRE_OK;
}

void fill_freqs(ilre::TurnArgs &a, const ilre_rope_freqs *f)
{
    a.rotary = f->rotary;
    a.magnitude = (float)f->magnitude;
    for (int j = 0; j < f->rotary / 2; ++j) a.turns[j] = f->inv_freq[j] / (2.0 * M_PI);
}

struct Cache {
    int64_t page_bytes, head_bytes, token_bytes, table_stride, kv_limit;
    int page_shift;
};

int check_cache(const ilre_paged_kv *c, int32_t Hq, int es, bool values, Cache &out)
{
    if (!c) return fail(ILRE_EINVAL, "cache is null");
    if (c->struct_size != (int32_t)sizeof(ilre_paged_kv)) return fail(ILRE_EINVAL, "cache->struct_size %d != %zu", c->struct_size, sizeof(ilre_paged_kv));
    if (!c->k_pages || (values && !c->v_pages)) return fail(ILRE_EINVAL, "k_pages or v_pages is null");
    if (!c->page_table || !c->kv_len || !c->cu_q) return fail(ILRE_EINVAL, "page_table, kv_len or cu_q is null");
    if (c->n_seq < 1 || c->num_pages < 1 || c->table_width < 1 || c->Hkv < 1) return fail(ILRE_EINVAL, "n_seq, num_pages, table_width and Hkv must be positive");
    if (Hq % c->Hkv != 0) return fail(ILRE_EINVAL, "Hq (%d) must be a multiple of Hkv (%d)", Hq, c->Hkv);
    const int P = c->page_tokens;
    if (P < 1 || (P & (P - 1))) return fail(ILRE_EINVAL, "page_tokens %d must be a power of two", P);
    if (P < ILRE_MIN_PAGE_TOKENS || P > ILRE_MAX_PAGE_TOKENS)
        return fail(ILRE_EUNSUPPORTED, "page_tokens %d unsupported (%d .. %d)", P, ILRE_MIN_PAGE_TOKENS, ILRE_MAX_PAGE_TOKENS);
    if (((uintptr_t)c->k_pages & 15) || ((uintptr_t)c->v_pages & 15)) return fail(ILRE_EINVAL, "k_pages and v_pages must be 16-byte aligned");
    const bool given = c->stride_page || c->stride_head || c->stride_token;
    const int64_t t = given ? c->stride_token : ILRE_HEAD_DIM, h = given ? c->stride_head : (int64_t)P * ILRE_HEAD_DIM,
                  p = given ? c->stride_page : (int64_t)c->Hkv * P * ILRE_HEAD_DIM;
    if (t < ILRE_HEAD_DIM || h < ILRE_HEAD_DIM || p < ILRE_HEAD_DIM) return fail(ILRE_EINVAL, "cache strides must be >= d (rows may not overlap)");
    if (t * es % 16 != 0 || h * es % 16 != 0 || p * es % 16 != 0) return fail(ILRE_EINVAL, "cache strides must be multiples of 16 bytes");
    if (t > (int64_t)0x7FFFFFF / es) return fail(ILRE_EUNSUPPORTED, "cache token stride %lld too large", (long long)t);
    if (c->table_stride != 0 && c->table_stride < c->table_width) return fail(ILRE_EINVAL, "table_stride is less than table_width");
    out.token_bytes = t * es;
    out.head_bytes = h * es;
    out.page_bytes = p * es;
    out.table_stride = c->table_stride ? c->table_stride : c->table_width;
    out.page_shift = __builtin_ctz((unsigned)P);
    const int64_t room = (int64_t)c->table_width * P, most = 0x7FFFFFFFll - 65536;
    out.kv_limit = room < most ? room : most;
    return ILRE_OK;
}

int check_attn(const ilre_attn *t)
{
    if (!t) return fail(ILRE_EINVAL, "attn is null");
    if (t->struct_size != (int32_t)sizeof(ilre_attn)) return fail(ILRE_EINVAL, "attn->struct_size %d != %zu", t->struct_size, sizeof(ilre_attn));
    if (t->causal != 0 && t->causal != 1) return fail(ILRE_EINVAL, "causal must be 0 or 1");
    if (t->sink < 0 || t->window < 0) return fail(ILRE_EINVAL, "sink and window must be non-negative");
    if (t->window > 0 && !t->causal) return fail(ILRE_EINVAL, "a window needs the causal mask");
    if (t->sink > 0 && t->window == 0) return fail(ILRE_EINVAL, "a sink part needs a window (without one every row sees it anyway)");
    if (t->max_q < 0 || t->max_kv < 0 || t->total_kv < 0) return fail(ILRE_EINVAL, "max_q, max_kv and total_kv must be non-negative");
    return ILRE_OK;
}

int run(ilre::AttnArgs &a, const ilre_attn *t, const ilre_opts *o)
{
    a.causal = t->causal;
    a.sink = t->sink;
    a.window = t->window;
    a.G = a.Hq / a.Hkv;
    a.c = (o->scale > 0.f ? o->scale : 1.0f / sqrtf((float)ILRE_HEAD_DIM)) * 1.4426950408889634f;
    if (a.lse && ((uintptr_t)a.lse & 3)) return fail(ILRE_EINVAL, "lse must be 4-byte aligned");
    if (o->workspace && ((uintptr_t)o->workspace & 255)) return fail(ILRE_EINVAL, "workspace must be 256-byte aligned");
    if (a.T == 0) return ILRE_OK;
    const ilre::AttnPlan p = ilre::make_attn_plan(o->dtype, a.T, a.n_seq, a.Hq, a.Hkv, t->max_q, t->max_kv, t->total_kv, t->sink, t->window,
                                                  o->workspace ? o->workspace_bytes : 0);
    if ((int64_t)p.nblocks * a.Hkv > ilre::kMaxUnits) return fail(ILRE_EUNSUPPORTED, "too many query rows");
    const hipError_t e = ilre::launch_attention(p, a, o->workspace, (hipStream_t)o->stream);
    return e == hipSuccess ? ILRE_OK : hip_fail(e, "attention launch");
}

}  // namespace

extern "C" {

int ilre_rope_frequencies(int32_t rotary, double base, int32_t scaling, double factor, double low, double high, int32_t original_len, ilre_rope_freqs *out)
{
    if (!out) return fail(ILRE_EINVAL, "out is null");
    if (rotary < 2 || rotary > ILRE_HEAD_DIM) return fail(ILRE_EINVAL, "rotary must be in [2, %d]", ILRE_HEAD_DIM);
    if (rotary % 16 != 0) return fail(ILRE_EUNSUPPORTED, "rotary %d unsupported (multiples of 16 only)", rotary);
    if (!(base > 0.0) || !isfinite(base)) return fail(ILRE_EINVAL, "base must be positive and finite");
    if (scaling < ILRE_ROPE_PLAIN || scaling > ILRE_ROPE_PARTS) return fail(ILRE_EUNSUPPORTED, "unknown scaling %d", scaling);
    if (scaling != ILRE_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return fail(ILRE_EINVAL, "factor must be finite and >= 1");
    if (scaling >= ILRE_ROPE_BANDS) {
        if (!(low > 0.0) || !(high > low) || !isfinite(high)) return fail(ILRE_EINVAL, "0 < low < high must hold");
        if (original_len < 1) return fail(ILRE_EINVAL, "original_len must be positive");
        if (scaling == ILRE_ROPE_PARTS && base == 1.0) return fail(ILRE_EINVAL, "base 1 has no pairs to part");
    }
    ilre_rope_freqs f{};
    f.struct_size = (int32_t)sizeof f;
    f.rotary = rotary;
    f.magnitude = scaling == ILRE_ROPE_PARTS ? 0.1 * log(factor) + 1.0 : 1.0;
    double first = 0.0, width = 1.0;
    if (scaling == ILRE_ROPE_PARTS) {
        auto pair = [&](double turns) { return rotary * log(original_len / (turns * 2.0 * M_PI)) / (2.0 * log(base)); };
        first = fmax(floor(pair(high)), 0.0);
        width = fmax(fmin(ceil(pair(low)), rotary - 1.0) - first, 1e-3);
    }
    for (int j = 0; j < rotary / 2; ++j) {
        const double x = pow(base, -2.0 * j / rotary);
        double keep = 1.0;  // of the frequency as it is; the rest of it divided
        if (scaling == ILRE_ROPE_LINEAR) keep = 0.0;
        if (scaling == ILRE_ROPE_BANDS) keep = fmin(1.0, fmax(0.0, (original_len * x / (2.0 * M_PI) - low) / (high - low)));
        if (scaling == ILRE_ROPE_PARTS) keep = 1.0 - fmin(1.0, fmax(0.0, (j - first) / width));
        f.inv_freq[j] = scaling == ILRE_ROPE_PLAIN ? x : x * keep + x / factor * (1.0 - keep);
    }
    *out = f;
    return ILRE_OK;
}

int ilre_rope(const void *x, void *out, int32_t T, int32_t H, int32_t d, const int32_t *positions, int32_t first_position, const ilre_rope_freqs *freqs,
              int32_t pairing, const ilre_strides *strides, const ilre_opts *opts)
{
    int rc = check_common(opts, T, H, d);
    if (rc || (rc = check_freqs(freqs, d, pairing))) return rc;
    if (!x || !out || !strides) return fail(ILRE_EINVAL, "x, out or strides is null");
    const int es = opts->dtype == ILRE_BF16 ? 2 : 4;
    ilre::TurnArgs a{};
    if ((rc = bytes_of("x", x, strides->q_token, strides->q_head, H, es, &a.q_token, &a.q_head))) return rc;
    if ((rc = bytes_of("out", out, strides->out_token, strides->out_head, H, es, &a.out_token, &a.out_head))) return rc;
    if (x == out && (a.q_token != a.out_token || a.q_head != a.out_head)) return fail(ILRE_EINVAL, "in place, out has to have the strides of x");
    if (T == 0) return ILRE_OK;
    a.q = (const unsigned char *)x;
    a.q_out = (unsigned char *)out;
    a.positions = positions;
    a.first_position = first_position;
    a.T = T;
    a.Hq = H;
    fill_freqs(a, freqs);
    const hipError_t e = ilre::launch_turn(a, opts->dtype, pairing, (hipStream_t)opts->stream);
    return e == hipSuccess ? ILRE_OK : hip_fail(e, "RoPE launch");
}

int ilre_rope_append(const void *q, void *q_out, const void *k, const void *v, int32_t T, int32_t Hq, int32_t d, const int32_t *positions,
                     const ilre_rope_freqs *freqs, int32_t pairing, const ilre_paged_kv *cache, const ilre_strides *strides, const ilre_opts *opts)
{
    int rc = check_common(opts, T, Hq, d);
    if (rc || (rc = check_freqs(freqs, d, pairing))) return rc;
    if (!k || !strides) return fail(ILRE_EINVAL, "k or strides is null");
    if (!q != !q_out) return fail(ILRE_EINVAL, "q and q_out go together");
    const int es = opts->dtype == ILRE_BF16 ? 2 : 4;
    Cache c;
    if ((rc = check_cache(cache, Hq, es, v != nullptr, c))) return rc;
    ilre::TurnArgs a{};
    if (q) {
        if ((rc = bytes_of("q", q, strides->q_token, strides->q_head, Hq, es, &a.q_token, &a.q_head))) return rc;
        if ((rc = bytes_of("q_out", q_out, strides->out_token, strides->out_head, Hq, es, &a.out_token, &a.out_head))) return rc;
        if (q == q_out && (a.q_token != a.out_token || a.q_head != a.out_head)) return fail(ILRE_EINVAL, "in place, q_out has to have the strides of q");
    }
    if ((rc = bytes_of("k", k, strides->k_token, strides->k_head, cache->Hkv, es, &a.k_token, &a.k_head))) return rc;
    if (v && (rc = bytes_of("v", v, strides->v_token, strides->v_head, cache->Hkv, es, &a.v_token, &a.v_head))) return rc;
    if (T == 0) return ILRE_OK;
    a.q = (const unsigned char *)q;
    a.q_out = (unsigned char *)q_out;
    a.k = (const unsigned char *)k;
    a.v = (const unsigned char *)v;
    a.positions = positions;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = cache->Hkv;
    a.k_pages = (unsigned char *)cache->k_pages;
    a.v_pages = (unsigned char *)cache->v_pages;
    a.page_bytes = c.page_bytes;
    a.head_bytes = c.head_bytes;
    a.token_bytes = c.token_bytes;
    a.table = cache->page_table;
    a.kv_len = cache->kv_len;
    a.cu_q = cache->cu_q;
    a.table_stride = c.table_stride;
    a.kv_limit = c.kv_limit;
    a.n_seq = cache->n_seq;
    a.num_pages = cache->num_pages;
    a.page_shift = c.page_shift;
    fill_freqs(a, freqs);
    const hipError_t e = ilre::launch_turn(a, opts->dtype, pairing, (hipStream_t)opts->stream);
    return e == hipSuccess ? ILRE_OK : hip_fail(e, "RoPE launch");
}

int ilre_attention_workspace_bytes(int32_t T, int32_t n_seq, int32_t Hq, int32_t Hkv, int32_t d, int32_t max_q, int32_t max_kv, int64_t total_kv, int32_t dtype,
                                   size_t *out_bytes)
{
    if (!out_bytes) return fail(ILRE_EINVAL, "out_bytes is null");
    if (T < 0 || n_seq < 1 || Hq < 1 || Hkv < 1 || max_q < 0 || max_kv < 0 || total_kv < 0)
        return fail(ILRE_EINVAL, "T, max_q, max_kv and total_kv must be non-negative, n_seq, Hq and Hkv positive");
    if (Hq % Hkv != 0) return fail(ILRE_EINVAL, "Hq (%d) must be a multiple of Hkv (%d)", Hq, Hkv);
    if (d != ILRE_HEAD_DIM) return fail(ILRE_EUNSUPPORTED, "head_dim %d unsupported (only %d)", d, ILRE_HEAD_DIM);
    if (dtype != ILRE_F32 && dtype != ILRE_BF16) return fail(ILRE_EUNSUPPORTED, "unknown dtype %d", dtype);
    if ((int64_t)Hq * T > 0x3FFFFFFF) return fail(ILRE_EUNSUPPORTED, "too many query rows");
    *out_bytes = T == 0 ? 0 : ilre::make_attn_plan(dtype, T, n_seq, Hq, Hkv, max_q, max_kv, total_kv, 0, 0, (size_t)1 << 62).bytes;
    return ILRE_OK;
}

int ilre_paged_attention(const void *q, void *out, float *lse, int32_t T, int32_t Hq, int32_t d, const ilre_attn *attn, const ilre_paged_kv *cache,
                         const ilre_strides *strides, const ilre_opts *opts)
{
    int rc = check_common(opts, T, Hq, d);
    if (rc || (rc = check_attn(attn))) return rc;
    if (!q || !out || !strides) return fail(ILRE_EINVAL, "q, out or strides is null");
    const int es = opts->dtype == ILRE_BF16 ? 2 : 4;
    Cache c;
    if ((rc = check_cache(cache, Hq, es, true, c))) return rc;
    ilre::AttnArgs a{};
    if ((rc = bytes_of("q", q, strides->q_token, strides->q_head, Hq, es, &a.q_token, &a.q_head))) return rc;
    if ((rc = bytes_of("out", out, strides->out_token, strides->out_head, Hq, es, &a.out_token, &a.out_head))) return rc;
    a.q = (const unsigned char *)q;
    a.out = (unsigned char *)out;
    a.lse = lse;
    a.k = (const unsigned char *)cache->k_pages;
    a.v = (const unsigned char *)cache->v_pages;
    a.k_page = a.v_page = c.page_bytes;
    a.k_head = a.v_head = c.head_bytes;
    a.k_token = a.v_token = c.token_bytes;
    a.table = cache->page_table;
    a.kv_len = cache->kv_len;
    a.cu_q = cache->cu_q;
    a.table_stride = c.table_stride;
    a.kv_limit = c.kv_limit;
    a.table_width = cache->table_width;
    a.page_shift = c.page_shift;
    a.num_pages = cache->num_pages;
    a.T = T;
    a.n_seq = cache->n_seq;
    a.Hq = Hq;
    a.Hkv = cache->Hkv;
    return run(a, attn, opts);
}

int ilre_prompt_attention(const void *q, const void *k, const void *v, void *out, float *lse, int32_t T, int32_t Tk, int32_t Hq, int32_t Hkv, int32_t d,
                          const int32_t *cu_q, const int32_t *cu_k, int32_t n_seq, const ilre_attn *attn, const ilre_strides *strides, const ilre_opts *opts)
{
    int rc = check_common(opts, T, Hq, d);
    if (rc || (rc = check_attn(attn))) return rc;
    if (!q || ((!k || !v) && Tk != 0) || !out || !strides || !cu_q) return fail(ILRE_EINVAL, "q, k, v, out, cu_q or strides is null");
    if (Hkv < 1 || n_seq < 1 || Tk < 0) return fail(ILRE_EINVAL, "Hkv and n_seq must be positive, Tk non-negative");
    if (Hq % Hkv != 0) return fail(ILRE_EINVAL, "Hq (%d) must be a multiple of Hkv (%d)", Hq, Hkv);
    if (!cu_k && Tk != T) return fail(ILRE_EINVAL, "without cu_k there are as many keys as queries");
    if (Tk > 0x7FFFFFFF - 65536) return fail(ILRE_EUNSUPPORTED, "too many keys");
    const int es = opts->dtype == ILRE_BF16 ? 2 : 4;
    ilre::AttnArgs a{};
    if ((rc = bytes_of("q", q, strides->q_token, strides->q_head, Hq, es, &a.q_token, &a.q_head))) return rc;
    if ((rc = bytes_of("out", out, strides->out_token, strides->out_head, Hq, es, &a.out_token, &a.out_head))) return rc;
    if ((rc = bytes_of("k", k, strides->k_token, strides->k_head, Hkv, es, &a.k_token, &a.k_head))) return rc;
    if ((rc = bytes_of("v", v, strides->v_token, strides->v_head, Hkv, es, &a.v_token, &a.v_head))) return rc;
    a.q = (const unsigned char *)q;
    a.k = (const unsigned char *)k;
    a.v = (const unsigned char *)v;
    a.out = (unsigned char *)out;
    a.lse = lse;
    a.cu_q = cu_q;
    a.cu_k = cu_k ? cu_k : cu_q;
    a.T = T;
    a.Tk = Tk;
    a.n_seq = n_seq;
    a.Hq = Hq;
    a.Hkv = Hkv;
    return run(a, attn, opts);
}

}  // extern "C"
