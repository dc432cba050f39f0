// C ABI of the rotation and the paged cache: argument validation and kernel
// sequencing, as in api.hip.
#include <float.h>
#include <math.h>
#include <string.h>

#include "cache.h"
#include "errors.h"
#include "internal.h"
#include "proxyattn.h"

namespace pa {

static int check_ints(const void* p, const char* name) {
    if (!p) return fail(PROXYATTN_E_INVALID, "%s is NULL", name);
    if ((uintptr_t)p & 3u) return fail(PROXYATTN_E_INVALID, "%s not 4-byte aligned", name);
    return PROXYATTN_OK;
}

// By the bits: the compiler takes floating comparisons to be free of NaN.
static bool finite(double x) {
    uint64_t u;
    memcpy(&u, &x, 8);
    return (u >> 52 & 0x7ff) != 0x7ff;
}

static int check_stride(int64_t stride, int esz, const char* name) {
    if (stride < 0) return fail(PROXYATTN_E_INVALID, "negative %s", name);
    if ((stride * esz) % 16)
        return fail(PROXYATTN_E_UNSUPPORTED, "%s must keep rows 16-byte aligned", name);
    return PROXYATTN_OK;
}

// Validates a norm and rotation of rows of d values.
static int resolve_rotary(const proxyattn_rotary* r, int d, int dtype, int64_t positions,
                          RotaryArgs* out) {
    if (!r) return fail(PROXYATTN_E_INVALID, "rotary is NULL");
    if (r->struct_size != sizeof(proxyattn_rotary))
        return fail(PROXYATTN_E_INVALID, "rotary struct_size %u != %zu", r->struct_size,
                    sizeof(proxyattn_rotary));
    if (r->rotary_dim < 0 || r->rotary_dim > d)
        return fail(PROXYATTN_E_INVALID, "rotary_dim %d outside [0, %d]", r->rotary_dim, d);
    if (r->rotary_dim % 16)
        return fail(PROXYATTN_E_UNSUPPORTED, "rotary_dim %d not a multiple of 16", r->rotary_dim);
    if (r->interleaved != 0 && r->interleaved != 1)
        return fail(PROXYATTN_E_INVALID, "interleaved must be 0 or 1");
    if (r->rotary_dim) {
        PA_TRY(check_ptr(r->cos, "cos"));
        PA_TRY(check_ptr(r->sin, "sin"));
        if (r->table_len < 1) return fail(PROXYATTN_E_INVALID, "table_len %d < 1", r->table_len);
        if (positions > r->table_len)
            return fail(PROXYATTN_E_INVALID, "table_len %d < %lld positions", r->table_len,
                        (long long)positions);
    }
    if (r->q_weight) PA_TRY(check_ptr(r->q_weight, "q_weight"));
    if (r->k_weight) PA_TRY(check_ptr(r->k_weight, "k_weight"));
    if ((r->q_weight || r->k_weight) &&
        (!finite(r->norm_eps) || r->norm_eps <= 0 || r->norm_eps > 1))
        return fail(PROXYATTN_E_INVALID, "norm_eps outside (0, 1]");
    const int esz = dtype == PROXYATTN_BF16 ? 2 : 4;
    PA_TRY(check_stride(r->q_out_tok_stride, esz, "q_out_tok_stride"));
    PA_TRY(check_stride(r->q_out_head_stride, esz, "q_out_head_stride"));
    PA_TRY(check_stride(r->k_out_tok_stride, esz, "k_out_tok_stride"));
    PA_TRY(check_stride(r->k_out_head_stride, esz, "k_out_head_stride"));
    *out = RotaryArgs{r->rotary_dim, r->interleaved, r->table_len, r->norm_eps, r->cos, r->sin,
                      r->q_weight, r->k_weight};
    return PROXYATTN_OK;
}

static int64_t pick(int64_t stride, int64_t packed) { return stride ? stride : packed; }

// An output over its own input reads each row before it writes it, where the
// rows lie on one another.
static int check_in_place(const void* in, const void* out, int64_t tok, int64_t head, int64_t otok,
                          int64_t ohead, const char* name) {
    if (in == out && (tok != otok || head != ohead))
        return fail(PROXYATTN_E_INVALID, "%s in place with other strides than its input's", name);
    return PROXYATTN_OK;
}

// Validates the descriptor and resolves it into a CacheShape.
static int resolve_cache(const proxyattn_cache* c, CacheShape* out) {
    if (!c) return fail(PROXYATTN_E_INVALID, "cache is NULL");
    if (c->struct_size != sizeof(proxyattn_cache))
        return fail(PROXYATTN_E_INVALID, "cache struct_size %u != %zu", c->struct_size,
                    sizeof(proxyattn_cache));
    if (c->num_seqs < 0 || c->num_tokens < 0)
        return fail(PROXYATTN_E_INVALID, "num_seqs %d or num_tokens %d < 0", c->num_seqs,
                    c->num_tokens);
    if (c->num_seqs > kMaxSeqs)
        return fail(PROXYATTN_E_UNSUPPORTED, "num_seqs %d > %d", c->num_seqs, kMaxSeqs);
    // workgroups of 256 threads to four tokens each: 2^31 threads, and a grid ends below 2^32
    if (c->num_tokens > 1 << 25)
        return fail(PROXYATTN_E_UNSUPPORTED, "num_tokens %d > 2^25", c->num_tokens);
    if (c->max_new < 1 || c->max_len < 1 || c->num_pages < 1 || c->table_width < 1)
        return fail(PROXYATTN_E_INVALID,
                    "max_new, max_len, num_pages and table_width must be positive");
    if (c->num_q_heads <= 0 || c->num_kv_heads <= 0)
        return fail(PROXYATTN_E_INVALID, "head counts must be positive");
    if (c->num_q_heads > 4096)
        return fail(PROXYATTN_E_UNSUPPORTED, "num_q_heads %d > 4096", c->num_q_heads);
    if (c->num_q_heads % c->num_kv_heads)
        return fail(PROXYATTN_E_UNSUPPORTED, "num_q_heads %% num_kv_heads != 0");
    if (c->head_dim != 64 && c->head_dim != 128)
        return fail(PROXYATTN_E_UNSUPPORTED, "head_dim %d not in {64, 128}", c->head_dim);
    int shift = 4;
    while (shift < 8 && (1 << shift) != c->page_size) ++shift;
    if ((1 << shift) != c->page_size)
        return fail(PROXYATTN_E_UNSUPPORTED, "page_size %d not in {16, 32, 64, 128, 256}",
                    c->page_size);
    if ((int64_t)c->table_width * c->page_size > (1 << 30))
        return fail(PROXYATTN_E_UNSUPPORTED, "table_width * page_size > 2^30");
    if (c->max_len > (int64_t)c->table_width * c->page_size)
        return fail(PROXYATTN_E_INVALID, "max_len %d > table_width * page_size", c->max_len);
    if (c->dtype != PROXYATTN_BF16 && c->dtype != PROXYATTN_F32)
        return fail(PROXYATTN_E_UNSUPPORTED, "dtype %d", c->dtype);
    if (c->cache_type != PROXYATTN_CACHE_SAME && c->cache_type != PROXYATTN_CACHE_FP4)
        return fail(PROXYATTN_E_UNSUPPORTED, "cache_type %d", c->cache_type);
    if (!finite((double)c->softmax_scale))
        return fail(PROXYATTN_E_INVALID, "softmax_scale is not finite");
    if (c->softmax_scale > 0.f && c->softmax_scale < FLT_MIN)
        return fail(PROXYATTN_E_INVALID, "softmax_scale below 2^-126");
    const int esz = c->dtype == PROXYATTN_BF16 ? 2 : 4;
    const int64_t d = c->head_dim;
    CacheShape s{};
    s.b = c->num_seqs;
    s.t = c->num_tokens;
    s.max_new = c->max_new;
    s.max_len = c->max_len;
    s.hq = c->num_q_heads;
    s.hkv = c->num_kv_heads;
    s.d = c->head_dim;
    s.rep = s.hq / s.hkv;
    s.page_shift = shift;
    s.num_pages = c->num_pages;
    s.width = c->table_width;
    s.dtype = c->dtype;
    s.fp4 = c->cache_type == PROXYATTN_CACHE_FP4;
    // Pages that fill over half of the MALL are not there any more when the next
    // step reads them again, and read faster past it (16 sequences to 64K tokens,
    // bf16, 600 MB: 128.7 -> 114.8 us; 131K in 4 bits, 143 MB: 38.4 -> 38.0); smaller
    // ones would lose what stays there (64 sequences, 109 MB: 36.9 -> 38.3).
    const size_t rows = (size_t)s.num_pages * s.hkv << shift;
    s.past = 2 * rows * (s.fp4 ? d / 2 + d / 32 : d * esz) > kMallBytes / 2;
    const float scale =
        c->softmax_scale > 0.f ? c->softmax_scale : (float)(1.0 / sqrt((double)c->head_dim));
    const double scale2 = (double)scale * 1.4426950408889634;
    s.scale2 = (float)scale2;
    if ((double)s.scale2 >= scale2) s.scale2 = nextafterf(s.scale2, 0.f);
    s.scale2_rest = fmaxf((float)(scale2 - (double)s.scale2), FLT_MIN);
    s.q_tok = pick(c->q_tok_stride, s.hq * d);
    s.q_head = pick(c->q_head_stride, d);
    s.kv_tok = pick(c->kv_tok_stride, s.hkv * d);
    s.kv_head = pick(c->kv_head_stride, d);
    s.o_tok = pick(c->o_tok_stride, s.hq * d);
    s.o_head = pick(c->o_head_stride, d);
    PA_TRY(check_stride(s.q_tok, esz, "q_tok_stride"));
    PA_TRY(check_stride(s.q_head, esz, "q_head_stride"));
    PA_TRY(check_stride(s.kv_tok, esz, "kv_tok_stride"));
    PA_TRY(check_stride(s.kv_head, esz, "kv_head_stride"));
    PA_TRY(check_stride(s.o_tok, esz, "o_tok_stride"));
    PA_TRY(check_stride(s.o_head, esz, "o_head_stride"));
    *out = s;
    return PROXYATTN_OK;
}

// Arrays of a batch and its pages.
static int check_batch(const CacheShape& s, const int32_t* page_table, const int32_t* seq_lens,
                       const int32_t* new_start, const void* kp, const void* vp, const void* ks,
                       const void* vs) {
    PA_TRY(check_ints(page_table, "page_table"));
    PA_TRY(check_ints(seq_lens, "seq_lens"));
    if (new_start)
        PA_TRY(check_ints(new_start, "new_start"));
    else if (s.t < s.b)
        return fail(PROXYATTN_E_INVALID, "num_tokens %d < num_seqs %d without new_start", s.t, s.b);
    PA_TRY(check_ptr(kp, "k_pages"));
    PA_TRY(check_ptr(vp, "v_pages"));
    if (s.fp4) {
        PA_TRY(check_ptr(ks, "k_scales"));
        PA_TRY(check_ptr(vs, "v_scales"));
    } else if (ks || vs) {
        return fail(PROXYATTN_E_INVALID, "scales of a cache in the problem's dtype");
    }
    return PROXYATTN_OK;
}

}  // namespace pa

using namespace pa;

extern "C" {

int proxyattn_norm_rotate(const proxyattn_problem* p, const proxyattn_rotary* r, const void* q,
                          const void* k, const int32_t* positions, int32_t first_position,
                          void* q_out, void* k_out, void* stream) {
    clear_error();
    Shape sh;
    PA_TRY(resolve(p, &sh));
    if (first_position < 0) return fail(PROXYATTN_E_INVALID, "first_position < 0");
    RotaryArgs ra;
    PA_TRY(resolve_rotary(r, sh.d, sh.dtype, positions ? 1 : (int64_t)first_position + sh.n, &ra));
    if (!q != !q_out || !k != !k_out)
        return fail(PROXYATTN_E_INVALID, "q and q_out, or k and k_out: one is NULL");
    if (sh.n == 0 || (!q && !k)) return PROXYATTN_OK;
    RotateRows w{};
    w.q = q;
    w.k = k;
    w.qo = q_out;
    w.ko = k_out;
    w.positions = positions;
    w.first = first_position;
    w.n = sh.n;
    w.hq = sh.hq;
    w.hkv = sh.hkv;
    w.d = sh.d;
    w.dtype = sh.dtype;
    w.q_tok = sh.q_tok;
    w.q_head = sh.q_head;
    w.k_tok = sh.kv_tok;
    w.k_head = sh.kv_head;
    w.qo_tok = pick(r->q_out_tok_stride, (int64_t)sh.hq * sh.d);
    w.qo_head = pick(r->q_out_head_stride, sh.d);
    w.ko_tok = pick(r->k_out_tok_stride, (int64_t)sh.hkv * sh.d);
    w.ko_head = pick(r->k_out_head_stride, sh.d);
    if (q) {
        PA_TRY(check_ptr(q, "q"));
        PA_TRY(check_ptr(q_out, "q_out"));
        PA_TRY(check_in_place(q, q_out, w.q_tok, w.q_head, w.qo_tok, w.qo_head, "q_out"));
    }
    if (k) {
        PA_TRY(check_ptr(k, "k"));
        PA_TRY(check_ptr(k_out, "k_out"));
        PA_TRY(check_in_place(k, k_out, w.k_tok, w.k_head, w.ko_tok, w.ko_head, "k_out"));
    }
    if (positions) PA_TRY(check_ints(positions, "positions"));
    PA_LAUNCH(launch_norm_rotate(w, ra, (hipStream_t)stream), "norm_rotate");
    return PROXYATTN_OK;
}

int proxyattn_cache_size(const proxyattn_cache* c, size_t* page_bytes, size_t* scale_bytes) {
    clear_error();
    CacheShape s;
    PA_TRY(resolve_cache(c, &s));
    if (!page_bytes || !scale_bytes) return fail(PROXYATTN_E_INVALID, "a size pointer is NULL");
    const size_t rows = (size_t)s.num_pages * s.hkv << s.page_shift;
    const size_t esz = s.dtype == PROXYATTN_BF16 ? 2 : 4;
    *page_bytes = s.fp4 ? rows * (s.d / 2) : rows * s.d * esz;
    *scale_bytes = s.fp4 ? rows * (s.d / 32) : 0;
    return PROXYATTN_OK;
}

int proxyattn_cache_append(const proxyattn_cache* c, const proxyattn_rotary* r, const void* q,
                           const void* k, const void* v, void* q_out, const int32_t* page_table,
                           const int32_t* seq_lens, const int32_t* new_start, void* k_pages,
                           void* v_pages, void* k_scales, void* v_scales, void* stream) {
    clear_error();
    CacheShape s;
    PA_TRY(resolve_cache(c, &s));
    RotaryArgs ra{};
    AppendArgs a{};
    if (r) {
        PA_TRY(resolve_rotary(r, s.d, s.dtype, s.max_len, &ra));
        a.norm_rotate = 1;
        a.qo_tok = pick(r->q_out_tok_stride, (int64_t)s.hq * s.d);
        a.qo_head = pick(r->q_out_head_stride, s.d);
    } else if (q || q_out) {
        return fail(PROXYATTN_E_INVALID, "q and q_out need a rotary");
    }
    if (!q != !q_out) return fail(PROXYATTN_E_INVALID, "q or q_out is NULL");
    if (s.b == 0 || s.t == 0) return PROXYATTN_OK;
    PA_TRY(check_ptr(k, "k"));
    PA_TRY(check_ptr(v, "v"));
    if (q) {
        PA_TRY(check_ptr(q, "q"));
        PA_TRY(check_ptr(q_out, "q_out"));
        PA_TRY(check_in_place(q, q_out, s.q_tok, s.q_head, a.qo_tok, a.qo_head, "q_out"));
    }
    PA_TRY(check_batch(s, page_table, seq_lens, new_start, k_pages, v_pages, k_scales, v_scales));
    a.q = q;
    a.k = k;
    a.v = v;
    a.qo = q_out;
    PA_LAUNCH(launch_cache_append(s, ra, a, page_table, seq_lens, new_start,
                                  PagePtrs{k_pages, v_pages, k_scales, v_scales},
                                  (hipStream_t)stream),
              "cache_append");
    return PROXYATTN_OK;
}

int proxyattn_cache_read(const proxyattn_cache* c, const int32_t* page_table,
                         const int32_t* seq_lens, const int32_t* new_start, const void* k_pages,
                         const void* v_pages, const void* k_scales, const void* v_scales,
                         void* k_out, void* v_out, void* stream) {
    clear_error();
    CacheShape s;
    PA_TRY(resolve_cache(c, &s));
    if (s.b == 0 || s.t == 0 || (!k_out && !v_out)) return PROXYATTN_OK;
    if (k_out) PA_TRY(check_ptr(k_out, "k_out"));
    if (v_out) PA_TRY(check_ptr(v_out, "v_out"));
    PA_TRY(check_batch(s, page_table, seq_lens, new_start, k_pages, v_pages, k_scales, v_scales));
    PA_LAUNCH(launch_cache_read(s, page_table, seq_lens, new_start,
                                PagePtrs{(void*)k_pages, (void*)v_pages, (void*)k_scales,
                                         (void*)v_scales},
                                k_out, v_out, (hipStream_t)stream),
              "cache_read");
    return PROXYATTN_OK;
}

static int resolve_cache_ws(const CacheShape& s, CacheWs* w) {
    if (!cache_ws(s, w))
        return fail(PROXYATTN_E_UNSUPPORTED, "too many (sequence, head, key) units: num_seqs %d, "
                    "max_new %d, max_len %d", s.b, s.max_new, s.max_len);
    return PROXYATTN_OK;
}

int proxyattn_cache_workspace_size(const proxyattn_cache* c, size_t* bytes) {
    clear_error();
    CacheShape s;
    PA_TRY(resolve_cache(c, &s));
    CacheWs w;
    PA_TRY(resolve_cache_ws(s, &w));
    if (!bytes) return fail(PROXYATTN_E_INVALID, "bytes is NULL");
    *bytes = s.b == 0 || s.t == 0 ? 0 : w.total;
    return PROXYATTN_OK;
}

int proxyattn_cache_attention(const proxyattn_cache* c, const void* q, const int32_t* page_table,
                              const int32_t* seq_lens, const int32_t* new_start,
                              const void* k_pages, const void* v_pages, const void* k_scales,
                              const void* v_scales, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
    clear_error();
    CacheShape s;
    PA_TRY(resolve_cache(c, &s));
    CacheWs w;
    PA_TRY(resolve_cache_ws(s, &w));
    if (s.b == 0 || s.t == 0) return PROXYATTN_OK;
    PA_TRY(check_ptr(q, "q"));
    PA_TRY(check_ptr(out, "out"));
    if (lse && ((uintptr_t)lse & 3u)) return fail(PROXYATTN_E_INVALID, "lse not 4-byte aligned");
    PA_TRY(check_batch(s, page_table, seq_lens, new_start, k_pages, v_pages, k_scales, v_scales));
    if (w.total) PA_TRY(check_ptr(workspace, "workspace"));
    if (workspace_bytes < w.total)
        return fail(PROXYATTN_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes,
                    w.total);
    PA_LAUNCH(launch_cache_attention(s, q, page_table, seq_lens, new_start,
                                     PagePtrs{(void*)k_pages, (void*)v_pages, (void*)k_scales,
                                              (void*)v_scales},
                                     out, lse, (char*)workspace, w, (hipStream_t)stream),
              "cache_attention");
    return PROXYATTN_OK;
}

}  // extern "C"
