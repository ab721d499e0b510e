// Argument checks of the attention side of a layer (see include/patch.h) and what the kernels are told.  No device arithmetic here.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/patch.h"
#include "attention.h"
#include "kernels.h"
#include "seqs.h"

using namespace patch;

static bool aligned(const void* p, uintptr_t n = 16) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
static bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

static patch_status launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PATCH_OK;
    patch_note_hip_error((int)e);
    return PATCH_ERR_HIP;
}

// writes: the call writes h->out, for so many tokens
static patch_status fill_heads(HeadArgs* to, const patch_heads* h, int head_dim, int f32, bool writes, int64_t n_tokens = 0) {
    if (!h->x || h->heads < 1 || h->heads > 16384 || (h->f32 != 0) != (f32 != 0)) return PATCH_ERR_ARG;
    const int size = f32 ? 4 : 2;
    if (!aligned(h->x) || !aligned(h->gamma)) return PATCH_ERR_ARG;
    const int64_t width = (int64_t)h->heads * head_dim;
    if (h->stride < width || h->stride > ((int64_t)1 << 40) || h->stride * size % 16) return PATCH_ERR_SHAPE;
    if (writes) {
        if (!h->out || !aligned(h->out)) return PATCH_ERR_ARG;
        if (h->out_stride < width || h->out_stride > ((int64_t)1 << 40) || h->out_stride % 8) return PATCH_ERR_SHAPE;
        // in place a head goes where it came from, or its workgroup would write what another has yet to read
        if (h->out == h->x && (f32 || (n_tokens > 1 && h->out_stride != h->stride))) return PATCH_ERR_ARG;
    }
    to->x = static_cast<const uint8_t*>(h->x);
    to->stride = h->stride * size;
    to->gamma = h->gamma;
    to->out = writes ? static_cast<uint8_t*>(h->out) : nullptr;
    to->out_stride = h->out_stride * 2;
    to->heads = h->heads;
    return PATCH_OK;
}

static patch_status fill_rope(RopeArgs* to, const patch_rope* r, int head_dim) {
    to->eps = 1e-6f;
    if (!r) return PATCH_OK;
    if (!r->table || !aligned(r->table) || r->n_pos < 1 || !(r->eps >= 0.f)) return PATCH_ERR_ARG;
    if (r->rot_dim < 8 || r->rot_dim > head_dim || r->rot_dim % 8) return PATCH_ERR_SHAPE;
    to->table = r->table;
    to->n_pos = r->n_pos;
    to->rot = r->rot_dim;
    to->interleaved = r->interleaved != 0;
    to->eps = r->eps;
    return PATCH_OK;
}

static patch_status fill_cache(CacheArgs* to, const patch_kv_cache* c) {
    if (!c->k || !c->v || !aligned(c->k) || !aligned(c->v) || c->n_pages < 1 || c->n_pages > INT32_MAX || c->kv_heads < 1 || c->kv_heads > 65535) return PATCH_ERR_ARG;
    if (!head_dim_ok(c->head_dim)) return PATCH_ERR_SHAPE;
    if (!c->e4m3 && (c->k_scale || c->v_scale)) return PATCH_ERR_ARG;
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return PATCH_ERR_ARG;
    int log2 = 4;
    while (log2 < 8 && (1 << log2) != c->page_size) ++log2;
    if ((1 << log2) != c->page_size) return PATCH_ERR_SHAPE;
    const int64_t cells = (int64_t)c->kv_heads * c->page_size * c->head_dim;
    if (c->page_stride != 0 && (c->page_stride < cells || c->page_stride > ((int64_t)1 << 40) || c->page_stride % 16)) return PATCH_ERR_SHAPE;
    to->k = static_cast<uint8_t*>(c->k);
    to->v = static_cast<uint8_t*>(c->v);
    to->page_bytes = (c->page_stride ? c->page_stride : cells) * (c->e4m3 ? 1 : 2);
    if (to->page_bytes >= ((int64_t)1 << 32)) return PATCH_ERR_SHAPE;
    to->k_scale = c->k_scale;
    to->v_scale = c->v_scale;
    to->n_pages = (int)c->n_pages;
    to->page_log2 = log2;
    to->kv_heads = c->kv_heads;
    to->head_dim = c->head_dim;
    to->e4m3 = c->e4m3 != 0;
    return PATCH_OK;
}

static patch_status fill_seqs(SeqArgs* to, const patch_seqs* s, int page_size) {
    if (!s->kv_len || !s->page_table || !aligned(s->q_start, 4) || !aligned(s->kv_len, 4) || !aligned(s->page_table, 4)) return PATCH_ERR_ARG;
    if (s->n_seqs < 1 || s->n_seqs > 65535 || s->n_tokens < 0 || s->n_tokens > (1 << 23) || s->max_q < 0 || s->max_kv < 0 || s->table_stride < 1) return PATCH_ERR_ARG;
    if (!s->q_start && s->n_tokens != s->n_seqs) return PATCH_ERR_SHAPE;
    if (s->table_stride > ((int64_t)1 << 32)) return PATCH_ERR_SHAPE;
    to->q_start = s->q_start;
    to->kv_len = s->kv_len;
    to->table = s->page_table;
    to->table_stride = s->table_stride;
    to->n_seqs = (int)s->n_seqs;
    to->n_tokens = (int)s->n_tokens;
    to->max_q = (int)(s->max_q < s->n_tokens ? s->max_q : s->n_tokens);
    int64_t most = s->table_stride * page_size;                       // tokens that a row of the table has pages for
    if (most > (1 << 30)) most = 1 << 30;
    to->max_kv = (int)(s->max_kv < most ? s->max_kv : most);
    return PATCH_OK;
}

#define TRY(expr)                                \
    do {                                         \
        const patch_status st_ = (expr);         \
        if (st_ != PATCH_OK) return st_;         \
    } while (0)

extern "C" {

patch_status patch_qk_rope(const patch_heads* q, const patch_heads* k, const int32_t* positions, int64_t n_tokens, int head_dim, const patch_rope* rope,
                           void* stream) {
    if (!q || !positions || !aligned(positions, 4) || n_tokens < 0 || n_tokens > (1 << 23)) return PATCH_ERR_ARG;
    if (!head_dim_ok(head_dim)) return PATCH_ERR_SHAPE;
    RopeArgs a = {};
    TRY(fill_heads(&a.q, q, head_dim, q->f32, true, n_tokens));
    if (k) TRY(fill_heads(&a.k, k, head_dim, q->f32, true, n_tokens));
    TRY(fill_rope(&a, rope, head_dim));
    a.positions = positions;
    a.n_tokens = n_tokens;
    a.head_dim = head_dim;
    a.f32 = q->f32 != 0;
    if (n_tokens == 0) return PATCH_OK;
    launch_rope(a, static_cast<hipStream_t>(stream));
    return launched();
}

patch_status patch_kv_append(const patch_heads* k, const patch_heads* v, const patch_heads* q, const patch_seqs* seqs, const patch_rope* rope,
                             const patch_kv_cache* cache, void* stream) {
    if (!k || !v || !seqs || !cache || v->gamma) return PATCH_ERR_ARG;
    RopeArgs a = {};
    TRY(fill_cache(&a.cache, cache));
    if (k->heads != cache->kv_heads || v->heads != cache->kv_heads) return PATCH_ERR_SHAPE;
    TRY(fill_heads(&a.k, k, cache->head_dim, k->f32, false));
    TRY(fill_heads(&a.v, v, cache->head_dim, k->f32, false));
    if (q) TRY(fill_heads(&a.q, q, cache->head_dim, k->f32, true, seqs->n_tokens));
    TRY(fill_rope(&a, rope, cache->head_dim));
    TRY(fill_seqs(&a.seqs, seqs, cache->page_size));
    a.n_tokens = seqs->n_tokens;
    a.head_dim = cache->head_dim;
    a.f32 = k->f32 != 0;
    if (seqs->n_tokens == 0) return PATCH_OK;
    launch_rope(a, static_cast<hipStream_t>(stream));
    return launched();
}

static patch_status fill_attention(AttnArgs* a, int heads, const patch_seqs* seqs, const patch_kv_cache* cache, const patch_attention_opts* opts) {
    if (!seqs || !cache || heads < 1 || heads > 65535) return PATCH_ERR_ARG;
    TRY(fill_cache(&a->cache, cache));
    TRY(fill_seqs(&a->seqs, seqs, cache->page_size));
    if (heads % cache->kv_heads) return PATCH_ERR_SHAPE;
    a->heads = heads;
    a->group = heads / cache->kv_heads;
    if (seqs->n_tokens * heads > (1 << 25) || seqs->n_seqs * cache->kv_heads > (1 << 22)) return PATCH_ERR_SHAPE;
    if (opts) {
        if (opts->prefix_len < 0) return PATCH_ERR_ARG;
        a->prefix = (int)(opts->prefix_len < (1 << 30) ? opts->prefix_len : 1 << 30);
    }
    return PATCH_OK;
}

patch_status patch_attention(const void* Q, int64_t q_stride, int heads, const patch_seqs* seqs, const patch_kv_cache* cache, void* O, int64_t o_stride,
                             void* stream, const patch_attention_opts* opts) {
    if (!Q || !O || !aligned(Q) || !aligned(O)) return PATCH_ERR_ARG;
    AttnArgs a = {};
    TRY(fill_attention(&a, heads, seqs, cache, opts));
    const int64_t width = (int64_t)heads * cache->head_dim;
    if (q_stride < width || o_stride < width || q_stride > ((int64_t)1 << 40) || o_stride > ((int64_t)1 << 40) || q_stride % 8 || o_stride % 8) return PATCH_ERR_SHAPE;
    float scale = 1.f / sqrtf((float)cache->head_dim);
    size_t ws_bytes = 0;
    if (opts) {
        if (!(fabsf(opts->scale) <= 3e38f)) return PATCH_ERR_ARG;
        if (!aligned(opts->workspace) || !aligned(opts->lse, 4)) return PATCH_ERR_ARG;
        if (opts->scale != 0.f) scale = opts->scale;
        a.lse = opts->lse;
        if (opts->workspace) {
            a.part_ml = static_cast<float*>(opts->workspace);
            ws_bytes = opts->workspace_bytes;
        }
    }
    a.Q = static_cast<const uint16_t*>(Q);
    a.O = static_cast<uint16_t*>(O);
    a.q_stride = q_stride;
    a.o_stride = o_stride;
    a.scale = scale * 1.4426950408889634f;
    if (seqs->n_tokens == 0 || seqs->max_q == 0) return PATCH_OK;
    if (Q == O) return PATCH_ERR_ARG;
    plan_attention(&a, ws_bytes);
    launch_attention(a, static_cast<hipStream_t>(stream));
    return launched();
}

size_t patch_attention_workspace_bytes(int heads, const patch_seqs* seqs, const patch_kv_cache* cache, const patch_attention_opts* opts) {
    AttnArgs a = {};
    if (fill_attention(&a, heads, seqs, cache, opts) != PATCH_OK || seqs->n_tokens == 0 || seqs->max_q == 0) return 0;
    return plan_attention(&a, (size_t)1 << 62);
}

// For tests on the host: what the kernels make of a sequence's numbers (first, n, len, pos0, bad), and of a page number.
void patch_test_seq(int t0, int t1, int len, int n_tokens, int max_kv, int* out) {
    const Seq q = seq_from(t0, t1, len, n_tokens, max_kv);
    out[0] = q.first; out[1] = q.n; out[2] = q.len; out[3] = q.pos0; out[4] = q.bad;
}
int patch_test_page(int id, int n_pages) { return page_or_none(id, n_pages); }
// ... which of its sequence's tokens a row of the call is, -1: none
int patch_test_place(int t0, int t1, int n_tokens, int t) { return place_of(seq_from(t0, t1, 1, n_tokens, 1), t); }
// ... a tile of new positions: whether there are any in it, its bounds, and the row that each of its positions is read from
void patch_test_new_tile(int t0, int t1, int len, int n_tokens, int max_kv, int tile, int* out) {
    const Seq q = seq_from(t0, t1, len, n_tokens, max_kv);
    const NewTile n = new_tile(q, tile);
    out[0] = !n.none; out[1] = n.begin; out[2] = n.base;
    for (int i = 0; i < kTurn; ++i) out[3 + i] = row_of_new(q, n, i);
}
// ... and how a call would split its keys: (prefix, own_chunk, prefix_chunk, prefix_parts, parts, bytes of the workspace, few, front_blocks, line_waves,
// least_steps); -1: refused
int patch_test_attention_plan(int heads, const patch_seqs* seqs, const patch_kv_cache* cache, const patch_attention_opts* opts, size_t ws_bytes, int64_t* out) {
    AttnArgs a = {};
    if (fill_attention(&a, heads, seqs, cache, opts) != PATCH_OK) return -1;
    out[5] = (int64_t)plan_attention(&a, ws_bytes);
    out[6] = a.few; out[7] = a.front_blocks; out[8] = a.line_waves; out[9] = a.least_steps;
    out[0] = a.prefix; out[1] = a.own_chunk; out[2] = a.prefix_chunk; out[3] = a.prefix_parts; out[4] = a.parts;
    return 0;
}

}  // extern "C"
