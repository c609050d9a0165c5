// Operators on a paged cache that several sequences live in: argument checks and launches (paged.hip), the fork of a
// session, the bookkeeping of shared pages, rotary tables for long contexts.
#include <cmath>
#include <new>

#include "host.h"

using namespace sb;
using namespace sbhost;

struct sb_pages {
    std::vector<int32_t> users;
    int32_t used;
};

namespace {

constexpr int64_t MAX_ITEMS = 0x7fffffff;

// Checks of the shared part; *empty: nothing to do (then only the counts are looked at).
int paged_check(const char* op, const sb_paged* kv, int32_t layer, int32_t x_dtype, int32_t n_heads, bool* empty) {
    if (!kv) return fail(SB_EINVAL, "%s: kv is NULL", op);
    if (kv->head_dim != 64 && kv->head_dim != 128) return fail(SB_EINVAL, "%s: head_dim must be 64 or 128", op);
    if (kv->n_kv_heads < 1 || n_heads < 1 || n_heads % kv->n_kv_heads) return fail(SB_EINVAL, "%s: head counts", op);
    if (n_heads > 65535 / 4) return fail(SB_EINVAL, "%s: more than %d heads", op, 65535 / 4);
    if (x_dtype != SB_FP32 && x_dtype != SB_BF16) return fail(SB_EINVAL, "%s: x_dtype", op);
    if (kv->n_seq < 0 || kv->n_rows < 0 || layer < 0) return fail(SB_EINVAL, "%s: negative count", op);
    if (kv->n_pages < 1 || kv->table_ld < 1) return fail(SB_EINVAL, "%s: n_pages and table_ld must be positive", op);
    if (kv->max_len < 1 || kv->max_len > (int64_t)kv->table_ld * SB_KV_BLOCK || kv->max_len > (1 << 24))
        return fail(SB_EINVAL, "%s: max_len must be in 1..16 table_ld, 2^24 at most", op);
    // (keys, rows times heads and work items are counted in 32 bits)
    if ((int64_t)kv->n_rows * n_heads + (int64_t)kv->n_seq * n_heads > MAX_ITEMS / 4)
        return fail(SB_EINVAL, "%s: %d rows and %d sequences of %d heads are too many for one call", op, kv->n_rows, kv->n_seq, n_heads);
    *empty = kv->n_seq == 0 || kv->n_rows == 0;
    if (*empty) return SB_OK;
    if (!kv->pool || !kv->table || !kv->row_start || !kv->kv_len) return fail(SB_EINVAL, "%s: NULL pool, table, row_start or kv_len", op);
    if ((uintptr_t)kv->pool & 15) return fail(SB_EINVAL, "%s: pool must be 16-byte aligned", op);
    if (((uintptr_t)kv->table | (uintptr_t)kv->row_start | (uintptr_t)kv->kv_len) & 3) return fail(SB_EINVAL, "%s: misaligned index array", op);
    return SB_OK;
}

size_t slab_elems(const sb_paged* kv) { return (size_t)kv->n_pages * kv->n_kv_heads * SB_KV_BLOCK * kv->head_dim; }

PagedKv device_kv(const sb_paged* kv, int32_t layer) {
    uint16_t* k = (uint16_t*)kv->pool + (size_t)layer * 2 * slab_elems(kv);
    return PagedKv{k, k + slab_elems(kv), kv->table, kv->row_start, kv->kv_len, kv->n_pages, kv->n_kv_heads, kv->head_dim, kv->n_seq,
                   kv->n_rows, kv->table_ld, kv->max_len};
}

// One operand of n_rows rows: aligned, wide enough, outside the layer's slabs.
int rows_check(const char* op, const char* name, const sb_paged* kv, int32_t layer, const void* x, int32_t x_dtype, int64_t ld, int64_t width) {
    const int64_t es = (int64_t)esize(x_dtype);
    if (!x) return fail(SB_EINVAL, "%s: %s is NULL", op, name);
    if (((uintptr_t)x & 15) || ld * es % 16) return fail(SB_EINVAL, "%s: %s: rows must be 16-byte aligned", op, name);
    if (ld < width || ld > ((int64_t)1 << 40)) return fail(SB_EINVAL, "%s: %s: rows are %lld apart and %lld wide", op, name, (long long)ld, (long long)width);
    const PagedKv d = device_kv(kv, layer);
    if (overlaps(x, (size_t)(((kv->n_rows - 1) * ld + width) * es), d.k, slab_elems(kv) * 4)) return fail(SB_EINVAL, "%s: %s lies in the pool", op, name);
    return SB_OK;
}

// `out` may be `in` itself, row by row, or apart from it.
int place_check(const char* op, const sb_paged* kv, int32_t x_dtype, const void* in, int64_t ld_in, int64_t w_in, const void* out, int64_t ld_out, int64_t w_out) {
    const size_t es = esize(x_dtype), n = (size_t)kv->n_rows - 1;
    if (in == out && ld_in == ld_out) return SB_OK;
    if (overlaps(in, (n * ld_in + w_in) * es, out, (n * ld_out + w_out) * es)) return fail(SB_EINVAL, "%s: the output overlaps the input without being it", op);
    return SB_OK;
}

}  // namespace

extern "C" {

int32_t sb_op_rope_append(const sb_paged* kv, int32_t layer, const void* qkv, int32_t x_dtype, int64_t ld_qkv, int32_t n_heads,
                          const float* q_gain, const float* k_gain, float eps, const float* rope_cos, const float* rope_sin,
                          int32_t n_pos, int32_t rot_dim, int32_t rope_layout, void* q_out, int64_t ld_q, void* stream) {
    static const char* op = "op_rope_append";
    bool empty;
    int rc = paged_check(op, kv, layer, x_dtype, n_heads, &empty);
    if (rc) return rc;
    if (rot_dim < 0 || rot_dim > kv->head_dim || rot_dim % 8) return fail(SB_EINVAL, "%s: rot_dim must be a multiple of 8 in 0..head_dim", op);
    if (rope_layout != SB_ROPE_HALF && rope_layout != SB_ROPE_INTERLEAVED) return fail(SB_EINVAL, "%s: rope_layout", op);
    if (rot_dim && n_pos < 1) return fail(SB_EINVAL, "%s: n_pos must be positive", op);
    if ((q_gain || k_gain) && !(eps >= 0.f)) return fail(SB_EINVAL, "%s: eps must be >= 0", op);
    if (empty) return SB_OK;
    if (rot_dim && (!rope_cos || !rope_sin)) return fail(SB_EINVAL, "%s: rope tables are NULL", op);
    if (((uintptr_t)rope_cos | (uintptr_t)rope_sin | (uintptr_t)q_gain | (uintptr_t)k_gain) & 15)
        return fail(SB_EINVAL, "%s: rope tables and gains must be 16-byte aligned", op);
    const int64_t w_in = (int64_t)(n_heads + 2 * kv->n_kv_heads) * kv->head_dim, w_q = (int64_t)n_heads * kv->head_dim;
    if ((rc = rows_check(op, "qkv", kv, layer, qkv, x_dtype, ld_qkv, w_in))) return rc;
    if ((rc = rows_check(op, "q_out", kv, layer, q_out, x_dtype, ld_q, w_q))) return rc;
    if ((rc = place_check(op, kv, x_dtype, qkv, ld_qkv, w_in, q_out, ld_q, w_q))) return rc;
    RopeAppendArgs a{};
    a.kv = device_kv(kv, layer);
    a.qkv = qkv; a.q_out = q_out; a.ld_qkv = ld_qkv; a.ld_q = ld_q; a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps;
    a.cos = rope_cos; a.sin = rope_sin; a.x_dtype = x_dtype; a.n_heads = n_heads; a.n_pos = n_pos; a.rot_dim = rot_dim;
    a.interleaved = rope_layout == SB_ROPE_INTERLEAVED;
    HIP_TRY(launch_rope_append(a, (hipStream_t)stream));
    return SB_OK;
}

size_t sb_op_paged_attention_scratch_bytes(const sb_paged* kv, int32_t n_heads) {
    bool empty;
    if (paged_check("op_paged_attention", kv, 0, SB_FP32, n_heads, &empty) || empty) return 0;
    return align_up(paged_attention_scratch(device_kv(kv, 0), n_heads), 256);
}

int32_t sb_op_paged_attention(const sb_paged* kv, int32_t layer, const void* q, int32_t x_dtype, int64_t ld_q, int32_t n_heads,
                              const sb_attn_rule* rule, void* out, int64_t ld_out, void* scratch, size_t scratch_bytes, void* stream) {
    static const char* op = "op_paged_attention";
    bool empty;
    int rc = paged_check(op, kv, layer, x_dtype, n_heads, &empty);
    if (rc) return rc;
    const sb_attn_rule r = rule ? *rule : sb_attn_rule{};
    if (!(r.scale >= 0.f) || r.scale > 1e38f) return fail(SB_EINVAL, "%s: scale must be positive, or 0 for 1 / sqrt(head_dim)", op);
    const float scale = r.scale > 0.f ? r.scale : 1.0f / sqrtf((float)kv->head_dim);
    if (!(r.softcap >= 0.f) || r.softcap > 1e30f) return fail(SB_EINVAL, "%s: softcap must be positive and 1e30 at most, or 0 for none", op);
    if (r.softcap > 0.f && !(scale / r.softcap >= 1e-34f && scale / r.softcap <= 1e6f)) return fail(SB_EINVAL, "%s: scale / softcap must be in 1e-34..1e6", op);
    if (r.window < 0) return fail(SB_EINVAL, "%s: window must be positive, or 0 for none", op);
    if (empty) return SB_OK;
    if (((uintptr_t)r.slopes | (uintptr_t)r.prefix_len | (uintptr_t)r.doc_start) & 3) return fail(SB_EINVAL, "%s: misaligned slopes, prefix_len or doc_start", op);
    const int64_t w = (int64_t)n_heads * kv->head_dim;
    if ((rc = rows_check(op, "q", kv, layer, q, x_dtype, ld_q, w))) return rc;
    if ((rc = rows_check(op, "out", kv, layer, out, x_dtype, ld_out, w))) return rc;
    if ((rc = place_check(op, kv, x_dtype, q, ld_q, w, out, ld_out, w))) return rc;
    const size_t need = sb_op_paged_attention_scratch_bytes(kv, n_heads);
    if (need) {
        if (!scratch || ((uintptr_t)scratch & 255)) return fail(SB_EINVAL, "%s: scratch is NULL or not 256-byte aligned", op);
        if (scratch_bytes < need) return fail(SB_ENOMEM, "%s: scratch too small (%zu < %zu)", op, scratch_bytes, need);
        const size_t n = (size_t)kv->n_rows - 1, es = esize(x_dtype);
        if (overlaps(scratch, need, q, (n * ld_q + w) * es) || overlaps(scratch, need, out, (n * ld_out + w) * es) ||
            overlaps(scratch, need, device_kv(kv, layer).k, slab_elems(kv) * 4))
            return fail(SB_EINVAL, "%s: scratch overlaps q, out or the pool", op);
    }
    PagedAttnArgs a{};
    a.kv = device_kv(kv, layer);
    a.q = q; a.out = out; a.ld_q = ld_q; a.ld_out = ld_out; a.x_dtype = x_dtype; a.n_heads = n_heads; a.group = n_heads / kv->n_kv_heads;
    a.scale = scale; a.cap = r.softcap; a.slopes = r.slopes; a.window = r.window; a.prefix_len = r.prefix_len; a.doc_start = r.doc_start;
    a.scratch = (float*)scratch;
    HIP_TRY(launch_paged_attention(a, (hipStream_t)stream));
    return SB_OK;
}

int32_t sb_op_copy_pages(void* dst, int32_t dst_n_pages, const void* src, int32_t src_n_pages, size_t page_bytes, int32_t n_slabs,
                         const int32_t* dst_pages, const int32_t* src_pages, int32_t n, void* stream) {
    static const char* op = "op_copy_pages";
    if (dst_n_pages < 1 || src_n_pages < 1 || n_slabs < 1 || n_slabs > 65535 || n < 0) return fail(SB_EINVAL, "%s: bad count", op);
    if (page_bytes < 16 || page_bytes % 16 || page_bytes > ((size_t)1 << 27)) return fail(SB_EINVAL, "%s: page_bytes must be a multiple of 16, 2^27 at most", op);
    if (n == 0) return SB_OK;
    if (!dst || !src || !dst_pages || !src_pages) return fail(SB_EINVAL, "%s: NULL argument", op);
    if (((uintptr_t)dst | (uintptr_t)src) & 15) return fail(SB_EINVAL, "%s: pools must be 16-byte aligned", op);
    const bool same = dst == src;
    if (same ? dst_n_pages != src_n_pages : overlaps(dst, dst_n_pages * page_bytes * n_slabs, src, src_n_pages * page_bytes * n_slabs))
        return fail(SB_EINVAL, "%s: the pools overlap without being the same", op);
    if (n > dst_n_pages) return fail(SB_EINVAL, "%s: more pages written than there are", op);
    std::vector<char> mark;
    try {
        mark.assign(dst_n_pages, 0);
    } catch (const std::bad_alloc&) {
        return fail(SB_ENOMEM, "%s: no host memory", op);
    }
    for (int i = 0; i < n; ++i) {
        if (dst_pages[i] < 0 || dst_pages[i] >= dst_n_pages || src_pages[i] < 0 || src_pages[i] >= src_n_pages)
            return fail(SB_EINVAL, "%s: pair %d: page %d -> %d outside the pools", op, i, src_pages[i], dst_pages[i]);
        if (mark[dst_pages[i]]) return fail(SB_EINVAL, "%s: page %d is written twice", op, dst_pages[i]);
        mark[dst_pages[i]] = 1;
    }
    if (same)
        for (int i = 0; i < n; ++i)
            if (mark[src_pages[i]]) return fail(SB_EINVAL, "%s: page %d is both read and written", op, src_pages[i]);
    CopyPagesArgs a{};
    a.src = (const char*)src; a.dst = (char*)dst; a.page_bytes = page_bytes;
    a.src_slab = src_n_pages * page_bytes; a.dst_slab = dst_n_pages * page_bytes;
    for (int i = 0; i < n; i += SB_COPY_PAGES) {
        const int m = n - i < SB_COPY_PAGES ? n - i : SB_COPY_PAGES;
        memcpy(a.from, src_pages + i, (size_t)m * 4);
        memcpy(a.to, dst_pages + i, (size_t)m * 4);
        HIP_TRY(launch_copy_pages(a, m, n_slabs, (hipStream_t)stream));
    }
    return SB_OK;
}

// ---------------------------------------------------------------- bookkeeping of pages
int32_t sb_new_pages(int32_t n_pages, sb_pages** out) {
    if (!out || n_pages < 1) return fail(SB_EINVAL, "new_pages: bad argument");
    try {
        *out = new sb_pages{std::vector<int32_t>(n_pages, 0), 0};
    } catch (const std::bad_alloc&) {
        return fail(SB_ENOMEM, "new_pages: no host memory");
    }
    return SB_OK;
}
void sb_free_pages(sb_pages* p) { delete p; }

int32_t sb_pages_alloc(sb_pages* p, int32_t n, int32_t* out) {
    if (!p || n < 0 || (n && !out)) return fail(SB_EINVAL, "pages_alloc: bad argument");
    const int32_t total = (int32_t)p->users.size();
    if (n > total - p->used) return fail(SB_ECAPACITY, "pages_alloc: %d pages asked for, %d free", n, total - p->used);
    for (int32_t i = 0, k = 0; k < n; ++i)
        if (!p->users[i]) { p->users[i] = 1; out[k++] = i; }
    p->used += n;
    return SB_OK;
}

static int pages_check(const char* op, const sb_pages* p, const int32_t* pages, int32_t n) {
    if (!p || n < 0 || (n && !pages)) return fail(SB_EINVAL, "%s: bad argument", op);
    for (int32_t i = 0; i < n; ++i) {
        if (pages[i] < 0 || pages[i] >= (int32_t)p->users.size()) return fail(SB_EINVAL, "%s: page %d out of range", op, pages[i]);
        if (!p->users[pages[i]]) return fail(SB_EINVAL, "%s: page %d is free", op, pages[i]);
    }
    return SB_OK;
}

int32_t sb_pages_share(sb_pages* p, const int32_t* pages, int32_t n) {
    int rc = pages_check("pages_share", p, pages, n);
    if (rc) return rc;
    for (int32_t i = 0; i < n; ++i)
        if (p->users[pages[i]] > 0x7fffffff - n) return fail(SB_ECAPACITY, "pages_share: page %d has too many users", pages[i]);
    for (int32_t i = 0; i < n; ++i) ++p->users[pages[i]];
    return SB_OK;
}

int32_t sb_pages_release(sb_pages* p, const int32_t* pages, int32_t n) {
    int rc = pages_check("pages_release", p, pages, n);
    if (rc) return rc;
    for (int32_t i = 0; i < n; ++i)
        if (--p->users[pages[i]] < 0) {   // named more often than it has users: taken back
            const int32_t bad = pages[i];
            for (int32_t k = 0; k <= i; ++k) ++p->users[pages[k]];
            return fail(SB_EINVAL, "pages_release: page %d has %d users", bad, p->users[bad]);
        }
    int32_t used = 0;
    for (int32_t u : p->users) used += u > 0;
    p->used = used;
    return SB_OK;
}

int32_t sb_pages_users(const sb_pages* p, int32_t page) {
    if (!p || page < 0 || page >= (int32_t)p->users.size()) return fail(SB_EINVAL, "pages_users: bad argument");
    return p->users[page];
}
int32_t sb_pages_used(const sb_pages* p) { return p ? p->used : 0; }

int32_t sb_pages_compact(sb_pages* p, int32_t* src, int32_t* dst, int32_t cap, int32_t* n_moves) {
    if (!p || !n_moves || cap < 0 || (cap && (!src || !dst))) return fail(SB_EINVAL, "pages_compact: bad argument");
    const int32_t total = (int32_t)p->users.size();
    int32_t need = 0;
    for (int32_t i = p->used; i < total; ++i) need += p->users[i] > 0;
    *n_moves = need;
    if (need > cap) return fail(SB_ECAPACITY, "pages_compact: %d moves, room for %d", need, cap);
    int32_t hole = 0, k = 0;
    for (int32_t i = p->used; i < total; ++i) {
        if (!p->users[i]) continue;
        while (p->users[hole]) ++hole;
        src[k] = i; dst[k++] = hole;
        p->users[hole] = p->users[i];
        p->users[i] = 0;
    }
    return SB_OK;
}

int32_t sb_rope_table_scaled_host(int32_t rot_dim, float base, int32_t n_pos, int32_t kind, float factor, int32_t orig_len, float slow,
                                  float fast, float magnitude, float* cos_out, float* sin_out) {
    static const char* op = "rope_table_scaled_host";
    if (rot_dim < 2 || (rot_dim & 1) || !(base > 0.f) || n_pos < 0 || !cos_out || !sin_out) return fail(SB_EINVAL, "%s: bad argument", op);
    if (kind < SB_ROPE_PLAIN || kind > SB_ROPE_PARTS) return fail(SB_EINVAL, "%s: kind", op);
    if (!(magnitude > 0.f)) return fail(SB_EINVAL, "%s: magnitude must be positive", op);
    if (kind != SB_ROPE_PLAIN && !(factor >= 1.f)) return fail(SB_EINVAL, "%s: factor must be 1 or more", op);
    if (kind == SB_ROPE_BASE && rot_dim == 2) return fail(SB_EINVAL, "%s: a single pair has no other frequency to keep", op);
    if (kind == SB_ROPE_PARTS && (orig_len < 1 || !(slow >= 0.f) || !(fast > slow))) return fail(SB_EINVAL, "%s: need orig_len >= 1 and 0 <= slow < fast", op);
    const int half = rot_dim / 2;
    double b = base;
    if (kind == SB_ROPE_BASE) b *= std::pow((double)factor, (double)rot_dim / (double)(rot_dim - 2));
    for (int i = 0; i < half; ++i) {
        double f = std::pow(b, -2.0 * (double)i / (double)rot_dim);
        if (kind == SB_ROPE_LINEAR) f /= (double)factor;
        if (kind == SB_ROPE_PARTS) {
            const double turns = (double)orig_len * f / (2.0 * M_PI);
            double t = (turns - (double)slow) / ((double)fast - (double)slow);
            t = t < 0.0 ? 0.0 : t > 1.0 ? 1.0 : t;
            f = (1.0 - t) * f / (double)factor + t * f;
        }
        for (int p = 0; p < n_pos; ++p) {
            const double x = (double)p * f;
            cos_out[(size_t)p * half + i] = (float)(std::cos(x) * (double)magnitude);
            sin_out[(size_t)p * half + i] = (float)(std::sin(x) * (double)magnitude);
        }
    }
    return SB_OK;
}

}  // extern "C"
