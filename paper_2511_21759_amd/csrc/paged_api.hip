// C entry points of the paged K/V operators (include/odb.h): argument checks, then one launch (two with split keys).
#include <math.h>
#include <stdint.h>

#include "errors.h"
#include "paged.h"

using namespace odb;

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

struct Range { const void *p; size_t bytes; };
bool overlap(const Range &a, const Range &b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

// log2 of a page size, or -1
int page_shift(int page_size) {
    if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1))) return -1;
    int s = 4;
    while ((1 << s) < page_size) s++;
    return s;
}

int check_pool(const char *who, int n_pages, int page_size) {
    if (page_shift(page_size) < 0) return fail(ODB_E_INVALID_ARG, "%s: page_size=%d is no power of two from 16 to 4096", who, page_size);
    if (n_pages < 1 || (long long)n_pages * page_size > 0x7fffffffll) return fail(ODB_E_INVALID_ARG, "%s: %d pages of %d positions", who, n_pages, page_size);
    return ODB_OK;
}

int check_columns(const char *who, int columns, int page_size) {
    if (columns < 1 || (long long)columns * page_size > (1ll << 30)) return fail(ODB_E_INVALID_ARG, "%s: tables of %d columns of %d positions", who, columns, page_size);
    return ODB_OK;
}

// align: of strides, in elements
int check_pages(const char *who, const odb_pages *p, bool buffers = true, int align = 8) {
    if (!p) return fail(ODB_E_INVALID_ARG, "%s: pages is NULL", who);
    int rc = check_pool(who, p->n_pages, p->page_size);
    if (rc) return rc;
    if (p->dtype != ODB_F16 && p->dtype != ODB_BF16) return fail(ODB_E_INVALID_ARG, "%s: pages of dtype %d", who, p->dtype);
    if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return fail(ODB_E_INVALID_ARG, "%s: head_dim=%d (64, 128 or 256)", who, p->head_dim);
    if (p->n_kv_heads < 1 || p->n_kv_heads > 65536) return fail(ODB_E_INVALID_ARG, "%s: n_kv_heads=%d", who, p->n_kv_heads);
    if (p->page_stride < 0 || p->head_stride < 0 || p->pos_stride < 0 || (p->page_stride | p->head_stride | p->pos_stride) & (align - 1) || p->pos_stride >= 1 << 24)
        return fail(ODB_E_INVALID_ARG, "%s: page strides %lld, %lld, %lld", who, p->page_stride, p->head_stride, p->pos_stride);
    if (buffers && (!p->k || !p->v || !aligned16(p->k) || !aligned16(p->v))) return fail(ODB_E_INVALID_ARG, "%s: pools are NULL or not aligned to 16 bytes", who);
    return ODB_OK;
}

int check_rows(const char *who, const char *name, const void *p, long long stride, int heads, int dim) {
    if (!p || !aligned16(p)) return fail(ODB_E_INVALID_ARG, "%s: %s is NULL or not aligned to 16 bytes", who, name);
    if (stride < (long long)heads * dim || stride & 7) return fail(ODB_E_INVALID_ARG, "%s: rows of %s are %lld elements apart", who, name, stride);
    return ODB_OK;
}

// Pages of 8-bit codes as the structures of the launchers have them
int check_quant_pages(const char *who, const odb_quant_pages *p, bool buffers, odb_pages &codes, QuantScales &s) {
    if (!p) return fail(ODB_E_INVALID_ARG, "%s: pages is NULL", who);
    codes = odb_pages{p->k, p->v, p->n_pages, p->page_size, p->n_kv_heads, p->head_dim, p->dtype, p->page_stride, p->head_stride, p->pos_stride};
    int rc = check_pages(who, &codes, buffers, 16);
    if (rc) return rc;
    if (p->codes != ODB_INT8 && p->codes != ODB_E4M3) return fail(ODB_E_INVALID_ARG, "%s: codes=%d", who, p->codes);
    if ((p->group != 1 && p->group != 16 && p->group != 32 && p->group != 64) || p->group > p->page_size)
        return fail(ODB_E_INVALID_ARG, "%s: groups of %d positions in pages of %d (1, 16, 32 or 64)", who, p->group, p->page_size);
    if (p->scale_page_stride < 0 || p->scale_head_stride < 0 || (p->group == 1 && (p->scale_page_stride | p->scale_head_stride) & 3))
        return fail(ODB_E_INVALID_ARG, "%s: scale strides %lld, %lld", who, p->scale_page_stride, p->scale_head_stride);
    if (buffers && (!p->k_scale || !p->v_scale || !aligned16(p->k_scale) || !aligned16(p->v_scale)))
        return fail(ODB_E_INVALID_ARG, "%s: scales are NULL or not aligned to 16 bytes", who);
    s = QuantScales{p->k_scale, p->v_scale, p->scale_page_stride, p->scale_head_stride, p->codes, p->group == 1 ? 0 : p->group == 16 ? 4 : p->group == 32 ? 5 : 6};
    return ODB_OK;
}

size_t span(int rows, long long stride, int heads, int dim, int bytes) {
    return rows < 1 ? 0 : ((size_t)(rows - 1) * (size_t)stride + (size_t)heads * dim) * bytes;
}

}  // namespace

// checks what does not need buffers, and fills the launch's fields that follow from it
// (the pages have been looked at)
template <class Plan>
static int plan_attention(const char *who, const odb_attention *a, const odb_pages *pages, Plan plan, PagedAttn &p, int &nt) {
    if (a->n < 1 || a->n > kMaxRequests) return fail(ODB_E_INVALID_ARG, "%s: n=%d outside [1, %d]", who, a->n, kMaxRequests);
    if (a->rows < 0 || a->rows > 1 << 24) return fail(ODB_E_INVALID_ARG, "%s: rows=%d outside [0, 2^24]", who, a->rows);
    if (a->n_heads < 1 || a->n_heads % pages->n_kv_heads) return fail(ODB_E_INVALID_ARG, "%s: %d query heads over %d K/V heads", who, a->n_heads, pages->n_kv_heads);
    int rc = check_columns(who, a->columns, pages->page_size);
    if (rc) return rc;
    if (!(a->scale > 0.f) || !isfinite(a->scale * 1.44269504088896340736f)) return fail(ODB_E_INVALID_ARG, "%s: scale=%g", who, (double)a->scale);
    if (a->window < 0 || a->window > 1 << 30 || a->sinks < 0 || a->sinks > 1 << 30) return fail(ODB_E_INVALID_ARG, "%s: window=%d, sinks=%d", who, a->window, a->sinks);
    if (a->max_rows < 0 || a->max_len < 0) return fail(ODB_E_INVALID_ARG, "%s: max_rows=%d, max_len=%d", who, a->max_rows, a->max_len);
    const long long most = (long long)a->columns * pages->page_size;
    p.columns = a->columns; p.n = a->n; p.rows = a->rows; p.heads = a->n_heads; p.group = a->n_heads / pages->n_kv_heads;
    p.pages = *pages;
    p.page_shift = page_shift(pages->page_size);
    p.rows_per_request = 1;
    const int max_rows = a->max_rows > 0 && a->max_rows < a->rows ? a->max_rows : a->rows;
    long long max_len = a->max_len > 0 && a->max_len < most ? a->max_len : most;
    if (a->window) {                                                   // what the rows of a request see together
        const long long seen = (a->causal ? 1ll : 2ll) * a->window + a->sinks + max_rows;
        max_len = seen < max_len ? seen : max_len;
    }
    plan(*pages, a->n, a->rows, p.group, max_rows, max_len, a->columns, &nt, &p.split, &p.items);
    if (a->rows == 0) p.split = 0;                                     // nothing is launched, no workspace
    // (a launch has fewer than 2^32 threads, 256 a workgroup; rows of a tile are counted in 32 bits, with room for a tile behind the last)
    if (p.items * pages->n_kv_heads >= 1 << 24 || (long long)a->rows * a->n_heads > 1 << 30)
        return fail(ODB_E_INVALID_ARG, "%s: %d rows of %d heads are too many for one launch", who, a->rows, a->n_heads);
    return ODB_OK;
}

int odb::plan_paged_attention(const odb_attention *a, const odb_pages *pages, bool buffers, PagedAttn &p, int &nt) {
    const char *who = "paged_attention";
    if (!a) return fail(ODB_E_INVALID_ARG, "%s: NULL argument", who);
    const int rc = check_pages(who, pages, buffers);
    if (rc) return rc;
    p = PagedAttn{};
    return plan_attention(who, a, pages, paged_attn_plan, p, nt);
}

int odb::plan_paged_attention_quant(const odb_attention *a, const odb_quant_pages *pages, bool buffers, PagedAttnQuant &p, int &nt) {
    const char *who = "paged_attention_quant";
    if (!a) return fail(ODB_E_INVALID_ARG, "%s: NULL argument", who);
    p = PagedAttnQuant{};
    odb_pages codes;
    const int rc = check_quant_pages(who, pages, buffers, codes, p.scales);
    if (rc) return rc;
    return plan_attention(who, a, &codes, [&](const odb_pages &q, int n, int rows, int group, int max_rows, long long max_len, long long columns, int *t, int *split,
                                              long long *items) { paged_attn_quant_plan(q, n, rows, group, max_rows, max_len, columns, t, split, items, &p.slots); }, p, nt);
}

// what an attention call needs beside its plan: buffers, a workspace; and the launch's fields that come from them
static int bind_attention(const char *who, const odb_attention *a, PagedAttn &p, int nt) {
    if (!a->cu_rows && a->rows != a->n) return fail(ODB_E_INVALID_ARG, "%s: without cu_rows every request has one row (%d rows, %d requests)", who, a->rows, a->n);
    const int dim = p.pages.head_dim;
    int rc;
    if ((rc = check_rows(who, "q", a->q, a->q_row, a->n_heads, dim)) || (rc = check_rows(who, "out", a->out, a->out_row, a->n_heads, dim))) return rc;
    if (!a->kv_len || !a->tables) return fail(ODB_E_INVALID_ARG, "%s: NULL kv_len or tables", who);
    if (overlap(Range{a->out, span(a->rows, a->out_row, a->n_heads, dim, 2)}, Range{a->q, span(a->rows, a->q_row, a->n_heads, dim, 2)}))
        return fail(ODB_E_INVALID_ARG, "%s: out overlaps q", who);
    const size_t need = paged_attn_workspace(p.pages, p.rows, p.heads, nt, p.split);
    if (need && (!a->workspace || (uintptr_t)a->workspace & 255 || a->workspace_bytes < need))
        return fail(ODB_E_INVALID_ARG, "%s: a workspace of %zu bytes aligned to 256, given %zu", who, need, a->workspace ? a->workspace_bytes : 0);
    p.q = a->q; p.out = a->out; p.q_row = a->q_row; p.out_row = a->out_row;
    p.cu_rows = a->cu_rows; p.first = a->first_pos; p.kv_len = a->kv_len; p.tables = a->tables;
    p.sc = a->scale * 1.44269504088896340736f;
    p.causal = a->causal != 0; p.window = a->window; p.sinks = a->sinks;
    return ODB_OK;
}

// sizes, gains and rows of a call that norms and turns, and that its queries go where nothing else is read (R: odb_qk_rows or odb_quant_rows)
template <class R, class TooMany>
static int check_turned_rows(const char *who, const R &r, const odb_pages &pages, TooMany too_many) {
    const int dim = pages.head_dim, kv = pages.n_kv_heads;
    if (r.rows < 0 || r.rows > 1 << 24) return fail(ODB_E_INVALID_ARG, "%s: rows=%d outside [0, 2^24]", who, r.rows);
    if (r.n_heads < 1 || r.n_heads > 65536) return fail(ODB_E_INVALID_ARG, "%s: n_heads=%d", who, r.n_heads);
    if (too_many()) return fail(ODB_E_INVALID_ARG, "%s: %d rows of %d heads are too many for one launch", who, r.rows, r.n_heads);
    if (r.in_dtype != ODB_F32 && r.in_dtype != pages.dtype) return fail(ODB_E_INVALID_ARG, "%s: rows of dtype %d into pages of dtype %d", who, r.in_dtype, pages.dtype);
    int rc;
    if (!(rc = check_rows(who, "q", r.q, r.q_row, r.n_heads, dim)) && !(rc = check_rows(who, "k", r.k, r.k_row, kv, dim)) &&
        !(rc = check_rows(who, "v", r.v, r.v_row, kv, dim)))
        rc = check_rows(who, "q_out", r.q_out, r.q_out_row, r.n_heads, dim);
    if (rc) return rc;
    if (!r.table || !aligned16(r.table) || !r.positions) return fail(ODB_E_INVALID_ARG, "%s: NULL table or positions", who);
    if ((r.q_gain == nullptr) != (r.k_gain == nullptr) || !aligned16(r.q_gain) || !aligned16(r.k_gain))
        return fail(ODB_E_INVALID_ARG, "%s: gains are given for q and k together, aligned to 16 bytes", who);
    if (r.q_gain && (!(r.eps >= 0.f) || !isfinite(r.eps))) return fail(ODB_E_INVALID_ARG, "%s: eps=%g", who, (double)r.eps);
    if (r.n_pos < 1 || r.n_pos > 1 << 22) return fail(ODB_E_INVALID_ARG, "%s: n_pos=%d outside [1, 2^22]", who, r.n_pos);
    if (r.rot_dim < 16 || r.rot_dim > dim || r.rot_dim % 16) return fail(ODB_E_INVALID_ARG, "%s: rot_dim=%d is no multiple of 16 in [16, %d]", who, r.rot_dim, dim);
    const bool in_place = r.q_out == r.q && r.in_dtype == pages.dtype && r.q_out_row == r.q_row;
    const int eb = r.in_dtype == ODB_F32 ? 4 : 2;
    const Range out{r.q_out, span(r.rows, r.q_out_row, r.n_heads, dim, 2)};
    if (!in_place && (overlap(out, Range{r.q, span(r.rows, r.q_row, r.n_heads, dim, eb)}) || overlap(out, Range{r.k, span(r.rows, r.k_row, kv, dim, eb)}) ||
                      overlap(out, Range{r.v, span(r.rows, r.v_row, kv, dim, eb)})))
        return fail(ODB_E_INVALID_ARG, "%s: q_out overlaps q, k or v without being q itself", who);
    // (in place, the rows of k and v may lie between those of q, as in a fused buffer, but a lane must not read what another has written)
    auto beside = [&](const void *x, long long row) {
        if (!overlap(out, Range{x, span(r.rows, row, kv, dim, eb)})) return true;
        if (r.rows > 1 && row != r.q_row) return false;
        const long long bytes = r.rows > 1 ? row * eb : 1ll << 62, gap = (((intptr_t)x - (intptr_t)r.q) % bytes + bytes) % bytes;
        return gap >= (long long)r.n_heads * dim * eb && gap + (long long)kv * dim * eb <= bytes;
    };
    if (in_place && !(beside(r.k, r.k_row) && beside(r.v, r.v_row)))
        return fail(ODB_E_INVALID_ARG, "%s: in place, k and v must not share elements with q (rows of one stride, or buffers apart)", who);
    return ODB_OK;
}

extern "C" {

int odb_page_tables(const int32_t *held, const int32_t *wanted, int n, int page_size, int32_t *tables, int columns, int32_t *free_pages,
                    int n_pages, const int32_t *n_free, const int32_t *row_first, const int32_t *row_count, int32_t *len, int32_t *cu_rows,
                    int32_t *slots, int32_t *positions, int rows_cap, int32_t *state, void *stream) {
    const char *who = "page_tables";
    if (!held || !wanted || !tables || !free_pages || !n_free || !len || !cu_rows || !slots || !positions || !state)
        return fail(ODB_E_INVALID_ARG, "%s: NULL buffer", who);
    if (n < 1 || n > kMaxRequests) return fail(ODB_E_INVALID_ARG, "%s: n=%d outside [1, %d]", who, n, kMaxRequests);
    int rc = check_pool(who, n_pages, page_size);
    if (!rc) rc = check_columns(who, columns, page_size);
    if (rc) return rc;
    if (rows_cap < 1 || rows_cap > 1 << 24) return fail(ODB_E_INVALID_ARG, "%s: rows_cap=%d outside [1, 2^24]", who, rows_cap);
    const size_t nb = (size_t)n * 4;
    const Range reads[] = {{held, nb}, {wanted, nb}, {n_free, 4}, {row_first, nb}, {row_count, nb}};
    const Range writes[] = {{tables, nb * columns}, {free_pages, (size_t)n_pages * 4}, {len, nb}, {cu_rows, nb + 4}, {slots, (size_t)rows_cap * 4},
                            {positions, (size_t)rows_cap * 4}, {state, 16}};
    for (size_t i = 0; i < sizeof(writes) / sizeof(writes[0]); i++) {
        for (const Range &r : reads)
            if (overlap(writes[i], r)) return fail(ODB_E_INVALID_ARG, "%s: a buffer that is written overlaps one that is read", who);
        for (size_t j = 0; j < i; j++)
            if (overlap(writes[i], writes[j])) return fail(ODB_E_INVALID_ARG, "%s: two buffers that are written overlap", who);
    }
    launch_page_tables(PageTables{held, wanted, row_first, row_count, n, page_shift(page_size), columns, n_pages, rows_cap, tables, free_pages, n_free, len,
                                  cu_rows, slots, positions, state, 0, 0}, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

int odb_rope_table(float *table, int n_pos, int rot_dim, const odb_rope *rope, void *stream) {
    const char *who = "rope_table";
    if (!table || !rope) return fail(ODB_E_INVALID_ARG, "%s: NULL argument", who);
    if (n_pos < 1 || n_pos > 1 << 22) return fail(ODB_E_INVALID_ARG, "%s: n_pos=%d outside [1, 2^22]", who, n_pos);
    if (rot_dim < 2 || rot_dim > 2 * kMaxRotPairs || rot_dim & 1) return fail(ODB_E_INVALID_ARG, "%s: rot_dim=%d", who, rot_dim);
    const odb_rope &r = *rope;
    if (r.scaling < ODB_ROPE_PLAIN || r.scaling > ODB_ROPE_YARN) return fail(ODB_E_INVALID_ARG, "%s: scaling=%d", who, r.scaling);
    if (!(r.base > 1.0) || !isfinite(r.base) || !(r.magnitude >= 0.0) || !isfinite(r.magnitude))
        return fail(ODB_E_INVALID_ARG, "%s: base=%g, magnitude=%g", who, r.base, r.magnitude);
    const bool scaled = r.scaling != ODB_ROPE_PLAIN, yarn = r.scaling == ODB_ROPE_YARN;
    if (scaled && (!(r.factor >= 1.0) || !isfinite(r.factor))) return fail(ODB_E_INVALID_ARG, "%s: factor=%g", who, r.factor);
    if (yarn && (r.original_len < 1 || !(r.beta_slow >= 0.0) || !(r.beta_fast > r.beta_slow) || !isfinite(r.beta_fast)))
        return fail(ODB_E_INVALID_ARG, "%s: original_len=%d, beta_fast=%g, beta_slow=%g", who, r.original_len, r.beta_fast, r.beta_slow);
    RopeTable a{};
    a.table = table;
    a.n_pos = n_pos;
    a.pairs = rot_dim / 2;
    a.magnitude = r.magnitude > 0.0 ? r.magnitude : yarn ? 0.1 * log(r.factor) + 1.0 : 1.0;
    const long double two_pi = 6.28318530717958647692528676655900577L;
    long double base = r.base;
    if (r.scaling == ODB_ROPE_NTK && rot_dim > 2) base *= powl(r.factor, (long double)rot_dim / (rot_dim - 2));
    // (a power for every 16th pair, products in between: they add at most 15 roundings of 2^-64)
    const long double ratio = powl(base, -2.0L / rot_dim);
    long double power = 1.0L;
    for (int j = 0; j < a.pairs; j++, power *= ratio) {
        if (j % 16 == 0) power = powl(base, -2.0L * j / rot_dim);
        long double f = power;
        if (r.scaling == ODB_ROPE_LINEAR) f /= r.factor;
        if (yarn) {
            long double w = (r.original_len * f / two_pi - r.beta_slow) / ((long double)r.beta_fast - r.beta_slow);
            w = w < 0.0L ? 0.0L : w > 1.0L ? 1.0L : w;
            f = f * w + f / r.factor * (1.0L - w);
        }
        f /= two_pi;
        a.hi[j] = (double)f;
        a.lo[j] = (double)(f - a.hi[j]);
    }
    launch_rope_angles(a, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

int odb_qk_norm_rope(const odb_qk_rows *rows, const odb_pages *pages, void *stream) {
    const char *who = "qk_norm_rope";
    if (!rows) return fail(ODB_E_INVALID_ARG, "%s: NULL argument", who);
    int rc = check_pages(who, pages);
    if (rc) return rc;
    const odb_qk_rows &r = *rows;
    if ((rc = check_turned_rows(who, r, *pages, [&] { return (long long)r.rows * qk_waves_per_row(r.n_heads, *pages) >= 1 << 26; }))) return rc;
    if (!r.slots) return fail(ODB_E_INVALID_ARG, "%s: NULL slots", who);
    if (r.rows == 0) return ODB_OK;
    launch_qk_norm_rope(QkNormRope{r.q, r.k, r.v, r.in_dtype, r.q_row, r.k_row, r.v_row, r.rows, r.n_heads, r.q_gain, r.k_gain, r.eps, r.table, r.n_pos,
                                   r.rot_dim, r.interleaved, r.positions, r.slots, r.q_out, r.q_out_row, *pages, r.row_end, nullptr}, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

int odb_qk_norm_rope_quant(const odb_quant_rows *rows, const odb_quant_pages *pages, void *stream) {
    const char *who = "qk_norm_rope_quant";
    if (!rows) return fail(ODB_E_INVALID_ARG, "%s: NULL argument", who);
    odb_pages codes;
    QuantScales scales;
    int rc = check_quant_pages(who, pages, true, codes, scales);
    if (rc) return rc;
    const odb_quant_rows &r = *rows;
    if (r.n < 1 || r.n > kMaxRequests) return fail(ODB_E_INVALID_ARG, "%s: n=%d outside [1, %d]", who, r.n, kMaxRequests);
    if ((rc = check_turned_rows(who, r, codes, [&] { return quant_workgroups(r.n, r.rows, r.n_heads, r.cu_rows != nullptr, 1, codes, scales) >= 1 << 24; })) ||
        (rc = check_columns(who, r.columns, codes.page_size)))
        return rc;
    if (!r.cu_rows && r.rows != r.n) return fail(ODB_E_INVALID_ARG, "%s: without cu_rows every request has one row (%d rows, %d requests)", who, r.rows, r.n);
    if (!r.kv_len || !r.tables) return fail(ODB_E_INVALID_ARG, "%s: NULL kv_len or tables", who);
    if (r.rows == 0) return ODB_OK;
    launch_qk_norm_rope_quant(QkNormRopeQuant{r.q, r.k, r.v, r.in_dtype, r.q_row, r.k_row, r.v_row, r.rows, r.n_heads, r.q_gain, r.k_gain, r.eps, r.table, r.n_pos,
                                              r.rot_dim, r.interleaved, r.positions, r.q_out, r.q_out_row, r.cu_rows, r.first_pos, r.kv_len, r.tables, 1, r.columns,
                                              r.n, page_shift(codes.page_size), codes, scales, (unsigned *)r.odd, 1u, nullptr}, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

int odb_paged_read_quant(const odb_quant_pages *pages, const int32_t *slots, int rows, int out_dtype, void *k_out, void *v_out, long long k_row,
                         long long v_row, void *stream) {
    const char *who = "paged_read_quant";
    if (!pages) return fail(ODB_E_INVALID_ARG, "%s: pages is NULL", who);
    odb_quant_pages any = *pages;
    any.dtype = ODB_F16;
    PagedReadQuant p{};
    int rc = check_quant_pages(who, &any, true, p.pages, p.scales);
    if (rc) return rc;
    const int dim = any.head_dim, kv = any.n_kv_heads;
    if (rows < 0 || rows > 1 << 24) return fail(ODB_E_INVALID_ARG, "%s: rows=%d outside [0, 2^24]", who, rows);
    if ((long long)rows * kv * dim >= 1ll << 33) return fail(ODB_E_INVALID_ARG, "%s: %d rows of %d heads are too many for one launch", who, rows, kv);
    if (!slots) return fail(ODB_E_INVALID_ARG, "%s: NULL slots", who);
    if (out_dtype != ODB_F16 && out_dtype != ODB_BF16 && out_dtype != ODB_F32) return fail(ODB_E_INVALID_ARG, "%s: out_dtype=%d", who, out_dtype);
    if ((rc = check_rows(who, "k_out", k_out, k_row, kv, dim)) || (rc = check_rows(who, "v_out", v_out, v_row, kv, dim))) return rc;
    const int eb = out_dtype == ODB_F32 ? 4 : 2;
    // (the rows of one may lie between those of the other)
    const Range ko{k_out, span(rows, k_row, kv, dim, eb)}, vo{v_out, span(rows, v_row, kv, dim, eb)};
    if (overlap(ko, vo)) {
        const long long bytes = k_row * eb, gap = rows > 1 ? (((intptr_t)v_out - (intptr_t)k_out) % bytes + bytes) % bytes : 0, own = (long long)kv * dim * eb;
        if (rows == 1 || k_row != v_row || gap < own || gap + own > bytes) return fail(ODB_E_INVALID_ARG, "%s: k_out and v_out overlap", who);
    }
    if (rows == 0) return ODB_OK;
    p.slots = slots; p.rows = rows; p.out_dtype = out_dtype;
    p.k = k_out; p.v = v_out; p.k_row = k_row; p.v_row = v_row;
    launch_paged_read_quant(p, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

long long odb_paged_attention_workspace(const odb_attention *a, const odb_pages *pages) {
    PagedAttn p;
    int nt;
    const int rc = plan_paged_attention(a, pages, false, p, nt);
    return rc ? rc : (long long)paged_attn_workspace(*pages, p.rows, p.heads, nt, p.split);
}

int odb_paged_attention(const odb_attention *a, const odb_pages *pages, void *stream) {
    PagedAttn p;
    int nt;
    int rc = plan_paged_attention(a, pages, true, p, nt);
    if (rc || (rc = bind_attention("paged_attention", a, p, nt))) return rc;
    if (a->rows == 0) return ODB_OK;
    launch_paged_attention(p, nt, a->workspace, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

long long odb_paged_attention_quant_workspace(const odb_attention *a, const odb_quant_pages *pages) {
    PagedAttnQuant p;
    int nt;
    const int rc = plan_paged_attention_quant(a, pages, false, p, nt);
    return rc ? rc : (long long)paged_attn_workspace(p.pages, p.rows, p.heads, nt, p.split);
}

int odb_paged_attention_quant(const odb_attention *a, const odb_quant_pages *pages, void *stream) {
    PagedAttnQuant p;
    int nt;
    int rc = plan_paged_attention_quant(a, pages, true, p, nt);
    if (rc || (rc = bind_attention("paged_attention_quant", a, p, nt))) return rc;
    if (a->rows == 0) return ODB_OK;
    launch_paged_attention_quant(p, nt, a->workspace, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return ODB_OK;
}

}  // extern "C"
