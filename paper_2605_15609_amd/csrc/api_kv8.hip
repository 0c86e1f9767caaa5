// C ABI of the head norms with rotary positions and of the caches in 8 bits: argument checks.
#include <math.h>

#include <algorithm>

#include "psd_internal.h"
#include "regions.h"

#define CHECK(expr)                  \
    do {                             \
        int32_t rc_ = (expr);        \
        if (rc_ != PSD_OK) return rc_; \
    } while (0)

namespace {

constexpr int32_t kMostPositions = 1 << 30;   // of a unit: the kernels count up to a stage's more in 32 bits

int32_t check_dtype(int32_t dtype) {
    if (dtype != PSD_DTYPE_BF16 && dtype != PSD_DTYPE_FP32) PSD_FAIL(PSD_ERR_UNSUPPORTED, "dtype %d", dtype);
    return PSD_OK;
}
int64_t size_of(int32_t dtype) { return dtype == PSD_DTYPE_BF16 ? 2 : 4; }

// `rows` rows of `heads` heads, `ld` elements apart
Region rows_region(const void *p, int64_t rows, int64_t ld, int64_t width, int64_t esz) {
    return {reinterpret_cast<uintptr_t>(p), 1, 0, p ? rows : 0, ld * esz, width * esz};
}

int32_t check_cache(const psd_kv8_cache *a, int32_t units, Kv8 *out) {
    if (!a) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL cache");
    if (a->reserved != 0) PSD_FAIL(PSD_ERR_INVALID_ARG, "cache: reserved is not 0");
    if (a->format != PSD_KV8_INT8 && a->format != PSD_KV8_E4M3) PSD_FAIL(PSD_ERR_UNSUPPORTED, "cache: format %d", a->format);
    if (a->block != 16 && a->block != 32 && a->block != 64 && a->block != 128) PSD_FAIL(PSD_ERR_UNSUPPORTED, "cache: %d positions to a scale (16, 32, 64, 128)", a->block);
    if (a->d_head != 16 && a->d_head != 32 && a->d_head != 64 && a->d_head != 128) PSD_FAIL(PSD_ERR_UNSUPPORTED, "cache: d_head %d (16, 32, 64, 128)", a->d_head);
    if (a->n_kv_heads < 1 || (int64_t)a->n_kv_heads * a->d_head >= 1 << 24) PSD_FAIL(PSD_ERR_SHAPE, "cache: %d KV heads", a->n_kv_heads);
    if (units < 1) PSD_FAIL(PSD_ERR_SHAPE, "%d units", units);
    if (a->capacity < 0 || a->capacity > kMostPositions || a->capacity % KV8_TILE || a->capacity % a->block)
        PSD_FAIL(PSD_ERR_SHAPE, "cache: %d positions are not whole blocks of %d", a->capacity, std::max(a->block, KV8_TILE));
    if (a->len < 0 || a->len > a->capacity) PSD_FAIL(PSD_ERR_SHAPE, "cache: %d positions of %d", a->len, a->capacity);
    if (a->stride_codes < 0 || a->stride_scales < 0) PSD_FAIL(PSD_ERR_SHAPE, "cache: negative stride");
    if (units > 1 && (double)units * std::max((double)a->stride_codes, 4.0 * a->stride_scales) >= 0x1p60)
        PSD_FAIL(PSD_ERR_SHAPE, "cache: %d units %lld bytes and %lld floats apart", units, (long long)a->stride_codes, (long long)a->stride_scales);
    if (a->capacity > 0) {
        if (!a->codes || !a->scales) PSD_FAIL(PSD_ERR_INVALID_ARG, "cache: codes or scales are NULL");
        if (misaligned16(a->codes) || a->stride_codes % 16) PSD_FAIL(PSD_ERR_SHAPE, "cache: codes must be 16-byte aligned");
        if (reinterpret_cast<uintptr_t>(a->scales) % 8 || a->stride_scales % 2) PSD_FAIL(PSD_ERR_SHAPE, "cache: scales must be 8-byte aligned");
    }
    if (reinterpret_cast<uintptr_t>(a->lens) % 4) PSD_FAIL(PSD_ERR_SHAPE, "cache: lens must be 4-byte aligned");
    out->codes = (uint8_t *)a->codes;
    out->scales = (float2 *)a->scales;
    out->lens = a->lens;
    out->stride_codes = a->stride_codes;
    out->stride_scales = a->stride_scales / 2;
    out->capacity = a->capacity;
    out->len = a->len;
    out->block_shift = a->block == 16 ? 4 : a->block == 32 ? 5 : a->block == 64 ? 6 : 7;
    out->format = a->format;
    out->n_kv_heads = a->n_kv_heads;
    out->d_head = a->d_head;
    out->seqs_per_unit = a->seqs_per_unit;
    return PSD_OK;
}

int64_t unit_codes(const Kv8 &c) { return (int64_t)c.n_kv_heads * c.capacity * c.d_head * 2; }
int64_t unit_scales(const Kv8 &c) { return (int64_t)c.n_kv_heads * (c.capacity >> c.block_shift) * 8; }
Region codes_region(const Kv8 &c, int64_t units) { return {reinterpret_cast<uintptr_t>(c.codes), units, c.stride_codes, c.capacity > 0 ? 1 : 0, 0, unit_codes(c)}; }
Region scales_region(const Kv8 &c, int64_t units) { return {reinterpret_cast<uintptr_t>(c.scales), units, c.stride_scales * 8, c.capacity > 0 ? 1 : 0, 0, unit_scales(c)}; }

int32_t check_rows(const char *what, const void *p, int64_t ld, int64_t width, int32_t dtype) {
    if (misaligned16(p) || ld % (16 / size_of(dtype))) PSD_FAIL(PSD_ERR_SHAPE, "%s: rows must be 16-byte aligned", what);
    if (ld < width) PSD_FAIL(PSD_ERR_SHAPE, "%s: rows of %lld elements", what, (long long)ld);
    return PSD_OK;
}

int32_t check_attention(const psd_attention_shape *a, const psd_kv8_cache *cache, SharedShape *sh, Kv8 *c) {
    if (!a || !cache) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL shape / cache");
    CHECK(check_dtype(a->dtype));
    if (!shared_attention_takes(a->dtype, a->d_head)) PSD_FAIL(PSD_ERR_UNSUPPORTED, "d_head %d (bf16: 64, 128; fp32: 16, 32, 64, 128)", a->d_head);
    if (a->S < 1 || a->L < 1 || a->L > PSD_MAX_BLOCK) PSD_FAIL(PSD_ERR_SHAPE, "%d sequences of %d rows (1..%d)", a->S, a->L, PSD_MAX_BLOCK);
    if (a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads) PSD_FAIL(PSD_ERR_SHAPE, "%d heads on %d KV heads", a->n_heads, a->n_kv_heads);
    if ((int64_t)a->n_heads * a->d_head >= 1 << 24 || (int64_t)a->S * a->L * a->n_heads >= 1ll << 31)
        PSD_FAIL(PSD_ERR_SHAPE, "%d sequences of %d rows of %d heads are too many", a->S, a->L, a->n_heads);
    const int64_t row = (int64_t)a->n_heads * a->d_head, chunk = 16 / size_of(a->dtype);
    if (a->ld_q < row || a->ld_q % chunk) PSD_FAIL(PSD_ERR_SHAPE, "query rows of %lld elements", (long long)a->ld_q);
    if (a->ld_out < row || a->ld_out % chunk) PSD_FAIL(PSD_ERR_SHAPE, "output rows of %lld elements", (long long)a->ld_out);
    if (cache->seqs_per_unit < 1 || a->S % cache->seqs_per_unit) PSD_FAIL(PSD_ERR_SHAPE, "units of %d sequences do not divide %d", cache->seqs_per_unit, a->S);
    CHECK(check_cache(cache, a->S / cache->seqs_per_unit, c));
    if (c->n_kv_heads != a->n_kv_heads || c->d_head != a->d_head)
        PSD_FAIL(PSD_ERR_SHAPE, "a cache of %d heads of %d for %d of %d", c->n_kv_heads, c->d_head, a->n_kv_heads, a->d_head);
    *sh = {a->S, a->L, a->n_heads, a->n_kv_heads, a->d_head, a->dtype, a->ld_q, a->ld_out, (int64_t)a->S * a->L * a->n_heads};
    return PSD_OK;
}

}   // namespace

int32_t psd_kv8_struct_sizes(int32_t *out, int32_t n) {
    const int32_t sizes[] = {(int32_t)sizeof(psd_rotary_shape), (int32_t)sizeof(psd_rotary_scaling), (int32_t)sizeof(psd_kv8_cache)};
    const int32_t count = (int32_t)(sizeof(sizes) / sizeof(sizes[0]));
    for (int32_t i = 0; i < n && i < count && out; ++i) out[i] = sizes[i];
    return count;
}

int32_t psd_rotary_frequencies(const psd_rotary_scaling *s, int32_t rotated, double *frequencies, double *factor) {
    if (!s || !frequencies) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL scaling / frequencies");
    if (s->reserved != 0) PSD_FAIL(PSD_ERR_INVALID_ARG, "scaling: reserved is not 0");
    if (rotated < 2 || rotated % 2 || rotated > PSD_MAX_ROTARY_HEAD) PSD_FAIL(PSD_ERR_SHAPE, "%d rotated channels (an even number up to %d)", rotated, PSD_MAX_ROTARY_HEAD);
    if (s->kind < PSD_ROTARY_PLAIN || s->kind > PSD_ROTARY_PARTS) PSD_FAIL(PSD_ERR_UNSUPPORTED, "scaling %d", s->kind);
    if (!(s->theta > 0.0) || !isfinite(s->theta)) PSD_FAIL(PSD_ERR_INVALID_ARG, "theta %g", s->theta);
    if (s->kind != PSD_ROTARY_PLAIN && (!(s->stretch >= 1.0) || !isfinite(s->stretch))) PSD_FAIL(PSD_ERR_INVALID_ARG, "stretch %g (1 or more)", s->stretch);
    if (s->kind == PSD_ROTARY_BASE && rotated == 2) PSD_FAIL(PSD_ERR_SHAPE, "the base of one pair says nothing");
    if (s->kind == PSD_ROTARY_PARTS && (!(s->trained > 0.0) || !(s->slow >= 0.0) || !(s->fast > s->slow) || !isfinite(s->trained) || !isfinite(s->fast)))
        PSD_FAIL(PSD_ERR_INVALID_ARG, "trained %g, slow %g, fast %g (slow < fast)", s->trained, s->slow, s->fast);
    const double theta = s->kind == PSD_ROTARY_BASE ? s->theta * pow(s->stretch, rotated / (rotated - 2.0)) : s->theta;
    for (int32_t j = 0; j < rotated / 2; ++j) {
        double f = pow(theta, -2.0 * j / rotated);
        if (s->kind == PSD_ROTARY_LINEAR) f /= s->stretch;
        if (s->kind == PSD_ROTARY_PARTS) {
            const double turns = s->trained * f / (2.0 * M_PI), as_is = std::min(std::max((turns - s->slow) / (s->fast - s->slow), 0.0), 1.0);
            f *= as_is + (1.0 - as_is) / s->stretch;
        }
        frequencies[j] = f;
    }
    if (factor) *factor = s->kind == PSD_ROTARY_PARTS ? 0.1 * log(s->stretch) + 1.0 : 1.0;
    return PSD_OK;
}

int32_t psd_rotary(const psd_rotary_shape *a, const void *q, const void *k, const double *frequencies, const int32_t *positions, const float *q_gain,
                   const float *k_gain, void *q_out, void *k_out, void *stream) {
    if (!a) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL shape");
    if (a->reserved != 0) PSD_FAIL(PSD_ERR_INVALID_ARG, "shape: reserved is not 0");
    CHECK(check_dtype(a->dtype));
    if (a->n_tokens < 1 || a->n_heads < 1 || a->n_kv_heads < 0) PSD_FAIL(PSD_ERR_SHAPE, "%lld tokens of %d and %d heads", (long long)a->n_tokens, a->n_heads, a->n_kv_heads);
    if (a->d_head < 2 || a->d_head % 2 || a->d_head > PSD_MAX_ROTARY_HEAD) PSD_FAIL(PSD_ERR_UNSUPPORTED, "d_head %d (an even number up to %d)", a->d_head, PSD_MAX_ROTARY_HEAD);
    if (((int64_t)a->n_heads + a->n_kv_heads) * a->d_head >= 1 << 24) PSD_FAIL(PSD_ERR_SHAPE, "%d and %d heads of %d", a->n_heads, a->n_kv_heads, a->d_head);
    if (a->rotated < 2 || a->rotated % 2 || a->rotated > a->d_head) PSD_FAIL(PSD_ERR_SHAPE, "%d rotated channels of %d", a->rotated, a->d_head);
    if (a->interleaved != 0 && a->interleaved != 1) PSD_FAIL(PSD_ERR_INVALID_ARG, "interleaved %d", a->interleaved);
    if (!isfinite(a->factor)) PSD_FAIL(PSD_ERR_INVALID_ARG, "factor %g", (double)a->factor);
    if (!(a->eps >= 0.f) || !isfinite(a->eps)) PSD_FAIL(PSD_ERR_INVALID_ARG, "eps %g", (double)a->eps);
    if (!positions && (a->rows_per_seq < 1 || a->first < 0 || (int64_t)a->first + a->rows_per_seq > 1ll << 31))
        PSD_FAIL(PSD_ERR_SHAPE, "positions %d .. of %d rows", a->first, a->rows_per_seq);
    if (!q || !q_out || !frequencies) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL q / q_out / frequencies");
    if (a->n_kv_heads > 0 && (!k || !k_out)) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL k / k_out");
    const int64_t esz = size_of(a->dtype);
    Rotary r;
    r.rows[0] = {q, q_out, q_gain, a->ld_q, a->ld_q_out, a->n_heads};
    if (a->n_kv_heads > 0) r.rows[1] = {k, k_out, k_gain, a->ld_k, a->ld_k_out, a->n_kv_heads};
    Region in[2], out[2];
    for (int i = 0; i < 2; ++i) {
        const RotaryRows &x = r.rows[i];
        const int64_t width = (int64_t)x.heads * a->d_head;
        if (x.heads > 0 && (x.ld_in < width || x.ld_out < width)) PSD_FAIL(PSD_ERR_SHAPE, "rows of %lld and %lld elements for %d heads", (long long)x.ld_in, (long long)x.ld_out, x.heads);
        if (reinterpret_cast<uintptr_t>(x.in) % esz || reinterpret_cast<uintptr_t>(x.out) % esz) PSD_FAIL(PSD_ERR_SHAPE, "rows must be aligned to their type");
        if (x.heads > 0 && (double)a->n_tokens * std::max(x.ld_in, x.ld_out) >= 0x1p60) PSD_FAIL(PSD_ERR_SHAPE, "%lld rows are too many", (long long)a->n_tokens);
        in[i] = rows_region(x.in, a->n_tokens, x.ld_in, width, esz);
        out[i] = rows_region(x.out, a->n_tokens, x.ld_out, width, esz);
    }
    if (reinterpret_cast<uintptr_t>(frequencies) % 8 || reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(q_gain) % 4 || reinterpret_cast<uintptr_t>(k_gain) % 4)
        PSD_FAIL(PSD_ERR_SHAPE, "frequencies, positions and gains must be aligned to their types");
    const Region read[] = {dense(frequencies, a->rotated / 2 * 8), dense(positions, a->n_tokens * 4), dense(q_gain, a->d_head * 4), dense(k_gain, a->d_head * 4)};
    for (int i = 0; i < 2; ++i) {
        for (int j = 0; j < 2; ++j) {
            const bool same = i == j && r.rows[i].in == r.rows[i].out && r.rows[i].ld_in == r.rows[i].ld_out;
            if (!same && !apart(out[i], in[j])) PSD_FAIL(PSD_ERR_INVALID_ARG, "an output overlaps an input without being it");
        }
        for (const Region &x : read)
            if (!apart(out[i], x)) PSD_FAIL(PSD_ERR_INVALID_ARG, "an output lies on frequencies, positions or gains");
    }
    if (!apart(out[0], out[1])) PSD_FAIL(PSD_ERR_INVALID_ARG, "the outputs overlap each other");
    r.frequencies = frequencies;
    r.positions = positions;
    r.n_tokens = a->n_tokens;
    r.d_head = a->d_head;
    r.rotated = a->rotated;
    r.interleaved = a->interleaved;
    r.first = a->first;
    r.rows_per_seq = a->rows_per_seq;
    r.dtype = a->dtype;
    r.factor = a->factor;
    r.eps = a->eps;
    if (!rotary_launchable(r)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    launch_rotary(r, (hipStream_t)stream);
    PSD_HIP(hipGetLastError());
    return PSD_OK;
}

int32_t psd_kv8_store(const psd_kv8_cache *cache, int32_t units, const void *k, const void *v, int64_t ld_k, int64_t ld_v, int32_t dtype, int32_t n,
                      int32_t first, const int32_t *starts, const int32_t *counts, void *stream) {
    Kv8 c;
    CHECK(check_cache(cache, units, &c));
    CHECK(check_dtype(dtype));
    if (n < 0 || n > kMostPositions || (int64_t)units * n >= 1ll << 40) PSD_FAIL(PSD_ERR_SHAPE, "%d rows of %d units", n, units);
    if (!starts && (first < 0 || (int64_t)first + n > c.capacity)) PSD_FAIL(PSD_ERR_SHAPE, "rows %d .. %lld of %d positions", first, (long long)first + n, c.capacity);
    if (units > 1 && (c.stride_codes < unit_codes(c) || c.stride_scales * 8 < unit_scales(c))) PSD_FAIL(PSD_ERR_SHAPE, "the units of the cache lie on each other");
    if (n == 0) return PSD_OK;
    if (!k || !v) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL k / v");
    const int64_t width = (int64_t)c.n_kv_heads * c.d_head, esz = size_of(dtype), rows = (int64_t)units * n;
    CHECK(check_rows("keys", k, ld_k, width, dtype));
    CHECK(check_rows("values", v, ld_v, width, dtype));
    if ((double)rows * std::max(ld_k, ld_v) >= 0x1p60) PSD_FAIL(PSD_ERR_SHAPE, "%lld rows are too many", (long long)rows);
    if (reinterpret_cast<uintptr_t>(starts) % 4 || reinterpret_cast<uintptr_t>(counts) % 4) PSD_FAIL(PSD_ERR_SHAPE, "starts and counts must be 4-byte aligned");
    const Region written[] = {codes_region(c, units), scales_region(c, units)};
    const Region read[] = {rows_region(k, rows, ld_k, width, esz), rows_region(v, rows, ld_v, width, esz), dense(starts, units * 4ll), dense(counts, units * 4ll),
                           dense(c.lens, units * 4ll)};
    if (!apart(written[0], written[1])) PSD_FAIL(PSD_ERR_INVALID_ARG, "codes and scales overlap");
    for (const Region &w : written)
        for (const Region &x : read)
            if (!apart(w, x)) PSD_FAIL(PSD_ERR_INVALID_ARG, "the cache overlaps what is read");
    if (!kv8_store_launchable(c, units, n)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    Kv8Rows r;
    r.k = const_cast<void *>(k);
    r.v = const_cast<void *>(v);
    r.ld_k = ld_k;
    r.ld_v = ld_v;
    r.n = n;
    r.first = first;
    r.dtype = dtype;
    launch_kv8_store(c, units, r, starts, counts, (hipStream_t)stream);
    PSD_HIP(hipGetLastError());
    return PSD_OK;
}

int32_t psd_kv8_load(const psd_kv8_cache *cache, int32_t units, int32_t first, int32_t n, void *k, void *v, int64_t ld_k, int64_t ld_v, int32_t dtype, void *stream) {
    Kv8 c;
    CHECK(check_cache(cache, units, &c));
    CHECK(check_dtype(dtype));
    if (n < 0 || first < 0 || (int64_t)first + n > c.capacity) PSD_FAIL(PSD_ERR_SHAPE, "rows %d .. %lld of %d positions", first, (long long)first + n, c.capacity);
    if (n == 0) return PSD_OK;
    if (!k || !v) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL k / v");
    const int64_t width = (int64_t)c.n_kv_heads * c.d_head, esz = size_of(dtype), rows = (int64_t)units * n;
    CHECK(check_rows("keys", k, ld_k, width, dtype));
    CHECK(check_rows("values", v, ld_v, width, dtype));
    if ((double)rows * std::max(ld_k, ld_v) >= 0x1p60) PSD_FAIL(PSD_ERR_SHAPE, "%lld rows are too many", (long long)rows);
    const Region written[] = {rows_region(k, rows, ld_k, width, esz), rows_region(v, rows, ld_v, width, esz)};
    if (!apart(written[0], written[1])) PSD_FAIL(PSD_ERR_INVALID_ARG, "keys and values overlap");
    for (const Region &w : written)
        for (const Region &x : {codes_region(c, units), scales_region(c, units), dense(c.lens, units * 4ll)})
            if (!apart(w, x)) PSD_FAIL(PSD_ERR_INVALID_ARG, "the rows lie on the cache");
    if (!kv8_load_launchable(c, units, n)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    Kv8Rows r;
    r.k = k;
    r.v = v;
    r.ld_k = ld_k;
    r.ld_v = ld_v;
    r.n = n;
    r.first = first;
    r.dtype = dtype;
    launch_kv8_load(c, units, r, (hipStream_t)stream);
    PSD_HIP(hipGetLastError());
    return PSD_OK;
}

int64_t psd_attention_kv8_bytes(const psd_attention_shape *shape, const psd_kv8_cache *cache, int32_t own_rows) {
    SharedShape sh;
    Kv8 c;
    Kv8Launch ln;
    CHECK(check_attention(shape, cache, &sh, &c));
    if (own_rows != 0 && own_rows != 1) PSD_FAIL(PSD_ERR_INVALID_ARG, "own_rows %d", own_rows);
    if (!plan_attention_kv8(sh, c, own_rows, &ln)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    return attention_parts_bytes(sh, ln);
}

int32_t psd_debug_attention_kv8_plan(const psd_attention_shape *shape, const psd_kv8_cache *cache, int32_t own_rows, int32_t *plan) {
    SharedShape sh;
    Kv8 c;
    Kv8Launch ln;
    CHECK(check_attention(shape, cache, &sh, &c));
    if (!plan) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL plan");
    if (!plan_attention_kv8(sh, c, own_rows != 0, &ln)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    const int32_t what[4] = {ln.tiled, ln.tiles, ln.splits, ln.chunk};
    std::copy(what, what + 4, plan);
    return PSD_OK;
}

int32_t psd_debug_force_attention_kv8(int32_t form, int32_t parts) {
    if (form < -1 || form > 1 || parts < 0) PSD_FAIL(PSD_ERR_INVALID_ARG, "form %d, %d parts", form, parts);
    force_attention_kv8(form, parts);
    return PSD_OK;
}

int32_t psd_attention_kv8(const psd_attention_shape *shape, const void *q, const psd_kv8_cache *cache, const void *k, const void *v, int64_t ld_k, int64_t ld_v, void *out,
                          float *lse, void *ws, int64_t ws_bytes, void *stream) {
    SharedShape sh;
    Kv8 c;
    CHECK(check_attention(shape, cache, &sh, &c));
    if (!q || !out) PSD_FAIL(PSD_ERR_INVALID_ARG, "NULL q / out");
    if (misaligned16(q) || misaligned16(out)) PSD_FAIL(PSD_ERR_SHAPE, "q and out must be 16-byte aligned");
    if (!k != !v) PSD_FAIL(PSD_ERR_INVALID_ARG, "keys and values of the rows' own blocks, or neither");
    const int64_t esz = size_of(sh.dtype), row = (int64_t)sh.n_heads * sh.d_head, width = (int64_t)sh.n_kv_heads * sh.d_head, n_tokens = (int64_t)sh.S * sh.L;
    if (k) {
        CHECK(check_rows("keys", k, ld_k, width, sh.dtype));
        CHECK(check_rows("values", v, ld_v, width, sh.dtype));
    }
    if ((double)n_tokens * std::max(std::max(sh.ld_q, sh.ld_out), k ? std::max(ld_k, ld_v) : 0) >= 0x1p60) PSD_FAIL(PSD_ERR_SHAPE, "%lld rows are too many", (long long)n_tokens);
    if (reinterpret_cast<uintptr_t>(lse) % 4) PSD_FAIL(PSD_ERR_SHAPE, "lse must be 4-byte aligned");
    const int64_t units = sh.S / c.seqs_per_unit;
    const Region to = rows_region(out, n_tokens, sh.ld_out, row, esz), sums = dense(lse, sh.n_rows * 4);
    if (!apart(to, sums)) PSD_FAIL(PSD_ERR_INVALID_ARG, "lse lies on out");
    const Region read[] = {rows_region(q, n_tokens, sh.ld_q, row, esz), rows_region(k, n_tokens, ld_k, width, esz), rows_region(v, n_tokens, ld_v, width, esz),
                           codes_region(c, units), scales_region(c, units), dense(c.lens, units * 4)};
    for (const Region &x : read)
        if (!apart(x, to) || !apart(x, sums)) PSD_FAIL(PSD_ERR_INVALID_ARG, "out or lse lies on what is read");
    Kv8Launch ln;
    if (!plan_attention_kv8(sh, c, k != nullptr, &ln)) PSD_FAIL(PSD_ERR_SHAPE, "more workgroups than a launch takes");
    const int64_t need = attention_parts_bytes(sh, ln);
    if (need > 0 && (!ws || ws_bytes < need)) PSD_FAIL(PSD_ERR_WORKSPACE, "workspace of %lld bytes, %lld needed", (long long)ws_bytes, (long long)need);
    if (need > 0 && (reinterpret_cast<uintptr_t>(ws) & 255) != 0) PSD_FAIL(PSD_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (need > 0) {
        const Region scratch = dense(ws, need);
        for (const Region &x : read)
            if (!apart(x, scratch)) PSD_FAIL(PSD_ERR_WORKSPACE, "the workspace lies on what is read");
        if (!apart(to, scratch) || !apart(sums, scratch)) PSD_FAIL(PSD_ERR_WORKSPACE, "the workspace lies on out or lse");
    }
    ln.k = k;
    ln.v = v;
    ln.ld_k = ld_k;
    ln.ld_v = ld_v;
    place_attention_parts(sh, ln, out, lse, ws);
    launch_attention_kv8(q, sh, ln, (hipStream_t)stream);
    PSD_HIP(hipGetLastError());
    return PSD_OK;
}
