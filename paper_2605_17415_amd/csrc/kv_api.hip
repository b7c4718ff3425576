// C ABI of the paged key-value cache (include/ivftq_kv.h): argument checks, the cache as kernels see it, launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "kv_pick.h"

namespace ivftq {

extern template hipError_t kv_attend_d<64>(const KvAttend&, const KvWork&, int, hipStream_t);
extern template hipError_t kv_attend_d<96>(const KvAttend&, const KvWork&, int, hipStream_t);
extern template hipError_t kv_attend_d<128>(const KvAttend&, const KvWork&, int, hipStream_t);
extern template hipError_t kv_attend_d<192>(const KvAttend&, const KvWork&, int, hipStream_t);
extern template hipError_t kv_attend_d<256>(const KvAttend&, const KvWork&, int, hipStream_t);
extern template hipError_t kv_score_d<64>(const KvAttend&, const void*, float*, int, hipStream_t);
extern template hipError_t kv_picked_d<64>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);
extern template hipError_t kv_score_d<96>(const KvAttend&, const void*, float*, int, hipStream_t);
extern template hipError_t kv_picked_d<96>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);
extern template hipError_t kv_score_d<128>(const KvAttend&, const void*, float*, int, hipStream_t);
extern template hipError_t kv_picked_d<128>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);
extern template hipError_t kv_score_d<192>(const KvAttend&, const void*, float*, int, hipStream_t);
extern template hipError_t kv_picked_d<192>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);
extern template hipError_t kv_score_d<256>(const KvAttend&, const void*, float*, int, hipStream_t);
extern template hipError_t kv_picked_d<256>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);

KvWork kv_work(int format, int d, int batch, int kv_heads, int64_t rows, int q_heads, int max_new, int64_t capacity) {
    KvWork w{};
    const int64_t cols = (int64_t)max_new * (q_heads / kv_heads), all = rows * q_heads;
    w.few = cols <= kFewRows;
    if (w.few) {
        w.col_tiles = (int)((cols + 15) / 16);
        w.split = capacity > 512;
    } else {
        w.row_tiles = (int)((cols + kManyRows - 1) / kManyRows);
        const int64_t wgs = (int64_t)batch * kv_heads * w.row_tiles, room = 256 * (d <= 128 ? 2 : 1);       // workgroups that the compute units hold (of d = 64 more would fit)
        // Up to twice as many, codes gain by sharing (752 workgroups of 16,000 keys: 1291 us, 1398 uncut), 16 bits do not (920
        // and 900).
        if (wgs < (format == IVFTQ_KV_CODE4 ? 2 : 1) * room && kv_heads <= room && capacity > 512) w.shared = (int)(room / kv_heads);
    }
    int64_t at = 0;
    auto room = [&](int64_t bytes) { const int64_t p = at; at += round_up64(bytes, 256); return p; };
    if (format == IVFTQ_KV_CODE4) {
        w.z = room(all * d * 4);
        w.zn = room(all * 4);
    }
    if (format == IVFTQ_KV_CODE4) w.whole = room(all * d * 4);
    if (w.shared) {
        const int64_t slots = (int64_t)2 * kv_heads * w.shared * kManyRows;
        w.part = room(slots * d * 4);
        w.ml = room(slots * 8);
        w.begin = room(8 * (1 + (int64_t)batch * w.row_tiles));
    }
    if (w.split) {
        w.part = room((int64_t)w.col_tiles * 2 * kFewMaxWgs * 16 * d * 4);
        w.ml = room((int64_t)w.col_tiles * 2 * kFewMaxWgs * 16 * 2 * 4);
    }
    w.bytes = at;
    return w;
}

hipError_t launch_kv_attend(const KvAttend& a, const KvWork& w, int d, int format, hipStream_t st) {
    switch (d) {
        case 64: return kv_attend_d<64>(a, w, format, st);
        case 96: return kv_attend_d<96>(a, w, format, st);
        case 128: return kv_attend_d<128>(a, w, format, st);
        case 192: return kv_attend_d<192>(a, w, format, st);
        default: return kv_attend_d<256>(a, w, format, st);
    }
}

PickWork pick_work(const ivftq_kv_cache& c, int64_t rows, int q_heads, int max_new, int count) {
    PickWork w{};
    const int format = c.format, d = c.d, group = q_heads / c.heads;
    const int64_t all = rows * q_heads;
    w.col_tiles = (group + 15) / 16;
    // Rows of a unit: their heads fill a product's columns, their columns' bits and their lists 16 KB and 4,096 places (a chunk of 794 rows, four
    // heads a group: 94 us, two rows each 121, one 153).  Where the rows alone are too few for the chip each is worked on by itself (eight
    // sequences of four new rows: 16 us, 23 together).
    w.words = (c.columns + 31) / 32;
    w.tokens = group < 16 && rows * c.heads >= 1024 ? 16 / group : 1;
    if (w.tokens > max_new) w.tokens = max_new;
    while (w.tokens > 1 && ((int64_t)w.tokens * w.words > 4096 || (int64_t)w.tokens * count > kMostPicks)) --w.tokens;
    if (w.tokens == 1) w.words = 0;
    w.list = w.tokens * count < c.columns || w.tokens == 1 ? w.tokens * count : c.columns;
    w.units = (int32_t)(w.tokens == 1 ? rows : rows / w.tokens + c.batch);
    // as many workgroups as the chip holds, but eight tiles for each, two for each of its wavefronts: the second kernel costs what those do
    const int64_t pairs = (int64_t)w.units * c.heads * w.col_tiles, most = (int64_t)(count < c.columns ? count : c.columns) * c.page / kFewTile / 8;
    const int64_t busy = (w.tokens == 1 ? rows : (rows / w.tokens > c.batch ? rows / w.tokens : c.batch)) * c.heads * w.col_tiles;
    int64_t splits = busy ? 256 * (d <= 64 ? 4 : (d <= 128 ? 3 : 1)) / busy : 1;
    splits = splits < most ? splits : most;
    w.splits = (int)(splits < 1 ? 1 : (splits < 64 ? splits : 64));
    int64_t at = 0;
    auto room = [&](int64_t bytes) { const int64_t p = at; at += round_up64(bytes, 256); return p; };
    if (format == IVFTQ_KV_CODE4) {
        w.z = room(all * d * 4);
        w.zn = room(all * 4);
        if (w.splits == 1) w.whole = room(all * d * 4);
    }
    if (w.splits > 1) {
        w.part = room(pairs * w.splits * 16 * d * 4);
        w.ml = room(pairs * w.splits * 16 * 8);
    }
    w.bytes = at;
    return w;
}

ScoreWork score_work(int format, int d, int64_t rows, int q_heads, int kv_heads, bool one) {
    ScoreWork w{};
    int64_t at = 0;
    auto room = [&](int64_t bytes) { const int64_t p = at; at += round_up64(bytes, 256); return p; };
    w.z = -1;
    if (format == IVFTQ_KV_CODE4 && (one || 16 % (q_heads / kv_heads))) {
        w.z = room(rows * q_heads * d * 4);
        w.zn = room(rows * q_heads * 4);
    }
    if (!one) {
        w.tiles = (int32_t)((rows + 15) / 16);
        w.sides = room((int64_t)w.tiles * 16 * kv_heads * (format == IVFTQ_KV_BF16 ? 3 : 2) * 2 * d * 2);
        w.unit = room((int64_t)w.tiles * 16 * kv_heads * 4);
    }
    w.bytes = at;
    return w;
}

hipError_t launch_kv_score(const KvAttend& a, const void* digests, float* scores, int d, int format, hipStream_t st) {
    switch (d) {
        case 64: return kv_score_d<64>(a, digests, scores, format, st);
        case 96: return kv_score_d<96>(a, digests, scores, format, st);
        case 128: return kv_score_d<128>(a, digests, scores, format, st);
        case 192: return kv_score_d<192>(a, digests, scores, format, st);
        default: return kv_score_d<256>(a, digests, scores, format, st);
    }
}
hipError_t launch_kv_picked(const KvAttend& a, const PickWork& w, const int32_t* chosen, int count, int d, int format, hipStream_t st) {
    switch (d) {
        case 64: return kv_picked_d<64>(a, w, chosen, count, format, st);
        case 96: return kv_picked_d<96>(a, w, chosen, count, format, st);
        case 128: return kv_picked_d<128>(a, w, chosen, count, format, st);
        case 192: return kv_picked_d<192>(a, w, chosen, count, format, st);
        default: return kv_picked_d<256>(a, w, chosen, count, format, st);
    }
}

}  // namespace ivftq

using namespace ivftq;

namespace {

ivftq_status refuse(ivftq_status code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}
ivftq_status done(hipError_t e, const char* what) {
    return e == hipSuccess ? IVFTQ_OK : refuse(e == hipErrorOutOfMemory ? IVFTQ_OOM : IVFTQ_HIP_ERROR, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool known_d(int d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }
bool known_page(int p) { return p >= 16 && p <= 1024 && (p & (p - 1)) == 0; }
bool known_format(int f) { return f == IVFTQ_KV_F16 || f == IVFTQ_KV_BF16 || f == IVFTQ_KV_CODE4; }

constexpr int kMaxHeads = 1024, kMaxColumns = 1 << 20, kMaxBatch = 1 << 20;

ivftq_status check_cache(const ivftq_kv_cache* c) {
    if (!c) return refuse(IVFTQ_INVALID_ARG, "cache is NULL");
    if (!known_format(c->format)) return refuse(IVFTQ_INVALID_ARG, "unknown cache format %d", c->format);
    if (!known_d(c->d)) return refuse(IVFTQ_UNSUPPORTED, "d = %d: a cache's heads have 64, 96, 128, 192 or 256 coordinates", c->d);
    if (!known_page(c->page)) return refuse(IVFTQ_UNSUPPORTED, "page = %d: a power of two from 16 to 1024", c->page);
    if (c->heads < 1 || c->heads > kMaxHeads) return refuse(IVFTQ_UNSUPPORTED, "heads = %d: 1 to %d", c->heads, kMaxHeads);
    if (c->pages < 1 || c->pages > INT32_MAX) return refuse(IVFTQ_INVALID_ARG, "pages = %lld", (long long)c->pages);
    if (c->batch < 0 || c->batch > kMaxBatch) return refuse(IVFTQ_INVALID_ARG, "batch = %d: 0 to %d", c->batch, kMaxBatch);
    if (c->columns < 1 || c->columns > kMaxColumns || c->table_stride < c->columns)
        return refuse(IVFTQ_INVALID_ARG, "table of %d columns (1 to %d) with stride %lld", c->columns, kMaxColumns, (long long)c->table_stride);
    if (!c->pool || !c->table || !c->lengths) return refuse(IVFTQ_INVALID_ARG, "pool, table or lengths is NULL");
    if (!aligned(c->pool, 16) || !aligned(c->table, 4) || !aligned(c->lengths, 4)) return refuse(IVFTQ_INVALID_ARG, "pool has to be 16-byte aligned");
    if (c->format == IVFTQ_KV_CODE4) {
        if (!c->rotation || !aligned(c->rotation, 16)) return refuse(IVFTQ_INVALID_ARG, "a cache of codes needs a rotation, 16-byte aligned");
        for (int i = 0; i < 8; ++i)
            if (!(c->levels[8 + i] > (i ? c->levels[7 + i] : 0.f)) || c->levels[7 - i] != -c->levels[8 + i] || !(c->levels[8 + i] < 1e4f))
                return refuse(IVFTQ_INVALID_ARG, "levels have to ascend and be symmetric about zero (level %d: %g)", 8 + i, (double)c->levels[8 + i]);
    }
    if (!c->asked != !c->granted || !aligned(c->asked, 4) || !aligned(c->granted, 4))
        return refuse(IVFTQ_INVALID_ARG, "asked and granted go together, 4-byte aligned");
    return IVFTQ_OK;
}

ivftq_status check_rows(const ivftq_kv_rows* r, const char* name, int heads, int d, const ivftq_kv_cache* c, bool starts) {
    if (!r || (!r->data && r->rows)) return refuse(IVFTQ_INVALID_ARG, "%s is NULL", name);
    if (r->type != IVFTQ_KV_F16 && r->type != IVFTQ_KV_BF16) return refuse(IVFTQ_INVALID_ARG, "%s: rows are float16 or bfloat16", name);
    if (c->format != IVFTQ_KV_CODE4 && r->type != c->format) return refuse(IVFTQ_INVALID_ARG, "%s: rows of a 16-bit cache have its type", name);
    if (r->heads != heads) return refuse(IVFTQ_INVALID_ARG, "%s has %d heads, not %d", name, r->heads, heads);
    if (r->rows < 0 || r->rows > INT32_MAX / 2 || r->rows * r->heads > INT32_MAX) return refuse(IVFTQ_INVALID_ARG, "%s: %lld rows", name, (long long)r->rows);
    if (!starts && r->rows != c->batch) return refuse(IVFTQ_INVALID_ARG, "%s: %lld rows for %d sequences without starts", name, (long long)r->rows, c->batch);
    if (r->row_stride % 8 || r->head_stride % 8 || r->row_stride < 0 || r->head_stride < (r->heads > 1 ? d : 0))
        return refuse(IVFTQ_INVALID_ARG, "%s: strides of %lld and %lld elements (multiples of 8, heads apart)", name, (long long)r->row_stride, (long long)r->head_stride);
    if (!aligned(r->data, 16)) return refuse(IVFTQ_INVALID_ARG, "%s has to be 16-byte aligned", name);
    return IVFTQ_OK;
}

ivftq_status check_workgroups(const ivftq_kv_cache& c, const KvWork& w) {
    if ((int64_t)c.batch * c.heads * (w.few ? 1 : (int64_t)w.row_tiles) <= INT32_MAX) return IVFTQ_OK;
    return refuse(IVFTQ_UNSUPPORTED, "more than 2^31 workgroups: %d sequences of %d heads and up to %d row tiles", c.batch, c.heads, w.row_tiles);
}

// The magnitudes' float16 table.  A table's common scale is free (scores and results are multiplied by it in float32), and the
// rounding of eight numbers to float16 depends on it: of 128 scales in [1, 2) the one that leaves the smallest mean square,
// levels weighted by how often a coordinate of variance 1 / d meets them and what a common factor mends left out, 4e-5 to 8e-5
// of a row where a scale taken blindly leaves 2e-4 (the rounding of a float16 result itself is 2.1e-4).  About a microsecond.
void level_table(KvView& v, int d) {
    constexpr int kScales = 128;
    float square[kScales] = {}, along[kScales] = {}, weight[8], energy = 0.f;
    for (int i = 0; i < 8; ++i) {
        int e;
        const float mantissa = ldexpf(frexpf(v.level[i], &e), 11), ulp = ldexpf(1.f, e - 11);          // [1024, 2048)
        const float low = i ? v.bound[i - 1] : 0.f, high = i < 7 ? v.bound[i] : 2.f * v.level[7] - v.bound[6];
        const float w = expf(-0.5f * v.level[i] * v.level[i] * (float)d) * (high - low);
        weight[i] = w;
        energy += w * v.level[i] * v.level[i];
        for (int k = 0; k < kScales; ++k) {
            const float x = mantissa * (1.f + (float)k * (1.f / kScales)), down = x >= 2048.f ? 0.5f : 1.f, up = x >= 2048.f ? 2.f : 1.f;
            const float y = x * down, off = (y - ((y + 12582912.f) - 12582912.f)) * (ulp * up);         // 1.5 * 2^23: to the next whole number
            square[k] += w * off * off;
            along[k] += w * off * v.level[i];
        }
    }
    float best = 1e30f, scale = 1.f;
    for (int k = 0; k < kScales; ++k) {
        const float s = 1.f + (float)k * (1.f / kScales), left = (square[k] - along[k] * along[k] / energy) / (s * s);
        if (left < best) { best = left; scale = s; }
    }
    double dot = 0, sum = 0;
    for (int i = 0; i < 8; ++i) {
        const _Float16 h = (_Float16)(v.level[i] * scale);
        uint16_t bits;
        memcpy(&bits, &h, 2);
        v.tab_lo[i / 4] |= (uint32_t)(bits & 0xff) << 8 * (i % 4);
        v.tab_hi[i / 4] |= (uint32_t)(bits >> 8) << 8 * (i % 4);
        dot += (double)weight[i] * (double)v.level[i] * (double)(float)h;
        sum += (double)weight[i] * (double)(float)h * (double)(float)h;
    }
    v.level_unit = sum > 0 ? (float)(dot / sum) : 1.f / scale;
}

// attends: the table of magnitudes is needed (rows are written and read with the levels themselves)
KvView view_of(const ivftq_kv_cache& c, const int32_t* starts, int64_t rows, bool attends) {
    KvView v{};
    v.pool = static_cast<char*>(c.pool);
    v.table = c.table;
    v.lengths = c.lengths;
    v.starts = starts;
    v.rotation = c.rotation;
    v.pages = c.pages;
    v.table_stride = c.table_stride;
    v.head_bytes = kv_head_bytes(c.format, c.page, c.d);
    v.page_bytes = v.head_bytes * c.heads;
    v.batch = c.batch;
    v.columns = c.columns;
    v.page = c.page;
    v.page_log2 = __builtin_ctz((unsigned)c.page);
    v.heads = c.heads;
    v.rows = (int32_t)rows;
    if (c.format == IVFTQ_KV_CODE4) {
        for (int i = 0; i < 8; ++i) {
            v.level[i] = c.levels[8 + i];
            if (i) v.bound[i - 1] = (float)(((double)c.levels[7 + i] + c.levels[8 + i]) / 2);
        }
        if (attends) level_table(v, c.d);
    }
    return v;
}

KvRows rows_of(const ivftq_kv_rows& r) {
    return KvRows{static_cast<char*>(r.data), r.row_stride, r.head_stride, (int32_t)r.rows, r.heads, r.type};
}

ivftq_status move_rows(const ivftq_kv_cache* cache, const ivftq_kv_rows* k, const ivftq_kv_rows* v, const int32_t* starts, void* stream, bool read) {
    if (ivftq_status e = check_cache(cache)) return e;
    if (ivftq_status e = check_rows(k, read ? "k_out" : "k", cache->heads, cache->d, cache, starts)) return e;
    if (ivftq_status e = check_rows(v, read ? "v_out" : "v", cache->heads, cache->d, cache, starts)) return e;
    if (k->rows != v->rows || k->type != v->type) return refuse(IVFTQ_INVALID_ARG, "keys and values have one number of rows and one type");
    if (!starts && k->rows * cache->heads > INT32_MAX / (cache->d / 8)) return refuse(IVFTQ_UNSUPPORTED, "%lld rows of %d heads in one call", (long long)k->rows, cache->heads);
    if (!k->rows || !cache->batch) return IVFTQ_OK;
    KvView c = view_of(*cache, starts, k->rows, false);
    if (!read) { c.asked = cache->asked; c.granted = cache->granted; }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = read ? launch_kv_read(c, rows_of(*k), rows_of(*v), cache->d, cache->format, st) : launch_kv_append(c, rows_of(*k), rows_of(*v), cache->d, cache->format, st);
    return done(e, read ? "ivftq_kv_read" : "ivftq_kv_append");
}

// Queries of a call on chosen pages, or of scores.
ivftq_status check_queries(const ivftq_kv_cache* c, const ivftq_kv_rows* q, const int32_t* starts, int32_t max_new) {
    if (ivftq_status e = check_cache(c)) return e;
    if (!q) return refuse(IVFTQ_INVALID_ARG, "q is NULL");
    if (q->heads < 1 || q->heads % c->heads) return refuse(IVFTQ_INVALID_ARG, "%d query heads over %d key-value heads", q->heads, c->heads);
    if (ivftq_status e = check_rows(q, "q", q->heads, c->d, c, starts)) return e;
    if (max_new < 1) return refuse(IVFTQ_INVALID_ARG, "max_new = %d", max_new);
    return IVFTQ_OK;
}
bool known_sizes(const ivftq_kv_cache* c, int64_t rows, int32_t q_heads) {
    if (rows >= 0 && rows <= INT32_MAX / 2 && q_heads >= 1 && q_heads % c->heads == 0 && rows * q_heads <= INT32_MAX) return true;
    refuse(IVFTQ_INVALID_ARG, "%lld rows of %d query heads over %d", (long long)rows, q_heads, c->heads);
    return false;
}
KvAttend attend_of(const ivftq_kv_cache& c, const ivftq_kv_rows& q, const int32_t* starts, int32_t max_new, void* workspace) {
    KvAttend a{};
    a.c = view_of(c, starts, q.rows, true);
    a.q = rows_of(q);
    a.group = q.heads / c.heads;
    a.max_new = !starts ? 1 : (max_new < q.rows ? max_new : (int32_t)q.rows);
    a.work = static_cast<char*>(workspace);
    return a;
}
ivftq_status check_work(const void* workspace, int64_t bytes, int64_t need) {
    if (!need || (workspace && bytes >= need && aligned(workspace, 256))) return IVFTQ_OK;
    return refuse(IVFTQ_INVALID_ARG, "workspace of %lld bytes where %lld are needed, 256-byte aligned", (long long)bytes, (long long)need);
}

ivftq_status check_pages(const ivftq_kv_pages* s, bool lengths = true) {
    if (!s) return refuse(IVFTQ_INVALID_ARG, "state is NULL");
    if (!known_page(s->page)) return refuse(IVFTQ_UNSUPPORTED, "page = %d: a power of two from 16 to 1024", s->page);
    if (s->pages < 1 || s->pages > INT32_MAX) return refuse(IVFTQ_INVALID_ARG, "pages = %lld", (long long)s->pages);
    if (s->rows < 0 || s->rows > kMaxBatch || s->columns < 1 || s->columns > kMaxColumns || s->table_stride < s->columns || (int64_t)s->columns * s->page > INT32_MAX)
        return refuse(IVFTQ_INVALID_ARG, "table of %d rows and %d columns with stride %lld", s->rows, s->columns, (long long)s->table_stride);
    if (!s->table || (lengths && !s->lengths) || !s->refs) return refuse(IVFTQ_INVALID_ARG, "table, lengths or refs is NULL");
    return IVFTQ_OK;
}
ivftq_status check_pools(const ivftq_kv_pools* p) {
    if (!p) return refuse(IVFTQ_INVALID_ARG, "pools is NULL");
    if (p->layers < 1 || p->pages < 1 || p->pages > INT32_MAX || p->page_bytes < 16 || p->page_bytes % 16 || p->layer_stride % 16 || !p->pool || !aligned(p->pool, 16) ||
        (p->layers > 1 && p->layer_stride < p->pages * p->page_bytes))
        return refuse(IVFTQ_INVALID_ARG, "pools: %d layers, %lld bytes apart, of %lld records of %lld bytes (multiples of 16)", p->layers, (long long)p->layer_stride,
                      (long long)p->pages, (long long)p->page_bytes);
    return IVFTQ_OK;
}

ivftq_status check_groups(const ivftq_kv_pages& state, const ivftq_kv_pools* p, int32_t groups) {
    if (groups < 1 || groups > 8) return refuse(IVFTQ_INVALID_ARG, "groups = %d: 1 to 8", groups);
    if (!p) return refuse(IVFTQ_INVALID_ARG, "pools is NULL");
    for (int i = 0; i < groups; ++i) {
        if (ivftq_status e = check_pools(p + i)) return e;
        if (p[i].pages != state.pages) return refuse(IVFTQ_INVALID_ARG, "pools of %lld pages, counts of %lld", (long long)p[i].pages, (long long)state.pages);
    }
    return IVFTQ_OK;
}

}  // namespace

extern "C" {

int64_t ivftq_kv_page_bytes(int format, int page, int heads, int d) {
    if (!known_format(format) || !known_page(page) || !known_d(d) || heads < 1 || heads > kMaxHeads) return 0;
    return kv_head_bytes(format, page, d) * heads;
}

ivftq_status ivftq_kv_append(const ivftq_kv_cache* cache, const ivftq_kv_rows* k, const ivftq_kv_rows* v, const int32_t* starts, void* stream) {
    return move_rows(cache, k, v, starts, stream, false);
}
ivftq_status ivftq_kv_read(const ivftq_kv_cache* cache, const ivftq_kv_rows* k_out, const ivftq_kv_rows* v_out, const int32_t* starts, void* stream) {
    return move_rows(cache, k_out, v_out, starts, stream, true);
}

int64_t ivftq_kv_attend_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new) {
    if (check_cache(cache)) return -1;
    if (rows < 0 || rows > INT32_MAX / 2 || q_heads < 1 || q_heads % cache->heads || max_new < 1 || rows * q_heads > INT32_MAX) {
        refuse(IVFTQ_INVALID_ARG, "%lld rows of %d query heads over %d, at most %d new ones", (long long)rows, q_heads, cache->heads, max_new);
        return -1;
    }
    if (max_new > rows) max_new = rows > 1 ? (int32_t)rows : 1;
    const KvWork w = kv_work(cache->format, cache->d, cache->batch, cache->heads, rows, q_heads, max_new, (int64_t)cache->columns * cache->page);
    return check_workgroups(*cache, w) ? -1 : w.bytes;
}

ivftq_status ivftq_kv_attend(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const ivftq_kv_rows* out, float* lse, const int32_t* starts,
                             int32_t max_new, int32_t window, int32_t sinks, float scale, void* workspace, int64_t workspace_bytes, void* stream) {
    if (ivftq_status e = check_cache(cache)) return e;
    if (!q || !out) return refuse(IVFTQ_INVALID_ARG, "q or out is NULL");
    if (q->heads < 1 || q->heads % cache->heads) return refuse(IVFTQ_INVALID_ARG, "%d query heads over %d key-value heads", q->heads, cache->heads);
    if (ivftq_status e = check_rows(q, "q", q->heads, cache->d, cache, starts)) return e;
    if (ivftq_status e = check_rows(out, "out", q->heads, cache->d, cache, starts)) return e;
    if (q->rows != out->rows || q->type != out->type) return refuse(IVFTQ_INVALID_ARG, "out has the rows and the type of q");
    if (max_new < 1 || window < 0 || sinks < 0) return refuse(IVFTQ_INVALID_ARG, "max_new = %d, window = %d, sinks = %d", max_new, window, sinks);
    if (!std::isfinite(scale)) return refuse(IVFTQ_INVALID_ARG, "scale is no number");
    if (!q->rows || !cache->batch) return IVFTQ_OK;
    if (!starts) max_new = 1;
    if (max_new > q->rows) max_new = (int32_t)q->rows;
    const KvWork w = kv_work(cache->format, cache->d, cache->batch, cache->heads, q->rows, q->heads, max_new, (int64_t)cache->columns * cache->page);
    if (ivftq_status e = check_workgroups(*cache, w)) return e;
    if (cache->format != IVFTQ_KV_CODE4 && q->data == out->data) return refuse(IVFTQ_INVALID_ARG, "out stands where q does: only a cache of codes allows that");
    if (w.bytes && (!workspace || workspace_bytes < w.bytes || !aligned(workspace, 256)))
        return refuse(IVFTQ_INVALID_ARG, "workspace of %lld bytes where %lld are needed, 256-byte aligned", (long long)workspace_bytes, (long long)w.bytes);
    KvAttend a{};
    a.c = view_of(*cache, starts, q->rows, true);
    a.q = rows_of(*q);
    a.out = rows_of(*out);
    a.lse = lse;
    a.group = q->heads / cache->heads;
    a.max_new = max_new;
    a.window = window;
    a.sinks = sinks;
    a.scale = scale;
    a.work = static_cast<char*>(workspace);
    return done(launch_kv_attend(a, w, cache->d, cache->format, static_cast<hipStream_t>(stream)), "ivftq_kv_attend");
}

ivftq_status ivftq_kv_digest(const ivftq_kv_cache* cache, void* digests, const int32_t* starts, void* stream) {
    if (ivftq_status e = check_cache(cache)) return e;
    if (!digests || !aligned(digests, 16)) return refuse(IVFTQ_INVALID_ARG, "digests is NULL or not 16-byte aligned");
    if (!cache->batch) return IVFTQ_OK;
    // the number of rows is not asked for: with starts it is what the last of them says
    KvView c = view_of(*cache, starts, starts ? INT32_MAX : cache->batch, false);
    c.asked = cache->asked;
    c.granted = cache->granted;
    return done(launch_kv_digest(c, digests, cache->d, cache->format, static_cast<hipStream_t>(stream)), "ivftq_kv_digest");
}

int64_t ivftq_kv_score_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new) {
    if (check_cache(cache) || !known_sizes(cache, rows, q_heads)) return -1;
    if (max_new < 1) {
        refuse(IVFTQ_INVALID_ARG, "max_new = %d", max_new);
        return -1;
    }
    return score_work(cache->format, cache->d, rows, q_heads, cache->heads, max_new == 1 || rows <= 1).bytes;
}
ivftq_status ivftq_kv_score(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const void* digests, float* scores, const int32_t* starts, int32_t max_new,
                            void* workspace, int64_t workspace_bytes, void* stream) {
    if (ivftq_status e = check_queries(cache, q, starts, max_new)) return e;
    if (!digests || !aligned(digests, 16)) return refuse(IVFTQ_INVALID_ARG, "digests is NULL or not 16-byte aligned");
    if (!q->rows || !cache->batch) return IVFTQ_OK;
    if (!scores || !aligned(scores, 4)) return refuse(IVFTQ_INVALID_ARG, "scores is NULL or not 4-byte aligned");
    const KvAttend a = attend_of(*cache, *q, starts, max_new, workspace);
    if ((int64_t)cache->batch * cache->heads * ((a.max_new + 15) / 16 + 1) > INT32_MAX)
        return refuse(IVFTQ_UNSUPPORTED, "more than 2^31 workgroups: %d sequences of %d heads and up to %d rows", cache->batch, cache->heads, a.max_new);
    if (ivftq_status e = check_work(workspace, workspace_bytes, score_work(cache->format, cache->d, q->rows, q->heads, cache->heads, a.max_new == 1).bytes)) return e;
    return done(launch_kv_score(a, digests, scores, cache->d, cache->format, static_cast<hipStream_t>(stream)), "ivftq_kv_score");
}

ivftq_status ivftq_kv_select(const float* scores, const int32_t* lengths, const int32_t* starts, int64_t rows, int32_t batch, int32_t heads, int32_t columns,
                             int32_t page, int32_t count, int32_t first, int32_t last, int32_t* chosen, void* stream) {
    if (!known_page(page)) return refuse(IVFTQ_UNSUPPORTED, "page = %d: a power of two from 16 to 1024", page);
    if (heads < 1 || heads > kMaxHeads) return refuse(IVFTQ_UNSUPPORTED, "heads = %d: 1 to %d", heads, kMaxHeads);
    if (batch < 0 || batch > kMaxBatch || columns < 1 || columns > kMaxColumns) return refuse(IVFTQ_INVALID_ARG, "%d sequences of %d columns", batch, columns);
    if (rows < 0 || rows * heads > INT32_MAX) return refuse(IVFTQ_INVALID_ARG, "%lld rows of %d heads", (long long)rows, heads);
    if (!starts && rows != batch) return refuse(IVFTQ_INVALID_ARG, "%lld rows for %d sequences without starts", (long long)rows, batch);
    if (count < 1 || count > kMostPicks) return refuse(IVFTQ_UNSUPPORTED, "count = %d: 1 to %d", count, kMostPicks);
    if (first < 0 || last < 0 || (int64_t)first + last > count) return refuse(IVFTQ_INVALID_ARG, "first = %d and last = %d of %d", first, last, count);
    if (!rows) return IVFTQ_OK;
    if (!scores || !chosen || (batch && !lengths)) return refuse(IVFTQ_INVALID_ARG, "scores, lengths or chosen is NULL");
    if (!aligned(scores, 4) || !aligned(chosen, 4) || !aligned(lengths, 4)) return refuse(IVFTQ_INVALID_ARG, "scores, lengths and chosen are 4-byte aligned");
    KvSelect s{scores, chosen, {}, count, first, last};
    s.c.lengths = lengths;
    s.c.starts = starts;
    s.c.batch = batch;
    s.c.columns = columns;
    s.c.page = page;
    s.c.page_log2 = __builtin_ctz((unsigned)page);
    s.c.heads = heads;
    s.c.rows = (int32_t)rows;
    return done(launch_kv_select(s, static_cast<hipStream_t>(stream)), "ivftq_kv_select");
}

int64_t ivftq_kv_attend_pages_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new, int32_t count) {
    if (check_cache(cache) || !known_sizes(cache, rows, q_heads)) return -1;
    if (max_new < 1 || count < 1 || count > kMostPicks) {
        refuse(IVFTQ_INVALID_ARG, "max_new = %d, count = %d: 1 to %d", max_new, count, kMostPicks);
        return -1;
    }
    return pick_work(*cache, rows, q_heads, max_new < rows ? max_new : (rows > 1 ? (int32_t)rows : 1), count).bytes;
}
ivftq_status ivftq_kv_attend_pages(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const ivftq_kv_rows* out, float* lse, const int32_t* starts,
                                   int32_t max_new, const int32_t* chosen, int32_t count, float scale, void* workspace, int64_t workspace_bytes, void* stream) {
    if (ivftq_status e = check_queries(cache, q, starts, max_new)) return e;
    if (!out) return refuse(IVFTQ_INVALID_ARG, "out is NULL");
    if (ivftq_status e = check_rows(out, "out", q->heads, cache->d, cache, starts)) return e;
    if (q->rows != out->rows || q->type != out->type) return refuse(IVFTQ_INVALID_ARG, "out has the rows and the type of q");
    if (count < 1 || count > kMostPicks) return refuse(IVFTQ_UNSUPPORTED, "count = %d: 1 to %d", count, kMostPicks);
    if (!std::isfinite(scale)) return refuse(IVFTQ_INVALID_ARG, "scale is no number");
    if (!q->rows || !cache->batch) return IVFTQ_OK;
    if (!chosen || !aligned(chosen, 4)) return refuse(IVFTQ_INVALID_ARG, "chosen is NULL or not 4-byte aligned");
    if (cache->format != IVFTQ_KV_CODE4 && q->data == out->data) return refuse(IVFTQ_INVALID_ARG, "out stands where q does: only a cache of codes allows that");
    KvAttend a = attend_of(*cache, *q, starts, max_new, workspace);
    const PickWork w = pick_work(*cache, q->rows, q->heads, a.max_new, count);
    if (ivftq_status e = check_work(workspace, workspace_bytes, w.bytes)) return e;
    a.out = rows_of(*out);
    a.lse = lse;
    a.scale = scale;
    return done(launch_kv_picked(a, w, chosen, count, cache->d, cache->format, static_cast<hipStream_t>(stream)), "ivftq_kv_attend_pages");
}

ivftq_status ivftq_kv_reserve(const ivftq_kv_pages* state, const int32_t* counts, int32_t* granted, int32_t* scratch, void* stream) {
    if (ivftq_status e = check_pages(state)) return e;
    if (!counts || !granted || !scratch) return refuse(IVFTQ_INVALID_ARG, "counts, granted or scratch is NULL");
    if (!state->rows) return IVFTQ_OK;
    return done(launch_kv_reserve(*state, counts, granted, scratch, static_cast<hipStream_t>(stream)), "ivftq_kv_reserve");
}
ivftq_status ivftq_kv_fork_pools(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t groups, const int32_t* parents, const int32_t* children,
                                 int32_t n, int32_t* done_out, int32_t* scratch, void* stream) {
    if (ivftq_status e = check_pages(state)) return e;
    if (ivftq_status e = check_groups(*state, pools, groups)) return e;
    if (n < 0 || n > 65536) return refuse(IVFTQ_INVALID_ARG, "n = %d: 0 to 65536", n);
    if (!n) return IVFTQ_OK;
    if (!parents || !children || !done_out || !scratch) return refuse(IVFTQ_INVALID_ARG, "parents, children, done or scratch is NULL");
    return done(launch_kv_fork(*state, pools, groups, parents, children, n, done_out, scratch, static_cast<hipStream_t>(stream)), "ivftq_kv_fork");
}
ivftq_status ivftq_kv_fork(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, const int32_t* parents, const int32_t* children, int32_t n,
                           int32_t* done_out, int32_t* scratch, void* stream) {
    return ivftq_kv_fork_pools(state, pools, 1, parents, children, n, done_out, scratch, stream);
}
ivftq_status ivftq_kv_free(const ivftq_kv_pages* state, const int32_t* rows, int32_t n, void* stream) {
    if (ivftq_status e = check_pages(state)) return e;
    if (n < 0 || (n && !rows)) return refuse(IVFTQ_INVALID_ARG, "n = %d rows", n);
    return done(launch_kv_free(*state, rows, n, static_cast<hipStream_t>(stream)), "ivftq_kv_free");
}
ivftq_status ivftq_kv_trim(const ivftq_kv_pages* state, int32_t window, int32_t sinks, void* stream) {
    if (ivftq_status e = check_pages(state)) return e;
    if (window < 1 || sinks < 0) return refuse(IVFTQ_INVALID_ARG, "window = %d, sinks = %d", window, sinks);
    return done(launch_kv_trim(*state, window, sinks, static_cast<hipStream_t>(stream)), "ivftq_kv_trim");
}
ivftq_status ivftq_kv_compact_pools(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t groups, int32_t* used_out, int32_t* scratch, void* stream) {
    if (ivftq_status e = check_pages(state, false)) return e;
    if (ivftq_status e = check_groups(*state, pools, groups)) return e;
    if (!used_out || !scratch) return refuse(IVFTQ_INVALID_ARG, "used_out or scratch is NULL");
    return done(launch_kv_compact(*state, pools, groups, used_out, scratch, static_cast<hipStream_t>(stream)), "ivftq_kv_compact");
}
ivftq_status ivftq_kv_compact(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t* used_out, int32_t* scratch, void* stream) {
    return ivftq_kv_compact_pools(state, pools, 1, used_out, scratch, stream);
}
ivftq_status ivftq_kv_copy(const ivftq_kv_pools* pools, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
    if (ivftq_status e = check_pools(pools)) return e;
    if (n < 0 || (n && (!src || !dst))) return refuse(IVFTQ_INVALID_ARG, "n = %d pairs", n);
    return done(launch_kv_copy(*pools, src, dst, nullptr, n, static_cast<hipStream_t>(stream)), "ivftq_kv_copy");
}

}  // extern "C"
