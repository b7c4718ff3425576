// Scores of pages by their digests, and attention over chosen pages.
//
// A score is linear in two sums over the group's heads, those of the queries' negative coordinates (which meet the lowest values) and of the
// others (the highest): sides[2][D].  One new row a sequence: sums and products in float32, a digest's sixteen-byte pieces over
// the lanes, bound by the digests' bytes.  Several: the sides are made once, in two (bfloat16: three) 16-bit parts, and meet the
// digests in v_mfma 16x16x32, 16 new rows x 16 pages.
//
// Attention: every new row has pages of its own for each key-value head.  A unit is what kv_few.h calls a sequence: as many neighbouring rows
// as their heads fill the sixteen columns of a product, and the pages that any of them has chosen (neighbours choose much alike).  A
// workgroup's wavefronts take every fourth tile of 32 tokens of those; a row that has not chosen a page has it masked.  Where the units are few
// several workgroups share a unit's tiles, and a second kernel joins their parts.
//
// Measured (kernels traced, medians): scores of four new rows over 42,000 (head, page) pairs of 128 coordinates in bfloat16 10.7 us (least 7.8) for 22 MB of
// digests, over codes 12.6 behind a rotation of 6.1; of 794 rows over up to 641 pages of codes 39 us (passes among others 36.6), 19 of them the products.
// Attention of 32 rows, 8 heads, over 64 pages of 64 tokens each in bfloat16: 96 us for 537 MB (5.6 TB/s); of 794 rows over 16 pages each: 104 us, and 93
// where passes follow one another, 1.9 GB from the L2 (20 TB/s).
#pragma once
#include "kv_many.h"
#include "wave_ops.h"

namespace ivftq {

struct ScoreArgs {
    KvAttend a;                       // c, q, group, max_new
    const uint16_t* digests;
    float* scores;
    const uint16_t* z;                // codes: rotated unit queries, two float16 parts, eights in the order of kv_levels8
    const float* zn;                  // codes: the queries' norms
    uint16_t* sides;                  // [heads][tiles][parts][2 D / 32][64 lanes][8]: operands as they are read
    float* unit;                      // [heads][tiles][16] what the parts are multiplied by
    int32_t tiles;                    // tiles of 16 rows: those of row r in tile r / 16, whatever sequence it is of
    int32_t row_tiles, each;          // tiles that a sequence's rows may lie in, and a workgroup's
};
template <int F> constexpr int kSideParts = F == IVFTQ_KV_BF16 ? 3 : 2;

// Eight values from the order of kv_levels8 into their own.
__device__ __forceinline__ uintx4 kv_in_order(uintx4 w) {
    return uintx4{__builtin_amdgcn_perm(w[2], w[0], 0x05040100u), __builtin_amdgcn_perm(w[2], w[0], 0x07060302u),
                  __builtin_amdgcn_perm(w[3], w[1], 0x05040100u), __builtin_amdgcn_perm(w[3], w[1], 0x07060302u)};
}

// Digests whose ends are not all finite.  A coordinate that is no number in every key has an empty interval, +infinity to -infinity, and counts for
// nothing: it is read as 0 to 0.  One end alone tells: a lowest value of +infinity, or a highest one of -infinity, stands otherwise only where every key has
// that infinity, and then the other end keeps it.  What is left of infinities makes a sum infinite or, times a query's zero or a part that is zero, no number.
template <bool BF>
__device__ __forceinline__ uintx4 kv_interval(uintx4 w, bool high) {
    const uint32_t none = (BF ? 0x7f80u : 0x7c00u) | (high ? 0x8000u : 0u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t a = w[e] & 0xffffu, b = w[e] >> 16;
        w[e] = (a == none ? 0u : a) | (b == none ? 0u : b) << 16;
    }
    return w;
}
// Nothing bounds the products of such a page: no number stands for the largest score, in one row's kernel as in that of several.
__device__ __forceinline__ float kv_score_of(float sum) { return sum == sum ? sum : INFINITY; }

// A query's coordinate that is no finite number counts for nothing: it would leave a row without scores to choose by (codes: the rotation makes all of the
// query's coordinates none).
__device__ __forceinline__ float kv_finite(float v) { return __builtin_fabsf(v) < INFINITY ? v : 0.f; }

// Eight coordinates from j on of the sides of a row and head: sums of the negative ones, and of the others.
template <int F, int D>
__device__ __forceinline__ void score_sides(const ScoreArgs& f, int64_t row, int h, int j, float (&low)[8], float (&high)[8]) {
    const KvAttend& a = f.a;
#pragma unroll
    for (int e = 0; e < 8; ++e) low[e] = high[e] = 0.f;
    auto add = [&](int e, float v) __attribute__((always_inline)) { v = kv_finite(v); low[e] += fminf(v, 0.f); high[e] += fmaxf(v, 0.f); };
#pragma unroll 4
    for (int i = 0; i < a.group; ++i) {
        const int64_t head = (int64_t)h * a.group + i;
        if constexpr (F == IVFTQ_KV_CODE4) {
            const int64_t at = row * a.q.heads + head, all = (int64_t)a.q.rows * a.q.heads;
            const halfx8 u = __builtin_bit_cast(halfx8, kv_in_order(*reinterpret_cast<const uintx4*>(f.z + at * D + j)));
            const halfx8 v = __builtin_bit_cast(halfx8, kv_in_order(*reinterpret_cast<const uintx4*>(f.z + (all + at) * D + j)));
            const float norm = f.zn[at] * (1.f / kSplitScale);
#pragma unroll
            for (int e = 0; e < 8; ++e) add(e, ((float)u[e] + (float)v[e]) * norm);
        } else {
            const uintx4 w = *reinterpret_cast<const uintx4*>(reinterpret_cast<const uint16_t*>(a.q.data) + row * a.q.row_stride + head * a.q.head_stride + j);
#pragma unroll
            for (int e = 0; e < 8; ++e) add(e, kv_to_float<F == IVFTQ_KV_BF16>(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffff));
        }
    }
}

// One new row a sequence.  A page's digest lies over kLanes lanes (a sixteen-byte piece each; 96 and 192 coordinates leave a quarter of them
// idle), a wavefront's load has kPages of them, 16 loads are on their way at once.
template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_score_one(ScoreArgs f) {
    constexpr int kPieces = D / 4, kLanes = kPieces <= 16 ? 16 : (kPieces <= 32 ? 32 : 64), kPages = 64 / kLanes, kLoads = 32 / kPages < 16 ? 32 / kPages : 16;
    constexpr int kAll = kPages * kLoads;                                 // pages of a wavefront
    constexpr bool bf = F == IVFTQ_KV_BF16;
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, piece = lane % kLanes, sub = lane / kLanes;
    const int64_t wg = kv_workgroup();
    const int h = (int)(wg % c.heads);
    const int64_t row = wg / c.heads;
    const int col0 = ((int)blockIdx.y * 4 + wave) * kAll;
    if (row >= c.rows || col0 >= c.columns) return;
    int first, count;
    const int b = kv_uniform(kv_sequence(c, row, first, count));
    if (b < 0 || row - first >= a.max_new) return;
    const int pos = kv_length(c, b) - count + (int)(row - first), reach = pos >> c.page_log2;      // a position under zero reaches column -1
    const int mine = col0 + lane;                                          // the column that this lane writes
    const int32_t id = lane < kAll && mine < c.columns && mine <= reach ? c.table[(int64_t)b * c.table_stride + mine] : -1;
    const bool there = (uint32_t)id < (uint32_t)c.pages;
    const int32_t page = there ? id : 0;
    float score = 0.f;
    if (col0 <= reach) {
        const uint16_t* box = f.digests + (int64_t)h * (2 * D) + (piece < kPieces ? piece : 0) * 8;
        uintx4 w[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w[i] = *reinterpret_cast<const uintx4*>(box + (int64_t)__shfl(page, i * kPages + sub) * c.heads * (2 * D));
        float low[8], high[8], side[8];
        const int j = piece < kPieces ? piece * 8 % D : 0;
        score_sides<F, D>(f, row, h, j, low, high);
#pragma unroll
        for (int e = 0; e < 8; ++e) side[e] = piece * 8 < D ? low[e] : (piece < kPieces ? high[e] : 0.f);
        auto add_up = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                float v = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) v = __builtin_fmaf(kv_to_float<bf>(e & 1 ? w[i][e >> 1] >> 16 : w[i][e >> 1] & 0xffff), side[e], v);
                if (kLanes > kPieces) v = piece < kPieces ? v : 0.f;
                v = lanes8(v, Sum());
                v += lane_moved<0x140>(v);
                if (kLanes >= 32) v = lane_pair<false>(v, Sum());
                if (kLanes == 64) v = lane_pair<true>(v, Sum());
                // the lanes that write the pages of this load
#pragma unroll
                for (int u = 0; u < kPages; ++u) {
                    const float of = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), u * kLanes));
                    score = lane == i * kPages + u ? of : score;
                }
            }
        };
        add_up();
        if (__ballot(there && !(__builtin_fabsf(score) < INFINITY))) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) w[i] = kv_interval<bf>(w[i], piece * 8 >= D);
            add_up();
        }
    }
    if (lane < kAll && mine < c.columns) f.scores[(row * c.heads + h) * c.columns + mine] = there ? kv_score_of(score) : -INFINITY;
}

// Sides of several rows: 32 lanes a (row, head) pair, of which D / 8 work.  (A row's operands one after the other, rows 8 KB apart,
// meet in one channel of the L2: the products took 36 us of a chunk's scores that way, 18 so.)
template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_sides(ScoreArgs f) {
    constexpr int kParts = kSideParts<F>;
    constexpr bool bf = F == IVFTQ_KV_BF16;
    const KvView& c = f.a.c;
    const int64_t pair = (int64_t)kv_workgroup() * 8 + threadIdx.x / 32, pairs = (int64_t)c.rows * c.heads;
    const int piece = threadIdx.x % 32, j = piece < D / 8 ? piece * 8 : 0;
    const int64_t used = pair < pairs ? pair : pairs - 1;
    float x[2][8], most = 0.f;
    score_sides<F, D>(f, used / c.heads, (int)(used % c.heads), j, x[0], x[1]);
    float by = 1.f;
    if constexpr (!bf) {                                      // float16: the largest value to 2^14, so that the second part keeps its bits
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(-x[0][e], x[1][e]));
        most = lanes8(most, Larger());
        most = fmaxf(most, lane_moved<0x140>(most));
        most = lane_pair<false>(most, Larger());
        const int e = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
        by = most > 0.f && most < INFINITY ? ldexpf(1.f, e < -100 ? 114 : 14 - e) : 1.f;
    }
    if (pair >= pairs || piece >= D / 8) return;
    const int row = (int)(pair / c.heads), h = (int)(pair % c.heads), i = row % 16;
    const int64_t tile = (int64_t)h * f.tiles + row / 16;
    if (piece == 0) f.unit[tile * 16 + i] = 1.f / by;
    uint16_t* to = f.sides + (tile * (kParts * 2 * D / 32) + j / 32) * 512 + (j % 32 / 8 * 16 + i) * 8;
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[side][e] *= by;
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            uintx4 w;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                w[e / 2] = kv_pack2<bf>(x[side][e], x[side][e + 1]);
                x[side][e] -= kv_to_float<bf>(w[e / 2] & 0xffff);
                x[side][e + 1] -= kv_to_float<bf>(w[e / 2] >> 16);
            }
            *reinterpret_cast<uintx4*>(to + (part * 2 + side) * (D / 32) * 512) = w;
        }
}

// Codes, where 16 rows of (row, query head) pairs are whole groups: sides made by the workgroup that rotates the queries, as k_kv_rotate_queries
// does it, which leaves nothing in between (25,000 pairs of 128: 20 us; in two kernels 17 and 9).
template <int D>
__global__ __launch_bounds__(D * 2) void k_kv_rotate_sides(ScoreArgs f, int tiles) {
    __shared__ UnitRows<D> unit;
    const KvRows& q = f.a.q;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, group = f.a.group;
    const int64_t all = (int64_t)q.rows * q.heads;
    const KvTurn<D, false> turn(f.a.c.rotation, wave);
    auto over_group = [&](float v) __attribute__((always_inline)) {              // the sum over the lanes of a group, in every one
        if (group > 1) v += lane_moved<0xb1>(v);
        if (group > 2) v += lane_moved<0x4e>(v);
        if (group > 4) v += lane_moved<0x141>(v);
        if (group > 8) v += lane_moved<0x140>(v);
        return v;
    };
    for (int64_t tile = (int64_t)blockIdx.x * tiles; tile < ((int64_t)blockIdx.x + 1) * tiles && tile * 16 < all; ++tile) {
        const int64_t i = tile * 16 + n;
        const bool in = i < all;
        const int64_t row = in ? i / q.heads : 0, head = in ? i % q.heads : 0;
        const uintx4 w = *reinterpret_cast<const uintx4*>(reinterpret_cast<const uint16_t*>(q.data) + row * q.row_stride + head * q.head_stride + 32 * wave + 8 * g);
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = w[e >> 1] >> 16 * (e & 1) & 0xffff;
            x[e] = q.type == IVFTQ_KV_BF16 ? kv_to_float<true>(bits) : kv_to_float<false>(bits);
        }
        const float norm = unit.bring(x);
        turn(unit, y);
        // no coordinate of the sums is larger than the norms' sum: that goes to 2^14
        const float most = over_group(kv_finite(norm));
        const int exponent = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
        const float by = most > 0.f && most < INFINITY ? ldexpf(1.f, exponent < -100 ? 113 : 13 - exponent) : 1.f;
        float low[8], high[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = kv_finite(y[e] * norm);
            low[e] = over_group(fminf(v, 0.f)) * by;
            high[e] = over_group(fmaxf(v, 0.f)) * by;
        }
        if (!in || n % group) continue;
        const int64_t place = (head / group) * f.tiles + row / 16;
        const int at = (int)(row % 16);
        if (wave == 0 && g == 0) f.unit[place * 16 + at] = 1.f / by;
        uint16_t* to = f.sides + (place * (2 * 2 * D / 32) + wave) * 512 + (g * 16 + at) * 8;
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                float(&v)[8] = side ? high : low;
                uintx4 u;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    u[e / 2] = kv_pack2<false>(v[e], v[e + 1]);
                    v[e] -= kv_to_float<false>(u[e / 2] & 0xffff);
                    v[e + 1] -= kv_to_float<false>(u[e / 2] >> 16);
                }
                *reinterpret_cast<uintx4*>(to + (part * 2 + side) * (D / 32) * 512) = u;
            }
    }
}

// Several new rows: a wavefront keeps the digests of its pages and walks the row tiles.
template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_score(ScoreArgs f) {
    constexpr int kSteps = 2 * D / 32, kTiles = D <= 128 ? 2 : 1, kParts = kSideParts<F>;
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const uint32_t wg = kv_workgroup(), groups = ((uint32_t)f.row_tiles + f.each - 1) / f.each;
    const int h = (int)(wg % (uint32_t)c.heads), rt0 = (int)(wg / (uint32_t)c.heads % groups) * f.each, b = (int)(wg / (uint32_t)c.heads / groups);
    if (b >= c.batch) return;
    int first, count;
    kv_new_rows(c, b, first, count);
    const int base = kv_length(c, b) - count - first;                      // a row's position: base + row
    if (count > a.max_new) count = a.max_new;
    const int end = first + count, tile0 = first / 16 + rt0, last = min(first / 16 + min(rt0 + f.each, f.row_tiles), (end + 15) / 16);
    if (!count || tile0 >= last) return;
    const int col0 = ((int)blockIdx.y * 4 + wave) * 16 * kTiles;
    if (col0 >= c.columns) return;
    uint32_t known[kTiles];
    int32_t id[kTiles];
    uintx4 box[kTiles][kSteps];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int col = col0 + 16 * t + n;                                 // this lane's page
        id[t] = c.table[(int64_t)b * c.table_stride + (col < c.columns ? col : 0)];
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const bool there = (uint32_t)id[t] < (uint32_t)c.pages && col0 + 16 * t + n < c.columns;
        known[t] = (uint32_t)__ballot(there) & 0xffffu;
        const uint16_t* p = f.digests + ((int64_t)(there ? id[t] : 0) * c.heads + h) * (2 * D) + 8 * g;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) box[t][k] = *reinterpret_cast<const uintx4*>(p + 32 * k);
    }
    // A tile's operands are asked for while the tile before is worked on, part by part (left alone the compiler asks for one ahead and waits).
    uintx4 w[kParts][kSteps];
    auto ask = [&](int part, int tile) __attribute__((always_inline)) {
        const uint16_t* p = f.sides + (((int64_t)h * f.tiles + tile) * kParts + part) * (kSteps * 512) + lane * 8;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) w[part][k] = *reinterpret_cast<const uintx4*>(p + 512 * k);
    };
#pragma unroll
    for (int part = 0; part < kParts; ++part) ask(part, tile0);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        if (__ballot(kv_any_not_finite<F == IVFTQ_KV_BF16>(box[t]))) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) box[t][k] = kv_interval<F == IVFTQ_KV_BF16>(box[t][k], k >= kSteps / 2);
        }
    for (int tile = tile0; tile < last; ++tile) {
        const int next = tile + 1 < last ? tile + 1 : tile;
        const float mine = f.unit[((int64_t)h * f.tiles + tile) * 16 + n];
        floatx4 acc[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) acc[t] = kv_mfma16<F>(w[part][k], box[t][k], acc[t]);
            __builtin_amdgcn_sched_barrier(0);
            ask(part, next);
            __builtin_amdgcn_sched_barrier(0);
        }
        // register r: row 4 g + r, page n: sixteen neighbouring scores a row
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * tile + 4 * g + r, reach = (base + row) >> c.page_log2;      // a position under zero reaches column -1
            const float unit = __shfl(mine, 4 * g + r);
            if (row < first || row >= end) continue;                       // of another sequence
            float* out = f.scores + ((int64_t)row * c.heads + h) * c.columns + col0 + n;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const int col = col0 + 16 * t + n;
                if (col < c.columns) out[16 * t] = col <= reach && (known[t] >> n & 1) ? kv_score_of(acc[t][r] * unit) : -INFINITY;
            }
        }
    }
}

// ---- attention ----------------------------------------------------------------------------------------------------

constexpr int kMostPicks = 4096;      // pages of a row and head

struct PickArgs {
    FewArgs f;                        // its KvAttend with max_new = tokens
    const int32_t* chosen;            // [rows][heads][count]
    int32_t count, max_new;
    int32_t tokens, units;            // new rows of a unit at most; units a head
    int32_t splits;                   // workgroups that share a unit's tiles
    int32_t list, words;              // several rows: places of the list, words of a row's bits
};

// What a workgroup works on: up to `tokens` neighbouring rows of a sequence, pos: the first one's position.
struct PickUnit { int b, row, count, pos; };
__device__ __forceinline__ PickUnit pick_unit(const PickArgs& p, int unit) {
    const KvView& c = p.f.a.c;
    int first, count;
    if (p.tokens == 1) {
        const int b = kv_sequence(c, unit, first, count);
        const bool none = b < 0 || unit - first >= p.max_new;
        return {none ? -1 : b, unit, 1, kv_length(c, b < 0 ? 0 : b) - count + unit - first};
    }
    int lo = 0, hi = c.batch;                        // units of sequence b: from starts[b] / tokens + b on, so that no two sequences' units meet
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1, s = kv_int(c.starts, mid);
        if ((s < 0 ? 0 : s) / p.tokens + mid <= unit) lo = mid; else hi = mid;
    }
    kv_new_rows(c, lo, first, count);
    const int base = kv_length(c, lo) - count, most = count < p.max_new ? count : p.max_new, at = (unit - first / p.tokens - lo) * p.tokens;
    return {at < 0 || at >= most ? -1 : lo, first + at, most - at < p.tokens ? most - at : p.tokens, base + at};
}

// A unit's pages in LDS, ascending: columns and page numbers, and which rows have chosen them.
struct Picked { int n, tiles; };
struct PickList { int2* page; uint16_t* by; uint32_t* bits; };
__device__ __forceinline__ PickList pick_lds(const PickArgs& p, int2* at) {
    uint16_t* by = reinterpret_cast<uint16_t*>(at + p.list);
    return {at, by, reinterpret_cast<uint32_t*>(by + ((p.list + 1) & ~1))};
}
// The entries of a row's list that count, 64 at a time, by a wavefront: f(column, whether the lane has one).
template <class Each>
__device__ __forceinline__ void pick_entries(const PickArgs& p, int64_t pair, int pos, Each&& f) {
    const KvView& c = p.f.a.c;
    const int lane = threadIdx.x & 63;
    uint32_t top = 0;                                // columns + 1: of the entries before these
    for (int i0 = 0; i0 < p.count; i0 += 64) {
        const int col = i0 + lane < p.count ? p.chosen[pair * p.count + i0 + lane] : -1;
        const uint32_t mine = col < 0 ? 0u : (uint32_t)col + 1, most = lanes_most_upto(mine);
        const uint32_t prev = __shfl_up(most, 1), before = lane && prev > top ? prev : top;
        f(col, mine > before && col < c.columns && (int64_t)col << c.page_log2 <= pos);
        const uint32_t last = (uint32_t)__builtin_amdgcn_readlane((int)most, 63);
        top = top > last ? top : last;
    }
}
__device__ __forceinline__ Picked pick_list(const PickArgs& p, const PickUnit& unit, int h, const PickList& list) {
    const KvView& c = p.f.a.c;
    __shared__ int many;
    const int lane = threadIdx.x & 63, wave = kv_wave();
    const int32_t* table = c.table + (int64_t)unit.b * c.table_stride;
    int n = 0;
    if (p.tokens == 1) {                             // one row: what names no page is left out too
        if (wave == 0) {
            pick_entries(p, (int64_t)unit.row * c.heads + h, unit.pos, [&](int col, bool in) __attribute__((always_inline)) {
                const int32_t id = in ? table[col] : -1;
                in = (uint32_t)id < (uint32_t)c.pages;
                const uint64_t all = __ballot(in);
                if (in) list.page[n + __popcll(all & ((1ull << lane) - 1))] = make_int2(col, id);
                n += __popcll(all);
            });
            if (lane == 0) many = n;
        }
        __syncthreads();
    } else {                                         // several: their columns as bits, put together
        for (int i = threadIdx.x; i < p.tokens * p.words; i += 256) list.bits[i] = 0;
        __syncthreads();
        for (int t = wave; t < unit.count; t += 4)
            pick_entries(p, (int64_t)(unit.row + t) * c.heads + h, unit.pos + t, [&](int col, bool in) __attribute__((always_inline)) {
                if (in) atomicOr(&list.bits[t * p.words + (col >> 5)], 1u << (col & 31));
            });
        __syncthreads();
        if (wave == 0) {
            for (int w0 = 0; w0 < p.words; w0 += 64) {
                const int w = w0 + lane;
                uint32_t any = 0;
                for (int t = 0; t < unit.count; ++t) any |= w < p.words ? list.bits[t * p.words + w] : 0;
                const int mine = __popc(any), upto = lanes_upto(mine);
                int at = n + upto - mine;
                for (; any; any &= any - 1) list.page[at++].x = w * 32 + __builtin_ctz(any);
                n += __builtin_amdgcn_readlane(upto, 63);
            }
            if (lane == 0) many = n;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < many; i += 256) {
            const int col = list.page[i].x;
            const int32_t id = table[col];
            uint32_t by = 0;
            for (int t = 0; t < unit.count; ++t) by |= (list.bits[t * p.words + (col >> 5)] >> (col & 31) & 1) << t;
            list.page[i].y = id;
            list.by[i] = (uint16_t)by;
        }
        __syncthreads();
    }
    Picked x;
    x.n = kv_uniform(many);
    if (c.page < kFewTile) {
        x.tiles = (x.n + 1) / 2;
    } else {                                         // of the last page, the only one that may end behind the rows, what they reach
        const int each = c.page / kFewTile;
        const int left = x.n ? (unit.pos + unit.count - 1 - (kv_uniform(list.page[x.n - 1].x) << c.page_log2)) / kFewTile + 1 : 0;
        x.tiles = x.n ? (x.n - 1) * each + (left < each ? left : each) : 0;
    }
    return x;
}

struct PickTable {
    PickList list;
    const char* head;
    int n, each_log2;                                // pages of 32 and more: log2 of a page's tiles
    bool several;
    __device__ __forceinline__ const char* record(const KvView& c, int id, bool& there) const {
        there = (uint32_t)id < (uint32_t)c.pages;
        return head + (int64_t)(there ? id : 0) * c.page_bytes;
    }
    __device__ __forceinline__ FewPlace operator()(const KvView& c, const FewSeq&, int i) const {
        FewPlace p;
        p.apart = 0;
        p.by0 = p.by1 = 1;
        if (c.page < kFewTile) {
            const int e0 = 2 * i, e1 = 2 * i + 1 < n ? 2 * i + 1 : 2 * i;
            const int2 x = list.page[e0], y = list.page[e1];
            const int xc = kv_uniform(x.x), yc = kv_uniform(y.x);
            p.t0 = xc * 16;
            p.apart = e1 > e0 ? (yc - xc - 1) * 16 : 0;
            p.r0 = record(c, kv_uniform(x.y), p.there0);
            p.r1 = record(c, kv_uniform(y.y), p.there1);
            p.there1 = p.there1 && e1 > e0;
            if (several) { p.by0 = (uint32_t)kv_uniform((int)list.by[e0]); p.by1 = (uint32_t)kv_uniform((int)list.by[e1]); }
        } else {
            const int2 x = list.page[i >> each_log2];
            p.t0 = (kv_uniform(x.x) << c.page_log2) + (i & ((1 << each_log2) - 1)) * kFewTile;
            p.r0 = p.r1 = record(c, kv_uniform(x.y), p.there0);
            p.there1 = p.there0;
            if (several) p.by0 = p.by1 = (uint32_t)kv_uniform((int)list.by[i >> each_log2]);
        }
        return p;
    }
};

// One wavefront's tiles [from, to) in steps of four, as few_walk.  careful: values that are no finite numbers, of pages that only some rows have
// chosen, are looked for in every tile.
template <int F, int D, bool LOW>
__device__ __forceinline__ void pick_walk(const FewArgs& f, const FewSeq& s, const PickTable& table, int h, int col0, int from, int to, bool careful, float& m, float& l,
                                          floatx4 (&o)[D / 16]) {
    const KvView& c = f.a.c;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) o[k] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (from >= to) return;
    FewQuery<F, D, LOW> q;
    FewPlace at = table(c, s, from);
    few_query<F, D, LOW, kQuads<F, D>>(f, s, h, col0, q);
    const FewLane<F, D, kQuads<F, D>> lane(c);
    if constexpr (F == IVFTQ_KV_CODE4) {
        FewTile<F, D> x, y;
        few_load<F, D, kQuads<F, D>>(c, at, lane, x);
        int i = from;
        auto step = [&](FewTile<F, D>& now, FewTile<F, D>& then) __attribute__((always_inline)) {      // past the end: a tile that is there, read and not used
            const FewPlace next = table(c, s, i + 4 < to ? i + 4 : i);
            few_load<F, D, kQuads<F, D>>(c, next, lane, then);
            few_step<F, D, LOW, true>(f.a, s, q, at, now, m, l, o, careful);
            at = next;
            i += 4;
        };
        while (true) {
            step(x, y);
            if (i >= to) break;
            step(y, x);
            if (i >= to) break;
        }
    } else {
        for (int i = from; i < to; i += 4) {
            FewTile<F, D> x;
            few_load<F, D, kQuads<F, D>>(c, at, lane, x);
            const FewPlace next = table(c, s, i + 4 < to ? i + 4 : i);
            few_step<F, D, LOW, true>(f.a, s, q, at, x, m, l, o, careful);
            at = next;
        }
    }
}

template <int F, int D, bool LOW>
__global__ __launch_bounds__(256, D <= 64 ? 4 : (D <= 128 ? 3 : 1)) void k_kv_picked(PickArgs p) {
    constexpr int kPass = D > 128 ? D / 2 : D;                 // coordinates that pass through LDS at a time
    __shared__ float ml[4][16][2];
    extern __shared__ int2 room[];                             // the list of pages; when they have been walked, the wavefronts' sums
    float(*sum)[16][kPass + 1] = reinterpret_cast<float(*)[16][kPass + 1]>(room);
    const FewArgs& f = p.f;
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, col0 = blockIdx.y * 16;
    const uint32_t wg = kv_workgroup();
    const int h = (int)(wg % (uint32_t)c.heads), at = (int)(wg / (uint32_t)c.heads % (uint32_t)p.units), share = (int)(wg / (uint32_t)c.heads / (uint32_t)p.units);
    if (share >= p.splits) return;
    const PickUnit unit = pick_unit(p, at);
    if (unit.b < 0) return;
    const PickList list = pick_lds(p, room);
    const Picked picked = pick_list(p, unit, h, list);
    FewSeq s{};
    s.first = unit.row;
    s.count = unit.count;
    s.base = unit.pos;
    s.end = unit.pos + unit.count > 0 ? unit.pos + unit.count : 0;
    s.beyond = -1;
    const int cols = unit.count * a.group;
    int from = 0, to = picked.tiles;
    if (p.splits > 1) {
        const int each = ((picked.tiles + p.splits - 1) / p.splits + 3) & ~3;
        from = share * each;
        to = from + each < to ? from + each : to;
    }
    float m, l;
    floatx4 o[D / 16];
    const PickTable table{list, c.pool + (int64_t)h * c.head_bytes, picked.n, c.page_log2 - 5, p.tokens > 1};
    // The weight of a value that a row does not see is zero, and zero times no finite number is none: only where a sum has become none
    // are such values looked for, by walking once more (looking in every tile: 64 of some 200 vector instructions).
    for (bool careful = F == IVFTQ_KV_CODE4 || unit.count == 1;; careful = true) {
        pick_walk<F, D, LOW>(f, s, table, h, col0, from + wave, to, careful, m, l, o);
        if (careful) break;
        float far = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) far = fmaxf(far, __builtin_fabsf(o[k][r])), far = o[k][r] == o[k][r] ? far : INFINITY;
        if (!__ballot(!(far < INFINITY))) break;
    }
    l = kv_sum4(l);
    if (g == 0) { ml[wave][n][0] = m; ml[wave][n][1] = l; }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][n][0]);
    const float turn = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int pass = 0; pass < D / kPass; ++pass) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = few_coord<F>(D, k, g, r) - pass * kPass;
                if (j >= 0 && j < kPass) sum[wave][n][j] = o[k][r] * turn;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * (kPass / 2); i += 256) {
            const int q = i / (kPass / 2), j = i % (kPass / 2) * 2, col = col0 + q;
            if (col >= cols) break;
            float tm = -INFINITY, tl = 0.f, u = 0.f, v = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) tm = fmaxf(tm, ml[w][q][0]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                tl += ml[w][q][0] == -INFINITY ? ml[w][q][1] * 0.f : ml[w][q][1] * __builtin_amdgcn_exp2f(ml[w][q][0] - tm);
                u += sum[w][q][j];
                v += sum[w][q][j + 1];
            }
            const int tok = p.tokens == 1 ? 0 : col / a.group, row = unit.row + tok, head = h * a.group + col - tok * a.group, jj = pass * kPass + j;
            if (p.splits == 1) {
                const float inv = tm == -INFINITY && tl == 0.f ? 0.f : 1.f / tl;
                if (F == IVFTQ_KV_CODE4) {
                    *reinterpret_cast<float2*>(f.whole + ((int64_t)row * a.q.heads + head) * D + jj) = make_float2(u * inv, v * inv);
                } else {
                    uint16_t* to16 = reinterpret_cast<uint16_t*>(a.out.data) + row * a.out.row_stride + head * a.out.head_stride + jj;
                    *reinterpret_cast<uint32_t*>(to16) = kv_pack2<F == IVFTQ_KV_BF16>(u * inv, v * inv);
                }
                if (a.lse && jj == 0) a.lse[(int64_t)row * a.q.heads + head] = tl > 0.f ? (tm + __builtin_amdgcn_logf(tl)) / kLog2e : (tl == 0.f ? -INFINITY : tl);
            } else {
                const int64_t slot = ((((int64_t)blockIdx.y * p.units + at) * c.heads + h) * p.splits + share) * 16 + q;
                *reinterpret_cast<float2*>(f.part + slot * D + jj) = make_float2(u, v);
                if (jj == 0) *reinterpret_cast<float2*>(f.part_ml + slot * 2) = make_float2(tm, tl);
            }
        }
        __syncthreads();
    }
}

struct NoRotation { __device__ __forceinline__ NoRotation(const float*, int) {} };

// The parts of a unit put together, a workgroup a unit and column tile, a wavefront a row; codes: rotated back, each wavefront a block
// of 32 coordinates.
template <int F, int D>
__global__ __launch_bounds__(512) void k_kv_picked_join(PickArgs p) {
    constexpr int kPart = D / 4, kBeside = D <= 64 ? 4 : (D <= 128 && D != 96 ? 2 : 1);
    __shared__ __align__(16) float row_sum[F == IVFTQ_KV_CODE4 ? 16 : 1][D + 4];
    const FewArgs& f = p.f;
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, col0 = blockIdx.y * 16;
    const uint32_t wg = kv_workgroup();
    // units are few here: the rotation is asked for before everything that it waits for
    const std::conditional_t<F == IVFTQ_KV_CODE4, KvTurnRows<D, true>, NoRotation> rotation(c.rotation, wave < D / 32 ? wave : 0);
    const int h = (int)(wg % (uint32_t)c.heads), at = (int)(wg / (uint32_t)c.heads);
    if (at >= p.units) return;
    const PickUnit unit = pick_unit(p, at);
    if (unit.b < 0) return;
    const int cols = unit.count * a.group;
    auto place = [&](int col, int& row, int& head) __attribute__((always_inline)) {
        const int tok = p.tokens == 1 ? 0 : col / a.group;
        row = unit.row + tok;
        head = h * a.group + col - tok * a.group;
    };
    for (int q = wave; q < 16 && col0 + q < cols; q += 8) {
        int row, head;
        place(col0 + q, row, head);
        const int64_t slot0 = ((((int64_t)blockIdx.y * p.units + at) * c.heads + h) * p.splits) * 16 + q;
        // a lane a part's maximum and sum (at most 64 parts)
        float2 u = make_float2(-INFINITY, 0.f);
        if (lane < p.splits) u = *reinterpret_cast<const float2*>(f.part_ml + (slot0 + lane * 16) * 2);
        float top = u.x;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float turn = u.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u.x - top);
        float l = u.x == -INFINITY ? u.y * 0.f : u.y * turn;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
        // kBeside parts side by side, one such load after the other: a loop with an exchange between lanes and a count that is not known is not unrolled (24 parts
        // of 128 coordinates: twelve trips to the L2, in a kernel of 10 us)
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const int beside = lane / kPart < kBeside ? lane / kPart : 0, j = lane % kPart * 4;
        for (int w = 0; w < p.splits; w += kBeside) {
            const bool there = w + beside < p.splits;
            const int part = there ? w + beside : w;
            const float t = __shfl(turn, part);
            const float4 x = *reinterpret_cast<const float4*>(f.part + (slot0 + part * 16) * D + j);
            acc.x += there ? x.x * t : 0.f; acc.y += there ? x.y * t : 0.f; acc.z += there ? x.z * t : 0.f; acc.w += there ? x.w * t : 0.f;
        }
#pragma unroll
        for (int o = kPart; o < kPart * kBeside; o <<= 1) {
            acc.x += __shfl(acc.x, lane + o); acc.y += __shfl(acc.y, lane + o); acc.z += __shfl(acc.z, lane + o); acc.w += __shfl(acc.w, lane + o);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
        if (a.lse && lane == 0) a.lse[(int64_t)row * a.q.heads + head] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
        if (lane >= kPart) continue;
        if constexpr (F == IVFTQ_KV_CODE4) {
            *reinterpret_cast<float4*>(&row_sum[q][j]) = acc;
        } else {
            constexpr bool bf = F == IVFTQ_KV_BF16;
            uint16_t* to16 = reinterpret_cast<uint16_t*>(a.out.data) + row * a.out.row_stride + head * a.out.head_stride + j;
            *reinterpret_cast<uint2*>(to16) = make_uint2(kv_pack2<bf>(acc.x, acc.y), kv_pack2<bf>(acc.z, acc.w));
        }
    }
    if constexpr (F == IVFTQ_KV_CODE4) {
        __syncthreads();
        if (wave >= D / 32) return;
        const int n = lane & 15, g = lane >> 4;
        const bool in = col0 + n < cols;
        float x[D / 32][8], y[8];
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = in ? row_sum[n][32 * k + 8 * g + e] : 0.f;
        const float norm = kv_unit_row<D>(x) * c.level_unit;
        KvTurn<D, true>{rotation}(x, y);
        int row, head;
        place(in ? col0 + n : 0, row, head);
        if (in) kv_store_turned(a.out, row, head, wave, y, norm);
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------

// Sizes of the workspaces' parts, as the launches and the caller's questions see them.
struct PickWork {
    int64_t z, zn, whole, part, ml, bytes;
    int32_t col_tiles, splits, tokens, units, list, words;
};
PickWork pick_work(const ivftq_kv_cache& c, int64_t rows, int q_heads, int max_new, int count);
struct ScoreWork { int64_t z, zn, sides, unit, bytes; int32_t tiles; };       // z < 0: not needed
ScoreWork score_work(int format, int d, int64_t rows, int q_heads, int kv_heads, bool one);

// 16-row tiles that a workgroup rotates, and workgroups (as kv_attend_launch; a chunk's scores: 36.2 us, where 512 workgroups are enough 37.1, 1,536 39.7).
struct TurnGrid {
    int tiles;
    unsigned wgs;
    explicit TurnGrid(int64_t all) {
        const int64_t fill = all / (16 * 768);
        tiles = fill < 1 ? 1 : (fill < kTurnTiles ? (int)fill : kTurnTiles);
        wgs = (unsigned)((all + 16 * tiles - 1) / (16 * tiles));
    }
};
template <int D>
void rotate_queries(const KvAttend& a, uint16_t* z, float* zn, hipStream_t st) {
    const TurnGrid grid((int64_t)a.q.rows * a.q.heads);
    k_kv_rotate_queries<D><<<grid.wgs, D * 2, 0, st>>>(a.q, a.c.rotation, z, zn, grid.tiles);
}

template <int F, int D>
hipError_t kv_score_launch(const KvAttend& a, const void* digests, float* scores, hipStream_t st) {
    const bool one = a.max_new == 1;
    const ScoreWork w = score_work(F, D, a.q.rows, a.q.heads, a.c.heads, one);
    uint16_t* z = w.z < 0 ? nullptr : reinterpret_cast<uint16_t*>(a.work + w.z);
    float* zn = reinterpret_cast<float*>(a.work + w.zn);
    ScoreArgs f{a, static_cast<const uint16_t*>(digests), scores, z, zn, reinterpret_cast<uint16_t*>(a.work + w.sides), reinterpret_cast<float*>(a.work + w.unit), w.tiles, (a.max_new + 15) / 16 + 1, 1};
    const int64_t pairs = (int64_t)a.c.rows * a.c.heads;
    const bool whole = F == IVFTQ_KV_CODE4 && !one && w.z < 0;   // sides straight from the queries
    if (F == IVFTQ_KV_CODE4 && !whole) rotate_queries<D>(a, z, zn, st);
    if (one) {
        constexpr int pages = 4 * (D <= 128 ? 32 : 16);
        k_kv_score_one<F, D><<<kv_grid(pairs, 256, (unsigned)((a.c.columns + pages - 1) / pages)), 256, 0, st>>>(f);
        return hipGetLastError();
    }
    if constexpr (F == IVFTQ_KV_CODE4) {
        const TurnGrid grid((int64_t)a.q.rows * a.q.heads);
        if (whole) k_kv_rotate_sides<D><<<grid.wgs, D * 2, 0, st>>>(f, grid.tiles);
    }
    if (!whole) k_kv_sides<F, D><<<kv_grid((pairs + 7) / 8, 256), 256, 0, st>>>(f);
    constexpr int pages = 4 * 16 * (D <= 128 ? 2 : 1);
    const unsigned blocks = (unsigned)((a.c.columns + pages - 1) / pages);
    // row tiles of a workgroup, which reads its digests once for them: as many as leave two workgroups a compute unit
    const int64_t wgs = (int64_t)a.c.batch * a.c.heads * f.row_tiles * blocks / 512;
    f.each = wgs < 1 ? 1 : (wgs < f.row_tiles ? (int)wgs : f.row_tiles);
    k_kv_score<F, D><<<kv_grid((int64_t)a.c.batch * a.c.heads * ((f.row_tiles + f.each - 1) / f.each), 256, blocks), 256, 0, st>>>(f);
    return hipGetLastError();
}
template <int D>
hipError_t kv_score_d(const KvAttend& a, const void* digests, float* scores, int format, hipStream_t st) {
    switch (format) {
        case IVFTQ_KV_F16: return kv_score_launch<IVFTQ_KV_F16, D>(a, digests, scores, st);
        case IVFTQ_KV_BF16: return kv_score_launch<IVFTQ_KV_BF16, D>(a, digests, scores, st);
        default: return kv_score_launch<IVFTQ_KV_CODE4, D>(a, digests, scores, st);
    }
}

template <int F, int D>
hipError_t kv_picked_launch(const KvAttend& a, const PickWork& w, const int32_t* chosen, int count, hipStream_t st) {
    uint16_t* z = reinterpret_cast<uint16_t*>(a.work + w.z);
    float *zn = reinterpret_cast<float*>(a.work + w.zn), *whole = reinterpret_cast<float*>(a.work + w.whole);
    if constexpr (F == IVFTQ_KV_CODE4) rotate_queries<D>(a, z, zn, st);
    PickArgs p{FewArgs{a, z, zn, whole, reinterpret_cast<float*>(a.work + w.part), reinterpret_cast<float*>(a.work + w.ml), 0, 0}, chosen, count, a.max_new, w.tokens, w.units,
               w.splits, w.list, w.words};
    p.f.a.max_new = w.tokens;
    const int64_t units = (int64_t)w.units * a.c.heads;
    const dim3 grid = kv_grid(units * w.splits, 256, (unsigned)w.col_tiles);
    // float16 results: the queries' second part matters beside the rounding of the result
    constexpr bool codes = F == IVFTQ_KV_CODE4;
    constexpr int sums = 4 * 16 * ((D > 128 ? D / 2 : D) + 1) * 4;
    const int pages = w.list * 8 + (w.list + 1) / 2 * 4 + w.tokens * w.words * 4;
    const unsigned lds = (unsigned)(pages > sums ? pages : sums);
    if (codes && a.q.type == IVFTQ_KV_F16) k_kv_picked<F, D, codes><<<grid, 256, lds, st>>>(p);
    else k_kv_picked<F, D, false><<<grid, 256, lds, st>>>(p);
    if (w.splits > 1) {
        k_kv_picked_join<F, D><<<kv_grid(units, 512, (unsigned)w.col_tiles), 512, 0, st>>>(p);
    } else if constexpr (codes) {
        const ManyArgs f{a, z, zn, whole, nullptr, nullptr, nullptr, 0, 0};
        const TurnGrid turn((int64_t)a.q.rows * a.q.heads);
        k_kv_rotate_back<D, false><<<turn.wgs, D * 2, 0, st>>>(f, turn.tiles);
    }
    return hipGetLastError();
}
template <int D>
hipError_t kv_picked_d(const KvAttend& a, const PickWork& w, const int32_t* chosen, int count, int format, hipStream_t st) {
    switch (format) {
        case IVFTQ_KV_F16: return kv_picked_launch<IVFTQ_KV_F16, D>(a, w, chosen, count, st);
        case IVFTQ_KV_BF16: return kv_picked_launch<IVFTQ_KV_BF16, D>(a, w, chosen, count, st);
        default: return kv_picked_launch<IVFTQ_KV_CODE4, D>(a, w, chosen, count, st);
    }
}

}  // namespace ivftq
