// Attention over the paged cache for few new rows: up to kFewRows query rows a key-value head (one token of every
// sequence, or a few), bound by the bytes of the cache.
//
// A workgroup walks tiles of 32 tokens; each of its four wavefronts takes every fourth tile and keeps everything in
// registers.  Scores are computed transposed, S^T = K Q^T (v_mfma 16x16x32: 16 tokens x 16 query rows), so a lane holds
// scores of one query row only; which token a row of the operand is can be chosen, and is chosen so that a lane's eight
// scores are those that the second product O^T = V^T P^T wants from that lane: no value crosses lanes between the two
// products.  Keys and values come straight from the pages in operand layout (that is why values stand in groups of eight
// tokens).  Running maximum and sum per query row, float32.
//
// Work is cut by tiles, not by sequences: the tiles of all (sequence, head) pairs, one after the other, are dealt to the
// workgroups in equal consecutive shares.  A pair that lies whole in a share is finished there; of the others each
// workgroup leaves at most two parts (one at its start, one at its end), which k_kv_few_join puts together.
//
// Measured (medians): 48 sequences of up to 9,000 tokens, 8 heads of 128 in bfloat16, four query heads each: 161 us for 912 MB (5.7
// TB/s, the rate of a read).  Four of 131,000 in codes, eight query heads each: 72 us for 328 MB (4.6 TB/s); there 263 vector
// instructions a tile take 63 % of the cycles, 224 of them make levels of codes.
#pragma once
#include "kv_kernels.h"

namespace ivftq {

// Query rows a key-value head: four column tiles of 16, each of which walks the cache.  Against the kernel of many rows (8 heads of 128,
// bfloat16, us): 16 sequences of 4,000 tokens 77 and 93 at 64 rows, 106 and 94 at 96; four of 20,000, which leave that kernel's row tiles
// few, 129 and 410, 182 and 410.  Codes gain more (70 and 165 at 64 rows of the first).  Where the sequences alone fill the chip and are
// short the other kernel is ahead from about 16 rows on (64 of 1,000 tokens: 40 and 35 at 16 rows, 101 and 36 at 64), but the host, which
// chooses, knows no lengths.
constexpr int kFewRows = 64;
constexpr int kFewTile = 32;          // tokens of a wavefront's step
constexpr int kFewMaxWgs = 1024;      // workgroups that share the tiles, at most: as many as the chip holds at once
constexpr float kLog2e = 1.44269504088896340736f;

// Weights are powers e^(score - reference) rounded to 16 bits; the reference is no maximum, and sums are only turned to another one
// when a score passes it by kWeightRoom (powers of two).  It is set kWeightLift under the maximum: float16 weights then keep their 11
// bits down to 2^-26 of the largest one, which counts where the heaviest token (a first token that most heads look at) has next to no
// value and the result is made of the others; bfloat16 has range enough.  Codes: weights meet the values' norms before they are rounded,
// so what is compared is the score plus the norm's exponent.
template <int F> constexpr float kWeightLift = F == IVFTQ_KV_BF16 ? 0.f : 12.f;
template <int F> constexpr float kWeightRoom = F == IVFTQ_KV_BF16 ? 8.f : 15.f;

// The exponent of a float16 norm, as a power of two that is above it (zero and what is under 2^-14: as 2^-14; no number: 2^17).
__device__ __forceinline__ float kv_norm_power(uint32_t bits) { return (float)(int)(__builtin_amdgcn_ubfe(bits, 10, 5)) - 14.f; }

struct FewArgs {
    KvAttend a;
    const uint16_t* z;                // codes: rotated unit queries, two float16 parts [2][rows][heads][D], eights in the order of kv_levels8
    const float* zn;                  // codes: the queries' norms
    float* whole;                     // codes: results of pairs that one workgroup finished, before they are rotated back
    float* part;                      // [column tile][2 * workgroups][16][D] unnormalised sums
    float* part_ml;                   // [column tile][2 * workgroups][16][2] maximum (in log2 units), sum
    int32_t wgs, split;               // workgroups that share the tiles; split == 0: one workgroup a pair
};

// Tiles of a sequence: those of the first tokens, then those of the window.
struct FewSeq {
    int first, count;                 // first new row, new rows that are computed
    int base, end;                    // position of the first new row, one past the last one's
    int low, beyond;                  // first token that the window of the earliest new row shows; last one outside that of the latest (-1: none)
    int sink_tiles, window_tile, tiles;
};

__device__ __forceinline__ FewSeq few_seq(const KvAttend& a, int b) {
    FewSeq s;
    const int len = kv_length(a.c, b);
    kv_new_rows(a.c, b, s.first, s.count);
    s.base = len - s.count;
    if (s.count > a.max_new) s.count = a.max_new;
    s.end = s.base + s.count > 0 ? s.base + s.count : 0;
    const int64_t low = a.window ? (int64_t)s.base - a.window + 1 : 0;
    s.low = low > 0 ? (int)low : 0;
    s.beyond = a.window && (int64_t)s.end - 1 - a.window >= 0 ? (int)((int64_t)s.end - 1 - a.window) : -1;
    const int end = (s.end + kFewTile - 1) / kFewTile, seen = a.sinks < s.end ? a.sinks : s.end;
    s.window_tile = s.low / kFewTile;
    if (s.window_tile > end) s.window_tile = end;
    s.sink_tiles = (seen + kFewTile - 1) / kFewTile;
    if (s.sink_tiles > s.window_tile) s.sink_tiles = s.window_tile;
    const int n = s.sink_tiles + end - s.window_tile;
    s.tiles = s.count ? (n ? n : 1) : 0;                    // an empty sequence keeps one tile, all of it masked
    return s;
}

__device__ __forceinline__ int few_tiles(const KvAttend& a, int b) { return b < a.c.batch ? few_seq(a, b).tiles : 0; }

// Tiles a workgroup takes.  At least four: one for each wavefront.
__device__ __forceinline__ int64_t few_share(int64_t total, int wgs) {
    const int64_t s = (total + wgs - 1) / wgs;
    return s < 4 ? 4 : (s + 3) & ~(int64_t)3;
}

// The share of workgroup `wg`, positions [x, end) in the order (sequence, head, tile): the sequence of x and that sequence's
// first position.  By a wavefront: a lane a sequence, scans over them; up to 64 sequences are looked at once.
__device__ __forceinline__ void few_find(const KvAttend& a, int wg, int wgs, int64_t& x, int64_t& end, int& seq, int64_t& at) {
    const int lane = threadIdx.x & 63;
    int tiles = 0;
    int64_t incl = 0, total = 0;
    auto scan = [&](int b0) __attribute__((always_inline)) {
        tiles = few_tiles(a, b0 + lane);
        incl = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int64_t u = __shfl_up(incl, o); if (lane >= o) incl += u; }
        return kv_uniform((int64_t)__shfl(incl, 63));
    };
    for (int b0 = 0; b0 < a.c.batch; b0 += 64) total += scan(b0);
    total *= a.c.heads;
    const int64_t share = few_share(total, wgs);
    x = wg * share;
    end = x + share < total ? x + share : total;
    seq = a.c.batch;
    at = 0;
    int64_t base = 0;
    for (int b0 = 0; x < end && b0 < a.c.batch; b0 += 64) {
        const int64_t all = a.c.batch <= 64 ? total / a.c.heads : scan(b0);
        const uint64_t past = __ballot((base + incl) * a.c.heads > x);
        if (past) {
            const int l = __builtin_ctzll(past);
            seq = b0 + l;
            at = kv_uniform(base + (int64_t)__shfl(incl - tiles, l)) * a.c.heads;
            return;
        }
        base += all;
    }
}

template <int F>
__device__ __forceinline__ floatx4 kv_mfma16(uintx4 x, uintx4 y, floatx4 acc) {
    if constexpr (F == IVFTQ_KV_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, x), __builtin_bit_cast(halfx8, y), acc, 0, 0, 0);
}

// What a tile of 32 tokens is read into.  Codes: a lane's words of the two key operands, its words of the value operands,
// the norms of its eight tokens; 16 bits: the operands themselves.
template <int F, int D>
struct FewTile {
    static constexpr bool kCodes = F == IVFTQ_KV_CODE4;
    uint32_t kw[2][kCodes ? D / 32 : 1], vw[kCodes ? D / 16 : 1];
    uintx4 kg, vg;
    uintx4 kk[2][kCodes ? 1 : D / 32], vv[kCodes ? 1 : D / 16];
};
// A tile's first token and the records of its page (pages of 16: of its two pages); page 0 where there is none.
struct FewPlace {
    int t0;
    const char *r0, *r1;
    bool there0, there1;
};
struct FewTable {                     // one pair's way into the cache
    const int32_t* row;
    const char* head;
    __device__ __forceinline__ FewTable(const KvView& c, int b, int h) : row(c.table + (int64_t)b * c.table_stride), head(c.pool + (int64_t)h * c.head_bytes) {}
    __device__ __forceinline__ const char* find(const KvView& c, int t, bool& there) const {
        const int col = t >> c.page_log2;
        const int32_t id = col < c.columns ? kv_int(row, col) : -1;
        there = (uint32_t)id < (uint32_t)c.pages;
        return head + (int64_t)(there ? id : 0) * c.page_bytes;
    }
    __device__ __forceinline__ FewPlace operator()(const KvView& c, const FewSeq& s, int i) const {
        FewPlace p;
        p.t0 = (i < s.sink_tiles ? i : i - s.sink_tiles + s.window_tile) * kFewTile;
        p.r0 = p.r1 = find(c, p.t0, p.there0);
        p.there1 = p.there0;
        if (c.page < kFewTile) p.r1 = find(c, p.t0 + 16, p.there1);
        return p;
    }
};

// Byte offsets of a lane's reads inside a tile of one page.
template <int F, int D>
struct FewLane {
    uint32_t key, value, norm;
    __device__ __forceinline__ explicit FewLane(const KvView& c) {
        const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
        // lane's token of the two key operands: 8 (n / 4) + (16 bits: 4 y + n % 4; codes: 2 (n % 4) + y)
        if constexpr (F == IVFTQ_KV_CODE4) {
            key = (8 * (n >> 2) + 2 * (n & 3)) * (D / 2) + g * (D / 8);
            value = c.page * (D / 2) + g * (D * 4) + n * (D / 4);
            norm = c.page * D + g * 16;
        } else {
            key = (8 * (n >> 2) + (n & 3)) * (D * 2) + g * 16;
            value = c.page * (D * 2) + (g * D + n) * 16;
            norm = 0;
        }
    }
};

template <int F, int D>
__device__ __forceinline__ void few_load(const KvView& c, const FewPlace& p, const FewLane<F, D>& at, FewTile<F, D>& x) {
    constexpr bool codes = F == IVFTQ_KV_CODE4;
    constexpr int row = codes ? D / 2 : D * 2;                        // bytes of a token's row
    const int in = p.t0 & (c.page - 1);
    const char* base = p.r0;
    auto read = [&](const char* keys, const char* values, const char* norms) {
        // every address is a scalar base and a lane's offset (pages of 32 and more), or a lane's own pointer
        if constexpr (codes) {
            const uint32_t *q = reinterpret_cast<const uint32_t*>(keys), *v = reinterpret_cast<const uint32_t*>(values);
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int k = 0; k < D / 32; ++k) x.kw[y][k] = q[y * (D / 8) + k];
#pragma unroll
            for (int k = 0; k < D / 16; ++k) x.vw[k] = v[k];
            x.kg = *reinterpret_cast<const uintx4*>(norms);
            x.vg = *reinterpret_cast<const uintx4*>(norms + 2 * c.page);
        } else {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int k = 0; k < D / 32; ++k) x.kk[y][k] = *reinterpret_cast<const uintx4*>(keys + y * 4 * row + k * 64);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) x.vv[k] = *reinterpret_cast<const uintx4*>(values + k * 256);
        }
    };
    if (c.page >= kFewTile) {
        const char* here = base + in * row;
        read(here + at.key, here + at.value, base + 2 * in + at.norm);
    } else {                                                          // pages of 16: the tile's halves lie in two pages
        const char* other = p.r1;
        const int lane = threadIdx.x & 63;
        const bool k1 = lane & 8, v1 = lane & 32;                     // second half: n / 8, g / 2
        read((k1 ? other - 16 * row : base) + at.key, (v1 ? other - 16 * row : base) + at.value, (v1 ? other - 32 : base) + at.norm);
    }
}

// One query row a lane: its operands, what its scores are multiplied by, its position.
template <int F, int D, bool LOW>
struct FewQuery {
    uintx4 q[D / 32], low[LOW ? D / 32 : 1];
    float gain;
    int pos, begin;                   // its position, the first token of its window
};

// The lowest n of eight bits.
__device__ __forceinline__ uint32_t few_below(int n) { return 0xffu >> (n <= 0 ? 8 : (n >= 8 ? 0 : 8 - n)); }

template <int F, int D, bool LOW>
__device__ __forceinline__ void few_query(const FewArgs& f, const FewSeq& s, int h, int col0, FewQuery<F, D, LOW>& x) {
    const KvAttend& a = f.a;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int cols = s.count * a.group, col = col0 + n < cols ? col0 + n : 0, tok = a.max_new == 1 ? 0 : col / a.group;
    x.pos = col0 + n < cols ? s.base + tok : s.end - 1;
    const int64_t low = a.window ? (int64_t)x.pos - a.window + 1 : 0;
    x.begin = low > 0 ? (int)low : 0;
    // scores are multiplied by a factor above zero, so that their maximum is that of the products: a negative scale turns the
    // queries' signs, and none at all is taken as next to none
    x.gain = fabsf(a.scale) * kLog2e;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    const int64_t row = s.first + tok, head = h * a.group + col - tok * a.group;
    if constexpr (F == IVFTQ_KV_CODE4) {
        const int64_t at = row * a.q.heads + head, all = (int64_t)a.q.rows * a.q.heads;
        x.gain *= f.zn[at] * (a.c.level_unit / kSplitScale);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            x.q[k] = *reinterpret_cast<const uintx4*>(f.z + at * D + g * (D / 4) + 8 * k);
            x.q[k] ^= sign;
            if constexpr (LOW) { x.low[k] = *reinterpret_cast<const uintx4*>(f.z + (all + at) * D + g * (D / 4) + 8 * k); x.low[k] ^= sign; }
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(a.q.data) + row * a.q.row_stride + head * a.q.head_stride + 8 * g;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) { x.q[k] = *reinterpret_cast<const uintx4*>(p + 32 * k); x.q[k] ^= sign; }
    }
    x.gain = fmaxf(x.gain, 1e-30f);
}

// A tile into the running maximum m, sum l (of this lane's tokens) and sums o (transposed: o[blk][r] = coordinate
// 16 blk + 4 g + r, or (4 g + r) * D / 16 + blk for codes).
template <int F, int D, bool LOW>
__device__ __forceinline__ void few_step(const KvAttend& a, const FewSeq& s, const FewQuery<F, D, LOW>& q, const FewPlace& at, FewTile<F, D>& x, float& m,
                                         float& l, floatx4 (&o)[D / 16]) {
    const KvView& c = a.c;
    constexpr bool codes = F == IVFTQ_KV_CODE4;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, t0 = at.t0;
    floatx4 st[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    float sc[8];                            // of the tokens t0 + 8 g + e
    if constexpr (F == IVFTQ_KV_CODE4) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const uintx4 w = __builtin_bit_cast(uintx4, kv_levels8(x.kw[y][k], c));
                st[y] = kv_mfma16<F>(w, q.q[k], st[y]);
                if constexpr (LOW) st[y] = kv_mfma16<F>(w, q.low[k], st[y]);
            }
        const halfx8 kn = __builtin_bit_cast(halfx8, x.kg);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e] = __builtin_fmaf((float)kn[e], st[e & 1][e >> 1], 0.f);        // one v_fma_mix
    } else {
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) st[y] = kv_mfma16<F>(x.kk[y][k], q.q[k], st[y]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e] = st[e >> 2][e & 3];
    }
    // every token of the tile visible to every row?
    const bool full = at.there0 && at.there1 && t0 + kFewTile - 1 <= s.base && (t0 > s.beyond || t0 + kFewTile <= a.sinks);
    uint32_t shown = 0xff;                  // of the lane's eight tokens: those that any row sees
    if (!full) {
        // bits and selects only: what the compiler makes of conditions here was found to be wrong
        const int tb = t0 + 8 * g;
        const uint32_t there = (g >> 1 ? at.there1 : at.there0) ? 0xffu : 0u, sinks = few_below(a.sinks - tb);
        shown = few_below(s.end - tb) & (~few_below(s.low - tb) | sinks) & there;
        const uint32_t mine = few_below(q.pos + 1 - tb) & (~few_below(q.begin - tb) | sinks) & shown;
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e] = mine >> e & 1 ? sc[e] : -INFINITY;
        if constexpr (codes) {                // norms of others may be anything, and 0 * NaN is no zero
#pragma unroll
            for (int e = 0; e < 4; ++e) x.vg[e] &= (mine >> 2 * e & 1 ? 0xffffu : 0u) | (mine >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
        }
    }
    float top = sc[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, sc[e]);
    top *= q.gain;
    if constexpr (codes) {                  // norms are not negative: the largest is that of the largest bits
        typedef uint16_t two __attribute__((ext_vector_type(2)));
        const uint32_t w0 = x.vg[0], w1 = x.vg[1], w2 = x.vg[2], w3 = x.vg[3];
        const two u = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(two, w0), __builtin_bit_cast(two, w1)),
                                                __builtin_elementwise_max(__builtin_bit_cast(two, w2), __builtin_bit_cast(two, w3)));
        top += kv_norm_power(u[0] > u[1] ? u[0] : u[1]);
    }
    if (__ballot(top > m + kWeightRoom<F>)) {
        const float all = kv_max4(top), now = all > m + kWeightRoom<F> ? all - kWeightLift<F> : m;
        const float turn = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= turn;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) o[k] *= turn;
    }
    const float less = m == -INFINITY ? 0.f : m;           // a row that has seen nothing: every score is -infinity
    float pr[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) pr[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], q.gain, -less));
#pragma unroll
    for (int e = 0; e < 8; ++e) l += pr[e];
    if constexpr (F == IVFTQ_KV_CODE4) {
        const halfx8 vn = __builtin_bit_cast(halfx8, x.vg);
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __builtin_fmaf((float)vn[e], pr[e], 0.f);
        const uintx4 p = {kv_pack2<false>(w[0], w[2]), kv_pack2<false>(w[4], w[6]), kv_pack2<false>(w[1], w[3]), kv_pack2<false>(w[5], w[7])};
#pragma unroll
        for (int k = 0; k < D / 16; ++k) o[k] = kv_mfma16<F>(__builtin_bit_cast(uintx4, kv_levels8(x.vw[k], c)), p, o[k]);
    } else {
        constexpr bool bf = F == IVFTQ_KV_BF16;
        const uintx4 p = {kv_pack2<bf>(pr[0], pr[1]), kv_pack2<bf>(pr[2], pr[3]), kv_pack2<bf>(pr[4], pr[5]), kv_pack2<bf>(pr[6], pr[7])};
        uint32_t dirty = 0;                 // of the lane's eight tokens: no finite value, and not the same to every row
        if (!full) {
            if (s.count > 1) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) dirty |= kv_not_finite<bf>(x.vv[k]);
#pragma unroll
                for (int w = 1; w < 16; w <<= 1) dirty |= __shfl_xor(dirty, w);
                dirty &= shown;
                shown &= ~dirty;
            }
            uintx4 keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) keep[e] = (shown >> 2 * e & 1 ? 0xffffu : 0u) | (shown >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) x.vv[k] &= keep;
        }
#pragma unroll
        for (int k = 0; k < D / 16; ++k) o[k] = kv_mfma16<F>(x.vv[k], p, o[k]);
        if (!full && __ballot(dirty != 0)) {         // such tokens one by one, for the rows that see them
            for (int t = 0; t < kFewTile; ++t) {
                const int from = t >> 3, e = t & 7;
                if (!(__shfl(dirty, 16 * from) >> e & 1)) continue;
                float v = sc[0], w = pr[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) { v = e == i ? sc[i] : v; w = e == i ? pr[i] : w; }
                v = __shfl(v, 16 * from + n);
                w = __shfl(w, 16 * from + n);
                const int in = (t0 + t) & (c.page - 1);
                const uint16_t* y = reinterpret_cast<const uint16_t*>((from >> 1 ? at.r1 : at.r0) + c.page * (D * 2)) + (in >> 3) * D * 8 + e;
                if (v == -INFINITY) continue;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[k][r] += w * kv_to_float<bf>(y[(16 * k + 4 * g + r) * 8]);
            }
        }
    }
}

// One wavefront's tiles [from, to) in steps of four.  Codes: the next tile's words are on their way while this one is
// worked on (a tile is 24 registers, its arithmetic as long as its loads), the pages of the one after are looked up.  16
// bits: a tile's 16 KB in flight are enough, only the pages are looked up ahead.
template <int F, int D, bool LOW>
__device__ __forceinline__ void few_walk(const FewArgs& f, const FewSeq& s, int b, int h, int col0, int from, int to, float& m, float& l,
                                         floatx4 (&o)[D / 16]) {
    const KvView& c = f.a.c;
    if (from >= to) return;
    FewQuery<F, D, LOW> q;
    const FewTable table(c, b, h);
    FewPlace at = table(c, s, from);
    few_query<F, D, LOW>(f, s, h, col0, q);
    const FewLane<F, D> lane(c);
    if constexpr (F == IVFTQ_KV_CODE4) {
        FewTile<F, D> x, y;
        few_load<F, D>(c, at, lane, x);
        FewPlace next = table(c, s, from + 4 < to ? from + 4 : from);
        int i = from;
        // past the end: a tile that is there, read and not used
        auto step = [&](FewTile<F, D>& now, FewTile<F, D>& then) {
            const FewPlace after = table(c, s, i + 8 < to ? i + 8 : i);
            few_load<F, D>(c, next, lane, then);
            few_step<F, D, LOW>(f.a, s, q, at, now, m, l, o);
            at = next;
            next = after;
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
            few_load<F, D>(c, at, lane, x);
            const FewPlace next = table(c, s, i + 4 < to ? i + 4 : i);
            few_step<F, D, LOW>(f.a, s, q, at, x, m, l, o);
            at = next;
        }
    }
}

template <int F>
__device__ __forceinline__ int few_coord(int D, int k, int g, int r) { return F == IVFTQ_KV_CODE4 ? (4 * g + r) * (D / 16) + k : 16 * k + 4 * g + r; }

template <int F, int D, bool LOW>
__global__ __launch_bounds__(256, D <= 64 ? 4 : (D <= 128 ? 3 : 1)) void k_kv_few(FewArgs f) {
    constexpr int kPass = D > 128 ? D / 2 : D;                 // coordinates that pass through LDS at a time
    __shared__ float sum[4][16][kPass + 1];
    __shared__ float ml[4][16][2];
    const KvAttend& a = f.a;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int col0 = blockIdx.y * 16;
    int64_t x = 0, end = 0, at = 0;
    int b = 0;
    if (f.split) {
        few_find(a, blockIdx.x, f.wgs, x, end, b, at);
        if (x >= end) return;
    } else {
        b = (int)(kv_workgroup() / (uint32_t)a.c.heads);
        if (b >= a.c.batch) return;
    }
    const int64_t begin = x;
    FewSeq s = few_seq(a, b);
    while (true) {
        int h, from, to;
        if (f.split) {
            while (b < a.c.batch && x >= at + (int64_t)s.tiles * a.c.heads) {        // the next sequence that has tiles
                at += (int64_t)s.tiles * a.c.heads;
                if (++b < a.c.batch) s = few_seq(a, b);
            }
            if (b >= a.c.batch) return;
            h = (int)((x - at) / s.tiles);
            const int64_t pair = at + (int64_t)h * s.tiles;
            from = (int)(x - pair);
            to = (int)(end - pair < s.tiles ? end - pair : s.tiles);
        } else {
            h = (int)(kv_workgroup() % (uint32_t)a.c.heads);
            from = 0;
            to = s.tiles;
            if (!s.tiles) return;
        }
        const int cols = s.count * a.group;
        const bool whole = from == 0 && to == s.tiles;
        if (col0 < cols) {
            float m = -INFINITY, l = 0.f;
            floatx4 o[D / 16];
#pragma unroll
            for (int k = 0; k < D / 16; ++k) o[k] = floatx4{0.f, 0.f, 0.f, 0.f};
            few_walk<F, D, LOW>(f, s, b, h, col0, from + wave, to, m, l, o);
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
                    const int row = i / (kPass / 2), j = i % (kPass / 2) * 2, col = col0 + row;
                    if (col >= cols) break;
                    float tm = -INFINITY, tl = 0.f, u = 0.f, v = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) tm = fmaxf(tm, ml[w][row][0]);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        tl += ml[w][row][0] == -INFINITY ? ml[w][row][1] * 0.f : ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - tm);
                        u += sum[w][row][j];
                        v += sum[w][row][j + 1];
                    }
                    const int64_t qrow = s.first + col / a.group;
                    const int qhead = h * a.group + col % a.group, jj = pass * kPass + j;
                    if (whole) {
                        const float inv = tm == -INFINITY && tl == 0.f ? 0.f : 1.f / tl;
                        if (F == IVFTQ_KV_CODE4) {
                            *reinterpret_cast<float2*>(f.whole + (qrow * a.q.heads + qhead) * D + jj) = make_float2(u * inv, v * inv);
                        } else {
                            uint16_t* p = reinterpret_cast<uint16_t*>(a.out.data) + qrow * a.out.row_stride + qhead * a.out.head_stride + jj;
                            *reinterpret_cast<uint32_t*>(p) = kv_pack2<F == IVFTQ_KV_BF16>(u * inv, v * inv);
                        }
                        if (a.lse && jj == 0) a.lse[qrow * a.q.heads + qhead] = tl > 0.f ? (tm + __builtin_amdgcn_logf(tl)) / kLog2e : (tl == 0.f ? -INFINITY : tl);
                    } else {
                        // a share's first part belongs to a pair that began before it, its last part to one that goes on
                        const int64_t slot = (int64_t)blockIdx.y * 2 * f.wgs + 2 * blockIdx.x + (x == begin && from != 0 ? 0 : 1);
                        *reinterpret_cast<float2*>(f.part + (slot * 16 + row) * D + jj) = make_float2(u, v);
                        if (jj == 0) *reinterpret_cast<float2*>(f.part_ml + (slot * 16 + row) * 2) = make_float2(tm, tl);
                    }
                }
                __syncthreads();
            }
        }
        if (!f.split) return;
        x += to - from;
        if (x >= end) return;
    }
}

// Pairs whose tiles lie in more than one share: their parts put together.  One workgroup a pair and column tile, a wavefront a
// row: D / 4 lanes read a part, the others the parts beside it, eight at a time.  Codes: every pair; its 16 rows are then
// rotated back, each wavefront computing a block of 32 coordinates.
template <int F, int D>
__global__ __launch_bounds__(512) void k_kv_few_join(FewArgs f) {
    constexpr int kPart = D / 4, kBeside = 64 / kPart > 0 ? 64 / kPart : 1;          // lanes of a part, parts side by side
    static_assert(kPart <= 64);
    __shared__ __align__(16) float row_sum[F == IVFTQ_KV_CODE4 ? 16 : 1][D + 4];
    __shared__ float weight[8][64];
    const KvAttend& a = f.a;
    const int wave = kv_wave(), lane = threadIdx.x & 63;
    const int b = (int)(kv_workgroup() / (uint32_t)a.c.heads), h = (int)(kv_workgroup() % (uint32_t)a.c.heads), col0 = blockIdx.y * 16;
    if (b >= a.c.batch) return;
    const FewSeq s = few_seq(a, b);
    const int cols = s.count * a.group;
    if (col0 >= cols) return;
    int64_t lo = 0, share = 1;
    int w0 = 0, w1 = 0;
    if (f.split) {
        int64_t total = 0, before = 0;
        for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
            const int i = b0 + lane;
            int v = few_tiles(a, i), u = i < b ? v : 0;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) { v += __shfl_xor(v, o); u += __shfl_xor(u, o); }
            total += v;
            before += u;
        }
        total = kv_uniform(total);
        before = kv_uniform(before);
        share = few_share(total * a.c.heads, f.wgs);
        lo = before * a.c.heads + (int64_t)h * s.tiles;
        w0 = (int)(lo / share);
        w1 = (int)((lo + s.tiles - 1) / share);
    }
    const bool joined = w0 != w1;
    if (!joined && F != IVFTQ_KV_CODE4) return;
    const int beside = lane / kPart, j = lane % kPart * 4;
    for (int row = wave; row < 16 && col0 + row < cols; row += 8) {
        const int col = col0 + row;
        const int64_t qrow = s.first + col / a.group;
        const int qhead = h * a.group + col % a.group;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        if (joined) {
            float top = -INFINITY, l = 0.f;
            // of the pair's first share the pair has the last part, of the others the first
            const int64_t base = (int64_t)blockIdx.y * 2 * f.wgs;
            for (int w = w0 + lane; w <= w1; w += 64)
                top = fmaxf(top, f.part_ml[((base + 2 * w + (w == w0)) * 16 + row) * 2]);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
            for (int v0 = w0; v0 <= w1; v0 += 64) {
                const int w = v0 + lane;
                float turn = 0.f;
                if (w <= w1) {
                    const float2 u = *reinterpret_cast<const float2*>(f.part_ml + ((base + 2 * w + (w == w0)) * 16 + row) * 2);
                    turn = u.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u.x - top);
                    l += u.y * turn;
                }
                weight[wave][lane] = turn;
                const int many = w1 - v0 + 1 < 64 ? w1 - v0 + 1 : 64;
#pragma unroll 8
                for (int i = beside; i < many; i += kBeside) {
                    if (kBeside * kPart < 64 && beside >= kBeside) break;
                    const int64_t slot = base + 2 * (v0 + i) + (v0 + i == w0);
                    const float t = weight[wave][i];
                    const float4 u = *reinterpret_cast<const float4*>(f.part + (slot * 16 + row) * D + j);
                    acc.x += u.x * t; acc.y += u.y * t; acc.z += u.z * t; acc.w += u.w * t;
                }
            }
#pragma unroll
            for (int o = kPart; o < kPart * kBeside; o <<= 1) {
                acc.x += __shfl(acc.x, lane + o); acc.y += __shfl(acc.y, lane + o); acc.z += __shfl(acc.z, lane + o); acc.w += __shfl(acc.w, lane + o);
            }
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
            const float inv = l == 0.f ? 0.f : 1.f / l;
            acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
            if (a.lse && lane == 0) a.lse[qrow * a.q.heads + qhead] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
        } else if (F == IVFTQ_KV_CODE4 && beside == 0) {
            acc = *reinterpret_cast<const float4*>(f.whole + (qrow * a.q.heads + qhead) * D + j);
        }
        if (beside) continue;
        if constexpr (F == IVFTQ_KV_CODE4) {
            *reinterpret_cast<float4*>(&row_sum[row][j]) = acc;
        } else {
            constexpr bool bf = F == IVFTQ_KV_BF16;
            uint16_t* p = reinterpret_cast<uint16_t*>(a.out.data) + qrow * a.out.row_stride + qhead * a.out.head_stride + j;
            *reinterpret_cast<uint2*>(p) = make_uint2(kv_pack2<bf>(acc.x, acc.y), kv_pack2<bf>(acc.z, acc.w));
        }
    }
    if constexpr (F == IVFTQ_KV_CODE4) {
        __syncthreads();
        if (wave >= D / 32) return;
        const int n = lane & 15, g = lane >> 4, col = col0 + n;
        const bool in = col < cols;
        float x[D / 32][8], y[8];
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = in ? row_sum[n][32 * k + 8 * g + e] : 0.f;
        const float norm = kv_unit_row<D>(x) * a.c.level_unit;
        KvTurn<D, true>(a.c.rotation, wave)(x, y);
        if (in) kv_store_turned(a.out, s.first + col / a.group, h * a.group + col % a.group, wave, y, norm);
    }
}

}  // namespace ivftq
