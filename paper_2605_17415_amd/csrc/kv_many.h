// Attention over the paged cache for many new rows a sequence (prompts, chunks of prompts): bound by the matrix cores and the
// exponentials beside them.
//
// A workgroup of four wavefronts owns 128 query rows of one (sequence, key-value head): rows are (token, head of the
// group) pairs, so the group's heads share every key and value that is read.  It walks the visible keys in tiles of 64
// tokens, staged in LDS (16-bit pages are copied, codes become float16 levels on the way).  As in kv_few.h the products
// are transposed, S^T = K Q^T and O^T = V^T P^T (v_mfma 32x32x16), and the token order of the key operand is chosen so
// that the scores a lane gets are those it puts into the second product: nothing goes through LDS but keys and values.
// Two workgroups a compute unit, which are not in step, so that one's exponentials run beside the other's products; each
// loads a tile into registers two steps before it is used and stores it to the second LDS buffer one step before.
#pragma once
#include <type_traits>

#include "kv_few.h"

namespace ivftq {

typedef float floatx16_ __attribute__((ext_vector_type(16)));

constexpr int kManyRows = 128;        // query rows of a workgroup
constexpr int kManyTile = 64;         // tokens of a step

struct ManyArgs {
    KvAttend a;
    const uint16_t* z;                // codes: rotated unit queries, two float16 parts, eights in the order of kv_levels8
    const float* zn;                  // codes: the queries' norms
    float* whole;                     // codes: results before they are rotated back; several parts: their sums [parts][rows][heads][D]
    float* part_ml;                   // several parts: maximum (in log2 units) and sum of weights
    int32_t row_tiles, parts;         // row tiles a (sequence, head): those of max_new; shares of a row tile's keys
};

template <int F>
__device__ __forceinline__ floatx16_ kv_mfma32(uintx4 x, uintx4 y, floatx16_ acc) {
    if constexpr (F == IVFTQ_KV_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, x), __builtin_bit_cast(halfx8, y), acc, 0, 0, 0);
}

// The tiles that a workgroup's rows see: those of the first tokens, then those of the window.
struct ManySpan {
    int end, low;                     // one past the last row's position, first token of the first row's window
    int sink_tiles, window_tile, tiles;
    __device__ __forceinline__ int first_token(int i) const { return (i < sink_tiles ? i : i - sink_tiles + window_tile) * kManyTile; }
};
__device__ __forceinline__ ManySpan many_span(const KvAttend& a, int pos0, int pos1) {
    ManySpan s;
    s.end = pos1 + 1 > 0 ? pos1 + 1 : 0;
    const int64_t low = a.window ? (int64_t)pos0 - a.window + 1 : 0;
    s.low = low > 0 ? (int)low : 0;
    const int end_tile = (s.end + kManyTile - 1) / kManyTile, seen = a.sinks < s.end ? a.sinks : s.end;
    s.window_tile = s.low / kManyTile < end_tile ? s.low / kManyTile : end_tile;
    s.sink_tiles = (seen + kManyTile - 1) / kManyTile;
    if (s.sink_tiles > s.window_tile) s.sink_tiles = s.window_tile;
    s.tiles = s.sink_tiles + end_tile - s.window_tile;
    return s;
}

// One wavefront's quarter of a tile on its way to LDS: 16 tokens, which lie in one page.
template <int F, int D>
struct ManyStage {
    static constexpr bool kCodes = F == IVFTQ_KV_CODE4;
    static constexpr int kKeyPitch = D * 2 + 16;                // bytes of a key row in LDS: rows 4 banks apart
    static constexpr int kKeyBytes = kManyTile * kKeyPitch, kBytes = kKeyBytes + kManyTile * D * 2 + (kCodes ? kManyTile * 8 : 0);
    using W = typename std::conditional<kCodes, uint32_t, uintx4>::type;      // eight coordinates of a key, eight tokens of a value
    W k[D / 32], v[D / 32];
    uint32_t norm;

    __device__ __forceinline__ void load(const KvView& c, int h, int64_t page, int t) {
        const int lane = threadIdx.x & 63, in = t & (c.page - 1);
        const char* rec = kv_record(c, page < 0 ? 0 : page, h);
        const int row = kCodes ? D / 2 : D * 2;
        const W* x = reinterpret_cast<const W*>(rec + in * row);
        const W* y = reinterpret_cast<const W*>(rec + c.page * row + in * row);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) { k[j] = x[lane + 64 * j]; v[j] = y[lane + 64 * j]; }
        if constexpr (kCodes)
            norm = reinterpret_cast<const uint16_t*>(rec + 2 * c.page * row)[(lane & 16 ? c.page : 0) + in + (lane & 15)];
    }
    // quarter: of the tile; a key chunk of eight coordinates goes to its row, a value chunk of eight tokens stays in order
    __device__ __forceinline__ void store(const KvView& c, char* to, int quarter) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int u = lane + 64 * j, t = 16 * quarter + u / (D / 8), w = u % (D / 8);
            uintx4 x, y;
            if constexpr (kCodes) { x = __builtin_bit_cast(uintx4, kv_levels8(k[j], c)); y = __builtin_bit_cast(uintx4, kv_levels8(v[j], c)); }
            else { x = k[j]; y = v[j]; }
            *reinterpret_cast<uintx4*>(to + t * kKeyPitch + w * 16) = x;
            *reinterpret_cast<uintx4*>(to + kKeyBytes + (quarter * 2 * D + u) * 16) = y;
        }
        if (kCodes && lane < 32)
            reinterpret_cast<float*>(to + kKeyBytes + kManyTile * D * 2)[(lane & 16) * 4 + 16 * quarter + (lane & 15)] = (float)__builtin_bit_cast(_Float16, (uint16_t)norm);
    }
};

// The lowest n bits.
__device__ __forceinline__ uint64_t many_below(int64_t n) { return n <= 0 ? 0 : (n >= 64 ? ~0ull : (1ull << n) - 1); }

template <int F, int D, bool LOW>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_kv_many(ManyArgs f) {
    using Stage = ManyStage<F, D>;
    constexpr bool codes = F == IVFTQ_KV_CODE4, bf = F == IVFTQ_KV_BF16;
    __shared__ __align__(16) char lds[2][Stage::kBytes];
    __shared__ uint32_t odd[2];
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
    // heads fastest: with eight heads each XCD reads one head's pages; then a row tile's shares, then sequences; the row tiles
    // with the longest reach first
    const int h = blockIdx.x % c.heads, part = blockIdx.x / c.heads % f.parts, b = blockIdx.x / c.heads / f.parts % c.batch;
    const int rt = f.row_tiles - 1 - (int)(blockIdx.x / c.heads / f.parts / c.batch);
    const FewSeq s = few_seq(a, b);
    const int cols = s.count * a.group;
    if (rt * kManyRows >= cols) return;
    const int col = rt * kManyRows + wave * 32 + n, used = col < cols ? col : cols - 1;
    const int pos = s.base + used / a.group;
    const int64_t qrow = s.first + used / a.group;
    const int qhead = h * a.group + used % a.group;
    const int last_col = (rt + 1) * kManyRows < cols ? (rt + 1) * kManyRows - 1 : cols - 1;
    const int pos0 = s.base + rt * kManyRows / a.group, pos1 = s.base + last_col / a.group;
    const ManySpan span = many_span(a, pos0, pos1);
    const int from = (int)((int64_t)span.tiles * part / f.parts), to = (int)((int64_t)span.tiles * (part + 1) / f.parts);

    // scores are multiplied by a factor above zero, so that their maximum is that of the products: a negative scale turns the
    // queries' signs, and none at all is taken as next to none
    uintx4 q[D / 16], ql[LOW ? D / 16 : 1];
    float gain = fabsf(a.scale) * kLog2e;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    if constexpr (codes) {
        const int64_t at = qrow * a.q.heads + qhead, all = (int64_t)a.q.rows * a.q.heads;
        gain *= f.zn[at] * (c.level_unit / kSplitScale);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            q[k] = *reinterpret_cast<const uintx4*>(f.z + at * D + 16 * k + 8 * half);
            q[k] ^= sign;
            if constexpr (LOW) { ql[k] = *reinterpret_cast<const uintx4*>(f.z + (all + at) * D + 16 * k + 8 * half); ql[k] ^= sign; }
        }
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(a.q.data) + qrow * a.q.row_stride + qhead * a.q.head_stride + 8 * half;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) { q[k] = *reinterpret_cast<const uintx4*>(p + 16 * k); q[k] ^= sign; }
    }
    gain = fmaxf(gain, 1e-30f);
    floatx16_ o[D / 32];
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[k][r] = 0.f;
    float m = -INFINITY, l = 0.f;              // m: in units of the exponent (log2)
    // the token (of 32) that this lane's operand row stands for
    const int tok = 16 * (n >> 4) + 8 * (n >> 2 & 1) + 4 * (n >> 3 & 1) + (n & 3);

    Stage stage;
    auto page_of = [&](int i) { return i < to ? kv_page(c, b, span.first_token(i) + 16 * wave) : -1; };
    auto load = [&](int i, int64_t page) { if (i < to) stage.load(c, h, page, span.first_token(i) + 16 * wave); };
    int64_t ahead = page_of(from);
    load(from, ahead);
    ahead = page_of(from + 1);
    if (from < to) stage.store(c, lds[0], wave);
    load(from + 1, ahead);
    ahead = page_of(from + 2);
    __syncthreads();

    for (int i = from; i < to; ++i) {
        const char* keys = lds[(i - from) & 1];
        const char* vals = keys + Stage::kKeyBytes;
        const float* gains = reinterpret_cast<const float*>(vals + kManyTile * D * 2);
        const int t0 = span.first_token(i);
        if (i + 1 < to) stage.store(c, lds[(i - from + 1) & 1], wave);
        load(i + 2, ahead);
        ahead = page_of(i + 3);

        floatx16_ st[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int r = 0; r < 16; ++r) st[x][r] = 0.f;
            const char* p = keys + (32 * x + tok) * Stage::kKeyPitch + 16 * half;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uintx4 w = *reinterpret_cast<const uintx4*>(p + 32 * k);
                st[x] = kv_mfma32<F>(w, q[k], st[x]);
                if constexpr (LOW) st[x] = kv_mfma32<F>(w, ql[k], st[x]);
            }
        }
        // register r of st[x]: token 32 x + 16 (r / 8) + 8 half + r % 8
        if constexpr (codes) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[x][r] *= gains[32 * x + 16 * (r >> 3) + 8 * half + (r & 7)];
        }
        uint32_t absent = 0;                        // quarters of 16 tokens whose page is missing
#pragma unroll
        for (int u = 0; u < 4; ++u) absent |= kv_page(c, b, t0 + 16 * u) < 0 ? 1u << u : 0u;
        const bool full = !absent && t0 + kManyTile - 1 <= pos0 &&
                          (!a.window || (int64_t)t0 > (int64_t)pos1 - a.window || t0 + kManyTile <= a.sinks);
        uint64_t dirty = 0;                         // tokens with a value that is no finite number, seen by some rows and not by others
        if (!full) {
            uint64_t none = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) none |= absent >> u & 1 ? 0xffffull << 16 * u : 0;
            const uint64_t sinks = many_below(a.sinks - (int64_t)t0);
            const uint64_t mine = (many_below((int64_t)pos - t0 + 1) & ~none & (a.window ? ~many_below((int64_t)pos - a.window + 1 - t0) | sinks : ~0ull)) >> 8 * half;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(mine >> (32 * x + 16 * (r >> 3) + (r & 7)) & 1)) st[x][r] = -INFINITY;
            // What no row of the workgroup sees may be anything, and 0 * NaN is no zero: such values are set to zero in LDS.  So are
            // values of no finite number that only some rows see; those rows get them one by one below.
            if constexpr (!codes) {
                const uint64_t shown = many_below((int64_t)span.end - t0) & ~none & (~many_below((int64_t)span.low - t0) | sinks);
                if (threadIdx.x < 2) odd[threadIdx.x] = 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    const int u = threadIdx.x + 256 * j;
                    const uint32_t bad = kv_not_finite<bf>(*reinterpret_cast<const uintx4*>(vals + u * 16)) << 8 * (u / D & 3);
                    if (bad) atomicOr(odd + u / D / 4, bad);
                }
                __syncthreads();
                const uint64_t found = (uint64_t)(uint32_t)kv_uniform((int)odd[0]) | (uint64_t)(uint32_t)kv_uniform((int)odd[1]) << 32;
                dirty = found & shown;
                const uint64_t keep = shown & ~found;
                if (~keep) {
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) {
                        const int u = threadIdx.x + 256 * j;
                        const uint32_t bits = (uint32_t)(keep >> 8 * (u / D));
                        uintx4* p = reinterpret_cast<uintx4*>(const_cast<char*>(vals) + u * 16);
                        uintx4 w = *p;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] &= (bits >> 2 * e & 1 ? 0xffffu : 0u) | (bits >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
                        *p = w;
                    }
                }
                __syncthreads();
            }
        }
        float top = st[0][0];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, st[x][r]);
        top = kv_max32(top) * gain;
        // 16 bits: a row's maximum may lag by 2^8, weights of up to 256 lose nothing; with codes they meet the norms in float16
        const bool grows = top > m + (codes || m == -INFINITY ? 0.f : 8.f);
        if (__ballot(grows)) {
            const float turn = grows ? __builtin_amdgcn_exp2f(m - top) : 1.f;
            m = grows ? top : m;
            l *= turn;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) o[k] *= turn;
        }
        const float less = m == -INFINITY ? 0.f : m;              // a row that has seen nothing: every score is -infinity
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int u = 0; u < 2; ++u) {           // 16 tokens: this lane's half of them in registers 8 u ..
                float pr[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    pr[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[x][8 * u + e], gain, -less));
                    l += pr[e];
                }
                const int og = 4 * x + 2 * u + half;             // group of eight tokens in the tile
                uintx4 p;
                if constexpr (codes) {
                    float w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = pr[e] * gains[kManyTile + 8 * og + e];
                    if (!full) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = st[x][8 * u + e] == -INFINITY ? 0.f : w[e];
                    }
                    p = uintx4{kv_pack2<bf>(w[0], w[2]), kv_pack2<bf>(w[4], w[6]), kv_pack2<bf>(w[1], w[3]), kv_pack2<bf>(w[5], w[7])};
                } else {
                    p = uintx4{kv_pack2<bf>(pr[0], pr[1]), kv_pack2<bf>(pr[2], pr[3]), kv_pack2<bf>(pr[4], pr[5]), kv_pack2<bf>(pr[6], pr[7])};
                }
#pragma unroll
                for (int k = 0; k < D / 32; ++k) o[k] = kv_mfma32<F>(*reinterpret_cast<const uintx4*>(vals + (og * D + 32 * k + n) * 16), p, o[k]);
            }
        for (uint64_t left = dirty; left; left &= left - 1) {           // such tokens one by one, for the rows that see them
            const int t = __builtin_ctzll(left);
            float v = -INFINITY;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) v = 32 * x + 16 * (r >> 3) + (r & 7) == (t & ~8) ? st[x][r] : v;
            v = __shfl(v, n + 32 * (t >> 3 & 1));
            const int64_t page = kv_page(c, b, t0 + t);
            const int in = (t0 + t) & (c.page - 1);
            const uint16_t* y = reinterpret_cast<const uint16_t*>(kv_record(c, page < 0 ? 0 : page, h) + c.page * (D * 2)) + (in >> 3) * D * 8 + (in & 7);
            if (v == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(v, gain, -less));
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[k][r] += w * kv_to_float<bf>(y[(32 * k + 8 * (r >> 2) + 4 * half + (r & 3)) * 8]);
        }
        __syncthreads();
    }
    l = kv_sum32(l);
    if (col >= cols) return;
    const float inv = f.parts > 1 ? 1.f : (l == 0.f ? 0.f : 1.f / l);
    const int64_t row_head = qrow * a.q.heads + qhead, all = (int64_t)a.q.rows * a.q.heads;
    // register r of o[k]: coordinate 32 k + 8 (r / 4) + 4 half + r % 4
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int j = 32 * k + 2 * r + 4 * half;
            if (codes || f.parts > 1) {
                *reinterpret_cast<float4*>(f.whole + (part * all + row_head) * D + j) =
                    make_float4(o[k][r] * inv, o[k][r + 1] * inv, o[k][r + 2] * inv, o[k][r + 3] * inv);
            } else {
                uint16_t* p = reinterpret_cast<uint16_t*>(a.out.data) + qrow * a.out.row_stride + qhead * a.out.head_stride + j;
                *reinterpret_cast<uint2*>(p) = make_uint2(kv_pack2<bf>(o[k][r] * inv, o[k][r + 1] * inv), kv_pack2<bf>(o[k][r + 2] * inv, o[k][r + 3] * inv));
            }
        }
    if (half) return;
    if (f.parts > 1) *reinterpret_cast<float2*>(f.part_ml + (part * all + row_head) * 2) = make_float2(m, l);
    else if (a.lse) a.lse[row_head] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
}

// Queries into the rotated frame: unit rows in float16, a second part with what the first rounds away, and their norms.
// Eights stand in the order of kv_levels8.  A wavefront takes 32 coordinates (blockIdx.y) of `tiles` times 16 rows: few
// rows are spread over many wavefronts (a chain of loads is what they cost), many share a block of Pi.
template <int D>
__global__ __launch_bounds__(64) void k_kv_rotate_queries(KvRows q, const float* __restrict__ pi, uint16_t* __restrict__ z, float* __restrict__ zn, int tiles) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4, block = blockIdx.y;
    const int64_t all = (int64_t)q.rows * q.heads;
    const KvTurn<D, false> turn(pi, block);
    for (int64_t tile = (int64_t)blockIdx.x * tiles; tile < ((int64_t)blockIdx.x + 1) * tiles && tile * 16 < all; ++tile) {
        const int64_t i = tile * 16 + n;
        const bool in = i < all;
        const int64_t row = in ? i / q.heads : 0, head = in ? i % q.heads : 0;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(q.data) + row * q.row_stride + head * q.head_stride + 8 * g;
        float x[D / 32][8], y[8];
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const uintx4 w = *reinterpret_cast<const uintx4*>(p + 32 * s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t bits = w[e >> 1] >> 16 * (e & 1) & 0xffff;
                x[s][e] = q.type == IVFTQ_KV_BF16 ? kv_to_float<true>(bits) : kv_to_float<false>(bits);
            }
        }
        const float norm = kv_unit_row<D>(x);
        turn(x, y);
        if (!in) continue;
        if (g == 0 && block == 0) zn[i] = norm;
        halfx8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = kv_slot(e);
            const float v = y[e] * kSplitScale;
            hi[at] = (_Float16)v;
            lo[at] = (_Float16)(v - (float)hi[at]);
        }
        *reinterpret_cast<halfx8*>(z + i * D + 32 * block + 8 * g) = hi;
        *reinterpret_cast<halfx8*>(z + (all + i) * D + 32 * block + 8 * g) = lo;
    }
}

// Parts of a row's result (one for each share of its keys) put together: eight coordinates from j on, divided by the sum of
// weights; lse where it is asked for.
template <int D>
__device__ __forceinline__ void many_join(const ManyArgs& f, int64_t i, int64_t all, int j, float (&x)[8], bool lse) {
    float top = -INFINITY, l = 0.f;
    for (int p = 0; p < f.parts; ++p) top = fmaxf(top, f.part_ml[(p * all + i) * 2]);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    for (int p = 0; p < f.parts; ++p) {
        const float2 u = *reinterpret_cast<const float2*>(f.part_ml + (p * all + i) * 2);
        const float turn = u.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u.x - top);
        const float4* w = reinterpret_cast<const float4*>(f.whole + (p * all + i) * D + j);
        const float4 a = w[0], b = w[1];
        l += u.y * turn;
        x[0] += a.x * turn; x[1] += a.y * turn; x[2] += a.z * turn; x[3] += a.w * turn;
        x[4] += b.x * turn; x[5] += b.y * turn; x[6] += b.z * turn; x[7] += b.w * turn;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    if (lse && f.a.lse) f.a.lse[i] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
}

// Rows that have a result: of a sequence, and not past max_new.
__device__ __forceinline__ bool many_has(const KvAttend& a, int64_t row) {
    if (!a.c.starts) return row < a.c.batch;
    int lo = 0, hi = a.c.batch;                     // first sequence that begins after the row, minus one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (kv_int(a.c.starts, mid) <= row) lo = mid; else hi = mid;
    }
    int first, count;
    kv_new_rows(a.c, lo, first, count);
    return row >= first && row < first + (count < a.max_new ? count : a.max_new);
}

template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_many_join(ManyArgs f) {
    const KvRows& out = f.a.out;
    const int64_t all = (int64_t)out.rows * out.heads, u = (int64_t)blockIdx.x * 256 + threadIdx.x, i = u / (D / 8);
    const int j = (int)(u % (D / 8)) * 8;
    if (i >= all || !many_has(f.a, i / out.heads)) return;
    float x[8];
    many_join<D>(f, i, all, j, x, j == 0);
    constexpr bool bf = F == IVFTQ_KV_BF16;
    uint16_t* p = reinterpret_cast<uint16_t*>(out.data) + i / out.heads * out.row_stride + i % out.heads * out.head_stride + j;
    *reinterpret_cast<uintx4*>(p) = uintx4{kv_pack2<bf>(x[0], x[1]), kv_pack2<bf>(x[2], x[3]), kv_pack2<bf>(x[4], x[5]), kv_pack2<bf>(x[6], x[7])};
}

// Results back into the rows' own frame, split the same way.
template <int D>
__global__ __launch_bounds__(64) void k_kv_rotate_back(ManyArgs f, int tiles) {
    const KvRows& out = f.a.out;
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
    const int64_t all = (int64_t)out.rows * out.heads;
    const KvTurn<D, true> turn(f.a.c.rotation, blockIdx.y);
    for (int64_t tile = (int64_t)blockIdx.x * tiles; tile < ((int64_t)blockIdx.x + 1) * tiles && tile * 16 < all; ++tile) {
        const int64_t i = tile * 16 + n;
        const bool in = i < all && many_has(f.a, i / out.heads);
        float x[D / 32][8], y[8];
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = 0.f;
            if (!in) continue;
            if (f.parts > 1) {
                many_join<D>(f, i, all, 32 * s + 8 * g, x[s], s == 0 && g == 0 && blockIdx.y == 0);
            } else {
                const float4* w = reinterpret_cast<const float4*>(f.whole + i * D + 32 * s + 8 * g);
                const float4 a = w[0], b = w[1];
                x[s][0] = a.x; x[s][1] = a.y; x[s][2] = a.z; x[s][3] = a.w; x[s][4] = b.x; x[s][5] = b.y; x[s][6] = b.z; x[s][7] = b.w;
            }
        }
        const float norm = kv_unit_row<D>(x) * f.a.c.level_unit;
        turn(x, y);
        if (in) kv_store_turned(out, i / out.heads, i % out.heads, blockIdx.y, y, norm);
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------

// Sizes of the workspace's parts, as the launch and the caller's question see them.
struct KvWork {
    int64_t z, zn, whole, part, ml, bytes;
    int32_t few, col_tiles, split, row_tiles, parts;
};
KvWork kv_work(int format, int d, int batch, int kv_heads, int64_t rows, int q_heads, int max_new, int64_t capacity);

template <int F, int D>
hipError_t kv_attend_launch(const KvAttend& a, const KvWork& w, hipStream_t st) {
    uint16_t* z = reinterpret_cast<uint16_t*>(a.work + w.z);
    float *zn = reinterpret_cast<float*>(a.work + w.zn), *whole = reinterpret_cast<float*>(a.work + w.whole), *ml = reinterpret_cast<float*>(a.work + w.ml);
    const int64_t all = (int64_t)a.q.rows * a.q.heads;
    const int tiles = all >= 16384 ? 8 : 1;              // 16-row tiles a wavefront rotates
    const dim3 rot((unsigned)((all + 16 * tiles - 1) / (16 * tiles)), D / 32);
    if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_queries<D><<<rot, 64, 0, st>>>(a.q, a.c.rotation, z, zn, tiles);
    const unsigned pairs = (unsigned)(a.c.batch * a.c.heads);
    if (w.few) {
        static ChipFill fill;
        unsigned wgs = 0;
        if (w.split) {
            if (hipError_t e = fill.get(reinterpret_cast<const void*>(&k_kv_few<F, D>), 256, 0, &wgs)) return e;
            if (wgs > (unsigned)kFewMaxWgs) wgs = kFewMaxWgs;
        }
        FewArgs f{a, z, zn, whole, reinterpret_cast<float*>(a.work + w.part), ml, (int32_t)wgs, w.split};
        k_kv_few<F, D><<<dim3(w.split ? wgs : pairs, (unsigned)w.col_tiles), 256, 0, st>>>(f);
        if (w.split || F == IVFTQ_KV_CODE4) k_kv_few_join<F, D><<<dim3(pairs, (unsigned)w.col_tiles), 512, 0, st>>>(f);
    } else {
        ManyArgs f{a, z, zn, whole, ml, w.row_tiles, w.parts};
        const unsigned wgs = pairs * (unsigned)w.row_tiles * (unsigned)w.parts;
        // float16 results: the queries' second part matters beside the rounding of the result
        if (F == IVFTQ_KV_CODE4 && a.q.type == IVFTQ_KV_F16) k_kv_many<F, D, F == IVFTQ_KV_CODE4><<<wgs, 256, 0, st>>>(f);
        else k_kv_many<F, D, false><<<wgs, 256, 0, st>>>(f);
        if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_back<D><<<rot, 64, 0, st>>>(f, tiles);
        else if (w.parts > 1) k_kv_many_join<F, D><<<(unsigned)((all * (D / 8) + 255) / 256), 256, 0, st>>>(f);
    }
    return hipGetLastError();
}

template <int D>
hipError_t kv_attend_d(const KvAttend& a, const KvWork& w, int format, hipStream_t st) {
    switch (format) {
        case IVFTQ_KV_F16: return kv_attend_launch<IVFTQ_KV_F16, D>(a, w, st);
        case IVFTQ_KV_BF16: return kv_attend_launch<IVFTQ_KV_BF16, D>(a, w, st);
        default: return kv_attend_launch<IVFTQ_KV_CODE4, D>(a, w, st);
    }
}

}  // namespace ivftq
