// Attention over the paged cache for many new rows a sequence (prompts, chunks of prompts): bound by the matrix cores and the
// exponentials beside them.
//
// A workgroup of four wavefronts owns 128 query rows of one (sequence, key-value head): rows are (token, head of the
// group) pairs, so the group's heads share every key and value that is read.  It walks the visible keys in tiles of 64
// tokens, staged in LDS (16-bit pages are copied, codes become float16 levels on the way).  As in kv_few.h the products
// are transposed, S^T = K Q^T and O^T = V^T P^T (v_mfma 32x32x16), and the token order of the key operand is chosen so
// that the scores a lane gets are those it puts into the second product: nothing goes through LDS but keys and values.
// Two workgroups a compute unit, which are not in step; inside a wavefront the products of one half tile stand between the
// exponentials of another.
//
// Measured: a prompt of 8,192 tokens, 32 heads of 128 over 8, window 4,096, bfloat16: 435 us, 0.95 PFLOP/s (an 8192^3 library
// product: 1.18), products 48 % of the cycles and vector instructions 42 %.  Chunks of 512 rows over 20,000 tokens in codes: 429 us,
// 0.63 PFLOP/s, vector instructions 54 %, a third of them for the levels, products 28 %.
#pragma once
#include <type_traits>

#include "kv_few.h"

namespace ivftq {

typedef float floatx16_ __attribute__((ext_vector_type(16)));

constexpr int kManyRows = 128;        // query rows of a workgroup
constexpr int kManyTile = 64;         // tokens of a step
constexpr int kTurnTiles = 8;         // tiles of 16 rows that a workgroup rotates where there are many

struct ManyArgs {
    KvAttend a;
    const uint16_t* z;                // codes: rotated unit queries, two float16 parts, eights in the order of kv_levels8
    const float* zn;                  // codes: the queries' norms
    float* whole;                     // codes: results before they are rotated back
    float* part;                      // shared tiles: [2 * workgroups][kManyRows][D] unnormalised sums
    float* part_ml;                   // [2 * workgroups][kManyRows][2] reference (in log2 units), sum of weights
    int64_t* begin;                   // a share's tiles, then [sequence][row tile] where a row tile begins among its head's tiles
    int32_t row_tiles, wgs;           // row tiles a (sequence, head): those of max_new; workgroups a head that share the tiles
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

// What a workgroup works on: one row tile (of 128 query rows) of a sequence.
struct ManyRowTile {
    FewSeq s;
    int cols, pos0, pos1;             // query rows of the sequence, positions of the first and the last row
    ManySpan span;
    __device__ __forceinline__ ManyRowTile(const KvAttend& a, int b, int rt) : s(few_seq(a, b)), cols(s.count * a.group) {
        const int last = (rt + 1) * kManyRows < cols ? (rt + 1) * kManyRows - 1 : cols - 1;
        pos0 = s.base + rt * kManyRows / a.group;
        pos1 = s.base + last / a.group;
        span = many_span(a, pos0, pos1);
        if (rt * kManyRows >= cols) span.tiles = 0;
        else if (!span.tiles) span.tiles = 1;             // rows that see nothing keep one tile, all of it masked
    }
};

// Where there are fewer row tiles than workgroups that keep the chip busy, or not many more, the key tiles of a head's row tiles, one
// after the other, are dealt out in equal consecutive shares, as in kv_few.h: a row tile that lies whole in a share is finished there, of
// the others each workgroup leaves at most two parts.  (Chunks of two sequences over 20,000 and 12,000 tokens in codes: the call
// 505 us with every row tile's keys cut in two, the longer sequence's workgroups last, and 474 us in equal shares; 737 us uncut.)
// Shares of few tiles are not worth their search and their parts (a prompt of 3,000 tokens, 94 row tiles a head, 35 tiles a share: 187
// us in shares, 102 us uncut); only the device knows the lengths, so it decides.
constexpr int kLeastShare = 64;
struct ManyShare { int64_t size; int b, rt, from, to; int64_t begin; };       // from, to: tiles of the row tile; begin: its first one's place

// The part of share `w` from its tile `x` on (x < size); to == from where there is none.
__device__ __forceinline__ ManyShare many_share(const KvAttend& a, int row_tiles, int wgs, int w, int64_t x) {
    const int lane = threadIdx.x & 63, items = a.c.batch * row_tiles;
    int tiles = 0;
    int64_t incl = 0;
    auto scan = [&](int e0) __attribute__((always_inline)) {
        const int e = e0 + lane;
        tiles = e < items ? ManyRowTile(a, e / row_tiles, e % row_tiles).span.tiles : 0;
        incl = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int64_t u = __shfl_up(incl, o); if (lane >= o) incl += u; }
        return kv_uniform((int64_t)__shfl(incl, 63));
    };
    int64_t total = 0;
    for (int e0 = 0; e0 < items; e0 += 64) total += scan(e0);
    ManyShare s{(total + wgs - 1) / wgs, 0, 0, 0, 0, 0};
    if (s.size < kLeastShare) {                       // a row tile a workgroup, those with the longest reach first; all lie in one share
        s.size = (int64_t)1 << 60;
        if (x == 0 && w < items) {
            s.b = w % a.c.batch;
            s.rt = row_tiles - 1 - w / a.c.batch;
            s.to = ManyRowTile(a, s.b, s.rt).span.tiles;
        }
        return s;
    }
    const int64_t at = w * s.size + x, end = (w + 1) * s.size < total ? (w + 1) * s.size : total;
    int64_t base = 0;
    for (int e0 = 0; at < end && e0 < items; e0 += 64) {
        const int64_t all = items <= 64 ? total : scan(e0);
        const uint64_t past = __ballot(base + incl > at);
        if (past) {
            const int l = __builtin_ctzll(past), e = e0 + l, n = kv_uniform(__shfl(tiles, l));
            s.b = e / row_tiles;
            s.rt = e % row_tiles;
            s.begin = base + kv_uniform((int64_t)__shfl(incl - tiles, l));
            s.from = (int)(at - s.begin);
            s.to = (int)(end - s.begin < n ? end - s.begin : n);
            break;
        }
        base += all;
    }
    return s;
}

// A tile in LDS.  Keys: rows of kRow 16-byte chunks, chunk w of token t in place w ^ turn(t), so that sixteen lanes that read one
// chunk of sixteen tokens use all banks; values: groups of eight tokens as they stand in a page; codes: the norms behind.
// A wavefront brings a quarter, 16 tokens, which lie in one page: 16 bits by loads that go to LDS directly (64 lanes write 1 KB
// in order, which is why keys are turned by choosing what a lane reads), codes through registers, where they become levels.
template <int F, int D>
struct ManyTile {
    static constexpr bool kCodes = F == IVFTQ_KV_CODE4;
    static constexpr int kRow = D <= 64 ? 8 : (D <= 128 ? 16 : 32);
    static constexpr int kKeyBytes = kManyTile * kRow * 16, kValueBytes = kManyTile * D * 2;
    char keys[2][kKeyBytes];
    char values[2][kValueBytes];
    // norms have four places: a tile's are written, a tile ahead, while others may still be at the tile before and read its own
    float key_gain[kCodes ? 4 : 1][kCodes ? kManyTile : 1], value_gain[kCodes ? 4 : 1][kCodes ? kManyTile : 1];
    float value_power[kCodes ? 4 : 1][4];      // of the quarters' largest norms
    alignas(8) uint16_t odd[2][4];             // masked tiles: tokens of each quarter with a value that is no finite number

    static __device__ __forceinline__ int turn(int t) { return kRow == 8 ? t >> 1 & 7 : t & 15; }
};

template <int F, int D>
struct ManyStage {
    using Tile = ManyTile<F, D>;
    static constexpr bool kCodes = F == IVFTQ_KV_CODE4;
    uint32_t k[kCodes ? D / 32 : 1], v[kCodes ? D / 32 : 1];      // eight coordinates of a key, eight tokens of a value
    uint32_t norm;                // lanes 0 .. 15: of the quarter's keys, 16 .. 31: of its values

    // keys (values) of a tile's quarter, which begins with token `in` of record `rec`, to buffer `to` of LDS
    __device__ __forceinline__ void bring_keys(const KvView& c, const char* rec, int in, Tile& lds, int to, int quarter) {
        const int lane = threadIdx.x & 63;
        if constexpr (kCodes) {
            const uint32_t* x = reinterpret_cast<const uint32_t*>(rec + in * (D / 2));
#pragma unroll
            for (int j = 0; j < D / 32; ++j) k[j] = x[lane + 64 * j];
            norm = reinterpret_cast<const uint16_t*>(rec + c.page * D)[(lane & 16 ? c.page : 0) + in + (lane & 15)];
        } else {
            // lane's place in the first 64 chunks; the next 64 are kRows rows on, where chunks are turned by a further xor
            constexpr int kRows = 64 / Tile::kRow, kTurn = Tile::kRow == 8 ? kRows / 2 : kRows;
            const char* from = rec + in * (D * 2);
            const uint32_t row = lane / Tile::kRow, chunk = (lane % Tile::kRow) ^ (Tile::kRow == 8 ? row / 2 : row);
#pragma unroll
            for (int j = 0; j < Tile::kRow / 4; ++j) {
                uint32_t w = chunk ^ (kTurn * j);
                if (D / 8 < Tile::kRow) w = w < D / 8 ? w : 0;                       // rows of 96 and 192: chunks that nobody reads
                kv_load_lds16(from + (row * (D * 2) + w * 16 + j * kRows * D * 2), lds.keys[to] + (quarter * 16 * Tile::kRow + 64 * j) * 16);
            }
        }
    }
    __device__ __forceinline__ void bring_values(const KvView& c, const char* rec, int in, Tile& lds, int to, int quarter) {
        const int lane = threadIdx.x & 63;
        if constexpr (kCodes) {
            const uint32_t* x = reinterpret_cast<const uint32_t*>(rec + (c.page + in) * (D / 2));
#pragma unroll
            for (int j = 0; j < D / 32; ++j) v[j] = x[lane + 64 * j];
        } else {
            const char* from = rec + (c.page + in) * (D * 2);
#pragma unroll
            for (int j = 0; j < D / 32; ++j) kv_load_lds16(from + (uint32_t)(lane * 16 + j * 1024), lds.values[to] + (quarter * 2 * D + 64 * j) * 16);
        }
    }
    // codes: what has been brought, into LDS
    __device__ __forceinline__ void store_keys(const KvView& c, Tile& lds, int to, int gain_to, int quarter) const {
        if constexpr (kCodes) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                const int u = lane + 64 * j, row = u / (D / 8), w = u % (D / 8);
                *reinterpret_cast<halfx8*>(lds.keys[to] + ((16 * quarter + row) * Tile::kRow + (w ^ Tile::turn(row))) * 16) = kv_levels8(k[j], c);
            }
            uint32_t most = norm;
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) { const uint32_t other = __shfl_xor(most, o); most = most > other ? most : other; }
            if (lane == 16) lds.value_power[gain_to][quarter] = kv_norm_power(most);
            if (lane < 32) (lane < 16 ? lds.key_gain : lds.value_gain)[gain_to][16 * quarter + (lane & 15)] = (float)__builtin_bit_cast(_Float16, (uint16_t)norm);
        }
    }
    __device__ __forceinline__ void store_values(const KvView& c, Tile& lds, int to, int quarter) const {
        if constexpr (kCodes) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) *reinterpret_cast<halfx8*>(lds.values[to] + (quarter * 2 * D + lane + 64 * j) * 16) = kv_levels8(v[j], c);
        }
    }
};

// A wavefront's priority on its SIMD: highest where products stand between exponentials, lowest where codes become levels and at the
// barrier, so that the other workgroup's wavefront takes the gaps (chunks over codes 465 -> 448 us, a long prompt 444 -> 435).  Heads of 64
// coordinates, three wavefronts a SIMD: not (ragged prompts 41 -> 44 us).
template <int D, int P>
__device__ __forceinline__ void many_priority() { if constexpr (D >= 96) __builtin_amdgcn_s_setprio(P); }

// The lowest n bits.
__device__ __forceinline__ uint64_t many_below(int64_t n) { return n <= 0 ? 0 : (n >= 64 ? ~0ull : (1ull << n) - 1); }

template <int F, int D, bool LOW, bool SHARED>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_kv_many(ManyArgs f) {
    using Tile = ManyTile<F, D>;
    constexpr int kSteps = D / 16;               // matrix instructions of a half tile's scores, and of its values
    constexpr int kLead = 3;                     // operands that are read ahead
    constexpr bool codes = F == IVFTQ_KV_CODE4, bf = F == IVFTQ_KV_BF16;
    __shared__ __align__(1024) Tile lds;
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
    // heads fastest: with eight heads each XCD reads one head's pages; then shares, or sequences and the row tiles with the longest
    // reach first
    const int h = (int)(kv_workgroup() % (uint32_t)c.heads), share = (int)(kv_workgroup() / (uint32_t)c.heads);
    int64_t x = 0;                               // the share's tiles that are done
  while (true) {                                 // a row tile, or what of it lies in the share
    int b, rt, from = 0, to = 0;
    bool last_part = true;
    if constexpr (SHARED) {
        const ManyShare now = many_share(a, f.row_tiles, f.wgs, share, x);
        if (threadIdx.x == 0 && share == 0 && h == 0 && x == 0) f.begin[0] = now.size;
        if (now.from >= now.to) return;
        b = now.b; rt = now.rt; from = now.from; to = now.to;
        if (threadIdx.x == 0 && h == 0 && from == 0) f.begin[1 + b * f.row_tiles + rt] = now.begin;
        last_part = x + (to - from) >= now.size || now.size > (int64_t)1 << 59;
        if (x) __syncthreads();                  // LDS is no longer read
    } else {
        b = share % c.batch;
        rt = f.row_tiles - 1 - share / c.batch;
        if (rt < 0) return;
    }
    const ManyRowTile tile(a, b, rt);
    const FewSeq& s = tile.s;
    const ManySpan& span = tile.span;
    const int cols = tile.cols, pos0 = tile.pos0, pos1 = tile.pos1;
    if (!SHARED) {
        if (rt * kManyRows >= cols) return;
        to = span.tiles;
    }
    const int col = rt * kManyRows + wave * 32 + n, used = col < cols ? col : cols - 1;
    const int pos = s.base + used / a.group;
    const int64_t qrow = s.first + used / a.group;
    const int qhead = h * a.group + used % a.group;

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

    ManyStage<F, D> stage;
    // What is known of a tile ahead of its turn: its first token, the record with this wavefront's quarter, quarters without a page.
    struct Ahead { int t; const char* rec; uint32_t absent; };
    const int32_t* const row = c.table + (int64_t)b * c.table_stride;
    const char* const head = c.pool + (int64_t)h * c.head_bytes;
    const int32_t pages = (int32_t)c.pages;
    // lane u % 4 asks for the page of quarter u % 4; the answer is taken up one tile later
    auto ask = [&](int i) __attribute__((always_inline)) {
        const int col = (span.first_token(i < to ? i : from) + 16 * (lane & 3)) >> c.page_log2;
        return col < c.columns ? row[col] : -1;
    };
    auto answer = [&](int i, int32_t id) __attribute__((always_inline)) {
        const bool none = (uint32_t)id >= (uint32_t)pages;
        const int32_t mine = __builtin_amdgcn_readlane(none ? 0 : id, wave);
        return Ahead{span.first_token(i < to ? i : from), head + (int64_t)mine * c.page_bytes, (uint32_t)__ballot(none) & 15u};
    };
    auto bring_keys = [&](int i, const Ahead& at, int buffer) __attribute__((always_inline)) {
        if (i < to) stage.bring_keys(c, at.rec, (at.t + 16 * wave) & (c.page - 1), lds, buffer, wave);
    };
    auto bring_values = [&](int i, const Ahead& at, int buffer) __attribute__((always_inline)) {
        if (i < to) stage.bring_values(c, at.rec, (at.t + 16 * wave) & (c.page - 1), lds, buffer, wave);
    };
    // S^T of tokens 32 x .. of a tile; register r: token 32 x + 16 (r / 8) + 8 half + r % 8
    const int key_at = tok * (Tile::kRow * 16) + ((half ^ Tile::turn(tok)) << 4);
    auto key_chunk = [&](int buffer, int x, int k) __attribute__((always_inline)) {
        return *reinterpret_cast<const uintx4*>(lds.keys[buffer] + 32 * x * (Tile::kRow * 16) + (key_at ^ (k << 5)));
    };
    auto value_chunk = [&](int buffer, int x, int j) __attribute__((always_inline)) {       // j: (16 tokens, block of 32 coordinates)
        return *reinterpret_cast<const uintx4*>(lds.values[buffer] + ((4 * x + 2 * (j / (D / 32)) + half) * D + 32 * (j % (D / 32)) + n) * 16);
    };
    auto score = [&](const uintx4& w, int k, floatx16_& st) __attribute__((always_inline)) {
        st = kv_mfma32<F>(w, q[k], st);
        if constexpr (LOW) st = kv_mfma32<F>(w, ql[k], st);
    };
    auto scores = [&](int buffer, int x, floatx16_& st) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) score(key_chunk(buffer, x, k), k, st);
    };
    auto product = [&](int buffer, int x, const uintx4 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) o[j % (D / 32)] = kv_mfma32<F>(value_chunk(buffer, x, j), p[j / (D / 32)], o[j % (D / 32)]);
    };
    // Each matrix instruction is followed by the vector instructions of a part of the sixteen scores, and the LDS read of the
    // one kLead further on stands before it; the compiler may not move anything from one such group to another (left alone it puts the
    // matrix instructions first, and the wavefront stands still behind them).
    //
    // O^T += V^T P^T of tokens 32 x .. of `buffer`; the maximum of the scores st of half `y` of tile `tile` (codes: times the
    // keys' norms; mine: the tokens that this lane's row sees, a bit each, from this lane's half on).
    auto product_and_maximum = [&](int buffer, int x, const uintx4 (&p)[2], int tile, int y, bool full, uint32_t mine, floatx16_& st) __attribute__((always_inline)) {
        uintx4 w[kSteps];
#pragma unroll
        for (int j = 0; j < kLead; ++j) w[j] = value_chunk(buffer, x, j);
        float gains[16];
        if constexpr (codes) {
#pragma unroll
            for (int r = 0; r < 16; ++r) gains[r] = lds.key_gain[(tile - from) & 3][32 * y + 8 * half + 16 * (r >> 3) + (r & 7)];
        }
        if (!full) {                                // (a norm that is no number: the product comes before the mask)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if constexpr (codes) { st[r] *= gains[r]; gains[r] = 1.f; }
                st[r] = mine >> (16 * (r >> 3) + (r & 7)) & 1 ? st[r] : -INFINITY;
            }
        }
        float power = 0.f;
        if constexpr (codes) {
            power = fmaxf(lds.value_power[(tile - from) & 3][2 * y], lds.value_power[(tile - from) & 3][2 * y + 1]);
            if (!full) {                            // of the tokens that the row sees: others' norms may be anything
                float most = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = lds.value_gain[(tile - from) & 3][32 * y + 8 * half + 16 * (r >> 3) + (r & 7)];
                    most = fmaxf(most, mine >> (16 * (r >> 3) + (r & 7)) & 1 ? v : 0.f);
                }
                const int e = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 126;
                power = (float)(e < -14 ? -14 : (e > 17 ? 17 : e));
            }
        }
        float top = -INFINITY;
        many_priority<D, 1>();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            if (j + kLead < kSteps) w[j + kLead] = value_chunk(buffer, x, j + kLead);
            o[j % (D / 32)] = kv_mfma32<F>(w[j], p[j / (D / 32)], o[j % (D / 32)]);
#pragma unroll
            for (int r = 16 * j / kSteps; r < 16 * (j + 1) / kSteps; ++r) {
                if constexpr (codes) st[r] *= gains[r];
                top = fmaxf(top, st[r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        top = codes && !full ? kv_max32(__builtin_fmaf(top, gain, power)) : __builtin_fmaf(kv_max32(top), gain, power);
        const bool grows = top > m + kWeightRoom<F>;
        top -= kWeightLift<F>;
        if (__ballot(grows)) {
            const float turn = grows ? __builtin_amdgcn_exp2f(m - top) : 1.f;
            m = grows ? top : m;
            l *= turn;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) o[k] *= turn;
        }
    };
    // S^T of tokens 32 x .. of `buffer` into `next`; the weights of the scores st of half `y` of tile `tile`.
    auto scores_and_weights = [&](int buffer, int x, floatx16_& next, int tile, int y, bool full, uint32_t mine, const floatx16_& st, uintx4 (&p)[2]) __attribute__((always_inline)) {
        uintx4 w[kSteps];
#pragma unroll
        for (int k = 0; k < kLead; ++k) w[k] = key_chunk(buffer, x, k);
        const float less = m == -INFINITY ? 0.f : m;              // a row that has seen nothing: every score is -infinity
        float gains[16], pr[16];
        if constexpr (codes) {
#pragma unroll
            for (int r = 0; r < 16; ++r) gains[r] = lds.value_gain[(tile - from) & 3][32 * y + 8 * half + 16 * (r >> 3) + (r & 7)];
            if (!full) {
#pragma unroll
                for (int r = 0; r < 16; ++r) gains[r] = mine >> (16 * (r >> 3) + (r & 7)) & 1 ? gains[r] : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) next[r] = 0.f;
        many_priority<D, 2>();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            if (k + kLead < kSteps) w[k + kLead] = key_chunk(buffer, x, k + kLead);
            score(w[k], k, next);
#pragma unroll
            for (int r = 16 * k / kSteps; r < 16 * (k + 1) / kSteps; ++r) {
                pr[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[r], gain, -less));
                l += pr[r];
                const int e = r & 7, u = r >> 3;
                if constexpr (codes) {                            // in the order of kv_levels8
                    pr[r] *= gains[r];
                    if (e & 2) p[u][(e & 1) * 2 + (e >> 2)] = kv_here(kv_pack2<false>(pr[r - 2], pr[r]));
                } else if (e & 1) {
                    p[u][e >> 1] = kv_here(kv_pack2<bf>(pr[r - 1], pr[r]));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        many_priority<D, 0>();
    };
    // Values that are no finite numbers, of tokens that some rows see and others do not: for the rows that see them, one by one.
    auto singly = [&](int t0, int x, uint32_t dirty, const floatx16_& st) __attribute__((always_inline)) {
        const float less = m == -INFINITY ? 0.f : m;
        for (uint32_t left = dirty; left; left &= left - 1) {
            const int t = __builtin_ctz(left);
            float v = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) v = 16 * (r >> 3) + (r & 7) == (t & ~8) ? st[r] : v;
            v = __shfl(v, n + 32 * (t >> 3 & 1));
            const int64_t page = kv_page(c, b, t0 + 32 * x + t);
            const int in = (t0 + 32 * x + t) & (c.page - 1);
            const uint16_t* y = reinterpret_cast<const uint16_t*>(kv_record(c, page < 0 ? 0 : page, h) + c.page * (D * 2)) + (in >> 3) * D * 8 + (in & 7);
            if (v == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(v, gain, -less));
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[k][r] += w * kv_to_float<bf>(y[(32 * k + 8 * (r >> 2) + 4 * half + (r & 3)) * 8]);
        }
    };

    // The order of things: keys and norms of tile i + 1 and values of tile i are there when tile i's second half begins, half way
    // through tile i (one barrier a tile); what the buffers are then free for, keys of tile i + 2 and values of tile i + 1, is on its
    // way from there on.
    Ahead now = answer(from, ask(from)), next = answer(from + 1, ask(from + 1));
    bring_keys(from, now, 0);
    if constexpr (codes) { if (from < to) stage.store_keys(c, lds, 0, 0, wave); }
    bring_keys(from + 1, next, 1);
    bring_values(from, now, 0);
    int32_t asked = ask(from + 2);
    // the first tile's step begins with the product of weights of zero and the other buffer's values: those have to be numbers
    for (int u = threadIdx.x; u < kManyTile * D / 8; u += 256) *reinterpret_cast<uintx4*>(lds.values[1] + u * 16) = uintx4{0, 0, 0, 0};
    kv_loads_done();
    __syncthreads();
    floatx16_ s0, s1;
    uintx4 p0[2], p1[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (from < to) scores(0, 0, s0);

    // A tile.  While a half tile's scores become weights (vector unit), the weights of the half before meet their values and the
    // next half's scores are made (matrix cores): no product waits for the weights beside it.
    const int beyond = a.window && (int64_t)pos1 - a.window >= 0 ? (int)((int64_t)pos1 - a.window) : -1;       // tokens up to this one are not in every row's window
    auto step = [&](int i, auto buffer) __attribute__((always_inline)) {
        constexpr int here = decltype(buffer)::value, other = here ^ 1;
        const int t0 = now.t;
        const uint32_t absent = now.absent;
        const bool full = !absent && t0 + kManyTile - 1 <= pos0 && (t0 > beyond || t0 + kManyTile <= a.sinks);       // every row sees every token
        const Ahead then = answer(i + 2, asked);
        asked = ask(i + 3);
        uint64_t mine = ~0ull;
        [[maybe_unused]] uint64_t shown = ~0ull, dirty = 0;
        if constexpr (codes) {
            if (i + 1 < to) stage.store_keys(c, lds, other, (i + 1 - from) & 3, wave);
            stage.store_values(c, lds, here, wave);
            bring_keys(i + 2, then, here);
            bring_values(i + 1, next, other);
        }
        if (!full) {
            uint64_t none = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) none |= absent >> u & 1 ? 0xffffull << 16 * u : 0;
            const uint64_t sinks = many_below(a.sinks - (int64_t)t0);
            mine = (many_below((int64_t)pos - t0 + 1) & ~none & (a.window ? ~many_below((int64_t)pos - a.window + 1 - t0) | sinks : ~0ull)) >> 8 * half;
            shown = many_below((int64_t)span.end - t0) & ~none & (~many_below((int64_t)span.low - t0) | sinks);
        }
        product_and_maximum(other, 1, p1, i, 0, full, (uint32_t)mine, s0);
        scores_and_weights(here, 1, s1, i, 0, full, (uint32_t)mine, s0, p0);
        if constexpr (!codes) kv_loads_done();
        if (!codes && !full) {
            // What no row of the workgroup sees may be anything, and 0 * NaN is no zero: such values are set to zero in LDS, each quarter
            // by the wavefront that has brought it, before the others read it.  So are values of no finite number that only some rows
            // see; those rows get them one by one.
            uint32_t found = 0;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                found |= kv_not_finite<bf>(*reinterpret_cast<const uintx4*>(lds.values[here] + (wave * 2 * D + lane + 64 * j) * 16)) << 8 * ((lane + 64 * j) / D);
            if (__ballot(found != 0)) {
#pragma unroll
                for (int w = 1; w < 64; w <<= 1) found |= __shfl_xor(found, w);
            }
            found = kv_uniform((int)found);
            if (lane == 0) lds.odd[here][wave] = (uint16_t)found;
            const uint32_t keep = (uint32_t)(shown >> 16 * wave) & ~found;
            if (~keep & 0xffffu) {
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    const uint32_t bits = keep >> 8 * ((lane + 64 * j) / D);
                    uintx4* p = reinterpret_cast<uintx4*>(lds.values[here] + (wave * 2 * D + lane + 64 * j) * 16);
                    uintx4 w = *p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] &= (bits >> 2 * e & 1 ? 0xffffu : 0u) | (bits >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
                    *p = w;
                }
            }
        }
        __syncthreads();
        if (!codes && !full) {
            const uint32_t* odd = reinterpret_cast<const uint32_t*>(lds.odd[here]);
            dirty = ((uint64_t)(uint32_t)kv_uniform((int)odd[0]) | (uint64_t)(uint32_t)kv_uniform((int)odd[1]) << 32) & shown;
            if ((uint32_t)dirty) singly(t0, 0, (uint32_t)dirty, s0);
        }
        if constexpr (!codes) {
            bring_keys(i + 2, then, here);
            bring_values(i + 1, next, other);
        }
        now = next;
        next = then;
        product_and_maximum(here, 0, p0, i, 1, full, (uint32_t)(mine >> 32), s1);
        scores_and_weights(other, 0, s0, i, 1, full, (uint32_t)(mine >> 32), s1, p1);       // past the last tile: of what LDS holds, not used
        if constexpr (!codes) {
            if (dirty >> 32) singly(t0, 1, (uint32_t)(dirty >> 32), s1);
        }
    };
    for (int i = from; i < to; i += 2) {
        step(i, std::integral_constant<int, 0>{});
        if (i + 1 < to) step(i + 1, std::integral_constant<int, 1>{});
    }
    if (from < to) product((to - from - 1) & 1, 1, p1);
    l = kv_sum32(l);
    // register r of o[k]: coordinate 32 k + 8 (r / 4) + 4 half + r % 4
    const bool whole = !SHARED || (from == 0 && to == span.tiles);
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    const int64_t row_head = qrow * a.q.heads + qhead, slot = (((int64_t)h * f.wgs + share) * 2 + (from == 0)) * kManyRows + wave * 32 + n;
    if (col < cols) {
        float* to_float = whole ? f.whole + row_head * D : f.part + slot * D;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int j = 32 * k + 2 * r + 4 * half;
                const float4 v = make_float4(o[k][r] * inv, o[k][r + 1] * inv, o[k][r + 2] * inv, o[k][r + 3] * inv);
                if (codes || !whole) {
                    *reinterpret_cast<float4*>(to_float + j) = v;
                } else {
                    uint16_t* p = reinterpret_cast<uint16_t*>(a.out.data) + qrow * a.out.row_stride + qhead * a.out.head_stride + j;
                    *reinterpret_cast<uint2*>(p) = make_uint2(kv_pack2<bf>(v.x, v.y), kv_pack2<bf>(v.z, v.w));
                }
            }
        if (half == 0) {
            if (!whole) *reinterpret_cast<float2*>(f.part_ml + slot * 2) = make_float2(m, l);
            else if (a.lse) a.lse[row_head] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
        }
    }
    if (!SHARED || last_part) return;
    x += to - from;
  }
}

// 16 unit rows in LDS as operands of the rotation: each of the workgroup's D / 32 wavefronts brings 32 coordinates of them
// (x[e] = coordinate 32 wave + 8 (lane / 16) + e of row lane % 16, any length) and gets all; returns the rows' lengths.
template <int D>
struct UnitRows {
    halfx8 hi[D / 32][64], lo[D / 32][64];
    float square[D / 32][16];

    __device__ __forceinline__ float bring(const float (&x)[8]) {
        const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15;
        float n2 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) n2 += x[e] * x[e];
        n2 = kv_sum4(n2);
        __syncthreads();                            // the rows before are no longer read
        if (lane < 16) square[wave][n] = n2;
        __syncthreads();
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) sum += square[s][n];
        const float norm = sqrtf(sum), scale = norm > 0.f ? kSplitScale / norm : 0.f;
        halfx8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = x[e] * scale;
            h[e] = (_Float16)v;
            l[e] = (_Float16)(v - (float)h[e]);
        }
        hi[wave][lane] = h;
        lo[wave][lane] = l;
        __syncthreads();
        return norm;
    }
};

// Queries into the rotated frame: unit rows in float16, a second part with what the first rounds away, and their norms.
// Eights stand in the order of kv_levels8.  A workgroup takes `tiles` times 16 rows, each of its wavefronts a block of 32
// coordinates of the result (and of the rows that it reads).
template <int D>
__global__ __launch_bounds__(D * 2) void k_kv_rotate_queries(KvRows q, const float* __restrict__ pi, uint16_t* __restrict__ z, float* __restrict__ zn, int tiles) {
    __shared__ UnitRows<D> unit;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int64_t all = (int64_t)q.rows * q.heads;
    const KvTurn<D, false> turn(pi, wave);
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
        if (!in) continue;
        if (g == 0 && wave == 0) zn[i] = norm;
        halfx8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = kv_slot(e);
            const float v = y[e] * kSplitScale;
            hi[at] = (_Float16)v;
            lo[at] = (_Float16)(v - (float)hi[at]);
        }
        *reinterpret_cast<halfx8*>(z + i * D + 32 * wave + 8 * g) = hi;
        *reinterpret_cast<halfx8*>(z + (all + i) * D + 32 * wave + 8 * g) = lo;
    }
}

// Where a row's result is: parts in the shares first .. last of its head (one share: finished), row `row` of each part; last < 0: none,
// because the row is of no sequence or past max_new.
struct ManyPlace { int first, last, row; };
template <bool SHARED>
__device__ __forceinline__ ManyPlace many_place(const ManyArgs& f, int64_t row, int qhead) {
    const KvAttend& a = f.a;
    int lo = 0, hi = a.c.batch;                     // first sequence that begins after the row, minus one
    if (a.c.starts) {
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (kv_int(a.c.starts, mid) <= row) lo = mid; else hi = mid;
        }
    } else {
        lo = row < a.c.batch ? (int)row : 0;
    }
    int first, count;
    kv_new_rows(a.c, lo, first, count);
    const int64_t i = row - first;
    if (i < 0 || i >= (count < a.max_new ? count : a.max_new)) return {0, -1, 0};
    if constexpr (!SHARED) return {0, 0, 0};
    const int col = (int)i * a.group + qhead % a.group, rt = col / kManyRows;
    const int64_t size = f.begin[0], begin = f.begin[1 + lo * f.row_tiles + rt];
    return {(int)(begin / size), (int)((begin + ManyRowTile(a, lo, rt).span.tiles - 1) / size), col % kManyRows};
}

// Parts of a row's result put together: eight coordinates from j on, divided by the sum of weights; lse where it is asked for.
template <int D>
__device__ __forceinline__ void many_join(const ManyArgs& f, const ManyPlace& at, int64_t i, int j, float (&x)[8], bool lse) {
    const int64_t h = i % f.a.q.heads / f.a.group;
    auto slot = [&](int w) { return ((h * f.wgs + w) * 2 + (w == at.first)) * kManyRows + at.row; };
    float top = -INFINITY, l = 0.f;
    for (int w = at.first; w <= at.last; ++w) top = fmaxf(top, f.part_ml[slot(w) * 2]);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    for (int w = at.first; w <= at.last; ++w) {
        const float2 u = *reinterpret_cast<const float2*>(f.part_ml + slot(w) * 2);
        const float turn = u.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(u.x - top);
        const float4* p = reinterpret_cast<const float4*>(f.part + slot(w) * D + j);
        const float4 a = p[0], b = p[1];
        l += u.y * turn;
        x[0] += a.x * turn; x[1] += a.y * turn; x[2] += a.z * turn; x[3] += a.w * turn;
        x[4] += b.x * turn; x[5] += b.y * turn; x[6] += b.z * turn; x[7] += b.w * turn;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    if (lse && f.a.lse) f.a.lse[i] = l > 0.f ? (top + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
}

// Rows whose tiles lie in more than one share.
template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_many_join(ManyArgs f) {
    const KvRows& out = f.a.out;
    const int64_t all = (int64_t)out.rows * out.heads, u = (int64_t)kv_workgroup() * 256 + threadIdx.x, i = u / (D / 8);
    const int j = (int)(u % (D / 8)) * 8;
    if (i >= all) return;
    const ManyPlace at = many_place<true>(f, i / out.heads, (int)(i % out.heads));
    if (at.last <= at.first) return;
    float x[8];
    many_join<D>(f, at, i, j, x, j == 0);
    constexpr bool bf = F == IVFTQ_KV_BF16;
    uint16_t* p = reinterpret_cast<uint16_t*>(out.data) + i / out.heads * out.row_stride + i % out.heads * out.head_stride + j;
    *reinterpret_cast<uintx4*>(p) = uintx4{kv_pack2<bf>(x[0], x[1]), kv_pack2<bf>(x[2], x[3]), kv_pack2<bf>(x[4], x[5]), kv_pack2<bf>(x[6], x[7])};
}

// Results back into the rows' own frame, split the same way.
template <int D, bool SHARED>
__global__ __launch_bounds__(D * 2) void k_kv_rotate_back(ManyArgs f, int tiles) {
    __shared__ UnitRows<D> unit;
    __shared__ ManyPlace places[16 * kTurnTiles];
    const KvRows& out = f.a.out;
    const int wave = kv_wave(), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int64_t all = (int64_t)out.rows * out.heads, first = (int64_t)blockIdx.x * tiles * 16;
    for (int u = threadIdx.x; u < 16 * tiles; u += D * 2)
        places[u] = first + u < all ? many_place<SHARED>(f, (first + u) / out.heads, (int)((first + u) % out.heads)) : ManyPlace{0, -1, 0};
    const KvTurn<D, true> turn(f.a.c.rotation, wave);
    __syncthreads();
    for (int tile = 0; tile < tiles && first + tile * 16 < all; ++tile) {
        const int64_t i = first + tile * 16 + n;
        const ManyPlace at = places[tile * 16 + n];
        const bool in = at.last >= 0;
        float x[8] = {}, y[8];
        if (in) {
            const int j = 32 * wave + 8 * g;
            if (SHARED && at.last > at.first) {
                many_join<D>(f, at, i, j, x, j == 0);
            } else {
                const float4* w = reinterpret_cast<const float4*>(f.whole + i * D + j);
                const float4 a = w[0], b = w[1];
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
            }
        }
        const float norm = unit.bring(x) * f.a.c.level_unit;
        turn(unit, y);
        if (in) kv_store_turned(out, i / out.heads, i % out.heads, wave, y, norm);
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------

// Sizes of the workspace's parts, as the launch and the caller's question see them.
struct KvWork {
    int64_t z, zn, whole, part, ml, begin, bytes;
    int32_t few, col_tiles, split, row_tiles, shared;        // shared: workgroups a head that share its tiles, 0: one a row tile
};
KvWork kv_work(int format, int d, int batch, int kv_heads, int64_t rows, int q_heads, int max_new, int64_t capacity);

template <int F, int D>
hipError_t kv_attend_launch(const KvAttend& a, const KvWork& w, hipStream_t st) {
    uint16_t* z = reinterpret_cast<uint16_t*>(a.work + w.z);
    float *zn = reinterpret_cast<float*>(a.work + w.zn), *whole = reinterpret_cast<float*>(a.work + w.whole), *ml = reinterpret_cast<float*>(a.work + w.ml);
    const int64_t all = (int64_t)a.q.rows * a.q.heads;
    // a workgroup's 16-row tiles: many rows share the rotation's operands, where that leaves three workgroups a compute unit (27,000 rows
    // of 128: eight tiles each 18 us there and 33 us back, two 16 and 20); rows whose workspace fits a card are far from 2^32 threads
    const int64_t fill = all / (16 * 768);
    const int tiles = fill < 1 ? 1 : (fill < kTurnTiles ? (int)fill : kTurnTiles);
    const unsigned rot = (unsigned)((all + 16 * tiles - 1) / (16 * tiles));
    if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_queries<D><<<rot, D * 2, 0, st>>>(a.q, a.c.rotation, z, zn, tiles);
    const unsigned pairs = (unsigned)(a.c.batch * a.c.heads);
    if (w.few) {
        FewArgs f{a, z, zn, whole, reinterpret_cast<float*>(a.work + w.part), ml, 0, w.split};
        // float16 results: the queries' second part matters beside the rounding of the result
        constexpr bool codes = F == IVFTQ_KV_CODE4;
        const bool low = codes && a.q.type == IVFTQ_KV_F16;
        auto launch = [&](auto kernel, ChipFill& fill) {
            unsigned wgs = pairs;
            if (w.split) {
                if (hipError_t e = fill.get(reinterpret_cast<const void*>(kernel), 256, 0, &wgs)) return e;
                if (wgs > (unsigned)kFewMaxWgs) wgs = kFewMaxWgs;
                f.wgs = (int32_t)wgs;
            }
            kernel<<<kv_grid(wgs, 256, (unsigned)w.col_tiles), 256, 0, st>>>(f);
            return hipGetLastError();
        };
        static ChipFill fill, fill_low;
        if (hipError_t e = low ? launch(&k_kv_few<F, D, codes>, fill_low) : launch(&k_kv_few<F, D, false>, fill)) return e;
        if (w.split || F == IVFTQ_KV_CODE4) k_kv_few_join<F, D><<<kv_grid(pairs, 512, (unsigned)w.col_tiles), 512, 0, st>>>(f);
    } else {
        const ManyArgs f{a, z, zn, whole, reinterpret_cast<float*>(a.work + w.part), ml, reinterpret_cast<int64_t*>(a.work + w.begin), w.row_tiles, w.shared};
        auto launch = [&](auto shared) {
            constexpr bool S = decltype(shared)::value;
            // shares: workgroups for either way
            const unsigned one_each = pairs * (unsigned)w.row_tiles, wgs = S && one_each < (unsigned)(a.c.heads * w.shared) ? (unsigned)(a.c.heads * w.shared) : one_each;
            // float16 results: the queries' second part matters beside the rounding of the result
            if (F == IVFTQ_KV_CODE4 && a.q.type == IVFTQ_KV_F16) k_kv_many<F, D, F == IVFTQ_KV_CODE4, S><<<kv_grid(wgs, 256), 256, 0, st>>>(f);
            else k_kv_many<F, D, false, S><<<kv_grid(wgs, 256), 256, 0, st>>>(f);
            if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_back<D, S><<<rot, D * 2, 0, st>>>(f, tiles);
            else if constexpr (S) k_kv_many_join<F, D><<<kv_grid((all * (D / 8) + 255) / 256, 256), 256, 0, st>>>(f);
        };
        if (w.shared) launch(std::true_type{}); else launch(std::false_type{});
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
