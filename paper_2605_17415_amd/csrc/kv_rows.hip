// Rows of the paged key-value cache: written to their pages (rotated and quantised where the cache holds codes) and read back.
#include <cstring>
#include <type_traits>

#include "kv_kernels.h"

namespace ivftq {
namespace {

// One row per sequence: where row r's token lives, its page's record part of head h and its place in the page; null where
// there is none.
template <bool READ>
__device__ __forceinline__ char* place_of(const KvView& c, int r, int h, int& t) {
    const int pos = kv_length(c, r) - 1;
    if (pos < 0 || (!READ && kv_refused(c, r))) return nullptr;
    const int64_t page = kv_page(c, r, pos);
    t = pos & (c.page - 1);
    return page < 0 ? nullptr : kv_record(c, page, h);
}

// ---- tiles of a sequence's new rows ---------------------------------------------------------------------------------
// Where a sequence has several new rows the work is cut into tiles of 32 positions of a sequence, aligned, so that a group
// of eight tokens (whose values share words) is written by one wavefront.  The tiles of all sequences stand one after the
// other; a wavefront takes a consecutive share of (tile, head) items.

struct NewTiles { int first_row, pos0, end, tile0, tiles; };      // pos0: position of the first new row (may be under zero)

template <bool READ>
__device__ __forceinline__ NewTiles new_tiles(const KvView& c, int b) {
    NewTiles t{0, 0, 0, 0, 0};
    if (b >= c.batch || (!READ && kv_refused(c, b))) return t;
    int count;
    kv_new_rows(c, b, t.first_row, count);
    t.end = kv_length(c, b);
    t.pos0 = t.end - count;
    const int lo = t.pos0 > 0 ? t.pos0 : 0;
    t.tile0 = lo / 32;
    t.tiles = count > 0 && t.end > lo ? (t.end + 31) / 32 - t.tile0 : 0;
    return t;
}

struct NewItem { int64_t left; int b, tile, sub; NewTiles s; };   // items left; sub: number inside a tile

// This wavefront's share of total * per_tile items.
template <bool READ>
__device__ __forceinline__ NewItem first_item(const KvView& c, int per_tile) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int b0 = 0; b0 < c.batch; b0 += 64) {
        int v = new_tiles<READ>(c, b0 + lane).tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
        total += v;
    }
    total = kv_uniform(total);
    const int64_t waves = (int64_t)gridDim.x * (blockDim.x / 64), items = total * per_tile, share = (items + waves - 1) / waves;
    const int64_t x = ((int64_t)blockIdx.x * (blockDim.x / 64) + kv_wave()) * share;
    NewItem it{items - x < share ? items - x : share, 0, 0, 0, {}};
    if (it.left <= 0) { it.left = 0; return it; }
    const int64_t tile = x / per_tile;
    it.sub = (int)(x % per_tile);
    int64_t base = 0;
    for (int b0 = 0; b0 < c.batch; b0 += 64) {
        const int v = new_tiles<READ>(c, b0 + lane).tiles;
        int64_t incl = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int64_t u = __shfl_up(incl, o); if (lane >= o) incl += u; }
        const uint64_t past = __ballot(base + incl > tile);
        if (past) {
            const int l = __builtin_ctzll(past);
            it.b = b0 + l;
            it.tile = kv_uniform((int)(tile - base - __shfl(incl - v, l)));
            break;
        }
        base += kv_uniform((int64_t)__shfl(incl, 63));
    }
    it.s = new_tiles<READ>(c, it.b);
    return it;
}
template <bool READ>
__device__ __forceinline__ void next_item(const KvView& c, int per_tile, NewItem& it) {
    if (--it.left <= 0) return;
    if (++it.sub < per_tile) return;
    it.sub = 0;
    if (++it.tile < it.s.tiles) return;
    it.tile = 0;
    do { it.s = new_tiles<READ>(c, ++it.b); } while (!it.s.tiles && it.b < c.batch);      // there is one: items are left
}

// Reading: new rows that stand before position zero (a sequence has more rows than tokens) have no place and give zeros.
__device__ __forceinline__ void no_place(const KvView& c, const KvRows& k, const KvRows& v, int d) {
    for (int b = blockIdx.x; b < c.batch; b += gridDim.x) {
        int first, count;
        kv_new_rows(c, b, first, count);
        const int64_t lost = count - kv_length(c, b);
        for (int64_t i = threadIdx.x; i < lost * c.heads * (d / 8); i += blockDim.x) {
            const int j = (int)(i % (d / 8)) * 8, h = (int)(i / (d / 8) % c.heads);
            const int64_t r = first + i / (d / 8) / c.heads;
            *reinterpret_cast<uintx4*>(reinterpret_cast<uint16_t*>(k.data) + r * k.row_stride + h * k.head_stride + j) = uintx4{0, 0, 0, 0};
            *reinterpret_cast<uintx4*>(reinterpret_cast<uint16_t*>(v.data) + r * v.row_stride + h * v.head_stride + j) = uintx4{0, 0, 0, 0};
        }
    }
}

// ---- 16 bits ---------------------------------------------------------------------------------------------------------

// One row per sequence (or a tile's ragged ends): eight coordinates of one row's key and value.
template <bool READ>
__device__ __forceinline__ void move16(const KvView& c, char* rec, int t, int d, int j, uint16_t* kr, uint16_t* vr) {
    uint16_t* kp = reinterpret_cast<uint16_t*>(rec) + (int64_t)t * d + j;
    uint16_t* vp = reinterpret_cast<uint16_t*>(rec) + (int64_t)c.page * d + ((int64_t)(t >> 3) * d + j) * 8 + (t & 7);
    if constexpr (READ) {
        uintx4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        if (rec) {
            a = *reinterpret_cast<const uintx4*>(kp);
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = (uint32_t)vp[16 * e] | (uint32_t)vp[16 * e + 8] << 16;
        }
        *reinterpret_cast<uintx4*>(kr) = a;
        *reinterpret_cast<uintx4*>(vr) = b;
    } else if (rec) {
        *reinterpret_cast<uintx4*>(kp) = *reinterpret_cast<const uintx4*>(kr);
        const uintx4 b = *reinterpret_cast<const uintx4*>(vr);
#pragma unroll
        for (int e = 0; e < 4; ++e) { vp[16 * e] = (uint16_t)b[e]; vp[16 * e + 8] = (uint16_t)(b[e] >> 16); }
    }
}

template <bool READ>
__global__ __launch_bounds__(256) void k_kv_move16(KvView c, KvRows k, KvRows v, int d) {
    const int chunks = d / 8, i = blockIdx.x * 256 + threadIdx.x;              // rows * heads * d / 8 is under 2^31 here
    const int row_head = i / chunks, j = i % chunks * 8, r = row_head / c.heads, h = row_head % c.heads;
    if (r >= c.rows) return;
    int t = 0;
    char* rec = place_of<READ>(c, r, h, t);
    move16<READ>(c, rec, t, d, j, reinterpret_cast<uint16_t*>(k.data) + r * k.row_stride + h * k.head_stride + j,
                 reinterpret_cast<uint16_t*>(v.data) + r * v.row_stride + h * v.head_stride + j);
}

// 8 x 8 16-bit numbers, rows in a[0..7], turned: three rounds of exchanges of halves, 24 byte permutations and moves.
__device__ __forceinline__ void turn8x8(uintx4 (&a)[8]) {
    uintx4 r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)              // row i of the result: value i of rows 2 e and 2 e + 1
            r[i][e] = __builtin_amdgcn_perm(a[2 * e + 1][i / 2], a[2 * e][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = r[i];
}

// Several rows a sequence: a lane moves eight tokens' eight coordinates, values turned in registers, so that both sides of
// the copy are whole 16-byte pieces.
template <bool READ>
__global__ __launch_bounds__(256) void k_kv_tiles16(KvView c, KvRows k, KvRows v, int d) {
    const int lane = threadIdx.x & 63, chunks = d / 8;
    if constexpr (READ) no_place(c, k, v, d);
    NewItem it = first_item<READ>(c, c.heads);
    for (; it.left > 0; next_item<READ>(c, c.heads, it)) {
        const int h = it.sub, t0 = (it.s.tile0 + it.tile) * 32;
        for (int u = lane; u < 4 * chunks; u += 64) {
            const int og = u / chunks, j = u % chunks * 8, t = t0 + 8 * og;
            const int64_t page = kv_page(c, it.b, t);
            char* rec = page < 0 ? nullptr : kv_record(c, page, h);
            const int in = t & (c.page - 1), row = it.s.first_row + t - it.s.pos0;
            uint16_t* kr = reinterpret_cast<uint16_t*>(k.data) + row * k.row_stride + h * k.head_stride + j;
            uint16_t* vr = reinterpret_cast<uint16_t*>(v.data) + row * v.row_stride + h * v.head_stride + j;
            if (rec && t >= it.s.pos0 && t + 8 <= it.s.end) {
                uintx4* kp = reinterpret_cast<uintx4*>(reinterpret_cast<uint16_t*>(rec) + (int64_t)in * d + j);
                uintx4* vp = reinterpret_cast<uintx4*>(reinterpret_cast<uint16_t*>(rec) + (int64_t)c.page * d + ((int64_t)(in >> 3) * d + j) * 8);
                uintx4 x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = READ ? kp[e * chunks] : *reinterpret_cast<const uintx4*>(kr + e * k.row_stride);
                    y[e] = READ ? vp[e] : *reinterpret_cast<const uintx4*>(vr + e * v.row_stride);
                }
                turn8x8(y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (READ) {
                        *reinterpret_cast<uintx4*>(kr + e * k.row_stride) = x[e];
                        *reinterpret_cast<uintx4*>(vr + e * v.row_stride) = y[e];
                    } else {
                        kp[e * chunks] = x[e];
                        vp[e] = y[e];
                    }
                }
            } else {
                for (int e = 0; e < 8; ++e)
                    if (t + e >= it.s.pos0 && t + e < it.s.end) move16<READ>(c, rec, in + e, d, j, kr + e * k.row_stride, vr + e * v.row_stride);
            }
        }
    }
}

// ---- codes ---------------------------------------------------------------------------------------------------------

// A 16-bit row in the operand layout: x[s][e] = coordinate 32 s + 8 (lane / 16) + e.
template <int D, bool BF>
__device__ __forceinline__ void load_row(const KvRows& x, int64_t row, int64_t head, float (&v)[D / 32][8]) {
    const int g = (threadIdx.x & 63) >> 4;
    const uint16_t* p = reinterpret_cast<const uint16_t*>(x.data) + row * x.row_stride + head * x.head_stride + 8 * g;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        const uintx4 w = *reinterpret_cast<const uintx4*>(p + 32 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[s][2 * e] = kv_to_float<BF>(w[e] & 0xffff); v[s][2 * e + 1] = kv_to_float<BF>(w[e] >> 16); }
    }
}

// One row per sequence: a wavefront takes 16 (row, head) pairs of keys or of values and 32 of the d codes (blockIdx.y), so
// that even a single row's rotation is spread over several wavefronts: such calls are bound by the latency of their chain
// of loads.  A key's codes are whole words; a value's code is one half byte in each of d words, which nothing else writes
// in this call.
template <int D, bool BF>
__global__ __launch_bounds__(64) void k_kv_append_row_codes(KvView c, KvRows k, KvRows v) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
    const bool value = blockIdx.y >= D / 32;
    const int block = blockIdx.y % (D / 32);
    const uint32_t i = blockIdx.x * 16u + n;                 // rows * heads is under 2^31
    const bool in = i < (uint32_t)c.rows * (uint32_t)c.heads;
    const int r = in ? (int)(i / (uint32_t)c.heads) : 0, h = in ? (int)(i % (uint32_t)c.heads) : 0;
    const KvTurnRows<D, false> pi(c.rotation, block);
    float x[D / 32][8], y[8];
    load_row<D, BF>(value ? v : k, r, h, x);          // (of lanes past the end: the first row, not used)
    const float norm = kv_unit_row<D>(x);
    int t = 0;
    char* rec = in ? place_of<false>(c, r, h, t) : nullptr;
    KvTurn<D, false>{pi}(x, y);
    if (!rec) return;
    const int codes = c.page * (D / 2), j = 32 * block + 8 * g;
    if (g == 0 && block == 0) reinterpret_cast<_Float16*>(rec + 2 * codes)[(value ? c.page : 0) + t] = (_Float16)norm;
    const uint32_t w = kv_nibbles8(y, c);
    if (!value) {
        reinterpret_cast<uint32_t*>(rec + (int64_t)t * (D / 2))[j / 8] = w;
    } else {
        uint8_t* p = reinterpret_cast<uint8_t*>(rec + codes) + ((int64_t)(t >> 3) * D + j) * 4 + (t & 7) / 2;
        uint32_t was[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) was[e] = p[4 * e];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[4 * e] = (uint8_t)(t & 1 ? (was[e] & 15) | (w >> 4 * e & 15) << 4 : (was[e] & 240) | (w >> 4 * e & 15));
    }
}

// 8 x 8 half bytes over eight neighbouring lanes, turned: lane i's half byte e becomes lane e's half byte i.  Exchanges inside a row of lanes
// (a lane 4 away: mirrored over eight, then over four), and byte permutations whose selectors depend on the lane.
template <int CTRL>
__device__ __forceinline__ uint32_t lanes_moved(uint32_t w) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)w, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t turn_nibbles(uint32_t w, int lane) {
    const uint32_t by4 = lane & 4 ? 0x03020706u : 0x05040100u, by2 = lane & 2 ? 0x03070105u : 0x06020400u;
    const uint32_t keep = lane & 1 ? 0xf0f0f0f0u : 0x0f0f0f0fu, right = lane & 1 ? 4u : 28u;
    w = __builtin_amdgcn_perm(lanes_moved<0x1b>(lanes_moved<0x141>(w)), w, by4);
    w = __builtin_amdgcn_perm(lanes_moved<0x4e>(w), w, by2);
    const uint32_t p = lanes_moved<0xb1>(w);
    return (w & keep) | (__builtin_amdgcn_alignbit(p, p, right) & ~keep);
}

// The eight levels, times 2^10 (levels from 32 on: a lower power of two, so that float16 holds the largest), as two float16 parts that
// keep them to 2^-22: byte tables like those of kv_levels8, the second part with a sign of its own.
struct KvExact {
    uint32_t hi[4], lo[4];          // of each part: low bytes, then high bytes
    float unit;                     // 2^10 over that power of two
};

KvExact kv_exact(const KvView& c) {
    KvExact x{};
    x.unit = 1.f;
    while (c.level[7] * kSplitScale >= 32768.f * x.unit) x.unit *= 2.f;          // levels are under 10^4
    for (int m = 0; m < 8; ++m) {
        const float v = c.level[m] * kSplitScale / x.unit;
        const _Float16 part[2] = {(_Float16)v, (_Float16)(v - (float)(_Float16)v)};
        for (int p = 0; p < 2; ++p) {
            uint16_t bits;
            memcpy(&bits, &part[p], 2);
            uint32_t* to = p ? x.lo : x.hi;
            to[m / 4] |= (uint32_t)(bits & 0xff) << 8 * (m % 4);
            to[2 + m / 4] |= (uint32_t)(bits >> 8) << 8 * (m % 4);
        }
    }
    return x;
}

__device__ __forceinline__ void kv_exact8(uint32_t w, const KvExact& x, halfx8& hi, halfx8& lo) {
    const uint32_t even = w & 0x07070707u, odd = (w >> 4) & 0x07070707u, even_sign = (w << 4) & 0x80808080u, odd_sign = w & 0x80808080u;
    uintx4 r[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint32_t* t = p ? x.lo : x.hi;
        const uint32_t el = __builtin_amdgcn_perm(t[1], t[0], even), eh = __builtin_amdgcn_perm(t[3], t[2], even) ^ even_sign;
        const uint32_t ol = __builtin_amdgcn_perm(t[1], t[0], odd), oh = __builtin_amdgcn_perm(t[3], t[2], odd) ^ odd_sign;
        r[p][0] = __builtin_amdgcn_perm(eh, el, 0x05010400u);
        r[p][1] = __builtin_amdgcn_perm(eh, el, 0x07030602u);
        r[p][2] = __builtin_amdgcn_perm(oh, ol, 0x05010400u);
        r[p][3] = __builtin_amdgcn_perm(oh, ol, 0x07030602u);
    }
    hi = __builtin_bit_cast(halfx8, r[0]);
    lo = __builtin_bit_cast(halfx8, r[1]);
}

// The rows that the codes stand for, one per sequence: levels, rotated back, times the norm.  Split as k_kv_append_row_codes is; what the
// rotation is read from is asked for before the chain length, table entry, words, and lanes without a page read page 0.
template <int D, bool BF>
__global__ __launch_bounds__(64) void k_kv_read_row_codes(KvView c, KvRows k, KvRows v, KvExact exact) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
    const bool value = blockIdx.y >= D / 32;
    const int block = blockIdx.y % (D / 32);
    const uint32_t i = blockIdx.x * 16u + n;                 // rows * heads is under 2^31
    const bool in = i < (uint32_t)c.rows * (uint32_t)c.heads;
    const int r = in ? (int)(i / (uint32_t)c.heads) : 0, h = in ? (int)(i % (uint32_t)c.heads) : 0;
    const KvTurnRows<D, true> pi(c.rotation, block);
    int t = 0;
    const char* const place = place_of<true>(c, r, h, t);
    const char* const rec = place ? place : kv_record(c, 0, h);
    const int codes = c.page * (D / 2);
    const _Float16 norm = reinterpret_cast<const _Float16*>(rec + 2 * codes)[(value ? c.page : 0) + t];
    uint32_t w[D / 32];
    if (!value) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(rec + (int64_t)t * (D / 2)) + g;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) w[s] = p[4 * s];
    } else {
        const uintx4* p = reinterpret_cast<const uintx4*>(reinterpret_cast<const uint32_t*>(rec + codes) + (int64_t)(t >> 3) * D + 8 * g);
        uintx4 u[D / 32][2];
#pragma unroll
        for (int s = 0; s < D / 32; ++s) { u[s][0] = p[8 * s]; u[s][1] = p[8 * s + 1]; }
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            w[s] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[s] |= (u[s][e >> 2][e & 3] >> 4 * (t & 7) & 15) << 4 * e;
        }
    }
    halfx8 hi[D / 32], lo[D / 32];
    float y[8];
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        kv_exact8(w[s], exact, hi[s], lo[s]);
        hi[s] = __builtin_shufflevector(hi[s], hi[s], 0, 4, 1, 5, 2, 6, 3, 7);
        lo[s] = __builtin_shufflevector(lo[s], lo[s], 0, 4, 1, 5, 2, 6, 3, 7);
    }
    KvTurn<D, true>{pi}(hi, lo, y);
    if (!in) return;
    kv_store_turned(value ? v : k, r, h, block, y, place ? (float)norm * exact.unit : 0.f);
}

// Several rows a sequence.  The rotation stands in LDS as two float16 parts in operand order, so that reading it costs 64
// KB of LDS traffic per 32 rows and none of L2 (at d = 256 and 192 a workgroup computes one half of the coordinates: 128
// and 72 KB).  A wavefront takes a tile of 32 tokens of one head's keys or values, two column tiles, and has the next
// tile's rows on their way meanwhile.  Writing: a row's values are float16 numbers as they are, or become such by a power of
// two that puts the row's length between 2^8 and 2^9 (what that loses lies 2^-25 under the row's largest value), so two
// products do, and the results are divided by the row's length afterwards.  Reading: the levels as two parts as well, three
// products.  Writing is bound by the vector unit, half of whose operations look for levels; 363,000 rows of keys and as many of values
// (float16, d = 128) take 125 us to write and 82 us to read back (medians; 114 and 75 at the least), where neighbouring lanes write
// neighbouring pieces (20 us more where a lane's pieces of a row lay 64 bytes apart).
template <int D> constexpr int kOutputs = D > 128 ? D / 2 : D;             // coordinates that a workgroup computes
template <int D> constexpr int kTurnBytes = kOutputs<D> * D * 4;
constexpr int kTileThreads = 512;

template <int D, bool READ>
struct TileRows {                                                          // a tile as it is read from memory
    static constexpr int NS = D / 32;
    typename std::conditional<READ, uint32_t, uintx4>::type w[2][NS];
    uint32_t norm[2];
    char* rec[2];
};

template <int D, bool READ>
__device__ __forceinline__ void load_tile(const KvView& c, const KvRows& rows, const NewItem& it, int h, bool value, TileRows<D, READ>& x) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, codes = c.page * (D / 2);
    const int t0 = (it.s.tile0 + it.tile) * 32;
#pragma unroll
    for (int ct = 0; ct < 2; ++ct) {
        const int64_t page = kv_uniform((int)kv_page(c, it.b, t0 + 16 * ct));          // 16 tokens lie in one page
        const int t = t0 + 16 * ct + n, at = t & (c.page - 1);
        const bool mine = t >= it.s.pos0 && t < it.s.end;
        x.rec[ct] = page < 0 ? nullptr : kv_record(c, page, h);
        x.norm[ct] = 0;
        if constexpr (READ) {
            const char* rec = page < 0 ? kv_record(c, 0, h) : x.rec[ct];
            x.norm[ct] = reinterpret_cast<const uint16_t*>(rec + 2 * codes)[(value ? c.page : 0) + at];
            const uint32_t* p = value ? reinterpret_cast<const uint32_t*>(rec + codes) + (at >> 3) * D + 8 * g + (n & 7)
                                      : reinterpret_cast<const uint32_t*>(rec + at * (D / 2)) + g;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) x.w[ct][s] = p[s * (value ? 32 : 4)];
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(rows.data) + (mine ? it.s.first_row + t - it.s.pos0 : 0) * rows.row_stride + h * rows.head_stride + 8 * g;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) x.w[ct][s] = *reinterpret_cast<const uintx4*>(p + 32 * s);
        }
    }
}

// Operands of a column tile: float16 values `hi` (writing) or levels in two parts (reading, in the order of kv_levels8);
// returns what the products are multiplied by, and the row's norm.
template <int D, bool BF>
__device__ __forceinline__ float row_operand(const uintx4 (&w)[D / 32], halfx8 (&x)[D / 32], float& norm) {
    float n2 = 0.f;
    if constexpr (BF) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = kv_to_float<true>(w[s][e] & 0xffff), hi = __builtin_bit_cast(float, w[s][e] & 0xffff0000u);
                n2 += lo * lo;
                n2 += hi * hi;
            }
        norm = sqrtf(kv_sum4(n2));
        // the power of two next under 2^9 / norm; norms of zero, none and infinity: any
        const int up = 8 + 127 - (int)(__builtin_bit_cast(uint32_t, norm) >> 23);
        const float scale = __builtin_bit_cast(float, (uint32_t)(up + 127 < 1 ? 1 : (up + 127 > 254 ? 254 : up + 127)) << 23);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            uintx4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = kv_pack2<false>(kv_to_float<true>(w[s][e] & 0xffff) * scale, __builtin_bit_cast(float, w[s][e] & 0xffff0000u) * scale);
            x[s] = __builtin_bit_cast(halfx8, y);
        }
        return norm > 0.f ? 1.f / (norm * scale * kSplitScale) : 0.f;
    } else {
        typedef _Float16 two __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            x[s] = __builtin_bit_cast(halfx8, w[s]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t u = w[s][e];          // (a bit cast of an element of a vector casts the first one, whichever is named)
                const two p = __builtin_bit_cast(two, u);
                n2 = __builtin_amdgcn_fdot2(p, p, n2, false);
            }
        }
        norm = sqrtf(kv_sum4(n2));
        return norm > 0.f ? 1.f / (norm * kSplitScale) : 0.f;
    }
}

template <int D, bool BF, bool READ>
__global__ __launch_bounds__(kTileThreads, D <= 128 ? 4 : 2) void k_kv_tiles_codes(KvView c, KvRows k, KvRows v, KvExact exact) {
    constexpr int NS = D / 32, NT = kOutputs<D> / 32;
    extern __shared__ __align__(16) char turn[];                           // [NT][2][NS][hi, lo][64 lanes] of 16 bytes
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int out0 = blockIdx.y * kOutputs<D>;
    if (READ && out0 == 0) no_place(c, k, v, D);
    for (int u = threadIdx.x; u < NT * 2 * NS * 64; u += kTileThreads) {
        const int l = u & 63, s = u / 64 % NS, half = u / 64 / NS & 1, t = u / 64 / NS / 2, m = l & 15;
        // a lane's results: coordinates out0 + 32 t + 8 g + 4 half + (0 .. 3), so that the four lanes of a row write neighbouring pieces
        const int i = out0 + 32 * t + 8 * (m >> 2) + 4 * half + (m & 3), k0 = 32 * s + 8 * (l >> 4);
        halfx8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = (READ ? c.rotation[(k0 + e) * D + i] : c.rotation[i * D + k0 + e]) * kSplitScale;
            const int at = READ ? kv_slot(e) : e;
            hi[at] = (_Float16)p;
            lo[at] = (_Float16)(p - (float)hi[at]);
        }
        halfx8* to = reinterpret_cast<halfx8*>(turn) + (u / 64) * 128 + l;
        to[0] = hi;
        to[64] = lo;
    }
    __syncthreads();
    const int codes = c.page * (D / 2), per_tile = 2 * c.heads;
    NewItem it = first_item<READ>(c, per_tile);
    if (it.left <= 0) return;
    TileRows<D, READ> next;
    load_tile<D, READ>(c, it.sub >= c.heads ? v : k, it, it.sub >= c.heads ? it.sub - c.heads : it.sub, it.sub >= c.heads, next);
    while (it.left > 0) {
        const bool value = it.sub >= c.heads;
        const int h = value ? it.sub - c.heads : it.sub, t0 = (it.s.tile0 + it.tile) * 32;
        const NewTiles seq = it.s;
        const KvRows& rows = value ? v : k;
        halfx8 xh[2][NS], xl[2][READ ? NS : 1];
        float norm[2], gain[2];
        char* rec[2];
        bool mine[2];
#pragma unroll
        for (int ct = 0; ct < 2; ++ct) {
            const int t = t0 + 16 * ct + n;
            mine[ct] = t >= seq.pos0 && t < seq.end;
            rec[ct] = next.rec[ct];
            if constexpr (READ) {
                norm[ct] = (float)__builtin_bit_cast(_Float16, (uint16_t)next.norm[ct]);
                gain[ct] = norm[ct] * exact.unit * (1.f / (kSplitScale * kSplitScale));
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const uint32_t w = value ? turn_nibbles(next.w[ct][s], lane) : next.w[ct][s];
                    kv_exact8(w, exact, xh[ct][s], xl[ct][s]);
                }
            } else {
                gain[ct] = row_operand<D, BF>(next.w[ct], xh[ct], norm[ct]);
            }
        }
        next_item<READ>(c, per_tile, it);
        if (it.left > 0) load_tile<D, READ>(c, it.sub >= c.heads ? v : k, it, it.sub >= c.heads ? it.sub - c.heads : it.sub, it.sub >= c.heads, next);
#pragma unroll 1
        for (int t = 0; t < NT; ++t) {
            float y[2][8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                const halfx8* from = reinterpret_cast<const halfx8*>(turn) + (t * 2 + half) * NS * 128 + lane;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const halfx8 ah = from[s * 128], al = from[s * 128 + 64];
#pragma unroll
                    for (int ct = 0; ct < 2; ++ct) {
                        acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, xh[ct][s], acc[ct], 0, 0, 0);
                        acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, xh[ct][s], acc[ct], 0, 0, 0);
                        if constexpr (READ) acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, xl[ct][s], acc[ct], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int ct = 0; ct < 2; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[ct][4 * half + r] = acc[ct][r] * gain[ct];
            }
            const int j = out0 + 32 * t + 8 * g;
#pragma unroll
            for (int ct = 0; ct < 2; ++ct) {
                const int at = (t0 + 16 * ct + n) & (c.page - 1);
                if constexpr (READ) {
                    if (!mine[ct]) continue;
                    uintx4 w = {0, 0, 0, 0};
                    if (rec[ct])
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = kv_pack2<BF>(y[ct][2 * e], y[ct][2 * e + 1]);
                    *reinterpret_cast<uintx4*>(reinterpret_cast<uint16_t*>(rows.data) + (int64_t)(seq.first_row + t0 + 16 * ct + n - seq.pos0) * rows.row_stride +
                                               h * rows.head_stride + j) = w;
                } else if (rec[ct]) {
                    uint32_t w = kv_nibbles8(y[ct], c);
                    if (!value) {
                        if (mine[ct]) reinterpret_cast<uint32_t*>(rec[ct] + at * (D / 2))[j / 8] = w;
                    } else {
                        w = turn_nibbles(w, lane);           // this lane: coordinate j + n % 8, tokens of its group of eight
                        const uint32_t given = (uint32_t)(__ballot(mine[ct]) >> (lane & 56)) & 0xff;
                        uint32_t* p = reinterpret_cast<uint32_t*>(rec[ct] + codes) + (at >> 3) * D + j + (n & 7);
                        if (given == 0xff) {
                            *p = w;
                        } else if (given) {                  // the other tokens' half bytes stay
                            uint32_t keep = 0;
#pragma unroll
                            for (int e = 0; e < 8; ++e) keep |= given >> e & 1 ? 0 : 15u << 4 * e;
                            *p = (*p & keep) | (w & ~keep);
                        }
                    }
                }
            }
        }
        if constexpr (!READ) {
#pragma unroll
            for (int ct = 0; ct < 2; ++ct)
                if (g == 0 && out0 == 0 && mine[ct] && rec[ct])
                    reinterpret_cast<_Float16*>(rec[ct] + 2 * codes)[(value ? c.page : 0) + ((t0 + 16 * ct + n) & (c.page - 1))] = (_Float16)norm[ct];
        }
    }
}

// Workgroups for the tiles: as many as the chip holds at once, or fewer where there cannot be that many items.
hipError_t tile_grid(ChipFill& fill, const void* kernel, int threads, size_t lds, const KvView& c, int per_tile, int slices, unsigned* wgs) {
    if (hipError_t e = fill.get(kernel, threads, lds, wgs)) return e;
    const int64_t waves = threads / 64, most = (((int64_t)c.rows / 32 + 2 * (int64_t)c.batch) * per_tile + waves - 1) / waves;
    *wgs = *wgs / slices ? *wgs / slices : 1;
    if (most < *wgs) *wgs = (unsigned)most;
    return hipSuccess;
}

template <int D, bool BF, bool READ>
hipError_t tiles_codes(const KvView& c, const KvRows& k, const KvRows& v, hipStream_t st) {
    static ChipFill fill;
    constexpr int slices = D / kOutputs<D>;
    const void* kernel = reinterpret_cast<const void*>(&k_kv_tiles_codes<D, BF, READ>);
    unsigned wgs;
    if (hipError_t e = tile_grid(fill, kernel, kTileThreads, kTurnBytes<D>, c, 2 * c.heads, slices, &wgs)) return e;
    k_kv_tiles_codes<D, BF, READ><<<dim3(wgs, slices), kTileThreads, kTurnBytes<D>, st>>>(c, k, v, READ ? kv_exact(c) : KvExact{});
    return hipGetLastError();
}

template <int D, bool BF>
hipError_t codes(const KvView& c, const KvRows& k, const KvRows& v, bool read, hipStream_t st) {
    if (c.starts) {
        if (read) return tiles_codes<D, BF, true>(c, k, v, st);
        return tiles_codes<D, BF, false>(c, k, v, st);
    }
    const dim3 grid((unsigned)(((int64_t)c.rows * c.heads + 15) / 16), 2 * (D / 32));
    if (read) k_kv_read_row_codes<D, BF><<<grid, 64, 0, st>>>(c, k, v, kv_exact(c)); else k_kv_append_row_codes<D, BF><<<grid, 64, 0, st>>>(c, k, v);
    return hipGetLastError();
}

template <int D>
hipError_t codes_d(const KvView& c, const KvRows& k, const KvRows& v, bool read, hipStream_t st) {
    return k.type == IVFTQ_KV_BF16 ? codes<D, true>(c, k, v, read, st) : codes<D, false>(c, k, v, read, st);
}

template <bool READ>
hipError_t tiles16(const KvView& c, const KvRows& k, const KvRows& v, int d, hipStream_t st) {
    static ChipFill fill;
    unsigned wgs;
    if (hipError_t e = tile_grid(fill, reinterpret_cast<const void*>(&k_kv_tiles16<READ>), 256, 0, c, c.heads, 1, &wgs)) return e;
    k_kv_tiles16<READ><<<wgs, 256, 0, st>>>(c, k, v, d);
    return hipGetLastError();
}

hipError_t move(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, bool read, hipStream_t st) {
    if (!c.rows) return hipSuccess;
    if (format == IVFTQ_KV_CODE4) {
        switch (d) {
            case 64: return codes_d<64>(c, k, v, read, st);
            case 96: return codes_d<96>(c, k, v, read, st);
            case 128: return codes_d<128>(c, k, v, read, st);
            case 192: return codes_d<192>(c, k, v, read, st);
            default: return codes_d<256>(c, k, v, read, st);
        }
    }
    if (c.starts) return read ? tiles16<true>(c, k, v, d, st) : tiles16<false>(c, k, v, d, st);
    const unsigned grid = (unsigned)(((int64_t)c.rows * c.heads * (d / 8) + 255) / 256);
    if (read) k_kv_move16<true><<<grid, 256, 0, st>>>(c, k, v, d); else k_kv_move16<false><<<grid, 256, 0, st>>>(c, k, v, d);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, hipStream_t st) {
    return move(c, k, v, d, format, false, st);
}
hipError_t launch_kv_read(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, hipStream_t st) {
    return move(c, k, v, d, format, true, st);
}

}  // namespace ivftq
