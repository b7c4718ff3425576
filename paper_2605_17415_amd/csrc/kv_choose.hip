// Digests of the key-value cache's pages, and the pages that a row is given for their scores.
#include <type_traits>

#include "kv_kernels.h"
#include "wave_ops.h"

namespace ivftq {
namespace {

// ---- digests ---------------------------------------------------------------------------------------------------------
// The smallest and the largest value of each key coordinate: comparisons only, so the order of its tokens does not matter and a digest in 16 bits
// is exact.  Over codes the ends are rounded to float16, to the nearest as all that is stored (once more, where a page goes on, changes nothing): an end may
// lie half a step, 2^-11 of it, inside the keys' range, and a score that much under a bound; scores only put pages in order.
// Prompts of 45,000 tokens, 8 heads of 128 in codes: 16 us for 27 MB; a wavefront has one page of one head, three dependent loads and five vector
// instructions a code.  One row a sequence: 3 us, its chain of loads.

// Pages of a sequence that hold new rows.
struct NewPages { int lo, end, col0, count; };          // positions of the new rows, first column, number of pages
__device__ __forceinline__ NewPages new_pages(const KvView& c, int b) {
    NewPages p{0, 0, 0, 0};
    if (b >= c.batch || kv_refused(c, b)) return p;
    int first, count;
    kv_new_rows(c, b, first, count);
    p.end = kv_length(c, b);
    p.lo = p.end > count ? p.end - count : 0;
    p.col0 = p.lo >> c.page_log2;
    p.count = count > 0 && p.end > p.lo ? ((p.end - 1) >> c.page_log2) - p.col0 + 1 : 0;
    return p;
}

// Eight coordinates of a key: 16 bits each, or codes and the row's norm.
template <int F>
struct KeyPiece {
    uintx4 w;
    uint32_t codes;
    float norm;
    __device__ __forceinline__ void load(const KvView& c, const char* rec, int t, int d, int j) {
        if constexpr (F == IVFTQ_KV_CODE4) {
            codes = *reinterpret_cast<const uint32_t*>(rec + (int64_t)t * (d / 2) + j / 2);
            norm = (float)reinterpret_cast<const _Float16*>(rec + (int64_t)c.page * d)[t];
        } else {
            w = *reinterpret_cast<const uintx4*>(rec + ((int64_t)t * d + j) * 2);
        }
    }
    // level: the sixteen levels by half byte, in LDS
    __device__ __forceinline__ float value(int e, const float* level) const {
        if constexpr (F == IVFTQ_KV_CODE4) return norm * level[codes >> 4 * e & 15];
        else return kv_to_float<F == IVFTQ_KV_BF16>(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffff);
    }
};

struct Box {
    float low[8], high[8];
    __device__ __forceinline__ Box() {
#pragma unroll
        for (int e = 0; e < 8; ++e) { low[e] = INFINITY; high[e] = -INFINITY; }
    }
    template <int F>
    __device__ __forceinline__ void add(const KeyPiece<F>& k, const float* level) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = k.value(e, level);
            low[e] = fminf(low[e], v);
            high[e] = fmaxf(high[e], v);
        }
    }
    // into the digest of a page (at: its eight lowest values, D values before its eight highest), with what stands there
    template <bool BF>
    __device__ __forceinline__ void store(uint16_t* at, int d, bool goes_on) {
        if (goes_on) {
            const uintx4 l = *reinterpret_cast<const uintx4*>(at), h = *reinterpret_cast<const uintx4*>(at + d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                low[e] = fminf(low[e], kv_to_float<BF>(l[e >> 1] >> 16 * (e & 1) & 0xffff));
                high[e] = fmaxf(high[e], kv_to_float<BF>(h[e >> 1] >> 16 * (e & 1) & 0xffff));
            }
        }
        uintx4 l, h;
#pragma unroll
        for (int e = 0; e < 4; ++e) { l[e] = kv_pack2<BF>(low[2 * e], low[2 * e + 1]); h[e] = kv_pack2<BF>(high[2 * e], high[2 * e + 1]); }
        *reinterpret_cast<uintx4*>(at) = l;
        *reinterpret_cast<uintx4*>(at + d) = h;
    }
};

__device__ __forceinline__ void level_table(const KvView& c, float* level) {
    if (threadIdx.x < 16) level[threadIdx.x] = threadIdx.x & 8 ? -c.level[threadIdx.x & 7] : c.level[threadIdx.x & 7];
    __syncthreads();
}

// One new row a sequence: a thread eight coordinates of a head.
template <int F>
__global__ __launch_bounds__(256) void k_kv_digest_row(KvView c, uint16_t* digests, int d) {
    __shared__ float level[16];
    if constexpr (F == IVFTQ_KV_CODE4) level_table(c, level);
    const int chunks = d / 8;
    const int64_t i = (int64_t)kv_workgroup() * 256 + threadIdx.x, row_head = i / chunks;
    const int j = (int)(i % chunks) * 8, r = (int)(row_head / c.heads), h = (int)(row_head % c.heads);
    if (row_head >= (int64_t)c.rows * c.heads || kv_refused(c, r)) return;
    const int pos = kv_length(c, r) - 1;
    const int64_t page = pos < 0 ? -1 : kv_page(c, r, pos);
    if (page < 0) return;
    const int t = pos & (c.page - 1);
    KeyPiece<F> k;
    k.load(c, kv_record(c, page, h), t, d, j);
    Box box;
    box.add<F>(k, level);
    box.store<F == IVFTQ_KV_BF16>(digests + (page * c.heads + h) * 2 * d + j, d, t > 0);
}

// Several: the (page, head) pairs of all sequences, one after the other, are dealt to the wavefronts in equal consecutive shares.  A
// wavefront's lanes are 64 / (D / 8) tokens of D / 8 pieces of eight coordinates.
template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_digest(KvView c, uint16_t* digests) {
    constexpr int kPieces = D / 8, kTokens = 64 / kPieces, kAhead = F == IVFTQ_KV_CODE4 ? 16 : 8;       // loads on their way: a page of 64 at once, half of one
    __shared__ float level[16];
    if constexpr (F == IVFTQ_KV_CODE4) level_table(c, level);
    const int lane = threadIdx.x & 63, token = lane / kPieces, j = lane % kPieces * 8;
    int64_t total = 0;
    for (int b0 = 0; b0 < c.batch; b0 += 64) {
        int v = new_pages(c, b0 + lane).count;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
        total += v;
    }
    const int64_t items = kv_uniform(total) * c.heads, waves = (int64_t)gridDim.x * 4, share = (items + waves - 1) / waves;
    const int64_t begin = ((int64_t)blockIdx.x * 4 + kv_wave()) * share, end = begin + share < items ? begin + share : items;
    int64_t base = 0;                                     // pages before the sequences of this round
    for (int b0 = 0; b0 < c.batch && base * c.heads < end; b0 += 64) {
        const int mine = new_pages(c, b0 + lane).count;
        int64_t incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int64_t u = __shfl_up(incl, o); if (lane >= o) incl += u; }
        for (uint64_t left = __ballot(mine && (base + incl) * c.heads > begin && (base + incl - mine) * c.heads < end); left; left &= left - 1) {
            const int l = __builtin_ctzll(left), b = b0 + l;
            const int64_t before = kv_uniform(base + (int64_t)__shfl(incl - mine, l));
            const NewPages p = new_pages(c, b);
            const int64_t to = before + p.count < (end + c.heads - 1) / c.heads ? (before + p.count) * c.heads : end;
            for (int64_t x = begin > before * c.heads ? begin : before * c.heads; x < to && x < end; ++x) {
                const int col = p.col0 + (int)(x / c.heads - before), h = (int)(x % c.heads), t_first = col << c.page_log2;
                const int64_t page = kv_page(c, b, t_first);
                if (page < 0) continue;
                const int from = p.lo > t_first ? p.lo - t_first : 0, past = p.end - t_first < c.page ? p.end - t_first : c.page;
                const char* rec = kv_record(c, page, h);
                Box box;
                if (token < kTokens) {
                    for (int t = from + token; t < past; t += kTokens * kAhead) {
                        KeyPiece<F> k[kAhead];
#pragma unroll
                        for (int u = 0; u < kAhead; ++u) k[u].load(c, rec, t + u * kTokens < past ? t + u * kTokens : t, D, j);       // past the end: once more
#pragma unroll
                        for (int u = 0; u < kAhead; ++u) box.add<F>(k[u], level);
                    }
                }
                // over the lanes of one piece
                if constexpr (kTokens * kPieces == 64) {
                    auto join = [](float v, auto op) __attribute__((always_inline)) {
                        if constexpr (kPieces <= 8) v = op(v, lane_moved<0x128>(v));          // row_ror:8
                        if constexpr (kPieces <= 16) v = lane_pair<false>(v, op);
                        return lane_pair<true>(v, op);
                    };
#pragma unroll
                    for (int e = 0; e < 8; ++e) { box.low[e] = join(box.low[e], Smaller()); box.high[e] = join(box.high[e], Larger()); }
                } else {
                    const Box own = box;
#pragma unroll
                    for (int u = 1; u < kTokens; ++u)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            box.low[e] = fminf(box.low[e], __shfl(own.low[e], (lane + u * kPieces) & 63));
                            box.high[e] = fmaxf(box.high[e], __shfl(own.high[e], (lane + u * kPieces) & 63));
                        }
                }
                if (lane < kPieces) box.store<F == IVFTQ_KV_BF16>(digests + (page * c.heads + h) * 2 * D + j, D, from > 0);
            }
        }
        base += kv_uniform((int64_t)__shfl(incl, 63));
    }
}

template <int F>
hipError_t digest(const KvView& c, uint16_t* digests, int d, hipStream_t st) {
    if (!c.starts) {
        k_kv_digest_row<F><<<kv_grid(((int64_t)c.rows * c.heads * (d / 8) + 255) / 256, 256), 256, 0, st>>>(c, digests, d);
        return hipGetLastError();
    }
    // no more pages than the table has, a wavefront each where the chip holds so many
    const int64_t most = (int64_t)c.batch * c.columns * c.heads;
    const unsigned wgs = (unsigned)(most < 4 * 2048 ? (most + 3) / 4 : 2048);
    switch (d) {
        case 64: k_kv_digest<F, 64><<<wgs, 256, 0, st>>>(c, digests); break;
        case 96: k_kv_digest<F, 96><<<wgs, 256, 0, st>>>(c, digests); break;
        case 128: k_kv_digest<F, 128><<<wgs, 256, 0, st>>>(c, digests); break;
        case 192: k_kv_digest<F, 192><<<wgs, 256, 0, st>>>(c, digests); break;
        default: k_kv_digest<F, 256><<<wgs, 256, 0, st>>>(c, digests); break;
    }
    return hipGetLastError();
}

// ---- pages of the highest scores --------------------------------------------------------------------------------------

// Scores as numbers whose order is theirs; 0: never chosen.  (Without branches: there are many of them.)
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v + 0.f);                 // no negative zero
    return (bits ^ (uint32_t)((int32_t)bits >> 31 | (int32_t)0x80000000)) & (v > -INFINITY ? ~0u : 0u);
}

// Sum of v over the threads before this one, and over all of the 256.
__device__ __forceinline__ uint32_t before256(uint32_t v, uint32_t* sums, uint32_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const uint32_t u = __shfl_up(incl, o); if (lane >= o) incl += u; }
    __syncthreads();
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) { before += w < wave ? sums[w] : 0; all += sums[w]; }
    return before + incl - v;
}

// W wavefronts a row and head, its scores in registers (lane l of wavefront w: columns 64 R w + l, + 64, ..): the order of the last one that is
// chosen is found by halving the range from the lowest to the highest, counting what is not under the middle, until the count is right
// (about twelve times for a thousand scores) or the range is one number, whose lowest columns are taken.
template <int R, int W>
__global__ __launch_bounds__(W < 4 ? 256 : 64 * W) void k_kv_select_held(KvSelect s) {
    constexpr int kUnits = W < 4 ? 4 / W : 1;             // of a workgroup
    __shared__ uint32_t shared[kUnits][2][W][2];
    const KvView& c = s.c;
    const int lane = threadIdx.x & 63, wave = kv_wave() % W, sub = kv_wave() / W;
    const int64_t unit = (int64_t)kv_workgroup() * kUnits + sub, last_unit = (int64_t)c.rows * c.heads - 1;
    const int64_t used = unit < last_unit ? unit : last_unit;                    // (past the end: the last one once more, for the barriers)
    const int row = (int)((uint32_t)used / (uint32_t)c.heads);                    // rows times heads are under 2^31
    int turn = 0;
    // two numbers of every wavefront
    auto exchange = [&](uint32_t a, uint32_t b, uint32_t (&as)[W], uint32_t (&bs)[W]) __attribute__((always_inline)) {
        if constexpr (W == 1) { as[0] = a; bs[0] = b; return; }
        if (lane == 0) { shared[sub][turn][wave][0] = a; shared[sub][turn][wave][1] = b; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) { as[w] = shared[sub][turn][w][0]; bs[w] = shared[sub][turn][w][1]; }
        turn ^= 1;
    };
    const int pos = kv_uniform(kv_position(c, row));
    const int reach = pos < 0 ? 0 : (pos >> c.page_log2) + 1, n = reach < c.columns ? reach : c.columns;
    const float* scores = s.scores + used * c.columns;
    int32_t* out = s.chosen + used * s.count;
    float score[R];
    uint32_t key[R], high = 0, low = 0xffffffffu, as[W], bs[W];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int col = 64 * (R * wave + j) + lane;
        score[j] = scores[col < c.columns ? col : c.columns - 1];
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int begin = 64 * (R * wave + j), col = begin + lane;
        key[j] = order_of(score[j]);
        if (begin < s.first || begin + 64 > n - s.last) key[j] &= col >= s.first && col < n - s.last ? ~0u : 0u;
        high = key[j] > high ? key[j] : high;
        low = key[j] - 1 < low - 1 ? key[j] : low;        // of those above zero
    }
    exchange(lanes64(high, Larger()), lanes64(low - 1, Smaller()), as, bs);
    high = as[0];
    low = bs[0];
#pragma unroll
    for (int w = 1; w < W; ++w) { high = as[w] > high ? as[w] : high; low = bs[w] < low ? bs[w] : low; }
    high = kv_uniform((int)high);
    low = kv_uniform((int)low) + 1;
    auto not_under = [&](uint32_t t) __attribute__((always_inline)) {
        uint32_t count = 0;
        if constexpr (W == 1) {                          // counted by the scalar unit: the vector unit is what bounds many wavefronts
#pragma unroll
            for (int j = 0; j < R; ++j) count += (uint32_t)__popcll(__ballot(key[j] >= t));
            return (int)count;
        }
#pragma unroll
        for (int j = 0; j < R; ++j) count += key[j] >= t;
        exchange(lanes64(count, Sum()), 0, as, bs);
        count = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) count += as[w];
        return kv_uniform((int)count);
    };
    // always: the first and the last columns; of the others `want`: those not under `low` (all of them: low = 1), of low's equals `ties`
    const int kept = (s.first < n ? s.first : n) + (s.last < n - s.first ? s.last : (n > s.first ? n - s.first : 0)), want = s.count - kept;
    int ties = 1 << 30;
    if (want <= 0) {
        low = 0xffffffffu;
    } else if (high == 0 || not_under(low) <= want) {
        low = 1;
    } else {
        // not_under(low) > want; not_under(past) < want (past: none is as large, at first)
        uint32_t past = high + 1;
        int above = 0;
        while (true) {
            if (past - low == 1) { ties = want - above; break; }
            const uint32_t mid = low + (past - low) / 2;
            const int count = not_under(mid);
            if (count >= want) low = mid; else { past = mid; above = count; }
            if (count == want) break;
        }
    }
    // what is above low, and of its equals the first `ties`, in order; the first columns before and the last ones behind
    const uint64_t before = (1ull << lane) - 1;
    const int head = s.first < n ? s.first : n;
    int at = head, equal = 0, total = 0;
    if constexpr (W > 1) {
        uint32_t better = 0, same = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) { better += key[j] > low; same += key[j] == low; }
        exchange(lanes64(better, Sum()), lanes64(same, Sum()), as, bs);
        int total_same = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            at += w < wave ? as[w] : 0;
            equal += w < wave ? bs[w] : 0;
            total += as[w];
            total_same += bs[w];
        }
        at += equal < ties ? equal : ties;
        total += total_same < ties ? total_same : ties;
    }
    if (unit > last_unit) return;
    const bool all_equals = ties == 1 << 30;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        uint64_t in = __ballot(key[j] >= low);
        if (!in) continue;
        if (!all_equals) {
            const uint64_t same = __ballot(key[j] == low);
            in = __ballot(key[j] > low || (key[j] == low && equal + __popcll(same & before) < ties));
            equal += __popcll(same);
        }
        if (in >> lane & 1) out[at + __popcll(in & before)] = 64 * (R * wave + j) + lane;
        at += __popcll(in);
    }
    if constexpr (W == 1) total = at - head;
    const int t = (int)(threadIdx.x % (64 * W)), tail = n > head ? (s.last < n - head ? s.last : n - head) : 0;
    for (int i = t; i < head; i += 64 * W) out[i] = i;
    for (int i = t; i < tail; i += 64 * W) out[head + total + i] = n - tail + i;
    for (int i = head + total + tail + t; i < s.count; i += 64 * W) out[i] = -1;
}

// Longer rows, a workgroup a row and head: the order of the count-th highest score is found eight bits at a time by counting, then what is above it, and
// of its equals the lowest columns, is written in order.
__global__ __launch_bounds__(256) void k_kv_select(KvSelect s) {
    __shared__ uint32_t counts[256], sums[4], found[2];
    const KvView& c = s.c;
    const int64_t unit = kv_workgroup();
    if (unit >= (int64_t)c.rows * c.heads) return;
    const int row = (int)(unit / c.heads);
    int32_t* out = s.chosen + unit * s.count;
    const int pos = kv_position(c, row);
    const int reach = pos < 0 ? 0 : (pos >> c.page_log2) + 1, n = reach < c.columns ? reach : c.columns;
    const float* scores = s.scores + unit * c.columns;
    auto key = [&](int col) { return col < s.first || col >= n - s.last ? 0xffffffffu : order_of(scores[col]); };
    uint32_t prefix = 0, want = (uint32_t)s.count;
    for (int shift = 24; shift >= 0; shift -= 8) {
        counts[threadIdx.x] = 0;
        if (threadIdx.x == 0) found[0] = 0xffffffffu;
        __syncthreads();
        for (int col = threadIdx.x; col < n; col += 256) {
            const uint32_t k = key(col);
            if (k && (shift == 24 || k >> (shift + 8) == prefix)) atomicAdd(&counts[k >> shift & 255], 1u);
        }
        __syncthreads();
        uint32_t all;
        const uint32_t mine = counts[255 - threadIdx.x], above = before256(mine, sums, all);
        if (above < want && above + mine >= want) { found[0] = 255 - threadIdx.x; found[1] = want - above; }
        __syncthreads();
        if (found[0] == 0xffffffffu) { prefix = 0; want = 0; break; }            // fewer than count: all of them
        prefix = prefix << 8 | found[0];
        want = found[1];
        __syncthreads();
    }
    // above `prefix` all, of its equals the first `want`
    uint32_t above = 0, equal = 0;
    for (int col0 = 0; col0 < n; col0 += 256) {
        const int col = col0 + threadIdx.x;
        const uint32_t k = col < n ? key(col) : 0;
        const uint32_t flags = k > prefix ? 1 : (k && k == prefix ? 1u << 16 : 0);
        uint32_t all;
        const uint32_t before = before256(flags, sums, all);
        const uint32_t a = above + (before & 0xffff), e = equal + (before >> 16);
        if (flags == 1 || (flags && e < want)) out[a + (e < want ? e : want)] = col;
        above += all & 0xffff;
        equal += all >> 16;
    }
    for (int i = (int)(above + (equal < want ? equal : want)) + threadIdx.x; i < s.count; i += 256) out[i] = -1;
}

}  // namespace

hipError_t launch_kv_digest(const KvView& c, void* digests, int d, int format, hipStream_t st) {
    uint16_t* p = static_cast<uint16_t*>(digests);
    switch (format) {
        case IVFTQ_KV_F16: return digest<IVFTQ_KV_F16>(c, p, d, st);
        case IVFTQ_KV_BF16: return digest<IVFTQ_KV_BF16>(c, p, d, st);
        default: return digest<IVFTQ_KV_CODE4>(c, p, d, st);
    }
}
hipError_t launch_kv_select(const KvSelect& s, hipStream_t st) {
    const int64_t units = (int64_t)s.c.rows * s.c.heads;
    // Many pairs: a wavefront each, with as many registers as its row is long (6,352 pairs of 1,251 columns: 20.5 us, four wavefronts each 36;
    // 1,024 of 516: 7.6 and 9.9); few, or rows so long that a single wavefront takes too long for them: four (32 of 2,048: 8.5 us, one each 12.9;
    // 1,024 of 2,032: 11.4 and 16).
    const int n = s.c.columns, of_one = (n + 255) / 256, of_four = (n + 511) / 512;
    auto one = [&](auto r) { k_kv_select_held<decltype(r)::value, 1><<<kv_grid((units + 3) / 4, 256), 256, 0, st>>>(s); };
    auto four = [&](auto r) { k_kv_select_held<decltype(r)::value, 4><<<kv_grid(units, 256), 256, 0, st>>>(s); };
    if (n > 4096) k_kv_select<<<kv_grid(units, 256), 256, 0, st>>>(s);
    else if (n <= 2048 && units >= (n <= 1280 ? 1024 : 4096))
        switch (of_one) {
            case 1: one(std::integral_constant<int, 4>{}); break;
            case 2: one(std::integral_constant<int, 8>{}); break;
            case 3: one(std::integral_constant<int, 12>{}); break;
            case 4: one(std::integral_constant<int, 16>{}); break;
            case 5: one(std::integral_constant<int, 20>{}); break;
            case 6: one(std::integral_constant<int, 24>{}); break;
            case 7: one(std::integral_constant<int, 28>{}); break;
            default: one(std::integral_constant<int, 32>{}); break;
        }
    else if (of_four <= 1) four(std::integral_constant<int, 2>{});
    else if (of_four <= 2) four(std::integral_constant<int, 4>{});
    else if (of_four <= 4) four(std::integral_constant<int, 8>{});
    else if (of_four <= 6) four(std::integral_constant<int, 12>{});
    else four(std::integral_constant<int, 16>{});
    return hipGetLastError();
}

}  // namespace ivftq
