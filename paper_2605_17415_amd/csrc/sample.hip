// The next token of each row from its logits.  No row is sorted: what decides is always within a short list of tokens, whose ranks are counted.
//   - k_sample_tops reads the logits once and leaves the largest one of every 4,096 tokens (a chunk) and of every 64 (a group).
//   - Few ranks are kept (top_k up to 1,024): at least k tokens are not under the k-th largest group maximum, so the tokens not under it, a
//     little more than k of them in as few groups, are the list (k_sample_rows).
//   - Otherwise a second reading (k_sample_chunks) adds up the weights of every chunk, and where a rank is looked for by its number or its mass, of
//     2,048 bins of logits.  A third reading (k_sample_bins) finds the bins in which the two ranks lie and lists their tokens, among which
//     k_sample_rows counts ranks.
//   - Shorter rows are one workgroup's (k_sample_row), all of it in one launch.
//   - The token is looked for in the chunk in which the sum passes u times all of it.
// Where a list would be too long (thousands of tokens within a bin) the row is worked through digit by digit of the logits' order by one
// workgroup.  For top_k up to 1,024 one group of 64 tokens that holds nothing but a finite value far under the others (a padded or masked vocabulary's lowest
// number, -1e9) is enough: the bins reach down to it, and all other logits fall into the first.  200 rows of 128,000 with top k and top p: 21 us, 791 with the
// last 256 tokens masked so; masked by -infinity 21.  (With the other ways the bins reach down 32 temperatures, whatever the lowest
// logit is; the last one is open, so that a top_k over 1,024 whose last rank lies beyond lists all that is there.)
//
// Weights are whole numbers of 2^-42, so that partial sums of any split and order agree to the last bit, and e^x is computed in 64 bits:
// a float32 weight is off by 2^-23, which over a hundred thousand tokens moves the drawn one in some of every thousand rows.
//
// Measured: 200 rows of 128,000 logits in bfloat16 with settings of all kinds 67 us, the first reading 11 (4.6 TB/s), the second and third 22 and 17,
// of which the weights of half the rows (14 operations in 64 bits each) take a third, the rows 19 (16 us those of 400 ranks: sixteen wavefronts'
// instructions, some 2,500 cycles a digit of ten bits).  One row of 32,000 with top k and top p: 9.2 us.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/ivftq_sample.h"
#include "kernels.h"
#include "wave_ops.h"

namespace ivftq {

void set_last_error(const char* text);

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBlock = kThreads;                 // tokens whose mass is one number of the second level
constexpr int kMostTokens = 1 << 20;
constexpr double kUnit = 4398046511104.0;        // 2^42

constexpr int kChunk = 4096, kGroup = 64, kGroups = kChunk / kGroup;
constexpr int kFewRanks = 1024;                  // top_k that goes by the groups
constexpr int kList = 2048;                      // tokens of a list
constexpr int kBins = 2048;
constexpr int kSliceRows = 1024;                 // rows that share a workspace's places
// Rows that are one workgroup's each, in one launch: of up to 65,536 tokens where there are 256 (64,000: 17 us with top k and top p, 68 with top p alone, 40
// with all tokens; by chunks 20, 109 and 41).  Fewer: up to 32,768 (one row of 32,000 with top k and top p: 9.3 us, 10.4 by chunks, which are three
// launches more), but where it is known that every row needs all of its weights up to 16,384 (top p alone 23 and 24, all tokens 12 and
// 12; of 32,000 34 and 24, 17 and 12).
constexpr int kOneRow = 1 << 16;
inline bool one_row(int64_t rows, int32_t vocabulary, bool weights) { return vocabulary <= (rows >= 256 ? kOneRow : (weights ? kOneRow / 4 : kOneRow / 2)); }

// What a row's search by bins has found.
struct RowBins {
    uint64_t before_k, before_p, total;          // mass of the bins before bin_k, before p0, of all
    int32_t bin_k, p0, p1;                       // the bin of the last rank of top_k (kBins: none), the first and the last that the mass top_p can end in
    uint32_t count_k;                            // tokens before bin_k
};

struct SampleArgs {
    const char* logits;
    int64_t row_stride;
    const float* u;
    ivftq_sampling how;
    int32_t *tokens;
    float* logprobs;
    int32_t vocabulary, rows, chunks;
    // workspace, for each row: chunks' largest and lowest logit, the largest one's place, groups' largest ones, masses; bins, what they tell, the list
    float *chunk_top, *chunk_low, *group_top;
    int32_t* chunk_at;
    uint64_t *chunk_mass, *bin_mass, *list;
    uint32_t *bin_count, *list_count;
    RowBins* found;
};

// How a row is sampled.
enum Way { kTop, kFew, kBinned, kAll };
struct Settings {
    Way way;
    int k;                                       // 0: all
    float p, temperature;                        // p: 1: all
    double least;                                // smallest weight
    __device__ __forceinline__ Settings(const SampleArgs& a, int r) {
        temperature = a.how.temperature ? a.how.temperature[r] : a.how.temperature_all;
        const int top_k = a.how.top_k ? a.how.top_k[r] : a.how.top_k_all;
        const float top_p = a.how.top_p ? a.how.top_p[r] : a.how.top_p_all, min_p = a.how.min_p ? a.how.min_p[r] : a.how.min_p_all;
        k = top_k > 0 && top_k < a.vocabulary ? top_k : 0;
        p = top_p < 1.f ? (top_p > 0.f ? top_p : 0.f) : 1.f;
        least = min_p > 0.f ? (min_p < 1.f ? (double)min_p : 1.0) : 0.0;
        // one rank is the largest logit
        way = !(temperature > 0.f) || k == 1 || p == 0.f ? kTop : (k && k <= kFewRanks ? kFew : (k || p < 1.f ? kBinned : kAll));
    }
};

// A logit and its order: larger numbers have larger keys, both zeros one, what is no number that of -infinity.
template <int T> constexpr int kSize = T == IVFTQ_LOGITS_F32 ? 4 : 2;
__device__ __forceinline__ float counted(float v) { return v == v ? v + 0.f : -INFINITY; }
template <int T>
__device__ __forceinline__ float logit(const char* row, int i) {
    if constexpr (T == IVFTQ_LOGITS_F32) return counted(reinterpret_cast<const float*>(row)[i]);
    else if constexpr (T == IVFTQ_LOGITS_F16) return counted((float)reinterpret_cast<const _Float16*>(row)[i]);
    else return counted(__builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16));
}
// N neighbouring ones from i on, in loads of 16 bytes wherever the row begins; behind the row's end -infinity.
template <int T, int N>
__device__ __forceinline__ void logits_of(const char* row, int i, int n, float (&v)[N]) {
    if (i + N <= n) {
        if constexpr (T == IVFTQ_LOGITS_F32) {
            float w[N];
            __builtin_memcpy(w, row + (int64_t)i * 4, N * 4);
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = counted(w[e]);
        } else {
            uint32_t w[N / 2];
            __builtin_memcpy(w, row + (int64_t)i * 2, N * 2);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t bits = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffff;
                v[e] = counted(T == IVFTQ_LOGITS_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)bits) : __builtin_bit_cast(float, bits << 16));
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = i + e < n ? logit<T>(row, i + e) : -INFINITY;
    }
}
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }
// A token's rank as a number, larger ones first: the key, without the bits that its type leaves alike, and the place from the end.
template <int T> constexpr int kSpare = T == IVFTQ_LOGITS_F32 ? 0 : (T == IVFTQ_LOGITS_F16 ? 13 : 16);
template <int T>
__device__ __forceinline__ uint64_t rank_of(float v, int i) { return (uint64_t)(key_of(v) >> kSpare<T>) << 20 | (uint32_t)(kMostTokens - 1 - i); }
template <int T>
__device__ __forceinline__ float of_rank(uint64_t r) {
    const uint32_t k = (uint32_t)(r >> 20) << kSpare<T>;
    return of_key(k >> 31 ? k : k | ((1u << kSpare<T>) - 1));
}

// e^x for x <= 0 to about 2^-50: x = n ln 2 + r, |r| <= ln 2 / 2, the series of e^r up to r^12.
__device__ __forceinline__ double exp64(double x) {
    if (!(x > -745.0)) return 0.0;
    const double n = __builtin_rint(x * 1.4426950408889634074);
    const double r = __builtin_fma(n, -(-1.904654299957768e-09), __builtin_fma(n, -0.693147182464599609375, x));      // ln 2 in two parts, the first of 24 bits
    double p = 1.0 / 479001600;
    p = __builtin_fma(p, r, 1.0 / 39916800);
    p = __builtin_fma(p, r, 1.0 / 3628800);
    p = __builtin_fma(p, r, 1.0 / 362880);
    p = __builtin_fma(p, r, 1.0 / 40320);
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// Weights of a row: 2^(t / 64) for t = 64 log2(e) (x - top) / temperature, the whole 64ths from a table of 2^(j / 64) in LDS, the rest, at most half a
// 64th, by the series up to its fifth power (2^-54).
__device__ __forceinline__ void fill_table(double* table) {
    if (threadIdx.x < 64) table[threadIdx.x] = threadIdx.x ? 2.0 * exp64((double)((int)threadIdx.x - 64) * (0.69314718055994530942 / 64)) : 1.0;
    __syncthreads();
}
struct Weights {
    float top;
    double first, by;
    const double* table;
    __device__ __forceinline__ Weights(float top_, float temperature, const double* table_) : top(top_), first((double)top_), by(92.332482616893656 / (double)temperature), table(table_) {}
    // top is finite.  -infinity: 2^-64, no mass
    __device__ __forceinline__ double operator()(float v) const {
        constexpr double c = 0.69314718055994530942 / 64, shift = 6755399441055744.0;        // 1.5 * 2^52: sums with it end in a whole number's bits
        const double t = __builtin_fmax(((double)v - first) * by, -4096.0), n = t + shift, r = t - (n - shift);
        double p = c * c * c * c * c / 120;
        p = __builtin_fma(p, r, c * c * c * c / 24);
        p = __builtin_fma(p, r, c * c * c / 6);
        p = __builtin_fma(p, r, c * c / 2);
        p = __builtin_fma(p, r, c);
        p = __builtin_fma(p, r, 1.0);
        const int k = (int)(uint32_t)__builtin_bit_cast(uint64_t, n);
        const uint64_t w = __builtin_bit_cast(uint64_t, table[k & 63] * p);
        return __builtin_bit_cast(double, w + ((uint64_t)(uint32_t)(k >> 6) << 52));
    }
    __device__ __forceinline__ uint64_t mass(float v) const { return whole((*this)(v)); }
    // to a whole number of 2^-42: the last bits of a number of 2^52
    static __device__ __forceinline__ uint64_t whole(double w) { return __builtin_bit_cast(uint64_t, __builtin_fma(w, kUnit, 4503599627370496.0)) & ((1ull << 52) - 1); }
};
// The same where the largest logit may be infinite.
struct AnyWeights : Weights {
    using Weights::Weights;
    __device__ __forceinline__ double operator()(float v) const { return v == top ? 1.0 : (top == INFINITY ? 0.0 : Weights::operator()(v)); }
    __device__ __forceinline__ uint64_t mass(float v) const { return whole((*this)(v)); }
};
// A share of a mass: the tokens that less than it comes before are those that less than this whole number does.
__device__ __forceinline__ uint64_t share_of(float p, uint64_t mass) { return (uint64_t)__builtin_ceil((double)p * (double)mass); }

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// Sum over the threads up to this one; all: over all threads.  sums: W numbers in LDS.
template <int W = kWaves>
__device__ __forceinline__ uint64_t scan(uint64_t v, uint64_t* sums, uint64_t& all) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint64_t incl = lanes_upto(v);
    __syncthreads();
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    const uint64_t of = lane < W ? sums[lane] : 0, upto = lanes_upto(of);
    all = lane_value(upto, W - 1);
    return lane_value(upto - of, wave) + incl;
}

struct Shared {
    uint64_t sums[kWaves], bins[256], blocks[kMostTokens / kBlock];
    uint32_t most[kWaves], digit;
    uint64_t above;
    double table[64];
};

// Digits of the keys, most significant first: the key at which sum(amount of larger keys) < want <= sum(amount of keys not smaller), and
// the first of the two sums.  Keys under `least` are left out.
template <int T, class Amount>
__device__ __forceinline__ uint32_t find_key(const char* row, int n, uint32_t least, uint64_t want, Shared& s, uint64_t& above, Amount amount) {
    uint32_t prefix = 0;
    above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) s.bins[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float v = logit<T>(row, i);
            const uint32_t k = key_of(v);
            if (k >= least && (shift == 24 || k >> (shift + 8) == prefix)) {
                const uint64_t m = amount(v);
                if (m) atomicAdd(reinterpret_cast<unsigned long long*>(&s.bins[k >> shift & 255]), (unsigned long long)m);
            }
        }
        if (threadIdx.x == 0) { s.digit = 0; s.above = 0; }
        __syncthreads();
        const uint64_t mine = threadIdx.x < 256 ? s.bins[255 - threadIdx.x] : 0;
        uint64_t all;
        const uint64_t upto = above + scan(mine, s.sums, all), before = upto - mine;
        if (mine && before < want && upto >= want) { s.digit = 255 - threadIdx.x; s.above = before; }
        __syncthreads();
        prefix = prefix << 8 | s.digit;
        above = s.above;
        __syncthreads();
    }
    return prefix;
}

// u of a whole number of masses: the token is the first up to which more than this has been added up.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t all) {
    if (u >= 1.f) return all - 1;
    const double want = (u > 0.f ? (double)u : 0.0) * (double)all;
    return want < (double)all ? (uint64_t)want : all - 1;
}
__device__ __forceinline__ void drawn(const SampleArgs& a, int r, int token, double weight, uint64_t all) {
    a.tokens[r] = token;
    if (a.logprobs) a.logprobs[r] = (float)log(weight / ((double)all / kUnit));
}
__device__ __forceinline__ void top_token(const SampleArgs& a, int r, float top, int at) {
    if (threadIdx.x) return;
    const bool none = top == -INFINITY;
    a.tokens[r] = none ? -1 : at;
    if (a.logprobs) a.logprobs[r] = none ? -INFINITY : 0.f;
}

// A row by one workgroup, whatever it holds.
template <int T>
__device__ void whole_row(const SampleArgs& a, int r, const Settings& how, Shared& s) {
    const int n = a.vocabulary, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    __syncthreads();
    fill_table(s.table);

    // the largest logit and its first place
    uint32_t best = 0;
    int at = n;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t k = key_of(logit<T>(row, i));
        if (k > best) { best = k; at = i; }
    }
    const uint32_t mine_best = best;
    best = lanes64(best, Larger());
    at = lanes64(mine_best == best ? at : n, Smaller());
    if (lane == 0) { s.most[wave] = best; s.sums[wave] = (uint64_t)at; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (s.most[w] > best || (s.most[w] == best && (int)s.sums[w] < at)) { best = s.most[w]; at = (int)s.sums[w]; }
    __syncthreads();
    const AnyWeights weight(of_key(best), how.temperature, s.table);
    if (weight.top == -INFINITY || how.way == kTop) {
        top_token(a, r, weight.top, at);
        return;
    }

    // kept: keys above `cut`, and of its equals the first `ties`
    uint32_t cut = 0;
    uint64_t ties = ~0ull, above = 0;
    if (how.k) {
        cut = find_key<T>(row, n, 0, (uint64_t)how.k, s, above, [](float) { return (uint64_t)1; });
        ties = (uint64_t)how.k - above;
    }
    if (how.p < 1.f) {
        uint64_t mass = 0, all;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float v = logit<T>(row, i);
            if (ties == ~0ull || key_of(v) > cut) mass += weight.mass(v);
        }
        scan(mass, s.sums, all);
        if (ties != ~0ull) all += ties * weight.mass(of_key(cut));
        const uint64_t want = share_of(how.p, all);
        const uint32_t key = find_key<T>(row, n, cut, want, s, above, [&](float v) { return weight.mass(v); });
        const uint64_t one = weight.mass(of_key(key));
        // rank i of its equals is kept where above + i * one < want
        const uint64_t i = (want - above + one - 1) / one;
        ties = key == cut && i > ties ? ties : i;
        cut = key;
    }
    // the place of the last of the equals that are kept
    int last = n;
    const int blocks = (n + kBlock - 1) / kBlock;
    if (ties != ~0ull) {
        for (int b = wave; b < blocks; b += kWaves) {
            uint32_t count = 0;
            for (int i = b * kBlock + lane; i < (b + 1) * kBlock; i += 64) count += (uint32_t)__popcll(__ballot(i < n && key_of(logit<T>(row, i < n ? i : 0)) == cut));
            if (lane == 0) s.blocks[b] = count;
        }
        __syncthreads();
        uint64_t all;
        const uint64_t mine = (int)threadIdx.x < blocks ? s.blocks[threadIdx.x] : 0, upto = scan(mine, s.sums, all);
        if (threadIdx.x == 0) s.digit = 0xffffffffu;
        __syncthreads();
        if (upto >= ties && upto - mine < ties) { s.digit = threadIdx.x; s.above = upto - mine; }
        __syncthreads();
        if (s.digit != 0xffffffffu) {
            const int i = (int)s.digit * kBlock + threadIdx.x;
            const uint64_t before = s.above, is = i < n && key_of(logit<T>(row, i)) == cut ? 1 : 0;
            __syncthreads();
            const uint64_t place = before + scan(is, s.sums, all);
            if (is && place == ties) s.digit = (uint32_t)i;
            __syncthreads();
            last = (int)s.digit;
        }
        __syncthreads();
    }
    auto kept = [&](int i, double& w) {
        const float v = logit<T>(row, i);
        const uint32_t k = key_of(v);
        w = weight(v);
        return (k > cut || (k == cut && i <= last)) && w >= how.least ? Weights::whole(w) : 0;
    };
    // masses of blocks, the block in which the sum passes u * all, the token in it
    for (int b = wave; b < blocks; b += kWaves) {
        uint64_t mass = 0;
        double w;
        for (int i = b * kBlock + lane; i < (b + 1) * kBlock && i < n; i += 64) mass += kept(i, w);
        mass = lanes64(mass, Sum());
        if (lane == 0) s.blocks[b] = mass;
    }
    __syncthreads();
    uint64_t all;
    const uint64_t mine = (int)threadIdx.x < blocks ? s.blocks[threadIdx.x] : 0, upto = scan(mine, s.sums, all);
    const uint64_t target = target_of(a.u[r], all);
    if (upto > target && upto - mine <= target) { s.digit = threadIdx.x; s.above = upto - mine; }
    __syncthreads();
    const int i = (int)s.digit * kBlock + threadIdx.x;
    const uint64_t before = s.above;
    __syncthreads();
    double w = 0.0;
    uint64_t total;
    const uint64_t one = i < n ? kept(i, w) : 0, sum = before + scan(one, s.sums, total);
    if (sum > target && sum - one <= target) drawn(a, r, i, w, all);
}

// ---- chunks ------------------------------------------------------------------------------------------------------------
constexpr int kChunkThreads = 256;
constexpr int kEach = kChunk / kChunkThreads / 8;         // a thread's pieces of eight tokens

// The first reading: 4,096 tokens a workgroup, bound by memory.
template <int T>
__global__ __launch_bounds__(kChunkThreads) void k_sample_tops(SampleArgs a) {
    __shared__ float tops[4], lows[4];
    __shared__ int places[4];
    const int r = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, n = a.vocabulary, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    const Settings how(a, r);
    float v[kEach][8], top = -INFINITY, low = INFINITY;
#pragma unroll
    for (int j = 0; j < kEach; ++j) logits_of<T, 8>(row, chunk * kChunk + (j * kChunkThreads + threadIdx.x) * 8, n, v[j]);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        float most = v[j][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) most = fmaxf(most, v[j][e]);
        top = fmaxf(top, most);
        if (how.way == kFew) {
            most = lanes8(most, Larger());
            if ((lane & 7) == 0) a.group_top[((int64_t)r * a.chunks + chunk) * kGroups + (j * kChunkThreads + threadIdx.x) / 8] = most;
        }
    }
    if (how.way == kBinned) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) low = v[j][e] > -INFINITY ? fminf(low, v[j][e]) : low;
        low = lanes64(low, Smaller());
    }
    top = lanes64(top, Larger());
    if (lane == 0) { tops[wave] = top; lows[wave] = low; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) { top = fmaxf(top, tops[w]); low = fminf(low, lows[w]); }
    const int64_t to = (int64_t)r * a.chunks + chunk;
    if (threadIdx.x == 0) { a.chunk_top[to] = top; a.chunk_low[to] = low; }
    if (how.way == kTop) {
        int at = n;
#pragma unroll
        for (int j = kEach - 1; j >= 0; --j)
#pragma unroll
            for (int e = 7; e >= 0; --e) at = v[j][e] == top ? chunk * kChunk + (j * kChunkThreads + (int)threadIdx.x) * 8 + e : at;
        at = lanes64(at, Smaller());
        if (lane == 0) places[wave] = at;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) at = places[w] < at ? places[w] : at;
        if (threadIdx.x == 0) a.chunk_at[to] = at;
    }
    if (how.way == kBinned) {                             // what the next readings add to
        for (int i = chunk * kChunkThreads + threadIdx.x; i < kBins; i += a.chunks * kChunkThreads) {
            a.bin_mass[(int64_t)r * kBins + i] = 0;
            a.bin_count[(int64_t)r * kBins + i] = 0;
        }
        if (chunk == 0 && threadIdx.x == 0) a.list_count[r] = 0;
    }
}

// A row's largest logit and the lowest one above -infinity (ways that need it), from those of its chunks; by the whole workgroup (W wavefronts).
struct RowTop { float top, low; };
template <int W>
__device__ __forceinline__ RowTop row_top(const SampleArgs& a, int r) {
    __shared__ float tops[W], lows[W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    RowTop x{-INFINITY, INFINITY};
    for (int c = threadIdx.x; c < a.chunks; c += W * 64) {
        x.top = fmaxf(x.top, a.chunk_top[(int64_t)r * a.chunks + c]);
        x.low = fminf(x.low, a.chunk_low[(int64_t)r * a.chunks + c]);
    }
    x.top = lanes64(x.top, Larger());
    x.low = lanes64(x.low, Smaller());
    if (lane == 0) { tops[wave] = x.top; lows[wave] = x.low; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) { x.top = fmaxf(x.top, tops[w]); x.low = fminf(x.low, lows[w]); }
    return x;
}

// Bins of logits: equally wide, from the largest logit down to the lowest one or 32 temperatures, the last one open; a bin's logits come before
// the next one's.
struct Bins {
    float top, by;
    int last;
    __device__ __forceinline__ Bins(float top_, float low, float reach, int bins) : top(top_), last(bins - 1) {
        const float wide = fminf(top - low, reach);
        by = wide > 0.f ? (float)bins / wide : 0.f;
        if (!(by < 1e30f)) by = 1e30f;
    }
    __device__ __forceinline__ float scaled(float v) const { return (top - v) * by; }
    __device__ __forceinline__ int operator()(float v) const {      // v above -infinity
        const float x = scaled(v);
        return x < (float)last ? (int)x : last;
    }
};
__device__ __forceinline__ Bins row_bins(const RowTop& x, const Settings& how) { return Bins(x.top, x.low, 32.f * how.temperature, kBins); }

// The second reading: chunks' masses, or the masses and numbers of the bins.
template <int T>
__global__ __launch_bounds__(kChunkThreads) void k_sample_chunks(SampleArgs a) {
    __shared__ double table[64];
    __shared__ uint64_t mass[kBins], sums[4];
    __shared__ uint32_t count[kBins];
    const int r = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, n = a.vocabulary;
    const Settings how(a, r);
    if (how.way == kTop || how.way == kFew) return;
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    float v[kEach][8];
#pragma unroll
    for (int j = 0; j < kEach; ++j) logits_of<T, 8>(row, chunk * kChunk + (j * kChunkThreads + threadIdx.x) * 8, n, v[j]);
    const RowTop x = row_top<4>(a, r);
    if (!(__builtin_fabsf(x.top) < INFINITY)) return;                  // one workgroup takes the row whole
    fill_table(table);
    const Weights weight(x.top, how.temperature, table);
    if (how.way == kAll) {
        uint64_t sum = 0;
        // a logit whose weight is surely too small: the logarithm and its product are good to 2^-20 of themselves (and under zero, for infinite
        // temperatures, whose weights are all 1)
        const float under = how.least > 0.0 ? x.top + how.temperature * (1.000002f * logf((float)how.least) - 1e-6f) - __builtin_fabsf(x.top) * 1e-6f : -INFINITY;
#pragma unroll
        for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!__ballot(v[j][e] >= under)) continue;
                const double w = weight(v[j][e]);
                sum += w >= how.least ? Weights::whole(w) : 0;
            }
        sum = lanes64(sum, Sum());
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0) a.chunk_mass[(int64_t)r * a.chunks + chunk] = sums[0] + sums[1] + sums[2] + sums[3];
        return;
    }
    for (int i = threadIdx.x; i < kBins; i += kChunkThreads) { mass[i] = 0; count[i] = 0; }
    __syncthreads();
    const Bins bins = row_bins(x, how);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!(v[j][e] > -INFINITY)) continue;
            const int bin = bins(v[j][e]);
            if (how.p < 1.f) {
                const uint64_t m = weight.mass(v[j][e]);
                if (m) atomicAdd(reinterpret_cast<unsigned long long*>(&mass[bin]), (unsigned long long)m);
            }
            if (how.k) atomicAdd(&count[bin], 1u);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kChunkThreads) {
        if (mass[i]) atomicAdd(reinterpret_cast<unsigned long long*>(&a.bin_mass[(int64_t)r * kBins + i]), (unsigned long long)mass[i]);
        if (count[i]) atomicAdd(&a.bin_count[(int64_t)r * kBins + i], count[i]);
    }
}

// What the bins tell; by W wavefronts, each thread kBins / 64 W of them.  sums: W numbers, value: 4, in LDS.
template <int W>
__device__ __forceinline__ RowBins look_up(const uint64_t* masses, const uint32_t* counts, const Settings& how, uint64_t* sums, uint64_t* value) {
    constexpr int kOwn = kBins / (64 * W);
    uint64_t m[kOwn], mass = 0, count = 0, all, many;
    uint32_t c[kOwn];
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        m[e] = masses[kOwn * threadIdx.x + e];
        c[e] = counts[kOwn * threadIdx.x + e];
        mass += m[e];
        count += c[e];
    }
    mass = scan<W>(mass, sums, all) - mass;
    __syncthreads();
    count = scan<W>(count, sums, many) - count;
    RowBins f{all, 0, all, kBins, kBins, kBins, 0};
    uint64_t in_k = 0;
    if (how.k && many > (uint64_t)how.k) {             // (otherwise every token above -infinity)
        uint64_t before_mass = mass, before = count;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            if (before < (uint64_t)how.k && before + c[e] >= (uint64_t)how.k) {
                value[0] = kOwn * threadIdx.x + e;
                value[1] = before;
                value[2] = before_mass;
                value[3] = m[e];
            }
            before += c[e];
            before_mass += m[e];
        }
        __syncthreads();
        f.bin_k = (int)value[0];
        f.count_k = (uint32_t)value[1];
        f.before_k = value[2];
        in_k = value[3];
        f.p0 = f.bin_k;
        f.p1 = f.bin_k;
        __syncthreads();
    }
    if (how.p < 1.f) {                                 // the mass of the ranks that top_k leaves is before_k to before_k + in_k
        const uint64_t low = share_of(how.p, f.before_k), high = share_of(how.p, f.before_k + in_k);
        if (threadIdx.x == 0) { value[0] = 0; value[1] = 0; value[2] = f.bin_k < kBins ? f.bin_k : kBins - 1; }
        __syncthreads();
        uint64_t before = mass;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            if (before < low && before + m[e] >= low) { value[0] = kOwn * threadIdx.x + e; value[1] = before; }
            if (before < high && before + m[e] >= high) value[2] = kOwn * threadIdx.x + e;
            before += m[e];
        }
        __syncthreads();
        f.p0 = (int)value[0];
        f.before_p = value[1];
        f.p1 = (int)value[2];
    }
    return f;
}

// The third reading: the masses of the chunks' tokens that are kept for certain, and the tokens whose ranks have to be counted.
template <int T>
__global__ __launch_bounds__(kChunkThreads) void k_sample_bins(SampleArgs a) {
    __shared__ double table[64];
    __shared__ uint64_t sums[4], value[4];
    __shared__ uint32_t many, begin;
    const int r = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, n = a.vocabulary;
    const Settings how(a, r);
    if (how.way != kBinned) return;
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    float v[kEach][8];
#pragma unroll
    for (int j = 0; j < kEach; ++j) logits_of<T, 8>(row, chunk * kChunk + (j * kChunkThreads + threadIdx.x) * 8, n, v[j]);
    if (threadIdx.x == 0) many = 0;
    const RowTop x = row_top<4>(a, r);
    if (!(__builtin_fabsf(x.top) < INFINITY)) return;
    fill_table(table);
    const Weights weight(x.top, how.temperature, table);
    const Bins bins = row_bins(x, how);
    const RowBins f = look_up<4>(a.bin_mass + (int64_t)r * kBins, a.bin_count + (int64_t)r * kBins, how, sums, value);
    if (chunk == 0 && threadIdx.x == 0) a.found[r] = f;
    __syncthreads();
    uint64_t sum = 0;
    uint32_t open = 0;                                     // of the thread's tokens: those of the list, a bit each
#pragma unroll
    for (int j = 0; j < kEach; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int bin = v[j][e] > -INFINITY ? bins(v[j][e]) : kBins + 1;
            if (bin < f.p0) {
                const double w = weight(v[j][e]);
                sum += w >= how.least ? Weights::whole(w) : 0;
            } else if (bin <= f.p1 || bin == f.bin_k) {
                open |= 1u << (8 * j + e);
            }
        }
    sum = lanes64(sum, Sum());
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    uint32_t at = open ? atomicAdd(&many, (uint32_t)__popc(open)) : 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        a.chunk_mass[(int64_t)r * a.chunks + chunk] = sums[0] + sums[1] + sums[2] + sums[3];
        begin = many ? atomicAdd(&a.list_count[r], many) : 0;
    }
    __syncthreads();
    at += begin;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (open >> (8 * j + e) & 1) {
                if (at < kList) a.list[(int64_t)r * kList + at] = rank_of<T>(v[j][e], chunk * kChunk + (j * kChunkThreads + (int)threadIdx.x) * 8 + e);
                ++at;
            }
}

// ---- rows --------------------------------------------------------------------------------------------------------------

struct ListShared {
    // Bins of find_rank, their amounts and tokens: one of the two is in use, the other one cleared for the next step.  Before, few_ranks keeps in the
    // second ones the numbers of the groups and what their bins count.
    uint64_t bins[2][1024], sums[8][kWaves], value[4];
    uint32_t tally[2][1024], many[3];
    uint64_t mass[kMostTokens / kChunk];           // of chunks
    uint64_t rank[kList];                          // the list's tokens
    double table[64];
    __device__ __forceinline__ void clear() { bins[0][threadIdx.x] = 0; tally[0][threadIdx.x] = 0; }       // for the first find_rank, a barrier before it
};

// Over all threads; at: a number a wavefront, not read since the last barrier.
template <class T, class Op>
__device__ __forceinline__ T all_threads(T v, uint64_t* sums, Op op) {
    T* at = reinterpret_cast<T*>(sums);
    v = lanes64(v, op);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    const T v8 = lanes8(at[threadIdx.x & (kWaves - 1)], op);
    return op(v8, lane_moved<0x140>(v8));
}

// The first of 1,024 bins up to which `want` is reached, the sums before it and up to it (the last bin where none does); the same for every
// thread, with one barrier: each wavefront reads the sums of all and the bins of the one that has it.  `clear` runs before the barrier.
struct FoundBin { int bin; uint64_t before, upto; };
template <class T, class Clear>
__device__ __forceinline__ FoundBin find_bin(const T* bins, uint64_t before, uint64_t want, uint64_t* sums, Clear clear) {
    const int lane = threadIdx.x & 63;
    const uint64_t incl = lanes_upto((uint64_t)bins[threadIdx.x]);
    if (lane == 63) sums[threadIdx.x >> 6] = incl;
    clear();
    __syncthreads();
    const uint64_t of_wave = lane < kWaves ? sums[lane] : 0, upto_wave = before + lanes_upto(of_wave), in_wave = __ballot(upto_wave >= want) & ((1ull << kWaves) - 1);
    const int wave = in_wave ? __builtin_ctzll(in_wave) : kWaves - 1;
    const uint64_t of = (uint64_t)bins[wave * 64 + lane], upto = lane_value(upto_wave - of_wave, wave) + lanes_upto(of), in = __ballot(upto >= want);
    const int at = in ? __builtin_ctzll(in) : 63;
    return {wave * 64 + at, lane_value(upto - of, at), lane_value(upto, at)};
}

// Of the tokens that have an amount, ordered by `by` (all different, the largest first), the one at which the sum reaches `want`: ten bits of `by`
// at a time, from bit `high` on, until one token is left, two barriers each.  Each thread holds two.
constexpr int kHeld = kList / kThreads;
__device__ __forceinline__ uint64_t find_rank(const uint64_t (&by)[kHeld], const uint64_t (&amount)[kHeld], int high, uint64_t before, uint64_t want, ListShared& s, int& turn) {
    uint32_t open = 0;
#pragma unroll
    for (int e = 0; e < kHeld; ++e) open |= amount[e] ? 1u << e : 0;
    int past = high + 1;                             // bits from this one on are alike
    while (true) {
        const int shift = past > 10 ? past - 10 : 0;
        const uint32_t mask = (1u << (past - shift)) - 1;
        uint64_t* bins = s.bins[turn];
        uint32_t* tally = s.tally[turn];
        turn ^= 1;
        uint32_t digit[kHeld];
#pragma unroll
        for (int e = 0; e < kHeld; ++e) {
            digit[e] = mask - ((uint32_t)(by[e] >> shift) & mask);           // the largest first
            if (open >> e & 1) {
                atomicAdd(reinterpret_cast<unsigned long long*>(&bins[digit[e]]), (unsigned long long)amount[e]);
                atomicAdd(&tally[digit[e]], 1u);
            }
        }
        __syncthreads();
        const FoundBin found = find_bin(bins, before, want, s.sums[7], [&]() __attribute__((always_inline)) { s.bins[turn][threadIdx.x] = 0; s.tally[turn][threadIdx.x] = 0; });
        before = found.before;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) open &= (int)digit[e] == found.bin ? ~0u : ~(1u << e);
        if (tally[found.bin] <= 1 || shift == 0) break;
        past = shift;
    }
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
        if (open >> e & 1) s.value[3] = by[e];
    __syncthreads();
    return s.value[3];
}

// The token among those of rank `cut` and better, by the masses of the chunks (in `mass`, a number a chunk).
template <int T>
__device__ __forceinline__ void locate(const SampleArgs& a, int r, const Weights& weight, double least, uint64_t cut, const uint64_t* mass, ListShared& s) {
    static_assert(kMostTokens / kChunk == 256, "a lane has four chunks");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    __syncthreads();
    // the chunk, by every wavefront
    uint64_t m[4], own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) own += m[e] = 4 * lane + e < a.chunks ? mass[4 * lane + e] : 0;
    const uint64_t upto = lanes_upto(own), all = lane_value(upto, 63), target = target_of(a.u[r], all), in = __ballot(upto > target);
    const int of = in ? __builtin_ctzll(in) : 63;
    uint64_t before = lane_value(upto - own, of);
    int chunk = 4 * of;
#pragma unroll
    for (int e = 0; e < 3; ++e) {
        const uint64_t past = before + lane_value(m[e], of);
        if (chunk == 4 * of + e && past <= target) { before = past; ++chunk; }
    }
    const int i = chunk * kChunk + (int)threadIdx.x * 4;
    float v[4];
    logits_of<T, 4>(a.logits + (int64_t)r * a.row_stride * kSize<T>, i, a.vocabulary, v);
    double w[4];
    uint64_t one[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        w[e] = weight(v[e]);
        one[e] = i + e < a.vocabulary && rank_of<T>(v[e], i + e) >= cut && w[e] >= least ? Weights::whole(w[e]) : 0;
        sum += one[e];
    }
    const uint64_t incl = lanes_upto(sum);
    if (lane == 63) s.sums[6][wave] = incl;
    __syncthreads();
    const uint64_t one_wave = lane < kWaves ? s.sums[6][lane] : 0;
    uint64_t at = before + lane_value(lanes_upto(one_wave) - one_wave, wave) + incl - sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (at + one[e] > target && at <= target) drawn(a, r, i + e, w[e], all);
        at += one[e];
    }
}

// Numbers over the lanes put in order, the largest first (a bitonic network: runs of 2, 4, .. 64 lanes, turn by turn rising and falling, are
// joined by comparing lanes J apart).
template <int J>
__device__ __forceinline__ uint64_t ordered(uint64_t v, bool larger) {
    if constexpr (J >= 16) {
        uint32_t a, b, c, d;
        lane_pair32<J == 32>((uint32_t)v, a, b);
        lane_pair32<J == 32>((uint32_t)(v >> 32), c, d);
        const uint64_t x = (uint64_t)c << 32 | a, y = (uint64_t)d << 32 | b;
        return (x > y) == larger ? x : y;
    } else {
        uint64_t other;
        if constexpr (J == 1) other = lane_moved<0xb1>(v);
        else if constexpr (J == 2) other = lane_moved<0x4e>(v);
        else if constexpr (J == 4) other = lane_moved<0x1b>(lane_moved<0x141>(v));      // the half row turned round, and its quads
        else other = lane_moved<0x128>(v);
        return (v > other) == larger ? v : other;
    }
}
template <int K, int J>
__device__ __forceinline__ uint64_t joined(uint64_t v) {
    const int lane = threadIdx.x & 63;
    v = ordered<J>(v, ((lane & J) == 0) == ((lane & K) == 0));
    if constexpr (J > 1) v = joined<K, J / 2>(v);
    return v;
}
__device__ __forceinline__ uint64_t in_order(uint64_t v) { return joined<64, 32>(joined<32, 16>(joined<16, 8>(joined<8, 4>(joined<4, 2>(joined<2, 1>(v)))))); }

// Up to 64 listed tokens: by one wavefront, without a barrier, in the order of their ranks and then of their places.  (Sixteen wavefronts take about
// 2,500 cycles a digit of find_rank, instructions of which each wavefront does its own; this takes as long as one or two.)
template <int T>
__device__ __forceinline__ void short_list(const SampleArgs& a, int r, const Settings& how, const Weights& weight, int n, const uint64_t* list) {
    constexpr uint64_t kMass = (1ull << 43) - 1;          // a token's is 2^42 at most
    const int lane = threadIdx.x & 63;
    const uint64_t rank = in_order(lane < n ? list[lane] : 0);
    const double w = weight(of_rank<T>(rank));
    uint64_t mass = rank && lane < how.k ? Weights::whole(w) : 0;
    if (how.p < 1.f) {
        const uint64_t upto = lanes_upto(mass);
        mass = upto - mass < share_of(how.p, lane_value(upto, 63)) ? mass : 0;
    }
    mass = w >= how.least ? mass : 0;
    const uint64_t place = rank & (kMostTokens - 1), by_place = in_order(mass ? place << 43 | mass : 0), one = by_place & kMass, upto = lanes_upto(one);
    const uint64_t all = lane_value(upto, 63), in = __ballot(upto > target_of(a.u[r], all));
    const uint64_t found = lane_value(by_place, in ? __builtin_ctzll(in) : 63) >> 43;
    if (mass && place == found) drawn(a, r, kMostTokens - 1 - (int)found, w, all);
}

// Few ranks: false where the list would be too long.
template <int T>
__device__ __forceinline__ bool few_ranks(const SampleArgs& a, int r, const Settings& how, float top, const Weights& weight, const float* tops, int groups, ListShared& s) {
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    uint32_t* counts = s.tally[1];
    int* of_groups = reinterpret_cast<int*>(s.bins[1]);
    int turn = 0;
    // the bin of the k-th largest group maximum
    float low = INFINITY;
    for (int g = threadIdx.x; g < groups; g += kThreads) { const float t = tops[g]; low = t > -INFINITY ? fminf(low, t) : low; }
    counts[threadIdx.x] = 0;
    s.clear();
    if (threadIdx.x < 3) s.many[threadIdx.x] = 0;
    low = all_threads(low, s.sums[0], Smaller());
    const Bins bins(top, low, INFINITY, 1024);
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        const float t = tops[g];
        if (t > -INFINITY) atomicAdd(&counts[bins(t)], 1u);
    }
    __syncthreads();
    const FoundBin of_k = find_bin(counts, 0, (uint64_t)how.k, s.sums[1], []() {});
    const int cut_bin = of_k.bin;
    if (of_k.upto > (uint64_t)kList) return false;
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        const float t = tops[g];
        if (t > -INFINITY && bins(t) <= cut_bin) of_groups[atomicAdd(&s.many[0], 1u)] = g;
    }
    __syncthreads();
    const int chosen = (int)s.many[0];
    // their tokens, eight a thread and two such pieces on their way: f(token, logit) for those in the bins up to last_bin.  Few of them are, and all
    // sixteen wavefronts' instructions count: what is not needed for the others is done for those alone (their bins and ranks for all: 15,000 cycles
    // for 411 groups; a group a wavefront: 22,000).
    auto tokens = [&](int last_bin, auto&& f) __attribute__((always_inline)) {
        constexpr int kAhead = 2, kPieces = kGroup / 8;
        const bool every = last_bin >= bins.last;
        const float past = (float)(last_bin + 1);          // of bins.scaled
        for (int u0 = threadIdx.x / kPieces; u0 < chosen; u0 += kThreads / kPieces * kAhead) {
            float v[kAhead][8];
            int i[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int u = u0 + j * (kThreads / kPieces);
                i[j] = u < chosen ? of_groups[u] * kGroup + (int)threadIdx.x % kPieces * 8 : a.vocabulary;
                logits_of<T, 8>(row, i[j], a.vocabulary, v[j]);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                uint32_t in = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) in |= (every ? v[j][e] > -INFINITY : bins.scaled(v[j][e]) < past) ? 1u << e : 0;
                for (; in; in &= in - 1) {
                    const int at = i[j] + __builtin_ctz(in);
                    f(at, logit<T>(row, at));
                }
            }
        }
    };
    auto list = [&](int last_bin, uint32_t& many) __attribute__((always_inline)) {
        tokens(last_bin, [&](int i, float v) __attribute__((always_inline)) {
            const uint32_t at = atomicAdd(&many, 1u);
            if (at < kList) s.rank[at] = rank_of<T>(v, i);
        });
        __syncthreads();
        return (int)many;
    };
    int n = list(cut_bin, s.many[1]);
    if (n > kList) {                               // large logits stand together: the bin of the k-th one, counted
        counts[threadIdx.x] = 0;
        __syncthreads();
        tokens(cut_bin, [&](int, float v) __attribute__((always_inline)) { atomicAdd(&counts[bins(v)], 1u); });
        __syncthreads();
        n = list(find_bin(counts, 0, (uint64_t)how.k, s.sums[2], []() {}).bin, s.many[2]);
        if (n > kList) return false;
    }
    if (n <= 64) {
        if (threadIdx.x < 64) short_list<T>(a, r, how, weight, n, s.rank);
        return true;
    }
    uint64_t rank[kHeld], amount[kHeld], place[kHeld], mixed = 0, sum = 0;
    double w[kHeld];
    const uint64_t any = s.rank[0];
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
        const int i = threadIdx.x + e * kThreads;
        rank[e] = i < n ? s.rank[i] : any;
        amount[e] = i < n;
        w[e] = i < n ? weight(of_rank<T>(rank[e])) : 0.0;
        place[e] = rank[e] & (kMostTokens - 1);
        mixed |= rank[e] ^ any;
    }
    mixed = all_threads(mixed, s.sums[3], Union());
    const int high = 63 - __builtin_clzll(mixed | 1);
    uint64_t cut = n > how.k ? find_rank(rank, amount, high, 0, (uint64_t)how.k, s, turn) : 0;
#pragma unroll
    for (int e = 0; e < kHeld; ++e) sum += amount[e] = amount[e] && rank[e] >= cut ? Weights::whole(w[e]) : 0;
    if (how.p < 1.f) cut = find_rank(rank, amount, high, 0, share_of(how.p, all_threads(sum, s.sums[4], Sum())), s, turn);
    // of what is kept, in the order of the tokens, the first up to which the mass passes the target
    sum = 0;
#pragma unroll
    for (int e = 0; e < kHeld; ++e) sum += amount[e] = rank[e] >= cut && w[e] >= how.least ? amount[e] : 0;
    const uint64_t kept = all_threads(sum, s.sums[5], Sum()), found = find_rank(place, amount, 31 - __builtin_clz((uint32_t)a.vocabulary | 1), 0, target_of(a.u[r], kept) + 1, s, turn);
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
        if (amount[e] && place[e] == found) drawn(a, r, kMostTokens - 1 - (int)found, w[e], kept);
    return true;
}

// Ranks by bins: where exactly they end among the n listed tokens, and the token.  The masses of the chunks' tokens that are kept for certain stand in
// s.mass.
template <int T>
__device__ __forceinline__ void cut_list(const SampleArgs& a, int r, const Settings& how, const Weights& weight, const Bins& bins, const RowBins& f, const uint64_t* list, int n,
                                         ListShared& s) {
    const uint64_t any = n ? list[0] : 0;
    uint64_t rank[kHeld], mass[kHeld], amount[kHeld], mixed = 0, cut = 0;
    int bin[kHeld], turn = 0;
    double w[kHeld];
    s.clear();
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
        const int i = threadIdx.x + e * kThreads;
        rank[e] = i < n ? list[i] : any;
        const float v = of_rank<T>(rank[e]);
        bin[e] = i < n ? bins(v) : kBins + 1;
        w[e] = i < n ? weight(v) : 0.0;
        mass[e] = i < n ? Weights::whole(w[e]) : 0;
        mixed |= rank[e] ^ any;
    }
    mixed = all_threads(mixed, s.sums[3], Union());
    const int high = 63 - __builtin_clzll(mixed | 1);
    uint64_t in_k = 0;
    if (f.bin_k < kBins) {
#pragma unroll
        for (int e = 0; e < kHeld; ++e) amount[e] = bin[e] == f.bin_k;
        cut = find_rank(rank, amount, high, f.count_k, (uint64_t)how.k, s, turn);
#pragma unroll
        for (int e = 0; e < kHeld; ++e) in_k += bin[e] == f.bin_k && rank[e] >= cut ? mass[e] : 0;
    }
    if (how.p < 1.f) {
        const uint64_t all = f.bin_k < kBins ? f.before_k + all_threads(in_k, s.sums[4], Sum()) : f.total;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) amount[e] = bin[e] >= f.p0 && bin[e] <= f.p1 && rank[e] >= cut ? mass[e] : 0;
        cut = find_rank(rank, amount, high, f.before_p, share_of(how.p, all), s, turn);
    }
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
        if (mass[e] && rank[e] >= cut && w[e] >= how.least) {
            const int place = kMostTokens - 1 - (int)((uint32_t)rank[e] & (kMostTokens - 1));
            atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[place / kChunk]), (unsigned long long)mass[e]);
        }
    locate<T>(a, r, weight, how.least, cut, s.mass, s);
}

// After the readings: each row's token.
template <int T>
__global__ __launch_bounds__(kThreads) void k_sample_rows(SampleArgs a) {
    __shared__ union { ListShared list; Shared whole; } s;
    const int r = blockIdx.x;
    const Settings how(a, r);
    const RowTop x = row_top<kWaves>(a, r);
    if (x.top == -INFINITY || how.way == kTop) {
        int at = a.vocabulary;
        if (how.way == kTop)
            for (int c = threadIdx.x; c < a.chunks; c += kThreads)
                if (a.chunk_top[(int64_t)r * a.chunks + c] == x.top) at = min(at, a.chunk_at[(int64_t)r * a.chunks + c]);
        top_token(a, r, x.top, all_threads(at, s.list.sums[0], Smaller()));
        return;
    }
    bool done = x.top < INFINITY;
    if (done) {
        const uint64_t* masses = a.chunk_mass + (int64_t)r * a.chunks;
        fill_table(s.list.table);
        const Weights weight(x.top, how.temperature, s.list.table);
        if (how.way == kFew) {
            done = few_ranks<T>(a, r, how, x.top, weight, a.group_top + (int64_t)r * a.chunks * kGroups, a.chunks * kGroups, s.list);
        } else if (how.way == kAll) {
            locate<T>(a, r, weight, how.least, 0, masses, s.list);
        } else {
            const int n = (int)a.list_count[r];
            done = n <= kList;
            if (done) {
                for (int c = threadIdx.x; c < a.chunks; c += kThreads) s.list.mass[c] = masses[c];
                cut_list<T>(a, r, how, weight, row_bins(x, how), a.found[r], a.list + (int64_t)r * kList, n, s.list);
            }
        }
    }
    if (!done) whole_row<T>(a, r, how, s.whole);
}

// The same by one workgroup a row, its numbers in LDS, in one launch.
template <int T>
__global__ __launch_bounds__(kThreads) void k_sample_row(SampleArgs a) {
    struct Parts {
        ListShared list;
        uint64_t bin_mass[kBins];
        uint32_t bin_count[kBins];
        float group_top[kOneRow / kGroup];
    };
    __shared__ union { Parts part; Shared whole; } shared;
    Parts& s = shared.part;
    const int r = blockIdx.x, n = a.vocabulary, lane = threadIdx.x & 63;
    const char* row = a.logits + (int64_t)r * a.row_stride * kSize<T>;
    const Settings how(a, r);
    RowTop x{-INFINITY, INFINITY};
    int at = n;
    for (int i0 = 0; i0 < n; i0 += kThreads * 8) {
        const int i = i0 + threadIdx.x * 8;
        float v[8], most;
        logits_of<T, 8>(row, i, n, v);
        most = v[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) most = fmaxf(most, v[e]);
        if (how.way == kTop) {
#pragma unroll
            for (int e = 7; e >= 0; --e) at = v[e] == most && most > x.top ? i + e : at;
        } else if (how.way == kFew) {
            const float group = lanes8(most, Larger());
            if ((lane & 7) == 0 && i < n) s.group_top[i / kGroup] = group;
        } else if (how.way == kBinned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x.low = v[e] > -INFINITY ? fminf(x.low, v[e]) : x.low;
        }
        x.top = fmaxf(x.top, most);
    }
    const float mine = x.top;
    x.top = all_threads(x.top, s.list.sums[6], Larger());
    if (x.top == -INFINITY || how.way == kTop) {
        top_token(a, r, x.top, all_threads(mine == x.top ? at : n, s.list.sums[0], Smaller()));
        return;
    }
    bool done = x.top < INFINITY;
    if (done) {
        fill_table(s.list.table);
        const Weights weight(x.top, how.temperature, s.list.table);
        if (how.way == kFew) {
            done = few_ranks<T>(a, r, how, x.top, weight, s.group_top, (n + kGroup - 1) / kGroup, s.list);
        } else {
            const bool binned = how.way == kBinned;
            x.low = all_threads(x.low, s.list.sums[0], Smaller());
            const Bins bins = row_bins(x, how);
            RowBins f{0, 0, 0, kBins, kBins, kBins, 0};
            if (threadIdx.x < kOneRow / kChunk) s.list.mass[threadIdx.x] = 0;
            if (threadIdx.x == 0) s.list.many[0] = 0;
            if (binned) {
                for (int i = threadIdx.x; i < kBins; i += kThreads) { s.bin_mass[i] = 0; s.bin_count[i] = 0; }
                __syncthreads();
                for (int i = threadIdx.x * 4; i < n; i += kThreads * 4) {
                    float v[4];
                    logits_of<T, 4>(row, i, n, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (!(v[e] > -INFINITY)) continue;
                        const int bin = bins(v[e]);
                        const uint64_t m = how.p < 1.f ? weight.mass(v[e]) : 0;
                        if (m) atomicAdd(reinterpret_cast<unsigned long long*>(&s.bin_mass[bin]), (unsigned long long)m);
                        if (how.k) atomicAdd(&s.bin_count[bin], 1u);
                    }
                }
                __syncthreads();
                f = look_up<kWaves>(s.bin_mass, s.bin_count, how, s.list.sums[1], s.list.value);
            }
            __syncthreads();
            for (int i0 = 0; i0 < n; i0 += kThreads * 4) {           // a chunk
                const int i = i0 + threadIdx.x * 4;
                float v[4];
                logits_of<T, 4>(row, i, n, v);
                uint64_t sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int bin = !binned ? 0 : (v[e] > -INFINITY ? bins(v[e]) : kBins + 1);
                    const double w = weight(v[e]);
                    sum += bin < f.p0 && w >= how.least ? Weights::whole(w) : 0;
                    if (bin >= f.p0 && (bin <= f.p1 || bin == f.bin_k)) {
                        const uint32_t to = atomicAdd(&s.list.many[0], 1u);
                        if (to < kList) s.list.rank[to] = rank_of<T>(v[e], i + e);
                    }
                }
                sum = lanes64(sum, Sum());
                if (lane == 0 && sum) atomicAdd(reinterpret_cast<unsigned long long*>(&s.list.mass[i0 / kChunk]), (unsigned long long)sum);
            }
            __syncthreads();
            const int many = (int)s.list.many[0];
            done = many <= kList;
            if (done && binned) cut_list<T>(a, r, how, weight, bins, f, s.list.rank, many, s.list);
            else if (done) locate<T>(a, r, weight, how.least, 0, s.list.mass, s.list);
        }
    }
    if (!done) whole_row<T>(a, r, how, shared.whole);
}

// What the settings of all rows tell: nothing without settings.
struct Needs {
    bool again, binned;                          // the second and the third reading are not ruled out
    bool weights;                                // every row needs all of its weights
    Needs(const ivftq_sampling* how, int32_t vocabulary) {
        if (!how) { again = binned = weights = true; return; }
        const bool k = how->top_k || (how->top_k_all > 1 && how->top_k_all < vocabulary), few = !how->top_k && k && how->top_k_all <= kFewRanks;
        const bool top = (!how->temperature && how->temperature_all == 0.f) || (!how->top_k && how->top_k_all == 1) || (!how->top_p && how->top_p_all == 0.f);
        again = !top && !few;
        binned = again && (k || how->top_p || how->top_p_all < 1.f);
        weights = again && !how->top_k && !how->temperature;
    }
};

struct SampleWork { int64_t chunk_top, chunk_low, chunk_at, group_top, chunk_mass, bin_mass, bin_count, list, list_count, found, bytes; };
SampleWork sample_work(int64_t rows, int32_t vocabulary, const Needs& needs) {
    SampleWork w{};
    if (one_row(rows, vocabulary, needs.weights)) return w;
    if (rows > kSliceRows) rows = kSliceRows;
    const int64_t chunks = (vocabulary + kChunk - 1) / kChunk;
    int64_t at = 0;
    auto room = [&](int64_t bytes) { const int64_t p = at; at += round_up64(bytes, 256); return p; };
    w.chunk_top = room(rows * chunks * 4);
    w.chunk_low = room(rows * chunks * 4);
    w.chunk_at = room(rows * chunks * 4);
    w.group_top = room(rows * chunks * kGroups * 4);
    w.chunk_mass = room(rows * chunks * 8);
    w.bin_mass = room(rows * kBins * 8);
    w.bin_count = room(rows * kBins * 4);
    w.list = room(rows * kList * 8);
    w.list_count = room(rows * 4);
    w.found = room(rows * (int64_t)sizeof(RowBins));
    w.bytes = at;
    return w;
}

template <int T>
hipError_t sample(SampleArgs a, const SampleWork& w, char* work, hipStream_t st) {
    a.chunks = (a.vocabulary + kChunk - 1) / kChunk;
    const Needs needs(&a.how, a.vocabulary);     // what it rules out is not launched
    if (one_row(a.rows, a.vocabulary, needs.weights)) {
        k_sample_row<T><<<(unsigned)a.rows, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    a.chunk_top = reinterpret_cast<float*>(work + w.chunk_top);
    a.chunk_low = reinterpret_cast<float*>(work + w.chunk_low);
    a.group_top = reinterpret_cast<float*>(work + w.group_top);
    a.chunk_at = reinterpret_cast<int32_t*>(work + w.chunk_at);
    a.chunk_mass = reinterpret_cast<uint64_t*>(work + w.chunk_mass);
    a.bin_mass = reinterpret_cast<uint64_t*>(work + w.bin_mass);
    a.bin_count = reinterpret_cast<uint32_t*>(work + w.bin_count);
    a.list = reinterpret_cast<uint64_t*>(work + w.list);
    a.list_count = reinterpret_cast<uint32_t*>(work + w.list_count);
    a.found = reinterpret_cast<RowBins*>(work + w.found);
    for (int64_t left = a.rows; left > 0; left -= kSliceRows) {
        const unsigned rows = (unsigned)(left < kSliceRows ? left : kSliceRows), wgs = rows * (unsigned)a.chunks;
        k_sample_tops<T><<<wgs, kChunkThreads, 0, st>>>(a);
        if (needs.again) k_sample_chunks<T><<<wgs, kChunkThreads, 0, st>>>(a);
        if (needs.binned) k_sample_bins<T><<<wgs, kChunkThreads, 0, st>>>(a);
        k_sample_rows<T><<<rows, kThreads, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        a.logits += (int64_t)rows * a.row_stride * kSize<T>;
        a.u += rows;
        a.tokens += rows;
        if (a.logprobs) a.logprobs += rows;
        if (a.how.temperature) a.how.temperature += rows;
        if (a.how.top_k) a.how.top_k += rows;
        if (a.how.top_p) a.how.top_p += rows;
        if (a.how.min_p) a.how.min_p += rows;
    }
    return hipSuccess;
}

ivftq_status refuse(ivftq_status code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}
bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

ivftq_status check_logits(const ivftq_logits* x) {
    if (!x) return refuse(IVFTQ_INVALID_ARG, "logits is NULL");
    if (x->type < IVFTQ_LOGITS_F16 || x->type > IVFTQ_LOGITS_F32) return refuse(IVFTQ_INVALID_ARG, "unknown type %d of logits", x->type);
    if (x->vocabulary < 1 || x->vocabulary > kMostTokens) return refuse(IVFTQ_UNSUPPORTED, "vocabulary = %d: 1 to %d", x->vocabulary, kMostTokens);
    if (x->rows < 0 || x->rows > (1 << 22) - 1) return refuse(IVFTQ_INVALID_ARG, "%lld rows: 0 to %d", (long long)x->rows, (1 << 22) - 1);
    if (x->rows > 1 && x->row_stride < x->vocabulary) return refuse(IVFTQ_INVALID_ARG, "rows of %d tokens %lld apart", x->vocabulary, (long long)x->row_stride);
    if (x->rows && (!x->data || !aligned(x->data, x->type == IVFTQ_LOGITS_F32 ? 4 : 2))) return refuse(IVFTQ_INVALID_ARG, "logits is NULL or not aligned to its type");
    return IVFTQ_OK;
}

}  // namespace
}  // namespace ivftq

using namespace ivftq;

extern "C" {

int64_t ivftq_sample_workspace(const ivftq_logits* logits, const ivftq_sampling* how) {
    return check_logits(logits) ? -1 : sample_work(logits->rows, logits->vocabulary, Needs(how, logits->vocabulary)).bytes;
}

ivftq_status ivftq_sample_tokens(const ivftq_logits* logits, const float* u, const ivftq_sampling* how, int32_t* tokens, float* logprobs, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
    if (ivftq_status e = check_logits(logits)) return e;
    if (!how) return refuse(IVFTQ_INVALID_ARG, "how is NULL");
    if (!how->temperature && !(how->temperature_all >= 0.f)) return refuse(IVFTQ_INVALID_ARG, "temperature = %g: 0 and above", (double)how->temperature_all);
    if (!how->top_k && how->top_k_all < 0) return refuse(IVFTQ_INVALID_ARG, "top_k = %d: 0 and above", how->top_k_all);
    if (!how->top_p && !(how->top_p_all >= 0.f && how->top_p_all <= 1.f)) return refuse(IVFTQ_INVALID_ARG, "top_p = %g: 0 to 1", (double)how->top_p_all);
    if (!how->min_p && !(how->min_p_all >= 0.f && how->min_p_all <= 1.f)) return refuse(IVFTQ_INVALID_ARG, "min_p = %g: 0 to 1", (double)how->min_p_all);
    if (!logits->rows) return IVFTQ_OK;
    if (!u || !tokens) return refuse(IVFTQ_INVALID_ARG, "u or tokens is NULL");
    if (!aligned(u, 4) || !aligned(tokens, 4) || !aligned(logprobs, 4) || !aligned(how->temperature, 4) || !aligned(how->top_k, 4) || !aligned(how->top_p, 4) ||
        !aligned(how->min_p, 4))
        return refuse(IVFTQ_INVALID_ARG, "u, tokens, logprobs and the arrays of settings are 4-byte aligned");
    const SampleWork w = sample_work(logits->rows, logits->vocabulary, Needs(how, logits->vocabulary));
    if (w.bytes && (!workspace || workspace_bytes < w.bytes || !aligned(workspace, 256)))
        return refuse(IVFTQ_INVALID_ARG, "workspace of %lld bytes where %lld are needed, 256-byte aligned", (long long)workspace_bytes, (long long)w.bytes);
    SampleArgs a{};
    a.logits = static_cast<const char*>(logits->data);
    a.row_stride = logits->row_stride;
    a.u = u;
    a.how = *how;
    a.tokens = tokens;
    a.logprobs = logprobs;
    a.vocabulary = logits->vocabulary;
    a.rows = (int32_t)logits->rows;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char* work = static_cast<char*>(workspace);
    const hipError_t e = logits->type == IVFTQ_LOGITS_F16    ? sample<IVFTQ_LOGITS_F16>(a, w, work, st)
                         : logits->type == IVFTQ_LOGITS_BF16 ? sample<IVFTQ_LOGITS_BF16>(a, w, work, st)
                                                             : sample<IVFTQ_LOGITS_F32>(a, w, work, st);
    return e == hipSuccess ? IVFTQ_OK : refuse(IVFTQ_HIP_ERROR, "ivftq_sample_tokens: %s", hipGetErrorString(e));
}

}  // extern "C"
