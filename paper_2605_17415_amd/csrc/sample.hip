// The next token of each row from its logits: the k-th rank and the rank where the mass reaches p are found by counting (and adding up weights)
// over the digits of the logits' order, most significant first; no row is sorted.
//
// Weights are whole numbers of 2^-42, so that partial sums of any split and order agree to the last bit, and e^x is computed in 64 bits:
// a float32 weight is off by 2^-23, which over a hundred thousand tokens moves the drawn one in some of every thousand rows.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/ivftq_sample.h"
#include "kernels.h"

namespace ivftq {

void set_last_error(const char* text);

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBlock = kThreads;                 // tokens whose mass is one number of the second level
constexpr int kMostTokens = 1 << 20;
constexpr double kUnit = 4398046511104.0;        // 2^42

struct SampleArgs {
    const char* logits;
    int64_t row_stride;
    const float* u;
    ivftq_sampling how;
    int32_t *tokens;
    float* logprobs;
    int32_t vocabulary, rows;
};

// A logit and its order: larger numbers have larger keys, both zeros one, what is no number that of -infinity.
template <int T>
__device__ __forceinline__ float logit(const char* row, int i) {
    float v;
    if constexpr (T == IVFTQ_LOGITS_F32) v = reinterpret_cast<const float*>(row)[i];
    else if constexpr (T == IVFTQ_LOGITS_F16) v = (float)reinterpret_cast<const _Float16*>(row)[i];
    else v = __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
    return v == v ? v + 0.f : -INFINITY;
}
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }

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

// Weights of a row.
struct Weights {
    float top;
    double by;                                   // 1 / temperature
    __device__ __forceinline__ double operator()(float v) const {
        if (v == top) return 1.0;                // both may be infinite
        return v == -INFINITY || top == INFINITY ? 0.0 : exp64(((double)v - (double)top) * by);
    }
    __device__ __forceinline__ uint64_t mass(float v) const { return whole((*this)(v)); }
    // to a whole number of 2^-42: the last bits of a number of 2^52
    static __device__ __forceinline__ uint64_t whole(double w) { return __builtin_bit_cast(uint64_t, __builtin_fma(w, kUnit, 4503599627370496.0)) & ((1ull << 52) - 1); }
};

template <class T>
__device__ __forceinline__ T wave_scan(T v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const T u = __shfl_up(v, o); if (lane >= o) v += u; }
    return v;
}
// Sum over the threads up to this one; all: over all threads.  sums: kWaves numbers in LDS.
template <class T>
__device__ __forceinline__ T scan(T v, T* sums, T& all) {
    const T incl = wave_scan(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = incl;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { before += w < (int)(threadIdx.x >> 6) ? sums[w] : 0; all += sums[w]; }
    return before + incl;
}

struct Shared {
    uint64_t sums[kWaves], bins[256], blocks[kMostTokens / kBlock];
    uint32_t most[kWaves], digit;
    uint64_t above;
};

// Digits of the keys, most significant first: the key at which sum(amount of larger keys) < want <= sum(amount of keys not smaller), and
// the first of the two sums.  Keys under `least` are left out.
template <int T, class Amount>
__device__ __forceinline__ uint32_t find_key(const char* row, int n, uint32_t least, double want, Shared& s, uint64_t& above, Amount amount) {
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
        if (mine && (double)before < want && (double)upto >= want) { s.digit = 255 - threadIdx.x; s.above = before; }
        __syncthreads();
        prefix = prefix << 8 | s.digit;
        above = s.above;
        __syncthreads();
    }
    return prefix;
}

// A workgroup a row.
template <int T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a) {
    __shared__ Shared s;
    const int r = blockIdx.x, n = a.vocabulary, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char* row = a.logits + (int64_t)r * a.row_stride * (T == IVFTQ_LOGITS_F32 ? 4 : 2);
    const float temperature = a.how.temperature ? a.how.temperature[r] : a.how.temperature_all;
    int top_k = a.how.top_k ? a.how.top_k[r] : a.how.top_k_all;
    const float top_p = a.how.top_p ? a.how.top_p[r] : a.how.top_p_all, min_p = a.how.min_p ? a.how.min_p[r] : a.how.min_p_all;

    // the largest logit and its first place
    uint32_t best = 0;
    int at = n;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t k = key_of(logit<T>(row, i));
        if (k > best) { best = k; at = i; }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t k = __shfl_xor(best, o);
        const int i = __shfl_xor(at, o);
        if (k > best || (k == best && i < at)) { best = k; at = i; }
    }
    if (lane == 0) { s.most[wave] = best; s.sums[wave] = (uint64_t)at; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (s.most[w] > best || (s.most[w] == best && (int)s.sums[w] < at)) { best = s.most[w]; at = (int)s.sums[w]; }
    __syncthreads();
    const Weights weight{of_key(best), 1.0 / (double)temperature};
    const bool none = weight.top == -INFINITY;
    if (none || !(temperature > 0.f)) {
        if (threadIdx.x == 0) {
            a.tokens[r] = none ? -1 : at;
            if (a.logprobs) a.logprobs[r] = none ? -INFINITY : 0.f;
        }
        return;
    }

    // kept: keys above `cut`, and of its equals the first `ties`
    uint32_t cut = 0;
    uint64_t ties = ~0ull, above = 0;
    if (top_k > 0 && top_k < n) {
        cut = find_key<T>(row, n, 0, (double)top_k, s, above, [](float) { return (uint64_t)1; });
        ties = (uint64_t)top_k - above;
    }
    if (top_p < 1.f) {
        uint64_t mass = 0, all;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float v = logit<T>(row, i);
            if (ties == ~0ull || key_of(v) > cut) mass += weight.mass(v);
        }
        scan(mass, s.sums, all);
        if (ties != ~0ull) all += ties * weight.mass(of_key(cut));
        const double want = (double)(top_p > 0.f ? top_p : 0.f) * (double)all;
        if (want > 0.0) {
            const uint32_t key = find_key<T>(row, n, cut, want, s, above, [&](float v) { return weight.mass(v); });
            const uint64_t one = weight.mass(of_key(key));
            // rank i of its equals is kept where above + i * one < want
            uint64_t i = (uint64_t)((want - (double)above) / (double)one);
            while (i > 0 && !((double)(above + (i - 1) * one) < want)) --i;
            while ((double)(above + i * one) < want) ++i;
            ties = key == cut && i > ties ? ties : i;
            cut = key;
        } else {
            cut = best;
            ties = 1;
        }
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
            const uint64_t before = s.above, is = i < n && key_of(logit<T>(row, i)) == cut;
            __syncthreads();
            const uint64_t place = before + scan(is, s.sums, all);
            if (is && place == ties) s.digit = (uint32_t)i;
            __syncthreads();
            last = (int)s.digit;
        }
        __syncthreads();
    }
    const double least = min_p > 0.f ? (min_p < 1.f ? (double)min_p : 1.0) : 0.0;
    auto kept = [&](int i, double& w) {
        const float v = logit<T>(row, i);
        const uint32_t k = key_of(v);
        w = weight(v);
        return (k > cut || (k == cut && i <= last)) && w >= least ? Weights::whole(w) : 0;
    };
    // masses of blocks, the block in which the sum passes u * all, the token in it
    for (int b = wave; b < blocks; b += kWaves) {
        uint64_t mass = 0;
        double w;
        for (int i = b * kBlock + lane; i < (b + 1) * kBlock && i < n; i += 64) mass += kept(i, w);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) mass += __shfl_xor(mass, o);
        if (lane == 0) s.blocks[b] = mass;
    }
    __syncthreads();
    uint64_t all;
    const uint64_t mine = (int)threadIdx.x < blocks ? s.blocks[threadIdx.x] : 0, upto = scan(mine, s.sums, all);
    const float u = a.u[r];
    const double want = (u > 0.f ? (double)u : 0.0) * (double)all;
    const uint64_t target = u < 1.f || !(u == u) ? (want < (double)all ? (uint64_t)want : all - 1) : all - 1;
    if (upto > target && upto - mine <= target) { s.digit = threadIdx.x; s.above = upto - mine; }
    __syncthreads();
    const int i = (int)s.digit * kBlock + threadIdx.x;
    const uint64_t before = s.above;
    __syncthreads();
    double w = 0.0;
    uint64_t total;
    const uint64_t one = i < n ? kept(i, w) : 0, sum = before + scan(one, s.sums, total);
    if (sum > target && sum - one <= target) {
        a.tokens[r] = i;
        if (a.logprobs) a.logprobs[r] = (float)log(w / ((double)all / kUnit));
    }
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

int64_t ivftq_sample_workspace(const ivftq_logits* logits) { return check_logits(logits) ? -1 : 0; }

ivftq_status ivftq_sample_tokens(const ivftq_logits* logits, const float* u, const ivftq_sampling* how, int32_t* tokens, float* logprobs, void*, int64_t,
                                 void* stream) {
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
    const SampleArgs a{static_cast<const char*>(logits->data), logits->row_stride, u, *how, tokens, logprobs, logits->vocabulary, (int32_t)logits->rows};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned rows = (unsigned)logits->rows;
    switch (logits->type) {
        case IVFTQ_LOGITS_F16: k_sample<IVFTQ_LOGITS_F16><<<rows, kThreads, 0, st>>>(a); break;
        case IVFTQ_LOGITS_BF16: k_sample<IVFTQ_LOGITS_BF16><<<rows, kThreads, 0, st>>>(a); break;
        default: k_sample<IVFTQ_LOGITS_F32><<<rows, kThreads, 0, st>>>(a); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? IVFTQ_OK : refuse(IVFTQ_HIP_ERROR, "ivftq_sample_tokens: %s", hipGetErrorString(e));
}

}  // extern "C"
