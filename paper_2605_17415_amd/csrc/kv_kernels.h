// What the translation units of the paged key-value cache share: the cache as kernels see it, the page look-up, the
// 4-bit levels, 16-row products with the rotation.  The public side is include/ivftq_kv.h.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/ivftq_kv.h"
#include "kernels.h"

namespace ivftq {

void set_last_error(const char* text);      // api.hip: the message of ivftq_last_error()

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// One layer's cache.  Magnitudes: the eight positive levels, scaled, as float16; low bytes in tab_lo, high bytes in tab_hi.
struct KvView {
    char* pool;
    const int32_t* table;
    const int32_t* lengths;
    const int32_t* starts;       // null: one row per sequence
    const int32_t *asked, *granted;      // append: null, or what the step's reservation was asked for and gave
    const float* rotation;
    int64_t pages, table_stride, head_bytes, page_bytes;
    int32_t batch, columns, page, page_log2, heads, rows;
    uint32_t tab_lo[2], tab_hi[2];
    float level[8], bound[7];    // positive levels and the boundaries between them
    float level_unit;            // level[m] = level_unit * magnitude m, but for the magnitudes' rounding
};

struct KvRows {
    char* data;
    int64_t row_stride, head_stride;      // elements
    int32_t rows, heads, type;
};

struct KvAttend {
    KvView c;
    KvRows q, out;
    float* lse;
    int32_t group, max_new, window, sinks;
    float scale;
    char* work;
};

hipError_t launch_kv_append(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, hipStream_t st);
hipError_t launch_kv_read(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, hipStream_t st);
hipError_t launch_kv_reserve(const ivftq_kv_pages& s, const int32_t* counts, int32_t* granted, int32_t* scratch, hipStream_t st);
hipError_t launch_kv_fork(const ivftq_kv_pages& s, const ivftq_kv_pools& p, const int32_t* parents, const int32_t* children, int n, int32_t* done,
                          int32_t* scratch, hipStream_t st);
hipError_t launch_kv_free(const ivftq_kv_pages& s, const int32_t* rows, int n, hipStream_t st);
hipError_t launch_kv_trim(const ivftq_kv_pages& s, int window, int sinks, hipStream_t st);
hipError_t launch_kv_compact(const ivftq_kv_pages& s, const ivftq_kv_pools& p, int32_t* used, int32_t* scratch, hipStream_t st);
hipError_t launch_kv_copy(const ivftq_kv_pools& p, const int32_t* src, const int32_t* dst, const int32_t* count, int n, hipStream_t st);

inline int64_t kv_head_bytes(int format, int page, int d) {
    return format == IVFTQ_KV_CODE4 ? (int64_t)page * (d + 4) : (int64_t)page * d * 4;
}

#ifdef __HIPCC__

// Workgroups in one row, as the kernel numbers them.  A dimension of a grid counts threads in 32 bits, and a launch of more takes what
// is left of the count without an error; so the row goes on in the third dimension (and a kernel passes over what lies past its end).
inline dim3 kv_grid(int64_t wgs, int threads, unsigned columns = 1) {
    const int64_t most = 0xffffffffll / threads, rows = (wgs + most - 1) / most;
    return dim3((unsigned)((wgs + rows - 1) / rows), columns, (unsigned)rows);
}
__device__ __forceinline__ uint32_t kv_workgroup() { return blockIdx.z * gridDim.x + blockIdx.x; }

// A value that all lanes hold, as a scalar.
__device__ __forceinline__ int kv_uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t kv_uniform(int64_t v) {
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) | (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}
__device__ __forceinline__ int kv_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Tables and lengths are read-only while a kernel runs: read through the constant address space, a uniform index gives a
// scalar load.
typedef const __attribute__((address_space(4))) int32_t* KvInts;
__device__ __forceinline__ int32_t kv_int(const int32_t* p, int64_t i) { return ((KvInts)(uintptr_t)p)[i]; }

// 16 bytes a lane from memory to LDS, without registers: lane l's go to `to` + 16 l (the same `to` in every lane).
__device__ __forceinline__ void kv_load_lds16(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// Before the barrier behind which others read what this wavefront has loaded.
__device__ __forceinline__ void kv_loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A value that is computed here and not further down, where it is used.
__device__ __forceinline__ uint32_t kv_here(uint32_t v) { asm volatile("" : "+v"(v)); return v; }

// ---- sequences and pages -------------------------------------------------------------------------------------------

__device__ __forceinline__ int kv_length(const KvView& c, int b) {
    const int64_t cap = (int64_t)c.columns << c.page_log2;
    const int n = kv_int(c.lengths, b);
    return n < 0 ? 0 : (int)(n < cap ? n : (cap < 0x7fffff00 ? cap : 0x7fffff00));
}

// First row and number of rows of sequence b; what `starts` says is held inside the rows that there are.
__device__ __forceinline__ void kv_new_rows(const KvView& c, int b, int& first, int& count) {
    if (!c.starts) { first = b; count = b < c.rows ? 1 : 0; return; }
    const int s = kv_int(c.starts, b), e = kv_int(c.starts, b + 1);
    first = s < 0 ? 0 : (s < c.rows ? s : c.rows);
    const int end = e < first ? first : (e < c.rows ? e : c.rows);
    count = end - first;
}

// Whether sequence b's reservation was refused: its length does not count the new rows.
__device__ __forceinline__ bool kv_refused(const KvView& c, int b) { return c.asked && kv_int(c.granted, b) < kv_int(c.asked, b); }

// Number of the page that holds token t of sequence b, -1 where there is none.
__device__ __forceinline__ int64_t kv_page(const KvView& c, int b, int t) {
    const int col = t >> c.page_log2;
    if ((unsigned)col >= (unsigned)c.columns) return -1;
    const int32_t id = kv_int(c.table, (int64_t)b * c.table_stride + col);
    return id >= 0 && id < c.pages ? id : -1;
}

__device__ __forceinline__ char* kv_record(const KvView& c, int64_t page, int head) {
    return c.pool + page * c.page_bytes + (int64_t)head * c.head_bytes;
}

// ---- 4-bit levels --------------------------------------------------------------------------------------------------

// Eight half bytes as eight float16 levels, in the order 0 2 4 6 1 3 5 7: the eight magnitudes' high and low bytes are
// each a table of eight bytes, which one byte permutation looks up for four codes at a time, and the sign bit goes into
// the high byte.  14 operations for eight values.
__device__ __forceinline__ halfx8 kv_levels8(uint32_t w, const KvView& c) {
    const uint32_t even = w & 0x07070707u, odd = (w >> 4) & 0x07070707u;
    const uint32_t even_hi = __builtin_amdgcn_perm(c.tab_hi[1], c.tab_hi[0], even) | ((w << 4) & 0x80808080u);
    const uint32_t odd_hi = __builtin_amdgcn_perm(c.tab_hi[1], c.tab_hi[0], odd) | (w & 0x80808080u);
    const uint32_t even_lo = __builtin_amdgcn_perm(c.tab_lo[1], c.tab_lo[0], even);
    const uint32_t odd_lo = __builtin_amdgcn_perm(c.tab_lo[1], c.tab_lo[0], odd);
    uintx4 r;
    r[0] = __builtin_amdgcn_perm(even_hi, even_lo, 0x05010400u);
    r[1] = __builtin_amdgcn_perm(even_hi, even_lo, 0x07030602u);
    r[2] = __builtin_amdgcn_perm(odd_hi, odd_lo, 0x05010400u);
    r[3] = __builtin_amdgcn_perm(odd_hi, odd_lo, 0x07030602u);
    return __builtin_bit_cast(halfx8, r);
}
// Place of half byte i in that order.
__device__ __forceinline__ constexpr int kv_slot(int i) { return (i & 1) * 4 + (i >> 1); }

// Signs and magnitudes of the levels next to eight values (no number: magnitude 0): three comparisons each, every one against
// the boundary that the one before leaves; a word's bits are shifted in from its top by additions with carry.
__device__ __forceinline__ uint32_t kv_nibbles8(const float (&y)[8], const KvView& c) {
    // (copies: a choice between elements of the argument would be branches around its reads)
    const float t0 = c.bound[0], t1 = c.bound[1], t2 = c.bound[2], t3 = c.bound[3], t4 = c.bound[4], t5 = c.bound[5], t6 = c.bound[6];
    uint32_t w = 0;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const float a = __builtin_fabsf(y[e]);
        const bool b2 = a >= t3, b1 = a >= (b2 ? t5 : t1);
        const float high = b1 ? t6 : t4, low = b1 ? t2 : t0;
        const bool b0 = a >= (b2 ? high : low);
        w = w + w + (y[e] < 0.f);
        w = w + w + b2;
        w = w + w + b1;
        w = w + w + b0;
    }
    return w;
}

// ---- 16-bit rows ---------------------------------------------------------------------------------------------------

template <bool BF>
__device__ __forceinline__ float kv_to_float(uint32_t bits) {
    if constexpr (BF) return __builtin_bit_cast(float, bits << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <bool BF>
__device__ __forceinline__ uint16_t kv_from_float(float v) {
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return __builtin_bit_cast(uint16_t, (_Float16)v);
}
template <bool BF>
__device__ __forceinline__ uint32_t kv_pack2(float a, float b) {
    typedef float two __attribute__((ext_vector_type(2)));
    typedef _Float16 two_f16 __attribute__((ext_vector_type(2)));
    typedef __bf16 two_bf16 __attribute__((ext_vector_type(2)));
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector((two{a, b}), two_bf16));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((two{a, b}), two_f16));
}

// Which of the eight 16-bit values of w are no finite numbers, a bit each.
template <bool BF>
__device__ __forceinline__ uint32_t kv_not_finite(uintx4 w) {
    constexpr uint32_t top = BF ? 0x7f80u : 0x7c00u;
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) bad |= ((w[e >> 1] >> 16 * (e & 1)) & top) == top ? 1u << e : 0u;
    return bad;
}

// A value of the lane 16, or 32, lanes away (of the other half of a pair), without the LDS unit: swapping the odd rows of
// one copy with the even rows of another leaves own and other value in two registers.
__device__ __forceinline__ void kv_pair16(float v, float& a, float& b) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned x = r[0], y = r[1];
    a = __builtin_bit_cast(float, x); b = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ void kv_pair32(float v, float& a, float& b) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned x = r[0], y = r[1];
    a = __builtin_bit_cast(float, x); b = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float kv_max32(float v) { float a, b; kv_pair32(v, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float kv_sum32(float v) { float a, b; kv_pair32(v, a, b); return a + b; }
// Over the four lanes of one column (16 apart).
__device__ __forceinline__ float kv_max4(float v) { float a, b; kv_pair16(v, a, b); return kv_max32(fmaxf(a, b)); }
__device__ __forceinline__ float kv_sum4(float v) { float a, b; kv_pair16(v, a, b); return kv_sum32(a + b); }

// ---- products with the rotation ------------------------------------------------------------------------------------

// A row in the operand layout, x[s][e] = coordinate 32 s + 8 (lane / 16) + e of row lane % 16, scaled to length one; returns
// its norm.  What is zero (or shorter than float32 can say) stays zero.
template <int D>
__device__ __forceinline__ float kv_unit_row(float (&x)[D / 32][8]) {
    float n2 = 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) n2 += x[s][e] * x[s][e];
    const float norm = sqrtf(kv_sum4(n2)), inv = norm > 0.f ? 1.f / norm : 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[s][e] *= inv;
    return norm;
}

// 32 coordinates (a block) of y = Pi x, or of Pi^T x, for 16 unit rows at a time.  A lane gets in y[e] of its row, for Pi,
// coordinate 32 block + 8 (lane / 16) + e: which coordinate a row of the matrix operand is can be chosen, and this choice
// leaves a lane with a whole word of codes; for Pi^T coordinate 32 block + 16 (e / 4) + 4 (lane / 16) + e % 4, so that the
// sixteen lanes' reads down a column of Pi are neighbours.  Both sides go in as sums of two float16 numbers, three products:
// y is good to about 2^-21 of the row's length, far under the distance of two levels; one product alone would move one code
// in two thousand.
// What it reads of Pi: asked for early where a chain of other loads comes first.
template <int D, bool TRANSPOSED>
struct KvTurnRows {
    float p[2][D / 32][8];
    __device__ __forceinline__ KvTurnRows(const float* __restrict__ pi, int block) {
        const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = 32 * block + (TRANSPOSED ? 16 * half + m : 8 * (m >> 2) + 4 * half + (m & 3));
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                float(&x)[8] = p[half][s];
                if constexpr (TRANSPOSED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = pi[(32 * s + 8 * g + e) * D + i];
                } else {
                    const float4* r = reinterpret_cast<const float4*>(pi + i * D + 32 * s + 8 * g);
                    const float4 u = r[0], w = r[1];
                    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
                }
            }
        }
    }
};

template <int D, bool TRANSPOSED>
struct KvTurn {
    halfx8 hi[2][D / 32], lo[2][D / 32];
    __device__ __forceinline__ KvTurn(const float* __restrict__ pi, int block) : KvTurn(KvTurnRows<D, TRANSPOSED>(pi, block)) {}
    __device__ __forceinline__ explicit KvTurn(const KvTurnRows<D, TRANSPOSED>& rows) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int s = 0; s < D / 32; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = rows.p[half][s][e] * kSplitScale;
                    hi[half][s][e] = (_Float16)v;
                    lo[half][s][e] = (_Float16)(v - (float)hi[half][s][e]);
                }
    }
    __device__ __forceinline__ void operator()(const float (&x)[D / 32][8], float (&y)[8]) const {
        floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            halfx8 h, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = x[s][e] * kSplitScale;
                h[e] = (_Float16)v;
                l[e] = (_Float16)(v - (float)h[e]);
            }
            product(h, l, s, acc);
        }
        finish(acc, y);
    }
    // Rows in two parts.
    __device__ __forceinline__ void operator()(const halfx8 (&h)[D / 32], const halfx8 (&l)[D / 32], float (&y)[8]) const {
        floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) product(h[s], l[s], s, acc);
        finish(acc, y);
    }
    // Rows that stand in LDS as two parts already (rows.hi[block][lane], rows.lo).
    template <class Rows>
    __device__ __forceinline__ void operator()(const Rows& rows, float (&y)[8]) const {
        const int lane = threadIdx.x & 63;
        floatx4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            product(rows.hi[s][lane], rows.lo[s][lane], s, acc);
        }
        finish(acc, y);
    }
    __device__ __forceinline__ void product(const halfx8& h, const halfx8& l, int s, floatx4 (&acc)[2]) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            acc[half] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[half][s], h, acc[half], 0, 0, 0);
            acc[half] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[half][s], l, acc[half], 0, 0, 0);
            acc[half] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[half][s], h, acc[half], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void finish(const floatx4 (&acc)[2], float (&y)[8]) const {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * half + r] = acc[half][r] * (1.f / (kSplitScale * kSplitScale));
    }
};

// A lane's eight coordinates of block t of Pi^T x into a 16-bit row.
__device__ __forceinline__ void kv_store_turned(const KvRows& out, int64_t row, int64_t head, int t, const float (&y)[8], float norm) {
    uint16_t* p = reinterpret_cast<uint16_t*>(out.data) + row * out.row_stride + head * out.head_stride + 32 * t + 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float a = y[4 * half] * norm, b = y[4 * half + 1] * norm, c = y[4 * half + 2] * norm, d = y[4 * half + 3] * norm;
        *reinterpret_cast<uint2*>(p + 16 * half) = out.type == IVFTQ_KV_BF16 ? make_uint2(kv_pack2<true>(a, b), kv_pack2<true>(c, d))
                                                                             : make_uint2(kv_pack2<false>(a, b), kv_pack2<false>(c, d));
    }
}

#endif
}  // namespace ivftq
