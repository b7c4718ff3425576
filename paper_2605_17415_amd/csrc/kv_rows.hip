// Rows of the paged key-value cache: written to their pages (rotated and quantised where the cache holds codes) and read back.
#include "kv_kernels.h"

namespace ivftq {
namespace {

// Where row r's token lives: its page's record part of head h and its place in the page; null where there is none.
__device__ __forceinline__ char* place_of(const KvView& c, int r, int h, int& t) {
    const int b = kv_sequence_of(c, r);
    int first, count;
    kv_new_rows(c, b, first, count);
    const int pos = kv_length(c, b) - count + (r - first);
    if (r < first || r >= first + count || pos < 0) return nullptr;
    const int64_t page = kv_page(c, b, pos);
    t = pos & (c.page - 1);
    return page < 0 ? nullptr : kv_record(c, page, h);
}

// ---- 16 bits: a thread moves eight coordinates of one row's key and value ------------------------------------------

template <bool READ>
__global__ __launch_bounds__(256) void k_kv_move16(KvView c, KvRows k, KvRows v, int d) {
    const int chunks = d / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row_head = i / chunks;
    const int j = (int)(i % chunks) * 8;
    const int r = (int)(row_head / c.heads), h = (int)(row_head % c.heads);
    if (r >= c.rows) return;
    int t = 0;
    char* rec = place_of(c, r, h, t);
    uint16_t* kr = reinterpret_cast<uint16_t*>(k.data) + r * k.row_stride + h * k.head_stride + j;
    uint16_t* vr = reinterpret_cast<uint16_t*>(v.data) + r * v.row_stride + h * v.head_stride + j;
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

// ---- codes ---------------------------------------------------------------------------------------------------------

// Loads the 16-bit row in the layout of kv_rotate16.
template <int D, bool BF>
__device__ __forceinline__ void load_row(const KvRows& x, int64_t row, int64_t head, bool valid, float (&v)[D / 32][8]) {
    const int g = (threadIdx.x & 63) >> 4;
    const uint16_t* p = reinterpret_cast<const uint16_t*>(x.data) + row * x.row_stride + head * x.head_stride + 8 * g;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        uintx4 w = {0, 0, 0, 0};
        if (valid) w = *reinterpret_cast<const uintx4*>(p + 32 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[s][2 * e] = kv_to_float<BF>(w[e] & 0xffff); v[s][2 * e + 1] = kv_to_float<BF>(w[e] >> 16); }
    }
}

// A wavefront takes 16 (row, head) pairs of keys or of values (blockIdx.y): norm, rotation, levels.  A key's codes are
// whole words of its lane.  A value's code is one half byte in each of d words that it shares with the seven other tokens
// of its group: those words are changed with atomic operations on the own half byte alone, whose order does not matter.
template <int D, bool BF>
__global__ __launch_bounds__(256) void k_kv_append_codes(KvView c, KvRows k, KvRows v) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const bool value = blockIdx.y;
    const int64_t i = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16 + n;
    const bool in = i < (int64_t)c.rows * c.heads;
    const int r = in ? (int)(i / c.heads) : 0, h = in ? (int)(i % c.heads) : 0;
    float x[D / 32][8], y[D / 32][8];
    load_row<D, BF>(value ? v : k, r, h, in, x);
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
    kv_rotate16<D, false>(c.rotation, x, y);
    int t = 0;
    char* rec = in ? place_of(c, r, h, t) : nullptr;
    if (!rec) return;
    const int codes = c.page * (D / 2);
    if (g == 0) reinterpret_cast<_Float16*>(rec + 2 * codes)[(value ? c.page : 0) + t] = (_Float16)norm;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        uint32_t w = 0, nib[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { nib[e] = kv_nibble(y[s][e], c); w |= nib[e] << 4 * e; }
        const int j = g * (D / 4) + 8 * s;
        if (!value) {
            reinterpret_cast<uint32_t*>(rec + (int64_t)t * (D / 2))[j / 8] = w;
        } else {
            uint32_t* p = reinterpret_cast<uint32_t*>(rec + codes) + (int64_t)(t >> 3) * D + j;
            const int shift = 4 * (t & 7);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                atomicAnd(p + e, ~(15u << shift));
                atomicOr(p + e, nib[e] << shift);
            }
        }
    }
}

// The rows that the codes stand for: levels, rotated back, times the norm.
template <int D, bool BF>
__global__ __launch_bounds__(256) void k_kv_read_codes(KvView c, KvRows k, KvRows v) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const bool value = blockIdx.y;
    const int64_t i = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16 + n;
    const bool in = i < (int64_t)c.rows * c.heads;
    const int r = in ? (int)(i / c.heads) : 0, h = in ? (int)(i % c.heads) : 0;
    int t = 0;
    const char* rec = in ? place_of(c, r, h, t) : nullptr;
    const int codes = c.page * (D / 2);
    float x[D / 32][8], y[D / 32][8], norm = 0.f;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        const int j = 32 * s + 8 * g;
        uint32_t w = 0;
        if (rec && !value) w = reinterpret_cast<const uint32_t*>(rec + (int64_t)t * (D / 2))[j / 8];
        if (rec && value) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(rec + codes) + (int64_t)(t >> 3) * D + j;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= (p[e] >> 4 * (t & 7) & 15) << 4 * e;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[s][e] = kv_level(w >> 4 * e & 15, c);
    }
    if (rec) norm = (float)reinterpret_cast<const _Float16*>(rec + 2 * codes)[(value ? c.page : 0) + t];
    kv_rotate16<D, true>(c.rotation, x, y);
    if (!in) return;
    const KvRows& o = value ? v : k;
    uint16_t* out = reinterpret_cast<uint16_t*>(o.data) + r * o.row_stride + h * o.head_stride + g * (D / 4);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        uintx4 w = {0, 0, 0, 0};
        if (rec)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = kv_pack2<BF>(y[s][2 * e] * norm, y[s][2 * e + 1] * norm);
        *reinterpret_cast<uintx4*>(out + 8 * s) = w;
    }
}

template <int D>
hipError_t codes(const KvView& c, const KvRows& k, const KvRows& v, bool read, hipStream_t st) {
    const int64_t tiles = ((int64_t)c.rows * c.heads + 63) / 64;
    const dim3 grid((unsigned)tiles, 2);
    const bool bf = k.type == IVFTQ_KV_BF16;
    if (read) {
        if (bf) k_kv_read_codes<D, true><<<grid, 256, 0, st>>>(c, k, v); else k_kv_read_codes<D, false><<<grid, 256, 0, st>>>(c, k, v);
    } else {
        if (bf) k_kv_append_codes<D, true><<<grid, 256, 0, st>>>(c, k, v); else k_kv_append_codes<D, false><<<grid, 256, 0, st>>>(c, k, v);
    }
    return hipGetLastError();
}

hipError_t move(const KvView& c, const KvRows& k, const KvRows& v, int d, int format, bool read, hipStream_t st) {
    if (!c.rows) return hipSuccess;
    if (format == IVFTQ_KV_CODE4) {
        switch (d) {
            case 64: return codes<64>(c, k, v, read, st);
            case 96: return codes<96>(c, k, v, read, st);
            case 128: return codes<128>(c, k, v, read, st);
            case 192: return codes<192>(c, k, v, read, st);
            default: return codes<256>(c, k, v, read, st);
        }
    }
    const int64_t threads = (int64_t)c.rows * c.heads * (d / 8);
    const unsigned grid = (unsigned)((threads + 255) / 256);
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
