// Attention over the paged cache for many new rows a sequence (prompts, chunks of prompts): bound by the matrix cores.
//
// A workgroup of four wavefronts owns 128 query rows of one (sequence, key-value head): rows are (token, head of the
// group) pairs, so the group's heads share every key and value that is read.  It walks the visible keys in tiles of 64
// tokens, staged in LDS (16-bit pages are copied, codes become float16 levels on the way).  As in kv_few.h the products
// are transposed, S^T = K Q^T and O^T = V^T P^T (v_mfma 32x32x16), and the token order of the key operand is chosen so
// that the scores a lane gets are those it puts into the second product: nothing goes through LDS but keys and values.
#pragma once
#include "kv_few.h"

namespace ivftq {

typedef float floatx16_ __attribute__((ext_vector_type(16)));

constexpr int kManyRows = 128;        // query rows of a workgroup
constexpr int kManyTile = 64;         // tokens of a step

struct ManyArgs {
    KvAttend a;
    const uint16_t* z;                // codes: rotated unit queries, float16, in coordinate order
    const float* zn;                  // codes: the queries' norms
    float* whole;                     // codes: results before they are rotated back
    int32_t row_tiles;                // row tiles a (sequence, head): those of max_new
};

template <int F>
__device__ __forceinline__ floatx16_ kv_mfma32(uintx4 x, uintx4 y, floatx16_ acc) {
    if constexpr (F == IVFTQ_KV_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, x), __builtin_bit_cast(halfx8, y), acc, 0, 0, 0);
}

template <int F, int D>
__global__ __launch_bounds__(256) void k_kv_many(ManyArgs f) {
    constexpr int kKeyPitch = D * 2 + 16;                       // bytes of a key row in LDS: rows 4 banks apart
    __shared__ __align__(16) char keys[kManyTile * kKeyPitch];
    __shared__ __align__(16) char vals[kManyTile / 8 * D * 16];
    __shared__ float key_gain[kManyTile], val_gain[kManyTile];
    const KvAttend& a = f.a;
    const KvView& c = a.c;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
    // heads fastest: with eight heads each XCD reads one head's pages; long row tiles (the last ones) first
    const int h = blockIdx.x % c.heads, rt = f.row_tiles - 1 - (int)(blockIdx.x / c.heads) % f.row_tiles, b = blockIdx.x / c.heads / f.row_tiles;
    const FewSeq s = few_seq(a, b);
    const int cols = s.count * a.group;
    if (rt * kManyRows >= cols) return;
    const int col = rt * kManyRows + wave * 32 + n, used = col < cols ? col : cols - 1;
    const int pos = s.base + used / a.group;
    const int64_t qrow = s.first + used / a.group;
    const int qhead = h * a.group + used % a.group;
    // positions of this workgroup's first and last row, and what they see
    const int last_col = (rt + 1) * kManyRows < cols ? (rt + 1) * kManyRows - 1 : cols - 1;
    const int pos0 = s.base + rt * kManyRows / a.group, pos1 = s.base + last_col / a.group;
    const int end = pos1 + 1 > 0 ? pos1 + 1 : 0;
    const int64_t low64 = a.window ? (int64_t)pos0 - a.window + 1 : 0;
    const int low = low64 > 0 ? (int)low64 : 0;
    const int end_tile = (end + kManyTile - 1) / kManyTile;
    int window_tile = low / kManyTile;
    if (window_tile > end_tile) window_tile = end_tile;
    const int seen = a.sinks < end ? a.sinks : end;
    int sink_tiles = (seen + kManyTile - 1) / kManyTile;
    if (sink_tiles > window_tile) sink_tiles = window_tile;
    const int tiles = sink_tiles + end_tile - window_tile;

    uintx4 q[D / 16];
    float gain = a.scale * kLog2e;
    if constexpr (F == IVFTQ_KV_CODE4) {
        const int64_t at = qrow * a.q.heads + qhead;
        gain *= f.zn[at] * (c.level_unit / kSplitScale);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = *reinterpret_cast<const uintx4*>(f.z + at * D + 16 * k + 8 * half);
    } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(a.q.data) + qrow * a.q.row_stride + qhead * a.q.head_stride + 8 * half;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = *reinterpret_cast<const uintx4*>(p + 16 * k);
    }
    floatx16_ o[D / 32];
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[k][r] = 0.f;
    float m = -INFINITY, l = 0.f;
    // the token (of 32) that this lane's operand row stands for
    const int tok = 16 * (n >> 4) + 8 * (n >> 2 & 1) + 4 * (n >> 3 & 1) + (n & 3);

    for (int i = 0; i < tiles; ++i) {
        const int t0 = (i < sink_tiles ? i : i - sink_tiles + window_tile) * kManyTile;
        __syncthreads();
        bool there = true;                          // every page of the tile exists
        if constexpr (F == IVFTQ_KV_CODE4) {
            const int codes = c.page * (D / 2);
            for (int u = threadIdx.x; u < kManyTile * (D / 8); u += 256) {          // a word of a key row: eight coordinates
                const int t = u / (D / 8), w = u % (D / 8);
                const int64_t page = kv_page(c, b, t0 + t);
                const char* rec = kv_record(c, page < 0 ? 0 : page, h) + (int64_t)((t0 + t) & (c.page - 1)) * (D / 2);
                const halfx8 x = kv_levels8(reinterpret_cast<const uint32_t*>(rec)[w], c);
                halfx8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[kv_slot(e)];
                *reinterpret_cast<halfx8*>(keys + t * kKeyPitch + w * 16) = y;
            }
            for (int u = threadIdx.x; u < kManyTile / 8 * D; u += 256) {            // a word of a value group: eight tokens
                const int og = u / D, j = u % D, t = t0 + 8 * og;
                const int64_t page = kv_page(c, b, t);
                const char* rec = kv_record(c, page < 0 ? 0 : page, h) + codes;
                const halfx8 x = kv_levels8(reinterpret_cast<const uint32_t*>(rec)[(int64_t)((t & (c.page - 1)) >> 3) * D + j], c);
                halfx8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[kv_slot(e)];
                *reinterpret_cast<halfx8*>(vals + u * 16) = y;
            }
            if (threadIdx.x < kManyTile) {
                const int t = t0 + threadIdx.x;
                const int64_t page = kv_page(c, b, t);
                const _Float16* norms = reinterpret_cast<const _Float16*>(kv_record(c, page < 0 ? 0 : page, h) + 2 * codes);
                key_gain[threadIdx.x] = (float)norms[t & (c.page - 1)];
                val_gain[threadIdx.x] = (float)norms[c.page + (t & (c.page - 1))];
            }
        } else {
            for (int u = threadIdx.x; u < kManyTile * (D / 8); u += 256) {
                const int t = u / (D / 8), w = u % (D / 8);
                const int64_t page = kv_page(c, b, t0 + t);
                const char* rec = kv_record(c, page < 0 ? 0 : page, h) + (int64_t)((t0 + t) & (c.page - 1)) * (D * 2);
                *reinterpret_cast<uintx4*>(keys + t * kKeyPitch + w * 16) = reinterpret_cast<const uintx4*>(rec)[w];
            }
            for (int u = threadIdx.x; u < kManyTile / 8 * D; u += 256) {
                const int og = u / D, j = u % D, t = t0 + 8 * og;
                const int64_t page = kv_page(c, b, t);
                const char* rec = kv_record(c, page < 0 ? 0 : page, h) + (int64_t)c.page * (D * 2);
                *reinterpret_cast<uintx4*>(vals + u * 16) = reinterpret_cast<const uintx4*>(rec)[(int64_t)((t & (c.page - 1)) >> 3) * D + j];
            }
        }
        uint32_t absent = 0;                        // quarters of 16 tokens whose page is missing
#pragma unroll
        for (int u = 0; u < 4; ++u) absent |= kv_page(c, b, t0 + 16 * u) < 0 ? 1u << u : 0u;
        there = !absent;
        __syncthreads();
        floatx16_ st[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int r = 0; r < 16; ++r) st[x][r] = 0.f;
            const char* p = keys + (32 * x + tok) * kKeyPitch + 16 * half;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) st[x] = kv_mfma32<F>(*reinterpret_cast<const uintx4*>(p + 32 * k), q[k], st[x]);
        }
        // register r of st[x]: token 32 x + 16 (r / 8) + 8 half + r % 8
        if constexpr (F == IVFTQ_KV_CODE4) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[x][r] *= key_gain[32 * x + 16 * (r >> 3) + 8 * half + (r & 7)] * gain;
        } else {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[x][r] *= gain;
        }
        const bool full = there && t0 + kManyTile - 1 <= pos0 &&
                          (!a.window || (int64_t)t0 > (int64_t)pos1 - a.window || t0 + kManyTile <= a.sinks);
        if (!full) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + 32 * x + 16 * (r >> 3) + 8 * half + (r & 7);
                    const bool mine = t <= pos && !(absent >> (2 * x + (r >> 3)) & 1) && (!a.window || (int64_t)t > (int64_t)pos - a.window || t < a.sinks);
                    if (!mine) st[x][r] = -INFINITY;
                }
        }
        // tokens of the tile with a value that is no finite number: a product would carry it to rows that do not see it
        uint64_t dirty = 0;
        if (F != IVFTQ_KV_CODE4 && !full) {
            for (int u = lane; u < kManyTile / 8 * D; u += 64)
                dirty |= (uint64_t)kv_not_finite<F == IVFTQ_KV_BF16>(*reinterpret_cast<const uintx4*>(vals + u * 16)) << 8 * (u / D);
#pragma unroll
            for (int w = 1; w < 64; w <<= 1) dirty |= __shfl_xor(dirty, w);
        }
        float top = st[0][0];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, st[x][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__ballot(top > m)) {
            const float now = fmaxf(m, top), turn = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= turn;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) o[k] *= turn;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int u = 0; u < 2; ++u) {           // 16 tokens: this lane's half of them in registers 8 u ..
                float pr[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = st[x][8 * u + e];
                    pr[e] = v == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(v - m);
                    l += pr[e];
                }
                const int og = 4 * x + 2 * u + half;             // group of eight tokens in the tile
                if constexpr (F == IVFTQ_KV_CODE4) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) pr[e] = pr[e] == 0.f ? 0.f : pr[e] * val_gain[8 * og + e];
                }
                constexpr bool bf = F == IVFTQ_KV_BF16;
                const uintx4 p = {kv_pack2<bf>(pr[0], pr[1]), kv_pack2<bf>(pr[2], pr[3]), kv_pack2<bf>(pr[4], pr[5]), kv_pack2<bf>(pr[6], pr[7])};
                uintx4 keep = {~0u, ~0u, ~0u, ~0u};
                if (F != IVFTQ_KV_CODE4 && !full) {               // what no row sees may be anything, and 0 * NaN is no zero
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int t = t0 + 8 * og + e;
                        const bool any = t < end && !(absent >> (2 * x + u) & 1) && (t >= low || t < a.sinks) && !(dirty >> (8 * og + e) & 1);
                        if (!any) keep[e >> 1] &= e & 1 ? 0xffffu : 0xffff0000u;
                    }
                }
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const uintx4 v = *reinterpret_cast<const uintx4*>(vals + (og * D + 32 * k + n) * 16);
                    o[k] = kv_mfma32<F>(v & keep, p, o[k]);
                }
            }
        for (uint64_t left = dirty; left; left &= left - 1) {           // one by one, for the rows that see them
            const int t = __builtin_ctzll(left);
            float v = -INFINITY;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) v = 32 * x + 16 * (r >> 3) + (r & 7) == (t & ~8) ? st[x][r] : v;
            v = __shfl(v, n + 32 * (t >> 3 & 1));
            const uint16_t* y = reinterpret_cast<const uint16_t*>(vals + (t >> 3) * D * 16) + (t & 7);
            if (v == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(v - m);
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[k][r] += w * kv_to_float<F == IVFTQ_KV_BF16>(y[(32 * k + 8 * (r >> 2) + 4 * half + (r & 3)) * 8]);
        }
    }
    l += __shfl_xor(l, 32);
    if (col >= cols) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    // register r of o[k]: coordinate 32 k + 8 (r / 4) + 4 half + r % 4
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int j = 32 * k + 2 * r + 4 * half;
            if constexpr (F == IVFTQ_KV_CODE4) {
                *reinterpret_cast<float4*>(f.whole + (qrow * a.q.heads + qhead) * D + j) =
                    make_float4(o[k][r] * inv, o[k][r + 1] * inv, o[k][r + 2] * inv, o[k][r + 3] * inv);
            } else {
                uint16_t* p = reinterpret_cast<uint16_t*>(a.out.data) + qrow * a.out.row_stride + qhead * a.out.head_stride + j;
                constexpr bool bf = F == IVFTQ_KV_BF16;
                *reinterpret_cast<uint2*>(p) = make_uint2(kv_pack2<bf>(o[k][r] * inv, o[k][r + 1] * inv), kv_pack2<bf>(o[k][r + 2] * inv, o[k][r + 3] * inv));
            }
        }
    if (a.lse && half == 0) a.lse[qrow * a.q.heads + qhead] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
}

// Queries into the rotated frame: unit rows in float16, a second part with what the first rounds away, and their norms.
// permuted: eights in the order of kv_levels8.  One wavefront takes 16 rows and 32 coordinates (blockIdx.y).
template <int D>
__global__ __launch_bounds__(64) void k_kv_rotate_queries(KvRows q, const float* __restrict__ pi, uint16_t* __restrict__ z, float* __restrict__ zn, int permuted) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4, block = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * 16 + n, all = (int64_t)q.rows * q.heads;
    const bool in = i < all;
    const int64_t row = in ? i / q.heads : 0, head = in ? i % q.heads : 0;
    const uint16_t* p = reinterpret_cast<const uint16_t*>(q.data) + row * q.row_stride + head * q.head_stride + 8 * g;
    float x[D / 32][8], y[1][8];
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
    kv_rotate16<D, false>(pi, block, x, y);
    if (!in) return;
    if (g == 0 && block == 0) zn[i] = norm;
    halfx8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int at = permuted ? kv_slot(e) : e;
        const float v = y[0][e] * kSplitScale;
        hi[at] = (_Float16)v;
        lo[at] = (_Float16)(v - (float)hi[at]);
    }
    *reinterpret_cast<halfx8*>(z + i * D + 32 * block + 8 * g) = hi;
    *reinterpret_cast<halfx8*>(z + (all + i) * D + 32 * block + 8 * g) = lo;
}

// Results back into the rows' own frame, split the same way.
template <int D>
__global__ __launch_bounds__(64) void k_kv_rotate_back(KvRows out, const float* __restrict__ pi, const float* __restrict__ whole, float unit) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4;
    const int64_t i = (int64_t)blockIdx.x * 16 + n, all = (int64_t)out.rows * out.heads;
    const bool in = i < all;
    const float* p = whole + (in ? i : 0) * D + 8 * g;
    float x[D / 32][8], y[1][8];
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[s][e] = p[32 * s + e];
    const float norm = kv_unit_row<D>(x) * unit;
    kv_rotate16<D, true>(pi, blockIdx.y, x, y);
    if (in) kv_store_turned(out, i / out.heads, i % out.heads, blockIdx.y, y[0], norm);
}

// ---- launches ------------------------------------------------------------------------------------------------------

// Sizes of the workspace's parts, as the launch and the caller's question see them.
struct KvWork {
    int64_t z, zn, whole, part, ml, bytes;
    int32_t few, col_tiles, wgs, split;
};
KvWork kv_work(int format, int d, int batch, int kv_heads, int64_t rows, int q_heads, int max_new, int64_t capacity);

template <int F, int D>
hipError_t kv_attend_launch(const KvAttend& a, const KvWork& w, hipStream_t st) {
    uint16_t* z = reinterpret_cast<uint16_t*>(a.work + w.z);
    float *zn = reinterpret_cast<float*>(a.work + w.zn), *whole = reinterpret_cast<float*>(a.work + w.whole);
    const dim3 rot((unsigned)(((int64_t)a.q.rows * a.q.heads + 15) / 16), D / 32);
    if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_queries<D><<<rot, 64, 0, st>>>(a.q, a.c.rotation, z, zn, w.few);
    const unsigned pairs = (unsigned)(a.c.batch * a.c.heads);
    if (w.few) {
        FewArgs f{a, z, zn, whole, reinterpret_cast<float*>(a.work + w.part), reinterpret_cast<float*>(a.work + w.ml), w.wgs, w.split};
        k_kv_few<F, D><<<dim3(w.split ? (unsigned)w.wgs : pairs, (unsigned)w.col_tiles), 256, 0, st>>>(f);
        if (w.split || F == IVFTQ_KV_CODE4) k_kv_few_join<F, D><<<dim3(pairs, (unsigned)w.col_tiles), 256, 0, st>>>(f);
    } else {
        const int row_tiles = (int)(((int64_t)a.max_new * a.group + kManyRows - 1) / kManyRows);
        ManyArgs f{a, z, zn, whole, row_tiles};
        k_kv_many<F, D><<<pairs * (unsigned)row_tiles, 256, 0, st>>>(f);
        if constexpr (F == IVFTQ_KV_CODE4) k_kv_rotate_back<D><<<rot, 64, 0, st>>>(a.out, a.c.rotation, whole, a.c.level_unit);
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
