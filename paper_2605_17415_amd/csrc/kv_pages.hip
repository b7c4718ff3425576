// Pages of the key-value cache: taken, shared, given back, brought together, copied.
//
// Who gets which page has to depend on the state alone, so free pages are found by scans over the reference counts (lowest
// first) and dealt out by scans over the rows: one workgroup does a whole call's bookkeeping, a few microseconds for some
// ten thousand pages, bound by the latency of its passes.  Records are moved by a kernel of their own, which fills the chip.
#include "kv_kernels.h"

namespace ivftq {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Sum of v over the threads before this one; total: over all.  Every thread of the workgroup calls it.
__device__ __forceinline__ int scan_before(int v, int& total) {
    __shared__ int sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(incl, o); if (lane >= o) incl += u; }
    __syncthreads();
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { if (w < wave) before += sums[w]; all += sums[w]; }
    total = all;
    return before + incl - v;
}

// The lowest `want` free pages into list; returns how many there are (at most `want`).
__device__ __forceinline__ int lowest_free(const ivftq_kv_pages& s, int want, int32_t* list) {
    int found = 0;
    for (int64_t p0 = 0; p0 < s.pages && found < want; p0 += kThreads) {
        const int64_t p = p0 + threadIdx.x;
        const int free = p < s.pages && s.refs[p] <= 0;
        int total;
        const int rank = found + scan_before(free, total);
        if (free && rank < want) list[rank] = (int32_t)p;
        found += total;
    }
    __syncthreads();
    return found < want ? found : want;
}

__device__ __forceinline__ int length_of(const ivftq_kv_pages& s, int r) {
    const int64_t cap = (int64_t)s.columns * s.page;
    const int n = s.lengths[r];
    return n < 0 ? 0 : (int)(n < cap ? n : cap);
}

__global__ __launch_bounds__(kThreads) void k_kv_reserve(ivftq_kv_pages s, const int32_t* counts, int32_t* granted, int32_t* list) {
    int want = 0;
    auto need_of = [&](int r, int& have, bool& fits) {
        const int n = length_of(s, r), more = counts[r] > 0 ? counts[r] : 0;
        have = (n + s.page - 1) / s.page;
        const int64_t all = ((int64_t)n + more + s.page - 1) / s.page;
        fits = all <= s.columns;
        return fits ? (int)all - have : 0;
    };
    for (int r0 = 0; r0 < s.rows; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        int have = 0, total;
        bool fits = false;
        const int need = r < s.rows ? need_of(r, have, fits) : 0;
        scan_before(need, total);
        want = want + total < s.pages ? want + total : (int)s.pages;      // a sum of two numbers of pages fits 32 bits
    }
    const int found = lowest_free(s, want, list);
    int64_t before = 0;
    for (int r0 = 0; r0 < s.rows; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        int have = 0, total;
        bool fits = false;
        const int need = r < s.rows ? need_of(r, have, fits) : 0;
        const int64_t at = before + scan_before(need, total);
        before += total;
        if (r >= s.rows) continue;
        fits = fits && (!need || at + need <= found);
        granted[r] = fits && counts[r] > 0 ? counts[r] : 0;
        if (!fits) continue;
        for (int i = 0; i < need; ++i) {
            const int32_t p = list[at + i];
            s.table[(int64_t)r * s.table_stride + have + i] = p;
            s.refs[p] = 1;
        }
        s.lengths[r] = length_of(s, r) + granted[r];
    }
}

// scratch: free pages [pages], copies' sources [n], destinations [n], first entry that names a row as child [rows], rows
// that are parents [rows].
__global__ __launch_bounds__(kThreads) void k_kv_fork(ivftq_kv_pages s, const int32_t* parents, const int32_t* children, int n, int32_t* done, int32_t* scratch) {
    int32_t *list = scratch, *src = list + s.pages, *dst = src + n, *claim = dst + n, *parent = claim + s.rows;
    for (int r = threadIdx.x; r < s.rows; r += kThreads) { claim[r] = 0x7fffffff; parent[r] = 0; }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        if ((unsigned)children[i] < (unsigned)s.rows) atomicMin(claim + children[i], i);
        if ((unsigned)parents[i] < (unsigned)s.rows) atomicOr(parent + parents[i], 1);
    }
    __threadfence_block();
    __syncthreads();
    auto ready = [&](int i) {
        const int p = parents[i], c = children[i];
        return (unsigned)p < (unsigned)s.rows && (unsigned)c < (unsigned)s.rows && __hip_atomic_load(claim + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i &&
               !__hip_atomic_load(parent + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) && s.lengths[c] <= 0;
    };
    int want = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        scan_before(i < n && ready(i) && length_of(s, parents[i]) % s.page, total);
        want += total;
    }
    const int found = lowest_free(s, want < s.pages ? want : (int)s.pages, list);
    int before = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const bool ok = i < n && ready(i);
        const bool part = ok && length_of(s, parents[i]) % s.page;
        const int at = before + scan_before(part, total);
        before += total;
        if (i >= n) continue;
        done[i] = ok && (!part || at < found);
        src[i] = dst[i] = -1;
        if (done[i] && part) {
            const int32_t from = s.table[(int64_t)parents[i] * s.table_stride + length_of(s, parents[i]) / s.page];
            src[i] = from >= 0 && from < s.pages ? from : -1;
            dst[i] = list[at];
        }
    }
    __syncthreads();
    for (int64_t u = threadIdx.x; u < (int64_t)n * s.columns; u += kThreads) {
        const int i = (int)(u / s.columns), col = (int)(u % s.columns);
        if (!done[i]) continue;
        const int whole = length_of(s, parents[i]) / s.page;
        int32_t p = -1;
        if (col < whole) {
            p = s.table[(int64_t)parents[i] * s.table_stride + col];
            if (p >= 0 && p < s.pages) atomicAdd(s.refs + p, 1); else p = -1;
        } else if (col == whole && dst[i] >= 0) {
            p = dst[i];
            s.refs[p] = 1;
        }
        s.table[(int64_t)children[i] * s.table_stride + col] = p;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (done[i]) s.lengths[children[i]] = length_of(s, parents[i]);
}

// Entries are taken out with an exchange, so that a row named twice gives its pages back once.
__device__ __forceinline__ void give_back(const ivftq_kv_pages& s, int r, int from, int to) {
    for (int col = from + threadIdx.x; col < to; col += blockDim.x) {
        const int32_t p = atomicExch(s.table + (int64_t)r * s.table_stride + col, -1);
        if (p >= 0 && p < s.pages) atomicSub(s.refs + p, 1);
    }
}
__global__ __launch_bounds__(256) void k_kv_free(ivftq_kv_pages s, const int32_t* rows) {
    const int r = rows[blockIdx.x];
    if ((unsigned)r >= (unsigned)s.rows) return;
    give_back(s, r, 0, s.columns);
    if (threadIdx.x == 0) s.lengths[r] = 0;
}
__global__ __launch_bounds__(256) void k_kv_trim(ivftq_kv_pages s, int window, int sinks) {
    const int r = blockIdx.x, n = length_of(s, r);
    const int64_t low = (int64_t)n - window + 1;              // first token that a row at position n sees
    if (low <= 0) return;
    const int from = (int)(((int64_t)sinks + s.page - 1) / s.page), to = (int)(low / s.page);
    give_back(s, r, from, to < s.columns ? to : s.columns);
}

// scratch: new number of each page [pages], sources [pages], destinations [pages], number of moves.
__global__ __launch_bounds__(kThreads) void k_kv_compact(ivftq_kv_pages s, int32_t* used_out, int32_t* scratch) {
    int32_t *to = scratch, *src = to + s.pages, *dst = src + s.pages;
    int used = 0;
    for (int64_t p0 = 0; p0 < s.pages; p0 += kThreads) {
        const int64_t p = p0 + threadIdx.x;
        int total;
        scan_before(p < s.pages && s.refs[p] > 0, total);
        used += total;
    }
    int moves = 0, holes = 0;
    for (int64_t p0 = 0; p0 < s.pages; p0 += kThreads) {
        const int64_t p = p0 + threadIdx.x;
        const bool in = p < s.pages, busy = in && s.refs[p] > 0;
        const bool move = busy && p >= used, hole = in && !busy && p < used;
        int total;
        const int rank = scan_before(move, total) + moves;
        moves += total;
        const int place = scan_before(hole, total) + holes;
        holes += total;
        if (in) to[p] = (int32_t)p;
        if (move) src[rank] = (int32_t)p;
        if (hole) dst[place] = (int32_t)p;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += kThreads) {
        to[src[i]] = dst[i];
        s.refs[dst[i]] = s.refs[src[i]];
        s.refs[src[i]] = 0;
    }
    if (threadIdx.x == 0) { *used_out = used; scratch[3 * s.pages] = moves; }
}
__global__ __launch_bounds__(256) void k_kv_renumber(ivftq_kv_pages s, const int32_t* to) {
    const int r = blockIdx.x;
    for (int col = threadIdx.x; col < s.columns; col += 256) {
        int32_t* e = s.table + (int64_t)r * s.table_stride + col;
        const int32_t p = *e;
        if (p >= 0 && p < s.pages) *e = to[p];
    }
}

// 16 KB of a record at a time.
constexpr int64_t kPiece = 16384;
__global__ __launch_bounds__(256) void k_kv_copy(ivftq_kv_pools p, const int32_t* src, const int32_t* dst, const int32_t* count, int n) {
    const int64_t pieces = (p.page_bytes + kPiece - 1) / kPiece, each = pieces * p.layers;
    const int moves = count ? (*count < n ? *count : n) : n;
    for (int64_t u = blockIdx.x; u < moves * each; u += gridDim.x) {
        const int i = (int)(u / each);
        const int64_t rest = u % each, layer = rest / pieces, at = rest % pieces * kPiece;
        const int32_t from = src[i], to = dst[i];
        if (from < 0 || from >= p.pages || to < 0 || to >= p.pages) continue;
        char* base = static_cast<char*>(p.pool) + layer * p.layer_stride + at;
        const int64_t bytes = p.page_bytes - at < kPiece ? p.page_bytes - at : kPiece;
        const uintx4* x = reinterpret_cast<const uintx4*>(base + from * p.page_bytes);
        uintx4* y = reinterpret_cast<uintx4*>(base + to * p.page_bytes);
        for (int j = threadIdx.x; j < bytes / 16; j += 256) y[j] = x[j];
    }
}

}  // namespace

hipError_t launch_kv_copy(const ivftq_kv_pools& p, const int32_t* src, const int32_t* dst, const int32_t* count, int n, hipStream_t st) {
    if (!n || !p.layers) return hipSuccess;
    const int64_t units = n * ((p.page_bytes + kPiece - 1) / kPiece) * p.layers;
    k_kv_copy<<<(unsigned)(units < 2048 ? units : 2048), 256, 0, st>>>(p, src, dst, count, n);
    return hipGetLastError();
}
hipError_t launch_kv_reserve(const ivftq_kv_pages& s, const int32_t* counts, int32_t* granted, int32_t* scratch, hipStream_t st) {
    k_kv_reserve<<<1, kThreads, 0, st>>>(s, counts, granted, scratch);
    return hipGetLastError();
}
hipError_t launch_kv_fork(const ivftq_kv_pages& s, const ivftq_kv_pools& p, const int32_t* parents, const int32_t* children, int n, int32_t* done,
                          int32_t* scratch, hipStream_t st) {
    if (!n) return hipSuccess;
    k_kv_fork<<<1, kThreads, 0, st>>>(s, parents, children, n, done, scratch);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_kv_copy(p, scratch + s.pages, scratch + s.pages + n, nullptr, n, st);
}
hipError_t launch_kv_free(const ivftq_kv_pages& s, const int32_t* rows, int n, hipStream_t st) {
    if (!n) return hipSuccess;
    k_kv_free<<<(unsigned)n, 256, 0, st>>>(s, rows);
    return hipGetLastError();
}
hipError_t launch_kv_trim(const ivftq_kv_pages& s, int window, int sinks, hipStream_t st) {
    if (!s.rows) return hipSuccess;
    k_kv_trim<<<(unsigned)s.rows, 256, 0, st>>>(s, window, sinks);
    return hipGetLastError();
}
hipError_t launch_kv_compact(const ivftq_kv_pages& s, const ivftq_kv_pools& p, int32_t* used, int32_t* scratch, hipStream_t st) {
    k_kv_compact<<<1, kThreads, 0, st>>>(s, used, scratch);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && s.rows) {
        k_kv_renumber<<<(unsigned)s.rows, 256, 0, st>>>(s, scratch);
        e = hipGetLastError();
    }
    const int most = (int)(s.pages / 2);              // every move has a hole
    return e != hipSuccess ? e : launch_kv_copy(p, scratch + s.pages, scratch + 2 * s.pages, scratch + 3 * s.pages, most, st);
}

}  // namespace ivftq
