// Pages of the key-value cache: taken, shared, given back, brought together, copied.
//
// Who gets which page has to depend on the state alone, so free pages are found by scans over the reference counts (lowest
// first) and dealt out by scans over the rows: one workgroup does a whole call's bookkeeping, a few microseconds for some
// ten thousand pages, bound by the latency of its passes (4,000 to 5,000 pages: fork 10 us, reserve 5, compact 10).  Records are moved by a
// kernel of their own, which fills the chip (316 MB: 121 us, 5.2 TB/s read and written).
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

// Pages are looked at four a thread, so that some thousands take one pass and one scan (a pass is a chain of loads and
// barriers, about 2 us).
constexpr int kPages = 4;
__device__ __forceinline__ void four_refs(const ivftq_kv_pages& s, int64_t p, int32_t (&refs)[kPages], int32_t past) {
#pragma unroll
    for (int e = 0; e < kPages; ++e) refs[e] = p + e < s.pages ? s.refs[p + e] : past;
}

// The lowest `want` free pages into list; returns how many there are (at most `want`).
__device__ __forceinline__ int lowest_free(const ivftq_kv_pages& s, int want, int32_t* list) {
    int found = 0;
    for (int64_t p0 = 0; p0 < s.pages && found < want; p0 += kThreads * kPages) {
        const int64_t p = p0 + threadIdx.x * kPages;
        int32_t refs[kPages];
        four_refs(s, p, refs, 1);
        int free = 0, total;
#pragma unroll
        for (int e = 0; e < kPages; ++e) free += refs[e] <= 0;
        int rank = found + scan_before(free, total);
#pragma unroll
        for (int e = 0; e < kPages; ++e)
            if (refs[e] <= 0 && rank < want) list[rank++] = (int32_t)(p + e);
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
    auto need_of = [&](int r, int& have, bool& fits) {
        const int n = length_of(s, r), more = counts[r] > 0 ? counts[r] : 0;
        have = (n + s.page - 1) / s.page;
        const int64_t all = ((int64_t)n + more + s.page - 1) / s.page;
        fits = all <= s.columns;
        return fits ? (int)all - have : 0;
    };
    // granted[r] first holds the number of pages that the rows before r need (as far as there can be pages)
    int64_t before = 0;
    for (int r0 = 0; r0 < s.rows; r0 += kThreads) {
        const int r = r0 + threadIdx.x;
        int have = 0, total;
        bool fits = false;
        const int need = r < s.rows ? need_of(r, have, fits) : 0;
        const int64_t at = before + scan_before(need, total);
        if (r < s.rows) granted[r] = (int32_t)(at < s.pages ? at : s.pages);
        before += total;
    }
    const int found = lowest_free(s, (int)(before < s.pages ? before : s.pages), list);
    for (int r = threadIdx.x; r < s.rows; r += kThreads) {
        int have = 0;
        bool fits = false;
        const int need = need_of(r, have, fits), at = granted[r];
        fits = fits && (!need || (int64_t)at + need <= found);
        const int more = fits && counts[r] > 0 ? counts[r] : 0;
        granted[r] = more;
        if (!fits) continue;
        for (int i = 0; i < need; ++i) {
            const int32_t p = list[at + i];
            s.table[(int64_t)r * s.table_stride + have + i] = p;
            s.refs[p] = 1;
        }
        s.lengths[r] = length_of(s, r) + more;
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
    // the parent's last page where it is not full, -1 where there is none (full, or the entry names no page: nothing to copy, and what
    // a page held before is not shown as the child's)
    auto last_part = [&](int i) {
        const int n = length_of(s, parents[i]);
        const int32_t p = n % s.page ? s.table[(int64_t)parents[i] * s.table_stride + n / s.page] : -1;
        return p >= 0 && p < s.pages ? p : -1;
    };
    // src[i] first holds how many pages the entries before i take, dst[i] whether this one takes one
    int want = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        int total;
        const bool ok = i < n && ready(i), part = ok && last_part(i) >= 0;
        const int at = want + scan_before(part, total);
        want += total;
        if (i < n) { done[i] = ok; src[i] = at; dst[i] = part; }
    }
    const int found = lowest_free(s, want < s.pages ? want : (int)s.pages, list);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int at = src[i], part = dst[i];
        done[i] = done[i] && (!part || at < found);
        src[i] = dst[i] = -1;
        if (done[i] && part) {
            src[i] = last_part(i);
            dst[i] = list[at];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x >> 6; i < n; i += kWaves) {         // a wavefront a row
        if (!done[i]) continue;
        const int whole = length_of(s, parents[i]) / s.page, last = dst[i];
        const int32_t* from = s.table + (int64_t)parents[i] * s.table_stride;
        int32_t* row = s.table + (int64_t)children[i] * s.table_stride;
        for (int col = threadIdx.x & 63; col < s.columns; col += 64) {
            int32_t p = -1;
            if (col < whole) {
                p = from[col];
                if (p >= 0 && p < s.pages) atomicAdd(s.refs + p, 1); else p = -1;
            } else if (col == whole && last >= 0) {
                p = last;
                s.refs[p] = 1;
            }
            row[col] = p;
        }
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
__global__ __launch_bounds__(256) void k_kv_free(ivftq_kv_pages s, const int32_t* rows, int n) {
    if (kv_workgroup() >= (uint32_t)n) return;
    const int r = rows[kv_workgroup()];
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
    for (int64_t p0 = 0; p0 < s.pages; p0 += kThreads * kPages) {
        int32_t refs[kPages];
        four_refs(s, p0 + threadIdx.x * kPages, refs, 0);
        int busy = 0, total;
#pragma unroll
        for (int e = 0; e < kPages; ++e) busy += refs[e] > 0;
        scan_before(busy, total);
        used += total;
    }
    int moves = 0, holes = 0;
    for (int64_t p0 = 0; p0 < s.pages; p0 += kThreads * kPages) {
        const int64_t p = p0 + threadIdx.x * kPages;
        int32_t refs[kPages];
        four_refs(s, p, refs, 0);
        int both = 0, total;                             // moves in the low half, holes in the high half: 4096 at most
#pragma unroll
        for (int e = 0; e < kPages; ++e) both += refs[e] > 0 ? p + e >= used : (p + e < s.pages && p + e < used ? 1 << 16 : 0);
        const int at = scan_before(both, total);
        int move = moves + (at & 0xffff), hole = holes + (at >> 16);
        moves += total & 0xffff;
        holes += total >> 16;
#pragma unroll
        for (int e = 0; e < kPages; ++e) {
            if (p + e >= s.pages) break;
            to[p + e] = (int32_t)(p + e);
            if (refs[e] > 0 && p + e >= used) src[move++] = (int32_t)(p + e);
            if (refs[e] <= 0 && p + e < used) dst[hole++] = (int32_t)(p + e);
        }
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
hipError_t launch_kv_fork(const ivftq_kv_pages& s, const ivftq_kv_pools* p, int groups, const int32_t* parents, const int32_t* children, int n, int32_t* done,
                          int32_t* scratch, hipStream_t st) {
    if (!n) return hipSuccess;
    k_kv_fork<<<1, kThreads, 0, st>>>(s, parents, children, n, done, scratch);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < groups && e == hipSuccess; ++i) e = launch_kv_copy(p[i], scratch + s.pages, scratch + s.pages + n, nullptr, n, st);
    return e;
}
hipError_t launch_kv_free(const ivftq_kv_pages& s, const int32_t* rows, int n, hipStream_t st) {
    if (!n) return hipSuccess;
    k_kv_free<<<kv_grid(n, 256), 256, 0, st>>>(s, rows, n);
    return hipGetLastError();
}
hipError_t launch_kv_trim(const ivftq_kv_pages& s, int window, int sinks, hipStream_t st) {
    if (!s.rows) return hipSuccess;
    k_kv_trim<<<(unsigned)s.rows, 256, 0, st>>>(s, window, sinks);
    return hipGetLastError();
}
hipError_t launch_kv_compact(const ivftq_kv_pages& s, const ivftq_kv_pools* p, int groups, int32_t* used, int32_t* scratch, hipStream_t st) {
    k_kv_compact<<<1, kThreads, 0, st>>>(s, used, scratch);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && s.rows) {
        k_kv_renumber<<<(unsigned)s.rows, 256, 0, st>>>(s, scratch);
        e = hipGetLastError();
    }
    const int most = (int)(s.pages / 2);              // every move has a hole
    for (int i = 0; i < groups && e == hipSuccess; ++i) e = launch_kv_copy(p[i], scratch + s.pages, scratch + 2 * s.pages, scratch + 3 * s.pages, most, st);
    return e;
}

}  // namespace ivftq
