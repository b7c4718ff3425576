// Reductions and sums up to a lane over a wavefront without the LDS unit, for numbers of 32 and 64 bits: a value of another lane of a row of
// sixteen comes with a data-parallel move, one of another row by exchanging registers' rows.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace ivftq {

// The value of the lane that CONTROL names; where there is none, zero.
template <int CONTROL, int ROWS = 0xf, class T>
__device__ __forceinline__ T lane_moved(T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xf, false));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CONTROL, ROWS, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CONTROL, ROWS, 0xf, false);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}
// The two values of a pair of lanes 16, or 32, apart.
template <bool FAR>
__device__ __forceinline__ void lane_pair32(uint32_t v, uint32_t& a, uint32_t& b) {
    if constexpr (FAR) { const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false); const uint32_t x = r[0], y = r[1]; a = x; b = y; }
    else { const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false); const uint32_t x = r[0], y = r[1]; a = x; b = y; }
}
template <bool FAR, class T, class Op>
__device__ __forceinline__ T lane_pair(T v, Op op) {
    if constexpr (sizeof(T) == 4) {
        uint32_t a, b;
        lane_pair32<FAR>(__builtin_bit_cast(uint32_t, v), a, b);
        return op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        uint32_t a, b, c, d;
        lane_pair32<FAR>((uint32_t)u, a, b);
        lane_pair32<FAR>((uint32_t)(u >> 32), c, d);
        return op(__builtin_bit_cast(T, (uint64_t)c << 32 | a), __builtin_bit_cast(T, (uint64_t)d << 32 | b));
    }
}

// Over eight neighbouring lanes, aligned; over all.  In every lane.
template <class T, class Op>
__device__ __forceinline__ T lanes8(T v, Op op) {
    v = op(v, lane_moved<0xb1>(v));              // quad_perm: lanes 1 apart
    v = op(v, lane_moved<0x4e>(v));              // 2 apart
    return op(v, lane_moved<0x141>(v));          // the half row turned round: the other four
}
template <class T, class Op>
__device__ __forceinline__ T lanes64(T v, Op op) {
    v = lanes8(v, op);
    v = op(v, lane_moved<0x140>(v));             // the row turned round: the other eight
    return lane_pair<true>(lane_pair<false>(v, op), op);
}
// The sum over the lanes up to this one.
template <class T>
__device__ __forceinline__ T lanes_upto(T v) {
    v += lane_moved<0x111>(v);                   // row_shr: 1, 2, 4, 8
    v += lane_moved<0x112>(v);
    v += lane_moved<0x114>(v);
    v += lane_moved<0x118>(v);
    v += lane_moved<0x142, 0xa>(v);              // the last lane of rows 0 and 2 to the rows behind them
    v += lane_moved<0x143, 0xc>(v);              // lane 31 to rows 2 and 3
    return v;
}

// The largest of the lanes up to this one (not negative).
__device__ __forceinline__ uint32_t lanes_most_upto(uint32_t v) {
    auto most = [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return a > b ? a : b; };
    v = most(v, lane_moved<0x111>(v));
    v = most(v, lane_moved<0x112>(v));
    v = most(v, lane_moved<0x114>(v));
    v = most(v, lane_moved<0x118>(v));
    v = most(v, lane_moved<0x142, 0xa>(v));
    return most(v, lane_moved<0x143, 0xc>(v));
}

struct Larger { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; } };
struct Smaller { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a < b ? a : b; } };
struct Sum { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; } };
struct Union { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a | b; } };

}  // namespace ivftq
