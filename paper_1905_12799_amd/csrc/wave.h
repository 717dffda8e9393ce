// Scans and reductions over a wave of 64 lanes in the vector ALU (data-parallel primitives: shifts within rows of 16 lanes, then
// the last lane of a row broadcast to the next ones).  Through LDS a step waits 64 cycles and more, here a few.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rls {

// lanes that have no source, or lie outside the rows of the mask, get `old`
template <int CTRL, int ROWS>
__device__ inline uint32_t lane_move(uint32_t old, uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ inline float lane_move(float old, float x)
{
    return __uint_as_float(lane_move<CTRL, ROWS>(__float_as_uint(old), __float_as_uint(x)));
}
template <int CTRL, int ROWS>
__device__ inline uint64_t lane_move(uint64_t old, uint64_t x)
{
    const uint32_t lo = lane_move<CTRL, ROWS>((uint32_t)old, (uint32_t)x), hi = lane_move<CTRL, ROWS>((uint32_t)(old >> 32), (uint32_t)(x >> 32));
    return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROWS>
__device__ inline double lane_move(double old, double x)
{
    return __longlong_as_double((long long)lane_move<CTRL, ROWS>((uint64_t)__double_as_longlong(old), (uint64_t)__double_as_longlong(x)));
}

// join of a lane's value with those of all lanes before it; join(earlier, later) is associative, `none` changes nothing
template <typename T, typename F>
__device__ inline T wave_scan(T x, T none, F join)
{
    x = join(lane_move<0x111, 0xf>(none, x), x);        // row_shr:1, 2, 4, 8
    x = join(lane_move<0x112, 0xf>(none, x), x);
    x = join(lane_move<0x114, 0xf>(none, x), x);
    x = join(lane_move<0x118, 0xf>(none, x), x);
    x = join(lane_move<0x142, 0xa>(none, x), x);        // row_bcast:15 into rows 1 and 3
    x = join(lane_move<0x143, 0xc>(none, x), x);        // row_bcast:31 into rows 2 and 3
    return x;
}
__device__ inline uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
__device__ inline float last_lane(float x) { return __uint_as_float(last_lane(__float_as_uint(x))); }
__device__ inline uint64_t last_lane(uint64_t x) { return (uint64_t)last_lane((uint32_t)(x >> 32)) << 32 | last_lane((uint32_t)x); }

__device__ inline double last_lane(double x) { return __longlong_as_double((long long)last_lane((uint64_t)__double_as_longlong(x))); }

// The same over rows of 16 lanes, each by itself: a scan, and a join that all lanes of the row get
template <typename T, typename F>
__device__ inline T row_scan(T x, T none, F join)
{
    x = join(lane_move<0x111, 0xf>(none, x), x);
    x = join(lane_move<0x112, 0xf>(none, x), x);
    x = join(lane_move<0x114, 0xf>(none, x), x);
    return join(lane_move<0x118, 0xf>(none, x), x);
}
template <typename T, typename F>
__device__ inline T row_reduce(T x, F join)
{
    x = join(lane_move<0x128, 0xf>(x, x), x);           // row_ror:8, 4, 2, 1
    x = join(lane_move<0x124, 0xf>(x, x), x);
    x = join(lane_move<0x122, 0xf>(x, x), x);
    return join(lane_move<0x121, 0xf>(x, x), x);
}

// over all lanes of a wave, all of them active; the same in every lane
template <typename T, typename F>
__device__ inline T wave_reduce(T x, T none, F join)
{
    return last_lane(wave_scan(x, none, join));
}
__device__ inline uint64_t wave_sum(uint64_t x)
{
    return wave_reduce(x, (uint64_t)0, [](uint64_t a, uint64_t b) { return a + b; });
}
__device__ inline float wave_max(float x)
{
    return wave_reduce(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float wave_min(float x)
{
    return wave_reduce(x, INFINITY, [](float a, float b) { return fminf(a, b); });
}

}  // namespace rls
