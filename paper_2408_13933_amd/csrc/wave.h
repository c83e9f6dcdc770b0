// Reductions and scans over the 64 lanes of a wave by data-parallel-primitive
// moves (a few cycles a step; a shuffle goes through LDS, about a hundred).
// All lanes have to be active.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mq {

template <int CTRL, int ROWS>
__device__ inline uint32_t dpp0(uint32_t v)  // 0 where a lane has no source
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
}

template <int CTRL, int ROWS>
__device__ inline int64_t scan_step(int64_t v)
{
    const uint32_t lo = dpp0<CTRL, ROWS>((uint32_t)v);
    const uint32_t hi = dpp0<CTRL, ROWS>((uint32_t)((uint64_t)v >> 32));
    return v + (int64_t)(((uint64_t)hi << 32) | lo);
}

// The sum of the values of the lanes up to and with this one: shifts inside
// each row of 16, then the rows' last lanes to the rows after them.
__device__ inline int64_t wave_scan(int64_t v)
{
    v = scan_step<0x111, 0xf>(v);  // row_shr:1
    v = scan_step<0x112, 0xf>(v);
    v = scan_step<0x114, 0xf>(v);
    v = scan_step<0x118, 0xf>(v);
    v = scan_step<0x142, 0xa>(v);  // row_bcast:15 to rows 1 and 3
    v = scan_step<0x143, 0xc>(v);  // row_bcast:31 to rows 2 and 3
    return v;
}

__device__ inline int32_t wave_scan(int32_t v)
{
    v += (int32_t)dpp0<0x111, 0xf>((uint32_t)v);
    v += (int32_t)dpp0<0x112, 0xf>((uint32_t)v);
    v += (int32_t)dpp0<0x114, 0xf>((uint32_t)v);
    v += (int32_t)dpp0<0x118, 0xf>((uint32_t)v);
    v += (int32_t)dpp0<0x142, 0xa>((uint32_t)v);
    v += (int32_t)dpp0<0x143, 0xc>((uint32_t)v);
    return v;
}

// A lane's value in all lanes.
__device__ inline int64_t wave_read(int64_t v, int lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)v >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// The sum over the wave, in all lanes.
__device__ inline int64_t wave_sum(int64_t v) { return wave_read(wave_scan(v), 63); }

// The largest over the wave, in all lanes.
__device__ inline uint32_t wave_max(uint32_t v)
{
    v = max(v, dpp0<0x121, 0xf>(v));  // row_ror:1, 2, 4, 8
    v = max(v, dpp0<0x122, 0xf>(v));
    v = max(v, dpp0<0x124, 0xf>(v));
    v = max(v, dpp0<0x128, 0xf>(v));
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

}  // namespace mq
