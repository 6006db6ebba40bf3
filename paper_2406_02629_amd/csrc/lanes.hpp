// Sums over the lanes of a wave by DPP.
#pragma once
#include "field.hpp"

namespace SS_NS {

// the value of another lane by DPP, 0 where there is none or its row is not in ROWS
template <int CTRL, int ROWS>
__device__ __forceinline__ u32 lane_of(u32 v) { return (u32)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 lane_of(u64 v) { return (u64)lane_of<CTRL, ROWS>((u32)(v >> 32)) << 32 | lane_of<CTRL, ROWS>((u32)v); }

__device__ __forceinline__ u32 read_lane(u32 v, int lane) { return (u32)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 read_lane(u64 v, int lane) { return (u64)read_lane((u32)(v >> 32), lane) << 32 | read_lane((u32)v, lane); }

template <typename T>
__device__ __forceinline__ T row_upto(T v)       // sum of the 16 lanes of a row up to one's own
{
    v += lane_of<0x111, 0xF>(v);                 // row_shr 1, 2, 4, 8
    v += lane_of<0x112, 0xF>(v);
    v += lane_of<0x114, 0xF>(v);
    v += lane_of<0x118, 0xF>(v);
    return v;
}

template <typename T>
__device__ __forceinline__ T wave_upto(T v)
{
    v = row_upto(v);
    v += lane_of<0x142, 0xA>(v);                 // row_bcast 15 to rows 1 and 3, row_bcast 31 to rows 2 and 3
    v += lane_of<0x143, 0xC>(v);
    return v;
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v) { return read_lane(wave_upto(v), 63); }

}  // namespace SS_NS
