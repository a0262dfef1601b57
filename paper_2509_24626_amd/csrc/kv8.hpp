// Block records held in 8 bits (SS_KV8_*): the layout that the writer, the
// reader and the attention share.  Not part of the public interface.
//
// Codes stand in the order in which the attention's matrix instructions take
// them, in subtiles of T = min(blk, 16) tokens, so that every wave-wide load
// of a record is 16 bytes a lane, 1 KiB in one piece (half as much for blocks
// of 8), with no staging:
//   K: 16 channels of one token a lane:   (c/16)*T*16 + t*16 + c%16
//   V: 4 tokens of 4 channels a lane:     (c%8/4)*T*64 + (t/4)*256 + (c/8)*16 + (c%4)*4 + t%4
// and a lane that holds 8 channels of 4 tokens (16 lanes read a row of bf16)
// has its V codes where they belong and its K codes half there, which one
// exchange between neighbouring lanes completes.
#pragma once

#include "internal.hpp"

namespace ss {

constexpr int kKv8Trailer = 128;  // the record's scales, in a line of their own

__host__ __device__ constexpr int kv8_record(int blk) { return 2 * blk * kHeadDim + kKv8Trailer; }

// A step of a team's search (T = 32 or 64 lanes, each with its own answer):
// the last b of [0, n) with b + begin[b] / BLK <= item.  Items are counted so
// that sequence b's blocks are items from b + begin[b] / BLK on: it has at
// most floor(rows / BLK) + 1 of them, and the next sequence's begin behind.
template <int BLK, int TEAM>
__device__ __forceinline__ int find_item(const int32_t *__restrict__ begin, int n, int64_t item, int lane)
{
    int lo = 0;
    for (int span = n; span > 1;) {
        const int step = (span + TEAM - 1) / TEAM, b = lo + (lane % TEAM) * step;
        unsigned long long at = __ballot(b < n && b + (int64_t)(begin[b < n ? b : n - 1] / BLK) <= item);
        if (TEAM == 32) at = lane & 32 ? at >> 32 : at & 0xFFFFFFFFull;
        lo += (at ? 63 - __builtin_clzll(at) : 0) * step;
        span = step;
    }
    return lo;
}

// inclusive sum over the wave's lanes
__device__ __forceinline__ uint32_t wave_scan_sum(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);  // lane 15 of rows 0, 2 to rows 1, 3
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2, 3
    return x;
}

__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// the other value of a lane pair (lane ^ 1)
__device__ __forceinline__ uint32_t pair_swap(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, false);
}

}  // namespace ss
