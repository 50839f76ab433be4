// Where the rows of a group lie, for kernels over rows ordered by group with offsets that only the device knows.
//
// The groups are [offsets[e], offsets[e + 1]), e < E, with offsets[0] = 0.  Offsets that a caller got wrong must not lead out of
// bounds: a group ends at the running maximum of the offsets, cut to [0, M], and starts where the one before it ended (the first at
// 0), so groups never overlap and their lengths never sum to more than M.  What is left behind the last one counts as group E.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fp8k {

// inclusive scans over the 64 lanes
__device__ __forceinline__ int wave_scan_add(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
__device__ __forceinline__ int wave_scan_max(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d, 64);
        if (lane >= d) v = o > v ? o : v;
    }
    return v;
}

struct GroupTile {
    int group;       // E: the rows behind the last group
    int row0, rows;  // of the tile
    int pad0;        // where the tile's first row lies when every group is padded to multiples of 128
    int total;       // tiles of all groups (with TAIL those behind the last one too)
    bool first;      // its group's first tile
};

// Tile number `index` of all groups cut into tiles of `height` rows, looked up by a whole wavefront; group = -1 where there is none.
// index < 0: only the total.
template <bool TAIL>
__device__ __forceinline__ GroupTile find_group_tile(const int32_t* __restrict__ offsets, int E, int M, int height, int index) {
    const int lane = threadIdx.x & 63;
    GroupTile t{-1, 0, 0, 0, 0, false};
    int end = 0, tiles_before = 0, pad_before = 0;
    for (int e0 = 0; e0 < E + (TAIL ? 1 : 0); e0 += 64) {
        const int e = e0 + lane;
        int b = e < E ? offsets[e + 1] : TAIL && e == E ? M : 0;
        b = b < end ? end : b > M ? M : b;
        b = wave_scan_max(b);
        int a = __shfl_up(b, 1, 64);
        if (lane == 0) a = end;
        const int n = b - a, tiles = (n + height - 1) / height, pad = (n + 127) & ~127;
        const int tiles_to = tiles_before + wave_scan_add(tiles), pad_to = pad_before + wave_scan_add(pad);
        const uint64_t hit = __ballot(index >= 0 && index < tiles_to);
        if (t.group < 0 && hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            const int in = index - (__shfl(tiles_to, l, 64) - __shfl(tiles, l, 64));
            const int a_l = __shfl(a, l, 64), n_l = __shfl(n, l, 64);
            t.group = e0 + l;
            t.row0 = a_l + in * height;
            t.first = in == 0;
            t.rows = n_l - in * height < height ? n_l - in * height : height;
            t.pad0 = __shfl(pad_to, l, 64) - __shfl(pad, l, 64) + in * height;
        }
        end = __shfl(b, 63, 64);
        tiles_before = __shfl(tiles_to, 63, 64);
        pad_before = __shfl(pad_to, 63, 64);
    }
    t.total = tiles_before;
    t.group = __builtin_amdgcn_readfirstlane(t.group);
    t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
    t.rows = __builtin_amdgcn_readfirstlane(t.rows);
    t.pad0 = __builtin_amdgcn_readfirstlane(t.pad0);
    t.total = __builtin_amdgcn_readfirstlane(t.total);
    return t;
}

// the rows of one group, and where it lies in the padded order
struct GroupSpan { int row0, rows, pad0; };
__device__ __forceinline__ GroupSpan find_group(const int32_t* __restrict__ offsets, int E, int M, int group) {
    const int lane = threadIdx.x & 63;
    GroupSpan s{0, 0, 0};
    int end = 0, pad_before = 0;
    for (int e0 = 0; e0 <= group; e0 += 64) {
        const int e = e0 + lane;
        int b = e < E ? offsets[e + 1] : 0;
        b = b < end ? end : b > M ? M : b;
        b = wave_scan_max(b);
        int a = __shfl_up(b, 1, 64);
        if (lane == 0) a = end;
        const int pad = (b - a + 127) & ~127;
        const int pad_to = pad_before + wave_scan_add(pad);
        if (group < e0 + 64) {
            const int l = group - e0;
            s.row0 = __shfl(a, l, 64);
            s.rows = __shfl(b - a, l, 64);
            s.pad0 = __shfl(pad_to, l, 64) - __shfl(pad, l, 64);
        }
        end = __shfl(b, 63, 64);
        pad_before = __shfl(pad_to, 63, 64);
    }
    s.row0 = __builtin_amdgcn_readfirstlane(s.row0);
    s.rows = __builtin_amdgcn_readfirstlane(s.rows);
    s.pad0 = __builtin_amdgcn_readfirstlane(s.pad0);
    return s;
}

}  // namespace fp8k
