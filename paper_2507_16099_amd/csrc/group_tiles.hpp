// Where the rows of a group lie, for kernels over rows ordered by group with offsets that only the device knows.
//
// The groups are [offsets[e], offsets[e + 1]), e < E, with offsets[0] = 0.  Offsets that a caller got wrong must not lead out of
// bounds: a group ends at the running maximum of the offsets, cut to [0, M], and starts where the one before it ended (the first at
// 0), so groups never overlap and their lengths never sum to more than M.  What is left behind the last one counts as group E.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fp8k {

// Inclusive scans over the 64 lanes in registers: shifts by 1, 2, 4, 8 within the rows of 16, then the last lane of a row to the next
// row and that of the first half to the second.
template <class F>
__device__ __forceinline__ int wave_scan(int v, int none, F f) {
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xF, 0xF, false));      // row_shr:1, 2, 4, 8
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xA, 0xF, false));      // row_bcast:15 into rows 1 and 3
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xC, 0xF, false));      // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ int wave_scan_add(int v) {
    return wave_scan(v, 0, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int wave_scan_max(int v) {      // of numbers that are not negative
    return wave_scan(v, 0, [](int a, int b) { return a > b ? a : b; });
}
// the lane before, lane 0 gets `first`
__device__ __forceinline__ int wave_before(int v, int first) { return __builtin_amdgcn_update_dpp(first, v, 0x138, 0xF, 0xF, false); }      // wave_shr:1

// the value of one lane, the same lane for all
__device__ __forceinline__ int at_lane(int v, int l) { return __builtin_amdgcn_readlane(v, __builtin_amdgcn_readfirstlane(l)); }

// offsets[e + 1] of 64 groups at a time, requested four sixty-fours ahead (one behind the other, 256 groups are four trips to memory)
struct OffsetChunks {
    const int32_t* offsets;
    int E, v[4];
    __device__ __forceinline__ int at(int e) const { return offsets[(e < E ? e : E - 1) + 1]; }
    __device__ __forceinline__ OffsetChunks(const int32_t* o, int E_) : offsets(o), E(E_) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i * 64 < E ? at(i * 64 + (int)(threadIdx.x & 63)) : 0;
    }
    // of the groups from e0 on; called for e0 = 0, 64, 128, ...
    __device__ __forceinline__ int get(int e0) {
        const int r = v[0];
        v[0] = v[1]; v[1] = v[2]; v[2] = v[3];
        if (e0 + 256 < E) v[3] = at(e0 + 256 + (int)(threadIdx.x & 63));
        return r;
    }
};

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
    OffsetChunks chunks(offsets, E);
    for (int e0 = 0; e0 < E + (TAIL ? 1 : 0); e0 += 64) {
        const int e = e0 + lane;
        int b = chunks.get(e0);
        if (e >= E) b = TAIL && e == E ? M : 0;
        b = b < end ? end : b > M ? M : b;
        b = wave_scan_max(b);
        const int a = wave_before(b, end);
        const int n = b - a, tiles = (n + height - 1) / height, pad = (n + 127) & ~127;
        const int tiles_to = tiles_before + wave_scan_add(tiles), pad_to = pad_before + wave_scan_add(pad);
        const uint64_t hit = __ballot(index >= 0 && index < tiles_to);
        if (t.group < 0 && hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            const int in = index - (at_lane(tiles_to, l) - at_lane(tiles, l));
            const int a_l = at_lane(a, l), n_l = at_lane(n, l);
            t.group = e0 + l;
            t.row0 = a_l + in * height;
            t.first = in == 0;
            t.rows = n_l - in * height < height ? n_l - in * height : height;
            t.pad0 = at_lane(pad_to, l) - at_lane(pad, l) + in * height;
        }
        end = at_lane(b, 63);
        tiles_before = at_lane(tiles_to, 63);
        pad_before = at_lane(pad_to, 63);
    }
    t.total = tiles_before;
    t.group = __builtin_amdgcn_readfirstlane(t.group);
    t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
    t.rows = __builtin_amdgcn_readfirstlane(t.rows);
    t.pad0 = __builtin_amdgcn_readfirstlane(t.pad0);
    t.total = __builtin_amdgcn_readfirstlane(t.total);
    return t;
}

// A persistent workgroup's share of `units` tiles: whole rounds, in which each of the eight XCDs takes a run of `slots` neighbouring ones,
// and its part of the last round, which is spread over the XCDs too, for each has its own way to memory (four experts 4096 x 14336 with
// 30, 2, 0 and 70 rows 67 us with the last round's tiles on the first XCDs, 45 so; 400 tokens, two of eight, 133 and 130; more rounds alike).
struct TileShare {
    int first, last, full, mine, step;
    __device__ __forceinline__ TileShare(int units) {
        const int slots = (int)gridDim.x / 8, xcd = (int)blockIdx.x % 8, slot = (int)blockIdx.x / 8;
        step = 8 * slots;
        full = units / step;
        const int rest = units - full * step, per = (rest + 7) / 8, at = xcd * per + slot;
        first = xcd * slots + slot;
        last = full * step + at;
        mine = full + (slot < per && at < rest ? 1 : 0);
    }
    // the j-th tile of it
    __device__ __forceinline__ int operator[](int j) const { return j < full ? first + j * step : last; }
};

// the rows of one group, where it lies in the padded order, and how many tiles of `height` rows the groups before it have
struct GroupSpan { int row0, rows, pad0, tile0; };
__device__ __forceinline__ GroupSpan find_group(const int32_t* __restrict__ offsets, int E, int M, int group, int height) {
    const int lane = threadIdx.x & 63;
    GroupSpan s{0, 0, 0, 0};
    int end = 0, pad_before = 0, tiles_before = 0;
    OffsetChunks chunks(offsets, E);
    for (int e0 = 0; e0 <= group; e0 += 64) {
        const int e = e0 + lane;
        int b = chunks.get(e0);
        if (e >= E) b = 0;
        b = b < end ? end : b > M ? M : b;
        b = wave_scan_max(b);
        const int a = wave_before(b, end);
        const int pad = (b - a + 127) & ~127, tiles = (b - a + height - 1) / height;
        const int pad_to = pad_before + wave_scan_add(pad), tiles_to = tiles_before + wave_scan_add(tiles);
        if (group < e0 + 64) {
            const int l = group - e0;
            s.row0 = at_lane(a, l);
            s.rows = at_lane(b - a, l);
            s.pad0 = at_lane(pad_to, l) - at_lane(pad, l);
            s.tile0 = at_lane(tiles_to, l) - at_lane(tiles, l);
        }
        end = at_lane(b, 63);
        pad_before = at_lane(pad_to, 63);
        tiles_before = at_lane(tiles_to, 63);
    }
    return s;
}

// The groups' table of a workgroup that walks many tiles, by one wavefront: starts[e] the first row of group e, tiles_to[e] the tiles of
// `height` rows of the groups before it, pads[e] its place when groups are padded to 128; group E is what lies behind the last one,
// and entry E + 1 the end.
__device__ __forceinline__ void list_groups(const int32_t* __restrict__ offsets, int E, int M, int height, int* starts, int* tiles_to, int* pads) {
    const int lane = threadIdx.x & 63;
    int end = 0, tiles_before = 0, pad_before = 0;
    OffsetChunks chunks(offsets, E);
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int e = e0 + lane;
        int b = chunks.get(e0);
        if (e >= E) b = e == E ? M : 0;
        b = b < end ? end : b > M ? M : b;
        b = wave_scan_max(b);
        const int a = wave_before(b, end);
        const int tiles = (b - a + height - 1) / height, pad = (b - a + 127) & ~127;
        const int tiles_sum = tiles_before + wave_scan_add(tiles), pad_sum = pad_before + wave_scan_add(pad);
        if (e <= E) {
            starts[e] = a;
            tiles_to[e] = tiles_sum - tiles;
            pads[e] = pad_sum - pad;
        }
        if (e == E) {
            starts[e + 1] = b;
            tiles_to[e + 1] = tiles_sum;
        }
        end = at_lane(b, 63);
        tiles_before = at_lane(tiles_sum, 63);
        pad_before = at_lane(pad_sum, 63);
    }
}
// the group of row tile tm, by a whole wavefront: as many groups end at or before it
__device__ __forceinline__ int group_of_tile(const int* tiles_to, int E, int tm) {
    int e = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int l = e0 + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (no register kept for the lane)
        e += __popcll(__ballot(l <= E && tiles_to[l <= E ? l + 1 : 0] <= tm));
    }
    return __builtin_amdgcn_readfirstlane(e);
}

}  // namespace fp8k
