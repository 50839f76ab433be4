// Quantization of the operands of products grouped by expert.
//
//   rows      codes and scales of x[row_token[r]], one scale per row: the rows of a token that several experts got are quantized
//             once per expert, which costs M K bytes of code but leaves the product's operand in group order.
//   columns   of each group: q[c, r] = fp8(x[r, c] s[e, c]), s from the largest |x[r, c]| over the group's rows, written
//             transposed, so that the weight gradient contracts over a contiguous axis.  Two passes: maxima of (group, strip of
//             columns, part of the rows) folded with an integer maximum (whose order does not matter), then the cast, in tiles
//             of 128 rows x 128 columns that turn through LDS.
// Scales, rounding and saturation are those of fp8_quantize.  All of it is bound by HBM.
#include "fp8_device.hpp"
#include "group_tiles.hpp"
#include "moe_launchers.hpp"

namespace fp8k {

namespace {

// ---- rows -----------------------------------------------------------------------------------------------------------

// one workgroup per row, the row in registers (NV pieces of eight per thread); NV == 0: any length, read twice
template <int FMT, int NTH, int NV>
__global__ __launch_bounds__(NTH) void rows_gather_kernel(const uint16_t* __restrict__ x, int64_t T, int64_t ldx,
                                                          const int32_t* __restrict__ row_token, int cols, int flags, uint8_t* __restrict__ q,
                                                          int64_t ld_q, float* __restrict__ scale) {
    __shared__ uint32_t part[NTH / 64];
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x;
    const int64_t t = row_token ? row_token[r] : r;
    const bool there = t >= 0 && t < T;
    const uint16_t* row = x + (there ? t : 0) * ldx;
    uint8_t* out = q + r * ld_q;
    constexpr int NR = NV > 0 ? NV : 1;
    uint4 v[NR];
    uint32_t m = 0;
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * NTH + tid) * 8;
            v[i] = there && c < cols ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) m = pk_absmax4(m, v[i]);
    } else if (there) {
        for (int c = tid * 8; c < cols; c += NTH * 8) m = pk_absmax4(m, *reinterpret_cast<const uint4*>(row + c));
    }
    m = wave_max_u32<64>(pk_fold(m));
    if constexpr (NTH > 64) {
        if ((tid & 63) == 0) part[tid >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NTH / 64; ++w) m = part[w] > m ? part[w] : m;
    }
    const float s = scale_from_amax(mag_to_float(m), FMT, flags);
    if (tid == 0) scale[r] = s;
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * NTH + tid) * 8;
            if (c < cols) store_vec(out + c, cast8<FMT>(v[i], s));
        }
    } else {
        for (int c = tid * 8; c < cols; c += NTH * 8)
            store_vec(out + c, cast8<FMT>(there ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0), s));
    }
}

template <int FMT>
hipError_t rows_gather(const uint16_t* x, int64_t T, int64_t ldx, const int32_t* row_token, int64_t M, int cols, int flags, uint8_t* q,
                       int64_t ld_q, float* scale, hipStream_t st) {
#define FP8K_ROWS(NTH_, NV_) rows_gather_kernel<FMT, NTH_, NV_><<<(unsigned)M, NTH_, 0, st>>>(x, T, ldx, row_token, cols, flags, q, ld_q, scale)
    if (cols <= 512) FP8K_ROWS(64, 1);
    else if (cols <= 1024) FP8K_ROWS(64, 2);
    else if (cols <= 2048) FP8K_ROWS(256, 1);
    else if (cols <= 4096) FP8K_ROWS(256, 2);
    else if (cols <= 8192) FP8K_ROWS(256, 4);
    else if (cols <= 16384) FP8K_ROWS(256, 8);
    else FP8K_ROWS(256, 0);
#undef FP8K_ROWS
    return hipGetLastError();
}

// ---- columns --------------------------------------------------------------------------------------------------------

struct ColArgs {
    const uint16_t* x;
    int64_t T, ldx;
    const int32_t *row_token, *offsets;      // offsets nullptr: groups of M / E rows
    int M, E, cols, flags;
    uint8_t* qt;
    int64_t ld_t, group_stride;
    float* scale;
    uint32_t* amax;
};

__device__ __forceinline__ GroupTile tile_of(const ColArgs& a, int height, int index) {
    if (a.offsets) return find_group_tile<false>(a.offsets, a.E, a.M, height, index);
    const int n = a.M / a.E, per = (n + height - 1) / height, e = index / per, in = index - e * per;
    return GroupTile{e < a.E ? e : -1, e * n + in * height, n - in * height < height ? n - in * height : height, in * height, per * a.E, in == 0};
}

// the row of x behind row r, or nullptr
__device__ __forceinline__ const uint16_t* row_of(const ColArgs& a, int r) {
    const int64_t t = a.row_token ? a.row_token[r] : r;
    return t >= 0 && t < a.T ? a.x + t * a.ldx : nullptr;
}

// Maxima: a workgroup takes 512 columns (a lane eight) of up to HEIGHT rows of a group, a wavefront every fourth row.
constexpr int AMAX_ROWS = 128;
__global__ __launch_bounds__(256) void cols_amax_kernel(ColArgs a) {
    __shared__ uint4 part[4][64];
    const GroupTile t = tile_of(a, AMAX_ROWS, blockIdx.x);
    if (t.group < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (int)blockIdx.y * 512 + lane * 8;
    uint4 m = make_uint4(0, 0, 0, 0);
    if (c < a.cols) {
        for (int r0 = wave; r0 < t.rows; r0 += 32) {
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint16_t* row = r0 + 4 * i < t.rows ? row_of(a, t.row0 + r0 + 4 * i) : nullptr;
                v[i] = row ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m.x = pk_absmax(m.x, v[i].x); m.y = pk_absmax(m.y, v[i].y);
                m.z = pk_absmax(m.z, v[i].z); m.w = pk_absmax(m.w, v[i].w);
            }
        }
    }
    part[wave][lane] = m;
    __syncthreads();
    // two columns a thread: dword d of lane l's eight columns
    const int l = threadIdx.x >> 2, d = threadIdx.x & 3;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w = pk_absmax(w, reinterpret_cast<const uint32_t*>(&part[i][l])[d]);
    const int col = (int)blockIdx.y * 512 + l * 8 + d * 2;
    if (col < a.cols) {
        uint32_t* to = a.amax + (int64_t)t.group * a.cols + col;
        atomicMax(to, w & 0xFFFFu);
        if (col + 1 < a.cols) atomicMax(to + 1, w >> 16);
    }
}

// Cast: 128 rows x 128 columns.  Thread (p, l) = (tid / 16, tid % 16) holds rows 4 p .. 4 p + 3 and 64 + those, eight columns from
// 8 l on; four rows turn into a dword of codes per column.  In LDS a column is 128 bytes, its sixteen-byte pieces exchanged by
// (column / 8) % 8, so that the sixteen lanes that write the same rows of sixteen columns eight apart meet in two of them at most.
template <int FMT>
__global__ __launch_bounds__(256) void cols_cast_kernel(ColArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
    const GroupTile t = tile_of(a, 128, blockIdx.x);
    if (t.group < 0) return;
    const int tid = threadIdx.x, p = tid >> 4, l = tid & 15;
    const int c = (int)blockIdx.y * 128 + l * 8;
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * p + (i & 3) + 64 * (i >> 2);
        const uint16_t* row = c < a.cols && r < t.rows ? row_of(a, t.row0 + r) : nullptr;
        v[i] = row ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0);
    }
    float s[8];
    if (c < a.cols) {
        const int64_t at = (int64_t)t.group * a.cols + c;
        const uint4 m0 = *reinterpret_cast<const uint4*>(a.amax + at), m1 = *reinterpret_cast<const uint4*>(a.amax + at + 4);
        const uint32_t m[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = scale_from_amax(mag_to_float(m[e]), FMT, a.flags);
        // (the group's first tile of rows leaves them for the product)
        if (t.first && p == 0) {
#pragma unroll
            for (int e = 0; e < 8; e += 4) *reinterpret_cast<float4*>(a.scale + at + e) = make_float4(s[e], s[e + 1], s[e + 2], s[e + 3]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = cast8<FMT>(v[4 * h + i], s);
        uint32_t o[8];
        {
            uint32_t lo[4], hi[4];
            transpose4x4_bytes(q[0].x, q[1].x, q[2].x, q[3].x, lo);
            transpose4x4_bytes(q[0].y, q[1].y, q[2].y, q[3].y, hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) { o[e] = lo[e]; o[4 + e] = hi[e]; }
        }
        const int d = p + 16 * h;      // dword of the column: rows 4 d .. 4 d + 3
#pragma unroll
        for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint32_t*>(turned + (l * 8 + e) * 128 + ((((d >> 2) ^ (l & 7)) << 4) | ((d & 3) << 2))) = o[e];
    }
    __syncthreads();
    // out: eight lanes write the 128 bytes of a column; sixteen-byte pieces past the group's rows, rounded up to sixteen, are left out
    const int rows16 = (t.rows + 15) & ~15;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = i * 32 + (tid >> 3), piece = tid & 7;
        const uint4 w = *reinterpret_cast<const uint4*>(turned + col * 128 + ((piece ^ ((col >> 3) & 7)) << 4));
        if ((int)blockIdx.y * 128 + col < a.cols && piece * 16 < rows16)
            store_vec(a.qt + t.group * a.group_stride + (int64_t)((int)blockIdx.y * 128 + col) * a.ld_t + t.pad0 + piece * 16, w);
    }
}

// scales of groups without rows, whose products are zero whatever they are: a finite one
__global__ __launch_bounds__(256) void clear_kernel(uint32_t* __restrict__ amax, float* __restrict__ scale, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) {
        amax[i] = 0u;
        scale[i] = 1.0f;
    }
}

}  // namespace

hipError_t launch_quant_rows_gather(const void* x, int64_t T, int64_t ldx, const int32_t* row_token, int64_t M, int64_t cols, int fmt, int flags,
                                    uint8_t* q, int64_t ld_q, float* scale, hipStream_t st) {
    if (M <= 0) return hipSuccess;
    auto* xs = static_cast<const uint16_t*>(x);
    return fmt == FMT_E4M3FN ? rows_gather<FMT_E4M3FN>(xs, T, ldx, row_token, M, (int)cols, flags, q, ld_q, scale, st)
                             : rows_gather<FMT_E5M2>(xs, T, ldx, row_token, M, (int)cols, flags, q, ld_q, scale, st);
}

hipError_t launch_quant_cols_grouped(const GroupedColOperand& op, const int32_t* offsets, int64_t E, int flags, hipStream_t st) {
    const ColArgs a{static_cast<const uint16_t*>(op.x), op.T, op.ldx, op.row_token, offsets, (int)op.M, (int)E, (int)op.cols, flags,
                    op.qt, op.ld_t, offsets ? 0 : op.cols * op.ld_t, op.scale, op.amax};
    const int64_t n = E * op.cols;
    clear_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(op.amax, op.scale, n);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (op.M <= 0) return hipSuccess;
    // tiles of 128 rows: what the groups can come to at most
    const int64_t per = op.M / E, tiles = offsets ? op.M / 128 + (E < op.M ? E : op.M) : E * ((per + 127) / 128);
    cols_amax_kernel<<<dim3((unsigned)tiles, (unsigned)((op.cols + 511) / 512)), 256, 0, st>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid((unsigned)tiles, (unsigned)((op.cols + 127) / 128));
    if (op.fmt == FMT_E4M3FN) cols_cast_kernel<FMT_E4M3FN><<<grid, 256, 0, st>>>(a);
    else cols_cast_kernel<FMT_E5M2><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace fp8k
