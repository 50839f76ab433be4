// Grouped linear layer of few rows per expert against quantized weights (decoding): out[r] = fp8(x[row_token[r]] s) wq[e]^T / (s sw[e]) for
// the rows r of expert e, the activations' quantization included.
//
// The persistent workgroups of gemm_fp8_few_stream.hip (which describes their rings, one eighth of K per wavefront, and the sum of
// the eight parts) over the weights of all experts that have rows.  A unit of work is 16 rows of an expert (or what it has) against 16 rows of its
// weight; units are numbered row tile by row tile, and every workgroup takes an equal run of them, so that the stream of the
// weights is spread evenly over the CUs whatever the groups' sizes are.  Where a run crosses into the next row tile, the fragments
// of A in registers are replaced.
//
// A is quantized in place of being read: each wavefront loads its eighth of the rows in the layout of its fragments, the
// eighths' maxima meet in LDS, scale and codes (those of fp8_quantize) are formed in registers.  The first time this happens behind
// the first requests of the weight stream, which take as long to arrive, instead of in a launch of its own.  A later row tile waits for
// its rows with the ring full: 1-2 us of the run.
//
// Bound: the weights' stream.  One token through two of eight experts 14336 x 4096 25.5 us (4.6 TB/s, start and end included), 64 tokens
// through six of 64 experts 1408 x 2048 34.5 us (5.3 TB/s); where it is not taken is measured at few_rows_pay.
#include "fp8_device.hpp"
#include "group_tiles.hpp"
#include "launchers.hpp"
#include "moe_launchers.hpp"
#include "tuning.hpp"

namespace fp8k {

namespace {

typedef int v8i_g __attribute__((ext_vector_type(8)));
typedef int v4i_g __attribute__((ext_vector_type(4)));
typedef float v4f_g __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_g __attribute__((ext_vector_type(2)));
typedef float f32x2_g __attribute__((ext_vector_type(2)));
constexpr int WAVES = 8;
constexpr int RING = 8;            // units (16 rows x 128 bytes) in flight per wavefront: what the LDS holds
constexpr int RUN = 32;            // most units of work of a workgroup (their scales sit in LDS)

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2_g v = {a, b};
    const bf16x2_g h = __builtin_convertvector(v, bf16x2_g);
    uint32_t r;
    __builtin_memcpy(&r, &h, 4);
    return r;
}
template <bool HINT>
__device__ __forceinline__ void dma16(v4i_g rsrc, uint32_t lds_addr, uint32_t voffset) {
    if constexpr (HINT)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                     :
                     : "s"(lds_addr), "v"(voffset), "s"(rsrc)
                     : "memory", "m0");
    else
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(lds_addr), "v"(voffset), "s"(rsrc)
                     : "memory", "m0");
}
template <int N_>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N_) : "memory"); }
__device__ __forceinline__ void barrier_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

struct FewArgs {
    const uint16_t* x; int64_t T;
    const int32_t *row_token, *offsets;
    const uint8_t* B; int64_t ldb;
    const float* scale_b;
    int E, M, N, K, flags, tiles_n;
    uint16_t* out; int64_t ld_out;
};
struct RowTile { int group, row0, rows, spare; };

// PER: most K steps of a wavefront
template <int FA, int FB, int PER, bool HINT>
__global__ __launch_bounds__(64 * WAVES) void grouped_few_kernel(FewArgs p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    v4f_g* const parts = reinterpret_cast<v4f_g*>(smem + WAVES * RING * 2048);      // [2][WAVES][64 lanes]
    float* const inv_sb = reinterpret_cast<float*>(parts + 2 * WAVES * 64);         // [RUN][16]
    uint32_t* const amax = reinterpret_cast<uint32_t*>(inv_sb + RUN * 16);          // [WAVES][16]
    RowTile* const tiles = reinterpret_cast<RowTile*>(amax + WAVES * 16);           // [RUN], the run's row tiles
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = lane & 15, g = lane >> 4;
    constexpr uint32_t OOB = 0x80000000u;

    // ---- this workgroup's run of units, and its row tiles
    const int total = find_group_tile<true>(p.offsets, p.E, p.M, 16, -1).total * p.tiles_n;
    const int share = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    const int u0 = (int)blockIdx.x * share, mine = total - u0 < share ? total - u0 : share;
    if (mine <= 0) return;
    const int r_first = u0 / p.tiles_n, n_tiles = (u0 + mine - 1) / p.tiles_n - r_first + 1;
    for (int r = wave; r < n_tiles; r += WAVES) {
        const GroupTile t = find_group_tile<true>(p.offsets, p.E, p.M, 16, r_first + r);
        if (lane == 0) tiles[r] = RowTile{t.group, t.row0, t.rows, 0};
    }
    __syncthreads();

    const int ksteps = (p.K + 127) >> 7, per = (ksteps + WAVES - 1) / WAVES;
    const int s_begin = wave * per;

    // ---- the weight's units.  Load h of a unit fetches rows 8 h + lane / 8; lane's chunk slot lane % 8 receives chunk slot ^ key(row)
    const int lrow = lane >> 3;
    const int c0 = (lane & 7) ^ ((lrow >> 1) & 7), c1 = (lane & 7) ^ ((4 + (lrow >> 1)) & 7);
    const uint32_t vb0 = (uint32_t)(lrow * (int)p.ldb + c0 * 16), vb1 = (uint32_t)((8 + lrow) * (int)p.ldb + c1 * 16);
    const uint32_t ring = (uint32_t)(size_t)smem + (uint32_t)wave * (RING * 2048u);
    const int k_begin = s_begin * 128, k_end = k_begin + per * 128;
    int next_k = k_begin, next_r = 0, next_n = u0 - r_first * p.tiles_n, left = mine;      // what is requested next
    v4i_g rsrc_b;
    auto point = [&] {
        const int e = __builtin_amdgcn_readfirstlane(tiles[next_r].group);
        const int rows = p.N - next_n * 16 < 16 ? p.N - next_n * 16 : 16;
        const uint64_t pb = reinterpret_cast<uint64_t>(p.B + ((int64_t)(e < p.E ? e : 0) * p.N + next_n * 16) * p.ldb);
        rsrc_b = v4i_g{(int)(uint32_t)pb, (int)(uint32_t)(pb >> 32), left > 0 && e < p.E ? (rows - 1) * (int)p.ldb + p.K : 0, 0x00020000};
    };
    auto issue = [&](uint32_t dst) {
        dma16<HINT>(rsrc_b, dst, next_k + c0 * 16 < p.K ? vb0 + (uint32_t)next_k : OOB);
        dma16<HINT>(rsrc_b, dst + 1024, next_k + c1 * 16 < p.K ? vb1 + (uint32_t)next_k : OOB);
        next_k += 128;
        if (next_k == k_end) {
            next_k = k_begin;
            left -= 1;
            if (++next_n == p.tiles_n) {
                next_n = 0;
                next_r = next_r + 1 < n_tiles ? next_r + 1 : next_r;
            }
            point();
        }
    };
    point();
#pragma unroll 1
    for (int u = 0; u < RING; ++u) issue(ring + u * 2048);

    // ---- reciprocals of the columns' scales, sixteen threads per unit of work
    {
        const int j = tid >> 4, u = u0 + j, r = u / p.tiles_n, n = (u - r * p.tiles_n) * 16 + (tid & 15);
        const int e = j < mine ? tiles[r - r_first].group : p.E;
        inv_sb[tid] = e < p.E && n < p.N ? 1.0f / p.scale_b[(int64_t)e * p.N + n] : 0.0f;
    }

    // ---- A: the rows of a row tile as fragments, chunks g and g + 4 of row i
    v8i_g af[PER];
    float inv_a = 0.f;
    auto take_rows = [&](int r) {
        const RowTile t = tiles[r];
        int64_t token = -1;
        if (t.group < p.E && i < t.rows) token = p.row_token ? p.row_token[t.row0 + i] : t.row0 + i;
        const bool there = token >= 0 && token < p.T;
        const uint16_t* row = p.x + (there ? token : 0) * p.K;
        int first_step = s_begin;      // (opaque: else the compares below are formed ahead of the units' loop and kept in scalar registers)
        asm volatile("" : "+s"(first_step));
        // piece h of step s: eight elements, or zeros where there are none (loaded from x's start all the same: no branches)
        auto piece = [&](int s, int h) {
            const int k = (first_step + s) * 128 + (h >> 1) * 64 + g * 16 + (h & 1) * 8;
            const bool real = there && s < per && k < p.K;
            const uint4 v = *reinterpret_cast<const uint4*>(real ? row + k : p.x);
            return make_uint4(real ? v.x : 0u, real ? v.y : 0u, real ? v.z : 0u, real ? v.w : 0u);
        };
        uint4 v[PER][4];
        uint32_t m = 0;
#pragma unroll
        for (int s = 0; s < PER; ++s)
#pragma unroll
            for (int h = 0; h < 4; ++h) v[s][h] = piece(s, h);
#pragma unroll
        for (int s = 0; s < PER; ++s)
#pragma unroll
            for (int h = 0; h < 4; ++h) m = pk_absmax4(m, v[s][h]);
        m = pk_absmax_xor<32>(pk_absmax_xor<16>(m));
        if (g == 0) amax[wave * 16 + i] = pk_fold(m);
        barrier_lds();
        uint32_t most = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = amax[w * 16 + i] > most ? amax[w * 16 + i] : most;
        const float s = scale_from_amax(mag_to_float(most), FA, p.flags);
        inv_a = t.group < p.E ? 1.0f / s : 0.0f;
#pragma unroll
        for (int st = 0; st < PER; ++st) {
            uint2 q[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) q[h] = cast8<FA>(v[st][h], s);
            af[st] = v8i_g{(int)q[0].x, (int)q[0].y, (int)q[1].x, (int)q[1].y, (int)q[2].x, (int)q[2].y, (int)q[3].x, (int)q[3].y};
        }
    };

    const int key = (i >> 1) & 7;
    const int f_lo = i * 128 + ((g ^ key) << 4), f_hi = i * 128 + (((g + 4) ^ key) << 4);
    const uint8_t* const ring_p = smem + wave * (RING * 2048);
    int slot = 0, r = 0, n = u0 - r_first * p.tiles_n;
    take_rows(0);
    for (int j = 0; j < mine; ++j) {
        v4f_g acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < PER; ++s) {
            if (s < per) {
                wait_loads<2 * (RING - 1)>();      // all but the younger units have landed
                const uint8_t* u = ring_p + slot * 2048;
                const uint4 lo = *reinterpret_cast<const uint4*>(u + f_lo), hi = *reinterpret_cast<const uint4*>(u + f_hi);
                const v8i_g bf = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bf, af[s], acc, FB, FA, 0, 0, 0, 0);
                issue(ring + (uint32_t)slot * 2048u);
                slot = slot + 1 == RING ? 0 : slot + 1;
            }
        }
        // ---- the parts of K: parked by every wavefront, summed by one (two sets: the next unit's are parked before it is done)
        v4f_g* const set = parts + (j & 1) * (WAVES * 64);
        set[wave * 64 + lane] = acc;
        barrier_lds();
        if (wave == (j & (WAVES - 1))) {
            const int row0 = tiles[r].row0, rows = tiles[r].rows;
            const int nb = n * 16 + 4 * g;
            const float4 ib = *reinterpret_cast<const float4*>(inv_sb + j * 16 + 4 * g);
            v4f_g sum = set[lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += set[w * 64 + lane];
            if (i < rows && nb < p.N)      // (columns are a multiple of eight)
                *reinterpret_cast<uint2*>(p.out + (int64_t)(row0 + i) * p.ld_out + nb) =
                    make_uint2(pack2((sum[0] * inv_a) * ib.x, (sum[1] * inv_a) * ib.y), pack2((sum[2] * inv_a) * ib.z, (sum[3] * inv_a) * ib.w));
        }
        if (++n == p.tiles_n) {
            n = 0;
            ++r;
            if (j + 1 < mine) take_rows(r);
        }
    }
    wait_loads<0>();       // trailing (out-of-range) refills must land before the LDS is handed back
}

template <int FA, int FB, int PER>
hipError_t launch_t(const FewArgs& a, int64_t grid, hipStream_t st) {
    constexpr int lds = WAVES * RING * 2048 + 2 * WAVES * 1024 + RUN * 16 * 4 + WAVES * 16 * 4 + RUN * (int)sizeof(RowTile);
    static_assert(lds <= 160 * 1024, "LDS");
    auto launch = [&](auto kern, DynamicLdsOnce& attr) {
        if (hipError_t e = attr.ensure(reinterpret_cast<const void*>(kern), lds); e != hipSuccess) return e;
        kern<<<dim3((unsigned)grid), dim3(64 * WAVES), lds, st>>>(a);
        return hipGetLastError();
    };
    static DynamicLdsOnce attr[2];
    if (stream_weight(a.B, a.ldb, (int64_t)a.E * a.N, a.K)) return launch(grouped_few_kernel<FA, FB, PER, true>, attr[1]);
    return launch(grouped_few_kernel<FA, FB, PER, false>, attr[0]);
}

}  // namespace

// Where this form is taken, against quantization and tiles in two launches (us, those / this; K shared evenly by the eight wavefronts,
// and no longer than 4096: longer rows would be read a second time for the cast, 4096 x 7168 with 2 rows 16.8 / 22.3):
//  * few units of work, where the second launch counts: one token of 8 experts 2048 x 2048, two of them, 11.9 / 9.3; of 128 experts 768 x
//    2048, eight, 11.1 / 9.7; 4096 x 4096, two of 8, 13.6 / 13.7; beyond: 2048 x 4096, six of 64, 14.3 / 20.4;
//  * weights enough that the stream decides, and rows few enough that the runs seldom cross: 14336 x 4096, two of 8 experts, 1, 4, 16
//    tokens 31.0 67.4 89.5 / 25.9 52.0 96.4; 4096 x 4096, two of 16, 8 tokens 45.0 / 35.1; 1408 x 2048, six of 64, 5, 16, 64, 128 tokens
//    17.2 24.6 37.3 40.7 / 17.8 23.2 35.4 64.0; 768 x 2048, eight of 128, 64 tokens 35.5 / 33.4.
static bool few_rows_pay(const GroupedGemm& g, int64_t cus) {
    const double busy = (double)(g.E < g.M ? g.E : g.M);
    if ((g.K + 127) / 128 % WAVES != 0) return false;
    if (g.M * ((g.N + 15) / 16) <= 2 * cus) return true;
    return g.M <= 6 * g.E && busy * (double)g.N * (double)g.K >= 64e6 && (g.M <= g.E || g.N * g.K <= (int64_t)16 << 20);
}

// hipErrorNotSupported (nothing launched): more rows, or a longer contraction, than it is for
hipError_t launch_grouped_few(const void* x, int64_t T, const int32_t* row_token, int fmt_x, int flags, const GroupedGemm& g, hipStream_t st) {
    const int forced = knob(KNOB_SKINNY_DMA);      // 0: never, 2: wherever it fits
    const int64_t cus = compute_units() > 0 ? compute_units() : 256;
    if (forced == 0 || g.K > 4096 || T < 1 || (forced < 2 && !few_rows_pay(g, cus))) return hipErrorNotSupported;
    const int64_t tiles_n = (g.N + 15) / 16, most = (g.M / 16 + (g.E + 1 < g.M ? g.E + 1 : g.M)) * tiles_n;
    if (most > 0x3FFFFFFF) return hipErrorNotSupported;
    int64_t grid = most < cus ? most : cus;
    if (grid * RUN < most) grid = (most + RUN - 1) / RUN;
    const FewArgs a{static_cast<const uint16_t*>(x), T, row_token, g.offsets, g.b, g.ldb, g.scale_b, (int)g.E, (int)g.M, (int)g.N, (int)g.K, flags,
                    (int)tiles_n, static_cast<uint16_t*>(g.out), g.ld_out};
    const int per = (int)(((g.K + 127) / 128 + WAVES - 1) / WAVES);
#define FP8K_FEW(FA_, FB_)                                                     \
    if (fmt_x == FA_ && g.fmt_b == FB_) {                                      \
        if (per <= 2) return launch_t<FA_, FB_, 2>(a, grid, st);               \
        return launch_t<FA_, FB_, 4>(a, grid, st);                             \
    }
    FP8K_FEW(FMT_E4M3FN, FMT_E4M3FN)
    FP8K_FEW(FMT_E5M2, FMT_E4M3FN)
    FP8K_FEW(FMT_E4M3FN, FMT_E5M2)
    FP8K_FEW(FMT_E5M2, FMT_E5M2)
#undef FP8K_FEW
    return hipErrorInvalidValue;
}

}  // namespace fp8k
