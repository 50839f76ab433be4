// Scaled FP8 products grouped by expert (gfx950), groups of any size that only the device knows:
//   rows      out[r] = A[r] B[e]^T / (sa[r] sb[e])        for the rows r of group e; one weight B[e] [N, K] per group
//   contract  out[e] = A_e B_e^T / (sa[e] sb[e])          A_e [N, n_e], B_e [K, n_e]: the columns of the group in A [N, lda], B [K, ldb]
// The K step is that of gemm_fp8_ring.hpp: a ring of R stages filled by LDS-DMA ahead of the matrix cores, one workgroup barrier a step,
// fragments of the next step read behind the matrix instructions of the present one; LDS layout, swizzle keys and operand
// order are described there.
//
// What is different: a workgroup walks many tiles and its ring never drains.  The refills run R steps ahead of the matrix instructions
// through the sequence of all steps of all its tiles, so that a tile's first operands arrive while the tile before it is computed; an
// expert's product is 4 to 32 steps long, and filling the ring for each tile again cost 3 to 5 us, as much as eight steps.
// Scales and the tile's place come a tile ahead in the same way, into one of R + 2 tables.  The epilogue goes from registers to memory:
// the lanes of a row exchange halves until each store instruction writes 64 bytes of it.  Measured: dX of 9186 rows in 64 groups, 1408 x
// 2048, 80 us with one tile a workgroup, 66 so.
// Bound: per step the matrix instructions and LDS reads of a tile (kForms has the times), with few rows a group the weights' stream.
//
// Which tiles: the host knows M rows and E groups; the workgroup reads the offsets and leaves in LDS where each group's rows start and how
// many tiles lie before it.  Tiles go round the workgroups in patches of GROUP_M row tiles, eight XCDs side by side (see
// gemm_fp8_grouped_stream.hip).  Rows behind the last group (slots that no expert took) are written as zeros: a tile without codes.
#include "gemm_fp8_ring.hpp"
#include "group_tiles.hpp"
#include "moe_launchers.hpp"

#include <algorithm>
#include <cmath>

namespace fp8k {

namespace {

struct GroupedArgs {
    const uint8_t* A; int64_t lda; const uint8_t* B; int64_t ldb;
    const float *scale_a, *scale_b;
    const int32_t* offsets;
    int E, M, N, K;              // rows: out is [M, N], contracting K.  contract: out is [E][N][K], contracting the group's rows
    uint16_t* out; int64_t ld_out;
    int tiles_n, tiles_m;        // tiles_m: of one group's output (contract)
};
typedef unsigned v2u_gr __attribute__((ext_vector_type(2)));

template <int FA, int FB, int TM, int TN, int WAVES_M, int WAVES_N, int R, int GROUP_M, bool CONTRACT>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void gemm_fp8_grouped_kernel(GroupedArgs p) {
    using namespace rg;
    constexpr int NW = WAVES_M * WAVES_N;
    constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N;
    constexpr int FM = WM / 16, FN = WN / 16;
    constexpr int GW = WN % 64 == 0 ? 64 : 32;
    constexpr int GT = GW / 16, NG = WN / GW;
    constexpr int SH = GW == 64 ? 4 : 3;
    constexpr int STAGE = (TM + TN) * BK;
    constexpr int UA = (TM + 63) / 64, TMS = 64 * UA, NU = UA + TN / 64;
    constexpr int NLA = TM / (8 * NW), NLB = TN / (8 * NW), NL = NLA + NLB;
    constexpr int NM = FM * FN;
    constexpr bool ACC_V = 4 * NM + 16 * (FM + FN) <= 176;
    constexpr int NTAB = R + 2, TAB = NU * 64;       // tables of scales: a tile's and those of the R + 1 tiles that may be entered before it is done
    static_assert(NW == 4 && WM % 16 == 0 && (GW == 64 || GW == 32) && WN % GW == 0 && TM % (8 * NW) == 0 && TN % 64 == 0, "tile");
    static_assert(R >= 3 && (R - 1) * NL <= 63 && TM <= 256 && TN <= 256, "vmcnt range, a scale per thread");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    float* const tabs = reinterpret_cast<float*>(smem + R * STAGE);
    int4* const places = reinterpret_cast<int4*>(tabs + NTAB * TAB);      // of those tiles: first row, rows, first column, contracted codes
    int* const starts = reinterpret_cast<int*>(places + NTAB);            // [E + 2] each
    int *const tiles_to = starts + p.E + 2, *const pads = tiles_to + p.E + 2;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = (wave / WAVES_N) * WM, wn0 = (wave % WAVES_N) * WN;
    if (wave == 0) list_groups(p.offsets, p.E, p.M, TM, starts, tiles_to, pads);
    __syncthreads();

    // ---- this workgroup's tiles
    const int tiles_n = p.tiles_n, per_group = p.tiles_m * tiles_n;
    const int row_tiles = CONTRACT ? p.tiles_m * p.E : __builtin_amdgcn_readfirstlane(tiles_to[p.E + 1]);
    const int units = row_tiles * tiles_n;
    const TileShare share(units);
    if (share.mine == 0) return;
    const int cols_all = CONTRACT ? p.K : p.N;
    const int64_t lda = p.lda, ldb = p.ldb;

    // ---- the tile whose operands are requested next: its panels, contracted codes, the step's first code
    v4i_t rsrc_a, rsrc_b;
    int k_tile = 0, k_next = 0, j_next = 0, tab_next = 0;
    auto enter_tile = [&] {
        int row = 0, rows = 1, n0 = 0, brow = 0;
        uint64_t pa = reinterpret_cast<uint64_t>(p.A), pb = reinterpret_cast<uint64_t>(p.B);
        const bool real = j_next < share.mine;
        k_tile = 0;
        k_next = 0;
        if (real) {
            const int u = share[j_next], e_c = CONTRACT ? u / per_group : 0;
            const int rest = u - e_c * per_group, in_group = GROUP_M * tiles_n, most_m = CONTRACT ? p.tiles_m : row_tiles;
            const int first_m = rest / in_group * GROUP_M, in = rest % in_group;
            const int gsize = most_m - first_m < GROUP_M ? most_m - first_m : GROUP_M;
            const int tm = first_m + in % gsize;
            n0 = in / gsize * TN;
            if constexpr (CONTRACT) {
                const int start = __builtin_amdgcn_readfirstlane(starts[e_c]), pad0 = __builtin_amdgcn_readfirstlane(pads[e_c]);
                k_tile = (__builtin_amdgcn_readfirstlane(starts[e_c + 1]) - start + 15) & ~15;
                const int m0 = tm * TM;
                row = e_c * p.N + m0;
                rows = p.N - m0 < TM ? p.N - m0 : TM;
                brow = e_c * p.K + n0;
                pa = reinterpret_cast<uint64_t>(p.A + (int64_t)m0 * lda + pad0);
                pb = reinterpret_cast<uint64_t>(p.B + (int64_t)n0 * ldb + pad0);
            } else {
                const int e = group_of_tile(tiles_to, p.E, tm);
                row = __builtin_amdgcn_readfirstlane(starts[e]) + (tm - __builtin_amdgcn_readfirstlane(tiles_to[e])) * TM;
                rows = __builtin_amdgcn_readfirstlane(starts[e + 1]) - row;
                if (rows > TM) rows = TM;
                k_tile = e < p.E ? p.K : 0;
                brow = (e < p.E ? e : p.E - 1) * p.N + n0;
                pa = reinterpret_cast<uint64_t>(p.A + (int64_t)row * lda);
                pb = reinterpret_cast<uint64_t>(p.B + (int64_t)brow * ldb);
            }
        }
        const int cols = cols_all - n0 < TN ? cols_all - n0 : TN;
        rsrc_a = v4i_t{(int)(uint32_t)pa, (int)(uint32_t)(pa >> 32), (int)((int64_t)(rows - 1) * lda + k_tile), 0x00020000};
        rsrc_b = v4i_t{(int)(uint32_t)pb, (int)(uint32_t)(pb >> 32), (int)((int64_t)(cols - 1) * ldb + k_tile), 0x00020000};
        if (real) {
            const uint64_t psa = reinterpret_cast<uint64_t>(p.scale_a + row), psb = reinterpret_cast<uint64_t>(p.scale_b + brow);
            const v4i_t rsrc_sa = {(int)(uint32_t)psa, (int)(uint32_t)(psa >> 32), rows * 4, 0x00020000};
            const v4i_t rsrc_sb = {(int)(uint32_t)psb, (int)(uint32_t)(psb >> 32), cols * 4, 0x00020000};
#pragma unroll
            for (int h = 0; h < (NU + NW - 1) / NW; ++h) {
                const int u = wave + NW * h, r = 64 * (u < UA ? u : u - UA) + lane;
                const uint32_t at = (uint32_t)(size_t)(tabs + tab_next * TAB) + (uint32_t)u * 256u;
                if (u < UA) lds_dma4(rsrc_sa, at, (uint32_t)(r < rows ? r : rows - 1) * 4u);
                else if (u < NU) lds_dma4(rsrc_sb, at, (uint32_t)(r < cols ? r : cols - 1) * 4u);
            }
        }
        if (tid == 0) places[tab_next] = make_int4(row, rows, n0, k_tile);
        ++j_next;
        tab_next = tab_next + 1 == NTAB ? 0 : tab_next + 1;
    };
    auto advance = [&] {      // to the next step of the sequence (a tile without codes has one, of zeros)
        k_next += BK;
        if (k_next >= k_tile) enter_tile();
    };

    const int lrow = lane >> 3;
    const int ca = (lane & 7) ^ ((4 * (wave & 1) + (lrow >> 1)) & 7);
    const int kb_e = SH == 4 ? (wave >> 1) : wave, kb_o = SH == 4 ? 2 + (wave >> 1) : kb_e;
    const int cb_e = (lane & 7) ^ (((lrow >> 1) & 1) | ((kb_e & 3) << 1));
    const int cb_o = (lane & 7) ^ (((lrow >> 1) & 1) | ((kb_o & 3) << 1));
    const uint32_t va0 = (uint32_t)((wave * 8 + lrow) * (int)lda + ca * 16);
    const uint32_t vb0_e = (uint32_t)((wave * 8 + lrow) * (int)ldb + cb_e * 16);
    const uint32_t vb0_o = (uint32_t)((wave * 8 + lrow) * (int)ldb + cb_o * 16);
    const uint32_t va_step = (uint32_t)(8 * NW * (int)lda), vb_step = (uint32_t)(8 * NW * (int)ldb);
    const uint32_t lds_base = (uint32_t)(size_t)smem + (uint32_t)wave * 1024u;
    constexpr uint32_t OOB = 0x80000000u;
    auto load_q = [&](int q, uint32_t stage_off, uint32_t ka, uint32_t ke, uint32_t ko) {
        if (q < NLB) lds_dma16<>(rsrc_b, lds_base + stage_off + TM * BK + q * (NW * 1024), ((q & 1) ? vb0_o + ko : vb0_e + ke) + (uint32_t)q * vb_step);
        else if (q < NL) lds_dma16<>(rsrc_a, lds_base + stage_off + (q - NLB) * (NW * 1024), va0 + (uint32_t)(q - NLB) * va_step + ka);
    };
    auto kofs = [&](int c) { return k_next + c * 16 < k_tile ? (uint32_t)k_next : OOB; };

    const int r16 = lane & 15, g = lane >> 4;
    const int key_a = (r16 >> 1) & 7;
    const int key_b = ((r16 >> 1) & 1) | ((r16 >> 2) << 1);
    int offa[2], offb[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        offa[c] = (wm0 + r16) * BK + (((g + 4 * c) ^ key_a) << 4);
        offb[c] = TM * BK + (wn0 + (GW / 4) * (r16 >> 2) + (r16 & 3)) * BK + (((g + 4 * c) ^ key_b) << 4);
    }
    v8i_t af[2][FM], bf[2][FN];
    auto read_q = [&](auto set_t, const uint8_t* s, int q) {
        constexpr int SET = decltype(set_t)::value;
        const bool is_b = q < FN;
        const int ro = is_b ? ((q / GT) * GW + (q % GT) * 4) * BK : (q - FN) * 16 * BK;
        const uint4 x0 = *reinterpret_cast<const uint4*>(s + (is_b ? offb[0] : offa[0]) + ro);
        const uint4 x1 = *reinterpret_cast<const uint4*>(s + (is_b ? offb[1] : offa[1]) + ro);
        const v8i_t v = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
        if (is_b) bf[SET][q < FN ? q : 0] = v; else af[SET][q < FN ? 0 : q - FN] = v;
    };

    v4f_t acc[FM][FN];
    auto clear = [&] {      // (the vector ALU's writes, two wait states ahead of any matrix instruction)
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            acc[i / FN][i % FN] = v4f_t{0.f, 0.f, 0.f, 0.f};
            if constexpr (ACC_V) asm volatile("" : "+v"(acc[i / FN][i % FN]));
            else asm volatile("" : "+a"(acc[i / FN][i % FN]));
        }
        asm volatile("s_nop 3" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    enter_tile();
#pragma unroll 1
    for (int r = 0; r < R; ++r) {
        const uint32_t ka = kofs(ca), ke = kofs(cb_e), ko = kofs(cb_o);
#pragma unroll
        for (int q = 0; q < NL; ++q) load_q(q, (uint32_t)(r * STAGE), ka, ke, ko);
        advance();
    }
    clear();
    wait_vmem_but_barrier<(R - 1) * NL>();      // stage 0 has landed for everyone (scale loads in between: the wait is the stricter)
#pragma unroll
    for (int q = 0; q < FM + FN; ++q) read_q(I0{}, smem, q);
    __builtin_amdgcn_sched_barrier(0);

    uint32_t cur = 0, nxt = STAGE;
    auto step = [&](auto par_t) {
        constexpr int P = decltype(par_t)::value;
        using NS = std::integral_constant<int, P ^ 1>;
        // (operations younger than stage s + 1's loads: those of R - 2 stages, and now and then scale loads and stores, with which the
        // wait is stricter than it need be; a wait that counts the stores was timed and is no faster)
        wait_vmem_but_barrier<(R - 2) * NL>();
        const uint32_t ka = kofs(ca), ke = kofs(cb_e), ko = kofs(cb_o), to = (uint32_t)__builtin_amdgcn_readfirstlane((int)cur);
        const uint8_t* rs = smem + nxt;
        constexpr int QR = NM >= 16 ? NM * 5 / 8 : (NM + 1) / 2;
#pragma unroll
        for (int t = 0; t < NM; ++t) {
            const int i = t / FN, j = (i & 1) ? FN - 1 - t % FN : t % FN;
            mfma<FA, FB, ACC_V>(acc[i][j], bf[P][j], af[P][i]);
            if (t < QR) {
#pragma unroll
                for (int q = t * (FM + FN) / QR; q < (t + 1) * (FM + FN) / QR; ++q) read_q(NS{}, rs, q);
            }
#pragma unroll
            for (int q = t * NL / NM; q < (t + 1) * NL / NM; ++q) load_q(q, to, ka, ke, ko);
            __builtin_amdgcn_sched_barrier(0);
        }
        cur = nxt;
        nxt = nxt + STAGE == R * STAGE ? 0 : nxt + STAGE;
        advance();
    };

    // ---- a tile's end: reciprocals of its scales, the results, and on to the next one
    int tab = 0, j = 0, left = 0;      // left: steps of the present tile to go
    auto steps_of = [&](int slot) {
        const int k = __builtin_amdgcn_readfirstlane(places[slot].w);
        return k > BK ? (k + BK - 1) / BK : 1;
    };
    const uint32_t lane_out = (uint32_t)(((wm0 + r16) * (int)p.ld_out + wn0 + 8 * g) * 2);
    auto finish = [&] {
        float* const t = tabs + tab * TAB;
        const int4 at = places[tab];
        const int row = __builtin_amdgcn_readfirstlane(at.x), rows = __builtin_amdgcn_readfirstlane(at.y), n0 = __builtin_amdgcn_readfirstlane(at.z);
        const bool some = __builtin_amdgcn_readfirstlane(at.w) != 0;      // (a tile without codes is zero whatever stands in its scales)
        if (tid < TM) t[tid] = some ? 1.0f / t[tid] : 0.0f;
        if (tid < TN) t[TMS + tid] = some ? 1.0f / t[TMS + tid] : 0.0f;
        asm volatile("s_nop 15\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const int cols = cols_all - n0 < TN ? cols_all - n0 : TN;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(p.out + (int64_t)row * p.ld_out + n0, 0,
                                                                             (int)(((int64_t)(rows - 1) * p.ld_out + cols) * 2), 0x00020000);
        constexpr int CE = GW / 4;      // consecutive columns of a lane in a group
#pragma unroll
        for (int grp = 0; grp < NG; ++grp) {
            float inv_b[CE];
#pragma unroll
            for (int e = 0; e < CE; e += 4) {
                const float4 t4 = *reinterpret_cast<const float4*>(t + TMS + wn0 + GW * grp + CE * g + e);
                inv_b[e] = t4.x; inv_b[e + 1] = t4.y; inv_b[e + 2] = t4.z; inv_b[e + 3] = t4.w;
            }
#pragma unroll
            for (int fi = 0; fi < FM; ++fi) {
                const float inv_a = t[wm0 + 16 * fi + r16];
                uint32_t pk[CE / 2];
#pragma unroll
                for (int e = 0; e < CE; e += 2)
                    pk[e / 2] = pack_bf16((acc[fi][grp * GT + (e >> 2)][e & 3] * inv_a) * inv_b[e],
                                          (acc[fi][grp * GT + ((e + 1) >> 2)][(e + 1) & 3] * inv_a) * inv_b[e + 1]);
                const uint32_t off = lane_out + (uint32_t)((16 * fi * (int)p.ld_out + GW * grp) * 2);
                const int col = wn0 + GW * grp + 8 * g;
                if constexpr (GW == 64) {
                    // lanes g = 0 .. 3 of a row hold its pieces (2 g, 2 g + 1) of eight columns; after the swaps pieces g and 4 + g
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const v2u_gr s1 = __builtin_amdgcn_permlane16_swap(pk[e], pk[4 + e], false, false);
                        const v2u_gr s2 = __builtin_amdgcn_permlane32_swap(s1[0], s1[1], false, false);
                        lo[e] = s2[0]; hi[e] = s2[1];
                    }
                    __builtin_amdgcn_raw_buffer_store_b128(v4u_t{lo[0], lo[1], lo[2], lo[3]}, rsrc, (int)(col < cols ? off : OOB), 0, 2);
                    __builtin_amdgcn_raw_buffer_store_b128(v4u_t{hi[0], hi[1], hi[2], hi[3]}, rsrc, (int)(col + 32 < cols ? off + 64u : OOB), 0, 2);
                } else {
                    __builtin_amdgcn_raw_buffer_store_b128(v4u_t{pk[0], pk[1], pk[2], pk[3]}, rsrc, (int)(col < cols ? off : OOB), 0, 2);
                }
            }
        }
        clear();
        ++j;
        tab = tab + 1 == NTAB ? 0 : tab + 1;
        left = steps_of(tab);
    };
    left = steps_of(0);
    while (true) {
        step(I0{});
        if (--left == 0) {
            finish();
            if (j == share.mine) break;
        }
        step(I1{});
        if (--left == 0) {
            finish();
            if (j == share.mine) break;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // trailing (out-of-range) refills must land before the LDS is handed back
}

template <int FA, int FB, int TM, int TN, int WAVES_M, int WAVES_N, int R, int GROUP_M, bool CONTRACT>
hipError_t launch_t(const GroupedGemm& g, hipStream_t st) {
    using namespace rg;
    auto kern = gemm_fp8_grouped_kernel<FA, FB, TM, TN, WAVES_M, WAVES_N, R, GROUP_M, CONTRACT>;
    constexpr int lds_fixed = R * (TM + TN) * BK + (R + 2) * (((TM + 63) / 64 + TN / 64) * 256 + 16);
    static_assert(lds_fixed + 12 * (GROUPED_MAX_EXPERTS + 2) <= 160 * 1024, "LDS");
    const int lds = lds_fixed + 12 * (int)(g.E + 2);
    static DynamicLdsOnce attr;
    if (hipError_t err = attr.ensure(reinterpret_cast<const void*>(kern), lds_fixed + 12 * (GROUPED_MAX_EXPERTS + 2)); err != hipSuccess) return err;
    const int64_t tiles_n = ((CONTRACT ? g.K : g.N) + TN - 1) / TN, tiles_m = (g.N + TM - 1) / TM;
    // rows: each group that has rows, and what lies behind the last one, has at most one tile that is not full
    const int64_t most = (CONTRACT ? tiles_m * g.E : g.M / TM + (g.E + 1 < g.M ? g.E + 1 : g.M)) * tiles_n;
    if (most > 0x3FFFFFFF) return hipErrorInvalidValue;
    int64_t cus = compute_units();
    if (const int forced = knob(KNOB_GEMM_STREAM); forced >= NUM_XCD) cus = forced;      // (few workgroups walk many tiles each)
    int64_t grid = std::max<int64_t>(cus, NUM_XCD) / NUM_XCD * NUM_XCD * (lds_fixed <= 72 * 1024 ? 2 : 1);
    if (const int64_t need = (most + NUM_XCD - 1) / NUM_XCD * NUM_XCD; grid > need) grid = need;
    const GroupedArgs a{g.a, g.lda, g.b, g.ldb, g.scale_a, g.scale_b, g.offsets, (int)g.E, (int)g.M, (int)g.N, (int)g.K,
                        static_cast<uint16_t*>(g.out), g.ld_out, (int)tiles_n, (int)tiles_m};
    kern<<<dim3((unsigned)grid), dim3(64 * WAVES_M * WAVES_N), lds, st>>>(a);
    return hipGetLastError();
}

// The tile forms: four of the kernel above, and those of gemm_fp8_grouped_stream.hip.
enum Form { F_64x64 = 0, F_64x128, F_128x128, F_128x256, F_192x256, F_256x256, FORMS };
// What a form takes, in us: a K step of 128 and the rest of a tile, times the rounds of tiles on the CUs (64 x 64: two tiles a CU), and
// the bytes at `rate`, whichever is more, as the fourth root of the sum of fourth powers (both count where they are close).  Fitted to 207
// forwards of 26 shapes (4 .. 128 experts, K and N 512 .. 14400, 2 .. 1024 rows an expert on average, groups a factor of 8 apart): off by
// 9 % in the root mean square, and the form with the least estimate is 3.6 % behind the best on average, 34 % at worst.  Without 64 x 64 4.5,
// without 128 x 256 4.3, without 256 x 256 5.1 % on average; 192 x 128 tiles give 0.1, 32 x 128, with a ring of six, nothing.
struct FormCost { int tm, tn, tiles_per_cu; double step, tile; };
constexpr FormCost kForms[FORMS] = {{64, 64, 2, 0.474, 0.3}, {64, 128, 1, 0.385, 1.0}, {128, 128, 1, 0.501, 1.8},
                                    {128, 256, 1, 0.787, 2.6}, {192, 256, 1, 0.956, 3.1}, {256, 256, 1, 1.101, 4.4}};
double form_cost(const FormCost& f, const GroupedGemm& g, int64_t cus) {
    constexpr double rate = 5.1e6;      // bytes a us
    const double busy = g.E < g.M ? (double)g.E : (double)g.M, mean = (double)g.M / (double)g.E;
    // row tiles: groups that have rows have one, longer ones half a tile more than their rows fill
    const double row_tiles = mean < 1 ? busy : busy * std::max(1.0, mean / f.tm + 0.5);
    const double full = row_tiles * (double)((g.N + f.tn - 1) / f.tn) / (double)(cus * f.tiles_per_cu);
    double rounds = (std::ceil(0.9 * full) + std::ceil(full) + std::ceil(1.1 * full)) / 3;      // (the number of tiles is an estimate)
    if (f.tiles_per_cu == 2 && 2 * full <= 1) rounds = 0.6;      // (a tile that has its CU to itself: one token, 64 experts 1408 x 2048, 64 x 64 11.1 us, 64 x 128 13.0)
    const double compute = 1.0 + rounds * ((double)((g.K + 127) / 128) * f.step + f.tile);
    const double bytes = (busy * (double)g.K * (double)g.N + (double)g.M * (double)g.K + 2.0 * (double)g.M * (double)g.N) / rate;
    return std::sqrt(std::sqrt(compute * compute * compute * compute + bytes * bytes * bytes * bytes));
}

template <int FA, int FB>
hipError_t launch_form(int form, const GroupedGemm& g, hipStream_t st) {
    switch (form) {
        case F_64x64: return launch_t<FA, FB, 64, 64, 2, 2, 4, 4, false>(g, st);
        case F_64x128: return launch_t<FA, FB, 64, 128, 2, 2, 4, 8, false>(g, st);
        case F_128x256: return launch_t<FA, FB, 128, 256, 2, 2, 3, 8, false>(g, st);
        default: return launch_t<FA, FB, 128, 128, 2, 2, 4, 4, false>(g, st);
    }
}

template <int FA, int FB>
hipError_t launch_rows(const GroupedGemm& g, hipStream_t st) {
    // the switches: 1 + form; the forms of the other file 0: never, 2: always the best of them
    const int forced = knob(KNOB_GEMM_RING), stream = knob(KNOB_GEMM_STREAM);
    int form = forced - 1;
    if (forced <= 0 || forced > FORMS) {
        const int64_t cus = compute_units() > 0 ? compute_units() : 256;
        const int first = stream >= 2 ? F_192x256 : 0, end = stream == 0 ? F_192x256 : FORMS;
        form = first;
        for (int f = first + 1; f < end; ++f)
            if (form_cost(kForms[f], g, cus) < form_cost(kForms[form], g, cus)) form = f;
    }
    if (form >= F_192x256) return launch_gemm_fp8_grouped_stream_rows(g, kForms[form].tm, st);
    return launch_form<FA, FB>(form, g, st);
}

}  // namespace

#define FP8K_FORMATS(CALL)                                                                      \
    if (g.fmt_a == FMT_E4M3FN && g.fmt_b == FMT_E4M3FN) return CALL<FMT_E4M3FN, FMT_E4M3FN>(g, st); \
    if (g.fmt_a == FMT_E5M2 && g.fmt_b == FMT_E4M3FN) return CALL<FMT_E5M2, FMT_E4M3FN>(g, st);     \
    if (g.fmt_a == FMT_E4M3FN) return CALL<FMT_E4M3FN, FMT_E5M2>(g, st);                            \
    return CALL<FMT_E5M2, FMT_E5M2>(g, st);

hipError_t launch_gemm_fp8_grouped_rows(const GroupedGemm& g, hipStream_t st) {
    if (g.M <= 0) return hipSuccess;
    FP8K_FORMATS(launch_rows)
}

// Short groups here, where a tile of one or two steps has the next tile's operands and the last one's stores under way (whole backward
// in us, the other file's 192 x 256 tiles of two steps at least / these of 128 x 256; at 256 rows its tiles of the rule below):
//   rows a group        24        90        143       192        256
//   64 of 1408 x 2048   321/303   361/331   380/345   400/366    412/404
//   32 of 4096 x 1408   391/360   434/395   437/398   486/450    456/453
//   128 of 768 x 2048   365/351   411/378   442/412   474/440    516/515
//   16 of 2048 x 5632   336/332   345/343   366/362   392/388    402/409
//   8 of 4096 x 4096    271/252   275/263   278/263   294/283    297/307
//   8 of 4096 x 14336   887/871   975/954   996/980   1031/998   1007/1043
//   8 of 14336 x 4096   862/803   888/831   912/850   965/887    903/924
// The switch GEMM_STREAM: 0 always here, 2 and more never.
template <int FA, int FB>
static hipError_t launch_contract(const GroupedGemm& g, hipStream_t st) {
    const int stream = knob(KNOB_GEMM_STREAM);
    if (stream == 0 || (stream < 0 && g.M <= 192 * g.E)) return launch_t<FA, FB, 128, 256, 2, 2, 3, 8, true>(g, st);
    return launch_gemm_fp8_grouped_stream_contract(g, st);
}
hipError_t launch_gemm_fp8_grouped_contract(const GroupedGemm& g, hipStream_t st) { FP8K_FORMATS(launch_contract) }

}  // namespace fp8k
