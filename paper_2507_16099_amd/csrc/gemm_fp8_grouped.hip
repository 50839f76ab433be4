// Scaled FP8 products grouped by expert (gfx950), groups of any size that only the device knows:
//   rows      out[r] = A[r] B[e]^T / (sa[r] sb[e])        for the rows r of group e; one weight B[e] [N, K] per group
//   contract  out[e] = A_e B_e^T / (sa[e] sb[e])          A_e [N, n_e], B_e [K, n_e]: the columns of the group in A [N, lda], B [K, ldb]
// The tile kernel is that of gemm_fp8_ring.hpp: a ring of R stages of K steps filled by LDS-DMA ahead of the matrix cores, one
// workgroup barrier a step, fragments of the next step read behind the matrix instructions of the present one; its LDS layout,
// swizzle keys and operand order are described there.
//
// What is different: which tile a workgroup has.  The host knows M rows and E groups, so it launches as many workgroups as the
// groups can come to (rows: M / TM + E row tiles); each finds its tile by a scan of the offsets over the lanes of a wavefront, and
// those beyond the last tile end.  The tiles in use are dealt to the XCDs in contiguous ranges, walked in patches of GROUP_M row
// tiles, as in the ungrouped kernels; neighbouring row tiles of one group share the weight's panel in that L2.
// Rows behind the last group (slots that no expert took) are written as zeros: a tile without K steps.
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
    constexpr bool ACC_V = 4 * NM + 16 * (FM + FN) <= (NW == 8 ? 208 : 192);
    static_assert((NW == 4 || NW == 8) && WM % 16 == 0 && (GW == 64 || GW == 32) && WN % GW == 0 && TM % (8 * NW) == 0 && TN % 64 == 0 && TN % (8 * NW) == 0, "tile");
    static_assert(R >= 3 && (R - 1) * NL <= 63, "vmcnt range");
    constexpr int CPR = WN / 8;
    constexpr bool POW2 = (CPR & (CPR - 1)) == 0;
    constexpr int PITCH = (CPR + (POW2 ? 0 : 1)) * 16;
    static_assert(NW * WM * PITCH <= R * STAGE, "the epilogue stages through the ring");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

    const int slot = (int)blockIdx.x / NUM_XCD, xcd = (int)blockIdx.x % NUM_XCD;
    int group, m0, n0, rows_a, rows_b, Kt;         // Kt: contracted elements (codes)
    const uint8_t *a0, *b0;
    const float *sa, *sb;
    uint16_t* out;
    if constexpr (!CONTRACT) {
        GroupTile t = find_group_tile<true>(p.offsets, p.E, p.M, TM, -1);
        const int tiles = t.total * p.tiles_n, per_xcd = (tiles + NUM_XCD - 1) / NUM_XCD;
        const int logical = xcd * per_xcd + slot;
        if (slot >= per_xcd || logical >= tiles) return;
        const int in_group = GROUP_M * p.tiles_n, first_m = logical / in_group * GROUP_M, in = logical % in_group;
        const int gsize = t.total - first_m < GROUP_M ? t.total - first_m : GROUP_M;
        const int tn = in / gsize, tm = first_m + in - tn * gsize;
        t = find_group_tile<true>(p.offsets, p.E, p.M, TM, tm);
        group = t.group;
        const int e = group < p.E ? group : p.E - 1;
        m0 = t.row0;
        rows_a = t.rows;
        n0 = tn * TN;
        rows_b = p.N - n0 < TN ? p.N - n0 : TN;
        Kt = group < p.E ? p.K : 0;
        a0 = p.A + (int64_t)m0 * p.lda;
        b0 = p.B + ((int64_t)e * p.N + n0) * p.ldb;
        sa = p.scale_a + m0;
        sb = p.scale_b + (int64_t)e * p.N + n0;
        out = p.out + (int64_t)m0 * p.ld_out;
    } else {
        const int per_group = p.tiles_m * p.tiles_n;
        const int64_t tiles = (int64_t)per_group * p.E, per_xcd = (tiles + NUM_XCD - 1) / NUM_XCD;
        const int64_t logical = xcd * per_xcd + slot;
        if (slot >= per_xcd || logical >= tiles) return;
        group = (int)(logical / per_group);
        const int rest = (int)(logical % per_group);
        const int in_group = GROUP_M * p.tiles_n, first_m = rest / in_group * GROUP_M, in = rest % in_group;
        const int gsize = p.tiles_m - first_m < GROUP_M ? p.tiles_m - first_m : GROUP_M;
        const int tn = in / gsize, tm = first_m + in - tn * gsize;
        const GroupSpan s = find_group(p.offsets, p.E, p.M, group);
        m0 = tm * TM;
        n0 = tn * TN;
        rows_a = p.N - m0 < TM ? p.N - m0 : TM;
        rows_b = p.K - n0 < TN ? p.K - n0 : TN;
        Kt = (s.rows + 15) & ~15;
        a0 = p.A + (int64_t)m0 * p.lda + s.pad0;
        b0 = p.B + (int64_t)n0 * p.ldb + s.pad0;
        sa = p.scale_a + (int64_t)group * p.N + m0;
        sb = p.scale_b + (int64_t)group * p.K + n0;
        out = p.out + ((int64_t)group * p.N + m0) * p.ld_out;
    }
    const int cols = CONTRACT ? p.K : p.N;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = (wave / WAVES_N) * WM, wn0 = (wave % WAVES_N) * WN;

    const int64_t lda = p.lda, ldb = p.ldb;
    const uint64_t pa = reinterpret_cast<uint64_t>(a0), pb = reinterpret_cast<uint64_t>(b0);
    const v4i_t rsrc_a = {(int)(uint32_t)pa, (int)(uint32_t)(pa >> 32), (int)((int64_t)(rows_a - 1) * lda + Kt), 0x00020000};
    const v4i_t rsrc_b = {(int)(uint32_t)pb, (int)(uint32_t)(pb >> 32), (int)((int64_t)(rows_b - 1) * ldb + Kt), 0x00020000};

    float* inv_tab = reinterpret_cast<float*>(smem + R * STAGE);
    {
        const uint64_t psa = reinterpret_cast<uint64_t>(sa), psb = reinterpret_cast<uint64_t>(sb);
        const v4i_t rsrc_sa = {(int)(uint32_t)psa, (int)(uint32_t)(psa >> 32), rows_a * 4, 0x00020000};
        const v4i_t rsrc_sb = {(int)(uint32_t)psb, (int)(uint32_t)(psb >> 32), rows_b * 4, 0x00020000};
#pragma unroll
        for (int h = 0; h < (NU + NW - 1) / NW; ++h) {
            const int u = wave + NW * h, r = 64 * (u < UA ? u : u - UA) + lane;
            const uint32_t at = (uint32_t)(size_t)inv_tab + (uint32_t)u * 256u;
            if (u < UA) lds_dma4(rsrc_sa, at, (uint32_t)(r < rows_a ? r : rows_a - 1) * 4u);
            else if (u < NU) lds_dma4(rsrc_sb, at, (uint32_t)(r < rows_b ? r : rows_b - 1) * 4u);
        }
    }
    auto scale_table = [&]() {       // (a tile without K steps is zero whatever stands in its scales)
        if (tid < TM) inv_tab[tid] = Kt ? 1.0f / inv_tab[tid] : 0.0f;
        if (tid < TN) inv_tab[TMS + tid] = Kt ? 1.0f / inv_tab[TMS + tid] : 0.0f;
    };

    const int lrow = lane >> 3;
    const int ca = (lane & 7) ^ ((4 * (wave & 1) + (lrow >> 1)) & 7);
    const int kb_e = SH == 4 ? (wave >> 1) : wave, kb_o = SH == 4 && NW == 4 ? 2 + (wave >> 1) : kb_e;
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
    auto kofs = [&](int k0, int c) { return k0 + c * 16 < Kt ? (uint32_t)k0 : OOB; };

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
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = v4f_t{0.f, 0.f, 0.f, 0.f};

    const int ksteps = (Kt + BK - 1) / BK;
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int k0 = r * BK;
        const uint32_t ka = kofs(k0, ca), ke = kofs(k0, cb_e), ko = kofs(k0, cb_o);
#pragma unroll
        for (int q = 0; q < NL; ++q) load_q(q, (uint32_t)(r * STAGE), ka, ke, ko);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
        if constexpr (ACC_V) asm volatile("" : "+v"(acc[i / FN][i % FN]));
        else asm volatile("" : "+a"(acc[i / FN][i % FN]));
    }
    wait_vmem_but_barrier<(R - 1) * NL>();
#pragma unroll
    for (int q = 0; q < FM + FN; ++q) read_q(I0{}, smem, q);
    scale_table();
    __builtin_amdgcn_sched_barrier(0);

    uint32_t cur = 0, nxt = STAGE;
    int k_refill = R * BK;
    auto step = [&](auto par_t) {
        constexpr int P = decltype(par_t)::value;
        using NS = std::integral_constant<int, P ^ 1>;
        wait_vmem_but_barrier<(R - 2) * NL>();
        const uint32_t ka = kofs(k_refill, ca), ke = kofs(k_refill, cb_e), ko = kofs(k_refill, cb_o);
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
            for (int q = t * NL / NM; q < (t + 1) * NL / NM; ++q) load_q(q, cur, ka, ke, ko);
            __builtin_amdgcn_sched_barrier(0);
        }
        cur = nxt;
        nxt = nxt + STAGE == R * STAGE ? 0 : nxt + STAGE;
        k_refill += BK;
    };
    int s = 0;
    if constexpr (ACC_V) {
        for (; s + 2 <= ksteps; s += 2) {
            step(I0{});
            step(I1{});
        }
        if (s < ksteps) step(I0{});
    } else {
        do {
            step(I0{});
            if (s + 1 < ksteps) step(I1{});
            s += 2;
        } while (s < ksteps);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    constexpr int CE = GW / 4;
    float inv_b[NG][CE];
#pragma unroll
    for (int grp = 0; grp < NG; ++grp)
#pragma unroll
        for (int e = 0; e < CE; e += 4) {
            const float4 t4 = *reinterpret_cast<const float4*>(inv_tab + TMS + wn0 + GW * grp + CE * g + e);
            inv_b[grp][e] = t4.x; inv_b[grp][e + 1] = t4.y; inv_b[grp][e + 2] = t4.z; inv_b[grp][e + 3] = t4.w;
        }
    float inv_a[FM];
#pragma unroll
    for (int fi = 0; fi < FM; ++fi) inv_a[fi] = inv_tab[wm0 + 16 * fi + r16];
    uint8_t* q_lds = smem + wave * (WM * PITCH);
#pragma unroll
    for (int fi = 0; fi < FM; ++fi) {
        uint8_t* row = q_lds + (16 * fi + r16) * PITCH;
#pragma unroll
        for (int grp = 0; grp < NG; ++grp) {
            float v[CE];
#pragma unroll
            for (int e = 0; e < CE; ++e) v[e] = (acc[fi][grp * GT + (e >> 2)][e & 3] * inv_a[fi]) * inv_b[grp][e];
#pragma unroll
            for (int h = 0; h < CE / 8; ++h) {
                const int c = (GW / 8) * grp + (CE / 8) * g + h;
                *reinterpret_cast<uint4*>(row + ((POW2 ? c ^ (r16 % CPR) : c) << 4)) =
                    make_uint4(pack_bf16(v[8 * h], v[8 * h + 1]), pack_bf16(v[8 * h + 2], v[8 * h + 3]),
                               pack_bf16(v[8 * h + 4], v[8 * h + 5]), pack_bf16(v[8 * h + 6], v[8 * h + 7]));
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int fi = 0; fi < FM; ++fi) {
#pragma unroll
        for (int it = 0; it < (CPR + 3) / 4; ++it) {
            const int piece = 64 * it + lane;
            if (piece >= 16 * CPR) continue;
            const int rr = 16 * fi + piece / CPR, c_rd = piece % CPR;
            const uint4 v = *reinterpret_cast<const uint4*>(q_lds + rr * PITCH + ((POW2 ? c_rd ^ ((rr & 15) % CPR) : c_rd) << 4));
            const int m = wm0 + rr, n = n0 + wn0 + c_rd * 8;
            // (the output's columns are a multiple of eight)
            if (m < rows_a && n < cols) *reinterpret_cast<v4u_t*>(out + (int64_t)m * p.ld_out + n) = v4u_t{v.x, v.y, v.z, v.w};
        }
    }
}

template <int FA, int FB, int TM, int TN, int WAVES_M, int WAVES_N, int R, int GROUP_M, bool CONTRACT>
hipError_t launch_t(const GroupedGemm& g, hipStream_t st) {
    using namespace rg;
    auto kern = gemm_fp8_grouped_kernel<FA, FB, TM, TN, WAVES_M, WAVES_N, R, GROUP_M, CONTRACT>;
    constexpr int lds = R * (TM + TN) * BK + ((TM + 63) / 64 + TN / 64) * 256;
    static_assert(lds <= 160 * 1024, "LDS");
    static DynamicLdsOnce attr;
    if (hipError_t err = attr.ensure(reinterpret_cast<const void*>(kern), lds); err != hipSuccess) return err;
    const int64_t tiles_n = ((CONTRACT ? g.K : g.N) + TN - 1) / TN, tiles_m = (g.N + TM - 1) / TM;
    // rows: each group that has rows, and what lies behind the last one, has at most one tile that is not full
    const int64_t most = CONTRACT ? tiles_m * g.E : g.M / TM + (g.E + 1 < g.M ? g.E + 1 : g.M);
    const int64_t tiles = most * tiles_n, grid = (tiles + NUM_XCD - 1) / NUM_XCD * NUM_XCD;
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    const GroupedArgs a{g.a, g.lda, g.b, g.ldb, g.scale_a, g.scale_b, g.offsets, (int)g.E, (int)g.M, (int)g.N, (int)g.K,
                        static_cast<uint16_t*>(g.out), g.ld_out, (int)tiles_n, (int)tiles_m};
    kern<<<dim3((unsigned)grid), dim3(64 * WAVES_M * WAVES_N), lds, st>>>(a);
    return hipGetLastError();
}

// The tile forms: those of RingTile (launchers.hpp) that pay here, one of 32 rows, and the persistent kernel's 256 x 256.
enum Form { F_32x128 = 0, F_64x64, F_64x128, F_128x128, F_192x128, F_128x256, F_STREAM, FORMS };
// What a form takes, in us: a K step of 128 and the rest of a tile, times the rounds of tiles on the CUs (64 x 64: two tiles a CU), and
// the bytes at `rate`, whichever is more, as the fourth root of the sum of fourth powers (both count where they are close).  Fitted to 207
// forwards of 26 shapes (4 .. 128 experts, K and N 512 .. 14400, 1/4 .. 4096 rows an expert on average, groups a factor of 8 apart): off by
// 11 % in the root mean square, and the form with the least estimate is 5 % behind the best of ten forms on average, 36 % at worst; by
// the mean number of rows alone (up to 16, 64, 256) 12 % and 86 %.  Others that were tried gain under 0.5 % together: 128 x 64, 96 x 128,
// 256 x 128.
struct FormCost { int tm, tn, tiles_per_cu; double step, tile; };
constexpr FormCost kForms[FORMS] = {{32, 128, 1, 0.303, 3.9}, {64, 64, 2, 0.408, 2.9}, {64, 128, 1, 0.382, 3.2}, {128, 128, 1, 0.508, 3.8},
                                    {192, 128, 1, 0.589, 4.7}, {128, 256, 1, 0.765, 5.6}, {256, 256, 1, 1.151, 7.2}};
double form_cost(const FormCost& f, const GroupedGemm& g, int64_t cus) {
    constexpr double rate = 5.1e6;      // bytes a us
    const double busy = g.E < g.M ? (double)g.E : (double)g.M, mean = (double)g.M / (double)g.E;
    // row tiles: groups that have rows have one, longer ones half a tile more than their rows fill
    const double row_tiles = mean < 1 ? busy : busy * std::max(1.0, mean / f.tm + 0.5);
    const double full = row_tiles * (double)((g.N + f.tn - 1) / f.tn) / (double)(cus * f.tiles_per_cu);
    const double rounds = (std::ceil(0.9 * full) + std::ceil(full) + std::ceil(1.1 * full)) / 3;      // (the number of tiles is an estimate)
    const double compute = rounds * ((double)((g.K + 127) / 128) * f.step + f.tile);
    const double bytes = (busy * (double)g.K * (double)g.N + (double)g.M * (double)g.K + 2.0 * (double)g.M * (double)g.N) / rate;
    return std::sqrt(std::sqrt(compute * compute * compute * compute + bytes * bytes * bytes * bytes));
}

template <int FA, int FB>
hipError_t launch_form(int form, const GroupedGemm& g, hipStream_t st) {
    switch (form) {
        case F_64x64: return launch_t<FA, FB, 64, 64, 2, 2, 4, 4, false>(g, st);
        case F_64x128: return launch_t<FA, FB, 64, 128, 2, 2, 4, 8, false>(g, st);
        case F_192x128: return launch_t<FA, FB, 192, 128, 2, 2, 3, 4, false>(g, st);
        case F_128x256: return launch_t<FA, FB, 128, 256, 2, 2, 3, 8, false>(g, st);
        case F_32x128: return launch_t<FA, FB, 32, 128, 1, 4, 6, 1, false>(g, st);
        default: return launch_t<FA, FB, 128, 128, 2, 2, 4, 4, false>(g, st);
    }
}

template <int FA, int FB>
hipError_t launch_rows(const GroupedGemm& g, hipStream_t st) {
    const int forced = knob(KNOB_GEMM_RING), stream = knob(KNOB_GEMM_STREAM);      // 1 + form; 0: never, 2: wherever it fits
    int form = 0;
    if (forced > 0) {
        form = forced - 1 < F_STREAM ? forced - 1 : F_128x128;
    } else {
        const int64_t cus = compute_units() > 0 ? compute_units() : 256;
        const bool fits = stream != 0 && gemm_fp8_grouped_stream_fits(g);
        for (int f = 1; f < (fits ? FORMS : F_STREAM); ++f)
            if (form_cost(kForms[f], g, cus) < form_cost(kForms[form], g, cus)) form = f;
        if (fits && stream >= 2) form = F_STREAM;
    }
    if (form == F_STREAM) return launch_gemm_fp8_grouped_stream_rows(g, st);
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

// dW: the persistent kernel (64 experts 1408 x 2048 of 16 .. 2048 rows: 86 to 430 us, 128 x 256 tiles 150 to 620), tiles for the
// tables of groups that its LDS has no room for
template <int FA, int FB>
static hipError_t launch_contract(const GroupedGemm& g, hipStream_t st) {
    if (knob(KNOB_GEMM_STREAM) != 0 && gemm_fp8_grouped_stream_fits(g)) return launch_gemm_fp8_grouped_stream_contract(g, st);
    return launch_t<FA, FB, 128, 128, 2, 2, 4, 4, true>(g, st);
}
hipError_t launch_gemm_fp8_grouped_contract(const GroupedGemm& g, hipStream_t st) { FP8K_FORMATS(launch_contract) }

}  // namespace fp8k
