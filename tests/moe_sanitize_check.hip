// Sanitizer driver for the HOST side of the mixture-of-experts and AdamW entry points (test infrastructure).
//
// Built by tests/test_moe_sanitizers.py from this file, moe_api.hip, tuning.hip and adamw.hip (for its table) with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code only.  The other kernels' launchers are the stubs below: they touch nothing but check that
// every place handed to them lies inside the workspace that was asked for and overlaps no other of the same call.
#include "../include/fp8mi355.h"
#include "../paper_2507_16099_amd/csrc/launchers.hpp"
#include "../paper_2507_16099_amd/csrc/moe_launchers.hpp"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

static uintptr_t g_ws = 0, g_ws_end = 0;      // the workspace of the call under test
static int g_launches = 0, g_few = 0, g_both = 0;
struct Span { uintptr_t a, b; };
static std::vector<Span> g_written;           // places of codes and scales of this call, each written by one launch

static void check(bool ok, const char* what) {
    if (ok) return;
    std::fprintf(stderr, "%s (%s)\n", what, fp8_last_error());
    std::exit(1);
}
static void inside(const void* p, size_t bytes, const char* what) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    check(a >= g_ws && a + bytes <= g_ws_end, what);
}
static void written(const void* p, size_t bytes, const char* what) {
    inside(p, bytes, what);
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    for (const Span& s : g_written) check(a >= s.b || a + bytes <= s.a, what);
    g_written.push_back({a, a + bytes});
}

namespace fp8k {
thread_local char g_text[256];
int api_error(int code, const char* text) {
    std::snprintf(g_text, sizeof(g_text), "%s", text);
    return code;
}
hipError_t launch_fill_u32(uint32_t* p, int64_t n, uint32_t, hipStream_t) {
    check(n >= 0 && n <= (int64_t)1 << 31 && p, "fill");
    ++g_launches;
    return hipSuccess;
}
size_t route_workspace_bytes(int64_t T, int64_t E) { return T <= 64 ? 256 : 256 * (size_t)E * 4; }
hipError_t launch_moe_route(const void*, bool, int64_t, int64_t, int64_t, int, bool, float*, int32_t*, int32_t*, int32_t*, int32_t*, void*, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_moe_route_bwd(const float*, const void*, bool, int64_t, int64_t, int64_t, int, bool, const float*, const int32_t*, void*, int64_t, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_moe_combine(const void*, int64_t, int64_t, const float*, const int32_t*, int64_t, int64_t, int, void*, int64_t, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_moe_combine_bwd(const void*, int64_t, const void*, int64_t, const float*, const int32_t*, const int32_t*, int64_t, int64_t, int64_t, int, void*, int64_t, float*, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_quant_rows_gather(const void*, int64_t, int64_t, const int32_t*, int64_t M, int64_t cols, int, int, uint8_t* q, int64_t ld_q, float* scale, hipStream_t) {
    check(ld_q >= cols, "row pitch");
    written(q, (size_t)M * ld_q, "row codes");
    written(scale, (size_t)M * 4, "row scales");
    ++g_launches;
    return hipSuccess;
}
static void cols(const GroupedColOperand& op, int64_t E) {
    const int64_t rows = op.uniform ? op.M / E : grouped_padded(op.M, E);
    check(op.ld_t >= rows, "column pitch");
    written(op.qt, (size_t)(op.uniform ? E : 1) * op.cols * op.ld_t, "column codes");
    written(op.scale, (size_t)E * op.cols * 4, "column scales");
    inside(op.amax, (size_t)E * op.cols * 4, "column maxima");
    ++g_launches;
}
hipError_t launch_quant_cols_grouped(const GroupedColOperand& op, const int32_t*, int64_t E, int, hipStream_t) { cols(op, E); return hipSuccess; }
hipError_t launch_quant_rows_cols_grouped(const GroupedColOperand& op, const int32_t* offsets, int64_t E, int flags, uint8_t* q, int64_t ld_q, float* scale, hipStream_t st) {
    if (++g_both & 1) return hipErrorNotSupported;      // (both ways)
    cols(op, E);
    return launch_quant_rows_gather(op.x, op.T, op.ldx, nullptr, op.M, op.cols, op.fmt, flags, q, ld_q, scale, st);
}
hipError_t launch_quant_strips_grouped(const GroupedColOperand& op, const GroupedColOperand* second, const int32_t*, int64_t E, int, hipStream_t) {
    cols(op, E);
    if (second) cols(*second, E);
    return hipSuccess;
}
static hipError_t gemm(const GroupedGemm& g) {
    check(g.lda >= 0 && g.a && g.b && g.out && g.offsets, "product");
    inside(g.a, 1, "product's codes");
    ++g_launches;
    return hipSuccess;
}
hipError_t launch_gemm_fp8_grouped_rows(const GroupedGemm& g, hipStream_t) { return gemm(g); }
hipError_t launch_gemm_fp8_grouped_contract(const GroupedGemm& g, hipStream_t) { return gemm(g); }
hipError_t launch_grouped_few(const void*, int64_t, const int32_t*, int, int, const GroupedGemm& g, hipStream_t) {
    if (++g_few & 1) return hipErrorNotSupported;
    inside(g.a, 1, "product's codes");
    ++g_launches;
    return hipSuccess;
}
}  // namespace fp8k

extern "C" const char* fp8_last_error(void) { return fp8k::g_text; }
extern "C" int fp8_quantize(const void*, int64_t rows, int64_t cols, int64_t, int, int, int, uint8_t* q, int64_t ld_q, float* scale, void*) {
    check(ld_q >= cols, "weight pitch");
    written(q, (size_t)rows * ld_q, "weight codes");
    written(scale, (size_t)rows * 4, "weight scales");
    return FP8_OK;
}

static void expect(int got, int want, const char* what) {
    if (got == want) return;
    std::fprintf(stderr, "%s: %d, expected %d (%s)\n", what, got, want, fp8_last_error());
    std::exit(1);
}
#define EXPECT(call, want) (g_written.clear(), expect((call), (want), #call))
static void workspace(void* p, size_t bytes) {
    g_ws = reinterpret_cast<uintptr_t>(p);
    g_ws_end = g_ws + bytes;
}

int main() {
    // never dereferenced by host code: a fake, suitably aligned "device" address
    void* p = reinterpret_cast<void*>(uintptr_t(1) << 32);
    float* f = static_cast<float*>(p);
    int32_t* i = static_cast<int32_t*>(p);
    const fp8_recipe row{FP8_ROW, FP8_E4M3FN, FP8_E4M3FN, FP8_E5M2, 0};
    // M, E, K, N
    const int64_t dims[][4] = {{0, 1, 0, 0}, {1, 1, 16, 16}, {5, 512, 48, 80}, {16384, 8, 4096, 14336}, {9186, 64, 2048, 1408}, {(1 << 24) - 1, 512, 16, 16},
                               {8000000, 1, 4096, 16}, {7, 2, (1 << 22) - 128, (1 << 22) - 128}, {1000, 500, 1 << 20, 16}, {100, 4, 0, 64}, {100, 4, 64, 0},
                               {6000, 8, 272, 9008}, {0, 8, 4096, 1 << 20}};
    for (const auto& d : dims) {
        const int64_t M = d[0], E = d[1], K = d[2], N = d[3];
        for (int bwd = 0; bwd < 2; ++bwd) {
            const size_t n = fp8_grouped_linear_workspace_bytes(M, E, K, N, &row, bwd);
            if (!n) {
                check(fp8_last_error()[0], "no reason given");
                continue;
            }
            workspace(p, n);
            for (int with_rows = 0; with_rows < 2; ++with_rows)
                for (int parts = 0; parts < 4; ++parts) {
                    const int32_t* rows = with_rows ? i : nullptr;
                    const int64_t T = with_rows ? 3 : M;
                    if (!bwd) EXPECT(fp8_grouped_linear_fwd(p, T, rows, p, i, E, M, K, N, &row, p, p, n, nullptr), FP8_OK);
                    else EXPECT(fp8_grouped_linear_bwd(p, p, T, rows, p, i, E, M, K, N, &row, parts & 1 ? p : nullptr, parts & 2 ? p : nullptr, p, n, nullptr), FP8_OK);
                }
            if (M && K && N) {
                if (!bwd) EXPECT(fp8_grouped_linear_fwd(p, M, nullptr, p, i, E, M, K, N, &row, p, p, n - 256, nullptr), FP8_ERR_WORKSPACE);
                else EXPECT(fp8_grouped_linear_bwd(p, p, M, nullptr, p, i, E, M, K, N, &row, p, p, p, n - 256, nullptr), FP8_ERR_WORKSPACE);
            }
        }
        const size_t n = fp8_grouped_linear_prequantized_workspace_bytes(M, K);
        check(n > 0, "workspace of the serving form");
        workspace(p, n);
        for (int twice = 0; twice < 2; ++twice)
            EXPECT(fp8_grouped_linear_fwd_prequantized(p, M, nullptr, 1, FP8_POW2_SCALE, static_cast<uint8_t*>(p), K, 0, f, i, E, M, K, N, p, p, n, nullptr), FP8_OK);
    }
    for (int64_t T : {int64_t(0), int64_t(1), int64_t(64), int64_t(65), int64_t(1) << 24})
        for (int k : {1, 2, 16}) {
            const size_t n = fp8_moe_route_workspace_bytes(T, 64, k);
            check(n > 0, "router's workspace");
            EXPECT(fp8_moe_route(p, T, 64, 72, k, FP8_ROUTE_RENORM | FP8_ROUTE_FP32, f, i, i, i, i, p, n, nullptr), FP8_OK);
            EXPECT(fp8_moe_route_bwd(f, p, T, 64, 72, k, 0, f, i, p, 64, nullptr), FP8_OK);
            if (T < 1 << 20) {
                EXPECT(fp8_moe_combine(p, T * k, 64, f, i, T, 64, k, p, 72, nullptr), FP8_OK);
                EXPECT(fp8_moe_combine_bwd(p, 64, p, T * k, 64, f, i, i, T, 64, k, p, 64, f, nullptr), FP8_OK);
            }
        }
    const int64_t most = INT64_MAX;
    EXPECT(fp8_moe_route(p, most, 64, 64, 16, 0, f, i, i, i, i, p, most, nullptr), FP8_ERR_SHAPE);
    EXPECT(fp8_moe_combine(p, most, most, f, i, most, most, 2, p, most, nullptr), FP8_ERR_SHAPE);
    EXPECT(fp8_grouped_linear_fwd(p, most, i, p, i, most, most, most, most, &row, p, p, most, nullptr), FP8_ERR_SHAPE);
    EXPECT(fp8_grouped_linear_bwd(p, p, most, i, p, i, 1, most, most, most, &row, p, p, p, most, nullptr), FP8_ERR_SHAPE);
    check(fp8_grouped_linear_prequantized_workspace_bytes(most, most) == 0, "no refusal");

    // tables in heap blocks of exactly the size that was asked for
    const std::vector<std::vector<int64_t>> lists = {{}, {0}, {1}, {2048, 2049, 0, 5}, {int64_t(1) << 37, 1}, {int64_t(16384) * 2048 + 1, 8193, 0, 3}, {most}};
    for (const auto& sizes : lists)
        for (int flags : {0, int(FP8_ADAMW_STATE_FP8), int(FP8_ADAMW_PARAM_FP32 | FP8_ADAMW_GRAD_FP32 | FP8_ADAMW_STATE_FP8)}) {
            std::vector<fp8_adamw_tensor> t;
            for (int64_t n : sizes) t.push_back({p, p, p, p, f, f, n});
            const size_t n = fp8_adamw_table_bytes(t.data(), (int64_t)t.size(), flags);
            if (!n) continue;
            void* table = std::malloc(n);
            int64_t blocks = 0;
            EXPECT(fp8_adamw_table(t.data(), (int64_t)t.size(), flags, table, n, &blocks), FP8_OK);
            EXPECT(fp8_adamw_table(t.data(), (int64_t)t.size(), flags, table, n - 1, &blocks), FP8_ERR_WORKSPACE);
            EXPECT(fp8_adamw_step(p, 0, flags, 1e-3, 0.9, 0.999, 1e-8, 0.1, most, f, nullptr), FP8_OK);
            std::free(table);
        }
    check(g_launches > 0 && g_few > 1 && g_both > 1, "stubs not reached");
    std::printf("moe_sanitize_check ok, %d launches\n", g_launches);
    return 0;
}
