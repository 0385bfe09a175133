// Driver of the block norms' and linear layers' entry points of the C ABI (include/tm.h) for the sanitizer
// build, as host_abi_driver.cpp for the others: descriptor and argument checks, sizes and their limits, the
// parts of rows and the shares of split tiles. Exit status 0 and "host block driver: all checks passed" when
// every check holds.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../paper_2506_03099_amd/csrc/tm_api.cpp"

namespace {

int g_failed = 0;
int g_checks = 0;

#define EXPECT(cond)                                                                        \
    do {                                                                                    \
        ++g_checks;                                                                         \
        if (!(cond)) {                                                                      \
            ++g_failed;                                                                     \
            std::fprintf(stderr, "FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, \
                         #cond, tm_last_error());                                           \
        }                                                                                   \
    } while (0)

// Aligned, non-null, and not memory the HIP runtime knows.
void* const FAKE = reinterpret_cast<void*>(uintptr_t(1) << 40);
float* const FAKE_F = static_cast<float*>(FAKE);

tm_block_norm_desc norm(int32_t E, int32_t pre = TM_NORM_LAYER, int32_t post = TM_NORM_NONE, int32_t B = 1,
                        int32_t groups = 1, int32_t group = 0, float eps = 1e-6f) {
    return tm_block_norm_desc{B, E, pre, post, TM_BF16, TM_F32, groups, group, eps};
}

tm_linear_desc linear(int32_t K, int32_t N, int32_t act = TM_ACT_NONE, int32_t B = 1, int32_t groups = 1, int32_t group = 0) {
    return tm_linear_desc{B, K, N, act, TM_BF16, groups, group};
}

tm_status norm_fwd(const tm_block_norm_desc* d, int32_t n, int64_t first, const void* y = nullptr, void* r = nullptr,
                   void* h = FAKE, const float* gate = nullptr, const float* scale = nullptr, const float* shift = nullptr,
                   const float* post_weight = nullptr, const float* pre_weight = nullptr) {
    return tm_block_norm_fwd(d, n, first, FAKE, y, gate, post_weight, pre_weight, nullptr, scale, shift, r, h, nullptr);
}

void norm_checks() {
    tm_block_norm_desc d = norm(5120);
    EXPECT(norm_fwd(nullptr, 1, 0) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 0, 0) == TM_OK);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);  // past the checks: an unknown pointer
    for (const int32_t E : {0, -8, 4, 12, 16392, INT_MAX}) {
        d = norm(E);
        EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    }
    d = norm(64, 3);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);
    d = norm(64, TM_NORM_RMS, -1);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);
    for (const float eps : {-1.f, float(INFINITY), float(NAN)}) {
        d = norm(64, TM_NORM_RMS, TM_NORM_NONE, 1, 1, 0, eps);
        EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);
    }
    d = norm(64);
    d.dtype = 7;
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_DTYPE);
    d = norm(64);
    d.stream_dtype = -1;
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_DTYPE);
    d = norm(64, TM_NORM_LAYER, TM_NORM_NONE, 0);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    d = norm(64, TM_NORM_LAYER, TM_NORM_NONE, 65536);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    // groups
    d = norm(64, TM_NORM_LAYER, TM_NORM_NONE, 1, 2, 0);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    d = norm(64, TM_NORM_LAYER, TM_NORM_NONE, 1, 3, 10);
    EXPECT(norm_fwd(&d, 30, 0) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 31, 0) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, 1, 30) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, 1, -1) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, -1, 0) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, 0, 30) == TM_OK);
    d = norm(64);
    EXPECT(norm_fwd(&d, INT_MAX, 0) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, 1, INT64_MAX) == TM_E_SHAPE);
    EXPECT(norm_fwd(&d, 1, (int64_t(1) << 30) - 1) == TM_E_ARG);
    d = norm(16384, TM_NORM_LAYER, TM_NORM_NONE, 65535, INT_MAX, 1);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    d = norm(8, TM_NORM_LAYER, TM_NORM_NONE, 1, 1 << 20, 1);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);
    d = norm(8, TM_NORM_LAYER, TM_NORM_NONE, 1, (1 << 20) + 1, 1);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    d = norm(2048, TM_NORM_LAYER, TM_NORM_NONE, 2, 1 << 19, 1);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_SHAPE);
    // which tensors go together
    d = norm(64);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, FAKE) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, FAKE, nullptr) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, nullptr) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, FAKE, FAKE_F) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, FAKE, nullptr, FAKE_F) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, FAKE, nullptr, nullptr, FAKE_F) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, FAKE, nullptr, nullptr, nullptr, FAKE_F) == TM_E_ARG);
    d = norm(64, TM_NORM_NONE);
    EXPECT(norm_fwd(&d, 1, 0, nullptr, nullptr, nullptr) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, FAKE, FAKE, FAKE) == TM_E_ARG);
    EXPECT(norm_fwd(&d, 1, 0, FAKE, FAKE, nullptr, nullptr, nullptr, nullptr, nullptr, FAKE_F) == TM_E_ARG);
    d = norm(64, TM_NORM_LAYER, TM_NORM_RMS);
    EXPECT(norm_fwd(&d, 1, 0) == TM_E_ARG);
    // the backward's
    d = norm(64);
    auto bwd = [&](int32_t n, const void* r, const void* dh, const void* dr, const void* y, void* dx, void* dy,
                   float* dgate = nullptr, const float* scale = nullptr, float* dscale = nullptr) {
        return tm_block_norm_bwd(&d, n, 0, r, dh, dr, y, nullptr, nullptr, nullptr, nullptr, scale, dx, dy, dgate, nullptr,
                                 nullptr, nullptr, dscale, nullptr, nullptr, 0, nullptr);
    };
    EXPECT(bwd(0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == TM_OK);
    EXPECT(bwd(1, nullptr, FAKE, FAKE, nullptr, FAKE, nullptr) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, nullptr, FAKE, nullptr, FAKE, nullptr) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, nullptr, nullptr, nullptr) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, FAKE, FAKE, nullptr) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, nullptr, FAKE, FAKE) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, FAKE, FAKE, FAKE, FAKE_F) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, FAKE, FAKE, FAKE, nullptr, nullptr, FAKE_F) == TM_E_ARG);
    EXPECT(bwd(1, FAKE, FAKE, nullptr, FAKE, FAKE, FAKE, nullptr, FAKE_F, FAKE_F) == TM_E_ARG);  // no workspace
    d = norm(64, TM_NORM_NONE);
    EXPECT(bwd(1, nullptr, nullptr, nullptr, FAKE, FAKE, FAKE) == TM_E_ARG);
    EXPECT(tm_block_norm_bwd_workspace(nullptr, 1, 0) == 0);
    EXPECT(tm_block_norm_bwd_workspace(&d, 0, 0) == 0);
    EXPECT(tm_block_norm_bwd_workspace(&d, 1, 0) == 3 * 64 * 4);
}

void linear_checks() {
    tm_linear_desc d = linear(5120, 5120);
    auto fwd = [&](int32_t n, int64_t first = 0) {
        return tm_linear_fwd(&d, n, first, FAKE, FAKE, nullptr, nullptr, nullptr, nullptr, FAKE, nullptr, 0, nullptr);
    };
    auto bwd = [&](int32_t n, const void* x, const void* w, const void* pre, float* dgate) {
        return tm_linear_bwd(&d, n, 0, x, w, FAKE, nullptr, pre, FAKE, FAKE, nullptr, dgate, nullptr, 0, nullptr);
    };
    EXPECT(tm_linear_fwd(nullptr, 1, 0, FAKE, FAKE, nullptr, nullptr, nullptr, nullptr, FAKE, nullptr, 0, nullptr) == TM_E_ARG);
    EXPECT(tm_linear_fwd(&d, 1, 0, nullptr, FAKE, nullptr, nullptr, nullptr, nullptr, FAKE, nullptr, 0, nullptr) == TM_E_ARG);
    EXPECT(fwd(0) == TM_OK);
    EXPECT(fwd(1) == TM_E_ARG);
    EXPECT(fwd(-1) == TM_E_SHAPE);
    EXPECT(fwd(INT_MAX) == TM_E_SHAPE);
    for (const int32_t w : {0, -8, 4, 20, (1 << 18) + 8, INT_MAX}) {
        d = linear(w, 64);
        EXPECT(fwd(1) == TM_E_SHAPE);
        d = linear(64, w);
        EXPECT(fwd(1) == TM_E_SHAPE);
    }
    d = linear(64, 64, 3);
    EXPECT(fwd(1) == TM_E_ARG);
    d = linear(64, 64);
    d.out_dtype = 2;
    EXPECT(fwd(1) == TM_E_DTYPE);
    d = linear(64, 64, 0, 1, 4, 25);
    EXPECT(fwd(100) == TM_E_ARG);
    EXPECT(fwd(101) == TM_E_SHAPE);
    EXPECT(fwd(1, 100) == TM_E_SHAPE);
    d = linear(1 << 18, 1 << 18);
    EXPECT(fwd(1 << 30) == TM_E_SHAPE);  // too many tiles
    d = linear(64, 64, TM_ACT_GELU);
    EXPECT(bwd(20, FAKE, FAKE, nullptr, nullptr) == TM_E_ARG);
    d = linear(64, 64);
    EXPECT(bwd(20, nullptr, FAKE, nullptr, nullptr) == TM_E_ARG);
    EXPECT(bwd(20, FAKE, nullptr, nullptr, nullptr) == TM_E_ARG);
    EXPECT(bwd(20, FAKE, FAKE, FAKE, FAKE_F) == TM_E_ARG);
    EXPECT(bwd(20, FAKE, FAKE, nullptr, nullptr) == TM_E_ARG);  // no workspace
    EXPECT(tm_linear_bwd_workspace(&d, 0, 0) == 0);
    EXPECT(tm_linear_bwd_workspace(nullptr, 1, 0) == 0);
    EXPECT(tm_linear_fwd_workspace(nullptr, 1) == 0);
    EXPECT(tm_linear_fwd_workspace(&d, 16) == 0);
}

// Every token of a run lies in exactly one part, that of its group.
void parts_checks() {
    struct Case { int64_t B, groups, group, n, first, want, least; };
    const Case cases[] = {{1, 1, 0, 4680, 0, 512, 8}, {2, 21, 1560, 4680, 4680, 512, 8}, {3, 5, 100, 333, 77, 512, 8},
                          {1, 40, 1, 40, 0, 512, 8},  {2, 9, 7, 50, 11, 4, 1},           {1, 3, 1 << 30, 17, 5, 512, 8},
                          {1, 1, 0, 1, 0, 512, 8},    {1, 1000, 3, 2999, 0, 16, 32}};
    for (const Case& c : cases) {
        Run r;
        EXPECT(check_run(int32_t(c.B), int32_t(c.groups), int32_t(c.group), int32_t(c.n), c.first, &r) == TM_OK);
        const tmk::RowParts p = row_parts(r, c.want, c.least);
        const tmk::TokenGroups t = token_groups(r);
        std::vector<int> seen(size_t(c.B * c.n), 0);
        EXPECT(int64_t(p.per_group) * p.rows_per_part >= p.len);
        for (int i = 0; i < p.count(); ++i) {
            // as the kernels count
            const int part = i % p.per_group, j = i / p.per_group % p.touched, b = i / p.per_group / p.touched;
            const int64_t at = int64_t(j) * p.len - p.f0, lo = at + int64_t(part) * p.rows_per_part;
            const int64_t hi = std::min(lo + p.rows_per_part, at + p.len);
            for (int64_t k = std::max<int64_t>(lo, 0); k < std::min(hi, c.n); ++k) {
                ++seen[size_t(b * c.n + k)];
                const int64_t g = c.group ? (c.first + k) / c.group : 0;
                EXPECT(p.g0 + j == g);
                EXPECT(t.g0 + t.by_group.of(int32_t(t.f0 + k)) == g);
                EXPECT(t.by_n.of(int32_t(b * c.n + k)) == b);
            }
        }
        for (const int s : seen) EXPECT(s == 1);
    }
}

// The shares of split tiles: every stage in one share, a share's stages in at most two tiles, and the merge's
// way of finding them.
void split_checks() {
    int split = 0;
    for (const int64_t M : {17, 130, 333, 600, 4680, 5376, 32760})
        for (const int64_t N : {64, 1032, 5120, 20480})
            for (const int64_t K : {8, 64, 1000, 5120, 20480}) {
                const GemmPlan p = plan_gemm(M, N, K, true);
                const int64_t tiles = p.tiles_m * p.tiles_n, rest = tiles - p.whole;
                EXPECT(p.tiles_m * p.tile >= M && p.tiles_n * p.tile >= N && p.stages * tmk::kGemmDepth >= K);
                EXPECT(rest >= 0);
                if (rest == 0) continue;
                ++split;
                const int64_t per_group = rest / p.groups, units = per_group * p.stages, W = p.shares;
                EXPECT(per_group * p.groups == rest && W >= per_group && W <= units);
                EXPECT(p.groups * W <= 256 * tmk::gemm_per_cu(p.tile));
                for (int64_t w = 0; w < W; ++w) {
                    const int64_t u0 = units * w / W, u1 = units * (w + 1) / W;
                    EXPECT(u0 < u1);
                    EXPECT((u1 - 1) / p.stages - u0 / p.stages <= 1);  // its two partial tiles
                }
                EXPECT(p.part_bytes() == size_t(2 * p.groups * W) * size_t(p.tile) * size_t(p.tile) * 4);
                for (int64_t t = 0; t < per_group; ++t) {
                    const int64_t u0 = t * p.stages, u1 = u0 + p.stages;
                    int64_t w = u0 * W / units;
                    EXPECT(units * w / W <= u0);
                    while (units * (w + 1) / W <= u0) ++w;
                    EXPECT(w < W && units * w / W <= u0);
                    int64_t covered = u0;
                    for (; w < W && units * w / W < u1; ++w) {
                        EXPECT(std::max(units * w / W, u0) == covered);
                        covered = std::min(units * (w + 1) / W, u1);
                    }
                    EXPECT(covered == u1);
                }
            }
    EXPECT(split > 20);
}

}  // namespace

int main() {
    norm_checks();
    linear_checks();
    parts_checks();
    split_checks();
    if (g_failed) {
        std::fprintf(stderr, "host block driver: %d of %d checks failed\n", g_failed, g_checks);
        return 1;
    }
    std::printf("host block driver: all checks passed (%d)\n", g_checks);
    return 0;
}
