// Driver of the plans behind the block norms and linear layers for the sanitizer build, with the functions
// of tm_internal.h that the kernels and their launchers themselves call. Arguments "product rows,in,out" and
// "sums batch,tokens,width,groups,group,first" are sizes of the GPU tests, which have to take every kernel variant
// between them. Exit status 0 and "host block plan driver: all checks passed" when every check holds.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include <string>
#include <vector>

#include "../../paper_2506_03099_amd/csrc/tm_api.cpp"

namespace {

int g_failed = 0;
int g_checks = 0;

#define EXPECT(cond)                                                            \
    do {                                                                        \
        ++g_checks;                                                             \
        if (!(cond)) {                                                          \
            ++g_failed;                                                         \
            std::fprintf(stderr, "FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
        }                                                                       \
    } while (0)

// Parts of a run as the kernels number them: none without a row, every token in one part of its group, a group's parts
// side by side, and as few rows a part as `want` parts allow.
void parts_checks() {
    struct Case {
        int64_t B, groups, group, n, first, want, least;
    };
    const Case cases[] = {
        {1, 21, 1560, 32760, 0, 512, 2},       // whole groups
        {1, 1, 0, 4680, 0, 256, 2},            // no groups
        {3, 5, 100, 333, 77, 512, 2},          // groups at both ends cut
        {1, 7, 1560, 4680, 4000, 256, 2},      // four groups of which two are cut
        {2, 3, 600, 700, 500, 512, 2},         // three
        {1, 2, 32760, 4680, 30420, 256, 2},    // over the border of two groups of more tokens than the run
        {1, 2, 1 << 28, 4680, (1 << 28) - 1, 256, 2},
        {1, 2, 1 << 28, 4680, (1 << 28) - 4679, 256, 2},
        {4, 2, 3000, 200, 2900, 512, 2},
        {1, 3, 1560, 1562, 1559, 512, 2},      // a token of the first, all of the second, a token of the third
        {2, 9, 7, 50, 11, 4, 2},               // more groups than parts are wanted
        {1, 40, 1, 40, 0, 512, 2},             // a token a group
        {1, 2, 1, 2, 0, 512, 2},
        {1, 1000, 3, 2999, 1, 16, 32},
        {1, 2, 4, 5, 3, 1, 32},
        {5, 3, 1000, 1, 999, 512, 2},          // a row
        {1, 5000, 200000, 1 << 29, 12345, 64, 2},  // offsets far past what a part holds
    };
    for (const Case& c : cases) {
        Run r;
        EXPECT(check_run(int32_t(c.B), int32_t(c.groups), int32_t(c.group), int32_t(c.n), c.first, &r) == TM_OK);
        const tmk::RowParts p = row_parts(r, c.want, c.least);
        const tmk::TokenGroups tg = token_groups(r);
        EXPECT(p.filled() == p.B * p.each() && p.each() > 0 && p.filled() <= p.count());
        EXPECT(p.filled() <= std::max(c.want, c.B * r.touched));
        // a group of so many rows has at most two parts more than rows / rows_per_part, so this many are enough
        const int64_t spare = c.want - 2 * c.B * r.touched;
        if (spare > 0) EXPECT(p.rows_per_part <= std::max(ceil_div(c.B * c.n, spare), c.least));
        std::vector<int32_t> group_end(size_t(c.B) * size_t(r.touched), 0);
        int64_t at = 0;
        for (int32_t i = 0; i < p.filled(); ++i) {
            int32_t b, t0, t1;
            int64_t mod;
            p.of(i, b, mod, t0, t1);
            EXPECT(b == at / c.n && t0 == at % c.n && t1 > t0 && t1 <= c.n);  // in order, and none is left out
            EXPECT(t1 - t0 <= p.rows_per_part);
            const int64_t g = c.group ? (c.first + t0) / c.group : 0;
            EXPECT((c.group ? (c.first + t1 - 1) / c.group : 0) == g && mod == b * c.groups + g);
            EXPECT(tg.row(int32_t(at)) == mod && tg.row(int32_t(at + t1 - t0 - 1)) == mod);
            int32_t i0, i1;
            p.of_group(b, int32_t(g - r.g0), i0, i1);
            EXPECT(i0 <= i && i < i1);
            group_end.at(size_t(b * r.touched + g - r.g0)) = i1;
            at += t1 - t0;
        }
        EXPECT(at == c.B * c.n);
        int32_t end = 0;
        for (const int32_t e : group_end) {  // each group's parts end where the next one's begin
            EXPECT(e > end);
            end = e;
        }
        EXPECT(end == p.filled());
    }
}

LinearBwdPlan backward_plan(int64_t rows, int64_t K, int64_t N) {
    tm_linear_desc d{1, int32_t(K), int32_t(N), TM_ACT_NONE, TM_BF16, 1, 0};
    LinearGeo g;
    EXPECT(check_linear(&d, int32_t(rows), 0, &g) == TM_OK);
    return plan_linear_bwd(g);
}

// dW sums over token rows, which lie side by side nowhere: its plan follows from the number of stages, not from
// whether the last one is whole.
void stage_checks() {
    const int64_t widths[][2] = {{1536, 2048}, {2048, 1536}, {1024, 4096}, {4096, 1024}, {1000, 1352}, {4096, 1000}, {5120, 5120}};
    for (const auto& w : widths)
        for (const int64_t stages : {5, 25, 74, 110, 512}) {
            const GemmPlan whole = backward_plan(64 * stages, w[0], w[1]).dw;
            EXPECT(whole.stages == stages);
            for (const int64_t rows : {64 * stages - 63, 64 * stages - 56, 64 * stages - 1}) {
                const GemmPlan p = backward_plan(rows, w[0], w[1]).dw;
                EXPECT(p.tile == whole.tile && p.stages == stages && p.whole == whole.whole);
                EXPECT(p.groups == whole.groups && p.shares == whole.shares);
            }
        }
}

// Shares of split tiles: each stage of each of these tiles in one share, which writes it into its first part, or its
// second where it began in the tile before; and the merge finds them.
void share_checks() {
    int split = 0;
    for (const int64_t M : {17, 130, 333, 600, 4680, 5376, 32760})
        for (const int64_t N : {64, 1032, 5120, 20480})
            for (const int64_t K : {8, 64, 1000, 5120, 20480, 1 << 30}) {
                const GemmPlan p = plan_gemm(M, N, K, true);
                const tmk::GemmArgs a = gemm_args(p, nullptr, nullptr, M, N, K, K, K, nullptr);
                const int tiles = a.tiles_m * a.tiles_n;
                if (tiles == a.whole) continue;
                ++split;
                EXPECT(a.share_begin(0) == 0 && a.share_begin(a.shares) == a.per_group() * a.stages);
                std::vector<int64_t> done(size_t(tiles), 0);  // stages of a tile that shares have taken so far
                std::vector<int> first(size_t(tiles), -1), last(size_t(tiles), -1);
                for (int c = 0; c < a.shares; ++c)
                    for (int g = 0; g < a.groups; ++g) {
                        // as a workgroup goes through its share
                        int seg = 0;
                        for (int u = a.share_begin(c), end = a.share_begin(c + 1); u < end; ++seg) {
                            const size_t t = size_t(a.split_tile(u / a.stages, g));
                            const int s0 = u % a.stages, s1 = std::min(a.stages, s0 + (end - u));
                            EXPECT(t >= size_t(a.whole) && t < size_t(tiles) && s0 < s1 && seg < 2);
                            EXPECT(done.at(t) == s0);
                            EXPECT((a.share_begin(c) < u / a.stages * a.stages ? 1 : 0) == seg);
                            EXPECT(a.share_of(u) == c && a.share_of(u + (s1 - s0) - 1) == c);
                            done.at(t) = s1;
                            if (first.at(t) < 0) first.at(t) = c;
                            last.at(t) = c;
                            u += s1 - s0;
                        }
                    }
                for (int t = a.whole; t < tiles; ++t) {
                    EXPECT(done.at(size_t(t)) == a.stages);
                    // as the merge looks them up
                    const int u0 = (t - a.whole) / a.groups * a.stages;
                    EXPECT(a.split_tile(u0 / a.stages, (t - a.whole) % a.groups) == t);
                    EXPECT(a.share_of(u0) == first.at(size_t(t)) && a.share_of(u0 + a.stages - 1) == last.at(size_t(t)));
                }
            }
    EXPECT(split > 20);
}

// The variants that sizes take.
class Variants {
    std::set<std::string> taken_;

    void product(const char* kind, const GemmPlan& p) {
        const tmk::GemmArgs a = gemm_args(p, nullptr, nullptr, 8, 8, 8, 8, 8, nullptr);
        const int wgs = tmk::gemm_workgroups(a, p.tile);
        const std::string form = std::string(kind) + " " + std::to_string(p.tile) + " ahead " + std::to_string(tmk::gemm_ahead(a, p.tile));
        if (a.whole > 0) taken_.insert(form + (a.whole > wgs ? " several" : " one"));
        if (p.tiles_m * p.tiles_n > p.whole) taken_.insert(form + " shared");
    }

public:
    void product(int64_t rows, int64_t K, int64_t N) {
        tm_linear_desc d{1, int32_t(K), int32_t(N), TM_ACT_NONE, TM_BF16, 1, 0};
        LinearGeo g;
        EXPECT(check_linear(&d, int32_t(rows), 0, &g) == TM_OK);
        const LinearBwdPlan b = plan_linear_bwd(g);
        if (rows > tmk::kFewRows) {
            product("forward", plan_gemm(rows, N, K, true));
            product("dx", b.dx);
            product("dW", b.dw);
            return;
        }
        taken_.insert(b.few ? "gradients of " + std::to_string(b.R) : std::string("gradients in 16 digits"));
        if (tiles_for_few(g)) {
            taken_.insert(rows <= 8 ? "8 rows by tiles" : "16 rows by tiles");
            return;
        }
        int pieces, waves;
        tmk::few_rows_shape(int(rows), int(N), &pieces, &waves);
        if (K / (64 * pieces) > 3 * waves)  // a wave's four runs at once
            taken_.insert(std::to_string(pieces) + " pieces, " + std::to_string(waves) + " waves");
    }

    void sums(const int64_t (&v)[6]) {
        tm_block_norm_desc d{int32_t(v[0]), int32_t(v[2]), TM_NORM_LAYER, TM_NORM_RMS, TM_BF16, TM_F32, int32_t(v[3]), int32_t(v[4]), 1e-6f};
        NormGeo g;
        EXPECT(check_norm(&d, int32_t(v[1]), v[5], &g) == TM_OK);
        plan_norm_bwd(&d, &g);
        int columns, threads;
        tmk::column_sums_shape(g.parts.filled(), d.width, &columns, &threads);
        taken_.insert("sums " + std::to_string(columns) + " x " + std::to_string(threads));
        if (g.parts.filled() > 512 && g.parts.per_group <= 4) taken_.insert("sums of groups");
    }

    void check() const {
        std::vector<std::string> all;
        for (const char* kind : {"forward ", "dx ", "dW "})
            for (const char* form : {"256 ahead 2", "128 ahead 2", "128 ahead 4", "64 ahead 2", "64 ahead 4"})
                for (const char* tiles : {" one", " several", " shared"})
                    if (std::strstr(form, "ahead 4") == nullptr || std::strcmp(tiles, " several") != 0)
                        all.push_back(std::string(kind) + form + tiles);
        for (const char* few : {"1", "2", "4"}) {
            all.push_back(std::string(few) + " pieces, 4 waves");
            all.push_back(std::string(few) + " pieces, 16 waves");
            all.push_back(std::string("gradients of ") + few);
        }
        for (const char* one : {"gradients in 16 digits", "8 rows by tiles", "16 rows by tiles", "sums 64 x 1", "sums 64 x 4", "sums 64 x 16",
                                "sums 32 x 32", "sums 16 x 64", "sums of groups"})
            all.push_back(one);
        for (const std::string& v : all) {
            ++g_checks;
            if (taken_.count(v)) continue;
            ++g_failed;
            std::fprintf(stderr, "FAILED: no size takes %s\n", v.c_str());
        }
    }
};

}  // namespace

int main(int argc, char** argv) {
    parts_checks();
    stage_checks();
    share_checks();
    if (argc > 1) {
        Variants variants;
        for (int i = 1; i + 1 < argc; i += 2) {
            int64_t v[6] = {};
            char* at = argv[i + 1];
            for (int64_t& x : v) x = std::strtoll(at + (*at == ','), &at, 10);
            if (std::strcmp(argv[i], "product") == 0)
                variants.product(v[0], v[1], v[2]);
            else
                variants.sums(v);
        }
        variants.check();
    }
    if (g_failed) {
        std::fprintf(stderr, "host block plan driver: %d of %d checks failed\n", g_failed, g_checks);
        return 1;
    }
    std::printf("host block plan driver: all checks passed (%d)\n", g_checks);
    return 0;
}
