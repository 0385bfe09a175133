// Driver of the rotary and 8-bit-cache entry points of the C ABI (include/tm.h)
// for the sanitizer build, as host_abi_driver.cpp for the others: tm_api.cpp is
// compiled with AddressSanitizer and UndefinedBehaviorSanitizer (host code only)
// into this file, the kernels come from libtm.so. Descriptor and argument checks,
// sizes and their limits, the division by multiplication that the kernels use, and
// the planner's layouts of attention calls. Exit status 0 and "host kv8 driver: all
// checks passed" when every check holds.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>

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

tm_attn_desc desc(int32_t B, int32_t H, int32_t D, int32_t T, int32_t C, int32_t R, int32_t W,
                  int32_t dtype = TM_BF16) {
    tm_attn_desc d{};
    d.batch = B;
    d.heads = H;
    d.head_dim = D;
    d.tokens_per_frame = T;
    d.chunk_frames = C;
    d.ref_frames = R;
    d.window = W;
    d.dtype = dtype;
    return d;
}

tm_rope_desc rope_desc(int32_t D = 128, int32_t frames = 21, int32_t h = 30, int32_t w = 52, int32_t pt = 22,
                       int32_t ph = 21, int32_t pw = 21, int32_t dtype = TM_BF16, float theta = 10000.f) {
    return tm_rope_desc{D, frames, h, w, pt, ph, pw, 0, dtype, theta};
}

void division_checks() {
    const uint32_t ds[] = {1, 2, 3, 5, 7, 52, 64, 1560, 2025, 3600, 65535, 65537, 1u << 20, (1u << 30) - 1, 1u << 30};
    for (const uint32_t d : ds) {
        const tmk::FastDiv f(d);
        for (int64_t k = 0; k < 2000; ++k) {
            // around the multiples of d, from both ends of the range
            for (int64_t n : {k * d - 1, k * d, k * d + 1, int64_t(INT32_MAX) - k * d, int64_t(INT32_MAX) - k}) {
                if (n < 0 || n > INT32_MAX) continue;
                if (f.of(int32_t(n)) != int32_t(n / d)) {
                    EXPECT(f.of(int32_t(n)) == int32_t(n / d));
                    return;
                }
            }
        }
        ++g_checks;
    }
}

void rope_checks() {
    tm_rope_desc r = rope_desc();
    EXPECT(tm_rope3d_table_bytes(&r) == size_t(8) * (21 * 22 + 30 * 21 + 52 * 21));
    tm_rope_desc none = rope_desc(64, 5, 2, 3, 0, 0, 0);
    EXPECT(tm_rope3d_table_bytes(&none) == 0 && tm_rope3d_table(&none, nullptr, nullptr) == TM_OK);
    const tm_rope_desc bad[] = {rope_desc(96), rope_desc(128, 0), rope_desc(128, 21, 0), rope_desc(128, 21, 30, 0),
                                rope_desc(128, 21, 30, 52, -1), rope_desc(128, 21, 30, 52, 22, 21, 22),
                                rope_desc(64), rope_desc(128, INT32_MAX, INT32_MAX, INT32_MAX),
                                rope_desc(128, INT32_MAX, 1, 1), rope_desc(128, 1 << 30, 1, 1, 64, 0, 0),
                                rope_desc(128, 21, 30, 52, INT32_MAX, INT32_MAX, INT32_MAX),
                                rope_desc(128, 21, 30, 52, 22, 21, 21, 7),
                                rope_desc(128, 21, 30, 52, 22, 21, 21, TM_BF16, 0.f),
                                rope_desc(128, 21, 30, 52, 22, 21, 21, TM_BF16, NAN),
                                rope_desc(128, 21, 30, 52, 22, 21, 21, TM_BF16, INFINITY)};
    for (const tm_rope_desc& b : bad) {
        EXPECT(tm_rope3d_table_bytes(&b) == 0);
        EXPECT(tm_rope3d_table(&b, FAKE_F, nullptr) != TM_OK);
    }
    EXPECT(tm_rope3d_table_bytes(nullptr) == 0);
    EXPECT(tm_rope3d_table(&r, nullptr, nullptr) == TM_E_ARG);
    EXPECT(tm_rope3d_table(&r, FAKE_F, nullptr) == TM_E_ARG);
    auto fwd = [&](int32_t batch, int32_t n, int64_t first, const void* q, int32_t H, const void* k, int32_t Hk) {
        return tm_rope3d_fwd(&r, FAKE_F, batch, n, first, q, H, k, Hk, FAKE, FAKE, nullptr);
    };
    EXPECT(fwd(0, 1, 0, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, 0, FAKE, 0, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, -1, 0, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, 0, FAKE, 1, FAKE, 0) == TM_E_ARG);
    EXPECT(fwd(1, 1, 0, FAKE, 1, nullptr, 1) == TM_E_ARG);
    EXPECT(fwd(INT32_MAX, 1, 0, FAKE, INT32_MAX, FAKE, INT32_MAX) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, -1, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, 21 * 1560, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, INT32_MAX, 0, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, INT64_MAX, FAKE, 1, nullptr, 0) == TM_E_SHAPE);
    EXPECT(fwd(1, 1, 21 * 1560 - 1, FAKE, 1, nullptr, 0) == TM_E_ARG);  // the pointers
    EXPECT(fwd(1, 0, 0, nullptr, 1, nullptr, 0) == TM_OK);              // nothing to do
    EXPECT(tm_rope3d_bwd(nullptr, FAKE_F, 1, 1, 0, FAKE, 1, nullptr, 0, FAKE, nullptr, nullptr) == TM_E_ARG);
}

void cache_checks() {
    tm_attn_desc d = desc(1, 40, 128, 1560, 3, 1, 1);
    EXPECT(tm_kv8_cache_tokens(&d) == 1600 + 2 * 4736);
    EXPECT(tm_kv8_cache_bytes(&d, 40) == size_t(2) * 40 * 11072 * 128 + size_t(2) * 40 * 173 * 4);
    EXPECT(tm_kv8_cache_bytes(&d, 5) == size_t(2) * 5 * 11072 * 128 + size_t(2) * 3472);  // 5 * 173 * 4 rounded up
    for (int32_t kv : {0, -1, 3, 41, INT32_MAX}) EXPECT(tm_kv8_cache_bytes(&d, kv) == 0);
    const tm_attn_desc bad[] = {desc(1, 40, 128, 1560, 3, 1, 1, TM_F32), desc(1, 40, 96, 1560, 3, 1, 1),
                                desc(1, 40, 128, 1560, 3, 1, 13), desc(0, 40, 128, 1560, 3, 1, 1),
                                desc(1, 40, 128, INT32_MAX, INT32_MAX, INT32_MAX, 12),
                                desc(1, 40, 128, 1 << 30, 1, 1, 0)};
    for (const tm_attn_desc& b : bad) {
        EXPECT(tm_kv8_cache_tokens(&b) == 0 && tm_kv8_cache_bytes(&b, 1) == 0);
        tm_kv8_cache* c = nullptr;
        EXPECT(tm_kv8_cache_create(&b, 1, FAKE, &c) != TM_OK && c == nullptr);
    }
    tm_kv8_cache* c = nullptr;
    EXPECT(tm_kv8_cache_create(&d, 40, nullptr, &c) == TM_E_ARG);
    EXPECT(tm_kv8_cache_create(&d, 40, FAKE, &c) == TM_E_ARG);
    EXPECT(tm_kv8_cache_create(&d, 40, FAKE, nullptr) == TM_E_ARG);
    tm_kv8_cache_destroy(nullptr);
    EXPECT(tm_kv8_cache_reset(nullptr) == TM_E_ARG && tm_kv8_cache_latest(nullptr) == -1);
    int32_t off = 0, n = 0;
    EXPECT(tm_kv8_cache_locate(nullptr, 0, &off, &n) == TM_E_ARG);
    EXPECT(tm_kv8_append(nullptr, 0, FAKE, FAKE, 1, nullptr) == TM_E_ARG);
    EXPECT(tm_kv8_read(nullptr, 0, FAKE, FAKE, 0, nullptr) == TM_E_ARG);
    EXPECT(tm_kv8_attn_workspace(nullptr, 0, 1) == 0);
    EXPECT(tm_kv8_attn_fwd(nullptr, FAKE, 0, 1, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_ARG);

    // a handle over memory that is not the device's: every call stops at its checks
    tm_kv8_cache fake{};
    fake.book.desc = d;
    fake.kv_heads = 8;
    fake.pool = FAKE;
    tm_kv_cache_reset(&fake.book);
    EXPECT(tm_kv8_append(&fake, 1, FAKE, FAKE, 1, nullptr) == TM_E_ORDER);
    EXPECT(tm_kv8_append(&fake, 0, FAKE, FAKE, 0, nullptr) == TM_E_SHAPE);
    EXPECT(tm_kv8_append(&fake, 0, FAKE, FAKE, 1561, nullptr) == TM_E_CAPACITY);
    EXPECT(tm_kv8_append(&fake, 0, FAKE, FAKE, 1560, nullptr) == TM_E_ARG);
    EXPECT(tm_qkv8_produce(&fake, 0, nullptr, FAKE, FAKE, nullptr, nullptr, 0.f, nullptr, nullptr, 0, FAKE, 1,
                           nullptr) == TM_E_ARG);
    EXPECT(tm_kv8_read(&fake, 0, FAKE, FAKE, 0, nullptr) == TM_E_ORDER);
    EXPECT(tm_kv8_attn_fwd(&fake, FAKE, 0, 1, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_ORDER);
    EXPECT(tm_kv8_cache_latest(&fake) == -1);
    fake.book.latest = 3;
    fake.book.ref_len = 1560;
    for (int t = 2; t <= 3; ++t) {
        fake.book.slot_chunk[(t - 1) % 2] = t;
        fake.book.slot_len[(t - 1) % 2] = t == 3 ? 77 : 4680;
    }
    EXPECT(tm_kv8_cache_locate(&fake, 3, &off, &n) == TM_OK && off == 1600 && n == 77);
    EXPECT(tm_kv8_cache_locate(&fake, 2, &off, &n) == TM_OK && off == 1600 + 4736 && n == 4680);
    EXPECT(tm_kv8_cache_locate(&fake, 1, &off, &n) == TM_E_ORDER);
    EXPECT(tm_kv8_attn_fwd(&fake, FAKE, 2, 1, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_ORDER);
    EXPECT(tm_kv8_attn_fwd(&fake, FAKE, 3, -1, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_SHAPE);
    EXPECT(tm_kv8_attn_fwd(&fake, FAKE, 3, INT32_MAX, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_SHAPE);
    EXPECT(tm_kv8_attn_fwd(&fake, nullptr, 3, 0, nullptr, 0, nullptr, nullptr, 0, nullptr) == TM_OK);
    EXPECT(tm_kv8_attn_fwd(&fake, FAKE, 3, 4, FAKE, 0, nullptr, nullptr, 0, nullptr) == TM_E_ARG);
}

// The layout of attention calls over a range of sizes: every key block is in some part, parts
// are not empty, the grid and the workspace are what the kernels index.
void plan_checks() {
    int cut = 0, few4 = 0, few8 = 0, many = 0, whole = 0;
    for (int32_t D : {64, 128})
        for (int32_t Hk : {1, 3, 8, 24, 40, 200})
            for (int32_t group : {1, 5})
                for (int32_t ref : {1, 64, 65, 1560, 14175, 100000, 3000000})
                    for (int32_t n_q : {1, 7, 33, 100, 257, 1000, 6075, 40000}) {
                        tm_kv8_cache c{};
                        c.book.desc = desc(2, Hk * group, D, 1, 128, ref, 1);
                        c.kv_heads = Hk;
                        tm_kv_cache_reset(&c.book);
                        c.book.latest = 2;
                        c.book.ref_len = ref;
                        c.book.slot_chunk[0] = 1;
                        c.book.slot_len[0] = 128;  // two full slots are one range
                        c.book.slot_chunk[1] = 2;
                        c.book.slot_len[1] = 9;
                        Kv8Geo z;
                        tmk::Kv8AttnArgs a{};
                        if (check_cache8(&c, &z) != TM_OK) {
                            EXPECT(false);
                            continue;
                        }
                        if (plan_attn8(&c, z, 2, n_q, &a) != TM_OK) {
                            EXPECT(false);
                            continue;
                        }
                        const int64_t rows = int64_t(n_q) * group, tiles = int64_t(a.n_tiles) * 2 * Hk;
                        const int64_t per = a.few ? tmk::kKv8FewRows : tmk::kTileRowsBf16;
                        int64_t blocks = 0;
                        for (int r = 0; r < a.n_ranges; ++r) {
                            EXPECT(a.range_keys[r] > 0 &&
                                   a.range_begin[r] + (a.range_keys[r] + 63) / 64 <= z.blocks);
                            blocks += (a.range_keys[r] + 63) / 64;
                        }
                        EXPECT(a.rows == rows && a.n_tiles == (rows + per - 1) / per);
                        EXPECT(a.n_kblocks == blocks && a.n_kblocks == (ref + 63) / 64 + 2 + 1);
                        EXPECT(a.n_whole >= 0 && a.n_whole <= tiles && a.parts >= 1 && a.parts <= tmk::kKv8MaxParts);
                        EXPECT(a.parts <= a.n_kblocks && (a.parts > 1) == (a.n_whole < tiles));
                        EXPECT(a.cut == 0 || (a.parts == 2 && !a.few && a.cut > 0 && a.cut < a.n_kblocks));
                        EXPECT(a.n_whole + (tiles - a.n_whole) * a.parts <= INT32_MAX);
                        const size_t ws = parts_bytes(z, a);
                        EXPECT(ws == size_t(tiles - a.n_whole) * (a.parts > 1 ? a.parts : 0) * per * (D + 2) * 4);
                        EXPECT(ws == tm_kv8_attn_workspace(&c, 2, n_q));
                        cut += a.cut > 0;
                        few4 += a.few == 4;
                        few8 += a.few == 8;
                        many += !a.few && a.parts > 1 && a.cut == 0;
                        whole += !a.few && a.parts == 1;
                    }
    EXPECT(cut > 0 && few4 > 0 && few8 > 0 && many > 0 && whole > 0);  // every layout was seen
}

}  // namespace

int main() {
    division_checks();
    rope_checks();
    cache_checks();
    plan_checks();
    std::printf("host kv8 driver: %d checks, %d failed\n", g_checks, g_failed);
    if (g_failed == 0) std::printf("host kv8 driver: all checks passed\n");
    return g_failed == 0 ? 0 : 1;
}
