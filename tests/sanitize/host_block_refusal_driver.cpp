// Driver of the refusals of the block norms' and linear layers' entry points for the sanitizer build: each by its
// status and its message, since the pointers are none that the HIP runtime knows and would be refused with
// TM_E_ARG as well; and calls that lack nothing get as far as that. Exit status 0 and "host block refusal driver:
// all checks passed" when every check holds.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "../../paper_2506_03099_amd/csrc/tm_api.cpp"

namespace {

int g_failed = 0;
int g_checks = 0;

#define REFUSED(call, status, message)                                                                           \
    do {                                                                                                         \
        ++g_checks;                                                                                              \
        g_err[0] = 0;                                                                                            \
        const tm_status st_ = (call);                                                                            \
        if (st_ != (status) || std::strstr(tm_last_error(), message) == nullptr) {                               \
            ++g_failed;                                                                                          \
            std::fprintf(stderr, "FAILED %s:%d: %s gave %d \"%s\"\n", __FILE__, __LINE__, #call, int(st_), tm_last_error()); \
        }                                                                                                        \
    } while (0)

const char* const PAST = "is not a pointer known to the HIP runtime";

// Aligned, non-null, and not memory the HIP runtime knows.
void* const FAKE = reinterpret_cast<void*>(uintptr_t(1) << 40);
float* const VEC = static_cast<float*>(FAKE);

struct Norm {
    tm_block_norm_desc d{1, 64, TM_NORM_LAYER, TM_NORM_NONE, TM_BF16, TM_F32, 1, 0, 1e-6f};
    int32_t n = 1;
    int64_t first = 0;
    const void *x = FAKE, *y = nullptr;
    const float *gate = nullptr, *post_weight = nullptr, *pre_weight = nullptr, *pre_bias = nullptr, *scale = nullptr, *shift = nullptr;
    void *r = nullptr, *h = FAKE;
    tm_status operator()() const {
        return tm_block_norm_fwd(&d, n, first, x, y, gate, post_weight, pre_weight, pre_bias, scale, shift, r, h, nullptr);
    }
};

struct NormBwd {
    tm_block_norm_desc d{1, 64, TM_NORM_LAYER, TM_NORM_NONE, TM_BF16, TM_F32, 1, 0, 1e-6f};
    int32_t n = 1;
    const void *r = FAKE, *dh = FAKE, *dr = nullptr, *y = nullptr;
    const float *gate = nullptr, *post_weight = nullptr, *pre_weight = nullptr, *pre_bias = nullptr, *scale = nullptr;
    void *dx = FAKE, *dy = nullptr;
    float *dgate = nullptr, *dpost_weight = nullptr, *dpre_weight = nullptr, *dpre_bias = nullptr, *dscale = nullptr, *dshift = nullptr;
    void* workspace = FAKE;
    size_t bytes = size_t(1) << 30;
    tm_status operator()() const {
        return tm_block_norm_bwd(&d, n, 0, r, dh, dr, y, gate, post_weight, pre_weight, pre_bias, scale, dx, dy, dgate, dpost_weight,
                                 dpre_weight, dpre_bias, dscale, dshift, workspace, bytes, nullptr);
    }
};

struct Linear {
    tm_linear_desc d{1, 64, 64, TM_ACT_NONE, TM_BF16, 1, 0};
    int32_t n = 1;
    int64_t first = 0;
    const void *x = FAKE, *w = FAKE;
    void* o = FAKE;
    tm_status operator()() const {
        return tm_linear_fwd(&d, n, first, x, w, nullptr, nullptr, nullptr, nullptr, o, nullptr, 0, nullptr);
    }
};

struct LinearBwd {
    tm_linear_desc d{1, 64, 64, TM_ACT_NONE, TM_BF16, 1, 0};
    int32_t n = 20;
    const void *x = FAKE, *w = FAKE, *dout = FAKE;
    const float* gate = nullptr;
    const void* pre = nullptr;
    void *dx = FAKE, *dw = FAKE;
    float *dbias = nullptr, *dgate = nullptr;
    void* workspace = FAKE;
    size_t bytes = size_t(1) << 30;
    tm_status operator()() const {
        return tm_linear_bwd(&d, n, 0, x, w, dout, gate, pre, dx, dw, dbias, dgate, workspace, bytes, nullptr);
    }
};

template <typename Call, typename Change>
Call with(const Change& change) {
    Call c;
    change(c);
    return c;
}
#define NORM(...) with<Norm>([](Norm& c) { __VA_ARGS__; })()
#define NORM_BWD(...) with<NormBwd>([](NormBwd& c) { __VA_ARGS__; })()
#define LINEAR(...) with<Linear>([](Linear& c) { __VA_ARGS__; })()
#define LINEAR_BWD(...) with<LinearBwd>([](LinearBwd& c) { __VA_ARGS__; })()

void sizes() {
    REFUSED(tm_block_norm_fwd(nullptr, 1, 0, FAKE, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, FAKE, nullptr),
            TM_E_ARG, "descriptor is NULL");
    REFUSED(tm_linear_fwd(nullptr, 1, 0, FAKE, FAKE, nullptr, nullptr, nullptr, nullptr, FAKE, nullptr, 0, nullptr), TM_E_ARG, "descriptor is NULL");
    REFUSED(NORM(), TM_E_ARG, PAST);
    REFUSED(NORM_BWD(), TM_E_ARG, PAST);
    REFUSED(LINEAR(), TM_E_ARG, PAST);
    REFUSED(LINEAR_BWD(), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.dtype = 7), TM_E_DTYPE, "neither TM_F32 nor TM_BF16");
    REFUSED(NORM(c.d.stream_dtype = -1), TM_E_DTYPE, "neither TM_F32 nor TM_BF16");
    REFUSED(LINEAR(c.d.out_dtype = 2), TM_E_DTYPE, "neither TM_F32 nor TM_BF16");
    REFUSED(NORM(c.d.width = 4), TM_E_SHAPE, "no multiple of 8");
    REFUSED(NORM(c.d.width = 12), TM_E_SHAPE, "no multiple of 8");
    REFUSED(NORM(c.d.width = 16392), TM_E_SHAPE, "no multiple of 8");
    REFUSED(NORM(c.d.width = 16384), TM_E_ARG, PAST);
    REFUSED(LINEAR(c.d.in_width = 20), TM_E_SHAPE, "no multiple of 8");
    REFUSED(LINEAR(c.d.out_width = (1 << 18) + 8), TM_E_SHAPE, "no multiple of 8");
    REFUSED(LINEAR(c.d.out_width = 1 << 18), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.pre = 3), TM_E_ARG, "unknown norm");
    REFUSED(NORM(c.d.pre = -1), TM_E_ARG, "unknown norm");
    REFUSED(NORM(c.d.post = 3; c.y = c.r = FAKE), TM_E_ARG, "unknown norm");
    REFUSED(NORM(c.d.post = -1), TM_E_ARG, "unknown norm");
    REFUSED(LINEAR(c.d.act = 3), TM_E_ARG, "unknown activation");
    REFUSED(LINEAR(c.d.act = -1), TM_E_ARG, "unknown activation");
    REFUSED(NORM(c.d.eps = -1e-30f), TM_E_ARG, "eps must be");
    REFUSED(NORM(c.d.eps = INFINITY), TM_E_ARG, "eps must be");
    REFUSED(NORM(c.d.eps = NAN), TM_E_ARG, "eps must be");
    REFUSED(NORM(c.d.eps = 0), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.batch = 0), TM_E_SHAPE, "batch must be");
    REFUSED(NORM(c.d.batch = 65536), TM_E_SHAPE, "batch must be");
    REFUSED(NORM(c.d.batch = 65535), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.groups = 0), TM_E_SHAPE, "groups must be >= 1");
    REFUSED(NORM(c.d.group_tokens = -1), TM_E_SHAPE, "groups must be >= 1");
    REFUSED(NORM(c.d.groups = 2), TM_E_SHAPE, "group_tokens 0 goes with one group");
    REFUSED(NORM(c.n = -1), TM_E_SHAPE, "n_tok must be >= 0");
    REFUSED(NORM(c.first = -1), TM_E_SHAPE, "positions must lie");
    REFUSED(NORM(c.first = INT64_MAX), TM_E_SHAPE, "positions must lie");
    REFUSED(NORM(c.n = INT_MAX), TM_E_SHAPE, "positions must lie");
    REFUSED(NORM(c.d.batch = 2; c.n = (1 << 29) + 1), TM_E_SHAPE, "more than 2^30 rows");
    REFUSED(NORM(c.d.groups = 3; c.d.group_tokens = 10; c.n = 30), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.groups = 3; c.d.group_tokens = 10; c.n = 31), TM_E_SHAPE, "lie past the 3 groups of 10");
    REFUSED(LINEAR(c.d.groups = 3; c.d.group_tokens = 10; c.first = 30), TM_E_SHAPE, "lie past the 3 groups of 10");
    REFUSED(NORM(c.d.groups = (1 << 20) + 1; c.d.group_tokens = 1; c.d.width = 8), TM_E_SHAPE, "modulations of more than");
    REFUSED(LINEAR(c.d.batch = 2; c.d.groups = 1 << 19; c.d.group_tokens = 1; c.d.out_width = 2048), TM_E_SHAPE, "modulations of more than");
    REFUSED(LINEAR(c.d.in_width = c.d.out_width = 1 << 18; c.n = 1 << 30), TM_E_SHAPE, "rows * width too large");
    REFUSED(LINEAR_BWD(c.d.in_width = c.d.out_width = 1 << 18; c.n = 1 << 30), TM_E_SHAPE, "rows * width too large");
    REFUSED(NORM(c.x = reinterpret_cast<void*>(uintptr_t(0x1008))), TM_E_ARG, "x is not 16-byte aligned");
}

void norm_sets() {
    REFUSED(NORM(c.gate = VEC), TM_E_ARG, "gate, post_weight and post need y");
    REFUSED(NORM(c.post_weight = VEC), TM_E_ARG, "gate, post_weight and post need y");
    REFUSED(NORM(c.d.post = TM_NORM_RMS), TM_E_ARG, "gate, post_weight and post need y");
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.y = c.r = FAKE; c.h = nullptr; c.pre_weight = VEC), TM_E_ARG, "need a norm before the block");
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.y = c.r = FAKE; c.h = nullptr; c.pre_bias = VEC), TM_E_ARG, "need a norm before the block");
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.y = c.r = FAKE; c.h = nullptr; c.scale = c.shift = VEC), TM_E_ARG, "need a norm before the block");
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.h = nullptr), TM_E_ARG, "nothing to do");
    REFUSED(NORM(c.scale = VEC), TM_E_ARG, "scale and shift: both or neither");
    REFUSED(NORM(c.shift = VEC), TM_E_ARG, "scale and shift: both or neither");
    REFUSED(NORM(c.y = FAKE), TM_E_ARG, "r goes with y");
    REFUSED(NORM(c.r = FAKE), TM_E_ARG, "r goes with y");
    REFUSED(NORM(c.h = nullptr), TM_E_ARG, "h goes with a norm");
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.y = c.r = FAKE), TM_E_ARG, "h goes with a norm");
    REFUSED(NORM(c.x = nullptr), TM_E_ARG, "x is NULL");
    REFUSED(NORM(c.y = c.r = FAKE; c.d.post = TM_NORM_RMS; c.gate = c.post_weight = c.pre_weight = c.pre_bias = c.scale = c.shift = VEC), TM_E_ARG, PAST);
    REFUSED(NORM(c.d.pre = TM_NORM_NONE; c.y = c.r = FAKE; c.h = nullptr; c.gate = VEC), TM_E_ARG, PAST);

    REFUSED(NORM_BWD(c.gate = VEC), TM_E_ARG, "gate, post_weight and post need y");
    REFUSED(NORM_BWD(c.d.pre = TM_NORM_NONE; c.dr = c.y = c.dy = FAKE; c.r = c.dh = nullptr; c.scale = VEC), TM_E_ARG, "need a norm before the block");
    REFUSED(NORM_BWD(c.r = nullptr), TM_E_ARG, "r and dh go with");
    REFUSED(NORM_BWD(c.dh = nullptr), TM_E_ARG, "r and dh go with");
    REFUSED(NORM_BWD(c.d.pre = TM_NORM_NONE; c.dr = c.y = c.dy = FAKE; c.dh = nullptr), TM_E_ARG, "r and dh go with");
    REFUSED(NORM_BWD(c.d.pre = TM_NORM_NONE; c.dr = c.y = c.dy = FAKE; c.r = nullptr), TM_E_ARG, "r and dh go with");
    REFUSED(NORM_BWD(c.d.pre = TM_NORM_NONE; c.y = c.dy = FAKE; c.r = c.dh = nullptr), TM_E_ARG, "dr is NULL");
    REFUSED(NORM_BWD(c.dx = nullptr), TM_E_ARG, "dx is NULL");
    REFUSED(NORM_BWD(c.y = FAKE), TM_E_ARG, "dy goes with y");
    REFUSED(NORM_BWD(c.dy = FAKE), TM_E_ARG, "dy goes with y");
    REFUSED(NORM_BWD(c.y = c.dy = FAKE; c.dgate = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.y = c.dy = FAKE; c.dpost_weight = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.dpre_weight = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.dpre_bias = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.dscale = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.dshift = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.scale = c.dshift = VEC; c.workspace = nullptr), TM_E_ARG, "workspace of 768 bytes needed");
    REFUSED(NORM_BWD(c.scale = c.dshift = VEC; c.bytes = 767), TM_E_ARG, "workspace of 768 bytes needed");
    REFUSED(NORM_BWD(c.scale = c.dshift = VEC; c.bytes = 768), TM_E_ARG, PAST);
    REFUSED(NORM_BWD(c.scale = VEC; c.workspace = nullptr), TM_E_ARG, PAST);  // no vector's gradient: none is needed
    REFUSED(NORM_BWD(c.n = 0; c.dpre_bias = VEC), TM_E_ARG, "a vector that is not there");
    REFUSED(NORM_BWD(c.n = 0; c.pre_bias = c.dpre_bias = VEC), TM_E_ARG, PAST);
}

void linear_sets() {
    REFUSED(LINEAR(c.x = nullptr), TM_E_ARG, "x, weight or o is NULL");
    REFUSED(LINEAR(c.w = nullptr), TM_E_ARG, "x, weight or o is NULL");
    REFUSED(LINEAR(c.o = nullptr), TM_E_ARG, "x, weight or o is NULL");
    REFUSED(LINEAR_BWD(c.pre = FAKE; c.dgate = VEC), TM_E_ARG, "dgate without gate");
    REFUSED(LINEAR_BWD(c.dout = nullptr), TM_E_ARG, "dout is NULL");
    REFUSED(LINEAR_BWD(c.w = nullptr), TM_E_ARG, "dx needs weight");
    REFUSED(LINEAR_BWD(c.x = nullptr), TM_E_ARG, "dweight needs x");
    REFUSED(LINEAR_BWD(c.d.act = TM_ACT_GELU), TM_E_ARG, "an activation and dgate need pre");
    REFUSED(LINEAR_BWD(c.gate = c.dgate = VEC), TM_E_ARG, "an activation and dgate need pre");
    REFUSED(LINEAR_BWD(c.workspace = nullptr), TM_E_ARG, "bytes needed");
    REFUSED(LINEAR_BWD(c.bytes = tm_linear_bwd_workspace(&c.d, c.n, 0) - 1), TM_E_ARG, "bytes needed");
    REFUSED(LINEAR_BWD(c.bytes = tm_linear_bwd_workspace(&c.d, c.n, 0)), TM_E_ARG, PAST);
    REFUSED(LINEAR_BWD(c.dx = nullptr; c.w = nullptr), TM_E_ARG, PAST);
    REFUSED(LINEAR_BWD(c.dw = nullptr; c.x = nullptr), TM_E_ARG, PAST);
    REFUSED(LINEAR_BWD(c.gate = c.dgate = VEC; c.pre = FAKE), TM_E_ARG, PAST);
}

}  // namespace

int main() {
    sizes();
    norm_sets();
    linear_sets();
    if (g_failed) {
        std::fprintf(stderr, "host block refusal driver: %d of %d checks failed\n", g_failed, g_checks);
        return 1;
    }
    std::printf("host block refusal driver: all checks passed (%d)\n", g_checks);
    return 0;
}
