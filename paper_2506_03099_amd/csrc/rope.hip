// Rotary positions with three axes (time, height, width) for gfx950.
//
// The student keeps the attention of its WAN2.1 teacher (TalkingMachines, Sec.
// 4.1), whose queries and keys carry their token's latent frame, row and column
// as rotations of pairs of their elements before the attention equation of Sec.
// 4.2. Pair i of the n_a pairs of axis a turns by pos_a * theta^(-i / n_a):
//     (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos),
// in fp32, rounded once. The rotation is orthogonal, so the backward pass is the
// rotation by the opposite angles of the incoming gradient.
//
// Bound by HBM: every element is read and written once. The angles come from a
// small table, (cos, sin) of each position of each axis and pair, formed in fp64
// (an angle of thousands of radians keeps its digits) and kept by the caller; a
// frame's rows and columns are some ten KB that stay in the L1. A lane holds 8
// pairs and takes the same 8 pairs of several heads of its token, so that the
// table is read once for them and their loads are in flight together. Measured:
// q and k of 32760 tokens with 40 heads of 128 in bf16 (1.34 GB) 233 us, 5.7 TB/s (a
// device copy of that size: 4.9 to 5.4); 6075 tokens, two streams, 10 heads of 64 in
// fp32 (62 MB) 9.5 us; one token 2.4 us, a launch.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tm_device.h"
#include "tm_internal.h"
#include "tm_rope.h"

namespace tmk {
namespace {

constexpr int kRopeThreads = 256;

// Tokens [tok0, tok0 + n) of batch element blockIdx.y, all heads of q, then all
// of k. Thread: lane g of the rows of heads s, s + S, s + 2 S, ... of a token
// (S = a.slices, at most U of them).
template <int EB, int D, bool HALVES, int U>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a) {
    constexpr int G = D / kRowElems;
    const uint32_t idx = blockIdx.x * static_cast<uint32_t>(kRopeThreads) + threadIdx.x;
    const int g = idx % G;
    const uint32_t r = idx / G;
    const int s = r % a.slices;
    const int64_t i = a.tok0 + r / a.slices;
    if (i >= a.tok_end) return;
    const int heads = a.H + a.Hk;
    const int64_t row = blockIdx.y * a.n + i;
    RowBits<EB> bits[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = s + u * a.slices;
        if (h < heads)
            bits[u] = h < a.H ? load_row<EB, D>(a.q + (row * a.H + h) * (D * EB), g)
                              : load_row<EB, D>(a.k + (row * a.Hk + (h - a.H)) * (D * EB), g);
    }
    float2 cs[8];
    load_turns<EB, D, HALVES>(a.table, a.first_token + i, g, cs);
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e].y *= a.sign;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = s + u * a.slices;
        if (h >= heads) continue;
        float x[kRowElems];
        unpack_row<EB>(bits[u], x);
        turn_row<HALVES>(x, cs);
        store_row<EB, D>(h < a.H ? a.q_out + (row * a.H + h) * (D * EB)
                                         : a.k_out + (row * a.Hk + (h - a.H)) * (D * EB), g, x);
    }
}

// (cos, sin)(pos * theta^(-i / pairs)) of positions [0, rows) and pairs, in fp64.
__global__ __launch_bounds__(kRopeThreads) void rope_table_kernel(float2* out, int64_t rows, int pairs, double log_theta) {
    const int64_t idx = blockIdx.x * static_cast<int64_t>(kRopeThreads) + threadIdx.x;
    if (idx >= rows * pairs) return;
    const int64_t pos = idx / pairs;
    const int i = static_cast<int>(idx - pos * pairs);
    const double angle = static_cast<double>(pos) * exp(-log_theta * i / pairs);
    double s, c;
    sincos(angle, &s, &c);
    out[idx] = make_float2(static_cast<float>(c), static_cast<float>(s));
}

template <int EB, int D, bool HALVES, int U>
hipError_t launch_u(RopeArgs a, hipStream_t s) {
    a.slices = (a.H + a.Hk + U - 1) / U;
    const int64_t per = static_cast<int64_t>(a.slices) * (D / kRowElems);  // threads of a token
    // Thread numbers are 32 bits wide: long runs take several launches.
    const int64_t most = (int64_t(1) << 31) / per;
    if (most < 1) return hipErrorInvalidValue;
    for (int64_t at = 0; at < a.n; at += most) {
        a.tok0 = at;
        a.tok_end = at + most < a.n ? at + most : a.n;
        const int64_t blocks = ((a.tok_end - at) * per + kRopeThreads - 1) / kRopeThreads;
        const hipError_t e = launch_with(rope_kernel<EB, D, HALVES, U>, dim3(static_cast<unsigned>(blocks), a.B),
                                         kRopeThreads, s, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int EB, int D, bool HALVES>
hipError_t launch(const RopeArgs& a, hipStream_t s) {
    // Four heads a thread once that leaves every CU its 1024 threads; few tokens are
    // bound by one thread's latency, so it takes one (one token: 2.4 us).
    const int64_t rows = static_cast<int64_t>(a.B) * a.n * (a.H + a.Hk);
    if (rows * (D / kRowElems) >= int64_t(4) * kCUs * 1024) return launch_u<EB, D, HALVES, 4>(a, s);
    return launch_u<EB, D, HALVES, 1>(a, s);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, int head_dim, int elem_bytes, bool halves, hipStream_t s) {
    if (a.B > 65535) return hipErrorInvalidValue;
#define TM_ROPE_CASE(EB_, D_)                     \
    if (elem_bytes == EB_ && head_dim == D_)      \
        return halves ? launch<EB_, D_, true>(a, s) : launch<EB_, D_, false>(a, s);
    TM_ROPE_CASE(2, 128)
    TM_ROPE_CASE(2, 64)
    TM_ROPE_CASE(4, 128)
    TM_ROPE_CASE(4, 64)
#undef TM_ROPE_CASE
    return hipErrorInvalidValue;
}

hipError_t launch_rope_table(const int64_t (&rows)[3], const int (&pairs)[3], double theta, float* out, hipStream_t s) {
    float2* at = reinterpret_cast<float2*>(out);
    for (int x = 0; x < 3; ++x) {
        const int64_t n = rows[x] * pairs[x];
        if (n == 0) continue;
        hipLaunchKernelGGL(rope_table_kernel, dim3(static_cast<unsigned>((n + kRopeThreads - 1) / kRopeThreads)),
                           dim3(kRopeThreads), 0, s, at, rows[x], pairs[x], log(theta));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        at += n;
    }
    return hipSuccess;
}

}  // namespace tmk
