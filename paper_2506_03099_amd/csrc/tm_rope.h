// Device-side helpers of the rotary positions (rope.hip) and of the producer of
// the 8-bit cache, which rotates keys and queries on their way (kv8_cache.hip):
// (cos, sin) of a token's pairs, and the rotation and normalisation of a row
// held by a few lanes. Not part of the public ABI.
//
// A row of D elements is held by D / 16 consecutive lanes, 16 elements each, in runs
// of 16 bytes: run i of lane g is the g-th 16 bytes of the row's i-th part of EB (2
// in bf16, 4 in fp32), so that a wave's load or store of a run touches whole lines
// (with a lane's 16 elements in one piece, every instruction touched 16 bytes of each
// 32 or 64: rotating 1.34 GB took 444 us). Pairs of neighbours lie in a run; the
// halves of a row are its first and second half of the runs. So element e of the lane
// pairs with e ^ 1, or with e + 8.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tm_device.h"
#include "tm_internal.h"

namespace tmk {

constexpr int kRowElems = 16;  // elements of a row per lane

// Element (of the row) of the first of lane g's elements 16 i / EB .. of run i.
template <int EB, int D>
__device__ __forceinline__ int run_of(int g, int i) {
    return i * (D / EB) + (16 / EB) * g;
}
// The pair (of the row's D / 2) that the lane's pair e (of 8) is.
template <int EB, int D, bool HALVES>
__device__ __forceinline__ int pair_of(int g, int e) {
    constexpr int N = 16 / EB;  // elements of a run
    return HALVES ? run_of<EB, D>(g, e / N) + e % N : (run_of<EB, D>(g, 2 * e / N) + 2 * e % N) / 2;
}

// A lane's 16 elements of the row at `row`, in fp32. EB: bytes per element.
template <int EB>
struct RowBits {
    u32x4_t v[EB];  // EB * 16 bytes
};
template <int EB, int D>
__device__ __forceinline__ RowBits<EB> load_row(const unsigned char* row, int g) {
    RowBits<EB> r;
#pragma unroll
    for (int i = 0; i < EB; ++i) r.v[i] = *reinterpret_cast<const u32x4_t*>(row + run_of<EB, D>(g, i) * EB);
    return r;
}
template <int EB>
__device__ __forceinline__ void unpack_row(const RowBits<EB>& r, float (&x)[kRowElems]) {
#pragma unroll
    for (int i = 0; i < EB; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (EB == 4) {
                x[4 * i + w] = __uint_as_float(r.v[i][w]);
            } else {
                x[8 * i + 2 * w] = __uint_as_float(r.v[i][w] << 16);
                x[8 * i + 2 * w + 1] = __uint_as_float(r.v[i][w] & 0xFFFF0000u);
            }
        }
}
// x rounded (nearest even) to the element type, through the L2.
template <int EB, int D>
__device__ __forceinline__ void store_row(unsigned char* row, int g, const float (&x)[kRowElems]) {
#pragma unroll
    for (int i = 0; i < EB; ++i) {
        u32x4_t v;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (EB == 4) {
                v[w] = __float_as_uint(x[4 * i + w]);
            } else {
                const bf16x2_t p{static_cast<__bf16>(x[8 * i + 2 * w]), static_cast<__bf16>(x[8 * i + 2 * w + 1])};
                v[w] = __builtin_bit_cast(uint32_t, p);
            }
        }
        store16_through(row + run_of<EB, D>(g, i) * EB, v);
    }
}

// (cos, sin) of lane g's 8 pairs of the token at position `pos`; (1, 0) of the
// pairs that no axis turns.
template <int EB, int D, bool HALVES>
__device__ __forceinline__ void load_turns(const RopeTable& t, int64_t pos, int g, float2 (&cs)[8]) {
    const int p = static_cast<int>(pos);  // below frames * frame_tokens <= 2^30
    const int f = t.by_frame.of(p), j = p - f * t.frame_tokens;
    const int y = t.by_w.of(j), x = j - y * t.grid_w;
    // pair i of the row is entry i of these, in its axis' span
    const int end_t = t.pairs_t, end_h = end_t + t.pairs_h, end_w = end_h + t.pairs_w;
    const int at = f * t.pairs_t, ay = t.first_h + y * t.pairs_h - end_t, ax = t.first_w + x * t.pairs_w - end_h;
    const bool all = end_w == D / 2;
    if (end_w == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = make_float2(1.f, 0.f);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = pair_of<EB, D, HALVES>(g, e);
        const int entry = (i < end_t ? at : i < end_h ? ay : ax) + i;
        // (an entry that exists for a pair that no axis turns)
        const uint32_t off = static_cast<uint32_t>(all || i < end_w ? entry : 0) * 8u;
        cs[e] = *reinterpret_cast<const float2*>(reinterpret_cast<const char*>(t.table) + off);
    }
    if (!all) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (pair_of<EB, D, HALVES>(g, e) >= end_w) cs[e] = make_float2(1.f, 0.f);
    }
}

// (x0, x1) -> (x0 c - x1 s, x0 s + x1 c) for the lane's 8 pairs.
template <bool HALVES>
__device__ __forceinline__ void turn_row(float (&x)[kRowElems], const float2 (&cs)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = HALVES ? e : 2 * e, j = HALVES ? e + 8 : 2 * e + 1;
        const float a = x[i], b = x[j];
        x[i] = fmaf(a, cs[e].x, -(b * cs[e].y));
        x[j] = fmaf(a, cs[e].y, b * cs[e].x);
    }
}

}  // namespace tmk
