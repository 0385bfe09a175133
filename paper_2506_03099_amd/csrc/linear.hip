// Linear layers with bias, activation, gate and residual for gfx950, forward and backward.
//
// The student keeps the blocks of its WAN2.1 teacher (TalkingMachines, Sec. 4.1): projections around the attention and
// a feed-forward layer, gated by frame into the residual stream.
//     z = x W^T + bias,  o = residual + gate * act(z);
//     dz = dout gate act'(z),  dx = dz W,  dW = dz^T x,  dbias = sums of dz,  dgate = sums of dout act(z).
// The three products differ in what lies side by side in memory: k of both operands (x W^T), k of the first (dz W), of
// neither (dz^T x). One kernel takes all, with transposing LDS reads where k is not side by side.
//
// Bound by the matrix cores from a few hundred rows on, by HBM (the bytes of W) below. Measured, with their
// epilogues: 4680 x 5120 x 20480, GELU, 781 us (1257 TFLOP/s, matrix cores busy for 76% of the cycles at 1.53 GHz,
// where power holds the clock); 4680 x 20480 x 5120, gated into an fp32 stream, 777 us (82%); dx and dW of 32760 x 5120 x
// 5120 1262 and 1272 us (1350 TFLOP/s); 130 rows of 5120 x 5120 24 us; one row of 5120 x 20480 32 us (6.6 TB/s).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "tm_device.h"
#include "tm_internal.h"

namespace tmk {
namespace {

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8_t;
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;

// ---------------------------------------------------------------------------
// An element's way from the sum of its products to the output
// ---------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
}

// gelu(z) = z sigmoid(2 c (z + a z^3)), c = sqrt(2 / pi), a = 0.044715: the tanh form, (1 + tanh u) / 2 = sigmoid(2 u).
constexpr float kGelu2C = 1.5957691216057308f, kGeluA = 0.044715f;
template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == kActGelu) {
        constexpr float k1 = -1.4426950408889634f * kGelu2C, k3 = k1 * kGeluA;
        return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * fmaf(k3, z * z, k1)));
    }
    if (ACT == kActSilu) return z * sigmoid(z);
    return z;
}

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(p), hi = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = lo[e];
        x[4 + e] = hi[e];
    }
}
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
    const bf16x8_t v = *reinterpret_cast<const bf16x8_t*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(v[e]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
    bf16x8_t v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(x[e]);
    *reinterpret_cast<bf16x8_t*>(p) = v;
}

// Eight neighbours at element `at` of the output: z holds the sums of products plus bias, g the gate, r the
// residual (which the caller loads, well ahead).
template <int ACT, bool F32>
__device__ __forceinline__ void finish8(const LinearEpilogue& ep, int64_t at, float (&z)[8], const float (&g)[8], const float (&r)[8]) {
    if (ep.pre != nullptr) store8(static_cast<__bf16*>(ep.pre) + at, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = activate<ACT>(z[e]);
    if (ep.gate != nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] *= g[e];
    }
    if (ep.residual != nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] += r[e];
    }
    if (F32)
        store8(static_cast<float*>(ep.o) + at, z);
    else
        store8(static_cast<__bf16*>(ep.o) + at, z);
}
template <bool F32>
__device__ __forceinline__ void load_residual(const LinearEpilogue& ep, int64_t at, float (&r)[8]) {
    if (F32)
        load8(static_cast<const float*>(ep.residual) + at, r);
    else
        load8(static_cast<const __bf16*>(ep.residual) + at, r);
}

// body(activation, whether the output is fp32) with both known to the compiler
template <typename Body>
__device__ __forceinline__ void by_kind(const LinearEpilogue& ep, const Body& body) {
    auto typed = [&](auto act) __attribute__((always_inline)) {
        if (ep.o_f32)
            body(act, std::true_type{});
        else
            body(act, std::false_type{});
    };
    if (ep.act == kActGelu)
        typed(std::integral_constant<int, kActGelu>{});
    else if (ep.act == kActSilu)
        typed(std::integral_constant<int, kActSilu>{});
    else
        typed(std::integral_constant<int, kActNone>{});
}

// ---------------------------------------------------------------------------
// The matrix product
// ---------------------------------------------------------------------------
// Why these tiles: a wave's 128 x 128 sums (16 MFMAs of 32x32x16 a k-step from 8 operands) take its SIMD's 256
// accumulation registers and ask 64 KB of LDS reads and 32 KB of writes per 32 k of a workgroup, 3/4 of what LDS moves
// in the MFMAs' time; 8 waves of 128 x 64 would ask 96 + 32 KB. So one wave a SIMD hides everything
// itself: operands are read a k-step ahead, in an order that is fixed (sched_barrier), loads a stage and more.
// Stages are 64 k deep since a row's 128 bytes are a line: at 32 k (64 bytes) the loads of 4680 x 5120 x
// 20480 kept the L2 busy for longer than the MFMAs (951 us, at 64 831). Smaller products take tiles of 128 (LDS
// reads bound them: 768 cycles a stage for 512 of MFMAs) or 64 (the reads' latency: 0.45 us a stage), which fill the CUs
// (130 rows, 5120 x 5120: 22 us; 1000 x 1000 x 1000: 8.7 us in tiles of 64, 12.3 of 128).

// One operand's part of a stage, T rows (its m or n) by 64 k, 128 * T bytes, in LDS.
// k side by side: rows of 128 bytes, 16-byte chunk c of row r at c ^ (r >> 1) % 8, so that the 16 rows that
// one cycle of a read covers lie in 16 different bank groups. A lane's operand of the MFMA, 8 k, is a chunk.
// TRANS: rows of one k and T elements, chunk c of row k at c ^ 4 (k % 4) (T = 64: c ^ 4 (k / 2 % 2)), so that the 4 rows
// by 64 bytes of a cycle of the transposing read lie apart. A lane's operand is two of these reads, 4 k each.
template <int T, bool TRANS>
struct Tile {
    static constexpr int kBytes = 2 * kGemmDepth * T;
    static constexpr int kLoads = kBytes / 4096;    // 1-KB direct loads per wave
    static constexpr int kChunks = TRANS ? T / 8 : kGemmDepth / 8;  // of a row
    uint32_t voff[kLoads];

    static __device__ __forceinline__ int swizzle(int row) {
        return !TRANS ? (row >> 1) & 7 : T == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
    }

    // Byte offsets in memory, from the stage's first element, of the chunks that this lane brings;
    // `rows`: of m (n) that exist from the tile's first one on. Past them the last ones come again.
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int rows) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int ch = (i * 4 + wave) * 64 + lane;
            const int row = ch / kChunks, c = (ch % kChunks) ^ swizzle(row);
            if (TRANS)
                voff[i] = static_cast<uint32_t>(row * ld + min(c * 8, rows - 8) * 2);
            else
                voff[i] = static_cast<uint32_t>(min(row, rows - 1) * ld + c * 16);
        }
    }

    // The stage of which only `left` < 64 k exist: direct loads in the lanes that have some (the others' 16 bytes of
    // LDS are left alone by them), zeros written in the others.
    __device__ __forceinline__ void load_rest(const void* base, lds_u8* lds, uint32_t lds_at, int wave, int lane, int left) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int ch = (i * 4 + wave) * 64 + lane;
            const int row = ch / kChunks, c = (ch % kChunks) ^ swizzle(row);
            if ((TRANS ? row : c * 8) < left)
                lds_dma16(base, voff[i], lds_at + (i * 4 + wave) * 1024);
            else
                *(lds_f32x4_t*)(lds + ch * 16) = f32x4_t{};
        }
    }

    // LDS offset of a lane's operand of rows [first, + 32), k-step 0. `perm`: lane l brings row k_perm(l), so
    // that 8 registers of the result in a row are 8 neighbours (of the transposing read's columns, the four
    // that each address stands for change places).
    static __device__ __forceinline__ uint32_t frag0(int first, int lane, bool perm) {
        const int l32 = lane & 31, hw = lane >> 5;
        if (!TRANS) {
            const int row = perm ? k_perm(l32) : l32;
            return (first + row) * (2 * kGemmDepth) + ((hw ^ swizzle(row)) << 4);
        }
        const int grp = lane >> 4, gi = lane & 15, k = 8 * hw + (gi >> 2);
        const int four = perm ? 2 * (gi & 1) + ((gi >> 1) & 1) : gi & 3;
        return k * (2 * T) + ((first * 2) ^ (swizzle(k) << 4)) + (2 * (grp & 1) + (four >> 1)) * 16 + (four & 1) * 8;
    }
    static __device__ __forceinline__ bf16x8_t frag(const lds_u8* lds, uint32_t at0, int i, int kk) {
        if (!TRANS) return *(const lds_bf16x8_t*)(lds + (at0 ^ (kk << 5)) + i * 32 * (2 * kGemmDepth));
        const lds_u8* p = lds + (at0 ^ (i << 6)) + kk * 16 * (2 * T);
        const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)p);
        const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(p + 4 * (2 * T)));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

template <int N>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The first row and column of tile t: tiles go in bands of 8 rows of tiles, so that those at work at one time
// share rows and columns.
__device__ __forceinline__ void tile_at(const GemmArgs& a, int t, int tile, int& m0, int& n0) {
    constexpr int BAND = 8;
    const int per = BAND * a.tiles_n, band = t / per, in = t % per;
    const int high = min(BAND, a.tiles_m - band * BAND);
    m0 = (band * BAND + in % high) * tile;
    n0 = in / high * tile;
}

// FULL: with all of the epilogue; else the sums are the output. Loads run AHEAD stages ahead of the MFMAs: 2, so
// that LDS holds 1 workgroup of tiles of 256, 2 of 128 or 4 of 64, or 4, since a smaller tile's workgroup that has a
// CU for itself waits for loads otherwise (512 rows, 5120 x 5120, 160 tiles of 128: 40.8 us with 2, 35.2 with 4).
template <int BT, bool AT, bool BTR, bool FULL, int AHEAD>
__global__ __launch_bounds__(256, gemm_per_cu(BT, AHEAD)) void gemm_kernel(const GemmArgs a) {
    constexpr int WT = BT / 2;      // a wave's rows and columns
    constexpr int F = WT / 32;      // its 32-wide blocks, either way
    using TA = Tile<BT, AT>;
    using TB = Tile<BT, BTR>;
    constexpr int SLOT = TA::kBytes;
    constexpr int LOADS = TA::kLoads, HALF = LOADS / 2;
    constexpr int kSlots = 2 * AHEAD + 1;  // operands' parts of stages in LDS
    static_assert(TB::kBytes == SLOT && TB::kLoads == LOADS, "both operands' parts take one slot");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kSlots * SLOT];
    lds_u8* const L = (lds_u8*)smem;
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(L));
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave & 1) * WT, wn = (wave >> 1) * WT;
    const uint32_t fa = TA::frag0(wm, lane, false), fb = TB::frag0(wn, lane, true);
    const int rest = a.K % kGemmDepth;

    // What a workgroup does, one after the other: whole tiles, those of its XCD dealt out to its XCD's
    // workgroups, then its share of the split ones' stages (of at most two tiles).
    struct Work {
        int m0, n0, s0, s1;
        float* part;
    };
    const int per_xcd = a.whole / 8, over = a.whole % 8, xcd = blockIdx.x % 8;
    const int first = xcd * per_xcd + min(xcd, over), end = first + per_xcd + (xcd < over ? 1 : 0);
    const int stride = (static_cast<int>(gridDim.x) - xcd + 7) / 8;
    int id = first + static_cast<int>(blockIdx.x) / 8, seg = 0;
    int u = 0, u_end = 0, group = 0, slot2 = 0;
    if (static_cast<int>(blockIdx.x) < a.groups * a.shares) {
        const int l = xcd_logical_id(blockIdx.x, a.groups * a.shares), c = l / a.groups;
        group = l % a.groups;
        slot2 = 2 * l;
        u = a.share_begin(c);
        u_end = a.share_begin(c + 1);
    }
    auto next_work = [&](Work& w) __attribute__((always_inline)) {
        int t;
        if (id < end) {
            t = id;
            id += stride;
            w.s0 = 0;
            w.s1 = a.stages;
            w.part = nullptr;
        } else if (u < u_end) {
            t = a.split_tile(u / a.stages, group);
            w.s0 = u % a.stages;
            w.s1 = min(a.stages, w.s0 + (u_end - u));
            w.part = a.part + static_cast<int64_t>(slot2 + seg) * (BT * BT);
            u += w.s1 - w.s0;
            ++seg;
        } else {
            return false;
        }
        tile_at(a, t, BT, w.m0, w.n0);
        return true;
    };

    // stage 0 is what K leaves over 64, if anything, so that all later ones are whole
    auto first_k = [&](int s) __attribute__((always_inline)) {
        return static_cast<int64_t>(rest ? (s == 0 ? a.K - rest : (s - 1) * kGemmDepth) : s * kGemmDepth);
    };
    auto base_a = [&](const Work& w, int s) __attribute__((always_inline)) {
        const int64_t k = first_k(s);
        return uniform_ptr(a.a + (AT ? k * a.lda + w.m0 * int64_t(2) : w.m0 * a.lda + k * 2));
    };
    auto base_b = [&](const Work& w, int s) __attribute__((always_inline)) {
        const int64_t k = first_k(s);
        return uniform_ptr(a.b + (BTR ? k * a.ldb + w.n0 * int64_t(2) : w.n0 * a.ldb + k * 2));
    };
    TA ta;
    TB tb;
    // load j of an operand's part from p into the slot at `slot`
    auto issue = [&](bool is_a, const void* p, uint32_t slot, int j) __attribute__((always_inline)) {
        lds_dma16(p, is_a ? ta.voff[j] : tb.voff[j], lds_base + slot + (j * 4 + wave) * 1024);
    };
    auto ahead = [](uint32_t slot, int by) __attribute__((always_inline)) {
        const uint32_t x = slot + by * SLOT;
        return x >= kSlots * SLOT ? x - kSlots * SLOT : x;
    };
    // The first loads of a tile: A and B of its first stages.
    auto begin = [&](const Work& w) __attribute__((always_inline)) {
        const int lane = fresh_thread_index() & 63;  // (what follows from it is not kept from tile to tile)
        ta.init(wave, lane, a.lda, a.M - w.m0);
        tb.init(wave, lane, a.ldb, a.N - w.n0);
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
            if (p >= w.s1 - w.s0) break;
            const void *pa = base_a(w, w.s0 + p), *pb = base_b(w, w.s0 + p);
            if (p == 0 && rest != 0 && w.s0 == 0) {
                ta.load_rest(pa, L, lds_base, wave, lane, rest);
                tb.load_rest(pb, L + SLOT, lds_base + SLOT, wave, lane, rest);
                continue;
            }
#pragma unroll
            for (int j = 0; j < LOADS; ++j) issue(true, pa, 2 * p * SLOT, j);
#pragma unroll
            for (int j = 0; j < LOADS; ++j) issue(false, pb, (2 * p + 1) * SLOT, j);
        }
    };
    // Waits until all but the last `left` stages' loads (and MORE later operations) are through, and for the
    // other waves.
    auto wait_but = [&](auto more, int left) __attribute__((always_inline)) {
        constexpr int MORE = decltype(more)::value;
        static_assert(2 * (AHEAD - 1) * LOADS + MORE < 64 && AHEAD <= 4, "s_waitcnt counts to 63");
        if (AHEAD > 3 && left >= 3)
            wait_and_meet<(AHEAD > 3 ? 6 : 0) * LOADS + MORE>();
        else if (AHEAD > 2 && left == 2)
            wait_and_meet<(AHEAD > 2 ? 4 : 0) * LOADS + MORE>();
        else if (left >= 1)
            wait_and_meet<2 * LOADS + MORE>();
        else
            wait_and_meet<MORE>();
    };

    f32x16_t acc[F][F];
    // a wave's operands of two k-steps; operand f: A's first block, B's blocks, A's others
    bf16x8_t af[2][F], bf[2][F];
    auto read = [&](const lds_u8* pa, const lds_u8* pb, int kk, int f) __attribute__((always_inline)) {
        if (f == 0)
            af[kk & 1][0] = TA::frag(pa, fa, 0, kk);
        else if (f <= F)
            bf[kk & 1][f - 1] = TB::frag(pb, fb, f - 1, kk);
        else
            af[kk & 1][f - F] = TA::frag(pa, fa, f - F, kk);
    };
    // Stage s, A in the slot at `at`, B in the one behind it: the MFMAs of its four k-steps, under those of
    // each the reads of the next one, and loads. Near the end of the third one, when the
    // wave's last reads of the stage are through, the wait for the next stage; its slots are free behind it.
    // Loads: A of s + AHEAD under the first two k-steps, B under the last, all at once, since it has the shorter
    // time until it is waited for.
    auto stage = [&](auto have1, auto have2, const Work& w, int s, uint32_t at) __attribute__((always_inline)) {
        constexpr bool ONE = decltype(have1)::value, TWO = decltype(have2)::value;
        const void *pa2 = nullptr, *pb2 = nullptr;
        if (TWO) {
            pa2 = base_a(w, s + AHEAD);
            pb2 = base_b(w, s + AHEAD);
        }
        const uint32_t a1 = ahead(at, 2), b1 = ahead(at, 3), a2 = ahead(at, 2 * AHEAD);
        constexpr int M = F * F;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            auto load = [&](int j) __attribute__((always_inline)) {
                if (kk == 3 && TWO) issue(false, pb2, at, j);
                if (kk == 0 && TWO) issue(true, pa2, a2, j);
                if (kk == 1 && TWO) issue(true, pa2, a2, HALF + j);
            };
            // (behind the last stage there is none to read of)
            auto next_read = [&](const lds_u8* qa, const lds_u8* qb, int of, int f) __attribute__((always_inline)) {
                if (of < 3 || ONE) read(qa, qb, (of + 1) & 3, f);
            };
            const lds_u8* pa = L + (kk == 3 ? a1 : at);
            const lds_u8* pbk = L + (kk == 3 ? b1 : ahead(at, 1));
#pragma unroll
            for (int m = 0; m < M; ++m) {
                acc[m / F][m % F] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[kk & 1][m % F], af[kk & 1][m / F], acc[m / F][m % F], 0, 0, 0);
                if (F == 4) {
                    if (kk == 2) {
                        if (m % 4 != 3 && m / 4 * 3 + m % 4 < 2 * F) read(pa, pbk, kk + 1, m / 4 * 3 + m % 4);
                    } else {
                        if (m % 2 == 0) next_read(pa, pbk, kk, m / 2);
                        if (kk == 3 && m % 2 == 1) load(m / 2);
                        if (kk < 2 && m % 4 == 1) load(m / 4);
                    }
                } else if (F == 1) {
                    next_read(pa, pbk, kk, 0);
                    next_read(pa, pbk, kk, 1);
                    load(0);
                    if (kk == 3) load(1);
                } else if (kk == 2) {
                    if (m < F) {
                        read(pa, pbk, kk + 1, 2 * m);
                        read(pa, pbk, kk + 1, 2 * m + 1);
                    }
                } else {
                    next_read(pa, pbk, kk, m);
                    if (kk == 3) load(m);
                    if (kk < 2 && m % 2 == 1) load(m / 2);
                }
                if (kk == 2 && m == (F == 4 ? 13 : F == 2 ? 2 : 0)) {
                    if (TWO)
                        wait_and_meet<(2 * AHEAD - 3) * LOADS>();
                    else
                        wait_but(std::integral_constant<int, 0>{}, w.s1 - 2 - s);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    // A tile's sums are read where they are used: the compiler would copy many of them at once, and spill them.
    auto here = [&](f32x16_t& x) __attribute__((always_inline)) {
        if (BT == 256)
            asm volatile("" : "+a"(x));
        else
            asm volatile("" : "+v"(x));
    };
    // Register 8 h + e of acc[i][j]: row wm + 32 i + l32, column wn + 32 j + 16 h + 8 hw + e (by B's order of
    // rows in the MFMA): a lane has 8 neighbours, the wave's store 32 bytes of each of 32 rows, and nothing goes
    // through LDS, where the next tile's first loads arrive meanwhile.
    auto finish = [&](const Work& w) __attribute__((always_inline)) {
        const int lane = fresh_thread_index() & 63, l32 = lane & 31, hw = lane >> 5;
        const int row0 = w.m0 + wm + l32, col0 = w.n0 + wn + 8 * hw;
        if (w.part != nullptr) {
            float* out = w.part + (wm + l32) * BT + wn + 8 * hw;
#pragma unroll
            for (int i = 0; i < F; ++i) {
                if (row0 + 32 * i >= a.M) break;
#pragma unroll
                for (int j = 0; j < 2 * F; ++j) {
                    float z[8];
                    if (j % 2 == 0) here(acc[i][j / 2]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = acc[i][j / 2][8 * (j % 2) + e];
                    store8(out + i * 32 * BT + 16 * j, z);
                }
            }
            return;
        }
        if (!FULL) {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                if (row0 + 32 * i >= a.M) break;
                const int64_t at = static_cast<int64_t>(row0 + 32 * i) * a.N + col0;
#pragma unroll
                for (int j = 0; j < 2 * F; ++j) {
                    if (col0 + 16 * j >= a.N) break;
                    float z[8];
                    if (j % 2 == 0) here(acc[i][j / 2]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = acc[i][j / 2][8 * (j % 2) + e];
                    if (a.ep.o_f32)
                        store8(static_cast<float*>(a.ep.o) + at + 16 * j, z);
                    else
                        store8(static_cast<__bf16*>(a.ep.o) + at + 16 * j, z);
                }
            }
            return;
        }
        by_kind(a.ep, [&](auto act, auto f32) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int row = row0 + 32 * i;
                if (row >= a.M) break;
                const int64_t at = static_cast<int64_t>(row) * a.N + col0;
                // gate and residual of a row of blocks at once
                constexpr bool F32 = decltype(f32)::value;
                float g[2 * F][8], r[2 * F][8];
                if (a.ep.gate != nullptr) {
                    const int64_t mod = a.ep.tg.row(row) * a.N + col0;
#pragma unroll
                    for (int j = 0; j < 2 * F; ++j)
                        if (col0 + 16 * j < a.N) load8(a.ep.gate + mod + 16 * j, g[j]);
                }
                if (a.ep.residual != nullptr) {
#pragma unroll
                    for (int j = 0; j < 2 * F; ++j)
                        if (col0 + 16 * j < a.N) load_residual<F32>(a.ep, at + 16 * j, r[j]);
                }
#pragma unroll
                for (int j = 0; j < 2 * F; ++j) {
                    if (col0 + 16 * j >= a.N) break;
                    float z[8];
                    if (j % 2 == 0) here(acc[i][j / 2]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = acc[i][j / 2][8 * (j % 2) + e];
                    finish8<decltype(act)::value, F32>(a.ep, at + 16 * j, z, g[j], r[j]);
                }
            }
        });
    };

    Work w, next;
    if (!next_work(w)) return;
    begin(w);
    // Vector-memory operations that follow begin()'s loads of the first stage: those of the second, and behind
    // them the stores of the tile before, where all of its rows and columns exist (they complete in order). With a bias,
    // whose loads come after all of them and are used at once, there is nothing left to wait for here.
    bool stores = false;
    constexpr int STORES = 2 * F * F;
    for (;;) {
        // the sums start from the bias (a split tile's get it where its parts are joined)
        const int hw = (fresh_thread_index() & 63) >> 5;
#pragma unroll
        for (int j = 0; j < 2 * F; ++j) {
            float bias[8] = {};
            const int col = w.n0 + wn + 16 * j + 8 * hw;
            if (FULL && a.ep.bias != nullptr && w.part == nullptr && col < a.N) load8(a.ep.bias + col, bias);
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[i][j / 2][8 * (j % 2) + e] = bias[e];
        }
        const int later = min(AHEAD, w.s1 - w.s0) - 1;
        if (stores)
            wait_but(std::integral_constant<int, STORES>{}, later);
        else
            wait_but(std::integral_constant<int, 0>{}, later);
#pragma unroll
        for (int f = 0; f < 2 * F; ++f) read(L, L + SLOT, 0, f);
        uint32_t at = 0;
        int s = w.s0;
        for (; s + AHEAD < w.s1; ++s, at = ahead(at, 2)) stage(std::true_type{}, std::true_type{}, w, s, at);
        for (; s + 1 < w.s1; ++s, at = ahead(at, 2)) stage(std::true_type{}, std::false_type{}, w, s, at);
        stage(std::false_type{}, std::false_type{}, w, s, at);
        // (since the last stage's wait no wave reads LDS)
        const bool more = next_work(next);
        if (more) begin(next);
        finish(w);
        if (!more) return;
        stores = w.m0 + wm + WT <= a.M && w.n0 + wn + WT <= a.N;
        w = next;
    }
}

// The split tiles' sums of products from their parts, in the order of k, and the rest of the way. A thread
// takes 8 columns of a row. Bound by the parts' bytes (124 tiles of 256 in 2 parts, 65 MB, with gate and residual: 23 us).
template <int BT>
__global__ __launch_bounds__(256) void gemm_merge_kernel(const GemmArgs a) {
    constexpr int LPR = BT / 8, ROWS = 256 / LPR, PER = BT / ROWS;
    const int t = blockIdx.x / PER, id = a.whole + t;
    int m0, n0;
    tile_at(a, id, BT, m0, n0);
    const int r = (blockIdx.x % PER) * ROWS + threadIdx.x / LPR, c = (threadIdx.x % LPR) * 8;
    const int row = m0 + r, col = n0 + c;
    if (row >= a.M || col >= a.N) return;
    // The shares that hold stages [u0, u1) of the group: w0 to w1. Only the first can have begun in the tile before,
    // so that this one is its second.
    const int group = t % a.groups;
    const int u0 = t / a.groups * a.stages, u1 = u0 + a.stages;
    const int w0 = a.share_of(u0), w1 = a.share_of(u1 - 1);
    const float* part = a.part + static_cast<int64_t>(w0 * a.groups + group) * 2 * (BT * BT) + r * BT + c;
    const int64_t step = static_cast<int64_t>(a.groups) * 2 * (BT * BT);
    float z[8] = {}, sum[8];
    if (a.ep.bias != nullptr) load8(a.ep.bias + col, z);
    load8(part + (a.share_begin(w0) < u0 ? BT * BT : 0), sum);
#pragma unroll 4
    for (int w = w0 + 1; w <= w1; ++w) {
        float x[8];
        load8(part + (w - w0) * step, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] += sum[e];
    const int64_t at = static_cast<int64_t>(row) * a.N + col;
    by_kind(a.ep, [&](auto act, auto f32) __attribute__((always_inline)) {
        float g[8], r[8];
        if (a.ep.gate != nullptr) load8(a.ep.gate + a.ep.tg.row(row) * a.N + col, g);
        if (a.ep.residual != nullptr) load_residual<decltype(f32)::value>(a.ep, at, r);
        finish8<decltype(act)::value, decltype(f32)::value>(a.ep, at, z, g, r);
    });
}

template <int BT, bool AT, bool BTR>
hipError_t launch_tiles(const GemmArgs& a, hipStream_t s) {
    const int rest = a.tiles_m * a.tiles_n - a.whole;
    const int wgs = gemm_workgroups(a, BT);
    hipError_t e = hipSuccess;
    if (gemm_ahead(a, BT) == 4)
        e = launch_with(gemm_kernel<BT, AT, BTR, !BTR, BT < 256 ? 4 : 2>, dim3(wgs), 256, s, a);
    else
        e = launch_with(gemm_kernel<BT, AT, BTR, !BTR, 2>, dim3(wgs), 256, s, a);
    if (e != hipSuccess || rest == 0) return e;
    constexpr int PER = BT / (256 / (BT / 8));
    return launch_with(gemm_merge_kernel<BT>, dim3(rest * PER), 256, s, a);
}

// ---------------------------------------------------------------------------
// Few rows: W streams by once
// ---------------------------------------------------------------------------
// A workgroup takes 16 / C columns of the output (rows of W) and its NW waves share K in runs of 64 C:
// v_mfma_f32_16x16x32_bf16 with W as the first operand and the rows of x as the second. Of its 16 rows and
// columns, C blocks of 16 / C take a run's C pieces of 64 each; the blocks on the diagonal hold the sums of
// a piece, the others nothing of use. (One or a few rows leave columns over, and 16 columns a workgroup
// leave CUs idle: 5120 columns are 320 workgroups for 256 CUs.) A lane brings 32 neighbouring bytes of its row of W,
// the k of two MFMAs, so that 4 lanes read a whole line; which k an operand's element is does not matter as
// long as x's are the same. Rows that do not exist repeat the last one. Bound by HBM up to 4 rows (one row: 5.2 to 6.6
// TB/s from 5120 x 5120 to 5120 x 20480), by each workgroup's reads of x above.
template <int NW, int C>
__global__ __launch_bounds__(NW * 64) void few_rows_kernel(const FewRowsArgs a) {
    constexpr int CO = 16 / C;  // columns, and the most rows
    __shared__ float sums[NW][16][17];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * CO;
    const int64_t K = a.K;
    const int piece = (lane & 15) / CO, k0 = piece * 64 + (lane >> 4) * 16;
    const __bf16* w = static_cast<const __bf16*>(a.w) + min(n0 + (lane & 15) % CO, a.N - 1) * K + k0;
    const __bf16* x = static_cast<const __bf16*>(a.x) + min((lane & 15) % CO, a.rows - 1) * K + k0;
    f32x4_t acc[2] = {f32x4_t{}, f32x4_t{}};
    constexpr int RUN = 64 * C;
    const int whole = a.K / RUN;
    constexpr int U = 4;
    int i = wave;
    for (; i + (U - 1) * NW < whole; i += U * NW) {
        bf16x8_t wf[U][2], xf[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) wf[u][h] = *reinterpret_cast<const bf16x8_t*>(w + (i + u * NW) * RUN + h * 8);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) xf[u][h] = *reinterpret_cast<const bf16x8_t*>(x + (i + u * NW) * RUN + h * 8);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[u][h], xf[u][h], acc[h], 0, 0, 0);
    }
    // the runs that are left, the last one perhaps with its first k only
    for (; i * RUN < a.K; i += NW) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8_t wf = bf16x8_t{}, xf = bf16x8_t{};
            if (i * RUN + k0 + h * 8 < a.K) {
                wf = *reinterpret_cast<const bf16x8_t*>(w + i * RUN + h * 8);
                xf = *reinterpret_cast<const bf16x8_t*>(x + i * RUN + h * 8);
            }
            acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf, acc[h], 0, 0, 0);
        }
    }
    // register e of a lane: column 4 (lane / 16) + e, row lane % 16
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][lane & 15][4 * (lane >> 4) + e] = acc[0][e] + acc[1][e];
    __syncthreads();
    if (tid >= CO * CO) return;
    const int row = tid / CO, c = tid % CO, col = n0 + c;
    if (row >= a.rows || col >= a.N) return;
    float z = a.ep.bias != nullptr ? a.ep.bias[col] : 0.f, sum = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v)
#pragma unroll
        for (int q = 0; q < C; ++q) sum += sums[v][q * CO + row][q * CO + c];
    z += sum;
    const int64_t at = static_cast<int64_t>(row) * a.N + col;
    if (a.ep.pre != nullptr) static_cast<__bf16*>(a.ep.pre)[at] = static_cast<__bf16>(z);
    z = a.ep.act == kActGelu ? activate<kActGelu>(z) : a.ep.act == kActSilu ? activate<kActSilu>(z) : z;
    if (a.ep.gate != nullptr) z *= a.ep.gate[a.ep.tg.row(row) * a.N + col];
    if (a.ep.residual != nullptr)
        z += a.ep.o_f32 ? static_cast<const float*>(a.ep.residual)[at]
                        : static_cast<float>(static_cast<const __bf16*>(a.ep.residual)[at]);
    if (a.ep.o_f32)
        static_cast<float*>(a.ep.o)[at] = z;
    else
        static_cast<__bf16*>(a.ep.o)[at] = static_cast<__bf16>(z);
}

// ---------------------------------------------------------------------------
// Backward: the gradient of the sums of products, and its sums over rows
// ---------------------------------------------------------------------------
// The activation and its slope: gelu with s = sigmoid(u), u = 2 c (z + a z^3): s + z s (1 - s) u'; silu: s + z s (1 - s).
// 1 - s = e s with e = exp(-u), to the last digit where s is near 1; it counts for nothing where s is 0 (e may be
// infinite there).
__device__ __forceinline__ void activate_both(float z, int act, float& value, float& slope) {
    value = z;
    slope = 1.f;
    if (act == kActNone) return;
    constexpr float k1 = -1.4426950408889634f * kGelu2C, k3 = k1 * kGeluA;
    const float zz = z * z;
    const float e = __builtin_amdgcn_exp2f(z * (act == kActGelu ? fmaf(k3, zz, k1) : -1.4426950408889634f));
    const float s = __builtin_amdgcn_rcpf(1.f + e);
    value = z * s;
    const float rest = s > 0.f ? e * s : 0.f;
    const float du = act == kActGelu ? fmaf(3.f * kGeluA * kGelu2C, zz, kGelu2C) : 1.f;
    slope = rest > 0.f ? s * fmaf(z * rest, du, 1.f) : s;
}

// One part of the rows per workgroup and 256 columns: 32 lanes of 8 columns, 8 rows at a time. dz is rounded to bf16
// here, to be an operand of the matrix instructions; its sums over rows are not. The roundings are independent of each other
// and leave dx and dW with an error of 0.0023 of their norm, which their own rounding alone makes 0.0017 (bf16, 64-bit
// reference). As two bf16 numbers, dz_rest beside dz, it would double the products' MFMAs, 2.5 ms of the 2.8 of 32760 x 5120 x
// 5120, so only up to kExactRows rows, where nothing averages them and the bytes of W count, take both. Bound by HBM: 32760 x 5120
// from fp32 1.34 GB in 265 us (5.1 TB/s); 5376 x 4096 with GELU 132 MB in 25 us, close to its arithmetic (17 us).
__global__ __launch_bounds__(256) void linear_dz_kernel(const LinearDzArgs a) {
    __shared__ float sums[8][256];
    int32_t b, t0, t1;
    int64_t mod;
    a.parts.of(blockIdx.x, b, mod, t0, t1);
    const int lane = threadIdx.x % 32, line = threadIdx.x / 32;
    const int col = blockIdx.y * 256 + lane * 8;
    const bool in = col < a.N;
    float gate[8], sum_dz[8] = {}, sum_u[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) gate[e] = 1.f;
    if (in && a.gate != nullptr) load8(a.gate + mod * a.N + col, gate);
    if (in) {
#pragma unroll 1  // (2 rows at a time: 148 for 140 us of 5376 rows of 4096 with both products)
        for (int t = t0 + line; t < t1; t += 8) {
            const int64_t row = static_cast<int64_t>(b) * a.parts.n + t, at = row * a.N + col;
            float d[8], z[8] = {};
            if (a.dout_f32)
                load8(static_cast<const float*>(a.dout) + at, d);
            else
                load8(static_cast<const __bf16*>(a.dout) + at, d);
            if (a.pre != nullptr) load8(static_cast<const __bf16*>(a.pre) + at, z);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float value, slope;
                activate_both(z[e], a.act, value, slope);
                sum_u[e] = fmaf(d[e], value, sum_u[e]);
                d[e] *= gate[e] * slope;
                sum_dz[e] += d[e];
            }
            if (a.dz != nullptr) store8(static_cast<__bf16*>(a.dz) + at, d);
            if (a.dz_rest != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float hi = static_cast<float>(static_cast<__bf16>(d[e]));
                    d[e] = __builtin_isfinite(hi) ? d[e] - hi : 0.f;  // (no NaN beside an infinity)
                }
                store8(static_cast<__bf16*>(a.dz_rest) + at, d);
            }
            if (a.dz_few != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e) a.dz_few[static_cast<int64_t>(col + e) * a.R + row] = d[e];
            }
        }
        // (the rows that fill dz_few up to R)
        if (a.dz_few != nullptr && blockIdx.x == 0) {
            for (int row = a.parts.B * a.parts.n + line; row < a.R; row += 8)
#pragma unroll
                for (int e = 0; e < 8; ++e) a.dz_few[static_cast<int64_t>(col + e) * a.R + row] = 0.f;
        }
    }
    if (a.part == nullptr) return;
    float* out = a.part + static_cast<int64_t>(blockIdx.x) * kLinearSums * a.N;
    for (int v = 0; v < (a.gate_sums ? 2 : 1); ++v) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[line][lane * 8 + e] = v == 0 ? sum_dz[e] : sum_u[e];
        __syncthreads();
        const int c = blockIdx.y * 256 + threadIdx.x;
        if (c < a.N) {
            float s = 0.f;
#pragma unroll
            for (int l = 0; l < 8; ++l) s += sums[l][threadIdx.x];
            out[v * a.N + c] = s;
        }
    }
}

// dx of R rows: 512 columns per wave, the 4 waves of a workgroup and the shares of the grid deal out N; the
// gradients are the same in every lane. In fp32: with so few rows nothing would average the roundings of dz. One row
// of 5120 x 5120, dx and dW: 27 us for 105 MB.
template <int R>
__global__ __launch_bounds__(256) void few_rows_dx_kernel(const FewRowsBwdArgs a) {
    __shared__ float sums[3][64][9];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = blockIdx.x * 512 + lane * 8;
    const int piece = blockIdx.y * 4 + wave, pieces = a.shares * 4;
    const int n0 = static_cast<int>(static_cast<int64_t>(a.N) * piece / pieces);
    const int n1 = static_cast<int>(static_cast<int64_t>(a.N) * (piece + 1) / pieces);
    float acc[R][8];
#pragma unroll
    for (int m = 0; m < R; ++m)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[m][e] = 0.f;
    const __bf16* w = static_cast<const __bf16*>(a.w) + min(col, a.K - 8);
#pragma unroll 4
    for (int n = n0; n < n1; ++n) {
        float x[8];
        load8(w + static_cast<int64_t>(n) * a.K, x);
        const float* g = a.dz + static_cast<int64_t>(n) * R;
#pragma unroll
        for (int m = 0; m < R; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[m][e] = fmaf(g[m], x[e], acc[m][e]);
    }
#pragma unroll
    for (int m = 0; m < R; ++m) {
        __syncthreads();
        if (wave > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[wave - 1][lane][e] = acc[m][e];
        }
        __syncthreads();
        if (wave == 0 && col < a.K) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                acc[m][e] = ((acc[m][e] + sums[0][lane][e]) + sums[1][lane][e]) + sums[2][lane][e];
            store8(a.part + (static_cast<int64_t>(blockIdx.y) * R + m) * a.K + col, acc[m]);
        }
    }
}

// 32 groups of 8 columns per workgroup, 8 threads a group, which deal out the shares.
__global__ __launch_bounds__(256) void few_rows_dx_merge_kernel(const FewRowsBwdArgs a) {
    __shared__ float sums[8][32][9];
    const int lane = threadIdx.x % 32, l = threadIdx.x / 32, per = a.K / 8;
    const int at = blockIdx.x * 32 + lane;
    const bool in = at < a.rows * per;
    const int row = in ? at / per : 0, col = in ? at % per * 8 : 0;
    float s[8] = {};
#pragma unroll 4
    for (int p = l; p < a.shares; p += 8) {
        float x[8];
        load8(a.part + (static_cast<int64_t>(p) * a.R + row) * a.K + col, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += x[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[l][lane][e] = s[e];
    __syncthreads();
    if (l > 0 || !in) return;
#pragma unroll
    for (int k = 1; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += sums[k][lane][e];
    store8(static_cast<__bf16*>(a.dx) + static_cast<int64_t>(row) * a.K + col, s);
}

// dW of R rows: 8 columns a lane, whose R values of x stay in registers over kDwRows rows of dW.
constexpr int kDwRows = 16;
template <int R>
__global__ __launch_bounds__(256) void few_rows_dw_kernel(const FewRowsBwdArgs a) {
    const int col = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.K) return;
    float x[R][8];
#pragma unroll
    for (int m = 0; m < R; ++m) load8(static_cast<const __bf16*>(a.x) + min(m, a.rows - 1) * static_cast<int64_t>(a.K) + col, x[m]);
    const int n1 = min(a.N, (static_cast<int>(blockIdx.y) + 1) * kDwRows);
    for (int n = blockIdx.y * kDwRows; n < n1; ++n) {
        const float* g = a.dz + static_cast<int64_t>(n) * R;
        float d[8] = {};
#pragma unroll
        for (int m = 0; m < R; ++m) {
            if (m < a.rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = fmaf(g[m], x[m][e], d[e]);
            }
        }
        store8(static_cast<__bf16*>(a.dw) + static_cast<int64_t>(n) * a.K + col, d);
    }
}

// x twice, one behind the other (n groups of 8), the second time for what dz's rounding left. Zeros stand there for
// infinities and NaN, which dz's first part takes along alone: the parts' signs differ, or the second one is zero.
__global__ __launch_bounds__(256) void twice_kernel(const TwiceArgs a) {
    const int64_t i = blockIdx.x * int64_t(256) + threadIdx.x;
    if (i >= a.n) return;
    bf16x8_t v = static_cast<const bf16x8_t*>(a.x)[i];
    static_cast<bf16x8_t*>(a.out)[i] = v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_isfinite(static_cast<float>(v[e])) ? v[e] : static_cast<__bf16>(0.f);
    static_cast<bf16x8_t*>(a.out)[a.n + i] = v;
}

// out = a + b, b behind a (n groups of 8); a alone where it is no finite number (of an infinite weight, as above).
__global__ __launch_bounds__(256) void halves_sum_kernel(const TwiceArgs a) {
    const int64_t i = (blockIdx.x * int64_t(256) + threadIdx.x) * 8;
    if (i >= a.n * 8) return;
    float u[8], v[8];
    load8(static_cast<const float*>(a.x) + i, u);
    load8(static_cast<const float*>(a.x) + a.n * 8 + i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = __builtin_isfinite(u[e]) ? u[e] + v[e] : u[e];
    store8(static_cast<__bf16*>(a.out) + i, u);
}

__global__ __launch_bounds__(256) void zero_kernel(uint32_t* p, int64_t n) {
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) p[i] = 0;
}

}  // namespace

hipError_t launch_gemm(const GemmArgs& a, int tile, bool a_trans, bool b_trans, hipStream_t s) {
#define TM_GEMM_CASE(T_, A_, B_) \
    if (tile == T_ && a_trans == A_ && b_trans == B_) return launch_tiles<T_, A_, B_>(a, s);
    TM_GEMM_CASE(256, false, false)
    TM_GEMM_CASE(128, false, false)
    TM_GEMM_CASE(64, false, false)
    TM_GEMM_CASE(256, false, true)
    TM_GEMM_CASE(128, false, true)
    TM_GEMM_CASE(64, false, true)
    TM_GEMM_CASE(256, true, true)
    TM_GEMM_CASE(128, true, true)
    TM_GEMM_CASE(64, true, true)
#undef TM_GEMM_CASE
    return hipErrorInvalidValue;
}

hipError_t launch_few_rows(const FewRowsArgs& a, hipStream_t s) {
    int pieces, waves;
    few_rows_shape(a.rows, a.N, &pieces, &waves);
    const int columns = 16 / pieces;
    const dim3 grid((a.N + columns - 1) / columns);
    const bool four = waves == 4;
    switch (pieces) {
        case 1: return four ? launch_with(few_rows_kernel<4, 1>, grid, 256, s, a) : launch_with(few_rows_kernel<16, 1>, grid, 1024, s, a);
        case 2: return four ? launch_with(few_rows_kernel<4, 2>, grid, 256, s, a) : launch_with(few_rows_kernel<16, 2>, grid, 1024, s, a);
    }
    return four ? launch_with(few_rows_kernel<4, 4>, grid, 256, s, a) : launch_with(few_rows_kernel<16, 4>, grid, 1024, s, a);
}

hipError_t launch_linear_dz(const LinearDzArgs& a, hipStream_t s) {
    return launch_with(linear_dz_kernel, dim3(a.parts.filled(), (a.N + 255) / 256), 256, s, a);
}

template <int R>
static hipError_t launch_few_bwd(const FewRowsBwdArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (a.dx != nullptr) {
        e = launch_with(few_rows_dx_kernel<R>, dim3((a.K + 511) / 512, a.shares), 256, s, a);
        if (e != hipSuccess) return e;
        e = launch_with(few_rows_dx_merge_kernel, dim3((static_cast<unsigned>(a.rows) * (a.K / 8) + 31) / 32), 256, s, a);
        if (e != hipSuccess) return e;
    }
    if (a.dw != nullptr)
        e = launch_with(few_rows_dw_kernel<R>, dim3((a.K + 2047) / 2048, (a.N + kDwRows - 1) / kDwRows), 256, s, a);
    return e;
}

hipError_t launch_few_rows_bwd(const FewRowsBwdArgs& a, hipStream_t s) {
    switch (a.R) {
        case 1: return launch_few_bwd<1>(a, s);
        case 2: return launch_few_bwd<2>(a, s);
        case 4: return launch_few_bwd<4>(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_twice(const TwiceArgs& a, hipStream_t s) {
    return launch_with(twice_kernel, dim3(static_cast<unsigned>((a.n + 255) / 256)), 256, s, a);
}
hipError_t launch_halves_sum(const TwiceArgs& a, hipStream_t s) {
    return launch_with(halves_sum_kernel, dim3(static_cast<unsigned>((a.n + 255) / 256)), 256, s, a);
}

hipError_t launch_zero(void* p, int64_t n, hipStream_t s) {
    if (n == 0) return hipSuccess;
    const int64_t blocks = (n + 255) / 256;
    hipLaunchKernelGGL(zero_kernel, dim3(static_cast<unsigned>(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s,
                       static_cast<uint32_t*>(p), n);
    return hipGetLastError();
}

}  // namespace tmk
