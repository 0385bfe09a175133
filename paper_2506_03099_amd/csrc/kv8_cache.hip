// The 8-bit KV cache: writing a chunk, with or without the normalisation and
// rotation of its queries and keys on the way, and reading a chunk back, for
// gfx950.
//
// The cache keeps the keys and values of c_0 and of the window's chunks so that
// context is never recomputed (TalkingMachines, Sec. 4.3, "KV & Embedding
// Cachings"); 80 caches of a 480p stream take 17.9 GB in bf16, half in 8 bits. A
// block of 64 tokens of a head shares a scale, of K and of V apart:
//     scale = max(largest magnitude of the block, 2^-60) / 127,
//     code = round(x / scale), to even at ties,
// so a value is off by at most half a scale, 1/254 of its block's largest
// magnitude. Rows of unit root mean square in blocks of 64 * 128 have a largest
// magnitude near 4, so the codes' error is near 0.9% of the rows' size (an 8-bit
// float with 3 bits of mantissa: 2.6%). A block that holds an infinity or a NaN
// cannot be coded: its scale is NaN, and all of it reads back as NaN. Chunks start
// on whole blocks, so writing one never touches another's scale.
//
// Writing: a workgroup per (batch, key head, block) takes the block's K and V
// rows in registers, forms their largest magnitudes over the workgroup, and puts
// the codes through LDS into the order of tm_kv8.h; nothing is read twice. The
// producer's queries are rows of their own, in workgroups of the same launch that
// go first (the other way round 1.4% slower). Bound by HBM: K and V in (2 bytes an
// element), codes out (1). Measured on a chunk of 4680 tokens, 40 heads of 128:
// written 25-32 us on different nodes (144 MB, 4.5-5.8 TB/s), read back 22.3 us (144 MB, 6.4), produced
// 53-61 us from cold inputs (240 MB, 3.9-4.5 TB/s; 39 where they are in the last-level cache).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tm_device.h"
#include "tm_internal.h"
#include "tm_kv8.h"
#include "tm_rope.h"

namespace tmk {
namespace {

constexpr int kKv8Threads = 256;
constexpr float kLeastMax = 0x1p-60f;  // a block's largest magnitude counts as at least this

// Sum over the N (4 or 8) consecutive lanes that hold a row, left in all of them.
template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
template <int N>
__device__ __forceinline__ float lanes_sum(float s) {
    static_assert(N == 4 || N == 8, "4 or 8 lanes per row");
    s += dpp_f<0xB1>(s);                          // quad_perm [1, 0, 3, 2]
    s += dpp_f<0x4E>(s);                          // quad_perm [2, 3, 0, 1]
    if constexpr (N == 8) s += dpp_f<0x141>(s);   // row_half_mirror
    return s;
}

// x / sqrt(mean(x^2) + eps) * gain of the row held by D / 16 lanes.
template <int D>
__device__ __forceinline__ void normalise(float (&x)[kRowElems], const float* gain, float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < kRowElems; ++e) ss = fmaf(x[e], x[e], ss);
    ss = lanes_sum<D / kRowElems>(ss);
    const float r = 1.f / sqrtf(ss / static_cast<float>(D) + eps);
#pragma unroll
    for (int e = 0; e < kRowElems; ++e) x[e] = x[e] * r * gain[e];
}

template <int D>
__device__ __forceinline__ void load_gains(const float* gain, int g, float (&w)[kRowElems]) {
#pragma unroll
    for (int e = 0; e < kRowElems; ++e) w[e] = 1.f;
    if (gain == nullptr) return;
#pragma unroll
    for (int e = 0; e < kRowElems; e += 4) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(gain + run_of<2, D>(g, e / 8) + e % 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[e + i] = v[i];
    }
}

// The largest magnitude among x, as bits: of non-negative floats the order of
// the bits is that of the values, infinity and then every NaN on top.
__device__ __forceinline__ uint32_t magnitude(const float (&x)[kRowElems], uint32_t m) {
#pragma unroll
    for (int e = 0; e < kRowElems; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    return m;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
    return m;
}

// The scale of a block of largest magnitude `m` (bits): NaN if it is not finite.
__device__ __forceinline__ float scale_of(uint32_t m) {
    if (m >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return fmaxf(__uint_as_float(m), kLeastMax) * (1.f / 127.f);
}

// 4 codes of x * inv, biased, in a word. The product is rounded to fp32 before it is
// rounded to a code (no fma): that defines the codes to the bit. Adding 2^23 + 2^22
// rounds to a whole number, to even at ties, and leaves it in the low bits.
__device__ __forceinline__ uint32_t codes4(const float* x, float inv) {
#pragma clang fp contract(off)
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float p = x[e] * inv;
        c[e] = __float_as_uint(p + 0x1.8p23f);
    }
    const uint32_t lo = pick_bytes(c[1], c[0], 0x0C0C0400), hi = pick_bytes(c[3], c[2], 0x04000C0C);
    return (lo | hi) ^ (kCodeZero * 0x01010101u);  // low bytes; + 128 in each
}

// D: head_dim. PRODUCE: the first a.q_wgs workgroups normalise and rotate queries, and
// the keys are normalised and rotated before they are coded (a.turn: rotated at all).
template <int D, bool PRODUCE, bool HALVES>
__global__ __launch_bounds__(kKv8Threads) void kv8_write_kernel(const Kv8WriteArgs a) {
    constexpr int G = D / kRowElems;                    // lanes per row
    constexpr int RPI = kKv8Threads / G;                // rows per pass
    constexpr int IT = kCacheBlock / RPI;               // passes: 2 at D = 128, 1 at D = 64
    constexpr int PITCH = D / 4 + 2;                    // words per LDS row: 32 rows' 8-byte reads of a
                                                        // column fall on 64 different banks
    constexpr int PIECES = kCacheBlock * D / 16;        // of one tensor of the block
    static_assert(IT >= 1 && IT * RPI == kCacheBlock, "whole passes");
    __shared__ __attribute__((aligned(16))) uint32_t tile[2][kCacheBlock * PITCH];
    __shared__ uint32_t tops[2][kKv8Threads / 64];

    const int tid = threadIdx.x;
    const int g = tid % G, r0 = tid / G;
    if constexpr (PRODUCE) {
        if (blockIdx.x < a.q_wgs) {
            // a lane takes this part of the rows of heads s, s + S, ... of a token
            constexpr int U = 4;
            const uint32_t idx = blockIdx.x * static_cast<uint32_t>(kKv8Threads) + tid;
            const uint32_t r = idx / G;
            const int s = r % a.q_slices;
            const int64_t row = r / a.q_slices;  // of [B, n]
            if (row >= static_cast<int64_t>(a.B) * a.n_tok) return;
            RowBits<2> bits[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = s + u * a.q_slices;
                if (h < a.H) bits[u] = load_row<2, D>(a.q + (row * a.H + h) * (D * 2), g);
            }
            float2 cs[8];
            if (a.turn) load_turns<2, D, HALVES>(a.table, a.first_token + row % a.n_tok, g, cs);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = s + u * a.q_slices;
                if (h >= a.H) continue;
                float x[kRowElems], w[kRowElems];
                unpack_row<2>(bits[u], x);
                load_gains<D>(a.q_gain != nullptr ? a.q_gain + h * D : nullptr, g, w);
                normalise<D>(x, w, a.eps);
                if (a.turn) turn_row<HALVES>(x, cs);
                store_row<2, D>(a.q_out + (row * a.H + h) * (D * 2), g, x);
            }
            return;
        }
    }

    const uint32_t wg = blockIdx.x - (PRODUCE ? a.q_wgs : 0);
    const int blk = wg % a.n_blk;
    const int bh = wg / a.n_blk;
    const int h = bh % a.Hk;
    const int64_t b = bh / a.Hk;
    const int64_t stride = static_cast<int64_t>(a.Hk) * D * 2;  // bytes per source token
    const int64_t first = b * a.n_tok * stride + static_cast<int64_t>(h) * D * 2;
    const int64_t t0 = static_cast<int64_t>(blk) * kCacheBlock;  // of the chunk

    RowBits<2> kb[IT], vb[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int64_t t = t0 + r0 + it * RPI;
#pragma unroll
        for (int i = 0; i < 2; ++i) kb[it].v[i] = vb[it].v[i] = u32x4_t{0, 0, 0, 0};
        if (t < a.n_tok) {
            kb[it] = load_row<2, D>(a.k + first + t * stride, g);
            vb[it] = load_row<2, D>(a.v + first + t * stride, g);
        }
    }
    float xk[IT][kRowElems], xv[IT][kRowElems];
    uint32_t mk = 0, mv = 0;
    float w[kRowElems];
    if constexpr (PRODUCE) load_gains<D>(a.k_gain != nullptr ? a.k_gain + h * D : nullptr, g, w);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        unpack_row<2>(kb[it], xk[it]);
        unpack_row<2>(vb[it], xv[it]);
        if constexpr (PRODUCE) {
            const int64_t t = t0 + r0 + it * RPI;
            float2 cs[8];
            if (a.turn) load_turns<2, D, HALVES>(a.table, a.first_token + min(t, static_cast<int64_t>(a.n_tok - 1)), g, cs);
            normalise<D>(xk[it], w, a.eps);
            if (a.turn) turn_row<HALVES>(xk[it], cs);
            // (eps 0 makes NaN of a row of zeros, which rows past the chunk's end are not)
            if (t >= a.n_tok) {
#pragma unroll
                for (int e = 0; e < kRowElems; ++e) xk[it][e] = 0.f;
            }
        }
        mk = magnitude(xk[it], mk);
        mv = magnitude(xv[it], mv);
    }
    mk = wave_max(mk);
    mv = wave_max(mv);
    if (tid % 64 == 0) {
        tops[0][tid / 64] = mk;
        tops[1][tid / 64] = mv;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kKv8Threads / 64; ++i) {
        mk = max(mk, tops[0][i]);
        mv = max(mv, tops[1][i]);
    }
    const float sk = scale_of(mk), sv = scale_of(mv);
    const float ik = 1.f / sk, iv = 1.f / sv;
    const int64_t at = (b * a.Hk + h) * a.n_blocks + a.first_blk + blk;  // block of the cache
    if (tid == 0) {
        a.k_scale[at] = sk;
        a.v_scale[at] = sv;
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int r = r0 + it * RPI;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int c = r * PITCH + run_of<2, D>(g, half) / 4;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                tile[0][c + i] = codes4(xk[it] + 8 * half + 4 * i, ik);
                tile[1][c + i] = codes4(xv[it] + 8 * half + 4 * i, iv);
            }
        }
    }
    __syncthreads();
    // K: a piece is two 8-byte runs of one key's row.
    unsigned char* const ko = a.k_codes + at * (kCacheBlock * D);
    for (int n = tid; n < PIECES; n += kKv8Threads) {
        const int lane = n % 64, s = n / 64 % (D / 32), half = n / 64 / (D / 32);
        const uint32_t* const from = &tile[0][(32 * half + k_perm(lane % 32)) * PITCH + 8 * s + 2 * (lane / 32)];
        store16_through(ko + 16 * n, u32x4_t{from[0], from[1], from[4], from[5]});
    }
    // V: 4 dimensions of 16 keys, transposed, are 4 pieces next to each other. They go through LDS
    // once more, so that a wave stores a whole KB: with four pieces a lane every store instruction
    // touched a quarter of 64 lines (with the rows loaded in the same manner, 38.7 us for 24.9).
    constexpr int QUADS = (PIECES / 4 + kKv8Threads - 1) / kKv8Threads;
    static_assert(QUADS == 1, "a thread transposes at most once");
    u32x4_t p[4];
    const int quad = tid % (D / 4), hw = tid / (D / 4) % 2, half = tid / (D / 4) / 2;
    if (tid < PIECES / 4) {
        const uint32_t* const from = &tile[1][(32 * half + 8 * hw) * PITCH + quad];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // keys 4 (i % 2) .. of the run's first or second 16
            uint32_t r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = from[(16 * (i / 2) + 4 * (i % 2) + e) * PITCH];
            transpose4x4(r);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e][i] = r[e];
        }
    }
    __syncthreads();
    u32x4_t* const pieces = reinterpret_cast<u32x4_t*>(tile);
    if (tid < PIECES / 4) {
        const int d = quad / 8, l = 4 * (quad % 8) + 32 * hw;
#pragma unroll
        for (int e = 0; e < 4; ++e) pieces[(half * (D / 32) + d) * 64 + l + e] = p[e];
    }
    __syncthreads();
    unsigned char* const vo = a.v_codes + at * (kCacheBlock * D);
    for (int n = tid; n < PIECES; n += kKv8Threads) store16_through(vo + 16 * n, pieces[n]);
}

// The values a chunk's codes stand for, [B, n_tok, Hk, D], rounded to bf16 (OF32:
// fp32). The writer's steps backwards: a workgroup per (batch, key head, block).
template <int D, bool OF32>
__global__ __launch_bounds__(kKv8Threads) void kv8_read_kernel(const Kv8ReadArgs a) {
    constexpr int G = D / kRowElems;
    constexpr int RPI = kKv8Threads / G;
    constexpr int IT = kCacheBlock / RPI;
    constexpr int PITCH = D / 4 + 2;
    constexpr int PIECES = kCacheBlock * D / 16;
    constexpr int EB = OF32 ? 4 : 2;
    __shared__ uint32_t tile[2][kCacheBlock * PITCH];
    const int tid = threadIdx.x;
    const int blk = blockIdx.x % a.n_blk;
    const int bh = blockIdx.x / a.n_blk;
    const int h = bh % a.Hk;
    const int64_t b = bh / a.Hk;
    const int64_t at = (b * a.Hk + h) * a.n_blocks + a.first_blk + blk;
    const unsigned char* const ki = a.k_codes + at * (kCacheBlock * D);
    const unsigned char* const vi = a.v_codes + at * (kCacheBlock * D);
    const float sk = a.k_scale[at], sv = a.v_scale[at];
    for (int n = tid; n < PIECES; n += kKv8Threads) {
        const int lane = n % 64, s = n / 64 % (D / 32), half = n / 64 / (D / 32);
        const u32x4_t p = *reinterpret_cast<const u32x4_t*>(ki + 16 * n);
        uint32_t* const to = &tile[0][(32 * half + k_perm(lane % 32)) * PITCH + 8 * s + 2 * (lane / 32)];
        to[0] = p[0];
        to[1] = p[1];
        to[4] = p[2];
        to[5] = p[3];
    }
    for (int n = tid; n < PIECES / 4; n += kKv8Threads) {
        const int quad = n % (D / 4), hw = n / (D / 4) % 2, half = n / (D / 4) / 2;
        uint32_t* const to = &tile[1][(32 * half + 8 * hw) * PITCH + quad];
        const int d = quad / 8, l = 4 * (quad % 8) + 32 * hw;
        u32x4_t p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            p[e] = *reinterpret_cast<const u32x4_t*>(vi + 16 * ((half * (D / 32) + d) * 64 + l + e));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r[4] = {p[0][i], p[1][i], p[2][i], p[3][i]};
            transpose4x4(r);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[(16 * (i / 2) + 4 * (i % 2) + e) * PITCH] = r[e];
        }
    }
    __syncthreads();
    const int g = tid % G, r0 = tid / G;
    const int64_t stride = static_cast<int64_t>(a.Hk) * D * EB;
    const int64_t first = b * a.n_tok * stride + static_cast<int64_t>(h) * D * EB;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const int r = r0 + it * RPI;
        const int64_t t = static_cast<int64_t>(blk) * kCacheBlock + r;
        if (t >= a.n_tok) continue;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float v[kRowElems];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = tile[x][r * PITCH + (run_of<EB, D>(g, 4 * i * EB / 16) + 4 * i % (16 / EB)) / 4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (128 off before the product: 128 scales of the largest values are past fp32)
                    v[4 * i + e] = (static_cast<float>((w >> (8 * e)) & 0xFFu) - 128.f) * (x == 0 ? sk : sv);
                }
            }
            store_row<EB, D>((x == 0 ? a.k_out : a.v_out) + first + t * stride, g, v);
        }
    }
}

}  // namespace

hipError_t launch_kv8_write(Kv8WriteArgs a, int head_dim, bool produce, bool halves, hipStream_t s) {
    a.n_blk = (a.n_tok + kCacheBlock - 1) / kCacheBlock;
    const int64_t kv = static_cast<int64_t>(a.n_blk) * a.B * a.Hk;
    a.q_slices = (a.H + 3) / 4;
    const int64_t q_threads = produce ? static_cast<int64_t>(a.B) * a.n_tok * a.q_slices * (head_dim / kRowElems) : 0;
    const int64_t grid = kv + (q_threads + kKv8Threads - 1) / kKv8Threads;
    if (grid > INT32_MAX || q_threads > UINT32_MAX - kKv8Threads) return hipErrorInvalidValue;
    a.q_wgs = static_cast<uint32_t>(grid - kv);
#define TM_KV8_WRITE(D_, P_, HV_)                         \
    if (head_dim == D_ && produce == P_ && halves == HV_) \
        return launch_with(kv8_write_kernel<D_, P_, HV_>, dim3(static_cast<unsigned>(grid)), kKv8Threads, s, a);
    TM_KV8_WRITE(128, false, false)
    TM_KV8_WRITE(64, false, false)
    TM_KV8_WRITE(128, true, false)
    TM_KV8_WRITE(64, true, false)
    TM_KV8_WRITE(128, true, true)
    TM_KV8_WRITE(64, true, true)
#undef TM_KV8_WRITE
    return hipErrorInvalidValue;
}

hipError_t launch_kv8_read(Kv8ReadArgs a, int head_dim, bool of32, hipStream_t s) {
    a.n_blk = (a.n_tok + kCacheBlock - 1) / kCacheBlock;
    const int64_t grid = static_cast<int64_t>(a.n_blk) * a.B * a.Hk;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
#define TM_KV8_READ(D_, F_)           \
    if (head_dim == D_ && of32 == F_) \
        return launch_with(kv8_read_kernel<D_, F_>, dim3(static_cast<unsigned>(grid)), kKv8Threads, s, a);
    TM_KV8_READ(128, false)
    TM_KV8_READ(64, false)
    TM_KV8_READ(128, true)
    TM_KV8_READ(64, true)
#undef TM_KV8_READ
    return hipErrorInvalidValue;
}

}  // namespace tmk
