// Attention over the 8-bit KV cache for gfx950.
//
// O_i = softmax_j(scale * q_i . k_j) v_j over the keys of c_0 and of the window's
// chunks (TalkingMachines, Sec. 4.2), with k = ks * code and v = vs * code, a
// scale ks and vs for each block of 64 tokens and head. Blocks belong to one
// chunk each, so a tile of 64 keys has one scale of K and one of V.
//
// Codes become fp16 operands, exactly: the byte code + 128 under the exponent of
// 1024 is the fp16 number 1152 + code, less 1152 (one byte permutation and one
// packed addition for two codes; the way over fp32 to bf16 takes twice that). So
// q is fp16 as well: its rows are scaled by a power of two that puts their largest
// element in [2^14, 2^15), which keeps every bf16 digit of elements down to 2^-28
// of it. The products q . code are summed in fp32; the scales follow on the sums:
//     x = (q . code) * (scale log2(e) ks / row's power) + log2(r) - m,
// one fma per score, P = 2^x in fp16 (11 digits, bf16 has 8), O += P . code, and
// the row sum takes P / r. r = vs / unit is V's scale in the unit, a power of two, that O
// is held in. Folding r into the exponent scales P, not the 8-bit operand, so nothing
// is rounded for it; a unit that follows the scales (struct Unit) keeps r in [1/8, 2), so
// that P stays where fp16 has its digits whatever the sizes of V. m is the running maximum of
// x + m less 8: P reaches 2^8 and a tile may exceed that by 2^7 before m is raised; what
// fp16 then loses at its lower end is below 2^-29 of the largest weight (2^-25 of 2^8 / 16).
//
// Both operands lose the bias of 128 before the products. (With K's codes as they are held
// and 128 times the row's sum of q taken off the score afterwards, a packed addition less for
// two codes, scores lose the digits by which 128 sum |q| exceeds sum |q code|: nearly all of
// P's where one channel of K sets the scale and the others' codes are small.)
//
// Tile kernel: as in the bf16 forward (attn_fwd.hip), 8 waves of 32 query rows share
// every 64-key tile in LDS, each wave's softmax in between its own MFMAs. The tiles come
// as codes into registers, half the bytes, one tile ahead, and are turned into fp16
// operands once per workgroup on the way into LDS; the cache's order makes every LDS
// access a contiguous KB (no bank conflicts). Bound by the MFMAs (58% of the cycles) and by
// what the waves wait for in between: 4680 queries over 10920 keys, 40 heads of 128,
// 889-950 us on different nodes (1102-1177 TFLOP/s; an 8192^3 bf16 product reaches 1627 at
// best), 10% more than the bf16 forward over a 16-bit cache. The decoding's place among
// the MFMAs hardly matters. Blocks of V that move the unit every time (scales 100 times
// apart) take 8% more.
//
// Few rows: a workgroup's waves share the keys of one block of 32 rows out, each with
// whole 64-key blocks, whose operands it loads straight from the cache; their results
// are merged through LDS, those of several workgroups by a second kernel, in a fixed
// order. Bound by the cache's bytes: one row, 65745 keys, 8 key heads, 4 streams (539
// MB) 95 us a call, 5 of them for the merge (5.7 TB/s); 10920 keys, 40 heads (112 MB) 26.2.
// Caches of some thousand keys are bound by a wave's chain of loads, decoding, products
// and softmax: 389 vector instructions a block of D = 128, with the masks behind a branch and
// one fma a score, behind the maximum (6517 keys, 18 rows, 20 heads 15.3 us a call).

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tm_device.h"
#include "tm_internal.h"
#include "tm_kv8.h"

namespace tmk {
namespace {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) f16x8_t lds_f16x8_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef __attribute__((address_space(3))) unsigned char lds_u8;

constexpr int kTileThreads = 512;
constexpr int kTileWaves = kTileThreads / 64;
constexpr int kTileRows = 32 * kTileWaves;
constexpr float kHeadroom = 8.f;      // log2 of the largest P after m is set
constexpr float kLargeScore = 0x1p10f;  // of m: a sum of its size is off by 2^-14 at most
constexpr float kRaise = 0x1p15f;     // a lane's sum of P over half a tile that raises m
static_assert(kTileRows == kTileRowsBf16, "the host counts tiles of this many rows");

__device__ __forceinline__ f32x16_t mfma(f16x8_t a, f16x8_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// 2 codes of a word as fp16: bytes 0 and 1 (HI: 2 and 3).
template <bool HI>
__device__ __forceinline__ f16x2_t decode2(uint32_t w) {
    const f16x2_t x = __builtin_bit_cast(f16x2_t, pick_bytes(0x64646464u, w, HI ? 0x04030402u : 0x04010400u));
    return x - f16x2_t{static_cast<_Float16>(1152.f), static_cast<_Float16>(1152.f)};
}
// 8 codes as an operand's 8 elements.
__device__ __forceinline__ f16x8_t decode8(uint32_t a, uint32_t b) {
    const f16x2_t p = decode2<false>(a), q = decode2<true>(a), r = decode2<false>(b), s = decode2<true>(b);
    return f16x8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

__device__ __forceinline__ float pin(float x) {
    asm volatile("" : "+v"(x));
    return x;
}
// Zero that the compiler takes to differ between lanes: an address formed with it
// is loaded through the vector unit, in order with the other vector loads (scalar
// loads share the counter of the LDS reads and come back in any order).
__device__ __forceinline__ int lane_zero() {
    int z = 0;
    asm volatile("" : "+v"(z));
    return z;
}

// T at byte `off` of the lane from a base that is the same in every lane (global
// memory by its type: a pointer put together from scalar registers would be loaded
// from as one that may point into LDS, and counted with the LDS reads).
template <typename T>
__device__ __forceinline__ T load_from(const void* base, uint32_t off) {
    typedef const __attribute__((address_space(1))) char* global_t;
    return *(const __attribute__((address_space(1))) T*)((global_t)(uniform_ptr(base)) + off);
}

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ float uniform_f(float x) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(static_cast<int>(__float_as_uint(x))));
}

// Larger of the two half-waves' values, in both.
__device__ __forceinline__ float both_max(float x) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// A row's maximum less the headroom. Where floats lie 16 apart that would round to 16 less, and 2^16 is
// past fp16: the maximum itself then (a difference of 0, 8 or 16 is exact).
__device__ __forceinline__ float below(float top) {
    const float m = top - kHeadroom;
    return top - m > kHeadroom ? top : m;
}

// Row r (of the n_q * group of a key head) of q and o: its offset in rows of D.
__device__ __forceinline__ int64_t row_at(const Kv8AttnArgs& a, int bat, int kvh, int r) {
    const int i = a.by_group.of(r), g = r - i * a.group;
    return (static_cast<int64_t>(bat) * a.n_q + i) * a.H + kvh * a.group + g;
}
__device__ __forceinline__ int64_t lse_at(const Kv8AttnArgs& a, int bat, int kvh, int r) {
    const int i = a.by_group.of(r), g = r - i * a.group;
    return (static_cast<int64_t>(bat) * a.H + kvh * a.group + g) * a.n_q + i;
}

// A query row's elements as the lane feeds them to the score MFMAs: dimensions 16 kk +
// 8 hw .. + 7. (Every lane loads a row that exists: with a row of zeros for the others
// the compiler made a branch and a wait of each load.)
template <int D>
__device__ __forceinline__ void load_q(const Kv8AttnArgs& a, int64_t row, int hw, u32x4_t (&raw)[D / 16]) {
    const u32x4_t* const p = reinterpret_cast<const u32x4_t*>(static_cast<const __bf16*>(a.q) + row * D + 8 * hw);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) raw[kk] = p[2 * kk];
}
// The same as B operands, scaled by a power of two; returns scale_log2 over that power.
// A row with an infinity or a NaN gets NaN, and so does its output.
template <int D>
__device__ __forceinline__ float scale_q(const u32x4_t (&raw)[D / 16], float scale_log2, f16x8_t (&qf)[D / 16]) {
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    u16x2_t tops{0, 0};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int w = 0; w < 4; ++w)
            tops = __builtin_elementwise_max(tops, __builtin_bit_cast(u16x2_t, raw[kk][w] & 0x7FFF7FFFu));
    uint32_t top = max(tops[0], tops[1]);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
    const uint32_t e = top >> 7;  // the exponent field
    const uint32_t up = min(127u + 14 + 127 - min(e, 254u), 253u);
    const float mult = __uint_as_float(up << 23);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            qf[kk][2 * w] = static_cast<_Float16>(__uint_as_float(raw[kk][w] << 16) * mult);
            qf[kk][2 * w + 1] = static_cast<_Float16>(__uint_as_float(raw[kk][w] & 0xFFFF0000u) * mult);
        }
    return e == 255 ? __uint_as_float(0x7FC00000u) : scale_log2 * __uint_as_float((254 - up) << 23);
}

// The factor of a tile's scores from that of the row's q and the scale of K. (Not zero, as a tiny
// row's may be: a masked score of -inf is still to be scaled; nor infinite, as that of large rows: a
// score of zero still is one. NaN stays.)
__device__ __forceinline__ float score_factor(float cq, float ks) {
    const float c = cq * ks, low = c < FLT_MIN ? FLT_MIN : c;
    return low > FLT_MAX ? FLT_MAX : low;
}

// The unit of O: 2^(e - 127), moved where a block's scale of V lies outside [1/8, 2) of it, by the whole
// wave, as a block's scale is the same in every lane. O follows by an exact factor, unless that takes it
// past the ends of fp32: so the unit is kept within 2^-kDown of the largest so far (O is at most 2^15 *
// 127 * 2^30 in it), and a block further down counts as one of 1/8 of that, off by less than 2^-60 of the
// largest value. Scales are 2^-60 / 127 at least, so normal numbers, or NaN, which moves nothing.
struct Unit {
    static constexpr int kDown = 64;
    int e = 0;    // (0: no block yet, and O is zero)
    int top = 0;
    __device__ __forceinline__ bool holds(float vs) const {
        return static_cast<uint32_t>(exponent(vs) - e + 3) <= 3u;
    }
    __device__ __forceinline__ void move(float& vs) {
        const int ev = exponent(vs);
        if (ev == 255) return;
        e = max(ev + 1, top - kDown);
        top = max(top, e);
        if (ev < e - 3) vs = __uint_as_float(static_cast<uint32_t>(e - 3) << 23);
    }
    __device__ __forceinline__ float inverse() const { return __uint_as_float(static_cast<uint32_t>(254 - e) << 23); }
    __device__ __forceinline__ float value() const { return __uint_as_float(static_cast<uint32_t>(e) << 23); }
    // What turns values held in the unit of exponent `from` into ones of this unit.
    __device__ __forceinline__ float from(int f) const {
        return f - e < -126 ? 0.f : __uint_as_float(static_cast<uint32_t>(f - e + 127) << 23);
    }
    static __device__ __forceinline__ int exponent(float vs) {
        return static_cast<int>(__builtin_amdgcn_readfirstlane(static_cast<int>(__float_as_uint(vs))) >> 23);
    }
};

// Waits for scalar loads, which share a counter with the LDS reads and come back in
// any order: after this no wait for one has to wait for every LDS read in flight.
__device__ __forceinline__ void wait_scalars() { __builtin_amdgcn_s_waitcnt(kWaitLgkmcnt0); }

// The key blocks of the call, one after the other.
struct Blocks {
    int r = 0;     // range
    int blk = 0;   // block of the cache
    int keys = 0;  // keys from this block to the range's end
    __device__ __forceinline__ void start(const Kv8AttnArgs& a, int skip) {
        r = 0;
        int n = (a.range_keys[0] + kCacheBlock - 1) / kCacheBlock;
        while (skip >= n && r + 1 < a.n_ranges) {
            skip -= n;
            ++r;
            n = (a.range_keys[r] + kCacheBlock - 1) / kCacheBlock;
        }
        blk = a.range_begin[r] + skip;
        keys = a.range_keys[r] - skip * kCacheBlock;
    }
    // On by one block; stays on the last one at the end. No else branch, and the kernel arguments
    // only on the rare path: its scalar loads are waited for there (see wait_scalars).
    __device__ __forceinline__ void step(const Kv8AttnArgs& a) {
        ++blk;
        keys -= kCacheBlock;
        if (__builtin_expect(keys <= 0, 0)) {
            if (r + 1 < a.n_ranges) {
                ++r;
                blk = a.range_begin[r];
                keys = a.range_keys[r];
            } else {
                --blk;
                keys += kCacheBlock;
            }
            wait_scalars();
        }
    }
    // On by `by` blocks; stays on the last one at the end.
    __device__ __forceinline__ void next(const Kv8AttnArgs& a, int by) {
        while (by > 0) {
            const int left = (keys - 1) / kCacheBlock;  // blocks behind this one in the range
            if (by <= left) {
                blk += by;
                keys -= by * kCacheBlock;
                return;
            }
            if (r + 1 >= a.n_ranges) {
                blk += left;
                keys -= left * kCacheBlock;
                return;
            }
            by -= left + 1;
            ++r;
            blk = a.range_begin[r];
            keys = a.range_keys[r];
        }
    }
};

// Rows [q0, q1) of tile `idx`: blocks of 32 shared out as evenly as they go.
__device__ __forceinline__ void split_rows(const Kv8AttnArgs& a, int idx, int& q0, int& q1) {
    q0 = 32 * (idx * a.row_blocks + min(idx, a.more_row_blocks));
    q1 = min(32 * ((idx + 1) * a.row_blocks + min(idx + 1, a.more_row_blocks)), a.rows);
}

// A workgroup's tile and share of its keys: whole tiles come first, then the split
// ones' parts, a tile's next to each other; with a cut, all first parts (up to the
// cut) and then all second ones. XCDS: consecutive tiles on one XCD. (Divisions by
// multiplication: with the runtime's own, of 64 bits where they split the keys, a
// workgroup spent some 300 instructions here.)
struct Share {
    int tile, bat, kvh, part;
    int split;  // number of the split tile, -1: whole
    int b0, n;  // first key block of the walk and how many
};
template <bool XCDS>
__device__ __forceinline__ Share share_of(const Kv8AttnArgs& a) {
    Share s;
    const int bid = blockIdx.x, splits = a.n_tiles * a.B * a.Hk - a.n_whole;
    int id;
    s.part = 0;
    s.split = -1;
    s.b0 = 0;
    s.n = a.n_kblocks;
    if (bid < a.n_whole) {
        id = XCDS ? xcd_logical_id(bid, a.n_whole) : bid;
    } else if (a.cut > 0) {
        const int j = bid - a.n_whole;
        s.part = j >= splits;
        s.split = xcd_logical_id(s.part ? j - splits : j, splits);
        id = a.n_whole + s.split;
        s.b0 = s.part ? a.cut : 0;
        s.n = s.part ? a.n_kblocks - a.cut : a.cut;
    } else {
        const int j = XCDS ? xcd_logical_id(bid - a.n_whole, splits * a.parts) : bid - a.n_whole;
        s.split = a.by_parts.of(j);
        s.part = j - s.split * a.parts;
        id = a.n_whole + s.split;
        s.b0 = s.part * a.part_blocks + min(s.part, a.more_part_blocks);
        s.n = a.part_blocks + (s.part < a.more_part_blocks);
    }
    const int bh = a.by_tiles.of(id);
    s.tile = id - bh * a.n_tiles;
    s.bat = a.by_heads.of(bh);
    s.kvh = bh - s.bat * a.Hk;
    return s;
}
// Kernel arguments that the start of a kernel needs, read together: left to itself the
// compiler reads them one after the other where they are first used, and waits each time.
__device__ __forceinline__ void read_args(const Kv8AttnArgs& a) {
    asm volatile("" ::"s"(a.q), "s"(a.k_codes), "s"(a.v_codes), "s"(a.k_scale), "s"(a.v_scale), "s"(a.B), "s"(a.H),
                 "s"(a.Hk), "s"(a.group), "s"(a.n_q), "s"(a.rows), "s"(a.n_blocks), "s"(a.n_tiles), "s"(a.n_whole),
                 "s"(a.parts), "s"(a.n_kblocks), "s"(a.range_begin[0]), "s"(a.range_keys[0]));
    asm volatile("" ::"s"(a.part_blocks), "s"(a.more_part_blocks), "s"(a.by_parts.mul), "s"(a.by_parts.shift),
                 "s"(a.by_tiles.mul), "s"(a.by_tiles.shift), "s"(a.by_heads.mul), "s"(a.by_heads.shift),
                 "s"(a.by_group.mul), "s"(a.by_group.shift), "s"(a.scale_log2), "s"(a.n_ranges), "s"(a.cut));
}
// A split tile's partial rows: O over the part's own row sum, [rows][D] (parts have units of their
// own), then each row's maximum and sum.
template <int D, int ROWS>
__device__ __forceinline__ float* part_at(const Kv8AttnArgs& a, int split, int part) {
    return a.part + (static_cast<int64_t>(split) * a.parts + part) * (ROWS * (D + 2));
}

// ----------------------------------------------------------------------------
// Few rows
// ----------------------------------------------------------------------------
// NW waves share the keys of a tile out.
template <int D, bool OF32, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_kv8_few_kernel(const Kv8AttnArgs a) {
    constexpr int KK = D / 16, DB = D / 32, NP = 2 * DB;  // pieces of K, and of V, of a block
    constexpr int PITCH = D + 4;                           // floats per row in LDS
    __shared__ float rows_o[NW][kKv8FewRows * PITCH];
    __shared__ float rows_m[NW][kKv8FewRows], rows_l[NW][kKv8FewRows], units[NW];
    const int lane = threadIdx.x & 63, hw = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    read_args(a);
    const Share s = share_of<false>(a);
    const int q0 = s.tile * kKv8FewRows, n_rows = min(kKv8FewRows, a.rows - q0);
    u32x4_t raw[KK];
    load_q<D>(a, row_at(a, s.bat, s.kvh, min(q0 + l32, a.rows - 1)), hw, raw);
    const int64_t head = (static_cast<int64_t>(s.bat) * a.Hk + s.kvh) * a.n_blocks;

    f32x16_t acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x16_t{};
    float m = kNegInf, l = 0.f;
    Unit unit;
    u32x4_t kc[NP], vc[NP];
    float ks = 0.f, vs = 0.f;
    const uint32_t lane16 = 16 * lane;
    auto load_k = [&](int blk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            kc[i] = load_from<u32x4_t>(a.k_codes + (head + blk) * (kCacheBlock * D) + 1024 * i, lane16);
    };
    auto load_v = [&](int blk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            vc[i] = load_from<u32x4_t>(a.v_codes + (head + blk) * (kCacheBlock * D) + 1024 * i, lane16);
    };
    // this wave's blocks: every NW-th of the share
    Blocks at;
    if (wave < s.n) {
        at.start(a, s.b0 + wave);
        load_k(at.blk);
        ks = a.k_scale[head + at.blk];
        load_v(at.blk);
        vs = a.v_scale[head + at.blk];
    }
    f16x8_t qf[KK];
    const float cq = scale_q<D>(raw, a.scale_log2, qf);
    for (int j = wave; j < s.n; j += NW) {
        const int keys = at.keys;
        f32x16_t x[2] = {f32x16_t{}, f32x16_t{}};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int kb = i / DB, st = i % DB;
            x[kb] = mfma(decode8(kc[i][0], kc[i][1]), qf[2 * st], x[kb]);
            x[kb] = mfma(decode8(kc[i][2], kc[i][3]), qf[2 * st + 1], x[kb]);
        }
        float c = score_factor(cq, ks);
        if (__builtin_expect(!unit.holds(vs), 0)) {
            const int was = unit.e;
            unit.move(vs);
            if (was != 0) {
                const float to = unit.from(was);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] *= to;
            }
        }
        const float share = vs * unit.inverse();
        const float iv = __builtin_amdgcn_rcpf(share), add = __builtin_amdgcn_logf(share);
        at.next(a, NW);  // (past the share's end: a block that exists)
        load_k(at.blk);
        ks = a.k_scale[head + at.blk];
        vs = a.v_scale[head + at.blk];
        if (__builtin_expect(keys < kCacheBlock, 0)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * kb + 16 * (i / 8) + 8 * hw + i % 8 >= keys) x[kb][i] = kNegInf;
        }
        // the maximum of x + m of the header's formula, from that of the sums (c is positive)
        float mx = x[0][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) mx = fmaxf(mx, x[e / 16][e % 16]);
        mx = below(fmaf(both_max(mx), c, add));
        if (__builtin_expect(__ballot(mx > m) != 0, 0)) {
            const float nm = fmaxf(m, mx);
            const float alpha = __builtin_amdgcn_exp2f(m == kNegInf ? kNegInf : m - nm);
            m = nm;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= alpha;
        }
        // (a row with only scores of -inf so far: P = 0)
        const float base = m == kNegInf ? 0.f : m;
        float less = add - base;
        // `less` is rounded at the size of m. Scores so large that it shows take their steps one by one,
        // which leaves the difference from the maximum exact (in the lanes of those rows alone: the
        // others keep their bits).
        if (__builtin_expect(fabsf(base) > kLargeScore, 0)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e / 16][e % 16] = fmaf(x[e / 16][e % 16], c, add) - base;
            c = 1.f;
            less = 0.f;
        }
        float lt = 0.f;
        f16x8_t pf[4];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(x[e / 16][e % 16], c, less));
            lt += p;
            pf[e / 8][e % 8] = static_cast<_Float16>(p);
        }
        l = fmaf(lt, iv, l);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int kb = i / DB, d = i % DB;
            acc[d] = mfma(decode8(vc[i][0], vc[i][1]), pf[2 * kb], acc[d]);
            acc[d] = mfma(decode8(vc[i][2], vc[i][3]), pf[2 * kb + 1], acc[d]);
        }
        load_v(at.blk);
    }
    // the waves' results, merged in order
    l += __shfl_xor(l, 32);
    if (l32 < n_rows) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4_t*>(&rows_o[wave][l32 * PITCH + 32 * d + 8 * g + 4 * hw]) =
                    f32x4_t{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]};
        if (hw == 0) {
            rows_m[wave][l32] = m;
            rows_l[wave][l32] = l;
        }
    }
    if (lane == 0) units[wave] = unit.value();
    __syncthreads();
    float* const part = s.split >= 0 ? part_at<D, kKv8FewRows>(a, s.split, s.part) : nullptr;
    for (int n = threadIdx.x; n < n_rows * (D / 4); n += 64 * NW) {
        const int r = n / (D / 4), d = 4 * (n % (D / 4));
        float top = kNegInf;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, rows_m[w][r]);
        const float base = top == kNegInf ? 0.f : top;
        float sum = 0.f, f[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            f[w] = __builtin_amdgcn_exp2f(rows_m[w][r] - base);
            sum = fmaf(f[w], rows_l[w][r], sum);
        }
        // (a part with only scores of -inf: zeros, which count for nothing in the merge)
        const float inv = part != nullptr && sum == 0.f ? 0.f : 1.f / sum;
        f32x4_t o{};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float to = f[w] * inv * units[w];
            const f32x4_t ow = *reinterpret_cast<const f32x4_t*>(&rows_o[w][r * PITCH + d]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(to, ow[e], o[e]);
        }
        if (part != nullptr) {
            *reinterpret_cast<f32x4_t*>(part + r * D + d) = o;
            if (d == 0) {
                part[kKv8FewRows * D + 2 * r] = top;
                part[kKv8FewRows * D + 2 * r + 1] = sum;
            }
            continue;
        }
        const int64_t at_o = row_at(a, s.bat, s.kvh, q0 + r) * D + d;
        if constexpr (OF32) {
            *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.o) + at_o) = o;
        } else {
            bf16x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = static_cast<__bf16>(o[e]);
            *reinterpret_cast<bf16x4_t*>(static_cast<__bf16*>(a.o) + at_o) = h;
        }
        if (a.lse != nullptr && d == 0)
            a.lse[lse_at(a, s.bat, s.kvh, q0 + r)] = (top + __log2f(sum)) * 0.69314718055994530942f;
    }
}

// ----------------------------------------------------------------------------
// Tiles of 256 rows
// ----------------------------------------------------------------------------
template <int D, bool OF32>
__global__ __launch_bounds__(kTileThreads, 1) void attn_kv8_tile_kernel(const Kv8AttnArgs a) {
    constexpr int KK = D / 16, DB = D / 32;
    constexpr int NK = 2 * KK, NV = 4 * DB, NF = NK + NV;  // operand fragments (1 KB) and MFMAs of a tile
    constexpr int TILEB = NK * 1024;                       // bytes of a K (or V) tile in LDS
    constexpr int NBUF = 4;
    constexpr int RING = 4;       // fragments read ahead of their MFMA
    constexpr int EPG = 32 / NK;  // P elements formed per score MFMA
    constexpr int FPG = 32 / NV;  // scores scaled per P V MFMA
    constexpr int NP = 2 * kCacheBlock * D / 16 / kTileThreads;  // pieces of codes per thread: K and V, or one
    static_assert(NF % RING == 0 && EPG % 2 == 0 && (NP == 1 || NP == 2), "layout");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * NBUF * TILEB];
    lds_u8* const L = (lds_u8*)(smem);

    const int tid = threadIdx.x, lane = tid & 63, hw = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    read_args(a);
    const Share s = share_of<true>(a);
    const int n = s.n;
    int q0, q1;
    split_rows(a, s.tile, q0, q1);
    const int64_t head = (static_cast<int64_t>(s.bat) * a.Hk + s.kvh) * a.n_blocks;

    // ---- codes: thread's pieces of a block, and where they go in a tile. NP = 2: piece
    // tid of K and of V; NP = 1: waves 0..3 take K's, the others V's. A piece is two fragments'
    // 16 bytes of the lane, next to each other in LDS.
    const bool v_first = NP == 1 && wave >= 4;
    const int pw = NP == 2 ? wave : wave & 3;  // piece's kb * DB + (s or d)
    const uint32_t lane16 = 16 * lane;
    const uint32_t lds_to = 2 * pw * 1024 + lane16;
    // (V's lane offset in a register of its own: it is past the reach of a read's immediate, and the
    // compiler would add it up for every read; 977 -> 964 us)
    uint32_t v_lane16 = NBUF * TILEB + lane16;
    asm volatile("" : "+v"(v_lane16));
    u32x4_t codes[NP];  // of the block that is turned into operands next
    float ks, vs;   // scales of the tile whose scores come next (the same in every lane)
    int blk[NBUF];  // block j of the walk in [j % 4]
    int cnt[NBUF];  // keys from it to its range's end
    const int z = lane_zero();
    Blocks at;
    at.start(a, s.b0);
    // The codes of the block that the walk stands on, block u of the tiles; the walk moves on by step().
    auto load = [&](u32x4_t (&to)[NP], int u) __attribute__((always_inline)) {
        const int64_t o = (head + at.blk) * (kCacheBlock * D) + 1024 * pw;
        if constexpr (NP == 2) {
            to[0] = load_from<u32x4_t>(a.k_codes + o, lane16);
            to[1] = load_from<u32x4_t>(a.v_codes + o, lane16);
        } else {
            to[0] = load_from<u32x4_t>((v_first ? a.v_codes : a.k_codes) + o, lane16);
        }
        blk[u & 3] = at.blk;
        cnt[u & 3] = at.keys;
    };
    auto load_scales = [&](int u) __attribute__((always_inline)) {
        ks = load_from<float>(a.k_scale + head + blk[u & 3], z);
        vs = load_from<float>(a.v_scale + head + blk[u & 3], z);
    };
    // Codes turned into operands two at a time: pair i of the thread's ND (piece i / 8, half i / 4 % 2), and
    // each half's 16 bytes into the buffers of block u once its four pairs are there.
    constexpr int ND = 8 * NP;
    f16x2_t half[4];
    auto put = [&](const u32x4_t (&from)[NP], int i, int u) __attribute__((always_inline)) {
        const int p = i / 8, h = i / 4 % 2;
        const uint32_t w = from[p][2 * h + i / 2 % 2];
        half[i % 4] = i % 2 ? decode2<true>(w) : decode2<false>(w);
        if (i % 4 != 3) return;
        const uint32_t base = NP == 2 ? p * NBUF * TILEB : v_first ? NBUF * TILEB : 0;
        *(lds_f16x8_t*)(L + lds_to + base + ((u & (NBUF - 1)) * TILEB + h * 1024)) =
            f16x8_t{half[0][0], half[0][1], half[1][0], half[1][1], half[2][0], half[2][1], half[3][0], half[3][1]};
    };
    // Fragment f of a tile's stream: K fragments (kk = f / 2, kb = f % 2) of buffer ku, then V
    // fragments (j = (f - NK) / DB, d) of buffer vu. In LDS: (kb, kk) and (j / 2, d, j % 2).
    auto read_frag = [&](int f, int ku, int vu) __attribute__((always_inline)) {
        const int j = (f - NK) / DB, d = (f - NK) % DB;
        if (f < NK) return *(const lds_f16x8_t*)(L + lane16 + ((ku & (NBUF - 1)) * TILEB + ((f & 1) * KK + (f >> 1)) * 1024));
        return *(const lds_f16x8_t*)(L + v_lane16 + ((vu & (NBUF - 1)) * TILEB + (((j >> 1) * DB + d) * 2 + (j & 1)) * 1024));
    };

    f32x16_t acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x16_t{};
    float m = 0.f, l = 0.f, iv = 0.f;  // iv: 1 / (scale of V in the unit) of the tile whose P is formed
    Unit unit;        // of that tile's P
    int acc_unit = 0;  // exponent of O's, which follows before the tile's P V
    uint64_t fresh = 0;  // lanes whose row has had no finite score yet (m is 0 until the first)
    auto mask_tile = [&](f32x16_t (&x)[2], int keys) __attribute__((always_inline)) {
        // register i of block kb is key 32 kb + 16 (i / 8) + 8 hw + i % 8 (the lane's bound formed
        // here, so that 32 keys per lane are not kept, spilled, across the loop)
        const int bound = keys - ((fresh_thread_index() >> 2) & 8);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * kb + 16 * (i / 8) + i % 8 >= bound) x[kb][i] = kNegInf;
    };
    auto row_max = [&](const f32x16_t (&x)[2]) __attribute__((always_inline)) {
        float mx = fmaxf(x[0][0], x[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, fmaxf(x[0][i], x[1][i]));
        return both_max(mx);
    };
    // P of elements e and e + 1 into their operand's word, summed into *lt. The word is pinned: else
    // the compiler rounds behind the check's branch and keeps 32 more registers until there.
    auto form_p2 = [&](const f32x16_t (&x)[2], u32x4_t (&pf)[4], int e, float& lt) __attribute__((always_inline)) {
        const float p0 = __builtin_amdgcn_exp2f(x[e >> 4][e & 15]);
        const float p1 = __builtin_amdgcn_exp2f(x[(e + 1) >> 4][(e + 1) & 15]);
        uint32_t w = __builtin_bit_cast(uint32_t, f16x2_t{static_cast<_Float16>(p0), static_cast<_Float16>(p1)});
        asm volatile("" : "+v"(w));
        pf[e >> 3][(e & 7) >> 1] = w;
        lt = e < 4 ? p0 + p1 : lt + (p0 + p1);
    };

    // ---- prologue: blocks 0..2 into LDS, block 3 in registers; every load is issued before the first
    // is waited for
    u32x4_t early[3][NP];
#pragma unroll
    for (int u = 0; u < 3; ++u) {
        load(early[u], u);
        at.step(a);
    }
    load(codes, 3);
    load_scales(0);
    const int qrow = q0 + wave * 32 + l32;
    f16x8_t qf[KK];
    u32x4_t raw[KK];
    load_q<D>(a, row_at(a, s.bat, s.kvh, min(qrow, a.rows - 1)), hw, raw);
    const float cq = scale_q<D>(raw, a.scale_log2, qf);
#pragma unroll
    for (int u = 0; u < 3; ++u)
#pragma unroll
        for (int i = 0; i < ND; ++i) put(early[u], i, u);
    __syncthreads();

    // A wave without rows takes part in the loads and barriers only.
    const bool busy = q0 + wave * 32 < q1;
    f32x16_t xa[2], xb[2];
    if (busy) {
        xa[0] = xa[1] = f32x16_t{};
#pragma unroll
        for (int f = 0; f < NK; ++f) xa[f & 1] = mfma(read_frag(f, 0, 0), qf[f >> 1], xa[f & 1]);
        const float c = score_factor(cq, ks);
        unit.move(vs);
        acc_unit = unit.e;
        const float share = vs * unit.inverse(), add = __builtin_amdgcn_logf(share);
        iv = uniform_f(__builtin_amdgcn_rcpf(share));
        load_scales(1);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) xa[kb][i] = fmaf(xa[kb][i], c, add);
        if (cnt[0] < kCacheBlock) mask_tile(xa, cnt[0]);
        const float mx = row_max(xa);
        m = mx == kNegInf ? 0.f : below(mx);
        fresh = __ballot(mx == kNegInf);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) xa[kb][i] -= m;
    }
    f16x8_t fr[RING];
#pragma unroll
    for (int f = 0; f < RING; ++f) fr[f] = read_frag(f, 1, 1);

    // ---- iteration t, with x = x(t) and nx receiving S(t+1); u = t % 4. Stage 1: the score
    // MFMAs of tile t+1, each with its share of P(t). Check: a lane's sum of P beyond the bound
    // (or not a number) raises m to the tile's maximum less the headroom, rescales O and the row
    // sum and forms P(t) again; O follows P(t) where that is in another unit. Stage 2: the P V
    // MFMAs of tile t, each with its share of x(t+1), of turning block t+3's codes into operands
    // in LDS, and of loading block t+4's. Block t+3 goes where block t-1 was, whose last reads
    // lie before the barrier that ended tile t-1. The barrier that ends tile t publishes block
    // t+3; K(t+2), read ahead here, was published by the one before.
    auto end_tile = [&](bool reads) __attribute__((always_inline)) {
        // this wave's LDS writes are done when at most the reads ahead behind them are not
        if (reads) __builtin_amdgcn_s_waitcnt(0xC07F | (RING << 8));
        else __builtin_amdgcn_s_waitcnt(kWaitLgkmcnt0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr int PUTS = NV - RING;  // MFMAs of stage 2 that have a share of the codes
    auto iteration = [&](int u, f32x16_t (&x)[2], f32x16_t (&nx)[2]) __attribute__((always_inline)) {
        at.step(a);
        u32x4_t pf[4];
        float lt0, lt1;
        nx[0] = nx[1] = f32x16_t{};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < NK; ++g) {
            nx[g & 1] = mfma(fr[g % RING], qf[g >> 1], nx[g & 1]);
            fr[g % RING] = read_frag(g + RING, u + 1, u);
#pragma unroll
            for (int e = EPG * g; e < EPG * (g + 1); e += 2) form_p2(x, pf, e, (e & 2) ? lt1 : lt0);
            __builtin_amdgcn_sched_barrier(0);
        }
        uint64_t raise = __ballot(!(lt0 + lt1 <= kRaise));
        // (one branch for all of it on the way past: two take 0.5% longer)
        if (__builtin_expect((raise | fresh | static_cast<uint32_t>(unit.e ^ acc_unit)) != 0, 0)) {
            const float to = unit.from(acc_unit);
            acc_unit = unit.e;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= to;
            if ((raise | fresh) != 0) {
                raise |= raise << 32 | raise >> 32;  // both lanes of a row; other rows keep their bits
                const float mx = row_max(x);
                const bool first = __builtin_amdgcn_inverse_ballot_w64(fresh) && mx != kNegInf;
                const float up = __builtin_amdgcn_inverse_ballot_w64(raise) ? fmaxf(below(mx), 0.f) : 0.f;
                const float dm = first ? below(mx) : up;
                const float alpha = first ? 1.f : __builtin_amdgcn_exp2f(-dm);  // (sum and O are still 0)
                fresh &= __ballot(mx == kNegInf);
                m += dm;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] *= alpha;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[kb][i] -= dm;
#pragma unroll
                for (int e = 0; e < 32; e += 2) form_p2(x, pf, e, (e & 2) ? lt1 : lt0);
            }
        }
        // (as one fma the compiler kept two copies of O: 200 registers spilled)
        l += pin(pin(lt0 + lt1) * iv);
        const float c = score_factor(cq, ks);
        if (__builtin_expect(!unit.holds(vs), 0)) unit.move(vs);
        const float share = vs * unit.inverse(), add = __builtin_amdgcn_logf(share) - m;
        iv = uniform_f(__builtin_amdgcn_rcpf(share));
        if (__builtin_expect(cnt[(u + 1) & 3] < kCacheBlock, 0)) mask_tile(nx, cnt[(u + 1) & 3]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            acc[k % DB] = mfma(fr[(NK + k) % RING], __builtin_bit_cast(f16x8_t, pf[k / DB]), acc[k % DB]);
            fr[(NK + k) % RING] = read_frag((NK + k + RING) % NF, NK + k + RING < NF ? u + 1 : u + 2, u);
#pragma unroll
            for (int e = FPG * k; e < FPG * (k + 1); ++e) nx[e >> 4][e & 15] = pin(fmaf(nx[e >> 4][e & 15], c, add));
            // (every write lies before the last RING reads ahead)
#pragma unroll
            for (int i = ND * k / PUTS; i < ND * (k + 1) / PUTS && k < PUTS; ++i) put(codes, i, u + 3);
            if (k == PUTS) load(codes, u + 4);
            if (k == PUTS + 1) load_scales(u + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        end_tile(true);
    };
    if (busy) {
        for (int t = 0; t < n; t += 4) {
            iteration(0, xa, xb);
            if (t + 1 >= n) break;
            iteration(1, xb, xa);
            if (t + 2 >= n) break;
            iteration(2, xa, xb);
            if (t + 3 >= n) break;
            iteration(3, xb, xa);
        }
    } else {
        auto idle = [&](int u) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < ND; ++i) put(codes, i, u + 3);
            at.step(a);
            load(codes, u + 4);
            end_tile(false);
        };
        for (int t = 0; t < n; t += 4) {
            idle(0);
            if (t + 1 >= n) break;
            idle(1);
            if (t + 2 >= n) break;
            idle(2);
            if (t + 3 >= n) break;
            idle(3);
        }
    }
    __syncthreads();

    // ---- the rows, through the wave's share of the LDS so that they are stored whole: O over
    // the row sum (a part's: in fp32)
    l += __shfl_xor(l, 32);
    const bool part_rows = s.split >= 0;
    float* const part = part_rows ? part_at<D, kTileRows>(a, s.split, s.part) : nullptr;
    const float inv = part_rows && l == 0.f ? 0.f : __uint_as_float(static_cast<uint32_t>(acc_unit) << 23) / l;
    if (busy) {
        constexpr int CPR = D / 4;  // 16-byte chunks of an fp32 row
        static_assert(kTileRows * D * 4 <= 2 * NBUF * TILEB, "output rows must fit the LDS");
        lds_u8* const rows = L + wave * (32 * D * 4);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4_t w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = acc[d][4 * g + e] * inv;
                *(lds_f32x4_t*)(rows + l32 * (D * 4) + (((8 * d + 2 * g + hw) ^ (l32 & 15)) << 4)) = w;
            }
        asm volatile("" ::: "memory");
#pragma unroll 4
        for (int i = 0; i < 32 * CPR / 64; ++i) {
            const int ch = 64 * i + lane, row = ch / CPR, cc = ch % CPR;
            const f32x4_t w = *(const lds_f32x4_t*)(rows + row * (D * 4) + ((cc ^ (row & 15)) << 4));
            const int r = q0 + wave * 32 + row;
            if (r >= q1) continue;
            if (part_rows) {
                *reinterpret_cast<f32x4_t*>(part + (wave * 32 + row) * D + 4 * cc) = w;
            } else if constexpr (OF32) {
                *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.o) + row_at(a, s.bat, s.kvh, r) * D + 4 * cc) = w;
            } else {
                bf16x4_t h;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = static_cast<__bf16>(w[e]);
                *reinterpret_cast<bf16x4_t*>(static_cast<__bf16*>(a.o) + row_at(a, s.bat, s.kvh, r) * D + 4 * cc) = h;
            }
        }
        if (qrow < q1 && hw == 0) {
            if (part_rows) {
                part[kTileRows * D + 2 * (wave * 32 + l32)] = m;
                part[kTileRows * D + 2 * (wave * 32 + l32) + 1] = l;
            } else if (a.lse != nullptr) {
                a.lse[lse_at(a, s.bat, s.kvh, qrow)] = (m + __log2f(l)) * 0.69314718055994530942f;
            }
        }
    }
}

// ----------------------------------------------------------------------------
// Merging the parts of split tiles
// ----------------------------------------------------------------------------
// PG = 1: a thread adds up all parts of 4 elements of a row, in order; PG = 8: 8
// threads take every 8th part each, their sums are added up in order.
constexpr int kMergeThreads = 256;
template <int D, bool OF32, int ROWS, int PG>
__global__ __launch_bounds__(kMergeThreads) void attn_kv8_merge_kernel(const Kv8AttnArgs a) {
    constexpr int TPR = D / 4;                           // threads that hold a row
    constexpr int RPW = kMergeThreads / (TPR * PG);      // rows of a workgroup
    constexpr int U = 4;                                 // parts loaded together
    static_assert(RPW >= 1 && ROWS % RPW == 0, "whole workgroups per tile");
    __shared__ f32x4_t sums[PG > 1 ? kMergeThreads : 1];
    __shared__ float lsums[PG > 1 ? kMergeThreads : 1], tops[PG > 1 ? kMergeThreads : 1];
    const int tid = threadIdx.x;
    const int d = 4 * (tid % TPR), pg = tid / TPR % PG;
    const int split = blockIdx.y;
    const int r = blockIdx.x * RPW + tid / (TPR * PG);  // row of the tile
    const int id = a.n_whole + split;
    const int bh = a.by_tiles.of(id), tile = id - bh * a.n_tiles;
    const int bat = a.by_heads.of(bh), kvh = bh - bat * a.Hk;
    int q0, q1;
    if constexpr (ROWS == kKv8FewRows) {
        q0 = tile * kKv8FewRows;
        q1 = min(q0 + kKv8FewRows, a.rows);
    } else {
        split_rows(a, tile, q0, q1);
    }
    const bool ok = q0 + r < q1;
    const float* const p = part_at<D, ROWS>(a, split, 0);
    constexpr int64_t step = ROWS * (D + 2);
    // one pass: O is the mean of the parts so far, by their shares of the row sum
    float top = kNegInf, sum = 0.f;
    f32x4_t o{};
    // (a part without a finite score has a sum of 0, any maximum and zeros)
    auto add = [&](const float (&mi)[U], const float (&li)[U], const f32x4_t (&oi)[U]) __attribute__((always_inline)) {
        float nm = top, share[U];
#pragma unroll
        for (int u = 0; u < U; ++u) nm = fmaxf(nm, li[u] == 0.f ? kNegInf : mi[u]);
        const float keep = sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f(top - nm);
        sum = keep;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            share[u] = li[u] == 0.f ? 0.f : li[u] * __builtin_amdgcn_exp2f(mi[u] - nm);
            sum += share[u];
        }
        top = nm;
        const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
        o *= keep * inv;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(share[u] * inv, oi[u][e], o[e]);
    };
    if (ok) {
        for (int i0 = pg; i0 < a.parts; i0 += U * PG) {
            float mi[U], li[U];
            f32x4_t oi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {  // (past the end: the last part again, which then counts for nothing)
                const float* const pi = p + min(i0 + u * PG, a.parts - 1) * step;
                mi[u] = pi[ROWS * D + 2 * r];
                li[u] = i0 + u * PG < a.parts ? pi[ROWS * D + 2 * r + 1] : 0.f;
                oi[u] = *reinterpret_cast<const f32x4_t*>(pi + r * D + d);
            }
            add(mi, li, oi);
        }
    }
    if constexpr (PG > 1) {
        sums[tid] = o;
        lsums[tid] = sum;
        tops[tid] = top;
        __syncthreads();
        if (pg != 0) return;
        static_assert(PG == 2 * U, "the others' sums, in two steps");
#pragma unroll
        for (int i = 0; i < PG; i += U) {
            float mi[U], li[U];
            f32x4_t oi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                mi[u] = tops[tid + (i + u) * TPR];
                li[u] = i + u == 0 ? 0.f : lsums[tid + (i + u) * TPR];  // (its own are there)
                oi[u] = sums[tid + (i + u) * TPR];
            }
            add(mi, li, oi);
        }
    }
    if (!ok) return;
    if (sum == 0.f) o *= 1.f / sum;  // only scores of -inf: NaN
    const int64_t at = row_at(a, bat, kvh, q0 + r) * D + d;
    if constexpr (OF32) {
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.o) + at) = o;
    } else {
        bf16x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = static_cast<__bf16>(o[e]);
        *reinterpret_cast<bf16x4_t*>(static_cast<__bf16*>(a.o) + at) = h;
    }
    if (a.lse != nullptr && d == 0) a.lse[lse_at(a, bat, kvh, q0 + r)] = (top + __log2f(sum)) * 0.69314718055994530942f;
}

template <int D, bool OF32>
hipError_t launch(const Kv8AttnArgs& a, hipStream_t s) {
    const int64_t total = static_cast<int64_t>(a.n_tiles) * a.B * a.Hk, split = total - a.n_whole;
    // (no more than one split tile a CU: the split is there for the CUs that a round leaves idle)
    if (split > kCUs) return hipErrorInvalidValue;
    const unsigned grid = static_cast<unsigned>(a.n_whole + split * a.parts);
    const hipError_t e = a.few == 4   ? launch_with(attn_kv8_few_kernel<D, OF32, 4>, dim3(grid), 256, s, a)
                         : a.few == 8 ? launch_with(attn_kv8_few_kernel<D, OF32, 8>, dim3(grid), 512, s, a)
                                      : launch_with(attn_kv8_tile_kernel<D, OF32>, dim3(grid), kTileThreads, s, a);
    if (e != hipSuccess || split == 0) return e;
    const int rows = min(a.rows, a.few ? kKv8FewRows : kTileRows);
    auto wgs = [&](int rpw) { return dim3((rows + rpw - 1) / rpw, static_cast<unsigned>(split)); };
    constexpr int kOne = kMergeThreads / (D / 4), kEight = kOne / 8;  // rows of a workgroup
    return a.few          ? launch_with(attn_kv8_merge_kernel<D, OF32, kKv8FewRows, 8>, wgs(kEight), kMergeThreads, s, a)
           : a.parts > 16 ? launch_with(attn_kv8_merge_kernel<D, OF32, kTileRows, 8>, wgs(kEight), kMergeThreads, s, a)
                          : launch_with(attn_kv8_merge_kernel<D, OF32, kTileRows, 1>, wgs(kOne), kMergeThreads, s, a);
}

}  // namespace

hipError_t launch_attn_kv8(Kv8AttnArgs a, int head_dim, hipStream_t s) {
    a.by_group = FastDiv(static_cast<uint32_t>(a.group));
    a.by_parts = FastDiv(static_cast<uint32_t>(a.parts));
    a.by_tiles = FastDiv(static_cast<uint32_t>(a.n_tiles));
    a.by_heads = FastDiv(static_cast<uint32_t>(a.Hk));
    a.part_blocks = a.n_kblocks / a.parts;
    a.more_part_blocks = a.n_kblocks % a.parts;
    const int blocks = (a.rows + 31) / 32;
    a.row_blocks = blocks / a.n_tiles;
    a.more_row_blocks = blocks % a.n_tiles;
    if (head_dim == 128) return a.o_f32 ? launch<128, true>(a, s) : launch<128, false>(a, s);
    if (head_dim == 64) return a.o_f32 ? launch<64, true>(a, s) : launch<64, false>(a, s);
    return hipErrorInvalidValue;
}

}  // namespace tmk
