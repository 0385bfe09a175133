// The norms before and after a branch of a block, with gate, residual and modulation, for gfx950.
//
// The student keeps the blocks of its WAN2.1 teacher (TalkingMachines, Sec. 4.1): a branch's output is gated by frame
// into the residual stream, which is normalised and modulated by frame for the next branch.
//     z = post(y) post_weight,  r = x + gate z,  h = (pre(r) pre_weight + pre_bias) (1 + scale) + shift
// with layer(v) = (v - mean) / sqrt(var + eps), rms(v) = v / sqrt(mean of squares + eps). Backward, with n = pre(r), v =
// post(y), t = dh (1 + scale) pre_weight, u = dx gate post_weight:
//     dx = dr + (t - mean t - n mean(t n)) / sigma_r,  dy = (u - mean u - v mean(u v)) / sigma_y
// (the means of t and u for a layer norm only), and from the sums over a group's rows of dh, dh n and dx v the gradients of
// all vectors.
//
// Bound by HBM: each element is read and written once, a row stays in registers between its sums, of which a layer norm
// takes two, one after the other (the variance from centred values). Measured: 4680 x 5120 into an fp32
// stream (287 MB) 58 us; 12150 x 1024 in bf16, both norms, (99 MB) 18 us; the backward of 32760 x 5120 (3.0 GB) 624 us,
// 4.9 TB/s in the kernel (a device copy of that size: 4.8); one token 3 us.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "tm_device.h"
#include "tm_internal.h"

namespace tmk {
namespace {

typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;

// Four neighbouring elements of a row in memory, and as fp32.
template <typename T>
struct Four;
template <>
struct Four<float> {
    typedef f32x4_t raw;
};
template <>
struct Four<__bf16> {
    typedef bf16x4_t raw;
};
template <typename T>
__device__ __forceinline__ f32x4_t as_f32(typename Four<T>::raw v) {
    return f32x4_t{static_cast<float>(v[0]), static_cast<float>(v[1]), static_cast<float>(v[2]), static_cast<float>(v[3])};
}
template <typename T>
__device__ __forceinline__ typename Four<T>::raw as_raw(f32x4_t v) {
    typename Four<T>::raw w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = static_cast<T>(v[e]);
    return w;
}
// Element `col` on of a row that begins at element `row` of p: the row is the same in all lanes and stays in scalar
// registers, the lane's part is a 32-bit offset.
template <typename T, typename P>
__device__ __forceinline__ auto* four_at(P* p, int64_t row, uint32_t col) {
    using B = std::conditional_t<std::is_const_v<P>, const char, char>;
    using R = std::conditional_t<std::is_const_v<P>, const typename Four<T>::raw, typename Four<T>::raw>;
    return reinterpret_cast<R*>(reinterpret_cast<B*>(p) + row * static_cast<int64_t>(sizeof(T)) + col * static_cast<uint32_t>(sizeof(T)));
}
template <typename T>
__device__ __forceinline__ typename Four<T>::raw load4(const void* p, int64_t row, uint32_t col) {
    return *four_at<T>(p, row, col);
}
template <typename T>
__device__ __forceinline__ void store4(void* p, int64_t row, uint32_t col, f32x4_t v) {
    *four_at<T>(p, row, col) = as_raw<T>(v);
}
// The same past the caches' order of use (the forward's outputs: 56.7 for 59.7 us for the 480p chunk; the backward
// writes the way it came, 640 for 648 us).
template <typename T>
__device__ __forceinline__ void store4_once(void* p, int64_t row, uint32_t col, f32x4_t v) {
    __builtin_nontemporal_store(as_raw<T>(v), four_at<T>(p, row, col));
}

// v of the lane that the DPP control CTRL names (0 where there is none, or where ROWS leaves the row out), added.
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_dpp(float v) {
    const int moved = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, true);
    return v + __builtin_bit_cast(float, moved);
}
// The sum over 16 lanes in lane 15 of each row of them, and over the wave in lane 63: row_shr 1, 2, 4, 8, then
// row_bcast 15 and 31. (A shuffle through LDS takes ten times as long as one of these steps, and a row's
// statistics wait for three such sums, one after the other.)
__device__ __forceinline__ float row_sum(float v) {
    v = add_dpp<0x111, 0xf>(v);
    v = add_dpp<0x112, 0xf>(v);
    v = add_dpp<0x114, 0xf>(v);
    return add_dpp<0x118, 0xf>(v);
}
__device__ __forceinline__ float wave_sum(float v) {
    v = row_sum(v);
    v = add_dpp<0x142, 0xa>(v);
    return add_dpp<0x143, 0xc>(v);
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

constexpr int kMaxWaves = 16;

// Sums of N values over the workgroup, the same in every lane, in a fixed order. `slots`: N * kMaxWaves
// floats that no wave of the workgroup still reads, zeros where there is no wave.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], lds_float* slots, int waves, int wave, int lane) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if (waves == 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = lane_value(v[k], 63);
        return;
    }
    if (lane == 63) {
#pragma unroll
        for (int k = 0; k < N; ++k) slots[k * kMaxWaves + wave] = v[k];
    }
    __syncthreads();
    float s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = slots[k * kMaxWaves + (lane & 15)];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane_value(row_sum(s[k]), 15);
}

// One row per workgroup, four neighbouring elements a lane, U times. ROWS > 1: a row per wave, for rows so short that
// starting a workgroup takes longer than its bytes (88311 rows of 128, bf16: 18.4 us, 22.2 with a workgroup each; of 256
// fp32 to bf16 25.5 and 22.4, so these stay).
template <typename S, typename A, int U, int ROWS>
__global__ __launch_bounds__(ROWS > 1 ? ROWS * 64 : 1024) void block_norm_kernel(const BlockNormArgs a) {
    __shared__ float smem[4 * kMaxWaves];
    lds_float* const L = (lds_float*)smem;
    const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int T = ROWS > 1 ? 64 : blockDim.x, waves = T / 64, tid = ROWS > 1 ? lane : threadIdx.x;
    const int wave = ROWS > 1 ? 0 : in_group, row = a.row0 + blockIdx.x * ROWS + (ROWS > 1 ? in_group : 0);
    if (ROWS > 1 && row >= a.rows) return;
    if (waves > 1 && tid < 4 * kMaxWaves) L[tid] = 0.f;
    const int64_t base = static_cast<int64_t>(row) * a.E;
    const int64_t mod = a.tg.row(row) * a.E;
    f32x4_t x[U];
    bool in[U];
    int col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        col[u] = (u * T + tid) * 4;
        in[u] = col[u] < a.E;
        x[u] = in[u] ? as_f32<S>(load4<S>(a.x, base, col[u])) : f32x4_t{};
    }
    typename Four<A>::raw y_raw[U];
    f32x4_t gate[U], scale[U], shift[U];
    const f32x4_t one = f32x4_t{1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        y_raw[u] = typename Four<A>::raw{};
        gate[u] = one;
        scale[u] = shift[u] = f32x4_t{};
        if (!in[u]) continue;
        if (a.y != nullptr) y_raw[u] = load4<A>(a.y, base, col[u]);
        if (a.gate != nullptr) gate[u] = load4<float>(a.gate, mod, col[u]);
        if (a.scale != nullptr) {
            scale[u] = load4<float>(a.scale, mod, col[u]);
            shift[u] = load4<float>(a.shift, mod, col[u]);
        }
    }
    if (waves > 1) __syncthreads();  // the slots are clear
    // Normalised values of v over the row, in place: (v - mean) / sqrt(var + eps) with the variance from the
    // centred values, or v / sqrt(mean of squares + eps); zeros stay where the row has ended.
    auto normalise = [&](f32x4_t (&v)[U], int kind, lds_float* slots) __attribute__((always_inline)) {
        if (kind == kNormLayer) {
            float s[1] = {0.f};
#pragma unroll
            for (int u = 0; u < U; ++u) s[0] += (v[u][0] + v[u][1]) + (v[u][2] + v[u][3]);
            group_sum(s, slots, waves, wave, lane);
            const float mean = s[0] * a.inv_E;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = in[u] ? v[u][e] - mean : 0.f;
        }
        float q[1] = {0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[0] = fmaf(v[u][e], v[u][e], q[0]);
        group_sum(q, slots + kMaxWaves, waves, wave, lane);
        const float by = 1.f / sqrtf(fmaf(q[0], a.inv_E, a.eps));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] *= by;
    };
    if (a.y != nullptr) {
        f32x4_t z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) z[u] = as_f32<A>(y_raw[u]);
        if (a.post != kNormNone) normalise(z, a.post, L);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            f32x4_t g = gate[u];
            if (a.post_weight != nullptr) g *= load4<float>(a.post_weight, 0, col[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[u][e] = fmaf(g[e], z[u][e], x[u][e]);
            store4_once<S>(a.r, base, col[u], x[u]);
        }
    }
    if (a.pre == kNormNone) return;
    normalise(x, a.pre, L + 2 * kMaxWaves);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!in[u]) continue;
        f32x4_t m = x[u];
        if (a.pre_weight != nullptr) m *= load4<float>(a.pre_weight, 0, col[u]);
        if (a.pre_bias != nullptr) m += load4<float>(a.pre_bias, 0, col[u]);
        if (a.scale != nullptr) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = fmaf(m[e], scale[u][e], m[e]) + shift[u][e];
        }
        store4_once<A>(a.h, base, col[u], m);
    }
}

// One part of the rows (of one group) per workgroup, one row after the other; each lane keeps the sums over
// rows of its columns.
template <typename S, typename A, int U>
__global__ __launch_bounds__(1024) void block_norm_bwd_kernel(const BlockNormBwdArgs a) {
    // Rows of more than 8192 (U = 4) leave no registers for all of it: a sum lives in LDS, and the vectors are
    // read anew for each row.
    constexpr bool WIDE = U > 2;
    __shared__ float smem[2 * 8 * kMaxWaves];
    __shared__ __attribute__((aligned(16))) float wide[WIDE ? kMaxNormWidth : 4];
    const int T = blockDim.x, waves = T / 64, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < 2 * 8 * kMaxWaves; i += T) ((lds_float*)smem)[i] = 0.f;  // no wave's slots stay so
    __syncthreads();
    int32_t b, t0, t1;
    int64_t mod;
    a.parts.of(blockIdx.x, b, mod, t0, t1);
    const bool has_pre = a.pre != kNormNone, has_y = a.y != nullptr, has_dr = a.dr != nullptr;
    const bool pre_layer = a.pre == kNormLayer, post_layer = a.post == kNormLayer;
    int col[U];
    bool in[U];
    const f32x4_t one = f32x4_t{1.f, 1.f, 1.f, 1.f};
    // (1 + scale) pre_weight and gate post_weight of a lane's columns
    auto load_by_pre = [&](int u) __attribute__((always_inline)) {
        f32x4_t v = one;
        if (in[u]) {
            if (a.scale != nullptr) v += load4<float>(a.scale, mod * a.E, col[u]);
            if (a.pre_weight != nullptr) v *= load4<float>(a.pre_weight, 0, col[u]);
        }
        return v;
    };
    auto load_by_post = [&](int u) __attribute__((always_inline)) {
        f32x4_t v = one;
        if (in[u]) {
            if (a.gate != nullptr) v = load4<float>(a.gate, mod * a.E, col[u]);
            if (a.post_weight != nullptr) v *= load4<float>(a.post_weight, 0, col[u]);
        }
        return v;
    };
    f32x4_t by_pre_kept[WIDE ? 1 : U], by_post_kept[WIDE ? 1 : U];
    f32x4_t sum_dh[WIDE ? 1 : U], sum_dhn[U], sum_av[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        col[u] = (u * T + tid) * 4;
        in[u] = col[u] < a.E;
        sum_dhn[u] = sum_av[u] = f32x4_t{};
        if (WIDE) {
            if (in[u]) *(lds_f32x4_t*)((lds_float*)wide + col[u]) = f32x4_t{};
        } else {
            by_pre_kept[u] = load_by_pre(u);
            by_post_kept[u] = load_by_post(u);
            sum_dh[u] = f32x4_t{};
        }
    }
    auto by_pre = [&](int u) __attribute__((always_inline)) { return WIDE ? load_by_pre(u) : by_pre_kept[WIDE ? 0 : u]; };
    auto by_post = [&](int u) __attribute__((always_inline)) { return WIDE ? load_by_post(u) : by_post_kept[WIDE ? 0 : u]; };
    for (int t = t0; t < t1; ++t) {
        // (sums of a row in slots that the row before does not use: a wave may still read those)
        lds_float* const L = (lds_float*)smem + (t & 1) * 8 * kMaxWaves;
        const int64_t base = (static_cast<int64_t>(b) * a.parts.n + t) * a.E;
        // (the columns anew for each row: the compiler would keep an address of each tensor for each of them)
        const int lane_now = fresh_thread_index();
#pragma unroll
        for (int u = 0; u < U; ++u) col[u] = (u * T + lane_now) * 4;
        // kept as they come, and turned into fp32 where they are used. (Loads a row ahead were no faster: 653 for
        // 655 us for the 480p clip, with 31 registers more.)
        typename Four<S>::raw r_raw[U], dr_raw[U];
        typename Four<A>::raw dh_raw[U], y_raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r_raw[u] = dr_raw[u] = typename Four<S>::raw{};
            dh_raw[u] = y_raw[u] = typename Four<A>::raw{};
            if (!in[u]) continue;
            if (has_pre) {
                r_raw[u] = load4<S>(a.r, base, col[u]);
                dh_raw[u] = load4<A>(a.dh, base, col[u]);
            }
            if (has_dr) dr_raw[u] = load4<S>(a.dr, base, col[u]);
            if (has_y) y_raw[u] = load4<A>(a.y, base, col[u]);
        }
        float mean_t = 0.f, mean_r = 0.f, mean_y = 0.f;
        if (pre_layer || post_layer) {
            float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const f32x4_t r = as_f32<S>(r_raw[u]), d = as_f32<A>(dh_raw[u]) * by_pre(u), y = as_f32<A>(y_raw[u]);
                s[0] += (r[0] + r[1]) + (r[2] + r[3]);
                s[1] += (d[0] + d[1]) + (d[2] + d[3]);
                s[2] += (y[0] + y[1]) + (y[2] + y[3]);
            }
            group_sum(s, L, waves, wave, lane);
            if (pre_layer) {
                mean_r = s[0] * a.inv_E;
                mean_t = s[1] * a.inv_E;
            }
            if (post_layer) mean_y = s[2] * a.inv_E;
        }
        // (zeros stay where the row has ended)
        auto r_centred = [&](int u, int e) __attribute__((always_inline)) {
            return in[u] ? static_cast<float>(r_raw[u][e]) - mean_r : 0.f;
        };
        auto y_centred = [&](int u, int e) __attribute__((always_inline)) {
            return in[u] ? static_cast<float>(y_raw[u][e]) - mean_y : 0.f;
        };
        float pre_by = 1.f, post_by = 1.f, along_r = 0.f;
        if (has_pre || a.post != kNormNone) {
            float s[3] = {0.f, 0.f, 0.f};  // squares of r and y, and t r
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const f32x4_t d = as_f32<A>(dh_raw[u]) * by_pre(u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float r = r_centred(u, e), y = y_centred(u, e);
                    s[0] = fmaf(r, r, s[0]);
                    s[1] = fmaf(d[e], r, s[1]);
                    s[2] = fmaf(y, y, s[2]);
                }
            }
            group_sum(s, L + 3 * kMaxWaves, waves, wave, lane);
            if (has_pre) {
                pre_by = 1.f / sqrtf(fmaf(s[0], a.inv_E, a.eps));
                along_r = s[1] * pre_by * a.inv_E;  // mean of t n
            }
            if (a.post != kNormNone) post_by = 1.f / sqrtf(fmaf(s[2], a.inv_E, a.eps));
        }
        f32x4_t dx[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            dx[u] = as_f32<S>(dr_raw[u]);
            if (has_pre) {
                const f32x4_t d = as_f32<A>(dh_raw[u]), by = by_pre(u);
                f32x4_t sum = WIDE ? f32x4_t{} : sum_dh[WIDE ? 0 : u];
                if (WIDE && in[u]) sum = *(lds_f32x4_t*)((lds_float*)wide + col[u]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float n = r_centred(u, e) * pre_by;
                    sum[e] += d[e];
                    sum_dhn[u][e] = fmaf(d[e], n, sum_dhn[u][e]);
                    dx[u][e] = fmaf(pre_by, fmaf(d[e], by[e], -mean_t) - n * along_r, dx[u][e]);
                }
                if (!WIDE)
                    sum_dh[WIDE ? 0 : u] = sum;
                else if (in[u])
                    *(lds_f32x4_t*)((lds_float*)wide + col[u]) = sum;
            }
            if (in[u]) store4<S>(a.dx, base, col[u], dx[u]);
        }
        if (!has_y) continue;
        float mean_u = 0.f, along = 0.f, s[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const f32x4_t by = by_post(u);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = y_centred(u, e) * post_by;
                sum_av[u][e] = fmaf(dx[u][e], v, sum_av[u][e]);
                dx[u][e] = in[u] ? dx[u][e] * by[e] : 0.f;
                s[0] += dx[u][e];
                s[1] = fmaf(dx[u][e], v, s[1]);
            }
        }
        if (a.post != kNormNone) {
            group_sum(s, L + 6 * kMaxWaves, waves, wave, lane);
            mean_u = post_layer ? s[0] * a.inv_E : 0.f;
            along = s[1] * a.inv_E;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f32x4_t d = dx[u];
            // (without a norm dy is u, whatever y holds: a product of an infinite y with an `along` of 0 would be NaN)
            if (a.post != kNormNone) {
#pragma unroll
                for (int e = 0; e < 4; ++e) d[e] = post_by * ((dx[u][e] - mean_u) - y_centred(u, e) * post_by * along);
            }
            if (in[u]) store4<A>(a.dy, base, col[u], d);
        }
    }
    if (a.part == nullptr) return;
    float* out = a.part + static_cast<int64_t>(blockIdx.x) * kNormSums * a.E;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!in[u]) continue;
        store4<float>(out, 0, col[u], WIDE ? *(lds_f32x4_t*)((lds_float*)wide + col[u]) : sum_dh[WIDE ? 0 : u]);
        store4<float>(out, a.E, col[u], sum_dhn[u]);
        store4<float>(out, 2 * a.E, col[u], sum_av[u]);
    }
}

// COLS columns of one sum, LANES threads a column, which deal out the parts (8 loads of each in flight). The first
// workgroups take the totals.
template <int COLS, int LANES>
__global__ __launch_bounds__(COLS * LANES) void column_sums_kernel(const ColumnSums a) {
    __shared__ float sums[2][LANES][COLS];
    const int blocks = (a.E + COLS - 1) / COLS;
    const int c = threadIdx.x % COLS, l = threadIdx.x / COLS;
    const int e = static_cast<int>(blockIdx.x % blocks) * COLS + c;
    const int which = static_cast<int>(blockIdx.x / blocks);
    const int64_t stride = static_cast<int64_t>(a.vectors) * a.E;
    const bool in = e < a.E;
    float s = 0.f, s_w = 0.f;
    if (which < a.n_total) {
        const TotalSum& o = a.total[which];
        const float* at = a.part + static_cast<int64_t>(o.v) * a.E + e;
        const int n = a.parts.filled();
        if (in) {
            if (o.mod != nullptr) {
#pragma unroll 8
                for (int i = l; i < n; i += LANES) {
                    const int b = a.by_each.of(i), j = a.by_parts.of(i - b * a.parts.each() + a.parts.before);
                    const int64_t mod = static_cast<int64_t>(b) * a.parts.groups + a.parts.g0 + j;
                    s = fmaf(at[i * stride], o.mod[mod * a.E + e] + o.add, s);
                }
            } else {
#pragma unroll 8
                for (int i = l; i < n; i += LANES) s += at[i * stride];
            }
        }
        sums[0][l][c] = s;
        __syncthreads();
        if (l > 0 || !in) return;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < LANES; ++i) s += sums[0][i][c];
        o.out[e] = s;
        return;
    }
    const int rows = a.parts.B * a.parts.touched;
    if (which >= a.n_total + a.n_group * rows) {
        // a group that the run does not touch: a workgroup for each, over all columns
        const int left = a.parts.groups - a.parts.touched;
        const int i = static_cast<int>(blockIdx.x) - blocks * (a.n_total + a.n_group * rows);
        const int r = i % (a.parts.B * left), b = r / left, j = r % left;
        float* out = a.group[i / (a.parts.B * left)].out +
                     (static_cast<int64_t>(b) * a.parts.groups + (j < a.parts.g0 ? j : j + a.parts.touched)) * a.E;
        for (int k = threadIdx.x; k < a.E; k += COLS * LANES) out[k] = 0.f;
        return;
    }
    const int touched = (which - a.n_total) % rows;
    const GroupSum& o = a.group[(which - a.n_total) / rows];
    const int b = touched / a.parts.touched, j = touched % a.parts.touched, row = b * a.parts.groups + a.parts.g0 + j;
    if (in) {
        int32_t i0, i1;
        a.parts.of_group(b, j, i0, i1);
        const float* v = a.part + static_cast<int64_t>(o.v) * a.E + e;
#pragma unroll 8
        for (int i = i0 + l; i < i1; i += LANES) s += v[i * stride];
        if (o.w >= 0) {
            const float* w = a.part + static_cast<int64_t>(o.w) * a.E + e;
#pragma unroll 8
            for (int i = i0 + l; i < i1; i += LANES) s_w += w[i * stride];
        }
    }
    if (LANES > 1) {
        sums[0][l][c] = s;
        sums[1][l][c] = s_w;
        __syncthreads();
        if (l > 0) return;
        s = s_w = 0.f;
#pragma unroll
        for (int i = 0; i < LANES; ++i) {
            s += sums[0][i][c];
            s_w += sums[1][i][c];
        }
    }
    if (!in) return;
    if (o.mul != nullptr) s *= o.mul[e];
    if (o.w >= 0) s = fmaf(s_w, o.mul_w[e], s);
    o.out[static_cast<int64_t>(row) * a.E + e] = s;
}

// The sums per group of many groups of at most 4 parts each, four columns a thread: a row of a modulation's gradient per
// workgroup and 4 * blockDim.x columns. Bound by HBM where the kernel above, a column a thread, has too little on its way
// (8000 groups of one row, 5120 wide, bf16 and fp32: the backward 972 us with it, 570 so).
__global__ __launch_bounds__(256) void group_sums_kernel(const ColumnSums a) {
    const int blocks = (a.E / 4 + blockDim.x - 1) / blockDim.x, rows = a.parts.B * a.parts.groups;
    const int col = (static_cast<int>(blockIdx.x % blocks) * blockDim.x + threadIdx.x) * 4;
    const int row = static_cast<int>(blockIdx.x / blocks) % rows, which = static_cast<int>(blockIdx.x / blocks) / rows;
    if (col >= a.E) return;
    const GroupSum& o = a.group[which];
    const int b = row / a.parts.groups, j = row % a.parts.groups - a.parts.g0;
    f32x4_t s = f32x4_t{}, s_w = f32x4_t{};
    if (j >= 0 && j < a.parts.touched) {
        const int64_t stride = static_cast<int64_t>(a.vectors) * a.E;
        int32_t i0, i1;
        a.parts.of_group(b, j, i0, i1);
        for (int i = i0; i < i1; ++i) {
            s += load4<float>(a.part, i * stride + static_cast<int64_t>(o.v) * a.E, col);
            if (o.w >= 0) s_w += load4<float>(a.part, i * stride + static_cast<int64_t>(o.w) * a.E, col);
        }
        if (o.mul != nullptr) s *= load4<float>(o.mul, 0, col);
        if (o.w >= 0) {
            const f32x4_t by = load4<float>(o.mul_w, 0, col);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fmaf(s_w[e], by[e], s[e]);
        }
    }
    store4<float>(o.out, static_cast<int64_t>(row) * a.E, col, s);
}

template <int COLS, int LANES>
hipError_t launch_sums(const ColumnSums& a, hipStream_t s) {
    const int64_t sums = a.n_total + static_cast<int64_t>(a.n_group) * a.parts.B * a.parts.touched;
    const int64_t zeros = static_cast<int64_t>(a.n_group) * a.parts.B * (a.parts.groups - a.parts.touched);
    return launch_with(column_sums_kernel<COLS, LANES>,
                       dim3(static_cast<unsigned>((a.E + COLS - 1) / COLS * sums + zeros)), COLS * LANES, s, a);
}

}  // namespace

template <typename S, typename A, int U, int ROWS>
static hipError_t launch_rows(BlockNormArgs a, int threads, hipStream_t s) {
    // Thread numbers are 32 bits wide: very many rows take several launches.
    const int64_t most = (int64_t(1) << 31) / threads;
    for (int64_t at = 0; at < a.rows; at += most) {
        a.row0 = static_cast<int32_t>(at);
        const int64_t groups = (std::min(most, a.rows - at) + ROWS - 1) / ROWS;
        const hipError_t e = launch_with(block_norm_kernel<S, A, U, ROWS>, dim3(static_cast<unsigned>(groups)), threads * ROWS, s, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_block_norm(const BlockNormArgs& a, bool stream_f32, bool act_f32, hipStream_t s) {
    int U, threads;
    block_norm_shape(a.E, false, &U, &threads);
#define TM_NORM_CASE(U_, ROWS_)                                                                                      \
    if (U == U_ && (ROWS_ == 1 || a.E <= 128)) {                                                                     \
        if (stream_f32)                                                                                              \
            return act_f32 ? launch_rows<float, float, U_, ROWS_>(a, threads, s)                                     \
                           : launch_rows<float, __bf16, U_, ROWS_>(a, threads, s);                                   \
        return act_f32 ? launch_rows<__bf16, float, U_, ROWS_>(a, threads, s)                                        \
                       : launch_rows<__bf16, __bf16, U_, ROWS_>(a, threads, s);                                      \
    }
    TM_NORM_CASE(1, 4)
    TM_NORM_CASE(1, 1)
    TM_NORM_CASE(2, 1)
    TM_NORM_CASE(5, 1)
#undef TM_NORM_CASE
    return hipErrorInvalidValue;
}

hipError_t launch_block_norm_bwd(const BlockNormBwdArgs& a, bool stream_f32, bool act_f32, hipStream_t s) {
    int U, threads;
    block_norm_shape(a.E, true, &U, &threads);
    const dim3 grid(a.parts.filled());
#define TM_NORM_CASE(U_)                                                                                 \
    if (U == U_) {                                                                                       \
        if (stream_f32)                                                                                  \
            return act_f32 ? launch_with(block_norm_bwd_kernel<float, float, U_>, grid, threads, s, a)       \
                           : launch_with(block_norm_bwd_kernel<float, __bf16, U_>, grid, threads, s, a);     \
        return act_f32 ? launch_with(block_norm_bwd_kernel<__bf16, float, U_>, grid, threads, s, a)          \
                       : launch_with(block_norm_bwd_kernel<__bf16, __bf16, U_>, grid, threads, s, a);        \
    }
    TM_NORM_CASE(1)
    TM_NORM_CASE(2)
    TM_NORM_CASE(4)
#undef TM_NORM_CASE
    return hipErrorInvalidValue;
}

static hipError_t launch_for(int parts, const ColumnSums& a, hipStream_t s) {
    int columns, threads;
    column_sums_shape(parts, a.E, &columns, &threads);
    switch (threads) {
        case 1: return launch_sums<64, 1>(a, s);
        case 4: return launch_sums<64, 4>(a, s);
        case 16: return launch_sums<64, 16>(a, s);
        case 32: return launch_sums<32, 32>(a, s);
    }
    return launch_sums<16, 64>(a, s);
}

hipError_t launch_column_sums(const ColumnSums& a, hipStream_t s) {
    ColumnSums t = a, g = a;
    t.by_parts = g.by_parts = FastDiv(a.parts.per_group);
    t.by_each = g.by_each = FastDiv(a.parts.each());
    // totals over many parts have a launch of their own, with more threads a column, if the groups have few
    if (a.n_total > 0 && (a.parts.filled() > std::max(512, a.parts.per_group) || a.n_group == 0)) {
        t.n_group = 0;
        g.n_total = 0;
        const hipError_t e = launch_for(a.parts.filled(), t, s);
        if (e != hipSuccess || a.n_group == 0) return e;
    }
    if (g.n_total == 0 && a.parts.per_group <= 4 && a.parts.filled() > 512) {
        const int threads = std::min(256, (a.E / 4 + 63) / 64 * 64);
        const int64_t blocks = (a.E / 4 + threads - 1) / threads;
        return launch_with(group_sums_kernel, dim3(static_cast<unsigned>(blocks * a.n_group * a.parts.B * a.parts.groups)), threads, s, g);
    }
    return launch_for(g.n_total > 0 ? a.parts.filled() : a.parts.per_group, g, s);
}

}  // namespace tmk
