// Layout of the 8-bit KV cache, shared by the kernels that write and read it
// (kv8_cache.hip, attn_kv8.hip). Not part of the public ABI.
//
// Tokens come in blocks of 64 (kCacheBlock) that belong to one chunk each. A
// (batch, key head, block) holds the codes of K and of V, 64 * D bytes each, and
// a scale of each. Codes are held as code + 128, and in the order in which the
// MFMAs of the attention take them: 16-byte pieces, one per lane of a wave, so
// that a wave's load of an operand is one contiguous KB.
//   K piece (kb, s, lane): key 32 kb + k_perm(lane % 32), dimensions 32 s + 8 hw
//     .. + 7 and 32 s + 16 + 8 hw .. + 7 (hw = lane / 32): the lane's elements of
//     the score MFMAs of dimensions 32 s .. + 15 and 32 s + 16 .. + 31;
//   V piece (kb, d, lane): dimension 32 d + lane % 32, keys 32 kb + 8 hw .. + 7
//     and 32 kb + 16 + 8 hw .. + 7: the lane's elements of the P V MFMAs of those
//     two groups of 16 keys.
// Piece n = (kb * (D / 32) + s or d) * 64 + lane sits at byte 16 n of the block.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tm_device.h"
#include "tm_internal.h"

namespace tmk {

constexpr uint32_t kCodeZero = 0x80;  // the byte of code 0

// Bytes 0 .. 3 of `lo` are selected by 0 .. 3, those of `hi` by 4 .. 7.
__device__ __forceinline__ uint32_t pick_bytes(uint32_t hi, uint32_t lo, uint32_t sel) {
    return __builtin_amdgcn_perm(hi, lo, sel);
}

// r[i] byte j -> r[j] byte i.
__device__ __forceinline__ void transpose4x4(uint32_t (&r)[4]) {
    const uint32_t a = pick_bytes(r[1], r[0], 0x05010400), b = pick_bytes(r[1], r[0], 0x07030602);
    const uint32_t c = pick_bytes(r[3], r[2], 0x05010400), d = pick_bytes(r[3], r[2], 0x07030602);
    r[0] = pick_bytes(c, a, 0x05040100);
    r[1] = pick_bytes(c, a, 0x07060302);
    r[2] = pick_bytes(d, b, 0x05040100);
    r[3] = pick_bytes(d, b, 0x07060302);
}

}  // namespace tmk
