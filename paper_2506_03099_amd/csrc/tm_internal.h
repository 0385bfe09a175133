// Internal interface between the host-side API (tm_api.cpp) and the HIP
// kernels. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tmk {

constexpr int kMaxRanges = 16;  // key ranges of one query segment (>= TM_MAX_WINDOW + 2)

// Rows per query tile of each attention kernel; the host needs them to count
// tiles per chunk.
constexpr int kTileRowsBf16 = 256;
constexpr int kKeyTile = 64;  // keys per tile of the bf16 kernel
constexpr int kCUs = 256;     // compute units of the target; one bf16 workgroup on each at a time

// Partial result of one wave (32 query rows) over a share of the keys: O in
// the MFMA layout, then each row's running max and row sum, in floats.
__host__ __device__ constexpr int64_t part_floats(int head_dim) { return 32 * int64_t(head_dim) + 128; }

// Key split of the query tiles that do not fill a whole round of the chip's
// CUs: `whole` tiles (a multiple of kCUs) run over all their keys, each of the
// others is shared out over `parts` workgroups, whose partial results a second
// kernel merges (without a workspace for these: the parts run one after the
// other in a workgroup, to the same bits). parts = 1: no split.
constexpr int kMaxParts = 16;
struct AttnSplit {
    int64_t whole = 0;
    int parts = 1;
};

// The fp32 kernel's workgroups have 4 waves (8 with 8 key groups, head_dim 64
// only), 32 query rows each; the waves are shared out between key groups and
// query rows, so a query tile has 32 * waves / key_groups rows.
constexpr int f32_tile_rows(int key_groups) { return 32 * (key_groups == 8 ? 8 : 4) / key_groups; }
// Waves (32 query rows and a share of the keys each) that fill the chip: two
// on every SIMD of its 256 CUs.
constexpr int64_t kF32FillWaves = 2 * 4 * 256;

// KV-cache pools are organised in blocks of this many token rows. The V pool
// stores each block dimension-major: [D][kCacheBlock] per (batch, head, block),
// so that the attention kernel's V^T operand is a contiguous 16-byte read.
constexpr int kCacheBlock = 64;
// Cache regions (c_0 and every ring slot) start on multiples of this many
// tokens, so that every 16-byte group of a V block row belongs to one region.
constexpr int kCacheAlign = 8;

// One attention launch. Element strides (not bytes) for batch, token and head.
// With v_blocked != 0, v is a cache V pool: element (token t, dim d) of a head
// sits at (t / 64) * 64 * D + d * 64 + t % 64 from the head's base, v_st is
// unused, and every key range starts on a multiple of kCacheAlign.
struct AttnArgs {
    const void* q;
    const void* k;
    const void* v;
    void* o;
    float* lse;  // [B, H, Lq] or null
    int64_t q_sb, q_st, q_sh;
    int64_t k_sb, k_st, k_sh;
    int64_t v_sb, v_st, v_sh;
    int64_t o_sb, o_st, o_sh;
    int32_t o_f32;  // bf16 kernel: store O as fp32 (the values before the final rounding)
    int32_t v_blocked;
    int32_t B, H, Lq;
    float scale_log2;  // softmax scale * log2(e)
    int32_t n_qtiles;  // query tiles per (batch, head)
    int32_t key_groups;  // fp32 kernel: shares of a tile's keys (1, 2, 4 or 8)
    int32_t n_whole;     // bf16 kernel: tiles (of all heads) that are not split
    int32_t parts;       // bf16 kernel: key shares of a split tile (1: none is split)
    float* part;         // bf16 kernel: [split tile][part][wave][part_floats], or null
    // mode 0: every query row of the buffer belongs to one chunk and sees the
    //         same key ranges (streaming form, or one chunk of a sequence);
    // mode 1: the buffer holds a whole sequence (row i = position i); each
    //         tile's chunk and key ranges follow from the geometry below.
    int32_t mode;
    int32_t n_ranges;  // mode 0
    int32_t n_ktiles;  // mode 0: 64-key tiles of all ranges
    int32_t range_begin[kMaxRanges];
    int32_t range_end[kMaxRanges];
    int32_t ref_tok;      // mode 1: R*T (clipped to the sequence)
    int32_t chunk_tok;    // mode 1: C*T
    int32_t window;       // mode 1: W
    int32_t seq_len;      // mode 1: tokens in the sequence
    int32_t ref_tiles;    // mode 1: query tiles of c_0
    int32_t chunk_tiles;  // mode 1: query tiles of a full chunk
};

hipError_t launch_attn_bf16(const AttnArgs& a, int head_dim, hipStream_t s);
hipError_t launch_attn_f32(const AttnArgs& a, int head_dim, hipStream_t s);

// Copy n_tok tokens of K and V from [B, n_tok, H, D] into the cache pools at
// token row `tok_offset` (a multiple of kCacheAlign): K into [B, H, capacity,
// D], V into [B, H, capacity / 64, D, 64]. The V columns from n_tok up to the
// next multiple of kCacheAlign are written as zeros. `capacity` is a multiple
// of kCacheBlock; elem_bytes is 2 or 4.
hipError_t launch_kv_append(const void* k_src, const void* v_src, void* k_pool, void* v_pool,
                            int B, int n_tok, int H, int D, int elem_bytes, int64_t capacity,
                            int64_t tok_offset, hipStream_t s);

// The same write of the chunk's V, while the chunk's queries (into q_out, same
// layout as q_src) and keys (into the K pool) are RMS-normalised per (token,
// head) row over D: x / sqrt(mean(x^2) + eps) * gain[h, :] (gain NULL: ones),
// in fp32, rounded to the element type. q_out may equal q_src.
hipError_t launch_qkv_produce(const void* q_src, const void* k_src, const void* v_src, void* q_out,
                              const float* q_gain, const float* k_gain, float eps, void* k_pool,
                              void* v_pool, int B, int n_tok, int H, int D, int elem_bytes,
                              int64_t capacity, int64_t tok_offset, hipStream_t s);

// Audio cross-attention of a run of latent-frame tokens (bf16). q, o: [B, n,
// H, D]; ak, av: [B, M, La, H, D] with La = F_a * A; face: [B, n] stream index
// per query token (ids outside [0, M) mean no face: zero output).
struct AudioArgs {
    const void* q;
    const void* ak;
    const void* av;
    const int32_t* face;
    void* o;
    int32_t B, n, H, M, La;
    int32_t T;             // query tokens per latent frame
    int32_t A;             // audio tokens per latent frame
    int32_t first_frame;   // latent frame of query row 0
    int32_t half_window;   // frames f - w .. f + w
    int32_t n_frames;      // latent frames the n rows span
    int32_t parts;         // workgroups per (batch, head, frame)
    int32_t max_keys_pad;  // most window keys of any frame, rounded up to 32
    int32_t o_f32;         // store o as fp32 (the values before the final rounding)
    float scale_log2;      // softmax scale * log2(e)
    int32_t n_cwg;         // compute workgroups (B * H * n_frames * parts, times M where each takes
                           // one stream); set by the launcher
    int32_t zrows;         // token rows per zero-fill workgroup; set by the launcher
    int32_t q_stage;       // queries (and bf16 output rows) staged in LDS; set by the launcher
};

// Most 32-row blocks of one frame per audio workgroup: a frame with more
// blocks is split over several workgroups, which take every parts-th block.
constexpr int kAudioBlocksPerPart = 64;

// LDS of one audio workgroup: a window of nk_pad keys as K rows and V rows of
// D bf16 each, then one word per wave (8), the face waves' row counts per
// segment (32), the count of one stream's rows (one word, padded to 16 bytes)
// and those rows compacted (16-bit indices). Staging the queries and the
// output through LDS adds one slot of 32 rows of D bf16 per wave.
constexpr size_t kAudioFaceLds = 4 * 8 + 4 * 32 + 16 + 2 * 32 * kAudioBlocksPerPart;
__host__ __device__ constexpr size_t audio_lds_bytes(int head_dim, int nk_pad) {
    return 2 * static_cast<size_t>(nk_pad) * head_dim * 2 + kAudioFaceLds;
}
__host__ __device__ constexpr size_t audio_stage_lds_bytes(int head_dim) {
    return static_cast<size_t>(8) * 32 * head_dim * 2;
}
constexpr size_t kAudioMaxLds = 160 * 1024;  // gfx950: 160 KiB of LDS per workgroup
// Most window keys (a multiple of 32) that fit: 288 at D = 128, 608 at D = 64.
template <int D>
constexpr int kAudioMaxKeys = static_cast<int>((kAudioMaxLds - kAudioFaceLds) / (2 * 2 * D)) / 32 * 32;

hipError_t launch_audio_attn_bf16(const AudioArgs& a, int head_dim, hipStream_t s);

// Backward of the whole-sequence attention (bf16): q, k, v, o, dout, dq, dk,
// dv are [B, L, H, D]; lse (natural log) and delta (written here) are fp32
// [B, H, L]. Query tiles of kBwdQTile rows and key tiles of kBwdKTile keys
// never straddle a chunk: ref tiles for c_0, then chunk tiles per chunk.
constexpr int kBwdQTile = 128;
constexpr int kBwdKTile = 128;
struct BwdArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* o;
    const float* lse;
    const void* dout;
    float* delta;
    void* dq;
    void* dk;
    void* dv;
    int32_t B, H, L;
    int32_t ref_tok, chunk_tok, window;  // R*T, C*T, W
    float scale, scale_log2;
    int32_t q_tiles, q_ref_tiles, q_chunk_tiles;
    int32_t k_tiles, k_ref_tiles, k_chunk_tiles;
    // Workgroups per key tile of c_0 and of the chunks, and per query tile (1:
    // the tile's own workgroup writes its result; else the partial sums of a
    // tile's parts, in fp32, are added up by another kernel).
    int32_t k_ref_parts, k_chunk_parts, q_parts;
    float* dkdv_part;  // [split key tile][part][wave][dK, dV][32 * D]
    float* dq_part;    // [query tile][part][wave][32 * D]
};
hipError_t launch_attn_bwd_bf16(const BwdArgs& a, int head_dim, hipStream_t s);

// The device-global workspace of the allocation-free backward: room for delta
// of B * H * L <= kBwdScratchFloats rows (8 MiB per GPU). bwd_scratch_address
// returns its address on the current device (looked up on the first call per
// device); kernels get that address, never the symbol.
constexpr int64_t kBwdScratchFloats = int64_t(1) << 21;
hipError_t bwd_scratch_address(float** out);

// Launches a kernel whose one argument is `args` by one call of the runtime (the launch syntax makes
// three, 0.15 us of a small call's 2.4).
template <typename Args>
hipError_t launch_with(void (*kernel)(Args), dim3 grid, unsigned threads, hipStream_t s, const Args& args) {
    void* params[] = {const_cast<Args*>(&args)};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), params, 0, s);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
}

// Division of 0 <= n < 2^31 by d, 1 <= d < 2^31: n * mul >> shift with mul = floor(2^shift / d) + 1 and
// shift = 31 + ceil(log2 d), exact since mul * d exceeds 2^shift by at most d <= 2^(shift - 31).
struct FastDiv {
    uint32_t mul = 0;
    int32_t shift = 0;
    FastDiv() = default;
    explicit FastDiv(uint32_t d) {
        int log2 = 0;
        while ((uint64_t(1) << log2) < d) ++log2;
        shift = 31 + log2;
        mul = static_cast<uint32_t>((uint64_t(1) << shift) / d + 1);
    }
    __host__ __device__ int32_t of(int32_t n) const {
        return static_cast<int32_t>(static_cast<uint64_t>(static_cast<uint32_t>(n)) * mul >> shift);
    }
};

// Rotary positions: (cos, sin) of every position and pair of the three axes, the
// frames' rows first, then the grid's rows, then its columns.
struct RopeTable {
    const float2* table;    // [frames][pairs_t], [grid_h][pairs_h], [grid_w][pairs_w]
    int32_t first_h, first_w;  // entries before the second and the third
    int32_t pairs_t, pairs_h, pairs_w;
    int32_t grid_w, frame_tokens;
    FastDiv by_w, by_frame;
};
constexpr int64_t kMaxRopeEntries = int64_t(1) << 28;  // of the table: 2 GiB, so that offsets fit 32 bits

// Rotation of q [B, n, H, D] and k [B, n, Hk, D] (Hk = 0: none) into q_out and
// k_out; row i is the token at position first_token + i.
struct RopeArgs {
    const unsigned char* q;
    const unsigned char* k;
    unsigned char* q_out;
    unsigned char* k_out;
    RopeTable table;
    int64_t first_token, n;
    int64_t tok0, tok_end;  // tokens of one launch; set by the launcher
    int32_t B, H, Hk;
    int32_t slices;  // threads that share a token's heads; set by the launcher
    float sign;      // of the angles: 1, or -1 for the backward pass
};
hipError_t launch_rope(const RopeArgs& a, int head_dim, int elem_bytes, bool halves, hipStream_t s);
hipError_t launch_rope_table(const int64_t (&rows)[3], const int (&pairs)[3], double theta, float* out, hipStream_t s);

// One chunk into the 8-bit cache (layout: tm_kv8.h): k, v [B, n_tok, Hk, D] in
// bf16, into the blocks of every (batch, key head) from first_blk on. The
// producer also takes q [B, n_tok, H, D] into q_out (which may be q), and
// RMS-normalises and, with turn, rotates q and k.
struct Kv8WriteArgs {
    const unsigned char* q;
    const unsigned char* k;
    const unsigned char* v;
    unsigned char* q_out;
    const float* q_gain;  // [H, D] or null
    const float* k_gain;  // [Hk, D] or null
    float eps;
    int32_t turn;
    RopeTable table;
    int64_t first_token;
    unsigned char* k_codes;  // [B, Hk, n_blocks][64 * D]
    unsigned char* v_codes;
    float* k_scale;  // [B, Hk, n_blocks]
    float* v_scale;
    int32_t B, n_tok, H, Hk;
    int32_t n_blocks;   // of 64 tokens per (batch, key head) of the cache
    int32_t first_blk;  // the chunk's first one
    int32_t n_blk;      // the chunk's; this and the next two set by the launcher
    int32_t q_slices;   // threads that share a token's query heads
    uint32_t q_wgs;     // workgroups for queries; those past them take K and V
};
hipError_t launch_kv8_write(Kv8WriteArgs a, int head_dim, bool produce, bool halves, hipStream_t s);

// A chunk of the 8-bit cache back into k_out, v_out [B, n_tok, Hk, D], bf16 or fp32.
struct Kv8ReadArgs {
    const unsigned char* k_codes;
    const unsigned char* v_codes;
    const float* k_scale;
    const float* v_scale;
    unsigned char* k_out;
    unsigned char* v_out;
    int32_t B, n_tok, Hk;
    int32_t n_blocks, first_blk;
    int32_t n_blk;  // set by the launcher
};
hipError_t launch_kv8_read(Kv8ReadArgs a, int head_dim, bool of32, hipStream_t s);

// Attention over the 8-bit cache. The n_q * group query rows of a (batch, key
// head), token by token, see the same keys: blocks [range_begin, range_begin +
// ceil(range_keys / 64)) of each range, the last one's first keys only.
struct Kv8AttnArgs {
    const void* q;  // [B, n_q, H, D] bf16
    void* o;        // the same, or fp32
    float* lse;     // [B, H, n_q] or null
    const unsigned char* k_codes;
    const unsigned char* v_codes;
    const float* k_scale;
    const float* v_scale;
    float* part;     // partial rows of the split tiles: [split tile][part][tile rows][D + 2], or null
    int32_t o_f32;
    int32_t B, H, Hk, group;  // group = H / Hk
    int32_t n_q, rows;        // rows = n_q * group
    int32_t n_blocks;         // per (batch, key head) of the cache
    float scale_log2;         // softmax scale * log2(e)
    int32_t few;              // 4 or 8: tiles of 32 rows, their keys shared out over so many waves; 0: of 256
    int32_t n_tiles;          // row tiles per (batch, key head)
    int32_t n_whole;          // tiles (of all heads) that are not split
    int32_t parts;            // key shares of a split tile
    int32_t cut;              // > 0: two parts, the first of this many key blocks; else parts are equal
    int32_t n_kblocks;        // key blocks of all ranges
    int32_t n_ranges;
    int32_t range_begin[kMaxRanges];  // in blocks
    int32_t range_keys[kMaxRanges];
    // set by the launcher: divisions by group, parts, n_tiles and Hk; key blocks of a part (of the first
    // more_part_blocks parts: one more), and 32-row blocks of a row tile of 256 likewise
    FastDiv by_group, by_parts, by_tiles, by_heads;
    int32_t part_blocks, more_part_blocks, row_blocks, more_row_blocks;
};
constexpr int kKv8FewRows = 32;  // rows of a tile where rows are few
constexpr int kKv8MaxParts = 256;
hipError_t launch_attn_kv8(Kv8AttnArgs a, int head_dim, hipStream_t s);

// Which row of a modulation [B, groups, width] a token row takes: token i of batch element b is at
// position first + i, group (first + i) / group_tokens, of which the host keeps the quotient of first
// (g0) and its remainder (f0). Without groups by_group divides by 2^31 - 1, which leaves 0.
struct TokenGroups {
    int32_t n, groups;
    int32_t f0, g0;
    FastDiv by_n, by_group;
    __host__ __device__ __forceinline__ int64_t row(int32_t r) const {
        const int32_t b = by_n.of(r);
        return int64_t(b) * groups + g0 + by_group.of(f0 + (r - b * n));
    }
};

// Linear layers. An element of the output from the sum z of its products: + bias, kept in pre (bf16) if
// wanted, through the activation, times the token's gate, + residual, rounded once.
constexpr int kActNone = 0, kActGelu = 1, kActSilu = 2;
struct LinearEpilogue {
    const float* bias;     // [N] or null
    const float* gate;     // [B, groups, N] or null
    const void* residual;  // [rows, N], of o's type, or null
    void* pre;             // [rows, N] bf16, or null
    void* o;               // [rows, N]
    int32_t act, o_f32;
    TokenGroups tg;
};

// C[m, n] = sum over k of A(m, k) B(n, k), bf16 operands, fp32 sums. An operand's rows in memory are its m
// (n), k side by side, or its k, m (n) side by side (TRANS).
struct GemmArgs {
    const unsigned char* a;
    const unsigned char* b;
    int64_t lda, ldb;   // bytes from row to row in memory
    int32_t M, N, K;
    int32_t tiles_m, tiles_n;
    int32_t stages;     // of kGemmDepth k each, the last one's first k only
    int32_t whole;      // tiles that a workgroup takes alone; the others' stages are dealt out
    int32_t groups;     // in so many groups of as many tiles each (group i: tiles whole + i, + groups, ...),
    int32_t shares;     // each to this many workgroups in equal shares, at most a tile's stages each
    float* part;        // [shares][groups][2][tile][tile], or null where none is split
    LinearEpilogue ep;
    __host__ __device__ __forceinline__ int per_group() const { return (tiles_m * tiles_n - whole) / groups; }
    // Tile i of a group.
    __host__ __device__ __forceinline__ int split_tile(int i, int group) const { return whole + i * groups + group; }
    // First of the stages of a group's tiles, in a row, that share c takes. Shares c of all groups go through the same k
    // at the same time, and neighbouring tiles lie in neighbouring groups: so their workgroups, which run on one
    // XCD, bring the same rows and columns to its L2 (dealt out without groups, each brought its own:
    // 42% of the reads missed).
    __host__ __device__ __forceinline__ int share_begin(int c) const {
        return static_cast<int>(static_cast<int64_t>(per_group()) * stages * c / shares);
    }
    // The share that takes stage u of a group.
    __host__ __device__ __forceinline__ int share_of(int u) const {
        int c = static_cast<int>(static_cast<int64_t>(u) * shares / (per_group() * stages));
        while (share_begin(c + 1) <= u) ++c;
        return c;
    }
};
constexpr int kGemmDepth = 64;
// Workgroups of a CU at a time: LDS holds 2 * ahead + 1 parts of 128 * tile bytes for each.
constexpr int gemm_per_cu(int tile, int ahead = 2) { return 160 * 1024 / ((2 * ahead + 1) * 128 * tile); }
// As many workgroups as the chip holds at a time; each takes one tile after the other.
inline int gemm_workgroups(const GemmArgs& a, int tile) {
    const int most = kCUs * gemm_per_cu(tile), wanted = a.whole > a.groups * a.shares ? a.whole : a.groups * a.shares;
    return wanted < most ? wanted : most;
}
// Stages that its loads run ahead of the MFMAs: more where a smaller tile's workgroup has a CU for itself.
inline int gemm_ahead(const GemmArgs& a, int tile) { return tile < 256 && gemm_workgroups(a, tile) <= kCUs ? 4 : 2; }
hipError_t launch_gemm(const GemmArgs& a, int tile, bool a_trans, bool b_trans, hipStream_t s);

// Token rows in parts that lie in one group each, for sums over a group's rows: group j of those that the
// run touches holds tokens [j * len - f0, (j + 1) * len - f0) of each batch element, cut to [0, n), and
// part p of it the rows_per_part from p * rows_per_part on. Only parts that have a row are counted and numbered, in the
// order of their rows: in the run's first and last group its ends leave out some.
struct RowParts {
    int32_t B, n;
    int32_t len, f0;        // tokens of a group (at most what the run has of one), and of the first one before the run
    int32_t touched;        // groups of the run
    int32_t per_group;      // parts of len tokens
    int32_t rows_per_part;
    int32_t g0, groups;     // the first one's index, of how many
    int32_t before, empty;  // of a batch element's parts those before its first row, and all without a row
    __host__ __device__ int32_t count() const { return B * touched * per_group; }  // with those without a row
    __host__ __device__ int32_t each() const { return touched * per_group - empty; }
    __host__ __device__ int32_t filled() const { return count() - B * empty; }
    // part `i` of filled(): its batch element, the modulation's row of its group, its tokens [t0, t1)
    __host__ __device__ __forceinline__ void of(int32_t i, int32_t& b, int64_t& mod, int32_t& t0, int32_t& t1) const {
        b = i / each();
        const int32_t q = i - b * each() + before, j = q / per_group, p = q - j * per_group;
        mod = int64_t(b) * groups + g0 + j;
        const int64_t at = int64_t(j) * len - f0;
        const int64_t lo = at + int64_t(p) * rows_per_part;
        const int64_t hi = lo + rows_per_part < at + len ? lo + rows_per_part : at + len;
        t0 = static_cast<int32_t>(lo > 0 ? lo : 0);
        t1 = static_cast<int32_t>(hi < n ? hi : n);
    }
    // parts [i0, i1) are those of group j of batch element b
    __host__ __device__ __forceinline__ void of_group(int32_t b, int32_t j, int32_t& i0, int32_t& i1) const {
        const int32_t lo = j * per_group - before, hi = lo + per_group;
        i0 = b * each() + (lo > 0 ? lo : 0);
        i1 = b * each() + (hi < each() ? hi : each());
    }
};

// Sums over rows from those over the parts, part [parts][vectors][E]: per group into out [B, groups, E] (zeros
// for groups outside the run), sum v times mul (null: 1) plus sum w times mul_w (w < 0: without); in total
// over all parts into out [E], sum v times what mod [B, groups, E] has for its group plus add (null: 1).
struct GroupSum {
    float* out;
    const float* mul;
    const float* mul_w;
    int32_t v, w;
};
struct TotalSum {
    float* out;
    const float* mod;
    float add;
    int32_t v;
};
struct ColumnSums {
    const float* part;
    int32_t vectors, E;
    RowParts parts;
    int32_t n_group, n_total;
    GroupSum group[3];
    TotalSum total[3];
    FastDiv by_parts, by_each;  // of a group, of a batch element; set by the launcher
};
// Columns of a workgroup and threads of a column, with so many parts to a sum. Few columns leave CUs idle, and their
// threads wait for one load after the other (2560 parts of 64 columns: 26 us of 92 for the backward with 32 threads a column
// and with 16); wide parts are bound by the lines that they read (2000 parts of 5120: 120 us of the backward with 64
// threads a column, 111 with 32).
inline void column_sums_shape(int parts, int E, int* columns, int* threads) {
    if (parts <= 512) {
        *columns = 64;
        *threads = parts <= 4 ? 1 : parts <= 64 ? 4 : 16;
    } else {
        *columns = E > 2048 ? 32 : 16;
        *threads = 1024 / *columns;
    }
}
hipError_t launch_column_sums(const ColumnSums& a, hipStream_t s);

// Norms around a block (rows of E): z = post(y) * post_weight, r = x + gate * z, m = pre(r) * pre_weight +
// pre_bias, h = m * (1 + scale) + shift. Null vectors are ones (weights, gate) or zeros.
constexpr int kNormNone = 0, kNormLayer = 1, kNormRms = 2;
constexpr int kMaxNormWidth = 16384;
struct BlockNormArgs {
    const void* x;  // backward: r
    const void* y;
    const float* gate;
    const float* post_weight;
    const float* pre_weight;
    const float* pre_bias;
    const float* scale;
    const float* shift;
    void* r;
    void* h;
    int32_t E, rows;
    int32_t row0;  // of one launch; set by the launcher
    int32_t pre, post;
    float eps, inv_E;
    TokenGroups tg;
};
hipError_t launch_block_norm(const BlockNormArgs& a, bool stream_f32, bool act_f32, hipStream_t s);

// Its backward: dx, dy, and per part the sums over rows of dh, of dh * pre(r) and of dx * post(y).
constexpr int kNormSums = 3;
struct BlockNormBwdArgs {
    const void* r;   // null without pre
    const void* dh;  // null without pre
    const void* dr;  // or null: zeros
    const void* y;   // or null
    const float* gate;
    const float* post_weight;
    const float* pre_weight;
    const float* scale;
    void* dx;
    void* dy;     // null without y
    float* part;  // [parts][kNormSums][E], or null: no sums wanted
    int32_t E, pre, post;
    float eps, inv_E;
    RowParts parts;
};
// Fours of a row that a lane takes, and lanes of a row. Forward: more work a lane takes less time (5120 wide, 4680
// rows: 55.4 us with 5, 59.9 with 2; 1024 wide: 42 with 2, 47 with 1; 88311 rows of 304, bf16, 33 with 2, in one wave,
// 43 with 1, in two) while there are lanes enough.
// Backward: as few as the registers of its sums allow, but two up to 512, whose rows one wave then takes (88311 rows of 304,
// bf16 and fp32: 138 us, 193 in two).
inline void block_norm_shape(int E, bool backward, int* fours, int* lanes) {
    const int all = E / 4;
    if (backward)
        *fours = all <= 64 ? 1 : all <= 128 ? 2 : all <= 256 ? 1 : all <= 2 * 1024 ? 2 : 4;
    else
        *fours = all <= 64 ? 1 : all <= 512 ? 2 : 5;
    *lanes = ((all + *fours - 1) / *fours + 63) / 64 * 64;
}
hipError_t launch_block_norm_bwd(const BlockNormBwdArgs& a, bool stream_f32, bool act_f32, hipStream_t s);

// o = epilogue(x W^T) for at most kFewRows rows x [rows, K], W [N, K] bf16: W streams by once.
constexpr int kFewRows = 16;
struct FewRowsArgs {
    const void* x;
    const void* w;
    int32_t rows, K, N;
    LinearEpilogue ep;
};
// Pieces of K that a workgroup takes side by side, and its waves: the fewest columns a workgroup that leave 1024
// workgroups, as far as the rows allow: one row of 5120 x 5120 14.2 us with 16, 11.1 with 8, 10.0 with 4; 20480 x 5120
// 51, 42, 37; 5120 x 20480 37, 39, 37; 2560 x 40960 39, 37, 45. Their four waves are sixteen where workgroups are few.
inline void few_rows_shape(int rows, int N, int* pieces, int* waves) {
    *pieces = 1;
    while (*pieces < 4 && rows * *pieces * 2 <= 16 && N / 16 * *pieces < 1024) *pieces *= 2;
    const int columns = 16 / *pieces;
    *waves = (N + columns - 1) / columns >= kCUs ? 4 : 16;
}
hipError_t launch_few_rows(const FewRowsArgs& a, hipStream_t s);

// dz = dout * gate * act'(pre) of a linear layer's rows, in bf16 [rows, N] (dz) or, of at most kFewRowsBwd rows,
// in fp32 [N][R] (dz_few, rows past the last one zero), and per part the sums over rows of dz and of
// dout * act(pre).
constexpr int kLinearSums = 2;
struct LinearDzArgs {
    const void* dout;
    const void* pre;    // bf16, or null
    const float* gate;  // or null
    void* dz;           // or null
    void* dz_rest;      // what dz's rounding left, in bf16, or null
    float* dz_few;      // or null
    float* part;        // [parts][kLinearSums][N], or null
    int32_t N, act, dout_f32, gate_sums;
    int32_t R;          // of dz_few
    RowParts parts;
};
hipError_t launch_linear_dz(const LinearDzArgs& a, hipStream_t s);

// dx = dz W and dW = dz^T x for at most kFewRowsBwd rows, from dz_few with R = 1, 2 or 4. More rows go through
// the matrix instructions: as 8 + 8 digits (dz and dz_rest) up to kExactRows, where nothing would average
// the roundings of dz.
constexpr int kFewRowsBwd = 4;
constexpr int kExactRows = 16;
struct FewRowsBwdArgs {
    const float* dz;  // [N][R]
    const void* x;    // [rows, K]
    const void* w;    // [N, K]
    void* dx;         // or null
    void* dw;         // or null
    float* part;      // of dx: [shares][R][K]
    int32_t rows, R, K, N;
    int32_t shares;   // of N that dx's sums are dealt out to
};
hipError_t launch_few_rows_bwd(const FewRowsBwdArgs& a, hipStream_t s);

// x twice into out, or (halves_sum) the sum of x's halves in fp32 into out in bf16; n: groups of 8 elements of x, or
// of one half.
struct TwiceArgs {
    const void* x;
    void* out;
    int64_t n;
};
hipError_t launch_twice(const TwiceArgs& a, hipStream_t s);
hipError_t launch_halves_sum(const TwiceArgs& a, hipStream_t s);

// n elements of 4 bytes to zero (a fill kernel: it may be captured).
hipError_t launch_zero(void* p, int64_t n, hipStream_t s);

}  // namespace tmk
