// Products of matrices in E4M3 codes with a scale for each block of 128: y[t, n] = sum over blocks b of sx[t, b] sw[n / 128, b] sum over b's k of x[t, k] W[n, k], and
// the same with W's other axis summed.
//
// All products run on the matrix instruction of 16 x 16 outputs and 128 products each, which is one block: its result, started from zero, is scaled and added
// to binary32 sums.  An operand fragment of a wavefront is 16 rows of 128 codes: lane l holds row l % 16, codes 16 g .. + 15 and 64 + 16 g .. + 15 with
// g = l / 16.  (Which codes a lane holds is free as long as both operands agree.)  Where the summed axis is the rows of a matrix in memory, tiles of it lie in
// LDS as they are and the transposing LDS load collects the fragment.  A result puts its column in lane l % 16 and its rows 4 (l / 16) .. + 3 in four registers.
#pragma once
#include "k_rows.h"

namespace condensa {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef u32 u32x8 __attribute__((ext_vector_type(8)));
typedef u32 u32x4_bytes __attribute__((ext_vector_type(4), aligned(1)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr u32 kStep = CONDENSA_FP8_BLOCK;       // codes of a row that a step sums

// Within eight neighbouring products what lies below 2^-13 of the largest (of its exponent) is cut, by this instruction and by the one for 32 products alike; the alternative is to widen
// codes to 16 bits, at half the rate and twice the LDS.  Random codes: 2.7e-5 of the largest of 128 products on the mean, 3e-5 of their sum; bfloat16 rounds by 1.7e-3.
__device__ inline f32x4 mfma_codes(u32x8 a, u32x8 b) {
    // (no scales of the instruction's own: zeros for them choose the form without)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, a), __builtin_bit_cast(i32x8, b), f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------------------

// Tiles with the summed axis along their rows: [rows][128], 16-byte pieces of a row at piece ^ (row & 7), so that eight rows of a fragment lie in
// different banks although rows are 128 bytes apart.
__device__ inline u32 codes_along_at(u32 row, u32 piece) { return row * kStep + ((piece ^ (row & 7u)) << 4); }
__device__ inline u32x8 codes_along_frag(const u8* tile, u32 row0) {
    const u32 l = threadIdx.x & 63, row = row0 + (l & 15), g = l >> 4;
    const u32x4 a = *reinterpret_cast<const u32x4*>(tile + codes_along_at(row, g)), b = *reinterpret_cast<const u32x4*>(tile + codes_along_at(row, g + 4));
    return u32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// Tiles with the summed axis across their rows: [128][COLS].  The transposing load hands 16 lanes eight rows of 16 columns: lane s reads row s / 2, columns
// 8 (s % 2) .. + 7, and receives column s of the eight rows.  Pieces of 16 bytes are moved so that the rows that 32 lanes read together (eight, and the
// eight that are 16 further on) lie in different banks.
template <u32 COLS>
__device__ inline u32 codes_across_at(u32 k, u32 piece) {
    constexpr u32 kPieces = COLS / 16;
    static_assert(kPieces % 16 == 0 || kPieces == 8 || kPieces % 4 == 0, "widths of tiles");
    const u32 slot = kPieces % 16 == 0 ? (k & 7u) | (k >> 1 & 8u) : (kPieces == 8 ? (k >> 1 & 3u) | (k >> 2 & 4u) : (k >> 2 & 1u) | (k >> 3 & 2u));
    return k * COLS + ((piece ^ slot) << 4);
}
template <u32 COLS>
__device__ inline u32x8 codes_across_frag(const u8* tile, u32 col0) {
    const u32 l = threadIdx.x & 63, s = l & 15, k0 = (l >> 4) * 16 + (s >> 1);
    u32x8 v;
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        const u8* at = tile + codes_across_at<COLS>(k0 + (i & 1) * 8 + (i >> 1) * 64, col0 >> 4) + (s & 1) * 8;
        const i32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)at);
        v[2 * i] = static_cast<u32>(t.x);
        v[2 * i + 1] = static_cast<u32>(t.y);
    }
    return v;
}

// Sixteen codes p[k .. k+15] of a row of n at any address, zeros past its end; what follows a row, up to the end of the matrix, is loaded and masked.  `left`: codes from
// p[k] to that end.
__device__ inline u32x4 load16_codes(const u8* p, i64 k, i64 n, i64 left) {
    const i64 rest = n - k;
    const int there = rest >= 16 ? 16 : (rest <= 0 ? 0 : static_cast<int>(rest));
    u32x4 v = {0u, 0u, 0u, 0u};
    if (there > 0) {
        if (left >= 16) {
            v = *reinterpret_cast<const u32x4_bytes*>(p + k);
        } else {
#pragma unroll
            for (int i = 0; i < 15; ++i) if (i < there) v[i >> 2] |= static_cast<u32>(p[k + i]) << (8 * (i & 3));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int in = there - 4 * i;                        // codes of this word
        v[i] &= in >= 4 ? ~0u : (in <= 0 ? 0u : (1u << (8 * in)) - 1u);
    }
    return v;
}

// ---- the product ----------------------------------------------------------------------------------------------------

struct ProductArgs {
    const u8* x; i64 ldx;                // [n_tokens, n_sum]
    const float* xs; i64 ldxs;           // [n_tokens, steps]
    const u8* w; i64 ldw;                // ALONG: [n_out, n_sum], else [n_sum, n_out]
    const float* ws; i64 ldws;           // a scale for 128 x 128 of w
    u16* y; i64 ldy;                     // [n_tokens, n_out]
    u32 n_tokens, n_out, n_sum;
    u32 splits, steps_each;              // steps of 128 codes that a split sums
    float* part;                         // [splits][n_tokens][n_out], or NULL: y is written
    u32 bf16;
};

// Two outputs in their 16-bit type, by the conversion instructions: in integer arithmetic the 65536 of a tile took 4 us more.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
__device__ inline u32 bf16_pair(float a, float b) { return __builtin_bit_cast(u32, b16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)}); }
__device__ inline u32 f16_pair(float a, float b) { return __builtin_bit_cast(u32, f16x2{static_cast<_Float16>(a), static_cast<_Float16>(b)}); }

// Four neighbouring outputs of a token.
__device__ inline void store_outputs(const ProductArgs& p, u32 t, u32 n, f32x4 v) {
    if (t >= p.n_tokens) return;
    u16* out = p.y + static_cast<i64>(t) * p.ldy;
    const u32x2 h = p.bf16 ? u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])} : u32x2{f16_pair(v[0], v[1]), f16_pair(v[2], v[3])};
    if (n + 4 <= p.n_out) {
        *reinterpret_cast<u32x2_any*>(out + n) = h;
    } else {
#pragma unroll
        for (u32 k = 0; k < 3; ++k) if (n + k < p.n_out) out[n + k] = static_cast<u16>(h[k >> 1] >> (16 * (k & 1)));
    }
}
// Parts of them.
__device__ inline void store_part(const ProductArgs& p, u32 split, u32 t, u32 n, f32x4 v) {
    if (t >= p.n_tokens) return;
    float* out = p.part + (static_cast<u64>(split) * p.n_tokens + t) * p.n_out;
    if (n + 4 <= p.n_out) {
        *reinterpret_cast<f32x4_any*>(out + n) = v;
    } else {
#pragma unroll
        for (u32 k = 0; k < 4; ++k) if (n + k < p.n_out) out[n + k] = v[k];
    }
}

// Tiles of 64 tokens by 64 outputs, rows at any address: steps go through registers, where what lies past the end of a row is masked.
template <bool ALONG>
__global__ __launch_bounds__(256) void k_product_any(ProductArgs p) {
    __shared__ __align__(16) u8 lds[2][128 * kStep];
    const u32 tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
    const u32 tiles_n = (p.n_out + 63) / 64;
    const u32 block = die_order(blockIdx.x, gridDim.x), tile = block / p.splits, split = block % p.splits;
    const u32 t0 = tile / tiles_n * 64, n0 = tile % tiles_n * 64;
    const u32 all = (p.n_sum + kStep - 1) / kStep, begin = split * p.steps_each, end = begin + p.steps_each < all ? begin + p.steps_each : all;
    f32x4 acc[2][2] = {};
    u32x4 rx[2], rw[2];
    auto fetch = [&](u32 s) {
        const i64 k0 = static_cast<i64>(s) * kStep;
#pragma unroll
        for (u32 i = 0; i < 2; ++i) {
            const u32 at = i * 256 + tid, row = at >> 3;
            const i64 k = k0 + (at & 7u) * 16;
            const u32 t = t0 + row < p.n_tokens ? t0 + row : p.n_tokens - 1;
            rx[i] = load16_codes(p.x + static_cast<i64>(t) * p.ldx, k, p.n_sum, static_cast<i64>(p.n_tokens - 1 - t) * p.ldx + p.n_sum - k);
            if (ALONG) {
                const u32 n = n0 + row < p.n_out ? n0 + row : p.n_out - 1;
                rw[i] = load16_codes(p.w + static_cast<i64>(n) * p.ldw, k, p.n_sum, static_cast<i64>(p.n_out - 1 - n) * p.ldw + p.n_sum - k);
            } else {
                const i64 r = k0 + (at >> 2), n = n0 + (at & 3u) * 16;
                rw[i] = load16_codes(p.w + r * p.ldw, n, r < p.n_sum ? p.n_out : 0, (p.n_sum - 1 - r) * p.ldw + p.n_out - n);
            }
        }
    };
    if (begin < end) fetch(begin);
    u32 to = 0;
    for (u32 s = begin; s < end; ++s) {
        u8* sx = lds[to];
        u8* sw = sx + 64 * kStep;
#pragma unroll
        for (u32 i = 0; i < 2; ++i) {
            const u32 at = i * 256 + tid;
            *reinterpret_cast<u32x4*>(sx + codes_along_at(at >> 3, at & 7u)) = rx[i];
            *reinterpret_cast<u32x4*>(sw + (ALONG ? codes_along_at(at >> 3, at & 7u) : codes_across_at<64>(at >> 2, at & 3u))) = rw[i];
        }
        const float by = p.ws[ALONG ? static_cast<i64>(n0 / kStep) * p.ldws + s : static_cast<i64>(s) * p.ldws + n0 / kStep];
        float scale[2];
#pragma unroll
        for (u32 j = 0; j < 2; ++j) {
            const u32 t = t0 + wm * 32 + j * 16 + (lane & 15);
            scale[j] = p.xs[static_cast<i64>(t < p.n_tokens ? t : p.n_tokens - 1) * p.ldxs + s] * by;
        }
        __syncthreads();
        if (s + 1 < end) fetch(s + 1);
        u32x8 fw[2];
#pragma unroll
        for (u32 i = 0; i < 2; ++i) fw[i] = ALONG ? codes_along_frag(sw, wn * 32 + i * 16) : codes_across_frag<64>(sw, wn * 32 + i * 16);
#pragma unroll
        for (u32 j = 0; j < 2; ++j) {
            const u32x8 fx = codes_along_frag(sx, wm * 32 + j * 16);
#pragma unroll
            for (u32 i = 0; i < 2; ++i) {
                const f32x4 v = mfma_codes(fw[i], fx);
#pragma unroll
                for (u32 k = 0; k < 4; ++k) acc[i][j][k] = __builtin_fmaf(v[k], scale[j], acc[i][j][k]);
            }
        }
        to ^= 1;                                              // the one that all have read since the barrier before this one
    }
#pragma unroll
    for (u32 j = 0; j < 2; ++j)
#pragma unroll
        for (u32 i = 0; i < 2; ++i) {
            const u32 t = t0 + wm * 32 + j * 16 + (lane & 15), n = n0 + wn * 32 + i * 16 + (lane >> 4) * 4;
            if (p.part) store_part(p, split, t, n, acc[i][j]);      // uniform
            else        store_outputs(p, t, n, acc[i][j]);
        }
}

// Rows at any address copied to rows that are 16-byte aligned, sixteen codes a thread: loads straight into LDS want those.
struct CodesCopy {
    const u8* src; i64 ld;
    u8* dst;
    u32 rows, cols, width;               // width: of a copied row, a multiple of sixteen
    u32 blocks;                          // workgroups that copy it
};
struct CopyArgs { CodesCopy m[2]; };
__global__ __launch_bounds__(256) void k_product_copy(CopyArgs a) {
    const bool second = blockIdx.x >= a.m[0].blocks;
    const CodesCopy& m = a.m[second];
    const u32 pieces = m.width / 16;
    const u64 at = static_cast<u64>(blockIdx.x - (second ? a.m[0].blocks : 0)) * 256 + threadIdx.x;
    const u64 row = at / pieces;
    if (row >= m.rows) return;
    const i64 k = static_cast<i64>(at % pieces) * 16;
    const u32x4 v = load16_codes(m.src + static_cast<i64>(row) * m.ld, k, m.cols, static_cast<i64>(m.rows - 1 - row) * m.ld + m.cols - k);
    *reinterpret_cast<u32x4*>(m.dst + row * m.width + k) = v;
}

// Tiles of BM tokens by BN outputs of rows that are 16-byte aligned, NB steps in LDS.  Loads go straight into LDS, NB - 1 steps ahead of their use, a few of them beside each sixteen tokens
// of a step; a token's and W's scales of a step come with it.  (A 16-byte piece may end past its row; it never leaves the sixteen bytes that hold the row's last code.)  Sixteen
// tokens at a time meet the wavefront's fragments of W, their results are scaled and added while the next sixteen are multiplied, and the fragments of the next step are read beside
// the last sixteen: wavefronts meet once a step, just before, when the next step has come and the last read of this one is done.
// 8192 tokens, 4608 -> 4096: 142 to 152 us by card, 2.0 to 2.2 PFLOP/s; backward, in two launches, 154 to 162.  What the time of 256 x 256 goes to, parts left out (150 us on that card): without loads 129, without LDS reads 142,
// with a quarter of the additions 139, without all three 109, of which 22 are two rounds of first loads and of outputs, and the rest the matrix instructions.  So none of them
// bounds it alone: they share a wavefront's issue and meet at its barrier.  Two groups of wavefronts in turns, one multiplying while the other reads LDS, took 150 us where this took 144.
constexpr u32 product_lds(u32 bm, u32 bn, u32 nb) { return nb * ((bm + bn) * kStep + bm * 4 + 256) + (bm == 256 ? 256 : 0); }
template <int BM, int BN, int WM, int WN, int NB, bool ALONG>
__device__ inline void product_tile(const ProductArgs& p, u32 block_id, u32 n_blocks, u8* lds) {
    constexpr u32 kThreads = 64 * WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr u32 kXLoads = BM * 8 / kThreads, kWLoads = BN * 8 / kThreads;
    constexpr bool kFar = BM == 256;                                // one workgroup a unit, two steps in LDS: lines of later steps are asked for
    constexpr u32 kLoads = kXLoads + kWLoads + 1 + kFar;
    constexpr u32 kTile = (BM + BN) * kStep, kBuffer = kTile + BM * 4 + 256;
    constexpr bool kOneBlock = (BN % 128 == 0 || BN == 64) && 128 % TN == 0;             // a wavefront's outputs lie in one block of W
    constexpr u32 kEach = (kLoads + FM / 2 - 1) / (FM / 2);         // loads beside sixteen tokens, in the first half of a step
    constexpr u32 kAhead = 2;
    static_assert(WM * WN > BM / 64, "a wavefront for W's scales");
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const u32 wm = wave / WN, wn = wave % WN;
    const u32 tiles_m = (p.n_tokens + BM - 1) / BM, tiles_n = (p.n_out + BN - 1) / BN;
    const u32 block = die_order(block_id, n_blocks);
    const u32 tile = block / p.splits, split = block % p.splits;
    // four rows of tiles at a time: tiles that run together share rows of x and of W
    const u32 band = tile / (4 * tiles_n), in_band = tile % (4 * tiles_n), high = tiles_m - band * 4 < 4 ? tiles_m - band * 4 : 4;
    const u32 t0 = (band * 4 + in_band % high) * BM, n0 = in_band / high * BN;
    const u32 all = (p.n_sum + kStep - 1) / kStep, begin = split * p.steps_each, end = begin + p.steps_each < all ? begin + p.steps_each : all;
    const u32 steps = end - begin;                                  // one at least
    const u32 valid = end == all ? p.n_sum - (all - 1) * kStep : kStep;                  // codes of the last step

    u32 xo[kXLoads], wo[kWLoads], so;                               // byte offsets of what this lane loads
#pragma unroll
    for (u32 i = 0; i < kXLoads; ++i) {
        const u32 at = i * kThreads + tid, row = at >> 3, r = t0 + row < p.n_tokens ? row : p.n_tokens - 1 - t0;
        xo[i] = r * static_cast<u32>(p.ldx) + ((at ^ row) & 7u) * 16;
    }
#pragma unroll
    for (u32 i = 0; i < kWLoads; ++i) {
        const u32 at = i * kThreads + tid;
        if (ALONG) {
            const u32 row = at >> 3, r = n0 + row < p.n_out ? row : p.n_out - 1 - n0;
            wo[i] = r * static_cast<u32>(p.ldw) + ((at ^ row) & 7u) * 16;
        } else {
            constexpr u32 kRow = BN / 16;
            const u32 k = at / kRow;
            u32 col = codes_across_at<BN>(k, at % kRow) - k * BN;
            if (n0 + col >= p.n_out) col = (p.n_out - 1 - n0) & ~15u;
            wo[i] = k * static_cast<u32>(p.ldw) + col;
        }
    }
    const char* xs = reinterpret_cast<const char*>(p.x + static_cast<i64>(t0) * p.ldx + begin * kStep);
    const char* ws = reinterpret_cast<const char*>(ALONG ? p.w + static_cast<i64>(n0) * p.ldw + begin * kStep : p.w + static_cast<i64>(begin) * kStep * p.ldw + n0);
    const char* ss;
    const bool of_x = wave < BM / 64;                               // the wavefront loads scales of 64 tokens; else those of W
    const u32 b0 = n0 / kStep, last_block = (p.n_out - 1) / kStep;
    if (of_x) {
        const u32 r = wave * 64 + lane;
        so = (t0 + r < p.n_tokens ? r : p.n_tokens - 1 - t0) * static_cast<u32>(p.ldxs) * 4;
        ss = reinterpret_cast<const char*>(p.xs + static_cast<i64>(t0) * p.ldxs + begin);
    } else {
        const u32 b = lane & 3u, at = b0 + b < last_block ? b : last_block - b0;
        so = (ALONG ? at * static_cast<u32>(p.ldws) : at) * 4;
        ss = reinterpret_cast<const char*>(p.ws + (ALONG ? static_cast<i64>(b0) * p.ldws + begin : static_cast<i64>(begin) * p.ldws + b0));
    }
    // Where only two steps fit LDS, a step's time does not hide a line that has to come from memory.  So one value of each line is loaded two steps before the
    // line is, which brings it into the die's cache: a part of the lines by each of the tiles that run together and share them, x's by even wavefronts, W's by odd ones.
    u32 fo = 0;
    if (kFar) {
        if ((wave & 1u) == 0) {
            const u32 row = n0 / BN % 8 * 32 + wave / 2 * 8 + (lane & 7u);
            fo = (t0 + row < p.n_tokens ? row : p.n_tokens - 1 - t0) * static_cast<u32>(p.ldx);
        } else {
            const u32 line = t0 / BM % 4 * 64 + wave / 2 * 16 + (lane & 15u);
            if (ALONG) {
                fo = (n0 + line < p.n_out ? line : p.n_out - 1 - n0) * static_cast<u32>(p.ldw);
            } else {
                const u32 col = (line & 1u) * kStep;
                fo = (line >> 1) * static_cast<u32>(p.ldw) + (n0 + col < p.n_out ? col : 0);
            }
        }
    }
    const i64 w_step = ALONG ? kStep : kStep * p.ldw, s_step = of_x || ALONG ? 4 : 4 * p.ldws;
    const u32 lds0 = static_cast<u32>(reinterpret_cast<uintptr_t>((lds_void*)lds)), s_at = kTile + (of_x ? wave * 256 : BM * 4);

    u32 loaded = 0, to = 0;
    // Loads of the next step, or of the last one again, part by part.
    auto load_begin = [&]() {
        if (loaded + 1 == steps && valid < kStep) {                 // what lies past the sum is loaded from its last codes
#pragma unroll
            for (u32 i = 0; i < kXLoads; ++i) {
                const u32 at = i * kThreads + tid, piece = (at ^ (at >> 3)) & 7u;
                xo[i] -= piece * 16 < valid ? 0 : (piece - (valid - 1) / 16) * 16;
            }
#pragma unroll
            for (u32 i = 0; i < kWLoads; ++i) {
                const u32 at = i * kThreads + tid;
                if (ALONG) {
                    const u32 piece = (at ^ (at >> 3)) & 7u;
                    wo[i] -= piece * 16 < valid ? 0 : (piece - (valid - 1) / 16) * 16;
                } else {
                    const u32 k = at / (BN / 16);
                    wo[i] -= k < valid ? 0 : (k - (valid - 1)) * static_cast<u32>(p.ldw);
                }
            }
        }
    };
    auto load_part = [&](u32 q) {
        if (q < kXLoads)             load_lds<16>(xo[q], xs, lds0 + to + (q * kThreads + wave * 64) * 16);
        else if (q < kXLoads + kWLoads) load_lds<16>(wo[q - kXLoads], ws, lds0 + to + BM * kStep + ((q - kXLoads) * kThreads + wave * 64) * 16);
        else if (q == kXLoads + kWLoads) load_lds<4>(so, ss, lds0 + to + s_at);
        else if (q < kLoads) {
            const bool there = loaded + kAhead < steps - (valid < kStep);          // a whole step; else the first value of what is loaded now
            const char* at = (wave & 1u) == 0 ? xs + (there ? kAhead * kStep : 0) : ws + (there ? kAhead * w_step : 0);
            load_lds<4>(there ? fo : 0u, at, lds0 + NB * kBuffer);
        }
    };
    auto load_end = [&]() {
        ++loaded;
        const bool more = loaded < steps;
        xs += more ? kStep : 0;
        ws += more ? w_step : 0;
        ss += more ? s_step : 0;
        to = to + kBuffer == NB * kBuffer ? 0 : to + kBuffer;
    };
    // zeros for what the last step has past the sum
    auto clear = [&](u8* buffer) {
        for (u32 at = tid; at < (ALONG ? BM + BN : BM) * 8; at += kThreads) {
            const u32 piece = at & 7u;
            if (piece * 16 + 16 <= valid) continue;
            u32x4* v = reinterpret_cast<u32x4*>(buffer + codes_along_at(at >> 3, piece));
            u32x4 t = *v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int in = static_cast<int>(valid) - static_cast<int>(piece * 16 + 4 * i);
                t[i] &= in >= 4 ? ~0u : (in <= 0 ? 0u : (1u << (8 * in)) - 1u);
            }
            *v = t;
        }
        if (!ALONG)
            for (u32 at = valid * (BN / 16) + tid; at < kStep * (BN / 16); at += kThreads) *reinterpret_cast<u32x4*>(buffer + BM * kStep + at * 16) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    };

    f32x4 acc[FN][FM] = {}, v[2][FN] = {};
    u32x8 fw[FN], fx;
    float scale[FM], by[FN], last = 0.0f, last_by[FN] = {};
    auto read_w = [&](const u8* buffer, u32 i) {
        fw[i] = ALONG ? codes_along_frag(buffer + BM * kStep, wn * TN + i * 16) : codes_across_frag<BN>(buffer + BM * kStep, wn * TN + i * 16);
    };
    auto read_x = [&](const u8* buffer, u32 j) { return codes_along_frag(buffer, wm * TM + j * 16); };
    auto read_scales = [&](const u8* buffer) {
        const float* s = reinterpret_cast<const float*>(buffer + kTile);
#pragma unroll
        for (u32 i = 0; i < (kOneBlock ? 1 : FN); ++i) by[i] = s[BM + (n0 % kStep + wn * TN + i * 16) / kStep];
#pragma unroll
        for (u32 j = 0; j < FM; ++j) scale[j] = s[wm * TM + j * 16 + (lane & 15)];
    };
    // results of sixteen tokens, scaled and added
    auto add = [&](u32 j, float s, const float* s_by) {
#pragma unroll
        for (u32 i = 0; i < FN; ++i) {
            const float f = s * s_by[kOneBlock ? 0 : i];
#pragma unroll
            for (u32 k = 0; k < 4; ++k) acc[i][j][k] = __builtin_fmaf(v[j & 1][i][k], f, acc[i][j][k]);
            asm volatile("" : "+v"(acc[i][j]));                     // here, and not all of them at the end of the step, where results would wait in registers that there are not
        }
    };
    static_assert(FM % 2 == 0, "two sets of results in turn");
#pragma unroll
    for (int i = 0; i + 1 < NB; ++i) {
        load_begin();
#pragma unroll
        for (u32 q = 0; q < kLoads; ++q) load_part(q);
        load_end();
    }
    meet_loads<(NB - 2) * kLoads + kFar>();
    if (steps == 1 && valid < kStep) clear(lds);
#pragma unroll
    for (u32 i = 0; i < FN; ++i) read_w(lds, i);
    fx = read_x(lds, 0);
    read_scales(lds);
    u32 from = 0;
    for (u32 s = 0; s < steps; ++s) {
        const u8* cur = lds + from;
        load_begin();                                               // where the step before this one was
#pragma unroll
        for (u32 j = 0; j + 1 < FM; ++j) {
            const u32x8 next = read_x(cur, j + 1);
#pragma unroll
            for (u32 q = j * kEach; q < (j + 1) * kEach; ++q) load_part(q);
#pragma unroll
            for (u32 i = 0; i < FN; ++i) v[j & 1][i] = mfma_codes(fw[i], fx);
            if (j == 0) add(FM - 1, last, last_by);
            else        add(j - 1, scale[j - 1], by);
            fx = next;
            // the order that is meant: the next sixteen tokens' reads, then products with the additions of the last ones' between them
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
            for (u32 i = 0; i < FN; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        load_end();
        meet_loads<(NB - 2) * kLoads + kFar>();
        from = from + kBuffer == NB * kBuffer ? 0 : from + kBuffer;
        u8* nxt = lds + from;
        if (s + 2 == steps && valid < kStep) clear(nxt);
#pragma unroll
        for (u32 i = 0; i < FN; ++i) {
            v[(FM - 1) & 1][i] = mfma_codes(fw[i], fx);
            read_w(nxt, i);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, ALONG ? 2 : 4, 0);
        }
        fx = read_x(nxt, 0);
        add(FM - 2, scale[FM - 2], by);
        last = scale[FM - 1];
#pragma unroll
        for (u32 i = 0; i < (kOneBlock ? 1 : FN); ++i) last_by[i] = by[i];
        read_scales(nxt);
    }
    add(FM - 1, last, last_by);
    meet_loads<0>();
    if (p.part) {                                                   // uniform
#pragma unroll
        for (u32 j = 0; j < FM; ++j)
#pragma unroll
            for (u32 i = 0; i < FN; ++i) store_part(p, split, t0 + wm * TM + j * 16 + (lane & 15), n0 + wn * TN + i * 16 + (lane >> 4) * 4, acc[i][j]);
        return;
    }
    // Outputs pass through LDS, so that rows are stored in whole cache lines; 16-byte pieces at piece ^ (row & 7).  (Eight bytes a lane in sixteen rows: 15 us for a tile.)
    constexpr u32 kPieces = BN / 8;
    auto out_at = [&](u32 row, u32 piece) { return lds + row * (BN * 2) + ((piece ^ (row & 7u)) << 4); };
    auto to_lds = [&](auto pair) {
#pragma unroll
        for (u32 j = 0; j < FM; ++j) {
            const u32 row = wm * TM + j * 16 + (lane & 15);
#pragma unroll
            for (u32 i = 0; i < FN; ++i) {
                const u32 col = wn * TN + i * 16 + (lane >> 4) * 4;
                *reinterpret_cast<u32x2*>(out_at(row, col / 8) + (col & 4u) * 2) = u32x2{pair(acc[i][j][0], acc[i][j][1]), pair(acc[i][j][2], acc[i][j][3])};
            }
        }
    };
    if (p.bf16) to_lds([](float a, float b) { return bf16_pair(a, b); });
    else        to_lds([](float a, float b) { return f16_pair(a, b); });
    __syncthreads();
#pragma unroll 4
    for (u32 at = tid; at < BM * kPieces; at += kThreads) {
        const u32 row = at / kPieces, piece = at % kPieces, t = t0 + row, n = n0 + piece * 8;
        if (t >= p.n_tokens || n >= p.n_out) continue;
        const u32x4 v = *reinterpret_cast<const u32x4*>(out_at(row, piece));
        u16* out = p.y + static_cast<i64>(t) * p.ldy + n;
        if (n + 8 <= p.n_out) *reinterpret_cast<u32x4_any*>(out) = v;
        else
#pragma unroll
            for (u32 k = 0; k < 7; ++k) if (n + k < p.n_out) out[k] = static_cast<u16>(v[k >> 1] >> (16 * (k & 1)));
    }
}
template <int BM, int BN, int WM, int WN, int NB, bool ALONG>
__global__ __launch_bounds__(64 * WM * WN, WM * WN <= 4 && product_lds(BM, BN, NB) > 80 * 1024 ? 1 : 2) void k_product(ProductArgs p) {
    __shared__ __align__(16) u8 lds[product_lds(BM, BN, NB)];
    product_tile<BM, BN, WM, WN, NB, ALONG>(p, blockIdx.x, gridDim.x, lds);
}

// ---- a few tokens, in one launch ------------------------------------------------------------------------------------

constexpr u32 kFewTokens = 64, kFewWaves = 8;

// Up to 16 TF tokens times sixteen rows of W a workgroup, whose wavefronts take steps of the sum in turn and add their sums up in LDS, in order.  W is read once, x comes out of
// the caches.  Loads take whole cache lines, eight lanes to a line (a lane each from sixteen rows, as the operands want them, costs the address unit four times as long), and the
// wavefront's own LDS turns them into fragments, without barriers.  Rows at any address.  us, with fragments loaded as they are, this way, and as split tiles of 64: 4608 -> 4096, 1 token 6.0,
// 6.8 and 8.4, 32 tokens 10.2, 7.6 and 9.4, 64 tokens 15.3, 10.2 and 10.3; 2048 -> 512, 64 tokens 8.3, 6.0 and 7.4.  Three and five steps under way, or sixteen wavefronts, gain nothing or
// half a microsecond.
template <int TF>
__global__ __launch_bounds__(64 * kFewWaves) void k_product_few(ProductArgs p) {
    __shared__ __align__(16) f32x4 sums[kFewWaves][TF][64];
    __shared__ __align__(16) u8 turns[kFewWaves][TF + 1][16 * kStep];
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, line = lane >> 3, piece = lane & 7;
    const u32 n0 = blockIdx.x * 16, all = (p.n_sum + kStep - 1) / kStep, whole = p.n_sum / kStep;
    constexpr u32 kAhead = TF > 2 ? 2 : 4;                          // steps whose codes are under way
    const u8 *w[2], *x[TF][2];
    i64 w_left[2], x_left[TF][2];
#pragma unroll
    for (u32 h = 0; h < 2; ++h) {
        const u32 n = n0 + h * 8 + line < p.n_out ? n0 + h * 8 + line : p.n_out - 1;
        w[h] = p.w + static_cast<i64>(n) * p.ldw;
        w_left[h] = static_cast<i64>(p.n_out - 1 - n) * p.ldw + p.n_sum;
#pragma unroll
        for (int f = 0; f < TF; ++f) {
            const u32 t = f * 16 + h * 8 + line < p.n_tokens ? f * 16 + h * 8 + line : p.n_tokens - 1;
            x[f][h] = p.x + static_cast<i64>(t) * p.ldx;
            x_left[f][h] = static_cast<i64>(p.n_tokens - 1 - t) * p.ldx + p.n_sum;
        }
    }
    const float* xs[TF];
#pragma unroll
    for (int f = 0; f < TF; ++f) {
        const u32 t = f * 16 + (lane & 15) < p.n_tokens ? f * 16 + (lane & 15) : p.n_tokens - 1;
        xs[f] = p.xs + static_cast<i64>(t) * p.ldxs;
    }
    const float* ws = p.ws + static_cast<i64>(n0 / kStep) * p.ldws;
    f32x4 acc[TF] = {};
    auto load = [&](const u8* row, i64 left, u32 s) {
        const i64 k = static_cast<i64>(s) * kStep + piece * 16;
        return s < whole ? *reinterpret_cast<const u32x4_bytes*>(row + k) : load16_codes(row, k, p.n_sum, left - k);         // the same way in the wavefront
    };
    auto turned = [&](const u32x4 (&v)[2], u32 f) {
        u8* room = turns[wave][f];
#pragma unroll
        for (u32 h = 0; h < 2; ++h) *reinterpret_cast<u32x4*>(room + codes_along_at(h * 8 + line, piece)) = v[h];
        return codes_along_frag(room, 0);
    };
    for (u32 s0 = wave; s0 < all; s0 += kAhead * waves) {
        u32x4 vw[kAhead][2], vx[kAhead][TF][2];
        float scale[kAhead][TF];
#pragma unroll
        for (u32 q = 0; q < kAhead; ++q) {
            const u32 s = s0 + q * waves;
            if (s >= all) break;                                    // the same in the wavefront
#pragma unroll
            for (u32 h = 0; h < 2; ++h) vw[q][h] = load(w[h], w_left[h], s);
            const float by = ws[s];
#pragma unroll
            for (int f = 0; f < TF; ++f) {
#pragma unroll
                for (u32 h = 0; h < 2; ++h) vx[q][f][h] = load(x[f][h], x_left[f][h], s);
                scale[q][f] = xs[f][s] * by;
            }
        }
#pragma unroll
        for (u32 q = 0; q < kAhead; ++q) {
            if (s0 + q * waves >= all) break;
            const u32x8 fw = turned(vw[q], TF);
#pragma unroll
            for (int f = 0; f < TF; ++f) {
                const f32x4 v = mfma_codes(fw, turned(vx[q][f], f));
#pragma unroll
                for (u32 k = 0; k < 4; ++k) acc[f][k] = __builtin_fmaf(v[k], scale[q][f], acc[f][k]);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < TF; ++f) sums[wave][f][lane] = acc[f];
    __syncthreads();
    for (u32 f = wave; f < TF; f += waves) {
        f32x4 v = sums[0][f][lane];
        for (u32 k = 1; k < waves; ++k) v += sums[k][f][lane];
        store_outputs(p, f * 16 + (lane & 15), n0 + (lane >> 4) * 4, v);
    }
}

// The parts of split sums, added in order, four outputs a thread.
__global__ __launch_bounds__(256) void k_product_join(ProductArgs p) {
    const u32 n = (blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y;
    if (n >= p.n_out) return;
    const u64 each = static_cast<u64>(p.n_tokens) * p.n_out;
    const float* from = p.part + static_cast<u64>(t) * p.n_out + n;
    f32x4 v = {};
    if (n + 4 <= p.n_out) {
        for (u32 s = 0; s < p.splits; ++s) v += *reinterpret_cast<const f32x4_any*>(from + s * each);
    } else {
        for (u32 s = 0; s < p.splits; ++s)
#pragma unroll
            for (u32 k = 0; k < 4; ++k) if (n + k < p.n_out) v[k] += from[s * each + k];
    }
    store_outputs(p, t, n, v);
}

}  // namespace condensa
