// Low-rank adapters of many requests beside one shared projection: y = x W^T + z B^T with z = s x A^T, and the gradients.
//
// All products run on the matrix instructions (16x16x32, 16-bit operands, binary32 sums).  An operand fragment of a wavefront is 16
// rows of 32 consecutive values along the summed axis: lane l holds row l % 16, values 8 (l / 16) .. + 7.  Where the summed axis is
// the rows of a matrix in memory, tiles of it lie in LDS as they are and the transposing LDS load collects the fragment.  A result
// tile puts its column in lane l % 16 and its rows 4 (l / 16) .. + 3 in four registers.
#pragma once
#include "common.h"

typedef int64_t i64;

namespace condensa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct ElemF16 {
    static __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ inline u16 enc(float x) { return f32_to_f16_rne(x); }
    static __device__ inline float dec(u16 h) { return f16_bits_to_f32(h); }
    static constexpr bool kNarrow = true;      // exponents of 5 bits: what is split into two values is scaled first
};
struct ElemBF16 {
    static __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
    static __device__ inline u16 enc(float x) { return f32_to_bf16_rne(x); }
    static __device__ inline float dec(u16 h) { return bf16_bits_to_f32(h); }
    static constexpr bool kNarrow = false;
};

struct AdapterDesc {
    const u16* a;              // [rank, n_in]
    const u16* b;              // [n_out, rank]
    float* grad_a;             // NULL where the list is for forward passes
    float* grad_b;
    float scale;
    u32 rank;
    u64 reserved;
};
static_assert(sizeof(AdapterDesc) == 48, "AdapterDesc layout");

constexpr int kAdapterPoke = 80;           // adapters that one launch writes into the device list
struct AdapterPoke { AdapterDesc d[kAdapterPoke]; };
__global__ __launch_bounds__(256) void k_adapter_list(AdapterDesc* __restrict__ dst, AdapterPoke src, u32 first, u32 count) {
    const u32 words = count * (sizeof(AdapterDesc) / 8);
    for (u32 i = threadIdx.x; i < words; i += 256) reinterpret_cast<u64*>(dst + first)[i] = reinterpret_cast<const u64*>(src.d)[i];
}

// ---- operand access ---------------------------------------------------------------------------------------------

// Eight consecutive 16-bit values p[k .. k+7] of a row of n, zeros past its end.  VEC: rows are 16-byte aligned and n and k are
// multiples of eight.
template <bool VEC>
__device__ inline u32x4 load8(const u16* __restrict__ p, i64 k, i64 n) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (VEC) {
        if (k < n) v = *reinterpret_cast<const u32x4*>(p + k);
    } else if ((reinterpret_cast<u64>(p + k) & 3u) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k + 2 * i + 2 <= n) v[i] = *reinterpret_cast<const u32*>(p + k + 2 * i);
            else if (k + 2 * i < n) v[i] = p[k + 2 * i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < n) v[i >> 1] |= static_cast<u32>(p[k + i]) << (16 * (i & 1));
    }
    return v;
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// Tiles with the summed axis along their rows: [rows][64], 16-byte pieces of a row at piece ^ (row & 7), so that the 16 rows of a
// fragment lie in different banks although rows are 128 bytes apart.
__device__ inline u32 along_at(u32 row, u32 piece) { return row * 64 + ((piece ^ (row & 7u)) << 3); }
__device__ inline u32x4 along_frag(const u16* tile, u32 row0, u32 sub) {        // sub: which 32 of the 64
    const u32 l = threadIdx.x & 63;
    return *reinterpret_cast<const u32x4*>(tile + along_at(row0 + (l & 15), sub * 4 + (l >> 4)));
}

// Tiles with the summed axis across their rows: [k][COLS].  The transposing load hands 16 lanes four rows of 16 columns: lane s reads
// row s / 4, columns 4 (s % 4) .. + 3, and receives column s of the four rows.  Pieces of 16 bytes are moved so that the rows that are read
// together lie in different banks.
template <u32 COLS>
__device__ inline u32 across_at(u32 k, u32 piece) {
    constexpr u32 kPieces = COLS / 8;
    const u32 slot = kPieces >= 16 ? ((k & 3u) | ((k >> 1) & 4u)) << 1 : (kPieces >= 8 ? (k & 3u) << 1 : 0u);
    return k * COLS + ((piece ^ slot) << 3);
}
template <u32 COLS>
__device__ inline u32x4 across_frag(const u16* tile, u32 col0, u32 sub) {
    const u32 l = threadIdx.x & 63, s = l & 15;
    const u32 k = sub * 32 + (l >> 4) * 8 + (s >> 2);
    const u32 piece = (col0 >> 3) + (s >> 1 & 1), half = (s & 1) * 4;
    const u16* lo = tile + across_at<COLS>(k, piece) + half;
    const u16* hi = tile + across_at<COLS>(k + 4, piece) + half;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lo), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)hi);
    u32x4 v;
    const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
    v.x = x.x; v.y = x.y; v.z = y.x; v.w = y.y;
    return v;
}

__device__ __align__(256) const u16 g_zeros[64] = {};        // where pieces outside a matrix are read from

// Ends a step whose next tile is on its way into LDS: a barrier alone orders LDS accesses, but loads into LDS count as loads from memory.
__device__ inline void sync_staged() {
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    __syncthreads();
}

// The adapter of a token; -1 for none and for values outside the list.
__device__ inline int adapter_of(const int* __restrict__ ids, u32 t, u32 n_tokens, u32 n_adapters) {
    const int a = t < n_tokens ? ids[t] : -1;
    return static_cast<u32>(a) < n_adapters ? a : -1;
}
// Smallest id above `last` among 64 lanes' ids (or INT_MAX).
__device__ inline int next_adapter(int id, int last) {
    int x = id > last ? id : 0x7FFFFFFF;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const int y = __shfl_xor(x, d, 64);
        x = x < y ? x : y;
    }
    return x;
}

// ---- down: the product with the narrow matrix -------------------------------------------------------------------

struct DownArgs {
    const u16* x; i64 ldx;               // [n_tokens, n_sum]
    u32 n_tokens, n_sum;
    const int* ids;
    const AdapterDesc* ad;
    u32 n_adapters, max_rank;
    u16* zp; u32 rp;                     // [n_tokens, rp] 16-bit, zeros past the rank; rp = max_rank rounded up to 32
    u16* z; i64 ldz;                     // the caller's copy, or NULL; all ldz columns are written
    float* z32;                          // [n_tokens, rp] before rounding, or NULL
    u32* row_max;                        // largest finite magnitude of each token's z (bits), or NULL
    u32 vec_x, vec_m;                    // 16-byte aligned rows of x / of the narrow matrix
    // blocks past the tiles sort the tokens by adapter (backward)
    u32 tiles;
    u32* order;                          // tokens of adapter 0, 1, ... in ascending order
    uint2* seg;                          // [n_adapters] first place in `order`, count
    u32* slots;                          // [n_slots] adapter of a run of tokens, or ~0
    u32 n_slots, run;                    // tokens of a run
};

constexpr int kDownTokens = 32, kDownWaves = 8, kDownRanks = 64;

// Places of the runs of an adapter whose tokens begin at `first`: run j of it is slot first / run + a + j.  (One slot at least for
// each adapter; the slots of different adapters never meet, since ceil(n / run) <= floor((first + n) / run) - floor(first / run) + 1.)
__device__ inline u32 first_slot(u32 first, u32 run, u32 a) { return first / run + a; }

// One wavefront an adapter: two passes over the ids, the first counts, the second writes.
__device__ inline void sort_tokens(const DownArgs& p, u32 a) {
    const u32 lane = threadIdx.x & 63;
    u32 less = 0, mine = 0;
    for (u32 t = 0; t < p.n_tokens; t += 256) {
        int id[4];
#pragma unroll
        for (u32 i = 0; i < 4; ++i) id[i] = adapter_of(p.ids, t + i * 64 + lane, p.n_tokens, p.n_adapters);
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            less += static_cast<u32>(__popcll(__ballot(id[i] >= 0 && id[i] < static_cast<int>(a))));
            mine += static_cast<u32>(__popcll(__ballot(id[i] == static_cast<int>(a))));
        }
    }
    if (lane == 0) p.seg[a] = make_uint2(less, mine);
    const u32 s0 = first_slot(less, p.run, a), s1 = a + 1 < p.n_adapters ? first_slot(less + mine, p.run, a + 1) : p.n_slots;
    const u32 runs = mine == 0 ? 1 : (mine + p.run - 1) / p.run;
    for (u32 s = s0 + lane; s < s1; s += 64) p.slots[s] = s - s0 < runs ? a : ~0u;
    u32 at = less;
    if (mine == 0) return;                                   // uniform
    for (u32 t = 0; t < p.n_tokens; t += 256) {
        int id[4];
#pragma unroll
        for (u32 i = 0; i < 4; ++i) id[i] = adapter_of(p.ids, t + i * 64 + lane, p.n_tokens, p.n_adapters);
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            const u64 same = __ballot(id[i] == static_cast<int>(a));
            if (id[i] == static_cast<int>(a)) p.order[at + static_cast<u32>(__popcll(same & ((1ull << lane) - 1ull)))] = t + i * 64 + lane;
            at += static_cast<u32>(__popcll(same));
        }
    }
}

// z = s x M_a^T for 32 tokens a workgroup, where M_a is the adapter's A [rank, n_sum] (ALONG), or its B [n_sum, rank] in the backward
// pass.  Reading x bounds it: each row is read once, by eight wavefronts that take every eighth piece of 32 values of it straight into
// operand registers (nothing of x is shared between wavefronts, so LDS would only add a trip) and add their sums up at the end.
// Thirty-two tokens share what is read of M_a.  Tokens of several adapters in one tile are done one adapter after the other.
template <typename E, bool ALONG, bool VECX>
__global__ __launch_bounds__(64 * kDownWaves) void k_adapter_down(DownArgs p) {
    __shared__ __align__(16) float sums[kDownWaves][kDownTokens][kDownRanks];
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (blockIdx.x >= p.tiles) {                             // uniform
        const u32 a = (blockIdx.x - p.tiles) * kDownWaves + wave;
        if (a < p.n_adapters) sort_tokens(p, a);
        return;
    }
    const u32 t0 = blockIdx.x * kDownTokens;
    const int my_id = lane < kDownTokens ? adapter_of(p.ids, t0 + lane, p.n_tokens, p.n_adapters) : -1;
    const u32 width = p.z && p.ldz > p.rp ? static_cast<u32>(p.ldz) : p.rp;
    // tokens without an adapter
    for (u32 i = wave; i < kDownTokens; i += kDownWaves) {
        const u32 t = t0 + i;
        if (t >= p.n_tokens || __shfl(my_id, static_cast<int>(i), 64) >= 0) continue;
        for (u32 j = lane; j < width; j += 64) {
            if (j < p.rp) { p.zp[static_cast<u64>(t) * p.rp + j] = 0; if (p.z32) p.z32[static_cast<u64>(t) * p.rp + j] = 0.0f; }
            if (p.z && j < p.ldz) p.z[static_cast<u64>(t) * p.ldz + j] = 0;
        }
    }
    const u32 steps = (p.n_sum + 31) / 32, row = lane & 15, sub = (lane >> 4) * 8;
    u32 ta = t0 + row, tb = t0 + 16 + row;
    if (ta >= p.n_tokens) ta = p.n_tokens - 1;               // their sums are not stored
    if (tb >= p.n_tokens) tb = p.n_tokens - 1;
    const u16* xa = p.x + static_cast<i64>(ta) * p.ldx;
    const u16* xb = p.x + static_cast<i64>(tb) * p.ldx;
    for (int a = next_adapter(my_id, -1); a != 0x7FFFFFFF; a = next_adapter(my_id, a)) {       // uniform over the workgroup
        const AdapterDesc& d = p.ad[a];
        const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
        const u16* m = ALONG ? d.a : d.b;
        for (u32 r0 = 0; r0 == 0 || r0 < rank; r0 += kDownRanks) {
            const u32 ranks = rank - r0 < static_cast<u32>(kDownRanks) ? rank - r0 : static_cast<u32>(kDownRanks);
            const u32 groups = (ranks + 15) / 16;
            f32x4 acc[2][4] = {};
            for (u32 s = wave; s < steps; s += kDownWaves) {
                const i64 k = static_cast<i64>(s) * 32 + sub;
                const u32x4 fa = load8<VECX>(xa, k, p.n_sum), fb = load8<VECX>(xb, k, p.n_sum);
#pragma unroll
                for (u32 g = 0; g < 4; ++g) {
                    if (g >= groups) continue;               // uniform
                    const u32 j = r0 + g * 16 + row;
                    u32x4 fm = {0u, 0u, 0u, 0u};
                    if (ALONG) {
                        if (j < rank) fm = p.vec_m ? load8<true>(m + static_cast<i64>(j) * p.n_sum, k, p.n_sum) : load8<false>(m + static_cast<i64>(j) * p.n_sum, k, p.n_sum);
                    } else if (j < rank) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (k + i < p.n_sum) fm[i >> 1] |= static_cast<u32>(m[(k + i) * rank + j]) << (16 * (i & 1));
                    }
                    acc[0][g] = E::mfma(fa, fm, acc[0][g]);
                    acc[1][g] = E::mfma(fb, fm, acc[1][g]);
                }
            }
            __syncthreads();                                 // the sums of the round before are read
#pragma unroll
            for (u32 h = 0; h < 2; ++h)
#pragma unroll
                for (u32 g = 0; g < 4; ++g) {
                    if (g >= groups) continue;
#pragma unroll
                    for (u32 i = 0; i < 4; ++i) sums[wave][h * 16 + (lane >> 4) * 4 + i][g * 16 + row] = acc[h][g][i];
                }
            __syncthreads();
            const bool last = r0 + kDownRanks >= rank;
            const u32 end = last ? width : r0 + kDownRanks;
            for (u32 i = wave; i < kDownTokens; i += kDownWaves) {
                if (__shfl(my_id, static_cast<int>(i), 64) != a) continue;       // uniform
                const u64 t = t0 + i;
                u32 most = 0;
                for (u32 j = r0 + lane; j < end; j += 64) {
                    float v = 0.0f;
                    if (j < rank) {
#pragma unroll
                        for (int w = 0; w < kDownWaves; ++w) v += sums[w][i][j - r0];
                        v *= d.scale;
                    }
                    const u16 h = E::enc(v);
                    if (j < p.rp) { p.zp[t * p.rp + j] = h; if (p.z32) p.z32[t * p.rp + j] = v; }
                    if (p.z && j < p.ldz) p.z[t * p.ldz + j] = h;
                    const u32 u = __float_as_uint(v) & 0x7FFFFFFFu;
                    if (u < 0x7F800000u) most = most > u ? most : u;
                }
                if (p.row_max) {                             // the same wavefront has the row in every round
#pragma unroll
                    for (int d2 = 32; d2 >= 1; d2 >>= 1) {
                        const u32 o = static_cast<u32>(__shfl_xor(static_cast<int>(most), d2, 64));
                        most = most > o ? most : o;
                    }
                    if (lane == 0) {
                        const u32 before = r0 ? p.row_max[t] : 0u;
                        p.row_max[t] = most > before ? most : before;
                    }
                }
            }
        }
    }
}

// ---- the wide product with the adapters' share added ------------------------------------------------------------

struct WideArgs {
    const u16* x; i64 ldx;               // [n_tokens, n_sum]
    const u16* w; i64 ldw;               // ALONG: [n_out, n_sum], else [n_sum, n_out]
    u16* y; i64 ldy;                     // [n_tokens, n_out]
    u32 n_tokens, n_out, n_sum;
    const u16* zp; u32 rp;
    const int* ids;
    const AdapterDesc* ad;
    u32 n_adapters, max_rank;
    u32 vec_m;                           // 16-byte aligned rows of the adapters' matrix
    u32 vec_y;                           // 8-byte aligned groups of four outputs
};

// Workgroups go round the eight dies one by one; this gives each die a run of neighbouring tiles, whose rows its cache keeps.
__device__ inline u32 die_order(u32 i, u32 n) {
    const u32 die = i & 7u, k = i >> 3, each = n >> 3, more = n & 7u;
    return die * each + (die < more ? die : more) + k;
}

// Tiles of BM tokens by BN outputs, summed 64 values a step.
template <typename E, int BM, int BN, int WM, int WN, bool ALONG, bool VEC>
__global__ __launch_bounds__(64 * WM * WN) void k_adapter_wide(WideArgs p) {
    constexpr u32 kThreads = 64 * WM * WN;
    constexpr u32 TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr u32 kXPieces = BM * 8 / kThreads, kWPieces = BN * 8 / kThreads;
    __shared__ __align__(16) u16 sx0[BM * 64], sw0[BN * 64], sx1[BM * 64], sw1[BN * 64];
    __shared__ int s_ids[BM];
    const u32 tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const u32 wm = wave / WN, wn = wave % WN;
    const u32 tiles_n = (p.n_out + BN - 1) / BN;
    const u32 tile = die_order(blockIdx.x, gridDim.x);
    const u32 t0 = tile / tiles_n * BM, n0 = tile % tiles_n * BN;
    f32x4 acc[FN][FM] = {};

    auto x_src = [&](u32 i, u32 k0) -> const u16* {            // piece i of this thread in step k0, or nullptr outside
        const u32 at = i * kThreads + tid, row = at >> 3, piece = (at & 7u) ^ (row & 7u);
        u32 t = t0 + row;
        if (t >= p.n_tokens) t = p.n_tokens - 1;
        return p.x + static_cast<i64>(t) * p.ldx + k0 + piece * 8;
    };
    auto stage = [&](u16* sx, u16* sw, u32 k0) {               // VEC: straight into LDS, 16 bytes a lane
#pragma unroll
        for (u32 i = 0; i < kXPieces; ++i) {
            const u32 at = i * kThreads + tid, piece = (at & 7u) ^ ((at >> 3) & 7u);
            const u16* src = k0 + piece * 8 < p.n_sum ? x_src(i, k0) : g_zeros;
            __builtin_amdgcn_global_load_lds((global_void*)src, (lds_void*)(sx + (i * kThreads + wave * 64) * 8), 16, 0, 0);
        }
#pragma unroll
        for (u32 i = 0; i < kWPieces; ++i) {
            const u32 at = i * kThreads + tid;
            const u16* src;
            if (ALONG) {
                const u32 row = at >> 3, piece = (at & 7u) ^ (row & 7u);
                u32 n = n0 + row;
                if (n >= p.n_out) n = p.n_out - 1;
                src = k0 + piece * 8 < p.n_sum ? p.w + static_cast<i64>(n) * p.ldw + k0 + piece * 8 : g_zeros;
            } else {
                constexpr u32 kRow = BN / 8;
                const u32 k = at / kRow, piece = ((across_at<BN>(k, at % kRow) - k * BN) >> 3);
                src = k0 + k < p.n_sum && n0 + piece * 8 < p.n_out ? p.w + static_cast<i64>(k0 + k) * p.ldw + n0 + piece * 8 : g_zeros;
            }
            __builtin_amdgcn_global_load_lds((global_void*)src, (lds_void*)(sw + (i * kThreads + wave * 64) * 8), 16, 0, 0);
        }
    };
    u32x4 rx[VEC ? 1 : kXPieces], rw[VEC ? 1 : kWPieces];
    auto fetch = [&](u32 k0) {                                 // not VEC: through registers
#pragma unroll
        for (u32 i = 0; i < kXPieces; ++i) {
            const u32 at = i * kThreads + tid, row = at >> 3, piece = at & 7u;
            u32 t = t0 + row;
            if (t >= p.n_tokens) t = p.n_tokens - 1;
            rx[VEC ? 0 : i] = load8<false>(p.x + static_cast<i64>(t) * p.ldx, k0 + piece * 8, p.n_sum);
        }
#pragma unroll
        for (u32 i = 0; i < kWPieces; ++i) {
            const u32 at = i * kThreads + tid;
            if (ALONG) {
                u32 n = n0 + (at >> 3);
                if (n >= p.n_out) n = p.n_out - 1;
                rw[VEC ? 0 : i] = load8<false>(p.w + static_cast<i64>(n) * p.ldw, k0 + (at & 7u) * 8, p.n_sum);
            } else {
                constexpr u32 kRow = BN / 8;
                const u32 k = at / kRow;
                rw[VEC ? 0 : i] = k0 + k < p.n_sum ? load8<false>(p.w + static_cast<i64>(k0 + k) * p.ldw, n0 + (at % kRow) * 8, p.n_out) : u32x4{0u, 0u, 0u, 0u};
            }
        }
    };
    auto put = [&](u16* sx, u16* sw) {
#pragma unroll
        for (u32 i = 0; i < kXPieces; ++i) {
            const u32 at = i * kThreads + tid;
            *reinterpret_cast<u32x4*>(sx + along_at(at >> 3, at & 7u)) = rx[VEC ? 0 : i];
        }
#pragma unroll
        for (u32 i = 0; i < kWPieces; ++i) {
            const u32 at = i * kThreads + tid;
            const u32 to = ALONG ? along_at(at >> 3, at & 7u) : across_at<BN>(at / (BN / 8), at % (BN / 8));
            *reinterpret_cast<u32x4*>(sw + to) = rw[VEC ? 0 : i];
        }
    };
    auto multiply = [&](const u16* sx, const u16* sw) {
#pragma unroll
        for (u32 sub = 0; sub < 2; ++sub) {
            u32x4 fx[FM], fw[FN];
#pragma unroll
            for (u32 i = 0; i < FM; ++i) fx[i] = along_frag(sx, wm * TM + i * 16, sub);
#pragma unroll
            for (u32 i = 0; i < FN; ++i) fw[i] = ALONG ? along_frag(sw, wn * TN + i * 16, sub) : across_frag<BN>(sw, wn * TN + i * 16, sub);
#pragma unroll
            for (u32 i = 0; i < FN; ++i)
#pragma unroll
                for (u32 j = 0; j < FM; ++j) acc[i][j] = E::mfma(fw[i], fx[j], acc[i][j]);
        }
    };

    // The adapter's product is added where the token is the adapter's and nowhere else: zeros in its place would spread infinities and
    // NaN of one request's adapter to its neighbours.
    auto multiply_own = [&](const u16* sx, const u16* sw, u32 subs, int a) {
#pragma unroll
        for (u32 sub = 0; sub < 2; ++sub) {
            if (sub >= subs) continue;
            u32x4 fw[FN];
#pragma unroll
            for (u32 i = 0; i < FN; ++i) fw[i] = ALONG ? along_frag(sw, wn * TN + i * 16, sub) : across_frag<BN>(sw, wn * TN + i * 16, sub);
#pragma unroll
            for (u32 j = 0; j < FM; ++j) {
                const bool mine = s_ids[wm * TM + j * 16 + (lane & 15)] == a;
                const u32x4 fx = along_frag(sx, wm * TM + j * 16, sub);
#pragma unroll
                for (u32 i = 0; i < FN; ++i) {
                    const f32x4 v = E::mfma(fw[i], fx, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                    for (u32 k = 0; k < 4; ++k) acc[i][j][k] = mine ? acc[i][j][k] + v[k] : acc[i][j][k];
                }
            }
        }
    };

    for (u32 i = tid; i < BM; i += kThreads) s_ids[i] = adapter_of(p.ids, t0 + i, p.n_tokens, p.n_adapters);
    if (VEC) {
        stage(sx0, sw0, 0);
        sync_staged();
        for (u32 k0 = 0; k0 < p.n_sum; k0 += 128) {
            if (k0 + 64 < p.n_sum) stage(sx1, sw1, k0 + 64);
            multiply(sx0, sw0);
            sync_staged();
            if (k0 + 64 < p.n_sum) {
                if (k0 + 128 < p.n_sum) stage(sx0, sw0, k0 + 128);
                multiply(sx1, sw1);
                sync_staged();
            }
        }
    } else {
        fetch(0);
        for (u32 k0 = 0; k0 < p.n_sum; k0 += 64) {
            put(sx0, sw0);
            __syncthreads();
            if (k0 + 64 < p.n_sum) fetch(k0 + 64);
            multiply(sx0, sw0);
            __syncthreads();
        }
    }

    // the adapters' share: one more step of the sum for each adapter that the tile's tokens have
    __syncthreads();
    int last = -1;
    for (;;) {
        int a = 0x7FFFFFFF;
        for (u32 i = lane; i < BM; i += 64) {
            const int id = s_ids[i];
            if (id > last && id < a) a = id;
        }
        a = next_adapter(a, -1);                               // the same in every wavefront
        if (a == 0x7FFFFFFF) break;
        last = a;
        const AdapterDesc& d = p.ad[a];
        const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
        const u16* m = ALONG ? d.b : d.a;
        for (u32 r0 = 0; r0 < rank; r0 += 64) {
            const u32 subs = rank - r0 > 32 ? 2 : 1;
            for (u32 at = tid; at < BM * 8; at += kThreads) {
                const u32 row = at >> 3, piece = at & 7u;
                if (piece >= subs * 4) continue;
                u32x4 v = {0u, 0u, 0u, 0u};
                if (s_ids[row] == a) v = load8<true>(p.zp + static_cast<u64>(t0 + row) * p.rp, r0 + piece * 8, p.rp);
                *reinterpret_cast<u32x4*>(sx0 + along_at(row, piece)) = v;
            }
            for (u32 at = tid; at < BN * 8; at += kThreads) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (ALONG) {
                    const u32 row = at >> 3, piece = at & 7u;
                    if (piece >= subs * 4) continue;
                    if (n0 + row < p.n_out) {
                        const u16* src = m + static_cast<i64>(n0 + row) * rank;
                        v = p.vec_m ? load8<true>(src, r0 + piece * 8, rank) : load8<false>(src, r0 + piece * 8, rank);
                    }
                    *reinterpret_cast<u32x4*>(sw0 + along_at(row, piece)) = v;
                } else {
                    constexpr u32 kRow = BN / 8;
                    const u32 k = at / kRow, piece = at % kRow;
                    if (k >= subs * 32) continue;
                    if (r0 + k < rank) {
                        const u16* src = m + static_cast<i64>(r0 + k) * p.n_out;
                        v = p.vec_m ? load8<true>(src, n0 + piece * 8, p.n_out) : load8<false>(src, n0 + piece * 8, p.n_out);
                    }
                    *reinterpret_cast<u32x4*>(sw0 + across_at<BN>(k, piece)) = v;
                }
            }
            __syncthreads();
            multiply_own(sx0, sw0, subs, a);
            __syncthreads();
        }
    }

#pragma unroll
    for (u32 j = 0; j < FM; ++j) {
        const u32 t = t0 + wm * TM + j * 16 + (lane & 15);
        if (t >= p.n_tokens) continue;
        u16* out = p.y + static_cast<i64>(t) * p.ldy;
#pragma unroll
        for (u32 i = 0; i < FN; ++i) {
            const u32 n = n0 + wn * TN + i * 16 + (lane >> 4) * 4;
            u16 h[4];
#pragma unroll
            for (u32 k = 0; k < 4; ++k) h[k] = E::enc(acc[i][j][k]);
            if (p.vec_y && n + 4 <= p.n_out) {
                u32x2 v;
                v.x = static_cast<u32>(h[0]) | static_cast<u32>(h[1]) << 16;
                v.y = static_cast<u32>(h[2]) | static_cast<u32>(h[3]) << 16;
                *reinterpret_cast<u32x2*>(out + n) = v;
            } else {
#pragma unroll
                for (u32 k = 0; k < 4; ++k) if (n + k < p.n_out) out[n + k] = h[k];
            }
        }
    }
}

// ---- few tokens -------------------------------------------------------------------------------------------------

struct FewArgs {
    WideArgs wide;
    float* part;                         // [splits][n_tokens][n_out]
    float* z32;                          // [n_tokens][max_rank]
    u16* z; i64 ldz;
    u32 tiles_n, splits, steps_each;     // steps of 32 values that a split sums
    u32 vec_a;
};

constexpr u32 kFewCols = 64, kFewWaves = 8;

// Up to 64 tokens: reading the weights once bounds it.  One launch reads everything that does not wait for anything: workgroups of
// 64 outputs and a part of the sum (two times 32 outputs by four interleaved quarters of it, added up in LDS) and one workgroup a token that
// makes z; the next launch adds the parts and z B^T.  Weights go from memory straight to operand registers; FM tiles of 16 tokens use
// them at once.
template <typename E, u32 FM, bool VEC>
__global__ __launch_bounds__(64 * kFewWaves) void k_adapter_few(FewArgs p) {
    __shared__ __align__(16) float sums[4 * 2 * 2 * FM * 256];
    const WideArgs& g = p.wide;
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, sub = (lane >> 4) * 8;
    const u32 steps = (g.n_sum + 31) / 32;
    if (blockIdx.x >= p.tiles_n * p.splits) {                  // z of one token: all eight wavefronts share its sum
        const u32 t = blockIdx.x - p.tiles_n * p.splits;
        const int a = adapter_of(g.ids, t, g.n_tokens, g.n_adapters);
        const u32 rank = a < 0 ? 0 : (g.ad[a].rank < g.max_rank ? g.ad[a].rank : g.max_rank);
        const u16* x = g.x + static_cast<i64>(t) * g.ldx;
        for (u32 r0 = 0; r0 < rank; r0 += 16) {
            f32x4 acc = {};
            const u32 j = r0 + row;
            const u16* m = g.ad[a].a + static_cast<i64>(j < rank ? j : 0) * g.n_sum;
#pragma unroll 4
            for (u32 s = wave; s < steps; s += kFewWaves) {
                const i64 k = static_cast<i64>(s) * 32 + sub;
                const u32x4 fm = p.vec_a ? load8<true>(m, k, g.n_sum) : load8<false>(m, k, g.n_sum);
                acc = E::mfma(fm, load8<VEC>(x, k, g.n_sum), acc);       // the token in every column
            }
            __syncthreads();
            if (row == 0)
#pragma unroll
                for (u32 i = 0; i < 4; ++i) sums[wave * 16 + (lane >> 4) * 4 + i] = acc[i];
            __syncthreads();
            if (threadIdx.x < 16 && r0 + threadIdx.x < rank) {
                float v = 0.0f;
#pragma unroll
                for (u32 w = 0; w < kFewWaves; ++w) v += sums[w * 16 + threadIdx.x];
                p.z32[static_cast<u64>(t) * g.max_rank + r0 + threadIdx.x] = v * g.ad[a].scale;
            }
        }
        return;
    }
    const u32 tile = blockIdx.x % p.tiles_n, split = blockIdx.x / p.tiles_n;
    const u32 part = wave >> 1, n0 = tile * kFewCols + (wave & 1) * 32;
    const u32 begin = split * p.steps_each, end = begin + p.steps_each < steps ? begin + p.steps_each : steps;
    const u16* w[2];
    const u16* x[FM];
#pragma unroll
    for (u32 i = 0; i < 2; ++i) {
        u32 n = n0 + i * 16 + row;
        if (n >= g.n_out) n = g.n_out - 1;
        w[i] = g.w + static_cast<i64>(n) * g.ldw;
    }
#pragma unroll
    for (u32 i = 0; i < FM; ++i) {
        u32 t = i * 16 + row;
        if (t >= g.n_tokens) t = g.n_tokens - 1;
        x[i] = g.x + static_cast<i64>(t) * g.ldx;
    }
    f32x4 acc[2][FM] = {};
#pragma unroll 2
    for (u32 s = begin + part; s < end; s += 4) {
        const i64 k = static_cast<i64>(s) * 32 + sub;
        u32x4 fw[2], fx[FM];
#pragma unroll
        for (u32 i = 0; i < 2; ++i) fw[i] = load8<VEC>(w[i], k, g.n_sum);
#pragma unroll
        for (u32 i = 0; i < FM; ++i) fx[i] = load8<VEC>(x[i], k, g.n_sum);
#pragma unroll
        for (u32 i = 0; i < 2; ++i)
#pragma unroll
            for (u32 j = 0; j < FM; ++j) acc[i][j] = E::mfma(fw[i], fx[j], acc[i][j]);
    }
#pragma unroll
    for (u32 i = 0; i < 2; ++i)
#pragma unroll
        for (u32 j = 0; j < FM; ++j) *reinterpret_cast<f32x4*>(&sums[((((part * 2 + (wave & 1)) * 2 + i) * FM + j) * 64 + lane) * 4]) = acc[i][j];
    __syncthreads();
    for (u32 at = threadIdx.x; at < 2 * 2 * FM * 64; at += 64 * kFewWaves) {
        f32x4 v = *reinterpret_cast<const f32x4*>(&sums[at * 4]);
#pragma unroll
        for (u32 q = 1; q < 4; ++q) v += *reinterpret_cast<const f32x4*>(&sums[(q * 2 * 2 * FM * 64 + at) * 4]);
        const u32 l = at & 63, j = at / 64 % FM, i = at / 64 / FM % 2, half = at / 64 / FM / 2;
        const u32 t = j * 16 + (l & 15), n = tile * kFewCols + half * 32 + i * 16 + (l >> 4) * 4;
        if (t >= g.n_tokens) continue;
        float* out = p.part + (static_cast<u64>(split) * g.n_tokens + t) * g.n_out + n;
        if ((g.n_out & 3u) == 0 && n + 4 <= g.n_out) *reinterpret_cast<f32x4*>(out) = v;
        else
#pragma unroll
            for (u32 q = 0; q < 4; ++q) if (n + q < g.n_out) out[q] = v[q];
    }
}

// y = the parts added in order + z B^T, one output a thread; z is kept in binary32 here.
template <typename E>
__global__ __launch_bounds__(256) void k_adapter_few_join(FewArgs p) {
    const WideArgs& g = p.wide;
    const u32 t = blockIdx.y, n = blockIdx.x * 256 + threadIdx.x;
    const int a = adapter_of(g.ids, t, g.n_tokens, g.n_adapters);
    const u32 rank = a < 0 ? 0 : (g.ad[a].rank < g.max_rank ? g.ad[a].rank : g.max_rank);
    const float* z = p.z32 + static_cast<u64>(t) * g.max_rank;
    if (p.z && blockIdx.x == 0)
        for (u32 j = threadIdx.x; j < p.ldz; j += 256) p.z[static_cast<u64>(t) * p.ldz + j] = j < rank ? E::enc(z[j]) : static_cast<u16>(0);
    if (n >= g.n_out) return;
    float v = 0.0f;
    for (u32 s = 0; s < p.splits; ++s) v += p.part[(static_cast<u64>(s) * g.n_tokens + t) * g.n_out + n];
    if (rank) {
        const u16* b = g.ad[a].b + static_cast<i64>(n) * rank;
        float u = 0.0f;
        for (u32 j = 0; j < rank; j += 8) {
            const u32x4 h = g.vec_m ? load8<true>(b, j, rank) : load8<false>(b, j, rank);
#pragma unroll
            for (u32 i = 0; i < 8; ++i) if (j + i < rank) u = __builtin_fmaf(z[j + i], E::dec(static_cast<u16>(h[i >> 1] >> (16 * (i & 1)))), u);
        }
        v += u;
    }
    g.y[static_cast<i64>(t) * g.ldy + n] = E::enc(v);
}

// ---- gradients of the adapters ----------------------------------------------------------------------------------

struct GradArgs {
    const u16* x; i64 ldx; u32 n_in;     // grad_a = sum of dz^T x
    const u16* dy; i64 ldy; u32 n_out;   // grad_b = sum of dy^T z
    const float* dz; u32 rp;
    const u16* z; i64 ldz;
    const u32* row_max;
    const u32* order;
    const uint2* seg;
    const u32* slots;
    const AdapterDesc* ad;
    u32 max_rank, run, tiles_in, tiles, vec;
    float* part;                         // [n_slots][max_rank (n_in + n_out)]
};

constexpr u32 kGradCols = 128, kGradStep = 64;

// One run of one adapter's tokens times 128 columns of x or of dy: 64 tokens a step, both operands across the rows of their tiles.
// dz enters as the sum of two 16-bit values, so that a binary32 gradient keeps 16 bits of it (22 with float16) and not 8; runs of
// float16 are scaled by a power of two first, so that the largest dz of the run sits near the top of the type's range.
template <typename E, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_grads(GradArgs p) {
    __shared__ __align__(16) u16 sv[kGradStep * kGradCols], su[kGradStep * 64], sl[kGradStep * 64];
    __shared__ u32 s_tok[kGradStep];
    __shared__ u32 s_max;
    const u32 tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const u32 slot = blockIdx.x / p.tiles, col_tile = blockIdx.x % p.tiles, r0 = blockIdx.y * 64;
    const u32 a = p.slots[slot];
    if (a == ~0u) return;                                      // uniform, as all that follow
    const AdapterDesc& d = p.ad[a];
    const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
    if (r0 >= rank) return;
    const uint2 seg = p.seg[a];
    const u32 j = slot - first_slot(seg.x, p.run, a);
    const u32 first = seg.x + j * p.run, count = seg.y < j * p.run ? 0 : (seg.y - j * p.run < p.run ? seg.y - j * p.run : p.run);
    const bool of_a = col_tile < p.tiles_in;
    const u32 c0 = (of_a ? col_tile : col_tile - p.tiles_in) * kGradCols;
    const u32 n_cols = of_a ? p.n_in : p.n_out;
    const u16* v_src = of_a ? p.x : p.dy;
    const i64 ldv = of_a ? p.ldx : p.ldy;
    float up = 1.0f, down = 1.0f;
    if (E::kNarrow && of_a) {
        if (tid == 0) s_max = 0;
        __syncthreads();
        u32 most = 0;
        for (u32 i = tid; i < count; i += 256) { const u32 m = p.row_max[p.order[first + i]]; most = most > m ? most : m; }
        atomicMax(&s_max, most);
        __syncthreads();
        int e = 14 - (static_cast<int>(s_max >> 23) - 127);    // the largest becomes 2^14 .. 2^15
        e = e > 120 ? 120 : (e < -100 ? -100 : e);
        up = __uint_as_float(static_cast<u32>(127 + e) << 23);
        down = __uint_as_float(static_cast<u32>(127 - e) << 23);
    }
    f32x4 acc[2][4] = {};
    for (u32 s = 0; s < count; s += kGradStep) {
        __syncthreads();
        if (tid < kGradStep) s_tok[tid] = s + tid < count ? p.order[first + s + tid] : ~0u;
        __syncthreads();
#pragma unroll
        for (u32 i = 0; i < kGradStep * kGradCols / 8 / 256; ++i) {
            const u32 at = i * 256 + tid, k = at / (kGradCols / 8), piece = at % (kGradCols / 8), t = s_tok[k];
            u32x4 v = {0u, 0u, 0u, 0u};
            if (t != ~0u) v = load8<VEC>(v_src + static_cast<i64>(t) * ldv, c0 + piece * 8, n_cols);
            *reinterpret_cast<u32x4*>(sv + across_at<kGradCols>(k, piece)) = v;
        }
        for (u32 at = tid; at < kGradStep * 8; at += 256) {
            const u32 k = at >> 3, piece = at & 7u, t = s_tok[k], c = r0 + piece * 8;
            u32x4 hi = {0u, 0u, 0u, 0u}, lo = {0u, 0u, 0u, 0u};
            if (t != ~0u && c < rank) {
                if (of_a) {
                    const float* src = p.dz + static_cast<u64>(t) * p.rp + c;        // zeros past the rank
#pragma unroll
                    for (u32 i = 0; i < 8; ++i) {
                        const float f = src[i] * up;
                        const u16 h = E::enc(f);
                        const float rest = f - E::dec(h);
                        const u16 l = __builtin_fabsf(rest) < INFINITY ? E::enc(rest) : static_cast<u16>(0);
                        hi[i >> 1] |= static_cast<u32>(h) << (16 * (i & 1));
                        lo[i >> 1] |= static_cast<u32>(l) << (16 * (i & 1));
                    }
                } else {
                    hi = load8<false>(p.z + static_cast<i64>(t) * p.ldz, c, rank);
                }
            }
            *reinterpret_cast<u32x4*>(su + across_at<64>(k, piece)) = hi;
            if (of_a) *reinterpret_cast<u32x4*>(sl + across_at<64>(k, piece)) = lo;
        }
        __syncthreads();
#pragma unroll
        for (u32 sub = 0; sub < 2; ++sub) {
            u32x4 fv[2];
#pragma unroll
            for (u32 i = 0; i < 2; ++i) fv[i] = across_frag<kGradCols>(sv, wave * 32 + i * 16, sub);
#pragma unroll
            for (u32 g = 0; g < 4; ++g) {
                if (r0 + g * 16 >= rank) continue;
                const u32x4 fu = across_frag<64>(su, g * 16, sub);
                if (of_a) {
                    const u32x4 fl = across_frag<64>(sl, g * 16, sub);
#pragma unroll
                    for (u32 i = 0; i < 2; ++i) acc[i][g] = E::mfma(fv[i], fl, E::mfma(fv[i], fu, acc[i][g]));
                } else {
#pragma unroll
                    for (u32 i = 0; i < 2; ++i) acc[i][g] = E::mfma(fu, fv[i], acc[i][g]);
                }
            }
        }
    }
    const bool whole = seg.y <= p.run;
    float* out = whole ? (of_a ? d.grad_a : d.grad_b)
                       : p.part + static_cast<u64>(slot) * p.max_rank * (static_cast<u64>(p.n_in) + p.n_out) + (of_a ? 0 : static_cast<u64>(rank) * p.n_in);
#pragma unroll
    for (u32 i = 0; i < 2; ++i)
#pragma unroll
        for (u32 g = 0; g < 4; ++g)
#pragma unroll
            for (u32 q = 0; q < 4; ++q) {
                const float v = acc[i][g][q] * down;
                if (of_a) {                                    // rows of the result are columns of x
                    const u32 r = r0 + g * 16 + (lane & 15), c = c0 + wave * 32 + i * 16 + (lane >> 4) * 4 + q;
                    if (r < rank && c < n_cols) out[static_cast<u64>(r) * p.n_in + c] = v;
                } else {
                    const u32 r = r0 + g * 16 + (lane >> 4) * 4 + q, c = c0 + wave * 32 + i * 16 + (lane & 15);
                    if (r < rank && c < n_cols) out[static_cast<u64>(c) * rank + r] = v;
                }
            }
}

// Adapters with several runs: their parts, added in order.
__global__ __launch_bounds__(256) void k_adapter_join(GradArgs p, u32 blocks_each) {
    const u32 a = blockIdx.x / blocks_each;
    const uint2 seg = p.seg[a];
    if (seg.y <= p.run) return;                                // uniform
    const AdapterDesc& d = p.ad[a];
    const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
    const u64 na = static_cast<u64>(rank) * p.n_in, n = na + static_cast<u64>(rank) * p.n_out;
    const u64 each = static_cast<u64>(p.max_rank) * (static_cast<u64>(p.n_in) + p.n_out);
    const u32 s0 = first_slot(seg.x, p.run, a), runs = (seg.y + p.run - 1) / p.run;
    for (u64 i = static_cast<u64>(blockIdx.x % blocks_each) * 256 + threadIdx.x; i < n; i += static_cast<u64>(blocks_each) * 256) {
        float v = p.part[s0 * each + i];
        for (u32 r = 1; r < runs; ++r) v += p.part[(s0 + r) * each + i];
        if (i < na) d.grad_a[i] = v;
        else d.grad_b[i - na] = v;
    }
}

}  // namespace condensa
