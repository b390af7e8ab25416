// Low-rank adapters of many requests beside one shared projection: y = x W^T + z B^T with z = s x A^T, and the gradients.
//
// All products run on the matrix instructions (16x16x32, 16-bit operands, binary32 sums).  An operand fragment of a wavefront is 16
// rows of 32 consecutive values along the summed axis: lane l holds row l % 16, values 8 (l / 16) .. + 7.  Where the summed axis is
// the rows of a matrix in memory, tiles of it lie in LDS as they are and the transposing LDS load collects the fragment.  A result
// tile puts its column in lane l % 16 and its rows 4 (l / 16) .. + 3 in four registers.
#pragma once
#include <type_traits>

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
    static __device__ inline u16 cut(float x) {
        const auto h = __builtin_amdgcn_cvt_pkrtz(x, 0.0f);
        return __builtin_bit_cast(u16, h[0]);
    }
};
struct ElemBF16 {
    static __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
    static __device__ inline u16 enc(float x) { return f32_to_bf16_rne(x); }
    static __device__ inline float dec(u16 h) { return bf16_bits_to_f32(h); }
    static constexpr bool kNarrow = false;
    static __device__ inline u16 cut(float x) { return static_cast<u16>(__float_as_uint(x) >> 16); }
};

struct AdapterDesc {
    const u16* a;              // [rank, n_in]
    const u16* b;              // [n_out, rank]
    float* grad_a;             // NULL where the list is for forward passes
    float* grad_b;
    float scale;
    u32 rank;
    u32 vec_a, vec_b;          // rows are 16-byte aligned and a multiple of eight long
};
static_assert(sizeof(AdapterDesc) == 48, "AdapterDesc layout");

constexpr int kAdapterPoke = 80;           // adapters that one launch writes into the device list
struct AdapterPoke { AdapterDesc d[kAdapterPoke]; };
__global__ __launch_bounds__(256) void k_adapter_list(AdapterDesc* __restrict__ dst, AdapterPoke src, u32 first, u32 count) {
    const u32 words = count * (sizeof(AdapterDesc) / 8);
    for (u32 i = threadIdx.x; i < words; i += 256) reinterpret_cast<u64*>(dst + first)[i] = reinterpret_cast<const u64*>(src.d)[i];
}

// ---- operand access ---------------------------------------------------------------------------------------------

// Sixteen bytes from global memory; of the second form at any address that a 16-bit value may have.  The address space is given because
// pointers that come out of the device list would otherwise be taken for pointers to any memory.
typedef u32 u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef u32 u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ inline u32x4 load16(const u16* p) { return *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>((u64)p); }
__device__ inline u32x4 load16_any(const u16* p) { return *reinterpret_cast<const __attribute__((address_space(1))) u32x4_any*>((u64)p); }
__device__ inline u16 load2(const u16* p) { return *reinterpret_cast<const __attribute__((address_space(1))) u16*>((u64)p); }

// Eight consecutive 16-bit values p[k .. k+7] of a row of n, zeros past its end.  VEC: rows are 16-byte aligned and n and k are
// multiples of eight.
template <bool VEC>
__device__ inline u32x4 load8(const u16* p, i64 k, i64 n) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (VEC) {
        if (k < n) v = load16(p + k);
    } else if (k + 8 <= n) {
        v = load16_any(p + k);
    } else if (k < n) {
        if (n >= 8) {                                        // the row's last eight, moved down
            const u32x4 t = load16_any(p + n - 8);
            u64 lo = static_cast<u64>(t.y) << 32 | t.x, hi = static_cast<u64>(t.w) << 32 | t.z;
            u32 drop = static_cast<u32>(k + 8 - n) * 16;     // 16 .. 112 bits
            if (drop >= 64) { lo = hi; hi = 0; drop -= 64; }
            if (drop) { lo = lo >> drop | hi << (64 - drop); hi >>= drop; }
            v = u32x4{static_cast<u32>(lo), static_cast<u32>(lo >> 32), static_cast<u32>(hi), static_cast<u32>(hi >> 32)};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (k + i < n) v[i >> 1] |= static_cast<u32>(load2(p + k + i)) << (16 * (i & 1));
        }
    }
    return v;
}
// The same at any address without a branch that waits: what follows a row, up to the end of the matrix, is loaded and masked.  `left`: values
// from p[k] to that end.
__device__ inline u32x4 load8_masked(const u16* p, i64 k, i64 n, i64 left) {
    const i64 rest = n - k;
    const int there = rest >= 8 ? 8 : (rest <= 0 ? 0 : static_cast<int>(rest));
    u32x4 v = {0u, 0u, 0u, 0u};
    if (there > 0) {
        if (left >= 8) v = load16_any(p + k);
        else v = load8<false>(p, k, n);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= there >= 2 * i + 2 ? ~0u : (there == 2 * i + 1 ? 0xFFFFu : 0u);
    return v;
}
template <bool VEC>
__device__ inline u32x4 load8_inside(const u16* p) { return VEC ? load16(p) : load16_any(p); }           // all eight are there

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

// Tiles with the summed axis along their rows: [rows][64], 16-byte pieces of a row at piece ^ (row & 7), so that eight rows of a
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
    const u32 slot = kPieces % 16 == 0 ? ((k & 3u) | ((k >> 1) & 4u)) << 1 : (kPieces % 8 == 0 ? (k & 3u) << 1 : (kPieces == 4 ? k & 2u : 0u));
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

// Every wavefront's loads into LDS but the last N and all its LDS reads are done, then the workgroup meets.  (A barrier alone orders LDS
// accesses, but loads into LDS count as loads from memory, and waiting for all of them would wait for tiles that are wanted later.)
// Nothing is moved across it.
template <u32 N>
__device__ inline void meet_loads() {
    static_assert(N < 64, "the counter has six bits");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15u) | (N >> 4 << 14) | 0x0070);      // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Bytes a lane from `base` (the same in all lanes) + `offset` straight into LDS, at byte `lds` + BYTES * lane.  Written out because the
// compiler, which cannot tell the tiles of one array apart, would wait for every such load before any LDS read; here meet_loads says
// what has come.  There is no output register that could be reused while the load is under way, and
// nothing else in these kernels keeps a value in m0.
template <u32 BYTES>
__device__ inline void load_lds(u32 offset, const void* any_base, u32 any_lds) {
    const u64 a = reinterpret_cast<u64>(any_base);
    const u32 hi = static_cast<u32>(__builtin_amdgcn_readfirstlane(static_cast<int>(a >> 32))), lo = static_cast<u32>(__builtin_amdgcn_readfirstlane(static_cast<int>(a)));
    const u64 base = static_cast<u64>(hi) << 32 | lo;
    const u32 lds = __builtin_amdgcn_readfirstlane(any_lds);
    if (BYTES == 16) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds) : "memory");
    else             asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(offset), "s"(base), "s"(lds) : "memory");
}

// How the rows of an operand lie: 16-byte aligned and a multiple of eight values long; 4-byte aligned (and, where the sum runs across
// them, an even number of values long); at any address.
enum : int { kRowsAny = 0, kRows4 = 1, kRows16 = 2 };

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
    return __builtin_amdgcn_readfirstlane(x);          // known to be the same in all lanes: what it selects comes in scalar registers
}

__device__ inline u32 wave_most(u32 x) {               // largest of 64 lanes' values
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const u32 y = static_cast<u32>(__shfl_xor(static_cast<int>(x), d, 64));
        x = x > y ? x : y;
    }
    return x;
}

// Power of two, as its exponent, that brings the largest of some finite magnitudes (its bits) to 2^14 .. 2^15, the top of float16's range.
__device__ inline int scale_exponent(u32 most) {
    const int e = 14 - (static_cast<int>(most >> 23) - 127);
    return e > 120 ? 120 : e;
}
__device__ inline float power_of_two(int e) { return __uint_as_float(static_cast<u32>(127 + e) << 23); }

// N 16-bit values of one sign whose sum is x, but for (2 u)^(N - 1) u of it (u: half a step of the type at 1): x cut off, what was cut, cut off again,
// and so on, and the last one rounded.  An infinity that all of them meet in a product stays one of that sign, so the type's smallest value stands where
// nothing is left.
template <typename E, u32 N>
__device__ inline void in_terms(float x, u16 (&h)[N]) {
    const u32 u = __float_as_uint(x), size = u & 0x7FFFFFFFu;
    const bool finite = size < 0x7F800000u;
    float rest = x;
#pragma unroll
    for (u32 t = 0; t < N; ++t) {
        if (t + 1 < N && (t > 0 || finite)) {
            h[t] = E::cut(rest);
            rest -= E::dec(h[t]);
        } else {
            h[t] = E::enc(rest);
            if (!finite) rest = 0.0f;
        }
        if (t > 0 && finite && size != 0 && (h[t] & 0x7FFFu) == 0) h[t] = static_cast<u16>((u >> 16 & 0x8000u) | 1u);
    }
}

// ---- down: the product with the narrow matrix -------------------------------------------------------------------

// Rows at any address and of any length, copied to rows that are 16-byte aligned and end in zeros.
struct PackArgs {
    const u16* src; i64 ld;              // [rows, cols]
    u16* dst;                            // [all_rows, width]: zeros beside and below
    u32 rows, cols, all_rows, width, blocks;
};

struct DownArgs {
    const u16* x; i64 ldx;               // [n_tokens, n_sum]
    u32 n_tokens, n_sum;
    const int* ids;
    const AdapterDesc* ad;
    u32 n_adapters, max_rank;
    u16* zp; u32 rp;                     // [n_tokens, rp / 32][2][32]: z as sums of two 16-bit values, zeros past the rank; rp = max_rank rounded up to 32
    u16* z; i64 ldz;                     // the caller's copy, or NULL; all ldz columns are written
    float* z32;                          // [n_tokens, rp] before rounding, or NULL
    u32* row_max;                        // [n_tokens, rp / 32] largest finite magnitude (bits) in 32 values of a token's z, or NULL;
                                         // those of zp are scaled by scale_exponent of it (float16)
    u32 vec_x;                           // 16-byte aligned rows of x
    u32 tiles, shares;                   // of 32 tokens; workgroups that share the adapters of a tile
    u32 sorters;                         // workgroups that sort the tokens by adapter (backward)
    u32* order;                          // tokens of adapter 0, 1, ... in ascending order
    uint4* slots;                        // [n_slots] of a run of tokens: adapter or ~0, first place in `order`, tokens, tokens of the adapter
    uint2* seg;                          // [n_adapters] first slot, slots
    u32 n_slots, run;                    // tokens of a run
    u32 by_token;                        // forward: a workgroup has one token instead of a share of a tile
    PackArgs pack[3];                    // copies made beside z (k_adapter_down)
};

constexpr int kDownTokens = 32, kDownRanks = 32;
constexpr u32 down_lds(u32 waves) { return waves * 8192; }

// Places of the runs of an adapter whose tokens begin at `first`: run j of it is slot first / run + a + j.  (One slot at least for
// each adapter; the slots of different adapters never meet, since ceil(n / run) <= floor((first + n) / run) - floor(first / run) + 1.)
__device__ inline u32 first_slot(u32 first, u32 run, u32 a) { return first / run + a; }
// Place of the parts of run j of adapter a, whose first slot is s0.  Only adapters with several runs have parts.  Where there are more adapters
// than runs of tokens, places are 2 (first / run) + j: several runs are at most twice as many as whole ones, so places do not meet either
// and 2 (tokens / run) of them are enough.
__device__ inline u32 part_place(u32 a, u32 s0, u32 j, bool many) { return many ? 2 * (s0 - a) + j : s0 + j; }

// One wavefront an adapter: two passes over the ids, the first counts, the second writes; 1024 ids are under way at once.
__device__ inline void sort_tokens(const DownArgs& p, u32 a) {
    const u32 lane = threadIdx.x & 63;
    constexpr u32 kIds = 16;
    u32 less = 0, mine = 0;
    for (u32 t = 0; t < p.n_tokens; t += 64 * kIds) {
        int id[kIds];
#pragma unroll
        for (u32 i = 0; i < kIds; ++i) { const u32 at = t + i * 64 + lane; id[i] = p.ids[at < p.n_tokens ? at : p.n_tokens - 1]; }
#pragma unroll
        for (u32 i = 0; i < kIds; ++i) {
            const bool there = t + i * 64 + lane < p.n_tokens;
            less += static_cast<u32>(__popcll(__ballot(there && static_cast<u32>(id[i]) < a)));
            mine += static_cast<u32>(__popcll(__ballot(there && static_cast<u32>(id[i]) == a)));
        }
    }
    const u32 s0 = first_slot(less, p.run, a), s1 = a + 1 < p.n_adapters ? first_slot(less + mine, p.run, a + 1) : p.n_slots;
    const u32 runs = mine == 0 ? 1 : (mine + p.run - 1) / p.run;
    if (lane == 0) p.seg[a] = make_uint2(s0, runs);
    for (u32 s = s0 + lane; s < s1; s += 64) {
        const u32 done = (s - s0) * p.run;
        p.slots[s] = make_uint4(s - s0 < runs ? a : ~0u, less + done, mine - done < p.run ? mine - done : p.run, mine);
    }
    u32 at = less;
    if (mine == 0) return;                                   // uniform
    for (u32 t = 0; t < p.n_tokens; t += 64 * kIds) {
        int id[kIds];
#pragma unroll
        for (u32 i = 0; i < kIds; ++i) { const u32 from = t + i * 64 + lane; id[i] = p.ids[from < p.n_tokens ? from : p.n_tokens - 1]; }
#pragma unroll
        for (u32 i = 0; i < kIds; ++i) {
            const bool is = t + i * 64 + lane < p.n_tokens && static_cast<u32>(id[i]) == a;
            const u64 same = __ballot(is);
            if (is) p.order[at + static_cast<u32>(__popcll(same & ((1ull << lane) - 1ull)))] = t + i * 64 + lane;
            at += static_cast<u32>(__popcll(same));
        }
    }
}

// Sums of 32 tokens and 16 G ranks from r0 on, over the steps of 64 values that are this wavefront's.  Loads take whole cache lines, eight
// lanes to a line (a lane each from sixteen rows, as the operands want them, costs the address unit four times as long), and this
// wavefront's 8 KB of LDS turn them into fragments.  ALONG: the narrow matrix is [rank, n_sum]; else it is [n_sum, rank], and the
// transposing LDS load makes its fragments.
template <typename E, bool ALONG, bool VECX, bool VECM, u32 WAVES, u32 G>
__device__ inline void down_sums(const DownArgs& p, u32 t0, const u16* m, u32 rank, u32 r0, u16* own, f32x4 (&acc)[2][2]) {
    u32 lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                         // keeps the places of each form out of the registers of the others
    const u32 wave = threadIdx.x >> 6, piece = lane & 7u;
    constexpr u32 kPieces = 2 * G;                         // 16-byte pieces of the narrow matrix for each lane and step
    u16* own_m = own + kDownTokens * 64;
    const u16* xr[4];
    const u16* mr[kPieces];
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {                          // sums of tokens past the last are not stored
        const u32 t = t0 + i * 8 + (lane >> 3);
        xr[i] = p.x + static_cast<i64>(t < p.n_tokens ? t : p.n_tokens - 1) * p.ldx;
    }
#pragma unroll
    for (u32 i = 0; i < kPieces; ++i) {                    // nor are those of rows past the rank
        const u32 j = r0 + i * 8 + (lane >> 3);
        mr[i] = ALONG ? m + static_cast<i64>(j < rank ? j : rank - 1) * p.n_sum : m;
    }
    // negative by what is left of the matrix behind the last piece of a step, at step 0
    const i64 last_row = 63 * static_cast<i64>(rank) + r0 + 16 * G - static_cast<i64>(p.n_sum) * rank - 1;
    // GUARD: the step may end past the sum
    auto fetch = [&](auto guard, u32 s, u32x4 (&x)[4], u32x4 (&v)[kPieces]) {
        constexpr bool GUARD = decltype(guard)::value;
        const i64 k = static_cast<i64>(s) * 64 + piece * 8;
#pragma unroll
        for (u32 i = 0; i < 4; ++i) x[i] = GUARD ? load8<VECX>(xr[i], k, p.n_sum) : load8_inside<VECX>(xr[i] + k);
#pragma unroll
        for (u32 i = 0; i < kPieces; ++i) {
            if (ALONG) {
                v[i] = GUARD ? load8<VECM>(mr[i], k, p.n_sum) : load8_inside<VECM>(mr[i] + k);
            } else {
                const u32 at = i * 64 + lane, r = r0 + at % (2 * G) * 8;
                const i64 n = static_cast<i64>(s) * 64 + at / (2 * G);
                // Rows follow each other without a gap, and what a lane has past the rank goes into sums that are not stored: only the
                // end of the matrix needs care.
                if (!VECM && last_row + s * 64 * static_cast<i64>(rank) < 0) v[i] = load16_any(m + n * rank + r);
                else v[i] = load8<VECM>(m + n * rank, r, !GUARD || n < p.n_sum ? rank : 0);
            }
        }
    };
    auto add = [&](const u32x4 (&x)[4], const u32x4 (&v)[kPieces]) {
#pragma unroll
        for (u32 i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(own + along_at(i * 8 + (lane >> 3), piece)) = x[i];
#pragma unroll
        for (u32 i = 0; i < kPieces; ++i) {
            const u32 at = i * 64 + lane;
            *reinterpret_cast<u32x4*>(own_m + (ALONG ? along_at(i * 8 + (lane >> 3), piece) : across_at<16 * G>(at / (2 * G), at % (2 * G)))) = v[i];
        }
#pragma unroll
        for (u32 h = 0; h < 2; ++h) {
            const u32x4 fa = along_frag(own, 0, h), fb = along_frag(own, 16, h);
#pragma unroll
            for (u32 g = 0; g < G; ++g) {
                const u32x4 fm = ALONG ? along_frag(own_m, g * 16, h) : across_frag<16 * G>(own_m, g * 16, h);
                acc[0][g] = E::mfma(fa, fm, acc[0][g]);
                acc[1][g] = E::mfma(fb, fm, acc[1][g]);
            }
        }
    };
    // Steps whose loads are under way at once.  A step is fetched where the one before it in the same registers has been multiplied.
    constexpr u32 kAhead = (G == 1 ? 3 : 2) + (WAVES > 4 ? 1 : 0);         // of four wavefronts three workgroups share a unit's registers
    constexpr bool kGuard = VECX;                          // costs nothing where rows are whole pieces; others take the last step by itself
    const u32 steps = kGuard ? (p.n_sum + 63) / 64 : p.n_sum / 64;
    u32x4 x[kAhead][4], v[kAhead][kPieces];
#pragma unroll
    for (u32 i = 0; i < kAhead; ++i)
        if (wave + i * WAVES < steps) fetch(std::bool_constant<kGuard>{}, wave + i * WAVES, x[i], v[i]);
    for (u32 s = wave; s < steps; s += kAhead * WAVES) {
#pragma unroll
        for (u32 i = 0; i < kAhead; ++i) {
            const u32 now = s + i * WAVES, later = now + kAhead * WAVES;
            if (now < steps) add(x[i], v[i]);
            if (later < steps) fetch(std::bool_constant<kGuard>{}, later, x[i], v[i]);
        }
    }
    if (!kGuard && (p.n_sum & 63u) && steps % WAVES == wave) {
        fetch(std::true_type{}, steps, x[0], v[0]);
        add(x[0], v[0]);
    }
}

// z = s x M_a^T for 32 tokens, where M_a is the adapter's A [rank, n_sum] (ALONG), or its B [n_sum, rank] in the backward pass.  Reading x
// bounds it: wavefronts take every WAVES-th 64 values of its rows (nothing of x is shared between them) and add their sums up at the
// end; thirty-two tokens share what is read of M_a.  Four to sixteen workgroups have the same tile and take its tokens' adapters, 32 ranks at a
// time, in turn: a tile where one request ends and the next begins takes no longer than the others, and up to 128 ranks no longer than 32.
// The first workgroups sort the tokens.  8192 tokens of 4608 values, rank 16: 30 us, 2.5 TB/s.
template <typename E, bool ALONG, bool VECX, u32 WAVES>
__device__ inline void down_tile(const DownArgs& p, u32 block, char* lds) {
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (block < p.sorters) {                                 // uniform
        const u32 a = block * WAVES + wave;
        if (a < p.n_adapters) sort_tokens(p, a);
        return;
    }
    block -= p.sorters;
    const u32 share = block / p.tiles, t0 = block % p.tiles * kDownTokens;
    const int my_id = lane < kDownTokens ? adapter_of(p.ids, t0 + lane, p.n_tokens, p.n_adapters) : -1;
    const u32 width = p.z && p.ldz > p.rp ? static_cast<u32>(p.ldz) : p.rp;
    auto put = [&](u64 t, u32 j, float v, float up) {
        if (j < p.rp) {
            if (p.zp) {
                u16 h[2];
                in_terms<E, 2>(E::kNarrow ? v * up : v, h);
                u16* to = p.zp + (t * p.rp + j / kDownRanks * kDownRanks) * 2 + j % kDownRanks;
                to[0] = h[0];
                to[kDownRanks] = h[1];
            }
            if (p.z32) p.z32[t * p.rp + j] = v;
        }
        if (p.z && j < p.ldz) p.z[t * p.ldz + j] = E::enc(v);
    };
    if (share == 0)                                          // tokens without an adapter
        for (u32 i = wave; i < kDownTokens; i += WAVES) {
            if (t0 + i >= p.n_tokens || __shfl(my_id, static_cast<int>(i), 64) >= 0) continue;
            for (u32 j = lane; j < width; j += 64) put(t0 + i, j, 0.0f, 1.0f);
        }
    float (*sums)[kDownTokens][kDownRanks] = reinterpret_cast<float (*)[kDownTokens][kDownRanks]>(lds);
    u16* own = reinterpret_cast<u16*>(lds) + wave * 4096;
    u32 turn = 0;
    for (int a = next_adapter(my_id, -1); a != 0x7FFFFFFF; a = next_adapter(my_id, a)) {       // uniform over the workgroup
        const AdapterDesc d = p.ad[a];
        const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
        const u16* m = ALONG ? d.a : d.b;
        const bool vec_m = ALONG ? d.vec_a : d.vec_b;
        for (u32 r0 = 0; r0 < rank; r0 += kDownRanks, ++turn) {
            if (turn % p.shares != share) continue;
            const u32 groups = rank - r0 <= 16 ? 1 : 2;
            f32x4 acc[2][2] = {};
            if (vec_m) {
                if (groups == 1) down_sums<E, ALONG, VECX, true, WAVES, 1>(p, t0, m, rank, r0, own, acc);
                else             down_sums<E, ALONG, VECX, true, WAVES, 2>(p, t0, m, rank, r0, own, acc);
            } else {
                if (groups == 1) down_sums<E, ALONG, VECX, false, WAVES, 1>(p, t0, m, rank, r0, own, acc);
                else             down_sums<E, ALONG, VECX, false, WAVES, 2>(p, t0, m, rank, r0, own, acc);
            }
            __syncthreads();                                 // sums take the place of the others' tiles
#pragma unroll
            for (u32 h = 0; h < 2; ++h)
#pragma unroll
                for (u32 g = 0; g < 2; ++g) {
                    if (g >= groups) continue;
#pragma unroll
                    for (u32 i = 0; i < 4; ++i) sums[wave][h * 16 + (lane >> 4) * 4 + i][g * 16 + (lane & 15)] = acc[h][g][i];
                }
            __syncthreads();
            const u32 end = r0 + kDownRanks >= rank ? width : r0 + kDownRanks;
            const u32 lane32 = lane & 31u;
            for (u32 i = wave * 2 + (lane >> 5); i < kDownTokens; i += WAVES * 2) {          // a token for each half of a wavefront
                if (__shfl(my_id, static_cast<int>(i), 64) != a) continue;
                const u64 t = t0 + i;
                const u32 j = r0 + lane32;
                float v = 0.0f, up = 1.0f;
                if (j < rank) {
#pragma unroll
                    for (u32 w = 0; w < WAVES; ++w) v += sums[w][i][lane32];
                    v *= d.scale;
                }
                if (p.row_max) {
                    const u32 u = __float_as_uint(v) & 0x7FFFFFFFu;
                    u32 most = u < 0x7F800000u ? u : 0u;
#pragma unroll
                    for (int k = 16; k >= 1; k >>= 1) {
                        const u32 y = static_cast<u32>(__shfl_xor(static_cast<int>(most), k, 64));
                        most = most > y ? most : y;
                    }
                    if (lane32 == 0) p.row_max[t * (p.rp / kDownRanks) + r0 / kDownRanks] = most;
                    up = power_of_two(scale_exponent(most));
                }
                put(t, j, v, up);
                for (u32 k = r0 + kDownRanks + lane32; k < end; k += 32) put(t, k, 0.0f, 1.0f);
            }
            __syncthreads();                                 // before tiles take the place of the sums
        }
    }
}

// z of one token, for batches where tokens that follow each other have adapters of their own: a wavefront takes every WAVES-th four rows of A,
// whose values meet x in order, 512 a load, and adds up its lanes.
template <typename E, bool VECX, u32 WAVES>
__device__ inline void down_token(const DownArgs& p, u32 t) {
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int a = __builtin_amdgcn_readfirstlane(adapter_of(p.ids, t, p.n_tokens, p.n_adapters));
    AdapterDesc d{};
    if (a >= 0) d = p.ad[a];
    const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
    const u32 width = p.z && p.ldz > p.rp ? static_cast<u32>(p.ldz) : p.rp;
    for (u32 j = rank + threadIdx.x; j < width; j += 64 * WAVES) {
        if (j < p.rp) p.z32[static_cast<u64>(t) * p.rp + j] = 0.0f;
        if (p.z && j < p.ldz) p.z[static_cast<u64>(t) * p.ldz + j] = 0;
    }
    const u16* x = p.x + static_cast<i64>(t) * p.ldx;
    for (u32 r0 = wave * 4; r0 < rank; r0 += 4 * WAVES) {
        float sum[4] = {};
        const u16* m[4];
#pragma unroll
        for (u32 r = 0; r < 4; ++r) m[r] = d.a + static_cast<i64>(r0 + r < rank ? r0 + r : rank - 1) * p.n_sum;
#pragma unroll 3
        for (u32 k0 = 0; k0 < p.n_sum; k0 += 512) {
            const i64 k = k0 + lane * 8;
            u32x4 vm[4];
            const u32x4 vx = load8<VECX>(x, k, p.n_sum);
#pragma unroll
            for (u32 r = 0; r < 4; ++r) vm[r] = d.vec_a ? load8<true>(m[r], k, p.n_sum) : load8<false>(m[r], k, p.n_sum);
#pragma unroll
            for (u32 i = 0; i < 8; ++i) {
                const float fx = E::dec(static_cast<u16>(vx[i >> 1] >> (16 * (i & 1))));
#pragma unroll
                for (u32 r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(fx, E::dec(static_cast<u16>(vm[r][i >> 1] >> (16 * (i & 1)))), sum[r]);
            }
        }
#pragma unroll
        for (u32 r = 0; r < 4; ++r) {
#pragma unroll
            for (int w = 32; w >= 1; w >>= 1) sum[r] += __shfl_xor(sum[r], w, 64);
            if (lane == r && r0 + r < rank) {
                const float v = sum[r] * d.scale;
                p.z32[static_cast<u64>(t) * p.rp + r0 + r] = v;
                if (p.z) p.z[static_cast<u64>(t) * p.ldz + r0 + r] = E::enc(v);
            }
        }
    }
}

constexpr u32 kDownWaves = 8;
constexpr u32 kPackRows = 4 * kDownWaves;                    // of a workgroup, four to a wavefront
__device__ inline void pack_rows(const PackArgs& p, u32 block) {
    const u32 lane = threadIdx.x & 63, r0 = block * kPackRows + (threadIdx.x >> 6) * 4;
    for (u32 k = lane * 8; k < p.width; k += 512) {
        u32x4 v[4];
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            const u32 r = r0 + i < p.rows ? r0 + i : p.rows - 1;
            v[i] = load8_masked(p.src + static_cast<i64>(r) * p.ld, k, r0 + i < p.rows ? p.cols : 0, static_cast<i64>(p.rows - 1 - r) * p.ld + p.cols - k);
        }
#pragma unroll
        for (u32 i = 0; i < 4; ++i)
            if (r0 + i < p.all_rows) *reinterpret_cast<u32x4*>(p.dst + static_cast<u64>(r0 + i) * p.width + k) = v[i];
    }
}

// z, and beside it aligned copies of what the wide product and the gradients read: loads of the wide product go straight into LDS, 16 bytes a
// lane, only from aligned rows.
template <typename E, bool ALONG, bool VECX>
__global__ __launch_bounds__(64 * kDownWaves) void k_adapter_down(DownArgs p) {
    __shared__ __align__(16) char lds[down_lds(kDownWaves)];
    const u32 down = ALONG && p.by_token ? p.n_tokens : p.sorters + p.tiles * p.shares;
    u32 block = blockIdx.x;
    if (block >= down) {                                     // uniform
        block -= down;
#pragma unroll
        for (u32 i = 0; i < 3; ++i) {
            if (block < p.pack[i].blocks) { pack_rows(p.pack[i], block); return; }
            block -= p.pack[i].blocks;
        }
        return;
    }
    if (ALONG && p.by_token) down_token<E, VECX, kDownWaves>(p, block);
    else down_tile<E, ALONG, VECX, kDownWaves>(p, block, lds);
}

// ---- the wide product with the adapters' share added ------------------------------------------------------------

struct WideArgs {
    const u16* x; i64 ldx;               // [n_tokens, n_sum]
    const u16* w; i64 ldw;               // ALONG: [n_out, n_sum], else [n_sum, n_out]
    u16* y; i64 ldy;                     // [n_tokens, n_out]
    u32 n_tokens, n_out, n_sum;
    u32 x_cols, w_cols;                  // values of a row of x and of W, with the zeros at the end of a copy
    const u16* zp; u32 rp;               // of DownArgs
    const u32* row_max;                  // of DownArgs (float16)
    const int* ids;
    const AdapterDesc* ad;
    u32 n_adapters, max_rank;
    u32 splits, steps_each;              // steps of 64 values that a split sums
    float* part;                         // [splits][n_tokens][n_out], or NULL: y is written
};

// Workgroups go round the eight dies one by one; this gives each die a run of neighbouring tiles, whose rows its cache keeps.
__device__ inline u32 die_order(u32 i, u32 n) {
    const u32 die = i & 7u, k = i >> 3, each = n >> 3, more = n & 7u;
    return die * each + (die < more ? die : more) + k;
}

// Tiles of BM tokens by BN outputs, summed 64 values a step (whole cache lines of x), NB steps in LDS.  Loads go straight into LDS, up to
// NB steps ahead of their use.  A fragment register is read again as soon as its last product has begun, half a step ahead, so that the
// matrix instructions wait for neither LDS nor memory; wavefronts meet once a step, in its middle, where the next step has come and the
// last read of this one is done.  Rows that are 4-byte aligned are loaded four bytes a lane; with others steps go through registers.
// With `part` a workgroup sums a part of the steps and stores it in binary32; the adapters' share is then added with the parts.
// Matrix instructions bound large products (8192 tokens, 4608 -> 4096: 263 us, 1.18 PFLOP/s; the units' matrix pipes are busy 63 % of the time, and
// 57 % backward, where the transposing LDS reads meet in banks in 21 % of LDS's cycles), reading W those of few tokens, latency those between
// (1333 tokens, 650 -> 2600: 27.4 us).
constexpr u32 wide_lds(u32 bm, u32 bn, u32 nb) { return nb * (bm + bn) * 128 + bm * 12; }
template <typename E, int BM, int BN, int WM, int WN, u32 NB, bool ALONG, int ROWS>
__device__ inline void wide_tile(const WideArgs& p, u32 block_id, u32 n_blocks, char* lds) {
    constexpr u32 kThreads = 64 * WM * WN;
    constexpr u32 TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr u32 kXPieces = BM * 8 / kThreads, kWPieces = BN * 8 / kThreads;          // 16-byte pieces of a step for each thread
    constexpr u32 kBytes = ROWS == kRows16 ? 16 : 4, kXLoads = kXPieces * 16 / kBytes, kWLoads = kWPieces * 16 / kBytes, kLoads = kXLoads + kWLoads;
    constexpr u32 kTile = (BM + BN) * 64, kEarly = FN < FM ? FN : FN / 2, kEach = FN / kEarly;
    u16* tiles = reinterpret_cast<u16*>(lds);
    int* s_ids = reinterpret_cast<int*>(lds + NB * kTile * 2);
    float* s_down = reinterpret_cast<float*>(s_ids + BM);          // what undoes the scale of a token's z, for two groups of 32 ranks (float16)
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const u32 wm = wave / WN, wn = wave % WN;
    const u32 tiles_m = (p.n_tokens + BM - 1) / BM, tiles_n = (p.n_out + BN - 1) / BN;
    const u32 block = die_order(block_id, n_blocks);
    const u32 tile = block / p.splits, split = block % p.splits;
    // four rows of tiles at a time: tiles that run together share rows of x and of W
    const u32 band = tile / (4 * tiles_n), in_band = tile % (4 * tiles_n), high = tiles_m - band * 4 < 4 ? tiles_m - band * 4 : 4;
    const u32 t0 = (band * 4 + in_band % high) * BM, n0 = in_band / high * BN;
    const u32 all_steps = (p.n_sum + 63) / 64;
    const u32 begin = split * p.steps_each, end = begin + p.steps_each < all_steps ? begin + p.steps_each : all_steps;
    const u32 steps = end > begin ? end - begin : 0;
    f32x4 acc[FN][FM] = {};
    u32x4 fx[FM], fw[FN];

    auto frag_x = [&](const u16* sx, u32 j, u32 sub) { return along_frag(sx, wm * TM + j * 16, sub); };
    auto frag_w = [&](const u16* sx, u32 i, u32 sub) {
        return ALONG ? along_frag(sx + BM * 64, wn * TN + i * 16, sub) : across_frag<BN>(sx + BM * 64, wn * TN + i * 16, sub);
    };

    for (u32 i = tid; i < BM; i += kThreads) s_ids[i] = adapter_of(p.ids, t0 + i, p.n_tokens, p.n_adapters);
    bool rest = false;                                             // a last step that ends past the sum is left
    if (ROWS != kRowsAny) {
        u32 xo[kXLoads], wo[kWLoads];                              // byte offsets of what this lane loads
        constexpr u32 kOf = 16 / kBytes;                           // loads of a piece
#pragma unroll
        for (u32 i = 0; i < kXLoads; ++i) {
            const u32 at = i * kThreads + tid, row = at / (8 * kOf), piece = (at / kOf & 7u) ^ (row & 7u);
            const u32 r = t0 + row < p.n_tokens ? row : p.n_tokens - 1 - t0;
            xo[i] = (r * static_cast<u32>(p.ldx) + piece * 8) * 2 + at % kOf * kBytes;
        }
#pragma unroll
        for (u32 i = 0; i < kWLoads; ++i) {
            const u32 at = i * kThreads + tid;
            if (ALONG) {
                const u32 row = at / (8 * kOf), piece = (at / kOf & 7u) ^ (row & 7u);
                const u32 r = n0 + row < p.n_out ? row : p.n_out - 1 - n0;
                wo[i] = (r * static_cast<u32>(p.ldw) + piece * 8) * 2 + at % kOf * kBytes;
            } else {
                constexpr u32 kRow = BN / 8;
                const u32 k = at / (kRow * kOf);
                u32 col = across_at<BN>(k, at / kOf % kRow) - k * BN + at % kOf * (kBytes / 2);
                if (n0 + col >= p.w_cols) col = p.w_cols - kBytes / 2 - n0;
                wo[i] = (k * static_cast<u32>(p.ldw) + col) * 2;
            }
        }
        const u32 full = begin + steps == all_steps && (p.n_sum & 63u) ? steps - 1 : steps;
        rest = full < steps;
        const char* xs = reinterpret_cast<const char*>(p.x + static_cast<i64>(t0) * p.ldx + begin * 64);
        const char* ws = reinterpret_cast<const char*>(ALONG ? p.w + static_cast<i64>(n0) * p.ldw + begin * 64 : p.w + static_cast<i64>(begin) * 64 * p.ldw + n0);
        const i64 w_step = (ALONG ? 64 : 64 * p.ldw) * 2;
        const u32 lds0 = static_cast<u32>(reinterpret_cast<uintptr_t>((lds_void*)tiles)) + wave * 64 * kBytes;
        u32 loaded = 0, to = 0;
        auto load = [&]() {                                        // the next step, or the last one again
#pragma unroll
            for (u32 i = 0; i < kXLoads; ++i) load_lds<kBytes>(xo[i], xs, lds0 + to + i * kThreads * kBytes);
#pragma unroll
            for (u32 i = 0; i < kWLoads; ++i) load_lds<kBytes>(wo[i], ws, lds0 + to + BM * 128 + i * kThreads * kBytes);
            ++loaded;
            const bool more = loaded < full;
            xs += more ? 128 : 0;
            ws += more ? w_step : 0;
            to = to + kTile * 2 == NB * kTile * 2 ? 0 : to + kTile * 2;
        };
        // products of the fragments in registers, which are replaced by those of half `sub` of the tile at `sx`
        auto half = [&](const u16* sx, u32 sub) {
            u32x4 next[FN];
#pragma unroll
            for (u32 j = 0; j < FM; ++j) {
#pragma unroll
                for (u32 i = 0; i < FN; ++i) acc[i][j] = E::mfma(fw[i], fx[j], acc[i][j]);
                fx[j] = frag_x(sx, j, sub);
                if (j < kEarly) {                                  // what the next half's first product waits for comes first
#pragma unroll
                    for (u32 i = j * kEach; i < (j + 1) * kEach; ++i) next[i] = frag_w(sx, i, sub);
                    __builtin_amdgcn_sched_group_barrier(0x008, FN, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1 + kEach * (ALONG ? 1 : 2), 0);
                } else {
                    __builtin_amdgcn_sched_group_barrier(0x008, FN, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
#pragma unroll
            for (u32 i = 0; i < FN; ++i) fw[i] = next[i];
        };
        if (full > 0) {
#pragma unroll
            for (u32 i = 0; i < NB; ++i) load();
            meet_loads<(NB - 1) * kLoads>();
#pragma unroll
            for (u32 i = 0; i < FN; ++i) fw[i] = frag_w(tiles, i, 0);
#pragma unroll
            for (u32 j = 0; j < FM; ++j) fx[j] = frag_x(tiles, j, 0);
            u32 from = 0;
            for (u32 s = 0; s < full; ++s) {
                half(tiles + from, 1);
                meet_loads<(NB - 2) * kLoads>();
                load();                                            // where this step was
                from = from + kTile == NB * kTile ? 0 : from + kTile;
                half(tiles + from, 0);
            }
            meet_loads<0>();
        }
    } else {
        constexpr u32 kAhead = 2;                                  // steps whose rows are under way
        u32x4 rx[kAhead][kXPieces], rw[kAhead][kWPieces];
        const i64 sum_end = static_cast<i64>(end) * 64 < p.n_sum ? static_cast<i64>(end) * 64 : p.n_sum;       // zeros from there on
        auto fetch = [&](u32 set, u32 s) {
            const i64 k0 = static_cast<i64>(s) * 64;
#pragma unroll
            for (u32 i = 0; i < kXPieces; ++i) {
                const u32 at = i * kThreads + tid, t = t0 + (at >> 3) < p.n_tokens ? t0 + (at >> 3) : p.n_tokens - 1;
                rx[set][i] = load8_masked(p.x + static_cast<i64>(t) * p.ldx, k0 + (at & 7u) * 8, sum_end, static_cast<i64>(p.n_tokens - 1 - t) * p.ldx + p.n_sum - (k0 + (at & 7u) * 8));
            }
#pragma unroll
            for (u32 i = 0; i < kWPieces; ++i) {
                const u32 at = i * kThreads + tid;
                if (ALONG) {
                    const u32 n = n0 + (at >> 3) < p.n_out ? n0 + (at >> 3) : p.n_out - 1;
                    rw[set][i] = load8_masked(p.w + static_cast<i64>(n) * p.ldw, k0 + (at & 7u) * 8, sum_end, static_cast<i64>(p.n_out - 1 - n) * p.ldw + p.n_sum - (k0 + (at & 7u) * 8));
                } else {
                    constexpr u32 kRow = BN / 8;
                    const i64 k = k0 + at / kRow;
                    rw[set][i] = load8_masked(p.w + k * p.ldw, n0 + (at % kRow) * 8, k < sum_end ? p.n_out : 0, (p.n_sum - 1 - k) * p.ldw + p.n_out - (n0 + (at % kRow) * 8));
                }
            }
        };
        if (steps > 0) {
#pragma unroll
            for (u32 q = 0; q < kAhead; ++q) fetch(q, begin + q);
        }
        u32 to = 0;
        for (u32 s = begin; s < end; s += kAhead) {
#pragma unroll
            for (u32 q = 0; q < kAhead; ++q) {                     // past the end: zeros
                u16* sx = tiles + to;
#pragma unroll
                for (u32 i = 0; i < kXPieces; ++i) {
                    const u32 at = i * kThreads + tid;
                    *reinterpret_cast<u32x4*>(sx + along_at(at >> 3, at & 7u)) = rx[q][i];
                }
#pragma unroll
                for (u32 i = 0; i < kWPieces; ++i) {
                    const u32 at = i * kThreads + tid;
                    const u32 w_at = ALONG ? along_at(at >> 3, at & 7u) : across_at<BN>(at / (BN / 8), at % (BN / 8));
                    *reinterpret_cast<u32x4*>(sx + BM * 64 + w_at) = rw[q][i];
                }
                __syncthreads();
                fetch(q, s + q + kAhead);
#pragma unroll
                for (u32 sub = 0; sub < 2; ++sub) {
#pragma unroll
                    for (u32 i = 0; i < FN; ++i) fw[i] = frag_w(sx, i, sub);
#pragma unroll
                    for (u32 j = 0; j < FM; ++j) fx[j] = frag_x(sx, j, sub);
#pragma unroll
                    for (u32 j = 0; j < FM; ++j)
#pragma unroll
                        for (u32 i = 0; i < FN; ++i) acc[i][j] = E::mfma(fw[i], fx[j], acc[i][j]);
                }
                to = to == 0 ? kTile : 0;                          // the one that all have read since the barrier before this one
            }
        }
    }
    __syncthreads();

    // What is left of the sum, then the adapters' share: 64 ranks at a time for each adapter that the tile's tokens have, in two groups of 32
    // with a tile in LDS each.  z comes as sums of two 16-bit values, 32 of the first beside 32 of the second, so its product keeps 16 bits of it or
    // more and y is rounded once; both meet the same fragments of the adapter's matrix.  A product is added where the token is the adapter's and
    // nowhere else: zeros in its place would spread infinities and NaN of one request's adapter to its neighbours.
    int a = -1;
    u32 r0 = 0, rank = 0;
    const u16* m = nullptr;
    bool vec_m = false;
    for (;;) {                                                     // uniform
        u32 me = tid;
        asm volatile("" : "+v"(me));                              // keeps the places below out of registers while the sum runs, and between passes
        if (!rest) {
            if (p.part) break;                                     // added with the parts
            r0 += 64;
            if (r0 >= rank) {
                int next = 0x7FFFFFFF;
                for (u32 i = me & 63u; i < BM; i += 64) {
                    const int id = s_ids[i];
                    if (id > a && id < next) next = id;
                }
                a = next_adapter(next, -1);                        // the same in every wavefront
                if (a == 0x7FFFFFFF) break;
                const AdapterDesc d = p.ad[a];
                rank = d.rank < p.max_rank ? d.rank : p.max_rank;
                m = ALONG ? d.b : d.a;
                vec_m = ALONG ? d.vec_b : d.vec_a;
                r0 = 0;
            }
        }
        const u32 groups = !rest && rank - r0 > kDownRanks ? 2 : 1;
        static_assert(BM * 2 <= kThreads, "a thread for each scale");
        float down = 1.0f;
        if (E::kNarrow && !rest && me < BM * groups) {
            const u64 t = t0 + me % BM < p.n_tokens ? t0 + me % BM : p.n_tokens - 1;
            down = power_of_two(-scale_exponent(p.row_max[t * (p.rp / kDownRanks) + r0 / kDownRanks + me / BM]));
        }
        const i64 k0 = rest ? static_cast<i64>(all_steps - 1) * 64 : r0;
        const i64 k_end = rest ? p.n_sum : rank;
        const u16* x = rest ? p.x : p.zp;
        const i64 ldx = rest ? p.ldx : static_cast<i64>(p.rp) * 2, x_end = rest ? p.x_cols : ldx, x0 = rest ? k0 : k0 * 2;
        const u16* w = rest ? p.w : m;
        const i64 ldw = rest ? p.ldw : (ALONG ? static_cast<i64>(rank) : static_cast<i64>(p.n_out));
        const i64 cols = rest ? p.w_cols : (ALONG ? rank : p.n_out), rows = ALONG ? p.n_out : k_end;
        const bool vec_w = rest ? ROWS == kRows16 : vec_m;
        auto load_x = [&](u32 at, u32 group) {
            const u32 row = at >> 3, t = t0 + row < p.n_tokens ? t0 + row : p.n_tokens - 1;
            const u16* src = x + static_cast<i64>(t) * ldx;
            const i64 k = x0 + group * 64 + (at & 7u) * 8;
            return ROWS == kRows16 || !rest ? load8<true>(src, k, x_end) : load8<false>(src, k, x_end);
        };
        auto store_x = [&](u32 at, u32 group, u32x4 v) { *reinterpret_cast<u32x4*>(tiles + group * kTile + along_at(at >> 3, at & 7u)) = v; };
        auto load_w = [&](u32 at) {
            const u32 row = ALONG ? at >> 3 : at / (BN / 8), piece = ALONG ? at & 7u : at % (BN / 8);
            const i64 want = ALONG ? n0 + row : k0 + row, r = want < rows ? want : rows - 1, from = ALONG ? k0 + piece * 8 : n0 + piece * 8;
            const i64 end_at = ALONG || want < rows ? cols : 0;
            return vec_w ? load8<true>(w + r * ldw, from, end_at) : load8_masked(w + r * ldw, from, end_at, (rows - 1 - r) * ldw + cols - from);
        };
        auto store_w = [&](u32 at, u32x4 v) {
            const u32 row = ALONG ? at >> 3 : at / (BN / 8), piece = ALONG ? at & 7u : at % (BN / 8);
            const u32 group = rest ? 0 : (ALONG ? piece / 4 : row / kDownRanks);
            const u32 to = ALONG ? along_at(row, piece - group * 4) : across_at<BN>(row - group * kDownRanks, piece);
            *reinterpret_cast<u32x4*>(tiles + group * kTile + BM * 64 + to) = v;
        };
        // All loads before the stores; tiles of 256 rows, which have no registers for that, one by one.
        constexpr bool kAtOnce = BM * BN <= 128 * 128;
        if (kAtOnce) {
            u32x4 vx[2][kXPieces], vw[kWPieces];
#pragma unroll
            for (u32 i = 0; i < kWPieces; ++i) vw[i] = load_w(me + i * kThreads);
#pragma unroll
            for (u32 i = 0; i < kXPieces; ++i) vx[0][i] = load_x(me + i * kThreads, 0);
            if (groups == 2) {
#pragma unroll
                for (u32 i = 0; i < kXPieces; ++i) vx[1][i] = load_x(me + i * kThreads, 1);
            }
#pragma unroll
            for (u32 i = 0; i < kWPieces; ++i) store_w(me + i * kThreads, vw[i]);
#pragma unroll
            for (u32 i = 0; i < kXPieces; ++i) store_x(me + i * kThreads, 0, vx[0][i]);
            if (groups == 2) {
#pragma unroll
                for (u32 i = 0; i < kXPieces; ++i) store_x(me + i * kThreads, 1, vx[1][i]);
            }
        } else {
            for (u32 group = 0; group < groups; ++group)
#pragma unroll 1
                for (u32 at = me; at < BM * 8; at += kThreads) store_x(at, group, load_x(at, group));
#pragma unroll 1
            for (u32 at = me; at < BN * 8; at += kThreads) {
                if (!rest && groups == 1 && (ALONG ? (at & 7u) >= 4 : at / (BN / 8) >= kDownRanks)) continue;      // not read
                store_w(at, load_w(at));
            }
        }
        if (E::kNarrow && me < BM * groups) s_down[me] = down;
        __syncthreads();
#pragma unroll 1
        for (u32 group = 0; group < groups; ++group) {
            const u16* sx = tiles + group * kTile;
            u32x4 second[FN];
#pragma unroll
            for (u32 i = 0; i < FN; ++i) {
                fw[i] = frag_w(sx, i, 0);
                second[i] = rest ? frag_w(sx, i, 1) : fw[i];
            }
#pragma unroll
            for (u32 j = 0; j < FM; ++j) {
                const u32 row = wm * TM + j * 16 + (me & 15u);
                const int id = s_ids[row];
                u32 mine = static_cast<u32>(rest) | static_cast<u32>(id == a) ? ~0u : 0u;
                if (kAtOnce && __ballot(mine != 0) == 0) continue;             // sixteen rows without a token of the adapter
                asm volatile("" : "+v"(mine));                    // a mask and no branch: with branches the tiles of 256 rows spilled 90 registers
                const u32x4 x_first = frag_x(sx, j, 0), x_second = frag_x(sx, j, 1);
                const float undo = E::kNarrow ? __uint_as_float(__float_as_uint(s_down[group * BM + row]) & mine) : 1.0f;
#pragma unroll
                for (u32 i = 0; i < FN; ++i) {
                    f32x4 v = E::mfma(second[i], x_second, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
                    v = E::mfma(fw[i], x_first, v);
#pragma unroll
                    for (u32 k = 0; k < 4; ++k) {
                        const float f = __uint_as_float(__float_as_uint(v[k]) & mine);
                        acc[i][j][k] = E::kNarrow ? __builtin_fmaf(f, undo, acc[i][j][k]) : acc[i][j][k] + f;
                    }
                }
                if (!kAtOnce) __builtin_amdgcn_sched_barrier(0);               // sixteen rows at a time: there are no registers for more
            }
        }
        __syncthreads();
        rest = false;
    }

    if (p.part) {                                                  // uniform
        float* part = p.part + static_cast<u64>(split) * p.n_tokens * p.n_out;
#pragma unroll
        for (u32 j = 0; j < FM; ++j) {
            const u32 t = t0 + wm * TM + j * 16 + (lane & 15);
            if (t >= p.n_tokens) continue;
            float* out = part + static_cast<u64>(t) * p.n_out;
#pragma unroll
            for (u32 i = 0; i < FN; ++i) {
                const u32 n = n0 + wn * TN + i * 16 + (lane >> 4) * 4;
                if (n + 4 <= p.n_out) *reinterpret_cast<f32x4_any*>(out + n) = acc[i][j];
                else
#pragma unroll
                    for (u32 k = 0; k < 4; ++k) if (n + k < p.n_out) out[n + k] = acc[i][j][k];
            }
        }
        return;
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
            if (n + 4 <= p.n_out) {                                // at any address: one by one they took ten times as long
                u32x2 v;
                v.x = static_cast<u32>(h[0]) | static_cast<u32>(h[1]) << 16;
                v.y = static_cast<u32>(h[2]) | static_cast<u32>(h[3]) << 16;
                *reinterpret_cast<u32x2_any*>(out + n) = v;
            } else {
#pragma unroll
                for (u32 k = 0; k < 4; ++k) if (n + k < p.n_out) out[n + k] = h[k];
            }
        }
    }
}

template <typename E, int BM, int BN, int WM, int WN, u32 NB, bool ALONG, int ROWS>
__global__ __launch_bounds__(64 * WM * WN, NB * (BM + BN) * 128 > 80 * 1024 && WM * WN <= 4 ? 1 : 2) void k_adapter_wide(WideArgs p) {
    __shared__ __align__(16) char lds[wide_lds(BM, BN, NB)];
    wide_tile<E, BM, BN, WM, WN, NB, ALONG, ROWS>(p, blockIdx.x, gridDim.x, lds);
}

// Where tiles of 64 outputs are few, the sum is split and z is made in the same launch: nothing in it waits for anything.  z comes first, its
// chain of loads is the longest.  64 tokens of 64 adapters, 4608 -> 4096: 17.4 us, 3.4 TB/s, and 5.8 us for the join.
template <typename E, bool ALONG, int ROWS, int BM>
__global__ __launch_bounds__(256, 3) void k_adapter_split(DownArgs d, WideArgs w, u32 down_blocks) {
    constexpr u32 NB = ROWS != kRowsAny ? 3 : 2;
    constexpr bool VECX = ROWS == kRows16;
    __shared__ __align__(16) char lds[wide_lds(BM, 64, NB) > down_lds(4) ? wide_lds(BM, 64, NB) : down_lds(4)];
    if (blockIdx.x >= down_blocks) wide_tile<E, BM, 64, BM / 32, 128 / BM, NB, ALONG, ROWS>(w, blockIdx.x - down_blocks, gridDim.x - down_blocks, lds);
    else if (ALONG && d.by_token) down_token<E, VECX, 4>(d, blockIdx.x);
    else down_tile<E, ALONG, VECX, 4>(d, blockIdx.x, lds);
}

// out = the parts added in order + z M_a (M_a: B^T or A), one output a thread; z in binary32.
template <typename E, bool ALONG>
__device__ inline void join_parts(const WideArgs& g, const float* z32, u32 ldz32, u32 t, u32 n) {
    const int a = __builtin_amdgcn_readfirstlane(adapter_of(g.ids, t, g.n_tokens, g.n_adapters));
    if (n >= g.n_out) return;
    const float* part = g.part + static_cast<u64>(t) * g.n_out + n;
    const u64 each = static_cast<u64>(g.n_tokens) * g.n_out;
    float v = 0.0f;
#pragma unroll 4
    for (u32 s = 0; s < g.splits; ++s) v += part[s * each];
    if (a >= 0) {
        const AdapterDesc d = g.ad[a];
        const u32 rank = d.rank < g.max_rank ? d.rank : g.max_rank;
        const float* z = z32 + static_cast<u64>(t) * ldz32;
        float u = 0.0f;
        if (ALONG) {
            const u16* b = d.b + static_cast<i64>(n) * rank;
            for (u32 j = 0; j < rank; j += 8) {
                const u32x4 h = d.vec_b ? load8<true>(b, j, rank) : load8<false>(b, j, rank);
#pragma unroll
                for (u32 i = 0; i < 8; ++i) if (j + i < rank) u = __builtin_fmaf(z[j + i], E::dec(static_cast<u16>(h[i >> 1] >> (16 * (i & 1)))), u);
            }
        } else {
            const u16* m = d.a + n;
#pragma unroll 8
            for (u32 j = 0; j < rank; ++j) u = __builtin_fmaf(z[j], E::dec(load2(m + static_cast<i64>(j) * g.n_out)), u);
        }
        v += u;
    }
    g.y[static_cast<i64>(t) * g.ldy + n] = E::enc(v);
}

template <typename E, bool ALONG>
__global__ __launch_bounds__(256) void k_adapter_split_join(WideArgs w, const float* z32, u32 ldz32) {
    join_parts<E, ALONG>(w, z32, ldz32, blockIdx.y, blockIdx.x * 256 + threadIdx.x);
}

// ---- a few tokens, in one launch -----------------------------------------------------------------------------------

constexpr u32 kFewTokens = 2, kFewWaves = 8, kFewRows = 4 * kFewWaves;

// One or two tokens beside a small A: every workgroup makes all of z for itself (A comes out of the caches), which saves the launch that would
// join the parts, and a wavefront takes four rows of W, whose values meet x in order.  z B^T is added as more of the same sum.  Latency bounds it: a
// launch, the first rows of W (under way before z is made), and one reduction over the lanes.  1 token 512 -> 2048 of rank 8: 7.5 us a call, 10.3 us
// with parts and a join; 2 tokens 2048 -> 512 of rank 32: 11.5 and 12.6 us; 3 and 4 tokens, whose adapters come one after the other: 13.9 and 12.0 us.
template <typename E, bool VEC>
__global__ __launch_bounds__(64 * kFewWaves) void k_adapter_few(WideArgs p, u16* z, i64 ldz) {
    __shared__ float sz[kFewTokens][CONDENSA_MAX_RANK];
    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32 n0 = blockIdx.x * kFewRows + wave * 4;
    const u16 *w[4], *x[kFewTokens];
#pragma unroll
    for (u32 r = 0; r < 4; ++r) w[r] = p.w + static_cast<i64>(n0 + r < p.n_out ? n0 + r : p.n_out - 1) * p.ldw;
#pragma unroll
    for (u32 t = 0; t < kFewTokens; ++t) x[t] = p.x + static_cast<i64>(t < p.n_tokens ? t : p.n_tokens - 1) * p.ldx;
    u32x4 vw[4];
#pragma unroll
    for (u32 r = 0; r < 4; ++r) vw[r] = load8<VEC>(w[r], lane * 8, p.n_sum);
    u32 turn = 0;
    for (u32 t = 0; t < p.n_tokens; ++t) {
        const int a = __builtin_amdgcn_readfirstlane(adapter_of(p.ids, t, p.n_tokens, p.n_adapters));
        if (a < 0) continue;                                   // uniform
        const AdapterDesc d = p.ad[a];
        const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
        for (u32 r0 = 0; r0 < rank; r0 += 4, ++turn) {
            if (turn % kFewWaves != wave) continue;
            float sum[4] = {};
            const u16* xt = p.x + static_cast<i64>(t) * p.ldx;
#pragma unroll 2
            for (u32 k0 = 0; k0 < p.n_sum; k0 += 512) {
                const i64 k = k0 + lane * 8;
                const u32x4 vx = load8<VEC>(xt, k, p.n_sum);
                u32x4 vm[4];
#pragma unroll
                for (u32 r = 0; r < 4; ++r) {
                    const u16* row = d.a + static_cast<i64>(r0 + r < rank ? r0 + r : rank - 1) * p.n_sum;
                    vm[r] = d.vec_a ? load8<true>(row, k, p.n_sum) : load8<false>(row, k, p.n_sum);
                }
#pragma unroll
                for (u32 i = 0; i < 8; ++i) {
                    const float fx = E::dec(static_cast<u16>(vx[i >> 1] >> (16 * (i & 1))));
#pragma unroll
                    for (u32 r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(fx, E::dec(static_cast<u16>(vm[r][i >> 1] >> (16 * (i & 1)))), sum[r]);
                }
            }
#pragma unroll
            for (u32 r = 0; r < 4; ++r) {
#pragma unroll
                for (int b = 32; b >= 1; b >>= 1) sum[r] += __shfl_xor(sum[r], b, 64);
                if (lane == r && r0 + r < rank) sz[t][r0 + r] = sum[r] * d.scale;
            }
        }
    }
    __syncthreads();
    float sum[4][kFewTokens] = {};
    for (u32 k0 = 0; k0 < p.n_sum; k0 += 512) {
        const i64 k = k0 + lane * 8;
        u32x4 vx[kFewTokens];
#pragma unroll
        for (u32 t = 0; t < kFewTokens; ++t) if (t < p.n_tokens) vx[t] = load8<VEC>(x[t], k, p.n_sum);
        if (k0 > 0) {
#pragma unroll
            for (u32 r = 0; r < 4; ++r) vw[r] = load8<VEC>(w[r], k, p.n_sum);
        }
#pragma unroll
        for (u32 t = 0; t < kFewTokens; ++t) {
            if (t >= p.n_tokens) continue;                     // uniform
#pragma unroll
            for (u32 i = 0; i < 8; ++i) {
                const float fx = E::dec(static_cast<u16>(vx[t][i >> 1] >> (16 * (i & 1))));
#pragma unroll
                for (u32 r = 0; r < 4; ++r) sum[r][t] = __builtin_fmaf(fx, E::dec(static_cast<u16>(vw[r][i >> 1] >> (16 * (i & 1)))), sum[r][t]);
            }
        }
    }
    float out = 0.0f;                                          // lane 4 t + r: row n0 + r of token t
#pragma unroll
    for (u32 t = 0; t < kFewTokens; ++t) {
        if (t >= p.n_tokens) continue;                         // uniform, as the next
        const int a = __builtin_amdgcn_readfirstlane(adapter_of(p.ids, t, p.n_tokens, p.n_adapters));
        u32 rank = 0;
        if (a >= 0) {
            const AdapterDesc d = p.ad[a];
            rank = d.rank < p.max_rank ? d.rank : p.max_rank;
            for (u32 j = lane; j < rank; j += 64) {
                const float fz = sz[t][j];
#pragma unroll
                for (u32 r = 0; r < 4; ++r) {
                    const u32 n = n0 + r < p.n_out ? n0 + r : p.n_out - 1;
                    sum[r][t] = __builtin_fmaf(fz, E::dec(load2(d.b + static_cast<i64>(n) * rank + j)), sum[r][t]);
                }
            }
        }
#pragma unroll
        for (u32 r = 0; r < 4; ++r) {
            float v = sum[r][t];
#pragma unroll
            for (int b = 32; b >= 1; b >>= 1) v += __shfl_xor(v, b, 64);
            if (lane == t * 4 + r) out = v;
        }
        if (z && blockIdx.x == 0)
            for (u32 j = threadIdx.x; j < ldz; j += 64 * kFewWaves) z[t * ldz + j] = j < rank ? E::enc(sz[t][j]) : static_cast<u16>(0);
    }
    const u32 t = lane >> 2, n = n0 + (lane & 3u);
    if (t < p.n_tokens && n < p.n_out) p.y[static_cast<i64>(t) * p.ldy + n] = E::enc(out);
}

// ---- gradients of the adapters ----------------------------------------------------------------------------------

struct GradArgs {
    const u16* x; i64 ldx; u32 n_in;     // grad_a = sum of dz^T x
    const u16* dy; i64 ldy; u32 n_out;   // grad_b = sum of dy^T z
    u32 x_cols, dy_cols;                 // values of a row, with the zeros at the end of a copy
    const float* dz; u32 rp;
    const u16* z; i64 ldz;
    const u32* row_max;
    const u32* order;
    const uint4* slots;
    const uint2* seg;
    const AdapterDesc* ad;
    u32 max_rank, run, tiles_in, tiles, rank_groups;
    u32 slot0;                           // of this launch
    u32 many;                            // how part_place numbers them
    float* part;                         // [places][max_rank (n_in + n_out)]
};

constexpr u32 kGradCols = 128, kGradWaves = 8, kGradPass = 32 * kGradWaves;

// One run of one adapter's tokens times 128 columns of x or of dy and 16 G ranks.  Reading x and dy once more bounds it; the columns are split and
// not the ranks, so that one workgroup only reads them (up to 32 ranks; with 64 in a workgroup registers were spilled).  Every wavefront has 32 tokens of each 256 to itself, what one matrix
// instruction sums, and meets the others only to add the sums up: with barriers for each step, wavefronts waited for memory together, and
// 212 tokens took 4 steps one after the other.  Rows of x and dy pass through 8 KB of LDS for the transposing load, dz and z come as
// fragments, a lane's eight tokens one by one; the next pass is on its way meanwhile.  dz enters as a sum of 16-bit values,
// three of bfloat16 or two of float16, since a binary32 gradient would keep no more than 8 or 11 bits of one; for float16 a wavefront scales its dz by a
// power of two first, so that the largest sits near the top of the type's range.
// 8192 tokens, 4608 -> 4096, 8 adapters of rank 16: 35 us, 4.0 TB/s.  Workgroups after the gradients' add the parts of dx.
template <typename E, bool VEC, int G>
__global__ __launch_bounds__(64 * kGradWaves, G == 1 ? 4 : 2) void k_adapter_grads(GradArgs p, WideArgs dx, u32 joins) {
    constexpr u32 kTerms = E::kNarrow ? 2 : 3;
    __shared__ __align__(16) u16 tiles[kGradWaves][32 * kGradCols];
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const u32 grads = gridDim.x - (joins + 1) / 2;
    if (blockIdx.x >= grads) {                                 // uniform
        const u32 cols = (dx.n_out + 255) / 256, block = (blockIdx.x - grads) * 2 + wave / 4;
        if (block < joins) join_parts<E, false>(dx, p.dz, p.rp, block / cols, block % cols * 256 + (tid & 255u));
        return;
    }
    const u32 col_tile = blockIdx.x % p.tiles, r0 = blockIdx.x / p.tiles % p.rank_groups * (16 * G), slot = p.slot0 + blockIdx.x / p.tiles / p.rank_groups;
    const uint4 of = p.slots[slot];
    const u32 a = __builtin_amdgcn_readfirstlane(of.x), first = __builtin_amdgcn_readfirstlane(of.y), count = __builtin_amdgcn_readfirstlane(of.z);
    const bool whole = of.w <= p.run;
    if (a == ~0u) return;                                      // uniform, as all that follow
    const AdapterDesc d = p.ad[a];
    const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
    if (r0 >= rank) return;
    const bool of_a = col_tile < p.tiles_in;
    const u32 c0 = (of_a ? col_tile : col_tile - p.tiles_in) * kGradCols;
    const u32 n_cols = of_a ? p.n_in : p.n_out, v_cols = of_a ? p.x_cols : p.dy_cols;
    const u16* v_src = of_a ? p.x : p.dy;
    const i64 ldv = of_a ? p.ldx : p.ldy;
    u16* own = tiles[wave];
    float up = 1.0f, down = 1.0f;
    f32x4 acc[8][G] = {};
    u32x4 rv[8];
    u32 ru[G][8];
    // the tokens of the pass that begins at `s` (lane l: l % 32), the last one again past the end
    auto tokens = [&](u32 s) { const u32 k = s + (lane & 31u); return p.order[first + (k < count ? k : count - 1)]; };
    // Columns past the last and ranks past the last are others again: their sums are not stored.
    const u32 col0 = c0 + (lane & 15u) * 8, col = VEC && col0 >= v_cols ? v_cols - 8 : col0;
    auto fetch = [&](u32 tok) {
#pragma unroll
        for (u32 i = 0; i < 8; ++i) {
            const u32 k = i * 4 + (lane >> 4);
            const i64 t = static_cast<u32>(__shfl(static_cast<int>(tok), static_cast<int>(k), 64));
            rv[i] = VEC ? load16(v_src + t * ldv + col) : load8<false>(v_src + t * ldv, col, v_cols);
        }
#pragma unroll
        for (u32 q = 0; q < 8; ++q) {
            const u32 k = (lane >> 4) * 8 + q;
            const u64 t = static_cast<u32>(__shfl(static_cast<int>(tok), static_cast<int>(k), 64));
#pragma unroll
            for (u32 g = 0; g < G; ++g) {
                const u32 j = r0 + g * 16 + (lane & 15u), there = j < rank ? j : rank - 1;
                ru[g][q] = of_a ? __float_as_uint(p.dz[t * p.rp + there]) : load2(p.z + t * p.ldz + there);
            }
        }
    };
    u32 s = wave * 32;
    if (s < count) {                                           // uniform in a wavefront
        const u32 tok = tokens(s);
        u32 next = tokens(s + kGradPass);
        fetch(tok);
        if (E::kNarrow && of_a) {
            u32 most = 0;
            const u32 groups = (rank + kDownRanks - 1) / kDownRanks;
            for (u32 k0 = s; k0 < count; k0 += 2 * kGradPass) {
                const u32 k = k0 + (lane >> 5) * kGradPass + (lane & 31u);
                if (k >= count) continue;
                const u64 t = p.order[first + k];
                for (u32 g = 0; g < groups; ++g) {
                    const u32 m = p.row_max[t * (p.rp / kDownRanks) + g];
                    most = most > m ? most : m;
                }
            }
            most = wave_most(most);
            const int e = scale_exponent(most);
            up = power_of_two(e);
            down = power_of_two(-e);
        }
        for (; s < count; s += kGradPass) {
            u32x4 fu[G][kTerms] = {};
            if (s + 32 > count) {                              // tokens past the last: zeros on both sides
#pragma unroll
                for (u32 i = 0; i < 8; ++i)
                    if (s + i * 4 + (lane >> 4) >= count) rv[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (u32 g = 0; g < G; ++g)
#pragma unroll
                    for (u32 q = 0; q < 8; ++q)
                        if (s + (lane >> 4) * 8 + q >= count) ru[g][q] = 0;
            }
#pragma unroll
            for (u32 i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(own + across_at<kGradCols>(i * 4 + (lane >> 4), lane & 15u)) = rv[i];
#pragma unroll
            for (u32 g = 0; g < G; ++g)
#pragma unroll
                for (u32 q = 0; q < 8; ++q) {
                    if (of_a) {
                        u16 h[kTerms];
                        in_terms<E, kTerms>(__uint_as_float(ru[g][q]) * up, h);
#pragma unroll
                        for (u32 t = 0; t < kTerms; ++t) fu[g][t][q >> 1] |= static_cast<u32>(h[t]) << (16 * (q & 1u));
                    } else {
                        fu[g][0][q >> 1] |= ru[g][q] << (16 * (q & 1u));
                    }
                }
            if (s + kGradPass < count) {
                fetch(next);
                next = tokens(s + 2 * kGradPass);
            }
#pragma unroll
            for (u32 c = 0; c < 8; ++c) {
                const u32x4 fv = across_frag<kGradCols>(own, c * 16, 0);
#pragma unroll
                for (u32 g = 0; g < G; ++g) {
                    if (r0 + g * 16 >= rank) continue;
                    if (of_a) {
#pragma unroll
                        for (u32 t = kTerms; t-- > 1;) acc[c][g] = E::mfma(fv, fu[g][t], acc[c][g]);
                    }
                    acc[c][g] = E::mfma(fv, fu[g][0], acc[c][g]);
                }
            }
        }
    }
    float* out = of_a ? d.grad_a : d.grad_b;
    if (!whole) {
        const u32 s0 = p.seg[a].x;
        out = p.part + static_cast<u64>(part_place(a, s0, slot - s0, p.many)) * p.max_rank * (static_cast<u64>(p.n_in) + p.n_out) + (of_a ? 0 : static_cast<u64>(rank) * p.n_in);
    }
    const u32 used = count < kGradPass ? (count + 31) / 32 : kGradWaves;       // wavefronts that had tokens
    f32x4* sums = reinterpret_cast<f32x4*>(&tiles[0][0]);
#pragma unroll
    for (u32 g = 0; g < G; ++g) {
        if (r0 + g * 16 >= rank) continue;                     // uniform over the workgroup
        __syncthreads();                                       // sums take the place of tiles and of the sums before
        if (wave < used) {
#pragma unroll
            for (u32 c = 0; c < 8; ++c) sums[wave * 512 + c * 64 + lane] = acc[c][g] * down;
        }
        __syncthreads();
        f32x4 v = {};
        for (u32 w = 0; w < used; ++w) v += sums[w * 512 + tid];
        const u32 r = r0 + g * 16 + (lane & 15u), c = c0 + wave * 16 + (lane >> 4) * 4;
        if (r >= rank) continue;
#pragma unroll
        for (u32 q = 0; q < 4; ++q)
            if (c + q < n_cols) out[of_a ? static_cast<u64>(r) * p.n_in + c + q : static_cast<u64>(c + q) * rank + r] = v[q];
    }
}

// Adapters with several runs: their parts, added in order.
__global__ __launch_bounds__(256) void k_adapter_join(GradArgs p, u32 blocks_each) {
    const u32 a = blockIdx.x / blocks_each;
    const uint2 seg = p.seg[a];
    if (seg.y <= 1) return;                                    // uniform
    const AdapterDesc d = p.ad[a];
    const u32 rank = d.rank < p.max_rank ? d.rank : p.max_rank;
    const u64 na = static_cast<u64>(rank) * p.n_in, n = na + static_cast<u64>(rank) * p.n_out;
    const u64 each = static_cast<u64>(p.max_rank) * (static_cast<u64>(p.n_in) + p.n_out);
    const u32 first = part_place(a, seg.x, 0, p.many), runs = seg.y;
    for (u64 i = static_cast<u64>(blockIdx.x % blocks_each) * 256 + threadIdx.x; i < n; i += static_cast<u64>(blocks_each) * 256) {
        float v = p.part[first * each + i];
#pragma unroll 4
        for (u32 r = 1; r < runs; ++r) v += p.part[(first + r) * each + i];
        if (i < na) d.grad_a[i] = v;
        else d.grad_b[i - na] = v;
    }
}

}  // namespace condensa
