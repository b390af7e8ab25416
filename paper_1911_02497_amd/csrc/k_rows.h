// Access to rows of 16-bit values at any address, loads straight into LDS, and the order of tiles: what the kernels of products and rows share.
#pragma once
#include "common.h"

typedef int64_t i64;

namespace condensa {

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

typedef __attribute__((address_space(3))) void lds_void;

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

__device__ inline u32 wave_most(u32 x) {               // largest of 64 lanes' values
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const u32 y = static_cast<u32>(__shfl_xor(static_cast<int>(x), d, 64));
        x = x > y ? x : y;
    }
    return x;
}

// Workgroups go round the eight dies one by one; this gives each die a run of neighbouring tiles, whose rows its cache keeps.
__device__ inline u32 die_order(u32 i, u32 n) {
    const u32 die = i & 7u, k = i >> 3, each = n >> 3, more = n & 7u;
    return die * each + (die < more ? die : more) + k;
}

}  // namespace condensa
