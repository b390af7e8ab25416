// AdamW over many tensors in one launch, states in 32 or in 8 bits, with the L-C penalty folded in.
#pragma once
#include "common.h"

namespace condensa {

constexpr int kStateBlock = CONDENSA_STATE_BLOCK;       // elements that share the scale of an 8-bit state: four to a lane of a wavefront
constexpr int kAdamwChunk = 8192;                       // elements of one tensor that an entry of the chunk map stands for
constexpr int kAdamwPoke = 40;                          // tensors that one launch writes into the device list

// One tensor as the kernel sees it.
struct AdamwDesc {
    float* w;
    const void* grad;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    const float* theta;        // NULL: no penalty on this tensor
    const float* lam;
    u16* codes;                // NULL: no 16-bit copy
    u64 n;
    u64 first_block;           // blocks of 256 elements in the tensors before this one
    u32 first_chunk;
    u32 vec;                   // all pointers aligned for four elements
};
static_assert(sizeof(AdamwDesc) == 96, "AdamwDesc layout");

struct AdamwArgs {
    const AdamwDesc* td;
    const u32* chunk_map;
    const float* grad_scale;   // device, or NULL
    float beta1, rest1, beta2, rest2;          // rest = 1 - beta, rounded from binary64
    float decay, step_size, correct, eps;      // 1 - lr wd, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    float mu;
    u32 seed_lo, seed_hi;
    u32 code_type;             // CONDENSA_TYPE_F16 / _BF16
};

struct AdamwPoke {
    AdamwDesc d[kAdamwPoke];
};

// The device list is made once for many steps: descriptors travel as kernel arguments, a graph that captures the call keeps them.
__global__ __launch_bounds__(256) void k_adamw_list(AdamwDesc* __restrict__ dst, u32* __restrict__ chunk_map, AdamwPoke src, u32 first, u32 count) {
    const u32 words = count * (sizeof(AdamwDesc) / 8);
    if (blockIdx.x == 0)
        for (u32 i = threadIdx.x; i < words; i += 256) reinterpret_cast<u64*>(dst + first)[i] = reinterpret_cast<const u64*>(src.d)[i];
    for (u32 t = 0; t < count; ++t) {
        const u64 chunks = (src.d[t].n + kAdamwChunk - 1) / kAdamwChunk;
        for (u64 c = blockIdx.x * 256ull + threadIdx.x; c < chunks; c += gridDim.x * 256ull) chunk_map[src.d[t].first_chunk + c] = first + t;
    }
}

// 32 bits from an element's position (256 times its block among all blocks of the list, plus its place in the block): the integer
// hash "lowbias32" (C. Wellons, hash-prospector), with one half of the seed mixed in before it and the other between its products.
__device__ inline u32 position_noise(u64 p, u32 seed_lo, u32 seed_hi) {
    u32 h = static_cast<u32>(p) ^ (static_cast<u32>(p >> 32) * 0x9E3779B9u) ^ seed_lo;
    h ^= h >> 16;
    h *= 0x7FEB352Du;
    h ^= h >> 15;
    h += seed_hi;
    h *= 0x846CA68Bu;
    return h ^ (h >> 16);
}

// Largest value of a wavefront's 64 lanes (patterns of non-negative floats order like integers).
__device__ inline u32 wave_max_u32(u32 x) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const u32 y = static_cast<u32>(__shfl_xor(static_cast<int>(x), d, 64));
        x = x > y ? x : y;
    }
    return x;
}

__device__ inline u32 finite_magnitude(float x) {
    const u32 a = __float_as_uint(x) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}

__device__ inline void unpack_e4m3(u32 c, float s, float v[4]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c), true);
    v[0] = __fmul_rn(lo.x, s); v[1] = __fmul_rn(lo.y, s); v[2] = __fmul_rn(hi.x, s); v[3] = __fmul_rn(hi.y, s);
}

// Four values of a block as e4m3 codes of x / scale, scale = (largest finite magnitude of the block) / 448.  Values outside the
// finite range saturate, NaN keeps a NaN code.  Rounding to nearest would hold the second moment still: one step changes it by
// at most (1 - beta2) of itself, a fraction of a percent, and neighbouring codes are 6 to 12 % apart.  So SR draws the neighbour
// with the probability that keeps the mean: 16 random bits are added below the kept fraction.  FLOOR keeps positive values
// positive, since the denominator of the update is made of them.
template <bool SR, bool FLOOR>
__device__ inline u32 pack_e4m3(const float x[4], const u32 noise[4], float* scale) {
    u32 top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) { const u32 a = finite_magnitude(x[k]); top = top > a ? top : a; }
    top = wave_max_u32(top);
    const float t = __uint_as_float(top);
    const bool kept = t >= 0x1p-100f;                    // below, the reciprocal would leave the range
    const float inv = kept ? __fmul_rn(448.0f, __fdiv_rn(1.0f, t)) : 0.0f;
    *scale = kept ? __fmul_rn(t, 1.0f / 448.0f) : 0.0f;
    u32 out = 0;
    if (!SR) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float q = __fmul_rn(x[k], inv);
            y[k] = __builtin_fabsf(x[k]) > t ? __builtin_copysignf(kept ? 448.0f : 0.0f, x[k]) : (__builtin_fabsf(q) > 448.0f ? __builtin_copysignf(448.0f, q) : q);
        }
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        out = static_cast<u32>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true));
        if (FLOOR) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const u32 c = (out >> (8 * k)) & 0xFFu;
                out |= (c == 0u && x[k] > 0.0f && kept) ? 1u << (8 * k) : 0u;
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const u32 u = __float_as_uint(x[k]), a = u & 0x7FFFFFFFu;
            const float y = __fmul_rn(__uint_as_float(a), inv);
            const u32 b = __float_as_uint(y);
            u32 code;
            if (y >= 0x1p-6f) code = ((b + (noise[k] << 4)) >> 20) - (120u << 3);
            else code = (static_cast<u32>(__fmul_rn(y, 0x1p29f)) + (noise[k] << 4)) >> 20;     // y 2^9 steps, 20 bits below the point
            if (code > 0x7Eu || (a == 0x7F800000u && kept)) code = 0x7Eu;
            if (a == 0x7F800000u && !kept) code = 0u;
            if (FLOOR) code = (code == 0u && x[k] > 0.0f && kept) ? 1u : code;
            if (a > 0x7F800000u) code = 0x7Fu;
            out |= (code | ((u >> 24) & 0x80u)) << (8 * k);
        }
    }
    return out;
}

template <int GRAD>
__device__ inline void load_grad4(const void* p, u64 e0, float g[4]) {            // aligned, all inside
    if (GRAD == CONDENSA_TYPE_F32) {
        const float4 t = ld4_stream(static_cast<const float*>(p) + e0);
        g[0] = t.x; g[1] = t.y; g[2] = t.z; g[3] = t.w;
    } else {
        const u32x2 t = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const u16*>(p) + e0));
        const u16 h[4] = {static_cast<u16>(t.x), static_cast<u16>(t.x >> 16), static_cast<u16>(t.y), static_cast<u16>(t.y >> 16)};
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = GRAD == CONDENSA_TYPE_F16 ? f16_bits_to_f32(h[k]) : bf16_bits_to_f32(h[k]);
    }
}
template <int GRAD>
__device__ inline float load_grad1(const void* p, u64 e) {
    if (GRAD == CONDENSA_TYPE_F32) return static_cast<const float*>(p)[e];
    const u16 h = static_cast<const u16*>(p)[e];
    return GRAD == CONDENSA_TYPE_F16 ? f16_bits_to_f32(h) : bf16_bits_to_f32(h);
}

// Per element, binary32, one rounding per operation:
//      g = grad [* grad_scale] [+ mu (w - theta) - lambda];  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g g;
//      w = w decay - step_size (m / (sqrt(v) correct + eps)).
// Every value is read once and written once and nothing is shared, so the bytes bound it.  A wavefront takes one block of 256
// elements, four to a lane: 128-bit accesses of what is held in 32 bits are contiguous across it, and the largest magnitude of a
// block of 8-bit states is found across its lanes alone.  604 M weights, states in 32 bits with penalty and 16-bit copy: 3.75 ms, 6.1 TB/s;
// 44 M weights with 8-bit states rounded by random bits: 158 us, 4.5 TB/s, held up by the hash and the rounding beside the memory.
template <int GRAD, bool STATE8, bool SR>
__global__ __launch_bounds__(64) void k_adamw(AdamwArgs a) {
    constexpr u32 kSub = kAdamwChunk / kStateBlock;
    const u32 c = blockIdx.x / kSub;
    const AdamwDesc& d = a.td[a.chunk_map[c]];
    const u64 block = static_cast<u64>(c - d.first_chunk) * kSub + blockIdx.x % kSub;        // of this tensor
    const u64 e0 = block * kStateBlock + threadIdx.x * 4;
    const u64 n = d.n;
    if (block * kStateBlock >= n) return;                                // uniform
    const bool full = d.vec && block * kStateBlock + kStateBlock <= n;   // uniform
    const int count = full ? 4 : (e0 + 4 <= n ? 4 : (e0 < n ? static_cast<int>(n - e0) : 0));
    const bool penalty = d.theta != nullptr;
    float w[4] = {}, g[4] = {}, m[4] = {}, v[4] = {}, th[4] = {}, l[4] = {};
    u32 mc = 0, vc = 0;
    if (full) {
        const float4 x = ld4_stream(d.w + e0);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        load_grad4<GRAD>(d.grad, e0, g);
        if (STATE8) {
            mc = __builtin_nontemporal_load(reinterpret_cast<const u32*>(static_cast<const u8*>(d.m) + e0));
            vc = __builtin_nontemporal_load(reinterpret_cast<const u32*>(static_cast<const u8*>(d.v) + e0));
        } else {
            const float4 y = ld4_stream(static_cast<const float*>(d.m) + e0), z = ld4_stream(static_cast<const float*>(d.v) + e0);
            m[0] = y.x; m[1] = y.y; m[2] = y.z; m[3] = y.w;
            v[0] = z.x; v[1] = z.y; v[2] = z.z; v[3] = z.w;
        }
        if (penalty) {
            const float4 y = ld4_stream(d.theta + e0), z = ld4_stream(d.lam + e0);
            th[0] = y.x; th[1] = y.y; th[2] = y.z; th[3] = y.w;
            l[0] = z.x; l[1] = z.y; l[2] = z.z; l[3] = z.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= count) continue;
            w[k] = d.w[e0 + k];
            g[k] = load_grad1<GRAD>(d.grad, e0 + k);
            if (STATE8) {
                mc |= static_cast<u32>(static_cast<const u8*>(d.m)[e0 + k]) << (8 * k);
                vc |= static_cast<u32>(static_cast<const u8*>(d.v)[e0 + k]) << (8 * k);
            } else {
                m[k] = static_cast<const float*>(d.m)[e0 + k];
                v[k] = static_cast<const float*>(d.v)[e0 + k];
            }
            if (penalty) { th[k] = d.theta[e0 + k]; l[k] = d.lam[e0 + k]; }
        }
    }
    if (STATE8) {
        unpack_e4m3(mc, d.m_scale[block], m);
        unpack_e4m3(vc, d.v_scale[block], v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __fmul_rn(v[k], v[k]);
    }
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    float r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        g[k] = __fmul_rn(g[k], gs);
        if (penalty) g[k] = __fsub_rn(__fadd_rn(g[k], __fmul_rn(a.mu, __fsub_rn(w[k], th[k]))), l[k]);
        m[k] = __fadd_rn(__fmul_rn(a.beta1, m[k]), __fmul_rn(a.rest1, g[k]));
        v[k] = __fadd_rn(__fmul_rn(a.beta2, v[k]), __fmul_rn(a.rest2, __fmul_rn(g[k], g[k])));
        r[k] = __builtin_sqrtf(v[k]);          // rounded once; __fsqrt_rn is the approximate instruction here
        const float u = __fdiv_rn(m[k], __fadd_rn(__fmul_rn(r[k], a.correct), a.eps));
        w[k] = __fsub_rn(__fmul_rn(w[k], a.decay), __fmul_rn(a.step_size, u));
    }
    if (STATE8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k >= count) { m[k] = 0.0f; r[k] = 0.0f; }
        u32 nm[4] = {}, nr[4] = {};
        if (SR) {
            const u64 p = (d.first_block + block) * kStateBlock + threadIdx.x * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const u32 h = position_noise(p + k, a.seed_lo, a.seed_hi);
                nm[k] = h & 0xFFFFu;
                nr[k] = h >> 16;
            }
        }
        float ms, vs;
        mc = pack_e4m3<SR, false>(m, nm, &ms);
        vc = pack_e4m3<SR, true>(r, nr, &vs);
        if (threadIdx.x == 0) { d.m_scale[block] = ms; d.v_scale[block] = vs; }
    }
    u16 h[4];
    if (d.codes) {
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = a.code_type == CONDENSA_TYPE_F16 ? f32_to_f16_rne(w[k]) : f32_to_bf16_rne(w[k]);
    }
    if (full) {
        st4_stream(d.w + e0, w[0], w[1], w[2], w[3]);
        if (STATE8) {
            __builtin_nontemporal_store(mc, reinterpret_cast<u32*>(static_cast<u8*>(d.m) + e0));
            __builtin_nontemporal_store(vc, reinterpret_cast<u32*>(static_cast<u8*>(d.v) + e0));
        } else {
            st4_stream(static_cast<float*>(d.m) + e0, m[0], m[1], m[2], m[3]);
            st4_stream(static_cast<float*>(d.v) + e0, v[0], v[1], v[2], v[3]);
        }
        if (d.codes) st_code4_stream(d.codes + e0, h[0], h[1], h[2], h[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= count) continue;
            d.w[e0 + k] = w[k];
            if (STATE8) {
                static_cast<u8*>(d.m)[e0 + k] = static_cast<u8>(mc >> (8 * k));
                static_cast<u8*>(d.v)[e0 + k] = static_cast<u8>(vc >> (8 * k));
            } else {
                static_cast<float*>(d.m)[e0 + k] = m[k];
                static_cast<float*>(d.v)[e0 + k] = v[k];
            }
            if (d.codes) d.codes[e0 + k] = h[k];
        }
    }
}

}  // namespace condensa
