// E4M3 codes with a scale for each block of 128: the codec of whole matrices, and the root-mean-square norm that answers in such codes, with its gradients.
//
// Lane l of a wavefront holds eight consecutive columns, 8 l .. 8 l + 7 of 512: sixteen lanes hold a block of 128 of a row.
#pragma once
#include "k_rows.h"

namespace condensa {

constexpr u32 kFp8Block = CONDENSA_FP8_BLOCK;
constexpr u32 kLaneCols = 8, kWaveCols = 64 * kLaneCols;

// ---- rows of eight values a lane ----------------------------------------------------------------------------------

typedef u32 u32x2_bytes __attribute__((ext_vector_type(2), aligned(1)));

struct RowsF16 {
    typedef u16 elem;
    template <bool VEC>
    static __device__ inline void load(const elem* p, i64 k, i64 n, float (&v)[8]) { unpack(load8<VEC>(p, k, n), v); }
    static __device__ inline void unpack(u32x4 t, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = CodecF16::dec(static_cast<u16>(t[i >> 1] >> (16 * (i & 1))));
    }
    static __device__ inline u16 enc(float x) { return CodecF16::enc(x); }
};
struct RowsBF16 {
    typedef u16 elem;
    template <bool VEC>
    static __device__ inline void load(const elem* p, i64 k, i64 n, float (&v)[8]) { unpack(load8<VEC>(p, k, n), v); }
    static __device__ inline void unpack(u32x4 t, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(t[i] << 16);
            v[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u);
        }
    }
    static __device__ inline u16 enc(float x) { return CodecBF16::enc(x); }
};
struct RowsF32 {
    typedef float elem;
    template <bool VEC>
    static __device__ inline void load(const elem* p, i64 k, i64 n, float (&v)[8]) {
        if (k + 8 <= n) {
            if (VEC) {
                const f32x4 a = *reinterpret_cast<const f32x4*>(p + k), b = *reinterpret_cast<const f32x4*>(p + k + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
            } else {
                const f32x4 a = *reinterpret_cast<const f32x4_any*>(p + k), b = *reinterpret_cast<const f32x4_any*>(p + k + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < n ? p[k + i] : 0.0f;
        }
    }
};

// Eight values of a row in its 16-bit type, from column k of n.
template <bool VEC>
__device__ inline void store8(u16* p, i64 k, i64 n, u32x4 t) {
    if (VEC) {
        if (k < n) *reinterpret_cast<u32x4*>(p + k) = t;
    } else if (k + 8 <= n) {
        *reinterpret_cast<u32x4_any*>(p + k) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i) if (k + i < n) p[k + i] = static_cast<u16>(t[i >> 1] >> (16 * (i & 1)));
    }
}
template <typename R>
__device__ inline u32x4 pack8(const float (&v)[8]) {
    u32x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = static_cast<u32>(R::enc(v[2 * i])) | static_cast<u32>(R::enc(v[2 * i + 1])) << 16;
    return t;
}
// Eight codes, at any address.
__device__ inline void store8_codes(u8* p, i64 k, i64 n, u32x2 t) {
    if (k + 8 <= n) {
        *reinterpret_cast<u32x2_bytes*>(p + k) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i) if (k + i < n) p[k + i] = static_cast<u8>(t[i >> 2] >> (8 * (i & 3)));
    }
}
__device__ inline u32x2 load8_codes(const u8* p, i64 k, i64 n) {
    u32x2 t = {0u, 0u};
    if (k + 8 <= n) {
        t = *reinterpret_cast<const u32x2_bytes*>(p + k);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i) if (k + i < n) t[i >> 2] |= static_cast<u32>(p[k + i]) << (8 * (i & 3));
    }
    return t;
}

// ---- codes of a block -----------------------------------------------------------------------------------------------

// Largest finite magnitude of eight values, as its bits.
__device__ inline u32 largest8(const float (&v)[8]) {
    u32 top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 a = __float_as_uint(v[i]) & 0x7FFFFFFFu, b = a < 0x7F800000u ? a : 0u;
        top = top > b ? top : b;
    }
    return top;
}
__device__ inline u32 largest_of16(u32 x) {                // of sixteen lanes' values
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) {
        const u32 y = static_cast<u32>(__shfl_xor(static_cast<int>(x), d, 64));
        x = x > y ? x : y;
    }
    return x;
}

// What makes codes of a block from the bits of its largest finite magnitude.
struct BlockBy {
    float top, by, scale;
    bool kept;
};
__device__ inline BlockBy block_by(u32 top_bits) {
    BlockBy b;
    b.top = __uint_as_float(top_bits);
    b.kept = b.top >= 0x1p-100f;                            // below, the reciprocal would leave the range
    b.by = b.kept ? __fdiv_rn(448.0f, b.top) : 0.0f;
    b.scale = b.kept ? __fdiv_rn(b.top, 448.0f) : 0.0f;
    return b;
}

// Four codes of x 448 / top, of the exact quotient.  The product with a rounded reciprocal is up to 1.5 units off, which decides wrongly where the quotient is the middle of
// two codes, as it often is for short significands, or within those units of one.  Its remainder, which two fused operations give, brings it to the nearest value; the
// sign of what then remains is put below its last bit, where it decides what would be a tie.
__device__ inline u32 codes4(const float* x, const BlockBy& b) {
    float y[4];
    const float pre = b.top >= 0x1p64f ? 0x1p-64f : 1.0f, top = b.top * pre, down = b.by * (1.0f / 448.0f) / pre;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = __builtin_fabsf(x[k]), p = a * pre * 448.0f, rest = __builtin_fmaf(a * pre, 448.0f, -p);
        float q = a * b.by;
        q = __builtin_fmaf(__builtin_fmaf(-q, top, p) + rest, down, q);
        const float left = __builtin_fmaf(-q, top, p) + rest;
        u32 bits = __float_as_uint(q);
        if (left != 0.0f && bits != 0) bits = (bits - (left < 0.0f ? 1u : 0u)) | 1u;
        q = __builtin_copysignf(__uint_as_float(bits), x[k]);
        // what is larger than the largest finite value is infinite
        y[k] = a > b.top ? __builtin_copysignf(b.kept ? 448.0f : 0.0f, x[k]) : (__builtin_fabsf(q) > 448.0f ? __builtin_copysignf(448.0f, q) : q);
        if (!b.kept && a == a) y[k] = __builtin_copysignf(0.0f, x[k]);
    }
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return static_cast<u32>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true));
}
__device__ inline u32x2 codes8(const float (&x)[8], const BlockBy& b) { return u32x2{codes4(x, b), codes4(x + 4, b)}; }

// ---- the codec ------------------------------------------------------------------------------------------------------

struct BlockArgs {
    void* x; i64 ldx;                    // values: read by one direction, written by the other
    u8* q; i64 ldq;
    float* scale; i64 lds;
    u64 items;                           // wavefronts' pieces of 512 columns (rows of scales of their own), or blocks of 128 x 128
    u32 rows, cols, across;              // across: pieces of a row, or blocks of a row
    u32 block_rows;
};

// A wavefront takes 512 columns of a row.
template <typename R, bool VEC>
__global__ __launch_bounds__(256) void k_block_encode_rows(BlockArgs p) {
    const u64 item = static_cast<u64>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (item >= p.items) return;
    const u32 row = static_cast<u32>(item / p.across), lane = threadIdx.x & 63;
    const i64 k = static_cast<i64>(item % p.across) * kWaveCols + lane * kLaneCols;
    float v[8];
    R::template load<VEC>(static_cast<const typename R::elem*>(p.x) + static_cast<i64>(row) * p.ldx, k, p.cols, v);
    const BlockBy b = block_by(largest_of16(largest8(v)));
    store8_codes(p.q + static_cast<i64>(row) * p.ldq, k, p.cols, codes8(v, b));
    if ((lane & 15u) == 0 && k < p.cols) p.scale[static_cast<i64>(row) * p.lds + k / kFp8Block] = b.scale;
}

// A workgroup takes a block of 128 x 128, sixteen rows at a time, and keeps it in registers between looking for its largest and making codes of it.
template <typename R, bool VEC>
__global__ __launch_bounds__(256) void k_block_encode_squares(BlockArgs p) {
    __shared__ u32 s_top[4];
    const u32 row0 = static_cast<u32>(blockIdx.x / p.across) * kFp8Block + (threadIdx.x >> 4);
    const u32 block = static_cast<u32>(blockIdx.x % p.across);
    const i64 k = static_cast<i64>(block) * kFp8Block + (threadIdx.x & 15u) * kLaneCols;
    float v[8][8];
    u32 top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 row = row0 + i * 16;
        R::template load<VEC>(static_cast<const typename R::elem*>(p.x) + static_cast<i64>(row < p.rows ? row : 0) * p.ldx, k, row < p.rows ? p.cols : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 t = largest8(v[i]);
        top = top > t ? top : t;
    }
    top = wave_most(top);
    if ((threadIdx.x & 63u) == 0) s_top[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) top = top > s_top[i] ? top : s_top[i];
    const BlockBy b = block_by(top);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32 row = row0 + i * 16;
        if (row < p.rows) store8_codes(p.q + static_cast<i64>(row) * p.ldq, k, p.cols, codes8(v[i], b));
    }
    if (threadIdx.x == 0) p.scale[static_cast<i64>(row0 / kFp8Block) * p.lds + block] = b.scale;
}

__device__ inline void decode8(u32x2 c, float s, float (&v)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[h]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[h]), true);
        v[4 * h] = lo.x * s; v[4 * h + 1] = lo.y * s; v[4 * h + 2] = hi.x * s; v[4 * h + 3] = hi.y * s;
    }
}

template <typename R, bool VEC>
__global__ __launch_bounds__(256) void k_block_decode(BlockArgs p) {
    const u64 item = static_cast<u64>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (item >= p.items) return;
    const u32 row = static_cast<u32>(item / p.across), lane = threadIdx.x & 63;
    const i64 k = static_cast<i64>(item % p.across) * kWaveCols + lane * kLaneCols;
    if (k >= p.cols) return;
    float v[8];
    const float s = p.scale[static_cast<i64>(p.block_rows == 1 ? row : row / kFp8Block) * p.lds + k / kFp8Block];
    decode8(load8_codes(p.q + static_cast<i64>(row) * p.ldq, k, p.cols), s, v);
    typename R::elem* out = static_cast<typename R::elem*>(p.x) + static_cast<i64>(row) * p.ldx;
    if constexpr (sizeof(typename R::elem) == 2) {
        store8<VEC>(out, k, p.cols, pack8<R>(v));
    } else {
        if (k + 8 <= p.cols) {
            const f32x4 a = {v[0], v[1], v[2], v[3]}, c = {v[4], v[5], v[6], v[7]};
            if (VEC) {
                *reinterpret_cast<f32x4*>(out + k) = a;
                *reinterpret_cast<f32x4*>(out + k + 4) = c;
            } else {
                *reinterpret_cast<f32x4_any*>(out + k) = a;
                *reinterpret_cast<f32x4_any*>(out + k + 4) = c;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i) if (k + i < p.cols) out[k + i] = v[i];
        }
    }
}

// ---- the norm -------------------------------------------------------------------------------------------------------

struct NormArgs {
    const u16* x; i64 ldx;
    const u16* res; i64 ldr;             // NULL: none
    const void* weight;
    u16* sum; i64 ldsum;                 // NULL: not wanted
    u16* y; i64 ldy;
    u8* q; i64 ldq;
    float* scale; i64 lds;
    u32 n_tokens, n;
    u32 waves;                           // of a row
    float eps;
};

__device__ inline float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}

constexpr u32 kNormWaves = 16;           // of a workgroup, at most

// Sums of the wavefronts of a row: of the only one, or in the order of the wavefronts.
template <u32 N>
__device__ inline void row_sums(float (&x)[N], u32 waves, float* s) {
#pragma unroll
    for (u32 i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
    if (waves == 1) return;                                   // the same in the whole workgroup
    const u32 wave = threadIdx.x >> 6;
    __syncthreads();                                          // what the call before this one left has been read
    if ((threadIdx.x & 63u) == 0)
#pragma unroll
        for (u32 i = 0; i < N; ++i) s[wave * N + i] = x[i];
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < N; ++i) {
        x[i] = 0.0f;
        for (u32 w = 0; w < waves; ++w) x[i] += s[w * N + i];
    }
}

// 1 / sqrt(mean + eps), and the power of two that values are multiplied by before they are squared: 2^-64 where squares would leave binary32's range.
struct RowNorm {
    float by, r;                         // u = (h by) r
};
__device__ inline float norm_factor(float squares, u32 n, float eps) { return __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(squares, static_cast<float>(n)) + eps)); }

// Rows of 512 CH columns a wavefront.
template <typename R, typename W, u32 CH, bool VEC>
__global__ __launch_bounds__(64 * kNormWaves) void k_rms_norm(NormArgs p) {
    __shared__ float s[kNormWaves];
    const u32 lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = (blockDim.x >> 6) / p.waves;        // rows of a workgroup: one where a row has several wavefronts
    const u32 row = blockIdx.x * per + wave / p.waves, part = wave % p.waves;
    if (row >= p.n_tokens) return;                            // then a row is one wavefront
    const i64 k0 = static_cast<i64>(part) * (CH * kWaveCols) + lane * kLaneCols;
    u32x4 h[CH];
#pragma unroll
    for (u32 c = 0; c < CH; ++c) h[c] = load8<VEC>(p.x + static_cast<i64>(row) * p.ldx, k0 + c * kWaveCols, p.n);
    if (p.res) {
        u32x4 t[CH];
#pragma unroll
        for (u32 c = 0; c < CH; ++c) t[c] = load8<VEC>(p.res + static_cast<i64>(row) * p.ldr, k0 + c * kWaveCols, p.n);
#pragma unroll
        for (u32 c = 0; c < CH; ++c) {
            float a[8], b[8];
            R::unpack(h[c], a);
            R::unpack(t[c], b);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] += b[i];
            h[c] = pack8<R>(a);
        }
    }
    float squares[1] = {0.0f};
#pragma unroll
    for (u32 c = 0; c < CH; ++c) {
        float a[8];
        R::unpack(h[c], a);
#pragma unroll
        for (int i = 0; i < 8; ++i) squares[0] = __builtin_fmaf(a[i], a[i], squares[0]);
    }
    row_sums(squares, p.waves, s);
    RowNorm m = {1.0f, norm_factor(squares[0], p.n, p.eps)};
    if (!(squares[0] < __builtin_inff())) {                   // the same in the whole row
        m.by = 0x1p-64f;
        squares[0] = 0.0f;
#pragma unroll
        for (u32 c = 0; c < CH; ++c) {
            float a[8];
            R::unpack(h[c], a);
#pragma unroll
            for (int i = 0; i < 8; ++i) squares[0] = __builtin_fmaf(a[i] * m.by, a[i] * m.by, squares[0]);
        }
        row_sums(squares, p.waves, s);
        m.r = norm_factor(squares[0], p.n, p.eps * 0x1p-128f);
    }
    if (p.sum) {
#pragma unroll
        for (u32 c = 0; c < CH; ++c) store8<VEC>(p.sum + static_cast<i64>(row) * p.ldsum, k0 + c * kWaveCols, p.n, h[c]);
    }
    if (!p.y && !p.q) return;
#pragma unroll
    for (u32 c = 0; c < CH; ++c) {
        const i64 k = k0 + c * kWaveCols;
        if (k - lane * kLaneCols >= p.n) break;               // the same in the wavefront
        float a[8], w[8];
        R::unpack(h[c], a);
        W::template load<VEC>(static_cast<const typename W::elem*>(p.weight), k, p.n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = a[i] * m.by * m.r * w[i];
        if (p.y) store8<VEC>(p.y + static_cast<i64>(row) * p.ldy, k, p.n, pack8<R>(a));
        if (p.q) {
            const BlockBy b = block_by(largest_of16(largest8(a)));
            store8_codes(p.q + static_cast<i64>(row) * p.ldq, k, p.n, codes8(a, b));
            if ((lane & 15u) == 0 && k < p.n) p.scale[static_cast<i64>(row) * p.lds + k / kFp8Block] = b.scale;
        }
    }
}

// ---- its gradients --------------------------------------------------------------------------------------------------

struct NormGradArgs {
    const u16* dy; i64 lddy;
    const u16* h; i64 ldh;
    const u16* dsum; i64 ldds;           // NULL: none
    const void* weight;
    u16* dx; i64 lddx;                   // NULL: not wanted
    u8* q; i64 ldq;
    float* scale; i64 lds;
    float* part;                         // [workgroups][n], NULL: the weight's gradient is not wanted
    u32 n_tokens, n;
    u32 waves;                           // of a row
    float eps;
};

// A workgroup takes rows in turn and keeps its lanes' columns of the weight's gradient.
template <typename R, typename W, u32 CH, bool VEC>
__global__ __launch_bounds__(64 * kNormWaves) void k_rms_norm_grad(NormGradArgs p) {
    __shared__ float s[2 * kNormWaves];
    const u32 lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const i64 k0 = static_cast<i64>(part) * (CH * kWaveCols) + lane * kLaneCols;
    float dw[CH][8] = {};
    for (u32 row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        u32x4 h[CH], dy[CH];
#pragma unroll
        for (u32 c = 0; c < CH; ++c) {
            h[c] = load8<VEC>(p.h + static_cast<i64>(row) * p.ldh, k0 + c * kWaveCols, p.n);
            dy[c] = load8<VEC>(p.dy + static_cast<i64>(row) * p.lddy, k0 + c * kWaveCols, p.n);
        }
        float sums[2];
        auto add = [&](float by) {
            sums[0] = sums[1] = 0.0f;
#pragma unroll
            for (u32 c = 0; c < CH; ++c) {
                float a[8], g[8], w[8];
                R::unpack(h[c], a);
                R::unpack(dy[c], g);
                W::template load<VEC>(static_cast<const typename W::elem*>(p.weight), k0 + c * kWaveCols, p.n, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sums[0] = __builtin_fmaf(a[i] * by, a[i] * by, sums[0]);
                    sums[1] = __builtin_fmaf(g[i] * w[i], a[i] * by, sums[1]);
                }
            }
            row_sums(sums, p.waves, s);
        };
        RowNorm m = {1.0f, 0.0f};
        add(1.0f);
        m.r = norm_factor(sums[0], p.n, p.eps);
        if (!(sums[0] < __builtin_inff())) {                  // the same in the workgroup
            m.by = 0x1p-64f;
            add(m.by);
            m.r = norm_factor(sums[0], p.n, p.eps * 0x1p-128f);
        }
        const float mean = __fdiv_rn(sums[1], static_cast<float>(p.n)) * m.r;        // of g u
#pragma unroll
        for (u32 c = 0; c < CH; ++c) {
            const i64 k = k0 + c * kWaveCols;
            if (k - lane * kLaneCols >= p.n) break;           // the same in the wavefront
            float a[8], g[8], w[8], d[8] = {};
            R::unpack(h[c], a);
            R::unpack(dy[c], g);
            W::template load<VEC>(static_cast<const typename W::elem*>(p.weight), k, p.n, w);
            if (p.dsum) R::template load<VEC>(p.dsum + static_cast<i64>(row) * p.ldds, k, p.n, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = a[i] * m.by * m.r;
                dw[c][i] = __builtin_fmaf(g[i], u, dw[c][i]);
                a[i] = __builtin_fmaf(__builtin_fmaf(-u, mean, g[i] * w[i]), m.r * m.by, d[i]);
            }
            if (p.dx) store8<VEC>(p.dx + static_cast<i64>(row) * p.lddx, k, p.n, pack8<R>(a));
            if (p.q) {
                const BlockBy b = block_by(largest_of16(largest8(a)));
                store8_codes(p.q + static_cast<i64>(row) * p.ldq, k, p.n, codes8(a, b));
                if ((lane & 15u) == 0 && k < p.n) p.scale[static_cast<i64>(row) * p.lds + k / kFp8Block] = b.scale;
            }
        }
    }
    if (!p.part) return;
    float* out = p.part + static_cast<u64>(blockIdx.x) * p.n;
#pragma unroll
    for (u32 c = 0; c < CH; ++c) {
        const i64 k = k0 + c * kWaveCols;
        if (k + 8 <= p.n) {
            *reinterpret_cast<f32x4_any*>(out + k) = f32x4{dw[c][0], dw[c][1], dw[c][2], dw[c][3]};
            *reinterpret_cast<f32x4_any*>(out + k + 4) = f32x4{dw[c][4], dw[c][5], dw[c][6], dw[c][7]};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i) if (k + i < p.n) out[k + i] = dw[c][i];
        }
    }
}

// The workgroups' parts of the weight's gradient: 64 columns a workgroup, every sixteenth part a wavefront, added in order.
__global__ __launch_bounds__(1024) void k_rms_norm_join(const float* __restrict__ part, u32 parts, u32 n, float* __restrict__ dweight) {
    __shared__ float s[16][64];
    const u32 col = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
    float x = 0.0f;
    if (col < n)
        for (u32 i = wave; i < parts; i += 16) x += part[static_cast<u64>(i) * n + col];
    s[wave][threadIdx.x & 63] = x;
    __syncthreads();
    if (wave != 0 || col >= n) return;
    for (u32 i = 1; i < 16; ++i) x += s[i][threadIdx.x];
    dweight[col] = x;
}

}  // namespace condensa
