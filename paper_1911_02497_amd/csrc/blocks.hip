// C-ABI entry points of matrices in 8 bits and of the norm that answers in them (include/condensa.h): checks, choice of form, launches.
#include <cmath>

#include "fp8_matrix.h"
#include "k_blocks.h"

namespace condensa {

constexpr u64 kMaxGroups = static_cast<u64>(1) << 24;        // workgroups of 256 threads that a launch holds; half as many of 512

static bool type_ok(int type, bool f32) { return type == CONDENSA_TYPE_F16 || type == CONDENSA_TYPE_BF16 || (f32 && type == CONDENSA_TYPE_F32); }
static u64 type_bytes(int type) { return type == CONDENSA_TYPE_F32 ? 4 : 2; }
// Rows that are 16-byte aligned and a multiple of eight values long.
static bool vec_rows(const void* p, i64 stride, i64 cols, int type) { return aligned_to(p, 16) && stride % (type == CONDENSA_TYPE_F32 ? 4 : 8) == 0 && cols % 8 == 0; }

enum { kEncodeRows, kEncodeSquares, kDecode };
template <typename R>
static void launch_codec(int what, bool vec, const BlockArgs& a, unsigned groups, hipStream_t st) {
    const dim3 grid(groups), threads(256);
    if (what == kEncodeRows) {
        if (vec) hipLaunchKernelGGL((k_block_encode_rows<R, true>), grid, threads, 0, st, a);
        else     hipLaunchKernelGGL((k_block_encode_rows<R, false>), grid, threads, 0, st, a);
    } else if (what == kEncodeSquares) {
        if (vec) hipLaunchKernelGGL((k_block_encode_squares<R, true>), grid, dim3(64 * kSquareWaves), 0, st, a);
        else     hipLaunchKernelGGL((k_block_encode_squares<R, false>), grid, dim3(64 * kSquareWaves), 0, st, a);
    } else {
        if (vec) hipLaunchKernelGGL((k_block_decode<R, true>), grid, threads, 0, st, a);
        else     hipLaunchKernelGGL((k_block_decode<R, false>), grid, threads, 0, st, a);
    }
}

static condensa_status codec(const condensa_fp8_matrix* m, void* x, int type, i64 stride, bool encode, void* stream) {
    const condensa_status rc = check_matrix(m, 0);
    if (rc != CONDENSA_OK) return rc;
    if (!type_ok(type, true)) return CONDENSA_ERR_ARG;
    if (stride < m->cols || stride > kMaxRowStride) return CONDENSA_ERR_SHAPE;
    if (m->rows > 0 && !x) return CONDENSA_ERR_NULL;
    if (!aligned_to(x, type_bytes(type))) return CONDENSA_ERR_ARG;
    if (m->rows == 0) return CONDENSA_OK;
    const bool squares = encode && m->block_rows != 1;
    BlockArgs a{};
    a.x = x; a.ldx = stride; a.q = m->q; a.ldq = m->q_stride; a.scale = m->scale; a.lds = m->scale_stride;
    a.rows = static_cast<u32>(m->rows); a.cols = static_cast<u32>(m->cols); a.block_rows = static_cast<u32>(m->block_rows);
    a.across = static_cast<u32>(squares ? blocks_of(m->cols) : (m->cols + kWaveCols - 1) / kWaveCols);
    a.items = static_cast<u64>(a.across) * (squares ? blocks_of(m->rows) : m->rows);
    const u64 groups = squares ? a.items : (a.items + 3) / 4;
    if (groups >= (squares ? kMaxGroups / 2 : kMaxGroups)) return CONDENSA_ERR_SIZE;
    ByteRange r[] = {byte_range(x, rows_bytes(m->rows, stride, m->cols, type_bytes(type)), !encode), codes_range(m, encode), scales_range(m, encode)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    const int what = squares ? kEncodeSquares : (encode ? kEncodeRows : kDecode);
    const bool vec = vec_rows(x, stride, m->cols, type);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (type == CONDENSA_TYPE_F32)      launch_codec<RowsF32>(what, vec, a, static_cast<unsigned>(groups), st);
    else if (type == CONDENSA_TYPE_F16) launch_codec<RowsF16>(what, vec, a, static_cast<unsigned>(groups), st);
    else                                launch_codec<RowsBF16>(what, vec, a, static_cast<unsigned>(groups), st);
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

// How a row is shared: pieces of 512 columns that a wavefront has, and wavefronts of a row.
struct RowShare {
    u32 each, waves;
};
static RowShare share_row(i64 width, u32 least_each) {
    const u32 pieces = static_cast<u32>((width + kWaveCols - 1) / kWaveCols);
    u32 each = least_each;
    while ((pieces + each - 1) / each > kNormWaves) each *= 2;
    return RowShare{each, (pieces + each - 1) / each};
}
static_assert(CONDENSA_MAX_NORM_WIDTH == kNormWaves * kWaveCols * 4, "the widest row: four pieces a wavefront");

// Workgroups that share the rows of a backward pass: 256, one a unit, for rows of eight wavefronts and more and for rows of one, of which a workgroup has eight at once; up to 1024 for those
// between; fewer for few tokens, so that each has rows enough and its part of the weight's gradient is small beside them.  8192 tokens of 4608, us with 256, 512 and 1024: 72, 77 and 78, and 2.7, 3.5 and 5.0 to add the parts up.
static u32 grad_groups(i64 n_tokens, i64 width) {
    const u32 waves = share_row(width, 1).waves;
    const u32 slots = waves == 1 ? kNormSlots : 1, most = 256 * (waves >= 8 || waves == 1 ? 1 : 8 / waves);
    const u64 rows = (static_cast<u64>(n_tokens) + 2 * slots - 1) / (2 * slots);
    return static_cast<u32>(rows < most ? rows : most);
}

// Calls launch(pieces of a wavefront, vec) with both as constants.
template <typename F>
static void with_share(u32 each, bool vec, F&& launch) {
    auto pick = [&](auto v) {
        switch (each) {
            case 1: launch(std::integral_constant<u32, 1>{}, v); break;
            case 2: launch(std::integral_constant<u32, 2>{}, v); break;
            default: launch(std::integral_constant<u32, 4>{}, v);
        }
    };
    if (vec) pick(std::true_type{});
    else     pick(std::false_type{});
}
// Calls launch(rows, weight) with objects of the two types.
template <typename F>
static void with_types(int type, int weight_type, F&& launch) {
    if (type == CONDENSA_TYPE_F16) {
        if (weight_type == CONDENSA_TYPE_F32) launch(RowsF16{}, RowsF32{});
        else                                  launch(RowsF16{}, RowsF16{});
    } else {
        if (weight_type == CONDENSA_TYPE_F32) launch(RowsBF16{}, RowsF32{});
        else                                  launch(RowsBF16{}, RowsBF16{});
    }
}

// What both directions check of their calls.
static condensa_status check_norm(i64 n_tokens, i64 width, int type, int weight_type, const void* weight, const condensa_fp8_matrix* codes, float eps, int32_t reserved) {
    if (n_tokens < 0 || n_tokens > kMaxFp8Rows) return CONDENSA_ERR_SIZE;
    if (width < 1 || width > CONDENSA_MAX_NORM_WIDTH) return CONDENSA_ERR_SHAPE;
    if (!type_ok(type, false) || (weight_type != type && weight_type != CONDENSA_TYPE_F32) || reserved != 0) return CONDENSA_ERR_ARG;
    if (!weight) return CONDENSA_ERR_NULL;
    if (!aligned_to(weight, type_bytes(weight_type))) return CONDENSA_ERR_ARG;
    if (!std::isfinite(eps) || eps <= 0.0f) return CONDENSA_ERR_DENSITY;
    if (codes) {
        const condensa_status rc = check_matrix(codes, 1);
        if (rc != CONDENSA_OK) return rc;
        if (codes->rows != n_tokens || codes->cols != width) return CONDENSA_ERR_SHAPE;
    }
    return CONDENSA_OK;
}
static condensa_status check_rows(const void* p, i64 stride, i64 width) {       // of an operand that is there
    if (!p) return CONDENSA_OK;
    if (stride < width || stride > kMaxRowStride) return CONDENSA_ERR_SHAPE;
    return aligned_to(p, 2) ? CONDENSA_OK : CONDENSA_ERR_ARG;
}
static bool vec_or_none(const void* p, i64 stride, i64 width) { return !p || vec_rows(p, stride, width, CONDENSA_TYPE_F16); }

}  // namespace condensa

using namespace condensa;

extern "C" {

condensa_status condensa_quantize_fp8_blocks(const void* x_dev, int type, int64_t x_stride, const condensa_fp8_matrix* m, void* stream) {
    return codec(m, const_cast<void*>(x_dev), type, x_stride, true, stream);
}

condensa_status condensa_dequantize_fp8_blocks(const condensa_fp8_matrix* m, void* dq_dev, int type, int64_t dq_stride, void* stream) {
    return codec(m, dq_dev, type, dq_stride, false, stream);
}

condensa_status condensa_rms_norm(const condensa_rms_norm_call* c, void* stream) {
    if (!c) return CONDENSA_ERR_NULL;
    condensa_status rc = check_norm(c->n_tokens, c->width, c->type, c->weight_type, c->weight, c->codes, c->eps, c->reserved);
    if (rc != CONDENSA_OK) return rc;
    if (c->n_tokens == 0) return CONDENSA_OK;
    if (!c->x || (!c->sum && !c->y && !c->codes)) return CONDENSA_ERR_NULL;
    const struct { const void* p; i64 stride; } rows[] = {{c->x, c->x_stride}, {c->residual, c->residual_stride}, {c->sum, c->sum_stride}, {c->y, c->y_stride}};
    bool vec = vec_rows(c->weight, 0, c->width, c->weight_type);
    for (const auto& r : rows) {
        rc = check_rows(r.p, r.stride, c->width);
        if (rc != CONDENSA_OK) return rc;
        vec = vec && vec_or_none(r.p, r.stride, c->width);
    }
    // sum may be what it is made of; that buffer is then entered once, as an output
    const bool over_x = c->sum && c->sum == c->x && c->sum_stride == c->x_stride, over_res = c->sum && c->sum == c->residual && c->sum_stride == c->residual_stride;
    auto range = [&](const void* p, i64 stride, bool written) { return byte_range(p, rows_bytes(c->n_tokens, stride, c->width, 2), written); };
    ByteRange r[] = {range(over_x ? nullptr : c->x, c->x_stride, false), range(over_res ? nullptr : c->residual, c->residual_stride, false),
                     range(c->sum, c->sum_stride, true), range(c->y, c->y_stride, true), byte_range(c->weight, c->width * type_bytes(c->weight_type), false),
                     c->codes ? codes_range(c->codes, true) : byte_range(nullptr, 0, true), c->codes ? scales_range(c->codes, true) : byte_range(nullptr, 0, true)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    NormArgs a{};
    a.x = c->x; a.ldx = c->x_stride; a.res = c->residual; a.ldr = c->residual_stride; a.weight = c->weight;
    a.sum = c->sum; a.ldsum = c->sum_stride; a.y = c->y; a.ldy = c->y_stride;
    if (c->codes) { a.q = c->codes->q; a.ldq = c->codes->q_stride; a.scale = c->codes->scale; a.lds = c->codes->scale_stride; }
    a.n_tokens = static_cast<u32>(c->n_tokens); a.n = static_cast<u32>(c->width); a.eps = c->eps;
    const RowShare share = share_row(c->width, 2);
    a.waves = share.waves;
    const u32 rows_each = share.waves == 1 ? 4 : 1;
    const dim3 grid((a.n_tokens + rows_each - 1) / rows_each), threads(64 * share.waves * rows_each);
    if (static_cast<u64>(grid.x) * threads.x >= kMaxGroups * 256) return CONDENSA_ERR_SIZE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    with_types(c->type, c->weight_type, [&](auto rows_type, auto weight_type) {
        with_share(share.each, vec, [&](auto each, auto v) {
            if constexpr (decltype(each)::value > 1) hipLaunchKernelGGL((k_rms_norm<decltype(rows_type), decltype(weight_type), decltype(each)::value, decltype(v)::value>), grid, threads, 0, st, a);
        });
    });
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

size_t condensa_rms_norm_workspace_bytes(int64_t n_tokens, int64_t width) {
    if (n_tokens < 0 || n_tokens > kMaxFp8Rows || width < 1 || width > CONDENSA_MAX_NORM_WIDTH) return 0;
    const size_t b = align_up(static_cast<u64>(grad_groups(n_tokens, width)) * width * 4);
    return b ? b : 256;
}

condensa_status condensa_rms_norm_backward(const condensa_rms_norm_grad_call* c, void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (!c) return CONDENSA_ERR_NULL;
    condensa_status rc = check_norm(c->n_tokens, c->width, c->type, c->weight_type, c->weight, c->codes, c->eps, c->reserved);
    if (rc != CONDENSA_OK) return rc;
    if (c->n_tokens == 0 && !c->dweight) return CONDENSA_OK;
    if (c->n_tokens > 0 && (!c->dy || !c->h || (!c->dx && !c->dweight && !c->codes))) return CONDENSA_ERR_NULL;
    if (!aligned_to(c->dweight, 4)) return CONDENSA_ERR_ARG;
    const struct { const void* p; i64 stride; } rows[] = {{c->dy, c->dy_stride}, {c->h, c->h_stride}, {c->dsum, c->dsum_stride}, {c->dx, c->dx_stride}};
    bool vec = vec_rows(c->weight, 0, c->width, c->weight_type);
    for (const auto& r : rows) {
        rc = check_rows(r.p, r.stride, c->width);
        if (rc != CONDENSA_OK) return rc;
        vec = vec && vec_or_none(r.p, r.stride, c->width);
    }
    const size_t need = condensa_rms_norm_workspace_bytes(c->n_tokens, c->width);
    if (c->dweight && (!workspace_dev || !aligned_to(workspace_dev, 256) || workspace_bytes < need)) return CONDENSA_ERR_WORKSPACE;
    const bool over_dsum = c->dx && c->dx == c->dsum && c->dx_stride == c->dsum_stride;
    auto range = [&](const void* p, i64 stride, bool written) { return byte_range(p, rows_bytes(c->n_tokens, stride, c->width, 2), written); };
    ByteRange r[] = {range(c->dy, c->dy_stride, false), range(c->h, c->h_stride, false), range(over_dsum ? nullptr : c->dsum, c->dsum_stride, false),
                     range(c->dx, c->dx_stride, true), byte_range(c->weight, c->width * type_bytes(c->weight_type), false),
                     byte_range(c->dweight, c->width * 4, true), byte_range(c->dweight ? workspace_dev : nullptr, need, true),
                     c->codes ? codes_range(c->codes, true) : byte_range(nullptr, 0, true), c->codes ? scales_range(c->codes, true) : byte_range(nullptr, 0, true)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    NormGradArgs a{};
    a.dy = c->dy; a.lddy = c->dy_stride; a.h = c->h; a.ldh = c->h_stride; a.dsum = c->dsum; a.ldds = c->dsum_stride; a.weight = c->weight;
    a.dx = c->dx; a.lddx = c->dx_stride;
    if (c->codes) { a.q = c->codes->q; a.ldq = c->codes->q_stride; a.scale = c->codes->scale; a.lds = c->codes->scale_stride; }
    a.part = c->dweight ? static_cast<float*>(workspace_dev) : nullptr;
    a.n_tokens = static_cast<u32>(c->n_tokens); a.n = static_cast<u32>(c->width); a.eps = c->eps;
    const RowShare share = share_row(c->width, 1);
    a.waves = share.waves;
    const u32 groups = grad_groups(c->n_tokens, c->width);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (groups) {
        with_types(c->type, c->weight_type, [&](auto rows_type, auto weight_type) {
            with_share(share.each, vec, [&](auto each, auto v) {
                hipLaunchKernelGGL((k_rms_norm_grad<decltype(rows_type), decltype(weight_type), decltype(each)::value, decltype(v)::value>), dim3(groups), dim3(64 * (share.waves == 1 ? kNormSlots : share.waves)), 0, st, a);
            });
        });
        CONDENSA_LAUNCH_CHECK();
    }
    if (c->dweight) {
        hipLaunchKernelGGL(k_rms_norm_join, dim3((a.n + kJoinCols - 1) / kJoinCols), dim3(kJoinCols * kJoinRows), 0, st, static_cast<const float*>(workspace_dev), groups, a.n, c->dweight);
        CONDENSA_LAUNCH_CHECK();
    }
    return CONDENSA_OK;
}

}  // extern "C"
