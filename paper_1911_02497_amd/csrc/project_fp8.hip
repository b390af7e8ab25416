// C-ABI entry points of products with matrices in 8 bits (include/condensa.h): checks, choice of form, launches.
#include "fp8_matrix.h"
#include "k_project_fp8.h"

namespace condensa {

struct ProductPlan {
    bool few = false;
    u32 splits = 1, steps_each = 0;
    size_t part = 0;                                          // bytes of the parts
};

constexpr u32 kMostSplits = 16;
constexpr u64 kSplitTiles = 512;                              // tiles of parts that sums are split into, at most

static ProductPlan make_plan(i64 T, i64 n_out, i64 n_sum, bool along) {
    ProductPlan p;
    p.few = along && T <= kFewTokens;
    if (p.few) return p;
    const u32 steps = static_cast<u32>(blocks_of(n_sum));
    const u64 tiles = static_cast<u64>((T + 63) / 64) * ((n_out + 63) / 64);
    u64 s = tiles ? kSplitTiles / tiles : 1;
    s = std::min<u64>(s, std::min<u64>(kMostSplits, steps / 2));
    s = s < 1 ? 1 : s;
    p.steps_each = static_cast<u32>((steps + s - 1) / s);
    p.splits = (steps + p.steps_each - 1) / p.steps_each;
    if (p.splits > 1) p.part = align_up(static_cast<u64>(p.splits) * T * n_out * 4);
    return p;
}
// What a call with T tokens and every call with fewer can do with: parts of most splits, or of as many tiles as sums are split into at all.
static size_t workspace_for(i64 T, i64 n_out) {
    const u64 b = std::min(static_cast<u64>(T) * n_out * 4 * kMostSplits, kSplitTiles * 64 * 64 * 4);
    return b ? align_up(b) : 256;
}

static bool grid_fits(i64 n_tokens, i64 n_wide) { return static_cast<u64>((n_tokens + 63) / 64) * ((n_wide + 63) / 64) < (static_cast<u64>(1) << 24); }

template <int BM, int BN, int WM, int WN, int NB, bool ALONG>
static void launch_tile(const ProductArgs& a, hipStream_t st) {
    const u64 tiles = (static_cast<u64>(a.n_tokens) + BM - 1) / BM * ((static_cast<u64>(a.n_out) + BN - 1) / BN) * a.splits;
    hipLaunchKernelGGL((k_product<BM, BN, WM, WN, NB, ALONG>), dim3(static_cast<unsigned>(tiles)), dim3(64 * WM * WN), 0, st, a);
}

template <bool ALONG>
static void launch_product(const ProductArgs& a, bool rows16, hipStream_t st) {
    const auto tiles = [&](u64 m, u64 n) { return (a.n_tokens + m - 1) / m * ((a.n_out + n - 1) / n); };
    if (!rows16) {
        hipLaunchKernelGGL((k_product_any<ALONG>), dim3(static_cast<unsigned>(tiles(64, 64) * a.splits)), dim3(256), 0, st, a);
    } else if (a.splits == 1 && tiles(256, 256) >= 192) {
        // A tile of 256 rows fills a compute unit.  The one whose rounds over the 256 of them cost less is taken: 8192 x 4608 outputs are 2.25 rounds
        // of 256 x 256, which take as long as three (193 us), and three of 256 x 192 (178 us).
        const auto cost = [&](u64 n) { return (tiles(256, n) + 255) / 256 * n; };
        if (cost(192) < cost(256)) launch_tile<256, 192, 2, 4, 2, ALONG>(a, st);
        else                       launch_tile<256, 256, 2, 4, 2, ALONG>(a, st);
    } else if (a.splits == 1 && tiles(128, 128) >= 192) {
        launch_tile<128, 128, 2, 2, 2, ALONG>(a, st);
    } else {
        launch_tile<64, 64, 2, 2, 4, ALONG>(a, st);
    }
}

// Rows that are 16-byte aligned.
static bool rows16(const void* p, i64 stride) { return aligned_to(p, 16) && stride % 16 == 0; }

static condensa_status product(const condensa_fp8_matrix* x, const condensa_fp8_matrix* w, uint16_t* y, i64 y_stride, int type, void* workspace, size_t workspace_bytes,
                               bool along, void* stream) {
    condensa_status rc = check_matrix(w, CONDENSA_FP8_BLOCK);
    if (rc == CONDENSA_OK) rc = check_matrix(x, 1);
    if (rc != CONDENSA_OK) return rc;
    if (w->rows < 1 || w->rows > kMaxFp8Cols) return CONDENSA_ERR_SHAPE;
    const i64 T = x->rows, n_sum = along ? w->cols : w->rows, n_out = along ? w->rows : w->cols;
    if (x->cols != n_sum || y_stride < n_out || y_stride > kMaxRowStride) return CONDENSA_ERR_SHAPE;
    if (type != CONDENSA_TYPE_F16 && type != CONDENSA_TYPE_BF16) return CONDENSA_ERR_ARG;
    if (T > 0 && !y) return CONDENSA_ERR_NULL;
    if (!aligned_to(y, 2)) return CONDENSA_ERR_ARG;
    if (T == 0) return CONDENSA_OK;
    if (!grid_fits(T, n_out)) return CONDENSA_ERR_SIZE;
    const ProductPlan p = make_plan(T, n_out, n_sum, along);
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < p.part) return CONDENSA_ERR_WORKSPACE;
    ByteRange r[] = {codes_range(x, false), scales_range(x, false), codes_range(w, false), scales_range(w, false),
                     byte_range(y, rows_bytes(T, y_stride, n_out, 2), true), byte_range(p.part ? workspace : nullptr, p.part, true)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    ProductArgs a{};
    a.x = x->q; a.ldx = x->q_stride; a.xs = x->scale; a.ldxs = x->scale_stride;
    a.w = w->q; a.ldw = w->q_stride; a.ws = w->scale; a.ldws = w->scale_stride;
    a.y = y; a.ldy = y_stride;
    a.n_tokens = static_cast<u32>(T); a.n_out = static_cast<u32>(n_out); a.n_sum = static_cast<u32>(n_sum);
    a.splits = p.splits; a.steps_each = p.steps_each;
    a.part = p.part ? static_cast<float*>(workspace) : nullptr;
    a.bf16 = type == CONDENSA_TYPE_BF16;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.few) {
        const u32 waves = std::min(kFewWaves, static_cast<u32>(blocks_of(n_sum)));
        const dim3 grid((a.n_out + 15) / 16), threads(64 * waves);
        if (T <= 16)      hipLaunchKernelGGL(k_product_few<1>, grid, threads, 0, st, a);
        else if (T <= 32) hipLaunchKernelGGL(k_product_few<2>, grid, threads, 0, st, a);
        else              hipLaunchKernelGGL(k_product_few<4>, grid, threads, 0, st, a);
        CONDENSA_LAUNCH_CHECK();
        return CONDENSA_OK;
    }
    const bool fast = rows16(a.x, a.ldx) && rows16(a.w, a.ldw);
    if (along) launch_product<true>(a, fast, st);
    else       launch_product<false>(a, fast, st);
    CONDENSA_LAUNCH_CHECK();
    if (a.part) {
        hipLaunchKernelGGL(k_product_join, dim3((a.n_out + 1023) / 1024, a.n_tokens), dim3(256), 0, st, a);
        CONDENSA_LAUNCH_CHECK();
    }
    return CONDENSA_OK;
}

}  // namespace condensa

using namespace condensa;

extern "C" {

size_t condensa_project_fp8_workspace_bytes(const condensa_fp8_matrix* w, int64_t n_tokens, int backward) {
    if (check_matrix(w, CONDENSA_FP8_BLOCK) != CONDENSA_OK || w->rows < 1 || w->rows > kMaxFp8Cols || n_tokens < 0 || n_tokens > kMaxFp8Rows) return 0;
    return workspace_for(n_tokens, backward ? w->cols : w->rows);
}

condensa_status condensa_project_fp8(const condensa_fp8_matrix* x, const condensa_fp8_matrix* w, uint16_t* y_dev, int64_t y_stride, int type,
                                     void* workspace_dev, size_t workspace_bytes, void* stream) {
    return product(x, w, y_dev, y_stride, type, workspace_dev, workspace_bytes, true, stream);
}

condensa_status condensa_project_fp8_backward(const condensa_fp8_matrix* dy, const condensa_fp8_matrix* w, uint16_t* dx_dev, int64_t dx_stride, int type,
                                              void* workspace_dev, size_t workspace_bytes, void* stream) {
    return product(dy, w, dx_dev, dx_stride, type, workspace_dev, workspace_bytes, false, stream);
}

}  // extern "C"
