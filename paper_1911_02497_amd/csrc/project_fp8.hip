// C-ABI entry points of products with matrices in 8 bits (include/condensa.h): checks, choice of form, launches.
#include "fp8_matrix.h"
#include "k_project_fp8.h"

namespace condensa {

struct ProductPlan {
    bool few = false;
    u32 splits = 1, steps_each = 0;
};

// Sums are split where tiles of 64 x 64 are few and steps many.  4608 -> 512, us whole and in four: 96 tokens (16 tiles, 36 steps) 13.1 and 9.0; 2600 -> 650, in two: 100 tokens
// (22 tiles, 21 steps) 10.4 and 10.2; 2048 -> 512: 100 tokens (16 tiles, 16 steps) 7.7 and 7.6.
// That is as far as the figures go: the border at 64 tiles is a quarter of the units, and what parts would gain between it and 256 tiles is not measured.
constexpr u64 kSplitTiles = 64;
constexpr u32 kSplitSteps = 20, kMostSplits = 4;

static ProductPlan make_plan(i64 T, i64 n_out, i64 n_sum, bool along) {
    ProductPlan p;
    p.few = along && T <= kFewTokens;
    const u32 steps = static_cast<u32>(blocks_of(n_sum));
    p.steps_each = steps;
    if (p.few) return p;
    const u64 tiles = static_cast<u64>((T + 63) / 64) * ((n_out + 63) / 64);
    if (tiles > kSplitTiles || steps < kSplitSteps) return p;
    const u32 s = std::min(kMostSplits, steps / 8);
    p.steps_each = (steps + s - 1) / s;
    p.splits = (steps + p.steps_each - 1) / p.steps_each;
    return p;
}
// Rows that are 16-byte aligned; the distance to the next one does not matter where there is none.
static bool rows16(const void* p, i64 stride, i64 rows) { return aligned_to(p, 16) && (stride % 16 == 0 || rows == 1); }
// Rows of a length that is no multiple of sixteen, one behind the other, are copied to aligned ones where tiles are more than the units or sums are long: 1333 tokens 2600 -> 650 (231
// tiles, 21 steps) 18.5 us with the copies and 24.6 as they are; 300 tokens 1003 -> 1999 (160 tiles, 8 steps), 12.8, gain nothing.  Rows of another length that lie at odd addresses
// are read as they are.
static i64 copied_width(i64 cols) { return (cols + 15) / 16 * 16; }
constexpr i64 kCopySum = 1024;
constexpr u64 kCopyTiles = 256, kCopyBytes = static_cast<u64>(1) << 34;                 // a launch's worth of copies, at most
static u64 bytes_of_copy(i64 rows, i64 cols) { return static_cast<u64>(rows) * copied_width(cols); }
static bool copies(const condensa_fp8_matrix* m) { return m->cols % 16 != 0 && !rows16(m->q, m->q_stride, m->rows) && bytes_of_copy(m->rows, m->cols) <= kCopyBytes; }

// What a call with T tokens and every call with fewer can do with: the most parts, of these tokens or of as many tiles as have any, and copies of x and of W.
static size_t part_bytes(i64 T, i64 n_out) { return align_up(kMostSplits * std::min(static_cast<u64>(T) * n_out, kSplitTiles * 64 * 64) * 4); }
static size_t copy_bytes(i64 rows, i64 cols) { return align_up(std::min(bytes_of_copy(rows, cols), kCopyBytes)); }
static size_t workspace_for(const condensa_fp8_matrix* w, i64 T, bool along) {
    const i64 n_sum = along ? w->cols : w->rows, n_out = along ? w->rows : w->cols;
    const size_t b = part_bytes(T, n_out) + (n_sum % 16 != 0 ? copy_bytes(T, n_sum) : 0) + (copies(w) ? copy_bytes(w->rows, w->cols) : 0);
    return b ? b : 256;
}

static bool grid_fits(i64 n_tokens, i64 n_wide) { return static_cast<u64>((n_tokens + 63) / 64) * ((n_wide + 63) / 64) < (static_cast<u64>(1) << 24); }

template <int BM, int BN, int WM, int WN, int NB, bool ALONG>
static void launch_tile(const ProductArgs& a, hipStream_t st) {
    const u64 tiles = (static_cast<u64>(a.n_tokens) + BM - 1) / BM * ((static_cast<u64>(a.n_out) + BN - 1) / BN) * a.splits;
    hipLaunchKernelGGL((k_product<BM, BN, WM, WN, NB, ALONG>), dim3(static_cast<unsigned>(tiles)), dim3(64 * WM * WN), 0, st, a);
}

// Forms of tiles, and what a call costs with each, in us of 36 steps of the sum.  Times below: 4608 -> 4096, 36 steps, and 512 -> 2048, 4 steps (long / short).
enum Form { kTiles64Deep, kTiles64, kTiles128Deep, kTiles128, kTiles192, kTiles256 };
struct FormCost {
    Form form;
    u64 cost;
};
static FormCost best_form(u64 n_tokens, u64 n_out) {
    const auto tiles = [&](u64 m, u64 n) { return (n_tokens + m - 1) / m * ((n_out + n - 1) / n); };
    const u64 t64 = tiles(64, 64), t128 = tiles(128, 128);
    // A tile a unit: 200 tokens 13.5 long, 4.1 short; with tiles of 128, four times fewer, 23.0 and 6.0.
    if (t64 <= 256) return {kTiles64Deep, 14};
    // Two a unit, room for three: 400 tokens (448 tiles) 20.5 long, 800 (416) 5.7 short; with four steps in LDS 21.1 and 6.0, with tiles of 128 23.3 and 6.8.  832 tiles: 36.7 and, of 128, 24.1.
    if (t64 <= 512) return {kTiles64, 21};
    // One a unit, eight wavefronts and four steps in LDS: 800 tokens 24.1; four wavefronts and two steps, which leave room for another workgroup, 35.8.
    if (t128 <= 256) return {kTiles128Deep, 24};
    // Rounds over the 256 units: a workgroup of 128 rows shares its unit with another (43 for two, 34 alone), one of 256 rows does not (70, or 59 with 192 outputs).  2048 tokens,
    // 512 tiles of 128: 43, and 62 with 128 of 256 x 256.  4096 tokens: 94, and 71 with 256 of 256 x 256.  2900 tokens, backward: 71, 59 and, with 288 of 256 x 192, 112.
    const auto rounds = [](u64 n, u64 each) { return (n + each - 1) / each; };
    const u64 c128 = t128 / 512 * 43 + (t128 % 512 == 0 ? 0 : (t128 % 512 <= 256 ? 34 : 43)), c192 = rounds(tiles(256, 192), 256) * 59, c256 = rounds(tiles(256, 256), 256) * 70;
    if (c128 <= c192 && c128 <= c256) return {kTiles128, c128};
    return c192 < c256 ? FormCost{kTiles192, c192} : FormCost{kTiles256, c256};
}

// Outputs that whole rounds of tiles of 256 x 256 make, where what is left costs less in a form of its own than another round; else 0.  8192 x 4608 outputs,
// backward: two rounds and 512 outputs in tiles of 128 161 us, three rounds of 256 x 192 176; 4096 x 4608 93 and 111; 4000 x 4400 forward 53 and 62.
static u32 whole_rounds(const ProductArgs& a, u64 cost) {
    const u64 rows = (a.n_tokens + 255) / 256, columns = a.n_out / 256, rounds = rows * columns / 256;
    if (rounds == 0 || a.n_sum < 16 * kStep) return 0;
    const u64 first = rounds * 256 / rows * 256;
    return first < a.n_out && rounds * 70 + best_form(a.n_tokens, a.n_out - first).cost < cost ? static_cast<u32>(first) : 0;
}

template <bool ALONG>
static condensa_status launch_product(const ProductArgs& a, bool rows16, hipStream_t st) {
    const FormCost best = best_form(a.n_tokens, a.n_out);
    if (!rows16) {
        const u64 tiles = static_cast<u64>((a.n_tokens + 63) / 64) * ((a.n_out + 63) / 64) * a.splits;
        hipLaunchKernelGGL((k_product_any<ALONG>), dim3(static_cast<unsigned>(tiles)), dim3(256), 0, st, a);
    } else if (const u32 first = a.splits > 1 ? 0 : whole_rounds(a, best.cost)) {
        ProductArgs r = a;
        r.n_out = first;
        launch_tile<256, 256, 2, 4, 2, ALONG>(r, st);
        CONDENSA_LAUNCH_CHECK();
        r.n_out = a.n_out - first;
        r.w += ALONG ? static_cast<i64>(first) * a.ldw : first;
        r.ws += ALONG ? static_cast<i64>(first / kStep) * a.ldws : first / kStep;
        r.y += first;
        return launch_product<ALONG>(r, rows16, st);
    } else {
        switch (a.splits > 1 ? kTiles64Deep : best.form) {
            case kTiles64Deep:  launch_tile<64, 64, 2, 2, 4, ALONG>(a, st); break;
            case kTiles64:      launch_tile<64, 64, 2, 2, 3, ALONG>(a, st); break;
            case kTiles128Deep: launch_tile<128, 128, 2, 4, 4, ALONG>(a, st); break;
            case kTiles128:     launch_tile<128, 128, 2, 2, 2, ALONG>(a, st); break;
            case kTiles192:     launch_tile<256, 192, 2, 4, 2, ALONG>(a, st); break;
            case kTiles256:     launch_tile<256, 256, 2, 4, 2, ALONG>(a, st); break;
        }
    }
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

// Names the copy of a matrix's rows and puts it in their place.
static CodesCopy copy_of(const u8** q, i64* ld, i64 rows, i64 cols, void* to) {
    CodesCopy c{};
    c.src = *q; c.ld = *ld; c.dst = static_cast<u8*>(to);
    c.rows = static_cast<u32>(rows); c.cols = static_cast<u32>(cols); c.width = static_cast<u32>(copied_width(cols));
    c.blocks = static_cast<u32>((static_cast<u64>(rows) * (c.width / 16) + 255) / 256);
    *q = c.dst;
    *ld = c.width;
    return c;
}

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
    const size_t need = workspace_for(w, T, along);
    if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < need) return CONDENSA_ERR_WORKSPACE;
    ByteRange r[] = {codes_range(x, false), scales_range(x, false), codes_range(w, false), scales_range(w, false),
                     byte_range(y, rows_bytes(T, y_stride, n_out, 2), true), byte_range(workspace, need, true)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    ProductArgs a{};
    a.x = x->q; a.ldx = x->q_stride; a.xs = x->scale; a.ldxs = x->scale_stride;
    a.w = w->q; a.ldw = w->q_stride; a.ws = w->scale; a.ldws = w->scale_stride;
    a.y = y; a.ldy = y_stride;
    a.n_tokens = static_cast<u32>(T); a.n_out = static_cast<u32>(n_out); a.n_sum = static_cast<u32>(n_sum);
    a.splits = p.splits; a.steps_each = p.steps_each;
    a.part = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
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
    const bool x16 = rows16(a.x, a.ldx, T), w16 = rows16(a.w, a.ldw, w->rows);
    if ((static_cast<u64>((T + 63) / 64) * ((n_out + 63) / 64) > kCopyTiles || n_sum > kCopySum) && !(x16 && w16) && (x16 || copies(x)) && (w16 || copies(w))) {
        CopyArgs c{};
        char* to = static_cast<char*>(workspace) + part_bytes(T, n_out);
        if (copies(x)) {
            c.m[0] = copy_of(&a.x, &a.ldx, T, n_sum, to);
            to += copy_bytes(T, n_sum);
        }
        if (copies(w)) c.m[1] = copy_of(&a.w, &a.ldw, w->rows, w->cols, to);
        hipLaunchKernelGGL(k_product_copy, dim3(c.m[0].blocks + c.m[1].blocks), dim3(256), 0, st, c);
        CONDENSA_LAUNCH_CHECK();
    }
    const bool fast = rows16(a.x, a.ldx, T) && rows16(a.w, a.ldw, w->rows);
    rc = along ? launch_product<true>(a, fast, st) : launch_product<false>(a, fast, st);
    if (rc != CONDENSA_OK) return rc;
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
    return workspace_for(w, n_tokens, !backward);
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
