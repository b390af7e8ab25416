// C-ABI entry points of the adapters beside a shared projection (include/condensa.h): checks, workspace, launches.
#include <cmath>
#include <memory>
#include <new>

#include "host_util.h"
#include "k_adapter.h"

namespace condensa {

constexpr i64 kMaxSide = static_cast<i64>(1) << 20;
constexpr i64 kMaxTokens = static_cast<i64>(1) << 24;
constexpr i64 kMaxStride = static_cast<i64>(1) << 22;       // 256 rows of a tile are less than 2^32 bytes apart
enum : int32_t { kHasGrads = 4 };

static bool aligned(const void* p, u64 bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
static u32 padded_rank(u32 r) { return (r + 31) / 32 * 32; }

static bool list_ok(const condensa_adapter_list* l) {
    return l && l->table_dev && l->n_adapters >= 0 && l->n_adapters <= CONDENSA_MAX_ADAPTERS && l->max_rank >= 0 && l->max_rank <= CONDENSA_MAX_RANK &&
           (l->type == CONDENSA_TYPE_F16 || l->type == CONDENSA_TYPE_BF16) && l->n_in >= 1 && l->n_in <= kMaxSide && l->n_out >= 1 && l->n_out <= kMaxSide;
}

// Tokens of a run of the gradients.  Up to 1536 tokens an adapter's are one run: six passes of a workgroup take no longer than a launch that adds parts.
// Longer lists: short enough that some 1024 workgroups share the columns of x and dy, long enough that the parts of a run, binary32 and as
// wide as a gradient, are small beside the 16-bit rows that it reads.
static u32 run_tokens(i64 n_tokens, i64 n_in, i64 n_out) {
    if (n_tokens <= 1536) return 1536;
    const i64 tiles = (n_in + kGradCols - 1) / kGradCols + (n_out + kGradCols - 1) / kGradCols;
    i64 run = n_tokens * tiles / 1024;
    run = run < 512 ? 512 : run;
    return static_cast<u32>((run + kGradPass - 1) / kGradPass * kGradPass);
}

// Ranks that a workgroup of the gradients takes, in sixteens.
static u32 grad_groups(u32 max_rank) { return max_rank <= 16 ? 1 : 2; }

// Workgroups that share the adapters of a tile of z: more where tiles are few.  us of a forward call, 4608 -> 4096, with 4, 8 and 16: 700 tokens of 64
// requests (22 tiles) 97, 90 and 90; 8192 tokens (256 tiles) 289, 292 and 304.
static u32 down_shares(u32 tiles) { return tiles >= 64 ? 4 : (tiles >= 16 ? 8 : 16); }

// Rows that are no multiple of eight long are copied to aligned rows beside z where more tokens than this use them.  650 -> 2600, us with copies and
// without: 40 tokens 17.7 and 12.1, 400 tokens 20.6 and 23.8.  Up to 256 tokens, whose sums are split, rows as they are would be the faster ones
// (96 tokens: 19.4 and 14.2).
constexpr i64 kPackTokens = 64;
// Sums run over whole steps of 64 of what is copied, into zeros: a last step of its own, with nothing under way before it, took 2 us.
static i64 up_to(i64 n, i64 unit) { return (n + unit - 1) / unit * unit; }

// Values of A that every workgroup of the form for a few tokens reads, at most.
constexpr i64 kFewWork = 1 << 17;

struct Plan {
    bool split = false, few = false;
    u32 rp = 0, splits = 1, steps_each = 0, bm = 64;
    u32 run = 0, n_slots = 0, tiles = 0;
    bool many = false;                                      // adapters than runs: how the parts of gradients are numbered
    bool pack_in = false, pack_out = false;                 // rows of n_in (x, W), rows of n_out (dy)
    i64 in_cols = 0, out_cols = 0, w_rows = 0;              // sizes of the copies, or of what is not copied
    size_t xq = 0, wq = 0, dyq = 0;
    size_t zp = 0, z32 = 0, part = 0, part_wide = 0, row_max = 0, order = 0, seg = 0, slots = 0, total = 0;
};

// Forward passes of up to this many tokens make z token by token and split their sums wherever tiles are few.  4608 -> 4096, us split and not: 192 tokens 27 and
// 64; 384 tokens of 16 adapters 41 and 73, so more tokens than these would gain too.
constexpr i64 kTokenwise = 256;

static Plan make_plan(i64 T, i64 n_in, i64 n_out, u32 n_adapters, u32 max_rank, bool backward) {
    Plan p;
    size_t at = 0;
    auto take = [&](u64 bytes) { const size_t o = at; at += align_up(bytes ? bytes : 1); return o; };
    p.rp = padded_rank(max_rank ? max_rank : 1);
    p.few = !backward && T <= kFewTokens && T * n_in * static_cast<i64>(max_rank) <= kFewWork;
    p.in_cols = n_in;
    if (p.few) return p;
    {
        // The wide product: where tiles of 32 or 64 tokens by 64 outputs would leave compute units without work, several share a sum.
        const i64 n_wide = backward ? n_in : n_out, n_sum = backward ? n_out : n_in;
        p.bm = T <= 32 ? 32 : 64;
        const u64 tiles = static_cast<u64>((T + p.bm - 1) / p.bm) * ((n_wide + 63) / 64);
        const u32 steps = static_cast<u32>((n_sum + 63) / 64);
        if (T > 0 && tiles < 512) {
            // three workgroups of a unit at once, those that make z among them
            const u64 others = backward || T > kTokenwise ? 128 : static_cast<u64>(T), room = 768 - others;
            u32 s = static_cast<u32>(room / tiles), most = steps / 2;
            s = s > most ? most : s;
            // At most 16: 32 tokens 4608 -> 2048 take 17.3 us with up to 32, 16.3 with 16, and 13.4 with 4, which write fewer parts.
            s = s > 16 ? 16 : (s < 1 ? 1 : s);
            // A tile a unit, with many steps under way.  us whole and split: 512 tokens 4608 -> 1024 (128 tiles) 39 and 25, 1000 tokens 512 -> 512 (128) 17.0
            // and 13.4, 1000 tokens 512 -> 1024 (256) 17.3 and 15.0: the border could lie higher.
            if (T > kTokenwise && tiles > 128) s = 1;
            p.split = s > 1 || T <= kTokenwise;
            p.steps_each = (steps + s - 1) / s;
            p.splits = (steps + p.steps_each - 1) / p.steps_each;
            if (p.split) p.part_wide = take(static_cast<u64>(p.splits) * T * n_wide * 4);
        }
        if (!p.split) p.zp = take(static_cast<u64>(T) * p.rp * 4);
        if (p.split || backward) p.z32 = take(static_cast<u64>(T) * p.rp * 4);
        if (!p.split || backward) p.row_max = take(static_cast<u64>(T) * (p.rp / kDownRanks) * 4);
        if (backward) {
            p.run = run_tokens(T, n_in, n_out);
            p.n_slots = static_cast<u32>(T / p.run) + n_adapters;
            p.order = take(static_cast<u64>(T) * 4);
            p.seg = take(static_cast<u64>(n_adapters) * sizeof(uint2));
            p.slots = take(static_cast<u64>(p.n_slots) * sizeof(uint4));
            p.many = n_adapters > T / p.run;
            if (T > p.run) p.part = take(static_cast<u64>(p.many ? 2 * (T / p.run) : p.n_slots) * max_rank * (n_in + n_out) * 4);
        }
    }
    p.pack_in = T > kPackTokens && n_in % 8 != 0;
    p.pack_out = backward && T > kPackTokens && n_out % 8 != 0;
    p.in_cols = p.pack_in ? up_to(n_in, backward ? 8 : 64) : n_in;
    p.out_cols = p.pack_out ? up_to(n_out, 64) : n_out;
    p.w_rows = p.pack_in && p.pack_out ? p.out_cols : n_out;
    if (p.pack_in) {
        p.xq = take(static_cast<u64>(T) * p.in_cols * 2);
        p.wq = take(static_cast<u64>(p.w_rows) * p.in_cols * 2);
    }
    if (p.pack_out) p.dyq = take(static_cast<u64>(T) * p.out_cols * 2);
    p.total = at;
    return p;
}

// Workspace that a call with n_tokens tokens and every call with fewer can do with: each piece of the plan, at least as large as it is at any
// number of tokens up to this one.  (A plan by itself is not: split sums have parts, larger batches none.)
static size_t workspace_for(i64 T, i64 n_in, i64 n_out, u32 n_adapters, u32 max_rank, bool backward) {
    const Plan p = make_plan(T, n_in, n_out, n_adapters, max_rank, backward);
    if (p.few || T == 0) return p.total;
    size_t total = 0;
    auto take = [&](u64 bytes) { total += align_up(bytes ? bytes : 1); };
    const u64 t = static_cast<u64>(T), n_wide = backward ? n_in : n_out, n_sum = backward ? n_out : n_in, columns = (n_wide + 63) / 64;
    // Split sums: below 512 tiles of 64 rows or fewer; at most 16 parts, at most half as many as steps, and 768 tiles of parts where there are several.
    const u64 split_tokens = std::min(t, 511 / columns * 64), steps = (n_sum + 63) / 64;
    const u64 splits = std::max<u64>(1, std::min<u64>(16, steps / 2));
    take(std::min(splits * split_tokens * n_wide * 4, static_cast<u64>(768) * 64 * 64 * 4));
    take(t * p.rp * 4);
    take((backward ? t : split_tokens) * p.rp * 4);
    take(t * (p.rp / kDownRanks) * 4);
    if (backward) {
        const u64 tiles = (n_in + kGradCols - 1) / kGradCols + (n_out + kGradCols - 1) / kGradCols;
        const u64 runs = T <= 1536 ? t / 1536 : std::min<u64>(t / 512, 1024 / tiles + 1);        // of run_tokens, whole ones
        take(t * 4);
        take(static_cast<u64>(n_adapters) * sizeof(uint2));
        take((runs + n_adapters) * sizeof(uint4));
        take(T <= 1536 ? 0 : std::min(2 * runs, runs + n_adapters) * max_rank * (n_in + n_out) * 4);
    }
    if (p.pack_in) {
        take(t * p.in_cols * 2);
        take(static_cast<u64>(p.w_rows) * p.in_cols * 2);
    }
    if (p.pack_out) take(t * p.out_cols * 2);
    return total;
}

template <typename E, bool ALONG>
static condensa_status launch_down(const DownArgs& a, u32 blocks, hipStream_t st) {
    for (const PackArgs& p : a.pack) blocks += p.blocks;
    if (a.vec_x) hipLaunchKernelGGL((k_adapter_down<E, ALONG, true>), dim3(blocks), dim3(64 * kDownWaves), 0, st, a);
    else         hipLaunchKernelGGL((k_adapter_down<E, ALONG, false>), dim3(blocks), dim3(64 * kDownWaves), 0, st, a);
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

template <typename E, int BM, int BN, int WM, int WN, u32 NB, bool ALONG, int ROWS>
static void launch_wide_tile(const WideArgs& a, hipStream_t st) {
    const u64 tiles = (static_cast<u64>(a.n_tokens) + BM - 1) / BM * ((static_cast<u64>(a.n_out) + BN - 1) / BN);
    hipLaunchKernelGGL((k_adapter_wide<E, BM, BN, WM, WN, NB, ALONG, ROWS>), dim3(static_cast<unsigned>(tiles)), dim3(64 * WM * WN), 0, st, a);
}

template <typename E, bool ALONG>
static condensa_status launch_wide(WideArgs a, int rows, hipStream_t st) {
    a.splits = 1;
    a.part = nullptr;
    a.steps_each = (a.n_sum + 63) / 64;
    const auto tiles = [&](u64 m, u64 n) { return (a.n_tokens + m - 1) / m * ((a.n_out + n - 1) / n); };
    // A tile of 256 rows fills a compute unit.  The one whose rounds over the 256 of them cost less is taken: 8192 x 4608 outputs are 2.25 rounds
    // of 256 x 256, which take as long as three, and three of 256 x 192.
    const auto cost = [&](u64 n) { return (tiles(256, n) + 255) / 256 * n; };
    // Short sums are left to smaller tiles.  8192 tokens -> 4096, us with 256 and with 128 rows: sums of 1024 113 and 120, of 512 88 and 91, of 256 76 and 75.
    // Three quarters of a round are wanted: 3584 tokens 4608 -> 4096 (224 tiles) take 134 and 152 us, 2048 tokens (128 tiles) 100 and 88; 2816 tokens (176
    // tiles), which this leaves to 128 rows, 109 and 132.
    if (rows == kRows16 && tiles(256, 256) >= 192 && a.n_sum >= 1024) {
        if (cost(192) < cost(256)) launch_wide_tile<E, 256, 192, 2, 4, 2, ALONG, kRows16>(a, st);
        else                       launch_wide_tile<E, 256, 256, 2, 4, 2, ALONG, kRows16>(a, st);
    } else if (rows != kRowsAny && tiles(128, 128) >= (rows == kRows16 ? 192 : 512)) {
        // One workgroup a unit, or two: what waits for memory is hidden by steps under way or by the other workgroup.
        if (rows != kRows16)                launch_wide_tile<E, 128, 128, 2, 2, 2, ALONG, kRows4>(a, st);
        else if (tiles(128, 128) <= 256)    launch_wide_tile<E, 128, 128, 2, 2, 4, ALONG, kRows16>(a, st);
        else                                launch_wide_tile<E, 128, 128, 2, 2, 2, ALONG, kRows16>(a, st);
    } else {
        if (rows == kRows16 && tiles(64, 64) <= 256)      launch_wide_tile<E, 64, 64, 2, 2, 8, ALONG, kRows16>(a, st);
        else if (rows == kRows16 && tiles(64, 64) <= 512) launch_wide_tile<E, 64, 64, 2, 2, 4, ALONG, kRows16>(a, st);
        else if (rows == kRows16)     launch_wide_tile<E, 64, 64, 2, 2, 3, ALONG, kRows16>(a, st);
        else if (rows == kRows4) launch_wide_tile<E, 64, 64, 2, 2, 3, ALONG, kRows4>(a, st);
        else                     launch_wide_tile<E, 64, 64, 2, 2, 2, ALONG, kRowsAny>(a, st);
    }
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

// The grid of the smallest tiles has to stay below 2^32 threads.
static bool grid_fits(i64 n_tokens, i64 n_wide) { return static_cast<u64>((n_tokens + 63) / 64) * ((n_wide + 63) / 64) < (static_cast<u64>(1) << 24); }

template <typename E, bool ALONG, int BM>
static void launch_split_tile(const DownArgs& d, const WideArgs& w, u32 down_blocks, int rows, hipStream_t st) {
    const dim3 blocks(down_blocks + (w.n_tokens + BM - 1) / BM * ((w.n_out + 63) / 64) * w.splits);
    if (rows == kRows16)     hipLaunchKernelGGL((k_adapter_split<E, ALONG, kRows16, BM>), blocks, dim3(256), 0, st, d, w, down_blocks);
    else if (rows == kRows4) hipLaunchKernelGGL((k_adapter_split<E, ALONG, kRows4, BM>), blocks, dim3(256), 0, st, d, w, down_blocks);
    else                     hipLaunchKernelGGL((k_adapter_split<E, ALONG, kRowsAny, BM>), blocks, dim3(256), 0, st, d, w, down_blocks);
}

template <typename E, bool ALONG>
static condensa_status launch_split(const DownArgs& d, const WideArgs& w, u32 bm, u32 down_blocks, int rows, hipStream_t st) {
    if (bm == 32) launch_split_tile<E, ALONG, 32>(d, w, down_blocks, rows, st);
    else          launch_split_tile<E, ALONG, 64>(d, w, down_blocks, rows, st);
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

template <typename E>
static condensa_status launch_grads(const GradArgs& q, const WideArgs& g, u32 joins, u32 grid, u32 groups, bool vec, hipStream_t st) {
    const dim3 threads(64 * kGradWaves);
    if (groups == 1) {
        if (vec) hipLaunchKernelGGL((k_adapter_grads<E, true, 1>), dim3(grid), threads, 0, st, q, g, joins);
        else     hipLaunchKernelGGL((k_adapter_grads<E, false, 1>), dim3(grid), threads, 0, st, q, g, joins);
    } else {
        if (vec) hipLaunchKernelGGL((k_adapter_grads<E, true, 2>), dim3(grid), threads, 0, st, q, g, joins);
        else     hipLaunchKernelGGL((k_adapter_grads<E, false, 2>), dim3(grid), threads, 0, st, q, g, joins);
    }
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

// Names the copy of rows in the call's workspace and puts it in their place.
static PackArgs pack_into(const u16** rows, i64* ld, i64 n, i64 cols, i64 all_rows, i64 width, u16* copy) {
    PackArgs p{};
    p.src = *rows; p.ld = *ld; p.dst = copy;
    p.rows = static_cast<u32>(n); p.cols = static_cast<u32>(cols);
    p.all_rows = static_cast<u32>(all_rows); p.width = static_cast<u32>(width);
    p.blocks = static_cast<u32>((all_rows + kPackRows - 1) / kPackRows);
    *rows = copy;
    *ld = width;
    return p;
}

// How rows lie that a sum runs along (x, W forward, dy) or across (W in the backward pass).
static int rows_of(const void* p, i64 stride, i64 cols, bool across) {
    if (aligned(p, 16) && stride % 8 == 0 && cols % 8 == 0) return kRows16;
    if (aligned(p, 4) && stride % 2 == 0 && (!across || cols % 2 == 0)) return kRows4;
    return kRowsAny;
}

// Checks that both directions share; `used`: the call has work to do.
static condensa_status check_call(bool used, i64 n_tokens, const void* ids, const void* workspace_dev, size_t workspace_bytes, const Plan& p) {
    if (n_tokens > 0 && !ids) return CONDENSA_ERR_NULL;
    if (!aligned(ids, 4)) return CONDENSA_ERR_ARG;
    if (used && (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < p.total)) return CONDENSA_ERR_WORKSPACE;
    return CONDENSA_OK;
}

static u64 rows_bytes(i64 rows, i64 ld, i64 cols, u64 elem) { return rows > 0 ? (static_cast<u64>(rows - 1) * ld + cols) * elem : 0; }

}  // namespace condensa

using namespace condensa;

template <typename T>
static T* at(void* ws, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(ws) + off); }

extern "C" {

size_t condensa_adapter_list_bytes(int n_adapters) {
    if (n_adapters < 0 || n_adapters > CONDENSA_MAX_ADAPTERS) return 0;
    return align_up((n_adapters ? static_cast<size_t>(n_adapters) : 1) * sizeof(AdapterDesc));
}

condensa_status condensa_adapter_list_init(const condensa_adapter* adapters, int n_adapters, int type, int64_t n_in, int64_t n_out,
                                           void* list_dev, size_t list_bytes, void* stream, condensa_adapter_list* list) {
    if (list == nullptr) return CONDENSA_ERR_NULL;
    if (n_adapters < 0 || n_adapters > CONDENSA_MAX_ADAPTERS) return CONDENSA_ERR_SIZE;
    if (n_adapters > 0 && adapters == nullptr) return CONDENSA_ERR_NULL;
    if (type != CONDENSA_TYPE_F16 && type != CONDENSA_TYPE_BF16) return CONDENSA_ERR_ARG;
    if (n_in < 1 || n_out < 1 || n_in > kMaxSide || n_out > kMaxSide) return CONDENSA_ERR_SHAPE;
    const size_t need = condensa_adapter_list_bytes(n_adapters);
    if (!list_dev || !aligned(list_dev, 256) || list_bytes < need) return CONDENSA_ERR_WORKSPACE;
    std::unique_ptr<ByteRange[]> ranges(new (std::nothrow) ByteRange[static_cast<size_t>(n_adapters) * 4 + 1]);
    if (!ranges) return CONDENSA_ERR_SIZE;
    size_t nr = 0;
    int32_t max_rank = 0, flags = kHasGrads;
    for (int i = 0; i < n_adapters; ++i) {
        const condensa_adapter& s = adapters[i];
        if (s.rank < 1 || s.rank > CONDENSA_MAX_RANK) return CONDENSA_ERR_SHAPE;
        if (!s.a || !s.b || (s.grad_a == nullptr) != (s.grad_b == nullptr)) return CONDENSA_ERR_NULL;
        if (!aligned(s.a, 2) || !aligned(s.b, 2) || !aligned(s.grad_a, 4) || !aligned(s.grad_b, 4)) return CONDENSA_ERR_ARG;
        if (!std::isfinite(s.scale)) return CONDENSA_ERR_DENSITY;
        max_rank = s.rank > max_rank ? s.rank : max_rank;
        if (!s.grad_a) flags &= ~kHasGrads;
        ranges[nr++] = byte_range(s.a, static_cast<u64>(s.rank) * n_in * 2, false);
        ranges[nr++] = byte_range(s.b, static_cast<u64>(s.rank) * n_out * 2, false);
        ranges[nr++] = byte_range(s.grad_a, static_cast<u64>(s.rank) * n_in * 4, true);
        ranges[nr++] = byte_range(s.grad_b, static_cast<u64>(s.rank) * n_out * 4, true);
    }
    ranges[nr++] = byte_range(list_dev, need, true);
    if (ranges_conflict(ranges.get(), nr)) return CONDENSA_ERR_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    for (int first = 0; first < n_adapters; first += kAdapterPoke) {
        AdapterPoke p{};
        const int k = n_adapters - first < kAdapterPoke ? n_adapters - first : kAdapterPoke;
        for (int i = 0; i < k; ++i) {
            const condensa_adapter& s = adapters[first + i];
            p.d[i].a = s.a; p.d[i].b = s.b; p.d[i].grad_a = s.grad_a; p.d[i].grad_b = s.grad_b;
            p.d[i].scale = s.scale; p.d[i].rank = static_cast<u32>(s.rank);
            p.d[i].vec_a = aligned(s.a, 16) && n_in % 8 == 0;
            p.d[i].vec_b = aligned(s.b, 16) && s.rank % 8 == 0;
        }
        hipLaunchKernelGGL(k_adapter_list, dim3(1), dim3(256), 0, st, static_cast<AdapterDesc*>(list_dev), p, static_cast<u32>(first), static_cast<u32>(k));
        CONDENSA_LAUNCH_CHECK();
    }
    list->table_dev = list_dev;
    list->n_in = n_in;
    list->n_out = n_out;
    list->n_adapters = n_adapters;
    list->max_rank = max_rank;
    list->type = type;
    list->flags = flags;
    return CONDENSA_OK;
}

size_t condensa_adapter_workspace_bytes(const condensa_adapter_list* list, int64_t n_tokens, int backward) {
    if (!list_ok(list) || n_tokens < 0 || n_tokens > kMaxTokens) return 0;
    const size_t b = workspace_for(n_tokens, list->n_in, list->n_out, static_cast<u32>(list->n_adapters), static_cast<u32>(list->max_rank), backward != 0);
    return b ? b : 256;
}

condensa_status condensa_adapter_project(const condensa_adapter_list* list, const uint16_t* x_dev, int64_t x_stride, int64_t n_tokens,
                                         const uint16_t* w_dev, int64_t w_stride, const int32_t* token_adapter_dev,
                                         uint16_t* y_dev, int64_t y_stride, uint16_t* z_dev, int64_t z_stride,
                                         void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (!list) return CONDENSA_ERR_NULL;
    if (!list_ok(list)) return CONDENSA_ERR_ARG;
    if (n_tokens < 0 || n_tokens > kMaxTokens) return CONDENSA_ERR_SIZE;
    if (n_tokens > 0 && (!x_dev || !w_dev || !y_dev)) return CONDENSA_ERR_NULL;
    if (x_stride < list->n_in || w_stride < list->n_in || y_stride < list->n_out || x_stride > kMaxStride || w_stride > kMaxStride || y_stride > kMaxStride ||
        (z_dev && (z_stride < list->max_rank || z_stride > kMaxSide)))
        return CONDENSA_ERR_SHAPE;
    if (!aligned(x_dev, 2) || !aligned(w_dev, 2) || !aligned(y_dev, 2) || !aligned(z_dev, 2)) return CONDENSA_ERR_ARG;
    const Plan p = make_plan(n_tokens, list->n_in, list->n_out, static_cast<u32>(list->n_adapters), static_cast<u32>(list->max_rank), false);
    const condensa_status rc = check_call(n_tokens > 0, n_tokens, token_adapter_dev, workspace_dev, workspace_bytes, p);
    if (rc != CONDENSA_OK) return rc;
    if (n_tokens == 0) return CONDENSA_OK;
    if (!grid_fits(n_tokens, list->n_out)) return CONDENSA_ERR_SIZE;
    ByteRange r[] = {byte_range(x_dev, rows_bytes(n_tokens, x_stride, list->n_in, 2), false), byte_range(w_dev, rows_bytes(list->n_out, w_stride, list->n_in, 2), false),
                     byte_range(token_adapter_dev, static_cast<u64>(n_tokens) * 4, false), byte_range(y_dev, rows_bytes(n_tokens, y_stride, list->n_out, 2), true),
                     byte_range(z_dev, static_cast<u64>(n_tokens) * z_stride * 2, true), byte_range(workspace_dev, p.total, true),
                     byte_range(list->table_dev, condensa_adapter_list_bytes(list->n_adapters), false)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool f16 = list->type == CONDENSA_TYPE_F16;
    const bool vec_x = aligned(x_dev, 16) && x_stride % 8 == 0 && list->n_in % 8 == 0;
    WideArgs g{};
    g.x = x_dev; g.ldx = x_stride; g.w = w_dev; g.ldw = w_stride; g.y = y_dev; g.ldy = y_stride;
    g.x_cols = g.w_cols = static_cast<u32>(p.in_cols);
    g.n_tokens = static_cast<u32>(n_tokens); g.n_out = static_cast<u32>(list->n_out); g.n_sum = static_cast<u32>(p.in_cols);
    g.rp = p.rp; g.ids = token_adapter_dev; g.ad = static_cast<const AdapterDesc*>(list->table_dev);
    g.n_adapters = static_cast<u32>(list->n_adapters); g.max_rank = static_cast<u32>(list->max_rank);
    g.splits = p.splits; g.steps_each = p.steps_each;
    g.part = p.split ? at<float>(workspace_dev, p.part_wide) : nullptr;
    g.zp = p.split ? nullptr : at<u16>(workspace_dev, p.zp);
    g.row_max = f16 && !p.split ? at<u32>(workspace_dev, p.row_max) : nullptr;
    if (p.few) {
        const dim3 grid((g.n_out + kFewRows - 1) / kFewRows), threads(64 * kFewWaves);
        const bool vec = vec_x && aligned(w_dev, 16) && w_stride % 8 == 0;
        if (f16) {
            if (vec) hipLaunchKernelGGL((k_adapter_few<ElemF16, true>), grid, threads, 0, st, g, z_dev, z_stride);
            else     hipLaunchKernelGGL((k_adapter_few<ElemF16, false>), grid, threads, 0, st, g, z_dev, z_stride);
        } else {
            if (vec) hipLaunchKernelGGL((k_adapter_few<ElemBF16, true>), grid, threads, 0, st, g, z_dev, z_stride);
            else     hipLaunchKernelGGL((k_adapter_few<ElemBF16, false>), grid, threads, 0, st, g, z_dev, z_stride);
        }
        CONDENSA_LAUNCH_CHECK();
        return CONDENSA_OK;
    }
    DownArgs d{};
    d.x = x_dev; d.ldx = x_stride; d.n_tokens = g.n_tokens; d.n_sum = static_cast<u32>(list->n_in); d.ids = g.ids; d.ad = g.ad; d.n_adapters = g.n_adapters; d.max_rank = g.max_rank;
    d.zp = p.split ? nullptr : at<u16>(workspace_dev, p.zp); d.rp = p.rp; d.z = z_dev; d.ldz = z_stride;
    d.z32 = p.split ? at<float>(workspace_dev, p.z32) : nullptr;
    d.row_max = f16 && !p.split ? at<u32>(workspace_dev, p.row_max) : nullptr;
    d.vec_x = vec_x;
    d.tiles = (g.n_tokens + kDownTokens - 1) / kDownTokens;
    d.shares = down_shares(d.tiles);
    d.by_token = p.split && n_tokens <= kTokenwise;
    u32 down = d.by_token ? g.n_tokens : d.tiles * d.shares;
    if (p.pack_in) {
        d.pack[0] = pack_into(&g.w, &g.ldw, list->n_out, list->n_in, list->n_out, p.in_cols, at<u16>(workspace_dev, p.wq));
        d.pack[1] = pack_into(&g.x, &g.ldx, n_tokens, list->n_in, n_tokens, p.in_cols, at<u16>(workspace_dev, p.xq));
    }
    const int rows = std::min(rows_of(g.x, g.ldx, p.in_cols, false), rows_of(g.w, g.ldw, p.in_cols, false));
    if (p.pack_in || !p.split) {
        const condensa_status s = f16 ? launch_down<ElemF16, true>(d, down, st) : launch_down<ElemBF16, true>(d, down, st);
        if (s != CONDENSA_OK) return s;
        down = 0;
    }
    if (p.split) {
        const condensa_status s = f16 ? launch_split<ElemF16, true>(d, g, p.bm, down, rows, st) : launch_split<ElemBF16, true>(d, g, p.bm, down, rows, st);
        if (s != CONDENSA_OK) return s;
        const dim3 grid((g.n_out + 255) / 256, g.n_tokens);
        if (f16) hipLaunchKernelGGL((k_adapter_split_join<ElemF16, true>), grid, dim3(256), 0, st, g, static_cast<const float*>(d.z32), p.rp);
        else     hipLaunchKernelGGL((k_adapter_split_join<ElemBF16, true>), grid, dim3(256), 0, st, g, static_cast<const float*>(d.z32), p.rp);
        CONDENSA_LAUNCH_CHECK();
        return CONDENSA_OK;
    }
    return f16 ? launch_wide<ElemF16, true>(g, rows, st) : launch_wide<ElemBF16, true>(g, rows, st);
}

condensa_status condensa_adapter_project_backward(const condensa_adapter_list* list, const uint16_t* dy_dev, int64_t dy_stride,
                                                  const uint16_t* x_dev, int64_t x_stride, int64_t n_tokens,
                                                  const uint16_t* w_dev, int64_t w_stride, const int32_t* token_adapter_dev,
                                                  const uint16_t* z_dev, int64_t z_stride, uint16_t* dx_dev, int64_t dx_stride,
                                                  void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (!list) return CONDENSA_ERR_NULL;
    if (!list_ok(list)) return CONDENSA_ERR_ARG;
    if (!(list->flags & kHasGrads)) return CONDENSA_ERR_NULL;
    if (n_tokens < 0 || n_tokens > kMaxTokens) return CONDENSA_ERR_SIZE;
    if (n_tokens > 0 && (!dy_dev || !x_dev || !w_dev || !z_dev)) return CONDENSA_ERR_NULL;
    if (x_stride < list->n_in || w_stride < list->n_in || dy_stride < list->n_out || x_stride > kMaxStride || w_stride > kMaxStride || dy_stride > kMaxStride ||
        z_stride < list->max_rank || z_stride > kMaxSide || (dx_dev && (dx_stride < list->n_in || dx_stride > kMaxStride)))
        return CONDENSA_ERR_SHAPE;
    if (!aligned(dy_dev, 2) || !aligned(x_dev, 2) || !aligned(w_dev, 2) || !aligned(z_dev, 2) || !aligned(dx_dev, 2)) return CONDENSA_ERR_ARG;
    const Plan p = make_plan(n_tokens, list->n_in, list->n_out, static_cast<u32>(list->n_adapters), static_cast<u32>(list->max_rank), true);
    const condensa_status rc = check_call(n_tokens > 0 || list->n_adapters > 0, n_tokens, token_adapter_dev, workspace_dev, workspace_bytes, p);
    if (rc != CONDENSA_OK) return rc;
    if (dx_dev && !grid_fits(n_tokens, list->n_in)) return CONDENSA_ERR_SIZE;
    ByteRange r[] = {byte_range(dy_dev, rows_bytes(n_tokens, dy_stride, list->n_out, 2), false), byte_range(x_dev, rows_bytes(n_tokens, x_stride, list->n_in, 2), false),
                     byte_range(w_dev, rows_bytes(list->n_out, w_stride, list->n_in, 2), false), byte_range(token_adapter_dev, static_cast<u64>(n_tokens) * 4, false),
                     byte_range(z_dev, static_cast<u64>(n_tokens) * z_stride * 2, false), byte_range(dx_dev, rows_bytes(n_tokens, dx_stride, list->n_in, 2), true),
                     byte_range(workspace_dev, p.total, true), byte_range(list->table_dev, condensa_adapter_list_bytes(list->n_adapters), false)};
    if (ranges_conflict(r, sizeof(r) / sizeof(r[0]))) return CONDENSA_ERR_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool f16 = list->type == CONDENSA_TYPE_F16;
    const bool vec_dy = aligned(dy_dev, 16) && dy_stride % 8 == 0 && list->n_out % 8 == 0;
    const u32 T = static_cast<u32>(n_tokens), n = static_cast<u32>(list->n_adapters);
    const AdapterDesc* ad = static_cast<const AdapterDesc*>(list->table_dev);
    DownArgs d{};
    d.x = dy_dev; d.ldx = dy_stride; d.n_tokens = T; d.n_sum = static_cast<u32>(list->n_out); d.ids = token_adapter_dev; d.ad = ad; d.n_adapters = n;
    d.max_rank = static_cast<u32>(list->max_rank);
    const bool wide = dx_dev && T > 0, split = wide && p.split;
    d.zp = p.split || !wide ? nullptr : at<u16>(workspace_dev, p.zp); d.rp = p.rp; d.z32 = at<float>(workspace_dev, p.z32); d.row_max = f16 ? at<u32>(workspace_dev, p.row_max) : nullptr;
    d.vec_x = vec_dy;
    d.tiles = (T + kDownTokens - 1) / kDownTokens;
    d.shares = down_shares(d.tiles);
    d.order = at<u32>(workspace_dev, p.order); d.seg = at<uint2>(workspace_dev, p.seg); d.slots = at<uint4>(workspace_dev, p.slots);
    d.n_slots = p.n_slots; d.run = p.run;
    const bool pack = p.pack_in || p.pack_out;                    // a launch of its own for z and the copies
    const u32 waves = split && !pack ? 4 : kDownWaves;
    d.sorters = (n + waves - 1) / waves;
    u32 blocks = d.tiles * d.shares + d.sorters;
    if (blocks == 0) return CONDENSA_OK;
    WideArgs g{};
    g.x = dy_dev; g.ldx = dy_stride; g.w = w_dev; g.ldw = w_stride; g.y = dx_dev; g.ldy = dx_stride;
    g.n_tokens = T; g.n_out = static_cast<u32>(list->n_in); g.n_sum = static_cast<u32>(p.w_rows);
    g.zp = d.zp; g.row_max = d.row_max; g.rp = p.rp; g.ids = token_adapter_dev; g.ad = ad; g.n_adapters = n; g.max_rank = d.max_rank;
    g.splits = p.splits; g.steps_each = p.steps_each;
    g.part = p.split ? at<float>(workspace_dev, p.part_wide) : nullptr;
    g.x_cols = static_cast<u32>(p.out_cols);
    g.w_cols = static_cast<u32>(p.in_cols);
    const u16* x_rows = x_dev;
    i64 ldx = x_stride;
    if (p.pack_out) d.pack[0] = pack_into(&g.x, &g.ldx, n_tokens, list->n_out, n_tokens, p.out_cols, at<u16>(workspace_dev, p.dyq));
    if (p.pack_in) {
        d.pack[1] = pack_into(&x_rows, &ldx, n_tokens, list->n_in, n_tokens, p.in_cols, at<u16>(workspace_dev, p.xq));
        if (wide) d.pack[2] = pack_into(&g.w, &g.ldw, list->n_out, list->n_in, p.w_rows, p.in_cols, at<u16>(workspace_dev, p.wq));
    }
    const int rows = std::min(rows_of(g.x, g.ldx, p.out_cols, false), rows_of(g.w, g.ldw, p.in_cols, true));
    condensa_status s;
    if (pack || !split) {
        s = f16 ? launch_down<ElemF16, false>(d, blocks, st) : launch_down<ElemBF16, false>(d, blocks, st);
        if (s != CONDENSA_OK) return s;
        blocks = 0;
    }
    if (split) {
        s = f16 ? launch_split<ElemF16, false>(d, g, p.bm, blocks, rows, st) : launch_split<ElemBF16, false>(d, g, p.bm, blocks, rows, st);
        if (s != CONDENSA_OK) return s;
    } else if (wide) {
        s = f16 ? launch_wide<ElemF16, false>(g, rows, st) : launch_wide<ElemBF16, false>(g, rows, st);
        if (s != CONDENSA_OK) return s;
    }
    const u32 joins = split ? (g.n_out + 255) / 256 * T : 0;
    if (n == 0 && joins == 0) return CONDENSA_OK;
    GradArgs q{};
    q.x = x_rows; q.ldx = ldx; q.n_in = static_cast<u32>(list->n_in); q.dy = g.x; q.ldy = g.ldx; q.n_out = static_cast<u32>(list->n_out);
    q.x_cols = g.w_cols; q.dy_cols = g.x_cols;
    q.dz = d.z32; q.rp = p.rp; q.z = z_dev; q.ldz = z_stride; q.row_max = d.row_max; q.order = d.order; q.seg = d.seg; q.slots = d.slots; q.ad = ad;
    q.max_rank = d.max_rank; q.run = p.run;
    q.tiles_in = (q.n_in + kGradCols - 1) / kGradCols;
    q.tiles = q.tiles_in + (q.n_out + kGradCols - 1) / kGradCols;
    q.many = p.many;
    q.part = n_tokens > p.run ? at<float>(workspace_dev, p.part) : nullptr;
    const u32 groups = grad_groups(q.max_rank);
    q.rank_groups = (q.max_rank + 16 * groups - 1) / (16 * groups);
    const bool vec = aligned(q.x, 16) && q.ldx % 8 == 0 && p.in_cols % 8 == 0 && aligned(q.dy, 16) && q.ldy % 8 == 0 && p.out_cols % 8 == 0;
    // As many slots a launch as keep it below 2^22 workgroups of 512; dx's parts are added beside the first.
    const u32 each_slot = q.rank_groups * q.tiles, all_slots = n > 0 && each_slot > 0 ? p.n_slots : 0;
    u32 join_blocks = joins;
    do {
        const u32 slots = all_slots ? std::min(all_slots - q.slot0, (1u << 22) / each_slot) : 0;
        const u32 grid = (join_blocks + 1) / 2 + slots * each_slot;
        s = f16 ? launch_grads<ElemF16>(q, g, join_blocks, grid, groups, vec, st) : launch_grads<ElemBF16>(q, g, join_blocks, grid, groups, vec, st);
        if (s != CONDENSA_OK) return s;
        q.slot0 += slots;
        join_blocks = 0;
    } while (q.slot0 < all_slots);
    if (n > 0 && n_tokens > p.run) {
        const u64 elems = static_cast<u64>(q.max_rank) * (list->n_in + list->n_out);
        u64 each = (elems + 1023) / 1024;
        each = each > 512 ? 512 : each;
        hipLaunchKernelGGL(k_adapter_join, dim3(static_cast<unsigned>(each * n)), dim3(256), 0, st, q, static_cast<u32>(each));
        CONDENSA_LAUNCH_CHECK();
    }
    return CONDENSA_OK;
}

}  // extern "C"
