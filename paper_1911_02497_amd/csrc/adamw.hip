// C-ABI entry points of the AdamW step (include/condensa.h): checks, the device list, one launch per step.
#include <cmath>
#include <memory>
#include <new>

#include "host_util.h"
#include "k_adamw.h"

namespace condensa {

static bool known_type(int t) { return t == CONDENSA_TYPE_F32 || t == CONDENSA_TYPE_F16 || t == CONDENSA_TYPE_BF16; }

static size_t adamw_table_bytes(u64 n_tensors) { return align_up((n_tensors ? n_tensors : 1) * sizeof(AdamwDesc)); }

// Chunks of all tensors, and their elements; false where a size is beyond what a launch numbers.
static bool adamw_sizes(const condensa_adamw_tensor* tensors, int n_tensors, u64* chunks, u64* elems) {
    *chunks = 0;
    *elems = 0;
    for (int t = 0; t < n_tensors; ++t) {
        if (tensors[t].n > kMaxElems) return false;
        *chunks += (tensors[t].n + kAdamwChunk - 1) / kAdamwChunk;
        *elems += tensors[t].n;
        if (*elems > kMaxElems) return false;
    }
    return true;
}

template <int GRAD>
static void launch_adamw(const AdamwArgs& a, unsigned grid, int state_bits, bool sr, hipStream_t st) {
    if (state_bits == 32) hipLaunchKernelGGL((k_adamw<GRAD, false, false>), dim3(grid), dim3(64), 0, st, a);
    else if (sr)          hipLaunchKernelGGL((k_adamw<GRAD, true, true>), dim3(grid), dim3(64), 0, st, a);
    else                  hipLaunchKernelGGL((k_adamw<GRAD, true, false>), dim3(grid), dim3(64), 0, st, a);
}

}  // namespace condensa

using namespace condensa;

extern "C" {

size_t condensa_adamw_list_bytes(const condensa_adamw_tensor* tensors, int n_tensors) {
    u64 chunks, elems;
    if (n_tensors < 0 || n_tensors > CONDENSA_MAX_TENSORS || (n_tensors > 0 && tensors == nullptr)) return 0;
    if (!adamw_sizes(tensors, n_tensors, &chunks, &elems)) return 0;
    return adamw_table_bytes(static_cast<u64>(n_tensors)) + align_up((chunks ? chunks : 1) * sizeof(u32));
}

condensa_status condensa_adamw_list_init(const condensa_adamw_tensor* tensors, int n_tensors, int state_bits, int grad_type,
                                         int code_type, void* list_dev, size_t list_bytes, void* stream, condensa_adamw_list* list) {
    if (list == nullptr) return CONDENSA_ERR_NULL;
    if (n_tensors < 0 || n_tensors > CONDENSA_MAX_TENSORS) return CONDENSA_ERR_SIZE;
    if (n_tensors > 0 && tensors == nullptr) return CONDENSA_ERR_NULL;
    if ((state_bits != 32 && state_bits != 8) || !known_type(grad_type) || (code_type != CONDENSA_TYPE_F16 && code_type != CONDENSA_TYPE_BF16))
        return CONDENSA_ERR_ARG;
    u64 chunks, elems;
    if (!adamw_sizes(tensors, n_tensors, &chunks, &elems)) return CONDENSA_ERR_SIZE;
    const size_t need = adamw_table_bytes(static_cast<u64>(n_tensors)) + align_up((chunks ? chunks : 1) * sizeof(u32));
    if (list_dev == nullptr || (reinterpret_cast<uintptr_t>(list_dev) & 255u) || list_bytes < need) return CONDENSA_ERR_WORKSPACE;
    const size_t count = static_cast<size_t>(n_tensors > 0 ? n_tensors : 1);
    std::unique_ptr<AdamwDesc[]> td(new (std::nothrow) AdamwDesc[count]);
    std::unique_ptr<ByteRange[]> ranges(new (std::nothrow) ByteRange[count * 9 + 1]);
    if (!td || !ranges) return CONDENSA_ERR_SIZE;
    size_t nr = 0;
    u64 chunk = 0, block = 0;
    const u64 gb = grad_type == CONDENSA_TYPE_F32 ? 4 : 2, sb = state_bits / 8;
    for (int t = 0; t < n_tensors; ++t) {
        const condensa_adamw_tensor& s = tensors[t];
        const u64 blocks = (s.n + kStateBlock - 1) / kStateBlock;
        if (s.n > 0) {
            if (!s.w || !s.grad || !s.exp_avg || !s.exp_avg_sq) return CONDENSA_ERR_NULL;
            if ((s.theta == nullptr) != (s.lambda == nullptr)) return CONDENSA_ERR_NULL;
            if (state_bits == 8 && (!s.exp_avg_scale || !s.exp_avg_sq_scale)) return CONDENSA_ERR_NULL;
            if (state_bits == 32 && (s.exp_avg_scale || s.exp_avg_sq_scale)) return CONDENSA_ERR_ARG;
            const uintptr_t odd4 = reinterpret_cast<uintptr_t>(s.w) | reinterpret_cast<uintptr_t>(s.theta) | reinterpret_cast<uintptr_t>(s.lambda) |
                                   reinterpret_cast<uintptr_t>(s.exp_avg_scale) | reinterpret_cast<uintptr_t>(s.exp_avg_sq_scale) |
                                   (gb == 4 ? reinterpret_cast<uintptr_t>(s.grad) : 0) |
                                   (sb == 4 ? reinterpret_cast<uintptr_t>(s.exp_avg) | reinterpret_cast<uintptr_t>(s.exp_avg_sq) : 0);
            if ((odd4 & 3u) || ((reinterpret_cast<uintptr_t>(s.grad) | reinterpret_cast<uintptr_t>(s.codes)) & 1u)) return CONDENSA_ERR_ARG;
        }
        AdamwDesc& d = td[t];
        d.w = s.w; d.grad = s.grad; d.m = s.exp_avg; d.v = s.exp_avg_sq; d.m_scale = s.exp_avg_scale; d.v_scale = s.exp_avg_sq_scale;
        d.theta = s.theta; d.lam = s.lambda; d.codes = s.codes; d.n = s.n;
        d.first_block = block;
        d.first_chunk = static_cast<u32>(chunk);
        const uintptr_t in32 = reinterpret_cast<uintptr_t>(s.w) | reinterpret_cast<uintptr_t>(s.theta) | reinterpret_cast<uintptr_t>(s.lambda);
        const uintptr_t states = reinterpret_cast<uintptr_t>(s.exp_avg) | reinterpret_cast<uintptr_t>(s.exp_avg_sq);
        d.vec = !(in32 & 15u) && !(states & (4 * sb - 1)) && !(reinterpret_cast<uintptr_t>(s.grad) & (4 * gb - 1)) &&
                !(reinterpret_cast<uintptr_t>(s.codes) & 7u);
        block += blocks;
        chunk += (s.n + kAdamwChunk - 1) / kAdamwChunk;
        ranges[nr++] = byte_range(s.w, s.n * 4, true);
        ranges[nr++] = byte_range(s.exp_avg, s.n * sb, true);
        ranges[nr++] = byte_range(s.exp_avg_sq, s.n * sb, true);
        ranges[nr++] = byte_range(s.exp_avg_scale, blocks * 4, true);
        ranges[nr++] = byte_range(s.exp_avg_sq_scale, blocks * 4, true);
        ranges[nr++] = byte_range(s.codes, s.n * 2, true);
        ranges[nr++] = byte_range(s.grad, s.n * gb, false);
        ranges[nr++] = byte_range(s.theta, s.n * 4, false);
        ranges[nr++] = byte_range(s.lambda, s.n * 4, false);
    }
    ranges[nr++] = byte_range(list_dev, need, true);
    if (ranges_conflict(ranges.get(), nr)) return CONDENSA_ERR_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    AdamwDesc* dst = static_cast<AdamwDesc*>(list_dev);
    u32* map = reinterpret_cast<u32*>(static_cast<char*>(list_dev) + adamw_table_bytes(static_cast<u64>(n_tensors)));
    for (int first = 0; first < n_tensors; first += kAdamwPoke) {
        AdamwPoke p{};
        const int k = n_tensors - first < kAdamwPoke ? n_tensors - first : kAdamwPoke;
        u64 most = 0;
        for (int i = 0; i < k; ++i) {
            p.d[i] = td[first + i];
            const u64 c = (p.d[i].n + kAdamwChunk - 1) / kAdamwChunk;
            most = c > most ? c : most;
        }
        const u64 grid = (most + 255) / 256;
        hipLaunchKernelGGL(k_adamw_list, dim3(static_cast<unsigned>(grid > 64 ? 64 : (grid ? grid : 1))), dim3(256), 0, st, dst, map, p,
                           static_cast<u32>(first), static_cast<u32>(k));
        CONDENSA_LAUNCH_CHECK();
    }
    list->table_dev = list_dev;
    list->map_dev = map;
    list->n_elems = elems;
    list->n_chunks = chunk;
    list->n_tensors = n_tensors;
    list->state_bits = state_bits;
    list->grad_type = grad_type;
    list->code_type = code_type;
    return CONDENSA_OK;
}

condensa_status condensa_lc_adamw_step(const condensa_adamw_list* list, const condensa_adamw_settings* s, void* stream) {
    if (list == nullptr || s == nullptr) return CONDENSA_ERR_NULL;
    if (list->table_dev == nullptr || list->map_dev == nullptr) return CONDENSA_ERR_NULL;
    if ((list->state_bits != 32 && list->state_bits != 8) || !known_type(list->grad_type) || (list->code_type != CONDENSA_TYPE_F16 && list->code_type != CONDENSA_TYPE_BF16) ||
        list->n_chunks > kMaxElems / kAdamwChunk + static_cast<u64>(CONDENSA_MAX_TENSORS))
        return CONDENSA_ERR_ARG;
    if (s->rounding != CONDENSA_ROUND_NEAREST && s->rounding != CONDENSA_ROUND_STOCHASTIC) return CONDENSA_ERR_ARG;
    if (s->rounding == CONDENSA_ROUND_STOCHASTIC && list->state_bits != 8) return CONDENSA_ERR_ARG;
    if (s->reserved != 0 || s->step < 1) return CONDENSA_ERR_ARG;
    if (!std::isfinite(s->lr) || !(s->beta1 >= 0.0 && s->beta1 < 1.0) || !(s->beta2 >= 0.0 && s->beta2 < 1.0) || !(s->eps >= 0.0) ||
        !std::isfinite(s->eps) || !std::isfinite(s->weight_decay) || !(s->mu >= 0.0) || !std::isfinite(s->mu))
        return CONDENSA_ERR_DENSITY;
    if (reinterpret_cast<uintptr_t>(s->grad_scale_dev) & 3u) return CONDENSA_ERR_ARG;
    if (list->n_chunks == 0) return CONDENSA_OK;
    AdamwArgs a{};
    a.td = static_cast<const AdamwDesc*>(list->table_dev);
    a.chunk_map = static_cast<const u32*>(list->map_dev);
    a.grad_scale = s->grad_scale_dev;
    a.beta1 = static_cast<float>(s->beta1);
    a.rest1 = static_cast<float>(1.0 - s->beta1);
    a.beta2 = static_cast<float>(s->beta2);
    a.rest2 = static_cast<float>(1.0 - s->beta2);
    a.decay = static_cast<float>(1.0 - s->lr * s->weight_decay);
    a.step_size = static_cast<float>(s->lr / (1.0 - std::pow(s->beta1, static_cast<double>(s->step))));
    a.correct = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(s->beta2, static_cast<double>(s->step))));
    a.eps = static_cast<float>(s->eps);
    a.mu = static_cast<float>(s->mu);
    a.seed_lo = static_cast<u32>(s->seed);
    a.seed_hi = static_cast<u32>(s->seed >> 32);
    a.code_type = static_cast<u32>(list->code_type);
    const unsigned grid = static_cast<unsigned>(list->n_chunks * (kAdamwChunk / kStateBlock));
    const bool sr = s->rounding == CONDENSA_ROUND_STOCHASTIC;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (list->grad_type == CONDENSA_TYPE_F32)      launch_adamw<CONDENSA_TYPE_F32>(a, grid, list->state_bits, sr, st);
    else if (list->grad_type == CONDENSA_TYPE_F16) launch_adamw<CONDENSA_TYPE_F16>(a, grid, list->state_bits, sr, st);
    else                                           launch_adamw<CONDENSA_TYPE_BF16>(a, grid, list->state_bits, sr, st);
    CONDENSA_LAUNCH_CHECK();
    return CONDENSA_OK;
}

}  // extern "C"
