// Host-side checks of condensa_fp8_matrix that its codec, the norm and the products share.
#pragma once
#include "host_util.h"

namespace condensa {

constexpr int64_t kMaxFp8Rows = static_cast<int64_t>(1) << 24;
constexpr int64_t kMaxFp8Cols = static_cast<int64_t>(1) << 20;
constexpr int64_t kMaxRowStride = static_cast<int64_t>(1) << 22;      // 256 rows of a tile are less than 2^31 bytes apart

inline bool aligned_to(const void* p, u64 bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline int64_t blocks_of(int64_t n) { return (n + CONDENSA_FP8_BLOCK - 1) / CONDENSA_FP8_BLOCK; }
inline u64 rows_bytes(int64_t rows, int64_t stride, int64_t cols, u64 elem) { return rows > 0 ? (static_cast<u64>(rows - 1) * stride + cols) * elem : 0; }

inline condensa_status check_matrix(const condensa_fp8_matrix* m, int block_rows) {           // block_rows 0: either
    if (!m) return CONDENSA_ERR_NULL;
    if (m->rows < 0 || m->rows > kMaxFp8Rows) return CONDENSA_ERR_SIZE;
    if (m->rows > 0 && (!m->q || !m->scale)) return CONDENSA_ERR_NULL;
    if (m->cols < 1 || m->cols > kMaxFp8Cols || m->q_stride < m->cols || m->q_stride > kMaxRowStride || m->scale_stride < blocks_of(m->cols) || m->scale_stride > kMaxFp8Cols)
        return CONDENSA_ERR_SHAPE;
    if ((m->block_rows != 1 && m->block_rows != CONDENSA_FP8_BLOCK) || (block_rows && m->block_rows != block_rows) || m->reserved != 0 || !aligned_to(m->scale, 4))
        return CONDENSA_ERR_ARG;
    return CONDENSA_OK;
}
inline ByteRange codes_range(const condensa_fp8_matrix* m, bool written) { return byte_range(m->q, rows_bytes(m->rows, m->q_stride, m->cols, 1), written); }
inline ByteRange scales_range(const condensa_fp8_matrix* m, bool written) {
    const int64_t rows = m->block_rows == 1 ? m->rows : blocks_of(m->rows);
    return byte_range(m->scale, rows_bytes(rows, m->scale_stride, blocks_of(m->cols), 4), written);
}

}  // namespace condensa
