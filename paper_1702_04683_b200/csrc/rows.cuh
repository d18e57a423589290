// Rows somewhere in device memory: the device view of adacomp_rows_t and the checks of it.
#pragma once

#include "numeric.cuh"

namespace adacomp {

// Device view of adacomp_rows_t.
struct Rows {
    char* data;
    int type;
    uint32_t group;
    uint64_t row_stride, group_stride;
    __device__ __forceinline__ uint64_t offset(uint32_t r) const {
        return group == 0 ? r * row_stride : (r / group) * group_stride + (r % group) * row_stride;
    }
};

// Checks `r` and turns it into its device view.  Distances that make the groups one plain run lose the group.
inline int rows_view(const adacomp_rows_t* r, uint64_t n_rows, bool tokens, Rows* out) {
    if (!r) return ADACOMP_ERR_INVALID;
    if (tokens ? (r->type != ADACOMP_I32 && r->type != ADACOMP_I64) : !known_type(r->type)) return ADACOMP_ERR_INVALID;
    const uint32_t size = tokens ? (r->type == ADACOMP_I64 ? 8u : 4u) : type_size(r->type);
    if (n_rows && (!r->d_data || !aligned(r->d_data, size))) return ADACOMP_ERR_INVALID;
    out->data = static_cast<char*>(r->d_data);
    out->type = r->type;
    out->group = r->group;
    out->row_stride = r->row_stride;
    out->group_stride = r->group_stride;
    if (r->group && (r->group >= n_rows || r->group_stride == r->group * r->row_stride)) out->group = 0;
    return ADACOMP_OK;
}

// Whether rows that are written keep clear of each other.
inline bool rows_apart(const Rows& r, uint64_t n_rows, uint64_t dim) {
    if (n_rows < 2) return true;
    if (r.group == 0) return r.row_stride >= dim;
    const uint64_t groups = (n_rows + r.group - 1) / r.group;
    const uint64_t in_group = r.group > 1 ? (r.group - 1) * r.row_stride + dim : dim;
    if ((r.group == 1 || r.row_stride >= dim) && r.group_stride >= in_group) return true;
    return r.group_stride >= dim && r.row_stride >= (groups - 1) * r.group_stride + dim;
}

// Whether every row starts on a boundary of so many bytes.
inline bool on_grid(const Rows& r, uint32_t bytes) {
    const uint32_t size = type_size(r.type);
    return reinterpret_cast<uintptr_t>(r.data) % bytes == 0 && r.row_stride * size % bytes == 0 &&
           (r.group == 0 || r.group_stride * size % bytes == 0);
}

}  // namespace adacomp
