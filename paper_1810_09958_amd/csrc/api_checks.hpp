// Argument checks shared by the C-ABI sources of the block operators (pure host code, no HIP call).
#pragma once

#include "api.hpp"

namespace isam {
namespace api {

// Workspaces start at the first multiple of 256 bytes of what the caller gives.
inline size_t room(size_t bytes) { return bytes ? bytes + 255 : 0; }
inline char* room_start(void* ws) { return reinterpret_cast<char*>(((uintptr_t)ws + 255) & ~(uintptr_t)255); }

// One tensor of a call: its address range, and whether the call writes it.
struct Tensor {
    const char* name;
    const void* p;
    size_t bytes;
    bool out;
};

// Outputs (and the workspace) must not overlap any other tensor of the call.
template <size_t N>
isam_status_t disjoint(const Tensor (&t)[N], const char* who) {
    for (size_t i = 0; i < N; ++i) {
        for (size_t j = i + 1; j < N; ++j) {
            if ((t[i].out || t[j].out) && overlaps(t[i].p, t[i].bytes, t[j].p, t[j].bytes))
                return fail(ISAM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, t[i].name, t[j].name);
        }
    }
    return ISAM_OK;
}

// Address range of rows (i, j), i < n, j < m, of `width` elements; false if it
// passes 2^46 bytes (no such tensor exists, and offsets stay within 64 bits).
inline bool extent(int64_t n, int64_t stride_n, int64_t m, int64_t stride_m, int64_t width, size_t es, size_t* bytes) {
    *bytes = 0;
    if (n == 0 || m == 0 || width == 0) return true;
    const __int128 e = ((__int128)(n - 1) * stride_n + (__int128)(m - 1) * stride_m + width) * (__int128)es;
    if (e > ((__int128)1 << 46)) return false;
    *bytes = (size_t)e;
    return true;
}

// Whether no two rows (i, j) of `width` elements share an element.
inline bool rows_apart(int64_t n, int64_t stride_n, int64_t m, int64_t stride_m, int64_t width) {
    const bool inner_m = m <= 1 || stride_m >= width, inner_n = n <= 1 || stride_n >= width;
    return (inner_m && (n <= 1 || (__int128)stride_n >= (__int128)(m - 1) * (m > 1 ? stride_m : 0) + width)) ||
           (inner_n && (m <= 1 || (__int128)stride_m >= (__int128)(n - 1) * (n > 1 ? stride_n : 0) + width));
}

// Address range of a matrix operand (0 bytes for NULL); false if a row is longer than
// its leading dimension or the range passes 2^46 bytes.
inline bool matrix(const void* p, int64_t rows, int64_t D, int64_t ld, size_t es, size_t* bytes) {
    *bytes = 0;
    if (!p) return true;
    return ld >= D && extent(rows, ld, 1, 0, D, es, bytes);
}

// A matrix operand whose extent must stay below 2^31 bytes; a null one has none.
inline isam_status_t small_matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t es, size_t* bytes,
                           const char* who) {
    *bytes = 0;
    if (!p || rows == 0 || cols == 0) return ISAM_OK;
    if (ld < cols) return fail(ISAM_ERR_INVALID_ARG, "%s: leading dimension %lld of %s below %lld", who, (long long)ld, name, (long long)cols);
    if (!extent(rows, ld, 1, 0, cols, es, bytes) || *bytes > (size_t)kMaxExtent)
        return fail(ISAM_ERR_UNSUPPORTED, "%s: %s spans more than 2^31 bytes", who, name);
    return ISAM_OK;
}

inline bool rows_aligned(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

// What a workspace has to hold.
inline isam_status_t need_room(size_t need, const void* workspace, size_t workspace_bytes, const char* who) {
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0, room(need));
    return ISAM_OK;
}

}  // namespace api
}  // namespace isam
