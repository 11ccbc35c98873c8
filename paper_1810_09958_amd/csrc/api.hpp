// Host-side helpers shared by the C-ABI sources (api.cpp defines them).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/isam.h"
#include "kernels.hpp"

namespace isam {
namespace api {

// Records the calling thread's reason and returns the status.
isam_status_t fail(isam_status_t st, const char* fmt, ...);
isam_status_t hip_fail(hipError_t e, const char* what);
void clear_error();
const char* last_error();
bool log_enabled();
bool overlaps(const void* a, size_t an, const void* b, size_t bn);
int device_cus();

inline bool valid_dtype(int t) { return t == ISAM_F32 || t == ISAM_BF16; }
inline size_t dsize(int t) { return t == ISAM_BF16 ? 2 : 4; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr int64_t kMaxExtent = (int64_t(1) << 31) - 1;

// The library's matrix product on validated operands (as isam_gemm, C overwritten).
isam_status_t product(int trans_a, int trans_b, int64_t M, int64_t N, int64_t K, int ab_type, const void* A, int64_t lda,
                      const void* B, int64_t ldb, int c_type, void* C, int64_t ldc, void* workspace, size_t workspace_bytes,
                      hipStream_t stream, const char* who);
size_t product_workspace(int trans_a, int trans_b, int64_t M, int64_t N, int64_t K, int ab_type);

}  // namespace api
}  // namespace isam
