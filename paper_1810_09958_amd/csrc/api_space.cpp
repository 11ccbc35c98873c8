// C-ABI layer of the operators of a state-space block: argument validation (pure
// host code, no HIP call) and dispatch.
#include <algorithm>

#include "api_checks.hpp"

using namespace isam;
using namespace isam::api;

namespace {

// A [T][batch] tensor of rows of `width` elements in a call.  Two of them that share their strides may
// lie in one wider tensor (as halves of its rows): they overlap only where their rows do.
struct RowsArg {
    const char* name;
    const void* p;
    int64_t st, sb, width;
    bool out;
};

bool rows_overlap(const RowsArg& a, size_t a_b, const RowsArg& b, size_t b_b, int64_t T, int64_t batch, size_t es) {
    if (!overlaps(a.p, a_b, b.p, b_b)) return false;
    if ((T > 1 && a.st != b.st) || (batch > 1 && a.sb != b.sb)) return true;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p, lo = std::min(pa, pb);
    const uint64_t gap = std::max(pa, pb) - lo, first = (uint64_t)(pa < pb ? a.width : b.width) * es;
    if (gap < first || gap % es) return true;  // the rows themselves meet
    const int64_t whole = (int64_t)(gap / es) + (pa < pb ? b.width : a.width);
    return !rows_apart(T, a.st, batch, a.sb, whole);
}

// Checks the strides, extents and overlaps of the rows of a call, and of the rows with its dense tensors.
template <size_t N, size_t M>
isam_status_t rows_check(RowsArg (&r)[N], const Tensor (&t)[M], int64_t T, int64_t batch, size_t es, const char* who) {
    size_t bytes[N];
    for (size_t i = 0; i < N; ++i) {
        bytes[i] = 0;
        if (!r[i].p) continue;
        if (T <= 1) r[i].st = 0;  // (one token: no second one to stride to)
        if (batch <= 1) r[i].sb = 0;
        if (r[i].st < 0 || r[i].sb < 0) return fail(ISAM_ERR_INVALID_ARG, "%s: negative stride of %s", who, r[i].name);
        if (!extent(T, r[i].st, batch, r[i].sb, r[i].width, es, &bytes[i]))
            return fail(ISAM_ERR_UNSUPPORTED, "%s: %s spans more than 2^46 bytes", who, r[i].name);
        if (r[i].out && !rows_apart(T, r[i].st, batch, r[i].sb, r[i].width))
            return fail(ISAM_ERR_INVALID_ARG, "%s: rows of %s overlap", who, r[i].name);
    }
    for (size_t i = 0; i < N; ++i) {
        if (!r[i].p) continue;
        for (size_t j = i + 1; j < N; ++j) {
            if (r[j].p && (r[i].out || r[j].out) && rows_overlap(r[i], bytes[i], r[j], bytes[j], T, batch, es))
                return fail(ISAM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, r[i].name, r[j].name);
        }
        for (size_t j = 0; j < M; ++j) {
            if ((r[i].out || t[j].out) && overlaps(r[i].p, bytes[i], t[j].p, t[j].bytes))
                return fail(ISAM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, r[i].name, t[j].name);
        }
    }
    return disjoint(t, who);
}

// Strides and extent of the reset marks.
isam_status_t reset_check(const uint8_t* reset, int64_t T, int64_t* st, int64_t batch, int64_t* sb, size_t* bytes, const char* who) {
    *bytes = 0;
    if (!reset) return ISAM_OK;
    if (T <= 1) *st = 0;
    if (batch <= 1) *sb = 0;
    if (*st < 0 || *sb < 0) return fail(ISAM_ERR_INVALID_ARG, "%s: negative stride of reset", who);
    if (!extent(T, *st, batch, *sb, 1, 1, bytes)) return fail(ISAM_ERR_UNSUPPORTED, "%s: reset spans more than 2^46 bytes", who);
    return ISAM_OK;
}

// Whether 32 tokens of every tensor lie within 31 bits.
template <size_t N>
isam_status_t rows_near(const RowsArg (&r)[N], size_t es, const uint8_t* reset, int64_t reset_st, const char* who) {
    for (const RowsArg& x : r) {
        if (x.p && !lingru_strides(x.st, x.width, (int64_t)es))
            return fail(ISAM_ERR_UNSUPPORTED, "%s: 32 tokens of %s span more than 2^31 bytes", who, x.name);
    }
    if (reset && !lingru_strides(reset_st, 1, 1)) return fail(ISAM_ERR_UNSUPPORTED, "%s: 32 tokens of reset span more than 2^31 bytes", who);
    return ISAM_OK;
}

ScanRows rows_of(const RowsArg& r) { return ScanRows{r.p, r.st, r.sb}; }

// ---------------------------------------------------------------------------
// Selective scan
// ---------------------------------------------------------------------------
// Sizes whose products stay far below 2^63 (states, partial sums and grids).
bool scan_sizes(int64_t T, int64_t batch, int64_t D, int64_t N) {
    return T < ((int64_t)1 << 40) && batch < ((int64_t)1 << 31) && D < ((int64_t)1 << 31) && N <= kScanMaxN &&
           (__int128)std::max<int64_t>(T, 1) * std::max<int64_t>(batch, 1) * (D + 2 * N) < ((__int128)1 << 42);
}

isam_status_t scan_check(int64_t T, int64_t batch, int64_t D, int64_t N, int type, const char* who) {
    if (T < 0 || batch < 0 || D < 0 || N <= 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size T=%lld batch=%lld D=%lld N=%lld", who, (long long)T, (long long)batch, (long long)D, (long long)N);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (!scan_sizes(T, batch, D, N))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: N=%lld above %lld, or sizes too large", who, (long long)N, (long long)kScanMaxN);
    return ISAM_OK;
}

// Workspace, in floats: the segments' sums and end states; backward also the partial sums of dB and dC (a row for each
// workgroup's channels and token) and of the parameters (one for each segment and sequence).
struct ScanPlan {
    int64_t segs, seg_len;
    size_t sum_f, end_f, bc_f, par_f;
    size_t total() const { return sum_f + end_f + bc_f + par_f; }
};
ScanPlan scan_plan(int64_t T, int64_t batch, int64_t D, int64_t N, bool backward) {
    ScanPlan p{};
    if (T <= 0 || batch <= 0 || D <= 0 || (!backward && T <= kScanFew)) {
        p.segs = 1;
        return p;
    }
    p.segs = scan_segments(T, batch, D, N, device_cus());
    p.seg_len = scan_segment_length(T, p.segs);
    if (p.segs > 1) {
        p.sum_f = (size_t)(p.segs * batch * D + 63) / 64 * 64;
        p.end_f = (size_t)(p.segs * batch * D * N + 63) / 64 * 64;
    }
    if (backward) {
        p.bc_f = (size_t)(cdiv(D, scan_channels(N)) * T * batch * 2 * N + 63) / 64 * 64;
        p.par_f = (size_t)(p.segs * batch * D * (N + 2));
    }
    return p;
}

isam_status_t need_room(size_t need, const void* workspace, size_t workspace_bytes, const char* who) {
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0, room(need));
    return ISAM_OK;
}

}  // namespace

extern "C" isam_status_t isam_selective_scan(int64_t T, int64_t batch, int64_t D, int64_t N, int type, const void* x,
                                             int64_t x_stride_t, int64_t x_stride_b, const void* dt, int64_t dt_stride_t,
                                             int64_t dt_stride_b, const float* A, const void* B, int64_t B_stride_t,
                                             int64_t B_stride_b, const void* C, int64_t C_stride_t, int64_t C_stride_b,
                                             const float* skip, const void* z, int64_t z_stride_t, int64_t z_stride_b,
                                             const float* dt_bias, const float* h0, const uint8_t* reset,
                                             int64_t reset_stride_t, int64_t reset_stride_b, void* y, int64_t y_stride_t,
                                             int64_t y_stride_b, float* h_T, float* states, void* workspace,
                                             size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_selective_scan";
    isam_status_t st = scan_check(T, batch, D, N, type, who);
    if (st != ISAM_OK || batch == 0 || D == 0) return st;
    if (!y && !h_T && !states) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    if (T > 0 && (!x || !dt || !A || !B || !C)) return fail(ISAM_ERR_INVALID_ARG, "%s: x, dt, A, B or C is NULL", who);
    const size_t es = dsize(type), state = (size_t)(batch * D * N) * sizeof(float);
    const ScanPlan p = scan_plan(T, batch, D, N, false);
    const size_t need = p.total() * sizeof(float);
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    RowsArg r[] = {{"x", x, x_stride_t, x_stride_b, D, false}, {"dt", dt, dt_stride_t, dt_stride_b, D, false},
                   {"B", B, B_stride_t, B_stride_b, N, false}, {"C", C, C_stride_t, C_stride_b, N, false},
                   {"z", z, z_stride_t, z_stride_b, D, false}, {"y", y, y_stride_t, y_stride_b, D, true}};
    size_t reset_b;
    if ((st = reset_check(reset, T, &reset_stride_t, batch, &reset_stride_b, &reset_b, who)) != ISAM_OK) return st;
    // (a few tokens: the state may be replaced in place, each thread reads its part before it writes it)
    const bool in_place = h_T && h_T == h0 && T <= kScanFew;
    const Tensor dense[] = {{"A", A, (size_t)(D * N) * 4, false},
                            {"skip", skip, (size_t)D * 4, false},
                            {"dt_bias", dt_bias, (size_t)D * 4, false},
                            {"h0", in_place ? nullptr : h0, state, false},
                            {"reset", reset, reset_b, false},
                            {"h_T", h_T, state, true},
                            {"states", states, (size_t)cdiv(T, kScanChunk) * state, true},
                            {"workspace", workspace, room(need), true}};
    if ((st = rows_check(r, dense, T, batch, es, who)) != ISAM_OK) return st;
    if (T > kScanFew && (st = rows_near(r, es, reset, reset_stride_t, who)) != ISAM_OK) return st;
    ScanArgs a{};
    a.T = T;
    a.batch = batch;
    a.D = D;
    a.N = N;
    a.type = type;
    a.x = rows_of(r[0]);
    a.dt = rows_of(r[1]);
    a.B = rows_of(r[2]);
    a.C = rows_of(r[3]);
    a.z = rows_of(r[4]);
    a.y = rows_of(r[5]);
    a.A = A;
    a.skip = skip;
    a.dt_bias = dt_bias;
    a.h0 = h0;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.h_T = h_T;
    a.states = states;
    a.segs = p.segs;
    a.seg_len = p.seg_len;
    float* const ws = reinterpret_cast<float*>(room_start(workspace));
    a.seg_sum = ws;
    a.seg_end = ws + p.sum_f;
    const hipError_t e = launch_scan_forward(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_selective_scan_workspace_size(int64_t T, int64_t batch, int64_t D, int64_t N, int type) {
    if (T <= 0 || batch <= 0 || D <= 0 || N <= 0 || !valid_dtype(type) || !scan_sizes(T, batch, D, N)) return 0;
    return room(scan_plan(T, batch, D, N, false).total() * sizeof(float));
}

extern "C" isam_status_t isam_selective_scan_backward(
    int64_t T, int64_t batch, int64_t D, int64_t N, int type, const void* x, int64_t x_stride_t, int64_t x_stride_b, const void* dt,
    int64_t dt_stride_t, int64_t dt_stride_b, const float* A, const void* B, int64_t B_stride_t, int64_t B_stride_b, const void* C,
    int64_t C_stride_t, int64_t C_stride_b, const float* skip, const void* z, int64_t z_stride_t, int64_t z_stride_b,
    const float* dt_bias, const uint8_t* reset, int64_t reset_stride_t, int64_t reset_stride_b, const float* states, const void* dy,
    int64_t dy_stride_t, int64_t dy_stride_b, const float* dh_T, void* dx, int64_t dx_stride_t, int64_t dx_stride_b, void* ddt,
    int64_t ddt_stride_t, int64_t ddt_stride_b, float* dA, void* dB, int64_t dB_stride_t, int64_t dB_stride_b, void* dC,
    int64_t dC_stride_t, int64_t dC_stride_b, float* dskip, void* dz, int64_t dz_stride_t, int64_t dz_stride_b, float* ddt_bias,
    float* dh0, void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_selective_scan_backward";
    isam_status_t st = scan_check(T, batch, D, N, type, who);
    if (st != ISAM_OK || D == 0) return st;
    const bool work = T > 0 && batch > 0;
    if (work && (!x || !dt || !A || !B || !C || !states)) return fail(ISAM_ERR_INVALID_ARG, "%s: x, dt, A, B, C or states is NULL", who);
    if (work && (!dx || !ddt || !dB || !dC)) return fail(ISAM_ERR_INVALID_ARG, "%s: dx, ddt, dB or dC is NULL", who);
    if (dz && work && !z) return fail(ISAM_ERR_INVALID_ARG, "%s: dz needs z", who);
    const size_t es = dsize(type), state = (size_t)(batch * D * N) * sizeof(float);
    const ScanPlan p = scan_plan(T, batch, D, N, true);
    const size_t need = p.total() * sizeof(float);
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    RowsArg r[] = {{"x", x, x_stride_t, x_stride_b, D, false},   {"dt", dt, dt_stride_t, dt_stride_b, D, false},
                   {"B", B, B_stride_t, B_stride_b, N, false},   {"C", C, C_stride_t, C_stride_b, N, false},
                   {"z", z, z_stride_t, z_stride_b, D, false},   {"dy", dy, dy_stride_t, dy_stride_b, D, false},
                   {"dx", dx, dx_stride_t, dx_stride_b, D, true}, {"ddt", ddt, ddt_stride_t, ddt_stride_b, D, true},
                   {"dB", dB, dB_stride_t, dB_stride_b, N, true}, {"dC", dC, dC_stride_t, dC_stride_b, N, true},
                   {"dz", dz, dz_stride_t, dz_stride_b, D, true}};
    size_t reset_b;
    if ((st = reset_check(reset, T, &reset_stride_t, batch, &reset_stride_b, &reset_b, who)) != ISAM_OK) return st;
    const Tensor dense[] = {{"A", A, (size_t)(D * N) * 4, false},
                            {"skip", skip, (size_t)D * 4, false},
                            {"dt_bias", dt_bias, (size_t)D * 4, false},
                            {"reset", reset, reset_b, false},
                            {"states", states, (size_t)cdiv(T, kScanChunk) * state, false},
                            {"dh_T", dh_T, state, false},
                            {"dA", dA, (size_t)(D * N) * 4, true},
                            {"dskip", dskip, (size_t)D * 4, true},
                            {"ddt_bias", ddt_bias, (size_t)D * 4, true},
                            {"dh0", dh0, state, true},
                            {"workspace", workspace, room(need), true}};
    if ((st = rows_check(r, dense, T, batch, es, who)) != ISAM_OK) return st;
    if (work && (st = rows_near(r, es, reset, reset_stride_t, who)) != ISAM_OK) return st;
    ScanArgs a{};
    a.T = T;
    a.batch = batch;
    a.D = D;
    a.N = N;
    a.type = type;
    a.x = rows_of(r[0]);
    a.dt = rows_of(r[1]);
    a.B = rows_of(r[2]);
    a.C = rows_of(r[3]);
    a.z = rows_of(r[4]);
    a.dy = rows_of(r[5]);
    a.dx = rows_of(r[6]);
    a.ddt = rows_of(r[7]);
    a.dB = rows_of(r[8]);
    a.dC = rows_of(r[9]);
    a.dz = rows_of(r[10]);
    a.A = A;
    a.skip = skip;
    a.dt_bias = dt_bias;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.states = const_cast<float*>(states);
    a.dh_T = dh_T;
    a.dA = dA;
    a.dskip = dskip;
    a.ddt_bias = ddt_bias;
    a.dh0 = dh0;
    a.segs = p.segs;
    a.seg_len = p.seg_len;
    float* const ws = reinterpret_cast<float*>(room_start(workspace));
    a.seg_sum = ws;
    a.seg_end = ws + p.sum_f;
    a.bc_part = ws + p.sum_f + p.end_f;
    a.par_part = a.bc_part + p.bc_f;
    const hipError_t e = launch_scan_backward(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_selective_scan_backward_workspace_size(int64_t T, int64_t batch, int64_t D, int64_t N, int type) {
    if (T <= 0 || batch <= 0 || D <= 0 || N <= 0 || !valid_dtype(type) || !scan_sizes(T, batch, D, N)) return 0;
    return room(scan_plan(T, batch, D, N, true).total() * sizeof(float));
}
