// C-ABI layer of the operators of a state-space block: argument validation (pure
// host code, no HIP call) and dispatch.
#include <algorithm>

#include "api_checks.hpp"

using namespace isam;
using namespace isam::api;

namespace {

// A [T][batch] tensor of rows of `width` elements in a call.  Two of them that share their strides may
// lie in one wider tensor (as halves of its rows, or turn by turn): they overlap only where their rows do.
struct RowsArg {
    const char* name;
    const void* p;
    int64_t st, sb, width;
    bool out;
};

// Integers k with lo < k n < hi, n > 0, |k| <= most: the first and the last.
struct Multiples {
    int64_t first, last;
};
Multiples multiples(int64_t lo, int64_t hi, int64_t n, int64_t most) {
    auto floor_div = [&](int64_t v) { return v >= 0 ? v / n : -((-v + n - 1) / n); };
    return {std::max(floor_div(lo) + 1, -most), std::min(-(floor_div(-hi) + 1), most)};
}

// (extents stay within 2^46 bytes)
bool rows_overlap(const RowsArg& a, size_t a_b, const RowsArg& b, size_t b_b, int64_t T, int64_t batch, size_t es) {
    if (!overlaps(a.p, a_b, b.p, b_b)) return false;
    if ((T > 1 && a.st != b.st) || (batch > 1 && a.sb != b.sb)) return true;
    const intptr_t bytes = (intptr_t)b.p - (intptr_t)a.p;
    if (bytes % (intptr_t)es) return true;
    // A row of b lies gap + k far + l near elements from one of a, |k| < fars, |l| < nears; the two meet where that is
    // above -b.width and below a.width.
    const int64_t gap = bytes / (intptr_t)es;
    const bool time_far = a.st >= a.sb;
    const int64_t far = time_far ? a.st : a.sb, fars = (time_far ? T : batch) - 1, near = time_far ? a.sb : a.st,
                  nears = (time_far ? batch : T) - 1;
    const int64_t reach = near * nears;
    const Multiples k = far ? multiples(-b.width - reach - gap, a.width + reach - gap, far, fars) : Multiples{0, 0};
    if (k.last - k.first > 8) return true;  // (rows far from nested: not looked into)
    for (int64_t i = k.first; i <= k.last; ++i) {
        const int64_t at = gap + i * far;
        if (near == 0 ? at > -b.width && at < a.width : [&] {
                const Multiples l = multiples(-b.width - at, a.width - at, near, nears);
                return l.first <= l.last;
            }())
            return true;
    }
    return false;
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
                            {"states", states, (size_t)cdiv(T, scan_chunk(N)) * state, true},
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
    if (st != ISAM_OK) return st;
    if (D == 0) {  // (dB and dC are sums of nothing)
        if (T == 0 || batch == 0) return ISAM_OK;
        if (!dB || !dC) return fail(ISAM_ERR_INVALID_ARG, "%s: dB or dC is NULL", who);
        RowsArg sums[] = {{"dB", dB, dB_stride_t, dB_stride_b, N, true}, {"dC", dC, dC_stride_t, dC_stride_b, N, true}};
        const Tensor none[] = {{"workspace", nullptr, 0, true}};
        if ((st = rows_check(sums, none, T, batch, dsize(type), who)) != ISAM_OK) return st;
        ScanArgs a{};
        a.T = T;
        a.batch = batch;
        a.N = N;
        a.type = type;
        a.dB = rows_of(sums[0]);
        a.dC = rows_of(sums[1]);
        const hipError_t e = launch_scan_backward(a, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
    }
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
                            {"states", states, (size_t)cdiv(T, scan_chunk(N)) * state, false},
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

// ---------------------------------------------------------------------------
// Causal convolution
// ---------------------------------------------------------------------------
namespace {

// (a lane's place in its row is kept in 32 bits)
bool conv_sizes(int64_t T, int64_t batch, int64_t C, int type) {
    return C <= ((int64_t)1 << 32) / (int64_t)dsize(type) && T < ((int64_t)1 << 40) && batch < ((int64_t)1 << 31) && C < ((int64_t)1 << 31) &&
           (__int128)std::max<int64_t>(T, 1) * std::max<int64_t>(batch, 1) * std::max<int64_t>(C, 1) < ((__int128)1 << 42);
}

isam_status_t conv_check(int64_t T, int64_t batch, int64_t C, int64_t K, int type, int act, const char* who) {
    if (T < 0 || batch < 0 || C < 0 || K <= 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size T=%lld batch=%lld C=%lld K=%lld", who, (long long)T, (long long)batch, (long long)C, (long long)K);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (act != ISAM_ACT_NONE && act != ISAM_ACT_SILU)
        return fail(ISAM_ERR_INVALID_ARG, "%s: activation must be ISAM_ACT_NONE or ISAM_ACT_SILU", who);
    if (K > kConvMaxK || !conv_sizes(T, batch, C, type))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: K=%lld above %lld, or sizes too large (a row: 2^32 bytes)", who, (long long)K, (long long)kConvMaxK);
    return ISAM_OK;
}

ConvArgs conv_args(int64_t T, int64_t batch, int64_t C, int64_t K, int type, int act, bool packed) {
    ConvArgs a{};
    a.T = T;
    a.batch = batch;
    a.C = C;
    a.K = K;
    a.type = type;
    a.act = act == ISAM_ACT_SILU;
    a.packed = packed;
    conv_plan(a, device_cus());
    return a;
}

size_t conv_part_bytes(const ConvArgs& a) { return (size_t)(a.rows * (a.K + 1) * a.C) * sizeof(float); }

}  // namespace

extern "C" isam_status_t isam_causal_conv(int64_t T, int64_t batch, int64_t C, int64_t K, int type, int act, const void* x,
                                          int64_t x_stride_t, int64_t x_stride_b, const float* w, const float* bias,
                                          const void* state, const uint8_t* reset, int64_t reset_stride_t,
                                          int64_t reset_stride_b, void* y, int64_t y_stride_t, int64_t y_stride_b,
                                          void* state_T, void* stream) {
    clear_error();
    const char* who = "isam_causal_conv";
    isam_status_t st = conv_check(T, batch, C, K, type, act, who);
    if (st != ISAM_OK || batch == 0 || C == 0) return st;
    if (T > 0 && (!x || !w)) return fail(ISAM_ERR_INVALID_ARG, "%s: x or w is NULL", who);
    if (!y && !state_T && T > 0 && K > 1) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    const size_t es = dsize(type), kept = (size_t)((K - 1) * batch * C) * es;
    RowsArg r[] = {{"x", x, x_stride_t, x_stride_b, C, false}, {"y", y, y_stride_t, y_stride_b, C, true}};
    size_t reset_b;
    if ((st = reset_check(reset, T, &reset_stride_t, batch, &reset_stride_b, &reset_b, who)) != ISAM_OK) return st;
    // (a few tokens: the state may be replaced in place, one thread reads a channel's before it writes it)
    const bool in_place = state_T && state_T == state && T <= kConvFew;
    const Tensor dense[] = {{"w", w, (size_t)(K * C) * 4, false},      {"bias", bias, (size_t)C * 4, false},
                            {"state", in_place ? nullptr : state, kept, false}, {"reset", reset, reset_b, false},
                            {"state_T", state_T, kept, true}};
    if ((st = rows_check(r, dense, T, batch, es, who)) != ISAM_OK) return st;
    ConvArgs a = conv_args(T, batch, C, K, type, act, conv_packs(rows_of(r[0]), C, type) && conv_packs(rows_of(r[1]), C, type));
    a.x = rows_of(r[0]);
    a.y = rows_of(r[1]);
    a.w = w;
    a.bias = bias;
    a.state = state;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.state_T = K > 1 ? state_T : nullptr;
    const hipError_t e = launch_causal_conv(a, false, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" isam_status_t isam_causal_conv_backward(int64_t T, int64_t batch, int64_t C, int64_t K, int type, int act, const void* x,
                                                   int64_t x_stride_t, int64_t x_stride_b, const float* w, const float* bias,
                                                   const void* state, const uint8_t* reset, int64_t reset_stride_t,
                                                   int64_t reset_stride_b, const void* dy, int64_t dy_stride_t,
                                                   int64_t dy_stride_b, const void* dstate_T, void* dx, int64_t dx_stride_t,
                                                   int64_t dx_stride_b, void* dstate, float* dw, float* dbias,
                                                   void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_causal_conv_backward";
    isam_status_t st = conv_check(T, batch, C, K, type, act, who);
    if (st != ISAM_OK || C == 0) return st;
    const bool work = T > 0 && batch > 0;
    if (work && (!x || !w)) return fail(ISAM_ERR_INVALID_ARG, "%s: x or w is NULL", who);
    if (work && !dx && !dstate && !dw && !dbias) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    const size_t es = dsize(type), kept = (size_t)((K - 1) * batch * C) * es;
    RowsArg r[] = {{"x", x, x_stride_t, x_stride_b, C, false},
                   {"dy", dy, dy_stride_t, dy_stride_b, C, false},
                   {"dx", dx, dx_stride_t, dx_stride_b, C, true}};
    bool packed = true;
    for (const RowsArg& v : r) packed = packed && conv_packs(ScanRows{v.p, 0, batch > 1 ? v.sb : 0}, C, type);
    ConvArgs a = conv_args(T, batch, C, K, type, act, packed);
    const size_t need = work && (dw || dbias) ? conv_part_bytes(a) : 0;
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    size_t reset_b;
    if ((st = reset_check(reset, T, &reset_stride_t, batch, &reset_stride_b, &reset_b, who)) != ISAM_OK) return st;
    const Tensor dense[] = {{"w", w, (size_t)(K * C) * 4, false},  {"bias", bias, (size_t)C * 4, false},
                            {"state", state, kept, false},         {"reset", reset, reset_b, false},
                            {"dstate_T", dstate_T, kept, false},   {"dstate", dstate, kept, true},
                            {"dw", dw, (size_t)(K * C) * 4, true}, {"dbias", dbias, (size_t)C * 4, true},
                            {"workspace", workspace, room(need), true}};
    if ((st = rows_check(r, dense, T, batch, es, who)) != ISAM_OK) return st;
    a.x = rows_of(r[0]);
    a.dy = rows_of(r[1]);
    a.dx = rows_of(r[2]);
    a.w = w;
    a.bias = bias;
    a.state = state;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.dstate_T = dstate_T;
    a.dstate = K > 1 ? dstate : nullptr;
    a.dw = dw;
    a.dbias = dbias;
    a.part = reinterpret_cast<float*>(room_start(workspace));
    const hipError_t e = launch_causal_conv(a, true, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_causal_conv_backward_workspace_size(int64_t T, int64_t batch, int64_t C, int64_t K, int type) {
    if (T <= 0 || batch <= 0 || C <= 0 || K <= 0 || K > kConvMaxK || !valid_dtype(type) || !conv_sizes(T, batch, C, type)) return 0;
    // (the rows' strides decide whether a wave has several sequences, and that how long its runs are)
    return room(std::max(conv_part_bytes(conv_args(T, batch, C, K, type, ISAM_ACT_NONE, true)),
                         conv_part_bytes(conv_args(T, batch, C, K, type, ISAM_ACT_NONE, false))));
}

// ---------------------------------------------------------------------------
// Beam search
// ---------------------------------------------------------------------------
namespace {

isam_status_t beam_check(int64_t batch, int64_t beams, int64_t V, int64_t width, const char* who) {
    if (batch < 0 || beams <= 0 || V <= 0 || width <= 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size batch=%lld beams=%lld V=%lld width=%lld", who, (long long)batch, (long long)beams, (long long)V, (long long)width);
    if (beams > kBeamMax || width > kBeamMax)
        return fail(ISAM_ERR_UNSUPPORTED, "%s: beams=%lld or width=%lld above %lld", who, (long long)beams, (long long)width, (long long)kBeamMax);
    if (V > INT32_MAX / beams || batch > ((int64_t)1 << 40) / (beams * V))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: beams x V passes 2^31, or sizes too large", who);
    if (width > beams * V) return fail(ISAM_ERR_INVALID_ARG, "%s: width=%lld above the %lld candidates", who, (long long)width, (long long)(beams * V));
    return ISAM_OK;
}

size_t beam_bytes(int64_t batch, int64_t beams, int64_t V, int64_t width) {
    return (size_t)(batch * beams * cdiv(V, kBeamPart)) * (16 + 8 * (size_t)width);
}

}  // namespace

extern "C" isam_status_t isam_beam_step(int64_t batch, int64_t beams, int64_t V, int64_t width, int type, const void* logits,
                                        int64_t logits_stride_b, int64_t logits_stride_n, const float* scores,
                                        const uint8_t* finished, int64_t end, float* scores_out, int32_t* parent,
                                        int32_t* token, uint8_t* finished_out, void* workspace, size_t workspace_bytes,
                                        void* stream) {
    clear_error();
    const char* who = "isam_beam_step";
    isam_status_t st = beam_check(batch, beams, V, width, who);
    if (st != ISAM_OK) return st;
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (end >= V) return fail(ISAM_ERR_INVALID_ARG, "%s: end=%lld is not below V=%lld", who, (long long)end, (long long)V);
    if (finished && end < 0) return fail(ISAM_ERR_INVALID_ARG, "%s: finished needs an end token", who);
    if (batch == 0) return ISAM_OK;
    if (!logits || !scores || !scores_out || !parent || !token)
        return fail(ISAM_ERR_INVALID_ARG, "%s: logits, scores, scores_out, parent or token is NULL", who);
    if (logits_stride_b < 0 || logits_stride_n < 0) return fail(ISAM_ERR_INVALID_ARG, "%s: negative stride", who);
    const size_t es = dsize(type), need = beam_bytes(batch, beams, V, width);
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    size_t lg_b;
    if (!extent(batch, logits_stride_b, beams, logits_stride_n, V, es, &lg_b))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: logits span more than 2^46 bytes", who);
    const size_t in = (size_t)(batch * beams), out = (size_t)(batch * width);
    const Tensor all[] = {{"logits", logits, lg_b, false},       {"scores", scores, in * 4, false},
                          {"finished", finished, in, false},     {"scores_out", scores_out, out * 4, true},
                          {"parent", parent, out * 4, true},     {"token", token, out * 4, true},
                          {"finished_out", finished_out, out, true}, {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    BeamArgs a{};
    a.batch = batch;
    a.beams = beams;
    a.V = V;
    a.width = width;
    a.type = type;
    a.logits = logits;
    a.lg_b = logits_stride_b;
    a.lg_n = logits_stride_n;
    a.scores = scores;
    a.finished = finished;
    a.end = end;
    a.scores_out = scores_out;
    a.parent = parent;
    a.token = token;
    a.finished_out = finished_out;
    a.parts = cdiv(V, kBeamPart);
    a.sums = reinterpret_cast<double2*>(room_start(workspace));
    a.best = reinterpret_cast<uint64_t*>(a.sums + batch * beams * a.parts);
    const hipError_t e = launch_beam_step(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_beam_step_workspace_size(int64_t batch, int64_t beams, int64_t V, int64_t width, int type) {
    if (batch <= 0 || !valid_dtype(type) || beams <= 0 || V <= 0 || width <= 0 || beams > kBeamMax || width > kBeamMax ||
        V > INT32_MAX / beams || batch > ((int64_t)1 << 40) / (beams * V))
        return 0;
    return room(beam_bytes(batch, beams, V, width));
}

extern "C" isam_status_t isam_beam_reorder(int64_t outer, int64_t batch, int64_t beams, int64_t width, int64_t row_bytes,
                                           const void* src, const int32_t* parent, void* dst, void* stream) {
    clear_error();
    const char* who = "isam_beam_reorder";
    if (outer < 0 || batch < 0 || beams <= 0 || width <= 0 || row_bytes < 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size outer=%lld batch=%lld beams=%lld width=%lld row_bytes=%lld", who, (long long)outer,
                    (long long)batch, (long long)beams, (long long)width, (long long)row_bytes);
    if (outer == 0 || batch == 0 || row_bytes == 0) return ISAM_OK;
    if (!src || !parent || !dst) return fail(ISAM_ERR_INVALID_ARG, "%s: src, parent or dst is NULL", who);
    size_t in, out;
    const int64_t lim = (int64_t)1 << 40;
    if (outer > lim || batch > lim || beams > lim || width > lim || row_bytes > lim ||
        (__int128)batch * std::max(beams, width) > lim || !extent(outer, batch * beams * row_bytes, 1, 0, batch * beams * row_bytes, 1, &in) ||
        !extent(outer, batch * width * row_bytes, 1, 0, batch * width * row_bytes, 1, &out))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: sizes too large", who);
    const Tensor all[] = {{"src", src, in, false}, {"parent", parent, (size_t)(batch * width) * 4, false}, {"dst", dst, out, true}};
    const isam_status_t st = disjoint(all, who);
    if (st != ISAM_OK) return st;
    const ReorderArgs a{outer, batch, beams, width, row_bytes, src, parent, dst};
    const hipError_t e = launch_beam_reorder(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

// ---------------------------------------------------------------------------
// Projection with its epilogue
// ---------------------------------------------------------------------------
namespace {

enum LinearWay { kLinearTokens, kLinearTiles, kLinearF32, kLinearProduct, kLinearDirect };

// Parts of the workspace, in order: copies of x (twice for the terms), W and dout with aligned rows, P or dP, the bias
// gradient's partial sums, the terms' dx, and what the matrix products use.
struct LinearPlan {
    LinearWay way;
    int tile;
    int64_t Kp, ld_pre, bias_rows;
    bool copy_x, copy_w, copy_d;
    size_t x_b, w_b, d_b, pre_b, bias_b, join_b, gemm_b;
    size_t total() const { return x_b + w_b + d_b + pre_b + bias_b + join_b + gemm_b; }
};

int64_t round8(int64_t v) { return cdiv(v, 8) * 8; }

void linear_copies(LinearPlan& p, int64_t M, int64_t K, int64_t N) {
    p.Kp = K;
    if (p.copy_x || p.copy_w) {
        // whole 64-deep tiles where that adds at most an eighth and both are copied (no range checks in the kernel)
        const int64_t K64 = cdiv(K, 64) * 64;
        p.Kp = p.copy_x && p.copy_w && (K64 - K) * 8 <= K ? K64 : round8(K);
    }
    if (p.copy_x) p.x_b = align256((size_t)(M * p.Kp) * 2);
    if (p.copy_w) p.w_b = align256((size_t)(N * p.Kp) * 2);
}

// Whether the kernel for a few rows takes them: always up to 16, and up to 64 where its work, in units of 16 rows of x
// and 1024 values of K to a round of its workgroups (16 columns each), is small.  It takes some 6 us and 1 (bf16) or 2.2
// (fp32) for each unit, the tiles (their copies of unaligned rows included) and the product with its pass, us of 17, 32, 64
// rows against it, gelu: bf16 1024x4096 (K x N) 11.4, 11.3, 11.5 against 7.2, 7.1, 8.4; 4096x1024 21.9, 21.6, 21.7 against
// 10.7, 13.6, 21.5; 4096x16384 36, 35, 36 against 41, 53, 84; fp32 1024x4096 18.5, 19.1, 18.9 against 9.3, 9.6, 15.4;
// 4096x1024 21, 24, 23 against 24, 27, 49.  Unaligned: bf16 6683x3905 57, 57, 57 against 37, 51, 83; fp32 92, 92, 91 against
// 44, 57, 90.
bool linear_few(int64_t M, int64_t K, int64_t N, bool aligned) {
    if (M <= kGatedTokens) return true;
    const int64_t rounds = cdiv(N, 16 * (int64_t)device_cus());
    return M <= kLinearFew && (__int128)M * K * rounds <= (aligned ? 4 : 16) * 16 * 1024;
}

// Whether the bf16 tiles would be too few and too deep: the product in slices of K and a pass take less than one round
// of 64 x 64 tiles, whose copies' latency costs 3.5 us for 1024 of K.  us of 64, 128, 256, 512 rows, tiles / product
// and pass, gelu: 2048x2048 (K x N) 15, 15, 15, 16 / 16, 17, 19, 21; 4096x1024 22, 22, 22, 23 / 18, 18, 20, 23; 4096x4096
// 24, 24, 26, 35 / 21, 24, 30, 38; 8192x2048 38, 38, 38, 40 / 23, 23, 32, 41; 16384x512 64, 64, 65, 64 / 24, 24, 27, 33.
bool linear_deep(int64_t M, int64_t K, int64_t N) { return K >= 4096 && 2 * cdiv(M, 64) * cdiv(N, 64) <= (int64_t)device_cus(); }

// fp32 grids of few tiles take linear_f32_kernel by the gated block's rule, up to 24 rounds of 64 values of K.  us of the
// product and pass / the kernel, silu, forward (rounds): 128x512x2048 17.5 / 10.2 (8), 100x333x5001 23.4 / 14.9 (12),
// 256x1024x1024 20.7 / 15.6 and 512x1024x1024 26.6 / 15.9 (16), 1000x768x1000 29.1 / 22.9 and 128x1536x2048 23.1 / 20.8 (24),
// 512x512x4096 30.2 / 31.9, 512x1024x2048 31.0 / 28.5, 128x2048x2048 26.2 / 25.9 and 1000x1000x1000 32.9 / 25.2 (32),
// 512x2048x2048 45 / 50 and 2048x512x2048 51 / 62 (64); whole gradients lie alike.  The bf16 tiles are chosen by that
// block's rounds too: 64 / 128 / 256 rows, us:
// 256x2048x2048 12.4 / 20.4 / 38.8, 576x256x4096 11.0 / 8.3 / 14.0, 1024x1024x8192 41 / 23.5 / 30.6, 1792x1024x8192 68 / 40 / 35.3,
// 2048x1024x8192 75 / 42.7 / 37.7, 2304x1024x8192 84 / 51.6 / 59, 2944x1024x8192 106 / 60.3 / 63.2, 3328x1024x8192 120 / 69.3 / 65.0.
//
// Forward.  plain: no activation, and no residual but out itself: the library's product has that epilogue in every
// one of its plans.
LinearPlan linear_forward_plan(int64_t M, int64_t K, int64_t N, int type, bool plain, bool x_ok, bool w_ok) {
    LinearPlan p{};
    const bool aligned = x_ok && w_ok && K % 8 == 0;
    if (linear_few(M, K, N, aligned)) {
        p.way = kLinearTokens;
    } else if (type == ISAM_F32 && gated_f32_direct(M, K, cdiv(N, 2), device_cus())) {
        p.way = kLinearF32;
    } else if (plain && (type == ISAM_F32 || (x_ok && w_ok))) {
        p.way = kLinearDirect;
        p.gemm_b = align256(product_workspace(0, 1, M, N, K, type));
    } else if (type == ISAM_BF16 && !(aligned && linear_deep(M, K, N))) {
        p.way = kLinearTiles;
        p.copy_x = !x_ok || K % 8;
        p.copy_w = !w_ok || K % 8;
        linear_copies(p, M, K, N);
        p.tile = gated_tile(M, cdiv(N, 2), device_cus());
    } else {
        p.way = kLinearProduct;
        p.ld_pre = N;
        p.pre_b = align256((size_t)(M * N) * sizeof(float));
        p.gemm_b = align256(product_workspace(0, 1, M, N, K, type));
    }
    return p;
}

// Gradient.  act: there is an activation, P is formed again and dP stands in the workspace; without one dP is dout.
LinearPlan linear_backward_plan(int64_t M, int64_t K, int64_t N, int type, bool act, bool x_ok, bool w_ok, bool d_ok) {
    LinearPlan p{};
    const size_t es = dsize(type);
    if (M == 0) {  // (zeros in dW and dbias; nothing is copied, formed or summed)
        p.way = kLinearDirect;
        return p;
    }
    p.gemm_b = std::max(product_workspace(0, 0, M, K, N, type), product_workspace(1, 0, N, K, M, type));
    p.Kp = K;
    p.ld_pre = round8(N);
    if (!act) {
        p.way = kLinearDirect;
        if (type == ISAM_BF16) {  // (rows off 16 bytes by size alone are the products' own matter)
            p.copy_x = !x_ok && K % 8 == 0;
            p.copy_w = !w_ok && K % 8 == 0;
            p.copy_d = !d_ok && N % 8 == 0;
            if (p.copy_x) p.x_b = align256((size_t)(M * K) * es);
            if (p.copy_w) p.w_b = align256((size_t)(N * K) * es);
            if (p.copy_d) p.d_b = align256((size_t)(M * N) * es);
        }
        p.bias_rows = cdiv(M, kLinearRows);
    } else if (type == ISAM_BF16 && M <= kGatedTokens && (__int128)2 * M * p.ld_pre * 2 <= kMaxExtent &&
               (__int128)2 * M * (K + 8) * 4 <= kMaxExtent) {
        p.way = kLinearTokens;  // dP in two bf16 terms, 2 M rows
        p.Kp = round8(K);
        p.x_b = align256((size_t)(2 * M * p.Kp) * es);
        p.pre_b = align256((size_t)(2 * M * p.ld_pre) * es);
        p.bias_rows = 1;
        p.join_b = align256((size_t)(2 * M * K) * sizeof(float));
        p.gemm_b = std::max(product_workspace(0, 0, 2 * M, K, N, type), product_workspace(1, 0, N, K, 2 * M, type));
    } else if (type == ISAM_BF16) {
        p.way = kLinearTiles;
        p.copy_x = !x_ok || K % 8;
        p.copy_w = !w_ok || K % 8;
        linear_copies(p, M, K, N);
        p.tile = gated_tile(M, cdiv(N, 2), device_cus());
        p.bias_rows = gated_bias_rows(p.tile, M);
        p.pre_b = align256((size_t)(M * p.ld_pre) * es);
    } else if (gated_f32_direct(M, K, cdiv(N, 2), device_cus())) {
        p.way = kLinearF32;
        p.bias_rows = cdiv(M, 32) * 2;
        p.pre_b = align256((size_t)(M * p.ld_pre) * es);
    } else {
        p.way = kLinearProduct;
        p.bias_rows = cdiv(M, kLinearRows);
        p.ld_pre = N;
        p.pre_b = align256((size_t)(M * N) * es);
        p.gemm_b = std::max(p.gemm_b, product_workspace(0, 1, M, N, K, type));
    }
    p.bias_b = align256((size_t)(p.bias_rows * N) * sizeof(float));
    p.gemm_b = align256(p.gemm_b);
    return p;
}

isam_status_t linear_check(int64_t M, int64_t K, int64_t N, int type, int act, const char* who) {
    if (M < 0 || K <= 0 || N < 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size M=%lld K=%lld N=%lld", who, (long long)M, (long long)K, (long long)N);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (act < ISAM_ACT_SIGMOID || act > ISAM_ACT_NONE)
        return fail(ISAM_ERR_INVALID_ARG, "%s: activation must be 0 (sigmoid), 1 (silu), 2 (gelu) or 3 (none)", who);
    return ISAM_OK;
}

// Sizes for which every buffer a plan adds stays below 2^31 bytes as well.
bool linear_sizes(int64_t M, int64_t K, int64_t N, int type) {
    const __int128 es = (__int128)dsize(type), most = kMaxExtent, Kp = (__int128)K + 64, Np = (__int128)N + 8;
    return (__int128)M * Np * es <= most && (__int128)M * Kp * es <= most && Np * Kp * es <= most;
}

// The copies of the plan, and the operands then read.
hipError_t linear_copy(const LinearPlan& p, char* ws, LinearArgs& a, hipStream_t s) {
    if (!p.copy_x && !p.copy_w) return hipSuccess;
    PackRows cx{}, cw{};
    if (p.copy_x) cx = PackRows{static_cast<const uint16_t*>(a.x), a.M, a.K, a.ld_x, reinterpret_cast<uint16_t*>(ws), p.Kp};
    if (p.copy_w) cw = PackRows{static_cast<const uint16_t*>(a.W), a.N, a.K, a.ld_w, reinterpret_cast<uint16_t*>(ws + p.x_b), p.Kp};
    const hipError_t e = launch_pack_rows(cx, cw, device_cus(), s);
    if (e != hipSuccess) return e;
    if (p.copy_x) {
        a.x = cx.dst;
        a.ld_x = p.Kp;
    }
    if (p.copy_w) {
        a.W = cw.dst;
        a.ld_w = p.Kp;
    }
    return hipSuccess;
}

}  // namespace

extern "C" isam_status_t isam_linear(int64_t M, int64_t K, int64_t N, int type, int act, const void* x, int64_t ldx, const void* W,
                                     int64_t ldw, const float* bias, const void* residual, int64_t ldr, void* out, int64_t ldo,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_linear";
    isam_status_t st = linear_check(M, K, N, type, act, who);
    if (st != ISAM_OK || M == 0 || N == 0) return st;
    if (!x || !W || !out) return fail(ISAM_ERR_INVALID_ARG, "%s: x, W or out is NULL", who);
    const size_t es = dsize(type);
    size_t x_b, w_b, r_b, o_b;
    if ((st = small_matrix("x", x, M, K, ldx, es, &x_b, who)) != ISAM_OK ||
        (st = small_matrix("W", W, N, K, ldw, es, &w_b, who)) != ISAM_OK ||
        (st = small_matrix("residual", residual, M, N, ldr, es, &r_b, who)) != ISAM_OK ||
        (st = small_matrix("out", out, M, N, ldo, es, &o_b, who)) != ISAM_OK)
        return st;
    if (!linear_sizes(M, K, N, type)) return fail(ISAM_ERR_UNSUPPORTED, "%s: M x N, M x K or N x K passes 2^31 bytes", who);
    const bool in_place = residual == out && (ldr == ldo || M == 1);
    const LinearPlan p = linear_forward_plan(M, K, N, type, act == ISAM_ACT_NONE && (!residual || in_place), rows_aligned(x, ldx),
                                             rows_aligned(W, ldw));
    const size_t need = p.total();
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    const Tensor all[] = {{"x", x, x_b, false},
                          {"W", W, w_b, false},
                          {"bias", bias, (size_t)N * 4, false},
                          {"residual", in_place ? nullptr : residual, r_b, false},
                          {"out", out, o_b, true},
                          {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* const ws = room_start(workspace);
    if (p.way == kLinearDirect)
        return product(0, 1, M, N, K, type, x, ldx, W, ldw, type, out, ldo, ws, p.gemm_b, s, who, residual ? 1 : 0, bias);
    LinearArgs a{};
    a.M = M;
    a.K = K;
    a.N = N;
    a.act = act;
    a.x = x;
    a.W = W;
    a.bias = bias;
    a.ld_x = ldx;
    a.ld_w = ldw;
    a.side = residual;
    a.ld_side = ldr;
    a.out = out;
    a.ld_out = ldo;
    hipError_t e;
    if (p.way == kLinearTokens) {
        e = launch_linear_tokens(a, type, false, s);
    } else if (p.way == kLinearF32) {
        e = launch_linear_f32(a, false, s);
    } else if (p.way == kLinearTiles) {
        e = linear_copy(p, ws, a, s);
        a.K = p.Kp;
        if (e == hipSuccess) e = launch_linear_tiles(a, p.tile, false, s);
    } else {
        float* const pre = reinterpret_cast<float*>(ws);
        st = product(0, 1, M, N, K, type, x, ldx, W, ldw, ISAM_F32, pre, N, ws + p.pre_b, p.gemm_b, s, who);
        if (st != ISAM_OK) return st;
        a.pre = pre;
        a.ld_pre = N;
        e = launch_linear_pass(a, type, false, s);
    }
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_linear_workspace_size(int64_t M, int64_t K, int64_t N, int type, int aligned) {
    if (M <= 0 || K <= 0 || N <= 0 || !valid_dtype(type) || !linear_sizes(M, K, N, type)) return 0;
    size_t most = 0;
    for (const bool plain : {false, true}) {
        most = std::max(most, linear_forward_plan(M, K, N, type, plain, true, true).total());
        if (!aligned) most = std::max(most, linear_forward_plan(M, K, N, type, plain, false, false).total());
    }
    return room(most);
}

extern "C" isam_status_t isam_linear_backward(int64_t M, int64_t K, int64_t N, int type, int act, const void* x, int64_t ldx,
                                              const void* W, int64_t ldw, const float* bias, const void* dout, int64_t lddo, void* dx,
                                              int64_t lddx, void* dW, int64_t lddw, float* dbias, void* workspace,
                                              size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_linear_backward";
    isam_status_t st = linear_check(M, K, N, type, act, who);
    if (st != ISAM_OK) return st;
    if (N == 0 && M > 0 && dx) return fail(ISAM_ERR_INVALID_ARG, "%s: N is 0", who);
    if (N == 0) return ISAM_OK;
    if (!dx && !dW && !dbias) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    if (M > 0 && (!x || !W || !dout)) return fail(ISAM_ERR_INVALID_ARG, "%s: x, W or dout is NULL", who);
    const size_t es = dsize(type);
    size_t x_b, w_b, do_b, dx_b, dw_b;
    if ((st = small_matrix("x", x, M, K, ldx, es, &x_b, who)) != ISAM_OK ||
        (st = small_matrix("W", W, N, K, ldw, es, &w_b, who)) != ISAM_OK ||
        (st = small_matrix("dout", dout, M, N, lddo, es, &do_b, who)) != ISAM_OK ||
        (st = small_matrix("dx", dx, M, K, lddx, es, &dx_b, who)) != ISAM_OK ||
        (st = small_matrix("dW", dW, N, K, lddw, es, &dw_b, who)) != ISAM_OK)
        return st;
    if (!linear_sizes(M, K, N, type)) return fail(ISAM_ERR_UNSUPPORTED, "%s: M x N, M x K or N x K passes 2^31 bytes", who);
    const LinearPlan p = linear_backward_plan(M, K, N, type, act != ISAM_ACT_NONE, rows_aligned(x, ldx), rows_aligned(W, ldw),
                                              rows_aligned(dout, lddo));
    const size_t need = p.total();
    if ((st = need_room(need, workspace, workspace_bytes, who)) != ISAM_OK) return st;
    const size_t b_b = (size_t)N * 4;
    const Tensor all[] = {{"x", x, x_b, false},       {"W", W, w_b, false},   {"bias", bias, b_b, false},
                          {"dout", dout, do_b, false}, {"dx", dx, dx_b, true}, {"dW", dW, dw_b, true},
                          {"dbias", dbias, b_b, true}, {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* const ws = room_start(workspace);
    char* const copy_d = ws + p.x_b + p.w_b;
    char* const pre = copy_d + p.d_b;
    float* const bias_part = reinterpret_cast<float*>(pre + p.pre_b);
    float* const join = reinterpret_cast<float*>(pre + p.pre_b + p.bias_b);
    char* const gemm_ws = pre + p.pre_b + p.bias_b + p.join_b;
    const void* dP = dout;
    int64_t ld_dP = lddo;
    LinearArgs a{};
    hipError_t e = hipSuccess;
    if (M > 0) {
        a.M = M;
        a.K = K;
        a.N = N;
        a.act = act;
        a.x = x;
        a.W = W;
        a.bias = bias;
        a.ld_x = ldx;
        a.ld_w = ldw;
        a.side = dout;
        a.ld_side = lddo;
        a.out = pre;
        a.ld_out = p.ld_pre;
        a.bias_part = dbias ? bias_part : nullptr;
        if ((e = linear_copy(p, ws, a, s)) != hipSuccess) return hip_fail(e, who);
        if (p.way != kLinearDirect) {
            dP = pre;
            ld_dP = p.ld_pre;
        }
        if (p.way == kLinearTokens) {
            e = launch_linear_tokens(a, type, true, s);
            if (e == hipSuccess && dW) {
                const PackRows x1{static_cast<const uint16_t*>(x), M, K, ldx, reinterpret_cast<uint16_t*>(ws), p.Kp};
                PackRows x2 = x1;
                x2.dst += M * p.Kp;
                e = launch_pack_rows(x1, x2, device_cus(), s);
            }
        } else if (p.way == kLinearTiles) {
            LinearArgs t = a;
            t.K = p.Kp;
            e = launch_linear_tiles(t, p.tile, true, s);
        } else if (p.way == kLinearF32) {
            e = launch_linear_f32(a, true, s);
        } else if (p.way == kLinearProduct) {
            st = product(0, 1, M, N, K, type, x, ldx, W, ldw, ISAM_F32, pre, N, gemm_ws, p.gemm_b, s, who);
            if (st != ISAM_OK) return st;
            a.pre = reinterpret_cast<const float*>(pre);
            a.ld_pre = N;
            e = launch_linear_pass(a, type, true, s);
        } else {
            if (p.copy_d) {
                const PackRows cd{static_cast<const uint16_t*>(dout), M, N, lddo, reinterpret_cast<uint16_t*>(copy_d), N};
                e = launch_pack_rows(cd, PackRows{}, device_cus(), s);
                dP = copy_d;
                ld_dP = N;
            }
            if (e == hipSuccess && dbias) e = launch_linear_pass(a, type, true, s);  // (column sums of dout)
        }
        if (e != hipSuccess) return hip_fail(e, who);
        if (p.way == kLinearTokens) {  // both terms' rows in one product, then their sum
            if (dx) {
                st = product(0, 0, 2 * M, K, N, type, dP, ld_dP, W, ldw, ISAM_F32, join, K, gemm_ws, p.gemm_b, s, who);
                if (st != ISAM_OK) return st;
                GatedArgs sum{};
                sum.M = M;
                sum.K = K;
                sum.gu = join;
                sum.out = dx;
                sum.ld_out = lddx;
                if ((e = launch_gated_join(sum, s)) != hipSuccess) return hip_fail(e, who);
            }
            if (dW) st = product(1, 0, N, K, 2 * M, type, dP, ld_dP, ws, p.Kp, type, dW, lddw, gemm_ws, p.gemm_b, s, who);
            if (st != ISAM_OK) return st;
            dx = dW = nullptr;
        }
        if (dx && (st = product(0, 0, M, K, N, type, dP, ld_dP, a.W, a.ld_w, type, dx, lddx, gemm_ws, p.gemm_b, s, who)) != ISAM_OK) return st;
    }
    if (dW && (st = product(1, 0, N, K, M, type, dP, M ? ld_dP : N, a.x, M ? a.ld_x : K, type, dW, lddw, gemm_ws, p.gemm_b, s, who)) != ISAM_OK)
        return st;
    if (dbias) {
        const ColSum sum{bias_part, dbias, M ? p.bias_rows : 0, N, 1, kF32};
        e = launch_colsum(&sum, 1, s);
    }
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_linear_backward_workspace_size(int64_t M, int64_t K, int64_t N, int type, int aligned) {
    if (M <= 0 || K <= 0 || N <= 0 || !valid_dtype(type) || !linear_sizes(M, K, N, type)) return 0;
    const bool ok = aligned != 0;
    size_t most = 0;
    for (const bool act : {false, true}) most = std::max(most, linear_backward_plan(M, K, N, type, act, ok, ok, ok).total());
    return room(most);
}
