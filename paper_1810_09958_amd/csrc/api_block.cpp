// C-ABI layer of the operators of a gated recurrent block: argument validation
// (pure host code, no HIP call) and dispatch.
#include <algorithm>

#include "api.hpp"

using namespace isam;
using namespace isam::api;

namespace {

// Workspaces start at the first multiple of 256 bytes of what the caller gives.
size_t room(size_t bytes) { return bytes ? bytes + 255 : 0; }
char* room_start(void* ws) { return reinterpret_cast<char*>(((uintptr_t)ws + 255) & ~(uintptr_t)255); }

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
bool extent(int64_t n, int64_t stride_n, int64_t m, int64_t stride_m, int64_t width, size_t es, size_t* bytes) {
    *bytes = 0;
    if (n == 0 || m == 0 || width == 0) return true;
    const __int128 e = ((__int128)(n - 1) * stride_n + (__int128)(m - 1) * stride_m + width) * (__int128)es;
    if (e > ((__int128)1 << 46)) return false;
    *bytes = (size_t)e;
    return true;
}

// Whether no two rows (i, j) of `width` elements share an element.
bool rows_apart(int64_t n, int64_t stride_n, int64_t m, int64_t stride_m, int64_t width) {
    const bool inner_m = m <= 1 || stride_m >= width, inner_n = n <= 1 || stride_n >= width;
    return (inner_m && (n <= 1 || (__int128)stride_n >= (__int128)(m - 1) * (m > 1 ? stride_m : 0) + width)) ||
           (inner_n && (m <= 1 || (__int128)stride_m >= (__int128)(n - 1) * (n > 1 ? stride_n : 0) + width));
}

// ---------------------------------------------------------------------------
// Linear GRU
// ---------------------------------------------------------------------------
// Sizes whose products stay far below 2^63 (states, partial sums and grids).
bool lingru_sizes(int64_t T, int64_t batch, int64_t H) {
    return T < ((int64_t)1 << 40) && batch < ((int64_t)1 << 31) && H < ((int64_t)1 << 31) &&
           (__int128)T * batch * H < ((__int128)1 << 46);
}

// Bytes of the bias gradient's partial sums, one row per tile of time and sequence.
size_t lingru_bias_bytes(int64_t T, int64_t batch, int64_t H) {
    return (size_t)(lingru_tiles(T, true) * batch * 2 * H) * sizeof(float);
}

isam_status_t lingru_check(int64_t T, int64_t batch, int64_t H, int type, int candidate, const char* who) {
    if (T < 0 || batch < 0 || H < 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: negative size T=%lld batch=%lld hidden=%lld", who, (long long)T,
                    (long long)batch, (long long)H);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (candidate != ISAM_LINEAR && candidate != ISAM_TANH)
        return fail(ISAM_ERR_INVALID_ARG, "%s: candidate must be ISAM_LINEAR (0) or ISAM_TANH (1)", who);
    if (!lingru_sizes(T, batch, H)) return fail(ISAM_ERR_UNSUPPORTED, "%s: sizes too large", who);
    return ISAM_OK;
}

}  // namespace

extern "C" isam_status_t isam_linear_gru(int64_t T, int64_t batch, int64_t hidden, int type, int candidate, const void* gx,
                                         int64_t gx_stride_t, int64_t gx_stride_b, const float* bias, const float* h0,
                                         const uint8_t* reset, int64_t reset_stride_t, int64_t reset_stride_b, void* h_seq,
                                         int64_t h_stride_t, int64_t h_stride_b, float* h_T, float* states,
                                         void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_linear_gru";
    isam_status_t st = lingru_check(T, batch, hidden, type, candidate, who);
    if (st != ISAM_OK || batch == 0 || hidden == 0) return st;
    if (!h_seq && !h_T && !states) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    if (T > 0 && !gx) return fail(ISAM_ERR_INVALID_ARG, "%s: gx is NULL", who);
    if (gx_stride_t < 0 || gx_stride_b < 0 || (h_seq && (h_stride_t < 0 || h_stride_b < 0)) ||
        (reset && (reset_stride_t < 0 || reset_stride_b < 0)))
        return fail(ISAM_ERR_INVALID_ARG, "%s: negative stride", who);
    if (h_seq && T > 0 && !rows_apart(T, h_stride_t, batch, h_stride_b, hidden))
        return fail(ISAM_ERR_INVALID_ARG, "%s: rows of h_seq overlap", who);
    const size_t es = dsize(type), state = (size_t)(batch * hidden) * sizeof(float);
    LinGruArgs a{};
    const size_t need = lingru_chain_bytes(T, batch, hidden, false);
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0,
                    room(need));
    if (T == 1) gx_stride_t = h_stride_t = reset_stride_t = 0;  // (one step: no second one to stride to)
    size_t gx_b, h_b, r_b;
    if (!extent(T, gx_stride_t, batch, gx_stride_b, 2 * hidden, es, &gx_b) ||
        !extent(h_seq ? T : 0, h_stride_t, batch, h_stride_b, hidden, es, &h_b) ||
        !extent(reset ? T : 0, reset_stride_t, batch, reset_stride_b, 1, 1, &r_b))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: a tensor spans more than 2^46 bytes", who);
    if (T > kLinGruFew && (!lingru_strides(gx_stride_t, 2 * hidden, es) || (h_seq && !lingru_strides(h_stride_t, hidden, es)) ||
                           (reset && !lingru_strides(reset_stride_t, 1, 1))))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: 32 steps of a tensor span more than 2^31 bytes", who);
    const Tensor all[] = {{"gx", gx, gx_b, false},
                          {"bias", bias, (size_t)(2 * hidden) * 4, false},
                          {"h0", h0, state, false},
                          {"reset", reset, r_b, false},
                          {"h_seq", h_seq, h_b, true},
                          {"h_T", h_T, state, true},
                          {"states", states, (size_t)cdiv(T, kLinGruChunk) * state, true},
                          {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    a.T = T;
    a.batch = batch;
    a.H = hidden;
    a.type = type;
    a.candidate = candidate;
    a.gx = gx;
    a.gx_t = gx_stride_t;
    a.gx_b = gx_stride_b;
    a.bias = bias;
    a.h0 = h0;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.h_seq = h_seq;
    a.h_t = h_stride_t;
    a.h_b = h_stride_b;
    a.h_T = h_T;
    a.states = states;
    a.chain = need ? reinterpret_cast<uint64_t*>(room_start(workspace)) : nullptr;
    const hipError_t e = launch_lingru_forward(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_linear_gru_workspace_size(int64_t T, int64_t batch, int64_t hidden, int type) {
    if (T <= 0 || batch <= 0 || hidden <= 0 || !valid_dtype(type) || !lingru_sizes(T, batch, hidden)) return 0;
    return room(lingru_chain_bytes(T, batch, hidden, false));
}

extern "C" isam_status_t isam_linear_gru_backward(int64_t T, int64_t batch, int64_t hidden, int type, int candidate,
                                                  const void* gx, int64_t gx_stride_t, int64_t gx_stride_b,
                                                  const float* bias, const uint8_t* reset, int64_t reset_stride_t,
                                                  int64_t reset_stride_b, const float* states, const void* dh_seq,
                                                  int64_t dh_stride_t, int64_t dh_stride_b, const float* dh_T, void* dgx,
                                                  int64_t dgx_stride_t, int64_t dgx_stride_b, float* dh0, float* dbias,
                                                  void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_linear_gru_backward";
    isam_status_t st = lingru_check(T, batch, hidden, type, candidate, who);
    if (st != ISAM_OK || hidden == 0) return st;
    if (T > 0 && batch > 0 && (!gx || !states || !dgx))
        return fail(ISAM_ERR_INVALID_ARG, "%s: gx, states or dgx is NULL", who);
    if (gx_stride_t < 0 || gx_stride_b < 0 || dgx_stride_t < 0 || dgx_stride_b < 0 ||
        (dh_seq && (dh_stride_t < 0 || dh_stride_b < 0)) || (reset && (reset_stride_t < 0 || reset_stride_b < 0)))
        return fail(ISAM_ERR_INVALID_ARG, "%s: negative stride", who);
    if (T > 0 && batch > 0 && !rows_apart(T, dgx_stride_t, batch, dgx_stride_b, 2 * hidden))
        return fail(ISAM_ERR_INVALID_ARG, "%s: rows of dgx overlap", who);
    const size_t es = dsize(type), state = (size_t)(batch * hidden) * sizeof(float);
    LinGruArgs a{};
    const size_t chain = align256(lingru_chain_bytes(T, batch, hidden, true));
    const size_t need = chain + (dbias ? lingru_bias_bytes(T, batch, hidden) : 0);
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0,
                    room(need));
    if (T == 1) gx_stride_t = dgx_stride_t = dh_stride_t = reset_stride_t = 0;
    size_t gx_b, dg_b, dh_b, r_b;
    if (!extent(T, gx_stride_t, batch, gx_stride_b, 2 * hidden, es, &gx_b) ||
        !extent(T, dgx_stride_t, batch, dgx_stride_b, 2 * hidden, es, &dg_b) ||
        !extent(dh_seq ? T : 0, dh_stride_t, batch, dh_stride_b, hidden, es, &dh_b) ||
        !extent(reset ? T : 0, reset_stride_t, batch, reset_stride_b, 1, 1, &r_b))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: a tensor spans more than 2^46 bytes", who);
    if (!lingru_strides(gx_stride_t, 2 * hidden, es) || !lingru_strides(dgx_stride_t, 2 * hidden, es) ||
        (dh_seq && !lingru_strides(dh_stride_t, hidden, es)) || (reset && !lingru_strides(reset_stride_t, 1, 1)))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: 32 steps of a tensor span more than 2^31 bytes", who);
    const Tensor all[] = {{"gx", gx, gx_b, false},
                          {"bias", bias, (size_t)(2 * hidden) * 4, false},
                          {"reset", reset, r_b, false},
                          {"states", states, (size_t)cdiv(T, kLinGruChunk) * state, false},
                          {"dh_seq", dh_seq, dh_b, false},
                          {"dh_T", dh_T, state, false},
                          {"dgx", dgx, dg_b, true},
                          {"dh0", dh0, state, true},
                          {"dbias", dbias, (size_t)(2 * hidden) * 4, true},
                          {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    a.T = T;
    a.batch = batch;
    a.H = hidden;
    a.type = type;
    a.candidate = candidate;
    a.gx = gx;
    a.gx_t = gx_stride_t;
    a.gx_b = gx_stride_b;
    a.bias = bias;
    a.reset = reset;
    a.rs_t = reset_stride_t;
    a.rs_b = reset_stride_b;
    a.states = const_cast<float*>(states);
    a.dh_seq = dh_seq;
    a.dh_t = dh_stride_t;
    a.dh_b = dh_stride_b;
    a.dh_T = dh_T;
    a.dgx = dgx;
    a.dg_t = dgx_stride_t;
    a.dg_b = dgx_stride_b;
    a.dh0 = dh0;
    a.dbias = dbias;
    char* ws = room_start(workspace);
    a.chain = chain ? reinterpret_cast<uint64_t*>(ws) : nullptr;
    a.bias_part = dbias ? reinterpret_cast<float*>(ws + chain) : nullptr;
    const hipError_t e = launch_lingru_backward(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_linear_gru_backward_workspace_size(int64_t T, int64_t batch, int64_t hidden, int type) {
    if (T < 0 || batch <= 0 || hidden <= 0 || !valid_dtype(type) || !lingru_sizes(T, batch, hidden)) return 0;
    return room(align256(lingru_chain_bytes(T, batch, hidden, true)) + lingru_bias_bytes(T, batch, hidden));
}

// ---------------------------------------------------------------------------
// Gated residual norm
// ---------------------------------------------------------------------------
namespace {

bool norm_sizes(int64_t rows, int64_t D) { return D <= kNormMaxD && rows < ((int64_t)1 << 40); }

isam_status_t norm_check(int64_t rows, int64_t D, int64_t* gates, int type, const void* gate, float scale, float eps,
                         const char* who) {
    if (rows < 0 || D < 0) return fail(ISAM_ERR_INVALID_ARG, "%s: negative size rows=%lld D=%lld", who, (long long)rows, (long long)D);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (!(eps >= 0.0f)) return fail(ISAM_ERR_INVALID_ARG, "%s: eps must not be negative", who);
    if (scale != scale) return fail(ISAM_ERR_INVALID_ARG, "%s: scale is NaN", who);
    if (!gate) *gates = 1;
    if (*gates < 0 || (rows > 0 && (*gates == 0 || rows % *gates)))
        return fail(ISAM_ERR_INVALID_ARG, "%s: gates=%lld must divide rows=%lld", who, (long long)*gates, (long long)rows);
    if (!norm_sizes(rows, D))
        return fail(ISAM_ERR_UNSUPPORTED, "%s: D=%lld above %lld, or too many rows", who, (long long)D, (long long)kNormMaxD);
    return ISAM_OK;
}

// Address range of a matrix operand (0 bytes for NULL); false if a row is longer than
// its leading dimension or the range passes 2^46 bytes.
bool matrix(const void* p, int64_t rows, int64_t D, int64_t ld, size_t es, size_t* bytes) {
    *bytes = 0;
    if (!p) return true;
    return ld >= D && extent(rows, ld, 1, 0, D, es, bytes);
}

}  // namespace

extern "C" isam_status_t isam_norm_residual(int64_t rows, int64_t D, int64_t gates, int type, const void* x, int64_t ldx,
                                            const void* r, int64_t ldr, const void* gate, const float* w_post,
                                            const float* w_pre, float scale, float eps, void* r_out, int64_t ldro, void* y,
                                            int64_t ldy, void* stream) {
    clear_error();
    const char* who = "isam_norm_residual";
    isam_status_t st = norm_check(rows, D, &gates, type, gate, scale, eps, who);
    if (st != ISAM_OK || rows == 0 || D == 0) return st;
    if (!r || !w_pre || !y) return fail(ISAM_ERR_INVALID_ARG, "%s: r, w_pre or y is NULL", who);
    if (x ? !r_out : (r_out || gate || w_post))
        return fail(ISAM_ERR_INVALID_ARG, "%s: x needs r_out; r_out, gate and w_post need x", who);
    const size_t es = dsize(type);
    size_t x_b, r_b, ro_b, y_b, g_b;
    if (!matrix(x, rows, D, ldx, es, &x_b) || !matrix(r, rows, D, ldr, es, &r_b) || !matrix(r_out, rows, D, ldro, es, &ro_b) ||
        !matrix(y, rows, D, ldy, es, &y_b) || !matrix(gate, gates, D, D, es, &g_b))
        return fail(ISAM_ERR_INVALID_ARG, "%s: a leading dimension is below D, or a tensor spans more than 2^46 bytes", who);
    const bool in_place = r_out == r && ldro == ldr;  // each row is read whole before it is written
    const Tensor all[] = {{"x", x, x_b, false},
                          {"r", r, r_b, false},
                          {"gate", gate, g_b, false},
                          {"w_post", w_post, (size_t)D * 4, false},
                          {"w_pre", w_pre, (size_t)D * 4, false},
                          {"r_out", in_place ? nullptr : r_out, ro_b, true},
                          {"y", y, y_b, true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    if (in_place) {
        const Tensor out[] = {{"r_out", r_out, ro_b, true}, {"x", x, x_b, false}, {"gate", gate, g_b, false},
                              {"w_post", w_post, (size_t)D * 4, false}, {"w_pre", w_pre, (size_t)D * 4, false}, {"y", y, y_b, true}};
        if ((st = disjoint(out, who)) != ISAM_OK) return st;
    }
    NormArgs a{};
    a.rows = rows;
    a.D = D;
    a.type = type;
    a.gates = gates;
    a.rows_per_gate = rows / gates;
    a.x = x;
    a.r = r;
    a.gate = gate;
    a.ld_x = ldx;
    a.ld_r = ldr;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.scale = scale;
    a.eps = eps;
    a.r_out = r_out;
    a.y = y;
    a.ld_ro = ldro;
    a.ld_y = ldy;
    const hipError_t e = launch_norm_forward(a, device_cus(), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" isam_status_t isam_norm_residual_backward(int64_t rows, int64_t D, int64_t gates, int type, const void* x,
                                                     int64_t ldx, const void* r_out, int64_t ldro, const void* gate,
                                                     const float* w_post, const float* w_pre, float scale, float eps,
                                                     const void* dy, int64_t lddy, const void* dr_out, int64_t lddro,
                                                     void* dx, int64_t lddx, void* dr, int64_t lddr, void* dgate,
                                                     float* dw_post, float* dw_pre, void* workspace,
                                                     size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_norm_residual_backward";
    const bool rows0 = rows == 0;
    const int64_t gate_rows = gates;
    isam_status_t st = norm_check(rows, D, &gates, type, gate, scale, eps, who);
    if (st != ISAM_OK || D == 0) return st;
    if (!rows0 && (!r_out || !w_pre || !dy || !dr)) return fail(ISAM_ERR_INVALID_ARG, "%s: r_out, w_pre, dy or dr is NULL", who);
    if (!rows0 && (x ? !dx : (dx || gate || w_post)))
        return fail(ISAM_ERR_INVALID_ARG, "%s: x needs dx; dx, gate and w_post need x", who);
    if (!rows0 && ((dgate && !gate) || (dw_post && !w_post)))
        return fail(ISAM_ERR_INVALID_ARG, "%s: dgate needs gate, dw_post w_post", who);
    if (rows0) gates = gate_rows;  // dgate is cleared whatever stands for the gate
    const size_t es = dsize(type);
    if (rows0 && dgate && (gates < 0 || gates > ((int64_t)1 << 40) / D))
        return fail(ISAM_ERR_INVALID_ARG, "%s: gates=%lld", who, (long long)gates);
    NormArgs a{};
    a.rows = rows;
    a.D = D;
    a.type = type;
    a.gates = gates;
    a.rows_per_gate = rows0 ? 1 : rows / gates;
    a.x = x;
    a.r = r_out;
    a.gate = gate;
    a.ld_x = ldx;
    a.ld_r = ldro;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.scale = scale;
    a.eps = eps;
    a.dy = dy;
    a.dr_out = dr_out;
    a.dx = dx;
    a.dr = dr;
    a.ld_dy = lddy;
    a.ld_dro = lddro;
    a.ld_dx = lddx;
    a.ld_dr = lddr;
    a.dgate = dgate;
    a.dw_post = dw_post;
    a.dw_pre = dw_pre;
    int64_t grid = 0;
    if (!rows0) norm_bwd_grid(a, device_cus(), &grid, &a.parts);
    const size_t need = (size_t)(3 * grid * D) * sizeof(float);
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0,
                    room(need));
    size_t x_b, r_b, dy_b, dro_b, dx_b, dr_b, g_b, dg_b;
    if (!matrix(x, rows, D, ldx, es, &x_b) || !matrix(r_out, rows, D, ldro, es, &r_b) || !matrix(dy, rows, D, lddy, es, &dy_b) ||
        !matrix(dr_out, rows, D, lddro, es, &dro_b) || !matrix(dx, rows, D, lddx, es, &dx_b) ||
        !matrix(dr, rows, D, lddr, es, &dr_b) || !matrix(gate, gates, D, D, es, &g_b) || !matrix(dgate, gates, D, D, es, &dg_b))
        return fail(ISAM_ERR_INVALID_ARG, "%s: a leading dimension is below D, or a tensor spans more than 2^46 bytes", who);
    const size_t w_b = (size_t)D * 4;
    const bool in_place = dr && dr == dr_out && lddr == lddro;
    const Tensor all[] = {{"x", x, x_b, false},           {"r_out", r_out, r_b, false},
                          {"gate", gate, g_b, false},     {"w_post", w_post, w_b, false},
                          {"w_pre", w_pre, w_b, false},   {"dy", dy, dy_b, false},
                          {"dr_out", in_place ? nullptr : dr_out, dro_b, false},
                          {"dx", dx, dx_b, true},         {"dr", dr, dr_b, true},
                          {"dgate", dgate, dg_b, true},   {"dw_post", dw_post, w_b, true},
                          {"dw_pre", dw_pre, w_b, true},  {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    a.partial = reinterpret_cast<float*>(room_start(workspace));
    const hipError_t e = launch_norm_backward(a, grid, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_norm_residual_backward_workspace_size(int64_t rows, int64_t D, int64_t gates, int type) {
    if (rows <= 0 || D <= 0 || !valid_dtype(type) || !norm_sizes(rows, D)) return 0;
    // without a gate the call has one gate row
    int64_t most = 0;
    for (const int64_t g : {gates, (int64_t)1}) {
        if (g <= 0 || rows % g) continue;
        NormArgs a{};
        a.rows = rows;
        a.D = D;
        a.type = type;
        a.gates = g;
        most = std::max(most, norm_bwd_most(a, device_cus()));
    }
    return room((size_t)(3 * most * D) * sizeof(float));
}

// ---------------------------------------------------------------------------
// Gated feed-forward block
// ---------------------------------------------------------------------------
namespace {

// Parts of the workspace, in order: copies of x (twice for the terms) and W with
// aligned rows, the projections (fp32) or their gradients, the bias gradient's
// partial sums, the terms' dx, and what the matrix products use.
struct GatedPlan {
    int64_t Kp;                       // row length of the copies
    int64_t ld_pair;                  // of the projections or their gradients
    bool copy_x, copy_w;
    bool terms;                       // a gradient of few rows: [dG dU] in two bf16 terms, 2 M rows
    bool direct;                      // fp32 projections formed in the block's own kernel
    int tile;
    int64_t bias_rows;                // partial sums of the bias gradient
    size_t x_b, w_b, pair_b, bias_b, join_b, gemm_b;
    size_t total() const { return x_b + w_b + pair_b + bias_b + join_b + gemm_b; }
};

bool rows_aligned(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

int64_t gated_ld_pair(int64_t F) { return cdiv(2 * F, 8) * 8; }

GatedPlan gated_plan(int64_t M, int64_t K, int64_t F, int type, bool x_ok, bool w_ok, bool backward) {
    GatedPlan p{};
    const size_t es = dsize(type);
    if (M == 0 || (!backward && M <= kGatedTokens)) return p;
    p.terms = backward && type == ISAM_BF16 && M <= kGatedTokens && (__int128)2 * M * gated_ld_pair(F) * 2 <= kMaxExtent &&
              (__int128)2 * M * (K + 8) * 4 <= kMaxExtent;
    if (p.terms) {
        p.Kp = cdiv(K, 8) * 8;
        p.x_b = align256((size_t)(2 * M * p.Kp) * es);  // x twice, a row for each row of the terms
        p.ld_pair = gated_ld_pair(F);
        p.pair_b = align256((size_t)(2 * M * p.ld_pair) * es);
        p.bias_rows = 1;
        p.bias_b = align256((size_t)(2 * F) * sizeof(float));
        p.join_b = align256((size_t)(2 * M * K) * sizeof(float));
        p.gemm_b = align256(std::max(product_workspace(0, 0, 2 * M, K, 2 * F, type), product_workspace(1, 0, 2 * F, K, 2 * M, type)));
        return p;
    }
    if (type == ISAM_BF16) {
        p.copy_x = !x_ok || K % 8;
        p.copy_w = !w_ok || K % 8;
        // whole 64-deep tiles where that adds at most an eighth (no range checks in the kernel)
        p.Kp = (cdiv(K, 64) * 64 - K) * 8 <= K ? cdiv(K, 64) * 64 : cdiv(K, 8) * 8;
        if (!(p.copy_x && p.copy_w)) p.Kp = cdiv(K, 8) * 8;
        if (p.copy_x) p.x_b = align256((size_t)(M * p.Kp) * es);
        if (p.copy_w) p.w_b = align256((size_t)(2 * F * p.Kp) * es);
        p.tile = gated_tile(M, F, device_cus());
    }
    p.direct = type == ISAM_F32 && gated_f32_direct(M, K, F, device_cus());
    // (rows of whole 16-byte pieces, so that the products after it need no copy of them)
    p.ld_pair = type == ISAM_F32 && !p.direct ? 2 * F : gated_ld_pair(F);
    if (backward || (type == ISAM_F32 && !p.direct)) p.pair_b = align256((size_t)(M * p.ld_pair) * es);
    p.bias_rows = type == ISAM_BF16 ? gated_bias_rows(p.tile, M) : p.direct ? cdiv(M, kGatedF32Tile) * 2 : cdiv(M, kGatedRows);
    if (backward) p.bias_b = align256((size_t)(p.bias_rows * 2 * F) * sizeof(float));
    if (type == ISAM_F32 && !p.direct) p.gemm_b = product_workspace(0, 1, M, 2 * F, K, type);
    if (backward) {
        p.gemm_b = std::max(p.gemm_b, product_workspace(0, 0, M, K, 2 * F, type));
        p.gemm_b = std::max(p.gemm_b, product_workspace(1, 0, 2 * F, K, M, type));
    }
    p.gemm_b = align256(p.gemm_b);
    return p;
}

isam_status_t gated_check(int64_t M, int64_t K, int64_t F, int type, int act, const char* who) {
    if (M < 0 || K <= 0 || F < 0)
        return fail(ISAM_ERR_INVALID_ARG, "%s: bad size M=%lld K=%lld F=%lld", who, (long long)M, (long long)K, (long long)F);
    if (!valid_dtype(type)) return fail(ISAM_ERR_INVALID_ARG, "%s: dtype must be ISAM_F32 (0) or ISAM_BF16 (1)", who);
    if (act < ISAM_ACT_SIGMOID || act > ISAM_ACT_GELU)
        return fail(ISAM_ERR_INVALID_ARG, "%s: activation must be 0 (sigmoid), 1 (silu) or 2 (gelu)", who);
    return ISAM_OK;
}

// A matrix operand whose extent must stay below 2^31 bytes; a null one has none.
isam_status_t gated_matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t es, size_t* bytes,
                           const char* who) {
    *bytes = 0;
    if (!p || rows == 0 || cols == 0) return ISAM_OK;
    if (ld < cols) return fail(ISAM_ERR_INVALID_ARG, "%s: leading dimension %lld of %s below %lld", who, (long long)ld, name, (long long)cols);
    if (!extent(rows, ld, 1, 0, cols, es, bytes) || *bytes > (size_t)kMaxExtent)
        return fail(ISAM_ERR_UNSUPPORTED, "%s: %s spans more than 2^31 bytes", who, name);
    return ISAM_OK;
}

// Sizes for which every buffer the plan adds stays below 2^31 bytes as well.
bool gated_sizes(int64_t M, int64_t K, int64_t F, int type) {
    const __int128 es = (__int128)dsize(type), most = kMaxExtent;
    const __int128 Kp = (__int128)K + 64;
    return (__int128)M * gated_ld_pair(F) * es <= most && (__int128)M * Kp * es <= most && (__int128)2 * F * Kp * es <= most &&
           (type == ISAM_BF16 || M <= 65535 * kGatedRows);
}

// Copies of x and W with aligned rows, where the plan has them; x, W and their
// leading dimensions become those of the copies.
hipError_t gated_copies(const GatedPlan& p, char* ws, GatedArgs& a, hipStream_t s) {
    if (!p.copy_x && !p.copy_w) return hipSuccess;
    PackRows cx{}, cw{};
    if (p.copy_x) cx = PackRows{static_cast<const uint16_t*>(a.x), a.M, a.K, a.ld_x, reinterpret_cast<uint16_t*>(ws), p.Kp};
    if (p.copy_w)
        cw = PackRows{static_cast<const uint16_t*>(a.W), 2 * a.F, a.K, a.ld_w, reinterpret_cast<uint16_t*>(ws + p.x_b), p.Kp};
    const hipError_t e = launch_pack_rows(cx, cw, device_cus(), s);
    if (e != hipSuccess) return e;
    // (one operand copied: rows of K rounded up to 8 there, K itself a multiple of 8)
    if (p.copy_x) {
        a.x = cx.dst;
        a.ld_x = p.Kp;
    }
    if (p.copy_w) {
        a.W = cw.dst;
        a.ld_w = p.Kp;
    }
    a.K = p.Kp;
    return hipSuccess;
}

}  // namespace

extern "C" isam_status_t isam_gated_ffn(int64_t M, int64_t K, int64_t F, int type, int act, const void* x, int64_t ldx,
                                        const void* W, int64_t ldw, const float* bias, void* out, int64_t ldo, void* workspace,
                                        size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_gated_ffn";
    isam_status_t st = gated_check(M, K, F, type, act, who);
    if (st != ISAM_OK || M == 0 || F == 0) return st;
    if (!x || !W || !out) return fail(ISAM_ERR_INVALID_ARG, "%s: x, W or out is NULL", who);
    const size_t es = dsize(type);
    size_t x_b, w_b, o_b;
    if ((st = gated_matrix("x", x, M, K, ldx, es, &x_b, who)) != ISAM_OK ||
        (st = gated_matrix("W", W, 2 * F, K, ldw, es, &w_b, who)) != ISAM_OK ||
        (st = gated_matrix("out", out, M, F, ldo, es, &o_b, who)) != ISAM_OK)
        return st;
    if (!gated_sizes(M, K, F, type)) return fail(ISAM_ERR_UNSUPPORTED, "%s: M x 2F, M x K or 2F x K passes 2^31 bytes", who);
    const GatedPlan p = gated_plan(M, K, F, type, rows_aligned(x, ldx), rows_aligned(W, ldw), false);
    const size_t need = p.total();
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0,
                    room(need));
    const Tensor all[] = {{"x", x, x_b, false},
                          {"W", W, w_b, false},
                          {"bias", bias, (size_t)(2 * F) * 4, false},
                          {"out", out, o_b, true},
                          {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = room_start(workspace);
    GatedArgs a{};
    a.M = M;
    a.K = K;
    a.F = F;
    a.act = act;
    a.x = x;
    a.W = W;
    a.bias = bias;
    a.ld_x = ldx;
    a.ld_w = ldw;
    a.out = out;
    a.ld_out = ldo;
    hipError_t e;
    if (M <= kGatedTokens) {
        e = launch_gated_tokens(a, type, false, s);
    } else if (type == ISAM_BF16) {
        e = gated_copies(p, ws, a, s);
        if (e == hipSuccess) e = launch_gated_tiles(a, p.tile, false, s);
    } else if (p.direct) {
        e = launch_gated_f32(a, false, s);
    } else {
        a.gu = reinterpret_cast<float*>(ws);
        st = product(0, 1, M, 2 * F, K, type, x, ldx, W, ldw, ISAM_F32, a.gu, 2 * F, ws + p.pair_b, p.gemm_b, s, who);
        if (st != ISAM_OK) return st;
        e = launch_gated_pairs(a, false, s);
    }
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_gated_ffn_workspace_size(int64_t M, int64_t K, int64_t F, int type, int aligned) {
    if (M <= 0 || K <= 0 || F <= 0 || !valid_dtype(type) || !gated_sizes(M, K, F, type)) return 0;
    return room(gated_plan(M, K, F, type, aligned != 0, aligned != 0, false).total());
}

extern "C" isam_status_t isam_gated_ffn_backward(int64_t M, int64_t K, int64_t F, int type, int act, const void* x, int64_t ldx,
                                                 const void* W, int64_t ldw, const float* bias, const void* dout, int64_t lddo,
                                                 void* dx, int64_t lddx, void* dW, int64_t lddw, float* dbias, void* workspace,
                                                 size_t workspace_bytes, void* stream) {
    clear_error();
    const char* who = "isam_gated_ffn_backward";
    isam_status_t st = gated_check(M, K, F, type, act, who);
    if (st != ISAM_OK) return st;
    if (F == 0 && M > 0 && dx) return fail(ISAM_ERR_INVALID_ARG, "%s: F is 0", who);
    if (F == 0) return ISAM_OK;
    if (!dx && !dW && !dbias) return fail(ISAM_ERR_INVALID_ARG, "%s: no output", who);
    if (M > 0 && (!x || !W || !dout)) return fail(ISAM_ERR_INVALID_ARG, "%s: x, W or dout is NULL", who);
    const size_t es = dsize(type);
    size_t x_b, w_b, do_b, dx_b, dw_b;
    if ((st = gated_matrix("x", x, M, K, ldx, es, &x_b, who)) != ISAM_OK ||
        (st = gated_matrix("W", W, 2 * F, K, ldw, es, &w_b, who)) != ISAM_OK ||
        (st = gated_matrix("dout", dout, M, F, lddo, es, &do_b, who)) != ISAM_OK ||
        (st = gated_matrix("dx", dx, M, K, lddx, es, &dx_b, who)) != ISAM_OK ||
        (st = gated_matrix("dW", dW, 2 * F, K, lddw, es, &dw_b, who)) != ISAM_OK)
        return st;
    if (!gated_sizes(M, K, F, type)) return fail(ISAM_ERR_UNSUPPORTED, "%s: M x 2F, M x K or 2F x K passes 2^31 bytes", who);
    const GatedPlan p = gated_plan(M, K, F, type, rows_aligned(x, ldx), rows_aligned(W, ldw), true);
    const size_t need = p.total();
    if (need && (!workspace || workspace_bytes < room(need)))
        return fail(ISAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0,
                    room(need));
    const size_t b_b = (size_t)(2 * F) * 4;
    const Tensor all[] = {{"x", x, x_b, false},       {"W", W, w_b, false},   {"bias", bias, b_b, false},
                          {"dout", dout, do_b, false}, {"dx", dx, dx_b, true}, {"dW", dW, dw_b, true},
                          {"dbias", dbias, b_b, true}, {"workspace", workspace, room(need), true}};
    if ((st = disjoint(all, who)) != ISAM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = room_start(workspace);
    char* const pairs = ws + p.x_b + p.w_b;
    float* const bias_part = reinterpret_cast<float*>(pairs + p.pair_b);
    float* const join = reinterpret_cast<float*>(pairs + p.pair_b + p.bias_b);
    char* const gemm_ws = pairs + p.pair_b + p.bias_b + p.join_b;
    hipError_t e = hipSuccess;
    GatedArgs a{};
    if (M > 0) {
        a.M = M;
        a.K = K;
        a.F = F;
        a.act = act;
        a.x = x;
        a.W = W;
        a.bias = bias;
        a.ld_x = ldx;
        a.ld_w = ldw;
        a.out = pairs;
        a.ld_out = p.ld_pair;
        a.dout = dout;
        a.ld_dout = lddo;
        a.bias_part = dbias ? bias_part : nullptr;
        if (p.terms) {
            e = launch_gated_tokens(a, type, true, s);
            if (e == hipSuccess && dW) {
                const PackRows x1{static_cast<const uint16_t*>(x), M, K, ldx, reinterpret_cast<uint16_t*>(ws), p.Kp};
                PackRows x2 = x1;
                x2.dst += M * p.Kp;
                e = launch_pack_rows(x1, x2, device_cus(), s);
            }
        } else if (type == ISAM_BF16) {
            e = gated_copies(p, ws, a, s);
            if (e == hipSuccess) e = launch_gated_tiles(a, p.tile, true, s);
        } else if (p.direct) {
            e = launch_gated_f32(a, true, s);
        } else {
            a.gu = reinterpret_cast<float*>(pairs);
            st = product(0, 1, M, 2 * F, K, type, x, ldx, W, ldw, ISAM_F32, a.gu, 2 * F, gemm_ws, p.gemm_b, s, who);
            if (st != ISAM_OK) return st;
            e = launch_gated_pairs(a, true, s);
        }
        if (e != hipSuccess) return hip_fail(e, who);
        if (p.terms && dx) {
            st = product(0, 0, 2 * M, K, 2 * F, type, pairs, p.ld_pair, W, ldw, ISAM_F32, join, K, gemm_ws, p.gemm_b, s, who);
            if (st != ISAM_OK) return st;
            GatedArgs sum{};
            sum.M = M;
            sum.K = K;
            sum.gu = join;
            sum.out = dx;
            sum.ld_out = lddx;
            if ((e = launch_gated_join(sum, s)) != hipSuccess) return hip_fail(e, who);
        }
        // (of x and W the aligned copies, where the plan has them)
        if (!p.terms && dx && (st = product(0, 0, M, K, 2 * F, type, pairs, p.ld_pair, a.W, a.ld_w, type, dx, lddx, gemm_ws, p.gemm_b, s, who)) != ISAM_OK)
            return st;
    }
    if (p.terms && dW) {
        st = product(1, 0, 2 * F, K, 2 * M, type, pairs, p.ld_pair, ws, p.Kp, type, dW, lddw, gemm_ws, p.gemm_b, s, who);
        if (st != ISAM_OK) return st;
    }
    if (!p.terms && dW && (st = product(1, 0, 2 * F, K, M, type, pairs, M ? p.ld_pair : 2 * F, a.x, M ? a.ld_x : K, type, dW, lddw, gemm_ws, p.gemm_b, s,
                            who)) != ISAM_OK)
        return st;
    if (dbias) {
        const ColSum sum{bias_part, dbias, p.bias_rows, 2 * F, 1, kF32};
        e = launch_colsum(&sum, 1, s);
    }
    return e == hipSuccess ? ISAM_OK : hip_fail(e, who);
}

extern "C" size_t isam_gated_ffn_backward_workspace_size(int64_t M, int64_t K, int64_t F, int type, int aligned) {
    if (M <= 0 || K <= 0 || F <= 0 || !valid_dtype(type) || !gated_sizes(M, K, F, type)) return 0;
    return room(gated_plan(M, K, F, type, aligned != 0, aligned != 0, true).total());
}
