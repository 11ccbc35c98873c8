// The linear GRU: a GRU whose gates do not see the state, so that the state is
// a scan over time, forward and backward.
//
//   z = sigmoid(gz + bz), n = tanh(gn + bn) or gn + bn, a = z (0 at a reset)
//   h_t = a_t h_{t-1} + (1 - z_t) n_t
//   e_t = a_t (dh_t + e_{t+1}), e_T = dh_T        (gradient that reaches h_{t-1})
//   d_t = dh_t + e_{t+1},  dgz = d (h_{t-1} - n) z (1 - z),  dgn = d (1 - z) n'
//
// Both are first-order recurrences of each channel: a run of steps maps the
// state v before it to A v + B, and two runs compose to (A1 A2, A2 B1 + B2).
// Per value the forward pass reads two gates and writes one state (6 bytes in
// bf16 against some 20 fp32 operations, four of them transcendental), so memory
// bounds it and the schedule is built to touch each value once:
//   * a workgroup owns one sequence's block of 128 bytes of channels (8 lanes x
//     16 bytes) and walks time in tiles of 256 steps: 64 groups of 8 lanes with
//     4 steps each.  A group composes its steps, the 8 groups of a wave are
//     scanned by lane exchanges, the 8 waves through LDS (one barrier), and the
//     state at the tile's end stays in registers for the next tile, whose gates
//     were requested before this tile's arithmetic;
//   * where sequences and channels alone leave compute units idle, time is cut
//     into segments: a first kernel composes each segment to its (A, B), and a
//     segment's workgroup starts from the state those of the segments before it
//     give.  Everything is combined in one order, so results repeat bit for bit;
//   * the backward pass keeps no sequence of states: the forward pass leaves the
//     state before every 256 steps, and each tile forms its states again in
//     registers while it scans e from its end (5 values moved per element, 6 with
//     stored states, which would have to be fp32 to give fp32 gradients).
// A reset must cut off whatever stands before it, NaN included, which 0 * NaN
// does not: its a is -0, and a sign bit in A (kept through products) makes a
// composition drop the left side.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

constexpr int kSteps = 4;  // steps per group and tile

__device__ __forceinline__ bool drops(float a) { return (int)__float_as_uint(a) < 0; }

// A of two runs: the product, with a sign bit if either has one.
template <bool RESET>
__device__ __forceinline__ float compose_a(float a1, float a2) {
    if constexpr (!RESET) return a1 * a2;
    return __uint_as_float(__float_as_uint(__builtin_fabsf(a1 * a2)) | ((__float_as_uint(a1) | __float_as_uint(a2)) & 0x80000000u));
}
// A v + B.
template <bool RESET>
__device__ __forceinline__ float apply(float a, float b, float v) {
    const float r = __builtin_fmaf(a, v, b);
    if constexpr (RESET) return drops(a) ? b : r;
    return r;
}

// What one workgroup works on: a block of channels of one sequence.
template <int ES>
struct Column {
    static constexpr int E = Row16<ES>::E;
    int64_t b, c;  // sequence, this lane's first channel
    int valid;     // channels of this lane that exist
    __device__ __forceinline__ Column(const LinGruArgs& a, int lane) {
        const int64_t blocks = (a.H + 8 * E - 1) / (8 * E);
        b = (int64_t)blockIdx.x / blocks;
        c = ((int64_t)blockIdx.x - b * blocks) * (8 * E) + (lane & 7) * E;
        valid = (int)max((int64_t)0, min((int64_t)E, a.H - c));
    }
};

// Inclusive scan over the wave's 8 groups in time order (UP) or against it.
template <int E, bool RESET, bool UP>
__device__ __forceinline__ void wave_scan(float (&A)[E], float (&B)[E], int lane) {
    static_for<3>([&](auto dc) {
        constexpr int d = 8 << decltype(dc)::value;
        const bool has = UP ? lane >= d : lane + d < 64;
        static_for<E>([&](auto e) {
            const float pa = UP ? __shfl_up(A[e], d) : __shfl_down(A[e], d);
            const float pb = UP ? __shfl_up(B[e], d) : __shfl_down(B[e], d);
            if (has) {
                B[e] = apply<RESET>(A[e], B[e], pb);
                A[e] = compose_a<RESET>(A[e], pa);
            }
        });
    });
}

// The state that reaches `seg` (from the end if BACK): `v` taken through the
// composed segments before it.
template <int E, bool RESET, bool BACK>
__device__ __forceinline__ void segment_in(const LinGruArgs& a, int64_t seg, int64_t b, int64_t c, int valid, float (&v)[E]) {
    const int64_t n = a.batch * a.H, at = b * a.H + c;
    const float* A = a.agg;
    const float* B = a.agg + a.segs * n;
    const int64_t count = BACK ? a.segs - 1 - seg : seg;
#pragma unroll 4
    for (int64_t i = 0; i < count; ++i) {
        const int64_t s = BACK ? a.segs - 1 - i : i;
        float sa[E], sb[E];
        load_f32<E>(A, s * n + at, valid, sa);
        load_f32<E>(B, s * n + at, valid, sb);
        static_for<E>([&](auto e) { v[e] = apply<RESET>(sa[e], sb[e], v[e]); });
    }
}

// Forward pass.  NW waves: tiles of NW * 32 steps.
template <int ES, int NW, bool RESET>
__global__ __launch_bounds__(NW * 64) void lingru_fwd_kernel(LinGruArgs a) {
    constexpr int E = Row16<ES>::E, R = kSteps, TS = NW * 8 * R;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = wid * 8 + (lane >> 3);
    const Column<ES> k(a, lane);
    __shared__ float totals[2][NW][2][8][E];

    float bz[E], bn[E], h[E];
    load_f32<E>(a.bias, k.c, k.valid, bz);
    load_f32<E>(a.bias, a.H + k.c, k.valid, bn);
    load_f32<E>(a.h0, k.b * a.H + k.c, k.valid, h);
    const int64_t tiles = (a.T + TS - 1) / TS;
    const int64_t tile0 = (int64_t)blockIdx.y * a.tiles_per_seg, tile1 = min(tiles, tile0 + a.tiles_per_seg);
    segment_in<E, RESET, false>(a, blockIdx.y, k.b, k.c, k.valid, h);

    const char* gx = static_cast<const char*>(a.gx) + k.b * a.gx_b * ES;
    char* hs = static_cast<char*>(a.h_seq) + k.b * a.h_b * ES;
    uint4 pz[R], pn[R];
    uint8_t pr[R];
    auto fetch = [&](int64_t tile) {
        static_for<R>([&](auto r) {
            const int64_t t = tile * TS + g * R + r;
            const int valid = tile < tile1 && t < a.T ? k.valid : 0;
            pz[r] = Row16<ES>::load(gx, t * a.gx_t + k.c, valid);
            pn[r] = Row16<ES>::load(gx, t * a.gx_t + a.H + k.c, valid);
            if constexpr (RESET) pr[r] = valid ? a.reset[t * a.rs_t + k.b * a.rs_b] : 0;
        });
    };
    fetch(tile0);
    for (int64_t tile = tile0; tile < tile1; ++tile) {
        if (a.states && g == 0) store_f32<E>(a.states, (tile * a.batch + k.b) * a.H + k.c, k.valid, h);
        const int64_t t0 = tile * TS + g * R;
        float ca[R][E], cb[R][E], A[E], B[E];
        static_for<R>([&](auto r) {
            float gz[E], gn[E];
            Row16<ES>::unpack(pz[r], gz);
            Row16<ES>::unpack(pn[r], gn);
            const bool in = t0 + r < a.T;
            static_for<E>([&](auto e) {
                float z, omz;
                sigmoid_pair(gz[e] + bz[e], z, omz);
                const float v = gn[e] + bn[e], n = a.candidate ? tanh_f32(v) : v;
                ca[r][e] = in ? z : 1.0f;
                cb[r][e] = in ? omz * n : 0.0f;
                if constexpr (RESET) ca[r][e] = in && pr[r] ? -0.0f : ca[r][e];
                A[e] = r == 0 ? ca[r][e] : compose_a<RESET>(A[e], ca[r][e]);
                B[e] = r == 0 ? cb[r][e] : apply<RESET>(ca[r][e], cb[r][e], B[e]);
            });
        });
        fetch(tile + 1);
        wave_scan<E, RESET, true>(A, B, lane);
        float (&tot)[NW][2][8][E] = totals[tile & 1];
        if ((lane >> 3) == 7) static_for<E>([&](auto e) {
            tot[wid][0][lane & 7][e] = A[e];
            tot[wid][1][lane & 7][e] = B[e];
        });
        __syncthreads();  // (the next tile writes the other half)
        float v[E];
        static_for<E>([&](auto e) { v[e] = h[e]; });
        static_for<NW>([&](auto w) {
            static_for<E>([&](auto e) {
                h[e] = apply<RESET>(tot[w][0][lane & 7][e], tot[w][1][lane & 7][e], h[e]);
                if (w < wid) v[e] = h[e];
            });
        });
        static_for<E>([&](auto e) {
            const float pa = __shfl_up(A[e], 8), pb = __shfl_up(B[e], 8);
            if (lane >= 8) v[e] = apply<RESET>(pa, pb, v[e]);
        });
        static_for<R>([&](auto r) {
            static_for<E>([&](auto e) { v[e] = apply<RESET>(ca[r][e], cb[r][e], v[e]); });
            if (a.h_seq) Row16<ES>::store(hs, (t0 + r) * a.h_t + k.c, Row16<ES>::pack(v), t0 + r < a.T ? k.valid : 0);
        });
    }
    if (a.h_T && tile1 == tiles && g == 0) store_f32<E>(a.h_T, k.b * a.H + k.c, k.valid, h);
}

// A few steps, one thread per channel: decoding (no tile to fill).
constexpr int kFewSteps = 8;
template <int ES>
__global__ __launch_bounds__(64) void lingru_few_kernel(LinGruArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (i >= a.batch * a.H) return;
    const int64_t b = i / a.H, c = i - b * a.H;
    const int T = (int)a.T;
    float gz[kFewSteps], gn[kFewSteps];
    bool drop[kFewSteps];
    float h = a.h0 ? a.h0[i] : 0.0f;
    const float bz = a.bias ? a.bias[c] : 0.0f, bn = a.bias ? a.bias[a.H + c] : 0.0f;
    static_for<kFewSteps>([&](auto t) {
        if (t < T) {
            gz[t] = Row16<ES>::get(a.gx, b * a.gx_b + t * a.gx_t + c);
            gn[t] = Row16<ES>::get(a.gx, b * a.gx_b + t * a.gx_t + a.H + c);
            drop[t] = a.reset && a.reset[t * a.rs_t + b * a.rs_b];
        }
    });
    if (a.states && T > 0) a.states[i] = h;
    static_for<kFewSteps>([&](auto t) {
        if (t < T) {
            float z, omz;
            sigmoid_pair(gz[t] + bz, z, omz);
            const float v = gn[t] + bn, n = a.candidate ? tanh_f32(v) : v;
            h = drop[t] ? omz * n : __builtin_fmaf(z, h, omz * n);
            if (a.h_seq) Row16<ES>::put(a.h_seq, b * a.h_b + t * a.h_t + c, h);
        }
    });
    if (a.h_T) a.h_T[i] = h;
}

// (A, B) of each segment, forward or (BACK) of e: the 64 groups of a workgroup
// take equal runs of the segment's steps, then compose.
template <int ES, bool RESET, bool BACK>
__global__ __launch_bounds__(512) void lingru_segment_kernel(LinGruArgs a) {
    constexpr int E = Row16<ES>::E, U = 4;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = wid * 8 + (lane >> 3);
    const Column<ES> k(a, lane);
    __shared__ float totals[8][2][8][E];
    float bz[E], bn[E], A[E], B[E];
    load_f32<E>(a.bias, k.c, k.valid, bz);
    load_f32<E>(a.bias, a.H + k.c, k.valid, bn);
    static_for<E>([&](auto e) { A[e] = 1.0f; B[e] = 0.0f; });
    const int64_t steps = a.tiles_per_seg * 256, t0 = (int64_t)blockIdx.y * steps, t1 = min(a.T, t0 + steps);
    const int run = (int)(steps / 64);  // a multiple of U
    const char* gx = static_cast<const char*>(a.gx) + k.b * a.gx_b * ES;
    const char* dh = static_cast<const char*>(a.dh_seq) + k.b * a.dh_b * ES;
    for (int i0 = 0; i0 < run; i0 += U) {
        uint4 pz[U], po[U];
        uint8_t pr[U];
        static_for<U>([&](auto u) {
            const int i = BACK ? run - 1 - (i0 + u) : i0 + u;
            const int64_t t = t0 + (int64_t)g * run + i;
            const int valid = t < t1 ? k.valid : 0;
            pz[u] = Row16<ES>::load(gx, t * a.gx_t + k.c, valid);
            if constexpr (BACK) po[u] = Row16<ES>::load(dh, t * a.dh_t + k.c, a.dh_seq ? valid : 0);
            else po[u] = Row16<ES>::load(gx, t * a.gx_t + a.H + k.c, valid);
            if constexpr (RESET) pr[u] = valid ? a.reset[t * a.rs_t + k.b * a.rs_b] : 0;
        });
        static_for<U>([&](auto u) {
            const int i = BACK ? run - 1 - (i0 + u) : i0 + u;
            const bool in = t0 + (int64_t)g * run + i < t1;
            float gz[E], o[E];
            Row16<ES>::unpack(pz[u], gz);
            Row16<ES>::unpack(po[u], o);
            static_for<E>([&](auto e) {
                float z, omz, b;
                sigmoid_pair(gz[e] + bz[e], z, omz);
                if constexpr (BACK) {
                    b = z * o[e];
                } else {
                    const float v = o[e] + bn[e];
                    b = omz * (a.candidate ? tanh_f32(v) : v);
                }
                float s = in ? z : 1.0f;
                if constexpr (RESET) {
                    s = in && pr[u] ? -0.0f : s;
                    if (BACK && in && pr[u]) b = 0.0f;
                }
                b = in ? b : 0.0f;
                B[e] = apply<RESET>(s, b, B[e]);
                A[e] = compose_a<RESET>(A[e], s);
            });
        });
    }
    wave_scan<E, RESET, !BACK>(A, B, lane);
    if ((lane >> 3) == (BACK ? 0 : 7)) static_for<E>([&](auto e) {
        totals[wid][0][lane & 7][e] = A[e];
        totals[wid][1][lane & 7][e] = B[e];
    });
    __syncthreads();
    if (g != 0) return;
    static_for<8>([&](auto i) {
        constexpr int w = BACK ? 7 - decltype(i)::value : decltype(i)::value;
        static_for<E>([&](auto e) {
            const float wa = totals[w][0][lane & 7][e], wb = totals[w][1][lane & 7][e];
            B[e] = i == 0 ? wb : apply<RESET>(wa, wb, B[e]);
            A[e] = i == 0 ? wa : compose_a<RESET>(A[e], wa);
        });
    });
    const int64_t n = a.batch * a.H, at = (int64_t)blockIdx.y * n + k.b * a.H + k.c;
    store_f32<E>(a.agg, at, k.valid, A);
    store_f32<E>(a.agg + a.segs * n, at, k.valid, B);
}

// Backward pass.  The tile's states are formed again from the one before it.
template <int ES, int NW, bool RESET>
__global__ __launch_bounds__(NW * 64) void lingru_bwd_kernel(LinGruArgs a) {
    constexpr int E = Row16<ES>::E, R = kSteps, TS = NW * 8 * R;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = wid * 8 + (lane >> 3);
    const Column<ES> k(a, lane);
    __shared__ float totals[2][NW][3][8][E];

    float bz[E], bn[E], er[E], sz[E], sn[E];
    load_f32<E>(a.bias, k.c, k.valid, bz);
    load_f32<E>(a.bias, a.H + k.c, k.valid, bn);
    load_f32<E>(a.dh_T, k.b * a.H + k.c, k.valid, er);
    static_for<E>([&](auto e) { sz[e] = 0.0f; sn[e] = 0.0f; });
    const int64_t tiles = (a.T + TS - 1) / TS;
    const int64_t tile0 = (int64_t)blockIdx.y * a.tiles_per_seg, tile1 = min(tiles, tile0 + a.tiles_per_seg);
    segment_in<E, RESET, true>(a, blockIdx.y, k.b, k.c, k.valid, er);

    const char* gx = static_cast<const char*>(a.gx) + k.b * a.gx_b * ES;
    const char* dh = static_cast<const char*>(a.dh_seq) + k.b * a.dh_b * ES;
    char* dg = static_cast<char*>(a.dgx) + k.b * a.dg_b * ES;
    uint4 pz[R], pn[R], pd[R];
    uint8_t pr[R];
    float ps[E];
    auto fetch = [&](int64_t tile) {
        const int vt = tile >= tile0 ? k.valid : 0;
        static_for<R>([&](auto r) {
            const int64_t t = tile * TS + g * R + r;
            const int valid = t < a.T ? vt : 0;
            pz[r] = Row16<ES>::load(gx, t * a.gx_t + k.c, valid);
            pn[r] = Row16<ES>::load(gx, t * a.gx_t + a.H + k.c, valid);
            pd[r] = Row16<ES>::load(dh, t * a.dh_t + k.c, a.dh_seq ? valid : 0);
            if constexpr (RESET) pr[r] = valid ? a.reset[t * a.rs_t + k.b * a.rs_b] : 0;
        });
        load_f32<E>(a.states, (tile * a.batch + k.b) * a.H + k.c, vt, ps);
    };
    fetch(tile1 - 1);
    for (int64_t tile = tile1 - 1; tile >= tile0; --tile) {
        const int64_t t0 = tile * TS + g * R;
        float z[R][E], omz[R][E], n[R][E], d[R][E], A[E], B[E], Z[E], C[E], hs[E];
        bool drop[R];
        static_for<R>([&](auto r) {
            float gz[E], gn[E];
            Row16<ES>::unpack(pz[r], gz);
            Row16<ES>::unpack(pn[r], gn);
            Row16<ES>::unpack(pd[r], d[r]);
            const bool in = t0 + r < a.T;
            drop[r] = RESET && in && pr[r];
            static_for<E>([&](auto e) {
                sigmoid_pair(gz[e] + bz[e], z[r][e], omz[r][e]);
                const float v = gn[e] + bn[e];
                n[r][e] = a.candidate ? tanh_f32(v) : v;
                if (!in) { z[r][e] = 1.0f; omz[r][e] = 0.0f; n[r][e] = 0.0f; }
                const float s = RESET && drop[r] ? -0.0f : z[r][e], b = omz[r][e] * n[r][e];
                A[e] = r == 0 ? s : compose_a<RESET>(A[e], s);
                B[e] = r == 0 ? b : apply<RESET>(s, b, B[e]);
            });
        });
        static_for<E>([&](auto e) {
            hs[e] = ps[e];
            Z[e] = A[e];
            C[e] = 0.0f;
            static_for<R>([&](auto i) {
                constexpr int r = R - 1 - decltype(i)::value;
                C[e] = RESET && drop[r] ? 0.0f : z[r][e] * (d[r][e] + C[e]);
            });
        });
        fetch(tile - 1);
        wave_scan<E, RESET, true>(A, B, lane);
        wave_scan<E, RESET, false>(Z, C, lane);
        float (&tot)[NW][3][8][E] = totals[tile & 1];
        if ((lane >> 3) == 7) static_for<E>([&](auto e) {
            tot[wid][0][lane & 7][e] = A[e];
            tot[wid][1][lane & 7][e] = B[e];
        });
        if ((lane >> 3) == 0) static_for<E>([&](auto e) { tot[wid][2][lane & 7][e] = C[e]; });
        __syncthreads();
        float en[E];
        static_for<E>([&](auto e) { en[e] = er[e]; });
        static_for<NW>([&](auto i) {
            constexpr int w = decltype(i)::value, wr = NW - 1 - w;
            static_for<E>([&](auto e) {
                if (w < wid) hs[e] = apply<RESET>(tot[w][0][lane & 7][e], tot[w][1][lane & 7][e], hs[e]);
                er[e] = apply<RESET>(tot[wr][0][lane & 7][e], tot[wr][2][lane & 7][e], er[e]);
                if (wr > wid) en[e] = er[e];
            });
        });
        // state before this group's steps, e after them
        float hb[R][E];
        static_for<E>([&](auto e) {
            const float pa = __shfl_up(A[e], 8), pb = __shfl_up(B[e], 8);
            if (lane >= 8) hs[e] = apply<RESET>(pa, pb, hs[e]);
            const float qa = __shfl_down(Z[e], 8), qc = __shfl_down(C[e], 8);
            if (lane < 56) en[e] = apply<RESET>(qa, qc, en[e]);
            static_for<R>([&](auto r) {
                hb[r][e] = RESET && drop[r] ? 0.0f : hs[e];
                hs[e] = RESET && drop[r] ? omz[r][e] * n[r][e] : __builtin_fmaf(z[r][e], hs[e], omz[r][e] * n[r][e]);
            });
        });
        static_for<R>([&](auto i) {
            constexpr int r = R - 1 - decltype(i)::value;
            const bool in = t0 + r < a.T;
            float oz[E], on[E];
            static_for<E>([&](auto e) {
                const float dt = d[r][e] + en[e], q = dt * omz[r][e];
                oz[e] = q * z[r][e] * (hb[r][e] - n[r][e]);
                on[e] = a.candidate ? q * (1.0f - n[r][e] * n[r][e]) : q;
                en[e] = RESET && drop[r] ? 0.0f : z[r][e] * dt;
                if (in) {
                    sz[e] += oz[e];
                    sn[e] += on[e];
                }
            });
            Row16<ES>::store(dg, (t0 + r) * a.dg_t + k.c, Row16<ES>::pack(oz), in ? k.valid : 0);
            Row16<ES>::store(dg, (t0 + r) * a.dg_t + a.H + k.c, Row16<ES>::pack(on), in ? k.valid : 0);
        });
        // (step by step, closer than the composition of the tile)
        if (a.dh0 && tile == 0 && g == 0) store_f32<E>(a.dh0, k.b * a.H + k.c, k.valid, en);
    }
    if (a.dh0 && tiles == 0 && g == 0) store_f32<E>(a.dh0, k.b * a.H + k.c, k.valid, er);
    if (!a.dbias) return;
    // this workgroup's sums over time: lanes of a wave, then waves
    static_for<3>([&](auto dc) {
        constexpr int d = 8 << decltype(dc)::value;
        static_for<E>([&](auto e) {
            sz[e] += __shfl_down(sz[e], d);
            sn[e] += __shfl_down(sn[e], d);
        });
    });
    __syncthreads();
    if ((lane >> 3) == 0) static_for<E>([&](auto e) {
        totals[0][wid][0][lane & 7][e] = sz[e];
        totals[0][wid][1][lane & 7][e] = sn[e];
    });
    __syncthreads();
    if (g != 0) return;
    static_for<NW - 1>([&](auto i) {
        static_for<E>([&](auto e) {
            sz[e] += totals[0][i + 1][0][lane & 7][e];
            sn[e] += totals[0][i + 1][1][lane & 7][e];
        });
    });
    const int64_t row = ((int64_t)blockIdx.y * a.batch + k.b) * 2 * a.H + k.c;
    store_f32<E>(a.bias_part, row, k.valid, sz);
    store_f32<E>(a.bias_part, row + a.H, k.valid, sn);
}

template <int ES>
int64_t columns(const LinGruArgs& a) {
    const int64_t cb = 8 * Row16<ES>::E;
    return a.batch * ((a.H + cb - 1) / cb);
}

template <int ES>
hipError_t forward(const LinGruArgs& a, hipStream_t s) {
    const int64_t cols = columns<ES>(a), n = a.batch * a.H;
    if (cols > INT32_MAX || (n + 63) / 64 > INT32_MAX) return hipErrorInvalidValue;
    if (a.T <= kFewSteps) {
        hipLaunchKernelGGL(lingru_few_kernel<ES>, dim3((unsigned)((n + 63) / 64)), dim3(64), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)cols, (unsigned)a.segs);
    if (a.segs > 1) {
        hipLaunchKernelGGL((a.reset ? lingru_segment_kernel<ES, true, false> : lingru_segment_kernel<ES, false, false>), grid,
                           dim3(512), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.T <= 64)
        hipLaunchKernelGGL((a.reset ? lingru_fwd_kernel<ES, 2, true> : lingru_fwd_kernel<ES, 2, false>), grid, dim3(128), 0, s, a);
    else
        hipLaunchKernelGGL((a.reset ? lingru_fwd_kernel<ES, 8, true> : lingru_fwd_kernel<ES, 8, false>), grid, dim3(512), 0, s, a);
    return hipGetLastError();
}

template <int ES>
hipError_t backward(const LinGruArgs& a, hipStream_t s) {
    const int64_t cols = columns<ES>(a);
    if (cols > INT32_MAX) return hipErrorInvalidValue;
    if (cols > 0) {
        const dim3 grid((unsigned)cols, (unsigned)a.segs);
        if (a.segs > 1) {
            hipLaunchKernelGGL((a.reset ? lingru_segment_kernel<ES, true, true> : lingru_segment_kernel<ES, false, true>), grid,
                               dim3(512), 0, s, a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (a.T <= 64)
            hipLaunchKernelGGL((a.reset ? lingru_bwd_kernel<ES, 2, true> : lingru_bwd_kernel<ES, 2, false>), grid, dim3(128), 0, s, a);
        else
            hipLaunchKernelGGL((a.reset ? lingru_bwd_kernel<ES, 8, true> : lingru_bwd_kernel<ES, 8, false>), grid, dim3(512), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return a.dbias ? launch_colsum(a.bias_part, a.segs * a.batch, 2 * a.H, 1, kF32, a.dbias, s) : hipSuccess;
}

}  // namespace

// Segments of time: none while sequences and channel blocks give every compute
// unit a workgroup, otherwise enough for two per unit, of two tiles or more.
void lingru_segments(int64_t T, int64_t batch, int64_t H, int type, int cus, int64_t* segs, int64_t* tiles_per_seg) {
    const int64_t cb = type == kBF16 ? 64 : 32, cols = batch * ((H + cb - 1) / cb), tiles = (T + kLinGruChunk - 1) / kLinGruChunk;
    int64_t s = 1;
    if (cols > 0 && cols < cus && tiles >= 4) s = (2 * (int64_t)cus) / cols;
    if (s > tiles / 2) s = tiles / 2;
    if (s < 1) s = 1;
    int64_t per = (tiles + s - 1) / s;
    if (per < 1) per = 1;
    *tiles_per_seg = per;
    *segs = tiles > 0 ? (tiles + per - 1) / per : 1;
}

hipError_t launch_lingru_forward(const LinGruArgs& a, hipStream_t s) {
    return a.type == kBF16 ? forward<2>(a, s) : forward<4>(a, s);
}

hipError_t launch_lingru_backward(const LinGruArgs& a, hipStream_t s) {
    return a.type == kBF16 ? backward<2>(a, s) : backward<4>(a, s);
}

}  // namespace isam
