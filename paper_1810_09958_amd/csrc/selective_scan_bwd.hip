// Gradient of the selective scan.  With dv_t = dy_t silu(z_t) and g_t the gradient of h_t:
//
//   g_t = C_t dv_t + a_{t+1} g_{t+1}, a = exp(d A)  (no second term before a reset; + dh_T at the last token)
//   dC_t = sum_c h_t dv_t,  dB_t = sum_c g_t d_t x_t,  dx_t = skip dv_t + d_t sum_n g_t B_t
//   dd_t = sum_n g_t a_t h_{t-1} A + x_t sum_n g_t B_t,  ddt_t = dd_t sigmoid(dt_t + dt_bias)
//   dA = sum g_t a_t h_{t-1} d_t,  dskip = sum dv x,  dz_t = dy_t v_t silu'(z_t),  dh0 = a_0 g_0
//
// Tiles from the end of time.  The states of 16 tokens (8 for N above 32) are formed again in registers from the one
// kept before them, with their a; then the tokens are walked backwards.  Running back by dividing by
// a would lose every digit where a is small, and keeping each state would move 4 N bytes a value.
// dB and dC are sums over channels: a wave halves its values lane bit by lane bit, the waves meet in
// LDS, and each workgroup leaves a row of partial sums for every token, which a second kernel
// adds in a fixed order.  dA, dskip and the bias' gradient are kept in registers over time.
#include <algorithm>

#include "selective_scan.hpp"

namespace isam {

namespace {

// Sums of NV values over the CW lanes of a group (lane bits below CW), halving the values with each
// bit from the highest on while there are several: the lane is left with LEFT values, the first of
// which is number `first`.
template <int BIT>
__device__ __forceinline__ float from_bit(float v) {
    if constexpr (BIT == 3) return dpp<kDppRor8>(v);
    else if constexpr (BIT == 2) return dpp<kDppHalfMirror>(v);  // (lane 7 - i of each eight)
    else if constexpr (BIT == 1) return dpp<kDppXor2>(v);
    else return dpp<kDppXor1>(v);
}
template <int BIT, int NV, int ALL>
__device__ __forceinline__ void sum_channels(float (&v)[ALL], int lane) {
    if constexpr (BIT >= 0) {
        if constexpr (NV > 1) {
            const bool up = lane >> BIT & 1;
            static_for<NV / 2>([&](auto j) {
                const float keep = up ? v[j + NV / 2] : v[j], send = up ? v[j] : v[j + NV / 2];
                v[j] = keep + from_bit<BIT>(send);
            });
            sum_channels<BIT - 1, NV / 2>(v, lane);
        } else {
            v[0] += from_bit<BIT>(v[0]);
            sum_channels<BIT - 1, 1>(v, lane);
        }
    }
}

template <int ES, bool VEC, int L, int R, bool SUM>
__global__ __launch_bounds__(256, 2) void scan_bwd_kernel(ScanArgs a) {
    using S = ScanShape<ES, VEC, L, R>;
    using P = typename S::P;
    constexpr int CH = S::CH, E = S::E, NP = S::NP, TT = kScanTile, CK = S::CK, CW = S::CW;
    constexpr int BITS = CW == 16 ? 4 : CW == 8 ? 3 : 2, LEFT = 2 * R > CW ? 2 * R / CW : 1;
    __shared__ __attribute__((aligned(16))) float4 dd[TT][CH];                    // d, d x, dv, v
    __shared__ __attribute__((aligned(16))) float2 back_sums[SUM ? 1 : TT][CH];   // sum q A, sum g B
    __shared__ __attribute__((aligned(16))) float bc[TT * NP * 2];
    __shared__ float2 par[CH];                            // dt_bias, skip
    __shared__ float2 own_sums[SUM ? 1 : E][SUM ? 1 : 256];  // a thread's sums of dv x and ddt
    __shared__ __attribute__((aligned(16))) float part[2][SUM ? 1 : kScanWaves][SUM ? 1 : CK][2 * NP];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane / CW, cl = wid * CW + lane % CW;
    const int64_t blocks = (a.D + CH - 1) / CH;
    const int64_t place = blockIdx.x / (a.batch * blocks), rest = blockIdx.x - place * a.batch * blocks;
    const int64_t seg = SUM ? place + 1 : place;  // (nobody asks for the first one's summary)
    const int64_t b = rest / blocks, blk = rest - b * blocks, c0 = blk * CH, ch = c0 + cl;
    const int64_t tbeg = seg * a.seg_len, tend = min(a.T, tbeg + a.seg_len);
    const bool in = ch < a.D;
    const bool ragged = !SUM && c0 + CH > a.D;  // some lanes' channels are none: their zeros must stay out of dB and dC
    const int N = (int)a.N;

    float A2[R], G[R], dA[R];
    static_for<R>([&](auto r) {
        const int n = g * R + r;
        const bool on = in && n < N;
        A2[r] = on ? a.A[ch * N + n] * kScanLog2e : 0.0f;
        G[r] = dA[r] = 0.0f;
        if (!SUM && on) {
            G[r] = a.dh_T ? a.dh_T[(b * a.D + ch) * N + n] : 0.0f;
#pragma unroll 4
            for (int64_t s = a.segs - 1; s > seg; --s) {
                const int64_t at = (s * a.batch + b) * a.D + ch;
                G[r] = pass_on(a.seg_sum[at], A2[r], G[r], a.seg_end[at * N + n]);
            }
        }
    });

    // This thread's piece of a tile: row tr, channels c0 + pc .. + E.  LEAN: the index goes through an empty asm wherever it
    // is used, so that what is computed from it is not held in registers across the walk (N above 32: 218 us with some
    // 45 spilled, 180 without; where they suffice, forming the places again costs more, N = 16: 430 against 400).
    constexpr bool LEAN = R >= 4;
    struct Mine {
        int tr, pc, valid;
    };
    auto mine = [&]() {
        int id = tid;
        if constexpr (LEAN) asm volatile("" : "+v"(id));
        const int pc = id % S::PPR * E;
        return Mine{id / S::PPR, pc, (int)max((int64_t)0, min((int64_t)E, a.D - (c0 + pc)))};
    };
    for (int i = tid; i < CH; i += 256) {
        const bool on = c0 + i < a.D;
        par[i] = make_float2(on && a.dt_bias ? a.dt_bias[c0 + i] : 0.0f, on && a.skip ? a.skip[c0 + i] : 0.0f);
    }
    if constexpr (!SUM) static_for<E>([&](auto e) { own_sums[e][tid] = make_float2(0.0f, 0.0f); });
    const int64_t tlast = tbeg + (tend - tbeg - 1) / TT * TT;
    TileRows<ES> rx(a.x, b, tlast), rd(a.dt, b, tlast), rz(a.z, b, tlast), ry(a.dy, b, tlast), rB(a.B, b, tlast), rC(a.C, b, tlast),
        rdx(a.dx, b, tlast), rdt(a.ddt, b, tlast), rdz(a.dz, b, tlast);
    auto offset = [&](const TileRows<ES>& r, const Mine& m, int left) {
        return r.p && m.tr < left && m.valid > 0 ? (uint32_t)m.tr * r.row + (uint32_t)((c0 + m.pc) * ES) : kOob;
    };
    P px, pd, pz, py;
    ScanWeights<ES, NP> wb, wc;
    ScanMarks marks;
    auto fetch = [&](int64_t t0) {  // (tiles before the segment: nothing is read)
        const int left = t0 >= tbeg ? (int)min((int64_t)TT, tend - t0) : 0;
        const Mine m = mine();
        int id = tid;
        if constexpr (LEAN) asm volatile("" : "+v"(id));
        pd.load(rd.buffer(), offset(rd, m, left), m.valid);
        pz.load(rz.buffer(), offset(rz, m, left), m.valid);
        py.load(ry.buffer(), offset(ry, m, left), m.valid);
        wc.load(rC.buffer(), rC.row, N, left, id);
        rd.back();
        rz.back();
        ry.back();
        rC.back();
        if constexpr (!SUM) {
            px.load(rx.buffer(), offset(rx, m, left), m.valid);
            wb.load(rB.buffer(), rB.row, N, left, id);
            rx.back();
            rB.back();
        }
        marks.load(a, b, max(t0, (int64_t)0), left, lane);
    };
    float total = 0.0f;
    bool dropped = false;
    fetch(tlast);
    __syncthreads();  // (par)
    using Token = ScanToken<L, R, true>;
    // the state kept before the next tokens to be walked
    float hnext[R];
    auto kept = [&](int64_t t) {
        const float* const from = a.states + ((t / CK * a.batch + b) * a.D + ch) * N + g * R;
        static_for<R>([&](auto r) { hnext[r] = t >= tbeg && in && g * R + r < N ? from[r] : 0.0f; });
    };
    if constexpr (!SUM) kept(tbeg + (tend - tbeg - 1) / CK * CK);
    // the first value that sum_channels leaves in this lane: the bits that halved the values, the highest first
    constexpr int USED = 2 * R >= CW ? BITS : (R == 1 ? 1 : 2);
    const int first = ((lane & (CW - 1)) >> (BITS - USED)) * LEFT;
    for (int64_t t0 = tlast; t0 >= tbeg; t0 -= TT) {
        const int left = (int)min((int64_t)TT, tend - t0);
        // (the pieces stay as they came; what the last step needs of them is formed again there)
        const P qx = px, qd = pd, qz = pz, qy = py;
        bool wild = false;
        {
            const Mine m = mine();
            float x[E], raw[E], zs[E], dv[E];
            if constexpr (!SUM) qx.unpack(x);
            qd.unpack(raw);
            qz.unpack(zs);
            qy.unpack(dv);
            static_for<E>([&](auto e) {
                const float step = m.tr < left && e < m.valid ? softplus(raw[e] + par[m.pc + e].x) : 0.0f;
                if (a.z.p) {
                    float gate, omz;
                    sigmoid_pair(zs[e], gate, omz);
                    dv[e] *= zs[e] * gate;
                }
                const float dx = SUM ? 0.0f : step * x[e];
                dd[m.tr][m.pc + e] = make_float4(step, dx, dv[e], 0.0f);
                wild = wild || not_finite(dx) || not_finite(dv[e]);
            });
        }
        {
            int id = tid;
            if constexpr (LEAN) asm volatile("" : "+v"(id));
            if (ragged) wild = wild || wb.wild() || wc.wild();
            wc.template put<R>(bc, 1, id);
            if constexpr (!SUM) wb.template put<R>(bc, 0, id);
        }
        const uint32_t reset = marks.bits();
        fetch(t0 - TT);  // (before the segment: zeros)
        wild = meet(N != NP || ragged, wild);
        auto walk = [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
            if constexpr (SUM) {
#pragma unroll 4
                for (int t = TT - 1; t >= 0; --t) {
                    const float4 s = dd[t][cl];
                    float Cv[R];
                    lds_get<R>(bc + (t * L + g) * 2 * R + R, Cv);
                    const bool drop = !FAST && (reset >> t & 1), live = FAST || t < left;
                    static_for<R>([&](auto r) {
                        const float back = __builtin_amdgcn_exp2f(s.x * A2[r]) * __builtin_fmaf(Cv[r], s.z, G[r]);
                        G[r] = drop ? 0.0f : live ? back : G[r];
                    });
                    total += s.x;
                    dropped = dropped || drop;
                }
                return;
            } else {
#pragma unroll 1
                for (int k = TT / CK - 1; k >= 0; --k) {
                    const int tc = k * CK;
                    if (!FAST && tc >= left) continue;
                    float h[CK + 1][R], av[CK][R];  // h[i]: the state before token i (reset or not)
                    static_for<R>([&](auto r) { h[0][r] = hnext[r]; });
                    kept(t0 + tc - CK);
                    float(*const to)[CK][2 * NP] = part[k & 1];
                    // Tokens' values on their way from LDS: two ahead of the one walked.
                    Token tok[4];
                    float dvs[4];
                    auto get = [&](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        tok[i & 3].get(*reinterpret_cast<const float2*>(&dd[tc + i][cl]), bc, tc + i, g);
                    };
                    get(std::integral_constant<int, 0>{});
                    get(std::integral_constant<int, 1>{});
                    float p[4];
                    static_for<CK>([&](auto ic) {
                        constexpr int i = decltype(ic)::value;
                        if constexpr (i + 2 < CK) get(std::integral_constant<int, (i + 2 < CK ? i + 2 : 0)>{});
                        __builtin_amdgcn_sched_barrier(0);
                        const Token& s = tok[i & 3];
                        const bool drop = !FAST && (reset >> (tc + i) & 1), live = tc + i < left;
                        float acc = 0.0f;
                        static_for<R>([&](auto r) {
                            const bool on = FAST || (live && in && g * R + r < N);
                            const float aw = on ? __builtin_amdgcn_exp2f(s.s.x * A2[r]) : 1.0f;
                            av[i][r] = aw;
                            const float hn = __builtin_fmaf(aw, drop ? 0.0f : h[i][r], s.s.y * s.B[r]);
                            h[i + 1][r] = on ? hn : h[i][r];
                            acc = r == 0 ? s.C[0] * h[i + 1][0] : __builtin_fmaf(s.C[r], h[i + 1][r], acc);
                        });
                        p[i & 3] = acc;
                        if constexpr ((i & 3) == 3) {
                            if (a.z.p) {
                                const float v = sum_lanes4<L>(p);
                                dd[tc + i - 3 + (lane >> 4)][cl].w = v;
                            }
                        }
                    });
                    // (what was read from LDS is read again on the way back, not held in registers)
                    asm volatile("" ::: "memory");
                    auto get_back = [&](auto ic) {
                        get(ic);
                        dvs[ic & 3] = dd[tc + ic][cl].z;
                    };
                    get_back(std::integral_constant<int, CK - 1>{});
                    get_back(std::integral_constant<int, CK - 2>{});
                    float pq[4], pg[4];
                    static_for<CK>([&](auto ir) {
                        constexpr int i = CK - 1 - decltype(ir)::value;
                        if constexpr (i >= 2) get_back(std::integral_constant<int, (i >= 2 ? i - 2 : 0)>{});
                        __builtin_amdgcn_sched_barrier(0);
                        const Token& s = tok[i & 3];
                        const float dv = dvs[i & 3];
                        const bool drop = !FAST && (reset >> (tc + i) & 1), live = FAST || tc + i < left;
                        float aq = 0.0f, gb = 0.0f, sums[2 * R];
                        static_for<R>([&](auto r) {
                            const float gn = __builtin_fmaf(s.C[r], dv, G[r]);
                            G[r] = FAST || (in && g * R + r < N) ? gn : 0.0f;
                            sums[r] = G[r] * s.s.y;
                            sums[R + r] = h[i + 1][r] * dv;
                            gb = r == 0 ? G[0] * s.B[0] : __builtin_fmaf(G[r], s.B[r], gb);
                            const float back = av[i][r] * G[r];
                            float qv = back * (drop ? 0.0f : h[i][r]);
                            if (!FAST) qv = live ? qv : 0.0f;
                            dA[r] = __builtin_fmaf(qv, s.s.x, dA[r]);
                            aq = r == 0 ? qv * A2[0] : __builtin_fmaf(qv, A2[r], aq);
                            G[r] = drop ? 0.0f : back;
                        });
                        pq[i & 3] = aq;
                        pg[i & 3] = gb;
                        sum_channels<BITS - 1, 2 * R>(sums, lane);
                        static_for<LEFT>([&](auto e) { to[wid][i][g * 2 * R + first + e] = sums[e]; });
                        if constexpr ((i & 3) == 0) {
                            const float sq = sum_lanes4<L>(pq), sg = sum_lanes4<L>(pg);
                            back_sums[tc + i + (lane >> 4)][cl] = make_float2(sq, sg);
                        }
                    });
                    __syncthreads();
                    int id = tid;
                    if constexpr (LEAN) asm volatile("" : "+v"(id));
                    for (int idx = id; idx < CK * 2 * NP; idx += 256) {
                        const int i = idx / (2 * NP), at = idx % (2 * NP), gg = at / (2 * R), w = at % (2 * R) / R, n = gg * R + at % R;
                        float s = to[0][i][at];
                        static_for<kScanWaves - 1>([&](auto k1) { s += to[k1 + 1][i][at]; });
                        if (n < N && tc + i < left) a.bc_part[((blk * a.T + t0 + tc + i) * a.batch + b) * 2 * N + w * N + n] = s;
                    }
                }
            }
        };
        if (left == TT && reset == 0 && !wild) walk(std::true_type{});
        else walk(std::false_type{});
        if constexpr (SUM) {
            __syncthreads();
        } else {
            const Mine m = mine();
            float x[E], raw[E], zs[E], dys[E], odx[E], odt[E], odz[E];
            qx.unpack(x);
            qd.unpack(raw);
            qz.unpack(zs);
            qy.unpack(dys);
            static_for<E>([&](auto e) {
                const float4 s = dd[m.tr][m.pc + e];
                const float2 q = back_sums[m.tr][m.pc + e], w = par[m.pc + e];
                float z, omz;
                sigmoid_pair(raw[e] + w.x, z, omz);
                odt[e] = __builtin_fmaf(q.y, x[e], q.x * 0.69314718f) * z;
                odx[e] = __builtin_fmaf(w.y, s.z, s.x * q.y);
                odz[e] = 0.0f;
                if (a.dz.p) {
                    sigmoid_pair(zs[e], z, omz);
                    odz[e] = dys[e] * __builtin_fmaf(w.y, x[e], s.w) * (z * __builtin_fmaf(zs[e], omz, 1.0f));
                }
                const bool live = m.tr < left && e < m.valid;
                float2 own = own_sums[e][tid];
                own.x += live ? s.z * x[e] : 0.0f;
                own.y += live ? odt[e] : 0.0f;
                own_sums[e][tid] = own;
            });
            P::store(rdx.buffer(), offset(rdx, m, left), m.valid, odx);
            P::store(rdt.buffer(), offset(rdt, m, left), m.valid, odt);
            P::store(rdz.buffer(), offset(rdz, m, left), m.valid, odz);
            rdx.back();
            rdt.back();
            rdz.back();
        }
    }
    if constexpr (SUM) {
        if (!in) return;
        const int64_t at = (seg * a.batch + b) * a.D + ch;
        if (g == 0) a.seg_sum[at] = dropped ? -1.0f : __builtin_fabsf(total);
        static_for<R>([&](auto r) {
            if (g * R + r < N) a.seg_end[at * N + g * R + r] = G[r];
        });
    } else {
        const int64_t row = seg * a.batch + b, rows = a.segs * a.batch;
        if (in) static_for<R>([&](auto r) {
            const int n = g * R + r;
            if (n < N) {
                if (a.dh0 && seg == 0) a.dh0[(b * a.D + ch) * N + n] = G[r];
                if (a.dA) a.par_part[(row * a.D + ch) * N + n] = dA[r];
            }
        });
        if (!a.dskip && !a.ddt_bias) return;
        // the threads with the same channels: 32 rows of the tile
        __syncthreads();
        for (int i = tid; i < 2 * CH; i += 256) {
            const int which = i / CH, c = i % CH;
            float s = 0.0f;
            for (int t = 0; t < TT; ++t) {
                const float2 v = own_sums[c % E][t * S::PPR + c / E];
                s += which ? v.y : v.x;
            }
            if (c0 + c < a.D) a.par_part[rows * a.D * N + (which * rows + row) * a.D + c0 + c] = s;
        }
    }
}

// dB and dC: the sums of the workgroups' rows, in order.
template <int ES>
__global__ __launch_bounds__(256) void scan_bc_kernel(ScanArgs a, int64_t blocks) {
    const int64_t n2 = 2 * a.N, all = a.T * a.batch * n2;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
#pragma unroll 8
        for (int64_t k = 0; k < blocks; ++k) s += a.bc_part[k * all + i];
        const int64_t row = i / n2, n = i - row * n2, t = row / a.batch, b = row - t * a.batch;
        const ScanRows& r = n < a.N ? a.dB : a.dC;
        Row16<ES>::put(const_cast<void*>(r.p), b * r.sb + t * r.st + (n < a.N ? n : n - a.N), s);
    }
}

typedef void (*ScanFn)(ScanArgs);

template <int ES, bool VEC, bool SUM>
ScanFn scan_bwd_fn(const ScanShapeOf& s) {
    if (s.L == 4) return scan_bwd_kernel<ES, VEC, 4, 1, SUM>;
    if (s.L == 8) return s.R == 1 ? scan_bwd_kernel<ES, VEC, 8, 1, SUM> : scan_bwd_kernel<ES, VEC, 8, 2, SUM>;
    return s.R == 2 ? scan_bwd_kernel<ES, VEC, 16, 2, SUM> : scan_bwd_kernel<ES, VEC, 16, 4, SUM>;
}

}  // namespace

hipError_t launch_scan_backward(const ScanArgs& a, hipStream_t s) {
    const int64_t rows = a.segs * a.batch;
    hipError_t e;
    if (a.T > 0 && a.batch > 0) {
        const int64_t blocks = (a.D + scan_channels(a.N) - 1) / scan_channels(a.N), groups = a.batch * blocks;
        if (blocks > 0) {
            if (groups * a.segs > INT32_MAX) return hipErrorInvalidValue;
            const ScanShapeOf shape = scan_shape(a.N);
            auto ok = [&](const ScanRows& r) { return scan_pieces(r, a.D, a.N, a.type); };
            const bool vec = ok(a.x) && ok(a.dt) && ok(a.z) && ok(a.dy) && ok(a.dx) && ok(a.ddt) && ok(a.dz);
            if (a.segs > 1) {
                const ScanFn fn = a.type == kBF16 ? (vec ? scan_bwd_fn<2, true, true>(shape) : scan_bwd_fn<2, false, true>(shape))
                                                  : (vec ? scan_bwd_fn<4, true, true>(shape) : scan_bwd_fn<4, false, true>(shape));
                hipLaunchKernelGGL(fn, dim3((unsigned)(groups * (a.segs - 1))), dim3(256), 0, s, a);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
            const ScanFn fn = a.type == kBF16 ? (vec ? scan_bwd_fn<2, true, false>(shape) : scan_bwd_fn<2, false, false>(shape))
                                              : (vec ? scan_bwd_fn<4, true, false>(shape) : scan_bwd_fn<4, false, false>(shape));
            hipLaunchKernelGGL(fn, dim3((unsigned)(groups * a.segs)), dim3(256), 0, s, a);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        const int64_t n = (a.T * a.batch * 2 * a.N + 255) / 256;
        hipLaunchKernelGGL((a.type == kBF16 ? scan_bc_kernel<2> : scan_bc_kernel<4>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(256), 0,
                           s, a, blocks);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else if (a.dh0 && a.batch > 0) {
        if ((e = launch_scan_copy(a.dh_T, a.dh0, a.batch * a.D * a.N, s)) != hipSuccess) return e;
    }
    const int64_t sums = a.T > 0 ? rows : 0;
    ColSum all[3];
    int count = 0;
    if (a.dA) all[count++] = ColSum{a.par_part, a.dA, sums, a.D * a.N, 1, kF32};
    if (a.dskip) all[count++] = ColSum{a.par_part + rows * a.D * a.N, a.dskip, sums, a.D, 1, kF32};
    if (a.ddt_bias) all[count++] = ColSum{a.par_part + rows * a.D * (a.N + 1), a.ddt_bias, sums, a.D, 1, kF32};
    return count ? launch_colsum(all, count, s) : hipSuccess;
}

}  // namespace isam
