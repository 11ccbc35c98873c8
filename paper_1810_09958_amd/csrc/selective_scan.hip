// The selective scan forward: tokens in tiles, single tokens, and the segments' summaries.
#include <algorithm>

#include "selective_scan.hpp"

namespace isam {

namespace {

// One workgroup: channels [block * CH, +CH) of one sequence over one segment of time.  SUM: only
// the state at the segment's end, from zero, and the sum of its steps.
template <int ES, bool VEC, int L, int R, bool SUM>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a) {
    using S = ScanShape<ES, VEC, L, R>;
    using P = typename S::P;
    constexpr int CH = S::CH, E = S::E, NP = S::NP, TT = kScanTile;
    __shared__ __attribute__((aligned(16))) float2 dd[TT][CH];          // d, d x; then v in .x
    __shared__ __attribute__((aligned(16))) float bc[TT * NP * 2];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane / S::CW, cl = wid * S::CW + lane % S::CW;        // group of n, channel in the workgroup
    const int64_t blocks = (a.D + CH - 1) / CH;
    const int64_t seg = blockIdx.x / (a.batch * blocks), rest = blockIdx.x - seg * a.batch * blocks;
    const int64_t b = rest / blocks, c0 = (rest - b * blocks) * CH, ch = c0 + cl;
    const int64_t tbeg = seg * a.seg_len, tend = min(a.T, tbeg + a.seg_len);
    const bool in = ch < a.D;
    const int N = (int)a.N;

    float A2[R], h[R];
    static_for<R>([&](auto r) {
        const int n = g * R + r;
        const bool on = in && n < N;
        A2[r] = on ? a.A[ch * N + n] * kScanLog2e : 0.0f;
        h[r] = 0.0f;
        if (!SUM && on) {
            h[r] = a.h0 ? a.h0[(b * a.D + ch) * N + n] : 0.0f;
#pragma unroll 4
            for (int64_t s = 0; s < seg; ++s) {
                const int64_t at = (s * a.batch + b) * a.D + ch;
                h[r] = pass_on(a.seg_sum[at], A2[r], h[r], a.seg_end[at * N + n]);
            }
        }
    });

    // this thread's piece of a tile: row tr, channels c0 + pc .. + E
    const int tr = tid / S::PPR, pc = (tid % S::PPR) * E;
    const int valid = (int)max((int64_t)0, min((int64_t)E, a.D - (c0 + pc)));
    float bias[E], skip[E];
    static_for<E>([&](auto e) {
        bias[e] = a.dt_bias && e < valid ? a.dt_bias[c0 + pc + e] : 0.0f;
        skip[e] = a.skip && e < valid ? a.skip[c0 + pc + e] : 0.0f;
    });
    TileRows<ES> rx(a.x, b, tbeg), rd(a.dt, b, tbeg), rz(a.z, b, tbeg), rB(a.B, b, tbeg), rC(a.C, b, tbeg), ry(a.y, b, tbeg);
    auto offset = [&](const TileRows<ES>& r, int left) {
        return tr < left && valid > 0 ? (uint32_t)tr * r.row + (uint32_t)((c0 + pc) * ES) : kOob;
    };
    P px, pd, pz;
    ScanWeights<ES, NP> wb, wc;
    ScanMarks marks;
    auto fetch = [&](int64_t t0) {
        const int left = (int)max((int64_t)0, min((int64_t)TT, tend - t0));
        px.load(rx.buffer(), offset(rx, left), valid);
        pd.load(rd.buffer(), offset(rd, left), valid);
        wb.load(rB.buffer(), rB.row, N, left, tid);
        rx.forth();
        rd.forth();
        rB.forth();
        if constexpr (!SUM) {
            pz.load(rz.buffer(), rz.p ? offset(rz, left) : kOob, valid);
            wc.load(rC.buffer(), rC.row, N, left, tid);
            rz.forth();
            rC.forth();
        }
        marks.load(a, b, t0, left, lane);
    };
    fetch(tbeg);
    float total = 0.0f;
    bool dropped = false;
    for (int64_t t0 = tbeg; t0 < tend; t0 += TT) {
        const int left = (int)min((int64_t)TT, tend - t0);
        float x[E], zs[E];
        bool wild = false;
        px.unpack(x);
        {
            float d[E];
            pd.unpack(d);
            static_for<E>([&](auto e) {
                const float step = tr < left && e < valid ? softplus(d[e] + bias[e]) : 0.0f;
                dd[tr][pc + e] = make_float2(step, step * x[e]);
                wild = wild || not_finite(step * x[e]);
            });
        }
        wb.template put<R>(bc, 0, tid);
        if constexpr (!SUM) {
            wc.template put<R>(bc, 1, tid);
            pz.unpack(zs);
        }
        const uint32_t reset = marks.bits();
        fetch(t0 + TT);  // (past the end: zeros)
        wild = meet(N != NP, wild);
        // FAST: a whole tile without a reset (or an infinity that would reach the padding of N).  The next four tokens' values are on their way from LDS while
        // four are walked.
        auto walk = [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
            using Token = ScanToken<L, R, !SUM>;
            Token next[4];
            auto ahead = [&](int q) { static_for<4>([&](auto i) { next[i].get(dd[q + i][cl], bc, q + i, g); }); };
            ahead(0);
#pragma unroll 2
            for (int q = 0; q < TT; q += 4) {
                Token now[4];
                static_for<4>([&](auto i) { now[i] = next[i]; });
                ahead(q + 4 < TT ? q + 4 : q);
                __builtin_amdgcn_sched_barrier(0);
                if (!SUM && (q & (S::CK - 1)) == 0 && a.states && (FAST || q < left)) {
                    float* const to = a.states + (((t0 + q) / S::CK * a.batch + b) * a.D + ch) * N + g * R;
                    static_for<R>([&](auto r) {
                        if (in && g * R + r < N) to[r] = h[r];
                    });
                }
                float p[4];
                static_for<4>([&](auto i) {
                    const int t = q + i;
                    const Token& v = now[i];
                    const bool drop = !FAST && (reset >> t & 1), live = FAST || t < left;
                    float acc = 0.0f;
                    static_for<R>([&](auto r) {
                        const float av = __builtin_amdgcn_exp2f(v.s.x * A2[r]);
                        const float hb = drop ? 0.0f : h[r];
                        const float hn = __builtin_fmaf(av, hb, v.s.y * v.B[r]);
                        h[r] = FAST || (live && g * R + r < N) ? hn : h[r];
                        if constexpr (!SUM) acc = r == 0 ? v.C[0] * h[0] : __builtin_fmaf(v.C[r], h[r], acc);
                    });
                    p[i] = acc;
                    if constexpr (SUM) {
                        total = drop ? v.s.x : total + v.s.x;
                        dropped = dropped || drop;
                    }
                });
                if constexpr (!SUM) {
                    // (each wave reads and writes its own channels' places)
                    const float v = sum_lanes4<L>(p);
                    dd[q + (lane >> 4)][cl].x = v;
                }
            }
        };
        if (left == TT && reset == 0 && !wild) walk(std::true_type{});
        else walk(std::false_type{});
        __syncthreads();
        if constexpr (!SUM) {
            float y[E];
            static_for<E>([&](auto e) {
                y[e] = __builtin_fmaf(skip[e], x[e], dd[tr][pc + e].x);
                if (a.z.p) {
                    float z, omz;
                    sigmoid_pair(zs[e], z, omz);
                    y[e] *= zs[e] * z;
                }
            });
            P::store(ry.buffer(), ry.p ? offset(ry, left) : kOob, valid, y);
            ry.forth();
        }
    }
    if (!in) return;
    if constexpr (SUM) {
        const int64_t at = (seg * a.batch + b) * a.D + ch;
        if (g == 0) a.seg_sum[at] = dropped ? -1.0f : __builtin_fabsf(total);  // (a NaN without its sign)
        static_for<R>([&](auto r) {
            if (g * R + r < N) a.seg_end[at * N + g * R + r] = h[r];
        });
    } else if (a.h_T && tend == a.T) {
        static_for<R>([&](auto r) {
            if (g * R + r < N) a.h_T[(b * a.D + ch) * N + g * R + r] = h[r];
        });
    }
}

// A few tokens: decoding.  G lanes to a channel (a power of two), four values of n to a lane, the
// state read and written once; h_T may be h0.  Bound by one pass over the state.
template <int ES, int G>
__global__ __launch_bounds__(256) void scan_few_kernel(ScanArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / G;                       // (b, channel)
    const int g = (int)(i % G), N = (int)a.N, T = (int)a.T, n0 = 4 * g;
    const bool in = row < a.batch * a.D;
    const int64_t b = in ? row / a.D : 0, ch = in ? row - b * a.D : 0;
    const bool whole = (N & 3) == 0;
    float A2[4], h[4];
    auto get4 = [&](const float* p, float (&f)[4]) {
        if (whole && n0 < N) {
            __builtin_memcpy(f, p + n0, 16);
        } else {
            static_for<4>([&](auto r) { f[r] = n0 + r < N ? p[n0 + r] : 0.0f; });
        }
    };
    auto put4 = [&](float* p) {
        if (!in || n0 >= N) return;
        if (whole) __builtin_memcpy(p + n0, h, 16);
        else static_for<4>([&](auto r) { if (n0 + r < N) p[n0 + r] = h[r]; });
    };
    const int64_t at = (b * a.D + ch) * N;
    get4(a.A + ch * N, A2);
    static_for<4>([&](auto r) { A2[r] *= kScanLog2e; });
    if (a.h0) get4(a.h0 + at, h);
    else static_for<4>([&](auto r) { h[r] = 0.0f; });
    if (a.states && T > 0) put4(a.states + at);
    const float bias = a.dt_bias ? a.dt_bias[ch] : 0.0f, skip = a.skip ? a.skip[ch] : 0.0f;
    auto row_get4 = [&](const ScanRows& r, int64_t at, float (&f)[4]) {
        const char* const p = static_cast<const char*>(r.p) + (at + n0) * ES;
        if (n0 + 4 <= N) {
            uint32_t w[ES];
            __builtin_memcpy(w, p, 4 * ES);
            static_for<4>([&](auto e) {
                if constexpr (ES == 4) f[e] = __uint_as_float(w[e]);
                else f[e] = e & 1 ? bf16hi(w[e / 2]) : bf16lo(w[e / 2]);
            });
        } else {
            static_for<4>([&](auto e) { f[e] = n0 + e < N ? Row16<ES>::get(r.p, at + n0 + e) : 0.0f; });
        }
    };
    for (int t = 0; t < T; ++t) {
        auto row_at = [&](const ScanRows& r) { return b * r.sb + t * r.st; };
        float Bv[4], Cv[4];
        row_get4(a.B, row_at(a.B), Bv);
        row_get4(a.C, row_at(a.C), Cv);
        const float x = Row16<ES>::get(a.x.p, row_at(a.x) + ch), raw = Row16<ES>::get(a.dt.p, row_at(a.dt) + ch);
        const float zv = a.z.p ? Row16<ES>::get(a.z.p, row_at(a.z) + ch) : 0.0f;
        const bool drop = a.reset && a.reset[t * a.rs_t + b * a.rs_b];
        const float d = softplus(raw + bias);
        float v = 0.0f;
        static_for<4>([&](auto r) {
            h[r] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * A2[r]), drop ? 0.0f : h[r], d * x * Bv[r]);
            v = n0 + r < N ? __builtin_fmaf(Cv[r], h[r], v) : v;
        });
        static_for<4>([&](auto k) {
            constexpr int m = 1 << decltype(k)::value;
            if constexpr (m < G) v += __shfl_xor(v, m);
        });
        v = __builtin_fmaf(skip, x, v);
        if (a.z.p) {
            float z, omz;
            sigmoid_pair(zv, z, omz);
            v *= zv * z;
        }
        if (a.y.p && in && g == 0) Row16<ES>::put(const_cast<void*>(a.y.p), row_at(a.y) + ch, v);
    }
    if (a.h_T) put4(a.h_T + at);
}

// dst = src, or zeros.
__global__ __launch_bounds__(256) void scan_copy_kernel(const float* src, float* dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) dst[i] = src ? src[i] : 0.0f;
}

typedef void (*ScanFn)(ScanArgs);

template <int ES, bool VEC, bool SUM>
ScanFn scan_fn(const ScanShapeOf& s) {
    if (s.L == 4) return scan_kernel<ES, VEC, 4, 1, SUM>;
    if (s.L == 8) return s.R == 1 ? scan_kernel<ES, VEC, 8, 1, SUM> : scan_kernel<ES, VEC, 8, 2, SUM>;
    return s.R == 2 ? scan_kernel<ES, VEC, 16, 2, SUM> : scan_kernel<ES, VEC, 16, 4, SUM>;
}

template <int ES>
hipError_t launch_few(const ScanArgs& a, hipStream_t s) {
    const int G = a.N <= 4 ? 1 : a.N <= 8 ? 2 : a.N <= 16 ? 4 : a.N <= 32 ? 8 : 16;
    const int64_t blocks = (a.batch * a.D * G + 255) / 256;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const ScanFn fn = G == 1 ? scan_few_kernel<ES, 1> : G == 2 ? scan_few_kernel<ES, 2> : G == 4 ? scan_few_kernel<ES, 4>
                    : G == 8 ? scan_few_kernel<ES, 8> : scan_few_kernel<ES, 16>;
    hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t scan_channels(int64_t N) { return kScanWaves * 64 / scan_shape(N).L; }

// Whether the rows of r are whole pieces of the tile's threads, on 4 bytes.
bool scan_pieces(const ScanRows& r, int64_t D, int64_t N, int type) {
    const int64_t e = scan_channels(N) * kScanTile / 256;
    return !r.p || (D % e == 0 && (type == kF32 || ((uintptr_t)r.p % 4 == 0 && r.st % 2 == 0 && r.sb % 2 == 0)));
}

// Segments of time, tiles of 32 tokens shared out over them: as many as make four workgroups to a compute unit, of two
// tiles at least, where the channels alone make fewer than two.  us forward / backward of 1, 2, 4, 8, 16 segments
// (workgroups of one; bf16, N 16): 512x2x1024 (64) 43, 39, 25, 21, 25 / 131, 93, 58, 48, 54; 4096x1x1024 (32)
// 301, -, 133, 73, 55 / 922, -, 309, 169, 122; 4096x2x2048 (128) 301, 255, 174, 156, 150 / 973, 633, 414, 404, 409;
// 2048x8x1024 (256) 161, 166, 150, 146 / 524, 419, 404, 412; 2048x8x2048 (512) 245, 257, 264, 277 / 678, 737, 745, 770.
int64_t scan_segments(int64_t T, int64_t batch, int64_t D, int64_t N, int cus) {
    if (T <= kScanFew) return 1;
    const int64_t groups = batch * ((D + scan_channels(N) - 1) / scan_channels(N)), tiles = (T + kScanTile - 1) / kScanTile;
    if (groups >= 2 * (int64_t)cus || tiles < 4) return 1;
    const int64_t segs = std::min({(4 * (int64_t)cus + groups - 1) / groups, tiles / 2, kScanMaxSegments});
    const int64_t per = (tiles + segs - 1) / segs;
    return (tiles + per - 1) / per;
}
int64_t scan_segment_length(int64_t T, int64_t segs) {
    const int64_t tiles = (T + kScanTile - 1) / kScanTile;
    return (tiles + segs - 1) / segs * kScanTile;
}

hipError_t launch_scan_copy(const float* src, float* dst, int64_t n, hipStream_t s) {
    const int64_t blocks = (n + 255) / 256;
    hipLaunchKernelGGL(scan_copy_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, src, dst, n);
    return hipGetLastError();
}

hipError_t launch_scan_forward(const ScanArgs& a, hipStream_t s) {
    if (a.T == 0) return a.h_T ? launch_scan_copy(a.h0, a.h_T, a.batch * a.D * a.N, s) : hipSuccess;
    if (a.T <= kScanFew) return a.type == kBF16 ? launch_few<2>(a, s) : launch_few<4>(a, s);
    const int64_t groups = a.batch * ((a.D + scan_channels(a.N) - 1) / scan_channels(a.N));
    if (groups * a.segs > INT32_MAX) return hipErrorInvalidValue;
    const ScanShapeOf shape = scan_shape(a.N);
    auto ok = [&](const ScanRows& r) { return scan_pieces(r, a.D, a.N, a.type); };
    const bool vec = ok(a.x) && ok(a.dt) && ok(a.z) && ok(a.y);
    if (a.segs > 1) {
        const ScanFn fn = a.type == kBF16 ? (vec ? scan_fn<2, true, true>(shape) : scan_fn<2, false, true>(shape))
                                          : (vec ? scan_fn<4, true, true>(shape) : scan_fn<4, false, true>(shape));
        hipLaunchKernelGGL(fn, dim3((unsigned)(groups * (a.segs - 1))), dim3(256), 0, s, a);  // (nobody asks for the last one's)
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const ScanFn fn = a.type == kBF16 ? (vec ? scan_fn<2, true, false>(shape) : scan_fn<2, false, false>(shape))
                                      : (vec ? scan_fn<4, true, false>(shape) : scan_fn<4, false, false>(shape));
    hipLaunchKernelGGL(fn, dim3((unsigned)(groups * a.segs)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace isam
