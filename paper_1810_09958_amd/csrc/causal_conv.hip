// The short causal convolution over time, and its gradient.
//
//   pre_t = bias + sum_{j < K} w[K-1-j] x_{t-j},  y_t = act(pre_t)     (inputs before a reset count as zeros)
//   e_t = dy_t act'(pre_t),  dx_s = sum_j w[K-1-j] e_{s+j},  dw[K-1-j] = sum_t e_t x_{t-j},  dbias = sum e_t
//
// Memory bounds both: one value read and one written forward, two and one backward, for K
// multiply-adds and the activation.  A thread takes a piece of E neighbouring channels (16 bytes
// forward) through a run of tokens with the last K - 1 inputs in registers, so a value is read once but
// for the K - 1 tokens before (backward also after) each run; four tokens are loaded while the four
// before them are used.  The gradient goes forward in time too: the K sums dx of the last tokens
// are kept in registers until they are complete, pre is formed again.  The gradients of w and bias are
// kept over a run, added over a workgroup's runs in LDS, and over workgroups by a second kernel.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

constexpr int kAhead = 4;  // tokens loaded together

// E values from p, `n` of them (the others zeros); any alignment of their own size.
template <int ES, int E>
struct Vals {
    static constexpr int B = E * ES;
    uint32_t w[(B + 3) / 4];
    __device__ __forceinline__ void load(const void* base, int64_t at, int n) {
        const char* const p = static_cast<const char*>(base) + at * ES;
        static_for<(B + 3) / 4>([&](auto k) { w[k] = 0; });
        if (n >= E) {
            __builtin_memcpy(w, p, B);
        } else {
            static_for<E>([&](auto e) {
                if (e < n) {
                    if constexpr (ES == 2) w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
                    else w[e] = reinterpret_cast<const uint32_t*>(p)[e];
                }
            });
        }
    }
    __device__ __forceinline__ void zero() { static_for<(B + 3) / 4>([&](auto k) { w[k] = 0; }); }
    __device__ __forceinline__ void get(float (&f)[E]) const {
        static_for<E>([&](auto e) {
            if constexpr (ES == 4) f[e] = __uint_as_float(w[e]);
            else if constexpr (e & 1) f[e] = bf16hi(w[e / 2]);
            else f[e] = bf16lo(w[e / 2]);
        });
    }
    // bf16: rounded to nearest even.
    __device__ __forceinline__ static void store(void* base, int64_t at, int n, const float (&f)[E]) {
        char* const p = static_cast<char*>(base) + at * ES;
        uint32_t o[(B + 3) / 4];
        static_for<(B + 3) / 4>([&](auto k) {
            if constexpr (ES == 4) o[k] = __float_as_uint(f[k]);
            else o[k] = pack_bf16_rne(f[2 * k], f[2 * k + 1]);
        });
        if (n >= E) {
            __builtin_memcpy(p, o, B);
        } else {
            static_for<E>([&](auto e) {
                if (e < n) {
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
                    else reinterpret_cast<uint32_t*>(p)[e] = o[e];
                }
            });
        }
    }
};

// Where a thread stands: channels c .. c + n, sequence b, tokens [t0, t1).
template <int E>
struct Place {
    int64_t c, b, t0, t1;
    int n;
    __device__ __forceinline__ explicit Place(const ConvArgs& a) {
        const int64_t cblocks = (a.C + a.lanes * E - 1) / (a.lanes * E), id = blockIdx.x;
        const int64_t tb = id / (cblocks * a.batch), rest = id - tb * cblocks * a.batch;
        b = rest / cblocks;
        c = ((rest - b * cblocks) * a.lanes + threadIdx.x % a.lanes) * E;
        t0 = (tb * (256 / a.lanes) + threadIdx.x / a.lanes) * a.run;
        t1 = min(a.T, t0 + a.run);
        n = (int)max((int64_t)0, min((int64_t)E, a.C - c));
    }
};

__device__ __forceinline__ bool marked(const ConvArgs& a, int64_t t, int64_t b) {
    return a.reset && t >= 0 && t < a.T && a.reset[t * a.rs_t + b * a.rs_b] != 0;
}

// The K - 1 inputs before token t as token t - 1 saw them: x[j - 1] is that of t - j, zero where a reset
// lies after it (or nothing is kept); seen[j - 1]: none does.
template <int ES, int K, int E>
__device__ __forceinline__ void before(const ConvArgs& a, const Place<E>& at, int64_t t, float (&x)[K > 1 ? K - 1 : 1][E],
                                       bool (&seen)[K > 1 ? K - 1 : 1]) {
    bool open = true;
    static_for<K - 1>([&](auto i) {
        const int64_t s = t - 1 - i;
        Vals<ES, E> v;
        if (s >= 0) v.load(a.x.p, s * a.x.st + at.b * a.x.sb + at.c, at.n);
        else if (a.state) v.load(a.state, ((K - 1 + s) * a.batch + at.b) * a.C + at.c, at.n);
        else v.zero();
        v.get(x[i]);
        static_for<E>([&](auto e) { x[i][e] = open ? x[i][e] : 0.0f; });
        seen[i] = open;
        open = open && !marked(a, s, at.b);
    });
}

template <int ES, int K, int E>
__global__ __launch_bounds__(256) void conv_fwd_kernel(ConvArgs a) {
    const Place<E> at(a);
    if (at.n == 0 || at.t0 >= at.t1) return;
    float w[K][E], bias[E];
    static_for<E>([&](auto e) {
        const bool on = e < at.n;
        bias[e] = on && a.bias ? a.bias[at.c + e] : 0.0f;
        static_for<K>([&](auto k) { w[k][e] = on ? a.w[k * a.C + at.c + e] : 0.0f; });
    });
    float x[K > 1 ? K - 1 : 1][E];
    bool seen[K > 1 ? K - 1 : 1];
    Vals<ES, E> next[kAhead];
    bool mark[kAhead];
    auto fetch = [&](int64_t t) {
        static_for<kAhead>([&](auto i) {
            next[i].zero();
            mark[i] = false;
            if (t + i < at.t1) {
                next[i].load(a.x.p, (t + i) * a.x.st + at.b * a.x.sb + at.c, at.n);
                mark[i] = marked(a, t + i, at.b);
            }
        });
    };
    fetch(at.t0);
    before<ES, K, E>(a, at, at.t0, x, seen);
    for (int64_t t = at.t0; t < at.t1; t += kAhead) {
        float now[kAhead][E];
        bool cut[kAhead];
        static_for<kAhead>([&](auto i) {
            next[i].get(now[i]);
            cut[i] = mark[i];
        });
        fetch(t + kAhead);
        static_for<kAhead>([&](auto i) {
            if (t + i < at.t1) {
                float y[E];
                static_for<E>([&](auto e) {
                    float p = __builtin_fmaf(w[K - 1][e], now[i][e], bias[e]);
                    static_for<K - 1>([&](auto j) {
                        x[j][e] = cut[i] ? 0.0f : x[j][e];
                        p = __builtin_fmaf(w[K - 2 - j][e], x[j][e], p);
                    });
                    y[e] = p;
                    if (a.act) {
                        float z, omz;
                        sigmoid_pair(p, z, omz);
                        y[e] *= z;
                    }
                    static_for<K - 1>([&](auto j) {
                        constexpr int to = K - 2 - decltype(j)::value;
                        x[to][e] = to == 0 ? now[i][e] : x[to > 0 ? to - 1 : 0][e];
                    });
                });
                if (a.y.p) Vals<ES, E>::store(const_cast<void*>(a.y.p), (t + i) * a.y.st + at.b * a.y.sb + at.c, at.n, y);
            }
        });
    }
    if (a.state_T && at.t1 == a.T)
        static_for<K - 1>([&](auto j) { Vals<ES, E>::store(a.state_T, ((K - 2 - j) * a.batch + at.b) * a.C + at.c, at.n, x[j]); });
}

template <int ES, int K, int E>
__global__ __launch_bounds__(256, 2) void conv_bwd_kernel(ConvArgs a) {
    __shared__ float sums[256 * E];
    const Place<E> at(a);
    float dw[K][E], db[E];
    static_for<E>([&](auto e) {
        db[e] = 0.0f;
        static_for<K>([&](auto k) { dw[k][e] = 0.0f; });
    });
    if (at.n > 0 && at.t0 < at.t1) {
        float w[K][E], bias[E];
        static_for<E>([&](auto e) {
            const bool on = e < at.n;
            bias[e] = on && a.bias ? a.bias[at.c + e] : 0.0f;
            static_for<K>([&](auto k) { w[k][e] = on ? a.w[k * a.C + at.c + e] : 0.0f; });
        });
        float x[K > 1 ? K - 1 : 1][E], dx[K][E];  // dx[j]: of token t - j
        bool seen[K > 1 ? K - 1 : 1];
        Vals<ES, E> nx[kAhead], nd[kAhead];
        bool mark[kAhead];
        const int64_t end = min(a.T, at.t1 + K - 1);  // the tokens that see this run's inputs
        auto fetch = [&](int64_t t) {
            static_for<kAhead>([&](auto i) {
                nx[i].zero();
                nd[i].zero();
                mark[i] = false;
                if (t + i < end) {
                    nx[i].load(a.x.p, (t + i) * a.x.st + at.b * a.x.sb + at.c, at.n);
                    if (a.dy.p) nd[i].load(a.dy.p, (t + i) * a.dy.st + at.b * a.dy.sb + at.c, at.n);
                    mark[i] = marked(a, t + i, at.b);
                }
            });
        };
        // dx of token s is complete: a row of dx, or of dstate before the first token
        auto done = [&](int64_t s, const float (&v)[E]) {
            if (s >= at.t0 && s < at.t1) {
                if (a.dx.p) Vals<ES, E>::store(const_cast<void*>(a.dx.p), s * a.dx.st + at.b * a.dx.sb + at.c, at.n, v);
            } else if (s < 0 && s >= -(K - 1) && at.t0 == 0 && a.dstate) {
                Vals<ES, E>::store(a.dstate, ((K - 1 + s) * a.batch + at.b) * a.C + at.c, at.n, v);
            }
        };
        fetch(at.t0);
        before<ES, K, E>(a, at, at.t0, x, seen);
        static_for<K>([&](auto j) { static_for<E>([&](auto e) { dx[j][e] = 0.0f; }); });
        for (int64_t t = at.t0; t < end; t += kAhead) {
            float now[kAhead][E], dy[kAhead][E];
            bool cut[kAhead];
            static_for<kAhead>([&](auto i) {
                nx[i].get(now[i]);
                nd[i].get(dy[i]);
                cut[i] = mark[i];
            });
            fetch(t + kAhead);
            static_for<kAhead>([&](auto i) {
                if (t + i < end) {
                    const bool own = t + i < at.t1;
                    static_for<K - 1>([&](auto j) { seen[j] = seen[j] && !cut[i]; });
                    static_for<E>([&](auto e) {
                        float p = __builtin_fmaf(w[K - 1][e], now[i][e], bias[e]);
                        static_for<K - 1>([&](auto j) {
                            x[j][e] = cut[i] ? 0.0f : x[j][e];
                            p = __builtin_fmaf(w[K - 2 - j][e], x[j][e], p);
                        });
                        float g = dy[i][e];
                        if (a.act) {
                            float z, omz;
                            sigmoid_pair(p, z, omz);
                            g *= z * __builtin_fmaf(p, omz, 1.0f);
                        }
                        const float mine = own ? g : 0.0f;
                        db[e] += mine;
                        dw[K - 1][e] = __builtin_fmaf(mine, now[i][e], dw[K - 1][e]);
                        dx[0][e] = w[K - 1][e] * g;
                        static_for<K - 1>([&](auto j) {
                            dw[K - 2 - j][e] = __builtin_fmaf(mine, x[j][e], dw[K - 2 - j][e]);
                            dx[j + 1][e] = __builtin_fmaf(w[K - 2 - j][e], seen[j] ? g : 0.0f, dx[j + 1][e]);
                        });
                    });
                    done(t + i - (K - 1), dx[K - 1]);
                    static_for<K - 1>([&](auto j) {
                        constexpr int to = K - 1 - decltype(j)::value;
                        static_for<E>([&](auto e) { dx[to][e] = dx[to - 1][e]; });
                    });
                    static_for<K - 1>([&](auto j) {
                        constexpr int to = K - 2 - decltype(j)::value;
                        seen[to] = to == 0 ? true : seen[to > 0 ? to - 1 : 0];
                        static_for<E>([&](auto e) { x[to][e] = to == 0 ? now[i][e] : x[to > 0 ? to - 1 : 0][e]; });
                    });
                }
            });
        }
        // what the inputs kept for the next call pass back (dx[j], j > 0: of token end - j)
        if (end == a.T) {
            static_for<K - 1>([&](auto j) {
                Vals<ES, E> v;
                float kept[E];
                v.zero();
                if (a.dstate_T) v.load(a.dstate_T, ((K - 2 - j) * a.batch + at.b) * a.C + at.c, at.n);
                v.get(kept);
                static_for<E>([&](auto e) { dx[j + 1][e] += seen[j] ? kept[e] : 0.0f; });
                done(a.T - 1 - j, dx[j + 1]);
            });
        }
    }
    if (!a.dw && !a.dbias) return;
    // one row of partial sums for a workgroup's runs
    const int64_t cblocks = (a.C + a.lanes * E - 1) / (a.lanes * E), row = blockIdx.x / cblocks, cb = blockIdx.x - row * cblocks;
    const int cols = a.lanes * E, runs = 256 / a.lanes;
    static_for<K + 1>([&](auto k) {
        __syncthreads();
        static_for<E>([&](auto e) { sums[threadIdx.x * E + e] = k < K ? dw[k < K ? decltype(k)::value : 0][e] : db[e]; });
        __syncthreads();
        for (int i = threadIdx.x; i < cols; i += 256) {
            const int64_t c = cb * cols + i;
            float s = 0.0f;
            for (int r = 0; r < runs; ++r) s += sums[r * cols + i];
            if (c < a.C) a.part[k < K ? row * K * a.C + k * a.C + c : a.rows * K * a.C + row * a.C + c] = s;
        }
    });
}

// T == 0: dst = src, or zeros.
template <int ES>
__global__ __launch_bounds__(256) void conv_copy_kernel(const void* src, void* dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        if constexpr (ES == 2) static_cast<uint16_t*>(dst)[i] = src ? static_cast<const uint16_t*>(src)[i] : (uint16_t)0;
        else static_cast<uint32_t*>(dst)[i] = src ? static_cast<const uint32_t*>(src)[i] : 0u;
    }
}

typedef void (*ConvFn)(ConvArgs);

// Channels of a piece: 16 bytes forward up to four taps, four channels where the registers are needed
// otherwise (a piece past the last channel is moved value by value).
constexpr int piece(int es, int K, bool backward) { return !backward && es == 2 && K <= 4 ? 8 : 4; }

template <int ES, bool BWD, int K>
ConvFn conv_fn() {
    if constexpr (BWD) return conv_bwd_kernel<ES, K, piece(ES, K, BWD)>;
    else return conv_fwd_kernel<ES, K, piece(ES, K, BWD)>;
}
template <int ES, bool BWD>
ConvFn conv_fn(int64_t K) {
    switch (K) {
        case 1: return conv_fn<ES, BWD, 1>();
        case 2: return conv_fn<ES, BWD, 2>();
        case 3: return conv_fn<ES, BWD, 3>();
        case 4: return conv_fn<ES, BWD, 4>();
        case 5: return conv_fn<ES, BWD, 5>();
        default: return conv_fn<ES, BWD, 6>();
    }
}

}  // namespace

// Lanes, run and rows of partial sums for these sizes.
void conv_plan(ConvArgs& a, bool backward, int cus) {
    const int64_t E = piece(a.type == kBF16 ? 2 : 4, (int)a.K, backward), pieces = (a.C + E - 1) / E;
    a.lanes = 1;
    while (a.lanes < 64 && a.lanes < pieces) a.lanes *= 2;
    const int64_t cblocks = (pieces + a.lanes - 1) / a.lanes, per = 256 / a.lanes;
    // runs as long as leave four workgroups to a compute unit; eight tokens at least
    auto blocks = [&](int64_t run) { return cblocks * a.batch * ((a.T + run * per - 1) / (run * per)); };
    a.run = 64;
    while (a.run > 8 && blocks(a.run) < 4 * (int64_t)cus) a.run /= 2;
    a.rows = a.batch * ((a.T + a.run * per - 1) / (a.run * per));
}

hipError_t launch_causal_conv(const ConvArgs& a, bool backward, hipStream_t s) {
    const int64_t E = piece(a.type == kBF16 ? 2 : 4, (int)a.K, backward);
    hipError_t e = hipSuccess;
    if (a.T > 0 && a.batch > 0) {
        const int64_t blocks = a.rows * ((a.C + a.lanes * E - 1) / (a.lanes * E));
        if (blocks > INT32_MAX) return hipErrorInvalidValue;
        const ConvFn fn = backward ? (a.type == kBF16 ? conv_fn<2, true>(a.K) : conv_fn<4, true>(a.K))
                                   : (a.type == kBF16 ? conv_fn<2, false>(a.K) : conv_fn<4, false>(a.K));
        hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(256), 0, s, a);
        e = hipGetLastError();
    } else {
        void* const to = backward ? a.dstate : a.state_T;
        const int64_t n = (a.K - 1) * a.batch * a.C, blocks = (n + 255) / 256;
        if (to && n > 0) {
            hipLaunchKernelGGL((a.type == kBF16 ? conv_copy_kernel<2> : conv_copy_kernel<4>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)),
                               dim3(256), 0, s, backward ? a.dstate_T : a.state, to, n);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess || !backward) return e;
    ColSum sums[2];
    int count = 0;
    const int64_t rows = a.T > 0 ? a.rows : 0;
    if (a.dw) sums[count++] = ColSum{a.part, a.dw, rows, a.K * a.C, 1, kF32};
    if (a.dbias) sums[count++] = ColSum{a.part + a.rows * a.K * a.C, a.dbias, rows, a.C, 1, kF32};
    return count ? launch_colsum(sums, count, s) : hipSuccess;
}

}  // namespace isam
