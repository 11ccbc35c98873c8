// The short causal convolution over time, and its gradient.
//
//   pre_t = bias + sum_{j < K} w[K-1-j] x_{t-j},  y_t = act(pre_t)     (inputs before a reset count as zeros)
//   e_t = dy_t act'(pre_t),  dx_s = sum_j w[K-1-j] e_{s+j},  dw[K-1-j] = sum_t e_t x_{t-j},  dbias = sum e_t
//
// Memory bounds both: one value read and one written forward, two and one backward, for K
// multiply-adds and the activation.  A thread takes a piece of 8 bytes of neighbouring channels through a
// run of tokens with the last K - 1 inputs in registers, so a value is read once but for the K - 1 tokens before
// (backward also after) each run; the next eight tokens are on their way while one is used, as the bytes in flight
// decide the rate.  The lanes of a wave are at one token, so that all but a lane's place in the row is scalar.
// The gradient goes forward in time too: the K sums dx of the last tokens are kept in registers until
// they are complete, pre is formed again.  The gradients of w and bias are kept over a run, added over a
// workgroup's four runs in LDS, and over workgroups by a second kernel.
// 4096x8x2048 (tokens, sequences, channels), K = 4, silu, bf16, resets, in a kernel trace: forward 60 us, 4.5 TB/s (268 MB),
// backward 127 and 4.9 for the sums (403 MB, 3.2 TB/s; the vector units are busy for 53 and 58 % of it, with the silu and,
// backward, its slope; 150 registers leave the gradient three waves a SIMD).  One token of 32x2048: 4.5 us.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

constexpr int kAhead = 8;  // tokens on their way

// E neighbouring values of a row, moved as one (gfx950 serves accesses at any alignment of the values).
template <int ES, int E>
struct Vals {
    static constexpr int B = E * ES;
    uint32_t w[(B + 3) / 4];
    __device__ __forceinline__ void load(const char* p) {
        if constexpr (B < 4) w[0] = *reinterpret_cast<const uint16_t*>(p);
        else __builtin_memcpy(w, p, B);
    }
    __device__ __forceinline__ void zero() { static_for<(B + 3) / 4>([&](auto k) { w[k] = 0; }); }
    __device__ __forceinline__ void get(float (&f)[E]) const {
        static_for<E>([&](auto e) {
            if constexpr (ES == 4) f[e] = __uint_as_float(w[e]);
            else if constexpr (e & 1) f[e] = bf16hi(w[e / 2]);
            else f[e] = bf16lo(w[e / 2]);
        });
    }
    // Values from `from` on.  bf16: rounded to nearest even.
    __device__ __forceinline__ static void store(char* p, int from, const float (&f)[E]) {
        uint32_t o[(B + 3) / 4];
        static_for<(B + 3) / 4>([&](auto k) {
            if constexpr (ES == 4) o[k] = __float_as_uint(f[k]);
            else if constexpr (E == 1) o[k] = pack_bf16_rne(f[0], 0.0f);
            else o[k] = pack_bf16_rne(f[2 * k], f[2 * k + 1]);
        });
        if (from == 0) {
            if constexpr (B < 4) *reinterpret_cast<uint16_t*>(p) = (uint16_t)o[0];
            else __builtin_memcpy(p, o, B);
        } else {
            static_for<E>([&](auto e) {
                if (e >= from) {
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
                    else reinterpret_cast<uint32_t*>(p)[e] = o[e];
                }
            });
        }
    }
};

// Where a thread stands: channels c .. c + E of sequence b, of which those from `from` on are its own (a last piece that
// would pass the row's end starts before), tokens [t0, t1).  A wave is 64 pieces (of several sequences where a row has
// fewer, if a.packed) at one run; lanes without a piece repeat the last one's loads and store nothing.
template <int E>
struct Place {
    int64_t c, b, b0, t0, t1;
    int from;
    bool on;
    __device__ __forceinline__ explicit Place(const ConvArgs& a) {
        const int64_t pieces = (a.C + E - 1) / E, cols = a.packed ? a.batch * pieces : a.batch * ((pieces + 63) / 64 * 64);
        const int64_t blocks = (cols + 63) / 64, tb = blockIdx.x / blocks, first = (blockIdx.x - tb * blocks) * 64;
        const int64_t per = a.packed ? pieces : cols / a.batch, id = min(first + (threadIdx.x & 63), cols - 1);
        b0 = first / per;
        b = id / per;
        const int64_t own = min(id - b * per, pieces - 1) * E;
        on = first + (threadIdx.x & 63) < cols && id - b * per < pieces;
        c = min(own, a.C - E);
        from = (int)(own - c);
        t0 = (tb * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * a.run;
        t1 = min(a.T, t0 + a.run);
    }
};

// Rows of a tensor as a wave's lanes see them.
template <int ES, int E>
struct Rows {
    char* base;     // of the wave's first sequence; null: no rows
    int64_t st;     // bytes from a token to the next
    uint32_t off;   // of the lane
    __device__ __forceinline__ Rows(const ScanRows& r, const Place<E>& at) {
        base = r.p ? static_cast<char*>(const_cast<void*>(r.p)) + at.b0 * r.sb * ES : nullptr;
        st = r.st * ES;
        off = (uint32_t)(((at.b - at.b0) * r.sb + at.c) * ES);
    }
    __device__ __forceinline__ char* at(int64_t t) const { return base + t * st + off; }
};
// The same of a state, [K-1][batch][C].
template <int ES, int E>
__device__ __forceinline__ char* kept_at(const ConvArgs& a, const void* p, const Place<E>& at, int64_t i) {
    return static_cast<char*>(const_cast<void*>(p)) + ((i * a.batch + at.b) * a.C + at.c) * ES;
}

__device__ __forceinline__ bool marked(const ConvArgs& a, int64_t t, int64_t b) {
    return a.reset && t >= 0 && a.reset[min(t, a.T - 1) * a.rs_t + b * a.rs_b] != 0;  // (past the end: not used)
}
// Reset marks of a run: where a wave has one sequence, a byte to a lane and then a bit to a token.
struct Marks {
    uint64_t bits = 0;
    bool whole = false;
    template <int E>
    __device__ __forceinline__ Marks(const ConvArgs& a, const Place<E>& at) {
        if (!a.reset) return;
        whole = __all(at.b == at.b0);
        if (whole) bits = __ballot(marked(a, at.t0 + (threadIdx.x & 63), at.b0));
    }
    // Whether token t0 + j may have one (the same answer for the whole wave).
    __device__ __forceinline__ bool may(const ConvArgs& a, int64_t j) const { return a.reset && !(whole && j < 64 && !(bits >> j & 1)); }
    // Of token t0 + j.
    template <int E>
    __device__ __forceinline__ bool at(const ConvArgs& a, const Place<E>& p, int64_t j) const {
        if (!a.reset) return false;
        return whole && j < 64 ? (bits >> j & 1) != 0 : marked(a, p.t0 + j, p.b);
    }
};

// The K - 1 inputs before token t as token t - 1 saw them: x[j - 1] is that of t - j, zero where a reset
// lies after it (or nothing is kept); seen[j - 1]: none does.
template <int ES, int K, int E>
__device__ __forceinline__ void before(const ConvArgs& a, const Place<E>& at, const Rows<ES, E>& rx, float (&x)[K > 1 ? K - 1 : 1][E],
                                       bool (&seen)[K > 1 ? K - 1 : 1]) {
    bool open = true;
    static_for<K - 1>([&](auto i) {
        const int64_t s = at.t0 - 1 - i;
        Vals<ES, E> v;
        if (s >= 0) v.load(rx.at(s));
        else if (a.state) v.load(kept_at<ES>(a, a.state, at, K - 1 + s));
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
    if (at.t0 >= at.t1) return;  // (the whole wave)
    const Marks marks(a, at);
    const Rows<ES, E> rx(a.x, at), ry(a.y, at);
    Vals<ES, E> next[kAhead];
    static_for<kAhead>([&](auto i) { next[i].load(rx.at(min(at.t0 + i, at.t1 - 1))); });
    float w[K][E], bias[E];
    static_for<E>([&](auto e) {
        bias[e] = a.bias ? a.bias[at.c + e] : 0.0f;
        static_for<K>([&](auto k) { w[k][e] = a.w[k * a.C + at.c + e]; });
    });
    float x[K > 1 ? K - 1 : 1][E];
    bool seen[K > 1 ? K - 1 : 1];
    before<ES, K, E>(a, at, rx, x, seen);
    for (int64_t j = 0; at.t0 + j < at.t1; j += kAhead) {
        static_for<kAhead>([&](auto i) {
            const int64_t t = at.t0 + j + i;
            if (t < at.t1) {
                float now[E], y[E];
                next[i].get(now);
                next[i].load(rx.at(min(t + kAhead, at.t1 - 1)));
                if (marks.may(a, j + i)) {
                    const bool cut = marks.at(a, at, j + i);
                    static_for<K - 1>([&](auto k) { static_for<E>([&](auto e) { x[k][e] = cut ? 0.0f : x[k][e]; }); });
                }
                static_for<E>([&](auto e) {
                    float p = __builtin_fmaf(w[K - 1][e], now[e], bias[e]);
                    static_for<K - 1>([&](auto k) { p = __builtin_fmaf(w[K - 2 - k][e], x[k][e], p); });
                    y[e] = p;
                    if (a.act) {
                        float z, omz;
                        sigmoid_pair(p, z, omz);
                        y[e] *= z;
                    }
                    static_for<K - 1>([&](auto k) {
                        constexpr int to = K - 2 - decltype(k)::value;
                        x[to][e] = to == 0 ? now[e] : x[to > 0 ? to - 1 : 0][e];
                    });
                });
                if (ry.base && at.on) Vals<ES, E>::store(ry.at(t), at.from, y);
            }
        });
    }
    if (a.state_T && at.t1 == a.T && at.on)
        static_for<K - 1>([&](auto k) { Vals<ES, E>::store(kept_at<ES>(a, a.state_T, at, K - 2 - k), at.from, x[k]); });
}

template <int ES, int K, int E>
__global__ __launch_bounds__(256, 2) void conv_bwd_kernel(ConvArgs a) {
    __shared__ float sums[4][64 * E];
    const Place<E> at(a);
    float dw[K][E], db[E];
    static_for<E>([&](auto e) {
        db[e] = 0.0f;
        static_for<K>([&](auto k) { dw[k][e] = 0.0f; });
    });
    if (at.t0 < at.t1) {  // (the whole wave)
        const Marks marks(a, at);
        const Rows<ES, E> rx(a.x, at), ry(a.dy, at), rd(a.dx, at);
        const int64_t end = min(a.T, at.t1 + K - 1);  // the tokens that see this run's inputs
        Vals<ES, E> nx[kAhead], nd[kAhead];
        auto fetch = [&](auto i, int64_t t) {
            t = min(t, end - 1);
            nx[i].load(rx.at(t));
            if (ry.base) nd[i].load(ry.at(t));
            else nd[i].zero();
        };
        static_for<kAhead>([&](auto i) { fetch(i, at.t0 + i); });
        float w[K][E], bias[E];
        static_for<E>([&](auto e) {
            bias[e] = a.bias ? a.bias[at.c + e] : 0.0f;
            static_for<K>([&](auto k) { w[k][e] = a.w[k * a.C + at.c + e]; });
        });
        float x[K > 1 ? K - 1 : 1][E], dx[K][E];  // dx[j]: of token t - j
        bool seen[K > 1 ? K - 1 : 1];
        // dx of token s is complete: a row of dx, or of dstate before the first token
        auto done = [&](int64_t s, const float (&v)[E]) {
            if (s >= at.t0 && s < at.t1) {
                if (rd.base && at.on) Vals<ES, E>::store(rd.at(s), at.from, v);
            } else if (s < 0 && at.t0 == 0 && a.dstate) {  // (s >= -(K - 1))
                if (at.on) Vals<ES, E>::store(kept_at<ES>(a, a.dstate, at, K - 1 + s), at.from, v);
            }
        };
        before<ES, K, E>(a, at, rx, x, seen);
        int closed = a.reset ? K : 0;  // tokens for which some input may not be seen any more (for the whole wave)
        static_for<K>([&](auto j) { static_for<E>([&](auto e) { dx[j][e] = 0.0f; }); });
        for (int64_t j = 0; at.t0 + j < end; j += kAhead) {
            static_for<kAhead>([&](auto i) {
                const int64_t t = at.t0 + j + i;
                if (t < end) {
                    float now[E], dy[E];
                    nx[i].get(now);
                    nd[i].get(dy);
                    fetch(i, t + kAhead);
                    const bool own = t < at.t1;
                    if (marks.may(a, j + i)) {
                        const bool cut = marks.at(a, at, j + i);
                        closed = K;
                        static_for<K - 1>([&](auto k) {
                            seen[k] = seen[k] && !cut;
                            static_for<E>([&](auto e) { x[k][e] = cut ? 0.0f : x[k][e]; });
                        });
                    }
                    float g[E];
                    static_for<E>([&](auto e) {
                        float p = __builtin_fmaf(w[K - 1][e], now[e], bias[e]);
                        static_for<K - 1>([&](auto k) { p = __builtin_fmaf(w[K - 2 - k][e], x[k][e], p); });
                        g[e] = dy[e];
                        if (a.act) {
                            float z, omz;
                            sigmoid_pair(p, z, omz);
                            g[e] *= z * __builtin_fmaf(p, omz, 1.0f);
                        }
                        dx[0][e] = w[K - 1][e] * g[e];
                    });
                    if (own) static_for<E>([&](auto e) {
                        db[e] += g[e];
                        dw[K - 1][e] = __builtin_fmaf(g[e], now[e], dw[K - 1][e]);
                        static_for<K - 1>([&](auto k) { dw[K - 2 - k][e] = __builtin_fmaf(g[e], x[k][e], dw[K - 2 - k][e]); });
                    });
                    if (closed > 0) {
                        --closed;
                        static_for<K - 1>([&](auto k) {
                            static_for<E>([&](auto e) { dx[k + 1][e] = __builtin_fmaf(w[K - 2 - k][e], seen[k] ? g[e] : 0.0f, dx[k + 1][e]); });
                        });
                    } else {
                        static_for<K - 1>([&](auto k) {
                            static_for<E>([&](auto e) { dx[k + 1][e] = __builtin_fmaf(w[K - 2 - k][e], g[e], dx[k + 1][e]); });
                        });
                    }
                    done(t - (K - 1), dx[K - 1]);
                    static_for<K - 1>([&](auto k) {
                        constexpr int to = K - 1 - decltype(k)::value;
                        static_for<E>([&](auto e) { dx[to][e] = dx[to - 1][e]; });
                    });
                    static_for<K - 1>([&](auto k) {
                        constexpr int to = K - 2 - decltype(k)::value;
                        seen[to] = to == 0 ? true : seen[to > 0 ? to - 1 : 0];
                        static_for<E>([&](auto e) { x[to][e] = to == 0 ? now[e] : x[to > 0 ? to - 1 : 0][e]; });
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
                if (a.dstate_T) v.load(kept_at<ES>(a, a.dstate_T, at, K - 2 - j));
                v.get(kept);
                static_for<E>([&](auto e) { dx[j + 1][e] += seen[j] ? kept[e] : 0.0f; });
                done(a.T - 1 - j, dx[j + 1]);
            });
        }
    }
    if (!a.dw && !a.dbias) return;
    // one row of partial sums for a workgroup's four runs (of each sequence)
    const int64_t pieces = (a.C + E - 1) / E, cols = a.packed ? a.batch * pieces : a.batch * ((pieces + 63) / 64 * 64);
    const int64_t row = blockIdx.x / ((cols + 63) / 64) * a.batch + at.b;
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    static_for<K + 1>([&](auto k) {
        __syncthreads();
        static_for<E>([&](auto e) { sums[wid][lane * E + e] = k < K ? dw[k < K ? decltype(k)::value : 0][e] : db[e]; });
        __syncthreads();
        // (each wave's lanes stand at the same pieces)
        if (wid < E && at.on && wid >= at.from) {
            const int i = lane * E + wid;
            const float s = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
            a.part[k < K ? (row * K + k) * a.C + at.c + wid : (a.rows * K + row) * a.C + at.c + wid] = s;
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

// Channels of a piece: 8 bytes, or one value where the row has fewer.
int piece(const ConvArgs& a) {
    const int e = a.type == kBF16 ? 4 : 2;
    return a.C >= e ? e : 1;
}

template <int ES, bool BWD, int K>
ConvFn conv_fn(int e) {
    constexpr int E = 8 / ES;
    if constexpr (BWD) return e == E ? conv_bwd_kernel<ES, K, E> : conv_bwd_kernel<ES, K, 1>;
    else return e == E ? conv_fwd_kernel<ES, K, E> : conv_fwd_kernel<ES, K, 1>;
}
template <int ES, bool BWD>
ConvFn conv_fn(int64_t K, int e) {
    switch (K) {
        case 1: return conv_fn<ES, BWD, 1>(e);
        case 2: return conv_fn<ES, BWD, 2>(e);
        case 3: return conv_fn<ES, BWD, 3>(e);
        case 4: return conv_fn<ES, BWD, 4>(e);
        case 5: return conv_fn<ES, BWD, 5>(e);
        default: return conv_fn<ES, BWD, 6>(e);
    }
}

// Workgroups to a block of four runs.
int64_t conv_blocks(const ConvArgs& a) {
    const int64_t E = piece(a), pieces = (a.C + E - 1) / E;
    return ((a.packed ? a.batch * pieces : a.batch * ((pieces + 63) / 64 * 64)) + 63) / 64;
}

}  // namespace

// Whether a wave may have several sequences: their places lie within 31 bits of the first's.
bool conv_packs(const ScanRows& r, int64_t C, int type) {
    const int64_t es = type == kBF16 ? 2 : 4, E = 8 / es, pieces = (C + E - 1) / E;
    return !r.p || ((__int128)(64 / pieces + 2) * r.sb + C) * es < ((__int128)1 << 31);
}

// Runs and rows of partial sums for these sizes.
void conv_plan(ConvArgs& a, int cus) {
    if (a.C <= 0) return;
    const int64_t blocks = conv_blocks(a);
    // runs as long as leave four workgroups to a compute unit; eight tokens at least
    a.run = 64;
    while (a.run > 8 && blocks * ((a.T + a.run * 4 - 1) / (a.run * 4)) < 4 * (int64_t)cus) a.run /= 2;
    a.rows = a.batch * ((a.T + a.run * 4 - 1) / (a.run * 4));
}

hipError_t launch_causal_conv(const ConvArgs& a, bool backward, hipStream_t s) {
    const int E = piece(a);
    hipError_t e = hipSuccess;
    if (a.T > 0 && a.batch > 0) {
        const int64_t blocks = a.rows / a.batch * conv_blocks(a);
        if (blocks > INT32_MAX) return hipErrorInvalidValue;
        const ConvFn fn = backward ? (a.type == kBF16 ? conv_fn<2, true>(a.K, E) : conv_fn<4, true>(a.K, E))
                                   : (a.type == kBF16 ? conv_fn<2, false>(a.K, E) : conv_fn<4, false>(a.K, E));
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
