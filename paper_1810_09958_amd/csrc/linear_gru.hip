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
// Per value the forward pass reads two gates and writes one state, the backward
// pass reads three and writes two.  The bytes bound them, with the vector units
// close behind (four transcendentals and some 20 plain instructions a value forward,
// twice that backward), so each value is loaded, and its gates are formed, once:
//   * a workgroup takes a tile of time x 64 channels of one sequence into
//     registers: 16 lanes x 4 channels make a row, a wave four groups of rows, each
//     group R consecutive steps.  A group composes its steps, the groups of a wave
//     are scanned by lane exchanges, the waves through LDS;
//   * tiles of one column of channels are chained in memory: a tile publishes its
//     composition (A, B) as soon as it has it, and takes the state before it from the
//     nearest earlier tile that has published one, through the compositions of
//     those between.  Workgroups draw their tiles from a counter in time order, so
//     those a tile waits for are always held by running workgroups: the chain needs
//     no co-residency.  A tile's published state is its composition applied to the state
//     before it wherever that came from, so results repeat bit for bit.  A word of
//     the chain is valid once it differs from the pattern a kernel before fills it
//     with (a captured launch replays), and is written and read with device scope, so
//     no ordering between words is needed;
//   * the backward pass keeps no sequence of states: the forward pass leaves the
//     state before every 128 steps, and each tile forms its states again in
//     registers while it scans e from its end (5 values moved per element, 6 with
//     stored states, which would have to be fp32 to give fp32 gradients).
// Measured, bf16: 32768 steps of 1 x 2048 forward 98-100 us, 4.1 TB/s (the residual norm streams
// at 5.4); forward and backward of 4096 x 8 x 1024 with resets 164 us, 3.3 TB/s, of which the
// forward kernel 62 and the backward kernel 98.  The vector units are busy 57 % of both
// (40 and 64 instructions a value) and half of the waves' time is waiting: a
// tile loads, computes, waits for the chain and stores, and only the two or three
// workgroups that the registers let a compute unit hold cover for each other.  The chain by
// itself, 32768 steps of a single column (1 x 64), takes 49 us forward and 97 backward.  fp32:
// 32768 x 1 x 2048 forward 153 us (5.3 TB/s), 4096 x 8 x 1024 84 and 149.  Of tile
// sizes: forward tiles of four waves (twice as many links) 122 us for the long sequence
// against 99; backward tiles of eight waves at two waves a SIMD 123, of four at two 113,
// of four at three 98 (a look of four tiles back instead of two takes the registers for
// that, 20 spilled: 115).
// A reset must cut off whatever stands before it, NaN included, which 0 * NaN
// does not.  Within a group's steps the state before it is replaced by 0; in a
// composition its A is -0, and a sign bit in A (kept through products) makes it drop
// the left side.
#include <type_traits>

#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

constexpr int kCols = 64;        // channels of a tile
constexpr int kChainWindow = 2;  // tiles that one look back along the chain sees

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

// (A, B) of a group's steps so far, then one more.  A's sign stays (also where z is NaN).
template <bool RESET>
__device__ __forceinline__ void step(bool drop, bool first, float z, float b, float& A, float& B) {
    if (first) {
        A = drop ? -0.0f : z;
        B = b;
    } else {
        A = drop ? -0.0f : RESET ? __builtin_copysignf(A * z, A) : A * z;
        B = __builtin_fmaf(z, drop ? 0.0f : B, b);
    }
}

// The four channels of a lane.  VEC (at least four of them, on 4 bytes): one
// piece of four, moved as one; otherwise channels 16 apart, moved one by one.  A
// block's lanes past the last channel repeat it (and a last piece off a multiple of four the
// channels before it: same loads, same values, same stores), so nothing below
// depends on how many of them exist, and no load or
// store stands in a branch of lanes (the compiler has copied registers inside such
// a branch, for its lanes only, in a kernel that uses nearly all of them).
template <bool VEC>
__device__ __forceinline__ int64_t channel(int64_t H, int64_t c0, int l, int e) {
    if constexpr (VEC) return min(c0 + 4 * l, H - 4) + e;
    return min(c0 + 16 * e + l, H - 1);
}

// Rows of one tensor as a wave sees them: row r of the lane's group of R steps at
// base + (group * R + r) * step + the lane's channels.  Rows outside are addressed
// past the buffer's end: loads give zeros, stores are dropped.
template <int ES, bool VEC, int R>
struct Rows {
    static constexpr int W = ES == 2 ? 2 : 4;  // 32-bit words of four values
    __amdgpu_buffer_rsrc_t rs;
    uint32_t off[VEC ? 1 : 4], step;
    // p: first row of the wave (null: no rows); stride in elements.
    __device__ __forceinline__ Rows(const void* p, int64_t at, int64_t stride, int64_t H, int64_t c0, int lane) {
        rs = make_rsrc(p ? static_cast<const char*>(p) + at * ES : nullptr, p ? 0x7fffffffu : 0u);
        step = (uint32_t)(stride * ES);
        static_for<VEC ? 1 : 4>([&](auto e) {
            off[e] = (uint32_t)(lane >> 4) * R * step + (uint32_t)channel<VEC>(H, c0, lane & 15, e) * ES;
        });
    }
    // `extra`: bytes added to every address (the second block of a row).
    __device__ __forceinline__ void load(uint32_t (&w)[W], int r, bool in, uint32_t extra) const {
        const int so = (int)(r * step + extra);
        if constexpr (VEC && ES == 4) {
            const i32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(in ? off[0] : kOob), so, 0);
            static_for<4>([&](auto e) { w[e] = (uint32_t)v[decltype(e)::value]; });
        } else if constexpr (VEC) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(in ? off[0] : kOob), so, 0);
            w[0] = (uint32_t)v[0];
            w[1] = (uint32_t)v[1];
        } else if constexpr (ES == 4) {
            static_for<4>([&](auto e) { w[e] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, (int)(in ? off[e] : kOob), so, 0); });
        } else {
            uint32_t h[4];
            static_for<4>([&](auto e) { h[e] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(in ? off[e] : kOob), so, 0) & 0xffffu; });
            w[0] = h[0] | h[1] << 16;
            w[1] = h[2] | h[3] << 16;
        }
    }
    // bf16: rounded to nearest even.
    __device__ __forceinline__ void store(const float (&f)[4], int r, bool in, uint32_t extra) const {
        const int so = (int)(r * step + extra);
        if constexpr (ES == 4) {
            if constexpr (VEC) {
                // The offset in the address register: after a 16-byte store whose offset sits in
                // a scalar register the compiler lets the next instruction overwrite the data,
                // and lanes have then stored the new value.
                const i32x4_t v = __builtin_bit_cast(i32x4_t, f32x4_t{f[0], f[1], f[2], f[3]});
                __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)(in ? off[0] + (uint32_t)so : kOob), 0, 0);
            } else {
                static_for<4>([&](auto e) { __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(f[e]), rs, (int)(in ? off[e] : kOob), so, 0); });
            }
        } else {
            const uint32_t w[2] = {pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3])};
            if constexpr (VEC) {
                __builtin_amdgcn_raw_buffer_store_b64((i32x2_t){(int)w[0], (int)w[1]}, rs, (int)(in ? off[0] : kOob), so, 0);
            } else {
                static_for<4>([&](auto e) {
                    __builtin_amdgcn_raw_buffer_store_b16((short)(w[e / 2] >> (16 * (e & 1))), rs, (int)(in ? off[e] : kOob), so, 0);
                });
            }
        }
    }
    __device__ __forceinline__ static void unpack(const uint32_t (&w)[W], float (&f)[4]) {
        static_for<4>([&](auto e) {
            if constexpr (ES == 4) f[e] = __uint_as_float(w[e]);
            else if constexpr (e & 1) f[e] = bf16hi(w[e / 2]);
            else f[e] = bf16lo(w[e / 2]);
        });
    }
};

// fp32 values of the lane's channels (zeros without a tensor).
template <bool VEC>
__device__ __forceinline__ void load_channels(const float* p, int64_t at, int64_t H, int64_t c0, int lane, float (&f)[4]) {
    static_for<4>([&](auto e) { f[e] = p ? p[at + channel<VEC>(H, c0, lane & 15, e)] : 0.0f; });
}
// The same stored, by the lanes with `on`.
template <bool VEC>
__device__ __forceinline__ void store_channels(float* p, int64_t at, int64_t H, int64_t c0, int lane, bool on, const float (&f)[4]) {
    const Rows<4, VEC, 0> rows(p, at, 0, H, c0, lane);
    rows.store(f, 0, on, 0);
}

constexpr float kLog2e = 1.44269504f;

// z = sigmoid(v) and 1 - z, each to fp32 accuracy also where it is small (1 - z formed
// from z would lose the digits that decide how long a state lives).  The bound on the
// exponent keeps 2^w z finite; a NaN passes.
__device__ __forceinline__ void gate_pair(float v, float& z, float& omz) {
    const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(v * -kLog2e, 126.0f));
    z = __builtin_amdgcn_rcpf(1.0f + e);
    omz = e * z;
}
// tanh(v), relative error of some 8 x 2^-24.  Through the exponential alone the difference
// from 1 would leave an absolute error (5e-5 of values of 1e-3), so below 1/4 it is v + v^3 P(v^2)
// with P fitted to tanh for the least relative error (0.05 x 2^-24 before rounding).
template <int ES>
__device__ __forceinline__ float gate_tanh(float v) {
    const float y = v * v, p = __builtin_fmaf(__builtin_fmaf(-0.05143003f, y, 0.13324237f), y, -0.3333324f);
    const float low = __builtin_fmaf(v, p * y, v);
    float high;
    if constexpr (ES == 4) {
        const float t = __builtin_amdgcn_exp2f(__builtin_fabsf(v) * (-2.0f * kLog2e));
        high = __builtin_copysignf((1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t), v);
    } else {
        high = __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * (2.0f * kLog2e))), 1.0f);
    }
    return __builtin_fabsf(v) < 0.25f ? low : high;
}

// Inclusive scan over the wave's four groups in time order (UP) or against it.
template <bool RESET, bool UP>
__device__ __forceinline__ void wave_scan(float (&A)[4], float (&B)[4], int lane) {
    static_for<2>([&](auto dc) {
        constexpr int d = 16 << decltype(dc)::value;
        const bool has = UP ? lane >= d : lane + d < 64;
        static_for<4>([&](auto e) {
            const float pa = UP ? __shfl_up(A[e], d) : __shfl_down(A[e], d);
            const float pb = UP ? __shfl_up(B[e], d) : __shfl_down(B[e], d);
            B[e] = has ? apply<RESET>(A[e], B[e], pb) : B[e];
            A[e] = has ? compose_a<RESET>(A[e], pa) : A[e];
        });
    });
}

// The chain of tiles: a counter, then for each tile 64 pairs (A, B) of 8 bytes and 64
// states after it, every bit set until they are published.  A published NaN is the
// canonical one, so no published word is all ones.
__device__ __forceinline__ uint64_t* chain_pair(const LinGruArgs& a, int64_t id, int ch) {
    return a.chain + 8 + id * (kCols + kCols / 2) + ch;
}
__device__ __forceinline__ uint32_t* chain_state(const LinGruArgs& a, int64_t id, int ch) {
    return reinterpret_cast<uint32_t*>(a.chain + 8 + id * (kCols + kCols / 2) + kCols) + ch;
}
__device__ __forceinline__ uint32_t chain_bits(float v) { return v != v ? 0x7fc00000u : __float_as_uint(v); }
template <bool RESET>
__device__ __forceinline__ void chain_put(const LinGruArgs& a, int64_t id, int ch, float ta, float tb) {
    // (an A that drops keeps its sign, also where it is NaN)
    const uint32_t wa = RESET && drops(ta) ? 0x80000000u : chain_bits(ta);
    __hip_atomic_store(chain_pair(a, id, ch), (uint64_t)wa | (uint64_t)chain_bits(tb) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void chain_put(const LinGruArgs& a, int64_t id, int ch, float v) {
    __hip_atomic_store(chain_state(a, id, ch), chain_bits(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// State that reaches the tile `id`, `before` tiles into its column (lane: channel;
// whole wave).  `first`: the state before the column's first tile.  The wait ends: a
// column's first tile waits for nobody, and every other one for tiles drawn before it, which
// running workgroups hold.  Only a foreign write to the workspace can take a word away
// for good; so that this ends too, a wait gives up after some seconds, with NaN.  It counts
// its looks, not the time: a queue that is taken off the device does not look.
template <bool RESET>
__device__ __forceinline__ float chain_in(const LinGruArgs& a, int64_t id, int64_t before, int64_t cols, int lane, float first) {
    constexpr int W = kChainWindow;  // tiles looked at together
    for (int looks = 0; looks < kLinGruLooks; ++looks) {
        uint64_t ab[W];
        uint32_t st[W];
        static_for<W>([&](auto i) {
            const int64_t p = id - (i + 1) * cols;
            st[i] = i == before ? chain_bits(first) : ~0u;
            ab[i] = ~0ull;
            if (i < before) {
                st[i] = __hip_atomic_load(chain_state(a, p, lane), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                ab[i] = __hip_atomic_load(chain_pair(a, p, lane), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        });
        int at = -1;
        bool open = true;
        static_for<W>([&](auto i) {
            if (open && __all(st[i] != ~0u)) {
                at = i;
                open = false;
            }
            open = open && __all(ab[i] != ~0ull);
        });
        if (at >= 0) {
            float v = 0.0f;
            static_for<W>([&](auto j) {
                constexpr int i = W - 1 - decltype(j)::value;
                if (i == at) v = __uint_as_float(st[i]);
                if (i < at) v = apply<RESET>(__uint_as_float((uint32_t)ab[i]), __uint_as_float((uint32_t)(ab[i] >> 32)), v);
            });
            return v;
        }
        __builtin_amdgcn_s_sleep(1);
    }
    return __builtin_nanf("");
}

// Which tile a workgroup has: number, place in its column (from the end if
// backward), sequence and first channel.
struct Tile {
    int64_t id, k, cols, b, c0;
    template <bool CHAIN>
    __device__ __forceinline__ static Tile take(const LinGruArgs& a, unsigned* shared) {
        Tile t;
        const int64_t blocks = (a.H + kCols - 1) / kCols;
        t.cols = a.batch * blocks;
        if constexpr (CHAIN) {
            if (threadIdx.x == 0)
                *shared = __hip_atomic_fetch_add(reinterpret_cast<unsigned*>(a.chain), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            t.id = __builtin_amdgcn_readfirstlane(*shared);
            t.k = t.id / t.cols;
        } else {
            t.id = blockIdx.x;
            t.k = 0;
        }
        const int64_t col = t.id - t.k * t.cols;
        t.b = col / blocks;
        t.c0 = (col - t.b * blocks) * kCols;
        return t;
    }
};

// Reset marks of a wave's 4 R steps: one byte a lane, then a bit for each of the group's steps.
template <int R, bool RESET>
struct Resets {
    static_assert(4 * R <= 32, "a lane for each step, a word of marks");
    uint32_t v = 0;
    __device__ __forceinline__ Resets(const LinGruArgs& a, int64_t b, int64_t tw, int lane, int left) {
        if constexpr (RESET) {
            const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.reset + b * a.rs_b + tw * a.rs_t, 0x7fffffffu);
            v = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rs, (int)(lane < left ? (uint32_t)lane * (uint32_t)a.rs_t : kOob), 0, 0);
        }
    }
    __device__ __forceinline__ uint32_t bits(int q) const {
        return RESET ? (uint32_t)__ballot((v & 0xffu) != 0) >> (q * R) : 0u;
    }
};

// A wave's totals: the lanes of its last group (or first) to the tile's row, the
// others to a row that nobody reads.
__device__ __forceinline__ void put4(float* row, float* spare, int lane, bool on, const float (&f)[4]) {
    *reinterpret_cast<float4*>((on ? row : spare) + (lane & 15) * 4) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void get4(const float* row, int lane, float (&f)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(row + (lane & 15) * 4);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}

// Forward pass: NW waves of 4 groups of R steps.
template <int ES, bool VEC, int NW, int R, bool RESET, bool CHAIN>
__global__ __launch_bounds__(NW * 64, 4) void lingru_fwd_kernel(LinGruArgs a) {
    using S = Rows<ES, VEC, R>;
    constexpr int TS = NW * 4 * R;
    __shared__ __attribute__((aligned(16))) float tot[NW][2][kCols];
    __shared__ __attribute__((aligned(16))) float start[NW][kCols];
    __shared__ __attribute__((aligned(16))) float spare[kCols];
    __shared__ unsigned ticket;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
    const Tile tile = Tile::take<CHAIN>(a, &ticket);
    const int64_t b = tile.b, c0 = tile.c0, tw = tile.k * TS + wid * 4 * R;
    const int left = (int)max((int64_t)0, min((int64_t)(4 * R), a.T - tw));  // steps of this wave that exist
    const bool last = (tile.k + 1) * TS >= a.T;

    const Resets<R, RESET> marks(a, b, tw, lane, left);
    const S gx(a.gx, b * a.gx_b + tw * a.gx_t, a.gx_t, a.H, c0, lane);
    uint32_t pz[R][S::W], pn[R][S::W];
    static_for<R>([&](auto r) {
        gx.load(pz[r], r, q * R + r < left, 0);
        gx.load(pn[r], r, q * R + r < left, (uint32_t)a.H * ES);
    });
    const uint32_t reset = marks.bits(q);
    float bz[4], bn[4];
    load_channels<VEC>(a.bias, 0, a.H, c0, lane, bz);
    load_channels<VEC>(a.bias, a.H, a.H, c0, lane, bn);

    // (a step that does not exist leaves the state as it is, whatever the bias)
    float ca[R][4], cb[R][4], A[4], B[4];
    static_for<R>([&](auto r) {
        const bool drop = RESET && (reset >> r & 1), in = q * R + r < left;
        float gz[4], n[4];
        S::unpack(pz[r], gz);
        S::unpack(pn[r], n);
        static_for<4>([&](auto e) { n[e] += bn[e]; });
        if (a.candidate) static_for<4>([&](auto e) { n[e] = gate_tanh<ES>(n[e]); });
        static_for<4>([&](auto e) {
            float z, omz;
            gate_pair(gz[e] + bz[e], z, omz);
            ca[r][e] = in ? z : 1.0f;
            cb[r][e] = in ? omz * n[e] : 0.0f;
            step<RESET>(drop, r == 0, ca[r][e], cb[r][e], A[e], B[e]);
        });
    });
    wave_scan<RESET, true>(A, B, lane);
    put4(tot[wid][0], spare, lane, q == 3, A);
    put4(tot[wid][1], spare, lane, q == 3, B);
    __syncthreads();
    if (wid == 0) {
        // lane: one of the tile's channels, in the lanes' order
        const int64_t ch = channel<VEC>(a.H, c0, lane >> 2, lane & 3);
        float wa[NW], wb[NW];
        static_for<NW>([&](auto w) {
            wa[w] = tot[w][0][lane];
            wb[w] = tot[w][1][lane];
        });
        const float first = a.h0 ? a.h0[b * a.H + ch] : 0.0f;
        float h = first;
        if constexpr (CHAIN) {
            float ta = wa[0], tb = wb[0];
            static_for<NW - 1>([&](auto w) {
                tb = apply<RESET>(wa[w + 1], wb[w + 1], tb);
                ta = compose_a<RESET>(ta, wa[w + 1]);
            });
            if (!last) chain_put<RESET>(a, tile.id, lane, ta, tb);
            h = chain_in<RESET>(a, tile.id, tile.k, tile.cols, lane, first);
            if (!last) chain_put(a, tile.id, lane, apply<RESET>(ta, tb, h));
        }
        static_for<NW>([&](auto w) {
            start[w][lane] = h;
            h = apply<RESET>(wa[w], wb[w], h);
        });
    }
    __syncthreads();
    float v[4];
    get4(start[wid], lane, v);
    static_for<4>([&](auto e) {
        const float pa = __shfl_up(A[e], 16), pb = __shfl_up(B[e], 16);
        v[e] = q > 0 ? apply<RESET>(pa, pb, v[e]) : v[e];
    });
    if (a.states && wid * 4 * R % kLinGruChunk == 0 && left > 0)
        store_channels<VEC>(a.states, (tw / kLinGruChunk * a.batch + b) * a.H, a.H, c0, lane, q == 0, v);
    const S hs(a.h_seq, b * a.h_b + tw * a.h_t, a.h_t, a.H, c0, lane);
    static_for<R>([&](auto r) {
        const bool drop = RESET && (reset >> r & 1);
        static_for<4>([&](auto e) { v[e] = __builtin_fmaf(ca[r][e], drop ? 0.0f : v[e], cb[r][e]); });
        hs.store(v, r, q * R + r < left, 0);
    });
    // (steps past the end leave the state as it is)
    if (a.h_T && last && wid == NW - 1) store_channels<VEC>(a.h_T, b * a.H, a.H, c0, lane, q == 3, v);
}

// A few steps, one thread per channel: decoding (no tile to fill).  Bound by one
// memory latency; a step of 32 x 1024 takes 7.7-8 us a call, most of it the host's.
template <int ES>
__global__ __launch_bounds__(64) void lingru_few_kernel(LinGruArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (i >= a.batch * a.H) return;
    const int64_t b = i / a.H, c = i - b * a.H;
    const int T = (int)a.T;
    float gz[kLinGruFew], gn[kLinGruFew];
    bool drop[kLinGruFew];
    float h = a.h0 ? a.h0[i] : 0.0f;
    const float bz = a.bias ? a.bias[c] : 0.0f, bn = a.bias ? a.bias[a.H + c] : 0.0f;
    static_for<kLinGruFew>([&](auto t) {
        if (t < T) {
            gz[t] = Row16<ES>::get(a.gx, b * a.gx_b + t * a.gx_t + c);
            gn[t] = Row16<ES>::get(a.gx, b * a.gx_b + t * a.gx_t + a.H + c);
            drop[t] = a.reset && a.reset[t * a.rs_t + b * a.rs_b];
        }
    });
    if (a.states && T > 0) a.states[i] = h;
    static_for<kLinGruFew>([&](auto t) {
        if (t < T) {
            float z, omz;
            gate_pair(gz[t] + bz, z, omz);
            const float v = gn[t] + bn, n = a.candidate ? gate_tanh<ES>(v) : v;
            h = drop[t] ? omz * n : __builtin_fmaf(z, h, omz * n);
            if (a.h_seq) Row16<ES>::put(a.h_seq, b * a.h_b + t * a.h_t + c, h);
        }
    });
    if (a.h_T) a.h_T[i] = h;
}

// Backward pass; tiles count from the end of time.  The tile's states are formed
// again from the one before it.
template <int ES, bool VEC, int NW, int R, bool RESET, bool CHAIN>
__global__ __launch_bounds__(NW * 64, ES == 2 && VEC ? 3 : 2) void lingru_bwd_kernel(LinGruArgs a) {
    using S = Rows<ES, VEC, R>;
    constexpr int TS = NW * 4 * R;
    static_assert(!CHAIN || TS % kLinGruChunk == 0, "a tile starts at a kept state");
    __shared__ __attribute__((aligned(16))) float tot[NW][3][kCols];
    __shared__ __attribute__((aligned(16))) float start[NW][2][kCols];
    __shared__ __attribute__((aligned(16))) float spare[kCols];
    __shared__ unsigned ticket;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
    const Tile tile = Tile::take<CHAIN>(a, &ticket);
    const int64_t tiles = (a.T + TS - 1) / TS, kt = tiles - 1 - tile.k;
    const int64_t b = tile.b, c0 = tile.c0, tw = kt * TS + wid * 4 * R;
    const int left = (int)max((int64_t)0, min((int64_t)(4 * R), a.T - tw));

    const Resets<R, RESET> marks(a, b, tw, lane, left);
    const S gx(a.gx, b * a.gx_b + tw * a.gx_t, a.gx_t, a.H, c0, lane);
    const S dh(a.dh_seq, b * a.dh_b + tw * a.dh_t, a.dh_t, a.H, c0, lane);
    uint32_t pz[R][S::W], pn[R][S::W], pd[R][S::W];
    static_for<R>([&](auto r) {
        gx.load(pz[r], r, q * R + r < left, 0);
        gx.load(pn[r], r, q * R + r < left, (uint32_t)a.H * ES);
        dh.load(pd[r], r, q * R + r < left, 0);
    });
    const uint32_t reset = marks.bits(q);
    float bz[4], bn[4];
    load_channels<VEC>(a.bias, 0, a.H, c0, lane, bz);
    load_channels<VEC>(a.bias, a.H, a.H, c0, lane, bn);

    // z, 1 - z and n of each step; (A, B) composes the state, (Z, C) e
    float z[R][4], omz[R][4], n[R][4], A[4], B[4], Z[4], C[4];
    static_for<R>([&](auto r) {
        const bool drop = RESET && (reset >> r & 1), in = q * R + r < left;
        float gz[4];
        S::unpack(pz[r], gz);
        S::unpack(pn[r], n[r]);
        static_for<4>([&](auto e) { n[r][e] += bn[e]; });
        if (a.candidate) static_for<4>([&](auto e) { n[r][e] = gate_tanh<ES>(n[r][e]); });
        static_for<4>([&](auto e) {
            gate_pair(gz[e] + bz[e], z[r][e], omz[r][e]);
            z[r][e] = in ? z[r][e] : 1.0f;
            omz[r][e] = in ? omz[r][e] : 0.0f;
            n[r][e] = in ? n[r][e] : 0.0f;
            step<RESET>(drop, r == 0, z[r][e], omz[r][e] * n[r][e], A[e], B[e]);
        });
    });
    static_for<R>([&](auto i) {
        constexpr int r = R - 1 - decltype(i)::value;
        float d[4];
        S::unpack(pd[r], d);
        static_for<4>([&](auto e) {
            const float w = z[r][e] * (i == 0 ? d[e] : d[e] + C[e]);
            C[e] = RESET && (reset >> r & 1) ? 0.0f : w;
            Z[e] = A[e];
        });
    });
    wave_scan<RESET, true>(A, B, lane);
    wave_scan<RESET, false>(Z, C, lane);
    put4(tot[wid][0], spare, lane, q == 3, A);
    put4(tot[wid][1], spare, lane, q == 3, B);
    put4(tot[wid][2], spare, lane, q == 0, C);
    __syncthreads();
    if (wid == 0) {
        const int64_t ch = channel<VEC>(a.H, c0, lane >> 2, lane & 3);
        float wa[NW], wc[NW];
        float h = a.states[(kt * TS / kLinGruChunk * a.batch + b) * a.H + ch];
        static_for<NW>([&](auto w) {
            wa[w] = tot[w][0][lane];
            wc[w] = tot[w][2][lane];
            start[w][0][lane] = h;
            h = apply<RESET>(wa[w], tot[w][1][lane], h);
        });
        const float first = a.dh_T ? a.dh_T[b * a.H + ch] : 0.0f;
        float g = first;
        if constexpr (CHAIN) {
            float ta = wa[NW - 1], tc = wc[NW - 1];
            static_for<NW - 1>([&](auto i) {
                constexpr int w = NW - 2 - decltype(i)::value;
                tc = apply<RESET>(wa[w], wc[w], tc);
                ta = compose_a<RESET>(ta, wa[w]);
            });
            if (kt > 0) chain_put<RESET>(a, tile.id, lane, ta, tc);
            g = chain_in<RESET>(a, tile.id, tile.k, tile.cols, lane, first);
            if (kt > 0) chain_put(a, tile.id, lane, apply<RESET>(ta, tc, g));
        }
        static_for<NW>([&](auto i) {
            constexpr int w = NW - 1 - decltype(i)::value;
            start[w][1][lane] = g;
            g = apply<RESET>(wa[w], wc[w], g);
        });
    }
    __syncthreads();
    // The states again; of each step then remain z and the factors of d in dgz and dgn, which
    // take the places of 1 - z and n.  The empty asm keeps the compiler from holding what it
    // formed of them before the scans (another 60 registers).
    static_for<R>([&](auto r) {
        static_for<4>([&](auto e) {
            float& v = omz[r][e];
            asm volatile("" : "+v"(v));
        });
        static_for<S::W>([&](auto w) {
            uint32_t& v = pd[r][w];
            asm volatile("" : "+v"(v));
        });
    });
    float hs[4], en[4], sz[4], sn[4];
    get4(start[wid][0], lane, hs);
    get4(start[wid][1], lane, en);
    static_for<4>([&](auto e) {
        const float pa = __shfl_up(A[e], 16), pb = __shfl_up(B[e], 16);
        hs[e] = q > 0 ? apply<RESET>(pa, pb, hs[e]) : hs[e];
        const float qa = __shfl_down(Z[e], 16), qc = __shfl_down(C[e], 16);
        en[e] = q < 3 ? apply<RESET>(qa, qc, en[e]) : en[e];
        sz[e] = sn[e] = 0.0f;
        static_for<R>([&](auto r) {
            const float hb = RESET && (reset >> r & 1) ? 0.0f : hs[e], w = omz[r][e], c = n[r][e];
            hs[e] = __builtin_fmaf(z[r][e], hb, w * c);
            omz[r][e] = w * z[r][e] * (hb - c);
            n[r][e] = a.candidate ? w * __builtin_fmaf(-c, c, 1.0f) : w;
        });
    });
    const S dg(a.dgx, b * a.dg_b + tw * a.dg_t, a.dg_t, a.H, c0, lane);
    static_for<R>([&](auto i) {
        constexpr int r = R - 1 - decltype(i)::value;
        float d[4], oz[4], on[4];
        S::unpack(pd[r], d);
        static_for<4>([&](auto e) {
            const float dt = d[e] + en[e];
            oz[e] = dt * omz[r][e];  // (0 past the end)
            on[e] = dt * n[r][e];
            const float back = z[r][e] * dt;
            en[e] = RESET && (reset >> r & 1) ? 0.0f : back;
            sz[e] += oz[e];
            sn[e] += on[e];
        });
        dg.store(oz, r, q * R + r < left, 0);
        dg.store(on, r, q * R + r < left, (uint32_t)a.H * ES);
    });
    if (a.dh0 && kt == 0 && wid == 0) store_channels<VEC>(a.dh0, b * a.H, a.H, c0, lane, q == 0, en);
    if (!a.dbias) return;
    // this tile's sums over time: groups of a wave, then waves
    static_for<4>([&](auto e) {
        static_for<2>([&](auto dc) {
            sz[e] += __shfl_xor(sz[e], 16 << decltype(dc)::value);
            sn[e] += __shfl_xor(sn[e], 16 << decltype(dc)::value);
        });
    });
    put4(tot[wid][0], spare, lane, q == 0, sz);  // (tot was last read before the second barrier)
    put4(tot[wid][1], spare, lane, q == 0, sn);
    __syncthreads();
    if (wid >= 2) return;
    float s = 0.0f;
    static_for<NW>([&](auto w) { s += tot[w][wid][lane]; });
    a.bias_part[(kt * a.batch + b) * 2 * a.H + wid * a.H + channel<VEC>(a.H, c0, lane >> 2, lane & 3)] = s;
}

// The chain before a launch: the counter's line of 64 bytes zero, every other bit set.
__global__ __launch_bounds__(256) void lingru_clear_kernel(uint4* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const uint32_t v = i < 4 ? 0u : ~0u;
        p[i] = make_uint4(v, v, v, v);
    }
}
// dst = src, or zeros.
__global__ __launch_bounds__(256) void lingru_copy_kernel(const float* src, float* dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) dst[i] = src ? src[i] : 0.0f;
}

typedef void (*LinGruFn)(LinGruArgs);

template <int ES, bool VEC, bool BWD, bool RESET>
LinGruFn tile_fn(bool few, bool chain) {
    constexpr int R = kLinGruSteps, NW = BWD ? kLinGruBwdWaves : kLinGruFwdWaves;
    if constexpr (BWD) {
        if (few) return lingru_bwd_kernel<ES, VEC, 2, R, RESET, false>;
        return chain ? lingru_bwd_kernel<ES, VEC, NW, R, RESET, true> : lingru_bwd_kernel<ES, VEC, NW, R, RESET, false>;
    } else {
        if (few) return lingru_fwd_kernel<ES, VEC, 2, R, RESET, false>;
        return chain ? lingru_fwd_kernel<ES, VEC, NW, R, RESET, true> : lingru_fwd_kernel<ES, VEC, NW, R, RESET, false>;
    }
}

// Whether every row of p has a whole piece of four, on 4 bytes (the last lanes' pieces may share
// channels, which both form alike).
bool pieces(const void* p, int64_t st, int64_t sb, const LinGruArgs& a) {
    return !p || (a.H >= 4 && (a.type == kF32 || (a.H % 2 == 0 && (uintptr_t)p % 4 == 0 && st % 2 == 0 && sb % 2 == 0)));
}

template <int ES, bool BWD>
hipError_t launch_tiles(const LinGruArgs& a, hipStream_t s) {
    const int64_t cols = a.batch * ((a.H + kCols - 1) / kCols);
    const bool few = a.T <= 64;
    const int64_t tiles = lingru_tiles(a.T, BWD), total = cols * tiles;
    if (total > INT32_MAX) return hipErrorInvalidValue;
    const bool chain = tiles > 1;
    if (chain) {
        const int64_t n = (int64_t)(lingru_chain_bytes(a.T, a.batch, a.H, BWD) / 16), blocks = (n + 255) / 256;
        hipLaunchKernelGGL(lingru_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s,
                           reinterpret_cast<uint4*>(a.chain), n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const bool vec = pieces(a.gx, a.gx_t, a.gx_b, a) && (BWD ? pieces(a.dh_seq, a.dh_t, a.dh_b, a) && pieces(a.dgx, a.dg_t, a.dg_b, a)
                                                             : pieces(a.h_seq, a.h_t, a.h_b, a));
    const LinGruFn fn = vec ? (a.reset ? tile_fn<ES, true, BWD, true>(few, chain) : tile_fn<ES, true, BWD, false>(few, chain))
                            : (a.reset ? tile_fn<ES, false, BWD, true>(few, chain) : tile_fn<ES, false, BWD, false>(few, chain));
    hipLaunchKernelGGL(fn, dim3((unsigned)total), dim3(few ? 128 : 64 * (BWD ? kLinGruBwdWaves : kLinGruFwdWaves)), 0, s, a);
    return hipGetLastError();
}

}  // namespace

// Whether a wave's rows lie within 31 bits of its first.
bool lingru_strides(int64_t stride_t, int64_t width, int64_t es) {
    return (__int128)stride_t * es * 32 + (__int128)width * es < ((__int128)1 << 31);
}

int64_t lingru_tiles(int64_t T, bool backward) {
    const int64_t ts = 4 * kLinGruSteps * (backward ? kLinGruBwdWaves : kLinGruFwdWaves);
    return T <= 64 ? (T > 0 ? 1 : 0) : (T + ts - 1) / ts;
}

// The counter's line and 12 bytes for each tile and channel; nothing for single tiles.
size_t lingru_chain_bytes(int64_t T, int64_t batch, int64_t H, bool backward) {
    const int64_t tiles = lingru_tiles(T, backward), cols = batch * ((H + kCols - 1) / kCols);
    return tiles > 1 ? 64 + (size_t)(tiles * cols) * kCols * 12 : 0;
}

hipError_t launch_lingru_forward(const LinGruArgs& a, hipStream_t s) {
    const int64_t n = a.batch * a.H;
    if (a.T > kLinGruFew) return a.type == kBF16 ? launch_tiles<2, false>(a, s) : launch_tiles<4, false>(a, s);
    if ((n + 63) / 64 > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((a.type == kBF16 ? lingru_few_kernel<2> : lingru_few_kernel<4>), dim3((unsigned)((n + 63) / 64)), dim3(64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_lingru_backward(const LinGruArgs& a, hipStream_t s) {
    const int64_t n = a.batch * a.H, tiles = lingru_tiles(a.T, true);
    hipError_t e = hipSuccess;
    if (n > 0 && tiles > 0) {
        e = a.type == kBF16 ? launch_tiles<2, true>(a, s) : launch_tiles<4, true>(a, s);
    } else if (n > 0 && a.dh0) {
        const int64_t blocks = (n + 255) / 256;
        hipLaunchKernelGGL(lingru_copy_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, a.dh_T, a.dh0, n);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !a.dbias) return e;
    const ColSum sum{a.bias_part, a.dbias, tiles * a.batch, 2 * a.H, 1, kF32};
    return launch_colsum(&sum, 1, s);
}

}  // namespace isam
