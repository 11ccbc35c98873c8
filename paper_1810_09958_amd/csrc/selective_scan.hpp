// The selective scan: a diagonal state space whose step, input and output weights depend on
// the token.
//
//   d_t = softplus(dt_t + dt_bias)                      (a step for each channel c)
//   h_t[n] = exp(d_t A[c][n]) h_{t-1}[n] + d_t x_t B_t[n]   (h_{t-1} = 0 at a reset)
//   v_t = sum_n C_t[n] h_t[n] + skip x_t,  y_t = v_t silu(z_t)
//
// Every value of the state is one first-order recurrence over time.  Per token, channel and n
// there are an exponential, two products and two multiply-adds against 2N-th of a few bytes of
// memory, so the vector units bound it and the layout serves them:
//   * a wave holds 64 / L channels, L lanes to a channel, R values of n to a lane (N <= L R), and
//     walks the tokens one by one with the state in registers.  Four waves make a workgroup
//     of 256 / L channels;
//   * tiles of 32 tokens pass through LDS: d and d x of each (token, channel), B and C in the order
//     the lanes want them, all in fp32, formed once by all lanes and read as broadcasts;
//   * the sums over n are left in the lanes for four tokens and then exchanged by half-wave and row
//     swaps that halve the values at each level, so a token costs one and a half exchanges.
// Where the channels are too few for the chip, time is cut into segments: a first kernel leaves
// each segment's end state from zero and the sum of its steps (its map is h -> exp(A sum d) h + end),
// and each workgroup of the scan composes those before its own.
// Counted over the whole kernels (bf16, N 16), a token costs a wave of 8 channels 18 vector instructions in 85 cycles
// forward and 62 in 268 backward, and the compute unit 58 and 170 cycles of LDS for its four waves (16 and 65 of them
// bank conflicts): the vector units are busy for 65-82 % of the time, the LDS for about half.
// 2048x8x1024 (tokens, sequences, channels), N 16, bf16, in a kernel trace: summaries 57 us and scan 111; backward
// summaries 65, gradient 347, sums of dB and dC 16.
#pragma once

#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

constexpr int kScanTile = 32;    // tokens of a tile
constexpr int kScanWaves = 4;    // waves of a workgroup
constexpr float kScanLog2e = 1.44269504f;

// softplus(v) = max(v, 0) + log(1 + u), u = exp(-|v|) in (0, 1]: log(1 + u) = 2 artanh(s) with
// s = u / (2 + u) <= 1/3, by its series (the first term left out is 2 s^15 / 15, below 2^-26 of the sum).
// To a few units of 2^-24 relative to itself, and for v below 0 another |v| 2^-24 from the exponential's rounded argument
// (2^-18 at -80); 0 below -87.3, where u is subnormal and flushed.  NaN passes.
__device__ __forceinline__ float softplus(float v) {
    const float u = __builtin_amdgcn_exp2f(__builtin_fabsf(v) * -kScanLog2e);
    const float s = u * __builtin_amdgcn_rcpf(2.0f + u), y = s * s;
    float p = __builtin_fmaf(y, 1.0f / 13, 1.0f / 11);
    p = __builtin_fmaf(p, y, 1.0f / 9);
    p = __builtin_fmaf(p, y, 1.0f / 7);
    p = __builtin_fmaf(p, y, 1.0f / 5);
    p = __builtin_fmaf(p, y, 1.0f / 3);
    p = __builtin_fmaf(p * y, s, s);
    return __builtin_fmaf(2.0f, p, v > 0.0f ? v : 0.0f);
}

// E consecutive values of a row, as words; from `off` bytes of a buffer (kOob: zeros, or not
// stored).  VEC: as one piece, on 4 bytes; otherwise one by one, `valid` of them.
template <int ES, bool VEC, int E>
struct Piece {
    static constexpr int W = (E * ES + 3) / 4;
    uint32_t w[W];

    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t off, int valid) {
        if constexpr (VEC && W >= 4) {
            static_for<W / 4>([&](auto q) {
                const uint4 v = buf_load16(rs, off == kOob ? kOob : off + 16u * q);
                w[4 * q] = v.x; w[4 * q + 1] = v.y; w[4 * q + 2] = v.z; w[4 * q + 3] = v.w;
            });
        } else if constexpr (VEC && W == 2) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)off, 0, 0);
            w[0] = (uint32_t)v[0];
            w[1] = (uint32_t)v[1];
        } else if constexpr (VEC) {
            w[0] = buf_load4(rs, off);
        } else {
            static_for<W>([&](auto k) { w[k] = 0; });
            static_for<E>([&](auto e) {
                const uint32_t at = e < valid ? off + (uint32_t)(e * ES) : kOob;
                if constexpr (ES == 4) w[e] = buf_load4(rs, at);
                else w[e / 2] |= (buf_load2(rs, at) & 0xffffu) << (16 * (e & 1));
            });
        }
    }
    __device__ __forceinline__ void unpack(float (&f)[E]) const {
        static_for<E>([&](auto e) {
            if constexpr (ES == 4) f[e] = __uint_as_float(w[e]);
            else if constexpr (e & 1) f[e] = bf16hi(w[e / 2]);
            else f[e] = bf16lo(w[e / 2]);
        });
    }
    // bf16: rounded to nearest even.
    __device__ __forceinline__ static void store(__amdgpu_buffer_rsrc_t rs, uint32_t off, int valid, const float (&f)[E]) {
        uint32_t o[W];
        static_for<W>([&](auto k) {
            if constexpr (ES == 4) o[k] = __float_as_uint(f[k]);
            else if constexpr (E == 1) o[k] = pack_bf16_rne(f[0], 0.0f);
            else o[k] = pack_bf16_rne(f[2 * k], f[2 * k + 1]);
        });
        if constexpr (VEC && W >= 4) {
            static_for<W / 4>([&](auto q) {
                __builtin_amdgcn_raw_buffer_store_b128((i32x4_t){(int)o[4 * q], (int)o[4 * q + 1], (int)o[4 * q + 2], (int)o[4 * q + 3]}, rs,
                                                       (int)(off == kOob ? kOob : off + 16u * q), 0, 0);
            });
        } else if constexpr (VEC && W == 2) {
            __builtin_amdgcn_raw_buffer_store_b64((i32x2_t){(int)o[0], (int)o[1]}, rs, (int)off, 0, 0);
        } else if constexpr (VEC) {
            __builtin_amdgcn_raw_buffer_store_b32((int)o[0], rs, (int)off, 0, 0);
        } else {
            static_for<E>([&](auto e) {
                const int at = (int)(e < valid ? off + (uint32_t)(e * ES) : kOob);
                if constexpr (ES == 4) __builtin_amdgcn_raw_buffer_store_b32((int)o[e], rs, at, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b16((short)(o[e / 2] >> (16 * (e & 1))), rs, at, 0, 0);
            });
        }
    }
};

// Rows of one sequence in a [T][batch] tensor, a tile at a time: from token t0 on, as a buffer.
template <int ES>
struct TileRows {
    const char* p;       // null: no rows
    uint32_t row;        // bytes from a token to the next (a tile stays below 2^31)
    __device__ __forceinline__ TileRows(const ScanRows& r, int64_t b, int64_t t0) {
        p = r.p ? static_cast<const char*>(r.p) + (b * r.sb + t0 * r.st) * ES : nullptr;
        row = r.p ? (uint32_t)(r.st * ES) : 0u;
    }
    __device__ __forceinline__ void forth() { p += row * (uint32_t)kScanTile; }
    __device__ __forceinline__ void back() { p -= row * (uint32_t)kScanTile; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const { return make_rsrc(p, p ? 0x7fffffffu : 0u); }
};

// How a workgroup's lanes stand to its channels, states and tiles.
template <int ES, bool VEC, int L, int R>
struct ScanShape {
    static constexpr int CW = 64 / L;              // channels of a wave
    static constexpr int CH = kScanWaves * CW;     // of the workgroup
    static constexpr int E = CH * kScanTile / 256; // values of a tile that a thread loads: one piece of a row
    static constexpr int PPR = CH / E;             // pieces of a row
    static constexpr int NP = L * R;               // N, padded
    static constexpr int CK = scan_chunk(NP);      // (the same for every N of this instance)
    static constexpr int BE = kScanTile * NP / 256;  // values of B (and of C) of a tile that a thread loads
    static_assert(PPR * kScanTile == 256, "one piece a thread");
    using P = Piece<ES, VEC, E>;
};

// B and C of a tile: value i of thread tid is n = (tid + 256 i) % NP of token (tid + 256 i) / NP.
template <int ES, int NP>
struct ScanWeights {
    static constexpr int BE = (kScanTile * NP + 255) / 256;
    uint16_t h[ES == 2 ? BE : 1];
    float f[ES == 4 ? BE : 1];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t row, int N, int left, int tid) {
        static_for<BE>([&](auto i) {
            const int idx = tid + 256 * i, t = idx / NP, n = idx % NP;
            const uint32_t off = t < left && n < N ? (uint32_t)t * row + (uint32_t)(n * ES) : kOob;  // (left <= the tile)
            if constexpr (ES == 4) f[i] = __uint_as_float(buf_load4(rs, off));
            else h[i] = (uint16_t)buf_load2(rs, off);
        });
    }
    // Whether one of them is an infinity or NaN.
    __device__ __forceinline__ bool wild() const {
        bool any = false;
        static_for<BE>([&](auto i) {
            if constexpr (ES == 4) any = any || (__float_as_uint(f[i]) & 0x7f800000u) == 0x7f800000u;
            else any = any || (h[i] & 0x7f80u) == 0x7f80u;
        });
        return any;
    }
    // To LDS: [token][lane group][B or C][R].
    template <int R>
    __device__ __forceinline__ void put(float* bc, int which, int tid) const {
        static_for<BE>([&](auto i) {
            const int idx = tid + 256 * i, t = idx / NP, n = idx % NP;
            float v;
            if constexpr (ES == 4) v = f[i];
            else v = bf16_to_f32(h[i]);
            if (kScanTile * NP % 256 == 0 || t < kScanTile) bc[t * NP * 2 + (n / R) * 2 * R + which * R + n % R] = v;
        });
    }
};

// R floats from LDS (aligned to their size).
template <int R>
__device__ __forceinline__ void lds_get(const float* p, float (&f)[R]) {
    if constexpr (R >= 4) {
        static_for<R / 4>([&](auto q) {
            const float4 v = *reinterpret_cast<const float4*>(p + 4 * q);
            f[4 * q] = v.x; f[4 * q + 1] = v.y; f[4 * q + 2] = v.z; f[4 * q + 3] = v.w;
        });
    } else if constexpr (R == 2) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        f[0] = v.x; f[1] = v.y;
    } else {
        f[0] = p[0];
    }
}

// What a token brings to a lane: d, d x and the lane's values of B and C.
template <int L, int R, bool WITH_C>
struct ScanToken {
    float2 s;
    float B[R], C[WITH_C ? R : 1];
    __device__ __forceinline__ void get(const float2& at, const float* bc, int t, int g) {
        s = at;
        lds_get<R>(bc + (t * L + g) * 2 * R, B);
        if constexpr (WITH_C) lds_get<R>(bc + (t * L + g) * 2 * R + R, C);
    }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int kDppXor1 = 0xb1, kDppXor2 = 0x4e, kDppHalfMirror = 0x141, kDppRor8 = 0x128;

// a and b with the upper half of a and the lower half of b exchanged (32: half waves; 16: rows of
// 16 within each half), then added.
__device__ __forceinline__ float swap_add32(float a, float b) {
    const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(v[0]) + __uint_as_float(v[1]);
}
__device__ __forceinline__ float swap_add16(float a, float b) {
    const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(v[0]) + __uint_as_float(v[1]);
}
// The sums over a channel's L lanes of four values: lane l has that of value l / 16 (for its
// channel l % CW, in every lane of the row with that channel).
template <int L>
__device__ __forceinline__ float sum_lanes4(const float (&p)[4]) {
    float s = swap_add16(swap_add32(p[0], p[2]), swap_add32(p[1], p[3]));
    if constexpr (L >= 8) s += dpp<kDppRor8>(s);
    if constexpr (L >= 16) s += dpp<0x124>(s);  // row_ror 4: each quad now holds the same sums
    return s;
}

// Reset marks of a tile's tokens: a byte to a lane, turned into a bit each where they are used (the loads of a
// tile are on their way during the one before).
struct ScanMarks {
    uint32_t byte = 0;
    __device__ __forceinline__ void load(const ScanArgs& a, int64_t b, int64_t t0, int left, int lane) {
        if (!a.reset) return;
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.reset + b * a.rs_b + t0 * a.rs_t, 0x7fffffffu);
        byte = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rs, (int)(lane < left ? (uint32_t)lane * (uint32_t)a.rs_t : kOob), 0, 0);
    }
    __device__ __forceinline__ uint32_t bits() const { return (uint32_t)__ballot((byte & 0xffu) != 0); }  // (left <= the tile)
};

__device__ __forceinline__ bool not_finite(float v) { return !(__builtin_fabsf(v) < __builtin_inff()); }

// A barrier; and, where N or the channels are padded, whether a thread before it had an infinity or NaN that meets the
// zeros there.
__device__ __forceinline__ bool meet(bool padded, bool wild) {
    if (padded) return __syncthreads_or(wild);
    __syncthreads();
    return false;
}

// Segments: [segment][batch][D] sums of steps (sign bit set: a reset lies inside, nothing passes),
// and [segment][batch][D][N] end states from zero.  What passes is at least 2^-126 of h, so that an infinity stays one
// where the tokens' factors are above zero and their product is not.  A product above 2^126 (states that grow) goes in
// three equal factors: no infinity meets a state of zero, and a small state grows as far as token by token.
__device__ __forceinline__ float pass_on(float sum, float a2, float h, float end) {
    const float e = sum * a2;
    const bool far = e > 126.0f;
    const float f = fmaxf(__builtin_amdgcn_exp2f(far ? fminf(e, 378.0f) * (1.0f / 3) : e), 0x1p-126f), again = far ? f : 1.0f;
    return (int)__float_as_uint(sum) < 0 ? end : __builtin_fmaf(f, h * again * again, end);
}

// Instances by N and type: (lanes to a channel, values to a lane).
struct ScanShapeOf {
    int L, R;
};
inline ScanShapeOf scan_shape(int64_t N) {
    if (N <= 4) return {4, 1};
    if (N <= 8) return {8, 1};
    if (N <= 16) return {8, 2};
    if (N <= 32) return {16, 2};
    return {16, 4};
}

}  // namespace isam
