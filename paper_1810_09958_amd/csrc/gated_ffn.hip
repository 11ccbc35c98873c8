// Launch of the gated feed-forward kernels, the kernel for a few tokens and the
// element-wise step of the fp32 path.
#include "gated_ffn.hpp"

namespace isam {

namespace {

typedef void (*GatedFn)(GatedArgs, TileMapArgs);

TileMapArgs tile_map(int64_t tiles_m, int64_t tiles_n) {
    TileMapArgs t{};
    t.tiles_m = (int)tiles_m;
    t.tiles_n = (int)tiles_n;
    t.group_m = 8;
    t.xcd_remap = 1;
    return t;
}

// A few tokens (M <= 16): the weights are streamed once, straight into the
// matrix instructions' operand registers, 16 rows of Wg and the same 16 of Wu
// per workgroup; its eight waves take every eighth K step and their sums meet
// in LDS.  x (the other operand: a column per token) comes from the caches.
// Bound by the stream of W: 16.8 MB at one token of 1024x4096 bf16, 6.7-7.0 us a call (16
// tokens 6.4; fp32 8.0 and 8.9).
// BWD (bf16): [dG dU] instead, in two bf16 terms, the high ones in rows 0 .. M - 1 and what they
// leave in rows M .. 2M - 1, so that dx and dW carry the rounding of the output alone: a norm error
// of 1.66e-3, against 2.35e-3 with dG and dU rounded once (at any number of rows: terms and errors
// grow alike). The price is twice the operations of both products: nothing while W's bytes bound
// them (dx and dW 12.8 and 14.1 us with one term and 12.9 and 14.2 with two at 16x1024x4096), 95 to
// 166 us for both at 2048x1024x4096, so blocks of more rows round dG and dU.
template <int ES, bool BWD>
__global__ __launch_bounds__(512) void gated_token_kernel(GatedArgs a) {
    using IO = Row16<ES>;
    constexpr int E = IO::E, KS = 4 * E, U = 4;  // values of K of a lane, of a step; steps in flight
    __shared__ float sums[8][2][4][64];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, li = lane & 15, g = lane >> 4;
    const int64_t f0 = (int64_t)blockIdx.x * 16, f = f0 + li;
    const int nk = (int)((a.K + KS - 1) / KS);
    f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int s0 = wid; s0 < nk; s0 += 8 * U) {
        uint4 wg[U], wu[U], x[U];
        static_for<U>([&](auto u) {
            const int64_t k = (int64_t)(s0 + 8 * u) * KS + g * E;
            const int valid = (int)max((int64_t)0, min((int64_t)E, a.K - k));
            wg[u] = IO::load(a.W, f * a.ld_w + k, f < a.F ? valid : 0);
            wu[u] = IO::load(a.W, (a.F + f) * a.ld_w + k, f < a.F ? valid : 0);
            x[u] = IO::load(a.x, li * a.ld_x + k, li < a.M ? valid : 0);
        });
        static_for<U>([&](auto u) {
            if constexpr (ES == 2) {
                mfma16_bf16(acc[0], wg[u], x[u]);
                mfma16_bf16(acc[1], wu[u], x[u]);
            } else {
                mfma16_f32x4(acc[0], wg[u], x[u]);
                mfma16_f32x4(acc[1], wu[u], x[u]);
            }
        });
    }
    static_for<2>([&](auto j) { static_for<4>([&](auto v) { sums[wid][j][v][lane] = acc[j][decltype(v)::value]; }); });
    __syncthreads();
    if (BWD && f0 + 16 >= a.F) {
        GatedArgs both = a;
        both.M = 2 * a.M;
        gated_pad<2>(both, 0, (int)both.M, threadIdx.x, 512);
    }
    // thread (v, lane) of the first four waves: f = f0 + 4 g + v, token li
    if (wid >= 4) return;
    const int v = wid;
    float G = 0.0f, Uv = 0.0f;
    for (int w = 0; w < 8; ++w) {
        G += sums[w][0][v][lane];
        Uv += sums[w][1][v][lane];
    }
    const int64_t fo = f0 + 4 * g + v;
    if (!BWD && (fo >= a.F || li >= a.M)) return;
    const bool on = fo < a.F && li < a.M;
    if (a.bias && fo < a.F) {
        G += a.bias[fo];
        Uv += a.bias[a.F + fo];
    }
    float slope;
    const float s = a.act == 0 ? gate_act<0>(G, slope) : a.act == 1 ? gate_act<1>(G, slope) : gate_act<2>(G, slope);
    if constexpr (!BWD) {
        IO::put(a.out, (int64_t)li * a.ld_out + fo, s * Uv);
    } else {
        const float dp = on ? IO::get(a.dout, (int64_t)li * a.ld_dout + fo) : 0.0f;
        float d[2] = {on ? dp * Uv * slope : 0.0f, on ? dp * s : 0.0f};
        if (on) {
            static_for<2>([&](auto h) {
                const int64_t at = (int64_t)li * a.ld_out + h * a.F + fo;
                const float high = bf16_to_f32((uint16_t)pack_bf16_rne(d[h], 0.0f)), low = d[h] - high;
                IO::put(a.out, at, high);
                // (nothing is left of what the high term cannot hold: infinities, NaN)
                IO::put(a.out, at + a.M * a.ld_out, low - low == 0.0f ? low : 0.0f);
            });
        }
        static_for<4>([&](auto k) {
            static_for<2>([&](auto h) { d[h] += __shfl_xor(d[h], 1 << decltype(k)::value); });
        });
        if (a.bias_part && li == 0 && fo < a.F) {
            a.bias_part[fo] = d[0];
            a.bias_part[a.F + fo] = d[1];
        }
    }
}

// dx = the sum of the two terms' products, [2][M][K] fp32 at a.gu.
__global__ __launch_bounds__(256) void gated_join_kernel(GatedArgs a) {
    const int64_t n = a.M * a.K;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / a.K;
        Row16<2>::put(a.out, m * a.ld_out + (i - m * a.K), a.gu[i] + a.gu[n + i]);
    }
}

// fp32 blocks of few tiles: 32 rows x 32 values of f, gate and up, on the fp32 matrix
// instructions, straight from memory (any alignment of 4 bytes) into their operand
// registers.  The four waves take every fourth 16-deep K step (32 matrix instructions
// on 6 loads, two steps in flight) and meet in LDS, each wave then holding one 16 x 16
// quarter of G and U for the epilogue.  G and U never reach memory, and no operand is
// copied or split into bf16 terms first, which is what bounds small products; larger
// ones are bound by the fp32 matrix rate (an eighth of what the terms need of bf16's)
// and go through the library's product.
template <bool BWD>
__global__ __launch_bounds__(256, 2) void gated_f32_kernel(GatedArgs a, TileMapArgs tmap) {
    __shared__ float sums[4][32][64];
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, g = lane >> 4;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * kGatedF32Tile, f0 = (int64_t)tn * kGatedF32Tile;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, (uint32_t)(((a.M - 1) * a.ld_x + a.K) * 4));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.W, (uint32_t)(((2 * a.F - 1) * a.ld_w + a.K) * 4));
    // rows of x, then gate and up rows of W: byte offset of the lane's four values of step 0
    uint32_t at[6];
    static_for<2>([&](auto i) {
        const int64_t m = m0 + 16 * i + li, f = f0 + 16 * i + li;
        at[i] = m < a.M ? (uint32_t)((m * a.ld_x + 4 * g) * 4) : kOob;
        at[2 + i] = f < a.F ? (uint32_t)((f * a.ld_w + 4 * g) * 4) : kOob;
        at[4 + i] = f < a.F ? (uint32_t)(((a.F + f) * a.ld_w + 4 * g) * 4) : kOob;
    });
    f32x4_t acc[2][2][2];  // [rows][f][gate, up]
    static_for<2>([&](auto i) {
        static_for<2>([&](auto j) { static_for<2>([&](auto h) { acc[i][j][h] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }); });
    });
    const int steps = (int)(a.K / 16);
    auto load = [&](uint4 (&v)[6], int s) {
        static_for<6>([&](auto o) {
            const uint32_t off = s < steps && at[o] != kOob ? at[o] + (uint32_t)s * 64u : kOob;
            v[o] = buf_load16(o < 2 ? rx : rw, off);
        });
    };
    auto multiply = [&](const uint4 (&v)[6]) {
        static_for<2>([&](auto i) {
            static_for<2>([&](auto j) {
                mfma16_f32x4(acc[i][j][0], v[i], v[2 + j]);
                mfma16_f32x4(acc[i][j][1], v[i], v[4 + j]);
            });
        });
    };
    uint4 b0[6], b1[6];
    load(b0, wid);
    load(b1, wid + 4);
    for (int s = wid; s < steps; s += 8) {  // (steps past the end are zeros)
        multiply(b0);
        load(b0, s + 8);
        multiply(b1);
        load(b1, s + 12);
    }
    if (a.K % 16 && wid == (steps & 3)) {  // the last values of the rows, one by one
        const int k = steps * 16 + 4 * g;
        uint4 v[6];
        static_for<6>([&](auto o) {
            uint32_t w[4];
            static_for<4>([&](auto e) {
                w[e] = buf_load4(o < 2 ? rx : rw, k + e < a.K && at[o] != kOob ? at[o] + (uint32_t)steps * 64u + 4u * e : kOob);
            });
            v[o] = make_uint4(w[0], w[1], w[2], w[3]);
        });
        multiply(v);
    }
    static_for<2>([&](auto i) {
        static_for<2>([&](auto j) {
            static_for<2>([&](auto h) {
                static_for<4>([&](auto v) { sums[wid][((i * 2 + j) * 2 + h) * 4 + v][lane] = acc[i][j][h][decltype(v)::value]; });
            });
        });
    });
    __syncthreads();
    // this wave's quarter: rows mq + 4 g + v, column f
    const int64_t mq = m0 + 16 * (wid >> 1), f = f0 + 16 * (wid & 1) + li;
    const bool in = f < a.F;
    const float bg = a.bias && in ? a.bias[f] : 0.0f, bu = a.bias && in ? a.bias[a.F + f] : 0.0f;
    const int64_t cols = BWD ? 2 * a.F : a.F;
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(BWD ? a.dout : nullptr, BWD ? (uint32_t)(((a.M - 1) * a.ld_dout + a.F) * 4) : 0u);
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, (uint32_t)(((a.M - 1) * a.ld_out + cols) * 4));
    float sg = 0.0f, su = 0.0f;
    static_for<4>([&](auto v) {
        const int64_t m = mq + 4 * g + v;
        const bool on = in && m < a.M;
        float G = bg, U = bu;
        static_for<4>([&](auto w) {
            G += sums[w][wid * 8 + v][lane];
            U += sums[w][wid * 8 + 4 + v][lane];
        });
        float slope;
        const float s = a.act == 0 ? gate_act<0>(G, slope) : a.act == 1 ? gate_act<1>(G, slope) : gate_act<2>(G, slope);
        const uint32_t to = on ? (uint32_t)((m * a.ld_out + f) * 4) : kOob;
        if constexpr (BWD) {
            const float dp = __uint_as_float(buf_load4(rp, on ? (uint32_t)((m * a.ld_dout + f) * 4) : kOob));
            const float dg = dp * U * slope, du = dp * s;
            __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(dg), ro, (int)to, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(du), ro, (int)(on ? to + (uint32_t)(a.F * 4) : kOob), 0, 0);
            sg += on ? dg : 0.0f;
            su += on ? du : 0.0f;
        } else {
            __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(s * U), ro, (int)to, 0, 0);
        }
    });
    if (BWD && f0 + kGatedF32Tile >= a.F) gated_pad<4>(a, m0, (int)min(kGatedF32Tile, a.M - m0), threadIdx.x, 256);
    if (BWD && a.bias_part) {  // one partial row for every 16 rows
        static_for<2>([&](auto k) {
            sg += __shfl_xor(sg, 16 << decltype(k)::value);
            su += __shfl_xor(su, 16 << decltype(k)::value);
        });
        float* const part = a.bias_part + (int64_t)(tm * 2 + (wid >> 1)) * 2 * a.F;
        if (in && g == 0) {
            part[f] = sg;
            part[a.F + f] = su;
        }
    }
}

// fp32: p, or (BWD) dG and dU in place, from G and U in memory ([M][2F] at
// a.gu).  A workgroup takes 64 columns of f and kGatedRows rows, four at a time,
// and leaves one partial row of the bias gradient.
template <bool BWD>
__global__ __launch_bounds__(256) void gated_pairs_kernel(GatedArgs a) {
    __shared__ float sums[2][4][64];
    const int cl = threadIdx.x & 63, rl = threadIdx.x >> 6;
    const int64_t f = (int64_t)blockIdx.x * 64 + cl, m0 = (int64_t)blockIdx.y * kGatedRows, m1 = min(a.M, m0 + kGatedRows);
    float sg = 0.0f, su = 0.0f;
    if (f < a.F) {
        const float bg = a.bias ? a.bias[f] : 0.0f, bu = a.bias ? a.bias[a.F + f] : 0.0f;
#pragma unroll 4
        for (int64_t m = m0 + rl; m < m1; m += 4) {
            float* const gu = a.gu + m * 2 * a.F + f;
            const float G = gu[0] + bg, U = gu[a.F] + bu;
            float slope;
            const float s = a.act == 0 ? gate_act<0>(G, slope) : a.act == 1 ? gate_act<1>(G, slope) : gate_act<2>(G, slope);
            if constexpr (BWD) {
                const float dp = static_cast<const float*>(a.dout)[m * a.ld_dout + f], dg = dp * U * slope, du = dp * s;
                gu[0] = dg;
                gu[a.F] = du;
                sg += dg;
                su += du;
            } else {
                static_cast<float*>(a.out)[m * a.ld_out + f] = s * U;
            }
        }
    }
    if constexpr (BWD) {
        sums[0][rl][cl] = sg;
        sums[1][rl][cl] = su;
        __syncthreads();
        if (!a.bias_part || rl != 0 || f >= a.F) return;
        float* const out = a.bias_part + (int64_t)blockIdx.y * 2 * a.F + f;
        out[0] = (sums[0][0][cl] + sums[0][1][cl]) + (sums[0][2][cl] + sums[0][3][cl]);
        out[a.F] = (sums[1][0][cl] + sums[1][1][cl]) + (sums[1][2][cl] + sums[1][3][cl]);
    }
}

template <bool BWD>
GatedFn tile_fn(int tile, bool k_full) {
    switch (tile) {
        case kGated256: return k_full ? gated_dma_kernel<256, 256, 2, 4, true, BWD> : gated_dma_kernel<256, 256, 2, 4, false, BWD>;
        case kGated128: return k_full ? gated_dma_kernel<128, 128, 2, 2, true, BWD> : gated_dma_kernel<128, 128, 2, 2, false, BWD>;
        default: return gated_ring_kernel<BWD>;
    }
}

}  // namespace

// bf16 tiles, by the rounds of workgroups they take on the compute units: 64 rows x 32 values of
// f (two workgroups to a compute unit) while they need one round; else 128 x 64 or 256 x 128, whose
// round does four times the work in 3.3 times the time. us forward of tiles of 256 / 128 / 64
// rows (tiles): 512x4096x2048 66 / 34 / 28 (32, 128, 512), 576x4096x2048 64 / 34 / 45 (48, 160, 640),
// 576x256x2048 10.3 / 6.9 / 8.3, 896x1024x2048 21.5 / 10.8 / 16.9 (64, 224, 896), 1024x1024x4096 25 / 20 / 35
// (128, 512), 1792x1024x4096 31 / 33 (224, 896), 2048x1024x4096 33 / 36 (256, 1024), 2304x1024x4096
// 51 / 43 (288, 1152), 2944x1024x4096 53 / 51 (384, 1472), 3328x1024x4096 55 / 58 (416, 1664), 5120x4096x4096
// 275 / 302 (640, 2560). The backward kernel's times lie alike.
int gated_tile(int64_t M, int64_t F, int cus) {
    auto tiles = [&](int64_t bm, int64_t hb) { return ((M + bm - 1) / bm) * ((F + hb - 1) / hb); };
    auto rounds = [&](int64_t n) { return (n + cus - 1) / cus; };
    if (tiles(64, 32) <= 2 * (int64_t)cus) return kGated64;
    return 10 * rounds(tiles(128, 64)) < 33 * rounds(tiles(256, 128)) ? kGated128 : kGated256;
}

int64_t gated_bias_rows(int tile, int64_t M) {
    const int64_t bm = tile == kGated256 ? 256 : tile == kGated128 ? 128 : 64;
    return (M + bm - 1) / bm * 2;  // two wave rows a tile
}

hipError_t launch_gated_tiles(const GatedArgs& a, int tile, bool backward, hipStream_t s) {
    const int64_t bm = tile == kGated256 ? 256 : tile == kGated128 ? 128 : 64, hb = bm / 2;
    const int64_t tm = (a.M + bm - 1) / bm, tn = (a.F + hb - 1) / hb;
    if (tm * tn > INT32_MAX || a.K <= 0) return hipErrorInvalidValue;
    const bool k_full = a.K % 64 == 0;
    const GatedFn fn = backward ? tile_fn<true>(tile, k_full) : tile_fn<false>(tile, k_full);
    GatedArgs p = a;
    auto on4 = [](const void* q, int64_t ld) { return (uintptr_t)q % 4 == 0 && ld % 2 == 0; };
    p.whole = a.F % 8 == 0 && on4(a.out, a.ld_out) && (!backward || on4(a.dout, a.ld_dout));
    hipLaunchKernelGGL(fn, dim3((unsigned)(tm * tn)), dim3(tile == kGated256 ? 512 : 256), 0, s, p, tile_map(tm, tn));
    return hipGetLastError();
}

hipError_t launch_gated_tokens(const GatedArgs& a, int type, bool backward, hipStream_t s) {
    if (a.M > kGatedTokens || (a.F + 15) / 16 > INT32_MAX || (backward && type != kBF16)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((backward ? gated_token_kernel<2, true> : type == kBF16 ? gated_token_kernel<2, false> : gated_token_kernel<4, false>),
                       dim3((unsigned)((a.F + 15) / 16)), dim3(512), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_gated_join(const GatedArgs& a, hipStream_t s) {
    const int64_t blocks = (a.M * a.K + 255) / 256;
    hipLaunchKernelGGL(gated_join_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Where gated_f32_kernel is taken: up to 24 rounds of 64 values of K on a compute unit.
// us forward, this kernel / product and element-wise step (rounds): 32x64x64 7.3 / 10.1 (1),
// 128x512x2048 10.2 / 17.8 (8), 64x1024x1024 15.7 / 15.6, 256x1024x1024 15.8 / 24.1 and
// 500x511x771 16.0 / 27.7 (16), 100x333x5001 18.6 / 27.0 (18), 512x512x2048 28.3 / 27.6 (32),
// 1000x1000x1000 41.3 / 42.2 and 32x4096x512 46.5 / 20.8 (64), 512x2048x2048 90 / 69 (128).
bool gated_f32_direct(int64_t M, int64_t K, int64_t F, int cus) {
    const int64_t tiles = ((M + kGatedF32Tile - 1) / kGatedF32Tile) * ((F + kGatedF32Tile - 1) / kGatedF32Tile);
    return (K + 63) / 64 <= 24 && (K + 63) / 64 * ((tiles + cus - 1) / cus) <= 24;
}

hipError_t launch_gated_f32(const GatedArgs& a, bool backward, hipStream_t s) {
    const int64_t tm = (a.M + kGatedF32Tile - 1) / kGatedF32Tile, tn = (a.F + kGatedF32Tile - 1) / kGatedF32Tile;
    if (tm * tn > INT32_MAX || a.K <= 0) return hipErrorInvalidValue;
    hipLaunchKernelGGL((backward ? gated_f32_kernel<true> : gated_f32_kernel<false>), dim3((unsigned)(tm * tn)), dim3(256), 0, s, a,
                       tile_map(tm, tn));
    return hipGetLastError();
}

hipError_t launch_gated_pairs(const GatedArgs& a, bool backward, hipStream_t s) {
    const int64_t gx = (a.F + 63) / 64, gy = (a.M + kGatedRows - 1) / kGatedRows;
    if (gx > INT32_MAX || gy > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL((backward ? gated_pairs_kernel<true> : gated_pairs_kernel<false>), dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, s,
                       a);
    return hipGetLastError();
}

}  // namespace isam
