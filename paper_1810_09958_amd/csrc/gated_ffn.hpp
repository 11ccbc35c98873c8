// The gated feed-forward block: both projections, the activation and the
// product in one kernel, and the gradient of the two projections in another.
//
//   G = x Wg^T + bg,  U = x Wu^T + bu,  p = act(G) U
//   dG = dp U act'(G),  dU = dp act(G)           (then dx = [dG dU] W, dW = [dG dU]^T x)
//
// With W = [Wg; Wu] ([2F][K]) this is one product x W^T whose output columns f
// and F + f meet in the epilogue.  So the tiles of the library's bf16 GEMMs are
// kept and only the choice of rows changes: of a tile's BN rows of W, blocks of
// 32 alternate between gate rows and the up rows of the same f, and since each
// wave's columns are one such pair of blocks, every lane holds G and U of the
// same (m, f) in matching accumulator registers.  G and U never reach memory: a
// tile of BM x BN accumulators leaves BM x BN / 2 bf16 values of p (through
// LDS, whole rows of the tile at a time).
// The backward kernel forms G and U again with the same main loop (4 M K F
// operations, against writing and reading 2 M F values and keeping them from the
// forward pass) and leaves dG and dU, rounded to bf16 as operands of the two
// products that follow (the second rounding in dx and dW; why not two terms stands at
// gated_token_kernel); the bias gradient is summed from the unrounded values.
// Bound by the rate of the large product: 8192x2048x8192 436 us, 1.26 PFLOP/s (8192^3
// without an epilogue 1.28-1.33 on the same cards).  Training step 2048x1024x4096: forward 35 us,
// this backward kernel 44, dx 51 (128 tiles of 128x128 in two K slices), dW 38 and the
// transposed copy of its operand 13.
#pragma once

#include "gemm_dma.hpp"
#include "gemm_ring.hpp"
#include "rowio.hpp"

namespace isam {

// act(g) and its derivative.  ACT: 0 sigmoid, 1 silu, 2 gelu (erf form).
template <int ACT>
__device__ __forceinline__ float gate_act(float g, float& slope) {
    if constexpr (ACT == 2) {
        const float cdf = 0.5f * erfcf(-0.70710678f * g);
        slope = cdf + g * (0.39894228f * __expf(-0.5f * g * g));
        return g * cdf;
    } else {
        float z, omz;
        sigmoid_pair(g, z, omz);
        slope = ACT == 0 ? z * omz : z * (1.0f + g * omz);
        return ACT == 0 ? z : g * z;
    }
}

// W row of tile row r of the tile whose first f is f0; -1 past F.
__device__ __forceinline__ int64_t gated_row(int64_t F, int64_t f0, int r) {
    const int64_t f = f0 + (r >> 6) * 32 + (r & 31);
    return f < F ? ((r >> 5) & 1) * F + f : -1;
}

// The direct-to-LDS copies of gemm_dma.hpp with W's rows paired.
template <int BM, int BN, int NW>
struct GatedCopier : DmaCopier<BM, BN, true, NW> {
    using Base = DmaCopier<BM, BN, true, NW>;
    __device__ __forceinline__ GatedCopier(const GemmArgs& a, int64_t F, int64_t m0, int64_t f0, int wid, int lane)
        : Base(a, m0, 0, a.K, wid, lane) {
        static_for<Base::B_INSTR>([&](auto q) {
            const int r = ((wid * Base::B_INSTR + q) * 64 + lane) >> 3;
            const int64_t row = gated_row(F, f0, r);
            this->b_off[q] = row >= 0 ? row * a.ldb : -1;
            this->b_base[q] = row >= 0 ? (uint32_t)((row * a.ldb + this->b_k[q]) * 2) : kOob;
        });
    }
};

// Eight bf16 values from `off` bytes of a matrix, of which `valid` exist.  WHOLE: all
// or none, on 4 bytes.  What does not exist loads as zeros and is not stored; no load
// or store stands in a branch of lanes (beside nearly all registers in use, the
// compiler has copied a register inside such a branch, for its lanes only).
template <bool WHOLE>
__device__ __forceinline__ uint4 gated_load8(__amdgpu_buffer_rsrc_t rs, uint32_t off, int valid) {
    if constexpr (WHOLE) return buf_load16(rs, valid > 0 ? off : kOob);
    uint32_t h[8];
    static_for<8>([&](auto e) { h[e] = buf_load2(rs, e < valid ? off + 2 * e : kOob) & 0xffffu; });
    return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}
template <bool WHOLE>
__device__ __forceinline__ void gated_store8(__amdgpu_buffer_rsrc_t rs, uint32_t off, int valid, uint4 v) {
    if constexpr (WHOLE) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4_t, v), rs, (int)(valid > 0 ? off : kOob), 0, 0);
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        static_for<8>([&](auto e) {
            __builtin_amdgcn_raw_buffer_store_b16((short)(w[e / 2] >> (16 * (e & 1))), rs, (int)(e < valid ? off + 2 * e : kOob), 0, 0);
        });
    }
}
__device__ __forceinline__ uint32_t gated_bytes(int64_t rows, int64_t cols, int64_t ld) { return (uint32_t)(((rows - 1) * ld + cols) * 2); }

// Zeros after the 2F gradients of each of a tile's rows, up to the end of the last 16-byte piece (the products
// that follow may multiply what they read there by zero).
template <int ES>
__device__ __forceinline__ void gated_pad(const GatedArgs& a, int64_t m0, int rows, int tid, int threads) {
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, (uint32_t)(a.M * a.ld_out * ES));
    const int pad = (int)(a.ld_out - 2 * a.F);
#pragma unroll 1
    for (int r = tid; r < rows; r += threads) {
        const uint32_t at = (uint32_t)(((m0 + r) * a.ld_out + 2 * a.F) * ES);
        static_for<6>([&](auto e) {  // (2F is even)
            if constexpr (ES == 2) __builtin_amdgcn_raw_buffer_store_b16((short)0, ro, (int)(e < pad ? at + 2u * e : kOob), 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b32(0, ro, (int)(e < pad ? at + 4u * e : kOob), 0, 0);
        });
    }
}

// Epilogue of a tile of BM rows and HB = BN / 2 values of f.  `smem` is idle.
template <int ACT, bool BWD, bool WHOLE, int BM, int HB, int WM, int WTM, int MI, int NT>
__device__ __forceinline__ void gated_epilogue(const GatedArgs& a, f32x16_t (&acc)[MI][2], char* smem, int64_t m0, int64_t f0,
                                               int tm, int wm, int wn, bool active, int tid, int lane) {
    // Both indexes go through an empty asm, so that what is computed from them is not
    // held in registers across the main loop or shared by the instances.
    asm volatile("" : "+v"(lane), "+v"(tid));
    constexpr int LD = HB * 2 + 16, TILE = BM * LD, PIECES = HB / 8, RPI = NT / PIECES;
    static_assert(NT % PIECES == 0 && BM % RPI == 0, "whole rows per pass");
    const int piece = tid % PIECES, row0 = tid / PIECES, rows = (int)min((int64_t)BM, a.M - m0);
    const int valid = (int)max((int64_t)0, min((int64_t)8, a.F - (f0 + piece * 8)));
    if constexpr (BWD) {
        // dp takes the place that dG will have
        const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.dout, gated_bytes(a.M, a.F, a.ld_dout));
        const uint32_t at = (uint32_t)((m0 * a.ld_dout + f0 + piece * 8) * 2), step = (uint32_t)(a.ld_dout * 2);
        constexpr int U = WHOLE && BM / RPI >= 4 ? 4 : 1;
#pragma unroll 1
        for (int r = row0; r < BM; r += U * RPI) {
            uint4 v[U];
            static_for<U>([&](auto i) {
                const int rr = r + i * RPI;
                v[i] = gated_load8<WHOLE>(rp, at + (uint32_t)rr * step, rr < rows ? valid : 0);
            });
            static_for<U>([&](auto i) { *reinterpret_cast<uint4*>(smem + (r + i * RPI) * LD + piece * 16) = v[i]; });
        }
        __syncthreads();
    }
    if (active) {
        const int64_t f = f0 + wn * 32 + (lane & 31);
        const bool in = f < a.F;
        const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.bias, a.bias ? (uint32_t)(a.F * 8) : 0u);
        const float bg = __uint_as_float(buf_load4(rb, in ? (uint32_t)(f * 4) : kOob));
        const float bu = __uint_as_float(buf_load4(rb, in ? (uint32_t)((a.F + f) * 4) : kOob));
        float sg = 0.0f, su = 0.0f;
        static_for<MI>([&](auto i) {
            static_for<16>([&](auto v) {
                const int r = wm * WTM + i * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
                uint16_t* const at = reinterpret_cast<uint16_t*>(smem + r * LD + (wn * 32 + (lane & 31)) * 2);
                const float u = acc[i][1][decltype(v)::value] + bu;
                float slope;
                const float s = gate_act<ACT>(acc[i][0][decltype(v)::value] + bg, slope);
                if constexpr (BWD) {
                    const float dp = bf16_to_f32(*at), dg = dp * u * slope, du = dp * s;
                    const uint32_t w = pack_bf16_rne(dg, du);
                    at[0] = (uint16_t)w;
                    at[TILE / 2] = (uint16_t)(w >> 16);
                    sg += r < rows ? dg : 0.0f;
                    su += r < rows ? du : 0.0f;
                } else {
                    *at = (uint16_t)pack_bf16_rne(s * u, 0.0f);
                }
                // Four values at a time: the compiler would hold all of dG and dU in registers
                // and sum them where the sums are used.
                if constexpr (BWD && (v & 3) == 3) {
                    asm volatile("" : "+v"(sg), "+v"(su));
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
        });
        if (BWD && a.bias_part) {
            // the two lane halves hold the other rows of the same f; one partial row per wave row
            sg += __shfl_xor(sg, 32);
            su += __shfl_xor(su, 32);
            const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.bias_part + ((int64_t)tm * WM + wm) * 2 * a.F, (uint32_t)(a.F * 8));
            const bool on = in && lane < 32;
            __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(sg), ro, (int)(on ? (uint32_t)(f * 4) : kOob), 0, 0);
            __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(su), ro, (int)(on ? (uint32_t)((a.F + f) * 4) : kOob), 0, 0);
        }
    }
    __syncthreads();
    const int64_t cols = BWD ? 2 * a.F : a.F;
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, gated_bytes(a.M, cols, a.ld_out));
    const uint32_t at = (uint32_t)((m0 * a.ld_out + f0 + piece * 8) * 2), step = (uint32_t)(a.ld_out * 2), half = (uint32_t)(a.F * 2);
#pragma unroll 2
    for (int r = row0; r < BM; r += RPI) {
        const char* const src = smem + r * LD + piece * 16;
        const int n = r < rows ? valid : 0;
        gated_store8<WHOLE>(ro, at + (uint32_t)r * step, n, *reinterpret_cast<const uint4*>(src));
        if constexpr (BWD) gated_store8<WHOLE>(ro, at + (uint32_t)r * step + half, n, *reinterpret_cast<const uint4*>(src + TILE));
    }
    if constexpr (BWD && !WHOLE) {
        if (f0 + HB >= a.F) gated_pad<2>(a, m0, rows, tid, NT);
    }
}

template <bool BWD, int BM, int HB, int WM, int WTM, int MI, int NT>
__device__ __forceinline__ void gated_finish(const GatedArgs& a, f32x16_t (&acc)[MI][2], char* smem, int64_t m0, int64_t f0, int tm,
                                             int wm, int wn, bool active, int tid, int lane) {
    auto act = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (a.act == 0) gated_epilogue<0, BWD, W, BM, HB, WM, WTM, MI, NT>(a, acc, smem, m0, f0, tm, wm, wn, active, tid, lane);
        else if (a.act == 1) gated_epilogue<1, BWD, W, BM, HB, WM, WTM, MI, NT>(a, acc, smem, m0, f0, tm, wm, wn, active, tid, lane);
        else gated_epilogue<2, BWD, W, BM, HB, WM, WTM, MI, NT>(a, acc, smem, m0, f0, tm, wm, wn, active, tid, lane);
    };
    if (a.whole) act(std::true_type{});
    else act(std::false_type{});
}

__device__ __forceinline__ GemmArgs gated_gemm(const GatedArgs& a) {
    GemmArgs p{};
    p.A = a.x;
    p.B = a.W;
    p.M = a.M;
    p.N = 2 * a.F;
    p.K = a.K;
    p.lda = a.ld_x;
    p.ldb = a.ld_w;
    return p;
}

// Large tiles: the three-stage ring of gemm_dma.hpp.
template <int BM, int BN, int WM, int WN, bool KFULL, bool BWD>
__global__ __launch_bounds__(64 * WM * WN, BM == 128 ? 2 : 1) void gated_dma_kernel(GatedArgs a, TileMapArgs tmap) {
    constexpr int NW = WM * WN, WTM = BM / WM, MI = WTM / 32, HB = BN / 2;
    static_assert(BN / WN == 64, "a wave's columns are one gate block and one up block");
    constexpr int LDS = BM * 128 * 2 + BN * 128 * 3;
    static_assert((BWD ? 2 : 1) * BM * (HB * 2 + 16) <= LDS, "epilogue staging must fit in LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid / WN, wn = wid % WN;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, f0 = (int64_t)tn * HB;
    const GemmArgs p = gated_gemm(a);
    const GatedCopier<BM, BN, NW> cp(p, a.F, m0, f0, wid, lane);
    f32x16_t acc[MI][2];
    static_for<MI>([&](auto i) {
        static_for<2>([&](auto j) { static_for<16>([&](auto v) { acc[i][j][decltype(v)::value] = 0.0f; }); });
    });
    ring3_main_loop<BM, BN, true, WM, WN, KFULL, false>(acc, smem, lds_addr_of(smem), cp, p, 0, (int)((a.K + 63) / 64), wm, wn, lane);
    vm_wait<0>();  // copies of tiles past the end still write (zeros) into LDS
    __syncthreads();
    gated_finish<BWD, BM, HB, WM, WTM, MI, 64 * NW>(a, acc, smem, m0, f0, tm, wm, wn, true, tid, lane);
}

// Small tiles (64 rows, 32 values of f): grids of up to two to a compute unit,
// bound by the copies' latency.  An LDS ring of four 64-deep K
// tiles; the four waves are two row blocks times two halves of each K tile's
// steps, summed through LDS at the end, so that each wave still holds a pair of
// column blocks.
template <bool BWD>
__global__ __launch_bounds__(256, 2) void gated_ring_kernel(GatedArgs a, TileMapArgs tmap) {
    constexpr int BM = 64, BN = 64, ST = 4, NW = 4, HB = 32;
    using Op = RingOperand<64, true, NW>;
    constexpr int STAGE = 2 * Op::BYTES, PER_TILE = 2 * Op::INSTR;
    __shared__ __attribute__((aligned(1024))) char smem[ST * STAGE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid >> 1, kw = wid & 1;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, f0 = (int64_t)tn * HB;
    const Op ox(a.x, (uint32_t)(((a.M - 1) * a.ld_x + a.K) * 2), a.ld_x, a.M, m0, wid, lane);
    Op ow(a.W, (uint32_t)(((2 * a.F - 1) * a.ld_w + a.K) * 2), a.ld_w, 2 * a.F, 0, wid, lane);
    static_for<Op::INSTR>([&](auto q) {
        const int unit = (wid * Op::INSTR + q) * 64 + lane, r = unit >> 3;
        const int64_t row = gated_row(a.F, f0, r);
        const int k = ((unit & 7) ^ dma_a_swz(r)) * 8;
        ow.kq[q] = row >= 0 ? k : 0x40000000;
        ow.base[q] = row >= 0 ? (uint32_t)((row * a.ld_w + k) * 2) : 0;
    });
    const uint32_t sbase = lds_addr_of(smem);
    const int K = (int)a.K, nk = (K + 63) / 64;
    auto copy = [&](int t) {
        const uint32_t dst = sbase + (uint32_t)((t % ST) * STAGE);
        static_for<Op::INSTR>([&](auto q) { ox.template copy<q>(t * 64, K, dst); });
        static_for<Op::INSTR>([&](auto q) { ow.template copy<q>(t * 64, K, dst + Op::BYTES); });
    };
    f32x16_t acc[1][2];
    static_for<2>([&](auto j) { static_for<16>([&](auto v) { acc[0][j][decltype(v)::value] = 0.0f; }); });
    static_for<ST - 1>([&](auto t) { copy(t); });  // (tiles past the end: zeros, no memory read)
    for (int t = 0; t < nk; ++t) {
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave is done with tile t - 1's stage
        vm_wait<(ST - 2) * PER_TILE>();
        block_sync();  // every wave's share of tile t has landed, and tile t - 1's stage is free
        copy(t + ST - 1);
        const char* const s = smem + (t % ST) * STAGE;
        static_for<2>([&](auto h) {
            const int ks = kw * 2 + h;
            const uint4 fx = Op::frag(s, wm * 32, ks, lane);
            static_for<2>([&](auto j) { mfma32_bf16(acc[0][j], fx, Op::frag(s + Op::BYTES, j * 32, ks, lane)); });
        });
    }
    vm_wait<0>();
    __syncthreads();
    // the second half's sums to the first's waves
    float* const part = reinterpret_cast<float*>(smem) + wm * 32 * 64;
    if (kw == 1) static_for<2>([&](auto j) {
        static_for<16>([&](auto v) { part[(j * 16 + v) * 64 + lane] = acc[0][j][decltype(v)::value]; });
    });
    __syncthreads();
    if (kw == 0) static_for<2>([&](auto j) {
        static_for<16>([&](auto v) { acc[0][j][decltype(v)::value] += part[(j * 16 + v) * 64 + lane]; });
    });
    __syncthreads();
    gated_finish<BWD, BM, HB, 2, 32, 1, 256>(a, acc, smem, m0, f0, tm, wm, 0, kw == 0, tid, lane);
}

}  // namespace isam
