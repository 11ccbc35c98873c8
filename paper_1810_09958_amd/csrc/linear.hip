// A projection with its epilogue, and the gradient before its products:
//
//   P = x W^T + b,  out = act(P) + residual                 dP = dout act'(P)   (then dx = dP W, dW = dP^T x)
//
// bf16: the main loops of the library's large tiles and of the small ring, whose accumulators pass bias,
// activation and residual on their way out: the residual's tile is copied to LDS while nothing else needs
// it, each lane replaces its values there, and whole rows leave.  P never reaches memory; backward it is
// formed again (2 M N K operations, against keeping M N values) and dP leaves rounded to bf16, as the
// operand of the two products after it, so that dx and dW carry two roundings (beyond 16 rows): a norm error of
// 2.35e-3, at any number of rows (terms and errors grow alike), against 1.66e-3 of the output's own.  Two bf16 terms
// would leave that alone at twice the operations of both products: dx 30.5 -> 54.2 and dW 32.3 -> 69.3 us at
// 2048x1024x4096 (M x K x N), 214 -> 438 and 268 -> 512 at 8192x2048x8192; fp32 operands do it for a caller who
// needs it.  (Bytes and latency hide the second term up to some 128 rows, 12 and 12 us either way at 128x1024x4096,
// but a tile's LDS has room for one term.)  The bias' gradient is summed before that rounding.
// Up to 16 rows (64 over little work) the weights are streamed once, straight into the matrix instructions' operand
// registers: 1x1024x4096 (M x K x N) 4.0 us, 2.1 TB/s between start and end of one launch.  bf16 tiles: 8192x8192x2048
// with a residual 212 us, 1.30 PFLOP/s, power, as the large product; 8192x2048x8192 280 us without an activation and 308
// with gelu, whose epilogue (67 M values on the vector units) nothing covers.  Gradient of 2048x1024x4096 with gelu 100 us:
// dP 29, dx 32, dW 26 and the transposed copy of its operand 13.
// fp32 grids of few tiles run on the fp32 matrix instructions, straight from memory; larger ones, and deep bf16 products
// of few tiles, go through the library's product and an element-wise pass.
#include "gated_ffn.hpp"

namespace isam {

namespace {

// p Phi(p) and its derivative Phi(p) + p phi(p).  Both halves need exp(-p^2 / 2) once: Phi(-|p|) = exp(-x^2) erfcx(x) / 2
// with x = |p| / sqrt 2, and erfcx(x) / (2 t) is a polynomial of t = 1 / (1 + 0.4 x) to 1.3e-7 of itself for all
// x >= 0 (a least-squares fit to it weighted towards its largest error, over the zeros of a Chebyshev polynomial).
__device__ __forceinline__ float gelu(float p, float& slope) {
    const float e = __builtin_amdgcn_exp2f(p * p * -0.72134752f), t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(p), 0.28284271f, 1.0f));
    float q = 0.0251324625f;
    q = __builtin_fmaf(q, t, -0.0914563082f);
    q = __builtin_fmaf(q, t, 0.0845517834f);
    q = __builtin_fmaf(q, t, -0.00281151942f);
    q = __builtin_fmaf(q, t, 0.0707194487f);
    q = __builtin_fmaf(q, t, 0.0842699833f);
    q = __builtin_fmaf(q, t, 0.103921491f);
    q = __builtin_fmaf(q, t, 0.11283479f);
    q = __builtin_fmaf(q, t, 0.112837931f);
    q *= t * e;
    const float cdf = p > 0.0f ? 1.0f - q : q;
    slope = __builtin_fmaf(p * 0.39894228f, e, cdf);
    return p * cdf;
}

// act(p) and its derivative.  ACT: 0 sigmoid, 1 silu, 2 gelu (erf form), 3 none.
template <int ACT>
__device__ __forceinline__ float linear_act(float p, float& slope) {
    if constexpr (ACT == 3) {
        slope = 1.0f;
        return p;
    } else if constexpr (ACT == 2) {
        return gelu(p, slope);
    } else {
        return gate_act<ACT>(p, slope);
    }
}
__device__ __forceinline__ float linear_act(int act, float p, float& slope) {
    return act == 0 ? linear_act<0>(p, slope) : act == 1 ? linear_act<1>(p, slope) : act == 2 ? linear_act<2>(p, slope) : linear_act<3>(p, slope);
}

// Zeros after the N gradients of each of a tile's rows, up to the end of the last 16-byte piece (the products that
// follow may multiply what they read there by zero).
template <int ES>
__device__ __forceinline__ void linear_pad(const LinearArgs& a, int64_t m0, int rows, int tid, int threads) {
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, (uint32_t)(a.M * a.ld_out * ES));
    const int pad = (int)(a.ld_out - a.N);
#pragma unroll 1
    for (int r = tid; r < rows; r += threads) {
        const uint32_t at = (uint32_t)(((m0 + r) * a.ld_out + a.N) * ES);
        static_for<7>([&](auto e) {
            if constexpr (ES == 2) __builtin_amdgcn_raw_buffer_store_b16((short)0, ro, (int)(e < pad ? at + 2u * e : kOob), 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b32(0, ro, (int)(e < pad ? at + 4u * e : kOob), 0, 0);
        });
    }
}

// Epilogue of a tile of BM rows and BN columns; `smem` is idle.  The wave holds rows wm WTM .. and columns
// wn 64 .. + 64.  The indexes go through an empty asm, so that what is computed from them is not held in
// registers across the main loop or shared by the instances; no load or store stands in a branch of lanes.
template <int ACT, bool BWD, bool WHOLE, int BM, int BN, int WM, int WTM, int MI, int NT>
__device__ __forceinline__ void linear_epilogue(const LinearArgs& a, f32x16_t (&acc)[MI][2], char* smem, int64_t m0, int64_t n0,
                                                int tm, int wm, int wn, bool active, int tid, int lane) {
    asm volatile("" : "+v"(lane), "+v"(tid));
    constexpr int LD = BN * 2 + 16, PIECES = BN / 8, RPI = NT / PIECES;
    static_assert(NT % PIECES == 0 && BM % RPI == 0, "whole rows per pass");
    const int piece = tid % PIECES, row0 = tid / PIECES, rows = (int)min((int64_t)BM, a.M - m0);
    const int valid = (int)max((int64_t)0, min((int64_t)8, a.N - (n0 + piece * 8)));
    const bool side = BWD || a.side;
    if (side) {  // the residual, or dout, takes the place that the result will have
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.side, gated_bytes(a.M, a.N, a.ld_side));
        const uint32_t at = (uint32_t)((m0 * a.ld_side + n0 + piece * 8) * 2), step = (uint32_t)(a.ld_side * 2);
        constexpr int U = WHOLE && BM / RPI >= 4 ? 4 : 1;
#pragma unroll 1
        for (int r = row0; r < BM; r += U * RPI) {
            uint4 v[U];
            static_for<U>([&](auto i) {
                const int rr = r + i * RPI;
                v[i] = gated_load8<WHOLE>(rs, at + (uint32_t)rr * step, rr < rows ? valid : 0);
            });
            static_for<U>([&](auto i) { *reinterpret_cast<uint4*>(smem + (r + i * RPI) * LD + piece * 16) = v[i]; });
        }
        __syncthreads();
    }
    if (active) {
        const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.bias, a.bias ? (uint32_t)(a.N * 4) : 0u);
        static_for<2>([&](auto j) {
            const int c = wn * 64 + j * 32 + (lane & 31);
            const int64_t n = n0 + c;
            const bool in = n < a.N;
            const float bias = __uint_as_float(buf_load4(rb, in ? (uint32_t)(n * 4) : kOob));
            float sum = 0.0f;
            static_for<MI>([&](auto i) {
                static_for<16>([&](auto v) {
                    const int r = wm * WTM + i * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
                    uint16_t* const at = reinterpret_cast<uint16_t*>(smem + r * LD + c * 2);
                    float slope;
                    const float s = linear_act<ACT>(acc[i][j][decltype(v)::value] + bias, slope);
                    if constexpr (BWD) {
                        const float d = bf16_to_f32(*at) * slope;
                        *at = (uint16_t)pack_bf16_rne(d, 0.0f);
                        sum += r < rows ? d : 0.0f;
                    } else {
                        *at = (uint16_t)pack_bf16_rne(side ? s + bf16_to_f32(*at) : s, 0.0f);
                    }
                    // Four values at a time: the compiler would hold all of them in registers.
                    if constexpr (BWD && (v & 3) == 3) {
                        asm volatile("" : "+v"(sum));
                        __builtin_amdgcn_sched_barrier(0);
                    }
                });
            });
            if (BWD && a.bias_part) {
                // the two lane halves hold the other rows of the same column; one partial row per wave row
                sum += __shfl_xor(sum, 32);
                const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.bias_part + ((int64_t)tm * WM + wm) * a.N, (uint32_t)(a.N * 4));
                __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(sum), ro, (int)(in && lane < 32 ? (uint32_t)(n * 4) : kOob), 0, 0);
            }
        });
    }
    __syncthreads();
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, gated_bytes(a.M, a.N, a.ld_out));
    const uint32_t at = (uint32_t)((m0 * a.ld_out + n0 + piece * 8) * 2), step = (uint32_t)(a.ld_out * 2);
#pragma unroll 2
    for (int r = row0; r < BM; r += RPI)
        gated_store8<WHOLE>(ro, at + (uint32_t)r * step, r < rows ? valid : 0, *reinterpret_cast<const uint4*>(smem + r * LD + piece * 16));
    if constexpr (BWD && !WHOLE) {
        if (n0 + BN >= a.N) linear_pad<2>(a, m0, rows, tid, NT);
    }
}

template <bool BWD, int BM, int BN, int WM, int WTM, int MI, int NT>
__device__ __forceinline__ void linear_finish(const LinearArgs& a, f32x16_t (&acc)[MI][2], char* smem, int64_t m0, int64_t n0, int tm,
                                              int wm, int wn, bool active, int tid, int lane) {
    auto act = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (a.act == 0) linear_epilogue<0, BWD, W, BM, BN, WM, WTM, MI, NT>(a, acc, smem, m0, n0, tm, wm, wn, active, tid, lane);
        else if (a.act == 1) linear_epilogue<1, BWD, W, BM, BN, WM, WTM, MI, NT>(a, acc, smem, m0, n0, tm, wm, wn, active, tid, lane);
        else if (a.act == 2) linear_epilogue<2, BWD, W, BM, BN, WM, WTM, MI, NT>(a, acc, smem, m0, n0, tm, wm, wn, active, tid, lane);
        else if constexpr (!BWD) linear_epilogue<3, BWD, W, BM, BN, WM, WTM, MI, NT>(a, acc, smem, m0, n0, tm, wm, wn, active, tid, lane);
    };
    if (a.whole) act(std::true_type{});
    else act(std::false_type{});
}

__device__ __forceinline__ GemmArgs linear_gemm(const LinearArgs& a) {
    GemmArgs p{};
    p.A = a.x;
    p.B = a.W;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.lda = a.ld_x;
    p.ldb = a.ld_w;
    return p;
}

// Large tiles: the three-stage ring of gemm_dma.hpp.
template <int BM, int BN, int WM, int WN, bool KFULL, bool BWD>
__global__ __launch_bounds__(64 * WM * WN, BM == 128 ? 2 : 1) void linear_dma_kernel(LinearArgs a, TileMapArgs tmap) {
    constexpr int NW = WM * WN, WTM = BM / WM, MI = WTM / 32;
    static_assert(BN / WN == 64, "64 columns to a wave");
    constexpr int LDS = BM * 128 * 2 + BN * 128 * 3;
    static_assert(BM * (BN * 2 + 16) <= LDS, "epilogue staging must fit in LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid / WN, wn = wid % WN;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const GemmArgs p = linear_gemm(a);
    const DmaCopier<BM, BN, true, NW> cp(p, m0, n0, a.K, wid, lane);
    f32x16_t acc[MI][2];
    static_for<MI>([&](auto i) {
        static_for<2>([&](auto j) { static_for<16>([&](auto v) { acc[i][j][decltype(v)::value] = 0.0f; }); });
    });
    ring3_main_loop<BM, BN, true, WM, WN, KFULL, false>(acc, smem, lds_addr_of(smem), cp, p, 0, (int)((a.K + 63) / 64), wm, wn, lane);
    vm_wait<0>();  // copies of tiles past the end still write (zeros) into LDS
    __syncthreads();
    linear_finish<BWD, BM, BN, WM, WTM, MI, 64 * NW>(a, acc, smem, m0, n0, tm, wm, wn, true, tid, lane);
}

// Small tiles (64 x 64): grids of up to two to a compute unit, bound by the copies' latency.  An LDS ring
// of four 64-deep K tiles; the four waves are two row blocks times two halves of each K tile's steps,
// summed through LDS at the end.
template <bool BWD>
__global__ __launch_bounds__(256, 2) void linear_ring_kernel(LinearArgs a, TileMapArgs tmap) {
    constexpr int BM = 64, BN = 64, ST = 4, NW = 4;
    using Op = RingOperand<64, true, NW>;
    constexpr int STAGE = 2 * Op::BYTES, PER_TILE = 2 * Op::INSTR;
    __shared__ __attribute__((aligned(1024))) char smem[ST * STAGE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wid >> 1, kw = wid & 1;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const Op ox(a.x, (uint32_t)(((a.M - 1) * a.ld_x + a.K) * 2), a.ld_x, a.M, m0, wid, lane);
    const Op ow(a.W, (uint32_t)(((a.N - 1) * a.ld_w + a.K) * 2), a.ld_w, a.N, n0, wid, lane);
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
    linear_finish<BWD, BM, BN, 2, 32, 1, 256>(a, acc, smem, m0, n0, tm, wm, 0, kw == 0, tid, lane);
}

// A few rows (MB blocks of 16): 16 rows of W per workgroup, streamed once into the operand registers; its
// eight waves take every eighth K step and their sums meet in LDS.  x (a column per row of it) comes from the
// caches, once for every 16 columns.
// BWD (bf16, one block): dP instead, in two bf16 terms, the high ones in rows 0 .. M - 1 and what they leave in rows
// M .. 2M - 1: over few rows the rounding of an operand is not averaged out, and twice the operations of both
// products cost nothing while W's bytes bound them.
template <int ES, bool BWD, int MB>
__global__ __launch_bounds__(512) void linear_token_kernel(LinearArgs a) {
    using IO = Row16<ES>;
    constexpr int E = IO::E, KS = 4 * E, U = 4;  // values of K of a lane, of a step; steps in flight
    static_assert(!BWD || MB == 1, "the gradient's terms are those of one block");
    __shared__ float sums[8][4 * MB][64];
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, li = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + li;
    const int nk = (int)((a.K + KS - 1) / KS);
    f32x4_t acc[MB];
    static_for<MB>([&](auto m) { acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
    for (int s0 = wid; s0 < nk; s0 += 8 * U) {
        uint4 w[U], x[U][MB];
        static_for<U>([&](auto u) {
            const int64_t k = (int64_t)(s0 + 8 * u) * KS + g * E;
            const int valid = (int)max((int64_t)0, min((int64_t)E, a.K - k));
            w[u] = IO::load(a.W, n * a.ld_w + k, n < a.N ? valid : 0);
            static_for<MB>([&](auto m) { x[u][m] = IO::load(a.x, (16 * m + li) * a.ld_x + k, 16 * m + li < a.M ? valid : 0); });
        });
        static_for<U>([&](auto u) {
            static_for<MB>([&](auto m) {
                if constexpr (ES == 2) mfma16_bf16(acc[m], w[u], x[u][m]);
                else mfma16_f32x4(acc[m], w[u], x[u][m]);
            });
        });
    }
    static_for<MB>([&](auto m) { static_for<4>([&](auto v) { sums[wid][4 * m + v][lane] = acc[m][decltype(v)::value]; }); });
    __syncthreads();
    if (BWD && n0 + 16 >= a.N) {
        LinearArgs both = a;
        both.M = 2 * a.M;
        linear_pad<2>(both, 0, (int)both.M, threadIdx.x, 512);
    }
    // thread (4 m + v, lane): n = n0 + 4 g + v, row 16 m + li
    for (int i = wid; i < 4 * MB; i += 8) {
        const int64_t no = n0 + 4 * g + (i & 3);
        const int row = 16 * (i >> 2) + li;
        const bool on = no < a.N && row < a.M;
        if (!BWD && !on) continue;
        float p = a.bias && no < a.N ? a.bias[no] : 0.0f;
        for (int w = 0; w < 8; ++w) p += sums[w][i][lane];
        float slope;
        const float s = linear_act(a.act, p, slope);
        const float other = on && a.side ? IO::get(a.side, (int64_t)row * a.ld_side + no) : 0.0f;
        if constexpr (!BWD) {
            IO::put(a.out, (int64_t)row * a.ld_out + no, s + other);
        } else {
            float d = on ? other * slope : 0.0f;
            if (on) {
                const int64_t at = (int64_t)row * a.ld_out + no;
                const float high = bf16_to_f32((uint16_t)pack_bf16_rne(d, 0.0f)), low = d - high;
                IO::put(a.out, at, high);
                // (nothing is left of what the high term cannot hold: infinities, NaN)
                IO::put(a.out, at + a.M * a.ld_out, low - low == 0.0f ? low : 0.0f);
            }
            static_for<4>([&](auto k) { d += __shfl_xor(d, 1 << decltype(k)::value); });
            if (a.bias_part && li == 0 && no < a.N) a.bias_part[no] = d;
        }
    }
}

// fp32 grids of few tiles: 32 rows x 64 columns on the fp32 matrix instructions, straight from memory
// (any alignment of 4 bytes) into their operand registers.  The eight waves take every eighth 16-deep K step (32
// matrix instructions on 6 loads, two steps in flight) and meet in LDS, each wave then holding a 16 x 16 block.
// 500x511x771 (M x K x N, 208 tiles) 13.5 us (four waves 15.5; the matrix instructions 4).  A call with two steps in
// flight, and with four: 128x512x2048 10.0, 11.1; 100x333x5001 14.8, 21.1; 256x1024x1024 15.6, 18.5; 1000x768x1000 22.8, 32.3;
// 1000x1000x1000 24.9, 33.1.
template <bool BWD>
__global__ __launch_bounds__(512) void linear_f32_kernel(LinearArgs a, TileMapArgs tmap) {
    constexpr int NW = 8, U = 2;  // waves, steps loaded together
    __shared__ float sums[NW][32][64];
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, g = lane >> 4;
    int tm, tn;
    map_tile(tmap, tm, tn);
    const int64_t m0 = (int64_t)tm * 32, n0 = (int64_t)tn * 64;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, (uint32_t)(((a.M - 1) * a.ld_x + a.K) * 4));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.W, (uint32_t)(((a.N - 1) * a.ld_w + a.K) * 4));
    // two blocks of 16 rows of x, four of W: byte offset of the lane's four values of step 0
    uint32_t at[6];
    static_for<6>([&](auto o) {
        const int64_t r = o < 2 ? m0 + 16 * o + li : n0 + 16 * (o - 2) + li;
        at[o] = r < (o < 2 ? a.M : a.N) ? (uint32_t)((r * (o < 2 ? a.ld_x : a.ld_w) + 4 * g) * 4) : kOob;
    });
    f32x4_t acc[2][4];
    static_for<2>([&](auto i) { static_for<4>([&](auto j) { acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }); });
    const int steps = (int)(a.K / 16);
    auto load = [&](uint4 (&v)[6], int s) {
        static_for<6>([&](auto o) {
            const uint32_t off = s < steps && at[o] != kOob ? at[o] + (uint32_t)s * 64u : kOob;
            v[o] = buf_load16(o < 2 ? rx : rw, off);
        });
    };
    auto multiply = [&](const uint4 (&v)[6]) {
        static_for<2>([&](auto i) { static_for<4>([&](auto j) { mfma16_f32x4(acc[i][j], v[i], v[2 + j]); }); });
    };
    uint4 b[U][6];
    static_for<U>([&](auto u) { load(b[u], wid + NW * u); });
    for (int s = wid; s < steps; s += NW * U) {  // (steps past the end are zeros)
        static_for<U>([&](auto u) {
            multiply(b[u]);
            load(b[u], s + NW * (U + u));
        });
    }
    if (a.K % 16 && wid == (steps & (NW - 1))) {  // the last values of the rows, one by one
        const int k = steps * 16 + 4 * g;
        uint4 tail[6];
        static_for<6>([&](auto o) {
            uint32_t w[4];
            static_for<4>([&](auto e) {
                w[e] = buf_load4(o < 2 ? rx : rw, k + e < a.K && at[o] != kOob ? at[o] + (uint32_t)steps * 64u + 4u * e : kOob);
            });
            tail[o] = make_uint4(w[0], w[1], w[2], w[3]);
        });
        multiply(tail);
    }
    static_for<2>([&](auto i) {
        static_for<4>([&](auto j) {
            static_for<4>([&](auto v) { sums[wid][(i * 4 + j) * 4 + v][lane] = acc[i][j][decltype(v)::value]; });
        });
    });
    __syncthreads();
    // this wave's eighth: row block wid / 4, column block wid % 4; rows 4 g + v, column li
    const int64_t mq = m0 + 16 * (wid >> 2), n = n0 + 16 * (wid & 3) + li;
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.side, a.side ? (uint32_t)(((a.M - 1) * a.ld_side + a.N) * 4) : 0u);
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.out, (uint32_t)(((a.M - 1) * a.ld_out + a.N) * 4));
    const bool in = n < a.N;
    const float bias = a.bias && in ? a.bias[n] : 0.0f;
    float sum = 0.0f;
    static_for<4>([&](auto v) {
        const int64_t m = mq + 4 * g + v;
        const bool on = in && m < a.M;
        float p = bias;
        static_for<NW>([&](auto w) { p += sums[w][wid * 4 + v][lane]; });
        float slope;
        const float s = linear_act(a.act, p, slope);
        const float other = __uint_as_float(buf_load4(rs, on && a.side ? (uint32_t)((m * a.ld_side + n) * 4) : kOob));
        const float out = BWD ? other * slope : s + other;
        __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(out), ro, (int)(on ? (uint32_t)((m * a.ld_out + n) * 4) : kOob), 0, 0);
        sum += on ? out : 0.0f;
    });
    if (BWD && a.bias_part) {  // one partial row for every 16 rows
        static_for<2>([&](auto k) { sum += __shfl_xor(sum, 16 << decltype(k)::value); });
        if (in && g == 0) a.bias_part[(int64_t)(tm * 2 + (wid >> 2)) * a.N + n] = sum;
    }
    if (BWD && n0 + 64 >= a.N) linear_pad<4>(a, m0, (int)min((int64_t)32, a.M - m0), threadIdx.x, 512);
}

// The element-wise pass: out = act(P + b) + residual, or (BWD) dP, from P in memory ([M][ld_pre] fp32, which dP
// replaces where out is P); PRE false: P is not needed, out = dout's column sums alone (no activation).
// A workgroup takes 64 columns and kLinearRows rows, four at a time, and leaves one partial row of the bias' gradient.
template <int ES, bool BWD, bool PRE>
__global__ __launch_bounds__(256) void linear_pass_kernel(LinearArgs a) {
    __shared__ float sums[4][64];
    const int cl = threadIdx.x & 63, rl = threadIdx.x >> 6;
    const int64_t n = (int64_t)blockIdx.x * 64 + cl;
    for (int64_t blk = blockIdx.y; blk * kLinearRows < a.M; blk += gridDim.y) {
        const int64_t m0 = blk * kLinearRows, m1 = min(a.M, m0 + kLinearRows);
        float sum = 0.0f;
        if (n < a.N) {
            const float bias = a.bias ? a.bias[n] : 0.0f;
#pragma unroll 4
            for (int64_t m = m0 + rl; m < m1; m += 4) {
                if constexpr (!PRE) {
                    sum += Row16<ES>::get(a.side, m * a.ld_side + n);
                } else {
                    float slope;
                    const float s = linear_act(a.act, a.pre[m * a.ld_pre + n] + bias, slope);
                    const float other = a.side ? Row16<ES>::get(a.side, m * a.ld_side + n) : 0.0f;
                    const float out = BWD ? other * slope : s + other;
                    Row16<ES>::put(a.out, m * a.ld_out + n, out);
                    sum += out;
                }
            }
        }
        if constexpr (BWD) {
            sums[rl][cl] = sum;
            __syncthreads();
            if (a.bias_part && rl == 0 && n < a.N) a.bias_part[blk * a.N + n] = (sums[0][cl] + sums[1][cl]) + (sums[2][cl] + sums[3][cl]);
            __syncthreads();
        }
    }
}

typedef void (*LinearFn)(LinearArgs, TileMapArgs);

TileMapArgs linear_map(int64_t tiles_m, int64_t tiles_n) {
    TileMapArgs t{};
    t.tiles_m = (int)tiles_m;
    t.tiles_n = (int)tiles_n;
    t.group_m = 8;
    t.xcd_remap = 1;
    return t;
}

template <bool BWD>
LinearFn linear_fn(int tile, bool k_full) {
    switch (tile) {
        case kGated256: return k_full ? linear_dma_kernel<256, 256, 2, 4, true, BWD> : linear_dma_kernel<256, 256, 2, 4, false, BWD>;
        case kGated128: return k_full ? linear_dma_kernel<128, 128, 2, 2, true, BWD> : linear_dma_kernel<128, 128, 2, 2, false, BWD>;
        default: return linear_ring_kernel<BWD>;
    }
}

}  // namespace

hipError_t launch_linear_tiles(const LinearArgs& a, int tile, bool backward, hipStream_t s) {
    const int64_t b = tile == kGated256 ? 256 : tile == kGated128 ? 128 : 64, tm = (a.M + b - 1) / b, tn = (a.N + b - 1) / b;
    if (tm * tn > INT32_MAX || a.K <= 0) return hipErrorInvalidValue;
    const LinearFn fn = backward ? linear_fn<true>(tile, a.K % 64 == 0) : linear_fn<false>(tile, a.K % 64 == 0);
    LinearArgs p = a;
    auto on4 = [](const void* q, int64_t ld) { return (uintptr_t)q % 4 == 0 && ld % 2 == 0; };
    p.whole = a.N % 8 == 0 && on4(a.out, a.ld_out) && (!a.side || on4(a.side, a.ld_side));
    hipLaunchKernelGGL(fn, dim3((unsigned)(tm * tn)), dim3(tile == kGated256 ? 512 : 256), 0, s, p, linear_map(tm, tn));
    return hipGetLastError();
}

hipError_t launch_linear_tokens(const LinearArgs& a, int type, bool backward, hipStream_t s) {
    if (a.M > (backward ? kGatedTokens : kLinearFew) || (a.N + 15) / 16 > INT32_MAX || (backward && type != kBF16)) return hipErrorInvalidValue;
    typedef void (*TokenFn)(LinearArgs);
    TokenFn fn;
    if (backward) fn = linear_token_kernel<2, true, 1>;
    else if (a.M <= 16) fn = type == kBF16 ? linear_token_kernel<2, false, 1> : linear_token_kernel<4, false, 1>;
    else if (a.M <= 32) fn = type == kBF16 ? linear_token_kernel<2, false, 2> : linear_token_kernel<4, false, 2>;
    else fn = type == kBF16 ? linear_token_kernel<2, false, 4> : linear_token_kernel<4, false, 4>;
    hipLaunchKernelGGL(fn, dim3((unsigned)((a.N + 15) / 16)), dim3(512), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_linear_f32(const LinearArgs& a, bool backward, hipStream_t s) {
    const int64_t tm = (a.M + 31) / 32, tn = (a.N + 63) / 64;
    if (tm * tn > INT32_MAX || a.K <= 0) return hipErrorInvalidValue;
    hipLaunchKernelGGL((backward ? linear_f32_kernel<true> : linear_f32_kernel<false>), dim3((unsigned)(tm * tn)), dim3(512), 0, s, a,
                       linear_map(tm, tn));
    return hipGetLastError();
}

hipError_t launch_linear_pass(const LinearArgs& a, int type, bool backward, hipStream_t s) {
    const int64_t gx = (a.N + 63) / 64, gy = (a.M + kLinearRows - 1) / kLinearRows;
    if (gx > INT32_MAX) return hipErrorInvalidValue;
    typedef void (*PassFn)(LinearArgs);
    PassFn fn;
    if (!a.pre) fn = type == kBF16 ? linear_pass_kernel<2, true, false> : linear_pass_kernel<4, true, false>;
    else if (backward) fn = type == kBF16 ? linear_pass_kernel<2, true, true> : linear_pass_kernel<4, true, true>;
    else fn = type == kBF16 ? linear_pass_kernel<2, false, true> : linear_pass_kernel<4, false, true>;
    hipLaunchKernelGGL(fn, dim3((unsigned)gx, (unsigned)(gy < 16384 ? gy : 16384)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace isam
