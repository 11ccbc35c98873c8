// The norm after a block, its gate and scale, the residual sum and the norm
// before the next block, in one pass over the rows, and their gradient in one.
//
//   q = 1 / sqrt(mean(x^2) + eps),  xn = q x,  u = xn w_post   (u = x without w_post)
//   r' = r + s g u
//   p = 1 / sqrt(mean(r'^2) + eps),  y = p r' w_pre
//
//   t = dy w_pre,  dr = dr' + p t - p^3 r' mean(t r'),  dg = sum over the gate's rows of s u dr
//   v = s g dr (w_post),  dx = q v - q^3 x mean(v x)    (dx = s g dr without w_post)
//   dw_pre = sum over rows of dy p r',  dw_post = sum over rows of s g dr xn
//
// Memory bounds both: per value the forward pass moves x, r, r' and y and the
// backward pass x, r', dy, dr', dx and dr, against some ten to thirty fp32
// operations.  A row stays in the registers of its threads between the two
// sums over it; the norm weights stay in registers over a workgroup's rows.  The
// sums over rows are kept in registers too, one partial row per workgroup, added
// in a fixed order by a second kernel (colsum.hip).  Everything is fp32 between
// the loads and the stores: y is normalised from the unrounded r'.  Measured, bf16: forward
// 32768 x 2048 99 us, 5.4 TB/s (a copy runs at 5.1); gradient of 8192 x 4096 with eight
// gate rows 94-97 us, 4.2 TB/s: 86 and a second launch of 9 for the sums over rows; fp32 gradient of
// 1001 x 1537 with a gate to each element 17 us; 32 x 1024 forward 7.7-8.3 us a call, most of it
// the host's.  fp32: 32768 x 2048 forward 201 us (5.3 TB/s), gradient of 8192 x 4096 186 us.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

// Sums of N values over a row's TPR threads (whole waves), the same in every thread.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*lds)[N], int slot0) {
    static_for<N>([&](auto n) {
        static_for<6>([&](auto k) { v[n] += __shfl_xor(v[n], 1 << decltype(k)::value); });
    });
    if constexpr (TPR > 64) {
        const int wid = threadIdx.x >> 6;
        static_for<N>([&](auto n) { lds[wid][n] = v[n]; });  // (every lane the same value: no branch of lanes)
        __syncthreads();
        static_for<N>([&](auto n) { v[n] = 0.0f; });
        static_for<TPR / 64>([&](auto w) {
            static_for<N>([&](auto n) { v[n] += lds[slot0 + w][n]; });
        });
    }
}

// Thread j of its row, row group ng of the workgroup, the group's first wave; the
// groups are whole waves, so ng is uniform over a wave.
template <int TPR, int BLOCK>
struct RowPart {
    static constexpr int NR = BLOCK / TPR, WAVES = BLOCK / 64;
    int j, ng, slot0;
    __device__ __forceinline__ RowPart() {
        const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        j = threadIdx.x % TPR;
        ng = wid / (TPR / 64);
        slot0 = ng * (TPR / 64);
    }
};

template <int ES, bool VEC, int TPR, int V, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_kernel(NormArgs a) {
    using P = RowPart<TPR, BLOCK>;
    constexpr int E = 16 / ES;
    using B = RowBuf<ES, VEC, TPR, E>;
    const P part;
    const int j = part.j;
    __shared__ float lds[2][P::WAVES][1];
    float wa[V][E], wb[V][E];
    using W = RowBuf<4, VEC, TPR, 4>;
    const __amdgpu_buffer_rsrc_t ra = W::row(a.w_post, 0, a.D, true), rb = W::row(a.w_pre, 0, a.D, true);
    static_for<V>([&](auto i) {
        B::load32(ra, i, j, wa[i]);
        B::load32(rb, i, j, wb[i]);
    });
    const float inv = 1.0f / (float)a.D;
    const int64_t step = (int64_t)gridDim.x * P::NR;
    for (int64_t base = (int64_t)blockIdx.x * P::NR; base < a.rows; base += step) {
        const int64_t row = base + part.ng;
        const bool live = row < a.rows;
        const __amdgpu_buffer_rsrc_t rx = B::row(a.x, row * a.ld_x, a.D, live), rr = B::row(a.r, row * a.ld_r, a.D, live),
                                     rg = B::row(a.gate, row / a.rows_per_gate * a.D, a.D, live);
        typename B::Piece px[V], pr[V], pg[V];
        static_for<V>([&](auto i) {
            pr[i] = B::load(rr, i, j);
            px[i] = B::load(rx, i, j);
            pg[i] = B::load(rg, i, j);
        });
        float r[V][E];
        static_for<V>([&](auto i) { B::unpack(pr[i], r[i]); });
        if (a.x) {
            float q = 1.0f;
            if (a.w_post) {
                float sum[1] = {0.0f};
                static_for<V>([&](auto i) {
                    float x[E];
                    B::unpack(px[i], x);
                    static_for<E>([&](auto e) { sum[0] += x[e] * x[e]; });
                });
                row_sum<TPR, 1>(sum, lds[0], part.slot0);
                q = 1.0f / sqrtf(sum[0] * inv + a.eps);
            }
            const __amdgpu_buffer_rsrc_t ro = B::row(a.r_out, row * a.ld_ro, a.D, live);
            static_for<V>([&](auto i) {
                float x[E], g[E];
                B::unpack(px[i], x);
                B::unpack(pg[i], g);
                static_for<E>([&](auto e) {
                    const float u = a.w_post ? x[e] * q * wa[i][e] : x[e];
                    r[i][e] += (a.gate ? a.scale * g[e] : a.scale) * u;
                });
                B::store(ro, i, j, r[i]);
            });
        }
        float sum[1] = {0.0f};
        static_for<V>([&](auto i) {
            static_for<E>([&](auto e) { sum[0] += r[i][e] * r[i][e]; });
        });
        row_sum<TPR, 1>(sum, lds[1], part.slot0);
        const float p = 1.0f / sqrtf(sum[0] * inv + a.eps);
        const __amdgpu_buffer_rsrc_t ry = B::row(a.y, row * a.ld_y, a.D, live);
        static_for<V>([&](auto i) {
            static_for<E>([&](auto e) { r[i][e] *= p * wb[i][e]; });
            B::store(ry, i, j, r[i]);
        });
        // The first sum of the next row writes lds[0], last read before this
        // row's second barrier; the second one lds[1], read before the next
        // row's first barrier -- if there is one.
        if (TPR > 64 && !(a.x && a.w_post)) __syncthreads();
    }
}

// Rows of the backward pass.  With few rows to a gate row (a.parts == 0) each row
// group takes whole gate rows and writes their gradient itself; otherwise a.parts
// workgroups share a gate row (one: writes the gradient; more: leave partial sums).
// HOLD: the weights stay in registers and the next row is requested before this
// row's arithmetic; the longest rows have no registers for that.
template <int ES, bool VEC, int TPR, int E, int V, int BLOCK, int MINW, bool HOLD>
__global__ __launch_bounds__(BLOCK, MINW) void norm_bwd_kernel(NormArgs a) {
    using P = RowPart<TPR, BLOCK>;
    constexpr int NR = P::NR, VH = HOLD ? V : 1;
    using B = RowBuf<ES, VEC, TPR, E>;
    using B4 = RowBuf<4, VEC, TPR, 4>;
    const P part;
    const int j = part.j;
    __shared__ float lds[2][P::WAVES][3];
    extern __shared__ float fold[];  // [TPR * V * E]
    float ha[VH][E], hb[VH][E], sa[V][E], sb[V][E], sg[V][E];
    const __amdgpu_buffer_rsrc_t ra = B4::row(a.w_post, 0, a.D, true), rb = B4::row(a.w_pre, 0, a.D, true);
    static_for<V>([&](auto i) {
        if constexpr (HOLD) {
            B::load32(ra, i, j, ha[i]);
            B::load32(rb, i, j, hb[i]);
        }
        static_for<E>([&](auto e) { sa[i][e] = 0.0f; sb[i][e] = 0.0f; sg[i][e] = 0.0f; });
    });
    // Weights of piece i.
    auto post = [&](auto i, float (&w)[E]) {
        if constexpr (HOLD) static_for<E>([&](auto e) { w[e] = ha[i][e]; });
        else B::load32(ra, i, j, w);
    };
    auto pre = [&](auto i, float (&w)[E]) {
        if constexpr (HOLD) static_for<E>([&](auto e) { w[e] = hb[i][e]; });
        else B::load32(rb, i, j, w);
    };
    const float inv = 1.0f / (float)a.D;
    const int64_t rpg = a.rows_per_gate, groups = a.gates;
    const int64_t workers = (int64_t)gridDim.x * NR, me = (int64_t)blockIdx.x * NR + part.ng;
    // Row k of gate row grp, `iters` of them in turn.
    int64_t iters, grp, k = 0, share = 0;
    if (a.parts == 0) {
        iters = (groups + workers - 1) / workers * rpg;
        grp = me;
    } else {
        grp = (int64_t)blockIdx.x / a.parts;
        share = (int64_t)a.parts * NR;
        k = ((int64_t)blockIdx.x - grp * a.parts) * NR + part.ng;
        iters = (rpg + share - 1) / share;
    }
    typename B::Piece px[V], pr[V], pg[V], py[V], pd[V];
    auto fetch = [&](int64_t row, int64_t gate, bool live) {
        const __amdgpu_buffer_rsrc_t rx = B::row(a.x, row * a.ld_x, a.D, live), rr = B::row(a.r, row * a.ld_r, a.D, live),
                                     ry = B::row(a.dy, row * a.ld_dy, a.D, live),
                                     rd = B::row(a.dr_out, row * a.ld_dro, a.D, live), rg = B::row(a.gate, gate * a.D, a.D, live);
        static_for<V>([&](auto i) {
            px[i] = B::load(rx, i, j);
            pr[i] = B::load(rr, i, j);
            py[i] = B::load(ry, i, j);
            pd[i] = B::load(rd, i, j);
            pg[i] = B::load(rg, i, j);
        });
    };
    auto is_live = [&] { return grp < groups && k < rpg; };
    if constexpr (HOLD) fetch(grp * rpg + k, grp, is_live());
    for (int64_t it = 0; it < iters; ++it) {
        const int64_t row = grp * rpg + k, cur = grp;
        const bool live = is_live();
        if constexpr (!HOLD) fetch(row, cur, live);
        bool last = false;
        if (a.parts == 0) {
            if (++k == rpg) {
                k = 0;
                grp += workers;
                last = true;
            }
        } else {
            k += share;
        }
        // (a row that does not exist is all zeros, and so is what it adds)
        float x[V][E], r[V][E], dr[V][E], dy[V][E], sum[3] = {0.0f, 0.0f, 0.0f};
        typename B::Piece gr[V];
        static_for<V>([&](auto i) {
            float w[E];
            pre(i, w);
            B::unpack(px[i], x[i]);
            B::unpack(pr[i], r[i]);
            B::unpack(py[i], dy[i]);
            B::unpack(pd[i], dr[i]);
            gr[i] = pg[i];
            static_for<E>([&](auto e) {
                sum[0] += x[i][e] * x[i][e];
                sum[1] += r[i][e] * r[i][e];
                sum[2] += dy[i][e] * w[e] * r[i][e];
            });
        });
        if constexpr (HOLD) fetch(grp * rpg + k, grp, it + 1 < iters && is_live());
        row_sum<TPR, 3>(sum, lds[0], part.slot0);
        const float q = a.w_post && live ? 1.0f / sqrtf(sum[0] * inv + a.eps) : 1.0f;
        const float p = live ? 1.0f / sqrtf(sum[1] * inv + a.eps) : 0.0f, c = sum[2] * inv * p * p * p;
        const __amdgpu_buffer_rsrc_t wr = B::row(a.dr, row * a.ld_dr, a.D, live);
        static_for<V>([&](auto i) {
            float w[E];
            pre(i, w);
            static_for<E>([&](auto e) {
                dr[i][e] += p * dy[i][e] * w[e] - c * r[i][e];
                sb[i][e] += dy[i][e] * p * r[i][e];
            });
            B::store(wr, i, j, dr[i]);
        });
        if (a.x) {
            float dot[1] = {0.0f};
            static_for<V>([&](auto i) {
                float w[E], g[E];
                post(i, w);
                B::unpack(gr[i], g);
                static_for<E>([&](auto e) {
                    const float u = a.w_post ? x[i][e] * q * w[e] : x[i][e];
                    const float du = (a.gate ? a.scale * g[e] : a.scale) * dr[i][e];
                    sg[i][e] += a.scale * u * dr[i][e];
                    sa[i][e] += du * x[i][e] * q;
                    dr[i][e] = a.w_post ? du * w[e] : du;
                    dot[0] += dr[i][e] * x[i][e];
                });
            });
            float m = 0.0f;
            if (a.w_post) {
                row_sum<TPR, 1>(dot, reinterpret_cast<float(*)[1]>(&lds[1][0][0]), part.slot0);
                m = dot[0] * inv * q * q * q;
            }
            const __amdgpu_buffer_rsrc_t wx = B::row(a.dx, row * a.ld_dx, a.D, live);
            static_for<V>([&](auto i) {
                if (a.w_post) static_for<E>([&](auto e) { dr[i][e] = q * dr[i][e] - m * x[i][e]; });
                B::store(wx, i, j, dr[i]);
            });
            if (last) {
                const __amdgpu_buffer_rsrc_t wg = B::row(a.dgate, cur * a.D, a.D, live);
                static_for<V>([&](auto i) {
                    B::store(wg, i, j, sg[i]);
                    static_for<E>([&](auto e) { sg[i][e] = 0.0f; });
                });
            }
        }
        // as in the forward pass
        if (TPR > 64 && !(a.x && a.w_post)) __syncthreads();
    }
    // The workgroup's sums: row groups one after the other through LDS, to the first.
    auto total = [&](float (&s)[V][E]) {
        static_for<NR - 1>([&](auto n) {
            __syncthreads();
            if (part.ng == n + 1) static_for<V>([&](auto i) {
                static_for<E>([&](auto e) { fold[(i * E + e) * TPR + j] = s[i][e]; });
            });
            __syncthreads();
            if (part.ng == 0) static_for<V>([&](auto i) {
                static_for<E>([&](auto e) { s[i][e] += fold[(i * E + e) * TPR + j]; });
            });
        });
    };
    auto leave = [&](float (&s)[V][E], float* out) {
        total(s);
        const __amdgpu_buffer_rsrc_t w = B4::row(out, (int64_t)blockIdx.x * a.D, a.D, part.ng == 0);
        static_for<V>([&](auto i) { B::store32(w, i, j, s[i]); });
    };
    const int64_t n = (int64_t)gridDim.x * a.D;
    if (a.dw_pre) leave(sb, a.partial);
    if (a.dw_post) leave(sa, a.partial + n);
    if (a.dgate && a.parts > 1) leave(sg, a.partial + 2 * n);
    if (a.dgate && a.parts == 1) {
        total(sg);
        const __amdgpu_buffer_rsrc_t w = B::row(a.dgate, (int64_t)blockIdx.x * a.D, a.D, part.ng == 0);
        static_for<V>([&](auto i) { B::store(w, i, j, sg[i]); });
    }
}

typedef void (*NormFn)(NormArgs);
struct Config {
    NormFn fn;
    int tpr, block, values;  // threads of a row, of a workgroup; values of a thread
    int per_cu;              // workgroups of a compute unit
};

// Forward: a wave holds a row of up to 2048 (bf16) values; longer rows take a
// workgroup.
template <int ES, bool VEC>
Config fwd_config(int64_t D) {
    constexpr int E = 16 / ES;
    const int64_t pieces = (D + E - 1) / E;
    if (pieces <= 64) return {norm_fwd_kernel<ES, VEC, 64, 1, 256>, 64, 256, E, 8};
    if (pieces <= 128) return {norm_fwd_kernel<ES, VEC, 64, 2, 256>, 64, 256, 2 * E, 8};
    if (pieces <= 256) return {norm_fwd_kernel<ES, VEC, 64, 4, 256>, 64, 256, 4 * E, 8};
    if (pieces <= 512) return {norm_fwd_kernel<ES, VEC, 256, 2, 256>, 256, 256, 2 * E, 8};
    if (pieces <= 1024) return {norm_fwd_kernel<ES, VEC, 256, 4, 256>, 256, 256, 4 * E, 8};
    if (pieces <= 2048) return {norm_fwd_kernel<ES, VEC, 1024, 2, 1024>, 1024, 1024, 2 * E, 2};
    return {norm_fwd_kernel<ES, VEC, 1024, 4, 1024>, 1024, 1024, 4 * E, 2};
}

// Backward: the sums, weights and values of a row take some 14 registers a value.
// bf16 rows in whole pieces of eight: sixteen values to a thread, so that a wave holds
// a row of 1024 and the sums over longer rows meet fewer waves; two waves to a
// SIMD.  fp32, and rows moved value by value: four values and four waves.  The
// longest rows: no registers for the weights and the next row.
template <int ES, bool VEC>
Config bwd_config(int64_t D) {
    if constexpr (ES == 2 && VEC) {
        if (D <= 512) return {norm_bwd_kernel<ES, VEC, 64, 8, 1, 256, 4, true>, 64, 256, 8, 4};
        if (D <= 1024) return {norm_bwd_kernel<ES, VEC, 64, 8, 2, 256, 2, true>, 64, 256, 16, 2};
        if (D <= 2048) return {norm_bwd_kernel<ES, VEC, 128, 8, 2, 256, 2, true>, 128, 256, 16, 2};
        if (D <= 4096) return {norm_bwd_kernel<ES, VEC, 256, 8, 2, 256, 2, true>, 256, 256, 16, 2};
        if (D <= 8192) return {norm_bwd_kernel<ES, VEC, 512, 8, 2, 512, 2, true>, 512, 512, 16, 1};
        return {norm_bwd_kernel<ES, VEC, 1024, 8, 2, 1024, 4, false>, 1024, 1024, 16, 1};
    } else {
        if (D <= 256) return {norm_bwd_kernel<ES, VEC, 64, 4, 1, 256, 4, true>, 64, 256, 4, 4};
        if (D <= 512) return {norm_bwd_kernel<ES, VEC, 128, 4, 1, 256, 4, true>, 128, 256, 4, 4};
        if (D <= 1024) return {norm_bwd_kernel<ES, VEC, 256, 4, 1, 256, 4, true>, 256, 256, 4, 4};
        if (D <= 2048) return {norm_bwd_kernel<ES, VEC, 512, 4, 1, 512, 4, true>, 512, 512, 4, 2};
        if (D <= 4096) return {norm_bwd_kernel<ES, VEC, 1024, 4, 1, 1024, 4, true>, 1024, 1024, 4, 1};
        if (D <= 8192) return {norm_bwd_kernel<ES, VEC, 1024, 4, 2, 1024, 4, false>, 1024, 1024, 8, 1};
        return {norm_bwd_kernel<ES, VEC, 1024, 4, 4, 1024, 4, false>, 1024, 1024, 16, 1};
    }
}

// Whole pieces in every row, on 4 bytes.
bool pieces(const NormArgs& a) {
    const int64_t E = a.type == kF32 ? 4 : 8, es = a.type == kF32 ? 4 : 2;
    auto ok = [&](const void* p, int64_t ld) { return !p || (ld * es % 4 == 0 && (uintptr_t)p % 4 == 0); };
    return a.D % E == 0 && ok(a.x, a.ld_x) && ok(a.r, a.ld_r) && ok(a.gate, a.D) && ok(a.r_out, a.ld_ro) && ok(a.y, a.ld_y) &&
           ok(a.dy, a.ld_dy) && ok(a.dr_out, a.ld_dro) && ok(a.dx, a.ld_dx) && ok(a.dr, a.ld_dr) && ok(a.dgate, a.D);
}

Config config(const NormArgs& a, bool backward) {
    if (a.type == kBF16) {
        if (pieces(a)) return backward ? bwd_config<2, true>(a.D) : fwd_config<2, true>(a.D);
        return backward ? bwd_config<2, false>(a.D) : fwd_config<2, false>(a.D);
    }
    if (pieces(a)) return backward ? bwd_config<4, true>(a.D) : fwd_config<4, true>(a.D);
    return backward ? bwd_config<4, false>(a.D) : fwd_config<4, false>(a.D);
}

}  // namespace

// Workgroups of the backward pass: those the device holds at once, as far as the
// rows go.  Gate rows of fewer than eight rows are owned by row
// groups (a workgroup to each would leave more partial sums than it reads).
void norm_bwd_grid(const NormArgs& a, int cus, int64_t* grid, int* parts) {
    const Config c = config(a, true);
    const int64_t nr = c.block / c.tpr, most = (int64_t)c.per_cu * cus, gates = a.gates, rpg = a.rows / gates;
    if (rpg < 8 && gates > 1) {
        const int64_t need = (gates + nr - 1) / nr;
        *parts = 0;
        *grid = need < most ? need : most;
        return;
    }
    const int64_t fill = (rpg + nr - 1) / nr;
    int64_t p = most / gates;
    if (p > fill) p = fill;
    if (p < 1) p = 1;
    *parts = (int)p;
    *grid = p * gates;
}

int64_t norm_bwd_most(const NormArgs& a, int cus) {
    NormArgs b = a;
    int64_t grid, most;
    int parts;
    norm_bwd_grid(b, cus, &most, &parts);
    b.r = reinterpret_cast<const void*>(2);  // (an address off 4 bytes)
    norm_bwd_grid(b, cus, &grid, &parts);
    return grid > most ? grid : most;
}

hipError_t launch_norm_forward(const NormArgs& a, int cus, hipStream_t s) {
    const Config c = config(a, false);
    const int64_t nr = c.block / c.tpr, need = (a.rows + nr - 1) / nr, most = (int64_t)cus * c.per_cu;
    hipLaunchKernelGGL(c.fn, dim3((unsigned)(need < most ? need : most)), dim3(c.block), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs& a, int64_t grid, hipStream_t s) {
    const Config c = config(a, true);
    hipError_t e = hipSuccess;
    if (grid > 0) {
        const size_t lds = (size_t)c.tpr * c.values * sizeof(float);
        if ((e = ensure_dynamic_lds(reinterpret_cast<const void*>(c.fn), lds)) != hipSuccess) return e;
        hipLaunchKernelGGL(c.fn, dim3((unsigned)grid), dim3(c.block), lds, s, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.rows == 0 && a.dgate) {
        ColSum z[1] = {{a.partial, a.dgate, 0, a.gates * a.D, 1, a.type}};
        if ((e = launch_colsum(z, 1, s)) != hipSuccess) return e;
    }
    const int64_t n = grid * a.D;
    ColSum sums[3];
    int count = 0;
    if (a.dw_pre) sums[count++] = ColSum{a.partial, a.dw_pre, grid, a.D, 1, kF32};
    if (a.dw_post) sums[count++] = ColSum{a.partial + n, a.dw_post, grid, a.D, 1, kF32};
    if (a.dgate && a.parts > 1) sums[count++] = ColSum{a.partial + 2 * n, a.dgate, a.parts, a.D, a.gates, a.type};
    return launch_colsum(sums, count, s);
}

}  // namespace isam
