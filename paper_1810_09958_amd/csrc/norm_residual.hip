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
// the loads and the stores: y is normalised from the unrounded r'.
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
        if ((threadIdx.x & 63) == 0) static_for<N>([&](auto n) { lds[wid][n] = v[n]; });
        __syncthreads();
        static_for<N>([&](auto n) { v[n] = 0.0f; });
        static_for<TPR / 64>([&](auto w) {
            static_for<N>([&](auto n) { v[n] += lds[slot0 + w][n]; });
        });
    }
}

template <int ES, int TPR, int V, int BLOCK>
struct RowPart {
    static constexpr int E = Row16<ES>::E, NR = BLOCK / TPR, WAVES = BLOCK / 64;
    int j, ng, slot0;  // thread in its row, row group in the workgroup, the group's first wave
    __device__ __forceinline__ RowPart() : j(threadIdx.x % TPR), ng(threadIdx.x / TPR), slot0(threadIdx.x / TPR * (TPR / 64)) {}
    __device__ __forceinline__ int64_t at(int i) const { return ((int64_t)i * TPR + j) * E; }
    __device__ __forceinline__ int valid(const NormArgs& a, int i) const {
        return (int)max((int64_t)0, min((int64_t)E, a.D - at(i)));
    }
};

template <int ES, int TPR, int V, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_kernel(NormArgs a) {
    using P = RowPart<ES, TPR, V, BLOCK>;
    using IO = Row16<ES>;
    constexpr int E = P::E;
    const P part;
    __shared__ float lds[2][P::WAVES][1];
    float wa[V][E], wb[V][E];
    static_for<V>([&](auto i) {
        load_f32<E>(a.w_post, part.at(i), part.valid(a, i), wa[i]);
        load_f32<E>(a.w_pre, part.at(i), part.valid(a, i), wb[i]);
    });
    const float inv = 1.0f / (float)a.D;
    const int64_t step = (int64_t)gridDim.x * P::NR;
    for (int64_t base = (int64_t)blockIdx.x * P::NR; base < a.rows; base += step) {
        const int64_t row = base + part.ng;
        const bool live = row < a.rows;
        uint4 px[V], pr[V], pg[V];
        static_for<V>([&](auto i) {
            const int valid = live ? part.valid(a, i) : 0;
            pr[i] = IO::load(a.r, row * a.ld_r + part.at(i), valid);
            px[i] = IO::load(a.x, row * a.ld_x + part.at(i), a.x ? valid : 0);
            pg[i] = IO::load(a.gate, row / a.rows_per_gate * a.D + part.at(i), a.gate ? valid : 0);
        });
        float r[V][E];
        if (a.x) {
            float q = 1.0f;
            if (a.w_post) {
                float sum[1] = {0.0f};
                static_for<V>([&](auto i) {
                    float x[E];
                    IO::unpack(px[i], x);
                    static_for<E>([&](auto e) { sum[0] += x[e] * x[e]; });
                });
                row_sum<TPR, 1>(sum, lds[0], part.slot0);
                q = 1.0f / sqrtf(sum[0] * inv + a.eps);
            }
            static_for<V>([&](auto i) {
                float x[E], g[E];
                IO::unpack(px[i], x);
                IO::unpack(pg[i], g);
                IO::unpack(pr[i], r[i]);
                static_for<E>([&](auto e) {
                    const float u = a.w_post ? x[e] * q * wa[i][e] : x[e];
                    r[i][e] += (a.gate ? a.scale * g[e] : a.scale) * u;
                });
                IO::store(a.r_out, row * a.ld_ro + part.at(i), IO::pack(r[i]), live ? part.valid(a, i) : 0);
            });
        } else {
            static_for<V>([&](auto i) { IO::unpack(pr[i], r[i]); });
        }
        float sum[1] = {0.0f};
        static_for<V>([&](auto i) {
            static_for<E>([&](auto e) { sum[0] += r[i][e] * r[i][e]; });
        });
        row_sum<TPR, 1>(sum, lds[1], part.slot0);
        const float p = 1.0f / sqrtf(sum[0] * inv + a.eps);
        static_for<V>([&](auto i) {
            static_for<E>([&](auto e) { r[i][e] *= p * wb[i][e]; });
            IO::store(a.y, row * a.ld_y + part.at(i), IO::pack(r[i]), live ? part.valid(a, i) : 0);
        });
        // The first sum of the next row writes lds[0], last read before this
        // row's second barrier; the second one lds[1], read before the next
        // row's first barrier -- if there is one.
        if (TPR > 64 && !(a.x && a.w_post)) __syncthreads();
    }
}

// Rows of the backward pass.  With at least as many gate rows as row groups
// (a.parts == 0) each row group takes whole gate rows and writes their
// gradient itself; otherwise a.parts workgroups share a gate row and leave
// partial sums.
template <int ES, int TPR, int V, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_kernel(NormArgs a) {
    using P = RowPart<ES, TPR, V, BLOCK>;
    using IO = Row16<ES>;
    constexpr int E = P::E, NR = P::NR;
    const P part;
    __shared__ float lds[2][P::WAVES][3];
    extern __shared__ float fold[];  // [TPR * V * E]
    float wa[V][E], wb[V][E], sa[V][E], sb[V][E], sg[V][E];
    static_for<V>([&](auto i) {
        load_f32<E>(a.w_post, part.at(i), part.valid(a, i), wa[i]);
        load_f32<E>(a.w_pre, part.at(i), part.valid(a, i), wb[i]);
        static_for<E>([&](auto e) { sa[i][e] = 0.0f; sb[i][e] = 0.0f; sg[i][e] = 0.0f; });
    });
    const float inv = 1.0f / (float)a.D;
    const int64_t rpg = a.rows_per_gate, groups = a.gates;
    const int64_t workers = (int64_t)gridDim.x * NR, me = (int64_t)blockIdx.x * NR + part.ng;
    // The row of iteration i and whether it exists.
    int64_t iters, grp, k = 0;
    int64_t share = 0;
    if (a.parts == 0) {
        iters = (groups + workers - 1) / workers * rpg;
        grp = me;
    } else {
        grp = (int64_t)blockIdx.x / a.parts;
        share = (int64_t)a.parts * NR;
        k = ((int64_t)blockIdx.x - grp * a.parts) * NR + part.ng;
        iters = (rpg + share - 1) / share;
    }
    uint4 px[V], pr[V], pg[V], py[V], pd[V];
    auto fetch = [&](int64_t row, bool live) {
        static_for<V>([&](auto i) {
            const int valid = live ? part.valid(a, i) : 0;
            const int64_t at = part.at(i);
            px[i] = IO::load(a.x, row * a.ld_x + at, a.x ? valid : 0);
            pr[i] = IO::load(a.r, row * a.ld_r + at, valid);
            py[i] = IO::load(a.dy, row * a.ld_dy + at, valid);
            pd[i] = IO::load(a.dr_out, row * a.ld_dro + at, a.dr_out ? valid : 0);
            pg[i] = IO::load(a.gate, row / rpg * a.D + at, a.gate ? valid : 0);
        });
    };
    auto is_live = [&] { return grp < groups && k < rpg; };
    fetch(grp * rpg + k, is_live());
    for (int64_t it = 0; it < iters; ++it) {
        const int64_t row = grp * rpg + k, cur = grp;
        const bool live = is_live();
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
        float x[V][E], r[V][E], dr[V][E], g[V][E], sum[3] = {0.0f, 0.0f, 0.0f};
        static_for<V>([&](auto i) {
            float dy[E];
            IO::unpack(px[i], x[i]);
            IO::unpack(pr[i], r[i]);
            IO::unpack(py[i], dy);
            IO::unpack(pd[i], dr[i]);
            IO::unpack(pg[i], g[i]);
            static_for<E>([&](auto e) {
                g[i][e] = a.gate ? a.scale * g[i][e] : a.scale;
                sum[0] += x[i][e] * x[i][e];
                sum[1] += r[i][e] * r[i][e];
                sum[2] += dy[e] * wb[i][e] * r[i][e];
            });
        });
        row_sum<TPR, 3>(sum, lds[0], part.slot0);
        const float q = a.w_post ? 1.0f / sqrtf(sum[0] * inv + a.eps) : 1.0f;
        const float p = 1.0f / sqrtf(sum[1] * inv + a.eps), c = sum[2] * inv * p * p * p;
        float dot[3] = {0.0f, 0.0f, 0.0f};
        static_for<V>([&](auto i) {
            float dy[E];
            IO::unpack(py[i], dy);
            static_for<E>([&](auto e) {
                dr[i][e] += p * dy[e] * wb[i][e] - c * r[i][e];
                if (live) sb[i][e] += dy[e] * p * r[i][e];
            });
            IO::store(a.dr, row * a.ld_dr + part.at(i), IO::pack(dr[i]), live ? part.valid(a, i) : 0);
        });
        // the next row's values arrive under the rest of this one's arithmetic
        fetch(grp * rpg + k, it + 1 < iters && is_live());
        if (a.x) {
            static_for<V>([&](auto i) {
                static_for<E>([&](auto e) {
                    const float u = a.w_post ? x[i][e] * q * wa[i][e] : x[i][e], du = g[i][e] * dr[i][e];
                    if (live) {
                        sg[i][e] += a.scale * u * dr[i][e];
                        sa[i][e] += du * x[i][e] * q;
                    }
                    dr[i][e] = a.w_post ? du * wa[i][e] : du;
                    dot[0] += dr[i][e] * x[i][e];
                });
            });
            float m = 0.0f;
            if (a.w_post) {
                float d1[1] = {dot[0]};
                row_sum<TPR, 1>(d1, reinterpret_cast<float(*)[1]>(&lds[1][0][0]), part.slot0);
                m = d1[0] * inv * q * q * q;
            }
            static_for<V>([&](auto i) {
                if (a.w_post) static_for<E>([&](auto e) { dr[i][e] = q * dr[i][e] - m * x[i][e]; });
                IO::store(a.dx, row * a.ld_dx + part.at(i), IO::pack(dr[i]), live ? part.valid(a, i) : 0);
                if (last) {
                    if (a.dgate) IO::store(a.dgate, cur * a.D + part.at(i), IO::pack(sg[i]), live ? part.valid(a, i) : 0);
                    static_for<E>([&](auto e) { sg[i][e] = 0.0f; });
                }
            });
        }
        // as in the forward pass
        if (TPR > 64 && !(a.x && a.w_post)) __syncthreads();
    }
    // The workgroup's sums: row groups one after the other through LDS.
    auto total = [&](float (&s)[V][E], float* out) {
        static_for<NR - 1>([&](auto n) {
            __syncthreads();
            if (part.ng == n + 1) static_for<V>([&](auto i) {
                static_for<E>([&](auto e) { fold[(i * E + e) * TPR + part.j] = s[i][e]; });
            });
            __syncthreads();
            if (part.ng == 0) static_for<V>([&](auto i) {
                static_for<E>([&](auto e) { s[i][e] += fold[(i * E + e) * TPR + part.j]; });
            });
        });
        if (part.ng == 0) static_for<V>([&](auto i) {
            store_f32<E>(out, (int64_t)blockIdx.x * a.D + part.at(i), part.valid(a, i), s[i]);
        });
    };
    const int64_t n = (int64_t)gridDim.x * a.D;
    if (a.dw_pre) total(sb, a.partial);
    if (a.dw_post) total(sa, a.partial + n);
    if (a.dgate && a.parts) total(sg, a.partial + 2 * n);
}

typedef void (*NormFn)(NormArgs);
struct Config {
    NormFn fn;
    int tpr, block, values;  // threads of a row, of a workgroup; values of a thread
};

// Forward: a wave holds a row of up to 2048 (bf16) values; longer rows take a
// workgroup.
template <int ES>
Config fwd_config(int64_t D) {
    constexpr int E = 16 / ES;
    const int64_t pieces = (D + E - 1) / E;
    if (pieces <= 64) return {norm_fwd_kernel<ES, 64, 1, 256>, 64, 256, E};
    if (pieces <= 128) return {norm_fwd_kernel<ES, 64, 2, 256>, 64, 256, 2 * E};
    if (pieces <= 256) return {norm_fwd_kernel<ES, 64, 4, 256>, 64, 256, 4 * E};
    if (pieces <= 512) return {norm_fwd_kernel<ES, 256, 2, 256>, 256, 256, 2 * E};
    if (pieces <= 1024) return {norm_fwd_kernel<ES, 256, 4, 256>, 256, 256, 4 * E};
    if (pieces <= 2048) return {norm_fwd_kernel<ES, 1024, 2, 1024>, 1024, 1024, 2 * E};
    return {norm_fwd_kernel<ES, 1024, 4, 1024>, 1024, 1024, 4 * E};
}

// Backward: eight values per thread (the sums and weights take six registers a
// value), sixteen for the longest rows.
template <int ES>
Config bwd_config(int64_t D) {
    constexpr int V = ES == 2 ? 1 : 2;
    if (D <= 512) return {norm_bwd_kernel<ES, 64, V, 512>, 64, 512, 8};
    if (D <= 1024) return {norm_bwd_kernel<ES, 128, V, 512>, 128, 512, 8};
    if (D <= 2048) return {norm_bwd_kernel<ES, 256, V, 512>, 256, 512, 8};
    if (D <= 4096) return {norm_bwd_kernel<ES, 512, V, 512>, 512, 512, 8};
    if (D <= 8192) return {norm_bwd_kernel<ES, 1024, V, 1024>, 1024, 1024, 8};
    return {norm_bwd_kernel<ES, 1024, 2 * V, 1024>, 1024, 1024, 16};
}

}  // namespace

// Workgroups of the backward pass: two per compute unit of 512 threads (one of
// 1024) as far as the rows go.
void norm_bwd_grid(int64_t rows, int64_t D, int64_t gates, int type, int cus, int64_t* grid, int* parts) {
    const Config c = type == kBF16 ? bwd_config<2>(D) : bwd_config<4>(D);
    const int64_t nr = c.block / c.tpr, most = (c.block == 1024 ? 1 : 2) * (int64_t)cus;
    if (gates >= most * nr) {
        *parts = 0;
        *grid = most;
        return;
    }
    const int64_t rpg = rows / gates, fill = (rpg + nr - 1) / nr;
    int64_t p = most / gates;
    if (p > fill) p = fill;
    if (p < 1) p = 1;
    *parts = (int)p;
    *grid = p * gates;
}

hipError_t launch_norm_forward(const NormArgs& a, int cus, hipStream_t s) {
    const Config c = a.type == kBF16 ? fwd_config<2>(a.D) : fwd_config<4>(a.D);
    const int64_t nr = c.block / c.tpr, need = (a.rows + nr - 1) / nr, most = (int64_t)cus * (c.block == 1024 ? 2 : 8);
    hipLaunchKernelGGL(c.fn, dim3((unsigned)(need < most ? need : most)), dim3(c.block), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs& a, int64_t grid, hipStream_t s) {
    const Config c = a.type == kBF16 ? bwd_config<2>(a.D) : bwd_config<4>(a.D);
    hipError_t e = hipSuccess;
    if (grid > 0) {
        const size_t lds = (size_t)c.tpr * c.values * sizeof(float);
        if ((e = ensure_dynamic_lds(reinterpret_cast<const void*>(c.fn), lds)) != hipSuccess) return e;
        hipLaunchKernelGGL(c.fn, dim3((unsigned)grid), dim3(c.block), lds, s, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int64_t n = grid * a.D;
    if (a.dw_pre && (e = launch_colsum(a.partial, grid, a.D, 1, kF32, a.dw_pre, s)) != hipSuccess) return e;
    if (a.dw_post && (e = launch_colsum(a.partial + n, grid, a.D, 1, kF32, a.dw_post, s)) != hipSuccess) return e;
    if (a.dgate && a.rows == 0) return launch_colsum(a.partial, 0, a.gates * a.D, 1, a.type, a.dgate, s);
    if (a.dgate && a.parts) e = launch_colsum(a.partial + 2 * n, a.parts, a.D, a.gates, a.type, a.dgate, s);
    return e;
}

}  // namespace isam
