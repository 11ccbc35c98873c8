// One step of beam search.  Of each text's beams x vocabulary candidates, of value
//   score_i + logits_i[v] - log(sum_w exp(logits_i[w])),
// the best `width`, equal ones by the lowest place i V + v.
//
// Bound by one pass over the logits.  Within a beam the order is that of the logits themselves, so
// the first kernel reads each once: a workgroup takes 4096 of a row into registers, sums their
// exponentials from their maximum, and leaves its best `width`, in order.  To find them without sorting,
// each lane takes its own best; of these the width-th (of the wave, or of the workgroup) is a bound that at most
// width lanes pass, so at most 16 width values are left to order (a few more than width, mostly), by counting for each
// how many are better.  Every key holds the place too, so no two are equal and ties need no care.
// The exponentials and their sum are in 64 bits, as the difference of two beams' sums decides between candidates (in fp32,
// 2^-23 to each, 32 texts of 8 beams over 32000 took 27.5 us instead of 33 and beams closer than that changed places).
// The second kernel, a workgroup to a text, forms the values of the candidates that are left, in 64 bits too (an fp32
// sum of scores and logits would make ties of what is none), and
// takes the best in the same way, the lists' first entries first: it ends where none of a piece is among the best.
// In a kernel trace: one text of 4 beams over 256 5.4 and 9.9 us; 32 texts of 8 beams over 32000 (33 MB) 19.8 and 15.9,
// 1.7 TB/s for the first (52 vector instructions a value, most of them the exponential in 64 bits, and the loads and
// exchanges of a workgroup's one piece before and after them).  Latency holds the second.
#include "kernels.hpp"
#include "rowio.hpp"

namespace isam {

namespace {

// A value's order as unsigned, never 0; both zeros are one.
__device__ __forceinline__ uint32_t order32(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return (int)u < 0 ? max(~u, 1u) : u | 0x80000000u;  // (one NaN would have 0)
}
__device__ __forceinline__ float value32(uint32_t o) { return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t order64(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
    return (int64_t)u < 0 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double value64(uint64_t o) {
    return __longlong_as_double((long long)((int64_t)o < 0 ? o & 0x7fffffffffffffffull : ~o));
}

constexpr int kEach = (int)(kBeamPart / 256);  // logits of a thread

// The n-th largest of the values of the lanes in `of` (0: there are fewer), bit by bit from the highest: one
// comparison of the wave and a count of its lanes each, the counts in scalar registers.
__device__ __forceinline__ uint32_t nth(uint32_t v, uint64_t of, int n) {
    uint32_t t = 0;
    if ((of & (of - 1)) == 0 && n == 1 && of) return (uint32_t)__builtin_amdgcn_readlane((int)v, __builtin_ctzll(of));
    static_for<32>([&](auto k) {
        const uint32_t more = t | 0x80000000u >> decltype(k)::value;
        if (__builtin_popcountll(__ballot(v >= more) & of) >= n) t = more;
    });
    return t;
}

template <int ES, bool ALL>
__global__ __launch_bounds__(256) void beam_part_kernel(BeamArgs a) {
    constexpr int E = 16 / ES, Q = kEach / E;  // values of a 16-byte piece, pieces of a thread
    extern __shared__ __attribute__((aligned(16))) uint64_t list[];  // of kEach width: at most width lanes (of each wave, without ALL) have any
    __shared__ double wsum[4];
    __shared__ float wmax[4];
    __shared__ uint64_t firsts[ALL ? 256 : 1];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int64_t row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts, b = row / a.beams, i = row - b * a.beams;
    const int64_t base = b * a.lg_b + i * a.lg_n, v0 = part * kBeamPart;
    const int W = (int)a.width;
    float v[kEach];
    static_for<Q>([&](auto q) {
        const int64_t at = v0 + (int64_t)(q * 256 + tid) * E;
        const int n = (int)max((int64_t)0, min((int64_t)E, a.V - at));
        const uint4 w = Row16<ES>::load(a.logits, base + at, n);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
        static_for<E>([&](auto e) {
            float f;
            if constexpr (ES == 4) f = __uint_as_float(ws[e]);
            else if constexpr (e & 1) f = bf16hi(ws[e / 2]);
            else f = bf16lo(ws[e / 2]);
            v[q * E + e] = e < n ? f : -INFINITY;
        });
    });
    // value k of the thread: place v0 + ((k / E) 256 + tid) E + k % E
    auto place = [&](int k) { return v0 + (int64_t)((k / E) * 256 + tid) * E + k % E; };
    auto key = [&](int k) { return (uint64_t)order32(v[k]) << 32 | (uint32_t)~(uint32_t)place(k); };
    // The thread's best: places rise with k, so the first of equal values is.  A NaN is above nothing, so whatever its bits
    // it hides none of the thread's values from the bound, which is what the list's size rests on (a NaN that passes for
    // want of a bound makes the row one without candidates).
    float most = -INFINITY;
    int at = 0;
    static_for<kEach>([&](auto k) {
        const bool up = v[k] > most;
        at = up ? (int)k : at;
        most = up ? v[k] : most;
    });
    const uint64_t first = place(0) < a.V ? (uint64_t)order32(most) << 32 | (uint32_t)~(uint32_t)place(at) : 0ull;
    for (int m = 32; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (lane == 0) wmax[wid] = most;
    if constexpr (ALL) firsts[tid] = first;
    if (tid == 0) count = 0;
    __syncthreads();
    most = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
    // the width-th of the firsts, by value and then (where that many are equal) by place; 0: fewer lanes have any.
    // ALL: of the workgroup's, four times the comparisons, which pays where many pass (32 texts of 8 beams over 32000
    // 13.0 of a wave's against 15.6 us, 4 texts of 64 beams 671 against 445 with the second kernel, with sums in fp32).
    uint64_t least = 0;
    if constexpr (ALL) {
        uint32_t hi[4], lo[4], low = 0, rest = 0;
        static_for<4>([&](auto k) {
            const uint64_t f = firsts[k * 64 + lane];
            hi[k] = (uint32_t)(f >> 32);
            lo[k] = (uint32_t)f;
        });
        auto lanes = [&](auto which) {
            int n = 0;
            static_for<4>([&](auto k) { n += __builtin_popcountll(__ballot(which(k))); });
            return n;
        };
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1) low = lanes([&](auto k) { return hi[k] >= (low | bit); }) >= W ? low | bit : low;
        if (low) {
            const int more = W - lanes([&](auto k) { return hi[k] > low; });
            if (lanes([&](auto k) { return hi[k] == low; }) > more)
                for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
                    rest = lanes([&](auto k) { return hi[k] == low && lo[k] >= (rest | bit); }) >= more ? rest | bit : rest;
        }
        least = (uint64_t)low << 32 | rest;
    } else {
        const uint32_t hi = (uint32_t)(first >> 32), low = nth(hi, ~0ull, W);
        if (low) least = (uint64_t)low << 32 | nth((uint32_t)first, __ballot(hi == low), W - __builtin_popcountll(__ballot(hi > low)));
    }
    const float bound = value32((uint32_t)(least >> 32));
    static_for<kEach>([&](auto k) {
        if (place(k) < a.V && (least == 0 || v[k] >= bound)) {
            const uint64_t u = key(k);
            if (u >= least) list[atomicAdd(&count, 1)] = u;
        }
    });
    // the sum; a NaN or an infinite maximum leaves NaN, which the second kernel takes as a row without candidates.  A part
    // of -inf has none, but a NaN may stand among them.
    double sum = 0.0;
    if (most == -INFINITY) static_for<kEach>([&](auto k) { sum = v[k] == v[k] ? sum : (double)v[k]; });
    else static_for<kEach>([&](auto k) { sum += exp((double)v[k] - (double)most); });
    for (int m = 32; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) wsum[wid] = sum;
    __syncthreads();
    const int n = count;
    uint64_t* const out = a.best + (row * a.parts + part) * W;
    for (int k = tid; k < n; k += 256) {
        const uint64_t u = list[k];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += list[j] > u;
        if (rank < W) out[rank] = u;
    }
    for (int k = n + tid; k < W; k += 256) out[k] = 0;
    if (tid == 0) a.sums[row * a.parts + part] = make_double2((double)most, (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]));
}

// A candidate: its value's order (0: none) and its place, lowest first; the order of its logit (0: none of a beam that goes on).
struct Cand {
    uint64_t order;
    uint32_t place, logit;
};
__device__ __forceinline__ bool ahead(const Cand& x, const Cand& y) {
    return x.order > y.order || (x.order == y.order && x.order && x.place < y.place);
}

constexpr int kAtOnce = 8;  // candidates of a thread

__global__ __launch_bounds__(256) void beam_join_kernel(BeamArgs a) {
    __shared__ double offset[kBeamMax];       // score - log sum; -inf: no candidate but of -inf
    __shared__ bool over[kBeamMax];           // finished
    __shared__ Cand list[4 * (kAtOnce + 1) * kBeamMax];
    __shared__ Cand best[kBeamMax];
    __shared__ int count, some[4];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, W = (int)a.width, parts = (int)a.parts, beams = (int)a.beams;
    const int64_t b = blockIdx.x;
    // candidate c: of list c % lists (a part of a beam) the c / lists-th
    const uint32_t lists = (uint32_t)beams * (uint32_t)parts, all = lists * (uint32_t)W, V = (uint32_t)a.V, end = (uint32_t)a.end;
    const uint64_t* const from = a.best + b * (int64_t)all;
    const uint64_t early = tid < all ? from[tid % lists * W + tid / lists] : 0ull;  // (on its way during the sums)
    int lanes = 1;
    while (lanes < 64 && lanes < parts) lanes *= 2;
    // a lane to a part, 64 / lanes beams to a wave
    const int at = lane & (lanes - 1), one = 64 / lanes;
    for (int i0 = wid * one; i0 < beams; i0 += 4 * one) {
        const int i = min(i0 + lane / lanes, beams - 1);
        const int64_t row = b * beams + i;
        const double2* const s = a.sums + row * parts;
        const double score = (double)a.scores[row];
        const bool done = a.finished && a.finished[row];
        const double2 own = at < parts ? s[at] : make_double2(-INFINITY, 0.0);
        double most = own.x;
        for (int p = at + 64; p < parts; p += 64) most = s[p].x > most ? s[p].x : most;
        for (int m = lanes / 2; m > 0; m >>= 1) {
            const double o = __shfl_xor(most, m);
            most = o > most ? o : most;
        }
        // (a part without a finite logit has the sum 0, or NaN)
        double2 v = own;
        double sum = 0.0;
        for (int p = at; p < parts;) {
            sum += v.x == -INFINITY ? v.y : v.y * exp(v.x - most);
            if ((p += 64) < parts) v = s[p];
        }
        for (int m = lanes / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
        const double o = done ? score : most == -INFINITY || most == INFINITY ? -INFINITY : score - (most + log(sum));
        if (at == 0) {
            offset[i] = o == o ? o : -INFINITY;
            over[i] = done;
        }
    }
    for (int k = tid; k < W; k += 256) best[k] = Cand{0, 0, 0};
    __syncthreads();
    // of a beam that can go on the parts' best, else the first tokens
    const double none = -INFINITY;
    auto candidate = [&](uint32_t c) {
        const uint32_t k = c / lists, l = c - k * lists, i = l / (uint32_t)parts;
        const double o = offset[i];
        if (over[i] || o == none) {
            // (a finished beam: its end token, then the others)
            if (l != i * (uint32_t)parts || k >= V) return Cand{0, 0, 0};
            if (over[i] && o != none) {
                const uint32_t v = k == 0 ? end : k - 1 < end ? k - 1 : k;
                return Cand{order64(k == 0 ? o : none), i * V + v, 0};
            }
            return Cand{order64(none), i * V + k, 0};
        }
        const uint64_t u = c < 256 ? early : from[l * W + k];
        if (!u) return Cand{0, 0, 0};
        const double v = o + (double)value32((uint32_t)(u >> 32));
        return Cand{order64(v == v ? v : none), i * V + ~(uint32_t)u, (uint32_t)(u >> 32)};
    };
    for (uint32_t c0 = 0; c0 < all; c0 += 256 * kAtOnce) {
        Cand mine[kAtOnce + 1];
        const Cand last = best[W - 1];  // (nothing behind it can be among the best any more)
        static_for<kAtOnce>([&](auto k) {
            const uint32_t c = c0 + k * 256 + tid;
            mine[k] = Cand{0, 0, 0};
            if (c0 + k * 256 < all && c < all) mine[k] = candidate(c);
            if (ahead(last, mine[k])) mine[k].order = 0;
        });
        mine[kAtOnce] = tid < W ? best[tid] : Cand{0, 0, 0};
        if (tid == 0) count = 0;
        Cand first{0, 0, 0};
        static_for<kAtOnce + 1>([&](auto k) { first = ahead(mine[k], first) ? mine[k] : first; });
        // the width-th of the wave's firsts, as above: its order in two halves, then (where that many are equal) its place
        const uint32_t hi = (uint32_t)(first.order >> 32), lo = (uint32_t)first.order;
        const uint64_t with = __ballot(first.order != 0);
        const uint32_t t1 = with ? nth(hi, with, W) : 0u;
        uint32_t t2 = 0, t3 = 0;
        if (t1) {
            const uint64_t tie = __ballot(hi == t1);
            const int n2 = W - __builtin_popcountll(__ballot(hi > t1));
            if (__builtin_popcountll(tie) > n2) {
                t2 = nth(lo, tie, n2);
                const uint64_t both = tie & __ballot(lo == t2);
                const int n3 = n2 - __builtin_popcountll(tie & __ballot(lo > t2));
                if (__builtin_popcountll(both) > n3) t3 = nth(~first.place, both, n3);
            }
        }
        const uint64_t least = (uint64_t)t1 << 32 | t2;
        __syncthreads();  // (best has been read, count is clear)
        bool fresh = false;
        static_for<kAtOnce + 1>([&](auto k) {
            if (mine[k].order > least || (mine[k].order == least && least && ~mine[k].place >= t3)) {
                list[atomicAdd(&count, 1)] = mine[k];
                fresh = fresh || k < kAtOnce;
            }
        });
        // (each list falls: where none of it is among the best, none behind is)
        if (!__syncthreads_or(fresh) && lists <= 256 * kAtOnce) break;
        const int n = count;
        for (int k = tid; k < n; k += 256) {
            const Cand u = list[k];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += ahead(list[j], u);
            if (rank < W) best[rank] = u;
        }
        __syncthreads();
    }
    // Unequal logits may have equal values (beside a score of the type's lowest value all have): of the last of the best's
    // value the lists hold their parts' largest logits, not the lowest places.  A place left out of a list, or behind where
    // the walk ended, is ahead of that last one only where the list has an entry of the same value that is not, behind it or
    // the last itself, and so only in the part of the last: its places of that value are looked through.
    const Cand low = best[W - 1];
    const uint32_t beam = low.place / V;
    auto order_of = [&](uint32_t logit) { return order64(offset[beam] + (double)value32(logit)); };
    const bool merged = low.logit && (order_of(low.logit + 1) == low.order ||
                                      order_of(low.logit - (low.logit == 0x80000000u ? 2 : 1)) == low.order);  // (past -0)
    if (merged) {
        const uint32_t v0 = (low.place - beam * V) / (uint32_t)kBeamPart * (uint32_t)kBeamPart, n = min(V - v0, (uint32_t)kBeamPart);
        const uint32_t p0 = beam * V + v0;
        const int64_t base = b * a.lg_b + beam * a.lg_n + v0;
        for (int k = tid; k < W; k += 256) {
            Cand u = best[k];
            if (u.order == low.order && u.place - p0 < n) u.order = 0;
            list[k] = u;
        }
        int found = 0;
        for (uint32_t v = 0; v < n && found < W; v += 256) {
            uint32_t logit = 0;
            if (v + tid < n) logit = order32(a.type == kBF16 ? Row16<2>::get(a.logits, base + v + tid) : Row16<4>::get(a.logits, base + v + tid));
            const bool same = logit && order_of(logit) == low.order;
            const uint64_t with = __ballot(same);
            if (lane == 0) some[wid] = __builtin_popcountll(with);
            __syncthreads();
            int at = found + __builtin_popcountll(with & ((1ull << lane) - 1));
            for (int w = 0; w < 4; ++w) {
                at += w < wid ? some[w] : 0;
                found += some[w];
            }
            if (same && at < W) list[W + at] = Cand{low.order, p0 + v + tid, logit};
            __syncthreads();
        }
        const int all = W + min(found, W);
        for (int k = tid; k < all; k += 256) {
            const Cand u = list[k];
            int rank = 0;
            for (int j = 0; j < all; ++j) rank += ahead(list[j], u);
            if (u.order && rank < W) best[rank] = u;
        }
        __syncthreads();
    }
    for (int k = tid; k < W; k += 256) {
        const Cand u = best[k];
        const uint32_t i = u.place / V, v = u.place - i * V;
        const int64_t at = b * W + k;
        a.scores_out[at] = (float)value64(u.order);
        a.parent[at] = (int32_t)i;
        a.token[at] = (int32_t)v;
        if (a.finished_out) a.finished_out[at] = (int64_t)v == a.end || over[i];
    }
}

// Rows of the beams that go on; a parent that is none of the beams leaves zeros.
template <typename V>
__global__ __launch_bounds__(256) void beam_reorder_kernel(ReorderArgs a) {
    constexpr int U = 4;
    const int64_t n = a.bytes / (int64_t)sizeof(V), blocks = (n + 256 * U - 1) / (256 * U);
    const int64_t row = blockIdx.x / blocks, at = (blockIdx.x - row * blocks) * 256 * U + threadIdx.x;
    const int64_t o = row / (a.batch * a.width), r = row - o * a.batch * a.width, b = r / a.width;
    const int64_t from = a.parent[r];
    const bool in = from >= 0 && from < a.beams;
    const V* const src = static_cast<const V*>(a.src) + ((o * a.batch + b) * a.beams + (in ? from : 0)) * n;
    V* const dst = static_cast<V*>(a.dst) + row * n;
    V v[U];
    static_for<U>([&](auto k) {
        const int64_t i = at + 256 * k;
        if (i < n) v[k] = src[i];
    });
    static_for<U>([&](auto k) {
        const int64_t i = at + 256 * k;
        if (i < n) dst[i] = in ? v[k] : V{};
    });
}

}  // namespace

hipError_t launch_beam_step(const BeamArgs& a, hipStream_t s) {
    const int64_t rows = a.batch * a.beams;
    if (rows * a.parts > INT32_MAX) return hipErrorInvalidValue;
    const bool all = a.width > 16;
    const size_t room = (size_t)((all ? 1 : 4) * kEach * a.width) * sizeof(uint64_t);
    typedef void (*PartFn)(BeamArgs);
    const PartFn fn = a.type == kBF16 ? (all ? beam_part_kernel<2, true> : beam_part_kernel<2, false>)
                                      : (all ? beam_part_kernel<4, true> : beam_part_kernel<4, false>);
    hipLaunchKernelGGL(fn, dim3((unsigned)(rows * a.parts)), dim3(256), room, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)a.batch), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_beam_reorder(const ReorderArgs& a, hipStream_t s) {
    const uintptr_t both = (uintptr_t)a.src | (uintptr_t)a.dst | (uintptr_t)a.bytes;
    const int64_t size = both % 16 == 0 ? 16 : both % 4 == 0 ? 4 : 1;
    const int64_t blocks = a.outer * a.batch * a.width * ((a.bytes / size + 1023) / 1024);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((size == 16 ? beam_reorder_kernel<uint4> : size == 4 ? beam_reorder_kernel<uint32_t> : beam_reorder_kernel<uint8_t>),
                       dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace isam
