// Rows of bf16 or fp32 values moved 16 bytes per lane at the elements' own
// alignment (gfx950 serves unaligned global accesses; a piece that passes the
// end of its row is moved element by element), and the gate functions.
#pragma once

#include "common.hpp"

namespace isam {

// ES: bytes per element (2: bf16, 4: fp32).
template <int ES>
struct Row16 {
    static constexpr int E = 16 / ES;  // values of one piece

    // E values from element `at` of p, those from `valid` on as zeros.
    __device__ __forceinline__ static uint4 load(const void* p, int64_t at, int valid) {
        const char* q = static_cast<const char*>(p) + at * ES;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (valid >= E) {
            __builtin_memcpy(&v, q, 16);
        } else if (valid > 0) {
            uint32_t w[4] = {0, 0, 0, 0};
            static_for<E>([&](auto ec) {
                constexpr int e = decltype(ec)::value;
                if (e < valid) {
                    if constexpr (ES == 2) w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(q)[e] << (16 * (e & 1));
                    else w[e] = reinterpret_cast<const uint32_t*>(q)[e];
                }
            });
            v = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return v;
    }
    __device__ __forceinline__ static void store(void* p, int64_t at, uint4 v, int valid) {
        char* q = static_cast<char*>(p) + at * ES;
        if (valid >= E) {
            __builtin_memcpy(q, &v, 16);
        } else if (valid > 0) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            static_for<E>([&](auto ec) {
                constexpr int e = decltype(ec)::value;
                if (e < valid) {
                    if constexpr (ES == 2) reinterpret_cast<uint16_t*>(q)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                    else reinterpret_cast<uint32_t*>(q)[e] = w[e];
                }
            });
        }
    }
    __device__ __forceinline__ static void unpack(uint4 v, float (&f)[E]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        static_for<4>([&](auto pc) {
            constexpr int p = decltype(pc)::value;
            if constexpr (ES == 2) {
                f[2 * p] = bf16lo(w[p]);
                f[2 * p + 1] = bf16hi(w[p]);
            } else {
                f[p] = __uint_as_float(w[p]);
            }
        });
    }
    // bf16: rounded to nearest, ties to even (NaN stays NaN).
    __device__ __forceinline__ static uint4 pack(const float (&f)[E]) {
        uint32_t w[4];
        static_for<4>([&](auto pc) {
            constexpr int p = decltype(pc)::value;
            if constexpr (ES == 2) w[p] = pack_bf16_rne(f[2 * p], f[2 * p + 1]);
            else w[p] = __float_as_uint(f[p]);
        });
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // One value.
    __device__ __forceinline__ static float get(const void* p, int64_t at) {
        if constexpr (ES == 2) return bf16_to_f32(static_cast<const uint16_t*>(p)[at]);
        else return static_cast<const float*>(p)[at];
    }
    __device__ __forceinline__ static void put(void* p, int64_t at, float v) {
        if constexpr (ES == 2) static_cast<uint16_t*>(p)[at] = (uint16_t)pack_bf16_rne(v, 0.0f);
        else static_cast<float*>(p)[at] = v;
    }
};

// E fp32 values (states, biases): zeros from `valid` on.
template <int E>
__device__ __forceinline__ void load_f32(const float* p, int64_t at, int valid, float (&f)[E]) {
    if (p && valid >= E) {
        __builtin_memcpy(f, p + at, E * 4);
    } else {
        static_for<E>([&](auto ec) { f[ec] = p && ec < valid ? p[at + ec] : 0.0f; });
    }
}
template <int E>
__device__ __forceinline__ void store_f32(float* p, int64_t at, int valid, const float (&f)[E]) {
    if (valid >= E) {
        __builtin_memcpy(p + at, f, E * 4);
    } else {
        static_for<E>([&](auto ec) {
            if (ec < valid) p[at + ec] = f[ec];
        });
    }
}

// sigmoid(v) and 1 - sigmoid(v), each to fp32 accuracy also where it is small
// (1 - z from z would lose the digits that decide how long a state lives).
__device__ __forceinline__ void sigmoid_pair(float v, float& z, float& omz) {
    const float e = __expf(-v);
    z = __builtin_amdgcn_rcpf(1.0f + e);
    omz = v > 0.0f ? e * z : 1.0f - z;
}
// tanh to an absolute error of a few 2^-24 (its uses add values of size 1 to it).
__device__ __forceinline__ float tanh_f32(float x) {
    const float t = __expf(-2.0f * __builtin_fabsf(x));
    return __builtin_copysignf((1.0f - t) * __builtin_amdgcn_rcpf(1.0f + t), x);
}

}  // namespace isam
