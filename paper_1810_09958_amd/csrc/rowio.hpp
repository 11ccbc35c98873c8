// Rows of bf16 or fp32 values at the elements' own alignment, and the gate function of the
// feed-forward block.  Row16: single values, and pieces of 16 bytes straight from memory
// (gfx950 serves unaligned global accesses; a piece that passes the end of its row is loaded
// value by value), for the kernels of a few rows.  RowBuf: whole rows as buffers of their own
// length, for the norms.
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

// One row of D values spread over TPR threads, pieces of E values (8 or 16 bytes)
// each.  VEC (D a multiple of E, rows on 4 bytes): piece i of thread j is E
// neighbouring values, moved as one; otherwise its values are TPR apart, moved one
// by one.  The row is a buffer of its own length, so what lies past its end loads as
// zeros and is not stored, and no load or store stands in a branch of lanes.
template <int ES, bool VEC, int TPR, int E>
struct RowBuf {
    static constexpr int BYTES = E * ES;
    static_assert(BYTES == 8 || BYTES == 16, "8- or 16-byte pieces");
    struct Piece {
        uint32_t w[BYTES / 4];
    };
    // p + at elements; null or not live: an empty row.  Uniform over a wave.
    __device__ __forceinline__ static __amdgpu_buffer_rsrc_t row(const void* p, int64_t at, int64_t D, bool live) {
        const bool on = p != nullptr && live;
        return make_rsrc(on ? static_cast<const char*>(p) + at * ES : nullptr, on ? (uint32_t)(D * ES) : 0u);
    }
    __device__ __forceinline__ static Piece load(__amdgpu_buffer_rsrc_t rs, int i, int j) {
        Piece v;
        if constexpr (VEC && BYTES == 16) {
            const uint4 q = buf_load16(rs, (uint32_t)((i * TPR + j) * 16));
            v.w[0] = q.x; v.w[1] = q.y; v.w[2] = q.z; v.w[3] = q.w;
        } else if constexpr (VEC) {
            const auto q = __builtin_amdgcn_raw_buffer_load_b64(rs, (i * TPR + j) * 8, 0, 0);
            v.w[0] = (uint32_t)q[0]; v.w[1] = (uint32_t)q[1];
        } else {
            static_for<BYTES / 4>([&](auto k) { v.w[k] = 0; });
            static_for<E>([&](auto e) {
                const uint32_t off = (uint32_t)(((i * E + e) * TPR + j) * ES);
                if constexpr (ES == 4) v.w[e] = buf_load4(rs, off);
                else v.w[e / 2] |= (buf_load2(rs, off) & 0xffffu) << (16 * (e & 1));
            });
        }
        return v;
    }
    __device__ __forceinline__ static void unpack(const Piece& v, float (&f)[E]) {
        static_for<E>([&](auto e) {
            if constexpr (ES == 4) f[e] = __uint_as_float(v.w[e]);
            else if constexpr (e & 1) f[e] = bf16hi(v.w[e / 2]);
            else f[e] = bf16lo(v.w[e / 2]);
        });
    }
    // bf16: rounded to nearest, ties to even (NaN stays NaN).
    __device__ __forceinline__ static void store(__amdgpu_buffer_rsrc_t rs, int i, int j, const float (&f)[E]) {
        uint32_t w[BYTES / 4];
        static_for<BYTES / 4>([&](auto k) {
            if constexpr (ES == 4) w[k] = __float_as_uint(f[k]);
            else w[k] = pack_bf16_rne(f[2 * k], f[2 * k + 1]);
        });
        if constexpr (VEC && BYTES == 16) {
            __builtin_amdgcn_raw_buffer_store_b128((i32x4_t){(int)w[0], (int)w[1], (int)w[2], (int)w[3]}, rs, (i * TPR + j) * 16, 0, 0);
        } else if constexpr (VEC) {
            __builtin_amdgcn_raw_buffer_store_b64((i32x2_t){(int)w[0], (int)w[1]}, rs, (i * TPR + j) * 8, 0, 0);
        } else {
            static_for<E>([&](auto e) {
                const int off = ((i * E + e) * TPR + j) * ES;
                if constexpr (ES == 4) __builtin_amdgcn_raw_buffer_store_b32((int)w[e], rs, off, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b16((short)(w[e / 2] >> (16 * (e & 1))), rs, off, 0, 0);
            });
        }
    }
    // The fp32 values (weights, sums) at the places of piece i; rs of D fp32 values.
    __device__ __forceinline__ static uint32_t off32(int i, int j, int e) {
        return (uint32_t)((VEC ? (i * TPR + j) * E + e : (i * E + e) * TPR + j) * 4);
    }
    __device__ __forceinline__ static void load32(__amdgpu_buffer_rsrc_t rs, int i, int j, float (&f)[E]) {
        if constexpr (VEC) {
            static_for<E / 4>([&](auto q) {
                const uint4 v = buf_load16(rs, off32(i, j, 4 * q));
                f[4 * q] = __uint_as_float(v.x);
                f[4 * q + 1] = __uint_as_float(v.y);
                f[4 * q + 2] = __uint_as_float(v.z);
                f[4 * q + 3] = __uint_as_float(v.w);
            });
        } else {
            static_for<E>([&](auto e) { f[e] = __uint_as_float(buf_load4(rs, off32(i, j, e))); });
        }
    }
    __device__ __forceinline__ static void store32(__amdgpu_buffer_rsrc_t rs, int i, int j, const float (&f)[E]) {
        static_for<E>([&](auto e) { __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint(f[e]), rs, (int)off32(i, j, e), 0, 0); });
    }
};

// sigmoid(v) and 1 - sigmoid(v), each to fp32 accuracy also where it is small
// (1 - z from z would lose the digits that decide how long a state lives).
__device__ __forceinline__ void sigmoid_pair(float v, float& z, float& omz) {
    const float e = __expf(-v);
    z = __builtin_amdgcn_rcpf(1.0f + e);
    omz = v > 0.0f ? e * z : 1.0f - z;
}

}  // namespace isam
