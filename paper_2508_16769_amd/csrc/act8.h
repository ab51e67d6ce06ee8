// 8-bit activation checkpoints: the arithmetic of a group of 32 columns, and how the lanes of a wavefront share rows.
#pragma once

#include "dr_internal.h"

namespace drc {

constexpr int kActGroup = DR_ACT8_GROUP;
__host__ __device__ inline int act_groups(int D) { return (D + kActGroup - 1) / kActGroup; }

// Scale byte of a group from the largest magnitude's bits (not-a-numbers are larger than infinities, infinities than
// anything finite): the least b >= 1 with magnitude < 127.5 * 2^(b - 127).  127.5 is 1.9921875 * 2^6, a mantissa of 0x7f0000:
// adding 0x10000 carries into the exponent from there on.
__device__ __forceinline__ uint32_t act_scale(uint32_t top) {
    const int b = (int)((top + 0x10000u) >> 23) - 6;
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(b, 1), 248);
}
// what a value of the group is multiplied with to become its code; 0 for a group that is not finite
__device__ __forceinline__ float act_inverse(uint32_t b) { return b == 255u ? 0.0f : __builtin_bit_cast(float, (254u - b) << 23); }
// 2^(b - 127); not-a-number for 255 (an infinity is what its bits would be)
__device__ __forceinline__ float act_factor(uint32_t b) { return b == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, b << 23); }
// Code of a value, as an integer in a float.  Exact but for the rounding: the scale is a power of two.  (inf * 0 and a not-a-number: 0.)
__device__ __forceinline__ int act_code(float x, float inverse) {
    const float v = __builtin_amdgcn_fmed3f(__builtin_rintf(x * inverse), -127.0f, 127.0f);
    return inverse == 0.0f ? 0 : (int)v;
}
// place of the scale byte of (row, group)
__device__ __forceinline__ size_t act_scale_at(int64_t row, int group, int groups) {
    return ((size_t)(row >> 3) * groups + group) * 8 + (size_t)(row & 7);
}

// Rows over lanes.  W consecutive columns per load (4: rows are multiples of 16 bytes; 1: any width), LPR lanes per row, V loads per
// lane: lane t holds columns W * (t + LPR * v) ...  A group of 32 columns is then 32 / W neighbouring lanes of one v.
template <int W_, int LPR_, int V_> struct RowTile {
    static constexpr int W = W_, LPR = LPR_, V = V_;
    static constexpr int E = V * W;                    // elements per lane
    static constexpr int GL = 32 / W < LPR ? 32 / W : LPR;      // lanes of a group
    static_assert(LPR <= kWave && (GL == LPR || GL == 32 / W));
};
template <typename T> __device__ __forceinline__ int tile_col(int t, int v) { return T::W * (t + T::LPR * v); }

template <int LANES> __device__ __forceinline__ float lane_sum(float s) {
#pragma unroll
    for (int d = LANES / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, kWave);
    return s;
}
template <int LANES> __device__ __forceinline__ uint32_t lane_max(uint32_t s) {
#pragma unroll
    for (int d = LANES / 2; d >= 1; d >>= 1) s = max(s, (uint32_t)__shfl_xor((int)s, d, kWave));
    return s;
}

// x[E]: a row's elements of this lane, zeros past the width
template <typename T> __device__ __forceinline__ void row_load(const float* __restrict__ row, int t, int D, bool on, float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        const int c = tile_col<T>(t, v);
        if constexpr (T::W == 4) {
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (on && c < D) f = *reinterpret_cast<const float4*>(row + c);
            x[4 * v] = f.x; x[4 * v + 1] = f.y; x[4 * v + 2] = f.z; x[4 * v + 3] = f.w;
        } else {
            x[v] = on && c < D ? row[c] : 0.f;
        }
    }
}
template <typename T> __device__ __forceinline__ void row_store(float* row, int t, int D, bool on, const float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        const int c = tile_col<T>(t, v);
        if (!on || c >= D) continue;
        if constexpr (T::W == 4) *reinterpret_cast<float4*>(row + c) = make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]);
        else row[c] = x[v];
    }
}
// the same from and to a checkpoint
template <typename T>
__device__ __forceinline__ void row_unpack(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, int64_t row, int t, int D, int groups,
                                           bool on, float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        const int c = tile_col<T>(t, v);
        const bool have = on && c < D;
        const float f = have ? act_factor(scale[act_scale_at(row, c / kActGroup, groups)]) : 0.f;
        if constexpr (T::W == 4) {
            const int w = have ? *reinterpret_cast<const int*>(q + (size_t)row * D + c) : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * v + j] = (float)(int8_t)(w >> (8 * j)) * f;
        } else {
            x[v] = have ? (float)q[(size_t)row * D + c] * f : 0.f;
        }
    }
}
// Every lane of the row group takes part.  Bytes of the rows behind the last one of the array are written by its row.
template <typename T>
__device__ __forceinline__ void row_pack(int8_t* q, uint8_t* scale, int64_t row, int64_t n, int t, int D, int groups, bool on, const float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        const int c = tile_col<T>(t, v);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < T::W; ++j) top = max(top, __builtin_bit_cast(uint32_t, x[T::W * v + j]) & 0x7fffffffu);
        const uint32_t b = act_scale(lane_max<T::GL>(top));
        const float inverse = act_inverse(b);
        if (!on || c >= D) continue;
        if constexpr (T::W == 4) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w |= ((uint32_t)act_code(x[4 * v + j], inverse) & 0xffu) << (8 * j);
            *reinterpret_cast<uint32_t*>(q + (size_t)row * D + c) = w;
        } else {
            q[(size_t)row * D + c] = (int8_t)act_code(x[v], inverse);
        }
        if (c % kActGroup == 0) {
            scale[act_scale_at(row, c / kActGroup, groups)] = (uint8_t)b;
            if (row == n - 1)
                for (int64_t r = n; r & 7; ++r) scale[act_scale_at(r, c / kActGroup, groups)] = 0;
        }
    }
}

// Calls f(RowTile<...>{}) with the narrowest tile that holds a row of D columns; `vector`: rows are read four columns at a time.
template <typename F> int with_row_tile(int D, bool vector, F f) {
    if (vector) {
        if (D <= 32) return f(RowTile<4, 8, 1>{});
        if (D <= 64) return f(RowTile<4, 16, 1>{});
        if (D <= 128) return f(RowTile<4, 32, 1>{});
        if (D <= 256) return f(RowTile<4, 64, 1>{});
        if (D <= 512) return f(RowTile<4, 64, 2>{});
        return f(RowTile<4, 64, 4>{});
    }
    if (D <= 4) return f(RowTile<1, 4, 1>{});
    if (D <= 8) return f(RowTile<1, 8, 1>{});
    if (D <= 16) return f(RowTile<1, 16, 1>{});
    if (D <= 32) return f(RowTile<1, 32, 1>{});
    if (D <= 64) return f(RowTile<1, 64, 1>{});
    if (D <= 128) return f(RowTile<1, 64, 2>{});
    if (D <= 256) return f(RowTile<1, 64, 4>{});
    if (D <= 512) return f(RowTile<1, 64, 8>{});
    return f(RowTile<1, 64, 16>{});
}

// host side ------------------------------------------------------------------------------------------
int launch_act8_pack(const float* X, int64_t n, int D, const dr_act8& out, hipStream_t s);
int launch_act8_unpack(const dr_act8& in, int64_t n, int D, float* X, hipStream_t s);
size_t act8_wgrad_workspace(int64_t n, int D, int F);
int launch_act8_wgrad(const dr_act8& A, int64_t n, int D, const float* dZ, int F, float* dW, bool accumulate, void* ws, hipStream_t s);
struct BlockFwd {
    dr_block b;
    int64_t n;
    int D;
    const float *X, *Y, *G;
    float *X_out, *N;
    dr_block_saved saved;
};
int launch_block_fwd(const BlockFwd& a, hipStream_t s);
struct BlockBwd {
    dr_block b;
    int64_t n;
    int D;
    const float *dX_out, *dN, *X_out, *Y, *G;
    dr_block_saved saved;
    dr_block_grads grads;
    float* part;                  // [workgroups][5][D]
    int parts;
};
size_t block_bwd_workspace(int64_t n, int D);
int launch_block_bwd(BlockBwd a, void* ws, hipStream_t s);

}  // namespace drc
