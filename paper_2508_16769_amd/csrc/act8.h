// Rows of embeddings over the lanes of a workgroup, and the arithmetic of 8-bit activation checkpoints.
#pragma once

#include "dr_internal.h"

namespace drc {

constexpr int kActGroup = DR_ACT8_GROUP;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t bits(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float of_bits(uint32_t x) { return __builtin_bit_cast(float, x); }

// ---- buffers --------------------------------------------------------------------------------------
// A view of the rows that a workgroup takes next: its base is their first byte and its size ends with the array, so rows past the end
// read as zeros and are not written, and neither is anything of a tensor that is absent.  No access is conditional, and the
// offsets of a lane are the same for every block of rows.
using Buf = __amdgpu_buffer_rsrc_t;
constexpr int kOutside = 0x40000000;               // an offset outside every view (so is a quarter of it)
__device__ __forceinline__ Buf buf_view(const void* p, int64_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), (short)0,
                                             __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
// `left` rows of `row_bytes` from row r0 on
__device__ __forceinline__ Buf rows_view(const void* p, int64_t r0, int left, int row_bytes) {
    return buf_view(static_cast<const char*>(p) + r0 * row_bytes, p ? left * row_bytes : 0);
}
// scale bytes from row r0 on, those of the rows that fill up the last eight among them (a block of rows is 64 at most)
__device__ __forceinline__ Buf scales_view(const uint8_t* p, int64_t r0, int64_t n, int groups) {
    const int64_t blocks = ((n + 7) >> 3) - (r0 >> 3);
    const int first = (int)(r0 & 7), have = (int)(blocks < 0 ? 0 : blocks > 8 ? 8 : blocks) * groups * 8;
    return buf_view(p + (r0 >> 3) * groups * 8 + first, p && have > first ? have - first : 0);
}

// ---- rows over lanes ------------------------------------------------------------------------------
// W consecutive columns per load (4: rows are multiples of 16 bytes; 1: any width), LPR lanes per row, V loads per lane: lane t holds
// columns W * (t + LPR * v) ...  A group of 32 columns is then 32 / W neighbouring lanes of one v.  No lane holds more than four elements,
// whatever the width: with 16 of them the backward pass took all registers of a SIMD for one wavefront.
constexpr int kRowThreads = 256;
template <int W_, int LPR_, int V_> struct RowTile {
    static constexpr int W = W_, LPR = LPR_, V = V_;
    static constexpr int E = V * W;                             // elements per lane
    static constexpr int R = kRowThreads / LPR;                 // rows per workgroup
    static constexpr int GL = 32 / W < LPR ? 32 / W : LPR;      // lanes of a group
    static_assert(E <= 4 && LPR <= kRowThreads && R <= 64 && (V == 1 || W * LPR % 32 == 0));
};
// this lane's places in the rows of a workgroup
template <typename T> struct RowLane {
    int row, t;                   // row of the workgroup's, lane of the row
    int at[T::V];                 // byte offset of fp32 elements; codes are at a quarter of it
    int scale[T::V];              // of the scale byte
    __device__ __forceinline__ RowLane(int D) : row((int)threadIdx.x / T::LPR), t((int)threadIdx.x % T::LPR) {
        const int groups = act_groups(D);
#pragma unroll
        for (int v = 0; v < T::V; ++v) {
            const int c = col(v);
            at[v] = c < D ? (row * D + c) * 4 : kOutside;
            scale[v] = c < D ? (row >> 3) * groups * 8 + c / kActGroup * 8 + (row & 7) : kOutside;
        }
    }
    __device__ __forceinline__ int col(int v) const { return T::W * (t + T::LPR * v); }
};

// Sums and maxima over lanes: within 16 by lane permutations inside the instruction, beyond by exchanges of rows of 16 and 32.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true); }
template <int LANES, typename F> __device__ __forceinline__ uint32_t over_lanes(uint32_t x, F f) {
    static_assert(LANES <= kWave);
    if constexpr (LANES >= 2) x = f(x, dpp<0xb1>(x));           // neighbours
    if constexpr (LANES >= 4) x = f(x, dpp<0x4e>(x));           // pairs of a quad
    if constexpr (LANES >= 8) x = f(x, dpp<0x141>(x));          // quads of a half row (mirrored)
    if constexpr (LANES >= 16) x = f(x, dpp<0x140>(x));         // half rows (mirrored)
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = f(p[0], p[1]);
    }
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = f(p[0], p[1]);
    }
    return x;
}
template <int LANES> __device__ __forceinline__ float lane_sum(float s) {
    return of_bits(over_lanes<LANES>(bits(s), [](uint32_t a, uint32_t b) { return bits(of_bits(a) + of_bits(b)); }));
}
template <int LANES> __device__ __forceinline__ uint32_t lane_max(uint32_t s) {
    return over_lanes<LANES>(s, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
// Sums over the lanes of a row, in every lane of it.  Rows of more than a wavefront meet in LDS; calls take the two halves of it in
// turn, so that one barrier is enough: a wavefront is at most one call ahead.
struct RowSums {
    float (*sh)[kRowThreads / kWave][2];                        // [2][wavefronts][2]
    int turn;
    template <typename T> __device__ __forceinline__ void sum(float& a, float& b) {
        if constexpr (T::LPR <= kWave) {
            a = lane_sum<T::LPR>(a);
            b = lane_sum<T::LPR>(b);
        } else {
            a = lane_sum<kWave>(a);
            b = lane_sum<kWave>(b);
            const int wave = threadIdx.x / kWave;
            if (threadIdx.x % kWave == 0) { sh[turn][wave][0] = a; sh[turn][wave][1] = b; }
            __syncthreads();
            constexpr int N = T::LPR / kWave;
            const int first = wave / N * N;
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < N; ++w) { a += sh[turn][first + w][0]; b += sh[turn][first + w][1]; }
            turn ^= 1;
        }
    }
    template <typename T> __device__ __forceinline__ float sum(float a) {
        if constexpr (T::LPR <= kWave) {
            return lane_sum<T::LPR>(a);
        } else {
            float b = 0.f;
            sum<T>(a, b);
            return a;
        }
    }
};

template <typename T> __device__ __forceinline__ void load_rows(Buf b, const RowLane<T>& l, uint32_t (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        if constexpr (T::W == 4) {
            const u32x4 f = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, l.at[v], 0, 0));
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * v + j] = f[j];
        } else {
            x[v] = __builtin_amdgcn_raw_buffer_load_b32(b, l.at[v], 0, 0);
        }
    }
}
// Elements in registers of their own: the loads of the next rows can then go where these came from.  (Left to itself the compiler loads the
// next rows elsewhere and copies them, which waits for the loads that have just been issued.)
template <int N> __device__ __forceinline__ void take(const uint32_t (&from)[N], float (&to)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        to[i] = of_bits(from[i]);
        asm volatile("" : "+v"(to[i]));
    }
}
constexpr int kStreamed = 2;      // cache policy of stores that nothing is to be read from soon
template <typename T, int POLICY = 0> __device__ __forceinline__ void store_rows(Buf b, const RowLane<T>& l, const float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        if constexpr (T::W == 4)
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{bits(x[4 * v]), bits(x[4 * v + 1]), bits(x[4 * v + 2]), bits(x[4 * v + 3])}, b, l.at[v], 0, POLICY);
        else
            __builtin_amdgcn_raw_buffer_store_b32(bits(x[v]), b, l.at[v], 0, POLICY);
    }
}

// ---- 8-bit checkpoints ----------------------------------------------------------------------------
// Scale byte of a group from the largest magnitude's bits (not-a-numbers are larger than infinities, infinities than
// anything finite): the least b >= 1 with magnitude < 127.5 * 2^(b - 127).  127.5 is 1.9921875 * 2^6, a mantissa of 0x7f0000:
// adding 0x10000 carries into the exponent from there on.
__device__ __forceinline__ uint32_t act_scale(uint32_t top) {
    const int b = (int)((top + 0x10000u) >> 23) - 6;
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(b, 1), 248);
}

// Codes and scale byte of a lane's elements; every lane of a row group takes part.  The one rounding is the code's: the scale is a power
// of two.  Rows at or behind the end (`on` false) have zeros as scale bytes, and no room for codes.
template <typename T>
__device__ __forceinline__ void store_codes(Buf q, Buf s, const RowLane<T>& l, bool on, const float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < T::W; ++j) top = max(top, bits(x[T::W * v + j]) & 0x7fffffffu);
        const uint32_t b = act_scale(lane_max<T::GL>(top));
        const float inverse = of_bits((254u - min(b, 253u)) << 23);
        uint32_t c[T::W];
#pragma unroll
        for (int j = 0; j < T::W; ++j)
            c[j] = (uint32_t)(int)__builtin_amdgcn_fmed3f(__builtin_rintf(x[T::W * v + j] * inverse), -127.0f, 127.0f);
        if constexpr (T::W == 4) {
            // lowest bytes of the four
            const uint32_t lo = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u);
            __builtin_amdgcn_raw_buffer_store_b32(b == 255u ? 0u : (lo | hi << 16), q, l.at[v] >> 2, 0, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b8((uint8_t)(b == 255u ? 0u : c[0]), q, l.at[v] >> 2, 0, 0);
        }
        __builtin_amdgcn_raw_buffer_store_b8((uint8_t)(on ? b : 0u), s, l.t % T::GL == 0 ? l.scale[v] : kOutside, 0, 0);
    }
}
// Codes and scale bytes as they come from memory
template <typename T> __device__ __forceinline__ void load_codes(Buf q, Buf s, const RowLane<T>& l, uint32_t (&code)[T::E], uint32_t (&scale)[T::V]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        if constexpr (T::W == 4) code[4 * v] = __builtin_amdgcn_raw_buffer_load_b32(q, l.at[v] >> 2, 0, 0);
        else code[v] = __builtin_amdgcn_raw_buffer_load_b8(q, l.at[v] >> 2, 0, 0);
        scale[v] = __builtin_amdgcn_raw_buffer_load_b8(s, l.scale[v], 0, 0);
    }
}
// What they stand for.  255 << 23 is an infinity and the codes of such a group are zeros: not-a-numbers.  Scale bytes of rows past the end
// (`on` false) may hold anything.
template <typename T>
__device__ __forceinline__ void decode(const uint32_t (&code)[T::E], const uint32_t (&scale)[T::V], bool on, float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v) {
        const float f = on ? of_bits(scale[v] << 23) : 0.f;
#pragma unroll
        for (int j = 0; j < T::W; ++j) x[T::W * v + j] = (float)(int8_t)(code[T::W * v] >> (8 * j)) * f;
    }
}

// Calls f(RowTile<...>{}) with the narrowest tile that holds a row of D columns; `vector`: rows are read four columns at a time.
template <typename F> int with_row_tile(int D, bool vector, F f) {
    if (vector) {
        if (D <= 32) return f(RowTile<4, 8, 1>{});
        if (D <= 64) return f(RowTile<4, 16, 1>{});
        if (D <= 128) return f(RowTile<4, 32, 1>{});
        if (D <= 256) return f(RowTile<4, 64, 1>{});
        if (D <= 512) return f(RowTile<4, 128, 1>{});
        return f(RowTile<4, 256, 1>{});
    }
    if (D <= 4) return f(RowTile<1, 4, 1>{});
    if (D <= 8) return f(RowTile<1, 8, 1>{});
    if (D <= 16) return f(RowTile<1, 16, 1>{});
    if (D <= 32) return f(RowTile<1, 32, 1>{});
    if (D <= 64) return f(RowTile<1, 32, 2>{});
    if (D <= 96) return f(RowTile<1, 32, 3>{});
    if (D <= 128) return f(RowTile<1, 32, 4>{});
    if (D <= 192) return f(RowTile<1, 64, 3>{});
    if (D <= 256) return f(RowTile<1, 64, 4>{});
    if (D <= 384) return f(RowTile<1, 128, 3>{});
    if (D <= 512) return f(RowTile<1, 128, 4>{});
    if (D <= 768) return f(RowTile<1, 256, 3>{});
    return f(RowTile<1, 256, 4>{});
}

}  // namespace drc
