// Residual block around a layer: norm behind it, gate, residual scale, residual sum and the norm in front of the next layer,
// one pass over the rows of a node type each way.
//
//   X_out = X + scale * sigmoid(G) * u,  u = yh * w_after + b_after,  yh = norm(Y);   N = xh * w_before + b_before,  xh = norm(X_out)
// Backward (r1, r2: the reciprocal deviations of X_out and Y):
//   g = dN * w_before;  d = dX_out + r1 * (g - [layer] mean(g) - xh * mean(g * xh));  dX = d
//   t = d * scale;  du = t * sig;  dG = t * u * sig * (1 - sig);  dscale = sum d * sig * u
//   g = du * w_after;  dY = r2 * (g - [layer] mean(g) - yh * mean(g * yh))
//   dw_after = sum du * yh, db_after = sum du, dw_before = sum dN * xh, db_before = sum dN          (sums over rows)
// A row stays in registers from its load to its stores; what bounds both passes is memory.
#include "act8.h"

#include <initializer_list>

namespace drc {

constexpr int kSums = 5;                       // dw_after, db_after, dscale, dw_before, db_before

// a parameter vector's elements of this lane; zeros past the width
template <typename T> __device__ __forceinline__ void vec_load(const float* p, const RowLane<T>& l, int D, float none, float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v)
#pragma unroll
        for (int j = 0; j < T::W; ++j) {
            const int c = l.col(v) + j;
            x[T::W * v + j] = c < D ? (p ? p[c] : none) : 0.f;
        }
}

// mean (0 for RMS) and reciprocal deviation of a row; elements past the width are zeros
template <typename T>
__device__ __forceinline__ void row_stats(const float (&x)[T::E], const RowLane<T>& l, RowSums& sums, int D, bool layer, float inv, float eps, float& m,
                                          float& r) {
    float s = 0.f;
    m = 0.f;
    if (layer) {
#pragma unroll
        for (int i = 0; i < T::E; ++i) s += x[i];
        m = sums.sum<T>(s) * inv;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            const float c = l.col(i / T::W) < D ? x[i] - m : 0.f;
            s = fmaf(c, c, s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < T::E; ++i) s = fmaf(x[i], x[i], s);
    }
    r = __builtin_amdgcn_rsqf(fmaf(sums.sum<T>(s), inv, eps));       // (off by an ulp at most)
}
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + expf(-g)); }

// Statistics are [n] or [n,2]: one load or store either way.
__device__ __forceinline__ Buf stats_view(const float* p, int64_t r0, int left, bool layer) { return rows_view(p, r0, left, layer ? 8 : 4); }
__device__ __forceinline__ void load_stats(Buf b, int row, bool layer, float& m, float& r) {
    if (layer) {
        const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, row * 8, 0, 0));
        m = of_bits(v[0]);
        r = of_bits(v[1]);
    } else {
        m = 0.f;
        r = of_bits(__builtin_amdgcn_raw_buffer_load_b32(b, row * 4, 0, 0));
    }
}
__device__ __forceinline__ void store_stats(Buf b, int row, bool first, bool layer, float m, float r) {
    if (layer) __builtin_amdgcn_raw_buffer_store_b64(u32x2{bits(m), bits(r)}, b, first ? row * 8 : kOutside, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(bits(r), b, first ? row * 4 : kOutside, 0, 0);
}

template <typename T> __device__ __forceinline__ void fill(uint32_t (&x)[T::E], uint32_t v) {
#pragma unroll
    for (int i = 0; i < T::E; ++i) x[i] = v;
}

// What a row brings, as it comes from memory: loaded a block of rows ahead.
template <typename T, bool GATED> struct FwdRow { uint32_t x[T::E], y[T::E], g[GATED ? T::E : 1]; };

// CKPT: checkpoints are kept (of any of the three tensors).
template <typename T, bool GATED, bool CKPT> __global__ __launch_bounds__(kRowThreads) void block_fwd_kernel(BlockFwd a) {
    __shared__ float sh[2][kRowThreads / kWave][2];
    RowSums sums{sh, 0};
    const int D = a.D, groups = act_groups(D);
    const RowLane<T> l(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER, full = a.b.gate_cols == D;
    const float inv = 1.0f / (float)D, eps = a.b.eps;
    float wa[T::E], ba[T::E], sc[T::E], wb[T::E], bb[T::E];
    vec_load<T>(a.b.w_after, l, D, 1.f, wa);
    vec_load<T>(a.b.b_after, l, D, 0.f, ba);
    vec_load<T>(a.b.scale, l, D, 1.f, sc);
    vec_load<T>(a.b.w_before, l, D, 1.f, wb);
    vec_load<T>(a.b.b_before, l, D, 0.f, bb);
    const int64_t end = CKPT ? (a.n + 7) & ~int64_t(7) : a.n, step = (int64_t)gridDim.x * T::R;
    const auto left_of = [&](int64_t r0) { return (int)(a.n - r0 < T::R ? (a.n > r0 ? a.n - r0 : 0) : T::R); };
    FwdRow<T, GATED> raw;
    const auto load = [&](int64_t r0) {
        const int left = left_of(r0);
        load_rows<T>(rows_view(a.X, r0, left, 4 * D), l, raw.x);
        load_rows<T>(rows_view(a.Y, r0, left, 4 * D), l, raw.y);
        if constexpr (GATED) {
            if (full) load_rows<T>(rows_view(a.G, r0, left, 4 * D), l, raw.g);
            else fill<T>(raw.g, __builtin_amdgcn_raw_buffer_load_b32(rows_view(a.G, r0, left, 4), l.row * 4, 0, 0));
        }
    };
    load((int64_t)blockIdx.x * T::R);
    for (int64_t r0 = (int64_t)blockIdx.x * T::R; r0 < end; r0 += step) {
        const int left = left_of(r0);
        const bool on = l.row < left;
        float x[T::E], y[T::E], g[T::E], m, r;
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            x[i] = of_bits(raw.x[i]);
            y[i] = of_bits(raw.y[i]);
            if constexpr (GATED) g[i] = of_bits(raw.g[i]);
        }
        load(r0 + step);
        if (a.Y) {
            row_stats<T>(y, l, sums, D, layer, inv, eps, m, r);
            store_stats(stats_view(a.saved.stats_after, r0, left, layer), l.row, l.t == 0, layer, m, r);
            if constexpr (CKPT) {
                if (a.saved.y.q) store_codes<T>(rows_view(a.saved.y.q, r0, left, D), scales_view(a.saved.y.scale, r0, a.n, groups), l, on, y);
                if constexpr (GATED)
                    if (a.saved.g.q) store_codes<T>(rows_view(a.saved.g.q, r0, left, D), scales_view(a.saved.g.scale, r0, a.n, groups), l, on, g);
            }
            if constexpr (GATED) {
                if (full) {
#pragma unroll
                    for (int i = 0; i < T::E; ++i) g[i] = sigmoid(g[i]);
                } else {
                    const float one = sigmoid(g[0]);
#pragma unroll
                    for (int i = 0; i < T::E; ++i) g[i] = one;
                }
            }
#pragma unroll
            for (int i = 0; i < T::E; ++i) x[i] = fmaf(GATED ? sc[i] * g[i] : sc[i], fmaf((y[i] - m) * r, wa[i], ba[i]), x[i]);
            store_rows<T>(rows_view(a.X_out, r0, left, 4 * D), l, x);
        }
        if constexpr (CKPT)
            if (a.saved.x.q) store_codes<T>(rows_view(a.saved.x.q, r0, left, D), scales_view(a.saved.x.scale, r0, a.n, groups), l, on, x);
        if (a.N) {
            row_stats<T>(x, l, sums, D, layer, inv, eps, m, r);
            store_stats(stats_view(a.saved.stats_before, r0, left, layer), l.row, l.t == 0, layer, m, r);
#pragma unroll
            for (int i = 0; i < T::E; ++i) x[i] = fmaf((x[i] - m) * r, wb[i], bb[i]);
            store_rows<T>(rows_view(a.N, r0, left, 4 * D), l, x);
        }
    }
}

// gradient of a norm's input from that of its result: r * (g - [layer] mean(g) - xh * mean(g * xh)), in place of g
template <typename T>
__device__ __forceinline__ void norm_back(float (&g)[T::E], const float (&xh)[T::E], RowSums& sums, float r, bool layer, float inv) {
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int i = 0; i < T::E; ++i) sx = fmaf(g[i], xh[i], sx);
    if (layer) {
#pragma unroll
        for (int i = 0; i < T::E; ++i) s += g[i];
        sums.sum<T>(s, sx);
        s *= inv;
    } else {
        sx = sums.sum<T>(sx);
    }
    sx *= inv;
#pragma unroll
    for (int i = 0; i < T::E; ++i) g[i] = r * fmaf(-xh[i], sx, g[i] - s);
}

// Columns past the width hold whatever the arithmetic makes of zeros: parameters are zeros there, so they add nothing to a row's sums, and
// they are neither stored nor part of the sums over rows.  Rows past the end are zeros throughout, their statistics among them.
template <typename T, bool GATED> struct BwdRow {
    uint32_t d[T::E], n[T::E], x[T::E], y[T::E], g[GATED ? T::E : 1], sx[T::V], sy[T::V], sg[T::V];
    float m1, r1, m2, r2;
};
template <typename T, bool GATED> __global__ __launch_bounds__(kRowThreads) void block_bwd_kernel(BlockBwd a) {
    __shared__ float sh[2][kRowThreads / kWave][2];
    __shared__ float all[T::R][T::LPR * T::E];
    RowSums sums{sh, 0};
    const int D = a.D, groups = act_groups(D);
    const RowLane<T> l(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER, full = a.b.gate_cols == D, after = a.Y || a.saved.y.q;
    const bool x8 = a.saved.x.q != nullptr, y8 = a.saved.y.q != nullptr, g8 = a.saved.g.q != nullptr;
    const float inv = 1.0f / (float)D;
    float wa[T::E], ba[T::E], sc[T::E], wb[T::E];
    vec_load<T>(a.b.w_after, l, D, 1.f, wa);
    vec_load<T>(a.b.b_after, l, D, 0.f, ba);
    vec_load<T>(a.b.scale, l, D, 1.f, sc);
    vec_load<T>(a.b.w_before, l, D, 1.f, wb);
    float sum[kSums][T::E];
#pragma unroll
    for (int p = 0; p < kSums; ++p)
#pragma unroll
        for (int i = 0; i < T::E; ++i) sum[p][i] = 0.f;
    const int64_t step = (int64_t)gridDim.x * T::R;
    const auto left_of = [&](int64_t r0) { return (int)(a.n - r0 < T::R ? (a.n > r0 ? a.n - r0 : 0) : T::R); };
    BwdRow<T, GATED> raw;
    // the same number of loads either way: the compiler counts how many may be outstanding
    const auto load_either = [&](bool eight, const float* f, const dr_act8& c, int64_t r0, int left, uint32_t (&x)[T::E], uint32_t (&s)[T::V]) {
        if (eight) {
            load_codes<T>(rows_view(c.q, r0, left, D), scales_view(c.scale, r0, a.n, groups), l, x, s);
        } else {
            load_rows<T>(rows_view(f, r0, left, 4 * D), l, x);
#pragma unroll
            for (int v = 0; v < T::V; ++v) s[v] = __builtin_amdgcn_raw_buffer_load_b8(buf_view(nullptr, 0), 0, 0, 0);
        }
    };
    const auto load = [&](int64_t r0) {
        const int left = left_of(r0);
        load_rows<T>(rows_view(a.dX_out, r0, left, 4 * D), l, raw.d);
        load_rows<T>(rows_view(a.dN, r0, left, 4 * D), l, raw.n);
        load_either(x8, a.X_out, a.saved.x, r0, left, raw.x, raw.sx);
        load_either(y8, a.Y, a.saved.y, r0, left, raw.y, raw.sy);
        load_stats(stats_view(a.saved.stats_before, r0, left, layer), l.row, layer, raw.m1, raw.r1);
        load_stats(stats_view(a.saved.stats_after, r0, left, layer), l.row, layer, raw.m2, raw.r2);
        if constexpr (GATED) {
            if (full) load_either(g8, a.G, a.saved.g, r0, left, raw.g, raw.sg);
            else fill<T>(raw.g, __builtin_amdgcn_raw_buffer_load_b32(rows_view(a.G, r0, left, 4), l.row * 4, 0, 0));
        }
    };
    load((int64_t)blockIdx.x * T::R);
    for (int64_t r0 = (int64_t)blockIdx.x * T::R; r0 < a.n; r0 += step) {
        const int left = left_of(r0);
        const bool on = l.row < left;
        float d[T::E], n[T::E], x[T::E], y[T::E], g[T::E];
        const auto values = [&](bool eight, const uint32_t (&from)[T::E], const uint32_t (&s)[T::V], float (&to)[T::E]) {
            if (eight) {
                decode<T>(from, s, on, to);
            } else {
#pragma unroll
                for (int i = 0; i < T::E; ++i) to[i] = of_bits(from[i]);
            }
        };
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            d[i] = of_bits(raw.d[i]);
            n[i] = of_bits(raw.n[i]);
        }
        values(x8, raw.x, raw.sx, x);
        values(y8, raw.y, raw.sy, y);
        if constexpr (GATED) {
            if (full) {
                values(g8, raw.g, raw.sg, g);
#pragma unroll
                for (int i = 0; i < T::E; ++i) g[i] = sigmoid(g[i]);
            } else {
                const float one = sigmoid(of_bits(raw.g[0]));
#pragma unroll
                for (int i = 0; i < T::E; ++i) g[i] = one;
            }
        }
        const float m1 = raw.m1, r1 = raw.r1, m2 = raw.m2, r2 = raw.r2;
        load(r0 + step);
        if (a.dN) {
#pragma unroll
            for (int i = 0; i < T::E; ++i) {
                x[i] = (x[i] - m1) * r1;
                sum[3][i] = fmaf(n[i], x[i], sum[3][i]);
                sum[4][i] += n[i];
                n[i] *= wb[i];
            }
            norm_back<T>(n, x, sums, r1, layer, inv);
#pragma unroll
            for (int i = 0; i < T::E; ++i) d[i] += n[i];
        }
        store_rows<T>(rows_view(a.grads.dX, r0, left, 4 * D), l, d);
        if (!after) continue;
        float dg[T::E], du[T::E], row = 0.f;
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            y[i] = (y[i] - m2) * r2;
            const float u = fmaf(y[i], wa[i], ba[i]), t = d[i] * sc[i];
            if constexpr (GATED) {
                const float dgate = d[i] * g[i];
                du[i] = t * g[i];
                dg[i] = du[i] * u * (1.0f - g[i]);
                sum[2][i] = fmaf(dgate, u, sum[2][i]);
            } else {
                du[i] = t;
                sum[2][i] = fmaf(d[i], u, sum[2][i]);
            }
            sum[0][i] = fmaf(du[i], y[i], sum[0][i]);
            sum[1][i] += du[i];
            du[i] *= wa[i];
        }
        if constexpr (GATED) {
            if (full) {
                store_rows<T>(rows_view(a.grads.dG, r0, left, 4 * D), l, dg);
            } else {
#pragma unroll
                for (int i = 0; i < T::E; ++i) row += dg[i];
                row = sums.sum<T>(row);
                __builtin_amdgcn_raw_buffer_store_b32(bits(row), rows_view(a.grads.dG, r0, left, 4), l.t == 0 ? l.row * 4 : kOutside, 0, 0);
            }
        }
        norm_back<T>(du, y, sums, r2, layer, inv);
        store_rows<T>(rows_view(a.grads.dY, r0, left, 4 * D), l, du);
    }
    float* const part = a.part + (size_t)blockIdx.x * kSums * D;
    for (int p = 0; p < kSums; ++p) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < T::V; ++v)
#pragma unroll
            for (int j = 0; j < T::W; ++j) all[l.row][l.col(v) + j] = sum[p][T::W * v + j];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += kRowThreads) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < T::R; ++k) s += all[k][c];
            part[(size_t)p * D + c] = s;
        }
    }
}

// The five sums over the workgroups' partials, in 64 bits and a fixed order: a wavefront sums every sixteenth partial of 64 columns, the
// sixteen sums are added in order.
constexpr int kSumWaves = 16, kSumAhead = 8;
__global__ __launch_bounds__(kWave* kSumWaves) void block_sums_kernel(const float* part, int parts, int D, dr_block_grads g) {
    __shared__ double sh[kSumWaves][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, count = kSums * D, i = blockIdx.x * kWave + lane;
    const float* const src = part + min(i, count - 1);
    double s = 0.0;
    int p = wave;
    for (; p + (kSumAhead - 1) * kSumWaves < parts; p += kSumAhead * kSumWaves) {
        float v[kSumAhead];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) v[u] = src[(size_t)(p + u * kSumWaves) * count];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) s += (double)v[u];
    }
    for (; p < parts; p += kSumWaves) s += (double)src[(size_t)p * count];
    sh[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || i >= count) return;
    float* const to[kSums] = {g.dw_after, g.db_after, g.dscale, g.dw_before, g.db_before};
    float* const o = to[i / D];
    if (!o) return;
    s = sh[0][lane];
#pragma unroll
    for (int w = 1; w < kSumWaves; ++w) s += sh[w][lane];
    o[i % D] = (float)s;
}

constexpr int kFwdWgs = 2048, kBwdWgs = 1024;
static bool vector_rows(int D, std::initializer_list<const void*> f32, std::initializer_list<const void*> q) {
    bool v = D % 4 == 0;
    for (const void* p : f32) v = v && aligned(p, 16);
    for (const void* p : q) v = v && aligned(p, 4);
    return v;
}

int launch_block_fwd(const BlockFwd& a, hipStream_t s) {
    const bool vector = vector_rows(a.D, {a.X, a.Y, a.b.gate_cols == a.D ? a.G : nullptr, a.X_out, a.N}, {a.saved.x.q, a.saved.y.q, a.saved.g.q});
    const bool ckpt = a.saved.x.q || a.saved.y.q || a.saved.g.q;
    return with_row_tile(a.D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        const int64_t rows = ckpt ? (a.n + 7) / 8 * 8 : a.n, blocks = (rows + T::R - 1) / T::R;
        const dim3 grid((unsigned)(blocks < kFwdWgs ? blocks : kFwdWgs));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRowThreads), 0, s, a); };
        if (a.G) {
            if (ckpt) go(block_fwd_kernel<T, true, true>);
            else go(block_fwd_kernel<T, true, false>);
        } else {
            if (ckpt) go(block_fwd_kernel<T, false, true>);
            else go(block_fwd_kernel<T, false, false>);
        }
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

size_t block_bwd_workspace(int64_t n, int D) {
    const int64_t most = n < kBwdWgs ? n : kBwdWgs;          // a workgroup takes a row at least
    return sizeof(float) * (size_t)(most < 1 ? 1 : most) * kSums * D;
}

int launch_block_bwd(BlockBwd a, void* ws, hipStream_t s) {
    const bool full = a.b.gate_cols == a.D;
    const bool vector = vector_rows(a.D, {a.dX_out, a.dN, a.X_out, a.Y, full ? a.G : nullptr, a.grads.dX, a.grads.dY, full ? a.grads.dG : nullptr},
                                    {a.saved.x.q, a.saved.y.q, a.saved.g.q});
    a.part = static_cast<float*>(ws);
    a.parts = 0;
    if (a.n > 0)
        DRC_TRY(with_row_tile(a.D, vector, [&](auto tile) -> int {
            using T = decltype(tile);
            const int64_t blocks = (a.n + T::R - 1) / T::R;
            a.parts = (int)(blocks < kBwdWgs ? blocks : kBwdWgs);
            auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)a.parts), dim3(kRowThreads), 0, s, a); };
            if (a.b.gate_cols) go(block_bwd_kernel<T, true>);
            else go(block_bwd_kernel<T, false>);
            DRC_HIP(hipGetLastError());
            return DR_OK;
        }));
    const dr_block_grads& g = a.grads;
    if (g.dw_after || g.db_after || g.dscale || g.dw_before || g.db_before) {
        hipLaunchKernelGGL(block_sums_kernel, dim3((unsigned)((kSums * a.D + kWave - 1) / kWave)), dim3(kWave * kSumWaves), 0, s, a.part, a.parts, a.D, g);
        DRC_HIP(hipGetLastError());
    }
    return DR_OK;
}

}  // namespace drc
