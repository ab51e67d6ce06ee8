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

constexpr int kBlockThreads = 256;
constexpr int kSums = 5;                       // dw_after, db_after, dscale, dw_before, db_before

template <typename T> __device__ __forceinline__ void vec_load(const float* __restrict__ p, int t, int D, float none, float (&x)[T::E]) {
#pragma unroll
    for (int v = 0; v < T::V; ++v)
#pragma unroll
        for (int j = 0; j < T::W; ++j) {
            const int c = tile_col<T>(t, v) + j;
            x[T::W * v + j] = c < D ? (p ? p[c] : none) : 0.f;
        }
}

// mean (0 for RMS) and reciprocal deviation of a row
template <typename T> __device__ __forceinline__ void row_stats(const float (&x)[T::E], int t, int D, bool layer, float eps, float& m, float& r) {
    const float inv = 1.0f / (float)D;
    m = 0.f;
    float s = 0.f;
    if (layer) {
#pragma unroll
        for (int i = 0; i < T::E; ++i) s += x[i];
        m = lane_sum<T::LPR>(s) * inv;
        s = 0.f;
    }
#pragma unroll
    for (int i = 0; i < T::E; ++i) {
        const bool in = tile_col<T>(t, i / T::W) < D;
        const float c = in ? x[i] - m : 0.f;
        s = fmaf(c, c, s);
    }
    r = 1.0f / sqrtf(lane_sum<T::LPR>(s) * inv + eps);
}
__device__ __forceinline__ void put_stats(float* p, int64_t row, bool layer, float m, float r) {
    if (layer) { p[2 * row] = m; p[2 * row + 1] = r; }
    else p[row] = r;
}
__device__ __forceinline__ void get_stats(const float* p, int64_t row, bool layer, float& m, float& r) {
    m = layer ? p[2 * row] : 0.f;
    r = layer ? p[2 * row + 1] : p[row];
}
__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + expf(-g)); }

template <typename T> __global__ __launch_bounds__(kBlockThreads) void block_fwd_kernel(BlockFwd a) {
    constexpr int R = kBlockThreads / T::LPR;
    const int t = threadIdx.x % T::LPR, D = a.D, groups = act_groups(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER;
    float wa[T::E], ba[T::E], sc[T::E], wb[T::E], bb[T::E];
    vec_load<T>(a.b.w_after, t, D, 1.f, wa);
    vec_load<T>(a.b.b_after, t, D, 0.f, ba);
    vec_load<T>(a.b.scale, t, D, 1.f, sc);
    vec_load<T>(a.b.w_before, t, D, 1.f, wb);
    vec_load<T>(a.b.b_before, t, D, 0.f, bb);
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.n; r0 += (int64_t)gridDim.x * R) {
        const int64_t row = r0 + threadIdx.x / T::LPR;
        const bool on = row < a.n;
        const size_t at = (size_t)row * D;
        float x[T::E];
        row_load<T>(a.X + at, t, D, on, x);
        if (a.Y) {
            float y[T::E], m, r;
            row_load<T>(a.Y + at, t, D, on, y);
            row_stats<T>(y, t, D, layer, a.b.eps, m, r);
            if (a.saved.y.q) row_pack<T>(a.saved.y.q, a.saved.y.scale, row, a.n, t, D, groups, on, y);
            if (on && t == 0 && a.saved.stats_after) put_stats(a.saved.stats_after, row, layer, m, r);
            float g[T::E];
            if (a.b.gate_cols == 0) {
#pragma unroll
                for (int i = 0; i < T::E; ++i) g[i] = 1.f;
            } else if (a.b.gate_cols == D) {
                row_load<T>(a.G + at, t, D, on, g);
                if (a.saved.g.q) row_pack<T>(a.saved.g.q, a.saved.g.scale, row, a.n, t, D, groups, on, g);
#pragma unroll
                for (int i = 0; i < T::E; ++i) g[i] = sigmoid(g[i]);
            } else {
                const float one = on ? sigmoid(a.G[row]) : 0.f;
#pragma unroll
                for (int i = 0; i < T::E; ++i) g[i] = one;
            }
#pragma unroll
            for (int i = 0; i < T::E; ++i) x[i] = fmaf(sc[i] * g[i], fmaf((y[i] - m) * r, wa[i], ba[i]), x[i]);
            row_store<T>(a.X_out + at, t, D, on, x);
        }
        if (a.saved.x.q) row_pack<T>(a.saved.x.q, a.saved.x.scale, row, a.n, t, D, groups, on, x);
        if (a.N) {
            float m, r;
            row_stats<T>(x, t, D, layer, a.b.eps, m, r);
            if (on && t == 0 && a.saved.stats_before) put_stats(a.saved.stats_before, row, layer, m, r);
#pragma unroll
            for (int i = 0; i < T::E; ++i) x[i] = fmaf((x[i] - m) * r, wb[i], bb[i]);
            row_store<T>(a.N + at, t, D, on, x);
        }
    }
}

// gradient of a norm's input from that of its result: r * (g - [layer] mean(g) - xh * mean(g * xh)), in place of g
template <typename T> __device__ __forceinline__ void norm_back(float (&g)[T::E], const float (&xh)[T::E], float r, bool layer, float inv) {
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int i = 0; i < T::E; ++i) {
        s += g[i];
        sx = fmaf(g[i], xh[i], sx);
    }
    sx = lane_sum<T::LPR>(sx) * inv;
    s = layer ? lane_sum<T::LPR>(s) * inv : 0.f;
#pragma unroll
    for (int i = 0; i < T::E; ++i) g[i] = r * (g[i] - s - xh[i] * sx);
}

template <typename T> __global__ __launch_bounds__(kBlockThreads) void block_bwd_kernel(BlockBwd a) {
    constexpr int R = kBlockThreads / T::LPR;
    __shared__ float sh[R][T::LPR * T::E];
    const int t = threadIdx.x % T::LPR, D = a.D, groups = act_groups(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER, after = a.Y || a.saved.y.q;
    const float inv = 1.0f / (float)D;
    float wa[T::E], ba[T::E], sc[T::E], wb[T::E];
    vec_load<T>(a.b.w_after, t, D, 1.f, wa);
    vec_load<T>(a.b.b_after, t, D, 0.f, ba);
    vec_load<T>(a.b.scale, t, D, 1.f, sc);
    vec_load<T>(a.b.w_before, t, D, 1.f, wb);
    float sum[kSums][T::E];
#pragma unroll
    for (int p = 0; p < kSums; ++p)
#pragma unroll
        for (int i = 0; i < T::E; ++i) sum[p][i] = 0.f;
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.n; r0 += (int64_t)gridDim.x * R) {
        const int64_t row = r0 + threadIdx.x / T::LPR;
        const bool on = row < a.n;
        const size_t at = (size_t)row * D;
        float d[T::E];
        if (a.dX_out) {
            row_load<T>(a.dX_out + at, t, D, on, d);
        } else {
#pragma unroll
            for (int i = 0; i < T::E; ++i) d[i] = 0.f;
        }
        if (a.dN) {
            float g[T::E], x[T::E], m = 0.f, r = 0.f;
            row_load<T>(a.dN + at, t, D, on, g);
            if (a.X_out) row_load<T>(a.X_out + at, t, D, on, x);
            else row_unpack<T>(a.saved.x.q, a.saved.x.scale, row, t, D, groups, on, x);
            if (on) get_stats(a.saved.stats_before, row, layer, m, r);
#pragma unroll
            for (int i = 0; i < T::E; ++i) {
                x[i] = tile_col<T>(t, i / T::W) < D ? (x[i] - m) * r : 0.f;
                sum[3][i] = fmaf(g[i], x[i], sum[3][i]);
                sum[4][i] += g[i];
                g[i] *= wb[i];
            }
            norm_back<T>(g, x, r, layer, inv);
#pragma unroll
            for (int i = 0; i < T::E; ++i) d[i] += g[i];
        }
        if (!after) {
            if (a.grads.dX) row_store<T>(a.grads.dX + at, t, D, on, d);
            continue;
        }
        float y[T::E], g[T::E], m = 0.f, r = 0.f;
        if (a.Y) row_load<T>(a.Y + at, t, D, on, y);
        else row_unpack<T>(a.saved.y.q, a.saved.y.scale, row, t, D, groups, on, y);
        if (on) get_stats(a.saved.stats_after, row, layer, m, r);
        if (a.b.gate_cols == 0) {
#pragma unroll
            for (int i = 0; i < T::E; ++i) g[i] = 1.f;
        } else if (a.b.gate_cols == D) {
            if (a.G) row_load<T>(a.G + at, t, D, on, g);
            else row_unpack<T>(a.saved.g.q, a.saved.g.scale, row, t, D, groups, on, g);
#pragma unroll
            for (int i = 0; i < T::E; ++i) g[i] = sigmoid(g[i]);
        } else {
            const float one = on ? sigmoid(a.G[row]) : 0.f;
#pragma unroll
            for (int i = 0; i < T::E; ++i) g[i] = one;
        }
        float dg[T::E], du[T::E], all = 0.f;
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            const bool in = on && tile_col<T>(t, i / T::W) < D;
            y[i] = in ? (y[i] - m) * r : 0.f;
            const float u = fmaf(y[i], wa[i], ba[i]), tt = d[i] * sc[i];
            du[i] = in ? tt * g[i] : 0.f;
            dg[i] = in ? tt * u * g[i] * (1.0f - g[i]) : 0.f;
            all += dg[i];
            sum[0][i] = fmaf(du[i], y[i], sum[0][i]);
            sum[1][i] += du[i];
            sum[2][i] += in ? d[i] * g[i] * u : 0.f;
            du[i] *= wa[i];
        }
        if (a.grads.dG) {
            if (a.b.gate_cols == D) {
                row_store<T>(a.grads.dG + at, t, D, on, dg);
            } else {
                all = lane_sum<T::LPR>(all);
                if (on && t == 0) a.grads.dG[row] = all;
            }
        }
        norm_back<T>(du, y, r, layer, inv);
        if (a.grads.dX) row_store<T>(a.grads.dX + at, t, D, on, d);       // (the rows that were read may be those that are written)
        if (a.grads.dY) row_store<T>(a.grads.dY + at, t, D, on, du);
    }
    for (int p = 0; p < kSums; ++p) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < T::V; ++v)
#pragma unroll
            for (int j = 0; j < T::W; ++j) sh[threadIdx.x / T::LPR][tile_col<T>(t, v) + j] = sum[p][T::W * v + j];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += kBlockThreads) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < R; ++k) s += sh[k][c];
            a.part[((size_t)blockIdx.x * kSums + p) * D + c] = s;
        }
    }
}

// the five sums over the workgroups' partials, in 64 bits and a fixed order
__global__ __launch_bounds__(256) void block_sums_kernel(const float* __restrict__ part, int parts, int D, dr_block_grads g) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= kSums * D) return;
    float* const to[kSums] = {g.dw_after, g.db_after, g.dscale, g.dw_before, g.db_before};
    float* const o = to[i / D];
    if (!o) return;
    double s = 0.0;
    for (int p = 0; p < parts; ++p) s += (double)part[(size_t)p * kSums * D + i];
    o[i % D] = (float)s;
}

constexpr int kBwdWgs = 1024;
static bool vector_rows(int D, std::initializer_list<const void*> f32, std::initializer_list<const void*> q) {
    bool v = D % 4 == 0;
    for (const void* p : f32) v = v && aligned(p, 16);
    for (const void* p : q) v = v && aligned(p, 4);
    return v;
}

int launch_block_fwd(const BlockFwd& a, hipStream_t s) {
    const bool vector = vector_rows(a.D, {a.X, a.Y, a.b.gate_cols == a.D ? a.G : nullptr, a.X_out, a.N}, {a.saved.x.q, a.saved.y.q, a.saved.g.q});
    return with_row_tile(a.D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        constexpr int R = kBlockThreads / T::LPR;
        const int64_t blocks = (a.n + R - 1) / R;
        hipLaunchKernelGGL((block_fwd_kernel<T>), dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kBlockThreads), 0, s, a);
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
            constexpr int R = kBlockThreads / T::LPR;
            const int64_t blocks = (a.n + R - 1) / R;
            a.parts = (int)(blocks < kBwdWgs ? blocks : kBwdWgs);
            hipLaunchKernelGGL((block_bwd_kernel<T>), dim3((unsigned)a.parts), dim3(kBlockThreads), 0, s, a);
            DRC_HIP(hipGetLastError());
            return DR_OK;
        }));
    const dr_block_grads& g = a.grads;
    if (g.dw_after || g.db_after || g.dscale || g.dw_before || g.db_before) {
        hipLaunchKernelGGL(block_sums_kernel, dim3((unsigned)((kSums * a.D + 255) / 256)), dim3(256), 0, s, a.part, a.parts, a.D, g);
        DRC_HIP(hipGetLastError());
    }
    return DR_OK;
}

}  // namespace drc
