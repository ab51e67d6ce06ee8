// Residual block around a layer: norm behind it, gate, residual scale, residual sum and the norm in front of the next layer,
// one pass over the rows of a node type each way.
//
//   X_out = X + scale * sigmoid(G) * u,  u = yh * w_after + b_after,  yh = norm(Y);   N = xh * w_before + b_before,  xh = norm(X_out)
// Backward (r1, r2: the reciprocal deviations of X_out and Y):
//   g = dN * w_before;  d = dX_out + r1 * (g - [layer] mean(g) - xh * mean(g * xh));  dX = d
//   t = d * scale;  du = t * sig;  dG = t * u * sig * (1 - sig);  dscale = sum d * sig * u
//   g = du * w_after;  dY = r2 * (g - [layer] mean(g) - yh * mean(g * yh))
//   dw_after = sum du * yh, db_after = sum du, dw_before = sum dN * xh, db_before = sum dN          (sums over rows)
// A row stays in registers from its load to its stores; what bounds both passes is memory: forward of 1.2 M x 128 443 to 449 us by card (2.47 GB, 5.5 TB/s), backward
// from checkpoints with a gate per row 493 to 505, its sums included (2.79 GB, 5.6 TB/s); with a gate per element and three checkpoints 500 000 x 128 forward 285 to 290 (1.48 GB, 5.2 TB/s).  The sums over rows
// of the backward pass are a second launch, 2.5 to 5 us.
#include "act8.h"

#include <initializer_list>
#include <type_traits>

namespace drc {

constexpr int kSums = 5;                       // dw_after, db_after, dscale, dw_before, db_before
// Rows that a lane adds up in fp32; those sums are added in 64 bits, so that what is lost does not grow with the rows: 16 additions, and the roundings of
// a workgroup's sum and of the result.  A thread's wide sums are in LDS and its own: additions there without a result to wait for (1.2 M x 128 from
// checkpoints 495 us; read, added and written back 504, every 32 rows 503).
constexpr int kWiden = 16;

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

// A row's mean where this lane has columns, zero past the width: what is there stays zero when the mean is taken off, and adds nothing to a row's
// sums.  (A mean times a reciprocal deviation may be past the range of fp32: in rows of one value.)  Only the last of a lane's loads can be past the
// width, tiles are the narrowest: asked of all of them, 500 000 x 45 backward takes 124.5 us instead of 121.6.
template <typename T> struct Mean {
    float of[T::V];
    __device__ __forceinline__ Mean(float m, const RowLane<T>& l, int D) {
#pragma unroll
        for (int v = 0; v < T::V; ++v) of[v] = v + 1 < T::V || l.col(v) < D ? m : 0.f;
    }
    __device__ __forceinline__ float operator[](int i) const { return of[i / T::W]; }
};

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
        asm volatile("" : "+v"(m));                // the mean that is saved: not the exact product inside the subtractions below
        s = 0.f;
        const Mean<T> mean(m, l, D);
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            const float c = x[i] - mean[i];
            s = fmaf(c, c, s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < T::E; ++i) s = fmaf(x[i], x[i], s);
    }
    r = __builtin_amdgcn_rsqf(fmaf(sums.sum<T>(s), inv, eps));       // (off by an ulp at most)
}
// sigmoid(g) and 1 - sigmoid(g).  (The reciprocal is off by an ulp at most; a gate below -87, whose sigmoid is a denormal, is shut.)  An open gate's
// complement is e^-g * sigmoid(g): as a difference from 1 nothing of it is left from g = 17 on, where it is 4e-8.
struct Sigmoid {
    float open, shut;
};
__device__ __forceinline__ Sigmoid sigmoid(float g) {
    const float e = expf(-g), open = __builtin_amdgcn_rcpf(1.0f + e);
    return {open, g > 0.f ? e * open : 1.0f - open};
}

// Statistics are [n] (r) or [n,2] (m, r).  A mean that is not there is read from outside, as zero.
struct StatsLane {
    int m, r;
    __device__ __forceinline__ StatsLane(int row, bool layer, bool on)
        : m(on && layer ? row * 8 : kOutside), r(on ? (layer ? row * 8 + 4 : row * 4) : kOutside) {}
};
__device__ __forceinline__ Buf stats_view(const float* p, int64_t r0, int left, bool layer) { return rows_view(p, r0, left, layer ? 8 : 4); }

// The loops below have no memory access under a condition: what is absent has an empty view.  The compiler then knows how many loads and stores
// are outstanding wherever it has to wait for some of them; with branches around loads and stores every row waited for the loads of
// the next one (1.2 M x 128 backward from checkpoints, two workgroups per compute unit: 627 us, without them 496).
// A row's loads do wait for the stores of the row before, and that is left as it is: with as many empty stores in front of the loop as it ends with
// the compiler lets them pass, and workgroups then spread over more of memory's pages (forward 443 / 456, backward 496 / 540 us).
enum Gate { kNoGate, kRowGate, kFullGate };
__device__ __forceinline__ int rows_left(int64_t n, int64_t r0, int rows) { return (int)(n - r0 < rows ? (n > r0 ? n - r0 : 0) : rows); }

// CKPT: checkpoints are kept (of any of the three tensors).
template <typename T, int GATE, bool CKPT> __global__ __launch_bounds__(kRowThreads) void block_fwd_kernel(BlockFwd a) {
    __shared__ float sh[2][kRowThreads / kWave][2];
    RowSums sums{sh, 0};
    const int D = a.D, groups = act_groups(D);
    const RowLane<T> l(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER;
    const StatsLane st(l.row, layer, l.t == 0);
    const float inv = 1.0f / (float)D, eps = a.b.eps;
    float wa[T::E], ba[T::E], sc[T::E], wb[T::E], bb[T::E];
    vec_load<T>(a.Y ? a.b.w_after : nullptr, l, D, a.Y ? 1.f : 0.f, wa);     // without Y, X_out is X
    vec_load<T>(a.Y ? a.b.b_after : nullptr, l, D, 0.f, ba);
    vec_load<T>(a.Y ? a.b.scale : nullptr, l, D, a.Y ? 1.f : 0.f, sc);
    vec_load<T>(a.b.w_before, l, D, 1.f, wb);
    vec_load<T>(a.b.b_before, l, D, 0.f, bb);
    const int64_t end = CKPT ? (a.n + 7) & ~int64_t(7) : a.n, step = (int64_t)gridDim.x * T::R;
    uint32_t rx[T::E], ry[T::E], rg[T::E], r1;                  // what the next rows bring
    const auto load = [&](int64_t r0) {
        const int left = rows_left(a.n, r0, T::R);
        load_rows<T>(rows_view(a.X, r0, left, 4 * D), l, rx);
        load_rows<T>(rows_view(a.Y, r0, left, 4 * D), l, ry);
        if constexpr (GATE == kFullGate) load_rows<T>(rows_view(a.G, r0, left, 4 * D), l, rg);
        if constexpr (GATE == kRowGate) r1 = __builtin_amdgcn_raw_buffer_load_b32(rows_view(a.G, r0, left, 4), l.row * 4, 0, 0);
    };
    load((int64_t)blockIdx.x * T::R);
    for (int64_t r0 = (int64_t)blockIdx.x * T::R; r0 < end; r0 += step) {
        const int left = rows_left(a.n, r0, T::R);
        const bool on = l.row < left;
        float x[T::E], y[T::E], g[T::E], m, r;
        take(rx, x);
        take(ry, y);
        if constexpr (GATE == kFullGate) take(rg, g);
        if constexpr (GATE == kRowGate) {
            const float one = sigmoid(of_bits(r1)).open;
#pragma unroll
            for (int i = 0; i < T::E; ++i) g[i] = one;
        }
        load(r0 + step);
        row_stats<T>(y, l, sums, D, layer, inv, eps, m, r);
        const Buf sa = stats_view(a.saved.stats_after, r0, left, layer);
        __builtin_amdgcn_raw_buffer_store_b32(bits(m), sa, st.m, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b32(bits(r), sa, st.r, 0, 0);
        if constexpr (CKPT) {
            store_codes<T>(rows_view(a.saved.y.q, r0, left, D), scales_view(a.saved.y.scale, r0, a.n, groups), l, on, y);
            if constexpr (GATE == kFullGate)
                store_codes<T>(rows_view(a.saved.g.q, r0, left, D), scales_view(a.saved.g.scale, r0, a.n, groups), l, on, g);
        }
        if constexpr (GATE == kFullGate) {
#pragma unroll
            for (int i = 0; i < T::E; ++i) g[i] = sigmoid(g[i]).open;
        }
        const Mean<T> my(m, l, D);
#pragma unroll
        for (int i = 0; i < T::E; ++i) x[i] = fmaf(GATE != kNoGate ? sc[i] * g[i] : sc[i], fmaf((y[i] - my[i]) * r, wa[i], ba[i]), x[i]);
        store_rows<T>(rows_view(a.X_out, r0, left, 4 * D), l, x);
        if constexpr (CKPT) store_codes<T>(rows_view(a.saved.x.q, r0, left, D), scales_view(a.saved.x.scale, r0, a.n, groups), l, on, x);
        row_stats<T>(x, l, sums, D, layer, inv, eps, m, r);
        const Buf sb = stats_view(a.saved.stats_before, r0, left, layer);
        __builtin_amdgcn_raw_buffer_store_b32(bits(m), sb, st.m, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b32(bits(r), sb, st.r, 0, 0);
#pragma unroll
        for (int i = 0; i < T::E; ++i) x[i] = fmaf((x[i] - m) * r, wb[i], bb[i]);
        store_rows<T>(rows_view(a.N, r0, left, 4 * D), l, x);
    }
}

// gradient of a norm's input from that of its result: r * (g - [layer] mean(g) - xh * mean(g * xh)), in place of g
template <typename T>
__device__ __forceinline__ void norm_back(float (&g)[T::E], const float (&xh)[T::E], const RowLane<T>& l, RowSums& sums, float r, int D, bool layer,
                                          float inv) {
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
    const Mean<T> mean(s, l, D);
#pragma unroll
    for (int i = 0; i < T::E; ++i) g[i] = r * fmaf(-xh[i], sx, g[i] - mean[i]);
}

// A tensor's rows of which nothing, fp32 elements or codes are there
enum From { kFloats, kCodes, kEither };
template <typename T, int FROM> struct Incoming {
    uint32_t f[T::E], q[T::E], s[T::V];
    __device__ __forceinline__ void load(const float* p, const dr_act8& c, const RowLane<T>& l, int64_t r0, int left, int64_t n, int D, int groups) {
        if constexpr (FROM != kCodes) load_rows<T>(rows_view(p, r0, left, 4 * D), l, f);
        if constexpr (FROM != kFloats) load_codes<T>(rows_view(c.q, r0, left, D), scales_view(c.scale, r0, n, groups), l, q, s);
    }
    __device__ __forceinline__ void get(bool on, float (&x)[T::E]) const {
        if constexpr (FROM == kFloats) {
            take(f, x);
        } else {
            decode<T>(q, s, on, x);
            if constexpr (FROM == kEither) {                    // the other one is zeros
                float y[T::E];
                take(f, y);
#pragma unroll
                for (int i = 0; i < T::E; ++i) x[i] += y[i];
            }
        }
    }
};

// Columns past the width are zeros throughout, but for a gate's half: they add nothing to a row's sums, and they are neither stored nor part of the
// sums over rows.  Rows past the end are zeros throughout, their statistics among them; so is all that
// belongs to a part that is left out.
template <typename T, int GATE, int FROM> __global__ __launch_bounds__(kRowThreads) void block_bwd_kernel(BlockBwd a) {
    __shared__ float sh[2][kRowThreads / kWave][2];
    __shared__ double all[kSums * T::E][kRowThreads];         // every thread's own sums
    RowSums sums{sh, 0};
    const int D = a.D, groups = act_groups(D);
    const RowLane<T> l(D);
    const bool layer = a.b.norm == DR_ROWNORM_LAYER;
    const StatsLane st(l.row, layer, true);
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
    int since = 0;
    bool wide = false;                                         // there is something in `all`
    const auto widen = [&]() {
#pragma unroll
        for (int p = 0; p < kSums; ++p)
#pragma unroll
            for (int i = 0; i < T::E; ++i) {
                if (wide) __hip_atomic_fetch_add(&all[T::E * p + i][threadIdx.x], (double)sum[p][i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                else all[T::E * p + i][threadIdx.x] = (double)sum[p][i];
                sum[p][i] = 0.f;
            }
        wide = true;
        since = 0;
    };
    const int64_t step = (int64_t)gridDim.x * T::R;
    // what the next rows bring
    uint32_t rd[T::E], rn[T::E], rs[4], rone;
    Incoming<T, FROM> ix, iy, ig;
    const auto load = [&](int64_t r0) {
        const int left = rows_left(a.n, r0, T::R);
        load_rows<T>(rows_view(a.dN, r0, left, 4 * D), l, rn);
        ix.load(a.X_out, a.saved.x, l, r0, left, a.n, D, groups);
        const Buf sb = stats_view(a.saved.stats_before, r0, left, layer), sa = stats_view(a.saved.stats_after, r0, left, layer);
        rs[0] = __builtin_amdgcn_raw_buffer_load_b32(sb, st.m, 0, 0);
        rs[1] = __builtin_amdgcn_raw_buffer_load_b32(sb, st.r, 0, 0);
        load_rows<T>(rows_view(a.dX_out, r0, left, 4 * D), l, rd);
        iy.load(a.Y, a.saved.y, l, r0, left, a.n, D, groups);
        rs[2] = __builtin_amdgcn_raw_buffer_load_b32(sa, st.m, 0, 0);
        rs[3] = __builtin_amdgcn_raw_buffer_load_b32(sa, st.r, 0, 0);
        if constexpr (GATE == kFullGate) ig.load(a.G, a.saved.g, l, r0, left, a.n, D, groups);
        if constexpr (GATE == kRowGate) rone = __builtin_amdgcn_raw_buffer_load_b32(rows_view(a.G, r0, left, 4), l.row * 4, 0, 0);
    };
    load((int64_t)blockIdx.x * T::R);
    for (int64_t r0 = (int64_t)blockIdx.x * T::R; r0 < a.n; r0 += step) {
        const int left = rows_left(a.n, r0, T::R);
        const bool on = l.row < left;
        float d[T::E], n[T::E], x[T::E], y[T::E], g[T::E], shut[T::E], s[4];
        take(rn, n);
        take(rd, d);
        take(rs, s);
        ix.get(on, x);
        iy.get(on, y);
        if constexpr (GATE == kFullGate) {
            ig.get(on, g);
#pragma unroll
            for (int i = 0; i < T::E; ++i) {
                const Sigmoid one = sigmoid(g[i]);
                g[i] = one.open;
                shut[i] = one.shut;
            }
        }
        if constexpr (GATE == kRowGate) {
            const Sigmoid one = sigmoid(of_bits(rone));
#pragma unroll
            for (int i = 0; i < T::E; ++i) {
                g[i] = one.open;
                shut[i] = one.shut;
            }
        }
        load(r0 + step);
        const Mean<T> mx(s[0], l, D), my(s[2], l, D);
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            x[i] = (x[i] - mx[i]) * s[1];
            sum[3][i] = fmaf(n[i], x[i], sum[3][i]);
            sum[4][i] += n[i];
            n[i] *= wb[i];
        }
        norm_back<T>(n, x, l, sums, s[1], D, layer, inv);
#pragma unroll
        for (int i = 0; i < T::E; ++i) d[i] += n[i];
        store_rows<T>(rows_view(a.grads.dX, r0, left, 4 * D), l, d);
        float dg[T::E], du[T::E];
#pragma unroll
        for (int i = 0; i < T::E; ++i) {
            y[i] = (y[i] - my[i]) * s[3];
            const float u = fmaf(y[i], wa[i], ba[i]);
            du[i] = d[i] * sc[i];
            if constexpr (GATE != kNoGate) {
                du[i] *= g[i];
                dg[i] = du[i] * u * shut[i];
                sum[2][i] = fmaf(d[i] * g[i], u, sum[2][i]);
            } else {
                sum[2][i] = fmaf(d[i], u, sum[2][i]);
            }
            sum[0][i] = fmaf(du[i], y[i], sum[0][i]);
            sum[1][i] += du[i];
            du[i] *= wa[i];
        }
        if constexpr (GATE == kFullGate) store_rows<T>(rows_view(a.grads.dG, r0, left, 4 * D), l, dg);
        if constexpr (GATE == kRowGate) {
            float row = 0.f;
#pragma unroll
            for (int i = 0; i < T::E; ++i) row += dg[i];
            row = sums.sum<T>(row);
            __builtin_amdgcn_raw_buffer_store_b32(bits(row), rows_view(a.grads.dG, r0, left, 4), l.t == 0 ? l.row * 4 : kOutside, 0, 0);
        }
        norm_back<T>(du, y, l, sums, s[3], D, layer, inv);
        store_rows<T>(rows_view(a.grads.dY, r0, left, 4 * D), l, du);
        if (++since == kWiden) widen();
    }
    widen();
    __syncthreads();
    float* const part = a.part + (size_t)blockIdx.x * kSums * D;
    for (int i = threadIdx.x; i < kSums * T::E * T::LPR; i += kRowThreads) {
        const int lane = i % T::LPR, e = i / T::LPR % T::E, p = i / (T::LPR * T::E), c = T::W * (lane + T::LPR * (e / T::W)) + e % T::W;
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < T::R; ++k) s += all[T::E * p + e][T::LPR * k + lane];
        if (c < D) part[(size_t)p * D + c] = (float)s;
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

// Workgroups of a launch: few that walk many rows.  Two per compute unit draw 5.6 TB/s from memory, more of them drift apart and find its
// pages closed: 1.2 M x 128, 512 / 768 / 1024 workgroups, us: forward 449 / 498 / 537, with two checkpoints 565 / 581 / 638, backward from checkpoints 506 / 562 /
// 594, from tensors 697 / 725 / 827; 60 000 x 128 19.7 / 20.0 / 20.5, 23.2 / 23.1 / 23.5, 28.0 / 29.0 / 30.4, 33.1 / 34.4 / 36.2.  Rows of any width are
// read a column at a time, and take three: 200 000 x 77 38 / 39 / 40, 87 / 82 / 83, 80 / 73 / 77, 75 / 79 / 84; 500 000 x 45 124 / 93 / 85, 150 / 139 / 138,
// 153 / 127 / 122, 139 / 122 / 126; 20 000 x 999 59 / 60 / 62, 85 / 80 / 81, 86 / 82 / 97, 96 / 104 / 114.
template <typename T> constexpr int kBlockWgs = T::W == 4 ? 512 : 768;
// Forward with a gate per element and checkpoints, ten tensors at once: one per compute unit from 2^25 elements on, where every lane has columns.  256 / 512
// workgroups, us: 12 M elements 61 / 57 (D = 64, 128 and 256), 25 M 116 / 117, 29 M 135 / 136, 34 M 153 / 153, 40 M 182 / 187, 64 M 291 / 320; with a
// quarter of the lanes idle (D = 96) 34 M 186 / 167, 64 M 350 / 325.
constexpr int64_t kManyTensorsFrom = int64_t(1) << 25;     // elements
static bool vector_rows(int D, std::initializer_list<const void*> f32, std::initializer_list<const void*> q) {
    bool v = D % 4 == 0;
    for (const void* p : f32) v = v && aligned(p, 16);
    for (const void* p : q) v = v && aligned(p, 4);
    return v;
}

template <typename F> static void by_gate(int gate_cols, int D, F go) {
    if (gate_cols == 0) go(std::integral_constant<int, kNoGate>{});
    else if (gate_cols == D) go(std::integral_constant<int, kFullGate>{});
    else go(std::integral_constant<int, kRowGate>{});
}

int launch_block_fwd(const BlockFwd& a, hipStream_t s) {
    const bool vector = vector_rows(a.D, {a.X, a.Y, a.b.gate_cols == a.D ? a.G : nullptr, a.X_out, a.N}, {a.saved.x.q, a.saved.y.q, a.saved.g.q});
    const bool ckpt = a.saved.x.q || a.saved.y.q || a.saved.g.q;
    return with_row_tile(a.D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        const int64_t rows = ckpt ? (a.n + 7) / 8 * 8 : a.n, blocks = (rows + T::R - 1) / T::R;
        const bool many = T::W == 4 && a.D == T::W * T::LPR && ckpt && a.b.gate_cols == a.D && a.n * a.D >= kManyTensorsFrom;
        const int64_t most = many ? kBlockWgs<T> / 2 : kBlockWgs<T>;
        const dim3 grid((unsigned)(blocks < most ? blocks : most));
        auto go = [&](auto gate) {
            constexpr int GATE = decltype(gate)::value;
            if (ckpt) hipLaunchKernelGGL((block_fwd_kernel<T, GATE, true>), grid, dim3(kRowThreads), 0, s, a);
            else hipLaunchKernelGGL((block_fwd_kernel<T, GATE, false>), grid, dim3(kRowThreads), 0, s, a);
        };
        by_gate(a.b.gate_cols, a.D, go);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

size_t block_bwd_workspace(int64_t n, int D) {
    constexpr int kMost = kBlockWgs<RowTile<1, 64, 1>>;
    const int64_t most = n < kMost ? n : kMost;              // a workgroup takes a row at least
    return sizeof(float) * (size_t)(most < 1 ? 1 : most) * kSums * D;
}

int launch_block_bwd(BlockBwd a, void* ws, hipStream_t s) {
    if (!a.dN) {                  // nothing of the norm in front is read, so that nothing in it counts
        a.X_out = nullptr;
        a.saved.x = dr_act8{};
        a.saved.stats_before = nullptr;
    }
    const bool full = a.b.gate_cols == a.D;
    const bool floats = a.X_out || a.Y || (full && a.G), codes = a.saved.x.q || a.saved.y.q || a.saved.g.q;
    // (some from tensors, some from checkpoints: the kernels of any width)
    const bool vector = !(floats && codes) && vector_rows(a.D,
                                                          {a.dX_out, a.dN, a.X_out, a.Y, full ? a.G : nullptr, a.grads.dX, a.grads.dY,
                                                           full ? a.grads.dG : nullptr},
                                                          {a.saved.x.q, a.saved.y.q, a.saved.g.q});
    a.part = static_cast<float*>(ws);
    a.parts = 0;
    if (a.n > 0)
        DRC_TRY(with_row_tile(a.D, vector, [&](auto tile) -> int {
            using T = decltype(tile);
            const int64_t blocks = (a.n + T::R - 1) / T::R;
            a.parts = (int)(blocks < kBlockWgs<T> ? blocks : kBlockWgs<T>);
            auto start = [&](auto gate, auto from) {
                hipLaunchKernelGGL((block_bwd_kernel<T, decltype(gate)::value, decltype(from)::value>), dim3((unsigned)a.parts), dim3(kRowThreads), 0, s, a);
            };
            auto go = [&](auto gate) {
                if (!codes) start(gate, std::integral_constant<int, kFloats>{});
                else if (!floats) start(gate, std::integral_constant<int, kCodes>{});
                else if constexpr (T::W == 1) start(gate, std::integral_constant<int, kEither>{});
            };
            by_gate(a.b.gate_cols, a.D, go);
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
