// 8-bit activation checkpoints: packing, unpacking, and weight gradients of projections whose input is held as one.
#include "act8.h"

namespace drc {

constexpr int kPackThreads = 256;

template <typename T>
__global__ __launch_bounds__(kPackThreads) void act8_pack_kernel(const float* __restrict__ X, int64_t n, int D, int groups, int8_t* __restrict__ q,
                                                                 uint8_t* __restrict__ scale) {
    constexpr int R = kPackThreads / T::LPR;
    const int t = threadIdx.x % T::LPR;
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < n; r0 += (int64_t)gridDim.x * R) {
        const int64_t row = r0 + threadIdx.x / T::LPR;
        const bool on = row < n;
        float x[T::E];
        row_load<T>(X + (size_t)row * D, t, D, on, x);
        row_pack<T>(q, scale, row, n, t, D, groups, on, x);
    }
}

template <typename T>
__global__ __launch_bounds__(kPackThreads) void act8_unpack_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, int64_t n, int D,
                                                                   int groups, float* __restrict__ X) {
    constexpr int R = kPackThreads / T::LPR;
    const int t = threadIdx.x % T::LPR;
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < n; r0 += (int64_t)gridDim.x * R) {
        const int64_t row = r0 + threadIdx.x / T::LPR;
        const bool on = row < n;
        float x[T::E];
        row_unpack<T>(q, scale, row, t, D, groups, on, x);
        row_store<T>(X + (size_t)row * D, t, D, on, x);
    }
}

static unsigned row_blocks(int64_t n, int rows_per_block, int64_t most) {
    const int64_t b = (n + rows_per_block - 1) / rows_per_block;
    return (unsigned)(b < most ? b : most);
}

int launch_act8_pack(const float* X, int64_t n, int D, const dr_act8& out, hipStream_t s) {
    const bool vector = D % 4 == 0 && aligned(X, 16) && aligned(out.q, 4);
    return with_row_tile(D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        hipLaunchKernelGGL((act8_pack_kernel<T>), dim3(row_blocks(n, kPackThreads / T::LPR, 8192)), dim3(kPackThreads), 0, s, X, n, D, act_groups(D),
                           out.q, out.scale);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

int launch_act8_unpack(const dr_act8& in, int64_t n, int D, float* X, hipStream_t s) {
    const bool vector = D % 4 == 0 && aligned(X, 16) && aligned(in.q, 4);
    return with_row_tile(D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        hipLaunchKernelGGL((act8_unpack_kernel<T>), dim3(row_blocks(n, kPackThreads / T::LPR, 8192)), dim3(kPackThreads), 0, s, in.q, in.scale, n, D,
                           act_groups(D), X);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

// ---------------------------------------------------------------------------------------------------
// dW[D,F] = A^T dZ.  A workgroup sums a 16 x 16 tile of dW over one span of rows; spans are added by a second kernel, in 64 bits
// and a fixed order.
// ---------------------------------------------------------------------------------------------------
constexpr int kWgTile = 16;
static int wgrad_spans(int64_t n) {
    const int64_t s = (n + 2047) / 2048;
    return (int)(s < 1 ? 1 : (s > 256 ? 256 : s));
}
size_t act8_wgrad_workspace(int64_t n, int D, int F) { return sizeof(float) * (size_t)wgrad_spans(n) * D * F; }

__global__ __launch_bounds__(kWgTile* kWgTile) void act8_wgrad_kernel(const int8_t* __restrict__ q, const uint8_t* __restrict__ scale, int64_t n, int D,
                                                                      int groups, const float* __restrict__ dZ, int F, int64_t span,
                                                                      float* __restrict__ part) {
    __shared__ float a[kWgTile][kWgTile + 1], b[kWgTile][kWgTile + 1];
    const int x = threadIdx.x % kWgTile, y = threadIdx.x / kWgTile;
    const int d = blockIdx.x * kWgTile + x, f = blockIdx.y * kWgTile + x;
    const int64_t end = min(n, (int64_t)(blockIdx.z + 1) * span);
    float acc = 0.f;
    for (int64_t r0 = (int64_t)blockIdx.z * span; r0 < end; r0 += kWgTile) {
        const int64_t row = r0 + y;
        const bool on = row < end;
        a[y][x] = on && d < D ? (float)q[(size_t)row * D + d] * act_factor(scale[act_scale_at(row, d / kActGroup, groups)]) : 0.f;
        b[y][x] = on && f < F ? dZ[(size_t)row * F + f] : 0.f;
        __syncthreads();
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kWgTile; ++k) sum = fmaf(a[k][y], b[k][x], sum);
        acc += sum;
        __syncthreads();
    }
    const int dd = blockIdx.x * kWgTile + y;
    if (dd < D && f < F) part[((size_t)blockIdx.z * D + dd) * F + f] = acc;
}

__global__ __launch_bounds__(256) void act8_wgrad_sum_kernel(const float* __restrict__ part, int spans, int64_t count, int accumulate, float* dW) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    double s = accumulate ? (double)dW[i] : 0.0;
    for (int p = 0; p < spans; ++p) s += (double)part[(size_t)p * count + i];
    dW[i] = (float)s;
}

int launch_act8_wgrad(const dr_act8& A, int64_t n, int D, const float* dZ, int F, float* dW, bool accumulate, void* ws, hipStream_t s) {
    const int spans = n == 0 ? 0 : wgrad_spans(n);
    if (spans) {
        const int64_t span = ((n + spans - 1) / spans + kWgTile - 1) / kWgTile * kWgTile;
        hipLaunchKernelGGL(act8_wgrad_kernel, dim3((D + kWgTile - 1) / kWgTile, (F + kWgTile - 1) / kWgTile, spans), dim3(kWgTile * kWgTile), 0, s, A.q,
                           A.scale, n, D, act_groups(D), dZ, F, span, static_cast<float*>(ws));
    }
    const int64_t count = (int64_t)D * F;
    hipLaunchKernelGGL(act8_wgrad_sum_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, s, static_cast<const float*>(ws), spans, count,
                       accumulate ? 1 : 0, dW);
    DRC_HIP(hipGetLastError());
    return DR_OK;
}

}  // namespace drc
