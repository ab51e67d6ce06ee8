// 8-bit activation checkpoints: packing, unpacking, and weight gradients of projections whose input is held as one.
#include "act8.h"

#include <cmath>
#include <type_traits>

namespace drc {

// Matrices of one width, each a range of the workgroups.
struct PackArgs {
    Act8Pack m[kMaxPacks];
    int first[kMaxPacks + 1];     // workgroup
    int D;
};
// Bound by memory, both ways: 1.2 M x 128 packed in 137 us (773 MB, 5.6 TB/s) and unpacked in 129.  A block of rows at a time: with two and four of them
// under way per workgroup both together take 310 and 319 us instead of 295 (8192 workgroups).
template <typename T> __global__ __launch_bounds__(kRowThreads) void act8_pack_kernel(PackArgs a) {
    const int D = a.D, groups = act_groups(D);
    const RowLane<T> l(D);
    int i = 0;
    while (i + 1 < kMaxPacks && (int)blockIdx.x >= a.first[i + 1]) ++i;
    const Act8Pack m = a.m[i];
    const int64_t n8 = (m.n + 7) & ~int64_t(7);                 // the rows that fill up the last eight have scale bytes
    const int64_t step = (int64_t)(a.first[i + 1] - a.first[i]) * T::R;
    for (int64_t r0 = (int64_t)((int)blockIdx.x - a.first[i]) * T::R; r0 < n8; r0 += step) {
        const int left = (int)(m.n - r0 < T::R ? (m.n > r0 ? m.n - r0 : 0) : T::R);
        uint32_t raw[T::E];
        float x[T::E];
        load_rows<T>(rows_view(m.X, r0, left, 4 * D), l, raw);
#pragma unroll
        for (int e = 0; e < T::E; ++e) x[e] = of_bits(raw[e]);
        store_codes<T>(rows_view(m.out.q, r0, left, D), scales_view(m.out.scale, r0, m.n, groups), l, l.row < left, x);
    }
}

template <typename T, int POLICY>
__global__ __launch_bounds__(kRowThreads) void act8_unpack_kernel(const int8_t* q, const uint8_t* scale, int64_t n, int D, float* X) {
    const RowLane<T> l(D);
    const int groups = act_groups(D);
    for (int64_t r0 = (int64_t)blockIdx.x * T::R; r0 < n; r0 += (int64_t)gridDim.x * T::R) {
        const int left = (int)(n - r0 < T::R ? n - r0 : T::R);
        uint32_t code[T::E], s[T::V];
        float x[T::E];
        load_codes<T>(rows_view(q, r0, left, D), scales_view(scale, r0, n, groups), l, code, s);
        decode<T>(code, s, l.row < left, x);
        store_rows<T, POLICY>(rows_view(X, r0, left, 4 * D), l, x);
    }
}

// Workgroups: so many that they come and go, which keeps those that are there close together in memory.  2048 / 8192 / 32768, us: 1.2 M x 128
// packed 152 / 157 / 141, 250 000 x 128 31.9 / 29.8 / 30.8, 30 011 x 99 7.2 / 8.5 / 8.4.
static unsigned row_blocks(int64_t rows, int rows_per_block) {
    const int64_t b = (rows + rows_per_block - 1) / rows_per_block;
    return (unsigned)(b < 32768 ? b : 32768);
}

// Elements from which on what is written outgrows the 256 MB that memory keeps in its own cache: it is streamed past the other caches
// (1.2 M x 128 packed and unpacked 294 / 272 us).
constexpr int64_t kStreamFrom = int64_t(1) << 26;

int launch_act8_packs(const Act8Pack* jobs, int n, int D, hipStream_t s) {
    bool vector = D % 4 == 0;
    for (int i = 0; i < n; ++i) vector = vector && aligned(jobs[i].X, 16) && aligned(jobs[i].out.q, 4);
    return with_row_tile(D, vector, [&](auto tile) -> int {
        using T = decltype(tile);
        PackArgs a{};
        a.D = D;
        unsigned blocks = 0;
        for (int i = 0; i < kMaxPacks; ++i) {
            a.first[i] = (int)blocks;
            if (i >= n) continue;
            a.m[i] = jobs[i];
            blocks += row_blocks((jobs[i].n + 7) / 8 * 8, T::R);
        }
        a.first[kMaxPacks] = (int)blocks;
        if (blocks == 0) return DR_OK;
        hipLaunchKernelGGL((act8_pack_kernel<T>), dim3(blocks), dim3(kRowThreads), 0, s, a);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}
int launch_act8_pack(const float* X, int64_t n, int D, const dr_act8& out, hipStream_t s) {
    const Act8Pack job{X, n, out};
    return launch_act8_packs(&job, 1, D, s);
}

int launch_act8_unpack(const dr_act8& in, int64_t n, int D, float* X, hipStream_t s) {
    return with_row_tile(D, D % 4 == 0 && aligned(X, 16) && aligned(in.q, 4), [&](auto tile) -> int {
        using T = decltype(tile);
        const dim3 grid(row_blocks(n, T::R));
        if (n * D > kStreamFrom) hipLaunchKernelGGL((act8_unpack_kernel<T, kStreamed>), grid, dim3(kRowThreads), 0, s, in.q, in.scale, n, D, X);
        else hipLaunchKernelGGL((act8_unpack_kernel<T, 0>), grid, dim3(kRowThreads), 0, s, in.q, in.scale, n, D, X);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

// ---------------------------------------------------------------------------------------------------
// dW[D,F] = A^T dZ, the contraction running over the rows.
//
// Arithmetic.  What a code stands for, q * 2^s, is a bf16 number exactly; dZ is cut into three bf16 numbers, x = x1 + x2 + x3,
// by taking the upper half of x, of x - x1 and of x - x1 - x2: 3 x 8 significant bits hold all 24 from 2^-110 upwards; below, bf16's steps end
// at 2^-133 and what is smaller is left out.  Three exact bf16 products per
// term then are the fp32 product (a projection whose input is held in fp32 needs six).  Leading products and small ones have
// accumulators of their own, which start from zero every kFlush chunks and are added to the running sum with one rounding:
// inside the matrix unit what lies below the running sum is cut off, always downwards, which over many rows adds up.
//
// Layout.  The matrix instructions take eight consecutive contraction indices, rows, per lane: a unit is eight rows of one
// column, 16 bytes.  A thread loads its column's eight rows (64 neighbouring columns per wavefront and row) and puts whole units
// into LDS, so nothing is transposed.  The scales of a unit's eight rows lie side by side: one load.  Rows past the end and columns
// past the widths read as zero through the buffer descriptors.
//
// Pipeline.  Eight wavefronts, LDS doubled, one barrier per chunk of rows; half of the wavefronts stage the next chunk before they
// multiply, the other half after, so that vector and matrix instructions of a SIMD's two wavefronts overlap.  A workgroup takes one tile of
// dW and every S-th chunk; partial sums go to the workspace and are added by a second kernel, in 64 bits and a fixed order.
//
// What bounds it is issue: 1.2 M x 128 x 128 takes 171 to 184 us by card, with the sums (773 MB, 4.5 to 4.2 TB/s); without the multiplication 127 (memory), with the
// multiplication and bare staging 138.  Vector and matrix instructions of a SIMD take turns for the most part, 99 of the former per wavefront and
// chunk (130 before: codes sign-extended as they are loaded, scale bytes shifted into place by one instruction, rows past the end looked for once per
// chunk, running sums added to every 16 chunks; 191 us).  60 013 x 96 x 200, 23 us: 15 chunks a workgroup one after the other, tiles of 128 columns
// for 72; 2 048 x 64 x 64, 8.3 us of two launches.
// ---------------------------------------------------------------------------------------------------
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kGradWaves = 8, kGradThreads = 64 * kGradWaves;
constexpr int kFlush = 16;                         // chunks that the matrix unit sums up by itself (4 / 8 / 16: 183 / 179 / 177 us, errors of 1e-7 each)
constexpr int kGradWgs = 256;                      // one workgroup per compute unit

// TD x TF entries of dW; WA x WB wavefronts side by side on them, WK groups of those on 32 rows of a chunk each.  A wavefront's part is made of
// 32 x 32 blocks where it is that wide: half as many matrix instructions as 16 x 16 ones take, each of which keeps vector instructions out
// as long.
template <int TD_, int TF_, int WA_, int WB_> struct GradTile {
    static constexpr int TD = TD_, TF = TF_, WA = WA_, WB = WB_, WK = kGradWaves / (WA * WB);
    static constexpr int CR = 32 * WK, RG = CR / 8;             // rows and units per column of a chunk
    static constexpr int AU = RG * TD, BU = RG * TF;            // units of A and of one part of dZ
    static constexpr int BUF = AU + 3 * BU;
    static constexpr int M = TD / WA % 32 == 0 && TF / WB % 32 == 0 ? 32 : 16;     // width of a block
    static constexpr int MA = TD / (M * WA), MB = TF / (M * WB);        // blocks per wavefront
    static constexpr int KS = M / 16;                                   // matrix instructions per block, part and chunk
    typedef float Block __attribute__((ext_vector_type(M * M / 64)));
    static_assert(AU <= kGradThreads && BU <= kGradThreads && AU % 64 == 0 && BU % 64 == 0);
    static_assert(MA * M * WA == TD && MB * M * WB == TF && TD * TF % 256 == 0);
};

struct GradArgs {
    const int8_t* q;
    const uint8_t* scale;
    const float* dZ;
    float* part;
    int64_t n;
    int D, groups, F, tiles_f, splits;
};

// the upper halves of a and b as two bf16 numbers
__device__ __forceinline__ uint32_t upper2(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// byte N of w as an exponent: in bits 23 .. 30, zeros around it
template <int N> __device__ __forceinline__ uint32_t byte_up(uint32_t w) {
    uint32_t r;
    const uint32_t by = 23;
    if constexpr (N == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(by), "v"(w));
    if constexpr (N == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(by), "v"(w));
    if constexpr (N == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(by), "v"(w));
    if constexpr (N == 3) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(by), "v"(w));
    return r;
}
template <int N, int I = 0, typename F> __device__ __forceinline__ void steps(F f) {       // f(0), ..., f(N - 1), each a constant
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        steps<N, I + 1>(f);
    }
}

template <typename T> __device__ __forceinline__ typename T::Block grad_mfma(const bf16x8& b, const bf16x8& a, const typename T::Block& c) {
    if constexpr (T::M == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
}

template <typename T> __global__ __launch_bounds__(kGradThreads, 2) void act8_wgrad_kernel(GradArgs a) {
    extern __shared__ bf16x8 smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = wave / (T::WA * T::WB), wa = wave % (T::WA * T::WB) / T::WB, wb = wave % T::WB;
    const int z = blockIdx.x % a.splits, tile = blockIdx.x / a.splits;
    const int d0 = tile / a.tiles_f * T::TD, f0 = tile % a.tiles_f * T::TF;
    const int ca = d0 + tid % T::TD, ra = tid / T::TD * 8;      // this thread's units: column and first row of A, of dZ
    const int cb = f0 + tid % T::TF, rb = tid / T::TF * 8;
    const bool has_a = T::AU == kGradThreads || wave * 64 < T::AU, has_b = T::BU == kGradThreads || wave * 64 < T::BU;    // whole wavefronts
    const int D = a.D, F = a.F, G8 = a.groups * 8;
    const int at_a = ca < D ? ra * D + ca : kOutside, at_b = cb < F ? (rb * F + cb) * 4 : kOutside;
    const int at_s = ca < D ? (ra >> 3) * G8 + ca / kActGroup * 8 : kOutside;
    const int chunks = (int)((a.n + T::CR - 1) / T::CR);

    struct Raw { int code[8]; u32x2 scales; float y[8]; } raw[2];
    auto load = [&](int chunk, Raw& r) {                        // past the last chunk: reads nothing
        const int64_t base = (int64_t)chunk * T::CR;
        const int64_t left = a.n > base ? (a.n - base < T::CR ? a.n - base : T::CR) : 0;
        if (has_a) {
            const Buf q = buf_view(a.q + base * D, left * D), s = buf_view(a.scale + base / 8 * G8, (left + 7) / 8 * G8);
#pragma unroll
            for (int j = 0; j < 8; ++j) r.code[j] = (int8_t)__builtin_amdgcn_raw_buffer_load_b8(q, at_a + j * D, 0, 0);
            r.scales = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(s, at_s, 0, 0));
        }
        if (has_b) {
            const Buf b = buf_view(a.dZ + base * F, left * F * 4);
#pragma unroll
            for (int j = 0; j < 8; ++j) r.y[j] = of_bits(__builtin_amdgcn_raw_buffer_load_b32(b, at_b + j * F * 4, 0, 0));
        }
    };
    auto commit = [&](int chunk, const Raw& r, int to) {
        bf16x8* const buf = smem + to * T::BUF;
        if (has_a) {
            // bytes of rows past the end may hold anything: they are zeros here
            u32x2 scales = r.scales;
            const int64_t left = a.n - (int64_t)chunk * T::CR;
            if (left < T::CR) {
                const int rows = (int)left - ra;
                const uint64_t keep = rows <= 0 ? 0 : rows >= 8 ? ~uint64_t(0) : (uint64_t(1) << (8 * rows)) - 1;
                scales[0] &= (uint32_t)keep;
                scales[1] &= (uint32_t)(keep >> 32);
            }
            uint32_t v[8], w[4];
            // 255 << 23 is an infinity and the codes of such a group are zeros: not-a-numbers
            steps<8>([&](auto at) {
                constexpr int j = decltype(at)::value;
                v[j] = bits((float)r.code[j] * of_bits(byte_up<j % 4>(scales[j / 4])));
            });
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = upper2(v[2 * j], v[2 * j + 1]);
            buf[tid] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        }
        if (has_b) {
            uint32_t x1[8], x2[8], x3[8];
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                most = fmaxf(most, fabsf(r.y[j]));
                x1[j] = bits(r.y[j]);
                const float rest = r.y[j] - of_bits(x1[j] & 0xffff0000u);
                x2[j] = bits(rest);
                x3[j] = bits(rest - of_bits(x2[j] & 0xffff0000u));
            }
            if (__builtin_amdgcn_ballot_w64(most == __builtin_inff())) {     // an infinity has no remainder
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (fabsf(r.y[j]) == __builtin_inff()) x2[j] = x3[j] = 0;
            }
            auto put = [&](int part, const uint32_t (&x)[8]) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = upper2(x[2 * j], x[2 * j + 1]);
                buf[T::AU + part * T::BU + tid] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
            };
            put(0, x1);
            put(1, x2);
            put(2, x3);
        }
    };

    using Block = typename T::Block;
    Block acc[T::MA][T::MB] = {}, hi[T::MA][T::MB] = {}, lo[T::MA][T::MB] = {};
    const auto flush = [&]() {
#pragma unroll
        for (int i = 0; i < T::MA; ++i)
#pragma unroll
            for (int j = 0; j < T::MB; ++j) {
                acc[i][j] += hi[i][j] + lo[i][j];
                hi[i][j] = Block{};
                lo[i][j] = Block{};
            }
    };
    const auto multiply = [&](int from) {
        const bf16x8* const buf = smem + from * T::BUF;
        const int col = lane % T::M;
        bf16x8 fa[T::MA][T::KS], fb[T::MB][3][T::KS];
#pragma unroll
        for (int k = 0; k < T::KS; ++k) {
            const int rg = 4 * wk + 4 / T::KS * k + lane / T::M;         // row group of this lane
#pragma unroll
            for (int i = 0; i < T::MA; ++i) fa[i][k] = buf[rg * T::TD + T::M * (wa * T::MA + i) + col];
#pragma unroll
            for (int j = 0; j < T::MB; ++j)
#pragma unroll
                for (int p = 2; p >= 0; --p) fb[j][p][k] = buf[T::AU + p * T::BU + rg * T::TF + T::M * (wb * T::MB + j) + col];
        }
        __builtin_amdgcn_sched_barrier(0);
        // consecutive instructions go to different sums
#pragma unroll
        for (int k = 0; k < T::KS; ++k)
#pragma unroll
            for (int j = 0; j < T::MB; ++j) {
#pragma unroll
                for (int i = 0; i < T::MA; ++i) lo[i][j] = grad_mfma<T>(fb[j][2][k], fa[i][k], lo[i][j]);
#pragma unroll
                for (int i = 0; i < T::MA; ++i) hi[i][j] = grad_mfma<T>(fb[j][0][k], fa[i][k], hi[i][j]);
#pragma unroll
                for (int i = 0; i < T::MA; ++i) lo[i][j] = grad_mfma<T>(fb[j][1][k], fa[i][k], lo[i][j]);
            }
    };
    // Two chunks are under way to the registers while one is in LDS and one is multiplied: 41 KB per compute unit (with one, 1.2 M x 128 x 128
    // took 184 us).
    const auto walk = [&](auto which) {
        constexpr bool first = decltype(which)::value;
        int chunk = z, since = 0;
        const auto step = [&](auto at) {
            constexpr int cur = decltype(at)::value;
            __syncthreads();                                    // this chunk is in LDS; the other buffer may be overwritten
            const int next = chunk + a.splits;
            if constexpr (first) {
                commit(next, raw[cur ^ 1], cur ^ 1);
                load(next + 2 * a.splits, raw[cur ^ 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(cur);
            if (++since == kFlush) {
                flush();
                since = 0;
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!first) {
                commit(next, raw[cur ^ 1], cur ^ 1);
                load(next + 2 * a.splits, raw[cur ^ 1]);
            }
            chunk = next;
        };
        if (chunk < chunks) {
            load(chunk, raw[0]);
            load(chunk + a.splits, raw[1]);
            commit(chunk, raw[0], 0);
            load(chunk + 2 * a.splits, raw[0]);
        }
        while (chunk < chunks) {
            step(std::integral_constant<int, 0>{});
            if (chunk >= chunks) break;
            step(std::integral_constant<int, 1>{});
        }
        flush();
    };
    if (wave < kGradWaves / 2) walk(std::true_type{});
    else walk(std::false_type{});
    // lane: row lane % M of a block of the tile, four columns each from 4 (lane / M) on, every 8 columns (32 x 32; 16 x 16 has four in all)
    float* const out = a.part + ((size_t)blockIdx.x * T::WK + wk) * T::TD * T::TF;
#pragma unroll
    for (int i = 0; i < T::MA; ++i)
#pragma unroll
        for (int j = 0; j < T::MB; ++j)
#pragma unroll
            for (int r = 0; r < T::M * T::M / 64; r += 4)
                *reinterpret_cast<f32x4*>(out + (size_t)(T::M * (wa * T::MA + i) + lane % T::M) * T::TF + T::M * (wb * T::MB + j) + 2 * r +
                                          4 * (lane / T::M)) = f32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
}

// dW = the sum over a tile's partials: wavefront w of the workgroup sums partials w, w + 16, ... of 64 x 4 consecutive entries, then
// the 16 sums are added in order, in 64 bits (up to 1024 partials of nearly equal size lose as much in 32-bit sums as everything before).
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void act8_wgrad_sum_kernel(const float* __restrict__ part, int parts, int TD, int TF, int tiles_f, int D,
                                                                        int F, int accumulate, float* dW) {
    __shared__ f64x4 sums[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = TD * TF / 256, tile = blockIdx.x / blocks;
    const int at = blockIdx.x % blocks * 256 + 4 * lane;
    const float* const src = part + (size_t)tile * parts * TD * TF + at;
    f64x4 s = {0., 0., 0., 0.};
    int b = wave;
    for (; b + 3 * kSumWaves < parts; b += 4 * kSumWaves) {     // four loads in flight
        f32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const f32x4*>(src + (size_t)(b + u * kSumWaves) * TD * TF);
#pragma unroll
        for (int u = 0; u < 4; ++u) s += __builtin_convertvector(v[u], f64x4);
    }
    for (; b < parts; b += kSumWaves) s += __builtin_convertvector(*reinterpret_cast<const f32x4*>(src + (size_t)b * TD * TF), f64x4);
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0) return;
    f64x4 t = sums[0][lane];
#pragma unroll
    for (int w = 1; w < kSumWaves; ++w) t += sums[w][lane];
    const int d = tile / tiles_f * TD + at / TF, f = tile % tiles_f * TF + at % TF;
    if (d >= D) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (f + r < F) {
            float* const o = dW + (size_t)d * F + f + r;
            *o = (float)(accumulate ? (double)*o + t[r] : t[r]);
        }
}

// Calls f(GradTile<...>{}): a tile as wide as the matrix, up to 128 either way.  Tiles of 96 columns for the layers' width: 250 000 x 96 x 96 41.5 / 38.5 us,
// 60 013 x 96 x 200 26.5 / 24.5 (128 x 128 / 96).
template <typename F> static int with_grad_tile(int D, int Fw, F f) {
    if (D <= 32) {
        if (Fw <= 32) return f(GradTile<32, 32, 2, 1>{});
        if (Fw <= 64) return f(GradTile<32, 64, 2, 2>{});
        return f(GradTile<32, 128, 2, 4>{});
    }
    if (D <= 64) {
        if (Fw <= 32) return f(GradTile<64, 32, 2, 2>{});
        if (Fw <= 64) return f(GradTile<64, 64, 2, 2>{});
        return f(GradTile<64, 128, 2, 4>{});
    }
    if (D <= 96 && Fw > 64) return f(GradTile<96, 128, 2, 4>{});
    if (Fw > 64 && Fw <= 96) return f(GradTile<128, 96, 4, 2>{});
    if (Fw <= 32) return f(GradTile<128, 32, 4, 2>{});
    if (Fw <= 64) return f(GradTile<128, 64, 4, 2>{});
    return f(GradTile<128, 128, 2, 4>{});
}
// Workgroups per tile of dW.  A workgroup's partial sums weigh as much as a few chunks, written once and read once: with r chunks a workgroup a launch
// takes about r * c + tiles * chunks / r * s, least at r = sqrt(tiles * chunks * s / c).  s / c is near 0.045 whatever the tile (best r measured: 32 x 32
// 157 / 469 / 1 953 chunks 4 / 5 / 10; 64 x 64 157 / 313 / 938 2.5 / 4 / 6.5; 128 x 128 128 / 250 / 500 2 / 3.5 / 4.5).  No more than one per compute
// unit in all, and all with the same number of chunks but for the last.  One per compute unit, or a chunk each / now: 10 000 x 64 x 64 13.0 / 10.6 us,
// 20 000 16.7 / 12.4, 8 000 x 128 x 128 17.7 / 13.6, 60 000 x 32 x 32 20.0 / 14.3.
template <typename T> static int grad_splits(int64_t n, int D, int F) {
    const int64_t tiles = (int64_t)((D + T::TD - 1) / T::TD) * ((F + T::TF - 1) / T::TF), chunks = (n + T::CR - 1) / T::CR;
    const int64_t most = tiles < kGradWgs ? kGradWgs / tiles : 1;
    int64_t r = (int64_t)(std::sqrt(0.045 * (double)(tiles * chunks)) + 0.5);
    if (r * most < chunks) r = (chunks + most - 1) / most;
    if (r < 1) r = 1;
    return chunks < 1 ? 1 : (int)((chunks + r - 1) / r);
}

size_t act8_wgrad_workspace(int64_t n, int D, int F) {
    size_t bytes = 0;
    with_grad_tile(D, F, [&](auto tile) -> int {
        using T = decltype(tile);
        const size_t tiles = (size_t)((D + T::TD - 1) / T::TD) * ((F + T::TF - 1) / T::TF);
        bytes = sizeof(float) * tiles * grad_splits<T>(n, D, F) * T::WK * T::TD * T::TF;
        return DR_OK;
    });
    return bytes;
}

int launch_act8_wgrad(const dr_act8& A, int64_t n, int D, const float* dZ, int F, float* dW, bool accumulate, void* ws, hipStream_t s) {
    return with_grad_tile(D, F, [&](auto tile) -> int {
        using T = decltype(tile);
        static PerDevice cache;
        constexpr size_t lds = sizeof(bf16x8) * 2 * T::BUF;
        int dev = 0, ready = 0;
        DRC_HIP(hipGetDevice(&dev));
        DRC_TRY(cache.get(dev, &ready, [&](int* r) -> int {
            DRC_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&act8_wgrad_kernel<T>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            *r = 1;
            return DR_OK;
        }));
        const int tiles_d = (D + T::TD - 1) / T::TD, tiles_f = (F + T::TF - 1) / T::TF;
        const int splits = n == 0 ? 0 : grad_splits<T>(n, D, F);
        if (splits) {
            const GradArgs a{A.q, A.scale, dZ, static_cast<float*>(ws), n, D, act_groups(D), F, tiles_f, splits};
            hipLaunchKernelGGL((act8_wgrad_kernel<T>), dim3((unsigned)(tiles_d * tiles_f * splits)), dim3(kGradThreads), lds, s, a);
        }
        hipLaunchKernelGGL(act8_wgrad_sum_kernel, dim3((unsigned)(tiles_d * tiles_f * (T::TD * T::TF / 256))), dim3(64 * kSumWaves), 0, s,
                           static_cast<const float*>(ws), splits * T::WK, T::TD, T::TF, tiles_f, D, F, accumulate ? 1 : 0, dW);
        DRC_HIP(hipGetLastError());
        return DR_OK;
    });
}

}  // namespace drc
