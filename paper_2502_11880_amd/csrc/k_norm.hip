// Root-mean-square norm of token rows, with the residual's addition before it and the int8 codes of the next product behind
// it (the quantiser of Sec. 2.1):
//   r      = x + residual                          (32 bits, then rounded to the residual's type: what is stored is what is normed)
//   inv    = fp32(1 / sqrt(sum_k r^2 / K + eps))   (64 bits)
//   n      = fp32(fp32(r inv) gamma)
//   s      = fp32(127 / max(max_k |n|, 1e-5)),  xq = clamp(rint(fp32(n s)), -128, 127),  rowsum = sum_k xq
// A sum of squares in 64 bits has the same 32-bit inv in any order but for one in some 2^29 rows, so the codes have one right
// value each, as those of the quantiser have; and squares of any 32-bit value fit it.  64-bit operations are as cheap as loads
// here: two an element, where the memory gives a CU less than one element a clock.
//
// Memory bounds it: a row is read once into registers (up to 8 quads a thread; rows past 16384 values 16, of which 1024 lanes spill 20 to
// 102 registers to scratch memory), summed, normed and quantised there, and written once; 13 bytes an element with everything in 32
// bits.  Two reductions over the work group stand in between.  Rows past 65536, which no linear of a model has, take three passes over
// memory.
//
// Measured (kernel times): 8192 rows of 4096, all in 32 bits, 76.8 us (5.7 TB/s; a large copy reaches 4.9, and here more is read
// than written) with 256 lanes a row, 512 the same, 128 79, 64 81, 1024 84; 333 rows of 8640, 32 bits onto a residual in bf16, 7.6 us
// with 512 lanes of five quads, 8.3 of eight, 9.1 with 1024 lanes; one row of 4096 3.3 us, of which an empty launch takes 1.7.
// Calls, all in 32 bits: 1000 rows of 20000 89 us (2.9 TB/s; three passes 97), 512 of 65536 112 (166), 256 of 100000 201; widths that are no
// multiple of four, by single values: 4096 rows of 4099 47 us (4.7 TB/s), 333 of 8641 11, 512 of 65535 132 (three passes 166), but 1000 of
// 20001 114 (97).
#include "rows.hpp"

namespace bitnet {
namespace {

__device__ __forceinline__ double wave_sum_all(double v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)dpp_row_step((int)(uint32_t)u, i), hi = (uint32_t)dpp_row_step((int)(uint32_t)(u >> 32), i);
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    double t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, 16 * i), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 16 * i);
        t[i] = __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    return (t[0] + t[1]) + (t[2] + t[3]);
}

// Reductions over the work group, the result in every thread.
template <int BLOCK>
__device__ __forceinline__ double block_sum(double v, double* red) {
    v = wave_sum_all(v);
    if constexpr (BLOCK > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v += red[w];
    }
    return v;
}
template <int BLOCK>
__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max_all(v);
    if constexpr (BLOCK > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v = fmaxf(v, red[w]);
    }
    return v;
}
template <int BLOCK>
__device__ __forceinline__ int block_sum(int v, int* red) {
    v = wave_sum_all(v);
    if constexpr (BLOCK > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; ++w) v += red[w];
    }
    return v;
}

__device__ __forceinline__ float inverse_rms(double sum, int K, float eps) { return (float)(1.0 / sqrt(sum / K + (double)eps)); }

// One row of up to VPT quads (QUAD) or 4 VPT single values a thread.
template <int X, int R, bool QUAD, int BLOCK, int VPT>
__global__ __launch_bounds__(BLOCK) void norm_rows_kernel(NormArgs a) {
    __shared__ double red_sum[BLOCK / 64];
    __shared__ float red_max[BLOCK / 64];
    __shared__ int red_codes[BLOCK / 64];
    const int64_t row = (a.first_row + blockIdx.x) * (int64_t)a.K;
    const int units = QUAD ? a.K >> 2 : a.K;              // what a thread takes at a time
    constexpr int N = QUAD ? VPT : 4 * VPT, E = QUAD ? 4 : 1;
    float v[N * E], g[N * E];
    // unit threadIdx.x + i BLOCK: a thread's loads are neighbours of its wave's
    auto at = [&](int i) { return (int)threadIdx.x + i * BLOCK; };
#pragma unroll
    for (int i = 0; i < N; ++i) load_units<X, E>(a.x, row, at(i), units, &v[i * E]);
    if (a.residual) {
        float b[N * E];
#pragma unroll
        for (int i = 0; i < N; ++i) load_units<R, E>(a.residual, row, at(i), units, &b[i * E]);
#pragma unroll
        for (int i = 0; i < N * E; ++i) v[i] = round_to<R>(v[i] + b[i]);
        if (a.residual_out) {
#pragma unroll
            for (int i = 0; i < N; ++i) store_units<R, E>(a.residual_out, row, at(i), units, &v[i * E]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (a.gamma) {
            load_units<kF32, E>(a.gamma, 0, at(i), units, &g[i * E]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) g[i * E + e] = 1.0f;
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N * E; ++i) sum = fma((double)v[i], (double)v[i], sum);   // exact products
    const float inv = inverse_rms(block_sum<BLOCK>(sum, red_sum), a.K, a.eps);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < N * E; ++i) {
        v[i] = v[i] * inv * g[i];
        top = fmaxf(top, fabsf(v[i]));
    }
    if (a.y) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (a.y_dtype == kF32) store_units<kF32, E>(a.y, row, at(i), units, &v[i * E]);
            else if (a.y_dtype == kBf16) store_units<kBf16, E>(a.y, row, at(i), units, &v[i * E]);
            else store_units<kF16, E>(a.y, row, at(i), units, &v[i * E]);
        }
    }
    if (!a.xq) return;
    const float s = 127.0f / fmaxf(block_max<BLOCK>(top, red_max), 1e-5f);
    int codes = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (at(i) >= units) continue;
        if constexpr (QUAD) {
            const uint32_t c = quant4(make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]), s);
            codes = byte_sum4(c, codes);
            reinterpret_cast<uint32_t*>(a.xq + row)[at(i)] = c;
        } else {
            const int c = quant1(v[i], s);
            codes += c;
            a.xq[row + at(i)] = (int8_t)c;
        }
    }
    if (threadIdx.x == 0) a.x_scale[a.first_row + blockIdx.x] = s;
    if (a.x_rowsum) {
        codes = block_sum<BLOCK>(codes, red_codes);
        if (threadIdx.x == 0) a.x_rowsum[a.first_row + blockIdx.x] = codes;
    }
}

// Rows of any length: the sum, the largest value and the codes in a pass each.  A thread reads in the later passes what it
// wrote itself in the first, where there is a residual_out (which may be the residual or x).
template <int X, int R, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_long_rows_kernel(NormArgs a) {
    __shared__ double red_sum[BLOCK / 64];
    __shared__ float red_max[BLOCK / 64];
    __shared__ int red_codes[BLOCK / 64];
    const int64_t row = (a.first_row + blockIdx.x) * (int64_t)a.K;
    const bool stored = a.residual && a.residual_out;
    auto sum_of = [&](int i) {
        float v = load_one<X>(a.x, row + i);
        return a.residual ? round_to<R>(v + load_one<R>(a.residual, row + i)) : v;
    };
    auto value_of = [&](int i) { return stored ? load_one<R>(a.residual_out, row + i) : sum_of(i); };
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.K; i += BLOCK) {
        const float v = sum_of(i);
        sum = fma((double)v, (double)v, sum);
        if (stored) store_one<R>(a.residual_out, row + i, v);
    }
    const float inv = inverse_rms(block_sum<BLOCK>(sum, red_sum), a.K, a.eps);
    float s = 0.0f;
    if (a.xq) {
        float top = 0.0f;
        for (int i = threadIdx.x; i < a.K; i += BLOCK) top = fmaxf(top, fabsf(value_of(i) * inv * (a.gamma ? a.gamma[i] : 1.0f)));
        s = 127.0f / fmaxf(block_max<BLOCK>(top, red_max), 1e-5f);
    }
    int codes = 0;
    for (int i = threadIdx.x; i < a.K; i += BLOCK) {
        const float n = value_of(i) * inv * (a.gamma ? a.gamma[i] : 1.0f);
        if (a.xq) {
            const int c = quant1(n, s);
            codes += c;
            a.xq[row + i] = (int8_t)c;
        }
        if (a.y) {
            if (a.y_dtype == kF32) store_one<kF32>(a.y, row + i, n);
            else if (a.y_dtype == kBf16) store_one<kBf16>(a.y, row + i, n);
            else store_one<kF16>(a.y, row + i, n);
        }
    }
    if (!a.xq) return;
    if (threadIdx.x == 0) a.x_scale[a.first_row + blockIdx.x] = s;
    if (a.x_rowsum) {
        codes = block_sum<BLOCK>(codes, red_codes);
        if (threadIdx.x == 0) a.x_rowsum[a.first_row + blockIdx.x] = codes;
    }
}

template <int X, int R, bool QUAD, int BLOCK, int VPT>
void launch_rows(const NormArgs& a, int rows, hipStream_t s) {
    hipLaunchKernelGGL((norm_rows_kernel<X, R, QUAD, BLOCK, VPT>), dim3((unsigned)rows), dim3(BLOCK), 0, s, a);
}

template <int X, int R, bool QUAD>
void launch_quads(const NormArgs& a, int rows, int64_t total_rows, hipStream_t s) {
    const int quads = (a.K + 3) >> 2;
    if (total_rows <= 64) {                               // few rows: spread each over many lanes
        if (quads <= 512) return launch_rows<X, R, QUAD, 512, 1>(a, rows, s);
        if (quads <= 1024) return launch_rows<X, R, QUAD, 1024, 1>(a, rows, s);
        if (quads <= 2048) return launch_rows<X, R, QUAD, 1024, 2>(a, rows, s);
    } else {
        if (quads <= 256) return launch_rows<X, R, QUAD, 64, 4>(a, rows, s);
        if (quads <= 512) return launch_rows<X, R, QUAD, 128, 4>(a, rows, s);
        if (quads <= 1024) return launch_rows<X, R, QUAD, 256, 4>(a, rows, s);
        if (quads <= 2048) return launch_rows<X, R, QUAD, 512, 4>(a, rows, s);
        if (quads <= 2560) return launch_rows<X, R, QUAD, 512, 5>(a, rows, s);
        if (quads <= 4096) return launch_rows<X, R, QUAD, 512, 8>(a, rows, s);
    }
    if (quads <= 4096) return launch_rows<X, R, QUAD, 1024, 4>(a, rows, s);
    if (quads <= 16384) return launch_rows<X, R, QUAD, 1024, 16>(a, rows, s);
    hipLaunchKernelGGL((norm_long_rows_kernel<X, R, 1024>), dim3((unsigned)rows), dim3(1024), 0, s, a);
}

template <int X, int R>
hipError_t launch_types(NormArgs a, int64_t M, hipStream_t s) {
    constexpr int64_t kMost = (int64_t)1 << 21;           // a grid has fewer than 2^32 threads
    for (int64_t at = 0; at < M; at += kMost) {
        a.first_row = at;
        const int rows = (int)(M - at < kMost ? M - at : kMost);
        if (a.K % 4 == 0) launch_quads<X, R, true>(a, rows, M, s);
        else launch_quads<X, R, false>(a, rows, M, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_quantize(const NormArgs& a, int x_dtype, int r_dtype, int64_t M, hipStream_t s) {
    if (x_dtype == kF32) {
        if (r_dtype == kBf16) return launch_types<kF32, kBf16>(a, M, s);
        if (r_dtype == kF16) return launch_types<kF32, kF16>(a, M, s);
        return launch_types<kF32, kF32>(a, M, s);
    }
    return x_dtype == kBf16 ? launch_types<kBf16, kBf16>(a, M, s) : launch_types<kF16, kF16>(a, M, s);
}

}  // namespace bitnet
