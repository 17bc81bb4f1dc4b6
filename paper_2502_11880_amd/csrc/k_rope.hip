// Rotary positions: the pairs of the first `rot` channels of every head turned by angles that grow with the token's position,
//   (a, b) -> gain (a cos p f_i - b sin p f_i, b cos p f_i + a sin p f_i)     (f_i: turns a position of pair i)
// and the frequencies f_i = theta^(-2i / rot) / 2 pi, as they are or stretched for contexts longer than the original.
//
// Memory bounds it: x is read and written once.  A work group takes some heads of one token: its threads work out the token's
// angles (in 64 bits, see turn_of), share them through LDS, and each then keeps its place in a head while it walks the heads.
//
// Measured (kernel times): 6001 tokens of 32 heads of 100, 48 channels turned, f16, 14.6 us (5.3 TB/s); seven tokens of 32 heads of 128
// 2.7, of which an empty launch takes 1.7.
#include "rows.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;

// One thread a pair.
//   linear: f / factor, every position that much closer.
//   base:   theta factor^(rot / (rot - 2)): the slowest pair stretched by the factor, the fastest hardly.
//   turns:  w f + (1 - w) f / factor, w rising from 0 at `low` turns over the original context to 1 at `high`.
//   index:  the same between the (whole) indices at which a pair would make `high` and `low` turns.
__global__ void rope_freqs_kernel(RopeScaling r, int rot, double* freqs) {
    const int i = threadIdx.x;
    if (i >= rot / 2) return;
    constexpr double kTwoPi = 6.283185307179586476925;
    const double theta = r.kind == kScaleBase ? r.theta * pow(r.factor, (double)rot / (rot - 2)) : r.theta;
    const double f = pow(theta, -2.0 * i / rot) / kTwoPi;
    double keep = 1.0;
    if (r.kind == kScaleLinear) {
        keep = 0.0;
    } else if (r.kind == kScaleTurns) {
        keep = fmin(1.0, fmax(0.0, (r.original * f - r.low) / (r.high - r.low)));
    } else if (r.kind == kScaleIndex) {
        const double per = rot / (2.0 * log(r.theta));
        const double lo = fmax(0.0, floor(per * log(r.original / (r.high * kTwoPi))));
        const double hi = fmin((double)(rot - 1), ceil(per * log(r.original / (r.low * kTwoPi))));
        keep = 1.0 - fmin(1.0, fmax(0.0, (i - lo) / fmax(hi - lo, 0.001)));
    }
    freqs[i] = r.kind == kScaleNone || r.kind == kScaleBase ? f : f * keep + f / r.factor * (1.0 - keep);
}

template <int T>
__global__ __launch_bounds__(kThreads) void rope_kernel(Rope r, const void* x, int heads, int dim, const int32_t* pos, void* out,
                                                        int per_group, int64_t first_token) {
    __shared__ float2 turns[kMostPairs];
    const int64_t token = first_token + blockIdx.x;
    if ((int)threadIdx.x < r.rot >> 1) turns[threadIdx.x] = turn_of(r, threadIdx.x, pos[token]);
    __syncthreads();
    const Items items = items_of(r, dim);
    const int at_once = kThreads / items.all;             // heads that the work group takes at a time
    const int mine = threadIdx.x / items.all, i = threadIdx.x - mine * items.all;
    if (mine >= at_once) return;
    if (i >= items.turning && x == out) return;           // in place, and nothing to do
    const int h0 = blockIdx.y * per_group, h1 = h0 + per_group < heads ? h0 + per_group : heads;
    for (int h = h0 + mine; h < h1; h += at_once) turn_item<T>(r, items, i, x, out, (token * heads + h) * dim, turns);
}

template <int T>
hipError_t launch(const Rope& r, const void* x, int64_t n_tokens, int heads, int dim, const int32_t* pos, void* out, hipStream_t s) {
    const int64_t want = (2048 + n_tokens - 1) / n_tokens;            // work groups a token
    const int at_once = kThreads / items_of(r, dim).all;
    const int most = (heads + at_once - 1) / at_once, splits = (int)(want < most ? want : most);
    const int per = (heads + splits - 1) / splits;
    constexpr int64_t kMost = (int64_t)1 << 22;           // a grid has fewer than 2^32 threads
    const int64_t step = kMost / splits;
    for (int64_t at = 0; at < n_tokens; at += step) {
        const unsigned n = (unsigned)(n_tokens - at < step ? n_tokens - at : step);
        hipLaunchKernelGGL((rope_kernel<T>), dim3(n, (unsigned)((heads + per - 1) / per)), dim3(kThreads), 0, s, r, x, heads, dim, pos, out, per, at);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_freqs(const RopeScaling& r, int rot, double* freqs, hipStream_t s) {
    hipLaunchKernelGGL(rope_freqs_kernel, dim3(1), dim3(kMostPairs), 0, s, r, rot, freqs);
    return hipGetLastError();
}

hipError_t launch_rope(const Rope& r, int dtype, const void* x, int64_t n_tokens, int heads, int dim, const int32_t* pos,
                       void* out, hipStream_t s) {
    if (dtype == kF32) return launch<kF32>(r, x, n_tokens, heads, dim, pos, out, s);
    if (dtype == kBf16) return launch<kBf16>(r, x, n_tokens, heads, dim, pos, out, s);
    return launch<kF16>(r, x, n_tokens, heads, dim, pos, out, s);
}

}  // namespace bitnet
