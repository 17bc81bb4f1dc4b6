// Rows of activations between the products of a layer: the norm and the position rotation.  Values of the three types, and
// the host launchers.
#pragma once

#include "bitnet_mi355x.h"
#include "kv_cache.hpp"

namespace bitnet {

template <int T>
__device__ __forceinline__ float load_one(const void* p, int64_t at) {
    if constexpr (T == kF32) return static_cast<const float*>(p)[at];
    else return Elem<T>::to(static_cast<const uint16_t*>(p)[at]);
}
template <int T>
__device__ __forceinline__ void store_one(void* p, int64_t at, float v) {
    if constexpr (T == kF32) static_cast<float*>(p)[at] = v;
    else static_cast<uint16_t*>(p)[at] = Elem<T>::from(v);
}
// Four values at a place that is a multiple of four.
template <int T>
__device__ __forceinline__ float4 load_quad(const void* p, int64_t at) {
    if constexpr (T == kF32) return load4<kBf16, true>(p, at);
    else return load4<T, false>(p, at);
}
template <int T>
__device__ __forceinline__ void store_quad(void* p, int64_t at, float4 v) {
    if constexpr (T == kF32) store4<kBf16, true>(p, at, v.x, v.y, v.z, v.w);
    else store4<T, false>(p, at, v.x, v.y, v.z, v.w);
}
// A value as type T holds it.
template <int T>
__device__ __forceinline__ float round_to(float v) {
    if constexpr (T == kF32) return v;
    else return Elem<T>::to(Elem<T>::from(v));
}

// Unit `unit` (E values: a quad, or one) of a row that starts at `row`; zeros, and nothing written, past its `units`.
template <int T, int E>
__device__ __forceinline__ void load_units(const void* p, int64_t row, int unit, int units, float* v) {
    if constexpr (E == 4) {
        const float4 q = unit < units ? load_quad<T>(p, row + 4 * (int64_t)unit) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        v[0] = q.x;
        v[1] = q.y;
        v[2] = q.z;
        v[3] = q.w;
    } else {
        v[0] = unit < units ? load_one<T>(p, row + unit) : 0.0f;
    }
}
template <int T, int E>
__device__ __forceinline__ void store_units(void* p, int64_t row, int unit, int units, const float* v) {
    if (unit >= units) return;
    if constexpr (E == 4) store_quad<T>(p, row + 4 * (int64_t)unit, make_float4(v[0], v[1], v[2], v[3]));
    else store_one<T>(p, row + unit, v[0]);
}

__device__ __forceinline__ int quant1(float v, float s) { return (int)fminf(fmaxf(rintf(v * s), -128.0f), 127.0f); }

// ------------------------------------------------------------------------------------------------
// The position rotation
// ------------------------------------------------------------------------------------------------
struct Rope {
    const double* freqs;      // turns a position, of rot / 2 pairs
    int rot;                  // rotated channels, the first of a head
    int interleaved;          // pairs (2i, 2i + 1), else (i, i + rot / 2)
    float gain;
};
constexpr int kMostPairs = 128;

// gain (cos, sin) of a position's angle for one pair.  The angle in turns and its reduction to an eighth of a turn are in 64 bits
// (positions of 2^24 leave 2^-29 of a turn), and so are the Taylor series: their next terms, x^15 / 15! and x^16 / 16! at
// pi / 4, are below 2^-45.  An angle is worked out once for all heads of its token: it costs nothing beside their loads.
__device__ __forceinline__ float2 turn_of(const Rope& r, int pair, int pos) {
    double t = (double)pos * r.freqs[pair];
    t -= rint(t);
    const double q = rint(4.0 * t);
    const double x = (t - 0.25 * q) * 6.283185307179586476925, x2 = x * x;
    double s = -1.0 / 39916800.0 + x2 * (1.0 / 6227020800.0);
    s = 1.0 / 362880.0 + x2 * s;
    s = -1.0 / 5040.0 + x2 * s;
    s = 1.0 / 120.0 + x2 * s;
    s = -1.0 / 6.0 + x2 * s;
    s = x + x * (x2 * s);
    double c = 1.0 / 479001600.0 - x2 * (1.0 / 87178291200.0);
    c = -1.0 / 3628800.0 + x2 * c;
    c = 1.0 / 40320.0 + x2 * c;
    c = -1.0 / 720.0 + x2 * c;
    c = 1.0 / 24.0 + x2 * c;
    c = -0.5 + x2 * c;
    c = 1.0 + x2 * c;
    const int quarter = (int)q & 3;
    const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    const double cs = quarter == 1 || quarter == 2 ? -a : a, sn = quarter >= 2 ? -b : b;
    return make_float2((float)(cs * r.gain), (float)(sn * r.gain));
}

// The two rotated values of a pair, in 32 bits.  Kept from being joined with their rounding to 16 (v_fma_mixlo_f16 rounds once what
// the others round twice): all forms and calls give the same bits.
__device__ __forceinline__ float held(float v) {
    asm("" : "+v"(v));
    return v;
}
__device__ __forceinline__ float turned_a(float a, float b, float2 t) { return held(fmaf(a, t.x, -(b * t.y))); }
__device__ __forceinline__ float turned_b(float a, float b, float2 t) { return held(fmaf(b, t.x, a * t.y)); }

// Channels d .. d + 3 (d a multiple of 4) of a head that starts at `head`, rotated; turns: of the pairs of its token.  What lies
// past the rotated channels comes as it is.
template <int T>
__device__ __forceinline__ float4 turned_quad(const Rope& r, const void* p, int64_t head, int d, const float2* turns) {
    const float4 x = load_quad<T>(p, head + d);
    if (d >= r.rot) return x;
    const int half = r.rot >> 1;
    float4 y = x;
    if (r.interleaved) {
        const float2 t0 = turns[d >> 1];
        y.x = turned_a(x.x, x.y, t0);
        y.y = turned_b(x.x, x.y, t0);
        if (d + 2 < r.rot) {
            const float2 t1 = turns[(d >> 1) + 1];
            y.z = turned_a(x.z, x.w, t1);
            y.w = turned_b(x.z, x.w, t1);
        }
    } else if ((half & 3) == 0) {
        const bool first = d < half;
        const int pair = first ? d : d - half;
        const float4 o = load_quad<T>(p, head + (first ? d + half : d - half));
        const float2 t0 = turns[pair], t1 = turns[pair + 1], t2 = turns[pair + 2], t3 = turns[pair + 3];
        y.x = first ? turned_a(x.x, o.x, t0) : turned_b(o.x, x.x, t0);
        y.y = first ? turned_a(x.y, o.y, t1) : turned_b(o.y, x.y, t1);
        y.z = first ? turned_a(x.z, o.z, t2) : turned_b(o.z, x.z, t2);
        y.w = first ? turned_a(x.w, o.w, t3) : turned_b(o.w, x.w, t3);
    } else {
        float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = d + e;
            if (at >= r.rot) continue;
            const bool first = at < half;
            const int pair = first ? at : at - half;
            const float o = load_one<T>(p, head + (first ? at + half : at - half));
            v[e] = first ? turned_a(v[e], o, turns[pair]) : turned_b(o, v[e], turns[pair]);
        }
        y = make_float4(v[0], v[1], v[2], v[3]);
    }
    return y;
}

// A head as items whose loads and stores no other item touches, so that a head may be rotated in place: both sides of four pairs
// (half layout, of quads), a quad of channels (interleaved pairs, or channels that are not rotated), a pair or a channel
// (half layout whose halves are no quads).
struct Items {
    int turning, all;         // items that turn come first
    bool quads;
};
__host__ __device__ __forceinline__ Items items_of(const Rope& r, int dim) {
    Items it;
    const int half = r.rot >> 1;
    it.quads = r.interleaved || (half & 3) == 0;
    it.turning = r.interleaved ? (r.rot + 3) >> 2 : it.quads ? half >> 2 : half;
    it.all = r.interleaved ? dim >> 2 : it.turning + (it.quads ? (dim - r.rot) >> 2 : dim - r.rot);
    return it;
}
template <int T>
__device__ __forceinline__ void turn_item(const Rope& r, const Items& items, int i, const void* in, void* out, int64_t head,
                                          const float2* turns) {
    const int half = r.rot >> 1;
    if (r.interleaved) {
        const int d = 4 * i;
        float4 x = load_quad<T>(in, head + d), y = x;
        if (d < r.rot) {
            const float2 t = turns[2 * i];
            y.x = turned_a(x.x, x.y, t);
            y.y = turned_b(x.x, x.y, t);
        }
        if (d + 2 < r.rot) {
            const float2 t = turns[2 * i + 1];
            y.z = turned_a(x.z, x.w, t);
            y.w = turned_b(x.z, x.w, t);
        }
        store_quad<T>(out, head + d, y);
    } else if (items.quads) {
        if (i >= items.turning) {
            const int d = r.rot + 4 * (i - items.turning);
            store_quad<T>(out, head + d, load_quad<T>(in, head + d));
            return;
        }
        const int d = 4 * i;
        const float4 a = load_quad<T>(in, head + d), b = load_quad<T>(in, head + half + d);
        const float2 t0 = turns[d], t1 = turns[d + 1], t2 = turns[d + 2], t3 = turns[d + 3];
        store_quad<T>(out, head + d, make_float4(turned_a(a.x, b.x, t0), turned_a(a.y, b.y, t1), turned_a(a.z, b.z, t2), turned_a(a.w, b.w, t3)));
        store_quad<T>(out, head + half + d, make_float4(turned_b(a.x, b.x, t0), turned_b(a.y, b.y, t1), turned_b(a.z, b.z, t2), turned_b(a.w, b.w, t3)));
    } else if (i >= items.turning) {
        const int d = r.rot + i - items.turning;
        store_one<T>(out, head + d, load_one<T>(in, head + d));
    } else {
        const float a = load_one<T>(in, head + i), b = load_one<T>(in, head + half + i);
        store_one<T>(out, head + i, turned_a(a, b, turns[i]));
        store_one<T>(out, head + half + i, turned_b(a, b, turns[i]));
    }
}

// ------------------------------------------------------------------------------------------------
// Host launchers (arguments checked by the caller)
// ------------------------------------------------------------------------------------------------
struct NormArgs {
    const void* x;
    const void* residual;     // or null
    void* residual_out;       // or null
    const float* gamma;       // or null: ones
    void* y;                  // or null
    int8_t* xq;               // or null (then x_scale and x_rowsum too)
    float* x_scale;
    int32_t* x_rowsum;        // or null
    int64_t first_row;
    int K, y_dtype;
    float eps;
};
// r_dtype: of the residual (x's where there is none).
hipError_t launch_norm_quantize(const NormArgs& a, int x_dtype, int r_dtype, int64_t M, hipStream_t s);

// How a rotation's frequencies are stretched (the values of bitnet_rope_scaling).
constexpr int kScaleNone = 0, kScaleLinear = 1, kScaleBase = 2, kScaleTurns = 3, kScaleIndex = 4;
struct RopeScaling {
    double theta, factor, original, low, high;
    int kind;
};
// A rotation's sizes and (where anything is to be done) its pointer, as the entry points check them; and as the kernels take it.
int check_rotation(const bitnet_rotation* r, int64_t head_dim, bool pointers);
Rope rope_of(const bitnet_rotation* r);
hipError_t launch_rope_freqs(const RopeScaling& r, int rot, double* freqs, hipStream_t s);
hipError_t launch_rope(const Rope& r, int dtype, const void* x, int64_t n_tokens, int heads, int dim, const int32_t* pos,
                       void* out, hipStream_t s);
// q null: keys and values only.
hipError_t launch_kv_append_rope(const KvCache& c, int dtype, const void* q, int heads, const void* k, const void* v, bool f32,
                                 const int32_t* q_start, int n_tokens, const Rope& r, void* q_out, hipStream_t s);

}  // namespace bitnet
