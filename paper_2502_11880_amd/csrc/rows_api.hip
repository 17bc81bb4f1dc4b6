// C entry points of the norm and of the position rotation: argument validation and dispatch.  As in bitnet_api.hip, every
// check runs on the host before anything is enqueued, and no call allocates, copies to the host or synchronises.
#include "bitnet_mi355x.h"
#include "rows.hpp"

#include <math.h>

namespace {

using bitnet::fail;
using bitnet::hip_status;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bitnet_status st(int code) { return (bitnet_status)code; }

bool dtype_ok(int d) { return d == BITNET_DTYPE_F32 || d == BITNET_DTYPE_BF16 || d == BITNET_DTYPE_F16; }
int64_t size_of(int dtype) { return dtype == BITNET_DTYPE_F32 ? 4 : 2; }

// A buffer of a call (null: not given).
struct Span {
    const void* p;
    int64_t bytes;
    int dtype;
};
bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

constexpr int64_t kMaxRows = (int64_t)1 << 24;
constexpr int64_t kMaxWidth = 1048576;

}  // namespace

extern "C" {

bitnet_status bitnet_norm_quantize(const void* x, int x_dtype, const void* residual, void* residual_out, int residual_dtype,
                                   const float* gamma, float eps, int64_t M, int64_t K, void* y, int y_dtype, int8_t* xq,
                                   float* x_scale, int32_t* x_rowsum, void* stream) {
    if (!dtype_ok(x_dtype) || (residual && !dtype_ok(residual_dtype)) || (y && !dtype_ok(y_dtype)))
        return st(fail(BITNET_E_INVALID, "unknown dtype (x %d, residual %d, y %d)", x_dtype, residual_dtype, y_dtype));
    if (residual && x_dtype != BITNET_DTYPE_F32 && x_dtype != residual_dtype)
        return st(fail(BITNET_E_INVALID, "x_dtype %d: f32 (0) or the residual's (%d) is needed", x_dtype, residual_dtype));
    if (residual_out && !residual) return st(fail(BITNET_E_INVALID, "residual_out without a residual"));
    if (!(eps > 0.0f) || !isfinite(eps)) return st(fail(BITNET_E_INVALID, "eps must be positive and finite"));
    if (M < 0 || M > kMaxRows || K < 1 || K > kMaxWidth)
        return st(fail(BITNET_E_SHAPE, "need 0 <= M <= 2^24 and 1 <= K <= %lld; got M=%lld K=%lld", (long long)kMaxWidth, (long long)M,
                       (long long)K));
    if (M == 0) return st(hip_status(hipSuccess, ""));
    if (!x) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!y && !xq) return st(fail(BITNET_E_INVALID, "nothing to write: y or xq is needed"));
    if ((xq != nullptr) != (x_scale != nullptr)) return st(fail(BITNET_E_INVALID, "xq and x_scale go together"));
    if (x_rowsum && !xq) return st(fail(BITNET_E_INVALID, "x_rowsum without xq"));
    if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(residual_out, 16) || !aligned(gamma, 16) || !aligned(y, 16) ||
        !aligned(xq, 16) || !aligned(x_scale, 4) || !aligned(x_rowsum, 4))
        return st(fail(BITNET_E_ALIGN, "rows, gamma and xq need 16-byte alignment, x_scale and x_rowsum 4-byte"));
    const int64_t n = M * K;
    const Span in[3] = {{x, n * size_of(x_dtype), x_dtype}, {residual, n * size_of(residual_dtype), residual_dtype}, {gamma, 4 * K, -1}};
    const Span out[5] = {{residual_out, n * size_of(residual_dtype), residual_dtype}, {y, n * size_of(y_dtype), y_dtype}, {xq, n, -2},
                         {x_scale, 4 * M, -3}, {x_rowsum, 4 * M, -4}};
    for (int i = 0; i < 5; ++i) {
        for (const Span& s : in)
            if (overlap(out[i], s) && !(out[i].p == s.p && out[i].dtype == s.dtype))
                return st(fail(BITNET_E_INVALID, "an output may be x or the residual, of its type, and overlap no input otherwise"));
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return st(fail(BITNET_E_INVALID, "outputs overlap"));
    }
    const bitnet::NormArgs a{x, residual, residual_out, gamma, y, xq, x_scale, x_rowsum, 0, (int)K, y_dtype, eps};
    return st(hip_status(bitnet::launch_norm_quantize(a, x_dtype, residual ? residual_dtype : x_dtype, M, (hipStream_t)stream),
                         "bitnet_norm_quantize launch"));
}

bitnet_status bitnet_rope_freqs(int scaling, double theta, int64_t rot_dim, double factor, double original, double low, double high,
                                double* freqs, void* stream) {
    if (scaling < BITNET_ROPE_NONE || scaling > BITNET_ROPE_INDEX) return st(fail(BITNET_E_INVALID, "unknown scaling %d", scaling));
    if (rot_dim < 2 || rot_dim > 256 || rot_dim % 2) return st(fail(BITNET_E_SHAPE, "need an even rot_dim, 2 <= rot_dim <= 256; got %lld", (long long)rot_dim));
    if (!(theta > 1.0) || !isfinite(theta)) return st(fail(BITNET_E_INVALID, "theta must be finite and above 1"));
    if (scaling != BITNET_ROPE_NONE && (!(factor > 0.0) || !isfinite(factor))) return st(fail(BITNET_E_INVALID, "factor must be positive and finite"));
    if (scaling == BITNET_ROPE_BASE && rot_dim < 4) return st(fail(BITNET_E_SHAPE, "a larger base needs rot_dim >= 4"));
    if (scaling >= BITNET_ROPE_TURNS && (!(original > 0.0) || !isfinite(original) || !(low > 0.0) || !(high > low) || !isfinite(high)))
        return st(fail(BITNET_E_INVALID, "need original > 0 and 0 < low < high"));
    if (!freqs) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(freqs, 8)) return st(fail(BITNET_E_ALIGN, "freqs needs 8-byte alignment"));
    const bitnet::RopeScaling r{theta, factor, original, low, high, scaling};
    return st(hip_status(bitnet::launch_rope_freqs(r, (int)rot_dim, freqs, (hipStream_t)stream), "bitnet_rope_freqs launch"));
}

bitnet_status bitnet_rope(const bitnet_rotation* rotation, const void* x, int dtype, int64_t n_tokens, int64_t n_heads,
                          int64_t head_dim, const int32_t* pos, void* out, void* stream) {
    if (!dtype_ok(dtype)) return st(fail(BITNET_E_INVALID, "unknown dtype %d", dtype));
    if (n_tokens < 0 || n_tokens > kMaxRows || n_heads < 1 || n_heads > 1024 || head_dim < 4 || head_dim > 256 || head_dim % 4)
        return st(fail(BITNET_E_SHAPE, "need 0 <= n_tokens <= 2^24, 1 <= n_heads <= 1024, head_dim %% 4 == 0, 4 <= head_dim <= 256; got "
                       "n_tokens=%lld n_heads=%lld head_dim=%lld", (long long)n_tokens, (long long)n_heads, (long long)head_dim));
    const bool work = n_tokens > 0;
    if (const int e = bitnet::check_rotation(rotation, head_dim, work)) return st(e);
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!x || !pos || !out) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(pos, 4))
        return st(fail(BITNET_E_ALIGN, "x and out need 16-byte alignment, pos 4-byte"));
    const int64_t bytes = n_tokens * n_heads * head_dim * size_of(dtype);
    if (x != out && overlap({x, bytes, 0}, {out, bytes, 0})) return st(fail(BITNET_E_INVALID, "out must be x or not overlap it"));
    return st(hip_status(bitnet::launch_rope(bitnet::rope_of(rotation), dtype, x, n_tokens, (int)n_heads, (int)head_dim, pos, out,
                                             (hipStream_t)stream),
                         "bitnet_rope launch"));
}

}  // extern "C"

namespace bitnet {

int check_rotation(const bitnet_rotation* r, int64_t head_dim, bool pointers) {
    if (!r) return fail(BITNET_E_INVALID, "null rotation");
    if (r->rot_dim < 2 || r->rot_dim > head_dim || r->rot_dim % 2)
        return fail(BITNET_E_SHAPE, "need an even rot_dim, 2 <= rot_dim <= head_dim; got %lld of %lld", (long long)r->rot_dim, (long long)head_dim);
    if (r->interleaved != 0 && r->interleaved != 1) return fail(BITNET_E_INVALID, "interleaved must be 0 or 1, got %d", r->interleaved);
    if (!pointers) return BITNET_OK;
    if (!r->freqs) return fail(BITNET_E_INVALID, "null freqs");
    if (!aligned(r->freqs, 8)) return fail(BITNET_E_ALIGN, "freqs needs 8-byte alignment");
    return BITNET_OK;
}

Rope rope_of(const bitnet_rotation* r) { return {r->freqs, (int)r->rot_dim, r->interleaved, r->gain}; }

}  // namespace bitnet
