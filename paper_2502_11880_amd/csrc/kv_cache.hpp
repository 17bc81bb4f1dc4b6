// The paged key-value cache: geometry, device helpers and host launchers shared by its kernels.
//
// A page holds ps tokens (16, 32, 64, 128 or 256) of every kv head:
//   keys    [Hkv, C, ps, 8], C = ceil(D / 8): chunk c of a token is its channels 8c .. 8c+7 (zeros past D);
//   values  [Hkv, ps / 8, D, 8]: channel d of eight consecutive tokens in one 16-byte word.
// Both are what one lane reads as its operand of a matrix instruction: S^T = K Q^T contracts over channels and takes 8
// channels of one key per lane, O^T = V^T P^T contracts over keys and takes 8 keys of one channel per lane.  So the values
// need no transposing when they are read, and a wave's loads are runs of 128 bytes (ps = 16: keys of two pages) and more.
// The price is paid once, when a token is appended: its values go out as single elements 16 bytes apart.
#pragma once

#include "bitnet_internal.hpp"
#include "status.hpp"

namespace bitnet {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types (the values of bitnet_dtype).
constexpr int kF32 = 0, kBf16 = 1, kF16 = 2;

struct KvCache {
    uint16_t* k;
    uint16_t* v;
    const int32_t* table;     // [n_seqs, max_pages]
    const int32_t* kv_len;    // [n_seqs]
    int64_t k_page, v_page;   // elements of one page
    int n_pages, max_pages, n_seqs;
    int shift;                // ps = 1 << shift
    int kv_heads, dim, chunks;
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();

// Tokens of sequence b that the cache can hold in its row of the table.
__device__ __forceinline__ int seq_len(const KvCache& c, int b) {
    const int n = c.kv_len[b], most = c.max_pages << c.shift;
    return n < 0 ? 0 : n < most ? n : most;
}

// A table entry that names a page of the pool; others stand for keys that are not there.
__device__ __forceinline__ bool page_ok(const KvCache& c, int page) { return (unsigned)page < (unsigned)c.n_pages; }

// The largest b in [0, n) with f(b) <= x, for increasing f with f(0) <= x: 64 lanes probe at once.  Whole waves only.
template <typename F>
__device__ __forceinline__ int find_last(int n, int x, F f) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int at = lane * step;
        const bool in = at < n && f(lo + (at < n ? at : 0)) <= x;
        const int count = __popcll(__ballot(in));
        const int skip = (count > 0 ? count - 1 : 0) * step;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    return lo;
}

// First token and number of tokens of sequence b in a ragged batch of n_tokens (q_start null: one each).
struct Span {
    int first, count;
};
__device__ __forceinline__ Span span_of(const int32_t* q_start, int b, int n_tokens) {
    if (!q_start) return {b, b < n_tokens ? 1 : 0};
    const int s = q_start[b], e = q_start[b + 1];
    if (s < 0 || e < s || e > n_tokens) return {0, 0};
    return {s, e - s};
}

// Other lanes' values of a float: the lane 16 and the lane 32 away.
__device__ __forceinline__ float max_xor16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_xor32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The cache's element types: conversions, matrix instructions, and 32-bit values as a sum of parts of that type.
// bf16: a part keeps the upper 16 bits of what is left (truncated, so every part has the value's sign); three parts hold all
// 24 bits of a value, which is exact, and two hold 16 (cut off: less than 2^-15 of it).  f16: a part is rounded to nearest; two parts
// hold 22 bits of a value near the top of the range, so values are brought there by a power of two first.  What is left out then,
// 2^-23 of a value or 2^-38 of its row's largest, is of the size of the roundings that 32-bit sums make anyway, and a third
// part would cost a third product.
template <int T>
struct Elem;

template <>
struct Elem<kBf16> {
    static constexpr int kExactParts = 3;
    static __device__ __forceinline__ uint16_t from(float x) {
        return __builtin_bit_cast(uint16_t, (__bf16)x);
    }
    static __device__ __forceinline__ float to(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {   // rounded to nearest even
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), bf16x2));
    }
    // sum + both values of a word
    static __device__ __forceinline__ float add2(uint32_t w, float sum) {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
    }
    // the leading part of two values, which lose it
    static __device__ __forceinline__ uint32_t part(float& a, float& b) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        a -= __uint_as_float(x & 0xFFFF0000u);
        b -= __uint_as_float(y & 0xFFFF0000u);
        return __builtin_amdgcn_perm(y, x, 0x07060302u);
    }
    static __device__ __forceinline__ v4f mfma16(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v16f mfma32(v4u a, v4u b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

template <>
struct Elem<kF16> {
    static constexpr int kExactParts = 2;
    static __device__ __forceinline__ uint16_t from(float x) {
        return __builtin_bit_cast(uint16_t, (_Float16)x);
    }
    static __device__ __forceinline__ float to(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), f16x2));
    }
    static __device__ __forceinline__ float add2(uint32_t w, float sum) {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), __builtin_bit_cast(f16x2, 0x3C003C00u), sum, false);
    }
    static __device__ __forceinline__ uint32_t part(float& a, float& b) {
        const f16x2 x = __builtin_convertvector((v2f{a, b}), f16x2);
        const uint32_t w = __builtin_bit_cast(uint32_t, x);
        // a - x[0] and b - x[1], exact, from the 16 bits in place (the compiler would convert them first)
        asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(a) : "v"(w), "v"(a));
        asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(b) : "v"(w), "v"(b));
        return w;
    }
    static __device__ __forceinline__ v4f mfma16(v4u a, v4u b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ v16f mfma32(v4u a, v4u b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// All ones in the halves of a word that hold an infinity or NaN of type T.
template <int T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t e = T == kBf16 ? 0x7F807F80u : 0x7C007C00u, one = T == kBf16 ? 0x00800080u : 0x04000400u;
    return ((((w & e) + one) & 0x80008000u) >> 15) * 0xFFFFu;
}
// A half that is not finite as a finite mark of its kind (1, 128 and 16384 for +inf, -inf and NaN), others as 0: marks of up to
// 64 keys add up without mixing.
template <int T>
__device__ __forceinline__ uint32_t mark_half(uint32_t h) {
    constexpr uint32_t inf = T == kBf16 ? 0x7F80u : 0x7C00u;
    constexpr uint32_t one = T == kBf16 ? 0x3F80u : 0x3C00u, b = T == kBf16 ? 0x4300u : 0x5800u, c = T == kBf16 ? 0x4680u : 0x7400u;
    return (h & 0x7FFFu) < inf ? 0u : h == inf ? one : h == (inf | 0x8000u) ? b : c;
}
// The halves of a word that are infinite as 1 or -1, others as 0; and the halves that are no 0 as 1 or -1, 0 as 0.
template <int T>
__device__ __forceinline__ uint32_t sign_of_infinite(uint32_t w) {
    constexpr uint32_t inf = T == kBf16 ? 0x7F80u : 0x7C00u, one = T == kBf16 ? 0x3F80u : 0x3C00u;
    const uint32_t a = w & 0xFFFFu, b = w >> 16;
    return ((a & 0x7FFFu) == inf ? one | (a & 0x8000u) : 0u) | ((b & 0x7FFFu) == inf ? one | (b & 0x8000u) : 0u) << 16;
}
template <int T>
__device__ __forceinline__ uint32_t sign_of(uint32_t w) {
    constexpr uint32_t one = T == kBf16 ? 0x3F80u : 0x3C00u;
    return (w & 0x7FFFu ? one | (w & 0x8000u) : 0u) | (w & 0x7FFF0000u ? one << 16 | (w & 0x80000000u) : 0u);
}
__device__ __forceinline__ float unmark(float sum) {
    const int n = (int)sum;
    const bool pos = (n & 127) != 0, neg = ((n >> 7) & 127) != 0;
    return n >= 16384 || (pos && neg) ? __builtin_nanf("") : pos ? -kNegInf : neg ? kNegInf : 0.0f;
}

__device__ __forceinline__ bool all_finite(const v4f& x) {
    return x[0] * 0.0f + x[1] * 0.0f + (x[2] * 0.0f + x[3] * 0.0f) == 0.0f;
}
// more + those of x that are not finite: what is left of partial outputs whose factors may be 0 in 32 bits.
__device__ __forceinline__ v4f add_infinite(v4f more, const v4f& x) {
#pragma unroll
    for (int t = 0; t < 4; ++t) more[t] += x[t] * 0.0f == 0.0f ? 0.0f : x[t];
    return more;
}
// o, but where a sum of infinite values has something
__device__ __forceinline__ v4f or_infinite(v4f o, const v4f& sum) {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = sum[t] == 0.0f ? o[t] : sum[t];
    return o;
}

// The softmax weights are exp2(x - m + kLift<T>): f16 parts hold small weights best near the top of their range.
template <int T>
constexpr float kLift = T == kF16 ? 14.0f : 0.0f;

// 2^e that brings a row whose largest |value| is `top` to [2^13, 2^14), in the exponents a float can scale by; 1 where the row
// is all zeros or not finite.  Only for f16.
__device__ __forceinline__ float row_gain(float top) {
    const int e = (int)((__float_as_uint(top) >> 23) & 0xFF);
    if (top == 0.0f || e == 255) return 1.0f;
    int shift = 13 - (e - 127);
    shift = shift < -100 ? -100 : shift > 100 ? 100 : shift;
    return __uint_as_float((uint32_t)(127 + shift) << 23);
}

// Four values of an input row that are 32-bit floats or of the cache's type T (8-byte aligned).
template <int T, bool F32>
__device__ __forceinline__ float4 load4(const void* p, int64_t at) {
    if constexpr (F32) {
        return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
        return make_float4(Elem<T>::to((uint16_t)w.x), Elem<T>::to((uint16_t)(w.x >> 16)), Elem<T>::to((uint16_t)w.y),
                           Elem<T>::to((uint16_t)(w.y >> 16)));
    }
}
template <int T, bool F32>
__device__ __forceinline__ void store4(void* p, int64_t at, float a, float b, float c, float d) {
    if constexpr (F32) {
        *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(a, b, c, d);
    } else {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + at) = make_uint2(Elem<T>::pack(a, b), Elem<T>::pack(c, d));
    }
}

// ------------------------------------------------------------------------------------------------
// Host launchers (arguments checked by the caller)
// ------------------------------------------------------------------------------------------------
hipError_t launch_kv_append(const KvCache& c, int dtype, const void* k, const void* v, bool f32, const int32_t* q_start,
                            int n_tokens, hipStream_t s);

struct AttnArgs {
    const void* q;
    void* out;
    const int32_t* q_start;   // prefill
    int n_tokens, heads;
    float scale;
    int window, n_sink;       // window 0: none
    bool f32;                 // q and out in 32 bits, else in the cache's type
};
// Decode: bytes for the partial results of rows that are split (0 where none can be, whatever the number of sequences), and
// whether a call splits any.
size_t attn_decode_workspace_bytes(int heads, int kv_heads, int dim, int page_size, int64_t max_pages, int window, int n_sink);
bool attn_decode_splits(int64_t n_seqs, int heads, int kv_heads, int page_size, int64_t max_pages, int window, int n_sink);
hipError_t launch_attn_decode(const KvCache& c, int dtype, const AttnArgs& a, void* ws, hipStream_t s);
// Prefill: ws null or smaller than this: nothing is split.
size_t attn_prefill_workspace_bytes(int64_t n_seqs, int64_t n_tokens, int heads, int kv_heads, int dim, int page_size,
                                    int64_t max_pages, int window, int n_sink, bool three_parts, bool f32);
hipError_t launch_attn_prefill(const KvCache& c, int dtype, const AttnArgs& a, void* ws, size_t ws_bytes, hipStream_t s);

// A pool: n_layers planes of keys and of values, each n_pages pages of k_bytes / v_bytes.
struct KvPool {
    uint8_t* k;
    uint8_t* v;
    int n_layers, n_pages;
    int64_t k_bytes, v_bytes;
};
struct KvTables {
    int32_t* table;           // [n_seqs, max_pages]
    int32_t* kv_len;          // [n_seqs]
    int32_t* refs;            // [n_pages]
    int n_seqs, max_pages, n_pages;
};
size_t kv_workspace_bytes(int64_t n_pages, int64_t n_seqs);
hipError_t launch_kv_copy(const KvPool& p, const int32_t* src, const int32_t* dst, int n, hipStream_t s);
hipError_t launch_kv_free(const KvTables& t, const int32_t* seqs, int n, hipStream_t s);
hipError_t launch_kv_trim(const KvTables& t, const int32_t* seqs, int n, int shift, int window, int n_sink, hipStream_t s);
hipError_t launch_kv_reserve(const KvTables& t, const int32_t* seqs, const int32_t* n_new, int n, int shift, int32_t* n_short,
                             void* ws, hipStream_t s);
hipError_t launch_kv_fork(const KvPool& p, const KvTables& t, const int32_t* parents, const int32_t* children, int n,
                          int shift, int32_t* n_short, void* ws, hipStream_t s);
hipError_t launch_kv_compact(const KvPool& p, const KvTables& t, int32_t* n_live, void* ws, hipStream_t s);

}  // namespace bitnet
