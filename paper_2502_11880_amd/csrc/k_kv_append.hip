// New tokens' keys and values written into their pages: token i of sequence b goes to position kv_len[b] - n_b + i.
//
// Memory bounds it: the rows are read once, the cache's type is written once.  Eight consecutive positions are one unit,
// because that is a word of the values' layout: a thread collects one channel of the eight tokens (its neighbours the next
// channels: whole rows are read) and writes 16 bytes; keys go as one thread a token and eight channels, tokens side by side.
// A unit that starts or ends inside such a word writes its values as single elements.
//
// Measured: five prompts, 8461 tokens in all, 32 heads of 100, 32 bits into f16, 74 us (325 MB, 4.4 TB/s; a large copy
// reaches 4.9); one token each of 64 sequences 5 us, of which a launch that does nothing takes 1.7: four reads in a row
// (length, page, row) before the first write.
#include "kv_cache.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;
constexpr int kWantGroups = 4096;    // sixteen work groups a CU (those prompts: 74 us, with eight a CU 78, four 85, 32 74)

// Units of sequence b start at floor(q_start[b] / 8) + 2 b: its tokens touch at most ceil(n / 8) + 1 of them, which never
// reach the next sequence's, so no prefix sum is needed (a few units stay empty).
__device__ __forceinline__ int first_unit(const int32_t* q_start, int b) { return (q_start ? q_start[b] : b) / 8 + 2 * b; }

template <int T, bool F32>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvCache c, const void* k, const void* v, const int32_t* q_start,
                                                             int n_tokens, int heads) {
    const int id = blockIdx.x;
    const int b = q_start ? find_last(c.n_seqs, id, [&](int i) { return first_unit(q_start, i); }) : id;
    const Span span = span_of(q_start, b, n_tokens);
    const int len = c.kv_len[b], p0 = len - span.count;
    const int low = p0 > 0 ? p0 : 0;
    const int unit = (low >> 3) + (q_start ? id - first_unit(q_start, b) : 0);
    const int base = unit * 8;
    // below 0: units before the first sequence's (offsets that start past 0 or decrease), lengths next to 2^31
    if (base < 0 || base >= len || span.count == 0) return;
    const int at = base >> c.shift;
    if (at >= c.max_pages) return;
    const int page = c.table[(int64_t)b * c.max_pages + at];
    if (!page_ok(c, page)) return;
    const int ps = 1 << c.shift, slot = base & (ps - 1);
    const int h0 = blockIdx.y * heads, h1 = h0 + heads < c.kv_heads ? h0 + heads : c.kv_heads;
    const int64_t row0 = (int64_t)span.first - p0;        // row of position p: row0 + p
    const int64_t row_step = (int64_t)c.kv_heads * c.dim;
    uint16_t* kp = c.k + (int64_t)page * c.k_page + (int64_t)slot * 8;
    uint16_t* vp = c.v + (int64_t)page * c.v_page + (int64_t)slot * c.dim;

    // keys: eight threads a chunk, one for each token
    const int p = base + (threadIdx.x & 7);
    const int64_t k_row = (row0 + p) * row_step;
    const int first_chunk = h0 * c.chunks, last_chunk = h1 * c.chunks;
    if (p >= low && p < len) {
#pragma unroll 2
        for (int i = first_chunk + (threadIdx.x >> 3); i < last_chunk; i += kThreads / 8) {
            const int h = i / c.chunks, chunk = i - h * c.chunks;
            const int64_t src = k_row + h * c.dim + 8 * chunk;
            const float4 x = load4<T, F32>(k, src);
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (8 * chunk + 4 < c.dim) y = load4<T, F32>(k, src + 4);
            *reinterpret_cast<uint4*>(kp + ((int64_t)i * ps + (threadIdx.x & 7)) * 8) =
                make_uint4(Elem<T>::pack(x.x, x.y), Elem<T>::pack(x.z, x.w), Elem<T>::pack(y.x, y.y), Elem<T>::pack(y.z, y.w));
        }
    }
    // values: a thread a channel of the eight tokens
    const bool whole = base >= low && base + 8 <= len;
    const int64_t v_row = (row0 + base) * row_step;
    for (int i = h0 * c.dim + threadIdx.x; i < h1 * c.dim; i += kThreads) {
        const int h = i / c.dim, d = i - h * c.dim;
        uint16_t* dst = vp + ((int64_t)h * ps * c.dim + d * 8);
        if (whole) {
            uint32_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int64_t src = v_row + t * row_step + i;
                if constexpr (F32) e[t] = __float_as_uint(static_cast<const float*>(v)[src]);
                else e[t] = static_cast<const uint16_t*>(v)[src];
            }
            uint4 w;
            if constexpr (F32)
                w = make_uint4(Elem<T>::pack(__uint_as_float(e[0]), __uint_as_float(e[1])), Elem<T>::pack(__uint_as_float(e[2]), __uint_as_float(e[3])),
                               Elem<T>::pack(__uint_as_float(e[4]), __uint_as_float(e[5])), Elem<T>::pack(__uint_as_float(e[6]), __uint_as_float(e[7])));
            else
                w = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
            *reinterpret_cast<uint4*>(dst) = w;
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if (base + t < low || base + t >= len) continue;
                const int64_t src = v_row + t * row_step + i;
                if constexpr (F32) dst[t] = Elem<T>::from(static_cast<const float*>(v)[src]);
                else dst[t] = static_cast<const uint16_t*>(v)[src];
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const KvCache& c, int dtype, const void* k, const void* v, bool f32, const int32_t* q_start,
                            int n_tokens, hipStream_t s) {
    const int64_t units = q_start ? (int64_t)n_tokens / 8 + 2 * (int64_t)c.n_seqs : c.n_seqs;
    // A prompt's units keep the device busy by themselves and one work group takes all heads of a unit (fewer, longer groups:
    // what a group looks up before its first row, four dependent reads, then costs little); few units are split by heads.
    const int64_t want = (kWantGroups + units - 1) / units;
    const int splits = (int)(want < c.kv_heads ? want : c.kv_heads), heads = (c.kv_heads + splits - 1) / splits;
    const dim3 grid((unsigned)units, (unsigned)((c.kv_heads + heads - 1) / heads));
    if (dtype == kBf16) {
        if (f32) hipLaunchKernelGGL((kv_append_kernel<kBf16, true>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens, heads);
        else hipLaunchKernelGGL((kv_append_kernel<kBf16, false>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens, heads);
    } else {
        if (f32) hipLaunchKernelGGL((kv_append_kernel<kF16, true>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens, heads);
        else hipLaunchKernelGGL((kv_append_kernel<kF16, false>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens, heads);
    }
    return hipGetLastError();
}

}  // namespace bitnet
