// New tokens' keys and values written into their pages: token i of sequence b goes to position kv_len[b] - n_b + i.
//
// Memory bounds it: the rows are read once, the cache's type is written once.  Eight consecutive positions are one unit,
// because that is a word of the values' layout: a thread collects one channel of the eight tokens (its neighbours the next
// channels: whole rows are read) and writes 16 bytes; keys go as one thread a token and eight channels, tokens side by side.
// A unit that starts or ends inside such a word writes its values as single elements.
#include "kv_cache.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;

// Units of sequence b start at floor(q_start[b] / 8) + 2 b: its tokens touch at most ceil(n / 8) + 1 of them, which never
// reach the next sequence's, so no prefix sum is needed (a few units stay empty).
__device__ __forceinline__ int first_unit(const int32_t* q_start, int b) { return (q_start ? q_start[b] : b) / 8 + 2 * b; }

template <int T, bool F32>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvCache c, const void* k, const void* v, const int32_t* q_start,
                                                             int n_tokens) {
    const int id = blockIdx.x;
    const int b = q_start ? find_last(c.n_seqs, id, [&](int i) { return first_unit(q_start, i); }) : id;
    const Span span = span_of(q_start, b, n_tokens);
    const int len = c.kv_len[b], p0 = len - span.count;
    const int low = p0 > 0 ? p0 : 0;
    const int unit = (low >> 3) + (q_start ? id - first_unit(q_start, b) : 0);
    const int base = unit * 8;
    if (base >= len || span.count == 0) return;
    const int at = base >> c.shift;
    if (at >= c.max_pages) return;
    const int page = c.table[(int64_t)b * c.max_pages + at];
    if (!page_ok(c, page)) return;
    const int ps = 1 << c.shift, slot = base & (ps - 1);
    const int h = blockIdx.y;
    const int64_t row0 = (int64_t)span.first - p0;        // row of position p: row0 + p
    uint16_t* kp = c.k + (int64_t)page * c.k_page + (int64_t)h * c.chunks * ps * 8;
    uint16_t* vp = c.v + (int64_t)page * c.v_page + (int64_t)h * c.dim * ps + (int64_t)slot * c.dim;
    const int k_items = c.chunks * 8;
    for (int i = threadIdx.x; i < k_items + c.dim; i += kThreads) {
        if (i < k_items) {
            const int p = base + (i & 7), chunk = i >> 3;
            if (p < low || p >= len) continue;
            const int64_t src = ((row0 + p) * c.kv_heads + h) * c.dim + 8 * chunk;
            const float4 x = load4<T, F32>(k, src);
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (8 * chunk + 4 < c.dim) y = load4<T, F32>(k, src + 4);
            *reinterpret_cast<uint4*>(kp + ((int64_t)chunk * ps + slot + (i & 7)) * 8) =
                make_uint4(Elem<T>::pack(x.x, x.y), Elem<T>::pack(x.z, x.w), Elem<T>::pack(y.x, y.y), Elem<T>::pack(y.z, y.w));
        } else {
            const int d = i - k_items;
            uint16_t e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int p = base + t;
                e[t] = 0;
                if (p < low || p >= len) continue;
                const int64_t src = ((row0 + p) * c.kv_heads + h) * c.dim + d;
                if constexpr (F32) e[t] = Elem<T>::from(static_cast<const float*>(v)[src]);
                else e[t] = static_cast<const uint16_t*>(v)[src];
            }
            uint16_t* dst = vp + (int64_t)d * 8;
            if (base >= low && base + 8 <= len) {
                *reinterpret_cast<uint4*>(dst) =
                    make_uint4((uint32_t)e[0] | (uint32_t)e[1] << 16, (uint32_t)e[2] | (uint32_t)e[3] << 16,
                               (uint32_t)e[4] | (uint32_t)e[5] << 16, (uint32_t)e[6] | (uint32_t)e[7] << 16);
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    if (base + t >= low && base + t < len) dst[t] = e[t];
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const KvCache& c, int dtype, const void* k, const void* v, bool f32, const int32_t* q_start,
                            int n_tokens, hipStream_t s) {
    const int64_t units = q_start ? (int64_t)n_tokens / 8 + 2 * (int64_t)c.n_seqs : c.n_seqs;
    const dim3 grid((unsigned)units, (unsigned)c.kv_heads);
    if (dtype == kBf16) {
        if (f32) hipLaunchKernelGGL((kv_append_kernel<kBf16, true>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens);
        else hipLaunchKernelGGL((kv_append_kernel<kBf16, false>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens);
    } else {
        if (f32) hipLaunchKernelGGL((kv_append_kernel<kF16, true>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens);
        else hipLaunchKernelGGL((kv_append_kernel<kF16, false>), grid, dim3(kThreads), 0, s, c, k, v, q_start, n_tokens);
    }
    return hipGetLastError();
}

}  // namespace bitnet
