// New tokens' keys rotated by their positions and written into their pages with the values, and the query heads of the same
// tokens rotated on the way: token i of sequence b is at position kv_len[b] - n_b + i.
//
// Memory bounds it: every row is read once, q and the cache's type written once.  Units of eight consecutive positions as in
// the append without rotation (the values' layout wants them); their angles are worked out once a work group (in 64 bits, see
// turn_of), shared through LDS, and used by all heads that it takes.
//
// Measured (kernel times): five prompts of up to 3001 tokens, 32 heads of 8 kv heads of 128, 32 bits into bf16, 79 us (381 MB, 4.8
// TB/s; a large copy reaches 5.0); one token each of 64 sequences 6.3; nine chunks of up to 509 tokens, 32 heads of 100, f16, 22 us
// where the pages are in the last cache, 30 to 31 a pass where they are not (3.1 TB/s), in pages of 16 as of 256; from 32 bits 40 (3.8
// TB/s): values of 16-bit rows are read two bytes a lane.
#include "rows.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;
constexpr int kWantGroups = 4096;    // sixteen work groups a CU

// Units of sequence b start at floor(q_start[b] / 8) + 2 b: its tokens touch at most ceil(n / 8) + 1 of them.
__device__ __forceinline__ int first_unit(const int32_t* q_start, int b) { return (q_start ? q_start[b] : b) / 8 + 2 * b; }

// T: the cache's type; I: the rows' (32 bits or T).
template <int T, int I>
__global__ __launch_bounds__(kThreads) void kv_append_rope_kernel(KvCache c, Rope r, const void* q, int group, const void* k, const void* v,
                                                                  void* q_out, const int32_t* q_start, int n_tokens, int heads) {
    __shared__ float2 turns[8][kMostPairs];
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
    const int page = at < c.max_pages ? c.table[(int64_t)b * c.max_pages + at] : -1;
    const int first = base > low ? base : low, last = len - base < 8 ? len : base + 8;   // positions of the unit

    const int pairs = r.rot >> 1;
    const int steps = (last - first) * pairs;
    for (int i = threadIdx.x; i < steps; i += kThreads) {
        const int t = i / pairs, pair = i - t * pairs;
        turns[first - base + t][pair] = turn_of(r, pair, first + t);
    }
    __syncthreads();

    const int h0 = blockIdx.y * heads, h1 = h0 + heads < c.kv_heads ? h0 + heads : c.kv_heads;
    const int64_t row0 = (int64_t)span.first - p0;        // row of position p: row0 + p
    if (q) {
        const Items items = items_of(r, c.dim);
        const int at_once = kThreads / items.all, mine = threadIdx.x / items.all, i = threadIdx.x - mine * items.all;
        const int count = (h1 - h0) * group;              // query heads of a token here
        const int rows = count * (last - first);
        if (mine < at_once && (i < items.turning || q != q_out)) {
            for (int j = mine; j < rows; j += at_once) {
                const int t = j / count, h = h0 * group + j - t * count;
                const int64_t head = ((row0 + first + t) * c.kv_heads * group + h) * c.dim;
                turn_item<I>(r, items, i, q, q_out, head, turns[first - base + t]);
            }
        }
    }
    if (!page_ok(c, page)) return;
    const int ps = 1 << c.shift, slot = base & (ps - 1);
    const int64_t row_step = (int64_t)c.kv_heads * c.dim;
    uint16_t* kp = c.k + (int64_t)page * c.k_page + (int64_t)slot * 8;
    uint16_t* vp = c.v + (int64_t)page * c.v_page + (int64_t)slot * c.dim;

    // keys: eight threads a chunk, one for each token
    const int p = base + (threadIdx.x & 7);
    if (p >= first && p < last) {
        const int64_t k_row = (row0 + p) * row_step;
        const float2* turn = turns[threadIdx.x & 7];
        for (int i = h0 * c.chunks + (threadIdx.x >> 3); i < h1 * c.chunks; i += kThreads / 8) {
            const int h = i / c.chunks, d = 8 * (i - h * c.chunks);
            const float4 x = turned_quad<I>(r, k, k_row + h * c.dim, d, turn);
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (d + 4 < c.dim) y = turned_quad<I>(r, k, k_row + h * c.dim, d + 4, turn);
            *reinterpret_cast<uint4*>(kp + ((int64_t)i * ps + (threadIdx.x & 7)) * 8) =
                make_uint4(Elem<T>::pack(x.x, x.y), Elem<T>::pack(x.z, x.w), Elem<T>::pack(y.x, y.y), Elem<T>::pack(y.z, y.w));
        }
    }
    // values: a thread a channel of the eight tokens
    const int64_t v_row = (row0 + base) * row_step;
    const bool whole = first == base && last == base + 8;
    for (int i = h0 * c.dim + threadIdx.x; i < h1 * c.dim; i += kThreads) {
        const int h = i / c.dim, d = i - h * c.dim;
        uint16_t* dst = vp + ((int64_t)h * ps * c.dim + d * 8);
        if (whole) {
            float e[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) e[t] = load_one<I>(v, v_row + t * row_step + i);
            *reinterpret_cast<uint4*>(dst) = make_uint4(Elem<T>::pack(e[0], e[1]), Elem<T>::pack(e[2], e[3]), Elem<T>::pack(e[4], e[5]), Elem<T>::pack(e[6], e[7]));
        } else {
            for (int t = first - base; t < last - base; ++t) dst[t] = Elem<T>::from(load_one<I>(v, v_row + t * row_step + i));
        }
    }
}

}  // namespace

hipError_t launch_kv_append_rope(const KvCache& c, int dtype, const void* q, int heads, const void* k, const void* v, bool f32,
                                 const int32_t* q_start, int n_tokens, const Rope& r, void* q_out, hipStream_t s) {
    const int64_t units = q_start ? (int64_t)n_tokens / 8 + 2 * (int64_t)c.n_seqs : c.n_seqs;
    const int64_t want = (kWantGroups + units - 1) / units;
    const int splits = (int)(want < c.kv_heads ? want : c.kv_heads), per = (c.kv_heads + splits - 1) / splits;
    const dim3 grid((unsigned)units, (unsigned)((c.kv_heads + per - 1) / per));
    const int group = heads / c.kv_heads;
    const auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, c, r, q, group, k, v, q_out, q_start, n_tokens, per);
    };
    if (dtype == kBf16) f32 ? launch(kv_append_rope_kernel<kBf16, kF32>) : launch(kv_append_rope_kernel<kBf16, kBf16>);
    else f32 ? launch(kv_append_rope_kernel<kF16, kF32>) : launch(kv_append_rope_kernel<kF16, kF16>);
    return hipGetLastError();
}

}  // namespace bitnet
