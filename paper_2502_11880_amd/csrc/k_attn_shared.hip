// Attention of one new token per sequence over the paged cache, where groups of neighbouring sequences share their first keys:
//   out[b, h] = sum_j p_j v_j,  p = softmax over the visible keys j of scale q[b, h] . k_j
// (visible as in the decode without groups: j < L, and with a window j >= L - window or j < n_sink; nothing visible: zeros).  Keys
// below the group's prefix are those of its first sequence, keys from there on the sequence's own.
//
// A wave takes one head of one sequence and walks its keys eight at a time (a word of the values) in plain 32-bit products.
#include "kv_cache.hpp"

namespace bitnet {
namespace {

constexpr int kThreads = 256;

struct SharedArgs {
    KvCache c;
    const void* q;
    void* out;
    const int32_t* group_start;
    const int32_t* prefix_len;
    int n_groups, heads, group;
    float scale2;                    // scale * log2 e
    int window, n_sink;
};

// Head h of sequence b over the keys [from, to) that it sees, in the pages of table row `row`, onto m, l, o and the values that are
// not finite (odd).  A lane holds channels d = 4 lane .. of q and of the output; every lane the maximum and the sum.
template <int T>
__device__ __forceinline__ void plain_keys(const SharedArgs& a, const float4& q, int row, int kvh, int from, int to, int len, int lo, int d,
                                           float& m, float& l, v4f& o, v4f& odd) {
    const KvCache& c = a.c;
    const int32_t* table = c.table + (int64_t)row * c.max_pages;
    const int ps = 1 << c.shift;
    const bool in = d < c.dim;
    const int ch = in ? d : 0;                            // lanes past D read the first channels and hold none
    for (int key = from & ~7; key < to; key += 8) {
        const int slot = key & (ps - 1);
        const int page = table[key >> c.shift];
        if (!page_ok(c, page)) continue;
        const int64_t k_at = (int64_t)page * c.k_page + ((int64_t)(kvh * c.chunks + (ch >> 3)) * ps + slot) * 8 + (ch & 4);
        const uint16_t* v_at = c.v + (int64_t)page * c.v_page + (int64_t)kvh * c.dim * ps + (slot >> 3) * c.dim * 8 + ch * 8;
        float x[8], top = m;
        uint32_t seen = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float4 k = load4<T, false>(c.k, k_at + 8 * e);
            x[e] = in ? q.x * k.x + q.y * k.y + (q.z * k.z + q.w * k.w) : 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t) x[e] += __int_as_float(dpp_row_step(__float_as_int(x[e]), t));
            const int j = key + e;
            const bool sees = (j >= from) & (j < to) & (j < len) & ((j >= lo) | (j < a.n_sink));
            seen |= sees ? 1u << e : 0u;
            x[e] = sees ? sum_xor32(sum_xor16(x[e])) * a.scale2 : kNegInf;
            top = fmaxf(top, x[e]);
        }
        const float alpha = m == top ? 1.0f : exp2_fast(m - top), base = (top == kNegInf ? 0.0f : top) - kLift<T>;
        m = top;
        l *= alpha;
        o *= alpha;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = exp2_fast(x[e] - base);
            l += x[e];
            if ((seen >> e) & 1) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float v = Elem<T>::to(v_at[8 * t + e]);
                    if (v * 0.0f == 0.0f) o[t] += x[e] * v;
                    else odd[t] += v;
                }
            }
        }
    }
}

template <int T, bool F32>
__global__ __launch_bounds__(kThreads) void attn_shared_kernel(SharedArgs a) {
    const KvCache& c = a.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_seq = (a.heads + 3) >> 2;
    const int b = blockIdx.x / per_seq, head = (blockIdx.x - b * per_seq) * 4 + wave;
    if (head >= a.heads) return;
    // the group that b belongs to
    int g = -1;
    for (int i = threadIdx.x & 63; __any(i < a.n_groups) && g < 0; i += 64) {
        const int start = i < a.n_groups ? a.group_start[i] : 0, end = i < a.n_groups ? a.group_start[i + 1] : 0;
        const uint64_t has = __ballot(start >= 0 && start <= b && b < end && end <= c.n_seqs);
        if (has) g = (i & ~63) + __builtin_ctzll(has);
    }
    if (g < 0) return;
    const int first = a.group_start[g];
    const int most = c.max_pages << c.shift, prefix = a.prefix_len[g] < 0 ? 0 : a.prefix_len[g] < most ? a.prefix_len[g] : most;
    const int len = seq_len(c, b), lo = a.window > 0 && len > a.window ? len - a.window : 0;
    const int d = 4 * (threadIdx.x & 63), kvh = head / a.group;
    const int64_t row = ((int64_t)b * a.heads + head) * c.dim;
    const float4 q = load4<T, F32>(a.q, row + (d < c.dim ? d : 0));
    float m = kNegInf, l = 0.0f;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f}, odd = o;
    plain_keys<T>(a, q, first, kvh, 0, prefix < len ? prefix : len, len, lo, d, m, l, o, odd);
    plain_keys<T>(a, q, b, kvh, prefix, len, len, lo, d, m, l, o, odd);
    if (d >= c.dim) return;
    o = or_infinite(o, odd);
    l = l == 0.0f ? 1.0f : l;
    store4<T, F32>(a.out, row + d, o[0] / l, o[1] / l, o[2] / l, o[3] / l);
}

}  // namespace

size_t attn_shared_workspace_bytes(int64_t n_seqs, int heads, int kv_heads, int dim) { return 0; }

hipError_t launch_attn_shared(const KvCache& c, int dtype, const AttnArgs& args, const int32_t* prefix_len, int n_groups, void* ws,
                              hipStream_t s) {
    SharedArgs a{};
    a.c = c;
    a.q = args.q;
    a.out = args.out;
    a.group_start = args.q_start;
    a.prefix_len = prefix_len;
    a.n_groups = n_groups;
    a.heads = args.heads;
    a.group = args.heads / c.kv_heads;
    a.scale2 = args.scale * kLog2e;
    a.window = args.window;
    a.n_sink = args.n_sink;
    const dim3 grid((unsigned)(c.n_seqs * ((args.heads + 3) / 4)));
    if (dtype == kBf16) {
        if (args.f32) hipLaunchKernelGGL((attn_shared_kernel<kBf16, true>), grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((attn_shared_kernel<kBf16, false>), grid, dim3(kThreads), 0, s, a);
    } else {
        if (args.f32) hipLaunchKernelGGL((attn_shared_kernel<kF16, true>), grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((attn_shared_kernel<kF16, false>), grid, dim3(kThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace bitnet
