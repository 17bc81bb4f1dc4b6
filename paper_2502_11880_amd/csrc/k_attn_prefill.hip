// Attention of a ragged batch of prompt tokens over the paged cache: the n_b tokens of sequence b are its last ones, at
// positions p = L - n_b + i, and see the keys j <= p (with a window those with j > p - window or j < n_sink):
//   out[i, h] = sum_j p_ij v_j,  p_i = softmax over the visible keys of scale q[i, h] . k_j   (none visible: zeros).
//
// The matrix instructions bound it (4 D operations a pair of query and visible key).  A work group takes 32 columns for each of
// its waves, a column being one token under one query head; the heads that share a kv head are neighbours, so one pass over
// the keys serves all of them and a tile's columns span few positions (little of a masked tile is wasted).  Keys go through
// LDS in tiles of 64, double-buffered.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 instructions: a column's scores lie in two
// lanes (maximum and sum need one exchange), and the rows of the key tiles are chosen so that a lane's scores are its operand of
// the second product.  Statistics and both products accumulate in 32 bits.  Inputs in the cache's type: weights are
// rounded once to that type (their sum is not), as the output is; 32-bit inputs go in as exact sums of parts (see Elem).
//
// A value that is not finite must not reach a query that does not see it, but 0 times it in the product is no 0.  Tiles that
// are masked for some query are looked through while they are staged; where one has such a value, the product takes the
// finite ones and a second one counts the others that each query sees.
#include "kv_cache.hpp"

namespace bitnet {
namespace {

constexpr int kTile = 64;            // keys of a tile

struct PrefillArgs {
    KvCache c;
    const void* q;
    void* out;
    const int32_t* q_start;
    int n_tokens, heads, group;
    float scale2;                    // scale * log2 e
    int window, n_sink;
    int tiles;                       // work groups of a kv head
};

// Work groups of sequence b start at floor(q_start[b] group / columns) + b.
__device__ __forceinline__ int first_tile(const int32_t* q_start, int b, int group, int columns) {
    return (int)((int64_t)q_start[b] * group / columns) + b;
}

template <int T, int DP, bool F32, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void attn_prefill_kernel(PrefillArgs a) {
    constexpr int kQParts = F32 ? Elem<T>::kExactParts : 1;
    constexpr int kPParts = F32 ? Elem<T>::kExactParts : 1;
    constexpr int kThreads = 64 * WAVES, kColumns = 32 * WAVES;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    constexpr int kWords = kTile * DP / 8;               // 16-byte words of a tile's keys (and at most of its values)
    constexpr int kLoads = kWords / kThreads;
    __shared__ uint4 kt[2][kWords];                       // [chunk][key]
    __shared__ uint4 vt[2][kWords + 32];                  // [eight keys][channel]; reads of channels past D run on
    __shared__ int odd_tile[2];                           // the last masked tile of the buffer with values that are not finite
    const KvCache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, n = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int dim = c.dim, ps = 1 << c.shift;
    const bool full = dim == DP;

    // work groups of one kv head follow each other at a distance of kv_heads (with 8 of them: on one XCD, whose L2 keeps the
    // head's keys), the last tiles, which have the most keys before them, first
    const int kvh = blockIdx.x % c.kv_heads;
    const int id = a.tiles - 1 - (int)(blockIdx.x / c.kv_heads);
    const int b = find_last(c.n_seqs, id, [&](int i) { return first_tile(a.q_start, i, a.group, kColumns); });
    const Span span = span_of(a.q_start, b, a.n_tokens);
    const int col0 = (id - first_tile(a.q_start, b, a.group, kColumns)) * kColumns;
    const int columns = span.count * a.group;
    if (col0 >= columns) return;
    const int len = seq_len(c, b);
    const int p0 = len - span.count;                      // position of the first token (below 0: it sees nothing)

    const int col = col0 + wave * 32 + n;
    const bool used = col < columns;
    const int token = (used ? col : columns - 1) / a.group, in_group = (used ? col : columns - 1) - token * a.group;
    const int pos = p0 + token;
    const int64_t row = ((int64_t)(span.first + token) * a.heads + kvh * a.group + in_group) * dim;

    // q as operands: chunk 2 s + half of this lane's column, in parts
    v4u qf[kQParts][kSteps];
    float gain = a.scale2;
    {
        float up = 1.0f;
        if constexpr (F32 && T == kF16) {
            float top = 0.0f;
            for (int d = 4 * half; d < dim; d += 8) {
                const float4 x = load4<T, F32>(a.q, row + d);
                top = fmaxf(top, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w))));
            }
            up = row_gain(max_xor32(top));
            gain = a.scale2 / up;
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 8 * (2 * s + half);
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f), y = x;
            if (full || d < dim) x = load4<T, F32>(a.q, row + d);
            if (full || d + 4 < dim) y = load4<T, F32>(a.q, row + d + 4);
            if constexpr (kQParts == 1) {
                qf[0][s] = v4u{Elem<T>::pack(x.x, x.y), Elem<T>::pack(x.z, x.w), Elem<T>::pack(y.x, y.y),
                               Elem<T>::pack(y.z, y.w)};
            } else {
                if constexpr (T == kF16) {
                    x.x *= up; x.y *= up; x.z *= up; x.w *= up;
                    y.x *= up; y.y *= up; y.z *= up; y.w *= up;
                }
#pragma unroll
                for (int p = 0; p < kQParts; ++p)
                    qf[p][s] = v4u{Elem<T>::part(x.x, x.y), Elem<T>::part(x.z, x.w), Elem<T>::part(y.x, y.y),
                                   Elem<T>::part(y.z, y.w)};
            }
        }
    }

    // Positions of the work group's and of this wave's columns, and the tiles they see: those of the sinks, then from the
    // window's first to the last position's.
    const int last_col = (col0 + kColumns < columns ? col0 + kColumns : columns) - 1;
    const int pos_lo = p0 + col0 / a.group, pos_hi = p0 + last_col / a.group;
    const int wcol0 = col0 + wave * 32, wcol1 = wcol0 + 31 < columns ? wcol0 + 31 : columns - 1;
    const bool wave_used = wcol0 < columns;
    const int wpos_lo = p0 + (wave_used ? wcol0 : columns - 1) / a.group, wpos_hi = p0 + (wave_used ? wcol1 : columns - 1) / a.group;
    const int lo = a.window > 0 && pos_lo >= a.window ? pos_lo - a.window + 1 : 0;
    const int sinks = a.n_sink < lo ? a.n_sink : lo;
    const int first = lo / kTile;
    int sink_tiles = (sinks + kTile - 1) / kTile;
    sink_tiles = sink_tiles < first ? sink_tiles : first;
    const int n_tiles = pos_hi < 0 ? 0 : sink_tiles + pos_hi / kTile + 1 - first;
    auto tile_key = [&](int t) { return (t < sink_tiles ? t : t - sink_tiles + first) * kTile; };

    const int32_t* table = c.table + (int64_t)b * c.max_pages;
    const int chunks = c.chunks;
    const int k_words = chunks * kTile, v_words = dim * (kTile / 8);
    const int64_t k_head = (int64_t)kvh * chunks * ps * 8, v_head = (int64_t)kvh * dim * ps;
    const int steps = (chunks + 1) / 2;

    // pages of the four quarters of a tile (-1 where there is none)
    int pages[4];
    auto load_pages = [&](int key) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = (key + 16 * i) >> c.shift;
            const int page = at < c.max_pages ? table[at] : -1;
            pages[i] = page_ok(c, page) ? page : -1;
        }
    };
    auto page_of = [&](int quarter) {
        const int x = quarter == 0 ? pages[0] : quarter == 1 ? pages[1] : quarter == 2 ? pages[2] : pages[3];
        return x < 0 ? 0 : x;
    };
    v4u stage_k[kLoads], stage_v[kLoads];
    auto load_tile = [&](int key) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int w = tid + i * kThreads;
            const int at = w & (kTile - 1), chunk = w / kTile;
            v4u x = {0u, 0u, 0u, 0u};
            if (full || w < k_words)
                x = *reinterpret_cast<const v4u*>(c.k + (int64_t)page_of(at >> 4) * c.k_page + k_head +
                                                  (int64_t)(chunk * ps + ((key + at) & (ps - 1))) * 8);
            stage_k[i] = x;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int w = tid + i * kThreads;
            const int eight = full ? w / DP : w / dim, d = w - eight * dim;
            v4u x = {0u, 0u, 0u, 0u};
            if (full || w < v_words)
                x = *reinterpret_cast<const v4u*>(c.v + (int64_t)page_of((eight >> 1) & 3) * c.v_page + v_head +
                                                  (int64_t)((key + 8 * eight) & (ps - 1)) * dim + d * 8);
            stage_v[i] = x;
        }
    };
    // there: whether the four quarters have pages.  Values of keys that the cache does not hold become zeros: whatever lies
    // there must not meet a weight of 0 in the product.
    auto store_tile = [&](int buf, int t, uint32_t there) {
        const int key = tile_key(t);
        // does every query of the work group see every key?
        const bool open = there == 15 && key + kTile - 1 <= pos_lo &&
                          (a.window <= 0 || key > pos_hi - a.window || key + kTile <= a.n_sink);
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) kt[buf][tid + i * kThreads] = __builtin_bit_cast(uint4, stage_k[i]);
        const bool whole = there == 15 && key + kTile <= len;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int w = tid + i * kThreads;
            v4u x = stage_v[i];
            if (!whole) {
                const int eight = full ? w / DP : w / dim;
                int held = len - (key + 8 * eight);
                held = (there >> ((eight >> 1) & 3)) & 1 ? held : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] &= (held > 2 * e ? 0x0000FFFFu : 0u) | (held > 2 * e + 1 ? 0xFFFF0000u : 0u);
            }
            if (!open) odd |= not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3]);
            if (full || w < v_words) vt[buf][w] = __builtin_bit_cast(uint4, x);
        }
        if (odd) odd_tile[buf] = t;
    };
    auto there_of = [&]() {
        return (pages[0] >= 0 ? 1u : 0u) | (pages[1] >= 0 ? 2u : 0u) | (pages[2] >= 0 ? 4u : 0u) | (pages[3] >= 0 ? 8u : 0u);
    };

    float m = kNegInf, l = 0.0f;
    v16f o[kBlocks];
#pragma unroll
    for (int t = 0; t < kBlocks; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;

    // key of a row of a 32-key block: the order in which a lane's 16 scores are its operand words of the second product
    const int key_row = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);

    uint32_t there = 0;
    if (tid < 2) odd_tile[tid] = -1;
    __syncthreads();
    if (n_tiles > 0) {
        load_pages(tile_key(0));
        there = there_of();
        load_tile(tile_key(0));
        store_tile(0, 0, there);
    }
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int key = tile_key(t), buf = t & 1;
        const uint32_t now = there;
        if (t + 1 < n_tiles) {
            load_pages(tile_key(t + 1));
            there = there_of();
            load_tile(tile_key(t + 1));
        }
        // does this wave see anything of the tile, and all of it?
        const bool near = key <= wpos_hi && (a.window <= 0 || key + kTile - 1 > wpos_lo - a.window);
        const bool sink = a.window > 0 && key < a.n_sink && key <= wpos_hi;
        if (wave_used && (near || sink)) {
            v16f s[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[blk][i] = 0.0f;
            }
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                if (!full && st >= steps) continue;
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const v4u kf = __builtin_bit_cast(v4u, kt[buf][(2 * st + half) * kTile + 32 * blk + key_row]);
#pragma unroll
                    for (int p = 0; p < kQParts; ++p) s[blk] = Elem<T>::mfma32(kf, qf[p][st], s[blk]);
                }
            }
            const bool whole = now == 15 && key + kTile - 1 <= wpos_lo &&
                               (a.window <= 0 || key > wpos_hi - a.window || key + kTile <= a.n_sink);
            float top = kNegInf;
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = s[blk][i] * gain;
                    if (!whole) {
                        const int quarter = 2 * blk + (i >> 3);
                        const int j = key + 16 * quarter + 8 * half + (i & 7);
                        const bool in = ((now >> quarter) & 1) && j <= pos && (a.window <= 0 || j > pos - a.window || j < a.n_sink);
                        x = in ? x : kNegInf;
                    }
                    s[blk][i] = x;
                    top = fmaxf(top, x);
                }
            }
            top = max_xor32(top);
            const float m_new = fmaxf(m, top);
            if (__any(m_new > m)) {
                const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(m - m_new);
                l *= alpha;
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) o[d] *= alpha;
                m = m_new;
            }
            const float base = (m == kNegInf ? 0.0f : m) - kLift<T>;
            float sum = 0.0f;
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[blk][i] = exp2_fast(s[blk][i] - base);
                    sum += s[blk][i];
                }
            }
            l += sum;
            const bool odd = !whole && odd_tile[buf] == t;
#pragma unroll
            for (int q = 0; q < 4; ++q) {                 // 16 keys
                const int blk = q >> 1, i0 = 8 * (q & 1);
                v4u pf[kPParts];
                if constexpr (kPParts == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) pf[0][e] = Elem<T>::pack(s[blk][i0 + 2 * e], s[blk][i0 + 2 * e + 1]);
                } else {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = s[blk][i0 + e];
#pragma unroll
                    for (int p = 0; p < kPParts; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) pf[p][e] = Elem<T>::part(x[2 * e], x[2 * e + 1]);
                }
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    if (!full && 32 * d >= dim) continue;
                    v4u vf = __builtin_bit_cast(v4u, vt[buf][(2 * q + half) * dim + 32 * d + n]);
                    if (odd) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) vf[e] &= ~not_finite<T>(vf[e]);
                    }
#pragma unroll
                    for (int p = 0; p < kPParts; ++p) o[d] = Elem<T>::mfma32(vf, pf[p], o[d]);
                }
            }
            if (odd) {
                constexpr uint32_t one = T == kBf16 ? 0x3F80u : 0x3C00u;
                for (int d = 0; d < kBlocks; ++d) {
                    if (!full && 32 * d >= dim) continue;
                    v16f count;
#pragma unroll
                    for (int i = 0; i < 16; ++i) count[i] = 0.0f;
                    for (int q = 0; q < 4; ++q) {
                        const uint4 w = vt[buf][(2 * q + half) * dim + 32 * d + n];
                        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
                        v4u mark, seen;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            mark[e] = mark_half<T>(x[e] & 0xFFFFu) | mark_half<T>(x[e] >> 16) << 16;
                            seen[e] = 0;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int j = key + 16 * q + 8 * half + 2 * e + h;
                                const bool in = ((now >> q) & 1) && j <= pos && (a.window <= 0 || j > pos - a.window || j < a.n_sink);
                                seen[e] |= in ? one << (16 * h) : 0u;
                            }
                        }
                        count = Elem<T>::mfma32(mark, seen, count);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float x = unmark(count[i]);
#pragma unroll
                        for (int k = 0; k < kBlocks; ++k) o[k][i] += k == d ? x : 0.0f;
                    }
                }
            }
        }
        if (t + 1 < n_tiles) store_tile(buf ^ 1, t + 1, there);
        __syncthreads();
    }

    l = sum_xor32(l);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;        // l is 0 where nothing was visible
    if (!used) return;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 32 * d + 8 * i + 4 * half;
            if (full || at < dim)
                store4<T, F32>(a.out, row + at, o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv,
                               o[d][4 * i + 3] * inv);
        }
    }
}

template <int T, int DP, bool F32, int WAVES>
hipError_t launch(PrefillArgs a, hipStream_t s) {
    a.tiles = (int)((int64_t)a.n_tokens * a.group / (32 * WAVES)) + a.c.n_seqs;
    hipLaunchKernelGGL((attn_prefill_kernel<T, DP, F32, WAVES>), dim3((unsigned)a.tiles * (unsigned)a.c.kv_heads),
                       dim3(64 * WAVES), 0, s, a);
    return hipGetLastError();
}

template <int T, bool F32>
hipError_t launch_dim(const PrefillArgs& a, hipStream_t s) {
    if (a.c.dim <= 64) return launch<T, 64, F32, 4>(a, s);
    if (a.c.dim <= 128) return launch<T, 128, F32, 4>(a, s);
    return launch<T, 256, F32, 4>(a, s);
}

}  // namespace

hipError_t launch_attn_prefill(const KvCache& c, int dtype, const AttnArgs& args, hipStream_t s) {
    PrefillArgs a{};
    a.c = c;
    a.q = args.q;
    a.out = args.out;
    a.q_start = args.q_start;
    a.n_tokens = args.n_tokens;
    a.heads = args.heads;
    a.group = args.heads / c.kv_heads;
    a.scale2 = args.scale * kLog2e;
    a.window = args.window;
    a.n_sink = args.n_sink;
    if (dtype == kBf16) return args.f32 ? launch_dim<kBf16, true>(a, s) : launch_dim<kBf16, false>(a, s);
    return args.f32 ? launch_dim<kF16, true>(a, s) : launch_dim<kF16, false>(a, s);
}

}  // namespace bitnet
