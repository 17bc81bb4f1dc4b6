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
// rounded once to that type (and summed as rounded), as the output is: a second part would double the longer half of the work,
// and the error against 64 bits is 2.1e-3 of the output's size where rounding the output alone makes 1.6e-3 (4096 tokens, bf16).
// 32-bit inputs go in as sums of parts (see Elem): three of bf16, which are exact, or two of f16, which hold 22 bits.
//
// A value that is not finite must not reach a query that does not see it, and makes its channel infinite for one that does, however
// small its weight.  The product does neither (0 times it is no number, and weights go in parts, some of them 0), but it leaves
// no such channel finite: finite outputs need no look at the values, and a work group that has others forms its products once
// more of the finite values and counts the rest that each query sees (careful).
//
// Measured (kernel times; D = 128, 32 heads of 8 kv heads unless said), TFLOP/s of the visible pairs: bf16 throughout, 4096
// tokens 148 us (930; a large library product reaches 1131 here); 32-bit inputs over bf16, 8192 tokens behind a window of 1024, 456
// us (284, 851 in its three parts); 32-bit inputs over f16, six chunks of up to 1500 tokens, 32 heads of 100, window 512, 175
// us (202, 403 in two parts); 37 tokens 11 us (a start of four reads in a row, then one tile).  At 4096 tokens the matrix cores are
// busy 37% of the kernel's cycles; a wave waits 31% of its time, is ready but not issued 31% and issues 38%: exponentials and
// weights of one wave against the products of the other.  Slower: softmax of one tile between the products of the next in one
// wave (190 us against 166), halves of the waves taking turns at a barrier (173), products in a fixed order (156), keys and
// values staged through the same registers (162), all against 151 to 152 then.
#include "attn_prefill.hpp"

namespace bitnet {
namespace {

template <int T, int DP, bool F32, int WAVES, int PER_SIMD, bool FULL, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, PER_SIMD) void attn_prefill_kernel(PrefillArgs a) {
    using P = Prefill<T, DP, F32, WAVES, FULL, SPLIT ? kSplit : kWhole>;
    __shared__ typename P::Lds lds;
    P(a, lds).run();
}

// The parts of every row in the order of the keys.  A thread four channels; blockIdx.y: slices of a work group's columns.
template <int T, bool F32>
__global__ __launch_bounds__(256) void attn_prefill_join_kernel(PrefillArgs a, int group_columns) {
    const KvCache& c = a.c;
    const int kvh = blockIdx.x % c.kv_heads, id = a.tiles - 1 - (int)(blockIdx.x / c.kv_heads);
    const int b = find_last(c.n_seqs, id, [&](int i) { return first_tile(a.q_start, i, a.n_tokens, a.group, group_columns); });
    const Span span = span_of(a.q_start, b, a.n_tokens);
    const int slice = group_columns / gridDim.y;
    const int col0 = (id - first_tile(a.q_start, b, a.n_tokens, a.group, group_columns)) * group_columns + (int)blockIdx.y * slice;
    const int columns = span.count * a.group;
    if (col0 < 0 || col0 >= columns) return;
    const int parts = parts_of(a, group_columns);
    if (parts == 1) return;                               // the work groups wrote out themselves
    const int quads = c.dim >> 2, held = held_parts(a.splits);
    for (int i = threadIdx.x; i < slice * quads; i += 256) {
        const int in_slice = i / quads, d = 4 * (i - in_slice * quads), col = col0 + in_slice;
        if (col >= columns) continue;
        const int token = col / a.group, head = kvh * a.group + col - token * a.group;
        const int64_t row = (int64_t)(span.first + token) * a.heads + head;
        const float* part = a.ws + row * row_floats(a.splits, c.dim);
        float m = kNegInf, l = 0.0f;
        v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int z = 0; z < parts; ++z) {
            const float pm = part[z], pl = part[held + z];
            const v4f po = *reinterpret_cast<const v4f*>(part + 2 * held + z * c.dim + d);
            const float top = fmaxf(m, pm);
            const float fa = m == kNegInf ? 0.0f : exp2_fast(m - top), fb = pm == kNegInf ? 0.0f : exp2_fast(pm - top);
            o = o * fa + po * fb;
            l = l * fa + pl * fb;
            m = top;
        }
        if (__builtin_expect(!all_finite(o) && l == l, 0)) {
            v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int z = 0; z < parts; ++z) sum = add_infinite(sum, *reinterpret_cast<const v4f*>(part + 2 * held + z * c.dim + d));
            o = or_infinite(o, sum);
        }
        const float inv = l == 0.0f ? 1.0f : 1.0f / l;
        store4<T, F32>(a.out, row * c.dim + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    }
}

// How a call is laid out.  Two waves a SIMD (256 registers each) cover each other's waits and softmax: one work group of 8 waves
// a CU, whose tiles are read once for 256 columns, or two of 4, of which one starts, ends or waits at a barrier while the
// other computes.  The large ones win where work groups go through many keys, the small ones where they are short (us, 8 waves /
// 4, bf16, 32 heads of 128: 4096 tokens 151 / 160, three prompts of 2048 155 / 144, eight of 1024 120 / 117, sixteen of 512
// 89 / 83; 8192 tokens behind a window of 4096 447 / 455, 2048 309 / 290, 1024 190 / 182; heads of 100, 512: 134 / 129) or
// where 8 waves do not divide a tile evenly (heads of 96: 124 / 102; of 100 without a window the large ones stay ahead, 170 / 176).
// Two parts of q fit 256 registers only in the large ones (f16 heads of 100 behind a window 174 / 220), three in neither: one
// wave a SIMD (8192 tokens, window 1024: 456; 8 waves with what does not fit in memory 525).
// Where they leave half of their places empty (a chunk of a prompt behind a long cache, a short prompt), each one's keys are split
// into parts of four tiles and more, and a second launch joins them (64 tokens behind 8000: 184 us whole, 31 split).  How many
// work groups have tokens is known on the device (parts_of); here the fewest that there can be give the most parts, so that a
// workspace holds no more rows of out than the places have columns (up to 42 MB).  Where all sequences turn out to have tokens
// the second launch and the parts left out cost some us (from 32 bits over f16, heads of 100: 8 sequences of 8 tokens behind 1000
// 44 us, whole 35); where one has them all the parts save several times that (64 tokens behind 8000 in one of 64 rows of the
// table 53 us, whole 187, of 1024 64 and 188; from 32 bits over f16, one of 32 rows, 66 and 360).  The large work groups are split
// where that gives kLargeParts parts and more: fewer cost more where they prove empty than they could save (8 sequences of 128 tokens
// behind 300, two parts: 32 us, whole 26; 1024 tokens in one of 8 rows 59 and 66).
// Sequences without tokens still cost work groups that find nothing; parts that would make more than kEmptyRounds rounds of those
// are not taken (one of 64, 256 and 1024 rows: 53, 59 and 64 us; 4 rounds 79, 81, 85; no bound 70, 80, 87).
// The keys are counted by the room of the table: in one much wider than its sequences some parts have nothing to do (37 tokens in
// a table of 8192 positions 16 us, in one of 64 11).
constexpr int kCus = 256;
constexpr int kEmptyRounds = 16;
constexpr int kLargeParts = 4;       // parts of groups of 8 waves, at least
constexpr int kMostSeqs = 1024;      // sequences that are counted on the device: past them nothing is split
struct Plan {
    int waves, splits, tiles;        // tiles: work groups of a kv head
    int places;
};
Plan plan_of(int64_t n_seqs, int64_t n_tokens, int heads, int kv_heads, int dim, int page_size, int64_t max_pages, int window,
             int n_sink, bool three_parts, bool f32) {
    const int64_t group = heads / kv_heads, rows = n_tokens * group, most_seqs = n_seqs < n_tokens ? n_seqs : n_tokens;
    const bool one_a_simd = three_parts ? dim > 64 : dim > 128 || (f32 && dim > 64);
    Plan p{4, 1, 0, one_a_simd ? kCus : 2 * kCus};
    constexpr int kLongKeys = 2048;
    const bool brief = (window > 0 && window <= kLongKeys) || (dim == 128 && n_tokens <= kLongKeys * n_seqs);
    const bool wide = !three_parts && dim > 64 && dim <= 128 && (f32 || (dim > 96 && !brief));
    if (wide && (rows / 256 + most_seqs) * kv_heads >= kCus) {
        p.waves = 8;
        p.places = kCus;
    }
    const int columns = 32 * p.waves;
    p.tiles = (int)(rows / columns + most_seqs);
    const int64_t busy = (rows + columns - 1) / columns * kv_heads;
    int64_t tiles = (max_pages * page_size + kTile - 1) / kTile;
    if (window > 0) {
        const int64_t near = ((int64_t)window + columns / group + kTile - 1) / kTile + 2 + ((int64_t)n_sink + kTile - 1) / kTile;
        tiles = near < tiles ? near : tiles;
    }
    int64_t splits = p.places / busy;
    splits = splits < tiles / 4 ? splits : tiles / 4;
    splits = splits < 32 ? splits : 32;
    const int64_t most = n_seqs > kMostSeqs ? 1 : kEmptyRounds * (int64_t)p.places / ((int64_t)p.tiles * kv_heads);
    splits = splits < most ? splits : most;
    if (p.waves == 8 && splits < kLargeParts) splits = 1;
    p.splits = (int)(splits < 1 ? 1 : splits);
    return p;
}

template <int T, int DP, bool F32, int WAVES, int PER_SIMD, bool FULL>
hipError_t launch_full(const PrefillArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)a.tiles * (unsigned)a.c.kv_heads, (unsigned)a.splits), block(64 * WAVES);
    if (a.splits == 1) {
        hipLaunchKernelGGL((attn_prefill_kernel<T, DP, F32, WAVES, PER_SIMD, FULL, false>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((attn_prefill_kernel<T, DP, F32, WAVES, PER_SIMD, FULL, true>), grid, block, 0, s, a);
    unsigned slices = 16;
    while (slices > 1 && grid.x * slices > 4096) slices /= 2;
    hipLaunchKernelGGL((attn_prefill_join_kernel<T, F32>), dim3(grid.x, slices), dim3(256), 0, s, a, 32 * WAVES);
    return hipGetLastError();
}

template <int T, int DP, bool F32, int WAVES, int PER_SIMD>
hipError_t launch(const PrefillArgs& a, hipStream_t s) {
    if (DP != 112 && a.c.dim == DP) return launch_full<T, DP, F32, WAVES, PER_SIMD, DP != 112>(a, s);
    return launch_full<T, DP, F32, WAVES, PER_SIMD, false>(a, s);
}

template <int T, bool F32, int DP>
hipError_t launch_waves(const PrefillArgs& a, int waves, hipStream_t s) {
    if constexpr (F32 && T == kBf16) {
        return launch<T, DP, F32, 4, 1>(a, s);
    } else if constexpr (!F32 && DP == 96) {
        return launch<T, DP, F32, 4, 2>(a, s);
    } else {
        if (waves == 8) return launch<T, DP, F32, 8, 2>(a, s);
        return launch<T, DP, F32, 4, F32 ? 1 : 2>(a, s);
    }
}

template <int T, bool F32>
hipError_t launch_dim(const PrefillArgs& a, int waves, hipStream_t s) {
    if (a.c.dim <= 64) return launch<T, 64, F32, 4, 2>(a, s);
    if (a.c.dim <= 96) return launch_waves<T, F32, 96>(a, waves, s);
    if (a.c.dim <= 112) return launch_waves<T, F32, 112>(a, waves, s);
    if (a.c.dim <= 128) return launch_waves<T, F32, 128>(a, waves, s);
    if (a.c.dim <= 192) return launch<T, 192, F32, 4, 1>(a, s);
    return launch<T, 256, F32, 4, 1>(a, s);
}

size_t parts_bytes(const Plan& p, int64_t n_tokens, int heads, int dim) {
    return p.splits > 1 ? (size_t)(n_tokens * heads) * (size_t)row_floats(p.splits, dim) * 4 : 0;
}

}  // namespace

size_t attn_prefill_workspace_bytes(int64_t n_seqs, int64_t n_tokens, int heads, int kv_heads, int dim, int page_size,
                                    int64_t max_pages, int window, int n_sink, bool three_parts, bool f32) {
    return parts_bytes(plan_of(n_seqs, n_tokens, heads, kv_heads, dim, page_size, max_pages, window, n_sink, three_parts, f32),
                       n_tokens, heads, dim);
}

hipError_t launch_attn_prefill(const KvCache& c, int dtype, const AttnArgs& args, void* ws, size_t ws_bytes, hipStream_t s) {
    Plan p = plan_of(c.n_seqs, args.n_tokens, args.heads, c.kv_heads, c.dim, 1 << c.shift, c.max_pages, args.window, args.n_sink,
                     args.f32 && dtype == kBf16, args.f32);
    if (!ws || ws_bytes < parts_bytes(p, args.n_tokens, args.heads, c.dim)) p.splits = 1;
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
    a.tiles = p.tiles;
    a.splits = p.splits;
    a.places = p.places;
    a.ws = static_cast<float*>(ws);
    if (dtype == kBf16) return args.f32 ? launch_dim<kBf16, true>(a, p.waves, s) : launch_dim<kBf16, false>(a, p.waves, s);
    return args.f32 ? launch_dim<kF16, true>(a, p.waves, s) : launch_dim<kF16, false>(a, p.waves, s);
}

}  // namespace bitnet
