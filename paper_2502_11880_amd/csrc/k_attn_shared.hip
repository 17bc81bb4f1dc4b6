// Attention of one new token per sequence over the paged cache, where groups of neighbouring sequences share their first keys:
//   out[b, h] = sum_j p_j v_j,  p = softmax over the visible keys j of scale q[b, h] . k_j
// (visible as in the decode without groups: j < L, and with a window j >= L - window or j < n_sink; nothing visible: zeros).  Keys
// below the group's prefix are those of its first sequence, keys from there on the sequence's own.
//
// A row of the work is a kv head's columns over a run of keys: all query heads of all sequences of a group over its prefix, and
// the query heads of one sequence over its own keys.  Up to W = 32 columns go through together (heads of up to 64 channels: 64; of 128
// 64 columns spilled, 100 us where 32 took 59), 16 to a tile of the matrix instruction; more are rows of their own, which lie in the
// line below so that work groups of one XCD read the same keys at about the same time (141 MB come from HBM where the keys and values
// are 124, though the prefix is gone through four times).  Keys go in units of 32 through registers (S^T = K Q^T, O^T = V^T P^T, as in
// the decode without groups: the weights never leave their lane), q waits in LDS.  Prefixes of many columns: k_attn_shared_wide.hip.
//
// All rows stand in one line, weighted by what a unit of their tiles costs, and every work group takes an equal share of it; its
// waves take the units in turn.  Every row leaves (maximum, sum, unnormalised output) records in the workspace, one for each share
// that it crosses, and a second launch joins those of a sequence's prefix and own keys.
//
// What is not finite: as in the decode without groups, finite results need no look at the inputs, and a share with others is gone
// through once more, key by key (redo).
//
// Measured (kernel times; 32 heads of 8 kv heads of 128, bf16, q from 32 bits unless said): 32 sequences with up to 1500 keys of their own
// behind 6016 41 us (127 MB) and 6.5 to join; four beams behind 352 13.8 and 4.2; five groups of up to 12, 32 heads of 100, f16, 76 us
// (314 MB, 4.1 TB/s) and 6.  Bound by the starts of rows where they are many or short: of a row of three units a wave, in cycles,
// index 5900, place 3600, q and pages 2000, keys 4750, end 3800.
#include "attn_shared.hpp"

#include <type_traits>

namespace bitnet {
namespace {

constexpr int kUnit = 32;            // keys of a unit
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kIds = 512;            // units whose pages a work group looks up at a time

__host__ __device__ constexpr int most_tiles(int dim) { return dim <= 64 ? 4 : 2; }
// What a unit of a row of one, two and four tiles costs, and what its start does (q, pages and first keys are three reads in a row,
// and in the end the waves' states become one).  Measured on the cases above (us a call: 32 sequences / four beams / five groups): two tiles
// at 3, 4, 6 and 8 51, 54, 56 and 56 / - / -, at 5 47; a start of 20 46 / 17.5 / 86, 24 47 / 17.4 / 81, 28 49 / 17.5 / 83, 36 53 / 16.8 / 81.
__host__ __device__ constexpr int cost_of(int tiles) { return tiles == 1 ? 4 : tiles == 2 ? 5 : 7; }
constexpr int kStartCost = 24;
// Rows of up to so many units are never split: the share that a row starts in takes it whole (none 47 / 21.6 / 85, 12 45 / 19.6 / 86, 24
// 50 / 19.7 / 84 then).
constexpr int kWholeUnits = 12;
__host__ __device__ __forceinline__ int tiles_of(int columns) { return columns <= 16 ? 1 : columns <= 32 ? 2 : 4; }

__device__ __forceinline__ int unit_key(const Keys& k, int u) {
    return (u < k.sink_units ? k.first_sink + u : k.first_unit + u - k.sink_units) * kUnit;
}
__device__ __forceinline__ int rows_of(const SharedArgs& a, int columns) { return (columns + a.columns - 1) / a.columns; }
// The keys of a sequence's own row, and of its group's prefix.
__device__ __forceinline__ Keys own_keys(const SharedArgs& a, const Index& x, int s) {
    if (x.lead[s] == kNobody) return {0, 0, 0, 0, 0, 0};
    const int len = x.len[s], prefix = x.prefix[x.lead[s]];
    return keys_of<kUnit>(prefix < len ? prefix : len, len, behind(a, len), a.n_sink);
}
__device__ __forceinline__ Keys all_prefix_keys(const SharedArgs& a, const Index& x, int s) {
    if (x.members[s] == 0) return {0, 0, 0, 0, 0, 0};
    return keys_of<kUnit>(0, x.prefix[s], x.low[s], a.n_sink);
}
__device__ __forceinline__ bool is_wide(const SharedArgs& a, const Index& x, int s) {
    return a.wide_groups && worth_wide(a.rule, x.members[s] * a.group, a.columns, a.wide_columns, (int64_t)all_prefix_keys(a, x, s).units * kUnit, a.c.kv_heads);
}
__device__ __forceinline__ Keys prefix_keys(const SharedArgs& a, const Index& x, int s) {
    const Keys k = all_prefix_keys(a, x, s);
    return is_wide(a, x, s) ? Keys{0, 0, 0, 0, 0, 0} : k;
}
__device__ __forceinline__ int cost_of_columns(const SharedArgs& a, int columns) {
    return cost_of(tiles_of(columns < a.columns ? columns : a.columns));
}
__device__ __forceinline__ int64_t cost_of_rows(const SharedArgs& a, int columns, int units) {
    return line_cost(units, cost_of_columns(a, columns), kStartCost) * rows_of(a, columns) * a.c.kv_heads;
}
// Of a group's wide prefix: its units, and the cost of its rows.
__device__ __forceinline__ int64_t wide_cost(const SharedArgs& a, const Index& x, int s) {
    const int columns = x.members[s] * a.group;
    if (!is_wide(a, x, s)) return 0;
    const int units = keys_of<kWideTile>(0, x.prefix[s], x.low[s], a.n_sink).units;
    return line_cost(units, kWideCost, kWideStart) * ((columns + a.wide_columns - 1) / a.wide_columns) * a.c.kv_heads;
}

// start[s]: the sum of cost(i) over i < s, for s up to n.
template <typename F>
__device__ __forceinline__ void sum_line(int n, F cost_at, int64_t* start, int64_t (&wave_cost)[kWaves]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t before_all = 0;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        const int s = s0 + tid;
        const int64_t cost = s < n ? cost_at(s) : 0;
        int64_t sum = cost;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const int64_t other = __shfl_up((long long)sum, i);
            if (lane >= i) sum += other;
        }
        if (lane == 63) wave_cost[wave] = sum;
        __syncthreads();
        int64_t before = before_all;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? wave_cost[w] : 0;
            before_all += wave_cost[w];
        }
        if (s < n) start[s] = before + sum - cost;
        __syncthreads();
    }
    if (tid == 0) start[n] = before_all;
}

// All of it worked out by every work group: the groups' marks, then sums and the last mark before each sequence in one scan.
__device__ void build_index(const SharedArgs& a, Index& x, int64_t (&wave_cost)[kWaves], int (&wave_lead)[kWaves]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, most = a.c.max_pages << a.c.shift;
    // groups from the one that the launch's first sequence belongs to; the first ones' bounds are asked for beside the lengths
    const int first_group = a.first_seq == 0 ? 0 : find_last(a.n_groups, a.first_seq, [&](int i) { return a.group_start[i]; });
    int g = first_group + tid, b0 = 0, b1 = 0, p = 0;
    auto ask = [&] {
        if (g >= a.n_groups) return;
        b0 = a.group_start[g];
        b1 = a.group_start[g + 1];
        p = a.prefix_len[g];
    };
    ask();
    for (int s = tid; s < a.n_seqs; s += kThreads) {
        x.members[s] = 0;
        x.low[s] = a.window > 0 ? most : 0;
        x.len[s] = seq_len(a.c, a.first_seq + s);
    }
    __syncthreads();
    for (; g < a.n_groups && b0 < a.first_seq + a.n_seqs; g += kThreads, ask()) {
        if (b0 < 0 || b1 <= b0 || b1 > a.c.n_seqs) continue;
        const int s0 = max(b0 - a.first_seq, 0), s1 = min(b1 - a.first_seq, a.n_seqs);
        if (s0 >= s1) continue;
        x.members[s0] = (uint16_t)(s1 - s0);
        x.prefix[s0] = p < 0 ? 0 : p < most ? p : most;
        if (s0 == 0) x.first_row = b0;
    }
    __syncthreads();
    int carry = -1;
    for (int s0 = 0; s0 < a.n_seqs; s0 += kThreads) {
        const int s = s0 + tid;
        int lead = s < a.n_seqs && x.members[s] > 0 ? s : -1;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const int other = __shfl_up(lead, i);
            if (lane >= i) lead = max(lead, other);
        }
        if (lane == 63) wave_lead[wave] = lead;
        __syncthreads();
        lead = max(lead, carry);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) lead = max(lead, wave_lead[w]);
            carry = max(carry, wave_lead[w]);
        }
        if (s < a.n_seqs) {
            const bool owned = lead >= 0 && s < lead + x.members[lead];
            x.lead[s] = owned ? (uint16_t)lead : kNobody;
            if (owned && a.window > 0) atomicMin(&x.low[lead], behind(a, x.len[s]));
        }
        __syncthreads();
    }
    sum_line(a.n_seqs, [&](int s) {
        return cost_of_rows(a, x.members[s] * a.group, prefix_keys(a, x, s).units) + cost_of_rows(a, a.group, own_keys(a, x, s).units);
    }, x.start, wave_cost);
    __syncthreads();
}

// No share lies within a unit, nor within a start; a short row costs about as much, so that few shares start two of them.
__device__ __forceinline__ int64_t share_of(const SharedArgs& a, int64_t all) {
    return line_share(all, gridDim.x, kStartCost + cost_of(tiles_of(a.columns)));
}

// A row, and the units [u0, u1) of it that the share from pos to end holds.
struct Place {
    int s, own;                      // the sequence (of the launch) that the row belongs to; its own keys or its group's prefix
    int kvh, col0, count, members;   // kv head, first column and number of them, sequences that the columns belong to
    int table_row;
    int u0, u1;
    int64_t next;                    // where the next row starts in the line
    Keys keys;
};
__device__ __forceinline__ Place place_of(const SharedArgs& a, const Index& x, int64_t pos, int64_t end) {
    int lo = 0, hi = a.n_seqs - 1;                        // the last sequence that starts at pos or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (x.start[mid] <= pos) lo = mid;
        else hi = mid - 1;
    }
    Place p;
    p.s = lo;
    p.own = 0;
    p.members = x.members[lo];
    p.keys = prefix_keys(a, x, lo);
    int64_t at = x.start[lo];
    const int64_t of_prefix = cost_of_rows(a, p.members * a.group, p.keys.units);
    if (pos - at >= of_prefix) {
        at += of_prefix;
        p.own = 1;
        p.members = 1;
        p.keys = own_keys(a, x, lo);
    }
    const int columns = p.members * a.group, rows = rows_of(a, columns);
    const int cost = cost_of_columns(a, columns);
    const int64_t row_cost = line_cost(p.keys.units, cost, kStartCost);
    const int row = (int)divide(pos - at, row_cost);
    at += row * row_cost;
    p.kvh = row / rows;
    p.col0 = (row - p.kvh * rows) * a.columns;
    p.count = columns - p.col0 < a.columns ? columns - p.col0 : a.columns;
    p.u0 = (int)line_unit(pos - at, cost, kStartCost);
    const int64_t room = line_unit(end - at, cost, kStartCost);
    p.u1 = room < p.keys.units ? (int)room : p.keys.units;
    if (p.keys.units <= kWholeUnits) {                    // whole, or of the share before
        p.u0 = pos > at ? p.keys.units : 0;
        p.u1 = p.keys.units;
    }
    p.next = at + row_cost;
    p.table_row = p.own == 0 && lo == 0 ? x.first_row : a.first_seq + lo;
    return p;
}

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

// A column's sequence (of the launch), head, and record.
struct Column {
    int s, head;
};
__device__ __forceinline__ Column column_of(const SharedArgs& a, const Place& p, int column) {
    const int c = p.col0 + column, member = c / a.group;
    return {p.s + member, p.kvh * a.group + c - member * a.group};
}
__device__ __forceinline__ float* record_of(const SharedArgs& a, const Place& p, int column) {
    if (p.u0 == 0 && p.u1 == p.keys.units) {
        const Column c = column_of(a, p, column);
        return whole_record(a, p.own, c.s, c.head);
    }
    return part_record(a, blockIdx.x, p.u0 > 0 ? 0 : 1, column);
}

// A wave's state of a row: running maximum, sum and unnormalised output; lane (m = lane & 15, g = lane >> 4) holds column m of
// tile n, channels 16 t + 4 g + i of o[n][t].
template <int DP, int NT>
struct Row {
    float m[NT], l[NT];
    v4f o[NT][DP / 16];
};

// The columns' lengths and windows.
struct Columns {
    float gain[64];
    int len[64], low[64];
};

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
struct Shared {
    static constexpr int kQParts = F32 ? Elem<T>::kExactParts : 1;
    static constexpr int kPParts = F32 ? Elem<T>::kExactParts : 2;
    static constexpr int kChunks = DP / 8;
    static constexpr int kMost = 16 * most_tiles(DP);     // columns
    static constexpr int kWords = kQParts * kChunks * kMost > kWaves * 16 * DP / 4 ? kQParts * kChunks * kMost : kWaves * 16 * DP / 4;

    struct Lds {
        uint4 q[kWords];                                  // q; then the waves' outputs of a tile
        Index index;
        Columns cols;
        float wave_m[kWaves][kMost], wave_l[kWaves][kMost];
        int ids[2][kIds];
        int64_t wave_cost[kWaves];
        int wave_lead[kWaves];
        int odd;                                          // some output is not finite
    };

    // q of the row's columns as operands in LDS: [part][chunk][column][8]; zeros past D and past the columns, which see everything.
    template <int NT>
    static __device__ __forceinline__ void stage_q(const SharedArgs& a, const Place& p, Lds& lds) {
        const int n = threadIdx.x >> 4, sub = threadIdx.x & 15;
#pragma unroll
        for (int tile = 0; tile < NT; ++tile) {
            const int column = 16 * tile + n;
            const bool used = column < p.count;
            const Column col = column_of(a, p, used ? column : 0);
            const int64_t at = ((int64_t)(a.first_seq + col.s) * a.heads + col.head) * a.c.dim;
            float x[DP / 128 ? DP / 128 : 1][8];
            float top = 0.0f;
#pragma unroll
            for (int r = 0; r < (DP + 127) / 128; ++r) {
                const int d = 8 * (sub + 16 * r);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (used && d + 4 * half < a.c.dim) v = load4<T, F32>(a.q, at + d + 4 * half);
                    x[r][4 * half] = v.x;
                    x[r][4 * half + 1] = v.y;
                    x[r][4 * half + 2] = v.z;
                    x[r][4 * half + 3] = v.w;
                    top = fmaxf(top, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
                }
            }
            float up = 1.0f;
            if constexpr (F32 && T == kF16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, __int_as_float(dpp_row_step(__float_as_int(top), i)));
                up = row_gain(top);
            }
            if (sub == 0) {
                const int len = lds.index.len[col.s];
                lds.cols.gain[column] = a.scale2 / up;
                lds.cols.len[column] = used ? len : 1 << 30;
                lds.cols.low[column] = used ? behind(a, len) : 0;
            }
#pragma unroll
            for (int r = 0; r < (DP + 127) / 128; ++r) {
                const int c = sub + 16 * r;
                if (c >= kChunks) continue;
                if constexpr (F32 && T == kF16) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[r][e] *= up;
                }
#pragma unroll
                for (int part = 0; part < kQParts; ++part) {
                    uint4 w;
                    if constexpr (kQParts == 1) {         // values of the cache's type: exact
                        w = make_uint4(Elem<T>::pack(x[r][0], x[r][1]), Elem<T>::pack(x[r][2], x[r][3]),
                                       Elem<T>::pack(x[r][4], x[r][5]), Elem<T>::pack(x[r][6], x[r][7]));
                    } else {
                        w.x = Elem<T>::part(x[r][0], x[r][1]);
                        w.y = Elem<T>::part(x[r][2], x[r][3]);
                        w.z = Elem<T>::part(x[r][4], x[r][5]);
                        w.w = Elem<T>::part(x[r][6], x[r][7]);
                    }
                    lds.q[(part * kChunks + c) * (16 * NT) + column] = w;
                }
            }
        }
    }

    // The pages of units u0 .. u1 - 1 (at most kIds), and, pages of 16, those of their upper halves: asked for, and put to LDS.
    struct Ids {
        int lower[kIds / kThreads], upper[kIds / kThreads];
    };
    static __device__ __forceinline__ Ids ask_ids(const KvCache& c, const Place& p, int u0, int u1) {
        const int32_t* table = c.table + (int64_t)p.table_row * c.max_pages;
        Ids ids;
#pragma unroll
        for (int k = 0; k < kIds / kThreads; ++k) {
            const int i = threadIdx.x + k * kThreads;
            if (i >= u1 - u0) continue;
            const int at = unit_key(p.keys, u0 + i) >> c.shift;
            ids.lower[k] = table[at];
            if (PAGE16) ids.upper[k] = at + 1 < c.max_pages ? table[at + 1] : -1;
        }
        return ids;
    }
    static __device__ __forceinline__ void put_ids(const Ids& ids, int u0, int u1, int (&to)[2][kIds]) {
#pragma unroll
        for (int k = 0; k < kIds / kThreads; ++k) {
            const int i = threadIdx.x + k * kThreads;
            if (i >= u1 - u0) continue;
            to[0][i] = ids.lower[k];
            if (PAGE16) to[1][i] = ids.upper[k];
        }
    }

    // Units u0 .. u1 - 1 of a row (their pages in ids), this wave's every fourth, into its state.
    template <int NT>
    static __device__ __forceinline__ void run(const SharedArgs& a, const Place& p, int u0, int u1, int least_len, int most_low, const Lds& lds,
                                               Row<DP, NT>& row) {
        const KvCache& c = a.c;
        const Keys keys = p.keys;
        const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int ps = PAGE16 ? 16 : 1 << c.shift;
        const int dim = FULL ? DP : c.dim, chunks = FULL ? DP / 8 : c.chunks;
        const int first = u0 + wave;
        const int count = first < u1 ? (u1 - first + kWaves - 1) / kWaves : 0;
        if (count == 0) return;
        const uint16_t* kbase = c.k + (int64_t)p.kvh * chunks * ps * 8;
        const uint16_t* vbase = c.v + (int64_t)p.kvh * dim * ps;
        // places of this lane's words in a unit: of the keys, key 8 (m / 4) + m % 4 (+ 4 in the second tile) of chunk g (+ 4 j);
        // of the values, channel m (+ 16 t) of the eight keys g
        const uint32_t k_lane = (uint32_t)(g * ps + 8 * (m >> 2) + (m & 3)) * 16, v_lane = (uint32_t)(g * dim + m) * 16;
        // rows of one tile are alone with their keys, which are read past the caches
        auto load = [](const uint16_t* base, uint32_t offset) {
            const v4u* at = reinterpret_cast<const v4u*>(reinterpret_cast<const uint8_t*>(base) + offset);
            if constexpr (NT == 1) return __builtin_nontemporal_load(at);
            else return *at;
        };
        auto page_of = [&](int half, int it) { return __builtin_amdgcn_readfirstlane(lds.ids[half][wave + kWaves * it]); };
        v4u kf[2][DP / 32], vf[DP / 16];
        auto issue_k = [&](int it) {
            const int key = unit_key(keys, first + kWaves * it);
            int p0 = page_of(0, it);
            p0 = page_ok(c, p0) ? p0 : 0;
            const uint16_t* kp = kbase + (int64_t)p0 * c.k_page + (PAGE16 ? 0 : (key & (ps - 1)) * 8);
            uint32_t at = k_lane;
            if (PAGE16 && m >= 8) {     // keys 16 to 31 of the unit: the second page's first 16
                int p1 = page_of(1, it);
                p1 = page_ok(c, p1) ? p1 : 0;
                kp = kbase + (int64_t)p1 * c.k_page;
                at -= 256;
            }
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    v4u w = {0u, 0u, 0u, 0u};
                    if (FULL || 4 * j + g < chunks) w = load(kp + j * 4 * ps * 8, at + 64 * t);
                    kf[t][j] = w;
                }
            }
        };
        auto issue_v = [&](int it) {
            const int key = unit_key(keys, first + kWaves * it);
            int p0 = page_of(0, it);
            p0 = page_ok(c, p0) ? p0 : 0;
            const uint16_t* vp = vbase + (int64_t)p0 * c.v_page + (PAGE16 ? 0 : (key & (ps - 1)) * dim);
            uint32_t at = v_lane;
            if (PAGE16 && g >= 2) {
                int p1 = page_of(1, it);
                p1 = page_ok(c, p1) ? p1 : 0;
                vp = vbase + (int64_t)p1 * c.v_page;
                at -= (uint32_t)dim * 32;
            }
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) {
                v4u w = {0u, 0u, 0u, 0u};
                if (FULL || 16 * t + m < dim) w = load(vp, at + 256 * t);
                vf[t] = w;
            }
        };

        float gain[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) gain[n] = lds.cols.gain[16 * n + m];
        issue_k(0);
        issue_v(0);
        // one unit; MORE: the next one's keys are asked for as soon as the scores are formed, its values after the product
        auto step = [&](int it, auto more_) {
            constexpr bool MORE = decltype(more_)::value;
            const int key = unit_key(keys, first + kWaves * it);
            const bool ok0 = page_ok(c, page_of(0, it)), ok1 = PAGE16 ? page_ok(c, page_of(1, it)) : ok0;
            v4f s[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            int q_at = g * (16 * NT) + m;
            asm volatile("" : "+v"(q_at));                // q stays in LDS
#pragma unroll
            for (int part = 0; part < kQParts; ++part) {
#pragma unroll
                for (int j = 0; j < DP / 32; ++j) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const v4u qf = __builtin_bit_cast(v4u, lds.q[(part * kChunks + 4 * j) * (16 * NT) + 16 * n + q_at]);
                        s[n][0] = Elem<T>::mfma16(kf[0][j], qf, s[n][0]);
                        s[n][1] = Elem<T>::mfma16(kf[1][j], qf, s[n][1]);
                    }
                }
            }
            if constexpr (MORE) issue_k(it + 1);
            const bool in_row = (ok0 & ok1 & (key >= keys.begin) & (key + kUnit <= keys.end)) != 0;
            const bool whole = in_row & (key + kUnit <= least_len) & ((key >= most_low) | (key + kUnit <= a.n_sink));
            if (!in_row) {
                // keys of no row, or of no page, do not enter the second product: 0 times an infinity would be no 0
                const bool there = g < 2 ? ok0 : ok1;
                v4u keep;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int j = key + 8 * g + 2 * w;
                    keep[w] = ((there & (j >= keys.begin) & (j < keys.end)) ? 0x0000FFFFu : 0u) |
                              ((there & (j + 1 >= keys.begin) & (j + 1 < keys.end)) ? 0xFFFF0000u : 0u);
                }
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) vf[t] &= keep;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                // scores of the keys key + 8 g + e, e = 4 t + i
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = s[n][e >> 2][e & 3] * gain[n];
                if (!whole) {
                    const bool there = g < 2 ? ok0 : ok1;
                    const int end = min(keys.end, lds.cols.len[16 * n + m]), low = lds.cols.low[16 * n + m];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int j = key + 8 * g + e;
                        x[e] = (there & (j >= keys.begin) & (j < end) & ((j >= low) | (j < a.n_sink))) ? x[e] : kNegInf;
                    }
                }
                float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
                top = max_xor32(max_xor16(top));
                const float m_new = fmaxf(row.m[n], top);
                if (__any(m_new > row.m[n])) {
                    const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(row.m[n] - m_new);
                    row.l[n] *= alpha;
#pragma unroll
                    for (int t = 0; t < DP / 16; ++t) row.o[n][t] *= alpha;
                    row.m[n] = m_new;
                }
                const float base = (row.m[n] == kNegInf ? 0.0f : row.m[n]) - kLift<T>;
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = exp2_fast(x[e] - base);
                    sum += x[e];
                }
                row.l[n] += sum;
#pragma unroll
                for (int part = 0; part < kPParts; ++part) {
                    const v4u pf = {Elem<T>::part(x[0], x[1]), Elem<T>::part(x[2], x[3]), Elem<T>::part(x[4], x[5]), Elem<T>::part(x[6], x[7])};
#pragma unroll
                    for (int t = 0; t < DP / 16; ++t) row.o[n][t] = Elem<T>::mfma16(vf[t], pf, row.o[n][t]);
                }
            }
            if constexpr (MORE) issue_v(it + 1);
        };
        for (int it = 0; it + 1 < count; ++it) step(it, std::true_type{});
        step(count - 1, std::false_type{});
    }

    // One row's units [u0, u1): its records.
    template <int NT>
    static __device__ __forceinline__ void do_row(const SharedArgs& a, const Place& p, Lds& lds) {
        const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, g = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int dim = a.c.dim;
        const Ids ids = ask_ids(a.c, p, p.u0, min(p.u1, p.u0 + kIds));   // on their way beside q
        stage_q<NT>(a, p, lds);
        put_ids(ids, p.u0, min(p.u1, p.u0 + kIds), lds.ids);
        __syncthreads();
        int least_len = lane < 16 * NT ? lds.cols.len[lane] : 1 << 30, most_low = lane < 16 * NT ? lds.cols.low[lane] : 0;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            least_len = min(least_len, __shfl_xor(least_len, i));
            most_low = max(most_low, __shfl_xor(most_low, i));
        }
        least_len = __builtin_amdgcn_readfirstlane(least_len);
        most_low = __builtin_amdgcn_readfirstlane(most_low);
        Row<DP, NT> r;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            r.m[n] = kNegInf;
            r.l[n] = 0.0f;
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) r.o[n][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        for (int v0 = p.u0; v0 < p.u1; v0 += kIds) {
            if (v0 > p.u0) {
                __syncthreads();
                put_ids(ask_ids(a.c, p, v0, min(p.u1, v0 + kIds)), v0, min(p.u1, v0 + kIds), lds.ids);
                __syncthreads();
            }
            run<NT>(a, p, v0, min(p.u1, v0 + kIds), least_len, most_low, lds, r);
        }

        // the four waves' states become one
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            r.l[n] = sum_xor32(sum_xor16(r.l[n]));
            if (g == 0) {
                lds.wave_m[wave][16 * n + m] = r.m[n];
                lds.wave_l[wave][16 * n + m] = r.l[n];
            }
        }
        float* wave_o = reinterpret_cast<float*>(lds.q);   // [wave][column][channel]
        const int quads = dim >> 2;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int count = p.count - 16 * n < 16 ? p.count - 16 * n : 16;
            if (count <= 0) break;
            __syncthreads();                              // q, and the tile before, have been read
            float top = lds.wave_m[0][16 * n + m];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds.wave_m[w][16 * n + m]);
            const float f = r.m[n] == kNegInf ? 0.0f : exp2_fast(r.m[n] - top);
            if (m < count) {
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) *reinterpret_cast<v4f*>(&wave_o[(wave * 16 + m) * DP + 16 * t + 4 * g]) = r.o[n][t] * f;
            }
            __syncthreads();
            for (int i = tid; i < count * quads; i += kThreads) {
                const int col = i / quads, d = 4 * (i - col * quads);
                v4f o = *reinterpret_cast<const v4f*>(&wave_o[col * DP + d]);
#pragma unroll
                for (int w = 1; w < kWaves; ++w) o += *reinterpret_cast<const v4f*>(&wave_o[(w * 16 + col) * DP + d]);
                if (!all_finite(o)) lds.odd = 1;
                float* rec = record_of(a, p, 16 * n + col);
                *reinterpret_cast<v4f*>(rec + 4 + d) = o;
                if (d == 0) {
                    float mm = kNegInf, ll = 0.0f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, lds.wave_m[w][16 * n + col]);
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) {
                        const float wm = lds.wave_m[w][16 * n + col];
                        ll += lds.wave_l[w][16 * n + col] * (wm == kNegInf ? 0.0f : exp2_fast(wm - mm));
                    }
                    rec[0] = mm;
                    rec[1] = ll;
                }
            }
        }
        __syncthreads();
    }
};

// The records of all that a work group has written, from plain products key by key.  A call, and everything worked out again from
// the kernel's arguments, so that the kernel keeps its registers to itself.
template <int T, bool F32>
__device__ __noinline__ void redo(uint64_t args, const Index* x) {
    const uint32_t low = __builtin_amdgcn_readfirstlane((int)args), high = __builtin_amdgcn_readfirstlane((int)(args >> 32));
    args = (uint64_t)high << 32 | low;
    const SharedArgs a = *(const SharedArgs*)(const __attribute__((address_space(4))) void*)args;
    const int dim = a.c.dim, d = 4 * (threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t all = x->start[a.n_seqs], share = share_of(a, all);
    int64_t pos = blockIdx.x * share;
    const int64_t end = pos + share < all ? pos + share : all;
    while (pos < end) {
        const Place p = place_of(a, *x, pos, end);
        pos = p.next;
        for (int column = wave; column < p.count; column += kWaves) {
            if (p.u0 >= p.u1) break;
            const Column col = column_of(a, p, column);
            const int len = x->len[col.s];
            const float4 q = load4<T, F32>(a.q, ((int64_t)(a.first_seq + col.s) * a.heads + col.head) * dim + (d < dim ? d : 0));
            float m = kNegInf, l = 0.0f;
            v4f o = {0.0f, 0.0f, 0.0f, 0.0f}, odd = o;
            for (int u = p.u0; u < p.u1; ++u) {
                const int key = unit_key(p.keys, u);
                plain_keys<T>(a, q, p.table_row, p.kvh, max(key, p.keys.begin), min(key + kUnit, p.keys.end), len, behind(a, len), d, m, l, o, odd);
            }
            o = or_infinite(o, odd);
            float* rec = record_of(a, p, column);
            if (d < dim) *reinterpret_cast<v4f*>(rec + 4 + d) = o;
            if (d == 0) {
                rec[0] = m;
                rec[1] = l;
            }
        }
    }
}

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : 2) void attn_shared_kernel(SharedArgs a) {
    using S = Shared<T, DP, F32, FULL, PAGE16>;
    __shared__ typename S::Lds lds;
    const int tid = threadIdx.x;
    if (tid == 0) lds.odd = 0;
    build_index(a, lds.index, lds.wave_cost, lds.wave_lead);
    const Index& x = lds.index;
    const int64_t all = x.start[a.n_seqs], share = share_of(a, all);
    if (blockIdx.x == gridDim.x - 1) {                    // the last one, which has the least to do
        Header* h = reinterpret_cast<Header*>(a.ws);
        if (tid == 0) {
            h->share = share;
            h->start[a.n_seqs] = all;
            h->first_row = x.first_row;
        }
        for (int s = tid; s < a.n_seqs; s += kThreads) {
            h->start[s] = x.start[s];
            const bool wide = is_wide(a, x, s);
            h->wide[s] = wide;
            h->prefix_units[s] = wide ? keys_of<kWideTile>(0, x.prefix[s], x.low[s], a.n_sink).units : prefix_keys(a, x, s).units;
            h->own_units[s] = own_keys(a, x, s).units;
            h->lead[s] = x.lead[s];
            h->members[s] = x.members[s];
            h->prefix[s] = x.prefix[s];
            h->low[s] = x.low[s];
        }
        if (a.wide_groups) {
            sum_line(a.n_seqs, [&](int s) { return wide_cost(a, x, s); }, h->wide_start, lds.wave_cost);
            if (tid == 0) h->wide_share = line_share(h->wide_start[a.n_seqs], a.wide_groups, kWideStart + 2 * kWideCost);
        }
    }
    int64_t pos = blockIdx.x * share;
    const int64_t end = pos + share < all ? pos + share : all;
    while (pos < end) {
        const Place p = place_of(a, x, pos, end);
        pos = p.next;
        if (p.u0 >= p.u1) continue;
        const int tiles = tiles_of(p.count);
        if (tiles == 1) S::template do_row<1>(a, p, lds);
        else if (most_tiles(DP) == 2 || tiles == 2) S::template do_row<2>(a, p, lds);
        else S::template do_row<most_tiles(DP)>(a, p, lds);
    }
    __syncthreads();
    if (__builtin_expect(lds.odd, 0)) redo<T, F32>((uint64_t)__builtin_amdgcn_kernarg_segment_ptr(), &lds.index);
}

// A sequence's records, first those of the prefix, in the order of the keys.  A work group 64 quads of channels (head, 4
// channels); its four waves take the records in turn and are added up in order.
template <int T, bool F32>
__global__ __launch_bounds__(256) void attn_shared_join_kernel(SharedArgs a) {
    __shared__ v4f part_o[4][64];
    __shared__ float part_m[4][64], part_l[4][64];
    const Header* h = reinterpret_cast<const Header*>(a.ws);
    const int dim = a.c.dim, quads = dim >> 2, s = blockIdx.x;
    const int lead = h->lead[s];
    if (lead == kNobody) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i = blockIdx.y * 64 + lane;
    const bool in = i < a.heads * quads;
    const int head = in ? i / quads : 0, d = in ? 4 * (i - head * quads) : 0;
    const int kvh = head / a.group, in_group = head - kvh * a.group;

    // the records of the prefix and of the own keys, and their columns
    const int members = h->members[lead], columns = members * a.group, col = (s - lead) * a.group + in_group;
    const bool wide = h->wide[lead];
    const int width = wide ? a.wide_columns : a.columns, rows = (columns + width - 1) / width, row = kvh * rows + col / width;
    const int units = h->prefix_units[lead], cost = wide ? kWideCost : cost_of_columns(a, columns), start = wide ? kWideStart : kStartCost;
    const Parts of_prefix = parts_of_row((wide ? h->wide_start : h->start)[lead] + row * line_cost(units, cost, start), units, wide ? 0 : kWholeUnits, cost, start,
                                         wide ? h->wide_share : h->share);
    const int own_units = h->own_units[s], own_cost = cost_of_columns(a, a.group), own_row = kvh * rows_of(a, a.group) + in_group / a.columns;
    const Parts of_own = parts_of_row(h->start[s] + cost_of_rows(a, h->members[s] * a.group, h->wide[s] ? 0 : h->prefix_units[s]) +
                                          own_row * line_cost(own_units, own_cost, kStartCost),
                                      own_units, kWholeUnits, own_cost, kStartCost, h->share);
    auto record = [&](int j) -> const float* {
        if (j < of_prefix.count) {
            if (of_prefix.count == 1) return whole_record(a, 0, s, head);
            return wide ? wide_record(a, of_prefix.first + j, j == 0 ? 1 : 0, col % width) : part_record(a, of_prefix.first + j, j == 0 ? 1 : 0, col % width);
        }
        j -= of_prefix.count;
        if (of_own.count == 1) return whole_record(a, 1, s, head);
        return part_record(a, of_own.first + j, j == 0 ? 1 : 0, in_group % a.columns);
    };
    const int total = of_prefix.count + of_own.count;
    float m = kNegInf, l = 0.0f;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int j = wave; j < total; j += 4) {
        const float* rec = record(j);
        const float pm = rec[0], pl = rec[1];
        const v4f po = *reinterpret_cast<const v4f*>(rec + 4 + d);
        const float top = fmaxf(m, pm);
        const float fa = m == kNegInf ? 0.0f : exp2_fast(m - top), fb = pm == kNegInf ? 0.0f : exp2_fast(pm - top);
        o = o * fa + po * fb;
        l = l * fa + pl * fb;
        m = top;
    }
    part_m[wave][lane] = m;
    part_l[wave][lane] = l;
    part_o[wave][lane] = o;
    __syncthreads();
    if (wave != 0 || !in) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float pm = part_m[w][lane];
        const float top = fmaxf(m, pm);
        const float fa = m == kNegInf ? 0.0f : exp2_fast(m - top), fb = pm == kNegInf ? 0.0f : exp2_fast(pm - top);
        o = o * fa + part_o[w][lane] * fb;
        l = l * fa + part_l[w][lane] * fb;
        m = top;
    }
    if (__builtin_expect(!all_finite(o) && l == l, 0)) {
        v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < total; ++j) sum = add_infinite(sum, *reinterpret_cast<const v4f*>(record(j) + 4 + d));
        o = or_infinite(o, sum);
    }
    l = l == 0.0f ? 1.0f : l;                             // no weight: o is 0
    const int64_t at = ((int64_t)(a.first_seq + s) * a.heads + head) * dim + d;
    store4<T, F32>(a.out, at, o[0] / l, o[1] / l, o[2] / l, o[3] / l);
}

// Columns of a row, at most: as many tiles as all of a launch's sequences could fill.
int columns_of(int64_t n_seqs, int group, int dim) {
    const int64_t all = (n_seqs < kSharedSeqs ? n_seqs : kSharedSeqs) * (int64_t)group;
    const int most = 16 * most_tiles(dim);
    return all <= 16 ? 16 : all <= 32 ? 32 : most;
}

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
hipError_t launch_page(SharedArgs a, hipStream_t s) {
    const int places = (DP > 128 ? 1 : 2) * device_cus(), groups = places < kSharedGroups ? places : kSharedGroups;
    const int total = a.c.n_seqs;
    a.rule = wide_rule(DP, F32, F32 && T == kBf16);
    a.wide_columns = wide_columns(DP, F32);
    for (int at = 0; at < total; at += kSharedSeqs) {
        a.first_seq = at;
        a.n_seqs = total - at < kSharedSeqs ? total - at : kSharedSeqs;
        const bool wide = attn_shared_may_be_wide((int64_t)a.n_seqs * a.group, (int64_t)a.c.max_pages << a.c.shift, a.c.kv_heads, a.c.dim, F32, F32 && T == kBf16);
        a.wide_groups = wide ? attn_shared_wide_groups(a.c.dim, F32) : 0;
        hipLaunchKernelGGL((attn_shared_kernel<T, DP, F32, FULL, PAGE16>), dim3((unsigned)groups), dim3(kThreads), 0, s, a);
        if (a.wide_groups) {
            const hipError_t e = launch_attn_shared_wide(a, T, F32, s);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((attn_shared_join_kernel<T, F32>), dim3((unsigned)a.n_seqs, (unsigned)((a.heads * (a.c.dim / 4) + 63) / 64)),
                           dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

template <int T, int DP, bool F32, bool FULL>
hipError_t launch(const SharedArgs& a, hipStream_t s) {
    return a.c.shift == 4 ? launch_page<T, DP, F32, FULL, true>(a, s) : launch_page<T, DP, F32, FULL, false>(a, s);
}

template <int T, bool F32>
hipError_t launch_dim(const SharedArgs& a, hipStream_t s) {
    if (a.c.dim <= 64) return a.c.dim == 64 ? launch<T, 64, F32, true>(a, s) : launch<T, 64, F32, false>(a, s);
    if (a.c.dim <= 128) return a.c.dim == 128 ? launch<T, 128, F32, true>(a, s) : launch<T, 128, F32, false>(a, s);
    return launch<T, 256, F32, false>(a, s);
}

}  // namespace

bool attn_shared_may_be_wide(int64_t columns, int64_t keys, int kv_heads, int dim, bool f32, bool three_parts) {
    const int width = wide_columns(dim, f32);
    for (const int64_t c : {columns, columns / width * width})
        if (worth_wide(wide_rule(dim, f32, three_parts), c, 16 * most_tiles(dim), width, keys, kv_heads)) return true;
    return false;
}

size_t attn_shared_workspace_bytes(int64_t n_seqs, int heads, int kv_heads, int dim, int64_t keys) {
    const int64_t n = n_seqs < kSharedSeqs ? n_seqs : kSharedSeqs, group = heads / kv_heads;
    const int narrow = columns_of(n, (int)group, dim);
    // (work groups times columns of the launch for wide prefixes: as many with 128 columns as with 256)
    bool wide = false;
    for (int f32 = 0; f32 < 2; ++f32)
        for (int three = 0; three <= f32; ++three) wide |= attn_shared_may_be_wide(n * group, keys, kv_heads, dim, f32 != 0, three != 0);
    const int64_t columns = narrow + (wide ? 128 : 0);
    const int64_t records = 2 * n * heads + 2 * kSharedGroups * columns;
    return (size_t)kHeaderBytes + (size_t)records * record_floats(dim) * 4;
}

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
    a.columns = columns_of(c.n_seqs, a.group, c.dim);
    a.ws = static_cast<uint8_t*>(ws);
    if (dtype == kBf16) return args.f32 ? launch_dim<kBf16, true>(a, s) : launch_dim<kBf16, false>(a, s);
    return args.f32 ? launch_dim<kF16, true>(a, s) : launch_dim<kF16, false>(a, s);
}

}  // namespace bitnet
