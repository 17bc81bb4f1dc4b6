// Attention of one new token per sequence over the paged cache:
//   out[b, h] = sum_j p_j v_j,  p = softmax over the visible keys j of scale q[b, h] . k_j
// (visible: j < L, and with a window j >= L - window or j < n_sink; nothing visible: zeros).
//
// The cache's bytes bound it: 4 Hkv D bytes a key for 4 Hq D operations.  Keys go through in units of 32, all query heads of
// a kv head (up to 16, a "row") at once on the 16 columns of the matrix instruction: S^T = K Q^T (two tiles of 16 keys) and
// O^T = V^T P^T.  The rows of the two key tiles are chosen so that a lane's eight scores are those of eight consecutive keys,
// which is its operand of the second product: the weights never leave their lane.  Maximum and sum of the softmax run along
// (one pass over the cache), in 32 bits; the matrix instructions have so much room here that q and the weights go in as sums
// of parts of the cache's type (see Elem): from 32-bit inputs three of bf16 (all 24 bits) or two of f16 (22 bits); of the cache's
// type q is one part as it is, and the weights two, 16 bits of bf16 and 22 of f16, beside a sum of all their bits: less than
// 2^-15 of the output, a 64th of its own rounding.
//
// Work is split evenly whatever the lengths: all units of the launch in one line (sequence, kv head, unit), one share of equal
// length for every work group, which its four waves take in turn.  A row that crosses shares leaves partial results (maximum,
// sum, unnormalised output) in the workspace, and a second launch joins them.
//
// A value that is infinite makes its channel so, whatever its weight, and a key whose score is -inf has no weight.  The products
// give NaN for both, because infinities meet weights, and parts of weights and of q, that are 0.  But they leave no such output
// finite: finite ones need no look at keys and values, and a share with others is gone through once more, key by key (plain).
//
// Measured (kernel times; D = 128, 32 heads of 8 kv heads unless said): one sequence of 131071 keys 82 us (6.5 TB/s of keys and
// values) and 5 to join; 32 sequences of up to 6000 keys 76 (5.3 TB/s) and 5; 24 sequences of 32 heads of 100, f16, behind a
// window of 1024, 57 us whole (5.3 TB/s); one of 61 keys 5.8 us (in a table of 5 pages; where the table has room for more than
// 256 keys, rows may be split and a second launch joins them: the pass takes 12 us, not 8).  A large plain read reaches 6.4 to
// 7.0 TB/s here.  What is left is a share's start: length, pages and first keys are three reads in a row, and rows that end inside
// a share start anew.
#include "kv_cache.hpp"

#include <type_traits>

namespace bitnet {
namespace {

constexpr int kUnit = 32;            // keys of a unit
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kMaxGroups = 1024;     // work groups of a split launch
constexpr int kMaxSeqs = 1024;       // sequences of a split launch (more go in several)
constexpr int kMinShare = 4;         // units of a share, at least: one for each wave
// Rows of up to kWholeUnits units are never split (61 keys: 5.8 us in one launch, where the join alone takes 4 to 5), nor rows of up
// to kManyUnits where there are kManyRows of them: a work group a row is enough then, and the join is saved (24 x 32 rows of
// 1028 keys: 57 us whole).
constexpr int kWholeUnits = 8;
constexpr int kManyUnits = 64;
constexpr int kManyRows = 512;
constexpr int kIds = 512;            // units whose pages a work group looks up at a time

// The keys that the last position of a sequence of length L sees: [0, sinks) and [lo, L).
struct Sight {
    int len, lo, sinks, sink_units, first_unit, units;   // units of the sinks, first unit of the window, all units
};
__host__ __device__ __forceinline__ Sight sight_of(int len, int window, int n_sink) {
    Sight s;
    s.len = len;
    s.lo = window > 0 && len > window ? len - window : 0;
    s.sinks = n_sink < s.lo ? n_sink : s.lo;
    s.first_unit = s.lo / kUnit;
    s.sink_units = (s.sinks + kUnit - 1) / kUnit;
    if (s.sink_units > s.first_unit) s.sink_units = s.first_unit;
    s.units = s.sink_units + (len + kUnit - 1) / kUnit - s.first_unit;
    return s;
}
__device__ __forceinline__ int unit_key(const Sight& s, int u) {
    return (u < s.sink_units ? u : u - s.sink_units + s.first_unit) * kUnit;
}

// Workspace of a split launch: header ints {share, units of all rows}, prefix of the units of the sequences, then two slots
// a work group of {max[16], sum[16], output [rows16, D]} floats.
constexpr int kHeadInts = 64;
__host__ __device__ __forceinline__ int64_t slot_floats(int rows, int dim) { return 32 + (int64_t)rows * dim; }
constexpr int64_t kPrefixBytes = 4 * (kHeadInts + ((kMaxSeqs + 1 + 63) / 64) * 64);

struct DecodeArgs {
    KvCache c;
    const void* q;
    void* out;
    int heads, group, tiles, rows;   // query heads, of a kv head, 16-head tiles of those, heads of a tile at most (<= 16)
    float scale2;                    // scale * log2 e
    int window, n_sink;
    int first_seq, n_seqs;           // of this launch
    int32_t* ws;                     // null: one work group a row
};

// What a work group is at: a row, or the units of one that its share reaches, from `pos` on (prefix: units of all sequences
// before each of them; unused where rows stay whole).
struct Place {
    int b, kvh, head0, count;            // sequence, kv head, first query head and number of them
    int u0, u1, units, stop;             // units [u0, u1) of the row's; those that hold keys end at stop
    Sight sight;
};
__device__ __forceinline__ Place place_of(const DecodeArgs& a, const int* prefix, int64_t pos, int64_t end) {
    const int per_seq = a.c.kv_heads * a.tiles;          // rows of a sequence
    Place p;
    int s, row;
    if (a.ws) {
        int lo = 0, hi = a.n_seqs - 1;                    // the last sequence that starts at pos or before
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((int64_t)prefix[mid] * per_seq <= pos) lo = mid;
            else hi = mid - 1;
        }
        s = lo;
        p.units = prefix[s + 1] - prefix[s];
        const int at = (int)(pos - (int64_t)prefix[s] * per_seq);
        row = at / p.units;
        p.u0 = at - row * p.units;
        p.u1 = end - pos < p.units - p.u0 ? p.u0 + (int)(end - pos) : p.units;
    } else {
        s = blockIdx.x / per_seq;
        row = blockIdx.x - s * per_seq;
        p.u0 = 0;
    }
    p.b = a.first_seq + s;
    p.sight = sight_of(seq_len(a.c, p.b), a.window, a.n_sink);
    if (!a.ws) p.u1 = p.units = p.sight.units;
    p.kvh = row / a.tiles;
    const int tile = row - p.kvh * a.tiles;
    p.head0 = p.kvh * a.group + tile * 16;
    p.count = a.group - tile * 16 < 16 ? a.group - tile * 16 : 16;
    p.stop = p.u1 < p.sight.units ? p.u1 : p.sight.units;
    return p;
}

// The share of this work group: units [pos, end) of the line of all (whole rows: one).
struct Share {
    int64_t pos, end;
    int units;
};
__device__ __forceinline__ Share share_of(const DecodeArgs& a, const int* prefix) {
    if (!a.ws) return {0, 1, 0};
    const int64_t all = (int64_t)prefix[a.n_seqs] * a.c.kv_heads * a.tiles;
    const int want = (int)((all + gridDim.x - 1) / gridDim.x), units = want < kMinShare ? kMinShare : want;
    const int64_t pos = (int64_t)blockIdx.x * units;
    return {pos, pos + units < all ? pos + units : all, units};
}

// A wave's state of one row: running maximum, sum and unnormalised output; lane (n = lane & 15, g = lane >> 4) holds head n,
// channels 16 t + 4 g + i of o[t].
template <int DP>
struct Row {
    float m, l;
    v4f o[DP / 16];
};

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
struct Decode {
    static constexpr int kQParts = F32 ? Elem<T>::kExactParts : 1;
    static constexpr int kPParts = F32 ? Elem<T>::kExactParts : 2;
    static constexpr int kChunks = DP / 8;
    static constexpr int kQBytes = kQParts * kChunks * 16 * 16;

    // q of up to 16 heads as operands in LDS: [part][chunk][head][8]; zeros past D and past the row's heads.  Returns the
    // factor of the scores of this lane's head (its column n).
    static __device__ __forceinline__ void stage_q(const DecodeArgs& a, int b, int head0, int count, uint4* qs, float* gain) {
        const int n = threadIdx.x >> 4, sub = threadIdx.x & 15;
        const int64_t at = ((int64_t)b * a.heads + head0 + n) * a.c.dim;
        float x[DP / 128 ? DP / 128 : 1][8];
        float top = 0.0f;
#pragma unroll
        for (int r = 0; r < (DP + 127) / 128; ++r) {
            const int d = 8 * (sub + 16 * r);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (n < count && d + 4 * half < a.c.dim) v = load4<T, F32>(a.q, at + d + 4 * half);
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
        if (sub == 0) gain[n] = a.scale2 / up;
#pragma unroll
        for (int r = 0; r < (DP + 127) / 128; ++r) {
            const int c = sub + 16 * r;
            if (c >= kChunks) continue;
            if constexpr (F32 && T == kF16) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[r][e] *= up;
            }
#pragma unroll
            for (int p = 0; p < kQParts; ++p) {
                uint4 w;
                if constexpr (kQParts == 1) {   // values of the cache's type: exact
                    w = make_uint4(Elem<T>::pack(x[r][0], x[r][1]), Elem<T>::pack(x[r][2], x[r][3]),
                                   Elem<T>::pack(x[r][4], x[r][5]), Elem<T>::pack(x[r][6], x[r][7]));
                } else {
                    w.x = Elem<T>::part(x[r][0], x[r][1]);
                    w.y = Elem<T>::part(x[r][2], x[r][3]);
                    w.z = Elem<T>::part(x[r][4], x[r][5]);
                    w.w = Elem<T>::part(x[r][6], x[r][7]);
                }
                qs[(p * kChunks + c) * 16 + n] = w;
            }
        }
    }

    // The pages of units u0 .. u1 - 1 (at most kIds), and, pages of 16, those of their upper halves.  In LDS, so that waiting for a
    // page number does not wait for the keys and values that are on their way.
    static __device__ __forceinline__ void stage_ids(const KvCache& c, int b, const Sight& sight, int u0, int u1, int (&ids)[2][kIds]) {
        const int32_t* table = c.table + (int64_t)b * c.max_pages;
        for (int i = threadIdx.x; i < u1 - u0; i += kThreads) {
            const int at = unit_key(sight, u0 + i) >> c.shift;
            ids[0][i] = table[at];
            if (PAGE16) ids[1][i] = at + 1 < c.max_pages ? table[at + 1] : -1;
        }
    }

    // Units u0 .. u1 - 1 of a row (their pages in ids), this wave's every fourth, into its state.
    static __device__ __forceinline__ void run(const DecodeArgs& a, int kvh, const Sight& sight, int u0, int u1,
                                               const int (&ids)[2][kIds], const uint4* qs, float gain, Row<DP>& row) {
        const KvCache& c = a.c;
        const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int ps = PAGE16 ? 16 : 1 << c.shift;
        const int dim = FULL ? DP : c.dim, chunks = FULL ? DP / 8 : c.chunks;
        const int first = u0 + wave;
        const int count = first < u1 ? (u1 - first + kWaves - 1) / kWaves : 0;
        if (count == 0) return;
        const uint16_t* kbase = c.k + (int64_t)kvh * chunks * ps * 8;
        const uint16_t* vbase = c.v + (int64_t)kvh * dim * ps;
        // places of this lane's words in a unit: of the keys, key 8 (m / 4) + m % 4 (+ 4 in the second tile) of chunk g (+ 4 j);
        // of the values, channel m (+ 16 t) of the eight keys g.  Read once, so past the caches (131071 keys 93 us, with
        // ordinary loads 104).
        const uint32_t k_lane = (uint32_t)(g * ps + 8 * (m >> 2) + (m & 3)) * 16, v_lane = (uint32_t)(g * dim + m) * 16;
        auto load = [](const uint16_t* base, uint32_t offset) {
            return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(reinterpret_cast<const uint8_t*>(base) + offset));
        };

        auto page_of = [&](int half, int it) { return __builtin_amdgcn_readfirstlane(ids[half][wave + kWaves * it]); };
        v4u kf[2][DP / 32], vf[DP / 16];
        auto issue_k = [&](int it) {
            const int key = unit_key(sight, first + kWaves * it);
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
            const int key = unit_key(sight, first + kWaves * it);
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

        issue_k(0);
        issue_v(0);
        // one unit; MORE: the next one's keys are asked for as soon as the scores are formed, its values after the product (known
        // when compiled: where a load may or may not be on its way, every wait is for all of them)
        auto step = [&](int it, auto more_) {
            constexpr bool MORE = decltype(more_)::value;
            const int key = unit_key(sight, first + kWaves * it);
            const bool ok0 = page_ok(c, page_of(0, it)), ok1 = PAGE16 ? page_ok(c, page_of(1, it)) : ok0;
            v4f s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            int q_at = g * 16 + m;
            asm volatile("" : "+v"(q_at));                // q stays in LDS: in registers it would halve the waves
#pragma unroll
            for (int p = 0; p < kQParts; ++p) {
#pragma unroll
                for (int j = 0; j < DP / 32; ++j) {
                    const uint4 qw = qs[(p * kChunks + 4 * j) * 16 + q_at];
                    const v4u qf = {qw.x, qw.y, qw.z, qw.w};
                    s[0] = Elem<T>::mfma16(kf[0][j], qf, s[0]);
                    s[1] = Elem<T>::mfma16(kf[1][j], qf, s[1]);
                }
            }
            if constexpr (MORE) {
                issue_k(it + 1);
            }
            // scores of the keys key + 8 g + e, e = 4 t + i
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * gain;
            const bool whole = (ok0 & ok1 & (key + kUnit <= sight.len) & ((key >= sight.lo) | (key + kUnit <= sight.sinks))) != 0;
            if (!whole) {
                const bool there = g < 2 ? ok0 : ok1;
                uint32_t seen = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = key + 8 * g + e;
                    const bool in = there & (j < sight.len) & ((j >= sight.lo) | (j < sight.sinks));
                    seen |= in ? 1u << e : 0u;
                    x[e] = in ? x[e] : kNegInf;
                }
                // nothing that is not visible enters the second product: 0 times an infinity would be no 0
                v4u keep;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    keep[w] = ((seen >> (2 * w)) & 1 ? 0x0000FFFFu : 0u) | ((seen >> (2 * w)) & 2 ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) vf[t] &= keep;
            }
            float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            top = max_xor32(max_xor16(top));
            const float m_new = fmaxf(row.m, top);
            if (__any(m_new > row.m)) {
                const float alpha = m_new == kNegInf ? 1.0f : exp2_fast(row.m - m_new);
                row.l *= alpha;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) row.o[t] *= alpha;
                row.m = m_new;
            }
            const float base = (row.m == kNegInf ? 0.0f : row.m) - kLift<T>;
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = exp2_fast(x[e] - base);
                sum += x[e];
            }
            row.l += sum;
#pragma unroll
            for (int p = 0; p < kPParts; ++p) {
                const v4u pf = {Elem<T>::part(x[0], x[1]), Elem<T>::part(x[2], x[3]), Elem<T>::part(x[4], x[5]),
                                Elem<T>::part(x[6], x[7])};
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) row.o[t] = Elem<T>::mfma16(vf[t], pf, row.o[t]);
            }
            if constexpr (MORE) issue_v(it + 1);
        };
        for (int it = 0; it + 1 < count; ++it) step(it, std::true_type{});
        step(count - 1, std::false_type{});
    }

    // A head's keys in units u0 .. u1 - 1 once more, in plain 32-bit products: the finite values weighted, and those that are not
    // finite added up beside them.  A lane holds channels d = 4 lane .. of q and of the output; every lane the maximum and the sum.
    static __device__ __forceinline__ void plain(const DecodeArgs& a, int b, int head, int kvh, const Sight& sight, int u0, int u1,
                                                 int d, float& m, float& l, v4f& o) {
        const KvCache& c = a.c;
        const int32_t* table = c.table + (int64_t)b * c.max_pages;
        const int ps = 1 << c.shift;
        const bool in = d < c.dim;
        const int ch = in ? d : 0;                        // lanes past D read the first channels and hold none
        const float4 q = load4<T, F32>(a.q, ((int64_t)b * a.heads + head) * c.dim + ch);
        v4f odd = {0.0f, 0.0f, 0.0f, 0.0f};
        m = kNegInf;
        l = 0.0f;
        o = odd;
        for (int i = 4 * u0; i < 4 * u1; ++i) {           // eight keys at a time: of one page, and of one word of the values
            const int key = unit_key(sight, i >> 2) + 8 * (i & 3), slot = key & (ps - 1);
            if (key >= sight.len) break;
            const int page = table[key >> c.shift];
            if (!page_ok(c, page)) continue;
            const int64_t k_at = (int64_t)page * c.k_page + ((int64_t)(kvh * c.chunks + (ch >> 3)) * ps + slot) * 8 + (ch & 4);
            const uint16_t* v_at = c.v + (int64_t)page * c.v_page + (int64_t)kvh * c.dim * ps + (slot >> 3) * c.dim * 8 + ch * 8;
            float x[8], top = m;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float4 k = load4<T, false>(c.k, k_at + 8 * e);
                x[e] = in ? q.x * k.x + q.y * k.y + (q.z * k.z + q.w * k.w) : 0.0f;
#pragma unroll
                for (int t = 0; t < 4; ++t) x[e] += __int_as_float(dpp_row_step(__float_as_int(x[e]), t));
                const int j = key + e;
                const bool seen = (j < sight.len) & ((j >= sight.lo) | (j < sight.sinks));
                x[e] = seen ? sum_xor32(sum_xor16(x[e])) * a.scale2 : kNegInf;
                top = fmaxf(top, x[e]);
            }
            const float alpha = m == top ? 1.0f : exp2_fast(m - top), base = (top == kNegInf ? 0.0f : top) - kLift<T>;
            m = top;
            l *= alpha;
            o *= alpha;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = key + e;
                x[e] = exp2_fast(x[e] - base);
                l += x[e];
                if (j < sight.len && (j >= sight.lo || j < sight.sinks)) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const float v = Elem<T>::to(v_at[8 * t + e]);
                        if (v * 0.0f == 0.0f) o[t] += x[e] * v;
                        else odd[t] += v;
                    }
                }
            }
        }
        o = or_infinite(o, odd);
    }
};

// What `plain` gives, in the place of all that a work group has written.  A call, and everything worked out again from the kernel's
// arguments, so that the kernel keeps its registers and its code to itself: inlined in several ways it cost batches of short rows 5
// to 10% (52 sequences of up to 110 keys, 16 heads of 100: 12.1 to 12.6 us, this way 11.7, without it 11.4).
template <int T, int DP, bool F32, bool FULL, bool PAGE16>
__device__ __noinline__ void redo(uint64_t args, const int* prefix) {
    const uint32_t low = __builtin_amdgcn_readfirstlane((int)args), high = __builtin_amdgcn_readfirstlane((int)(args >> 32));
    args = (uint64_t)high << 32 | low;
    const DecodeArgs a = *(const DecodeArgs*)(const __attribute__((address_space(4))) void*)args;
    const int dim = a.c.dim, d = 4 * (threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Share share = share_of(a, prefix);
    for (int64_t pos = share.pos; pos < share.end;) {
        const Place p = place_of(a, prefix, pos, share.end);
        const bool whole = p.u0 == 0 && p.u1 == p.units;
        float* part = reinterpret_cast<float*>(a.ws) + kPrefixBytes / 4 +
                      (2 * (int64_t)blockIdx.x + (pos == share.pos ? 0 : 1)) * slot_floats(a.rows, dim);
        for (int head = wave; head < p.count; head += kWaves) {
            float m, l;
            v4f o;
            Decode<T, DP, F32, FULL, PAGE16>::plain(a, p.b, p.head0 + head, p.kvh, p.sight, p.u0, p.stop, d, m, l, o);
            if (d >= dim) continue;
            if (whole) {
                l = l == 0.0f ? 1.0f : l;                 // no weight: o is 0
                store4<T, F32>(a.out, ((int64_t)p.b * a.heads + p.head0 + head) * dim + d, o[0] / l, o[1] / l, o[2] / l, o[3] / l);
            } else {
                part[head] = m;
                part[16 + head] = l;
                *reinterpret_cast<v4f*>(part + 32 + (int64_t)head * dim + d) = o;
            }
        }
        if (!a.ws) break;
        pos += p.u1 - p.u0;
    }
}

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
__global__ __launch_bounds__(kThreads, DP > 128 ? 1 : FULL ? 2 : 3) void attn_decode_kernel(DecodeArgs a) {
    using D = Decode<T, DP, F32, FULL, PAGE16>;
    __shared__ uint4 qs[D::kQBytes / 16];
    __shared__ float gain[16];
    __shared__ float wave_m[kWaves][16], wave_l[kWaves][16];
    __shared__ int prefix[kMaxSeqs + 1];
    __shared__ int wave_total[kWaves];
    __shared__ int ids[2][kIds];
    __shared__ int odd;                                   // some output is not finite
    extern __shared__ float wave_o[];                     // [wave][head][channel]
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int per_seq = a.c.kv_heads * a.tiles;           // rows of a sequence
    const int dim = a.c.dim;

    if (tid == 0) odd = 0;
    if (a.ws) {
        // units of all sequences before each of them
        int carry = 0;
        for (int s0 = 0; s0 < a.n_seqs; s0 += kThreads) {
            const int s = s0 + tid;
            int u = 0;
            if (s < a.n_seqs) {
                u = sight_of(seq_len(a.c, a.first_seq + s), a.window, a.n_sink).units;
                u = u > 0 ? u : 1;
            }
            int sum = u;
#pragma unroll
            for (int i = 1; i < 64; i <<= 1) {
                const int other = __shfl_up(sum, i);
                if (lane >= i) sum += other;
            }
            if (lane == 63) wave_total[wave] = sum;
            __syncthreads();
            int before = carry;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) before += w < wave ? wave_total[w] : 0;
            if (s < a.n_seqs) prefix[s] = before + sum - u;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) carry += wave_total[w];
            __syncthreads();
        }
        if (tid == 0) prefix[a.n_seqs] = carry;
        __syncthreads();
    }
    const Share share = share_of(a, prefix);
    if (a.ws && blockIdx.x == 0) {
        if (tid == 0) a.ws[0] = share.units;
        for (int s = tid; s <= a.n_seqs; s += kThreads) a.ws[kHeadInts + s] = prefix[s];
    }
    int64_t pos = share.pos;
    const int64_t end = share.end;
    const int64_t start = pos;

    while (pos < end) {
        const Place at = place_of(a, prefix, pos, end);
        const int b = at.b, head0 = at.head0, count = at.count, kvh = at.kvh, u0 = at.u0, u1 = at.u1, units = at.units, stop = at.stop;
        const Sight sight = at.sight;
        D::stage_q(a, b, head0, count, qs, gain);
        D::stage_ids(a.c, b, sight, u0, stop < u0 + kIds ? stop : u0 + kIds, ids);
        __syncthreads();

        Row<DP> r;
        r.m = kNegInf;
        r.l = 0.0f;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) r.o[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for (int v0 = u0; v0 < stop; v0 += kIds) {
            if (v0 > u0) {
                __syncthreads();
                D::stage_ids(a.c, b, sight, v0, stop < v0 + kIds ? stop : v0 + kIds, ids);
                __syncthreads();
            }
            D::run(a, kvh, sight, v0, stop < v0 + kIds ? stop : v0 + kIds, ids, qs, gain[n], r);
        }

        // the four waves' states become one
        r.l = sum_xor32(sum_xor16(r.l));
        if (g == 0) {
            wave_m[wave][n] = r.m;
            wave_l[wave][n] = r.l;
        }
        __syncthreads();
        float top = wave_m[0][n];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, wave_m[w][n]);
        const float f = r.m == kNegInf ? 0.0f : exp2_fast(r.m - top);
        if (n < count) {
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) {
                const v4f o = r.o[t] * f;
                *reinterpret_cast<v4f*>(&wave_o[(wave * a.rows + n) * DP + 16 * t + 4 * g]) = o;
            }
        }
        __syncthreads();
        const bool complete = u0 == 0 && u1 == units;
        float* slot = nullptr;
        if (!complete) {
            slot = reinterpret_cast<float*>(a.ws) + kPrefixBytes / 4 +
                   (2 * (int64_t)blockIdx.x + (pos == start ? 0 : 1)) * slot_floats(a.rows, dim);
            if (tid < 16) {
                float mm = kNegInf, ll = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, wave_m[w][tid]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    ll += wave_l[w][tid] * (wave_m[w][tid] == kNegInf ? 0.0f : exp2_fast(wave_m[w][tid] - mm));
                slot[tid] = mm;
                slot[16 + tid] = ll;
            }
        }
        const int quads = dim >> 2;
        for (int i = tid; i < count * quads; i += kThreads) {
            const int head = i / quads, d = 4 * (i - head * quads);
            v4f o = *reinterpret_cast<const v4f*>(&wave_o[head * DP + d]);
#pragma unroll
            for (int w = 1; w < kWaves; ++w) o += *reinterpret_cast<const v4f*>(&wave_o[(w * a.rows + head) * DP + d]);
            if (!all_finite(o)) odd = 1;
            if (complete) {
                float mm = kNegInf, ll = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, wave_m[w][head]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    ll += wave_l[w][head] * (wave_m[w][head] == kNegInf ? 0.0f : exp2_fast(wave_m[w][head] - mm));
                const bool none = ll == 0.0f;             // nothing visible
                store4<T, F32>(a.out, ((int64_t)b * a.heads + head0 + head) * dim + d, none ? 0.0f : o[0] / ll,
                               none ? 0.0f : o[1] / ll, none ? 0.0f : o[2] / ll, none ? 0.0f : o[3] / ll);
            } else {
                *reinterpret_cast<v4f*>(slot + 32 + (int64_t)head * dim + d) = o;
            }
        }
        if (!a.ws) break;
        pos += u1 - u0;
        __syncthreads();
    }
    __syncthreads();
    if (__builtin_expect(odd, 0)) redo<T, DP, F32, FULL, PAGE16>((uint64_t)__builtin_amdgcn_kernarg_segment_ptr(), prefix);
}

// Rows that crossed shares: their partial results, in the order of the keys.  One work group a row and 64 quads of channels
// (head, 4 channels); its four waves take the parts in turn and are added up in order.
template <int T, bool F32>
__global__ __launch_bounds__(256) void attn_join_kernel(DecodeArgs a) {
    __shared__ v4f part_o[4][64];
    __shared__ float part_m[4][64], part_l[4][64];
    const int per_seq = a.c.kv_heads * a.tiles, dim = a.c.dim;
    const int s = blockIdx.x / per_seq, row = blockIdx.x - s * per_seq;
    const int kvh = row / a.tiles, tile = row - kvh * a.tiles;
    const int count = a.group - tile * 16 < 16 ? a.group - tile * 16 : 16;
    const int share = a.ws[0];
    const int64_t before = a.ws[kHeadInts + s];
    const int units = a.ws[kHeadInts + s + 1] - (int)before;
    const int64_t first = before * per_seq + (int64_t)row * units, last = first + units - 1;
    const int w0 = (int)(first / share), w1 = (int)(last / share);
    if (w0 == w1) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i = blockIdx.y * 64 + lane, quads = dim >> 2;
    const bool in = i < count * quads;
    const int head = in ? i / quads : 0, d = in ? 4 * (i - head * quads) : 0;
    const float* slots = reinterpret_cast<const float*>(a.ws) + kPrefixBytes / 4;
    const int64_t step = slot_floats(a.rows, dim);
    float m = kNegInf, l = 0.0f;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int w = w0 + wave; w <= w1; w += 4) {
        const int which = w == w0 && first != (int64_t)w0 * share ? 1 : 0;
        const float* slot = slots + (2 * (int64_t)w + which) * step;
        const float pm = slot[head], pl = slot[16 + head];
        const v4f po = *reinterpret_cast<const v4f*>(slot + 32 + (int64_t)head * dim + d);
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
        for (int w = w0; w <= w1; ++w) {
            const int which = w == w0 && first != (int64_t)w0 * share ? 1 : 0;
            sum = add_infinite(sum, *reinterpret_cast<const v4f*>(slots + (2 * (int64_t)w + which) * step + 32 + (int64_t)head * dim + d));
        }
        o = or_infinite(o, sum);
    }
    l = l == 0.0f ? 1.0f : l;                             // no weight: o is 0
    const int64_t at = ((int64_t)(a.first_seq + s) * a.heads + kvh * a.group + tile * 16 + head) * dim + d;
    store4<T, F32>(a.out, at, o[0] / l, o[1] / l, o[2] / l, o[3] / l);
}

template <int T, int DP, bool F32, bool FULL, bool PAGE16>
hipError_t launch_page(DecodeArgs a, bool split, hipStream_t s) {
    const size_t lds = (size_t)kWaves * a.rows * DP * 4;
    const int rows = a.c.kv_heads * a.tiles;
    const int total = a.n_seqs, first = a.first_seq;
    const auto kern = attn_decode_kernel<T, DP, F32, FULL, PAGE16>;
    if (!split) {
        a.ws = nullptr;
        const int64_t most = (1 << 23) / rows;            // a grid has fewer than 2^32 threads
        for (int64_t at = 0; at < total; at += most) {
            a.first_seq = first + (int)at;
            a.n_seqs = (int)(total - at < most ? total - at : most);
            hipLaunchKernelGGL(kern, dim3((unsigned)(a.n_seqs * rows)), dim3(kThreads), lds, s, a);
        }
        return hipGetLastError();
    }
    // One round of work groups, each with keys and values of 16 DP KiB on their way: two a CU (DP <= 64: four) keep the memory
    // busy, and a third only starts and joins more parts (131071 keys of 8 heads 95 us against 98, 32 sequences 81 against 83).
    const int resident = resident_groups(reinterpret_cast<const void*>(kern), kThreads, lds), most = DP <= 64 ? 4 : 2;
    const int groups = (resident < most ? resident : most) * device_cus() < kMaxGroups ? (resident < most ? resident : most) * device_cus()
                                                                                      : kMaxGroups;
    for (int at = 0; at < total; at += kMaxSeqs) {
        a.first_seq = first + at;
        a.n_seqs = total - at < kMaxSeqs ? total - at : kMaxSeqs;
        hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kThreads), lds, s, a);
        hipLaunchKernelGGL((attn_join_kernel<T, F32>), dim3((unsigned)(a.n_seqs * rows), (unsigned)((a.rows * a.c.dim / 4 + 63) / 64)),
                           dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

template <int T, int DP, bool F32, bool FULL>
hipError_t launch(const DecodeArgs& a, bool split, hipStream_t s) {
    return a.c.shift == 4 ? launch_page<T, DP, F32, FULL, true>(a, split, s) : launch_page<T, DP, F32, FULL, false>(a, split, s);
}

// Heads of exactly 64 and 128 channels load without asking whether a word is there.  Of 256 they do not: with nothing to hold them
// back the next unit's loads come so early that registers spill (8 sequences of up to 8000 keys: 66 us as it is, 72 so).
template <int T, bool F32>
hipError_t launch_dim(const DecodeArgs& a, bool split, hipStream_t s) {
    if (a.c.dim <= 64) return a.c.dim == 64 ? launch<T, 64, F32, true>(a, split, s) : launch<T, 64, F32, false>(a, split, s);
    if (a.c.dim <= 128) return a.c.dim == 128 ? launch<T, 128, F32, true>(a, split, s) : launch<T, 128, F32, false>(a, split, s);
    return launch<T, 256, F32, false>(a, split, s);
}

int most_units(int64_t max_pages, int page_size, int window, int n_sink) {
    const int64_t keys = max_pages * page_size;
    int64_t units = (keys + kUnit - 1) / kUnit;
    if (window > 0) {
        const int64_t near = (window + kUnit - 1) / kUnit + 1 + ((int64_t)n_sink + kUnit - 1) / kUnit;
        units = near < units ? near : units;
    }
    return (int)units;
}

// Whether rows are split: not where the longest takes little longer than starting and joining parts would, nor where they are
// many and a window or a short table keeps them about alike (then the work groups are enough and the second launch is saved).
bool rows_split(int64_t n_seqs, int heads, int kv_heads, int page_size, int64_t max_pages, int window, int n_sink) {
    const int units = most_units(max_pages, page_size, window, n_sink);
    const int64_t rows = n_seqs * kv_heads * ((heads / kv_heads + 15) / 16);
    return units > kWholeUnits && (units > kManyUnits || rows < kManyRows);
}

}  // namespace

size_t attn_decode_workspace_bytes(int heads, int kv_heads, int dim, int page_size, int64_t max_pages, int window, int n_sink) {
    if (most_units(max_pages, page_size, window, n_sink) <= kWholeUnits) return 0;
    const int group = heads / kv_heads;
    return (size_t)kPrefixBytes + (size_t)(2 * kMaxGroups * slot_floats(group < 16 ? group : 16, dim)) * 4;
}

bool attn_decode_splits(int64_t n_seqs, int heads, int kv_heads, int page_size, int64_t max_pages, int window, int n_sink) {
    return rows_split(n_seqs, heads, kv_heads, page_size, max_pages, window, n_sink);
}

hipError_t launch_attn_decode(const KvCache& c, int dtype, const AttnArgs& args, void* ws, hipStream_t s) {
    DecodeArgs a{};
    a.c = c;
    a.q = args.q;
    a.out = args.out;
    a.heads = args.heads;
    a.group = args.heads / c.kv_heads;
    a.tiles = (a.group + 15) / 16;
    a.rows = a.group < 16 ? a.group : 16;
    a.scale2 = args.scale * kLog2e;
    a.window = args.window;
    a.n_sink = args.n_sink;
    a.n_seqs = c.n_seqs;
    a.ws = static_cast<int32_t*>(ws);
    const bool split = rows_split(c.n_seqs, args.heads, c.kv_heads, 1 << c.shift, c.max_pages, args.window, args.n_sink);
    if (dtype == kBf16) return args.f32 ? launch_dim<kBf16, true>(a, split, s) : launch_dim<kBf16, false>(a, split, s);
    return args.f32 ? launch_dim<kF16, true>(a, split, s) : launch_dim<kF16, false>(a, split, s);
}

}  // namespace bitnet
