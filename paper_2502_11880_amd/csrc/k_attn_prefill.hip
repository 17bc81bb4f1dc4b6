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
    int splits;                      // parts that the keys of each are divided into, at most
    int places;                      // work groups that the device holds at a time
    float* ws;                       // the parts' results, where there are several
};

// What the parts of a row of out (a token under a head) leave for joining: their references and sums, then their outputs.  By rows
// of out, not by work groups: sequences without tokens take no room.
__host__ __device__ __forceinline__ int held_parts(int splits) { return (splits + 1) & ~1; }   // outputs start at 16 bytes
__host__ __device__ __forceinline__ int64_t row_floats(int splits, int dim) { return (int64_t)held_parts(splits) * (2 + dim); }

// Work groups of sequence b start at floor(q group / columns) + min(b, q), q = q_start[b]: its n tokens take at most
// floor(n group / columns) + 1 of them, and no more than q sequences before it have tokens.
__device__ __forceinline__ int first_tile(const int32_t* q_start, int b, int n_tokens, int group, int columns) {
    const int q = min(max(q_start[b], 0), n_tokens);
    return (int)((int64_t)q * group / columns) + min(b, q);
}

// Parts of this call: as many as find a place beside the work groups that have tokens, which only the device can count where
// there are several sequences (one without tokens has none, one with a single token as many as kv heads).  Whole waves only.
__device__ __forceinline__ int parts_of(const PrefillArgs& a, int columns) {
    if (a.c.n_seqs == 1) return a.splits;
    int tiles = 0;
    for (int b = threadIdx.x & 63; b < a.c.n_seqs; b += 64)
        tiles += (span_of(a.q_start, b, a.n_tokens).count * a.group + columns - 1) / columns;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) tiles += __shfl_xor(tiles, i);
    tiles = __builtin_amdgcn_readfirstlane(tiles);
    if (tiles <= 0 || tiles > a.places) return 1;
    const int parts = a.places / (tiles * a.c.kv_heads);
    return parts < 1 ? 1 : parts < a.splits ? parts : a.splits;
}

template <int T, int DP, bool F32, int WAVES, bool FULL, bool SPLIT>
struct Prefill {
    static constexpr int kQParts = F32 ? Elem<T>::kExactParts : 1;
    static constexpr int kPParts = kQParts;
    static constexpr int kThreads = 64 * WAVES, kColumns = 32 * WAVES;
    static constexpr int kSteps = DP / 16, kBlocks = (DP + 31) / 32;
    static constexpr int kWords = kTile * DP / 8;         // 16-byte words of a tile's keys (and at most of its values)
    static constexpr int kLoads = (kWords + kThreads - 1) / kThreads;
    static constexpr int kAhead = 4;                      // words of the keys on their way from LDS
    static constexpr int kSchedMfma = 0x8, kSchedLds = 0x100;

    struct Lds {
        uint4 k[2][kLoads * kThreads];                    // [chunk][key]
        uint4 v[2][kWords + 32];                          // [eight keys][channel]; reads of channels past D run on
        int odd;                                          // an output is not finite
    };

    const PrefillArgs& a;
    Lds& lds;
    int tid, half, n, dim, ps, dim_magic;
    int kvh, b, len;
    int pos, low;                                         // of this column; keys up to low are behind its window
    int wave_first, wave_last, open_first, open_last;     // tiles that this wave sees, and those that all its columns see
    int group_first, group_last;                          // tiles that all columns of the work group see
    int sink_end;                                         // tiles with sinks end here
    int sink_tiles, first, n_tiles, part_first;           // (n_tiles from part_first on are this work group's)
    int parts;                                            // of every work group's keys
    const int32_t* table;
    const uint16_t *kbase, *vbase;
    int key_row;

    v4u stage_k[kLoads], stage_v[kLoads];

    static __device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
    __device__ __forceinline__ Prefill(const PrefillArgs& args, Lds& l) : a(args), lds(l) {}

    // Tiles are numbered by their first key / 64; the t-th that the work group looks at:
    __device__ __forceinline__ int tile_of(int t) const {
        if constexpr (SPLIT) t += part_first;
        return t < sink_tiles ? t : t - sink_tiles + first;
    }
    __device__ __forceinline__ int channels() const { return FULL ? DP : dim; }

    // Pages of a tile's four quarters (pages of 64 and more: all the same, and only p0 is kept).
    struct Pages {
        int p0, p1, p2, p3;
    };
    __device__ __forceinline__ int page_at(int key) const {
        const int at = key >> a.c.shift;
        return at < a.c.max_pages ? table[at] : -1;
    }
    __device__ __forceinline__ Pages ask_pages(int tile) const {
        const int key = tile * kTile;
        Pages p{page_at(key), 0, 0, 0};
        if (a.c.shift < 6) {
            p.p1 = page_at(key + 16);
            p.p2 = page_at(key + 32);
            p.p3 = page_at(key + 48);
        }
        return p;
    }
    // A bit for each quarter that has a page; where there is none, page 0 is read and nothing of it used.
    __device__ __forceinline__ uint32_t settle(Pages& p) const {
        const int p0 = uniform(p.p0);
        const bool a0 = page_ok(a.c, p0);
        p.p0 = a0 ? p0 : 0;
        if (a.c.shift >= 6) return a0 ? 15u : 0u;
        const int p1 = uniform(p.p1), p2 = uniform(p.p2), p3 = uniform(p.p3);
        const bool a1 = page_ok(a.c, p1), a2 = page_ok(a.c, p2), a3 = page_ok(a.c, p3);
        p.p1 = a1 ? p1 : 0;
        p.p2 = a2 ? p2 : 0;
        p.p3 = a3 ? p3 : 0;
        return (a0 ? 1u : 0u) | (a1 ? 2u : 0u) | (a2 ? 4u : 0u) | (a3 ? 8u : 0u);
    }
    static __device__ __forceinline__ int of_quarter(int quarter, int p0, int p1, int p2, int p3) {
        return quarter & 2 ? (quarter & 1 ? p3 : p2) : (quarter & 1 ? p1 : p0);
    }
    // Which eight keys of a tile word w of its values belongs to: w / dim.
    __device__ __forceinline__ int eight_of(int w) const {
        if constexpr (FULL) return w / DP;
        else return (w * dim_magic) >> 20;                // exact: w < 8 dim <= 2048
    }

    static __device__ __forceinline__ v4u load16(const void* base, uint32_t offset) {
        return *reinterpret_cast<const v4u*>(static_cast<const uint8_t*>(base) + offset);
    }
    // A tile's words on their way to registers: word tid + i threads of the keys (chunk-major: a wave reads 64 keys of a chunk)
    // and of the values.  In pages of 64 and more a tile is one run of either but for the keys' chunks, and a thread's place in
    // it never changes.
    // Words past the last chunk or channel are read again from the last one and not stored: a load that may or may not
    // be on its way would make every wait one for all of them (heads of 96 with 8 waves: 142 us against 102).
    static constexpr bool kEven = FULL && kWords % kThreads == 0;
    __device__ __forceinline__ int chunk_of(int i) const { return uniform(tid / kTile) + i * WAVES; }
    __device__ __forceinline__ int held_chunk(int i) const {
        const int chunk = chunk_of(i);
        return kEven || chunk < a.c.chunks ? chunk : a.c.chunks - 1;
    }
    __device__ __forceinline__ int held_word(int i) const {
        const int w = tid + i * kThreads, last = (kTile / 8) * channels() - 1;
        return kEven || w < last ? w : last;
    }
    __device__ __forceinline__ void load_keys(int tile, const Pages p) {
        const KvCache& c = a.c;
        const int key = tile * kTile, at = tid & 63;
        if (c.shift >= 6) {
            const uint16_t* kp = kbase + (int64_t)p.p0 * c.k_page + (key & (ps - 1)) * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage_k[i] = load16(kp + held_chunk(i) * ps * 8, (uint32_t)at * 16);
        } else {
            const uint16_t* kp = kbase + (int64_t)of_quarter(at >> 4, p.p0, p.p1, p.p2, p.p3) * c.k_page + ((key + at) & (ps - 1)) * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage_k[i] = load16(kp + held_chunk(i) * ps * 8, 0);
        }
    }
    __device__ __forceinline__ void load_values(int tile, const Pages p) {
        const KvCache& c = a.c;
        const int key = tile * kTile;
        if (c.shift >= 6) {
            const uint16_t* vp = vbase + (int64_t)p.p0 * c.v_page + (key & (ps - 1)) * channels();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if constexpr (kEven) stage_v[i] = load16(vp + i * kThreads * 8, (uint32_t)tid * 16);
                else stage_v[i] = load16(vp, (uint32_t)held_word(i) * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int w = held_word(i), eight = eight_of(w), d = w - eight * channels();
                const int page = of_quarter((eight >> 1) & 3, p.p0, p.p1, p.p2, p.p3);
                stage_v[i] = load16(vbase + (int64_t)page * c.v_page + ((key + 8 * eight) & (ps - 1)) * channels(), (uint32_t)d * 16);
            }
        }
    }
    // Into LDS.  Values of keys that the cache does not hold become zeros: whatever lies there must not meet a weight of 0 in
    // the product.
    __device__ __forceinline__ void store_keys(int buf) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (kEven || chunk_of(i) < a.c.chunks) lds.k[buf][tid + i * kThreads] = __builtin_bit_cast(uint4, stage_k[i]);
    }
    __device__ __forceinline__ void store_values(int buf, int tile, uint32_t there) {
        if (there != 15 || tile < group_first || tile > group_last) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int eight = eight_of(held_word(i));
                int held = len - (tile * kTile + 8 * eight);
                held = (there >> ((eight >> 1) & 3)) & 1 ? held : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) stage_v[i][e] &= (held > 2 * e ? 0x0000FFFFu : 0u) | (held > 2 * e + 1 ? 0xFFFF0000u : 0u);
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int w = tid + i * kThreads;
            if (kEven || w < (kTile / 8) * channels()) lds.v[buf][w] = __builtin_bit_cast(uint4, stage_v[i]);
        }
    }

    // Does this wave see anything of the tile?  And every column all of it?
    __device__ __forceinline__ bool sees(int tile) const {
        return (tile >= wave_first || tile < sink_end) && tile <= wave_last;
    }
    __device__ __forceinline__ bool sees_all(int tile, uint32_t there) const {
        return there == 15 && tile >= open_first && tile <= open_last;
    }
    // Which of the eight keys from `base` on this column sees, a bit each.
    static __device__ __forceinline__ uint32_t first_bits(int n) { return (1u << (n < 0 ? 0 : n > 8 ? 8 : n)) - 1u; }
    __device__ __forceinline__ uint32_t visible(int base, int p, int low, uint32_t there, int quarter) const {
        const uint32_t seen = first_bits(p + 1 - base) & (~first_bits(low + 1 - base) | first_bits(a.n_sink - base));
        return (there >> quarter) & 1 ? seen : 0u;
    }

    // Scores of 64 keys: s[block][i] is key 32 block + 16 (i / 8) + 8 half + i % 8 against this lane's column.
    __device__ __forceinline__ void scores(int buf, const v4u (&qf)[kQParts][kSteps], v16f (&s)[2]) const {
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[blk][i] = 0.0f;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const v4u kf = __builtin_bit_cast(v4u, lds.k[buf][(2 * st + half) * kTile + 32 * blk + key_row]);
#pragma unroll
                for (int p = 0; p < kQParts; ++p) s[blk] = Elem<T>::mfma32(kf, qf[p][st], s[blk]);
            }
        }
    }
    // The order of the scores' instructions: kAhead words of the keys on their way (by itself the compiler keeps two).
    static __device__ __forceinline__ void order_scores() {
        __builtin_amdgcn_sched_group_barrier(kSchedLds, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, kQParts, 0);
            if (i < 2 * kSteps - kAhead) __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
        }
    }

    __device__ __forceinline__ void mask(int key, uint32_t there, v16f (&s)[2]) const {
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter) {
            const int seen = (int)visible(key + 16 * quarter + 8 * half, pos, low, there, quarter);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int keep = (seen << (31 - e)) >> 31, i = 8 * (quarter & 1) + e;
                const float x = s[quarter >> 1][i];
                s[quarter >> 1][i] = __int_as_float((__float_as_int(x) & keep) | (__float_as_int(kNegInf) & ~keep));
            }
        }
    }

    // The reference m of the weights (of the scaled scores) and the running sum; s becomes the weights exp2(s - m).  m moves
    // only where the maximum has grown by more than kSlack: what is there then needs no factor in most tiles, and a weight of
    // up to 2^kSlack loses nothing.  Returns the factor.
    static constexpr float kSlack = 8.0f;
    static constexpr float kLiftLow = T == kF16 ? 6.0f : 0.0f;   // 2^(kSlack + lift) stays in the type's range
    __device__ __forceinline__ float softmax(v16f (&s)[2], float gain, float& m, float& l) const {
        float top = kNegInf;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, s[blk][i]), s[blk][i + 1]);
        top = max_xor32(top) * gain;
        float alpha = 1.0f;
        if (__any(top > m + kSlack)) {
            const float m_new = top > m + kSlack ? top : m;
            alpha = m_new == m ? 1.0f : exp2_fast(m - m_new);
            m = m_new;
            l *= alpha;
        }
        const float base = kLiftLow - (m == kNegInf ? 0.0f : m);
        float sum = 0.0f;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[blk][i] = exp2_fast(__builtin_fmaf(s[blk][i], gain, base));
                if constexpr (kPParts > 1) sum += s[blk][i];
            }
        if constexpr (kPParts > 1) l += sum;
        return alpha;
    }

    // Operands of the second product: the weights of 16 keys (quarter) in parts.  Rounded weights are summed as rounded: the
    // sum then belongs to the product it divides, and takes half the instructions.
    __device__ __forceinline__ void weights(const v16f (&s)[2], int quarter, v4u (&pf)[kPParts], float& l) const {
        const int blk = quarter >> 1, i0 = 8 * (quarter & 1);
        if constexpr (kPParts == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pf[0][e] = Elem<T>::pack(s[blk][i0 + 2 * e], s[blk][i0 + 2 * e + 1]);
                l = Elem<T>::add2(pf[0][e], l);
            }
        } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[blk][i0 + e];
#pragma unroll
            for (int p = 0; p < kPParts; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) pf[p][e] = Elem<T>::part(x[2 * e], x[2 * e + 1]);
        }
    }

    // The first tile's words on their way, and the pages of the second asked for.
    __device__ __forceinline__ void begin(Pages& pages, uint32_t& there) {
        if (n_tiles <= 0) return;
        there = settle(pages);
        load_keys(tile_of(0), pages);
        load_values(tile_of(0), pages);
        if (n_tiles > 1) pages = ask_pages(tile_of(1));
    }

    // Scores, softmax and product of every tile, the next tile's words on their way.  pages: of the tile after the one being
    // loaded; there: quarters of the latter that have one.
    __device__ __forceinline__ void all_tiles(Pages pages, uint32_t there, const v4u (&qf)[kQParts][kSteps], float gain, float& m,
                                              float& l, v16f (&o)[kBlocks]) {
        __syncthreads();
        if (n_tiles > 0) {
            store_keys(0);
            store_values(0, tile_of(0), there);
        }
        __syncthreads();
        for (int t = 0; t < n_tiles; ++t) {
            const int tile = tile_of(t), buf = t & 1;
            const uint32_t now = there;
            if (t + 1 < n_tiles) {
                there = settle(pages);
                load_keys(tile_of(t + 1), pages);
                load_values(tile_of(t + 1), pages);
                if (t + 2 < n_tiles) pages = ask_pages(tile_of(t + 2));
            }
            if (sees(tile)) {
                v16f s[2];
                scores(buf, qf, s);
                order_scores();
                if (!sees_all(tile, now)) mask(tile * kTile, now, s);
                const float alpha = softmax(s, gain, m, l);
                if (__any(alpha != 1.0f)) {
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d) o[d] *= alpha;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v4u pf[kPParts];
                    weights(s, q, pf, l);
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d) {
                        const v4u vf = __builtin_bit_cast(v4u, lds.v[buf][(2 * q + half) * channels() + 32 * d + n]);
#pragma unroll
                        for (int p = 0; p < kPParts; ++p) o[d] = Elem<T>::mfma32(vf, pf[p], o[d]);
                    }
                }
            }
            if (t + 1 < n_tiles) {
                store_keys(buf ^ 1);
                store_values(buf ^ 1, tile_of(t + 1), there);
            }
            __syncthreads();
        }
    }

    // Scores of infinite keys, whose products with parts of q that are 0 are no numbers: of 32 keys, the finite channels' products,
    // and where there are others an infinity if all of those meet a q of their sign, or all one of the other sign, else NaN.
    __device__ __forceinline__ void careful_scores(const v4u (&qf)[kQParts][kSteps], v16f (&s)[2]) const {
        constexpr uint32_t one = T == kBf16 ? 0x3F803F80u : 0x3C003C00u;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            v16f sum, signs, count;                       // of the finite; of the infinite, by sign; how many are not finite
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = signs[i] = count[i] = 0.0f;
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                const v4u ones = {one, one, one, one};
                v4u kf = __builtin_bit_cast(v4u, lds.k[0][(2 * st + half) * kTile + 32 * blk + key_row]), inf, odd, sq;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bad = not_finite<T>(kf[e]);
                    inf[e] = sign_of_infinite<T>(kf[e]);
                    odd[e] = bad & one;
                    kf[e] &= ~bad;
                    sq[e] = sign_of<T>(qf[0][st][e]);     // (a value's first part has its sign, and is 0 where the value is next to none)
                }
                signs = Elem<T>::mfma32(inf, sq, signs);
                count = Elem<T>::mfma32(odd, ones, count);
#pragma unroll
                for (int p = 0; p < kQParts; ++p) sum = Elem<T>::mfma32(kf, qf[p][st], sum);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[blk][i] = count[i] == 0.0f         ? sum[i]
                            : signs[i] == count[i]  ? -kNegInf
                            : signs[i] == -count[i] ? kNegInf
                                                    : __builtin_nanf("");
        }
    }

    // All tiles once more, twice for every block of 32 channels: first the values that are not finite, counted as the marks of
    // each kind that a column sees (see mark_half), then the product without them.
    __device__ __forceinline__ void careful(const v4u (&qf)[kQParts][kSteps], float gain, bool used, int64_t row) {
        constexpr uint32_t one = T == kBf16 ? 0x3F80u : 0x3C00u;
        for (int d = 0; 32 * d < channels(); ++d) {
            float m = kNegInf, l = 0.0f;
            v16f o, odd;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = odd[i] = 0.0f;
            for (int turn = 0; turn < 2 * n_tiles; ++turn) {
                const int t = turn < n_tiles ? turn : turn - n_tiles, tile = tile_of(t), key = tile * kTile;
                __syncthreads();
                Pages p = ask_pages(tile);
                const uint32_t there = settle(p);
                load_keys(tile, p);
                load_values(tile, p);
                store_keys(0);
                store_values(0, tile, there);
                __syncthreads();
                if (!sees(tile)) continue;
                if (turn < n_tiles) {
                    v16f marks;
#pragma unroll
                    for (int i = 0; i < 16; ++i) marks[i] = 0.0f;
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t bits = visible(key + 16 * q + 8 * half, pos, low, there, q);
                        const v4u vf = __builtin_bit_cast(v4u, lds.v[0][(2 * q + half) * channels() + 32 * d + n]);
                        v4u mark, seen;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            mark[e] = mark_half<T>(vf[e] & 0xFFFFu) | mark_half<T>(vf[e] >> 16) << 16;
                            seen[e] = ((bits >> (2 * e)) & 1 ? one : 0u) | ((bits >> (2 * e)) & 2 ? one << 16 : 0u);
                        }
                        marks = Elem<T>::mfma32(mark, seen, marks);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) odd[i] += unmark(marks[i]);
                } else {
                    v16f s[2];
                    if constexpr (kQParts > 1) careful_scores(qf, s);
                    else scores(0, qf, s);
                    if (!sees_all(tile, there)) mask(key, there, s);
                    o *= softmax(s, gain, m, l);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        v4u pf[kPParts];
                        weights(s, q, pf, l);
                        v4u vf = __builtin_bit_cast(v4u, lds.v[0][(2 * q + half) * channels() + 32 * d + n]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) vf[e] &= ~not_finite<T>(vf[e]);
#pragma unroll
                        for (int p = 0; p < kPParts; ++p) o = Elem<T>::mfma32(vf, pf[p], o);
                        __builtin_amdgcn_sched_barrier(0);   // one quarter's registers at a time
                    }
                }
            }
            l = sum_xor32(l);
            if (used) store_block(d, o, odd, m, l, row);
        }
    }

    // Channels 32 d .. of this lane's column: divided by the sum, or, where the keys are split, as they are, with m and l.
    __device__ __forceinline__ void store_block(int d, const v16f& o, const v16f& more, float m, float l, int64_t row) const {
        if (SPLIT && parts > 1) {
            const int held = held_parts(a.splits), z = blockIdx.y;
            float* part = a.ws + row * row_floats(a.splits, dim);
            if (d == 0 && half == 0) {
                part[z] = m;
                part[held + z] = l;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 32 * d + 8 * i + 4 * half;
                if (FULL || at < dim)
                    *reinterpret_cast<v4f*>(part + 2 * held + z * dim + at) =
                        v4f{o[4 * i] + more[4 * i], o[4 * i + 1] + more[4 * i + 1], o[4 * i + 2] + more[4 * i + 2], o[4 * i + 3] + more[4 * i + 3]};
            }
            return;
        }
        const float inv = l == 0.0f ? 1.0f : 1.0f / l;    // no weight, nothing visible: o is 0
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 32 * d + 8 * i + 4 * half;
            if (FULL || at < dim)
                store4<T, F32>(a.out, row * dim + at, o[4 * i] * inv + more[4 * i], o[4 * i + 1] * inv + more[4 * i + 1],
                               o[4 * i + 2] * inv + more[4 * i + 2], o[4 * i + 3] * inv + more[4 * i + 3]);
        }
    }

    __device__ __forceinline__ void run() {
        const KvCache& c = a.c;
        tid = threadIdx.x;
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        half = lane >> 5;
        n = lane & 31;
        dim = c.dim;
        ps = 1 << c.shift;
        dim_magic = ((1 << 20) + dim - 1) / dim;
        // key of a row of a 32-key block: the order in which a lane's 16 scores are its operand words of the second product
        key_row = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);

        // work groups of one kv head follow each other at a distance of kv_heads (with 8 of them: on one XCD, whose L2 keeps
        // the head's keys), the last tiles, which have the most keys before them, first
        kvh = blockIdx.x % c.kv_heads;
        const int id = a.tiles - 1 - (int)(blockIdx.x / c.kv_heads);
        b = find_last(c.n_seqs, id, [&](int i) { return first_tile(a.q_start, i, a.n_tokens, a.group, kColumns); });
        b = uniform(b);
        Span span = span_of(a.q_start, b, a.n_tokens);
        span = {uniform(span.first), uniform(span.count)};
        const int col0 = (id - uniform(first_tile(a.q_start, b, a.n_tokens, a.group, kColumns))) * kColumns;
        const int columns = span.count * a.group;
        if (col0 < 0 || col0 >= columns) return;          // below 0: before the first sequence's tokens, or offsets that decrease
        if constexpr (SPLIT) {
            parts = parts_of(a, kColumns);
            if ((int)blockIdx.y >= parts) return;
        }
        len = uniform(seq_len(c, b));
        const int p0 = len - span.count;                  // position of the first token (below 0: it sees nothing)
        table = c.table + (int64_t)b * c.max_pages;
        kbase = c.k + (int64_t)kvh * c.chunks * ps * 8;
        vbase = c.v + (int64_t)kvh * dim * ps;

        const int col = col0 + wave * 32 + n;
        const bool used = col < columns;
        const int token = (used ? col : columns - 1) / a.group, in_group = (used ? col : columns - 1) - token * a.group;
        pos = p0 + token;
        low = a.window > 0 ? pos - a.window : -1;
        const int64_t row = (int64_t)(span.first + token) * a.heads + kvh * a.group + in_group;   // of q and out

        // The tiles of the work group: those of the sinks, then from the window's first to the last position's.  Positions of
        // its and of this wave's columns (an unused wave sees nothing):
        const int last_col = (col0 + kColumns < columns ? col0 + kColumns : columns) - 1;
        const int pos_lo = p0 + col0 / a.group, pos_hi = p0 + last_col / a.group;
        const int wcol0 = col0 + wave * 32, wcol1 = wcol0 + 31 < columns ? wcol0 + 31 : columns - 1;
        const int wpos_lo = p0 + wcol0 / a.group, wpos_hi = wcol0 < columns ? p0 + wcol1 / a.group : -1;
        auto behind = [&](int p) { return a.window > 0 && p >= a.window ? p - a.window + 1 : 0; };   // first key in the window
        const int lo = behind(pos_lo), sinks = a.n_sink < lo ? a.n_sink : lo;
        first = lo / kTile;
        sink_tiles = (sinks + kTile - 1) / kTile;
        sink_tiles = sink_tiles < first ? sink_tiles : first;
        n_tiles = pos_hi < 0 ? 0 : sink_tiles + pos_hi / kTile + 1 - first;
        sink_end = (a.n_sink + kTile - 1) / kTile;
        if constexpr (SPLIT) {                            // (a row has up to 2^18 tiles, a call 32 parts)
            part_first = n_tiles * (int)blockIdx.y / parts;
            n_tiles = n_tiles * ((int)blockIdx.y + 1) / parts - part_first;
        }
        wave_first = uniform(behind(wpos_lo) / kTile);
        wave_last = uniform(wpos_hi < 0 ? -1 : wpos_hi / kTile);
        open_first = uniform((behind(wpos_hi) + kTile - 1) / kTile);
        open_last = uniform((wpos_lo + 1) / kTile - 1);
        group_first = (behind(pos_hi) + kTile - 1) / kTile;
        group_last = (pos_lo + 1) / kTile - 1;

        if (tid == 0) lds.odd = 0;
        if constexpr (!FULL) {                            // chunks past D: q has zeros there, and 0 times them has to be 0
            for (int w = c.chunks * kTile + tid; w < DP / 8 * kTile; w += kThreads) lds.k[0][w] = lds.k[1][w] = make_uint4(0, 0, 0, 0);
        }
        // A work group starts with three loads that follow each other (pages, then keys and values); q comes beside them.
        Pages pages{};
        uint32_t there = 0;
        if (n_tiles > 0) pages = ask_pages(tile_of(0));
        float4 x[kSteps][2];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 8 * (2 * s + half);
            x[s][0] = x[s][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (FULL || d < dim) x[s][0] = load4<T, F32>(a.q, row * dim + d);
            if (FULL || d + 4 < dim) x[s][1] = load4<T, F32>(a.q, row * dim + d + 4);
        }
        if constexpr (kQParts < 3) begin(pages, there);
        // q as operands: chunk 2 s + half of this lane's column, in parts.  The factor of the scores is positive (a negative
        // scale changes q's sign, a scale of 0 makes q 0), so that it can be applied after the maximum.
        v4u qf[kQParts][kSteps];
        float gain = fabsf(a.scale2), up = a.scale2 < 0.0f ? -1.0f : a.scale2 == 0.0f ? 0.0f : 1.0f;
        if constexpr (F32 && T == kF16) {
            float top = 0.0f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    top = fmaxf(top, fmaxf(fmaxf(fabsf(x[s][i].x), fabsf(x[s][i].y)), fmaxf(fabsf(x[s][i].z), fabsf(x[s][i].w))));
            const float g = row_gain(max_xor32(top));
            up *= g;
            gain /= g;
        }
        if (a.scale2 == 0.0f) gain = 1.0f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            float4 u = x[s][0], w = x[s][1];
            u.x *= up; u.y *= up; u.z *= up; u.w *= up;
            w.x *= up; w.y *= up; w.z *= up; w.w *= up;
#pragma unroll
            for (int p = 0; p < kQParts; ++p) {
                if constexpr (kQParts == 1)
                    qf[p][s] = v4u{Elem<T>::pack(u.x, u.y), Elem<T>::pack(u.z, u.w), Elem<T>::pack(w.x, w.y), Elem<T>::pack(w.z, w.w)};
                else
                    qf[p][s] = v4u{Elem<T>::part(u.x, u.y), Elem<T>::part(u.z, u.w), Elem<T>::part(w.x, w.y), Elem<T>::part(w.z, w.w)};
            }
        }

        if constexpr (kQParts == 3) begin(pages, there);
        float m = kNegInf, l = 0.0f;
        v16f o[kBlocks];
#pragma unroll
        for (int t = 0; t < kBlocks; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;

        all_tiles(pages, there, qf, gain, m, l, o);
        l = sum_xor32(l);
        float odd = 0.0f;                                 // of channels past D nothing is known
#pragma unroll
        for (int t = 0; t < kBlocks; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (FULL || 32 * t + 8 * (i >> 2) + 4 * half < dim) odd += o[t][i] * 0.0f;
        // A score that is no number makes all of its row so, and there is nothing to be careful about, unless an infinite key met a
        // part of q that is 0 (one part: the score is what it has to be).
        if (used && odd != 0.0f && (kQParts > 1 || l == l)) lds.odd = 1;
        __syncthreads();
        if (__builtin_expect(uniform(lds.odd), 0)) {
            careful(qf, gain, used, row);
            return;
        }
        if (!used) return;
        v16f none;
#pragma unroll
        for (int i = 0; i < 16; ++i) none[i] = 0.0f;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) store_block(d, o[d], none, m, l, row);
    }
};

template <int T, int DP, bool F32, int WAVES, int PER_SIMD, bool FULL, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, PER_SIMD) void attn_prefill_kernel(PrefillArgs a) {
    using P = Prefill<T, DP, F32, WAVES, FULL, SPLIT>;
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
