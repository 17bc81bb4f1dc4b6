// The work group of the prompt kernels: 32 columns (a query row under a head) for each wave, tiles of 64 keys through
// double-buffered LDS, both products on 32x32x16 instructions.  Used by the attention of prompts (run) and by the decode over
// shared prefixes of many columns (run_prefix); what it computes and why it is laid out so stands at the former.
#pragma once

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

// How the keys of a work group's columns are gone through: all of them, in parts that are joined, or as runs of a shared prefix
// whose results go to records.
constexpr int kWhole = 0, kSplit = 1, kPrefix = 2;

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

template <int T, int DP, bool F32, int WAVES, bool FULL, int MODE>
struct Prefill {
    static constexpr bool SPLIT = MODE != kWhole;
    static constexpr int kQParts = F32 ? Elem<T>::kExactParts : 1;
    // Weights in as many parts as q; over a shared prefix in two at least, as the decode's are (a sequence's result must not be less
    // exact for its neighbours).
    static constexpr int kPParts = MODE == kPrefix && !F32 ? 2 : kQParts;
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
    float* record;                                        // of this column: [maximum, sum, -, -, output] (prefix)

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

    // The same of words in stages of the caller's.  Bodies of their own: with the prompts' loop going through these, 4096 tokens took
    // 173 us where they take 154.
    using Stage = v4u[kLoads];
    __device__ __forceinline__ void load_keys(int tile, const Pages p, Stage& stage) const {
        const KvCache& c = a.c;
        const int key = tile * kTile, at = tid & 63;
        if (c.shift >= 6) {
            const uint16_t* kp = kbase + (int64_t)p.p0 * c.k_page + (key & (ps - 1)) * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage[i] = load16(kp + held_chunk(i) * ps * 8, (uint32_t)at * 16);
        } else {
            const uint16_t* kp = kbase + (int64_t)of_quarter(at >> 4, p.p0, p.p1, p.p2, p.p3) * c.k_page + ((key + at) & (ps - 1)) * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) stage[i] = load16(kp + held_chunk(i) * ps * 8, 0);
        }
    }
    __device__ __forceinline__ void load_values(int tile, const Pages p, Stage& stage) const {
        const KvCache& c = a.c;
        const int key = tile * kTile;
        if (c.shift >= 6) {
            const uint16_t* vp = vbase + (int64_t)p.p0 * c.v_page + (key & (ps - 1)) * channels();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if constexpr (kEven) stage[i] = load16(vp + i * kThreads * 8, (uint32_t)tid * 16);
                else stage[i] = load16(vp, (uint32_t)held_word(i) * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int w = held_word(i), eight = eight_of(w), d = w - eight * channels();
                const int page = of_quarter((eight >> 1) & 3, p.p0, p.p1, p.p2, p.p3);
                stage[i] = load16(vbase + (int64_t)page * c.v_page + ((key + 8 * eight) & (ps - 1)) * channels(), (uint32_t)d * 16);
            }
        }
    }
    __device__ __forceinline__ void store_keys(int buf, const Stage& stage) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (kEven || chunk_of(i) < a.c.chunks) lds.k[buf][tid + i * kThreads] = __builtin_bit_cast(uint4, stage[i]);
    }
    __device__ __forceinline__ void store_values(int buf, int tile, uint32_t there, Stage& stage) {
        if (there != 15 || tile < group_first || tile > group_last) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int eight = eight_of(held_word(i));
                int held = len - (tile * kTile + 8 * eight);
                held = (there >> ((eight >> 1) & 3)) & 1 ? held : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) stage[i][e] &= (held > 2 * e ? 0x0000FFFFu : 0u) | (held > 2 * e + 1 ? 0xFFFF0000u : 0u);
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int w = tid + i * kThreads;
            if (kEven || w < (kTile / 8) * channels()) lds.v[buf][w] = __builtin_bit_cast(uint4, stage[i]);
        }
    }

    // Scores, softmax and product of one tile in LDS.
    __device__ __forceinline__ void one_tile(int tile, int buf, uint32_t now, const v4u (&qf)[kQParts][kSteps], float gain, float& m, float& l,
                                             v16f (&o)[kBlocks]) const {
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
    }

    // As all_tiles, with the words of two tiles on their way: a prefix's keys come from memory, where those of a prompt are in the caches
    // that its other work groups fill.  Page numbers are asked for 64 tiles at a time, one a lane, so that nothing waits for them
    // in between; past the last tile that one is loaded again (a load that may or may not be on its way would make every wait one
    // for all).
    __device__ __forceinline__ void prefix_tiles(const v4u (&qf)[kQParts][kSteps], float gain, float& m, float& l, v16f (&o)[kBlocks]) {
        if (n_tiles <= 0) return;
        const int lane = tid & 63;
        Pages held{};
        auto hold = [&](int from) { held = ask_pages(tile_of(min(from + lane, n_tiles - 1))); };
        auto pages_of = [&](int t, uint32_t& there) {
            const int at = t & 63;
            Pages p{__builtin_amdgcn_readlane(held.p0, at), 0, 0, 0};
            if (a.c.shift < 6) {
                p.p1 = __builtin_amdgcn_readlane(held.p1, at);
                p.p2 = __builtin_amdgcn_readlane(held.p2, at);
                p.p3 = __builtin_amdgcn_readlane(held.p3, at);
            }
            there = settle(p);
            return p;
        };
        Stage ka, va, kb, vb;
        uint32_t there_now, there_a, there_b;
        hold(0);
        const int second = min(1, n_tiles - 1);
        {
            const Pages p = pages_of(0, there_now), p1 = pages_of(second, there_a);
            load_keys(tile_of(0), p, ka);
            load_values(tile_of(0), p, va);
            load_keys(tile_of(second), p1, kb);
            load_values(tile_of(second), p1, vb);
        }
        __syncthreads();
        store_keys(0, ka);
        store_values(0, tile_of(0), there_now, va);
        __syncthreads();
        // the next tile's words in (k, v), and the one's after it asked for in (k2, v2)
        auto step = [&](int t, Stage& k, Stage& v, uint32_t& there, Stage& k2, Stage& v2, uint32_t& there2) {
            const int next = min(t + 1, n_tiles - 1), after = min(t + 2, n_tiles - 1);
            if ((after & 63) == 0 && after == t + 2) hold(after);
            const Pages p = pages_of(after, there2);
            load_keys(tile_of(after), p, k2);
            load_values(tile_of(after), p, v2);
            one_tile(tile_of(t), t & 1, there_now, qf, gain, m, l, o);
            store_keys((t + 1) & 1, k);
            store_values((t + 1) & 1, tile_of(next), there, v);
            there_now = there;
            __syncthreads();
        };
        for (int t = 0; t < n_tiles; t += 2) {
            step(t, kb, vb, there_a, ka, va, there_b);
            if (t + 1 < n_tiles) step(t + 1, ka, va, there_b, kb, vb, there_a);
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
        if constexpr (MODE == kPrefix) {
            if (d == 0 && half == 0) {
                record[0] = m + (kLift<T> - kLiftLow);    // the reference of weights that are lifted as the decode's are
                record[1] = l;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 32 * d + 8 * i + 4 * half;
                if (FULL || at < dim)
                    *reinterpret_cast<v4f*>(record + 4 + at) =
                        v4f{o[4 * i] + more[4 * i], o[4 * i + 1] + more[4 * i + 1], o[4 * i + 2] + more[4 * i + 2], o[4 * i + 3] + more[4 * i + 3]};
            }
            return;
        }
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

        go(row, used);
    }

    // Tiles [u0, u1) of a shared prefix of `prefix` keys in the pages of table row `table_row` for this wave's columns: each sees keys
    // up to `last`, those up to `behind` only among the sinks (below 0: all of them), and is row `q_row` of q.  first_tile and
    // before: the window's first tile and the sinks' tiles before it.
    __device__ __forceinline__ void run_prefix(int table_row, int head, int prefix, int last, int behind, int first_tile, int before,
                                               int u0, int u1, bool used, int64_t q_row, float* to) {
        const KvCache& c = a.c;
        tid = threadIdx.x;
        const int lane = tid & 63;
        half = lane >> 5;
        n = lane & 31;
        dim = c.dim;
        ps = 1 << c.shift;
        dim_magic = ((1 << 20) + dim - 1) / dim;
        // key of a row of a 32-key block: the order in which a lane's 16 scores are its operand words of the second product
        key_row = (n & 16) | ((n & 4) << 1) | ((n & 8) >> 1) | (n & 3);
        kvh = head;
        len = prefix;
        table = c.table + (int64_t)table_row * c.max_pages;
        kbase = c.k + (int64_t)kvh * c.chunks * ps * 8;
        vbase = c.v + (int64_t)kvh * dim * ps;
        record = to;
        pos = last;
        low = behind;
        first = first_tile;
        sink_tiles = before;
        part_first = u0;
        n_tiles = u1 - u0;
        sink_end = (a.n_sink + kTile - 1) / kTile;
        int pos_lo = pos, pos_hi = pos, low_lo = low, low_hi = low;
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            pos_lo = min(pos_lo, __shfl_xor(pos_lo, i));
            pos_hi = max(pos_hi, __shfl_xor(pos_hi, i));
            low_lo = min(low_lo, __shfl_xor(low_lo, i));
            low_hi = max(low_hi, __shfl_xor(low_hi, i));
        }
        const bool any = __any(used) != 0;                // a wave without columns sees nothing
        wave_first = uniform((low_lo + 1) / kTile);
        wave_last = uniform(any && pos_hi >= 0 ? pos_hi / kTile : -1);
        open_first = uniform((low_hi + kTile) / kTile);
        open_last = uniform((pos_lo + 1) / kTile - 1);
        group_first = 0;                                  // of tiles that the prefix fills nothing is put to zero
        group_last = prefix / kTile - 1;
        go(q_row, used);
    }

    // The columns' products over all tiles, and their results.
    __device__ __forceinline__ void go(int64_t row, bool used) {
        const KvCache& c = a.c;
        if (tid == 0) lds.odd = 0;
        if constexpr (!FULL) {                            // chunks past D: q has zeros there, and 0 times them has to be 0
            for (int w = c.chunks * kTile + tid; w < DP / 8 * kTile; w += kThreads) lds.k[0][w] = lds.k[1][w] = make_uint4(0, 0, 0, 0);
        }
        // A work group starts with three loads that follow each other (pages, then keys and values); q comes beside them.
        Pages pages{};
        uint32_t there = 0;
        if (MODE != kPrefix && n_tiles > 0) pages = ask_pages(tile_of(0));
        float4 x[kSteps][2];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 8 * (2 * s + half);
            x[s][0] = x[s][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (FULL || d < dim) x[s][0] = load4<T, F32>(a.q, row * dim + d);
            if (FULL || d + 4 < dim) x[s][1] = load4<T, F32>(a.q, row * dim + d + 4);
        }
        if constexpr (kQParts < 3 && MODE != kPrefix) begin(pages, there);
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

        if constexpr (kQParts == 3 && MODE != kPrefix) begin(pages, there);
        float m = kNegInf, l = 0.0f;
        v16f o[kBlocks];
#pragma unroll
        for (int t = 0; t < kBlocks; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;

        if constexpr (MODE == kPrefix) prefix_tiles(qf, gain, m, l, o);
        else all_tiles(pages, there, qf, gain, m, l, o);
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

}  // namespace
}  // namespace bitnet
