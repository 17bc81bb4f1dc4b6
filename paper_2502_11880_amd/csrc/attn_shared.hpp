// Decode over shared prefixes: the rows of a launch, where their results go, and how the parts of a call find them.
#pragma once

#include "kv_cache.hpp"

namespace bitnet {

constexpr int kSharedSeqs = 1024;    // sequences of a launch (more go in several)
constexpr int kSharedGroups = 512;   // work groups of a launch
constexpr uint16_t kNobody = 0xFFFF;
// A prefix is gone through in registers, up to 64 columns (query heads of a kv head, of all sequences of the group) a pass, or
// in shared memory, 128 or 256 a pass, in a launch of its own.
constexpr int kNarrowColumns = 64;   // up to so many: always the former
// Columns of a wide pass: four waves' or eight waves' (q in one part leaves registers for two waves a SIMD).
constexpr int wide_columns(int dim, bool f32) { return !f32 && dim > 64 && dim <= 128 ? 256 : 128; }
// What decides past that: picoseconds a key and kv head of a pass of either, and the microseconds that the second launch costs by
// itself, fitted to 576 pairs of calls that were sent either way (heads of 32 to 256; 80, 128, 256 and 512 columns; 1, 8 and 32 kv
// heads; 1024, 6016 and 32768 keys).  Past heads of 64 the slower side was taken 4% too slow at the worst, up to them 14% (one kv
// head or 32 have not the costs of 8).  us, in registers / in shared memory, 8 kv heads, behind 1024, 6016 and 32768 keys:
//   heads of 64, bf16: 80 columns 22 / 33, 31 / 34, 55 / 50; 256 columns 32 / 35, 44 / 41, 94 / 68, from 32 bits 35 / 37, 48 / 46, 96 / 83;
//   heads of 128, bf16: 80 columns 27 / 38, 38 / 41, 79 / 69; 256 columns 32 / 49, 58 / 56, 182 / 90; 512 columns 44 / 61, 90 / 73, 351 / 147,
//     from 32 bits 46 / 63, 92 / 91, 347 / 251, from 32 bits over f16 45 / 59, 92 / 80, 350 / 198;
//   heads of 256, bf16: 80 columns 49 / 65, 66 / 76, 178 / 150; 512 columns 98 / 111, 207 / 166, 930 / 437, from 32 bits 110 / 144, 216 / 248,
//     894 / 773, from 32 bits over f16 103 / 128, 209 / 215, 912 / 642.
struct WideRule {
    int narrow, wide, start;
};
constexpr WideRule wide_rule(int dim, bool f32, bool three_parts) {
    // Heads between 128 and 256 never: their words past D and the masks take the registers (185 to 318 spilled).  128 columns behind 32768
    // keys, 8 kv heads, in registers / in shared memory: heads of 132 191 / 322, of 192 203 / 363, of 192 from 32 bits 213 / 417; 512 columns
    // 732 / 1111, 786 / 1205 and 810 / 1405.
    if (dim > 128 && dim < 256) return WideRule{0, 0, 0};
    if (dim <= 64) return three_parts ? WideRule{66, 86, 4} : f32 ? WideRule{66, 68, 4} : WideRule{66, 60, 3};
    if (dim <= 128) return three_parts ? WideRule{67, 166, 20} : f32 ? WideRule{67, 143, 12} : WideRule{58, 83, 13};
    return three_parts ? WideRule{230, 792, 50} : f32 ? WideRule{230, 704, 50} : WideRule{230, 410, 40};
}
__host__ __device__ __forceinline__ bool worth_wide(const WideRule& r, int64_t columns, int narrow_columns, int wide_columns, int64_t keys,
                                                    int kv_heads) {
    if (columns <= kNarrowColumns) return false;
    const int64_t narrow = (columns + narrow_columns - 1) / narrow_columns * r.narrow, wide = (columns + wide_columns - 1) / wide_columns * r.wide;
    return keys * kv_heads * (narrow - wide) > (int64_t)r.start * 1000000;
}
// Whether it could be for some group of up to `columns` columns behind up to `keys`: the difference grows with the columns but for where a
// wide pass begins.  What the launch for wide prefixes goes by, and the workspace (for any type of q).  (keys: of a row of the table)
bool attn_shared_may_be_wide(int64_t columns, int64_t keys, int kv_heads, int dim, bool f32, bool three_parts);
constexpr int kWideTile = 64;        // keys
constexpr int kWideCost = 2, kWideStart = 6;   // of a tile, and of a row's start

struct SharedArgs {
    KvCache c;
    const void* q;
    void* out;
    const int32_t* group_start;
    const int32_t* prefix_len;
    int n_groups, heads, group;
    float scale2;                    // scale * log2 e
    int window, n_sink;
    int first_seq, n_seqs;           // of this launch
    int columns;                     // of a row, at most (W)
    int wide_groups;                 // work groups of the launch for wide prefixes; 0: none could be worth it
    int wide_columns;
    WideRule rule;
    uint8_t* ws;
};

// The launch's sequences: what each belongs to, and the line.
struct Index {
    int64_t start[kSharedSeqs + 1];     // cost of the rows of all sequences before (a group's prefix rows are its first sequence's)
    int prefix[kSharedSeqs];            // of the group whose first sequence (of this launch) it is
    int low[kSharedSeqs];               // and the first key that any window of that group reaches
    int len[kSharedSeqs];
    uint16_t lead[kSharedSeqs];         // first sequence of its group; kNobody: of none
    uint16_t members[kSharedSeqs];      // of the group whose first sequence it is
    int first_row;                   // the first group's first sequence, which may be of a launch before
};
// What the later launches need of it, at the start of the workspace: the line, and the line of the prefixes that have a launch of
// their own (units of kWideTile keys).
struct Header {
    int64_t share, wide_share;
    int64_t start[kSharedSeqs + 1], wide_start[kSharedSeqs + 1];
    int prefix_units[kSharedSeqs], own_units[kSharedSeqs], prefix[kSharedSeqs], low[kSharedSeqs];
    uint16_t lead[kSharedSeqs], members[kSharedSeqs];
    uint8_t wide[kSharedSeqs];       // whether the group's prefix has its rows in the other line
    int first_row;
};
constexpr int64_t kHeaderBytes = (sizeof(Header) + 255) / 256 * 256;

// Records of [maximum, sum, -, -, output of dim channels]: of whole rows by (kind, sequence, head), then of parts of rows, two slots
// of W a work group: for the row that it goes on with and for the one that it leaves unfinished.  Then those of the launch for wide
// prefixes.
__host__ __device__ __forceinline__ int record_floats(int dim) { return dim + 4; }
__device__ __forceinline__ float* whole_record(const SharedArgs& a, int own, int s, int head) {
    return reinterpret_cast<float*>(a.ws + kHeaderBytes) + (((int64_t)own * a.n_seqs + s) * a.heads + head) * record_floats(a.c.dim);
}
__device__ __forceinline__ float* part_record(const SharedArgs& a, int64_t share, int slot, int column) {
    return reinterpret_cast<float*>(a.ws + kHeaderBytes) +
           ((int64_t)2 * a.n_seqs * a.heads + (2 * share + slot) * a.columns + column) * record_floats(a.c.dim);
}

__device__ __forceinline__ float* wide_record(const SharedArgs& a, int64_t share, int slot, int column) {
    return reinterpret_cast<float*>(a.ws + kHeaderBytes) +
           ((int64_t)2 * a.n_seqs * a.heads + (int64_t)2 * kSharedGroups * a.columns + (2 * share + slot) * a.wide_columns + column) *
               record_floats(a.c.dim);
}

// The keys of a row: those of [begin, end) at `low` and past it, and those below n_sink.  In units: first those of the sinks
// that lie before the others'.
struct Keys {
    int begin, end, first_sink, sink_units, first_unit, units;
};
template <int kUnit>
__device__ __forceinline__ Keys keys_of(int begin, int end, int low, int n_sink) {
    Keys k;
    k.begin = begin;
    k.end = end;
    const int from = low > begin ? low : begin, sinks = min(min(n_sink, low), end);
    k.first_unit = from / kUnit;
    const int near = from < end ? (end + kUnit - 1) / kUnit - k.first_unit : 0;
    k.first_sink = begin / kUnit;
    k.sink_units = sinks > begin ? (sinks + kUnit - 1) / kUnit - k.first_sink : 0;
    if (near > 0) k.sink_units = min(k.sink_units, k.first_unit - k.first_sink);
    k.units = k.sink_units + near;
    return k;
}

__device__ __forceinline__ int behind(const SharedArgs& a, int len) { return a.window > 0 && len > a.window ? len - a.window : 0; }

// a / b of numbers that are not negative: a 64-bit division is a hundred instructions and more.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// The line: a row of n units costs start + n cost, and nothing where it has none.
__device__ __forceinline__ int64_t line_cost(int units, int cost, int start) { return units == 0 ? 0 : start + (int64_t)units * cost; }
// The first unit of a row that starts `before` or later in it: the first at 0, the others behind the start's cost.
__device__ __forceinline__ int64_t line_unit(int64_t before, int cost, int start) {
    return before <= 0 ? 0 : before <= start + cost ? 1 : divide(before - start + cost - 1, cost);
}
// The share of every work group; none lies within one unit, nor within a start.
__device__ __forceinline__ int64_t line_share(int64_t all, int groups, int64_t least) {
    const int64_t want = (all + groups - 1) / groups;
    return want < least ? least : want;
}
// Where a row's parts lie: shares first .. first + count - 1 (a row of up to `whole` units is one part).
struct Parts {
    int64_t first;
    int count;
};
__device__ __forceinline__ Parts parts_of_row(int64_t at, int units, int whole, int cost, int start, int64_t share) {
    if (units <= whole) return {0, units > 0 ? 1 : 0};
    const int64_t first = divide(at, share), last = divide(units < 2 ? at : at + start + (int64_t)(units - 1) * cost, share);
    return {first, (int)(last - first) + 1};
}

// The prefixes of more than kNarrowColumns columns (k_attn_shared_wide.hip).
int attn_shared_wide_groups(int dim, bool f32);
hipError_t launch_attn_shared_wide(const SharedArgs& a, int dtype, bool f32, hipStream_t s);

}  // namespace bitnet
