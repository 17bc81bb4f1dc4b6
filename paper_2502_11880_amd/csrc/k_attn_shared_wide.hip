// Decode over shared prefixes, the prefixes of many columns: all query heads of a kv head of all sequences of a group, 128 to a work
// group of the prompt kernel (Prefill::run_prefix), so that a tile of 64 keys is read once for them and its products keep the
// matrix cores busy.  Every column sees the prefix whole, or what its length and window leave of it.
//
// The rows (group, kv head, 128 columns) stand in a line of their own, which the launch before worked out (Header), and every work
// group takes an equal share of its tiles.  Results go to records, as those of the other rows.  Weights go in two parts at least, as in the
// other rows (rounded once, they were 2^-9 off in bf16, for the sequences with enough neighbours only; the call took 131 us then).
//
// Measured: 64 sequences of 4 query heads a kv head behind 65536 keys, bf16 throughout, 130 us (68.7 GFLOP, 529 TFLOP/s, 793 in its parts),
// the whole call 154; in registers (32 columns a pass) 475.  The matrix cores are busy 40% of the time, a wave waits 49% of its own: each
// work group reads keys that no other is about to.  With weights in one part it took 99 to 104, with one tile of keys on its way 109 then,
// with 128 columns a pass 113.
#include "attn_prefill.hpp"
#include "attn_shared.hpp"

namespace bitnet {
namespace {

// Waves of a SIMD: q in parts leaves registers for one.
constexpr int per_simd(int dim, bool f32) { return dim <= 64 || (dim <= 128 && !f32) ? 2 : 1; }

// The last of n sequences that starts at x or before: 64 lanes probe at once.
__device__ __forceinline__ int find_start(const int64_t* start, int n, int64_t x) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const bool in = at < n && start[lo + (at < n ? at : 0)] <= x;
        const int count = __popcll(__ballot(in));
        const int skip = (count > 0 ? count - 1 : 0) * step;
        lo += skip;
        n = n - skip < step ? n - skip : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

template <int T, int DP, bool F32, int PER_SIMD, int WAVES, bool FULL>
__global__ __launch_bounds__(64 * WAVES, PER_SIMD) void attn_shared_wide_kernel(SharedArgs a) {
    using P = Prefill<T, DP, F32, WAVES, FULL, kPrefix>;
    constexpr int kColumns = 32 * WAVES;
    __shared__ typename P::Lds lds;
    const Header* h = reinterpret_cast<const Header*>(a.ws);
    const int64_t all = h->wide_start[a.n_seqs], share = h->wide_share;
    int64_t pos = blockIdx.x * share;
    const int64_t end = pos + share < all ? pos + share : all;
    PrefillArgs args{};
    args.c = a.c;
    args.q = a.q;
    args.heads = a.heads;
    args.group = a.group;
    args.scale2 = a.scale2;
    args.window = a.window;
    args.n_sink = a.n_sink;
    while (pos < end) {
        const int s = find_start(h->wide_start, a.n_seqs, pos);
        const int columns = h->members[s] * a.group, rows = (columns + kColumns - 1) / kColumns;
        const Keys keys = keys_of<kWideTile>(0, h->prefix[s], h->low[s], a.n_sink);
        const int64_t row_cost = line_cost(keys.units, kWideCost, kWideStart);
        const int row = (int)divide(pos - h->wide_start[s], row_cost);
        const int64_t at = h->wide_start[s] + row * row_cost;
        const int u0 = (int)line_unit(pos - at, kWideCost, kWideStart);
        const int64_t room = line_unit(end - at, kWideCost, kWideStart);
        const int u1 = room < keys.units ? (int)room : keys.units;
        pos = at + row_cost;
        if (u0 >= u1) continue;
        const int kvh = row / rows, col0 = (row - kvh * rows) * kColumns;
        // this lane's column; past the last one, that one once more
        const int col = col0 + (int)(threadIdx.x >> 6) * 32 + (int)(threadIdx.x & 31);
        const bool used = col < columns;
        const int member = (used ? col : columns - 1) / a.group, head = kvh * a.group + (used ? col : columns - 1) - member * a.group;
        const int len = seq_len(a.c, a.first_seq + s + member);
        const int last = (keys.end < len ? keys.end : len) - 1, low = a.window > 0 ? behind(a, len) - 1 : -1;
        float* record = u0 == 0 && u1 == keys.units ? whole_record(a, 0, s + member, head)
                                                    : wide_record(a, blockIdx.x, u0 > 0 ? 0 : 1, col - col0);
        P(args, lds).run_prefix(s == 0 ? h->first_row : a.first_seq + s, kvh, keys.end, last, low, keys.first_unit, keys.sink_units, u0, u1,
                                used, (int64_t)(a.first_seq + s + member) * a.heads + head, record);
        __syncthreads();
    }
}

template <int T, int DP, bool F32>
hipError_t launch(const SharedArgs& a, hipStream_t s) {
    constexpr int kWaves = wide_columns(DP, F32) / 32, kPerSimd = per_simd(DP, F32);
    const dim3 grid((unsigned)a.wide_groups), block(64 * kWaves);
    if (DP == 256 || a.c.dim == DP) hipLaunchKernelGGL((attn_shared_wide_kernel<T, DP, F32, kPerSimd, kWaves, true>), grid, block, 0, s, a);
    else if constexpr (DP < 256) hipLaunchKernelGGL((attn_shared_wide_kernel<T, DP, F32, kPerSimd, kWaves, false>), grid, block, 0, s, a);
    return hipGetLastError();
}

template <int T, bool F32>
hipError_t launch_dim(const SharedArgs& a, hipStream_t s) {
    if (a.c.dim <= 64) return launch<T, 64, F32>(a, s);
    if (a.c.dim <= 128) return launch<T, 128, F32>(a, s);
    return launch<T, 256, F32>(a, s);                     // 256: others past 128 have no wide prefixes (wide_rule)
}

}  // namespace

// One round of work groups; with their columns at most kSharedGroups times 128.
int attn_shared_wide_groups(int dim, bool f32) {
    const int waves = wide_columns(dim, f32) / 32, groups = 4 * per_simd(dim, f32) / waves * device_cus(), most = kSharedGroups * 4 / waves;
    return groups < most ? groups : most;
}

hipError_t launch_attn_shared_wide(const SharedArgs& a, int dtype, bool f32, hipStream_t s) {
    if (dtype == kBf16) return f32 ? launch_dim<kBf16, true>(a, s) : launch_dim<kBf16, false>(a, s);
    return f32 ? launch_dim<kF16, true>(a, s) : launch_dim<kF16, false>(a, s);
}

}  // namespace bitnet
