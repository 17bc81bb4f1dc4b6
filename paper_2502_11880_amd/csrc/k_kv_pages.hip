// Pages of the cache: copying, forking, freeing and compacting them, and pages for new tokens.
//
// Which page a sequence owns is device data (table, kv_len, refs), so a serving loop never waits for the host and a captured
// graph stays valid: every call is a few launches that work out their page numbers themselves.  Pages are handed out lowest
// number first, in the order of the call's sequences, whatever the launch shape: results are reproducible.  Only copying
// moves bytes that count; it reads and writes every page once, in pieces of 16 KiB that a fixed grid shares out.
//
// Measured: compacting a pool of which half is live (1678 MB read and written) 328 to 342 us for the moves (4.9 to 5.1 TB/s; a large
// copy reaches 4.9) and 5 for the pairs; forking beams over 32 layers (235 MB) 30 us (the source pages are still in the last
// cache) and 5.6 for the plan, freeing 4 and reserving 5.6.  Plans take one work group because a page number depends on
// all before it: up to 8192 pages one pass of 1024 threads, and for compaction past that a work group for each 8192 of them.
#include "kv_cache.hpp"

namespace bitnet {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyWords = 4;                              // 16-byte words a thread holds at a time
constexpr int kPiece = kCopyThreads * kCopyWords * 16;     // bytes of a piece
constexpr int kCountIds = 8192;                            // page ids of one group of the compaction's counts

// Workspace: a header, three ints for every sequence of a call, three for every page, and the counts.
constexpr int kHeader = 64;                                // [0] pages to copy, [1] live pages
__host__ __device__ __forceinline__ int64_t ws_seq(int64_t n_seqs, int which) { return kHeader + which * n_seqs; }
__host__ __device__ __forceinline__ int64_t ws_page(int64_t n_seqs, int64_t n_pages, int which) {
    return kHeader + 3 * n_seqs + which * n_pages;
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int other = __shfl_up(v, i);
        if (lane >= i) v += other;
    }
    return v;
}

// Exclusive sum over the work group; total: of all threads.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int* part, int& total) {
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int incl = wave_scan(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wave] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < waves; ++w) {
        before += w < wave ? part[w] : 0;
        total += part[w];
    }
    return before + incl - v;
}

// The lowest `want` free pages into ids; returns how many there were (at most want).  One work group.
__device__ int lowest_free(const int32_t* refs, int n_pages, int want, int32_t* ids, int* part) {
    int found = 0;
    for (int at = 0; at < n_pages && found < want; at += 4 * kPlanThreads) {
        const int p = at + 4 * threadIdx.x;
        bool free_[4];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            free_[i] = p + i < n_pages && refs[p + i] == 0;
            mine += free_[i];
        }
        int total;
        int k = found + block_scan(mine, part, total);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (free_[i] && k < want) ids[k] = p + i;
            k += free_[i];
        }
        found += total;
    }
    __syncthreads();                                       // the ids of all threads
    return found < want ? found : want;
}

// Pages for new tokens.  One work group; a thread a sequence.  What a sequence wants counts against all after it whether it
// gets it or not: the list's order is kept, and one running sum decides.
__global__ __launch_bounds__(kPlanThreads) void kv_reserve_kernel(KvTables t, const int32_t* seqs, const int32_t* n_new, int n,
                                                                  int shift, int32_t* n_short, int32_t* ws) {
    __shared__ int part[kPlanThreads / 64];
    int32_t* offset = ws + ws_seq(t.n_seqs, 0);
    int32_t* ids = ws + ws_page(t.n_seqs, t.n_pages, 0);
    const int64_t most = (int64_t)t.max_pages << shift;
    // first table entry and number of pages that sequence i needs; false: it cannot have them
    auto need_of = [&](int i, int& s, int& first, int& count) {
        s = seqs[i];
        if ((unsigned)s >= (unsigned)t.n_seqs) return false;
        const int64_t len = t.kv_len[s], now = len + n_new[i];
        if (len < 0 || now < len || now > most) return false;
        first = (int)((len + (1 << shift) - 1) >> shift);
        count = (int)((now + (1 << shift) - 1) >> shift) - first;
        return true;
    };
    int want = 0, refused = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int s, first, count = 0;
        const bool ok = i < n && need_of(i, s, first, count);
        if (!ok) count = 0;
        int total;
        const int before = want + block_scan(count, part, total);
        if (i < n) offset[i] = ok ? before : -1;
        refused += i < n && !ok;
        want = want + total < t.n_pages + 1 ? want + total : t.n_pages + 1;   // more than there are: all later ones fail too
    }
    const int found = lowest_free(t.refs, t.n_pages, want < t.n_pages ? want : t.n_pages, ids, part);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        if (offset[i] < 0) continue;
        int s, first, count;
        need_of(i, s, first, count);
        if (count > 0 && (int64_t)offset[i] + count > found) {
            ++refused;
            continue;
        }
        for (int j = 0; j < count; ++j) {
            const int page = ids[offset[i] + j];
            t.table[(int64_t)s * t.max_pages + first + j] = page;
            t.refs[page] = 1;
        }
        t.kv_len[s] += n_new[i];
    }
    int total;
    block_scan(refused, part, total);
    if (threadIdx.x == 0) *n_short = total;
}

// Forking, first half: a new page for every child whose parent ends inside a page.  One work group.
__global__ __launch_bounds__(kPlanThreads) void kv_fork_plan_kernel(KvTables t, const int32_t* parents,
                                                                    const int32_t* children, int n, int shift,
                                                                    int32_t* n_short, int32_t* ws) {
    __shared__ int part[kPlanThreads / 64];
    int32_t* state = ws + ws_seq(t.n_seqs, 0);             // the child's place among the new pages; -1: needs none, -2: none left, -3: left out
    int32_t* src = ws + ws_seq(t.n_seqs, 1);
    int32_t* dst = ws + ws_seq(t.n_seqs, 2);
    int32_t* ids = ws + ws_page(t.n_seqs, t.n_pages, 0);
    int want = 0, refused = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        bool ok = false;
        int last = -1;
        if (i < n) {
            const int p = parents[i], c = children[i];
            ok = (unsigned)p < (unsigned)t.n_seqs && (unsigned)c < (unsigned)t.n_seqs && p != c;
            if (ok) {
                const int len = t.kv_len[p], full = len >> shift;
                ok = len >= 0 && (int64_t)len <= (int64_t)t.max_pages << shift;
                if (ok && (len & ((1 << shift) - 1))) last = t.table[(int64_t)p * t.max_pages + full];
                if ((unsigned)last >= (unsigned)t.n_pages) last = -1;
            }
        }
        int total;
        const int before = want + block_scan(last >= 0, part, total);
        if (i < n) {
            state[i] = !ok ? -3 : last >= 0 ? before : -1;
            src[i] = last;
        }
        refused += i < n && !ok;
        want += total;
    }
    const int found = lowest_free(t.refs, t.n_pages, want < t.n_pages ? want : t.n_pages, ids, part);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        int page = -1;
        if (state[i] >= 0) {
            if (state[i] < found) {
                page = ids[state[i]];
            } else {
                state[i] = -2;
                ++refused;
            }
        }
        dst[i] = page;
    }
    int total;
    block_scan(refused, part, total);
    if (threadIdx.x == 0) *n_short = total;
}

// Bytes of the pairs (src[i], dst[i]), i < n, in every plane: this work group's share, as number `group` of `groups`.  Pairs out
// of range are skipped.
__device__ void copy_pages(const KvPool& p, const int32_t* src, const int32_t* dst, int n, int group, int groups) {
    const int k_pieces = (int)((p.k_bytes + kPiece - 1) / kPiece), v_pieces = (int)((p.v_bytes + kPiece - 1) / kPiece);
    const int per_layer = k_pieces + v_pieces;
    const int64_t per_pair = (int64_t)per_layer * p.n_layers;
    const int64_t all = per_pair * n;
    for (int64_t w = group; w < all; w += groups) {
        const int pair = (int)(w / per_pair);
        const int64_t rest = w - pair * per_pair;
        const int layer = (int)(rest / per_layer);
        int piece = (int)(rest - (int64_t)layer * per_layer);
        const int from = src[pair], to = dst[pair];
        if ((unsigned)from >= (unsigned)p.n_pages || (unsigned)to >= (unsigned)p.n_pages || from == to) continue;
        const bool value = piece >= k_pieces;
        if (value) piece -= k_pieces;
        const int64_t bytes = value ? p.v_bytes : p.k_bytes;
        uint8_t* plane = (value ? p.v : p.k) + (int64_t)layer * p.n_pages * bytes;
        const uint8_t* a = plane + from * bytes + (int64_t)piece * kPiece;
        uint8_t* b = plane + to * bytes + (int64_t)piece * kPiece;
        const int left = (int)(bytes - (int64_t)piece * kPiece < kPiece ? bytes - (int64_t)piece * kPiece : kPiece);
        v4u x[kCopyWords];
#pragma unroll
        for (int i = 0; i < kCopyWords; ++i) {
            const int at = (threadIdx.x + i * kCopyThreads) * 16;
            if (at < left) x[i] = *reinterpret_cast<const v4u*>(a + at);
        }
#pragma unroll
        for (int i = 0; i < kCopyWords; ++i) {
            const int at = (threadIdx.x + i * kCopyThreads) * 16;
            if (at < left) *reinterpret_cast<v4u*>(b + at) = x[i];
        }
    }
}

__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(KvPool p, const int32_t* src, const int32_t* dst, int n) {
    copy_pages(p, src, dst, n, blockIdx.x, gridDim.x);
}

// Forking, second half: the children's rows and the reference counts by the first row_groups work groups, the last pages' bytes
// by the others.
__global__ __launch_bounds__(kCopyThreads) void kv_fork_kernel(KvPool pool, KvTables t, const int32_t* parents,
                                                               const int32_t* children, int n, int shift, const int32_t* ws,
                                                               int row_groups) {
    if ((int)blockIdx.x >= row_groups) {
        copy_pages(pool, ws + ws_seq(t.n_seqs, 1), ws + ws_seq(t.n_seqs, 2), n, blockIdx.x - row_groups, gridDim.x - row_groups);
        return;
    }
    const int64_t entries = (int64_t)n * t.max_pages;
    for (int64_t e = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (int64_t)row_groups * kCopyThreads) {
        const int i = (int)(e / t.max_pages), col = (int)(e - (int64_t)i * t.max_pages);
        const int state = ws[ws_seq(t.n_seqs, 0) + i];
        if (state == -3) continue;
        const int c = children[i], p = parents[i];
        const bool ok = state != -2;
        const int len = ok ? t.kv_len[p] : 0, full = len >> shift;
        if (col == 0) t.kv_len[c] = len;
        int page = -1;
        if (ok && col < full) {
            page = t.table[(int64_t)p * t.max_pages + col];
            if ((unsigned)page < (unsigned)t.n_pages) atomicAdd(&t.refs[page], 1);
        } else if (ok && col == full && state >= 0) {
            page = ws[ws_seq(t.n_seqs, 2) + i];
            t.refs[page] = 1;
        }
        t.table[(int64_t)c * t.max_pages + col] = page;
    }
}

// Freeing: every entry is taken by exactly one thread, so a sequence that is named twice is freed once.  With keep_window the
// sequence stays and loses the pages that no later token sees.
__global__ __launch_bounds__(256) void kv_free_kernel(KvTables t, const int32_t* seqs, int shift, bool keep_window, int window,
                                                      int n_sink) {
    const int s = seqs[blockIdx.x];
    if ((unsigned)s >= (unsigned)t.n_seqs) return;
    const int col = blockIdx.y * 256 + threadIdx.x;
    if (!keep_window && col == 0) t.kv_len[s] = 0;
    if (col >= t.max_pages) return;
    if (keep_window) {
        const int64_t from = (int64_t)col << shift, to = from + (1 << shift);
        if (from < n_sink || to > (int64_t)t.kv_len[s] + 1 - window) return;
    }
    const int page = atomicExch(&t.table[(int64_t)s * t.max_pages + col], -1);
    if ((unsigned)page < (unsigned)t.n_pages) atomicSub(&t.refs[page], 1);
}

// Compaction: the k-th lowest hole below the number of live pages takes the k-th highest live page above it.
// Live pages of every kCountIds ids (only where there are more than so many).
__global__ __launch_bounds__(256) void kv_count_kernel(const int32_t* refs, int n_pages, int32_t* counts) {
    __shared__ int part[4];
    int mine = 0;
#pragma unroll 8
    for (int i = 0; i < kCountIds / 256; ++i) {
        const int id = blockIdx.x * kCountIds + i * 256 + threadIdx.x;
        mine += id < n_pages && refs[id] > 0;
    }
    int total;
    block_scan(mine, part, total);
    if (threadIdx.x == 0) counts[blockIdx.x] = total;
}

// Pairs, and every page's place among the moved ones (-1: it stays).
__global__ __launch_bounds__(kPlanThreads) void kv_pairs_kernel(const int32_t* refs, int n_pages, int n_seqs, int groups,
                                                                int32_t* n_live_out, int32_t* ws) {
    __shared__ int part[kPlanThreads / 64];
    constexpr int kIds = kCountIds / kPlanThreads;
    const int32_t* counts = ws + ws_page(n_seqs, n_pages, 3);
    int32_t* src = ws + ws_page(n_seqs, n_pages, 0);
    int32_t* dst = ws + ws_page(n_seqs, n_pages, 1);
    int32_t* rank = ws + ws_page(n_seqs, n_pages, 2);
    const int id0 = blockIdx.x * kCountIds + threadIdx.x * kIds;
    int on[kIds], mine = 0;
#pragma unroll
    for (int i = 0; i < kIds; ++i) {
        on[i] = id0 + i < n_pages && refs[id0 + i] > 0;
        mine += on[i];
    }
    int before = 0, live, total;
    int k = block_scan(mine, part, total);                 // live pages below the id
    if (groups == 1) {
        live = total;
    } else {
        int lower = 0, all = 0;
        for (int g = threadIdx.x; g < groups; g += kPlanThreads) {
            const int c = counts[g];
            lower += g < (int)blockIdx.x ? c : 0;
            all += c;
        }
        block_scan(lower, part, before);
        block_scan(all, part, live);
    }
    k += before;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *n_live_out = live;
        if (live == 0) ws[0] = 0;
    }
#pragma unroll
    for (int i = 0; i < kIds; ++i) {
        const int id = id0 + i;
        if (id < n_pages) {
            int r = -1;
            if (on[i] && id >= live) {
                r = live - 1 - k;
                src[r] = id;
            } else if (!on[i] && id < live) {
                dst[id - k] = id;
            }
            rank[id] = r;
            if (id == live - 1) ws[0] = live - (k + on[i]);  // holes below the number of live pages
        }
        k += on[i];
    }
}

// The moves: tables and reference counts by the first row_groups work groups, the pages' bytes by the others.
__global__ __launch_bounds__(kCopyThreads) void kv_compact_kernel(KvPool pool, KvTables t, const int32_t* ws, int row_groups) {
    const int32_t* src = ws + ws_page(t.n_seqs, t.n_pages, 0);
    const int32_t* dst = ws + ws_page(t.n_seqs, t.n_pages, 1);
    const int32_t* rank = ws + ws_page(t.n_seqs, t.n_pages, 2);
    const int moves = ws[0];
    if ((int)blockIdx.x >= row_groups) {
        copy_pages(pool, src, dst, moves, blockIdx.x - row_groups, gridDim.x - row_groups);
        return;
    }
    const int64_t entries = (int64_t)t.n_seqs * t.max_pages, step = (int64_t)row_groups * kCopyThreads;
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += step) {
        const int page = t.table[i];
        if ((unsigned)page >= (unsigned)t.n_pages) continue;
        const int r = rank[page];
        if (r >= 0) t.table[i] = dst[r];
    }
    for (int64_t r = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; r < moves; r += step) {
        t.refs[dst[r]] = t.refs[src[r]];
        t.refs[src[r]] = 0;
    }
}

int copy_groups() { return device_cus() * 8; }
// Work groups for the entries of tables, up to 512.
int row_groups(int64_t entries) {
    const int64_t groups = (entries + kCopyThreads - 1) / kCopyThreads;
    return (int)(groups < 512 ? groups : 512);
}

int64_t pieces_of(const KvPool& p) {
    return ((p.k_bytes + kPiece - 1) / kPiece + (p.v_bytes + kPiece - 1) / kPiece) * p.n_layers;
}

}  // namespace

size_t kv_workspace_bytes(int64_t n_pages, int64_t n_seqs) {
    return (size_t)(ws_page(n_seqs, n_pages, 3) + (n_pages + kCountIds - 1) / kCountIds) * 4;
}

hipError_t launch_kv_copy(const KvPool& p, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
    const int64_t all = pieces_of(p) * n, most = copy_groups();
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(all < most ? all : most)), dim3(kCopyThreads), 0, s, p, src, dst, n);
    return hipGetLastError();
}

hipError_t launch_kv_free(const KvTables& t, const int32_t* seqs, int n, hipStream_t s) {
    hipLaunchKernelGGL(kv_free_kernel, dim3((unsigned)n, (unsigned)((t.max_pages + 255) / 256)), dim3(256), 0, s, t, seqs, 0,
                       false, 0, 0);
    return hipGetLastError();
}

hipError_t launch_kv_trim(const KvTables& t, const int32_t* seqs, int n, int shift, int window, int n_sink, hipStream_t s) {
    hipLaunchKernelGGL(kv_free_kernel, dim3((unsigned)n, (unsigned)((t.max_pages + 255) / 256)), dim3(256), 0, s, t, seqs,
                       shift, true, window, n_sink);
    return hipGetLastError();
}

hipError_t launch_kv_reserve(const KvTables& t, const int32_t* seqs, const int32_t* n_new, int n, int shift, int32_t* n_short,
                             void* ws, hipStream_t s) {
    hipLaunchKernelGGL(kv_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, s, t, seqs, n_new, n, shift, n_short,
                       static_cast<int32_t*>(ws));
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvPool& p, const KvTables& t, const int32_t* parents, const int32_t* children, int n,
                          int shift, int32_t* n_short, void* ws, hipStream_t s) {
    int32_t* w = static_cast<int32_t*>(ws);
    hipLaunchKernelGGL(kv_fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, t, parents, children, n, shift, n_short, w);
    if (n == 0) return hipGetLastError();
    const int64_t most = copy_groups(), all = pieces_of(p) * n;
    const int rows = row_groups((int64_t)n * t.max_pages);
    hipLaunchKernelGGL(kv_fork_kernel, dim3((unsigned)(rows + (all < most ? all : most))), dim3(kCopyThreads), 0, s, p, t, parents,
                       children, n, shift, w, rows);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const KvPool& p, const KvTables& t, int32_t* n_live, void* ws, hipStream_t s) {
    int32_t* w = static_cast<int32_t*>(ws);
    const int groups = (t.n_pages + kCountIds - 1) / kCountIds;
    if (groups > 1)
        hipLaunchKernelGGL(kv_count_kernel, dim3((unsigned)groups), dim3(256), 0, s, t.refs, t.n_pages,
                           w + ws_page(t.n_seqs, t.n_pages, 3));
    hipLaunchKernelGGL(kv_pairs_kernel, dim3((unsigned)groups), dim3(kPlanThreads), 0, s, t.refs, t.n_pages, t.n_seqs, groups,
                       n_live, w);
    const int64_t entries = (int64_t)t.n_seqs * t.max_pages > t.n_pages ? (int64_t)t.n_seqs * t.max_pages : t.n_pages;
    const int rows = row_groups(entries);
    const int64_t all = pieces_of(p) * (t.n_pages / 2 + 1), most = copy_groups();
    hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)(rows + (all < most ? all : most))), dim3(kCopyThreads), 0, s, p, t, w,
                       rows);
    return hipGetLastError();
}

}  // namespace bitnet
