// Page operations of the 4-bit cache: release, share, grow (copying a shared
// page first) and keep the accepted path of a draft tree.
//
// All decisions are integers on the device, so a captured call replays on
// whatever the cache holds then, and they do not depend on the order in which
// workgroups run: free pages (page_refs <= 0) are given out in order of their
// numbers, entries are served in order of the list.  What an operation has to
// move is small (tables, one page a sequence, a path of some tokens a layer),
// so these kernels are bound by launches and by the latency of dependent
// loads: one launch that decides (a single workgroup where entries depend on
// each other), then one over all layers for the bytes.  32 streams' 64-node
// trees: room 7.0 us and 2.2 for no copy, path judged in 4.0 and moved in 3.8
// (8 layers of 8 heads); 64 forks that each copy a page in every layer: 46.8
// us, 5.4 TB/s.
#include "internal.h"
#include "kv.h"

namespace sense {
namespace {

constexpr int kThreads = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

enum : int { kOk = 0, kNoPages = 1, kTooLong = 2, kRefused = 3 };

__device__ __forceinline__ int pages_of(const KvCache& c, int tokens) {
    return (tokens + c.page() - 1) >> c.lg_page;
}

// Pages [from, to) of a sequence leave it.
__device__ __forceinline__ void release(const KvCache& c, int s, int from, int to, int thread,
                                        int threads) {
    int32_t* table = c.page_table + (int64_t)s * c.max_pages;
    for (int i = from + thread; i < to; i += threads) {
        const int id = table[i];
        if (kv_page_ok(c, id)) atomicSub(&c.page_refs[id], 1);
        table[i] = -1;
    }
}

// One workgroup an entry.  The minimum is taken atomically, so entries that
// name one sequence twice release disjoint ranges of its pages.
__global__ __launch_bounds__(kThreads) void kv_truncate_kernel(KvCache c, const int32_t* seqs,
                                                               const int32_t* lens,
                                                               int32_t* status) {
    __shared__ int s_old;
    const int i = blockIdx.x;
    const int s = kv_seq(c, seqs, i);
    const int to = lens ? lens[i] : 0;
    if (s < 0 || to < 0) {
        if (status && threadIdx.x == 0) status[i] = kRefused;
        return;
    }
    if (threadIdx.x == 0) {
        s_old = atomicMin(&c.seq_len[s], to);
        if (status) status[i] = kOk;
    }
    __syncthreads();
    const int old = s_old < c.capacity() ? s_old : c.capacity();
    if (old > to) release(c, s, pages_of(c, to), pages_of(c, old), threadIdx.x, kThreads);
}

// One workgroup a pair.  A pair is refused when its destination holds tokens
// or was listed before, or when its source is some pair's destination: then no
// workgroup reads what another writes.
__global__ __launch_bounds__(kThreads) void kv_fork_kernel(KvCache c, const int32_t* src,
                                                           const int32_t* dst, int n,
                                                           int32_t* status) {
    const int i = blockIdx.x;
    const int from = kv_seq(c, src, i), to = kv_seq(c, dst, i);
    bool bad = from < 0 || to < 0;
    for (int t = threadIdx.x; t < n; t += kThreads) {
        const int d = dst[t];
        bad |= (t < i && d == to) || d == from;
    }
    if (__syncthreads_or(bad)) {
        if (status && threadIdx.x == 0) status[i] = kRefused;
        return;
    }
    // No other workgroup writes `to`'s length or reads it past this point.
    const int held = c.seq_len[to];
    __syncthreads();
    if (held > 0) {
        if (status && threadIdx.x == 0) status[i] = kRefused;
        return;
    }
    const int len = kv_length(c, from);
    const int32_t* a = c.page_table + (int64_t)from * c.max_pages;
    int32_t* b = c.page_table + (int64_t)to * c.max_pages;
    for (int p = threadIdx.x; p < pages_of(c, len); p += kThreads) {
        const int id = a[p];
        b[p] = id;
        if (kv_page_ok(c, id)) atomicAdd(&c.page_refs[id], 1);
    }
    if (threadIdx.x == 0) {
        c.seq_len[to] = len;
        if (status) status[i] = kOk;
    }
}

// ------------------------------------------------------------------- grow

// A page to be copied: the filled slots of `src` to `dst`, in every layer.
struct Copy {
    int32_t src, dst, fill;
};

// Workspace of a reserve: copies[0].src = their number, then the copies, then
// the free pages that are given out.
__global__ __launch_bounds__(kPlanThreads) void kv_reserve_kernel(KvCache c, const int32_t* seqs,
                                                                  const int32_t* counts, int n,
                                                                  int32_t* status, Copy* copies,
                                                                  int32_t* free_ids) {
    __shared__ int s_seq[kKvMaxEntries];
    __shared__ int s_last[kKvMaxEntries];    // partly filled last page that grows, or -1
    __shared__ int s_need[kKvMaxEntries];    // pages, the copy among them
    __shared__ int64_t s_wave[kPlanThreads / 64];
    __shared__ int s_copies;
    const int tid = threadIdx.x;
    if (tid == 0) s_copies = 0;
    for (int i = tid; i < n; i += kPlanThreads) s_seq[i] = kv_seq(c, seqs, i);
    __syncthreads();
    // What each entry asks for.
    for (int i = tid; i < n; i += kPlanThreads) {
        const int s = s_seq[i], count = counts[i];
        int state = s < 0 || count < 0 ? kRefused : kOk;
        if (seqs && state == kOk)
            for (int t = 0; t < i; ++t)
                if (s_seq[t] == s) {
                    state = kRefused;
                    break;
                }
        int last = -1, need = 0;
        if (state == kOk) {
            const int len = kv_length(c, s);
            if (count > c.capacity() - len) {
                state = kTooLong;
            } else {
                need = pages_of(c, len + count) - pages_of(c, len);
                if (count > 0 && (len & (c.page() - 1))) {
                    last = c.page_table[(int64_t)s * c.max_pages + (len >> c.lg_page)];
                    if (!kv_page_ok(c, last)) last = -1;
                }
            }
        }
        s_last[i] = last;
        s_need[i] = state == kOk ? need : -state;    // refused ones below 0
    }
    __syncthreads();
    // A partly filled page that others hold too is copied; of the entries that
    // share one, the last holder keeps it.
    for (int i = tid; i < n; i += kPlanThreads) {
        const int last = s_last[i];
        if (last < 0 || s_need[i] < 0) continue;
        if (c.page_refs[last] <= 1) s_last[i] = -1 - last;   // nobody else: not copied
    }
    __syncthreads();
    int mine[kKvMaxEntries / kPlanThreads];
#pragma unroll
    for (int q = 0; q < kKvMaxEntries / kPlanThreads; ++q) {
        const int i = q * kPlanThreads + tid;
        mine[q] = 0;
        if (i >= n || s_last[i] < 0 || s_need[i] < 0) continue;
        int before = 0;
        for (int t = 0; t < i; ++t) before += s_last[t] == s_last[i];
        mine[q] = c.page_refs[s_last[i]] - before > 1;
    }
    __syncthreads();
    // Entries in order take free pages in order; from the first that does not
    // fit on, none is served.  `want` counts what all in front asked for.
    int64_t want = 0;
    int64_t first[kKvMaxEntries / kPlanThreads];
#pragma unroll
    for (int q = 0; q < kKvMaxEntries / kPlanThreads; ++q) {
        first[q] = 0;
        if (q * kPlanThreads >= n) break;            // the same for every thread
        const int i = q * kPlanThreads + tid;
        const int need = i < n && s_need[i] >= 0 ? s_need[i] + mine[q] : 0;
        int64_t all;
        const int64_t upto = block_scan(need, s_wave, &all);
        first[q] = want + upto - need;
        want += all;
    }
    int64_t have = 0;
    const bool vec = ((uintptr_t)c.page_refs & 15) == 0;
    for (int64_t at = 0; at < c.n_pages && have < want; at += 4 * kPlanThreads) {
        const int64_t p = at + 4 * tid;
        i32x4 refs = {1, 1, 1, 1};
        if (vec && p + 4 <= c.n_pages) {
            refs = *(const i32x4*)(c.page_refs + p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (p + e < c.n_pages) refs[e] = c.page_refs[p + e];
        }
        int here = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) here += refs[e] <= 0;
        int64_t all;
        int64_t to = have + block_scan(here, s_wave, &all) - here;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (refs[e] <= 0) {
                if (to < want) free_ids[to] = (int32_t)(p + e);
                ++to;
            }
        have += all;
    }
    __syncthreads();                                 // free_ids written, page_refs read
#pragma unroll
    for (int q = 0; q < kKvMaxEntries / kPlanThreads; ++q) {
        const int i = q * kPlanThreads + tid;
        if (i >= n) break;
        const int s = s_seq[i];
        int state = s_need[i] < 0 ? -s_need[i] : kOk;
        const int need = s_need[i] < 0 ? 0 : s_need[i] + mine[q];
        if (state == kOk && first[q] + need > have) state = kNoPages;
        if (status) status[i] = state;
        if (state != kOk) continue;
        const int len = kv_length(c, s), count = counts[i];
        int32_t* table = c.page_table + (int64_t)s * c.max_pages;
        int64_t at = first[q];
        if (mine[q]) {
            const int id = free_ids[at++];
            const int slot = atomicAdd(&s_copies, 1);
            Copy& k = copies[1 + slot];
            k.src = s_last[i];
            k.dst = id;
            k.fill = len & (c.page() - 1);
            table[len >> c.lg_page] = id;
            c.page_refs[id] = 1;
            atomicSub(&c.page_refs[s_last[i]], 1);
        }
        for (int p = pages_of(c, len); p < pages_of(c, len + count); ++p) {
            const int id = free_ids[at++];
            table[p] = id;
            c.page_refs[id] = 1;
        }
        c.seq_len[s] = len + count;
    }
    __syncthreads();
    if (tid == 0) copies[0].src = s_copies;
}

// The copies of a reserve: workgroups take (copy, layer, K or V, head) in turn.
__global__ __launch_bounds__(kThreads) void kv_copy_kernel(KvCache c, const Copy* copies) {
    const int n = copies[0].src;
    const int64_t parts = (int64_t)n * c.n_layers * 2 * c.heads;
    for (int64_t at = blockIdx.x; at < parts; at += gridDim.x) {
        const int head = (int)(at % c.heads);
        const int which = (int)(at / c.heads % 2);
        const int64_t rest = at / (2 * c.heads);
        const Copy k = copies[1 + rest / c.n_layers];
        const int layer = (int)(rest % c.n_layers);
        const int64_t from = c.rows_before(layer, k.src, which, head);
        const int64_t to = c.rows_before(layer, k.dst, which, head);
        const u32x4* a = (const u32x4*)(c.codes + from * (c.d / 2));
        u32x4* b = (u32x4*)(c.codes + to * (c.d / 2));
        for (int i = threadIdx.x; i < k.fill * c.d / 32; i += kThreads) b[i] = a[i];
        const u32x4* sa = (const u32x4*)(c.scales + from * (c.d / kKvBlock));
        u32x4* sb = (u32x4*)(c.scales + to * (c.d / kKvBlock));
        const int slots = (c.d / kKvBlock) << c.lg_page;    // a multiple of 16
        for (int i = threadIdx.x; i < slots / 16; i += kThreads) sb[i] = sa[i];
    }
}

// ---------------------------------------------------------------- compact

// Workspace: per entry the length to cut to (-1: refused), the number of rows
// to move, then the moves themselves (page * page size + slot) as pairs.
struct Move {
    int64_t src, dst;
};

__device__ __forceinline__ int64_t cell_of(const KvCache& c, int s, int pos) {
    const int id = c.page_table[(int64_t)s * c.max_pages + (pos >> c.lg_page)];
    if (!kv_page_ok(c, id)) return -1;
    return ((int64_t)id << c.lg_page) + (pos & (c.page() - 1));
}

// Judges the entries, a wave an entry: the moves are written down from the
// table as it is, and the length to cut to.  Nothing is changed yet, so no
// entry sees another's pages released.
__global__ __launch_bounds__(kThreads) void kv_judge_kernel(KvCache c, const int32_t* seqs,
                                                            KvKeep k, int n, int32_t* status,
                                                            int32_t* ends, int32_t* count,
                                                            Move* moves) {
    const int lane = threadIdx.x & 63;
    const int i = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (i >= n) return;
    const int s = kv_seq(c, seqs, i), tail = k.tails[i];
    const int pick = k.pick ? k.pick[i] : 0;
    bool bad = s < 0 || tail < 0 || (unsigned)pick >= (unsigned)k.keep_rows;
    if (seqs)
        for (int t = lane; t < i; t += 64) bad |= seqs[t] == s;
    const int len = s < 0 ? 0 : kv_length(c, s);
    bad |= tail > len;
    bool refuse = __any(bad);
    int kept = 0, n_moves = 0;
    const int base = len - tail;
    if (!refuse) {
        const int64_t row = (int64_t)i * k.keep_rows + pick;
        const int32_t* keep = k.keep + row * k.keep_ld;
        int most = k.keep_len[row];
        most = most < 0 ? 0 : (most < k.keep_ld ? most : k.keep_ld);
        // The leading run of strictly ascending nodes of the tail, and of them
        // the rows that move; whether a page they go to is shared.
        bool shared = false, more = true;
        Move* out = moves + (int64_t)i * k.keep_ld;
        for (int j0 = 0; j0 < most && more; j0 += 64) {
            const int j = j0 + lane;
            const int node = j < most ? keep[j] : 0;
            const int prev = j < most && j > 0 ? keep[j - 1] : -1;
            const uint64_t stop = __ballot(j >= most || node <= prev || node >= tail);
            const int wide = stop ? __builtin_ctzll(stop) : 64;
            more = wide == 64;
            kept += wide;
            bool go = lane < wide && node != j;
            int64_t src = -1, dst = -1;
            if (go) {
                src = cell_of(c, s, base + node);
                dst = cell_of(c, s, base + j);
                go = src >= 0 && dst >= 0;
                if (go) shared |= c.page_refs[dst >> c.lg_page] > 1;
            }
            const uint64_t who = __ballot(go);
            if (go) {
                Move& m = out[n_moves + __popcll(who & ((1ull << lane) - 1))];
                m.src = src;
                m.dst = dst;
            }
            n_moves += __popcll(who);
        }
        refuse = __any(shared);
    }
    if (lane == 0) {
        ends[i] = refuse ? -1 : base + kept;
        count[i] = refuse ? 0 : n_moves;
        if (status) status[i] = refuse ? kRefused : kOk;
    }
}

// The moves of a (layer, K or V, head): a wave an entry's, in order.  A path's
// nodes ascend, so a row goes to its own place or further to the front and
// never onto a row that a later move reads; a wave's rows are all read before
// the first of them is written.  The first waves cut the sequences instead:
// the moves are in the list, so no other wave needs the table any more.
template <int D>
__global__ __launch_bounds__(kThreads) void kv_move_kernel(KvCache c, const int32_t* seqs, int n,
                                                           int keep_ld, const int32_t* ends,
                                                           const int32_t* count,
                                                           const Move* moves) {
    constexpr int kPer = D / 32;                     // 16-byte parts of a row
    constexpr int kRows = 64 / kPer;                 // rows of a wave's step
    const int lane = threadIdx.x & 63;
    int64_t at = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (at < n) {
        const int end = ends[at];
        if (end < 0) return;
        const int s = kv_seq(c, seqs, (int)at);
        const int len = kv_length(c, s);
        release(c, s, pages_of(c, end), pages_of(c, len), lane, 64);
        if (lane == 0) c.seq_len[s] = end;
        return;
    }
    at -= n;
    const int heads2 = 2 * c.heads;
    if (at >= (int64_t)n * c.n_layers * heads2) return;
    const int head = (int)(at % heads2);
    const int64_t rest = at / heads2;
    const int i = (int)(rest % n), layer = (int)(rest / n);
    const int m = count[i];
    const Move* list = moves + (int64_t)i * keep_ld;
    const int part = lane % kPer;
    for (int j0 = 0; j0 < m; j0 += kRows) {
        const int j = j0 + lane / kPer;
        const bool on = j < m;
        u32x4 x = {0, 0, 0, 0};
        uint8_t sc = 0;
        u32x4* to = nullptr;
        uint8_t* sto = nullptr;
        if (on) {
            const Move v = list[j];
            const int page = c.page();
            const int64_t pre = c.rows_before(layer, 0, 0, 0) + ((int64_t)head << c.lg_page);
            const int64_t a = pre + (v.src >> c.lg_page) * heads2 * page;
            const int64_t b = pre + (v.dst >> c.lg_page) * heads2 * page;
            const int sa = (int)(v.src & (page - 1)), sb = (int)(v.dst & (page - 1));
            x = *(const u32x4*)(c.codes + (a + sa) * (D / 2) + part * 16);
            sc = c.scales[a * kPer + (part << c.lg_page) + sa];
            to = (u32x4*)(c.codes + (b + sb) * (D / 2) + part * 16);
            sto = c.scales + b * kPer + (part << c.lg_page) + sb;
        }
        // All lanes' rows have arrived before any lane writes one.
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_wave_barrier();
        if (on) {
            *to = x;
            *sto = sc;
        }
    }
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

hipError_t launch_kv_truncate(const KvCache& c, const int32_t* seqs, const int32_t* lens, int n,
                              int32_t* status, hipStream_t st) {
    hipLaunchKernelGGL(kv_truncate_kernel, dim3((unsigned)n), dim3(kThreads), 0, st, c, seqs, lens,
                       status);
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvCache& c, const int32_t* src, const int32_t* dst, int n,
                          int32_t* status, hipStream_t st) {
    hipLaunchKernelGGL(kv_fork_kernel, dim3((unsigned)n), dim3(kThreads), 0, st, c, src, dst, n,
                       status);
    return hipGetLastError();
}

size_t kv_reserve_workspace_bytes(int n, int n_pages) {
    return align256((size_t)(n + 1) * sizeof(Copy)) + align256((size_t)n_pages * sizeof(int32_t));
}

hipError_t launch_kv_reserve(const KvCache& c, const int32_t* seqs, const int32_t* counts, int n,
                             int32_t* status, void* workspace, hipStream_t st) {
    Copy* copies = (Copy*)workspace;
    int32_t* ids = (int32_t*)((char*)workspace + align256((size_t)(n + 1) * sizeof(Copy)));
    hipLaunchKernelGGL(kv_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, st, c, seqs, counts, n,
                       status, copies, ids);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t parts = (int64_t)n * c.n_layers * 2 * c.heads, most = 16 * device_cus();
    hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)(parts < most ? parts : most)),
                       dim3(kThreads), 0, st, c, copies);
    return hipGetLastError();
}

size_t kv_compact_workspace_bytes(int n, int keep_ld) {
    return align256((size_t)2 * n * sizeof(int32_t)) + align256((size_t)n * keep_ld * sizeof(Move));
}

hipError_t launch_kv_compact(const KvCache& c, const int32_t* seqs, const KvKeep& k, int n,
                             int32_t* status, void* workspace, hipStream_t st) {
    int32_t* ends = (int32_t*)workspace;
    int32_t* count = ends + n;
    Move* moves = (Move*)((char*)workspace + align256((size_t)2 * n * sizeof(int32_t)));
    constexpr int kWaves = kThreads / 64;
    hipLaunchKernelGGL(kv_judge_kernel, dim3((unsigned)((n + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, st, c, seqs, k, n, status, ends, count, moves);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t waves = n + (int64_t)n * c.n_layers * 2 * c.heads;
    const dim3 grid((unsigned)((waves + kWaves - 1) / kWaves));
    if (c.d == 64)
        hipLaunchKernelGGL((kv_move_kernel<64>), grid, dim3(kThreads), 0, st, c, seqs, n,
                           k.keep_ld, ends, count, moves);
    else if (c.d == 128)
        hipLaunchKernelGGL((kv_move_kernel<128>), grid, dim3(kThreads), 0, st, c, seqs, n,
                           k.keep_ld, ends, count, moves);
    else
        hipLaunchKernelGGL((kv_move_kernel<256>), grid, dim3(kThreads), 0, st, c, seqs, n,
                           k.keep_ld, ends, count, moves);
    return hipGetLastError();
}

}  // namespace sense
