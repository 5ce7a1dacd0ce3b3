// The paged key/value cache held in 4 bits: its layout, and the launchers of
// the kernels that work on it (kv_rows.hip, kv_attention.hip, kv_pages.hip).
//
// A row is one token's key (or value) of one head: d values in blocks of 32.
// A block is 32 E2M1 codes (sign, 0 .5 1 1.5 2 3 4 6) in units of
// 2^(scale - 127), scale a byte; scale 255 makes the block NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sense {

constexpr int kKvBlock = 32;             // values that share a scale
constexpr int kKvMaxEntries = 4096;      // entries of one page operation
constexpr int kKvMaxRows = 1 << 20;      // rows of one entry in a call

// Sequence sizes on the device are clamped to what the cache can hold and
// page ids are checked before use, so no table content reads out of range.
struct KvCache {
    uint8_t* codes;       // [layer][page][K, V][head][slot][d / 2]
    uint8_t* scales;      // [layer][page][K, V][head][d / 32][slot]
    int32_t* page_table;  // [seq][max_pages]
    int32_t* seq_len;     // [seq]
    int32_t* page_refs;   // [page], <= 0: free
    int n_layers, n_pages, lg_page, heads, d, n_seqs, max_pages;

    __host__ __device__ int page() const { return 1 << lg_page; }
    __host__ __device__ int capacity() const { return max_pages << lg_page; }
    // Rows in front of (layer, page, which, head): which 0 = K, 1 = V.
    __host__ __device__ int64_t rows_before(int layer, int page_id, int which, int head) const {
        return ((((int64_t)layer * n_pages + page_id) * 2 + which) * heads + head) << lg_page;
    }
};

#ifdef __HIPCC__
__device__ __forceinline__ int kv_length(const KvCache& c, int seq) {
    const int n = c.seq_len[seq];
    return n < 0 ? 0 : (n < c.capacity() ? n : c.capacity());
}
__device__ __forceinline__ bool kv_page_ok(const KvCache& c, int id) {
    return (unsigned)id < (unsigned)c.n_pages;
}
#endif

// The entries of a call: entry i is sequence seqs[i] (i itself when seqs is
// NULL), whose last row_len[i] cached positions (max_rows when NULL) meet the
// rows row_start[i].. (i * max_rows when NULL) of the tensors of n_rows rows.
struct KvBatch {
    const int32_t* seqs;
    const int32_t* row_start;
    const int32_t* row_len;
    int n;
    int max_rows;
    int64_t n_rows;
};

#ifdef __HIPCC__
// Entry i's sequence, or -1 when there is none of that number.
__device__ __forceinline__ int kv_seq(const KvCache& c, const int32_t* seqs, int i) {
    const int s = seqs ? seqs[i] : i;
    return (unsigned)s < (unsigned)c.n_seqs ? s : -1;
}
__device__ __forceinline__ int kv_rows(const KvBatch& b, int i) {
    const int m = b.row_len ? b.row_len[i] : b.max_rows;
    return m < 0 ? 0 : (m < b.max_rows ? m : b.max_rows);
}
__device__ __forceinline__ int64_t kv_start(const KvBatch& b, int i) {
    return b.row_start ? (int64_t)b.row_start[i] : (int64_t)i * b.max_rows;
}

// Inclusive prefix sums over the threads of a workgroup that plans alone, in
// their order; s_wave is its scratch, a number a wave.
constexpr int kPlanThreads = 1024;
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* s_wave, int64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int64_t o = __shfl_up((long long)v, s);
        if (lane >= s) v += o;
    }
    if (lane == 63) s_wave[wave] = v;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += s_wave[w];
        all += s_wave[w];
    }
    __syncthreads();
    *total = all;
    return v + before;
}
#endif

// Rows of n_layers layers from `layer` on; strides in elements, head h of a
// row at h * d.
struct KvRows {
    void* k;
    void* v;
    int dtype;
    int64_t row_stride;
    int64_t layer_stride;
    int layer;
    int n_layers;
};
hipError_t launch_kv_write(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st);
hipError_t launch_kv_read(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st);

struct KvAttention {
    const void* q;
    void* out;
    int dtype;               // F16 or BF16
    int layer;
    int n_heads;
    int64_t q_stride;
    int64_t out_stride;
    const uint8_t* mask;     // NULL: causal
    int64_t mask_ld;
    int64_t mask_stride;
    float scale;
    int max_kv;              // the caller's bound on the lengths (a hint)
};
// Workgroups of a call (its largest launch).
int64_t kv_rows_blocks(const KvCache& c, const KvBatch& b);
int64_t kv_attention_blocks(int n, int max_rows, int n_heads, int kv_heads, int d);
size_t kv_attention_workspace_bytes(int n, int max_rows, int n_heads, int kv_heads, int d,
                                    int max_kv);
hipError_t launch_kv_attention(const KvCache& c, const KvBatch& b, const KvAttention& a,
                               void* workspace, hipStream_t st);

// Page operations (kv_pages.hip); status may be NULL.
size_t kv_reserve_workspace_bytes(int n, int n_pages);
hipError_t launch_kv_truncate(const KvCache& c, const int32_t* seqs, const int32_t* lens, int n,
                              int32_t* status, hipStream_t st);
hipError_t launch_kv_fork(const KvCache& c, const int32_t* src, const int32_t* dst, int n,
                          int32_t* status, hipStream_t st);
hipError_t launch_kv_reserve(const KvCache& c, const int32_t* seqs, const int32_t* counts, int n,
                             int32_t* status, void* workspace, hipStream_t st);
struct KvKeep {
    const int32_t* tails;
    const int32_t* keep;
    const int32_t* keep_len;
    const int32_t* pick;
    int keep_rows;           // rows of `keep` per entry
    int keep_ld;
};
size_t kv_compact_workspace_bytes(int n, int keep_ld);
hipError_t launch_kv_compact(const KvCache& c, const int32_t* seqs, const KvKeep& k, int n,
                             int32_t* status, void* workspace, hipStream_t st);

}  // namespace sense
