// Rows of keys and values into the 4-bit paged cache, and back out of it.
//
// Writing a block of 32 values: with a its largest magnitude, the unit is
// 2^(floor(log2 a) - 2), so a lies in [4, 8) units; every value goes to the
// nearest of 0 .5 1 1.5 2 3 4 6 units (a tie to the even code, beyond 6 to
// 6), which is what v_cvt_scalef32_pk_fp4_f32 does in one rounding from fp32.
// Reading is exact: a code times a power of two.
//
// Both move every byte once (2.53 bytes a 16-bit value) and do a few
// operations on it.  A thread has 8 values: 16 bytes of a 16-bit row, 4 bytes
// of codes; the four threads of a block find its largest value with two lane
// exchanges.  A workgroup takes up to 16 tokens (of 128 values) of one head
// side by side, so that the codes of a page's head leave as one run and a
// block's scales as neighbouring bytes; a call of few tokens fills the
// workgroup with more heads instead.
#include "internal.h"
#include "kv.h"

namespace sense {
namespace {

constexpr int kThreads = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float from_bits16(uint32_t b, int dt) {
    if (dt == DT_BF16) return __builtin_bit_cast(float, b << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)b);
}

template <int DT>
__device__ __forceinline__ void load8(const void* p, int64_t at, float* x) {
    if constexpr (DT == DT_F32) {
        const f32x4* s = (const f32x4*)((const float*)p + at);
        const f32x4 a = s[0], b = s[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        const u32x4 a = *(const u32x4*)((const uint16_t*)p + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = from_bits16(a[i] & 0xFFFFu, DT);
            x[2 * i + 1] = from_bits16(a[i] >> 16, DT);
        }
    }
}

template <int DT>
__device__ __forceinline__ void store8(void* p, int64_t at, const float* x) {
    if constexpr (DT == DT_F32) {
        const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        f32x4* d = (f32x4*)((float*)p + at);
        d[0] = a;
        d[1] = b;
    } else {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = (uint32_t)to_bits16(x[2 * i], DT) | (uint32_t)to_bits16(x[2 * i + 1], DT) << 16;
        *(u32x4*)((uint16_t*)p + at) = a;
    }
}

// One thread's 8 values: which entry, layer, K or V, head and token.
struct Place {
    int64_t cell;    // rows in front in the cache, slot included
    int64_t row;     // row of the tensor
    int head, which, layer;
    bool ok;         // the token exists
    bool page_ok;
};

template <int D>
__device__ __forceinline__ Place place(const KvCache& c, const KvBatch& b, const KvRows& r,
                                       int lg_tokens, int blocks_per_entry, int token_tiles,
                                       int* entry, int* seq) {
    constexpr int kRows = kThreads / (D / 8);       // rows of a workgroup
    const int row = threadIdx.x / (D / 8);
    const int tokens = 1 << lg_tokens;              // token run of a workgroup
    const int per = kRows >> lg_tokens;             // (K or V, head) pairs of a workgroup
    const int i = blockIdx.x / blocks_per_entry;
    const int rest = blockIdx.x % blocks_per_entry;
    const int tile = rest % token_tiles;
    const int pair = (rest / token_tiles) * per + (row >> lg_tokens);
    const int j = tile * tokens + (row & (tokens - 1));
    Place p;
    *entry = i;
    const int s = kv_seq(c, b.seqs, i);
    *seq = s;
    p.layer = blockIdx.y;
    p.which = pair >= c.heads;
    p.head = pair - (p.which ? c.heads : 0);
    p.ok = s >= 0 && pair < 2 * c.heads;
    p.page_ok = false;
    p.cell = p.row = 0;
    if (!p.ok) return p;
    const int m = kv_rows(b, i);
    const int pos = kv_length(c, s) - m + j;
    p.row = kv_start(b, i) + j;
    p.ok = j < m && pos >= 0 && p.row >= 0 && p.row < b.n_rows;
    if (!p.ok) return p;
    const int id = c.page_table[(int64_t)s * c.max_pages + (pos >> c.lg_page)];
    p.page_ok = kv_page_ok(c, id);
    if (p.page_ok)
        p.cell = c.rows_before(r.layer + p.layer, id, p.which, p.head) + (pos & (c.page() - 1));
    return p;
}

// Bytes in front of block `blk` of the row at `cell`: scales lie block-major
// in a page's head, so that neighbouring tokens' scales are neighbours.
__device__ __forceinline__ int64_t scale_at(const KvCache& c, int64_t cell, int blk) {
    const int64_t slot = cell & (c.page() - 1);
    return (cell - slot) * (c.d / kKvBlock) + ((int64_t)blk << c.lg_page) + slot;
}

template <int D, int DT>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, KvBatch b, KvRows r,
                                                            int lg_tokens, int blocks_per_entry,
                                                            int token_tiles) {
    int i, s;
    const Place p = place<D>(c, b, r, lg_tokens, blocks_per_entry, token_tiles, &i, &s);
    // A sequence that is listed again: its first entry is the one written.
    bool again = false;
    if (b.seqs) {
        for (int t = threadIdx.x; t < i; t += kThreads) again |= b.seqs[t] == s;
        again = __syncthreads_or(again);
    }
    const int vec = threadIdx.x % (D / 8);
    float x[8] = {};
    const bool on = p.ok && p.page_ok && !again;
    if (on)
        load8<DT>(p.which ? r.v : r.k, p.layer * r.layer_stride + p.row * r.row_stride +
                                           (int64_t)p.head * D + vec * 8, x);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x[e]) & 0x7FFFFFFFu;
        top = u > top ? u : top;
    }
#pragma unroll
    for (int step = 1; step < 4; step <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)top, step);
        top = o > top ? o : top;
    }
    if (!on) return;
    const bool finite = top < 0x7F800000u;
    const int e = (int)(top >> 23) - 2;
    const uint32_t sc = finite ? (uint32_t)(e > 0 ? e : 0) : 255u;
    const float unit = __builtin_bit_cast(float, sc << 23);   // only its exponent is used
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
    *(uint32_t*)(c.codes + p.cell * (D / 2) + vec * 4) = finite ? w : 0u;
    if (vec % 4 == 0) c.scales[scale_at(c, p.cell, vec / 4)] = (uint8_t)sc;
}

template <int D, int DT>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, KvBatch b, KvRows r,
                                                           int lg_tokens, int blocks_per_entry,
                                                           int token_tiles) {
    int i, s;
    const Place p = place<D>(c, b, r, lg_tokens, blocks_per_entry, token_tiles, &i, &s);
    if (!p.ok) return;
    const int vec = threadIdx.x % (D / 8);
    float x[8] = {};
    if (p.page_ok) {
        const uint32_t w = *(const uint32_t*)(c.codes + p.cell * (D / 2) + vec * 4);
        const float unit =
            __builtin_bit_cast(float, (uint32_t)c.scales[scale_at(c, p.cell, vec / 4)] << 23);
        const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0);
        const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
        const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2);
        const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3);
        x[0] = a0.x, x[1] = a0.y, x[2] = a1.x, x[3] = a1.y;
        x[4] = a2.x, x[5] = a2.y, x[6] = a3.x, x[7] = a3.y;
    }
    store8<DT>(p.which ? r.v : r.k, p.layer * r.layer_stride + p.row * r.row_stride +
                                        (int64_t)p.head * D + vec * 8, x);
}

// Token run (its logarithm), token runs of an entry, workgroups of an entry.
struct Shape {
    int lg, tiles, blocks;
};
Shape shape_of(const KvCache& c, const KvBatch& b) {
    const int rows = kThreads / (c.d / 8);
    Shape s = {0, 0, 0};
    while ((1 << s.lg) < b.max_rows && (1 << s.lg) < rows) ++s.lg;
    s.tiles = (b.max_rows + (1 << s.lg) - 1) >> s.lg;
    const int per = rows >> s.lg;
    s.blocks = (2 * c.heads + per - 1) / per * s.tiles;
    return s;
}

template <bool WRITE, int D>
hipError_t launch_d(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    const Shape h = shape_of(c, b);
    const dim3 grid((unsigned)((int64_t)h.blocks * b.n), (unsigned)r.n_layers);
#define SENSE_KV_ROWS(T)                                                                     \
    if constexpr (WRITE)                                                                     \
        hipLaunchKernelGGL((kv_write_kernel<D, T>), grid, dim3(kThreads), 0, st, c, b, r,     \
                           h.lg, h.blocks, h.tiles);                                         \
    else                                                                                     \
        hipLaunchKernelGGL((kv_read_kernel<D, T>), grid, dim3(kThreads), 0, st, c, b, r,      \
                           h.lg, h.blocks, h.tiles)
    if (r.dtype == DT_F32) {
        SENSE_KV_ROWS(DT_F32);
    } else if (r.dtype == DT_F16) {
        SENSE_KV_ROWS(DT_F16);
    } else {
        SENSE_KV_ROWS(DT_BF16);
    }
#undef SENSE_KV_ROWS
    return hipGetLastError();
}

template <bool WRITE>
hipError_t launch_rows(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    if (c.d == 64) return launch_d<WRITE, 64>(c, b, r, st);
    if (c.d == 128) return launch_d<WRITE, 128>(c, b, r, st);
    return launch_d<WRITE, 256>(c, b, r, st);
}

}  // namespace

int64_t kv_rows_blocks(const KvCache& c, const KvBatch& b) {
    return (int64_t)shape_of(c, b).blocks * b.n;
}
hipError_t launch_kv_write(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    return launch_rows<true>(c, b, r, st);
}
hipError_t launch_kv_read(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    return launch_rows<false>(c, b, r, st);
}

}  // namespace sense
