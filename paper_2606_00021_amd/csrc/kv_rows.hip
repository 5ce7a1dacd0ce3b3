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
// exchanges.  A workgroup takes up to 16 tokens (of 128 values) side by side,
// so that the codes of a page's head leave as one run and a block's scales as
// neighbouring bytes, of one head after the other where there is work for the
// whole device; a call of few tokens puts heads beside each other instead.
// 8 x 2048 rows of 8 heads of 128, keys and values, 85 MB: written in 17.0 us
// (5.0 TB/s), read back in 18.1 (4.7), a large copy reaches 4.9; 61 rows 3.3
// and 3.0 us.
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

// A thread's token: which row of the tensors, and where in the cache.
struct Place {
    int64_t row;     // row of the tensors
    int64_t page;    // its number; slot: the token's place in it
    int slot;
    int seq;
    bool ok;         // the token exists
    bool page_ok;    // and has a page
};

// How a launch is cut: a workgroup has 2^lg tokens of one entry side by side
// and `per` (K or V, head) pairs beside them, `loops` times.
struct Shape {
    int lg, tiles;       // tokens of a workgroup; workgroups along an entry's tokens
    int per, loops;
    int groups;          // workgroups along the pairs
    int64_t blocks() const { return (int64_t)tiles * groups; }
};

__device__ __forceinline__ Place place(const KvCache& c, const KvBatch& b, int entry, int j) {
    Place p;
    p.row = 0;
    p.page = 0;
    p.slot = 0;
    p.ok = p.page_ok = false;
    p.seq = kv_seq(c, b.seqs, entry);
    if (p.seq < 0) return p;
    const int m = kv_rows(b, entry);
    const int pos = kv_length(c, p.seq) - m + j;
    p.row = kv_start(b, entry) + j;
    p.ok = j < m && pos >= 0 && p.row >= 0 && p.row < b.n_rows;
    if (!p.ok) return p;
    const int id = c.page_table[(int64_t)p.seq * c.max_pages + (pos >> c.lg_page)];
    p.page_ok = kv_page_ok(c, id);
    p.page = p.page_ok ? id : 0;
    p.slot = pos & (c.page() - 1);
    return p;
}

// A workgroup's entry, first pair and token, from its number.
struct Work {
    int entry, pair, j;
};
template <int D>
__device__ __forceinline__ Work work_of(const Shape& h) {
    const int row = threadIdx.x / (D / 8);
    const int at = blockIdx.x;
    Work w;
    const int blocks = h.tiles * h.groups;
    w.entry = at / blocks;
    const int rest = at % blocks;
    w.j = (rest % h.tiles << h.lg) + (row & ((1 << h.lg) - 1));
    w.pair = rest / h.tiles * h.per * h.loops + (row >> h.lg);
    return w;
}

constexpr int kUnroll = 4;      // pairs whose bytes are on their way together

template <int D, int DT>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, KvBatch b, KvRows r,
                                                            Shape h) {
    const Work w = work_of<D>(h);
    const Place p = place(c, b, w.entry, w.j);
    const int vec = threadIdx.x % (D / 8);
    // A sequence that is listed again: its first entry is the one written.
    bool again = false;
    if (b.seqs) {
        for (int t = threadIdx.x; t < w.entry; t += kThreads) again |= b.seqs[t] == p.seq;
        again = __syncthreads_or(again);
    }
    const int64_t from = blockIdx.y * r.layer_stride + p.row * r.row_stride + vec * 8;
    for (int l0 = 0; l0 < h.loops; l0 += kUnroll) {
        float x[kUnroll][8];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int pair = w.pair + (l0 + u) * h.per;
            const bool v = pair >= c.heads;
            if (p.ok && l0 + u < h.loops && pair < 2 * c.heads) {
                load8<DT>(v ? r.v : r.k, from + (int64_t)(pair - (v ? c.heads : 0)) * D, x[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int pair = w.pair + (l0 + u) * h.per;
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t bits = __builtin_bit_cast(uint32_t, x[u][e]) & 0x7FFFFFFFu;
                top = bits > top ? bits : top;
            }
#pragma unroll
            for (int step = 1; step < 4; step <<= 1) {
                const uint32_t o = (uint32_t)__shfl_xor((int)top, step);
                top = o > top ? o : top;
            }
            if (!p.page_ok || again || l0 + u >= h.loops || pair >= 2 * c.heads) continue;
            const bool finite = top < 0x7F800000u;
            const int e = (int)(top >> 23) - 2;
            const uint32_t sc = finite ? (uint32_t)(e > 0 ? e : 0) : 255u;
            const float unit = __builtin_bit_cast(float, sc << 23);   // only its exponent is used
            uint32_t code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][0], x[u][1], unit, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][2], x[u][3], unit, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][4], x[u][5], unit, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][6], x[u][7], unit, 3);
            // K and V pairs lie one after the other in a page.
            const int64_t base =
                c.rows_before(r.layer + (int)blockIdx.y, (int)p.page, 0, 0) + ((int64_t)pair << c.lg_page);
            *(uint32_t*)(c.codes + (base + p.slot) * (D / 2) + vec * 4) = finite ? code : 0u;
            if (vec % 4 == 0)
                c.scales[base * (D / kKvBlock) + (vec / 4 << c.lg_page) + p.slot] = (uint8_t)sc;
        }
    }
}

template <int D, int DT>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, KvBatch b, KvRows r,
                                                           Shape h) {
    const Work w = work_of<D>(h);
    const Place p = place(c, b, w.entry, w.j);
    if (!p.ok) return;
    const int vec = threadIdx.x % (D / 8);
    const int64_t to = blockIdx.y * r.layer_stride + p.row * r.row_stride + vec * 8;
    for (int l0 = 0; l0 < h.loops; l0 += kUnroll) {
        uint32_t code[kUnroll], sc[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int pair = w.pair + (l0 + u) * h.per;
            const bool on = l0 + u < h.loops && pair < 2 * c.heads;
            const int64_t base = c.rows_before(r.layer + (int)blockIdx.y, (int)p.page, 0, 0) +
                                 ((int64_t)(on ? pair : 0) << c.lg_page);
            code[u] = *(const uint32_t*)(c.codes + (base + p.slot) * (D / 2) + vec * 4);
            sc[u] = c.scales[base * (D / kKvBlock) + (vec / 4 << c.lg_page) + p.slot];
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int pair = w.pair + (l0 + u) * h.per;
            if (l0 + u >= h.loops || pair >= 2 * c.heads) continue;
            const uint32_t x = p.page_ok ? code[u] : 0u;      // no page: zeros
            const float unit = __builtin_bit_cast(float, (p.page_ok ? sc[u] : 0u) << 23);
            const f32x2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, unit, 0);
            const f32x2 a1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, unit, 1);
            const f32x2 a2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, unit, 2);
            const f32x2 a3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, unit, 3);
            const float y[8] = {a0.x, a0.y, a1.x, a1.y, a2.x, a2.y, a3.x, a3.y};
            const bool v = pair >= c.heads;
            store8<DT>(v ? r.v : r.k, to + (int64_t)(pair - (v ? c.heads : 0)) * D, y);
        }
    }
}

Shape shape_of(const KvCache& c, const KvBatch& b, int n_layers) {
    const int rows = kThreads / (c.d / 8);
    Shape s;
    s.lg = 0;
    while ((1 << s.lg) < b.max_rows && (1 << s.lg) < rows) ++s.lg;
    s.tiles = (b.max_rows + (1 << s.lg) - 1) >> s.lg;
    s.per = rows >> s.lg;
    const int pairs = (2 * c.heads + s.per - 1) / s.per;
    // Workgroups take several pairs, so that a token's place is found once for
    // them, while there are enough workgroups for the device.
    const int64_t all = (int64_t)s.tiles * pairs * b.n * n_layers, enough = 4 * device_cus();
    s.loops = 1;
    while (s.loops < pairs && s.loops < 16 && all / (2 * s.loops) >= enough) s.loops *= 2;
    s.groups = (pairs + s.loops - 1) / s.loops;
    return s;
}

template <bool WRITE, int D>
hipError_t launch_d(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    const Shape h = shape_of(c, b, r.n_layers);
    const dim3 grid((unsigned)(h.blocks() * b.n), (unsigned)r.n_layers);
#define SENSE_KV_ROWS(T)                                                                      \
    if constexpr (WRITE)                                                                      \
        hipLaunchKernelGGL((kv_write_kernel<D, T>), grid, dim3(kThreads), 0, st, c, b, r, h); \
    else                                                                                      \
        hipLaunchKernelGGL((kv_read_kernel<D, T>), grid, dim3(kThreads), 0, st, c, b, r, h)
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
    const Shape s = shape_of(c, b, 1);
    return (int64_t)s.tiles * ((2 * c.heads + s.per - 1) / s.per) * b.n;
}
hipError_t launch_kv_write(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    return launch_rows<true>(c, b, r, st);
}
hipError_t launch_kv_read(const KvCache& c, const KvBatch& b, const KvRows& r, hipStream_t st) {
    return launch_rows<false>(c, b, r, st);
}

}  // namespace sense
