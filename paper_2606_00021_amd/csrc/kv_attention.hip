// Attention of new tokens over the 4-bit paged cache.
//
//   o_j = sum_p w_jp v_p / sum_p w_jp,  w_jp = exp(scale q_j . k_p) over the
//   positions p that row j sees
//
// in one pass over the cache: the running maximum m and the sums of
// exp(s - m) and exp(s - m) v are kept in fp32, rescaled only when a score
// passes m by more than 2^8 (see kSlack).
//
// A unit is the rows of one entry that share a key head: new tokens times
// query heads per key head, in tiles of 16 MT rows.  A unit's keys are cut
// into runs of C keys; an item is one tile over one run, and a workgroup has
// one item, its four waves taking steps of 32 keys in turn.  C is computed on
// the device from the lengths themselves (plan()), so that about `target`
// workgroups share the work whatever the lengths are; runs of one unit are
// joined by a second kernel.
//
// Both products run on the matrix cores, transposed:
//   S^T = K Q^T   A = K (16 keys x 32 dims), B = Q^T (32 dims x 16 rows)
//   O^T = V^T P^T A = V^T (16 dims x 32 keys), B = P^T (32 keys x 16 rows)
// In both results a lane holds one row (lane & 15), so softmax statistics stay
// in the lane, and the scores of two key tiles are, as they lie, the B operand
// of the second product.  Contractions may take dims and keys in any order:
//   - lane group g = lane >> 4 takes dims [g d/4, (g+1) d/4) of a key, d/8
//     bytes in one load, the tiles' key rows being 8 (m >> 2) + 4 t + (m & 3);
//   - in the second product lane (m, g) has keys 8g .. 8g+7 and dims
//     [m d/16, (m+1) d/16): whole bytes of codes, of one scale a key.  Codes
//     of two keys are widened by v_cvt_scalef32_pk and exchanged in pairs by
//     v_perm, so nothing passes through LDS.
// 4-bit values times their scales are exact in bf16, and in f16 where they lie
// in its range.  Probabilities are rounded to the query's type (nearest);
// their sum is taken of the rounded ones, by a product with ones, so that the
// weights that are used add up to 1.
#include "internal.h"
#include "kv.h"

namespace sense {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kStep = 32;              // keys of a wave's step
constexpr int kTile = kStep * kWaves;  // keys of a workgroup's step
constexpr float kSlack = 8.f;          // scores may pass the reference by 2^8
// A unit is not cut below this many keys: a shorter run costs more in joining
// than its parallelism gains.
constexpr int kMinRun = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct Args {
    KvCache c;
    KvBatch b;
    KvAttention a;
    int group;          // query heads per key head
    int target;         // workgroups that the work is cut for (0: units stay whole)
    float* part_o;      // [item][rows][d]
    f32x2* part_ml;     // [item][rows]: reference, sum
};

// Where one unit tile's items lie, and which keys one of them has.
struct Plan {
    int item;           // this workgroup's item
    int entry, seq;     // entry of the item (-1: none)
    int rows, len;      // new tokens of the entry, cached positions
    int first;          // first item of the entry
    int splits;         // runs of a unit of the entry
    int run;            // tiles of kTile keys in a run
};

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor((long long)v, s);
    return v;
}

// The items of the entries, in order, computed by every wave for itself from
// the entries' lengths.  entry < 0: the entry that this workgroup's item
// belongs to; else that entry.  Items go to the XCDs in runs (workgroups are
// dealt to the 8 XCDs in turn): tiles of one unit, which read the same keys,
// then share an L2.
template <int ROWS>
__device__ __forceinline__ Plan plan(const Args& g, int entry) {
    const int lane = threadIdx.x & 63;
    const int n = g.b.n, per = (n + 63) / 64;
    const int e0 = lane * per < n ? lane * per : n;
    const int e1 = e0 + per < n ? e0 + per : n;
    int64_t work = 0;
    for (int e = e0; e < e1; ++e) {
        const int s = kv_seq(g.c, g.b.seqs, e);
        if (s < 0) continue;
        const int m = kv_rows(g.b, e);
        const int units = (m * g.group + ROWS - 1) / ROWS;
        work += (int64_t)units * ((kv_length(g.c, s) + kTile - 1) / kTile);
    }
    work = wave_sum64(work) * g.c.heads;
    int64_t run64 = g.target ? (work + g.target - 1) / g.target : 1 << 24;
    if (run64 < kMinRun / kTile) run64 = kMinRun / kTile;
    Plan p;
    p.run = (int)(run64 < (1 << 24) ? run64 : (1 << 24));
    int mine = 0;
    for (int e = e0; e < e1; ++e) {
        const int s = kv_seq(g.c, g.b.seqs, e);
        if (s < 0) continue;
        const int units = (kv_rows(g.b, e) * g.group + ROWS - 1) / ROWS;
        const int tiles = (kv_length(g.c, s) + kTile - 1) / kTile;
        const int splits = tiles > p.run ? (tiles + p.run - 1) / p.run : 1;
        mine += units * splits * g.c.heads;
    }
    int upto = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_up(upto, s);
        if (lane >= s) upto += o;
    }
    const int total = __shfl(upto, 63), share = (total + 7) >> 3;
    const int idx = (int)(blockIdx.x >> 3);
    const int item = idx < share ? (int)(blockIdx.x & 7) * share + idx : total;
    p.item = item;
    const bool owner = entry < 0 ? (item >= upto - mine && item < upto)
                                 : (entry >= e0 && entry < e1);
    const uint64_t who = __ballot(owner);
    p.entry = -1;
    p.seq = -1;
    p.rows = p.len = p.first = 0;
    p.splits = 1;
    if (!who) return p;
    const int src = __builtin_ctzll(who);
    // Walked by every lane alike: the owner's chunk.
    int at = __shfl(upto - mine, src);
    const int c0 = __shfl(e0, src), c1 = __shfl(e1, src);
    for (int e = c0; e < c1; ++e) {
        const int s = kv_seq(g.c, g.b.seqs, e);
        if (s < 0) continue;
        const int m = kv_rows(g.b, e);
        const int units = (m * g.group + ROWS - 1) / ROWS;
        const int len = kv_length(g.c, s);
        const int tiles = (len + kTile - 1) / kTile;
        const int splits = tiles > p.run ? (tiles + p.run - 1) / p.run : 1;
        const int mine_e = units * splits * g.c.heads;
        if (entry < 0 ? item < at + mine_e : e == entry) {
            p.entry = __builtin_amdgcn_readfirstlane(e);
            p.seq = __builtin_amdgcn_readfirstlane(s);
            p.rows = __builtin_amdgcn_readfirstlane(m);
            p.len = __builtin_amdgcn_readfirstlane(len);
            p.first = __builtin_amdgcn_readfirstlane(at);
            p.splits = __builtin_amdgcn_readfirstlane(splits);
            break;
        }
        at += mine_e;
    }
    return p;
}

template <bool F16>
__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Two codes (byte SEL of w) times 2^(exponent of unit), as a pair of 16 bits.
template <bool F16, int SEL>
__device__ __forceinline__ uint32_t widen(uint32_t w, float unit) {
    if constexpr (F16)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, SEL));
    else
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, SEL));
}
template <bool F16>
__device__ __forceinline__ u32x4 widen8(uint32_t w, float unit) {
    u32x4 r;
    r[0] = widen<F16, 0>(w, unit);
    r[1] = widen<F16, 1>(w, unit);
    r[2] = widen<F16, 2>(w, unit);
    r[3] = widen<F16, 3>(w, unit);
    return r;
}
template <bool F16>
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const f32x2 v = {a, b};
    if constexpr (F16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ float unit_of(uint32_t byte) {
    return __builtin_bit_cast(float, byte << 23);
}

// One step's codes and scales of a lane.
template <int D>
struct Step {
    uint32_t k[2][D / 32];              // d/8 bytes of a key, per key tile
    uint32_t ks[2];                     // its scales: one byte, two of 256 dims
    uint32_t v[8 * D / 128 + (D == 64 ? 4 : 0)];   // d/32 bytes of each of 8 keys
    uint32_t vs[2];                     // 8 scale bytes
    int bad;                            // halves of the step without a page
};

template <int D, bool F16, int MT>
__global__ __launch_bounds__(kThreads) void kv_attention_kernel(Args g) {
    constexpr int kRows = 16 * MT;
    constexpr int kKs = D / 32;         // matrix steps of the first product
    constexpr int DV = D / 16;          // dims of a lane in the second
    constexpr int kPad = D + 4;
    __shared__ float s_o[kWaves][kRows][kPad];
    __shared__ float s_m[kWaves][kRows];
    __shared__ float s_l[kWaves][kRows];

    const Plan p = plan<kRows>(g, -1);
    if (p.entry < 0) return;
    const int item = p.item;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int n_tiles = (p.rows * g.group + kRows - 1) / kRows;
    const int local = item - p.first;
    const int rt = local % n_tiles;
    const int head = (local / n_tiles) % g.c.heads;
    const int split = local / n_tiles / g.c.heads;
    const int r0 = rt * kRows;
    const int base = p.len - p.rows;            // position of the first new token
    const int64_t start = kv_start(g.b, p.entry);

    // Rows of the lane's column: token and whether it exists.
    int tok[MT];
    int64_t qrow[MT];
    u32x4 qf[MT][kKs];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = r0 + mt * 16 + col;
        tok[mt] = r / g.group;
        const int64_t row = start + tok[mt];
        const bool on = tok[mt] < p.rows && row >= 0 && row < g.b.n_rows;
        qrow[mt] = on ? row : -1;
        const u32x4* src = (const u32x4*)((const uint16_t*)g.a.q + (on ? row : 0) * g.a.q_stride +
                                          ((int64_t)head * g.group + r % g.group) * D +
                                          grp * (D / 4));
#pragma unroll
        for (int s = 0; s < kKs; ++s) qf[mt][s] = on ? src[s] : u32x4{0, 0, 0, 0};
    }

    // Keys of the item.  Up to `full` every row sees every key.
    int key0 = split * p.run * kTile;
    int key1 = p.splits == 1 ? p.len : key0 + p.run * kTile;
    if (key1 > p.len) key1 = p.len;
    int full = base;
    if (!g.a.mask) {
        const int last = (r0 + kRows - 1) / g.group;
        const int seen = base + (last < p.rows ? last : p.rows - 1) + 1;
        if (key1 > seen) key1 = seen;
        full = base + r0 / g.group + 1;
    }

    f32x4 o[DV][MT];
    f32x4 lsum[MT];
    float ref[MT], neg[MT];             // reference of the exponents, and its negative or 0
    constexpr float kLift = F16 ? 7.f : 0.f;    // f16: probabilities up to 2^15, not 2^8
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int t = 0; t < DV; ++t) o[t][mt] = f32x4{0, 0, 0, 0};
        lsum[mt] = f32x4{0, 0, 0, 0};
        ref[mt] = -INFINITY;
        neg[mt] = kLift;
    }
    const float cs = g.a.scale * 1.4426950408889634f;
    const uint32_t one = F16 ? 0x3C003C00u : 0x3F803F80u;
    const u32x4 ones = {one, one, one, one};

    const int32_t* table = g.c.page_table + (int64_t)p.seq * g.c.max_pages;
    const int lg = g.c.lg_page, slot_mask = g.c.page() - 1;
    const int64_t page_rows = (int64_t)2 * g.c.heads << lg;
    const int64_t k_rows = g.c.rows_before(g.a.layer, 0, 0, head);
    const int64_t v_rows = g.c.rows_before(g.a.layer, 0, 1, head);

    auto load = [&](Step<D>& f, int key) {
        // Pages of the step's halves (one page where pages hold 32 or more).
        int id0 = table[key >> lg];
        int id1 = key + 16 < p.len ? table[(key + 16) >> lg] : -1;
        f.bad = (kv_page_ok(g.c, id0) ? 0 : 1) | (kv_page_ok(g.c, id1) ? 0 : 2);
        id0 = f.bad & 1 ? 0 : id0;
        id1 = f.bad & 2 ? 0 : id1;
        const int kin = 8 * (col >> 2) + (col & 3);         // + 4 t
        const int64_t kpage = (kin >= 16 ? id1 : id0) * page_rows + k_rows;
        const int kslot = (key + kin) & slot_mask;
        const uint8_t* kc = g.c.codes + (kpage + kslot) * (D / 2) + grp * (D / 8);
        const uint8_t* ksc = g.c.scales + kpage * (D / 32) + kslot;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* at = kc + t * 4 * (D / 2);
#pragma unroll
            for (int w = 0; w < D / 32; ++w) f.k[t][w] = ((const uint32_t*)at)[w];
            if constexpr (D == 256) {
                f.ks[t] = ksc[4 * t + ((2 * grp) << lg)] | ksc[4 * t + ((2 * grp + 1) << lg)] << 8;
            } else {
                f.ks[t] = ksc[4 * t + ((D == 64 ? grp >> 1 : grp) << lg)];
            }
        }
        const int64_t vpage = (grp >= 2 ? id1 : id0) * page_rows + v_rows;
        const int vslot = (key + 8 * grp) & slot_mask;
        const uint8_t* vc = g.c.codes + (vpage + vslot) * (D / 2) + col * (D / 32);
        const uint32_t* vsc = (const uint32_t*)(g.c.scales + vpage * (D / 32) + vslot +
                                                (((col * DV) / 32) << lg));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (D == 64) {
                f.v[i] = *(const uint16_t*)(vc + i * (D / 2));
            } else {
#pragma unroll
                for (int w = 0; w < D / 128; ++w)
                    f.v[i * (D / 128) + w] = ((const uint32_t*)(vc + i * (D / 2)))[w];
            }
        }
        f.vs[0] = vsc[0];
        f.vs[1] = vsc[1];
    };

    auto compute = [&](Step<D>& f, int key) {
        // S^T: two tiles of 16 keys.
        u32x4 kf[2][kKs];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < kKs; ++s)
                kf[t][s] = widen8<F16>(
                    f.k[t][s], unit_of(D == 256 ? (f.ks[t] >> (s >= 4 ? 8 : 0)) & 0xFFu : f.ks[t]));
        const bool plain = key + kStep <= full && f.bad == 0;
        uint32_t vis[MT];               // bit 4t + r: the row sees the key (masked steps)
        u32x4 pf[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            f32x4 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < kKs; ++q) s[t] = mfma<F16>(kf[t][q], qf[mt][q], s[t]);
            }
            if (!plain) {
                uint32_t bits = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int pos = key + 8 * grp + e;
                    bool see = pos < key1 && !(f.bad & (grp >= 2 ? 2 : 1));
                    const int u = pos - base;
                    if (!g.a.mask) {
                        see = see && u <= tok[mt];
                    } else if (see && u >= 0) {
                        see = tok[mt] < p.rows &&
                              g.a.mask[p.entry * g.a.mask_stride + tok[mt] * g.a.mask_ld + u] != 0;
                    }
                    bits |= (uint32_t)see << e;
                    if (!see) s[e >> 2][e & 3] = -INFINITY;
                }
                vis[mt] = bits;
            }
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                              fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) *
                        cs;
            if (__any(top > ref[mt] + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = fmaxf(ref[mt], top);
                const float keep = now == -INFINITY ? 1.f : exp2f(ref[mt] - now);
                ref[mt] = now;
                neg[mt] = now == -INFINITY ? kLift : kLift - now;
#pragma unroll
                for (int t = 0; t < DV; ++t) o[t][mt] *= keep;
                lsum[mt] *= keep;
            }
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                e[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], cs, neg[mt]));
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[mt][i] = pack<F16>(e[2 * i], e[2 * i + 1]);
            lsum[mt] = mfma<F16>(ones, pf[mt], lsum[mt]);
        }
        // V^T: dims DV m + t of the lane's 8 keys.
        float unit[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) unit[i] = unit_of((f.vs[i >> 2] >> (8 * (i & 3))) & 0xFFu);
        if (!plain) {
            // A key that a row does not see leaves it alone even where its
            // value is NaN: such values count as 0 in the product, and the
            // rows that do see them become NaN by a product of indicators.
            u32x4 nan = {0, 0, 0, 0};
            bool some = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool here = __builtin_bit_cast(uint32_t, unit[i]) == 0x7F800000u;
                some |= here;
                nan[i >> 1] |= here ? (i & 1 ? one & 0xFFFF0000u : one & 0xFFFFu) : 0u;
                unit[i] = here ? 0.f : unit[i];
            }
            if (__any(some)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    u32x4 seen;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        seen[i] = ((vis[mt] >> (2 * i)) & 1 ? one & 0xFFFFu : 0u) |
                                  ((vis[mt] >> (2 * i + 1)) & 1 ? one & 0xFFFF0000u : 0u);
                    const f32x4 hit = mfma<F16>(nan, seen, f32x4{0, 0, 0, 0});
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int t = 0; t < DV; ++t)
                            if (hit[r] > 0.f) o[t][mt][r] = NAN;
                }
            }
        }
#pragma unroll
        for (int w = 0; w < (D == 256 ? 2 : 1); ++w) {
#pragma unroll
            for (int by = 0; by < (D == 64 ? 2 : 4); ++by) {
                uint32_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t word = f.v[D == 256 ? 2 * i + w : i];
                    x[i] = by == 0   ? widen<F16, 0>(word, unit[i])
                           : by == 1 ? widen<F16, 1>(word, unit[i])
                           : by == 2 ? widen<F16, 2>(word, unit[i])
                                     : widen<F16, 3>(word, unit[i]);
                }
                u32x4 lo, hi;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
                    hi[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
                }
                const int t = 8 * w + 2 * by;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    o[t][mt] = mfma<F16>(lo, pf[mt], o[t][mt]);
                    o[t + 1][mt] = mfma<F16>(hi, pf[mt], o[t + 1][mt]);
                }
            }
        }
    };

    int key = key0 + wave * kStep;
    if (key < key1) {
        Step<D> cur, nxt;
        load(cur, key);
        for (;;) {
            const int ahead = key + kTile;
            if (ahead < key1) load(nxt, ahead);
            compute(cur, key);
            if (ahead >= key1) break;
            cur = nxt;
            key = ahead;
        }
    }

    // The waves' sums to a common reference.
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = mt * 16 + col;
        if (grp == 0) {
            s_m[wave][r] = ref[mt];
            s_l[wave][r] = lsum[mt][0];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int t = 0; t < DV; t += 4)
                *(f32x4*)&s_o[wave][r][4 * DV * grp + DV * q + t] =
                    f32x4{o[t][mt][q], o[t + 1][mt][q], o[t + 2][mt][q], o[t + 3][mt][q]};
    }
    __syncthreads();
    for (int at = threadIdx.x; at < kRows * (D / 4); at += kThreads) {
        const int r = at / (D / 4), dim = at % (D / 4) * 4;
        const int rr = r0 + r, token = rr / g.group;
        const int64_t row = start + token;
        if (token >= p.rows || row < 0 || row >= g.b.n_rows) continue;
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        float l = 0.f;
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            // A wave that saw no key has sums of 0 (or of NaN scores).
            const float f = s_m[w][r] == -INFINITY ? 1.f : exp2f(s_m[w][r] - top);
            l += s_l[w][r] * f;
            sum += *(const f32x4*)&s_o[w][r][dim] * f;
        }
        if (p.splits == 1) {
            // Nothing seen: 0.  A sum of NaN is not 0.
            const float inv = l == 0.f ? 0.f : 1.f / l;
            uint32_t* dst = (uint32_t*)((uint16_t*)g.a.out + row * g.a.out_stride +
                                        ((int64_t)head * g.group + rr % g.group) * D + dim);
            dst[0] = pack<F16>(sum[0] * inv, sum[1] * inv);
            dst[1] = pack<F16>(sum[2] * inv, sum[3] * inv);
        } else {
            *(f32x4*)(g.part_o + ((int64_t)item * kRows + r) * D + dim) = sum;
            if (dim == 0) g.part_ml[(int64_t)item * kRows + r] = f32x2{top, l};
        }
    }
}

// Joins the runs of a unit: RB rows of a tile for a workgroup, each row's runs
// dealt to 4 / RB' waves.
template <int D, bool F16, int MT, int RB>
__global__ __launch_bounds__(kThreads) void kv_join_kernel(Args g, int tiles_max) {
    constexpr int kRows = 16 * MT;
    constexpr int kLanes = D / 4;                 // threads of a row
    constexpr int kTeams = kThreads / kLanes;     // 16, 8, 4
    __shared__ f32x4 s_o[kTeams][kLanes];
    __shared__ f32x2 s_ml[kTeams];
    const int per_tile = kRows / RB;
    const int sub = blockIdx.x % per_tile;
    const int rt = blockIdx.x / per_tile % tiles_max;
    const int head = blockIdx.x / per_tile / tiles_max % g.c.heads;
    const int entry = blockIdx.x / per_tile / tiles_max / g.c.heads;
    const Plan p = plan<kRows>(g, entry);
    if (p.entry < 0 || p.splits == 1) return;
    const int n_tiles = (p.rows * g.group + kRows - 1) / kRows;
    if (rt >= n_tiles) return;
    const int team = threadIdx.x / kLanes, dim = threadIdx.x % kLanes * 4;
    const int64_t start = kv_start(g.b, p.entry);
    // RB == 1: the teams share a row's runs.  Else a team has rows of its own.
    for (int r = sub * RB + (RB == 1 ? 0 : team); r < (sub + 1) * RB; r += kTeams) {
        const int rr = rt * kRows + r, token = rr / g.group;
        const int64_t row = start + token;
        const bool on = token < p.rows && row >= 0 && row < g.b.n_rows;
        if (RB == 1 && !on) return;               // the whole workgroup
        float top = -INFINITY, l = 0.f;
        f32x4 sum = {0, 0, 0, 0};
        if (on) {
            const int step = RB == 1 ? kTeams : 1;
#pragma unroll 4
            for (int s = RB == 1 ? team : 0; s < p.splits; s += step) {
                const int64_t at =
                    ((int64_t)p.first + (s * g.c.heads + head) * n_tiles + rt) * kRows + r;
                const f32x2 ml = g.part_ml[at];
                const f32x4 x = *(const f32x4*)(g.part_o + at * D + dim);
                const float now = fmaxf(top, ml[0]);
                const float a = top == -INFINITY ? 1.f : exp2f(top - now);
                const float b = ml[0] == -INFINITY ? 1.f : exp2f(ml[0] - now);
                l = l * a + ml[1] * b;
                sum = sum * a + x * b;
                top = now;
            }
        }
        if constexpr (RB == 1) {
            s_o[team][threadIdx.x % kLanes] = sum;
            if (dim == 0) s_ml[team] = f32x2{top, l};
            __syncthreads();
            if (team != 0) return;
            for (int t = 1; t < kTeams; ++t) {
                const float now = fmaxf(top, s_ml[t][0]);
                const float a = top == -INFINITY ? 1.f : exp2f(top - now);
                const float b = s_ml[t][0] == -INFINITY ? 1.f : exp2f(s_ml[t][0] - now);
                l = l * a + s_ml[t][1] * b;
                sum = sum * a + s_o[t][threadIdx.x % kLanes] * b;
                top = now;
            }
        }
        if (on) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            uint32_t* dst = (uint32_t*)((uint16_t*)g.a.out + row * g.a.out_stride +
                                        ((int64_t)head * g.group + rr % g.group) * D + dim);
            dst[0] = pack<F16>(sum[0] * inv, sum[1] * inv);
            dst[1] = pack<F16>(sum[2] * inv, sum[3] * inv);
        }
    }
}

// Row tiles of a wave: as many as the rows of a unit fill, up to 64 rows (32
// of 256 dims, whose sums take twice the registers).  A tile of more rows
// widens each key and value once for all of them.
int row_tiles(int max_rows, int group, int d) {
    const int64_t rows = (int64_t)max_rows * group;
    const int most = d == 256 ? 2 : 4;
    const int mt = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    return mt < most ? mt : most;
}

// Workgroups to cut the work for: what is resident at once.
int target_items(int mt) { return device_cus() * (mt == 1 ? 4 : (mt == 2 ? 2 : 1)); }

int64_t units_most(int n, int max_rows, int n_heads, int kv_heads, int mt) {
    const int64_t tiles = ((int64_t)max_rows * (n_heads / kv_heads) + 16 * mt - 1) / (16 * mt);
    return tiles * kv_heads * n;
}

template <int D, bool F16, int MT>
hipError_t launch_mt(const Args& g, hipStream_t st) {
    const int64_t units = units_most(g.b.n, g.b.max_rows, g.a.n_heads, g.c.heads, MT);
    // ceil(total / 8) workgroups for each XCD; total <= target + units.
    const int64_t most = units + g.target;
    hipLaunchKernelGGL((kv_attention_kernel<D, F16, MT>), dim3((unsigned)((most + 7) / 8 * 8)),
                       dim3(kThreads), 0, st, g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !g.target) return e;
    const int tiles = (int)(units / g.c.heads / g.b.n);
    const int64_t rows = (int64_t)g.b.max_rows * g.group;
    if (rows <= 16) {
        hipLaunchKernelGGL((kv_join_kernel<D, F16, MT, 1>), dim3((unsigned)(units * 16 * MT)),
                           dim3(kThreads), 0, st, g, tiles);
    } else {
        hipLaunchKernelGGL((kv_join_kernel<D, F16, MT, 16>), dim3((unsigned)(units * MT)),
                           dim3(kThreads), 0, st, g, tiles);
    }
    return hipGetLastError();
}

template <int D, bool F16>
hipError_t launch_d(Args& g, int mt, hipStream_t st) {
    if (mt == 1) return launch_mt<D, F16, 1>(g, st);
    if (mt == 2) return launch_mt<D, F16, 2>(g, st);
    if constexpr (D != 256) return launch_mt<D, F16, 4>(g, st);
    return hipErrorInvalidValue;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t kv_attention_blocks(int n, int max_rows, int n_heads, int kv_heads, int d) {
    const int mt = row_tiles(max_rows, n_heads / kv_heads, d);
    const int64_t units = units_most(n, max_rows, n_heads, kv_heads, mt);
    // Of the attention itself, and of the join (a workgroup for 1 or 16 rows).
    return units * ((int64_t)max_rows * (n_heads / kv_heads) <= 16 ? 16 * mt : mt) +
           target_items(mt);
}

size_t kv_attention_workspace_bytes(int n, int max_rows, int n_heads, int kv_heads, int d,
                                    int max_kv) {
    if (max_kv <= kMinRun) return 0;
    const int mt = row_tiles(max_rows, n_heads / kv_heads, d);
    const int64_t items = units_most(n, max_rows, n_heads, kv_heads, mt) + target_items(mt);
    const size_t rows = (size_t)items * 16 * mt;
    return align256(rows * d * sizeof(float)) + align256(rows * sizeof(f32x2));
}

hipError_t launch_kv_attention(const KvCache& c, const KvBatch& b, const KvAttention& a,
                               void* workspace, hipStream_t st) {
    Args g;
    g.c = c;
    g.b = b;
    g.a = a;
    g.group = a.n_heads / c.heads;
    const int mt = row_tiles(b.max_rows, g.group, c.d);
    g.target = a.max_kv > kMinRun ? target_items(mt) : 0;
    const int64_t items = units_most(b.n, b.max_rows, a.n_heads, c.heads, mt) + g.target;
    g.part_o = (float*)workspace;
    g.part_ml = (f32x2*)((char*)workspace +
                         align256((size_t)items * 16 * mt * c.d * sizeof(float)));
    const bool f16 = a.dtype == DT_F16;
    if (c.d == 64) return f16 ? launch_d<64, true>(g, mt, st) : launch_d<64, false>(g, mt, st);
    if (c.d == 128) return f16 ? launch_d<128, true>(g, mt, st) : launch_d<128, false>(g, mt, st);
    return f16 ? launch_d<256, true>(g, mt, st) : launch_d<256, false>(g, mt, st);
}

}  // namespace sense
