// Attention of new tokens over the 4-bit paged cache.
//
//   o_j = sum_p w_jp v_p / sum_p w_jp,  w_jp = exp(scale q_j . k_p) over the
//   positions p that row j sees
//
// in one pass over the cache: the running maximum m and the sums of
// exp(s - m) and exp(s - m) v are kept in fp32, rescaled only when a weight
// passes 2^8.
//
// The rows of one entry that share a key head (new tokens times query heads
// per key head) are cut into tiles; a unit is one tile.  A unit's keys are cut
// into runs, an item is a unit over one run, and a workgroup has one item.
// The length of a run is computed on the device from the sequences' lengths
// (plan()), so that about `target` workgroups share the work whatever the
// lengths are; a second kernel joins the runs of a unit.  Up to 32 rows the
// four waves of a workgroup have the same rows and take steps of 32 keys in
// turn (kv_few_kernel), beyond they have rows of their own and share the keys
// (kv_many_kernel).
//
// Few rows are bound by the bytes of the cache: 64 streams of 8000 positions
// (32 / 8 heads of 128, 558 MB) take 97 to 103 us, 5.4 to 5.8 TB/s, where a plain
// read of as many bytes takes 78 to 80.  Many rows are bound by the matrix and
// vector units (exponentials): two 2048-token chunks, of 2048 and 10000
// positions, 341 us, 984 TFLOP/s, where a large bf16 product of the library
// reaches 1170.
//
// Both products run on the matrix cores, transposed:
//   S^T = K Q^T   A = K (16 keys x 32 dims), B = Q^T (32 dims x 16 rows)
//   O^T = V^T P^T A = V^T (16 dims x 32 keys), B = P^T (32 keys x 16 rows)
// In both results a lane holds one row (lane & 15), so softmax statistics stay
// in the lane, and the scores of two key tiles are, as they lie, the B operand
// of the second product.  Contractions may take dims and keys in any order:
//   - lane group g = lane >> 4 takes dims [g d/4, (g+1) d/4) of a key, d/8
//     bytes in one load;
//   - in the second product lane (m, g) has keys 4g .. 4g+3 of both key tiles
//     and dims [m d/16, (m+1) d/16): whole bytes of codes, of one scale a key.
//     Codes of two keys are widened by v_cvt_scalef32_pk and exchanged in
//     pairs by v_perm.
// A key tile lies in one page, so every load has a base that is the same for
// the wave and an offset that is the same for all steps.
// 4-bit values times their scales are exact in bf16, and in f16 where they lie
// in its range.  Weights of entries of up to 64 rows enter as the sum of two
// numbers of 16 bits, so that only the result is rounded.  Of larger ones, which
// the matrix units bound, they are rounded once (nearest), to f16 whatever the
// query's type: 11 bits, so a bf16 result is off by its own rounding and 1 % more
// (weights of 8 bits: 40 %), an f16 one by 40 % more.  Values then enter in f16;
// the few that it does not hold in bf16 beside it (kv_many_kernel).  The weights'
// sum is taken of what enters, by a product with ones, so that the weights that
// are used add up to 1.
#include <type_traits>

#include "internal.h"
#include "kv.h"

namespace sense {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kStep = 32;              // keys of a wave's step
constexpr int kTile = kStep * kWaves;  // keys of a workgroup's step
// A unit is not cut into runs of fewer keys (one token over 2000 positions, 8
// key heads: 10.4 us with 256, 11.5 with 512, 14.1 with 1024; 16 of them 17.9,
// 16.8, 17.2), nor at all where no sequence is longer than kWhole, which saves
// the second launch (500 positions 7.5 us whole, 10.0 cut; 1000 the same;
// 2000 15.8 and 10.4).
constexpr int kMinRun = 256;
constexpr int kWhole = 1024;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The page table is not written while these kernels run: scalar loads.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

constexpr int kTries = 3;              // run lengths tried

struct Args {
    KvCache c;
    KvBatch b;
    KvAttention a;
    int group;          // query heads per key head
    int target;         // workgroups that the work is cut for (0: units stay whole)
    float* part_o;      // [item of a cut unit][rows][d]
    f32x2* part_ml;     // [the same][rows]: reference (a score), sum
    i32x4* plans;       // [entry]: new tokens, first item, runs of a unit, first cut item
};

// Where one unit tile's items lie, and which keys one of them has.
struct Plan {
    int item;           // this workgroup's item
    int entry, seq;     // entry of the item (-1: none)
    int rows, len;      // new tokens of the entry, cached positions
    int first;          // first item of the entry
    int part;           // the item's place among those of cut units
    int splits;         // runs of a unit of the entry
    int run;            // tiles of kTile keys in a run
};

// Inclusive prefix sums over a wave, in registers.
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // row_bcast:15
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);     // row_bcast:31
    return v;
}
__device__ __forceinline__ int wave_total(int v) {
    return __builtin_amdgcn_readlane(wave_scan(v), 63);
}

// An entry's tiles of rows (of one head) and of keys.
struct Size {
    int seq, rows, len, units, tiles;
};
template <int ROWS>
__device__ __forceinline__ Size size_of(const Args& g, int e) {
    Size z = {kv_seq(g.c, g.b.seqs, e), 0, 0, 0, 0};
    if (z.seq < 0) return z;
    z.rows = kv_rows(g.b, e);
    z.len = kv_length(g.c, z.seq);
    z.units = (z.rows * g.group + ROWS - 1) / ROWS;
    z.tiles = (z.len + kTile - 1) / kTile;
    return z;
}
__device__ __forceinline__ int splits_of(int tiles, int run) {
    return tiles > run ? (int)((unsigned)(tiles + run - 1) / (unsigned)run) : 1;
}
__device__ __forceinline__ int64_t divide(int64_t a, int b) {
    return a >> 31 ? a / b : (int64_t)((unsigned)a / (unsigned)b);
}

// The items of up to 64 entries, in order, computed by every wave for itself
// from the entries' lengths, a lane an entry.  The first workgroup leaves them
// for the join.
template <int ROWS>
__device__ __forceinline__ Plan plan_few(const Args& g) {
    const int lane = threadIdx.x & 63;
    Size z0 = {-1, 0, 0, 0, 0};
    if (lane < g.b.n) z0 = size_of<ROWS>(g, lane);
    const int64_t work = (int64_t)z0.units * z0.tiles;
    const int units = z0.units;
    // Fewer than 2^24 units of fewer than 2^24 tiles: two sums of 31 bits.
    const int64_t all = ((int64_t)wave_total((int)(work >> 20)) << 20) +
                        wave_total((int)(work & 0xFFFFF));
    const int64_t whole = (int64_t)wave_total(units) * g.c.heads;
    int64_t run64 = g.target ? divide(all * g.c.heads + g.target - 1, g.target) : 1 << 24;
    if (run64 < kMinRun / kTile) run64 = kMinRun / kTile;
    int run = __builtin_amdgcn_readfirstlane((int)(run64 < (1 << 24) ? run64 : (1 << 24)));
    // Items of the lane's entry with runs of that length.  Rounding up makes
    // more of them than `target`, and the last few would have the device to
    // themselves: the runs are made longer until they fit (or units are whole).
    int mine, upto;
    for (int tries = 0;; ++tries) {
        mine = z0.units * splits_of(z0.tiles, run) * g.c.heads;
        upto = wave_scan(mine);
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (total <= g.target || whole >= g.target || tries == kTries) break;
        const int longer = (int)divide((int64_t)run * total, g.target);
        run = __builtin_amdgcn_readfirstlane(longer > run ? longer : run + 1);
    }
    const int cut = splits_of(z0.tiles, run) > 1 ? mine : 0, cut_first = wave_scan(cut) - cut;
    if (g.target && blockIdx.x == 0 && threadIdx.x < g.b.n)
        g.plans[threadIdx.x] =
            i32x4{z0.rows, upto - mine, splits_of(z0.tiles, run), cut_first};
    Plan p;
    p.item = (int)blockIdx.x;
    p.entry = -1;
    const uint64_t who = __ballot(p.item >= upto - mine && p.item < upto);
    if (!who) return p;
    const int src = __builtin_ctzll(who);
    p.entry = src;
    p.seq = __builtin_amdgcn_readlane(z0.seq, src);
    p.rows = __builtin_amdgcn_readlane(z0.rows, src);
    p.len = __builtin_amdgcn_readlane(z0.len, src);
    p.first = __builtin_amdgcn_readlane(upto - mine, src);
    p.part = __builtin_amdgcn_readlane(cut_first, src) + p.item - p.first;
    p.run = run;
    p.splits = __builtin_amdgcn_readfirstlane(
        splits_of(__builtin_amdgcn_readlane(z0.tiles, src), run));
    return p;
}

// The same for more entries, by one workgroup in front of the attention.
template <int ROWS>
__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(Args g) {
    __shared__ int64_t s_wave[kPlanThreads / 64];
    int64_t work = 0, units = 0, all, whole;
    for (int e = threadIdx.x; e < g.b.n; e += kPlanThreads) {
        const Size z = size_of<ROWS>(g, e);
        work += (int64_t)z.units * z.tiles;
        units += z.units;
    }
    block_scan(work, s_wave, &all);
    block_scan(units, s_wave, &whole);
    whole *= g.c.heads;
    int64_t run64 = g.target ? divide(all * g.c.heads + g.target - 1, g.target) : 1 << 24;
    if (run64 < kMinRun / kTile) run64 = kMinRun / kTile;
    int run = (int)(run64 < (1 << 24) ? run64 : (1 << 24));
    for (int tries = 0; whole < g.target && tries < kTries; ++tries) {
        int64_t mine = 0, total;
        for (int e = threadIdx.x; e < g.b.n; e += kPlanThreads) {
            const Size z = size_of<ROWS>(g, e);
            mine += z.units * splits_of(z.tiles, run);
        }
        block_scan(mine, s_wave, &total);
        total *= g.c.heads;
        if (total <= g.target) break;
        const int longer = (int)divide((int64_t)run * total, g.target);
        run = longer > run ? longer : run + 1;
    }
    // Items, and in the high half those of cut units: fewer than 2^25 of either.
    int64_t at = 0;
    for (int e0 = 0; e0 < g.b.n; e0 += kPlanThreads) {
        const int e = e0 + threadIdx.x;
        Size z = {-1, 0, 0, 0, 0};
        if (e < g.b.n) z = size_of<ROWS>(g, e);
        const int splits = splits_of(z.tiles, run);
        const int64_t items = (int64_t)z.units * splits * g.c.heads;
        const int64_t mine = items + (splits > 1 ? items << 32 : 0);
        int64_t total;
        const int64_t first = at + block_scan(mine, s_wave, &total) - mine;
        if (e < g.b.n) g.plans[e] = i32x4{z.rows, (int)first, splits, (int)(first >> 32)};
        at += total;
    }
    if (threadIdx.x == 0) g.plans[g.b.n] = i32x4{0, (int)at, 1, run};
}

// This workgroup's item in that plan: the last entry whose first item is not
// behind it (entries without items share theirs with the next), 64 at a time.
template <int ROWS>
__device__ __forceinline__ Plan plan_many(const Args& g) {
    const int lane = threadIdx.x & 63;
    Plan p;
    p.item = (int)blockIdx.x;
    p.entry = -1;
    int from = 0, to = g.b.n + 1;               // the one behind the last holds the total
    while (to - from > 1) {
        const int step = (to - from + 63) / 64;
        const int e = from + lane * step;
        const uint64_t not_behind = __ballot(e < to && g.plans[e < to ? e : from][1] <= p.item);
        // The first is never behind: bit 0 is set.
        const int last = 63 - __builtin_clzll(not_behind);
        to = from + (last + 1) * step < to ? from + (last + 1) * step : to;
        from = from + last * step;
    }
    if (from == g.b.n) return p;
    const Size z = size_of<ROWS>(g, from);
    p.entry = from;
    p.seq = __builtin_amdgcn_readfirstlane(z.seq);
    p.rows = __builtin_amdgcn_readfirstlane(z.rows);
    p.len = __builtin_amdgcn_readfirstlane(z.len);
    const i32x4 x = g.plans[from];
    p.first = __builtin_amdgcn_readfirstlane(x[1]);
    p.splits = __builtin_amdgcn_readfirstlane(x[2]);
    p.part = __builtin_amdgcn_readfirstlane(x[3]) + p.item - p.first;
    p.run = __builtin_amdgcn_readfirstlane(g.plans[g.b.n][3]);
    return p;
}

template <int ROWS>
__device__ __forceinline__ Plan plan(const Args& g) {
    return g.b.n <= 64 ? plan_few<ROWS>(g) : plan_many<ROWS>(g);
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

// The two numbers of a pair.
template <bool F16>
__device__ __forceinline__ float low(uint32_t w) {
    if constexpr (F16)
        return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
    else
        return __builtin_bit_cast(float, w << 16);
}
template <bool F16>
__device__ __forceinline__ float high(uint32_t w) {
    if constexpr (F16)
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
    else
        return __builtin_bit_cast(float, w & 0xFFFF0000u);
}

// Whether a weight of the lane's row, in any of its four lanes, is beyond
// `limit`.  A row takes a new reference only then, so that its result does not
// depend on the rows that it shares a wave with.
__device__ __forceinline__ bool row_over(uint32_t most, uint32_t limit) {
    const uint64_t over = __ballot(most > limit);
    return (over | over >> 16 | over >> 32 | over >> 48) >> (threadIdx.x & 15) & 1;
}

// The exponent of the weight of a row's reference, and the bits of the largest
// weight that leaves the reference as it is: f16 weights up to 2^15, not 2^8.
constexpr float lift_of(bool f16) { return f16 ? 7.f : 0.f; }
constexpr uint32_t most_bits(bool f16) { return (uint32_t)(127 + (f16 ? 15 : 8)) << 23; }

// Weights of a row with the reference `now` (a score): 2^(cs s + neg), one fma,
// neg = lift - cs now rounded once.  What neg is off by is a factor of all
// weights of this reference; surplus() is its exponent, which is taken out where
// sums of different references meet.  From cs now = 2^24 on, where it passes 1,
// weights are 2^(cs (s - now) + lift) instead; such rows, and those that have
// seen nothing, have neg infinite in the step, so that each step comes back here.
struct Exponent {
    float sub, add, neg;                // 2^(cs (s - sub) + add); neg for the step
};
__device__ __forceinline__ Exponent exponent(float now, float cs, float lift) {
    const bool none = now == -INFINITY, far = !none && fabsf(now * cs) >= 0x1p24f;
    Exponent x;
    x.sub = far ? now : 0.f;
    x.add = none || far ? lift : fmaf(-now, cs, lift);
    x.neg = none || far ? INFINITY : x.add;
    return x;
}
__device__ __forceinline__ float surplus(float now, float cs, float lift) {
    const bool exact = now == -INFINITY || fabsf(now * cs) >= 0x1p24f;
    return exact ? 0.f : fmaf(now, cs, fmaf(-now, cs, lift)) - lift;
}
// What sums of reference `was` are worth at the reference `now`, `more` the
// difference of their surpluses.  A row that has seen nothing has sums of 0 (or
// of NaN scores).
__device__ __forceinline__ float fade(float was, float now, float cs, float more = 0.f) {
    return was == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fmaf(was - now, cs, more));
}

__device__ __forceinline__ float unit_of(uint32_t byte) {
    return __builtin_bit_cast(float, byte << 23);
}
// The largest unit whose codes are all finite in the type.  A weight of 0 must
// meet a finite value, whatever lies in a position that a row does not see.
template <bool F16>
__device__ __forceinline__ float finite_unit(float unit) {
    return fminf(unit, F16 ? 0x1p13f : 0x1p125f);
}

// Codes of a scale byte that f16 does not hold: units of 2^-23 to 2^13 it does,
// and zeros of any.  (A NaN block has no values.)
template <int N>
__device__ __forceinline__ bool beyond_f16(uint32_t byte, const uint32_t (&codes)[N]) {
    uint32_t some = codes[0];
    if constexpr (N == 2) some |= codes[1];
    return byte - 104u > 36u && byte != 255u && (some & 0x77777777u) != 0;
}

// Which of 4 N positions a row sees: bit 4t + r is position first + 16t + r,
// with `none` the tiles that have no page (bit `stride` t).  A row whose own
// position would be below 0 sees none.  The mask's bytes are read together, from
// places inside it whether they count or not.
template <int N>
__device__ __forceinline__ uint32_t seen_bits(const Args& g, const Plan& p, int token, int first,
                                              int end, uint32_t none, int stride) {
    const int base = p.len - p.rows;
    uint8_t byte[4 * N];
    if (g.a.mask) {
        const int row = token < p.rows ? token : p.rows - 1;
        const uint8_t* m = g.a.mask + p.entry * g.a.mask_stride + row * g.a.mask_ld;
#pragma unroll
        for (int e = 0; e < 4 * N; ++e) {
            const int u = first + 16 * (e >> 2) + (e & 3) - base;
            byte[e] = m[u < 0 ? 0 : (u < p.rows ? u : p.rows - 1)];
        }
    }
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 4 * N; ++e) {
        const int pos = first + 16 * (e >> 2) + (e & 3), u = pos - base;
        bool see = pos < end && !(none >> (stride * (e >> 2)) & 1);
        if (!g.a.mask)
            see = see && u <= token;
        else
            see = see && (u < 0 || (byte[e] != 0 && token < p.rows && base + token >= 0));
        bits |= (uint32_t)see << e;
    }
    return bits;
}

// One step's codes and scales of a lane.
template <int D>
struct Step {
    uint32_t k[2][D / 32];              // d/8 bytes of a key, per key tile
    uint32_t ks[2][D == 256 ? 2 : 1];   // its scale bytes
    uint32_t v[2][4][D == 256 ? 2 : 1]; // d/32 bytes of four keys, per key tile
    uint32_t vs[2];                     // their scale bytes
};

// Pages of a step's two key tiles; bit t of `bad`: tile t has none.
struct Pages {
    int id[2];
    int bad;
};

template <int D, bool F16, int MT>
__global__ __launch_bounds__(kThreads, MT * D > 128 || MT == 2 ? 2 : (D == 128 ? 3 : 4))
    void kv_few_kernel(Args g) {
    constexpr int kRows = 16 * MT;
    constexpr int kKs = D / 32;         // matrix steps of the first product
    constexpr int DV = D / 16;          // dims of a lane in the second
    constexpr int kPad = D + 4;
    __shared__ float s_o[kWaves][kRows][kPad];
    __shared__ float s_m[kWaves][kRows];
    __shared__ float s_l[kWaves][kRows];
    __shared__ float s_more[kWaves][kRows];

    const Plan p = plan<kRows>(g);
    if (p.entry < 0) return;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int local = p.item - p.first;
    const int split = local / g.c.heads, head = local - split * g.c.heads;
    const int base = p.len - p.rows;            // position of the first new token
    const int64_t start = kv_start(g.b, p.entry);

    // Rows of the lane's column: token and whether it exists.
    int tok[MT];
    u32x4 qf[MT][kKs];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = mt * 16 + col;
        tok[mt] = r / g.group;
        const int64_t row = start + tok[mt];
        const bool on = tok[mt] < p.rows && row >= 0 && row < g.b.n_rows;
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
        const int last = (kRows - 1) / g.group;
        const int seen = base + (last < p.rows ? last : p.rows - 1) + 1;
        if (key1 > seen) key1 = seen;
        full = base + 1;
    }

    f32x4 o[DV][MT];
    f32x4 lsum[MT];
    f32x4 hit[MT];                      // NaN values that a row sees, for its dims
    float ref[MT], neg[MT];             // reference of the weights, see exponent()
    constexpr float kLift = lift_of(F16);
    constexpr uint32_t kMostBits = most_bits(F16);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int t = 0; t < DV; ++t) o[t][mt] = f32x4{0, 0, 0, 0};
        lsum[mt] = f32x4{0, 0, 0, 0};
        hit[mt] = f32x4{0, 0, 0, 0};
        ref[mt] = -INFINITY;
        neg[mt] = INFINITY;
    }
    const float cs = g.a.scale * 1.4426950408889634f;
    const uint32_t one = F16 ? 0x3C003C00u : 0x3F803F80u;
    const u32x4 ones = {one, one, one, one};

    const ScalarInts table =
        (ScalarInts)(uintptr_t)(g.c.page_table + (int64_t)p.seq * g.c.max_pages);
    const int lg = g.c.lg_page, slot_mask = g.c.page() - 1;
    const int64_t page_rows = (int64_t)2 * g.c.heads << lg;
    const int64_t k_rows = g.c.rows_before(g.a.layer, 0, 0, head);
    const int64_t v_rows = k_rows + ((int64_t)g.c.heads << lg);
    const uint32_t kc_at = col * (D / 2) + grp * (D / 8);
    const uint32_t ks_at = ((D == 64 ? grp >> 1 : (D == 128 ? grp : 2 * grp)) << lg) + col;
    const uint32_t vc_at = 4 * grp * (D / 2) + col * (D / 32);
    const uint32_t vs_at = ((col * DV / 32) << lg) + 4 * grp;
    constexpr int kWide = D == 64 ? 2 : 4;      // words of a load
    typedef uint32_t KeyBytes __attribute__((ext_vector_type(kWide)));

    auto pages = [&](int key) {
        Pages f;
        f.id[0] = table[key >> lg];
        f.id[1] = key + 16 < p.len ? table[(key + 16) >> lg] : -1;
        return f;
    };
    auto load = [&](Step<D>& f, Pages& ids, int key) {
        ids.bad = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            int id = ids.id[t];
            if (!kv_page_ok(g.c, id)) {
                ids.bad |= 1 << t;
                id = 0;
            }
            const int slot = (key + 16 * t) & slot_mask;
            const int64_t kr = id * page_rows + k_rows, vr = id * page_rows + v_rows;
            const uint8_t* kc = g.c.codes + (kr + slot) * (D / 2);
            const uint8_t* vc = g.c.codes + (vr + slot) * (D / 2);
            const uint8_t* ks = g.c.scales + kr * (D / 32) + slot;
            const uint8_t* vs = g.c.scales + vr * (D / 32) + slot;
#pragma unroll
            for (int w = 0; w < D / 32; w += kWide) {
                // Streamed: read once, they would push everything else out of L2.
                const KeyBytes x = __builtin_nontemporal_load((const KeyBytes*)(kc + kc_at + 4 * w));
#pragma unroll
                for (int i = 0; i < kWide; ++i) f.k[t][w + i] = x[i];
            }
#pragma unroll
            for (int w = 0; w < (D == 256 ? 2 : 1); ++w) f.ks[t][w] = (ks + (w << lg))[ks_at];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (D == 64) {
                    f.v[t][i][0] = *(const uint16_t*)(vc + vc_at + i * (D / 2));
                } else {
#pragma unroll
                    for (int w = 0; w < D / 128; ++w)
                        f.v[t][i][w] = ((const uint32_t*)(vc + vc_at + i * (D / 2)))[w];
                }
            }
            f.vs[t] = *(const uint32_t*)(vs + vs_at);
        }
    };

    // One step of 32 keys.  plain: every row sees every key of it.
    auto compute = [&](const Step<D>& f, int bad, int key, bool plain) {
        // S^T: two tiles of 16 keys.
        f32x4 s[MT][2];
#pragma unroll
        for (int q = 0; q < kKs; ++q) {
            u32x4 kf[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
                kf[t] = widen8<F16>(f.k[t][q], unit_of(f.ks[t][D == 256 ? q >> 2 : 0]));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    s[mt][t] = mfma<F16>(kf[t], qf[mt][q], q ? s[mt][t] : f32x4{0, 0, 0, 0});
        }
        uint32_t vis[MT] = {};          // bit 4t + r: the row sees key 4 grp + r of tile t
        if (!plain) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                vis[mt] = seen_bits<2>(g, p, tok[mt], key + 4 * grp, key1, bad, 1);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    s[mt][e >> 2][e & 3] = vis[mt] >> e & 1 ? s[mt][e >> 2][e & 3] : -INFINITY;
            }
        }
        // Weights 2^(cs s + neg).  One beyond the slack, or any of a row whose
        // reference is not set (neg infinite: its weights are infinite or NaN),
        // gives its row a new reference; weights are positive, so their bits
        // compare as integers.
        float w[MT][8];
        uint32_t most[MT] = {}, all = 0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[mt][i] = __builtin_amdgcn_exp2f(fmaf(s[mt][i >> 2][i & 3], cs, neg[mt]));
                const uint32_t bits = __builtin_bit_cast(uint32_t, w[mt][i]);
                most[mt] = bits > most[mt] ? bits : most[mt];
            }
            all = most[mt] > all ? most[mt] : all;
        }
        if (__any(all > kMostBits)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float now = s[mt][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) now = fmaxf(now, s[mt][i >> 2][i & 3]);
                now = fmaxf(now, __shfl_xor(now, 16));
                now = fmaxf(fmaxf(now, __shfl_xor(now, 32)), ref[mt]);
                now = row_over(most[mt], kMostBits) ? now : ref[mt];
                const float keep = fade(
                    ref[mt], now, cs, surplus(now, cs, kLift) - surplus(ref[mt], cs, kLift));
                const Exponent x = exponent(now, cs, kLift);
                ref[mt] = now;
                neg[mt] = x.neg;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[mt][i] =
                        __builtin_amdgcn_exp2f(fmaf(s[mt][i >> 2][i & 3] - x.sub, cs, x.add));
#pragma unroll
                for (int t = 0; t < DV; ++t) o[t][mt] *= keep;
                lsum[mt] *= keep;
            }
        }
        // Weights as the sum of two numbers of the type.
        u32x4 pf[MT], pl[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = w[mt][2 * i], b = w[mt][2 * i + 1];
                const uint32_t hi = pack<F16>(a, b);
                pf[mt][i] = hi;
                pl[mt][i] = pack<F16>(a - low<F16>(hi), b - high<F16>(hi));
            }
            lsum[mt] = mfma<F16>(ones, pf[mt], lsum[mt]);
            lsum[mt] = mfma<F16>(ones, pl[mt], lsum[mt]);
        }
        // V^T: dims DV m + t of the lane's 8 keys.
        float unit[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) unit[i] = unit_of((f.vs[i >> 2] >> (8 * (i & 3))) & 0xFFu);
        if (!plain) {
            // A key that a row does not see leaves it alone even where its
            // value is NaN: such values count as 0 in the product, and the
            // rows that do see them become NaN at the end, where a product of
            // indicators has counted any.
            u32x4 nan = {0, 0, 0, 0};
            bool some = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool here = __builtin_bit_cast(uint32_t, unit[i]) == 0x7F800000u;
                some |= here;
                nan[i >> 1] |= here ? (i & 1 ? one & 0xFFFF0000u : one & 0xFFFFu) : 0u;
                unit[i] = here ? 0.f : finite_unit<F16>(unit[i]);
            }
            if (__any(some)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    u32x4 seen;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        seen[i] = ((vis[mt] >> (2 * i)) & 1 ? one & 0xFFFFu : 0u) |
                                  ((vis[mt] >> (2 * i + 1)) & 1 ? one & 0xFFFF0000u : 0u);
                    hit[mt] = mfma<F16>(nan, seen, hit[mt]);
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
                    const uint32_t word = f.v[i >> 2][i & 3][w];
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
                    o[t][mt] = mfma<F16>(lo, pl[mt], o[t][mt]);
                    o[t + 1][mt] = mfma<F16>(hi, pl[mt], o[t + 1][mt]);
                }
            }
        }
    };

    // The next step's bytes and the pages of the one behind it are on their way
    // while a step is worked on.
    int key = key0 + wave * kStep;
    if (key < key1) {
        Step<D> f[2];
        Pages now = pages(key), next = pages(key + kTile < key1 ? key + kTile : key);
        load(f[0], now, key);
        while (key < key1) {
            const int ahead = key + kTile < key1 ? key + kTile : key;
            load(f[1], next, ahead);
            const Pages then = pages(ahead + kTile < key1 ? ahead + kTile : ahead);
            compute(f[0], now.bad, key, key + kStep <= full && key + kStep <= key1 && now.bad == 0);
            f[0] = f[1];
            now = next;
            next = then;
            key += kTile;
        }
    }

    // The waves' sums to a common reference.
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = mt * 16 + col;
        if (grp == 0) {
            s_m[wave][r] = ref[mt];
            s_l[wave][r] = lsum[mt][0];
            s_more[wave][r] = surplus(ref[mt], cs, kLift);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int t = 0; t < DV; t += 4)
                *(f32x4*)&s_o[wave][r][4 * DV * grp + DV * q + t] =
                    f32x4{o[t][mt][q], o[t + 1][mt][q], o[t + 2][mt][q], o[t + 3][mt][q]} +
                    (hit[mt][q] > 0.f ? NAN : 0.f);
    }
    __syncthreads();
    for (int at = threadIdx.x; at < kRows * (D / 4); at += kThreads) {
        const int r = at / (D / 4), dim = at % (D / 4) * 4;
        const int token = r / g.group;
        const int64_t row = start + token;
        if (token >= p.rows || row < 0 || row >= g.b.n_rows) continue;
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        float l = 0.f;
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = fade(s_m[w][r], top, cs, -s_more[w][r]);
            l += s_l[w][r] * f;
            sum += *(const f32x4*)&s_o[w][r][dim] * f;
        }
        if (p.splits == 1) {
            // Nothing seen: 0.  A sum of NaN is not 0.
            const float inv = l == 0.f ? 0.f : 1.f / l;
            uint32_t* dst = (uint32_t*)((uint16_t*)g.a.out + row * g.a.out_stride +
                                        ((int64_t)head * g.group + r % g.group) * D + dim);
            dst[0] = pack<F16>(sum[0] * inv, sum[1] * inv);
            dst[1] = pack<F16>(sum[2] * inv, sum[3] * inv);
        } else {
            *(f32x4*)(g.part_o + ((int64_t)p.part * kRows + r) * D + dim) = sum;
            if (dim == 0) g.part_ml[(int64_t)p.part * kRows + r] = f32x2{top, l};
        }
    }
}

// The same for many rows (draft trees, prompt chunks): a workgroup's four
// waves have 16 MT rows each and share the keys.  A tile of KT keys is widened
// once for all of them and laid into LDS in the order in which the matrix
// instructions take it, in fragments of 16 bytes a lane (bank conflicts are 14 % of
// the LDS's cycles, in which it is busy a third of the time), two tiles
// in turn, so that one is read while the next is written; a wave widens 16
// keys (or their keys or values alone).  Each wave ends with whole rows, so
// nothing is joined but runs.
//
// Keys are widened to the query's type, values to f16.  A part with a scale
// outside 2^-19 .. 2^12 (one test of four bytes) is looked at value by value: what
// f16 does not hold is 0 in LDS, and each wave fetches it again in bf16, for
// products of its own.  Two 2048-token chunks take 341 us, as with weights and
// values in bf16 (344; with values of both kinds in LDS and a mask: 391).  Where
// every value is beyond f16 they take 2.8 times as long.
template <int D, bool F16, int MT>
__global__ __launch_bounds__(kThreads, D >= 128 ? 2 : (MT == 1 ? 4 : 3))
    void kv_many_kernel(Args g) {
    constexpr int kRows = 64 * MT;
    constexpr int kKs = D / 32;
    constexpr int DV = D / 16;
    constexpr int KT = D == 256 ? 32 : 64;          // keys of a tile
    constexpr int kTiles = 2;                       // parts of 16 keys worked on at a time
    __shared__ u32x4 s_k[2][KT / 16][kKs][64];
    __shared__ u32x4 s_v[2][KT / 32][DV][64];
    __shared__ u32x4 s_nan[2][KT / 32][64]; // 1 where a value is NaN
    __shared__ int s_flag[2][KT / 16];      // 1: no page, 2: some value is NaN, 4: some beyond f16

    const Plan p = plan<kRows>(g);
    if (p.entry < 0) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int n_tiles = (p.rows * g.group + kRows - 1) / kRows;
    const int local = p.item - p.first;
    const int split = local / (n_tiles * g.c.heads);
    // Tiles of one run from the last on (causal, they see the most keys), the
    // heads of each side by side: workgroups are dealt to the 8 XCDs in turn,
    // so the tiles of a head meet in one L2 where there are 8 heads.
    const int at = local - split * n_tiles * g.c.heads;
    const int rt = n_tiles - 1 - at / g.c.heads, head = at % g.c.heads;
    const int r0 = rt * kRows;
    const int w0 = r0 + wave * 16 * MT;         // the wave's rows
    const int base = p.len - p.rows;
    const int64_t start = kv_start(g.b, p.entry);

    int tok[MT];
    u32x4 qf[MT][kKs];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = w0 + mt * 16 + col;
        tok[mt] = r / g.group;
        const int64_t row = start + tok[mt];
        const bool on = tok[mt] < p.rows && row >= 0 && row < g.b.n_rows;
        const u32x4* src = (const u32x4*)((const uint16_t*)g.a.q + (on ? row : 0) * g.a.q_stride +
                                          ((int64_t)head * g.group + r % g.group) * D +
                                          grp * (D / 4));
#pragma unroll
        for (int s = 0; s < kKs; ++s) qf[mt][s] = on ? src[s] : u32x4{0, 0, 0, 0};
    }

    // Keys of the item; of a causal tile up to what its last row sees.  The
    // wave's own rows see every key in front of `full` and none from `end` on.
    const int key0 = split * p.run * kTile;
    int key1 = p.splits == 1 ? p.len : key0 + p.run * kTile;
    if (key1 > p.len) key1 = p.len;
    int full = base, end = key1;
    if (!g.a.mask) {
        const int last = (r0 + kRows - 1) / g.group, mine = (w0 + 16 * MT - 1) / g.group;
        const int seen = base + (last < p.rows ? last : p.rows - 1) + 1;
        if (key1 > seen) key1 = seen;
        const int own = base + (mine < p.rows ? mine : p.rows - 1) + 1;
        full = base + w0 / g.group + 1;
        end = own < key1 ? own : key1;
    }
    if (w0 / g.group >= p.rows) end = 0;        // no rows: the wave only widens
    // Weights as two numbers where the entry has no more rows than this, whatever
    // lies beside it: 48 rows of 128 dims over 200 to 4100 positions 25.8 -> 28.4
    // us; 183 rows of 64 would pay 33.8 -> 38.1, 1204 of 128 over 8500 positions
    // 75 -> 91, two 2048-token chunks 337 -> 444.
    const bool two = p.rows * g.group <= 64;

    f32x4 o[DV][MT];
    f32x4 lsum[MT];
    f32x4 hit[MT];
    float ref[MT], neg[MT];
    constexpr float kLift = lift_of(true);
    constexpr uint32_t kMostBits = most_bits(true);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int t = 0; t < DV; ++t) o[t][mt] = f32x4{0, 0, 0, 0};
        lsum[mt] = f32x4{0, 0, 0, 0};
        hit[mt] = f32x4{0, 0, 0, 0};
        ref[mt] = -INFINITY;
        neg[mt] = INFINITY;
    }
    const float cs = g.a.scale * 1.4426950408889634f;
    constexpr uint32_t one = 0x3C003C00u;
    const u32x4 ones = {one, one, one, one};

    const ScalarInts table =
        (ScalarInts)(uintptr_t)(g.c.page_table + (int64_t)p.seq * g.c.max_pages);
    const int lg = g.c.lg_page, slot_mask = g.c.page() - 1;
    const int64_t page_rows = (int64_t)2 * g.c.heads << lg;
    const int64_t k_rows = g.c.rows_before(g.a.layer, 0, 0, head);
    const int64_t v_rows = k_rows + ((int64_t)g.c.heads << lg);

    // The wave's part of a tile: 16 keys, both products' side of them or one.
    const int part = KT == 64 ? wave : wave >> 1;
    const bool do_k = KT == 64 || (wave & 1) == 0, do_v = KT == 64 || (wave & 1) == 1;
    uint32_t rk[D / 32], rks[D == 256 ? 2 : 1], rv[4][D == 256 ? 2 : 1], rvs;
    int bad = 0;
    typedef uint32_t Codes[4][D == 256 ? 2 : 1];
    auto load_v = [&](int id, int slot, Codes& codes, uint32_t& bytes) {
        const int64_t vr = id * page_rows + v_rows;
        const uint8_t* vc = g.c.codes + (vr + slot) * (D / 2) + 4 * grp * (D / 2) + col * (D / 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (D == 64) {
                codes[i][0] = *(const uint16_t*)(vc + i * (D / 2));
            } else {
#pragma unroll
                for (int w = 0; w < D / 128; ++w)
                    codes[i][w] = ((const uint32_t*)(vc + i * (D / 2)))[w];
            }
        }
        bytes = *(const uint32_t*)(g.c.scales + vr * (D / 32) + slot + 4 * grp +
                                   ((col * DV / 32) << lg));
    };
    auto fetch = [&](int key) {
        int id = key + 16 * part < p.len ? table[(key + 16 * part) >> lg] : -1;
        bad = !kv_page_ok(g.c, id);
        if (bad) id = 0;
        const int slot = (key + 16 * part) & slot_mask;
        if (do_k) {
            const int64_t kr = id * page_rows + k_rows;
            const uint8_t* kc = g.c.codes + (kr + slot) * (D / 2) + col * (D / 2) + grp * (D / 8);
            const uint8_t* ks = g.c.scales + kr * (D / 32) + slot + col +
                                ((D == 64 ? grp >> 1 : (D == 128 ? grp : 2 * grp)) << lg);
#pragma unroll
            for (int w = 0; w < D / 32; ++w) rk[w] = ((const uint32_t*)kc)[w];
#pragma unroll
            for (int w = 0; w < (D == 256 ? 2 : 1); ++w) rks[w] = ks[w << lg];
        }
        if (do_v) load_v(id, slot, rv, rvs);
    };
    auto spread = [&](int buf) {
        if (do_k) {
#pragma unroll
            for (int q = 0; q < kKs; ++q)
                s_k[buf][part][q][lane] = widen8<F16>(rk[q], unit_of(rks[D == 256 ? q >> 2 : 0]));
        }
        if (do_v) {
            const int step = part >> 1, half = part & 1;
            float unit[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) unit[i] = unit_of((rvs >> (8 * i)) & 0xFFu);
            int flag = bad;
            // All four scales 108 to 139: finite in f16.  Where the sum carries, a
            // byte of 236 or more shows itself.
            if (__any(((rvs + 0x14141414u) & 0xE0E0E0E0u) != 0x80808080u)) {
                uint32_t nan[2] = {0, 0};
                bool some = false, odd = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t byte = (rvs >> (8 * i)) & 0xFFu;
                    const bool here = byte == 255u, out = !F16 && beyond_f16(byte, rv[i]);
                    some |= here;
                    odd |= out;
                    nan[i >> 1] |= here ? (i & 1 ? one & 0xFFFF0000u : one & 0xFFFFu) : 0u;
                    unit[i] = here || out ? 0.f : finite_unit<true>(unit[i]);
                }
                flag |= (__any(some) ? 2 : 0) | (__any(odd) ? 4 : 0);
                ((u32x2*)&s_nan[buf][step][lane])[half] = u32x2{nan[0], nan[1]};
            }
            if (lane == 0) s_flag[buf][part] = flag;
#pragma unroll
            for (int w = 0; w < (D == 256 ? 2 : 1); ++w)
#pragma unroll
                for (int by = 0; by < (D == 64 ? 2 : 4); ++by) {
                    uint32_t x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[i] = by == 0   ? widen<true, 0>(rv[i][w], unit[i])
                               : by == 1 ? widen<true, 1>(rv[i][w], unit[i])
                               : by == 2 ? widen<true, 2>(rv[i][w], unit[i])
                                         : widen<true, 3>(rv[i][w], unit[i]);
                    const int t = 8 * w + 2 * by;
                    ((u32x2*)&s_v[buf][step][t][lane])[half] =
                        u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u),
                              __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)};
                    ((u32x2*)&s_v[buf][step][t + 1][lane])[half] =
                        u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u),
                              __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
                }
        }
    };

    // The 16-key parts of a tile from t0 on, `key` the first of their keys.
    // plain: every row of the wave sees all of them, and their flags are 0.
    auto compute = [&](int buf, int t0, int key, int flags, bool plain) {
        uint32_t vis[MT] = {};          // bit 4t + r: the row sees key 4 grp + r of quarter t
        if (!plain) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                vis[mt] = seen_bits<kTiles>(g, p, tok[mt], key + 4 * grp, key1, flags, 3);
        }
        f32x4 s[MT][kTiles];
        auto scores = [&]() {
            // All reads on their way before the first product waits.
            u32x4 kf[kKs][kTiles];
#pragma unroll
            for (int q = 0; q < kKs; ++q)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) kf[q][t] = s_k[buf][t0 + t][q][lane];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < kKs; ++q)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        s[mt][t] = mfma<F16>(kf[q][t], qf[mt][q], q ? s[mt][t] : f32x4{0, 0, 0, 0});
            if (!plain) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            s[mt][t][r] = vis[mt] >> (4 * t + r) & 1 ? s[mt][t][r] : -INFINITY;
            }
        };
        scores();
        uint32_t most[MT] = {}, all = 0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[mt][t][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][t][r], cs, neg[mt]));
                    const float w = s[mt][t][r];
                    const uint32_t bits = __builtin_bit_cast(uint32_t, w);
                    most[mt] = bits > most[mt] ? bits : most[mt];
                }
            all = most[mt] > all ? most[mt] : all;
        }
        if (__any(all > kMostBits)) {
            scores();                           // again: they are not kept
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float now = s[mt][0][0];
#pragma unroll
                for (int i = 1; i < 4 * kTiles; ++i) now = fmaxf(now, s[mt][i >> 2][i & 3]);
                now = fmaxf(now, __shfl_xor(now, 16));
                now = fmaxf(fmaxf(now, __shfl_xor(now, 32)), ref[mt]);
                now = row_over(most[mt], kMostBits) ? now : ref[mt];
                const float keep = fade(
                    ref[mt], now, cs, surplus(now, cs, kLift) - surplus(ref[mt], cs, kLift));
                const Exponent x = exponent(now, cs, kLift);
                ref[mt] = now;
                neg[mt] = x.neg;
#pragma unroll
                for (int i = 0; i < 4 * kTiles; ++i)
                    s[mt][i >> 2][i & 3] =
                        __builtin_amdgcn_exp2f(fmaf(s[mt][i >> 2][i & 3] - x.sub, cs, x.add));
#pragma unroll
                for (int t = 0; t < DV; ++t) o[t][mt] *= keep;
                lsum[mt] *= keep;
            }
        }
        const int at = t0 / 2;
        constexpr int kBatch = DV < 8 ? DV : 8;
        u32x4 pf[MT];
#pragma unroll
        for (int d0 = 0; d0 < DV; d0 += kBatch) {
            u32x4 vf[kBatch];
#pragma unroll
            for (int t = 0; t < kBatch; ++t) vf[t] = s_v[buf][at][d0 + t][lane];
            __builtin_amdgcn_sched_barrier(0);
            if (d0 == 0) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        pf[mt][i] =
                            pack<true>(s[mt][i >> 1][2 * i & 3], s[mt][i >> 1][(2 * i & 3) + 1]);
                    lsum[mt] = mfma<true>(ones, pf[mt], lsum[mt]);
                }
            }
#pragma unroll
            for (int t = 0; t < kBatch; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    o[d0 + t][mt] = mfma<true>(vf[t], pf[mt], o[d0 + t][mt]);
        }
        if (!two && !(flags & 0x36)) return;            // most often
        // What pf leaves of the weights.
        u32x4 pl[MT];
        if (two) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t hi = pf[mt][i];
                    pl[mt][i] = pack<true>(s[mt][i >> 1][2 * i & 3] - low<true>(hi),
                                           s[mt][i >> 1][(2 * i & 3) + 1] - high<true>(hi));
                }
                lsum[mt] = mfma<true>(ones, pl[mt], lsum[mt]);
            }
#pragma unroll
            for (int t = 0; t < DV; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    o[t][mt] = mfma<true>(s_v[buf][at][t][lane], pl[mt], o[t][mt]);
        }
        if (!F16 && (flags & 0x24)) {
            // Values beyond f16 are 0 in s_v.  They come from the cache again, in
            // bf16, and meet the same weights: two numbers of bf16 hold one of
            // f16, a third what pl has.
            Codes codes[2];
            float unit[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from = key + 16 * h;
                const int id = from < p.len ? table[from >> lg] : -1;
                uint32_t bytes;
                load_v(kv_page_ok(g.c, id) ? id : 0, from & slot_mask, codes[h], bytes);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t byte = (bytes >> (8 * i)) & 0xFFu;
                    unit[4 * h + i] = beyond_f16(byte, codes[h][i])
                                          ? finite_unit<false>(unit_of(byte)) : 0.f;
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                u32x4 p0, p1, p2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = low<true>(pf[mt][i]), b = high<true>(pf[mt][i]);
                    p0[i] = pack<false>(a, b);
                    p1[i] = pack<false>(a - low<false>(p0[i]), b - high<false>(p0[i]));
                    p2[i] = two ? pack<false>(low<true>(pl[mt][i]), high<true>(pl[mt][i])) : 0u;
                }
#pragma unroll
                for (int w = 0; w < (D == 256 ? 2 : 1); ++w)
#pragma unroll
                    for (int by = 0; by < (D == 64 ? 2 : 4); ++by) {
                        uint32_t x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint32_t word = codes[i >> 2][i & 3][w];
                            x[i] = by == 0   ? widen<false, 0>(word, unit[i])
                                   : by == 1 ? widen<false, 1>(word, unit[i])
                                   : by == 2 ? widen<false, 2>(word, unit[i])
                                             : widen<false, 3>(word, unit[i]);
                        }
#pragma unroll
                        for (int odd = 0; odd < 2; ++odd) {
                            u32x4 v;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                v[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i],
                                                             odd ? 0x07060302u : 0x05040100u);
                            const int t = 8 * w + 2 * by + odd;
                            o[t][mt] = mfma<false>(v, p0, o[t][mt]);
                            o[t][mt] = mfma<false>(v, p1, o[t][mt]);
                            o[t][mt] = mfma<false>(v, p2, o[t][mt]);
                        }
                    }
            }
        }
        if (flags & 0x12) {
            u32x4 nan = s_nan[buf][at][lane];           // of a half that has none: anything
#pragma unroll
            for (int i = 0; i < 4; ++i) nan[i] = flags & (i < 2 ? 2 : 0x10) ? nan[i] : 0u;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                u32x4 seen;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    seen[i] = (vis[mt] >> (2 * i) & 1 ? one & 0xFFFFu : 0u) |
                              (vis[mt] >> (2 * i + 1) & 1 ? one & 0xFFFF0000u : 0u);
                hit[mt] = mfma<true>(nan, seen, hit[mt]);
            }
        }
    };

    if (key0 < key1) {
        fetch(key0);
        spread(0);
        if (key0 + KT < key1) fetch(key0 + KT);
        __syncthreads();
        int buf = 0;
        for (int key = key0; key < key1; key += KT) {
            // Flags of the tile's parts, three bits each.
            int flags = 0;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) flags |= s_flag[buf][t] << (3 * t);
            flags = __builtin_amdgcn_readfirstlane(flags);
#pragma unroll
            for (int t0 = 0; t0 < KT / 16; t0 += kTiles) {
                const int at = key + 16 * t0, part = flags >> (3 * t0) & ((1 << 3 * kTiles) - 1);
                if (at < end)
                    compute(buf, t0, at, part, at + 16 * kTiles <= full && at + 16 * kTiles <= end &&
                                                   part == 0);
            }
            if (key + KT < key1) {
                spread(buf ^ 1);
                if (key + 2 * KT < key1) fetch(key + 2 * KT);
                __syncthreads();
            }
            buf ^= 1;
        }
    }

    // A lane has 4 DV neighbouring dims of each of its rows.
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = wave * 16 * MT + mt * 16 + col, rr = r0 + r;
        const int64_t row = start + tok[mt];
        if (tok[mt] >= p.rows || row < 0 || row >= g.b.n_rows) continue;
        const float l = lsum[mt][0];
        if (p.splits == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            u32x4* dst = (u32x4*)((uint16_t*)g.a.out + row * g.a.out_stride +
                                  ((int64_t)head * g.group + rr % g.group) * D + 4 * DV * grp);
#pragma unroll
            for (int at = 0; at < 4 * DV; at += 8) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int a = at + 2 * i, q = a / DV;
                    const float nan = hit[mt][q] > 0.f ? NAN : 0.f;
                    x[i] = pack<F16>(o[a % DV][mt][q] * inv + nan, o[a % DV + 1][mt][q] * inv + nan);
                }
                dst[at / 8] = x;
            }
        } else {
            float* dst = g.part_o + ((int64_t)p.part * kRows + r) * D + 4 * DV * grp;
            const float less = __builtin_amdgcn_exp2f(-surplus(ref[mt], cs, kLift));
#pragma unroll
            for (int at = 0; at < 4 * DV; at += 4) {
                const int q = at / DV, t = at % DV;
                *(f32x4*)(dst + at) =
                    f32x4{o[t][mt][q], o[t + 1][mt][q], o[t + 2][mt][q], o[t + 3][mt][q]} * less +
                    (hit[mt][q] > 0.f ? NAN : 0.f);
            }
            if (grp == 0) g.part_ml[(int64_t)p.part * kRows + r] = f32x2{ref[mt], l * less};
        }
    }
}

// Joins the runs of a unit: RB rows of a tile of ROWS for a workgroup.  RB 1:
// the row's runs are dealt to teams of threads, who add up at the end; else
// each row has a team.
template <int D, bool F16, int ROWS, int RB>
__global__ __launch_bounds__(kThreads) void kv_join_kernel(Args g, int tiles_max, int per_tile) {
    constexpr int kLanes = D / 4;                 // threads of a row
    constexpr int kTeams = kThreads / kLanes;     // 16, 8, 4
    __shared__ f32x4 s_o[kTeams][kLanes];
    __shared__ f32x2 s_ml[kTeams];
    const int sub = blockIdx.x % per_tile;
    const int rt = blockIdx.x / per_tile % tiles_max;
    const int head = blockIdx.x / per_tile / tiles_max % g.c.heads;
    const int entry = blockIdx.x / per_tile / tiles_max / g.c.heads;
    const i32x4 plan = g.plans[entry];
    const int rows = plan[0], splits = plan[2], first_part = plan[3];
    if (splits == 1) return;
    const int n_tiles = (rows * g.group + ROWS - 1) / ROWS;
    if (rt >= n_tiles) return;
    const int place = (n_tiles - 1 - rt) * g.c.heads + head;
    const int team = threadIdx.x / kLanes, dim = threadIdx.x % kLanes * 4;
    const int64_t start = kv_start(g.b, entry);
    const float cs = g.a.scale * 1.4426950408889634f;
    for (int r = sub * RB + (RB == 1 ? 0 : team); r < (sub + 1) * RB; r += kTeams) {
        const int rr = rt * ROWS + r, token = rr / g.group;
        const int64_t row = start + token;
        const bool on = token < rows && row >= 0 && row < g.b.n_rows;
        if (RB == 1 && !on) return;               // the whole workgroup
        float top = -INFINITY, l = 0.f;
        f32x4 sum = {0, 0, 0, 0};
        if (on) {
            // The partial sums come from far (other XCDs wrote them): many at
            // a time; places behind the last read the first again, weight 0.
            constexpr int kEvery = RB == 1 ? kTeams : 1;
            const int64_t first = ((int64_t)first_part + place) * ROWS + r;
            const int64_t apart = (int64_t)g.c.heads * n_tiles * ROWS;
            auto add = [&](auto batch) {
                constexpr int kBatch = decltype(batch)::value;
                for (int s0 = RB == 1 ? team : 0; s0 < splits; s0 += kBatch * kEvery) {
                    f32x2 ml[kBatch];
                    f32x4 x[kBatch];
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        const int s = s0 + i * kEvery;
                        const int64_t at = first + (s < splits ? s : s0) * apart;
                        ml[i] = g.part_ml[at];
                        x[i] = *(const f32x4*)(g.part_o + at * D + dim);
                    }
                    // Left alone, most of the loads are moved behind the
                    // exponentials, one after the other.
                    __builtin_amdgcn_sched_barrier(0);
                    float now = top;
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) now = fmaxf(now, ml[i][0]);
                    const float a = fade(top, now, cs);
                    l *= a;
                    sum *= a;
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        float w = fade(ml[i][0], now, cs);
                        w = s0 + i * kEvery < splits ? w : 0.f;
                        l += ml[i][1] * w;
                        sum += x[i] * w;
                    }
                    top = now;
                }
            };
            if (splits > 4 * kEvery)
                add(std::integral_constant<int, RB == 1 ? 16 : 8>());
            else
                add(std::integral_constant<int, 4>());
        }
        if constexpr (RB == 1) {
            s_o[team][threadIdx.x % kLanes] = sum;
            if (dim == 0) s_ml[team] = f32x2{top, l};
            __syncthreads();
            if (team != 0) return;
            for (int t = 1; t < kTeams; ++t) {
                const float now = fmaxf(top, s_ml[t][0]);
                const float a = fade(top, now, cs), b = fade(s_ml[t][0], now, cs);
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

// Rows of a tile.  Up to 32 rows of a unit are one tile of the kernel whose
// waves share rows (24 rows of 128 dims over 3000 positions, 4 entries: 17.7
// us, 18.5 by the other); more go to the one whose waves share keys, in tiles
// of 128: two 2048-token chunks 341 us, 497 in tiles of 64.
// Tiles of 64 where the unit has no more, of 256 dims, whose sums take twice
// the registers, and of 64 dims where they leave a quarter of the rows less
// empty, which is from 129 to 192 rows.  Tiles of 64 and 128 there, us: 16 entries
// over 200 to 4100 positions of 129, 183, 192 rows 32.7, 35.0, 34.7 and 38.9,
// 40.6, 39.3; 1 of 183 over 8000 24.2 and 26.9; 32 over 1500 50.8 and 56.9; 8 of
// 140 over 1000 26.5 and 34.6; 16 of 188 over 4000 73 and 63.  And where it is
// not a quarter: 65 rows 31.9 and 29.7, 210 44.8 and 40.7, 300 51.8 and 49.8.
int tile_rows(int max_rows, int group, int d) {
    const int64_t rows = (int64_t)max_rows * group;
    if (rows <= 16) return 16;
    if (rows <= 32 && d != 256) return 32;
    if (rows <= 64 || d == 256) return 64;
    const int64_t by64 = (rows + 63) / 64 * 64, by128 = (rows + 127) / 128 * 128;
    return d == 64 && 4 * by64 <= 3 * by128 ? 64 : 128;
}

// Workgroups to cut the work for: what is resident at once (twice and three
// times as many took 41 -> 46, 48 us for one token over 131K positions: each
// costs its start and a partial sum).  Tiles of 64 rows of 64 dims leave room for
// four on a compute unit; four against three, us: 16 entries over 200 to 4100
// positions of 129, 183, 192 rows 32.7, 35.0, 34.7 and 36.5, 38.7, 38.6; 32 of 183
// over 1500 50.8 and 50.3; 2 of 150 over 300 and 9000 29.7 and 27.1; 16 of 188
// over 4000 each, where the last few have the device to themselves, 73 and 63.
int target_items(int rows, int d) {
    if (rows > 32) return device_cus() * (d >= 128 ? 2 : (rows == 64 ? 4 : 3));
    return device_cus() * (rows > 16 || d == 256 ? 2 : (d == 128 ? 3 : 4));
}

int64_t units_most(int n, int max_rows, int n_heads, int kv_heads, int rows) {
    const int64_t tiles = ((int64_t)max_rows * (n_heads / kv_heads) + rows - 1) / rows;
    return tiles * kv_heads * n;
}

template <int D, bool F16, int ROWS>
hipError_t launch_rows(const Args& g, hipStream_t st) {
    const int64_t units = units_most(g.b.n, g.b.max_rows, g.a.n_heads, g.c.heads, ROWS);
    if (g.b.n > 64) {
        hipLaunchKernelGGL((kv_plan_kernel<ROWS>), dim3(1), dim3(kPlanThreads), 0, st, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)(units + g.target));      // items, at most
    if constexpr (ROWS <= 32)
        hipLaunchKernelGGL((kv_few_kernel<D, F16, ROWS / 16>), grid, dim3(kThreads), 0, st, g);
    else
        hipLaunchKernelGGL((kv_many_kernel<D, F16, ROWS / 64>), grid, dim3(kThreads), 0, st, g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !g.target) return e;
    const int tiles = (int)(units / g.c.heads / g.b.n);
    constexpr int RB = ROWS == 16 ? 1 : 16;
    const int per_tile = ROWS == 16 ? g.b.max_rows * g.group : ROWS / RB;
    hipLaunchKernelGGL((kv_join_kernel<D, F16, ROWS, RB>), dim3((unsigned)(units * per_tile)),
                       dim3(kThreads), 0, st, g, tiles, per_tile);
    return hipGetLastError();
}

template <int D, bool F16>
hipError_t launch_d(const Args& g, int rows, hipStream_t st) {
    if (rows == 16) return launch_rows<D, F16, 16>(g, st);
    if (rows == 64) return launch_rows<D, F16, 64>(g, st);
    if constexpr (D != 256)
        return rows == 32 ? launch_rows<D, F16, 32>(g, st) : launch_rows<D, F16, 128>(g, st);
    return hipErrorInvalidValue;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t kv_attention_blocks(int n, int max_rows, int n_heads, int kv_heads, int d) {
    const int rows = tile_rows(max_rows, n_heads / kv_heads, d);
    const int64_t units = units_most(n, max_rows, n_heads, kv_heads, rows);
    // Of the attention itself, and of the join (a workgroup for 1 or 16 rows).
    return units * (rows == 16 ? 16 : rows / 16) + target_items(rows, d);
}

// Partial sums of the items of cut units, and the entries' plans.  There are at
// most `target` more items than units, and at most 2 target of cut units: a run
// has at least (tiles of all units) / target tiles and a cut unit more than one
// run, so all cut units' tiles are at most target runs, and there are fewer cut
// units than that; each unit's last run may be a part of one.
struct Layout {
    int rows, target;
    size_t ml, plans, total;
};
Layout layout_of(int n, int max_rows, int n_heads, int kv_heads, int d, int max_kv) {
    Layout l;
    l.rows = tile_rows(max_rows, n_heads / kv_heads, d);
    l.target = max_kv > kWhole ? target_items(l.rows, d) : 0;
    const int64_t units = units_most(n, max_rows, n_heads, kv_heads, l.rows);
    const size_t rows =
        (size_t)(units < l.target ? units + l.target : 2 * (int64_t)l.target) * l.rows *
        (l.target != 0);
    l.ml = align256(rows * d * sizeof(float));
    l.plans = l.ml + align256(rows * sizeof(f32x2));
    l.total = l.plans + (l.target || n > 64 ? align256((size_t)(n + 1) * sizeof(i32x4)) : 0);
    return l;
}

size_t kv_attention_workspace_bytes(int n, int max_rows, int n_heads, int kv_heads, int d,
                                    int max_kv) {
    return layout_of(n, max_rows, n_heads, kv_heads, d, max_kv).total;
}

hipError_t launch_kv_attention(const KvCache& c, const KvBatch& b, const KvAttention& a,
                               void* workspace, hipStream_t st) {
    Args g;
    g.c = c;
    g.b = b;
    g.a = a;
    g.group = a.n_heads / c.heads;
    const Layout l = layout_of(b.n, b.max_rows, a.n_heads, c.heads, c.d, a.max_kv);
    const int rows = l.rows;
    g.target = l.target;
    g.part_o = (float*)workspace;
    g.part_ml = (f32x2*)((char*)workspace + l.ml);
    g.plans = (i32x4*)((char*)workspace + l.plans);
    const bool f16 = a.dtype == DT_F16;
    if (c.d == 64) return f16 ? launch_d<64, true>(g, rows, st) : launch_d<64, false>(g, rows, st);
    if (c.d == 128)
        return f16 ? launch_d<128, true>(g, rows, st) : launch_d<128, false>(g, rows, st);
    return f16 ? launch_d<256, true>(g, rows, st) : launch_d<256, false>(g, rows, st);
}

}  // namespace sense
