// Attention over the paged cache (siso_kv_attend, siso_kv_attend_tree).  Layout of the pages: kv_internal.h.
#include <math.h>
#include <type_traits>

#include "kv_internal.h"

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// A row of work is one query head of one token; the heads that share a kv head are rows of the same tile (row = token * group
// + head in the group), so that a tile of 32 rows reads a key once for all of them.
struct KvAttend {
    KvPool pool;
    KvBatch batch;
    const bf16_t *q;
    long q_token, q_head;
    int vec;
    int group;         // query heads of a kv head
    float scale;       // its size times log2(e), above zero: the softmax is one of powers of two
    unsigned negate;   // a scale below zero: the queries' signs are turned
    int window;        // 0 = all
    int few;           // a sequence of more rows of work is k_kv_attend_chunk's, all others k_kv_attend_few's
    bf16_t *out;
    float *lse;
    float *parts;       // [2 * KV_STRETCHES]: sums [32][DP], then maximum and sum of each row
    unsigned *arrived;  // [2 * KV_STRETCHES]: parts of a tile that are there, by the number of its first; zeros between calls
    struct KvPlan *plan;
    long item0, items;  // of this launch the first; how many there may be
    const unsigned *mask;  // of a tree's rows, [rows][KV_MASK_WORDS]
};

struct KvTile {
    KvSequence s;
    int row0, rows;      // of the sequence's rows of work: the first one of the tile, how many there are
    int lo, hi;          // positions that some row of the tile sees
    int all_lo, all_hi;  // positions that all rows of the tile see
};
__device__ __forceinline__ int kv_window_from(const KvAttend &a, int pos) {  // the first position that a row at `pos` sees
    return a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
}
// A tree's rows stand at most as deep as they lie: of what lies behind the context a row sees what its mask has.
template <bool TREE>
__device__ __forceinline__ void kv_tile(const KvAttend &a, int row0, int size, KvTile &t) {
    const int work = t.s.rows * a.group;  // (2^30 at most)
    t.row0 = row0;
    t.rows = work - row0 < size ? work - row0 : size;
    const int first = t.s.start + row0 / a.group, last = t.s.start + (row0 + t.rows - 1) / a.group;
    t.hi = last + 1 > 0 ? last + 1 : 0;
    t.lo = kv_window_from(a, TREE ? t.s.start : first);
    t.all_hi = TREE ? t.s.start : first + 1;
    t.all_lo = kv_window_from(a, last);
}

// A row's mask in LDS: a word of ones (of the context), the words, a word of zeros; rows lie so that lanes meet in no bank.
#define KV_MASK_WORDS (SISO_KV_TREE / 32)
#define KV_MASK_ROW (KV_MASK_WORDS + 3)
// Lanes l and l + 32 bring the row of work of lane l: half of its words each.  A window leaves it the last `window` rows of its own.  Returns
// its depth.  Only lanes of one wave share what is written here.
__device__ __forceinline__ int kv_mask_row(const KvAttend &a, const KvTile &t, int token, bool valid, unsigned *lds) {
    constexpr int HALF = KV_MASK_WORDS / 2;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    u32x4_t w = u32x4_t{0, 0, 0, 0};
    static_assert(HALF == 4, "16 bytes for a lane");
    if (valid) w = *(const u32x4_t *)(a.mask + (size_t)(t.s.first + token) * KV_MASK_WORDS + HALF * h);
    int seen = 0;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {  // (no row behind this one)
        const int over = token + 1 - 32 * (HALF * h + i);
        w[i] &= over >= 32 ? 0xFFFFFFFFu : over <= 0 ? 0u : (1u << over) - 1u;
        seen += __popc(w[i]);
    }
    const int upper = __shfl(seen, n + 32), lower = __shfl(seen, n);
    const int depth = upper + lower > 0 ? upper + lower - 1 : 0;
    if (a.window > 0) {
        int drop = upper + lower - a.window;  // the first so many of the row's
        if (h) drop -= lower;
#pragma unroll
        for (int i = 0; i < HALF; ++i) {
            const int has = __popc(w[i]);
            if (drop >= has) w[i] = 0;
            else
                for (int k = 0; k < drop; ++k) w[i] &= w[i] - 1;
            drop -= has;
        }
    }
    unsigned *const row = lds + n * KV_MASK_ROW;
#pragma unroll
    for (int i = 0; i < HALF; ++i) row[1 + HALF * h + i] = w[i];
    row[h ? KV_MASK_WORDS + 1 : 0] = h ? 0u : 0xFFFFFFFFu;
    return depth;
}
// Bits of 32 positions, the first of them `off` (the same in every lane) behind the tree's first row: what lies ahead of that is the context.
__device__ __forceinline__ unsigned kv_mask_bits(const unsigned *lds, int row, int off) {
    if (off < -32) return 0xFFFFFFFFu;
    if (off >= SISO_KV_TREE) return 0u;
    const unsigned *w = lds + row * KV_MASK_ROW + 1 + (off >> 5);
    return (unsigned)((((u64)w[1] << 32) | w[0]) >> (off & 31));
}

__device__ __forceinline__ bf16x8_t kv_as_bf16(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }
// eight codes, exactly
__device__ __forceinline__ bf16x8_t kv_codes_bf16(unsigned a, unsigned b) {
    struct {
        bf16x2_t v[4];
    } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return __builtin_bit_cast(bf16x8_t, r);
}
__device__ __forceinline__ bool kv_not_finite(unsigned two) {
    return (two & 0x7F80u) == 0x7F80u || (two & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ float kv_both_halves_max(float v) {
    const LanePair<float> p = lane_pair<32>(v);
    return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float kv_both_halves_sum(float v) {
    const LanePair<float> p = lane_pair<32>(v);
    return p.a + p.b;
}

#define KV_PART(DP) (32 * ((DP) + 2))

// Parts go from one workgroup to another within a kernel, past the caches of each XCD: single stores and loads at the scope of the
// device.  A fence of that scope instead writes back and empties the XCD's whole L2, once for each workgroup: with it 64 sequences took 260
// to 560 us, the more the finer they were split.
__device__ __forceinline__ void kv_leave(float *at, float a, float b) {
    __hip_atomic_store((u64 *)at, (u64)__float_as_uint(a) | ((u64)__float_as_uint(b) << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 kv_found(const float *at) {
    const u64 v = __hip_atomic_load((const u64 *)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}

// Four sums of a row and what goes with them, brought from their own maximum to `top`.
__device__ __forceinline__ void kv_add_part(float mj, float top, float lj, float4 y, float &sum, float4 &x) {
    const float f = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj - top);
    sum += lj * f;
    x.x += y.x * f, x.y += y.y * f, x.z += y.z * f, x.w += y.w * f;
}
__device__ __forceinline__ void kv_finish(const KvAttend &a, const KvTile &t, int head, int r, int d, float top, float sum, float4 x) {
    const int work = t.row0 + r, tok = work / a.group, hd = head * a.group + work % a.group;
    const size_t at = (size_t)(t.s.first + tok) * a.group * a.pool.kv_heads + hd;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    if (d < a.pool.dim)
        *(uint2 *)(a.out + at * a.pool.dim + d) = make_uint2((unsigned)f32_to_bf16(x.x * inv) | ((unsigned)f32_to_bf16(x.y * inv) << 16),
                                                             (unsigned)f32_to_bf16(x.z * inv) | ((unsigned)f32_to_bf16(x.w * inv) << 16));
    if (d == 0 && a.lse) a.lse[at] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718056f;
}

// Sequences of few rows of work (at most KV_FEW: one token, a draft's few).  Each has tiles of 32 rows for each of its kv heads, each tile a
// number of units of KS positions.  The units of all tiles together, on the device, say how many make a stretch: KV_STRETCHES of them hold
// them all.  A tile of more is cut into stretches, each a workgroup's: nobody has more to do than one stretch, whatever the lengths
// are, and nobody but the device knows them.  Tiles and stretches are at most tiles + KV_STRETCHES items, at most 2 * KV_STRETCHES of them
// parts of a tile that is cut.
#define KV_FEW 128
// Of up to 128 elements all sequences go to the one kernel, whatever their rows, where the work is light: its latency is
// lower, as it has no stages that wait for each other, but every 32 rows read the keys again.  Light are so many tiles times positions times
// elements at most, all taken to be as long as the longest: KV_LIGHT where all sequences have as many new rows (16 heads over 4, 250 rows of
// 4,000: 25 us for elements of 128, two kernels 35; of 64 21 and 26; 400 rows: 41 and 39, 21 and 26; 1,000 rows of 3,000: 60 and 46, 38 and
// 32), KV_LIGHT_MIXED where not: then both kernels would run, one after the other, and this one's stretches are alike however lengths
// differ (8 heads, 24 sequences of 1 to 1,500 rows and 1 to 5,000 positions, elements of 128: 80 us, two kernels 128;
// 32 heads, 64 sequences of up to 4,000 rows and 9,000 positions: 1,377 and 1,007).
#define KV_LIGHT (1L << 26)
#define KV_LIGHT_MIXED (1L << 30)
#define KV_STRETCHES 1024
#define KV_LEAST 4  // units of a stretch, at least, one for each wave (one token of 2,001 positions gets 5: the launch has no workgroup for the last part of 4, and the fifth
                    // unit is a second step of one wave)
// Trees of up to 128 elements go to the chunks' kernel where its tiles of 256 rows are filled by half, the work is not light, and there are so few tiles (those that
// are likely) that they are cut into pieces of one length (heads of 128, 4 rows of work for each new one over 8 kv heads, us by the first kernel and by the
// chunks': one tree of 256 rows behind 4,000 positions 45 and 47, behind 8,000 64 and 59, in 8 bits behind 30,000 182 and 156; 3 of 40 behind 9,000 to
// 20,000 84 and 68, 3 of 24 behind 30,000 122 and 145; 8 of 100 behind 4,000 126 and 105; 12 of 60 to 100 behind 1,000 to 5,000 98 and 107, in 8 bits 87
// and 117; 24 of 35 to 64 in 8 bits 151 and 176).
#define KV_TREE_LIGHT (250L << 20)
#define KV_TREE_TILES 160
#define KV_TREE_WHOLE 20
#define KV_TREE_ROOT 2.0f
#define KV_ENOUGH 32 // units that are worth being joined
#define KV_FULL 256  // workgroups
#define KV_PLAN_CHUNKS 1024  // 65,535 sequences, 64 each
struct KvPlan {  // more than 64 sequences: made by a launch of its own
    unsigned stretch;
    unsigned items[KV_PLAN_CHUNKS], parts[KV_PLAN_CHUNKS];  // before each 64 sequences
};
static_assert(sizeof(KvPlan) <= SISO_KV_PLAN_BYTES, "room for the plan");

template <int KS, bool TREE>
struct KvFew {
    int first, rows, length;  // of this lane's sequence
    int tiles, range;         // its tiles (of all kv heads; 0: not one of these sequences) and the units of each
    __device__ __forceinline__ static int range_of(const KvAttend &a, int start, int length, int &from) {
        from = kv_window_from(a, start) & ~(KS - 1);
        const int r = (length - from + KS - 1) / KS;
        return r > 1 ? r : 1;
    }
    __device__ __forceinline__ void load(const KvAttend &a, int b) {
        tiles = range = first = rows = length = 0;
        if (b >= a.batch.n) return;
        const KvSequence s = kv_sequence(a.batch, b);
        first = s.first;
        rows = s.rows;
        length = s.length;
        if (rows == 0 || rows * a.group > a.few || (TREE && rows > SISO_KV_TREE)) return;
        int from;
        tiles = ((rows * a.group + 31) >> 5) * a.pool.kv_heads;
        range = range_of(a, s.start, length, from);
    }
    __device__ __forceinline__ u64 units() const { return (u64)tiles * (unsigned)range; }
    // Units of a stretch, from how many there are of units and tiles: KV_ENOUGH of them at least, less only where that would not
    // fill the chip, and so many that there are no more than KV_STRETCHES, nor than the launch has workgroups for.  More tiles than the launch
    // counted (first rows that decrease) are not cut: a part that no workgroup comes for would leave its tile's count for the next call.
    __device__ __forceinline__ static unsigned stretch_of(const KvAttend &a, u64 all, u64 all_tiles) {
        if (all_tiles >= (u64)a.items) return 0x7FFFFFFFu;
        const u64 room = a.items - all_tiles < KV_STRETCHES ? a.items - all_tiles : KV_STRETCHES;
        unsigned s = all < KV_FULL * KV_ENOUGH ? (unsigned)all / KV_FULL : KV_ENOUGH;
        if constexpr (TREE) {
            // A part of a full tile takes about as long to join as a step of its four waves: both together are least for twice the root of a tile's
            // units, and a tile of few is not cut (16 rows of 32 heads over 8 behind 2,001 positions: 16.2 us, with stretches of 4 20.9; behind 8,000:
            // 21.2 and 29.8; behind 500: 12.5 and 14.0).
            const float units = all_tiles ? (float)all / (float)all_tiles : 0.f;
            const unsigned best = units <= KV_TREE_WHOLE ? KV_TREE_WHOLE : (unsigned)(KV_TREE_ROOT * __builtin_amdgcn_sqrtf(units));
            s = s > best ? s : best;
        } else s = s > KV_LEAST ? s : KV_LEAST;
        const u64 most = (all + room - 1) / room;
        return most > 0x7FFFFFFFu ? 0x7FFFFFFFu : s > most ? s : (unsigned)most;
    }
    __device__ __forceinline__ unsigned cuts(unsigned stretch) const { return tiles ? ((unsigned)range + stretch - 1) / stretch : 0; }
    __device__ __forceinline__ static unsigned running_sum(unsigned v) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const unsigned x = __shfl_up(v, off);
            if (lane >= off) v += x;
        }
        return v;
    }
};
__device__ __forceinline__ u64 kv_wave_sum(u64 v) {
    return wave_fold(v, [](u64 a, u64 b) __attribute__((always_inline)) { return a + b; });
}

// What every workgroup of k_kv_attend_few has to know of all sequences, where they are more than a wave takes in.
template <int KS, bool TREE>
__global__ __launch_bounds__(1024) void k_kv_plan(KvAttend a) {
    __shared__ u64 sums[32];
    __shared__ unsigned items[KV_PLAN_CHUNKS], parts[KV_PLAN_CHUNKS], waves[2][16];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, chunks = (a.batch.n + 63) / 64;
    KvFew<KS, TREE> few;
    u64 all = 0, all_tiles = 0;
    for (int b = t; b < a.batch.n; b += 1024) {
        few.load(a, b);
        all += few.units();
        all_tiles += few.tiles;
    }
    all = kv_wave_sum(all);
    all_tiles = kv_wave_sum(all_tiles);
    if (lane == 0) {
        sums[w] = all;
        sums[16 + w] = all_tiles;
    }
    __syncthreads();
    all = all_tiles = 0;
    for (int i = 0; i < 16; ++i) {
        all += sums[i];
        all_tiles += sums[16 + i];
    }
    const unsigned stretch = KvFew<KS, TREE>::stretch_of(a, all, all_tiles);
    for (int c = w; c < chunks; c += 16) {
        few.load(a, 64 * c + lane);
        const unsigned cuts = few.cuts(stretch), mine = few.tiles * cuts;
        const u64 both = kv_wave_sum(((u64)mine << 32) | (cuts > 1 ? mine : 0u));
        if (lane == 0) {
            items[c] = (unsigned)(both >> 32);
            parts[c] = (unsigned)both;
        }
    }
    __syncthreads();
    const unsigned mine = t < chunks ? items[t] : 0, my_parts = t < chunks ? parts[t] : 0;
    unsigned upto = KvFew<KS, TREE>::running_sum(mine), upto_parts = KvFew<KS, TREE>::running_sum(my_parts);
    if (lane == 63) {
        waves[0][w] = upto;
        waves[1][w] = upto_parts;
    }
    __syncthreads();
    for (int i = 0; i < w; ++i) {
        upto += waves[0][i];
        upto_parts += waves[1][i];
    }
    if (t < chunks) {
        a.plan->items[t] = upto - mine;
        a.plan->parts[t] = upto_parts - my_parts;
    }
    if (t == 0) a.plan->stretch = stretch;
}

// One workgroup for a stretch of a tile's units; its four waves take every fourth of them, each with sums of its own, which are
// joined through LDS in the order of the waves.  Keys and values go straight from memory to registers: no wave reads what another does.
// A tile that is cut is finished by the workgroup that is done last, from all parts, in their order.
// KS: positions of a step.  A wave has one step's operands on their way while it works on the last one's.
// Bound by the reading of keys and values: 64 sequences of one token over 282,144 positions, 32 heads over 8 of 128 in 8 bits, 597 MB, in 120 us, 5.0
// TB/s (a large copy on the same card: 5.0), two over 232,244 in 16 bits, 951 MB, in 177 us, 5.4 TB/s.  Short ones are bound by latency: one
// token over 2,001 positions takes 10 us, of which the join is about 3.
// Up to 64 elements a step of 64 positions, where two waves on a SIMD unit have to have enough on their way (24 sequences of up to 12 rows and 30,000
// positions, 16 bits: 36 us; steps of 32 and three waves 40, four 48), but of codes, which are half the bytes, 32 and four waves (with 64 and two
// 25 and 25 us; 5,261 rows of 40 sequences under a window of 1,000, 12 heads: 49 and 38; 250 rows over 4,000, 16 heads over 4: 24.0 and 17.8.  It
// costs where there are few workgroups: 60 rows over 4,000 12.1 and 14.3 us, 400 rows 23.1 and 26.2).
template <int DP, bool FP8>
constexpr int kv_step() { return DP <= 64 && !FP8 ? 64 : 32; }
template <int DP, bool FP8, bool TREE>
__global__ __launch_bounds__(256, DP <= 64 && FP8 ? 4 : DP <= 128 ? 2 : 1) void k_kv_attend_few(KvAttend a) {
    constexpr int ES = FP8 ? 1 : 2;
    constexpr int KS = kv_step<DP, FP8>(), SUBS = KS / 32, BLOCKS = KS / 16;
    constexpr int NF = FP8 ? DP / 32 : DP / 16;  // 16-byte operands of a lane for 32 keys, and for 32 values
    constexpr int NU = DP / 32;
    constexpr int RS = DP + 4;  // floats of a row in LDS
    __shared__ __attribute__((aligned(16))) float sh[4 * 32 * RS];  // sums of each wave
    __shared__ float sh_m[4 * 32], sh_l[4 * 32];
    __shared__ int sh_last;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    KvTile t;
    int head, from, to, piece, count;  // of the tile's pieces
    unsigned first_part;               // of the tile
    {
        const unsigned item = (unsigned)(a.item0 + blockIdx.x);
        using Few = KvFew<KS, TREE>;
        Few few;
        unsigned stretch, items_before = 0, parts_before = 0;
        int chunk = 0;
        if (a.batch.n <= 64) {
            few.load(a, lane);
            u64 all = few.units(), all_tiles = few.tiles;
            if (a.batch.n > 1) {
                all = kv_wave_sum(all);
                all_tiles = kv_wave_sum(all_tiles);
            }
            stretch = __builtin_amdgcn_readfirstlane(Few::stretch_of(a, all, all_tiles));
        } else {  // the last 64 with no more items before them than this one
            int count = (a.batch.n + 63) / 64;
            while (count > 1) {
                const int step = (count + 63) / 64;
                const bool before = lane * step < count && a.plan->items[chunk + lane * step] <= item;
                const int k = __popcll(__ballot(before)) - 1;  // (the first is 0)
                chunk += k * step;
                count = count - k * step < step ? count - k * step : step;
            }
            stretch = __builtin_amdgcn_readfirstlane(a.plan->stretch);
            items_before = __builtin_amdgcn_readfirstlane(a.plan->items[chunk]);
            parts_before = __builtin_amdgcn_readfirstlane(a.plan->parts[chunk]);
            few.load(a, 64 * chunk + lane);
        }
        const unsigned cuts = few.cuts(stretch), mine = few.tiles * cuts, my_parts = cuts > 1 ? mine : 0;
        const unsigned upto = items_before + (a.batch.n > 1 ? Few::running_sum(mine) : mine);
        const unsigned upto_parts = parts_before + (a.batch.n > 1 ? Few::running_sum(my_parts) : my_parts);
        const u64 over = __ballot(upto > item);
        if (over == 0) return;  // (there are not as many items)
        const int at = __ffsll((long long)over) - 1;
        t.s.b = 64 * chunk + at;
        t.s.first = __builtin_amdgcn_readlane(few.first, at);
        t.s.rows = __builtin_amdgcn_readlane(few.rows, at);
        t.s.length = __builtin_amdgcn_readlane(few.length, at);
        t.s.start = t.s.length - t.s.rows;
        count = __builtin_amdgcn_readlane(cuts, at);
        const unsigned in = item - __builtin_amdgcn_readlane(upto - mine, at);
        if (in >= (unsigned)__builtin_amdgcn_readlane(mine, at)) return;  // (more tiles than 32 bits count)
        unsigned tile;
        if constexpr (TREE) {
            // All tiles read the same stretches: those of a stretch and head follow each other at a distance of eight, so that one XCD reads it once (2 trees of
            // 30 to 50 rows, 4 heads for each of 8, behind 30,000 positions: 115 us, tile after tile 140).
            const unsigned tiles = (unsigned)(t.s.rows * a.group + 31) >> 5, units = (unsigned)(count * a.pool.kv_heads);
            const unsigned eight = __builtin_amdgcn_readfirstlane(in / (8 * tiles)), rest = in - 8 * tiles * eight;
            const unsigned wide = units - 8 * eight < 8 ? units - 8 * eight : 8;
            tile = __builtin_amdgcn_readfirstlane(rest / wide);
            const unsigned unit = 8 * eight + rest - tile * wide;
            piece = __builtin_amdgcn_readfirstlane(unit / (unsigned)a.pool.kv_heads);
            head = unit - piece * a.pool.kv_heads;
        } else {
            // heads first, then pieces: neighbours read the same pages
            const unsigned rest = __builtin_amdgcn_readfirstlane(in / (unsigned)a.pool.kv_heads);
            head = in - rest * a.pool.kv_heads;
            tile = __builtin_amdgcn_readfirstlane(rest / (unsigned)count);
            piece = rest - tile * count;
        }
        first_part = __builtin_amdgcn_readlane(upto_parts - my_parts, at) + (tile * a.pool.kv_heads + head) * count;
        kv_tile<TREE>(a, tile * 32, 32, t);
        int base;
        Few::range_of(a, t.s.start, t.s.length, base);
        if constexpr (TREE) stretch = ((unsigned)__builtin_amdgcn_readlane(few.range, at) + count - 1) / count;  // (its pieces alike)
        from = base + KS * (int)(piece * stretch);
        to = piece == count - 1 ? t.hi : from + KS * (int)stretch;
        if (from < (t.lo & ~(KS - 1))) from = t.lo & ~(KS - 1);
        if (to > t.hi) to = t.hi;
    }

    // this lane's row (of both halves) as the operand Q^T
    const int row = t.row0 + n, token = row / a.group, qh = head * a.group + row % a.group;
    const bool valid = n < t.rows;
    const int pos = t.s.start + token;
    u32x4_t qx[DP / 16];
    unsigned *const masks = (unsigned *)(sh + w * 32 * RS) + 64;  // (TREE) this wave's, behind its scales
    static_assert(64 + 32 * KV_MASK_ROW <= 32 * RS, "room for the masks");
    int depth = 0;
    if constexpr (TREE) depth = kv_mask_row(a, t, valid ? token : 0, valid, masks);
    const bf16_t *const q_row = a.q + (long)(t.s.first + (valid ? token : 0)) * a.q_token + (long)(valid ? qh : 0) * a.q_head;
    auto q_at = [&](int s) { return FP8 ? 16 * (2 * (s >> 1) + h) + 8 * (s & 1) : 16 * s + 8 * h; };
    if (a.vec) {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) qx[s] = *(const u32x4_t *)(q_row + (q_at(s) < a.pool.dim ? q_at(s) : 0));
    } else {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16_t *two = q_row + (q_at(s) < a.pool.dim ? q_at(s) : 0) + 2 * i;
                qx[s][i] = (unsigned)two[0] | ((unsigned)two[1] << 16);
            }
    }

    f32x16_t o[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) o[u] = f32x16_t{};
    float m = -INFINITY, l = 0.f;

    u32x4_t kf[SUBS * NF], vf[SUBS * NF];
    static_assert(!FP8 || KS == 32, "a lane for each key's scale, one for each value's");
    float scale;  // (8 bits) a key's, in the other half of the lanes a value's
    int page[BLOCKS], next_page[BLOCKS];
    // what the table says of the blocks from `at` on; of a block ahead of or beyond what the tile sees, whose page may be given up, of the first or last one
    auto find_pages = [&](int at, int (&p)[BLOCKS]) {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) p[i] = kv_page_entry(a.pool, a.batch, t.s.b, kv_clamp(at + 16 * i, t.lo & ~15, t.hi - 1));
    };
    auto load_keys = [&](int at, const int (&p)[BLOCKS]) {
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            const size_t b0 = kv_block_at(a.pool, kv_is_page(a.pool, p[2 * sub]) ? p[2 * sub] : 0, head, at + 32 * sub),
                         b1 = kv_block_at(a.pool, kv_is_page(a.pool, p[2 * sub + 1]) ? p[2 * sub + 1] : 0, head, at + 32 * sub + 16);
            const char *from_k = a.pool.k + ((lane >> 4) & 1 ? b1 : b0) * ES + h * 256 + (lane & 15) * 16;
#pragma unroll
            for (int s = 0; s < NF; ++s) kf[sub * NF + s] = *(const u32x4_t *)(from_k + s * 512);
        }
        if constexpr (FP8) {
            const int key = lane & (KS - 1);
            size_t from_s = 0;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                const size_t x = kv_scale_at(a.pool, kv_is_page(a.pool, p[i]) ? p[i] : 0, head, at + 16 * i);
                from_s = key >> 4 == i ? x : from_s;
            }
            from_s += key & 15;
            scale = (h ? a.pool.vs : a.pool.ks)[from_s];
        }
    };
    auto load_values = [&](int at, const int (&p)[BLOCKS]) {
#pragma unroll
        for (int blk = 0; blk < BLOCKS; ++blk) {
            const char *from_v = a.pool.v + kv_block_at(a.pool, kv_is_page(a.pool, p[blk]) ? p[blk] : 0, head, at + 16 * blk) * ES + (h * (NF / 2) * 32 + n) * 16;
#pragma unroll
            for (int u = 0; u < NF / 2; ++u) vf[blk * (NF / 2) + u] = *(const u32x4_t *)(from_v + u * 512);
        }
    };
    float *const sh_scales = sh + w * 32 * RS;  // this wave's: keys' [KS], values' [KS]

    // One step: KS positions from `at` on, while the next ones' keys, then values, are fetched, as soon as their registers are free.
    // (Whether there are any is known when this is compiled: what is fetched on one way only would be waited for on both.)
    auto step = [&](int at, auto has_next) __attribute__((always_inline)) {
        constexpr bool more = decltype(has_next)::value;
        f32x16_t s[SUBS];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            s[sub] = f32x16_t{};
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                const u32x4_t x = kf[sub * NF + i];
                if constexpr (FP8) {
                    s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(x[0], x[1]), kv_as_bf16(qx[2 * i]), s[sub], 0, 0, 0);
                    s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(x[2], x[3]), kv_as_bf16(qx[2 * i + 1]), s[sub], 0, 0, 0);
                } else s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_as_bf16(x), kv_as_bf16(qx[i]), s[sub], 0, 0, 0);
            }
        }
        if constexpr (FP8) {  // a lane has one position's scales and needs those of its registers': through LDS
            sh_scales[lane] = scale;
#pragma unroll
            for (int g = 0; g < 4 * SUBS; ++g) {
                const float4 x = *(const float4 *)(sh_scales + 8 * g + 4 * h);
                s[g >> 2][4 * (g & 3)] *= x.x;
                s[g >> 2][4 * (g & 3) + 1] *= x.y;
                s[g >> 2][4 * (g & 3) + 2] *= x.z;
                s[g >> 2][4 * (g & 3) + 3] *= x.w;
            }
        }
        if constexpr (more) load_keys(at + 4 * KS, next_page);

        // register r of a 32 holds position 8 (r / 4) + 4 h + r % 4 of this lane's row
        bool none = false;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) none = none || !kv_is_page(a.pool, page[i]);
        const bool edge = at + KS > t.all_hi || at < t.all_lo || none;
        unsigned seen[SUBS];
        if (edge) {
            if (lane == 0 && none) atomicAdd(a.pool.bad, 1ull);
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                seen[sub] = 0;
                const unsigned own = TREE ? kv_mask_bits(masks, n, at + 32 * sub - t.s.start) >> 4 * h : 0u;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int p = at + 32 * sub + 8 * (r >> 2) + 4 * h + (r & 3);
                    bool sees;
                    if constexpr (TREE) sees = (own >> (8 * (r >> 2) + (r & 3)) & 1) && (a.window == 0 || p >= t.s.start || p > t.s.start + depth - a.window);
                    else sees = p <= pos && (a.window == 0 || p > pos - a.window);
                    if (sees && kv_is_page(a.pool, page[2 * sub + (r >> 3)])) seen[sub] |= 1u << r;
                    s[sub][r] = seen[sub] >> r & 1 ? s[sub][r] : -INFINITY;
                }
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int r = 1; r < 16 * SUBS; ++r) top = fmaxf(top, s[r >> 4][r & 15]);
        top = fmaxf(m, kv_both_halves_max(top));
        if (__ballot(top > m) != 0) {  // (a maximum that stays needs no new sums)
            const float down = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.scale);
            l *= down;
#pragma unroll
            for (int u = 0; u < NU; ++u) o[u] *= down;
            m = top;
        }
        const float base = m == -INFINITY ? 0.f : m * a.scale;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16 * SUBS; ++r) {
            s[r >> 4][r & 15] = __builtin_amdgcn_exp2f(__fmaf_rn(s[r >> 4][r & 15], a.scale, -base));
            sum += s[r >> 4][r & 15];
        }
        l += sum;
        if constexpr (FP8) {
#pragma unroll
            for (int g = 0; g < 4 * SUBS; ++g) {
                const float4 x = *(const float4 *)(sh_scales + KS + 8 * g + 4 * h);
                s[g >> 2][4 * (g & 3)] *= x.x;
                s[g >> 2][4 * (g & 3) + 1] *= x.y;
                s[g >> 2][4 * (g & 3) + 2] *= x.z;
                s[g >> 2][4 * (g & 3) + 3] *= x.w;
            }
            if (edge)
#pragma unroll
                for (int r = 0; r < 16 * SUBS; ++r) s[r >> 4][r & 15] = seen[r >> 4] >> (r & 15) & 1 ? s[r >> 4][r & 15] : 0.f;  // (the scale there may be NaN)
        }
        // Powers are rounded to 16 bits, the operands of the matrix cores' fast products (those of 32 bits have a sixteenth of the rate); the
        // sum that they are divided by is of the unrounded ones.  In relation to the definition in 64 bits outputs are off by 0.0019 to 0.0024
        // where rounding the outputs alone leaves 0.0017.
        bf16x8_t pf[BLOCKS];
#pragma unroll
        for (int r = 0; r < 16 * SUBS; ++r) pf[r >> 3][r & 7] = (__bf16)s[r >> 4][r & 15];
        if (!FP8 && edge) {
            // Nothing times an infinity is NaN: where some rows do not see a position, its value's infinities and NaN are
            // taken out of the product and added, position by position, for the rows that see it.
            bool odd = false;
#pragma unroll
            for (int i = 0; i < SUBS * NF; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) odd = odd || kv_not_finite(vf[i][c]);
            if (__ballot(odd) != 0) {
#pragma unroll
                for (int blk = 0; blk < BLOCKS; ++blk)
#pragma unroll 1
                    for (int slot = 0; slot < 16; ++slot) {  // (the lane half, then the position among its eight)
                        const unsigned half = slot >> 3 == h ? (slot & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
                        const u64 seen_by = __ballot(seen[blk >> 1] >> (8 * (blk & 1) + (slot & 7)) & 1);
                        const bool sees = seen_by >> (n + 32 * (slot >> 3)) & 1;
#pragma unroll
                        for (int u = 0; u < NU; ++u) {
                            u32x4_t x;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const unsigned v = vf[blk * (NF / 2) + u % (NF / 2)][c] & (c == (slot & 7) >> 1 ? half : 0u);
                                x[c] = kv_not_finite(v) ? v : 0u;
                            }
                            const f32x16_t add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_as_bf16(x), pf[blk], f32x16_t{}, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 16; ++r) o[u][r] += sees ? add[r] : 0.f;
                        }
                    }
#pragma unroll
                for (int i = 0; i < SUBS * NF; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if ((vf[i][c] & 0x7F80u) == 0x7F80u) vf[i][c] &= 0xFFFF0000u;
                        if ((vf[i][c] & 0x7F800000u) == 0x7F800000u) vf[i][c] &= 0xFFFFu;
                    }
            }
        }
#pragma unroll
        for (int blk = 0; blk < BLOCKS; ++blk) {
            if constexpr (FP8) {
#pragma unroll
                for (int u = 0; u < NF / 2; ++u) {
                    const u32x4_t x = vf[blk * (NF / 2) + u];
                    o[2 * u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(x[0], x[1]), pf[blk], o[2 * u], 0, 0, 0);
                    o[2 * u + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(x[2], x[3]), pf[blk], o[2 * u + 1], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int u = 0; u < NU; ++u) o[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_as_bf16(vf[blk * NU + u]), pf[blk], o[u], 0, 0, 0);
            }
        }
        if constexpr (more) {
            load_values(at + 4 * KS, next_page);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) page[i] = next_page[i];
        }
    };

    // Pages are looked up two steps ahead.
    int at = from + KS * w;
    if (at < to) {
        int over_next_page[BLOCKS];
        find_pages(at, page);
        find_pages(at + 4 * KS, next_page);
        load_keys(at, page);
        load_values(at, page);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            asm volatile("" : "+v"(qx[i]));  // waited for here, and not at every step along with what has just been asked for
#pragma unroll
            for (int c = 0; c < 4; ++c) qx[i][c] = valid && q_at(i) < a.pool.dim ? qx[i][c] ^ a.negate : 0u;
        }
        for (; at + 4 * KS < to; at += 4 * KS) {
            find_pages(at + 8 * KS, over_next_page);
            step(at, std::true_type());
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) next_page[i] = over_next_page[i];
        }
        step(at, std::false_type());
    }

    l = kv_both_halves_sum(l);
    if (h == 0) {
        sh_m[w * 32 + n] = m * a.scale;
        sh_l[w * 32 + n] = l;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4 *)(sh + (w * 32 + n) * RS + 32 * u + 8 * g + 4 * h) = make_float4(o[u][4 * g], o[u][4 * g + 1], o[u][4 * g + 2], o[u][4 * g + 3]);
    __syncthreads();
    float *part = a.parts + (size_t)(first_part + piece) * KV_PART(DP);
    for (int i = threadIdx.x; i < t.rows * (DP / 4); i += 256) {
        const int r = i / (DP / 4), d = i % (DP / 4) * 4;
        float mj[4], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mj[j] = sh_m[j * 32 + r];
            top = fmaxf(top, mj[j]);
        }
        float sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) kv_add_part(mj[j], top, sh_l[j * 32 + r], *(const float4 *)(sh + (j * 32 + r) * RS + d), sum, x);
        if (count <= 1) kv_finish(a, t, head, r, d, top, sum, x);
        else {
            kv_leave(part + r * DP + d, x.x, x.y);
            kv_leave(part + r * DP + d + 2, x.z, x.w);
            if (d == 0) kv_leave(part + 32 * DP + 2 * r, top, sum);
        }
    }
    if (count > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's numbers are where all workgroups see them
        __syncthreads();
        if (threadIdx.x == 0) {
            sh_last = atomicAdd(a.arrived + first_part, 1u) == (unsigned)(count - 1);
            if (sh_last) a.arrived[first_part] = 0;  // (for the next call: nobody else comes)
        }
        __syncthreads();
        if (sh_last) {
            const float *parts = a.parts + (size_t)first_part * KV_PART(DP);
            auto part_of = [&](int s) { return parts + (size_t)s * KV_PART(DP); };
            // few rows leave threads idle: these take every second, fourth or eighth part
            const int work = t.rows * (DP / 4), across = work > 128 ? 1 : work > 64 ? 2 : work > 32 ? 4 : 8, wide = 256 / across;
            const int mine = threadIdx.x & (wide - 1), lead = threadIdx.x / wide;
            // ITEMS of a thread's fours of sums at a time, from part `lead` on every `across`th one, PARTS of them on their way at once (what is beyond the
            // last weighs nothing): two by five for whole tiles, of which four or five parts are usual (40 rows over 400 positions, 16 heads: 13.2 us,
            // four by four 12.6, one by eight 15.7; 24 drafts of up to 9 tokens: 25.8, 27.1, 25.9)
            auto add_parts = [&](auto items, auto parts_at_once, int i0, float (&top)[decltype(items)::value], float (&sum)[decltype(items)::value],
                                 float4 (&x)[decltype(items)::value]) __attribute__((always_inline)) {
                constexpr int ITEMS = decltype(items)::value, PARTS = decltype(parts_at_once)::value;
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    top[k] = -INFINITY;
                    sum[k] = 0.f;
                    x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                for (int s0 = lead; s0 < count; s0 += PARTS * across) {
                    float2 ml[ITEMS][PARTS], y[ITEMS][PARTS], z[ITEMS][PARTS];
#pragma unroll
                    for (int k = 0; k < ITEMS; ++k) {
                        const int i = i0 + k * wide < work ? i0 + k * wide : 0, r = i / (DP / 4), d = i % (DP / 4) * 4;
#pragma unroll
                        for (int j = 0; j < PARTS; ++j) {
                            const float *p = part_of(s0 + j * across < count ? s0 + j * across : 0);
                            ml[k][j] = kv_found(p + 32 * DP + 2 * r);
                            y[k][j] = kv_found(p + r * DP + d);
                            z[k][j] = kv_found(p + r * DP + d + 2);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < ITEMS; ++k) {
                        float now = top[k];
#pragma unroll
                        for (int j = 0; j < PARTS; ++j)
                            if (s0 + j * across < count) now = fmaxf(now, ml[k][j].x);
                        const float4 had = x[k];
                        const float had_sum = sum[k];
                        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                        sum[k] = 0.f;
                        kv_add_part(top[k], now, had_sum, had, sum[k], x[k]);
#pragma unroll
                        for (int j = 0; j < PARTS; ++j)
                            if (s0 + j * across < count)
                                kv_add_part(ml[k][j].x, now, ml[k][j].y, make_float4(y[k][j].x, y[k][j].y, z[k][j].x, z[k][j].y), sum[k], x[k]);
                        top[k] = now;
                    }
                }
            };
            if (across == 1) {
                constexpr int ITEMS = 2;
                for (int i0 = mine; i0 < work; i0 += ITEMS * wide) {
                    float top[ITEMS], sum[ITEMS];
                    float4 x[ITEMS];
                    add_parts(std::integral_constant<int, ITEMS>(), std::integral_constant<int, 5>(), i0, top, sum, x);
#pragma unroll
                    for (int k = 0; k < ITEMS; ++k) {
                        const int i = i0 + k * wide;
                        if (i < work) kv_finish(a, t, head, i / (DP / 4), i % (DP / 4) * 4, top[k], sum[k], x[k]);
                    }
                }
            } else {
                float top[1], sum[1];
                float4 x[1];
                add_parts(std::integral_constant<int, 1>(), std::integral_constant<int, 8>(), mine, top, sum, x);
                *(float4 *)(sh + 8 * threadIdx.x) = x[0];
                *(float2 *)(sh + 8 * threadIdx.x + 4) = make_float2(top[0], sum[0]);
                __syncthreads();
                if (lead == 0 && mine < work) {
                    for (int j = 1; j < across; ++j) top[0] = fmaxf(top[0], sh[8 * (j * wide + mine) + 4]);
                    x[0] = make_float4(0.f, 0.f, 0.f, 0.f);
                    sum[0] = 0.f;
                    for (int j = 0; j < across; ++j) {
                        const float *other = sh + 8 * (j * wide + mine);
                        kv_add_part(other[4], top[0], other[5], *(const float4 *)other, sum[0], x[0]);
                    }
                    kv_finish(a, t, head, mine / (DP / 4), mine % (DP / 4) * 4, top[0], sum[0], x[0]);
                }
            }
        }
    }
}

// Sequences of more rows of work: a prompt's chunk.  One workgroup for a tile of NW * 32 rows, each wave for 32 of them over all
// positions, in stages of KEYS.  A wave goes through a stage in two phases with a barrier behind each: one of products, the scores of the next
// stage and the sums of this one, and one of powers, of the next stage's scores.  Both take about as long, the one on the matrix cores, the
// other on the vector units, and of the two waves on a SIMD unit one is always a phase behind: each has the unit that the other leaves.
// (4,096 rows of 32 heads of 128 behind 8,193: 660 us, 1,040 TFLOP/s; in step, with one barrier a stage, both waited for the same unit: 785 us.)
// Keys and values pass through LDS, two stages of each: keys are read a stage earlier than values.  A wave writes its share of the next ones
// and asks for those after them in its phase of products, whose vector units are idle.  Codes become 16-bit numbers (exactly) on the way in.
template <int DP, bool FP8>
struct KvChunk {
    // Waves: two on each SIMD unit.  Of 64 elements they are those of two workgroups (of one of eight waves 1,500 rows at most and windows of 1,000
    // took 84 us, not 61; three workgroups do not have the registers: 68), of more than 128 there is room for one.
    static constexpr int NW = DP == 128 ? 8 : 4;
    static constexpr int NT = 64 * NW, ROWS = 32 * NW, PER_SIMD = DP <= 128 ? 2 : 1;
    static constexpr int KEYS = DP <= 192 ? 64 : 32, SUBS = KEYS / 32, BLOCKS = KEYS / 16;
    static constexpr int ES = FP8 ? 1 : 2;
    static constexpr int NS = DP / 16, NU = DP / 32;
    static constexpr int BLOCK_CHUNKS = DP * ES;           // 16-byte chunks of a block of 16 positions in memory
    static constexpr int CHUNKS = BLOCKS * BLOCK_CHUNKS;   // of a stage's keys
    static constexpr int NL = (CHUNKS + NT - 1) / NT;      // of a thread
    static constexpr int HALF = KEYS * DP * 2;             // bytes of a stage's keys in LDS
    static constexpr int SCALES = 4 * HALF;                // (8 bits) where the scales begin: of four stages, keys' and values'
    static constexpr int FOUND = SCALES + (FP8 ? 4 * 2 * KEYS * 4 : 0);  // three words: a value that is not finite, a maximum that grew too far, a page that is none
    static constexpr int LDS = FOUND + 16 + 4 * BLOCKS * 4;  // and which blocks of four stages have a page
    static constexpr int MASKS = ROWS * KV_MASK_ROW * 4;     // (trees) behind that
    static_assert(LDS + MASKS <= 160 * 1024 && NT >= 2 * KEYS, "fits LDS; a thread for each scale");
};
#define KV_CHUNK_PART(ROWS, DP) ((size_t)(ROWS) * ((DP) + 2))

struct KvPieces {
    long slots, slot0;
    int ways;      // a tile's positions are cut into at most so many pieces
    int at_once;   // (trees) workgroups that run at once
    int room;      // parts that the workspace holds (0: no tile is cut)
};
struct KvPiece {
    int head, piece, pieces;
    int from, blocks, per;  // where the tile's positions begin, its blocks of KEYS positions, those of a piece
    long part, next_part;   // where the tile's first part is, and how far apart they are
};
#define KV_PIECE_LEAST 256  // positions
// A phase of products: operands are read so many products ahead (4: 1% slower, 8: 2%), and the work of the next stages begins behind this one.
#define KV_AHEAD 6
#define KV_FORWARD 4
// What may pass a product in the compiler's order: vector and scalar arithmetic, memory reads and writes, writes to LDS; reads of LDS
// and products may not.  (Nothing bounded, the compiler moves operands' reads to where they are waited for: 8% slower.)
#define KV_MASK 0x276
// The tile of a slot, of `rows` rows of work, and how its positions are cut: pieces of `per` blocks of KEYS positions from `from` on.
template <int ROWS, int KEYS, bool TREE>
__device__ __forceinline__ bool kv_chunk_tile(const KvAttend &a, const KvPieces &p, long slot, KvTile &t, int &from, int &blocks, int &per, int &pieces) {
    constexpr int SHIFT = ROWS == 256 ? 8 : 7;
    static_assert(ROWS == 1 << SHIFT, "rows of a tile");
    t.s = kv_sequence_of(a.batch, slot, a.group, SHIFT, 1);
    const long j = slot - kv_slots_before(t.s.first, t.s.b, a.group, SHIFT, 1), work = (long)t.s.rows * a.group;
    if (j < 0 || j * ROWS >= work || work <= a.few || (TREE && t.s.rows > SISO_KV_TREE)) return false;
    kv_tile<TREE>(a, (int)(j * ROWS), ROWS, t);
    from = t.lo & ~15;  // (no block that nobody sees: its page may be given up)
    blocks = t.hi > from ? (t.hi - from + KEYS - 1) / KEYS : 0;
    per = (blocks + p.ways - 1) / p.ways;
    if (per < KV_PIECE_LEAST / KEYS) per = KV_PIECE_LEAST / KEYS;
    pieces = blocks > 0 ? (blocks + per - 1) / per : 1;
    return true;
}

// Trees of up to 64 sequences: every workgroup knows all lengths, and cuts the tiles so that all pieces together are as many as run at once, or twice as many,
// and so on where there are more tiles than that: the smallest number of blocks with which they are no more.  (`tile_of`: number `index` counts tiles
// and heads, not pieces.)  All tiles of a sequence are cut as its whole length is.  False: there are not as many.
// (24 trees of 35 to 64 rows, 4 heads for each of 8, behind 2,000 to 6,000 positions in 8 bits: 176 us, cut by the tiles that are likely 227.)
template <int ROWS, int KEYS>
__device__ __forceinline__ bool kv_tree_piece(const KvAttend &a, const KvPieces &p, long index, bool tile_of, KvTile &t, KvPiece &k) {
    const int lane = threadIdx.x & 63, heads = a.pool.kv_heads;
    const KvSequence s = kv_sequence(a.batch, lane < a.batch.n ? lane : a.batch.n - 1);
    const bool has = lane < a.batch.n && s.rows > 0 && s.rows <= SISO_KV_TREE;
    const int from = kv_window_from(a, s.start) & ~15;  // (no block that nobody sees: its page may be given up)
    const unsigned tiles = has ? ((unsigned)(s.rows * a.group) + ROWS - 1) / ROWS * (unsigned)heads : 0u;
    const unsigned blocks = s.length > from ? ((unsigned)(s.length - from) + KEYS - 1) / KEYS : 0u;
    auto sum = [](auto v) __attribute__((always_inline)) { return wave_fold(v, [](auto x, auto y) __attribute__((always_inline)) { return x + y; }); };
    auto most = [](unsigned v) __attribute__((always_inline)) { return wave_fold(v, [](unsigned x, unsigned y) __attribute__((always_inline)) { return x > y ? x : y; }); };
    const unsigned all = sum(tiles), top = most(tiles && blocks ? blocks : 1u), goal = (all + p.at_once - 1) / p.at_once * p.at_once;
    if (all == 0) return false;
    auto cut = [&](unsigned by) __attribute__((always_inline)) { return blocks ? (blocks + by - 1) / by : 1u; };
    unsigned per = top;
    if (tile_of) per = *(const unsigned *)a.plan;  // (what the pieces' workgroups found)
    else if (goal <= (unsigned)p.room) {
        const u64 work = sum((u64)tiles * blocks);
        unsigned low = (unsigned)((work + goal - 1) / goal);  // (fewer are too many pieces)
        if (low < KV_PIECE_LEAST / KEYS) low = KV_PIECE_LEAST / KEYS;
        while (low < per) {
            const unsigned middle = (low + per) / 2;
            if (sum(tiles * cut(middle)) <= goal) per = middle;
            else low = middle + 1;
        }
        per = per > low ? per : low;
    }
    per = __builtin_amdgcn_readfirstlane(per);
    if (!tile_of && index == 0 && threadIdx.x == 0) *(unsigned *)a.plan = per;
    const unsigned pieces = cut(per), mine = tile_of ? tiles : tiles * pieces;
    unsigned upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned x = __shfl_up(upto, off);
        if (lane >= off) upto += x;
    }
    unsigned before_parts = upto - mine;  // parts of the sequences before
    if (tile_of) {
        before_parts = tiles * pieces;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const unsigned x = __shfl_up(before_parts, off);
            if (lane >= off) before_parts += x;
        }
        before_parts -= tiles * pieces;
    }
    const u64 over = __ballot((long)upto > index);
    if (over == 0) return false;
    const int at = __ffsll((long long)over) - 1;
    t.s.b = at;
    t.s.first = __builtin_amdgcn_readlane(s.first, at);
    t.s.rows = __builtin_amdgcn_readlane(s.rows, at);
    t.s.length = __builtin_amdgcn_readlane(s.length, at);
    t.s.start = t.s.length - t.s.rows;
    const unsigned in = (unsigned)index - (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), at), of_tiles = (unsigned)__builtin_amdgcn_readlane((int)tiles, at);
    k.piece = (int)(in / of_tiles);  // heads first, then tiles: neighbours read the same pages
    const unsigned tile = in - (unsigned)k.piece * of_tiles;
    k.head = (int)(tile % (unsigned)heads);
    k.pieces = __builtin_amdgcn_readlane((int)pieces, at);
    k.from = __builtin_amdgcn_readlane(from, at);
    k.per = (int)per;
    k.part = (long)(unsigned)__builtin_amdgcn_readlane((int)before_parts, at) + tile;
    k.next_part = of_tiles;
    kv_tile<true>(a, (int)(tile / (unsigned)heads) * ROWS, ROWS, t);
    // (a tile ends where its own rows do: of rows below position 0 there is no block, and no entry of the table.  Pieces behind that are empty.)
    k.blocks = t.hi > k.from ? (t.hi - k.from + KEYS - 1) / KEYS : 0;
    return true;
}
// The piece of a workgroup of k_kv_attend_chunk, or the tile of one of k_kv_attend_join (`tile_of`).
template <int ROWS, int KEYS, bool TREE>
__device__ __forceinline__ bool kv_chunk_piece(const KvAttend &a, const KvPieces &p, bool tile_of, KvTile &t, KvPiece &k) {
    if constexpr (TREE)
        if (a.batch.n <= 64) return kv_tree_piece<ROWS, KEYS>(a, p, p.slot0 + blockIdx.x, tile_of, t, k);
    // (the tiles of one kv head follow each other at a distance of kv_heads, those that see most first)
    const int heads = a.pool.kv_heads, ways = tile_of ? 1 : p.ways;
    const long at_slot = blockIdx.x / (heads * ways);
    k.head = blockIdx.x % heads;
    k.piece = blockIdx.x / heads % ways;
    k.part = at_slot * p.ways * heads + k.head;
    k.next_part = heads;
    return kv_chunk_tile<ROWS, KEYS, TREE>(a, p, p.slot0 + p.slots - 1 - at_slot, t, k.from, k.blocks, k.per, k.pieces) && k.piece < k.pieces;
}

template <int DP, bool FP8, bool TREE>
__global__ __launch_bounds__((KvChunk<DP, FP8>::NT), (KvChunk<DP, FP8>::PER_SIMD)) void k_kv_attend_chunk(KvAttend a, KvPieces p) {
    using C = KvChunk<DP, FP8>;
    constexpr int KEYS = C::KEYS, SUBS = C::SUBS, BLOCKS = C::BLOCKS, NS = C::NS, NU = C::NU, NL = C::NL;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    KvTile t;
    KvPiece k;
    if (!kv_chunk_piece<C::ROWS, KEYS, TREE>(a, p, false, t, k)) return;
    const int head = k.head, pieces = k.pieces, done = k.piece * k.per, first = k.from + done * KEYS, stages = k.blocks - done < k.per ? k.blocks - done : k.per;

    // this wave's rows; `any`: there are some
    const bool any = w * 32 < t.rows;
    KvTile mine;
    mine.s = t.s;
    kv_tile<TREE>(a, any ? t.row0 + w * 32 : t.row0, 32, mine);
    const int row = t.row0 + w * 32 + n;
    const bool valid = row < t.row0 + t.rows;
    const int token = valid ? row / a.group : 0, qh = head * a.group + (valid ? row % a.group : 0), pos = t.s.start + token;
    auto q_at = [&](int s) { return FP8 ? 16 * (2 * (s >> 1) + h) + 8 * (s & 1) : 16 * s + 8 * h; };
    unsigned *const masks = (unsigned *)(lds + C::LDS) + w * 32 * KV_MASK_ROW;  // (TREE) this wave's
    int depth = 0;
    if constexpr (TREE) depth = kv_mask_row(a, t, token, valid, masks);
    u32x4_t qx[NS];
    {
        const bf16_t *q_row = a.q + (long)(t.s.first + token) * a.q_token + (long)qh * a.q_head;
        if (a.vec) {
#pragma unroll
            for (int s = 0; s < NS; ++s) qx[s] = *(const u32x4_t *)(q_row + (q_at(s) < a.pool.dim ? q_at(s) : 0));
        } else {
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bf16_t *two = q_row + (q_at(s) < a.pool.dim ? q_at(s) : 0) + 2 * i;
                    qx[s][i] = (unsigned)two[0] | ((unsigned)two[1] << 16);
                }
        }
    }
    f32x16_t o[NU];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < NU; ++u) o[u] = f32x16_t{};

    // ---- stages: pages from the table, a stage from memory to registers, from registers to LDS
    // Every thread looks up the pages of its own chunks, a stage before it fetches them: what the scalar unit would have to work out
    // for all of them takes longer than the products.  Stages beyond the last are fetched and written as others (at positions of the last page), and not read.
    const int late = C::NW == 8 ? w >> 2 : 0;  // this wave is a phase behind
    u32x4_t gk[NL], gv[NL];
    float gs = 0.f;
    int entry[NL], scale_entry = 0;       // what the table says of the stage whose keys are fetched next
    const char *k_at[NL], *v_at[NL];      // where this thread's chunks of its keys are; of the values of the one before
    unsigned k_held = 0, v_held = 0, gv_held = 0;  // a bit for each of them that is in a page of the cache; of those in gv
    // What hardly ever is, is only looked for, in `odd`, and the tile done again with care if it is found: pages that are none, and values that
    // are not finite (nothing times an infinity is NaN, so they must not reach the rows that do not see them).
    bool careful = false;
    unsigned odd = 0;
    const int *const table = a.batch.pages + (long)t.s.b * a.batch.width;
    const long page_bytes = ((long)a.pool.kv_heads << a.pool.shift) * DP * C::ES, head_bytes = ((long)head << a.pool.shift) * DP * C::ES;
    const int in_page = (1 << a.pool.shift) - 1;
    auto position = [&](int stage, int blk) {
        const int p = first + stage * KEYS + 16 * blk;
        return p < t.hi ? p : (t.hi - 1) & ~15;
    };
    auto look_up = [&](int stage) {
#pragma unroll
        for (int i = 0; i < NL; ++i) entry[i] = table[position(stage, (threadIdx.x + C::NT * i) / C::BLOCK_CHUNKS % BLOCKS) >> a.pool.shift];
        if constexpr (FP8) scale_entry = table[position(stage, (threadIdx.x & (KEYS - 1)) >> 4) >> a.pool.shift];
    };
    auto fetch_keys = [&](int stage) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int c = threadIdx.x + C::NT * i, at = position(stage, c / C::BLOCK_CHUNKS % BLOCKS);
            const bool held = kv_is_page(a.pool, entry[i]);
            k_held = (k_held & ~(1u << i)) | (unsigned)held << i;
            odd |= held ? 0u : 1u;
            const long off = (held ? entry[i] : 0) * page_bytes + head_bytes + ((at & in_page) >> 4) * (C::BLOCK_CHUNKS * 16) + c % C::BLOCK_CHUNKS * 16;
            gk[i] = *(const u32x4_t *)(a.pool.k + off);
            k_at[i] = a.pool.v + off;
        }
        if constexpr (FP8) {
            const int key = threadIdx.x & (KEYS - 1), at = position(stage, key >> 4);
            const bool held = kv_is_page(a.pool, scale_entry);
            const float *scales = threadIdx.x & KEYS ? a.pool.vs : a.pool.ks;
            gs = scales[(((long)(held ? scale_entry : 0) * a.pool.kv_heads + head) << a.pool.shift) + (at & in_page) + (key & 15)];
            gs = held ? gs : 0.f;
        }
    };
    auto fetch_values = [&]() {
#pragma unroll
        for (int i = 0; i < NL; ++i) gv[i] = *(const u32x4_t *)v_at[i];
        gv_held = v_held;
    };
    auto next = [&]() {  // the stage whose keys are fetched becomes that whose values are
#pragma unroll
        for (int i = 0; i < NL; ++i) v_at[i] = k_at[i];
        v_held = k_held;
    };
    int *const found = (int *)(lds + C::FOUND);
    int *const held = found + 4;  // [4][BLOCKS]: of four stages the blocks that have a page
    auto put_keys = [&](int stage) __attribute__((always_inline)) {
        char *k = lds + (stage & 1) * C::HALF;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int c = threadIdx.x + C::NT * i, blk = c / C::BLOCK_CHUNKS, r = c % C::BLOCK_CHUNKS;
            if (!(C::CHUNKS % C::NT == 0 || c < C::CHUNKS)) continue;
            if constexpr (FP8) {
                // chunk (2 t + h) of 16 codes and a token; two operands of 8
                const int kc = r >> 4, key = r & 15, even = 2 * (2 * (kc >> 1)) + (kc & 1);
                *(bf16x8_t *)(k + blk * 32 * DP + (even * 16 + key) * 16) = kv_codes_bf16(gk[i][0], gk[i][1]);
                *(bf16x8_t *)(k + blk * 32 * DP + ((even + 2) * 16 + key) * 16) = kv_codes_bf16(gk[i][2], gk[i][3]);
            } else *(u32x4_t *)(k + c * 16) = gk[i];
        }
        if (FP8 && (C::NT == 2 * KEYS || threadIdx.x < 2 * KEYS)) ((float *)(lds + C::SCALES))[(stage & 3) * 2 * KEYS + threadIdx.x] = gs;
    };
    auto put_values = [&](int stage) __attribute__((always_inline)) {
        char *v = lds + (2 + (stage & 1)) * C::HALF;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int c = threadIdx.x + C::NT * i, blk = c / C::BLOCK_CHUNKS, r = c % C::BLOCK_CHUNKS;
            if constexpr (!FP8)
#pragma unroll
                for (int k = 0; k < 4; ++k) odd |= (gv[i][k] & 0x7F807F80u) + 0x00800080u;  // (the top bit of a half: its exponent is all ones)
            if (!(C::CHUNKS % C::NT == 0 || c < C::CHUNKS)) continue;
            if constexpr (FP8) {
                // [h][dimension / 64][32] of two operands
                const int vh = r / (DP / 2), vu = r % (DP / 2) >> 5, vm = r & 31;
                *(bf16x8_t *)(v + blk * 32 * DP + (vh * DP + 64 * vu + vm) * 16) = kv_codes_bf16(gv[i][0], gv[i][1]);
                *(bf16x8_t *)(v + blk * 32 * DP + (vh * DP + 64 * vu + 32 + vm) * 16) = kv_codes_bf16(gv[i][2], gv[i][3]);
            } else *(u32x4_t *)(v + c * 16) = gv[i];
        }
    };
    auto take_care = [&](int stage) {  // before these: of the stage whose keys are put, which blocks have a page; values that are numbers only
#pragma unroll 1
        for (int i = 0; i < NL; ++i) {
            const int c = threadIdx.x + C::NT * i, blk = c / C::BLOCK_CHUNKS;
            if (c >= C::CHUNKS || c % C::BLOCK_CHUNKS != 0) continue;
            held[(stage & 3) * BLOCKS + blk] = k_held >> i & 1;
            if (!(k_held >> i & 1) && stage < stages) atomicAdd(a.pool.bad, 1ull);
        }
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                unsigned x = gv_held >> i & 1 ? gv[i][c] : 0u;
                if (!FP8 && (x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
                if (!FP8 && (x & 0x7F800000u) == 0x7F800000u) x &= 0xFFFFu;
                gv[i][c] = x;
            }
    };

    // ---- a stage's work
    auto keys_at = [&](int stage, int sub, int i) { return lds + (stage & 1) * C::HALF + (lane >> 4 & 1) * 32 * DP + h * 256 + (lane & 15) * 16 + sub * 64 * DP + i * 512; };
    auto values_at = [&](int stage, int blk, int u) { return lds + (2 + (stage & 1)) * C::HALF + blk * 32 * DP + (h * DP + 32 * u + n) * 16; };
    auto scaled = [&](int stage, int which, f32x16_t (&s)[SUBS]) __attribute__((always_inline)) {
        if constexpr (FP8)
#pragma unroll
            for (int g = 0; g < 4 * SUBS; ++g) {
                const float4 x = *(const float4 *)((const float *)(lds + C::SCALES) + ((stage & 3) * 2 + which) * KEYS + 8 * g + 4 * h);
                s[g >> 2][4 * (g & 3)] *= x.x;
                s[g >> 2][4 * (g & 3) + 1] *= x.y;
                s[g >> 2][4 * (g & 3) + 2] *= x.z;
                s[g >> 2][4 * (g & 3) + 3] *= x.w;
            }
    };
    auto scores = [&](int stage, f32x16_t (&s)[SUBS]) __attribute__((always_inline)) {
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            s[sub] = f32x16_t{};
#pragma unroll
            for (int i = 0; i < NS; ++i)
                s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t *)keys_at(stage, sub, i), kv_as_bf16(qx[i]), s[sub], 0, 0, 0);
        }
    };
    auto add_values = [&](int stage, const bf16x8_t (&pf)[BLOCKS]) __attribute__((always_inline)) {
#pragma unroll
        for (int blk = 0; blk < BLOCKS; ++blk)
#pragma unroll
            for (int u = 0; u < NU; ++u) o[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t *)values_at(stage, blk, u), pf[blk], o[u], 0, 0, 0);
    };
    // A stage's phase of powers: its scores become operands of the products with its values.  Rows are weighed against the maximum of the first
    // stage in which they see something, as long as they can be (see below).
    // (rounded to 16 bits for them, as in k_kv_attend_few)
    bf16x8_t pf[BLOCKS];
    float peak = -INFINITY;
    auto weigh = [&](int stage, f32x16_t (&s)[SUBS]) __attribute__((always_inline)) {
        const int at = first + stage * KEYS;
        const bool edge = at + KEYS > mine.all_hi || at < mine.all_lo || careful;
        unsigned seen[SUBS];
        scaled(stage, 0, s);
        if (edge) {
            const u64 bits = careful ? __ballot(held[(stage & 3) * BLOCKS + (lane & (BLOCKS - 1))] != 0) : ~0ull;  // (bit `blk` is block blk's)
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                seen[sub] = 0;
                const unsigned own = TREE ? kv_mask_bits(masks, n, at + 32 * sub - t.s.start) >> 4 * h : 0u;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int p = at + 32 * sub + 8 * (r >> 2) + 4 * h + (r & 3);
                    bool sees;
                    if constexpr (TREE) sees = (own >> (8 * (r >> 2) + (r & 3)) & 1) && (a.window == 0 || p >= t.s.start || p > t.s.start + depth - a.window);
                    else sees = p <= pos && (a.window == 0 || p > pos - a.window);
                    if (sees && (bits >> (2 * sub + (r >> 3)) & 1)) seen[sub] |= 1u << r;
                    s[sub][r] = seen[sub] >> r & 1 ? s[sub][r] : -INFINITY;
                }
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int r = 1; r < 16 * SUBS; ++r) top = fmaxf(top, s[r >> 4][r & 15]);
        top = kv_both_halves_max(top);
        peak = fmaxf(peak, top);
        m = m == -INFINITY ? top : m;
        const float base = m == -INFINITY ? 0.f : m * a.scale;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16 * SUBS; ++r) {
            s[r >> 4][r & 15] = __builtin_amdgcn_exp2f(__fmaf_rn(s[r >> 4][r & 15], a.scale, -base));
            sum += s[r >> 4][r & 15];
        }
        l += sum;
        scaled(stage, 1, s);
        if (FP8 && edge)  // (the scale of what nobody sees may be NaN)
#pragma unroll
            for (int r = 0; r < 16 * SUBS; ++r) s[r >> 4][r & 15] = seen[r >> 4] >> (r & 15) & 1 ? s[r >> 4][r & 15] : 0.f;
#pragma unroll
        for (int r = 0; r < 16 * SUBS; ++r) pf[r >> 3][r & 7] = (__bf16)s[r >> 4][r & 15];
    };

#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) qx[i][c] = valid && q_at(i) < a.pool.dim ? qx[i][c] ^ a.negate : 0u;
    // The sums are changed by the products and by nothing else: were they brought down where a maximum grows, the compiler would move
    // all of them from registers to registers in every stage.  A maximum that grows too far, to powers that could leave the range, has the
    // tile done again, with the maxima that are known by then.  Pages that are none are read as the first page in the first
    // turn: its maxima do not count then, the careful turn begins without any, and there may be a third.
#pragma unroll 1
    for (int turn = 0; stages > 0; ++turn) {
        if (threadIdx.x < 3) found[threadIdx.x] = 0;
        if (threadIdx.x < 4 * BLOCKS) held[threadIdx.x] = 1;
        __syncthreads();
        odd = 0;
        look_up(0);
        fetch_keys(0);
        look_up(1);
        if (careful) take_care(0);  // (no values yet)
        put_keys(0);
        next();
        fetch_keys(1);
        fetch_values();
        next();
        look_up(2);
        __syncthreads();
        if (late) __syncthreads();
        // what was fetched goes to LDS: keys that the next phase of products reads and values of the one after; the next are asked for
        auto forward = [&](int i) __attribute__((always_inline)) {
            put_keys(i + 2);
            put_values(i + 1);
            fetch_keys(i + 3);
            fetch_values();
            next();
            look_up(i + 4);
        };
        f32x16_t s[SUBS];
        if (careful) take_care(1);
        forward(-1);
        scores(0, s);
        __syncthreads();
        weigh(0, s);
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i + 1 < stages; ++i) {
            if (careful) take_care(i + 2);
            __builtin_amdgcn_sched_barrier(0);
            // scores and sums in turn, so that no product waits for the one before it
            constexpr int PRODUCTS = SUBS * NS + BLOCKS * NU;
            static_assert(SUBS * NS == BLOCKS * NU, "as many scores as sums");
            bf16x8_t x[KV_AHEAD];
            auto operand = [&](int c) __attribute__((always_inline)) {
                return *(const bf16x8_t *)(c & 1 ? values_at(i, (c >> 1) / NU, (c >> 1) % NU) : keys_at(i + 1, (c >> 1) % SUBS, (c >> 1) / SUBS));
            };
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) s[sub] = f32x16_t{};
#pragma unroll
            for (int c = 0; c < KV_AHEAD; ++c) x[c] = operand(c);
#pragma unroll
            for (int c = 0; c < PRODUCTS; ++c) {
                const int d = c >> 1;
                if (c & 1) o[d % NU] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c % KV_AHEAD], pf[d / NU], o[d % NU], 0, 0, 0);
                else s[d % SUBS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c % KV_AHEAD], kv_as_bf16(qx[d / SUBS]), s[d % SUBS], 0, 0, 0);
                if (c + KV_AHEAD < PRODUCTS) x[c % KV_AHEAD] = operand(c + KV_AHEAD);
                __builtin_amdgcn_sched_barrier(KV_MASK);
                if (c == KV_FORWARD) {
                    forward(i);
                    __builtin_amdgcn_sched_barrier(KV_MASK);
                }
            }
            __syncthreads();
            weigh(i + 1, s);
            __syncthreads();
        }
        add_values(stages - 1, pf);
        if (C::NW == 8 && !late) __syncthreads();
        // Powers beyond 2^32, or sums that left the range with powers above one?
        bool again = (peak - m) * a.scale > 32.f;
        if ((peak - m) * a.scale > 0.f) {
            again = again || !(fabsf(l) <= 3.4e38f);
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) again = again || !(fabsf(o[u][r]) <= 3.4e38f);
        }
        if (any && again) found[1] = 1;
        if (odd & 0x80008000u) found[0] = 1;
        if (odd & 1u) found[2] = 1;
        __syncthreads();
        const int grown = found[1], no_page = found[2], strange = found[0] | no_page;
        __syncthreads();
        if (turn == 0 ? !(grown | strange) : turn > 1 || !(grown & no_page)) break;
        careful = strange != 0;
        if (turn == 0 && no_page) peak = -INFINITY;
        m = peak;
        l = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u) o[u] = f32x16_t{};
    }
    if (!FP8 && any && careful) {  // values that were taken out, for the rows that see them: whatever their weight, they decide
        const int past = first + stages * KEYS, to = mine.hi < past ? mine.hi : past;
#pragma unroll 1
        for (int at = mine.lo > first ? mine.lo & ~15 : first; at < to; at += 16) {
            const int e = kv_page_entry(a.pool, a.batch, t.s.b, at);
            if (!kv_is_page(a.pool, e)) continue;
            const bf16_t *block = (const bf16_t *)a.pool.v + kv_block_at(a.pool, e, head, at);
            bool odd = false;
            for (int c = lane; c < 2 * DP; c += 64) {
                const u32x4_t x = *(const u32x4_t *)(block + c * 8);
#pragma unroll
                for (int k = 0; k < 4; ++k) odd = odd || kv_not_finite(x[k]);
            }
            if (__ballot(odd) == 0) continue;
#pragma unroll 1
            for (int key = 0; key < 16; ++key) {
                const int p = at + key;
                bool sees;
                if constexpr (TREE) sees = (kv_mask_bits(masks, n, p - t.s.start) & 1) && (a.window == 0 || p >= t.s.start || p > t.s.start + depth - a.window);
                else sees = p <= pos && (a.window == 0 || p > pos - a.window);
                const bf16_t *v = block + (size_t)kv_half(key) * DP * 8 + kv_slot(key);
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bf16_t x = v[(32 * u + 8 * (r >> 2) + 4 * h + (r & 3)) * 8];
                        if ((x & 0x7F80u) == 0x7F80u && sees) o[u][r] += bf16_to_f32(x);
                    }
            }
        }
    }
    if (!any) return;

    const int r = w * 32 + n;  // of the tile
    const float sum = kv_both_halves_sum(l), top = m * a.scale;
    if (pieces > 1) {
        float *part = a.parts + (size_t)(k.part + k.piece * k.next_part) * KV_CHUNK_PART(C::ROWS, DP);
        if (!valid) return;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * u + 8 * g < a.pool.dim) *(float4 *)(part + r * DP + 32 * u + 8 * g + 4 * h) = make_float4(o[u][4 * g], o[u][4 * g + 1], o[u][4 * g + 2], o[u][4 * g + 3]);
        if (h == 0) *(float2 *)(part + C::ROWS * DP + 2 * r) = make_float2(top, sum);
        return;
    }
    const size_t at_out = (size_t)(t.s.first + token) * a.group * a.pool.kv_heads + qh;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    // the halves change places: each lane has eight elements side by side
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            unsigned x[2], y[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = (unsigned)f32_to_bf16(o[u][8 * k + 2 * i] * inv) | ((unsigned)f32_to_bf16(o[u][8 * k + 2 * i + 1] * inv) << 16);
                y[i] = (unsigned)f32_to_bf16(o[u][8 * k + 4 + 2 * i] * inv) | ((unsigned)f32_to_bf16(o[u][8 * k + 4 + 2 * i + 1] * inv) << 16);
            }
            const auto p0 = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false), p1 = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
            const int d = 32 * u + 16 * k + 8 * h;
            if (valid && d < a.pool.dim) *(u32x4_t *)(a.out + at_out * a.pool.dim + d) = u32x4_t{p0[0], p1[0], p0[1], p1[1]};
        }
    if (valid && h == 0 && a.lse) a.lse[at_out] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718056f;
}

// Joins the pieces of the tiles that were cut, in their order, four elements a thread.
template <int DP, bool FP8, bool TREE>
__global__ __launch_bounds__(256) void k_kv_attend_join(KvAttend a, KvPieces p) {
    using C = KvChunk<DP, FP8>;
    KvTile t;
    KvPiece k;
    if (!kv_chunk_piece<C::ROWS, C::KEYS, TREE>(a, p, true, t, k) || k.pieces <= 1) return;
    const int head = k.head, pieces = k.pieces;
    const float *parts = a.parts + (size_t)k.part * KV_CHUNK_PART(C::ROWS, DP);
    const size_t next = (size_t)k.next_part * KV_CHUNK_PART(C::ROWS, DP);
    const int i = blockIdx.y * 256 + threadIdx.x;
    const int r = i / (DP / 4), d = i % (DP / 4) * 4;
    if (r < t.rows && d < a.pool.dim) {
        float top = -INFINITY, sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int MANY = 4;  // pieces whose loads do not wait for each other
        for (int s0 = 0; s0 < pieces; s0 += MANY) {
            float y[MANY];
#pragma unroll
            for (int k = 0; k < MANY; ++k) y[k] = parts[(s0 + k < pieces ? s0 + k : s0) * next + C::ROWS * DP + 2 * r];
#pragma unroll
            for (int k = 0; k < MANY; ++k) top = fmaxf(top, y[k]);
        }
        for (int s0 = 0; s0 < pieces; s0 += MANY) {
            float2 ml[MANY];
            float4 y[MANY];
#pragma unroll
            for (int k = 0; k < MANY; ++k) {
                const float *part = parts + (s0 + k < pieces ? s0 + k : s0) * next;
                ml[k] = *(const float2 *)(part + C::ROWS * DP + 2 * r);
                y[k] = *(const float4 *)(part + r * DP + d);
            }
#pragma unroll
            for (int k = 0; k < MANY; ++k)
                if (s0 + k < pieces) kv_add_part(ml[k].x, top, ml[k].y, y[k], sum, x);
        }
        kv_finish(a, t, head, r, d, top, sum, x);
    }
}

// Workgroups that run at once on 256 compute units.
static int kv_chunk_workgroups(int dp) { return dp == 64 ? 512 : 256; }

template <int DP, bool FP8, bool TREE>
static int attend_chunks(siso_kv *kv, const KvAttend &a) {
    using C = KvChunk<DP, FP8>;
    KvPieces p;
    p.slots = kv_slots_before(a.batch.rows, a.batch.n, a.group, C::ROWS == 256 ? 8 : 7, 1);
    const long tiles = p.slots * kv->kv_heads, room = (long)(SISO_KV_PARTS / KV_CHUNK_PART(C::ROWS, DP));
    long ways = tiles <= kv_chunk_workgroups(DP) / 2 ? kv_chunk_workgroups(DP) / tiles : 1;
    if (ways > room / tiles) ways = room / tiles;
    if (ways > 64) ways = 64;
    if (ways < 1) ways = 1;
    p.ways = (int)ways;
    constexpr int LDS = C::LDS + (TREE ? C::MASKS : 0);
    if (LDS > 64 * 1024) KV_TRY(kv, hipFuncSetAttribute((const void *)k_kv_attend_chunk<DP, FP8, TREE>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
    p.at_once = kv_chunk_workgroups(DP);
    p.room = (int)room;
    if (TREE && a.batch.n <= 64) {
        // There are at most `tiles`; how many pieces the device makes of them it knows by itself.
        auto rounds = [&](long of) { return (of + p.at_once - 1) / p.at_once * p.at_once; };
        auto launch = [&](auto kernel, long all, int threads, int high, int shared) {
            const long most = (1L << 31) / threads / high;
            for (p.slot0 = 0; p.slot0 < all; p.slot0 += most)
                hipLaunchKernelGGL(kernel, dim3((unsigned)(all - p.slot0 < most ? all - p.slot0 : most), high), dim3(threads), shared, kv->stream, a, p);
        };
        const bool join = rounds((long)a.batch.rows * a.group / C::ROWS * kv->kv_heads) <= room;
        if (!join) p.room = 0;  // (more tiles than that are cut)
        launch(k_kv_attend_chunk<DP, FP8, TREE>, rounds(tiles), C::NT, 1, LDS);
        KV_TRY(kv, hipGetLastError());
        if (join) launch(k_kv_attend_join<DP, FP8, TREE>, tiles, 256, C::ROWS * (DP / 4) / 256, 0);
        KV_TRY(kv, hipGetLastError());
        return SISO_OK;
    }
    const long slots = p.slots, piece = ((1L << 31) / C::NT) / (kv->kv_heads * ways);  // (a launch has fewer than 2^32 threads)
    for (p.slot0 = 0; p.slot0 < slots; p.slot0 += piece) {
        p.slots = slots - p.slot0 < piece ? slots - p.slot0 : piece;
        hipLaunchKernelGGL((k_kv_attend_chunk<DP, FP8, TREE>), dim3((unsigned)(p.slots * ways * kv->kv_heads)), dim3(C::NT), LDS, kv->stream, a, p);
        KV_TRY(kv, hipGetLastError());
        if (ways > 1) {
            hipLaunchKernelGGL((k_kv_attend_join<DP, FP8, TREE>), dim3((unsigned)(p.slots * kv->kv_heads), C::ROWS * (DP / 4) / 256), dim3(256), 0, kv->stream, a, p);
            KV_TRY(kv, hipGetLastError());
        }
    }
    return SISO_OK;
}

template <int DP, bool FP8, bool TREE>
static int attend(siso_kv *kv, KvAttend &a, long max_length, long max_new) {
    // Which sequences there are is known on the device only: where both kinds can be, both kernels are launched, and each leaves the other's.
    const long seen = a.window > 0 && a.window + 32L < max_length ? a.window + 32L : max_length;
    const long light = (((long)a.batch.rows * a.group >> 5) + a.batch.n) * kv->kv_heads * seen;
    bool by_few = DP <= 128 && light * DP <= (a.batch.rows >= max_new * a.batch.n ? KV_LIGHT : KV_LIGHT_MIXED);
    if (TREE) {  // all by one kernel (both, each for its own, took 5 to 20% longer than the chunks' alone)
        const long tiles = ((long)a.batch.rows * a.group / KvChunk<DP, FP8>::ROWS + (a.batch.n + 1) / 2) * kv->kv_heads;
        by_few = max_new * a.group <= KV_FEW ||
                 (DP <= 128 && (light * DP <= KV_TREE_LIGHT || tiles > KV_TREE_TILES || (long)a.batch.rows * a.group < KV_FEW * (long)a.batch.n));
    }
    a.few = by_few ? 1 << 30 : TREE ? 0 : KV_FEW;
    if (max_new * a.group > a.few) {
        const int rc = attend_chunks<DP, FP8, TREE>(kv, a);
        if (rc != SISO_OK || TREE || a.batch.rows >= max_new * a.batch.n) return rc;  // (all have max_new rows)
    }
    constexpr int KS = kv_step<DP, FP8>();
    const long tiles = (((long)a.batch.rows * a.group >> 5) + a.batch.n) * kv->kv_heads, cuts = (max_length / KS + 2 + KV_LEAST - 1) / KV_LEAST;
    const long items = tiles * cuts < tiles + KV_STRETCHES ? tiles * cuts : tiles + KV_STRETCHES, piece = 1L << 23;
    a.items = items;
    a.item0 = 0;
    static_assert((size_t)2 * KV_STRETCHES * KV_PART(256) <= SISO_KV_PARTS && 2 * KV_STRETCHES <= SISO_KV_JOINS, "room for the parts");
    if (a.batch.n > 64) {
        hipLaunchKernelGGL((k_kv_plan<KS, TREE>), dim3(1), dim3(1024), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
    }
    for (; a.item0 < items; a.item0 += piece) {  // (a launch has fewer than 2^32 threads)
        const dim3 grid((unsigned)(items - a.item0 < piece ? items - a.item0 : piece));
        hipLaunchKernelGGL((k_kv_attend_few<DP, FP8, TREE>), grid, dim3(256), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}

template <bool TREE>
static int attend(siso_kv *kv, const char *call, int layer, const siso_kv_batch *batch, const unsigned *mask, const void *q, long q_token, long q_head,
                  int heads, float scale, int window, void *out, float *lse) {
    if (!kv) return SISO_EINVAL;
    if (layer < 0) return kv_fail(kv, SISO_EINVAL, "%s: layer %d", call, layer);
    KvAttend a;
    const int rc = kv_batch(kv, call, layer, batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (TREE && kv_max_new(batch) > SISO_KV_TREE) return kv_fail(kv, SISO_EINVAL, "%s: trees of %ld rows", call, kv_max_new(batch));
    if (heads < 1 || heads % kv->kv_heads != 0 || heads / kv->kv_heads > 128)
        return kv_fail(kv, SISO_EINVAL, "%s: %d heads over %d kv heads", call, heads, kv->kv_heads);
    if (!isfinite(scale) || window < 0) return kv_fail(kv, SISO_EINVAL, "%s: scale %g, window %d", call, (double)scale, window);
    if ((long)a.batch.rows * heads > 1L << 30) return kv_fail(kv, SISO_EINVAL, "%s: %d rows of %d heads", call, a.batch.rows, heads);
    if (a.batch.n == 0 || a.batch.rows == 0) return SISO_OK;
    if (!q || !out || ((uintptr_t)q & 1) || ((uintptr_t)out & 15) || ((uintptr_t)lse & 3))
        return kv_fail(kv, SISO_EINVAL, "%s: queries and outputs must be there, outputs 16-byte aligned", call);
    if (TREE && (!mask || ((uintptr_t)mask & 15))) return kv_fail(kv, SISO_EINVAL, "%s: masks must be there, 16-byte aligned", call);
    a.pool = kv_pool(kv, layer);
    a.q = (const bf16_t *)q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.vec = ((uintptr_t)q & 15) == 0 && q_token % 8 == 0 && q_head % 8 == 0;
    a.group = heads / kv->kv_heads;
    // (zero as the smallest number: a score of minus infinity times it stays one; and what would leave the range as the largest: a score of zero stays one)
    a.scale = fminf(fmaxf(fabsf(scale) * 1.44269504089f, 1.17549435e-38f), 3.40282347e38f);
    a.negate = scale < 0.f ? 0x80008000u : 0u;
    a.window = window < a.batch.most ? window : 0;  // (all that there can be; what a row at a position below zero would see cannot wrap)
    a.out = (bf16_t *)out;
    a.lse = lse;
    a.parts = kv->parts;
    a.arrived = kv->arrived;
    a.plan = (KvPlan *)kv->plan;
    a.mask = mask;
    const long max_new = kv_max_new(batch);
    const long max_length = batch->max_length > 0 && batch->max_length < a.batch.most ? batch->max_length : a.batch.most;
    switch (kv->dp / 64 + (kv->dtype == SISO_FP8 ? 4 : 0)) {
        case 1: return attend<64, false, TREE>(kv, a, max_length, max_new);
        case 2: return attend<128, false, TREE>(kv, a, max_length, max_new);
        case 3: return attend<192, false, TREE>(kv, a, max_length, max_new);
        case 4: return attend<256, false, TREE>(kv, a, max_length, max_new);
        case 5: return attend<64, true, TREE>(kv, a, max_length, max_new);
        case 6: return attend<128, true, TREE>(kv, a, max_length, max_new);
        case 7: return attend<192, true, TREE>(kv, a, max_length, max_new);
        default: return attend<256, true, TREE>(kv, a, max_length, max_new);
    }
}

extern "C" int siso_kv_attend(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *q, long q_token, long q_head, int heads,
                              float scale, int window, void *out, float *lse) {
    return attend<false>(kv, "siso_kv_attend", layer, batch, nullptr, q, q_token, q_head, heads, scale, window, out, lse);
}

extern "C" int siso_kv_attend_tree(siso_kv *kv, int layer, const siso_kv_batch *batch, const unsigned *mask, const void *q, long q_token, long q_head,
                                   int heads, float scale, int window, void *out, float *lse) {
    return attend<true>(kv, "siso_kv_attend_tree", layer, batch, mask, q, q_token, q_head, heads, scale, window, out, lse);
}
