// Attention weights of cached positions, added up (siso_kv_weigh).  Layout of the pages: kv_internal.h.
#include <math.h>
#include <type_traits>

#include "kv_internal.h"

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// The weight of position j in row r is 2^(scale * <q_r, k_j> - lse_r): with the rows' sums known there is no maximum to run along, and a
// position's sum is its own.  The product is S = Q K^T, rows of work (row = token * group + head in the group) by positions: a lane of
// v_mfma_f32_32x32x16_bf16 then has one position and 16 of 32 rows, and adds up its own registers; the two halves meet once, at the end.
struct KvWeigh {
    KvPool pool;
    KvBatch batch;
    const bf16_t *q;
    long q_token, q_head;
    int vec;  // rows are aligned to 16 bytes; 2: and a stage's lie within 31 bits
    int heads, group;
    float scale;  // times log2(e): the weights are powers of two
    int window;
    int ahead;  // what is ahead of it stays as it is, if it is not noted anew
    const float *lse;
    const int *fresh, *newest;
    float decay;
    float *mass;
    int *born;
    float *parts;                // [SISO_KV_JOINS][block]: sums of a block's positions over a stretch of the rows
    unsigned *arrived;           // [SISO_KV_JOINS] how many of a block's stretches are there; zeros between calls
    struct KvWeighPlan *plan;
    long items, item0;           // of k_kv_weigh_few: workgroups, and the first of this launch
    int block, rows;             // of k_kv_weigh_rows: positions of a block, rows of work of a stretch
};

// Sequences of few rows of work: a workgroup takes a stretch of the positions, KV_STEP at a time, against all rows, which it holds in LDS.
#define KV_WEIGH_FEW 128
#define KV_STEP 128
// Workgroups: of up to 32 rows of work more than are on the chip at once (64 single tokens over 217,173 positions: 61.6 us a pass, 1,024 62.8, 512 66.2, 8,192
// 66.2), of more, whose rows every workgroup brings to LDS first, as many (64 rows over 21,608 positions: 20.8 us a pass, 2,048 25.2, 512 22.1).
#define KV_WEIGH_FILL(work) ((work) > 32 ? 1024 : 2048)
// Of more rows: a workgroup takes a block of positions, whose keys its waves hold in registers, against a stretch of the rows, which pass through LDS.
// (two tiles of 32 positions a wave, of more than 128 elements one: the registers hold no more)
constexpr int kv_subs(int dp) { return dp <= 128 ? 2 : 1; }
constexpr int kv_block(int dp) { return 128 * kv_subs(dp); }
constexpr int kv_stage(int dp) { return dp <= 128 ? 128 : 64; }  // rows that pass through LDS at a time
#define KV_WEIGH_AHEAD 4  // operands are read so many products ahead
#define KV_WEIGH_MASK 0x274  // what may pass a product in the compiler's order: scalar arithmetic, memory, writes to LDS

struct KvWeighPlan {  // more than 64 sequences: made by a launch of its own
    u64 all, tiles;
    u64 before[SISO_KV_PLAN_BYTES / 8 - 2];  // of each 64 sequences
};
static_assert(sizeof(KvWeighPlan) <= SISO_KV_PLAN_BYTES && SISO_KV_PLAN_BYTES / 8 - 2 >= 65536 / 64, "room for the plan");

__device__ __forceinline__ bf16x8_t kv_as_bf16(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }
__device__ __forceinline__ bf16x8_t kv_codes_bf16(unsigned a, unsigned b) {  // eight codes, exactly
    struct {
        bf16x2_t v[4];
    } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return __builtin_bit_cast(bf16x8_t, r);
}

// ---------------------------------------------------------------------------- who does what
// A lane's sequence, and how many units of work it has: of k_kv_weigh_few steps of positions, of k_kv_weigh_rows blocks of positions times stretches of
// rows.  Lengths are known on the device only.
// Positions ahead of `fresh` that no row sees keep their weight where it does not decay: they are not met (attention does not meet them either), their
// pages may be given up, or be another sequence's by now.  The rest begins with the first block that has one of the others (8 tokens, 4 heads for each of 8 of
// 128, behind 32,768 positions in 16 bits: 108 us, under a window of 1,024 9.4).
__device__ __forceinline__ int kv_weigh_from(const KvWeigh &a, const KvSequence &s) {
    if (!a.ahead) return 0;
    const int seen = s.start - a.window + 1, fresh = a.fresh ? a.fresh[s.b] : s.start, from = fresh < seen ? fresh : seen;
    return from > 0 ? from & ~(SISO_KV_BLOCK - 1) : 0;  // (below the length: the last row sees itself)
}
template <bool FEW>
struct KvShare {
    using Count = typename std::conditional<FEW, unsigned, u64>::type;  // (of few rows there are at most 2^24 steps of a sequence, and 2^27 pieces of work)
    int first, rows, length, from;
    Count units;
    __device__ __forceinline__ void load(const KvWeigh &a, int b, int stretch) {
        first = rows = length = from = 0;
        units = 0;
        if (b >= a.batch.n) return;
        const KvSequence s = kv_sequence(a.batch, b);
        first = s.first;
        rows = s.rows;
        length = s.length;
        if (rows == 0 || length == 0 || (rows * a.group <= KV_WEIGH_FEW) != FEW) return;
        from = kv_weigh_from(a, s);
        if constexpr (FEW) units = ((unsigned)(length - from) + KV_STEP - 1) / KV_STEP;
        else units = (u64)(((unsigned)(length - from) + a.block - 1) / (unsigned)a.block) * (((unsigned)(rows * a.group) + stretch - 1) / (unsigned)stretch);
    }
    // Pieces of work of the sequence, of all heads.
    __device__ __forceinline__ Count pieces(const KvWeigh &a, unsigned stretch) const {
        return (FEW ? ((unsigned)units + stretch - 1) / stretch : units) * (unsigned)a.pool.kv_heads;
    }
};
__device__ __forceinline__ u64 kv_wave_sum(u64 v) {
    return wave_fold(v, [](u64 a, u64 b) __attribute__((always_inline)) { return a + b; });
}
template <class V>
__device__ __forceinline__ V kv_running_sum(V v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const V x = __shfl_up(v, off);
        if (lane >= off) v += x;
    }
    return v;
}
__device__ __forceinline__ u64 kv_divide(u64 a, u64 b) { return (a | b) >> 32 ? a / b : (u64)((unsigned)a / (unsigned)b); }
// Steps of a stretch: so many that there are not more stretches than workgroups.
__device__ __forceinline__ unsigned kv_weigh_stretch(const KvWeigh &a, u64 all, u64 sequences) {
    const u64 ends = sequences * a.pool.kv_heads, room = (u64)a.items > ends ? a.items - ends : 0;
    const u64 s = room ? kv_divide(all * a.pool.kv_heads + room - 1, room) : 0x7FFFFFFFu;
    return s < 1 ? 1u : s > 0x7FFFFFFFu ? 0x7FFFFFFFu : (unsigned)s;
}
// Rows of work of a stretch: those asked for, or all where the workspace has no room for the sums of so many.
__device__ __forceinline__ int kv_weigh_rows(const KvWeigh &a, u64 all) { return all * a.pool.kv_heads <= SISO_KV_JOINS ? a.rows : 1 << 30; }
static_assert((size_t)SISO_KV_JOINS * kv_block(128) <= SISO_KV_PARTS, "room for the sums");

template <bool FEW>
__global__ __launch_bounds__(1024) void k_kv_weigh_plan(KvWeigh a) {
    __shared__ u64 sums[16], tiles[16], before[1024];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, chunks = (a.batch.n + 63) / 64;
    KvShare<FEW> share;
    u64 all = 0, sequences = 0;
    for (int b = t; b < a.batch.n; b += 1024) {
        share.load(a, b, a.rows);
        all += share.units;
        sequences += share.units > 0;
    }
    all = kv_wave_sum(all);
    sequences = kv_wave_sum(sequences);
    if (lane == 0) {
        sums[w] = all;
        tiles[w] = sequences;
    }
    __syncthreads();
    all = sequences = 0;
    for (int i = 0; i < 16; ++i) {
        all += sums[i];
        sequences += tiles[i];
    }
    const unsigned stretch = FEW ? kv_weigh_stretch(a, all, sequences) : (unsigned)kv_weigh_rows(a, all);
    __syncthreads();  // (the sums' places are used again)
    for (int c = w; c < chunks; c += 16) {
        share.load(a, 64 * c + lane, (int)stretch);
        const u64 mine = kv_wave_sum((u64)share.pieces(a, stretch));
        if (lane == 0) before[c] = mine;
    }
    __syncthreads();
    const u64 mine = t < chunks ? before[t] : 0;
    u64 upto = kv_running_sum(mine);
    if (lane == 63) sums[w] = upto;
    __syncthreads();
    for (int i = 0; i < w; ++i) upto += sums[i];
    if (t < chunks) a.plan->before[t] = upto - mine;
    if (t == 0) {
        a.plan->all = all;
        a.plan->tiles = sequences;
    }
}

struct KvWork {
    KvSequence s;
    int head;
    int from;          // where the sequence's positions begin
    unsigned stretch;  // in steps of positions, or rows of work
    u64 in;            // which of the sequence's and head's
};
// The piece of work `item`, the same in every lane; false: there are not as many.
template <bool FEW>
__device__ __forceinline__ bool kv_weigh_find(const KvWeigh &a, u64 item, KvWork &k) {
    using Count = typename KvShare<FEW>::Count;
    const int lane = threadIdx.x & 63;
    KvShare<FEW> share;
    int chunk = 0;
    u64 wanted = item;  // of the 64 sequences
    if (a.batch.n <= 64) {
        share.load(a, lane, a.rows);
        const u64 all = a.batch.n == 1 ? __shfl((u64)share.units, 0) : kv_wave_sum((u64)share.units);
        if constexpr (FEW) k.stretch = kv_weigh_stretch(a, all, __popcll(__ballot(share.units > 0)));
        else k.stretch = (unsigned)kv_weigh_rows(a, all);
        if (!FEW && (int)k.stretch != a.rows) share.load(a, lane, (int)k.stretch);
    } else {  // the last 64 with no more work before them than this piece
        int count = (a.batch.n + 63) / 64;
        while (count > 1) {
            const int step = (count + 63) / 64;
            const bool before = lane * step < count && a.plan->before[chunk + lane * step] <= item;
            const int at = __popcll(__ballot(before)) - 1;  // (the first is 0)
            chunk += at * step;
            count = count - at * step < step ? count - at * step : step;
        }
        chunk = __builtin_amdgcn_readfirstlane(chunk);
        k.stretch = FEW ? kv_weigh_stretch(a, a.plan->all, a.plan->tiles) : (unsigned)kv_weigh_rows(a, a.plan->all);
        wanted = item - a.plan->before[chunk];
        share.load(a, 64 * chunk + lane, (int)k.stretch);
    }
    k.stretch = __builtin_amdgcn_readfirstlane(k.stretch);
    const Count mine = share.pieces(a, k.stretch), upto = a.batch.n == 1 ? mine : kv_running_sum(mine);
    const u64 over = __ballot((u64)upto > wanted);
    if (over == 0) return false;
    const int at = __ffsll((long long)over) - 1;
    k.s.b = 64 * chunk + at;
    k.s.first = __builtin_amdgcn_readlane(share.first, at);
    k.s.rows = __builtin_amdgcn_readlane(share.rows, at);
    k.s.length = __builtin_amdgcn_readlane(share.length, at);
    k.s.start = k.s.length - k.s.rows;
    k.from = __builtin_amdgcn_readlane(share.from, at);
    const u64 before = (u64)(upto - mine);
    const u64 in = wanted - (((u64)(unsigned)__builtin_amdgcn_readlane((int)(before >> 32), at) << 32) | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)before, at));
    k.in = kv_divide(in, (unsigned)a.pool.kv_heads);
    k.head = (int)(in - k.in * (unsigned)a.pool.kv_heads);
    return true;
}

// ---------------------------------------------------------------------------- rows
// Rows of work lie in LDS as the lanes take them: 16-byte pieces [fragment][half][row], 33 rows apart so that neither the writing of a row's pieces
// nor the reading of a fragment meets in one bank.
#define KV_ROWS_APART 33
template <bool FP8>
__device__ __forceinline__ int kv_piece(int c) { return FP8 ? 4 * (c >> 2) + 2 * (c & 1) + ((c >> 1) & 1) : c; }  // where eight elements from 8 c on are
template <int DP>
constexpr int kv_tile_bytes() { return DP / 8 * KV_ROWS_APART * 16; }  // of 32 rows

// Rows to tokens, for numbers below 256 (and a group of 128 at most): (x * magic) >> 16 is x / group.
__device__ __forceinline__ unsigned kv_group_magic(int group) { return 65536u / (unsigned)group + 1; }
__device__ __forceinline__ const bf16_t *kv_row_at(const KvWeigh &a, const KvWork &k, int token, int in_group) {
    return a.q + (long)(k.s.first + token) * a.q_token + (long)(k.head * a.group + in_group) * a.q_head;
}
__device__ __forceinline__ const float *kv_lse_at(const KvWeigh &a, const KvWork &k, int token, int in_group) {
    return a.lse + (size_t)(k.s.first + token) * a.heads + k.head * a.group + in_group;
}
__device__ __forceinline__ u32x4_t kv_eight_of(const bf16_t *q, int vec) {
    if (vec) return *(const u32x4_t *)q;
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (unsigned)q[2 * i] | ((unsigned)q[2 * i + 1] << 16);
    return x;
}
// What is added to a row's scores: minus infinity for a row that adds nothing.
__device__ __forceinline__ float kv_row_less(float lse) { return lse == -INFINITY ? -INFINITY : -lse * 1.44269504089f; }

// Rows that see a position: from `from` up to `to` of the sequence's rows of work.
__device__ __forceinline__ int kv_rows_from(const KvWeigh &a, const KvWork &k, int pos) {
    const long r = ((long)pos - k.s.start) * a.group;
    return r > 0 ? (r < 1 << 30 ? (int)r : 1 << 30) : 0;
}
__device__ __forceinline__ int kv_rows_to(const KvWeigh &a, const KvWork &k, int pos) {
    const long r = a.window > 0 ? ((long)pos + a.window - k.s.start) * a.group : 1L << 30, all = (long)k.s.rows * a.group;
    return r < 0 ? 0 : r < all ? (int)r : (int)all;
}

// What a lane's 16 rows of a tile have subtracted: register r is row 8 (r / 4) + 4 h + r % 4.
__device__ __forceinline__ void kv_less(const float *less, float (&l)[16]) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4 x = *(const float4 *)(less + 8 * g + 4 * h);
        l[4 * g] = x.x, l[4 * g + 1] = x.y, l[4 * g + 2] = x.z, l[4 * g + 3] = x.w;
    }
}
// The powers of 8 * `groups` rows of a tile, summed for this lane's position, which they all see.  What fills a tile up repeats the last row, with a
// power of zero: nothing but what that row's own score may be comes of it.
__device__ __forceinline__ float kv_powers(const f32x16_t &s, float scale, const float (&l)[16], int groups = 4) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (g > 0 && g >= groups) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += __builtin_amdgcn_exp2f(__fmaf_rn(s[4 * g + j], scale, l[4 * g + j]));
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
// Of the rows from row0 on only those from `from` up to `to` that add something.
__device__ __forceinline__ float kv_powers_seen(const f32x16_t &s, float scale, const float (&l)[16], int row0, int from, int to) {
    const int h = (threadIdx.x >> 5) & 1;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[r], scale, l[r]));
        const int row = row0 + 8 * (r >> 2) + 4 * h + (r & 3);
        sum[r & 3] += row >= from && row < to && l[r] != -INFINITY ? p : 0.f;
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__device__ __forceinline__ void kv_weigh_note(const KvWeigh &a, const KvSequence &s, int pos, size_t spot, float had, float sum) {
    const int fresh = a.fresh ? a.fresh[s.b] : s.start;
    a.mass[spot] = (pos < fresh && a.decay > 0.f ? a.decay * had : 0.f) + sum;  // (decay 0: whatever was there)
    if (a.born && pos >= fresh) a.born[spot] = (a.newest ? a.newest[s.b] : s.length - 1) - (s.length - 1 - pos);
}

__device__ __forceinline__ void kv_weigh_position(const KvWeigh &a, const KvWork &k, int pos, float sum) {
    const int page = a.batch.pages[(long)k.s.b * a.batch.width + (pos >> a.pool.shift)];
    if (!kv_is_page(a.pool, page)) return;
    const size_t spot = kv_scale_at(a.pool, page, k.head, pos);
    kv_weigh_note(a, k.s, pos, spot, a.mass[spot], sum);
}

// ---------------------------------------------------------------------------- few rows
// One workgroup for a stretch of a sequence's and head's positions; its rows stay in LDS, its four waves take 32 positions each at a time, whose keys go
// straight to registers, the next step's while this one is worked on.  Bound by the reading of the keys: 64 tokens, 4 heads for each of 8, over 217,173
// positions in 8 bits 57 us, 244 MB at 4.3 TB/s; 2 sequences' last 32 over 21,608 in 16 bits 17, a few us of them launch and plan.
template <int DP, bool FP8>
__global__ __launch_bounds__(256, DP <= 128 ? 4 : 2) void k_kv_weigh_few(KvWeigh a) {
    constexpr int ES = FP8 ? 1 : 2;
    constexpr int NF = FP8 ? DP / 32 : DP / 16, NS = DP / 16;
    __shared__ __attribute__((aligned(16))) char rows[KV_WEIGH_FEW / 32 * kv_tile_bytes<DP>()];
    __shared__ __attribute__((aligned(16))) float less[KV_WEIGH_FEW];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, n = lane & 31;
    KvWork k;
    if (!kv_weigh_find<true>(a, (u64)a.item0 + blockIdx.x, k)) return;
    const int work = k.s.rows * a.group, tiles = (work + 31) >> 5;
    const long begin = k.from + (long)k.in * k.stretch * KV_STEP;
    const int from = (int)begin, to = begin + (long)k.stretch * KV_STEP < k.s.length ? (int)(begin + (long)k.stretch * KV_STEP) : k.s.length;
    // positions ahead of every row's window (that decay, or are noted anew) have no products
    const long seen_from = a.window > 0 ? (long)k.s.start - a.window + 1 : 0;
    int at = from + 32 * w;
    auto pages_of = [&](int p, int (&page)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) page[i] = kv_page_entry(a.pool, a.batch, k.s.b, p + 16 * i < k.s.length ? p + 16 * i : k.s.length - 1);
    };
    u32x4_t kf[NF];
    float ks = 1.f, had = 0.f;
    auto spot_of = [&](int p, const int (&page)[2]) {
        const int mine = page[n >> 4];
        return kv_scale_at(a.pool, kv_is_page(a.pool, mine) ? mine : 0, k.head, p + n);
    };
    auto load = [&](int p, const int (&page)[2]) {
        const int mine = page[n >> 4];
        const char *from_k = a.pool.k + kv_block_at(a.pool, kv_is_page(a.pool, mine) ? mine : 0, k.head, p + 16 * (n >> 4)) * ES + h * 256 + (lane & 15) * 16;
#pragma unroll
        for (int i = 0; i < NF; ++i) kf[i] = *(const u32x4_t *)(from_k + i * 512);
        if constexpr (FP8) ks = a.pool.ks[spot_of(p, page)];
        had = a.mass[spot_of(p, page)];
    };
    int page[2], next_page[2], over_next_page[2];
    if (at < to) {
        pages_of(at, page);
        pages_of(at + KV_STEP < to ? at + KV_STEP : at, next_page);
        load(at, page);
    }
    const unsigned magic = kv_group_magic(a.group);
    for (int i = t; i < 32 * tiles * (DP / 8); i += 256) {
        const int row = i / (DP / 8), c = i % (DP / 8), of = row < work ? row : work - 1, token = (int)((unsigned)of * magic >> 16);
        u32x4_t x = u32x4_t{0, 0, 0, 0};
        if (8 * c < a.pool.dim) x = kv_eight_of(kv_row_at(a, k, token, of - token * a.group) + 8 * c, a.vec);
        *(u32x4_t *)(rows + (row >> 5) * kv_tile_bytes<DP>() + (kv_piece<FP8>(c) * KV_ROWS_APART + (row & 31)) * 16) = x;
    }
    bool none = false;
    if (t < 32 * tiles) {
        const int token = (int)((unsigned)t * magic >> 16);
        const float l = t < work ? kv_row_less(*kv_lse_at(a, k, token, t - token * a.group)) : -INFINITY;
        less[t] = l;
        none = t < work && l == -INFINITY;
    }
    const bool odd = __syncthreads_or(none);
    // positions that all rows see
    const int all_from = a.window > 0 ? k.s.length - a.window : 0, all_to = odd ? 0 : k.s.start + 1;

    for (; at < to; at += KV_STEP) {
        const int pos = at + n;
        const bool held = kv_is_page(a.pool, page[n >> 4]);
        if (k.head == 0 && (lane == 0 || lane == 16) && pos < k.s.length && !held) atomicAdd(a.pool.bad, 1ull);
        const size_t spot = spot_of(at, page);
        const float before = had, scale = FP8 ? a.scale * ks : a.scale;
        bf16x8_t kx[NS];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            if constexpr (FP8) {
                kx[2 * i] = kv_codes_bf16(kf[i][0], kf[i][1]);
                kx[2 * i + 1] = kv_codes_bf16(kf[i][2], kf[i][3]);
            } else kx[i] = kv_as_bf16(kf[i]);
        }
        const int next = at + KV_STEP;
        if (next < to) {
            pages_of(next + KV_STEP < to ? next + KV_STEP : next, over_next_page);
            load(next, next_page);
        }
        float sum = 0.f;
        if (at + 31 >= seen_from) {
            const bool all = at >= all_from && at + 32 <= all_to;
            int r0 = 0, r1 = 0;
            if (!all) {
                r0 = pos < k.s.length ? kv_rows_from(a, k, pos) : 1 << 30;
                r1 = kv_rows_to(a, k, pos);
            }
            for (int tile = 0; tile < tiles; ++tile) {
                f32x16_t s = f32x16_t{};
                float l[16];
                const char *q = rows + tile * kv_tile_bytes<DP>() + (h * KV_ROWS_APART + n) * 16;
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t *)(q + i * 2 * KV_ROWS_APART * 16), kx[i], s, 0, 0, 0);
                kv_less(less + 32 * tile, l);
                sum += all ? kv_powers(s, scale, l, (work - 32 * tile + 7) >> 3) : kv_powers_seen(s, scale, l, 32 * tile, r0, r1);
            }
            const LanePair<float> both = lane_pair<32>(sum);
            sum = both.a + both.b;
        }
        if (h == 0 && pos < k.s.length && held) kv_weigh_note(a, k.s, pos, spot, before, sum);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            page[i] = next_page[i];
            next_page[i] = over_next_page[i];
        }
    }
}

// ---------------------------------------------------------------------------- many rows
// Where the 16-byte piece c of row r of a stage lies: rows one after the other, their pieces in an order of each row's own, so that the 16 rows whose
// pieces of one number are read at a time lie in 16 different banks.
template <int DP>
__device__ __forceinline__ int kv_swizzled(int r, int c) {
    constexpr int P = DP / 8;
    if constexpr (P == 8) return c ^ ((r >> 1) & 7);
    else if constexpr (P == 24) return (c + (r >> 1 & 7)) % 24;
    else return c ^ (r & 15);
}
template <int DP>
__device__ __forceinline__ int kv_unswizzled(int r, int slot) {
    constexpr int P = DP / 8;
    if constexpr (P == 24) return (slot + 24 - (r >> 1 & 7)) % 24;
    else return kv_swizzled<DP>(r, slot);
}
// 16 bytes of each lane, from memory to LDS: lane l's to `to` + 16 l.  The compiler does not know of it: kv_landed() has to come before a barrier
// before they are read.
__device__ __forceinline__ void kv_to_lds(const void *from, unsigned off, unsigned at) {
    const unsigned to = __builtin_amdgcn_readfirstlane(at);  // (both are the same in every lane)
    const u64 p = (u64)from, base = ((u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)p);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void kv_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// One workgroup for a block of positions and a stretch of the rows.  Each of its four waves holds 64 positions' keys in registers (of more than 128
// elements 32); the rows pass through LDS in stages, the next from memory while these are worked on.  VEC: their pieces are aligned, and a
// stage's lie within 31 bits.
// Bound by the matrix cores, the powers and the LDS reads of the rows between them: 4,096 rows of 32 heads of 128 over 12,289 positions, 344 GFLOP, 400 us, 860
// TFLOP/s or 0.70 of a large library product (without fetching the same loop takes 359 us, without powers 307, with neither 270).  Stretches of 1,024 rows
// take 422 us, of 4,096 400, stages of 64 rows 413, operands read eight products ahead 419, no bound on the compiler's order 410.
template <int DP, bool FP8, bool VEC>
__global__ __launch_bounds__(256, 2) void k_kv_weigh_rows(KvWeigh a) {
    constexpr int ES = FP8 ? 1 : 2;
    constexpr int NF = FP8 ? DP / 32 : DP / 16, NS = DP / 16, PIECES = DP / 8, SUBS = kv_subs(DP), BLOCK = kv_block(DP), ROWS = kv_stage(DP), TILES = ROWS / 32;
    constexpr int STAGE = ROWS * DP * 2, NL = STAGE / 4096;  // bytes; a thread's pieces
    static_assert(TILES % 2 == 0, "two sets of scores in turn");
    __shared__ __attribute__((aligned(1024))) char rows[2 * STAGE];
    __shared__ __attribute__((aligned(16))) float less[4][ROWS];  // of four stages: the one before is still read where the next is written
    __shared__ int odd[2][2];  // a row of a half of the stage adds nothing
    __shared__ int last;
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5, n = lane & 31;
    for (u64 item = blockIdx.x;; item += gridDim.x) {
        KvWork k;
        if (!kv_weigh_find<false>(a, item, k)) return;
        const unsigned stretches = ((unsigned)(k.s.rows * a.group) + k.stretch - 1) / k.stretch;
        const unsigned block = (unsigned)kv_divide(k.in, stretches), piece = (unsigned)(k.in - (u64)block * stretches);
        const int p0 = k.from + (int)(block * BLOCK), at = p0 + 32 * SUBS * w;  // the block's positions, this wave's
        bf16x8_t kx[SUBS][NS];
        float scale[SUBS], sum[SUBS] = {};
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            const int blk = at + 32 * sub + 16 * (n >> 4), page = a.batch.pages[(long)k.s.b * a.batch.width + ((blk < k.s.length ? blk : k.s.length - 1) >> a.pool.shift)];
            const bool held = kv_is_page(a.pool, page);
            if (k.head == 0 && piece == 0 && (lane == 0 || lane == 16) && blk < k.s.length && !held) atomicAdd(a.pool.bad, 1ull);
            const int pg = held ? page : 0;
            const char *from_k = a.pool.k + kv_block_at(a.pool, pg, k.head, blk) * ES + h * 256 + (lane & 15) * 16;
            u32x4_t kf[NF];
#pragma unroll
            for (int i = 0; i < NF; ++i) kf[i] = *(const u32x4_t *)(from_k + i * 512);
            scale[sub] = FP8 ? a.scale * a.pool.ks[kv_scale_at(a.pool, pg, k.head, at + 32 * sub + n)] : a.scale;
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                if constexpr (FP8) {
                    kx[sub][2 * i] = kv_codes_bf16(kf[i][0], kf[i][1]);
                    kx[sub][2 * i + 1] = kv_codes_bf16(kf[i][2], kf[i][3]);
                } else kx[sub][i] = kv_as_bf16(kf[i]);
            }
        }
        // the stretch's rows that see a position of the block; those that see all of this wave's
        const long cut = (long)piece * k.stretch;
        int begin = kv_rows_from(a, k, p0), end = kv_rows_to(a, k, p0 + BLOCK - 1);
        begin = begin > cut ? begin : (int)cut;
        end = end < cut + k.stretch ? end : (int)(cut + k.stretch);
        const int all_from = at + 32 * SUBS - 1 < k.s.length ? kv_rows_from(a, k, at + 32 * SUBS - 1) : 1 << 30, all_to = kv_rows_to(a, k, at);
        // Stages.  `token` and `in_first`: of the next one's first row.
        const int stages = end > begin ? (end - begin + ROWS - 1) / ROWS : 0;
        const unsigned magic = kv_group_magic(a.group);
        const int jump = ROWS / a.group, jump_in = ROWS - jump * a.group;
        int row0 = begin, token = begin / a.group, in_first = begin - token * a.group;
        const bf16_t *q_first = kv_row_at(a, k, token, 0);
        const float *lse_first = kv_lse_at(a, k, token, 0);
        // A wave's pieces: 64 that lie side by side in LDS, and every fourth 64.  Where 4 KB hold whole tokens, these are as far apart for all lanes (the order of
        // pieces repeats itself every 16 rows).
        constexpr int ROWS_4K = 2048 / DP, OFFS = ROWS_4K < 16 ? 16 / ROWS_4K : 1;
        const bool even = 2048 % DP == 0 && ROWS_4K % a.group == 0;
        const long step = even ? ROWS_4K / a.group * a.q_token : 0;
        auto offset = [&](int x, int most) __attribute__((always_inline)) {  // from the first token's row on (rows beyond `most` as that one: they weigh nothing)
            const int row = x / PIECES, c = kv_unswizzled<DP>(row, x % PIECES), over = in_first + (row < most ? row : most), d = (int)((unsigned)over * magic >> 16);
            return 2u * ((unsigned)d * (unsigned)a.q_token + (unsigned)(over - d * a.group) * (unsigned)a.q_head + (8 * c < a.pool.dim ? 8u * c : 0u));
        };
        unsigned off[OFFS];
        auto offsets = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < OFFS; ++i) off[i] = offset(t + 256 * i, ROWS);
        };
        if constexpr (VEC) offsets();
        float gl = -INFINITY;
        auto fetch = [&](int buffer) __attribute__((always_inline)) {
            if constexpr (VEC) {  // (beyond the dimension, where the keys are zeros, lies what is: a row's own first elements)
                const unsigned to = (unsigned)(size_t)(__attribute__((address_space(3))) char *)rows + buffer * STAGE + w * 1024;
                if (even && row0 + ROWS <= end) {
#pragma unroll
                    for (int i = 0; i < NL; ++i) kv_to_lds(q_first + i / OFFS * OFFS * step, off[i % OFFS], to + i * 4096);
                } else {
                    const int most = end - 1 - row0;
#pragma unroll 1
                    for (int i = 0; i < NL; ++i) kv_to_lds(q_first, offset(t + 256 * i, most), to + i * 4096);
                }
            } else {
#pragma unroll 1
                for (int x = t; x < ROWS * PIECES; x += 256) {
                    const int row = x / PIECES, c = kv_unswizzled<DP>(row, x % PIECES), over = in_first + (row0 + row < end ? row : end - 1 - row0), d = (int)((unsigned)over * magic >> 16);
                    u32x4_t y = u32x4_t{0, 0, 0, 0};
                    if (8 * c < a.pool.dim) y = kv_eight_of(q_first + (long)d * a.q_token + (long)(over - d * a.group) * a.q_head + 8 * c, 0);
                    *(u32x4_t *)(rows + buffer * STAGE + x * 16) = y;
                }
            }
            if (t < ROWS) gl = row0 + t < end ? kv_row_less(lse_first[in_first + t + (unsigned)((in_first + t) * magic >> 16) * (a.heads - a.group)]) : INFINITY;  // (infinity: no row)
            row0 += ROWS;
            q_first += jump * a.q_token;
            lse_first += jump * a.heads;
            if (jump_in) {
                in_first += jump_in;
                if (in_first >= a.group) {
                    in_first -= a.group;
                    q_first += a.q_token;
                    lse_first += a.heads;
                }
                if constexpr (VEC) offsets();
            }
        };
        auto put_less = [&](int stage) __attribute__((always_inline)) {
            if (t < ROWS) {
                less[stage & 3][t] = gl == INFINITY ? -INFINITY : gl;
                const u64 none = __ballot(gl == -INFINITY);
                if (lane == 0) odd[stage & 1][w] = none != 0;
            }
        };
        if (stages > 0) {
            fetch(0);
            put_less(0);
            kv_landed();
        }
        __syncthreads();
        // The products of a tile and the powers of the one before it stand side by side, one on the matrix cores, the other on the vector units: a
        // product takes as long as two rows' powers.  The last tile of a stage leaves its powers to the next stage: `pending`.
        f32x16_t s[2][SUBS];
        bool pending = false;
        const float *of_pending = less[0];  // what is added to its rows' scores
        auto four = [&](const float *of, int g) __attribute__((always_inline)) { return *(const float4 *)(of + 8 * g + 4 * h); };
        auto power = [&](const f32x16_t (&of)[SUBS], int sub, int r, float4 l, float (&part)[SUBS]) __attribute__((always_inline)) {
            part[sub] += __builtin_amdgcn_exp2f(__fmaf_rn(of[sub][r], scale[sub], (r & 3) == 0 ? l.x : (r & 3) == 1 ? l.y : (r & 3) == 2 ? l.z : l.w));
        };
        auto finish = [&]() __attribute__((always_inline)) {
            if (pending) {
                float part[SUBS] = {};
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float4 l = four(of_pending, r >> 2);
#pragma unroll
                    for (int sub = 0; sub < SUBS; ++sub) power(s[1], sub, r, l, part);
                }
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub) sum[sub] += part[sub];
            }
            pending = false;
        };
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) s[1][sub] = f32x16_t{};
        const char *const mine = rows + n * DP * 2;  // this lane's row of a tile
        auto place = [&](int j) __attribute__((always_inline)) {  // of its piece of fragment j
            const int c = FP8 ? 2 * (2 * (j >> 1) + h) + (j & 1) : 2 * j + h;
            return kv_swizzled<DP>(n, c) * 16;
        };
#pragma unroll 1
        for (int i = 0; i < stages; ++i) {
            const int buffer = i & 1, first = begin + i * ROWS;
            if (i + 1 < stages) fetch(buffer ^ 1);
            const bool all = first >= all_from && (first + ROWS < end ? first + ROWS : end) <= all_to && !(odd[buffer][0] | (ROWS > 64 ? odd[buffer][1] : 0));
            if (all) {
                auto operand = [&](int j) __attribute__((always_inline)) { return *(const bf16x8_t *)(mine + buffer * STAGE + j / NS * 64 * DP + place(j % NS)); };
                bf16x8_t x[KV_WEIGH_AHEAD];
#pragma unroll
                for (int j = 0; j < KV_WEIGH_AHEAD; ++j) x[j] = operand(j);
                float4 l = four(of_pending, 0), next_l;
#pragma unroll
                for (int tile = 0; tile < TILES; ++tile) {
                    float part[SUBS] = {};
#pragma unroll
                    for (int sub = 0; sub < SUBS; ++sub) s[tile & 1][sub] = f32x16_t{};
#pragma unroll
                    for (int c = 0; c < NS * SUBS; ++c) {
                        const int j = c / SUBS, sub = c % SUBS, J = tile * NS + j;
                        s[tile & 1][sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[J % KV_WEIGH_AHEAD], kx[sub][j], s[tile & 1][sub], 0, 0, 0);
                        if (sub == SUBS - 1 && J + KV_WEIGH_AHEAD < TILES * NS) x[J % KV_WEIGH_AHEAD] = operand(J + KV_WEIGH_AHEAD);
                        // the same share of the powers behind each product: row by row, of all positions
#pragma unroll
                        for (int p = 16 * c / NS; p < 16 * (c + 1) / NS; ++p) {
                            const int r = p / SUBS;
                            if (p % (4 * SUBS) == 0) next_l = r < 12 ? four(of_pending, (r >> 2) + 1) : four(less[i & 3] + 32 * tile, 0);
                            power(s[~tile & 1], p % SUBS, r, l, part);
                            if (p % (4 * SUBS) == 4 * SUBS - 1) l = next_l;
                        }
                        __builtin_amdgcn_sched_barrier(KV_WEIGH_MASK);
                    }
#pragma unroll
                    for (int sub = 0; sub < SUBS; ++sub) sum[sub] += tile > 0 || pending ? part[sub] : 0.f;
                    of_pending = less[i & 3] + 32 * tile;
                }
                pending = true;
            } else {
                finish();
#pragma unroll 1
                for (int tile = 0; tile < TILES; ++tile) {
                    float l[16];
                    kv_less(less[i & 3] + 32 * tile, l);
#pragma unroll
                    for (int sub = 0; sub < SUBS; ++sub) {
                        const int pos = at + 32 * sub + n;
                        f32x16_t x = f32x16_t{};
#pragma unroll
                        for (int j = 0; j < NS; ++j)
                            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t *)(mine + buffer * STAGE + tile * 64 * DP + place(j)), kx[sub][j], x, 0, 0, 0);
                        sum[sub] += kv_powers_seen(x, scale[sub], l, first + 32 * tile, pos < k.s.length ? kv_rows_from(a, k, pos) : 1 << 30, kv_rows_to(a, k, pos));
                    }
                }
            }
            if (i + 1 < stages) put_less(i + 1);
            if constexpr (VEC) kv_landed();
            __syncthreads();
        }
        finish();
        const bool parts = (int)k.stretch != 1 << 30 && stretches > 1;
        const u64 block_item = item - (u64)piece * a.pool.kv_heads;  // the block's first piece: its sums begin there, and its count is there
        const int pos = p0 + t;
        float total[SUBS];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            const LanePair<float> both = lane_pair<32>(sum[sub]);
            total[sub] = both.a + both.b;
        }
        if (parts) {
            // The workgroup that is done last with a block adds up all sums, in the order of the rows.  They pass the caches of the XCDs.
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
                if (h == 0) __hip_atomic_store(a.parts + item * BLOCK + 32 * (SUBS * w + sub) + n, total[sub], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (t == 0) {
                last = atomicAdd(a.arrived + block_item, 1u) == stretches - 1;
                if (last) a.arrived[block_item] = 0;  // (for the next call: nobody else comes)
            }
            __syncthreads();
            if (last && t < BLOCK && pos < k.s.length) {
                float all = 0.f;
#pragma unroll 8
                for (unsigned i = 0; i < stretches; ++i)
                    all += __hip_atomic_load(a.parts + (block_item + (u64)i * a.pool.kv_heads) * BLOCK + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                kv_weigh_position(a, k, pos, all);
            }
        } else {
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
                if (h == 0 && at + 32 * sub + n < k.s.length) kv_weigh_position(a, k, at + 32 * sub + n, total[sub]);
        }
        __syncthreads();  // (`last` is used again)
    }
}

template <int DP, bool FP8>
static int weigh(siso_kv *kv, KvWeigh &a, long max_length, long max_new) {
    const long heads = kv->kv_heads;
    const bool many = max_new * a.group > KV_WEIGH_FEW, few = !many || a.batch.rows < max_new * a.batch.n;  // (otherwise all have max_new rows)
    if (few) {
        const long most = (long)a.batch.n * heads * ((max_length + KV_STEP - 1) / KV_STEP), ends = (long)a.batch.n * heads;
        const long fill = KV_WEIGH_FILL(max_new * a.group);
        a.items = most < fill + ends ? most : fill + ends;
        a.rows = 1 << 30;
        a.block = 0;
        if (a.batch.n > 64) {
            hipLaunchKernelGGL(k_kv_weigh_plan<true>, dim3(1), dim3(1024), 0, kv->stream, a);
            KV_TRY(kv, hipGetLastError());
        }
        const long piece = 1L << 23;  // (a launch has fewer than 2^32 threads)
        for (a.item0 = 0; a.item0 < a.items; a.item0 += piece) {
            hipLaunchKernelGGL((k_kv_weigh_few<DP, FP8>), dim3((unsigned)(a.items - a.item0 < piece ? a.items - a.item0 : piece)), dim3(256), 0, kv->stream, a);
            KV_TRY(kv, hipGetLastError());
        }
    }
    if (many) {
        a.block = kv_block(DP);
        const long blocks = (long)a.batch.n * heads * ((max_length + a.block - 1) / a.block), work = max_new * a.group;
        a.rows = 1 << 30;
        long items = blocks;
        for (int rows = 2048; rows >= 256; rows /= 2) {
            if (rows < work) {
                a.rows = rows;
                items = blocks * ((work + rows - 1) / rows);
            }
            if (items >= 1024) break;
        }
        const unsigned grid = (unsigned)(items < 1 << 16 ? items : 1 << 16);
        if (a.batch.n > 64) {
            hipLaunchKernelGGL(k_kv_weigh_plan<false>, dim3(1), dim3(1024), 0, kv->stream, a);
            KV_TRY(kv, hipGetLastError());
        }
        if (a.vec == 2) hipLaunchKernelGGL((k_kv_weigh_rows<DP, FP8, true>), dim3(grid), dim3(256), 0, kv->stream, a);
        else hipLaunchKernelGGL((k_kv_weigh_rows<DP, FP8, false>), dim3(grid), dim3(256), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}

extern "C" int siso_kv_weigh(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *q, long q_token, long q_head, int heads, float scale,
                             int window, const float *lse, const int *fresh, const int *newest, float decay, float *mass, int *born) {
    if (!kv) return SISO_EINVAL;
    if (layer < 0) return kv_fail(kv, SISO_EINVAL, "siso_kv_weigh: layer %d", layer);
    KvWeigh a;
    const int rc = kv_batch(kv, "siso_kv_weigh", layer, batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (heads < 1 || heads % kv->kv_heads != 0 || heads / kv->kv_heads > 128)
        return kv_fail(kv, SISO_EINVAL, "siso_kv_weigh: %d heads over %d kv heads", heads, kv->kv_heads);
    if (!isfinite(scale) || window < 0 || !(decay >= 0.f && decay <= 1.f))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_weigh: scale %g, window %d, decay %g", (double)scale, window, (double)decay);
    if ((long)a.batch.rows * heads > 1L << 30) return kv_fail(kv, SISO_EINVAL, "siso_kv_weigh: %d rows of %d heads", a.batch.rows, heads);
    if (a.batch.n == 0 || a.batch.rows == 0) return SISO_OK;
    if (!q || !lse || !mass || ((uintptr_t)q & 1) || (((uintptr_t)lse | (uintptr_t)mass | (uintptr_t)born) & 3))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_weigh: queries, lse and mass must be there, all aligned to their type");
    if (a.batch.most == 0) return SISO_OK;  // (no position: launches without workgroups are errors)
    a.pool = kv_pool(kv, layer);
    a.q = (const bf16_t *)q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.vec = ((uintptr_t)q & 15) == 0 && q_token % 8 == 0 && q_head % 8 == 0;
    if (a.vec && q_token >= 0 && q_head >= 0 && q_token < 1 << 20 && q_head < 1 << 20) a.vec = 2;
    a.heads = heads;
    a.group = heads / kv->kv_heads;
    a.scale = copysignf(fminf(fmaxf(fabsf(scale) * 1.44269504089f, 1.17549435e-38f), 3.40282347e38f), scale);  // (as siso_kv_attend takes it)
    a.window = window < a.batch.most ? window : 0;
    a.ahead = a.window > 0 && decay == 1.f;
    a.lse = lse;
    a.fresh = fresh;
    a.newest = newest;
    a.decay = decay;
    a.mass = mass + (size_t)layer * kv->layer_scales;
    a.born = born ? born + (size_t)layer * kv->layer_scales : nullptr;
    const long max_length = batch->max_length > 0 && batch->max_length < a.batch.most ? batch->max_length : a.batch.most;
    a.parts = kv->parts;
    a.arrived = kv->arrived;
    a.plan = (KvWeighPlan *)kv->plan;
    const long max_new = kv_max_new(batch);
    switch (kv->dp / 64 + (kv->dtype == SISO_FP8 ? 4 : 0)) {
        case 1: return weigh<64, false>(kv, a, max_length, max_new);
        case 2: return weigh<128, false>(kv, a, max_length, max_new);
        case 3: return weigh<192, false>(kv, a, max_length, max_new);
        case 4: return weigh<256, false>(kv, a, max_length, max_new);
        case 5: return weigh<64, true>(kv, a, max_length, max_new);
        case 6: return weigh<128, true>(kv, a, max_length, max_new);
        case 7: return weigh<192, true>(kv, a, max_length, max_new);
        default: return weigh<256, true>(kv, a, max_length, max_new);
    }
}
