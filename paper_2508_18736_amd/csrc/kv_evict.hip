// Eviction from the paged cache by accumulated attention weight (siso_kv_evict).  Layout of the pages: kv_internal.h.
#include <type_traits>

#include "kv_internal.h"

typedef unsigned char byte_t;

struct KvEvict {
    KvPool pool;
    KvBatch batch;
    int keep, recent, early;
    float *mass;
    int *born;
    const int *to;  // NULL: in place
    long to_width;
    long layer_bytes, layer_scales;
    int layers;
    long unit0, units;  // of this launch: a unit is a kv head of a layer of a sequence
    int *from;          // [units][keep]: where what stands in a slot comes from: itself, another one, or -1: nothing is to be done
    int *list;          // [units][keep]: slots from `keep` on that stay, in order
};

struct KvUnit {
    KvSequence s;
    int head, layer;
    int stay;  // positions that it has afterwards
};
__device__ __forceinline__ KvUnit kv_unit(const KvEvict &a, long unit) {
    KvUnit u;
    u.head = (int)(unit % a.pool.kv_heads);
    u.layer = (int)(unit / a.pool.kv_heads % a.layers);
    const int b = (int)(unit / a.pool.kv_heads / a.layers);
    u.s.b = b;
    u.s.first = u.s.rows = u.s.start = 0;
    u.s.length = kv_clamp(a.batch.length[b], 0, a.batch.most);
    u.stay = u.s.length < a.keep ? u.s.length : a.keep;
    return u;
}
// Where a slot's numbers are, of mass and born (of the layer): below 2^32, a place has 64 bytes of keys and 64 of values at least.
#define KV_NOWHERE 0xFFFFFFFFu  // its page is none
__device__ __forceinline__ unsigned kv_spot(const KvPool &pool, const int *table, int head, int at) {
    const int page = table[at >> pool.shift];
    return kv_is_page(pool, page) ? (((unsigned)page * (unsigned)pool.kv_heads + (unsigned)head) << pool.shift) + (unsigned)(at & ((1 << pool.shift) - 1)) : KV_NOWHERE;
}
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
// Numbers that are ordered as the masses are; NaN is less than all else (and 0, of positions without a page, is less than that).
__device__ __forceinline__ unsigned kv_order(float mass) {
    const unsigned x = __float_as_uint(mass + 0.f);  // (the two zeros are equal)
    return mass != mass ? 1u : x >> 31 ? ~x : x | 0x80000000u;
}

// ---------------------------------------------------------------------------- which positions stay
#define KV_CHOOSE_ROOM 32768  // words of LDS: two for each position (its number and its age), or one; of more positions both are read from memory whenever they are asked for
// Threads of a workgroup: 1,024, or 256 where there are more units than CUs, of at most so many positions each: workgroups of 1,024 that share a CU wait for
// one another at barriers (8 heads, us a call with 256 and with 1,024 threads: 48 sequences of 400 positions 57 and 61, of 1,900 239 and 241, 96 of 1,000 262
// and 271; 16 of 1,900 87 and 84).
#define KV_CHOOSE_FEW 2048
#define KV_DIGIT 2048

// Of numbers of a wave's lanes the sum of those before this lane's, and of all, in each lane.
template <int OFF = 1>
__device__ __forceinline__ unsigned kv_before(unsigned &all) {
    const LanePair<unsigned> pair = lane_pair<OFF>(all);
    const unsigned both = pair.a + pair.b, less = threadIdx.x & OFF ? both - all : 0u;
    all = both;
    if constexpr (OFF < 32) return less + kv_before<2 * OFF>(all);
    else return less;
}
// One workgroup a unit.  Its positions' numbers are brought to LDS once, four positions a load; the `keep`-th largest is found digit by digit (11, 11 and 10 bits),
// from counts of each digit's values, until what is left is one group.  A thread then has a stretch of the slots, in order: ranks are sums over threads, so that
// nothing depends on scheduling.  Bound by latency: some ten passes over LDS, a barrier each, behind three loads that wait for each other (length, page, mass): 5
// sequences of 25,683 positions down to 2,048 each, 8 heads: 18.9 us, 264 units of 900 to 1,064 13.9 us (ranks from ballots, 64 slots after 64, 29 and 17.9).
template <int NT>
__global__ __launch_bounds__(NT) void k_kv_choose(KvEvict a, int room) {
    extern __shared__ __attribute__((aligned(16))) unsigned numbers[];
    constexpr int NW = NT / 64, EACH = KV_DIGIT / NT, TURNS = 3, NEVER = -0x7FFFFFFF - 1;
    __shared__ unsigned counts[TURNS][KV_DIGIT];
    __shared__ unsigned waves[TURNS + 2][NW];
    __shared__ int newest_of[NW];
    __shared__ int last_equal, moving;
    const KvUnit u = kv_unit(a, a.unit0 + blockIdx.x);
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), length = u.s.length, keep = a.keep;
    int *const from = a.from + (long)blockIdx.x * keep;
    float *const mass = a.mass + u.layer * a.layer_scales;
    int *const born = a.born ? a.born + u.layer * a.layer_scales : nullptr;
    const int *const table = a.batch.pages + (long)u.s.b * a.batch.width, *const to = a.to ? a.to + (long)u.s.b * a.to_width : nullptr;
    const int quads = (length + 3) >> 2;  // (a page has whole ones)
    const bool all = length <= keep, cached = 4L * quads <= room, roomy = 8L * quads <= room;
    if (all && !to) return;
    unsigned *const ages = numbers + 4 * quads;  // (if there is room)
    for (int i = t; i < TURNS * KV_DIGIT; i += NT) counts[0][i] = 0;
    auto largest = [](int x, int y) __attribute__((always_inline)) { return x > y ? x : y; };
    // (a page that is none is counted at its first four positions, where they are first asked for: what is never kept of it nothing else meets)
    auto met = [&](int q, unsigned at) __attribute__((always_inline)) {
        if (at == KV_NOWHERE && u.head == 0 && (4 * q & ((1 << a.pool.shift) - 1)) == 0) atomicAdd(a.pool.bad, 1ull);
    };
    // Four positions' places and what is there, AHEAD times; f(quad, place, weights, ages).
    constexpr int AHEAD = 4;
    auto each = [&](bool weights, bool times, auto f) __attribute__((always_inline)) {
#pragma unroll 1
        for (int q0 = t; q0 < quads; q0 += AHEAD * NT) {
            unsigned at[AHEAD];
            f32x4u_t weight[AHEAD];
            i32x4u_t when[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) at[k] = kv_spot(a.pool, table, u.head, 4 * (q0 + k * NT < quads ? q0 + k * NT : q0));
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const unsigned there = at[k] == KV_NOWHERE ? 0u : at[k];
                if (weights) weight[k] = *(const f32x4u_t *)(mass + there);
                if (times) when[k] = *(const i32x4u_t *)(born + there);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (q0 + k * NT < quads) {
                    met(q0 + k * NT, at[k]);
                    f(q0 + k * NT, at[k], weight[k], when[k]);
                }
        }
    };
    int newest = length - 1;
    if (!all && born) {
        newest = NEVER;
        auto note = [&](int q, unsigned at, f32x4u_t weight, i32x4u_t when) __attribute__((always_inline)) {
            u32x4_t x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool is = at != KV_NOWHERE && 4 * q + j < length;
                y[j] = is ? when[j] : NEVER;
                newest = largest(newest, (int)y[j]);
                x[j] = is ? kv_order(weight[j]) : 0u;
            }
            if (roomy) {
                *(u32x4_t *)(numbers + 4 * q) = x;
                *(u32x4_t *)(ages + 4 * q) = y;
            }
        };
        if (roomy) each(true, true, note);
        else each(false, true, [&](int q, unsigned at, f32x4u_t, i32x4u_t when) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) newest = largest(newest, at != KV_NOWHERE && 4 * q + j < length ? when[j] : NEVER);
        });
        newest = wave_fold(newest, largest);
        if (lane == 0) newest_of[w] = newest;
        __syncthreads();
        newest = wave_fold(newest_of[lane & (NW - 1)], largest);
    }
    const long recent_from = (long)newest - a.recent;  // above that
    auto safe = [&](int when) { return when > recent_from || when < a.early; };
    if (!all && cached) {
        if (born && roomy) {  // (a thread's own)
#pragma unroll 1
            for (int q = t; q < quads; q += NT) {
                u32x4_t x = *(const u32x4_t *)(numbers + 4 * q), y = *(const u32x4_t *)(ages + 4 * q);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = x[j] != 0 && safe((int)y[j]) ? 0xFFFFFFFFu : x[j];
                *(u32x4_t *)(numbers + 4 * q) = x;
            }
        } else {
            auto put = [&](int q, unsigned at, f32x4u_t weight, i32x4u_t when) __attribute__((always_inline)) {
                u32x4_t x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = at == KV_NOWHERE || 4 * q + j >= length ? 0u : safe(born ? when[j] : 4 * q + j) ? 0xFFFFFFFFu : kv_order(weight[j]);
                *(u32x4_t *)(numbers + 4 * q) = x;
            };
            each(true, born != nullptr, put);
        }
    }
    __syncthreads();
    // What a thread has summed over its slots, before it over all threads' (`place`: one for each call).
    auto before_all = [&](int place, unsigned mine) __attribute__((always_inline)) {
        unsigned sum = mine;
        const unsigned before = kv_before(sum);
        if (lane == 0) waves[place][w] = sum;
        __syncthreads();
        unsigned others = lane < NW ? waves[place][lane & (NW - 1)] : 0u;
        const unsigned ahead = kv_before(others);
        return before + (unsigned)__builtin_amdgcn_readlane((int)ahead, w);
    };
    auto rest = [&](auto here) __attribute__((always_inline)) {  // `here`: the numbers are in LDS
        constexpr bool HERE = decltype(here)::value;
        auto four = [&](int q) {  // (what fills up the last four is less than all else)
            if constexpr (HERE) return *(const u32x4_t *)(numbers + 4 * q);
            u32x4_t x = u32x4_t{0, 0, 0, 0};
            const unsigned at = kv_spot(a.pool, table, u.head, 4 * q);
            if (at == KV_NOWHERE) return x;
            const f32x4u_t weight = *(const f32x4u_t *)(mass + at);
            i32x4u_t when = {4 * q, 4 * q + 1, 4 * q + 2, 4 * q + 3};
            if (born) when = *(const i32x4u_t *)(born + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = 4 * q + j >= length ? 0u : safe(when[j]) ? 0xFFFFFFFFu : kv_order(weight[j]);
            return x;
        };
        unsigned bar = 0, ties = keep;  // what is above the bar stays, and of what is equal the first `ties`
        bool every = all;               // all that is equal
#pragma unroll 1
        for (int turn = 0; turn < TURNS && !every; ++turn) {
            const int shift = turn == 0 ? 21 : turn == 1 ? 10 : 0, bits = turn == 2 ? 10 : 11;
#pragma unroll 1
            for (int q = t; q < quads; q += NT) {
                const u32x4_t x = four(q);
                if (!HERE && turn == 0 && !born && x[0] == 0) met(q, KV_NOWHERE);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (turn == 0 || ((x[j] ^ bar) >> (shift + bits)) == 0) atomicAdd(&counts[turn][(x[j] >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // from the top: thread t has EACH digits from KV_DIGIT - 1 - EACH t down.  All waves find the wave, the lane and the digit that reach `ties`.
            auto digits_of = [&](int thread, unsigned (&c)[EACH]) __attribute__((always_inline)) {
                unsigned sum = 0;
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    c[k] = counts[turn][KV_DIGIT - 1 - EACH * thread - k];
                    sum += c[k];
                }
                return sum;
            };
            unsigned c[EACH], sum = digits_of(t, c);
            kv_before(sum);
            if (lane == 0) waves[turn][w] = sum;
            __syncthreads();
            auto reaching = [&](unsigned mine, unsigned before) { return __ffsll((long long)__ballot(before < ties && before + mine >= ties)) - 1; };
            unsigned mine = lane < NW ? waves[turn][lane & (NW - 1)] : 0u, before;
            sum = mine;
            before = kv_before(sum);
            const int of_wave = reaching(mine, before);
            const unsigned ahead = (unsigned)__builtin_amdgcn_readlane((int)before, of_wave);
            sum = mine = digits_of(64 * of_wave + lane, c);
            before = ahead + kv_before(sum);
            const int of_lane = reaching(mine, before);
            unsigned digit = 0, above = 0, same = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                if (before < ties && before + c[k] >= ties) {
                    digit = KV_DIGIT - 1 - EACH * (64 * of_wave + lane) - k;
                    above = before;
                    same = c[k];
                }
                before += c[k];
            }
            bar |= (unsigned)__builtin_amdgcn_readlane((int)digit, of_lane) << shift;
            ties -= (unsigned)__builtin_amdgcn_readlane((int)above, of_lane);
            every = (unsigned)__builtin_amdgcn_readlane((int)same, of_lane) == ties;  // (with whatever digits follow)
        }
        // a thread's slots, in order
        const int each_of = (quads + NT - 1) / NT, begin = t * each_of, end = begin + each_of < quads ? begin + each_of : quads;
        int cut = 0x7FFFFFFF;  // the last one of the equal ones that stay
        if (!every) {
            unsigned mine = 0;
#pragma unroll 1
            for (int q = begin; q < end; ++q) {
                const u32x4_t x = four(q);
#pragma unroll
                for (int j = 0; j < 4; ++j) mine += x[j] == bar ? 1u : 0u;
            }
            unsigned before = before_all(TURNS, mine);
            if (before < ties && before + mine >= ties)
                for (int q = begin; q < end; ++q) {
                    const u32x4_t x = four(q);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (x[j] == bar && ++before == ties) last_equal = 4 * q + j;
                }
            __syncthreads();
            cut = last_equal;
        }
        auto stays = [&](int i, unsigned x) { return i < length && (x > bar || (x == bar && i <= cut)); };
        unsigned so_far = 0;
#pragma unroll 1
        for (int q = begin; q < end; ++q) {
            const u32x4_t x = four(q);
#pragma unroll
            for (int j = 0; j < 4; ++j) so_far += stays(4 * q + j, x[j]) ? 1u : 0u;
        }
        so_far = before_all(TURNS + 1, so_far);
        // `where`: of a slot below `keep` -1, or (it becomes free) the number of free ones before it.  `movers`: the slots from `keep` on that stay, the last one first.
        auto ranked = [&](int *where, int *movers) __attribute__((always_inline)) {
            int stayed = (int)so_far;
#pragma unroll 1
            for (int q = begin; q < end; ++q) {
                const u32x4_t x = four(q);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * q + j;
                    const bool yes = stays(i, x[j]);
                    if (i == keep) moving = keep - stayed;
                    if (i < u.stay) where[i] = yes ? -1 : i - stayed;
                    else if (yes) movers[keep - 1 - stayed] = i;
                    stayed += yes;
                }
            }
            __syncthreads();  // (what the workgroup has written its own threads see)
            const int last = all ? 0 : moving - 1, to_most = a.to_width > (SISO_KV_MOST >> a.pool.shift) ? (int)SISO_KV_MOST : (int)(a.to_width << a.pool.shift);
            constexpr int MOVES = NT == 1024 ? 2 : 4;
#pragma unroll 1
            for (int i0 = t; i0 < u.stay; i0 += MOVES * NT) {
                int of[MOVES];
                unsigned at[MOVES], spot[MOVES];
                float weight[MOVES];
                int when[MOVES];
#pragma unroll
                for (int k = 0; k < MOVES; ++k) {
                    const int i = i0 + k * NT, rank = i < u.stay ? where[i] : -1;
                    of[k] = rank >= 0 ? movers[last - rank] : to && i < u.stay ? i : -1;
                    if (i < u.stay) from[i] = of[k];
                }
#pragma unroll
                for (int k = 0; k < MOVES; ++k) {
                    const int i = i0 + k * NT;
                    at[k] = of[k] >= 0 ? kv_spot(a.pool, table, u.head, of[k]) : KV_NOWHERE;
                    spot[k] = of[k] < 0 || (to && i >= to_most) ? KV_NOWHERE : kv_spot(a.pool, to ? to : table, u.head, i);
                }
#pragma unroll
                for (int k = 0; k < MOVES; ++k) {
                    weight[k] = at[k] != KV_NOWHERE ? mass[at[k]] : 0.f;
                    when[k] = born && at[k] != KV_NOWHERE ? born[at[k]] : 0;
                }
#pragma unroll
                for (int k = 0; k < MOVES; ++k)
                    if (spot[k] != KV_NOWHERE) {
                        mass[spot[k]] = weight[k];
                        if (born) born[spot[k]] = when[k];
                    }
            }
        };
        // (where the ages were: `keep` numbers and of those that move at most length - keep)
        if (HERE && roomy) ranked((int *)ages, (int *)ages + u.stay);
        else ranked(from, a.list + (long)blockIdx.x * keep);
    };
    if (cached) rest(std::true_type{});
    else rest(std::false_type{});
}

// ---------------------------------------------------------------------------- what moves
// One wave for a block of 16 slots of a unit.  A lane has every fourth chunk of one slot's key, and of every 64th dimension (in the order in which they lie) the
// eight tokens of each half, from as many places, whose addresses are the wave's.  What is read in place lies behind all that is written.
// Bound by lines that are read for a part: of a token's value every eighth element of its half's lines is its own (10,240 positions of 8 heads out of
// 25,683 in 8 bits: 15 us, where 21 MB out and in would take 9; 264 heads of 64 elements that lose up to 64 of 1,064 positions: 9 us).
template <int DP, bool FP8>
__global__ __launch_bounds__(256) void k_kv_move(KvEvict a, int blocks) {
    constexpr int ES = FP8 ? 1 : 2, CHUNKS = DP * ES / 16, NC = CHUNKS * 16 / 64;
    using E = typename std::conditional<FP8, byte_t, bf16_t>::type;
    using Eight = typename std::conditional<FP8, uint2, u32x4_t>::type;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), four = (blocks + 3) / 4;
    const long in_launch = blockIdx.x / four;
    const int at = 16 * ((int)(blockIdx.x % four) * 4 + w);
    const KvUnit u = kv_unit(a, a.unit0 + in_launch);
    if (at >= u.stay || (!a.to && u.s.length <= a.keep)) return;
    const int *const table = a.batch.pages + (long)u.s.b * a.batch.width;
    const int key = lane & 15;
    const int of = at + key < u.stay ? a.from[in_launch * a.keep + at + key] : -1;  // (the same in every 16 lanes)
    if (__ballot(of >= 0) == 0) return;
    int of_page = of >= 0 ? table[of >> a.pool.shift] : -1;
    if (a.to && (at >> a.pool.shift) >= a.to_width) return;
    const int page = a.to ? a.to[(long)u.s.b * a.to_width + (at >> a.pool.shift)] : table[at >> a.pool.shift];
    if (of >= 0 && !kv_is_page(a.pool, of_page)) {
        of_page = -1;
        if (u.head == 0 && lane < 16) atomicAdd(a.pool.bad, 1ull);
    }
    if (!kv_is_page(a.pool, page)) {
        if (lane == 0 && u.head == 0) atomicAdd(a.pool.bad, 1ull);
        return;
    }
    char *const pool_k = a.pool.k + u.layer * a.layer_bytes, *const pool_v = a.pool.v + u.layer * a.layer_bytes;
    const size_t to_block = kv_block_at(a.pool, page, u.head, at) * ES;
    u32x4_t k[NC];
    {
        const char *from_k = pool_k + kv_block_at(a.pool, of_page >= 0 ? of_page : 0, u.head, of >= 0 ? of : 0) * ES + (of & 15) * 16;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            k[c] = u32x4_t{0, 0, 0, 0};
            if (of_page >= 0) k[c] = *(const u32x4_t *)(from_k + ((lane >> 4) + 4 * c) * 256);
        }
    }
    const bool full = (__ballot(of_page >= 0) & 0xFFFFu) == 0xFFFFu;  // all 16 come from pages: loads that wait for nothing but their addresses
    float scale = 0.f;
    float *const scales = (lane < 16 ? a.pool.ks : a.pool.vs) + u.layer * a.layer_scales;
    if (FP8 && lane < 32 && of_page >= 0) scale = scales[kv_scale_at(a.pool, of_page, u.head, of)];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        E *const to_v = (E *)(pool_v + to_block) + (size_t)h * DP * 8;
        if (full) {
            E x[8][DP / 64];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int token = (s & 3) + 4 * h + 8 * (s >> 2), slot = __builtin_amdgcn_readlane(of, token), from_page = __builtin_amdgcn_readlane(of_page, token);
                const E *from_v = (const E *)(pool_v + kv_block_at(a.pool, from_page, u.head, slot) * ES) + (size_t)kv_half(slot & 15) * DP * 8 + kv_slot(slot & 15);
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) x[s][i] = from_v[(lane + 64 * i) * 8];
            }
#pragma unroll
            for (int i = 0; i < DP / 64; ++i) {
                unsigned y[2 * ES];
#pragma unroll
                for (int c = 0; c < 2 * ES; ++c) {
                    y[c] = 0;
#pragma unroll
                    for (int s = 0; s < 4 / ES; ++s) y[c] |= (unsigned)x[4 / ES * c + s][i] << (8 * ES * s);
                }
                Eight z;
                __builtin_memcpy(&z, y, sizeof(z));
                *(Eight *)(to_v + (lane + 64 * i) * 8) = z;
            }
            continue;
        }
        E x[DP / 64][8];
        bool whole = true;
        unsigned mine = 0;  // which of the eight are written
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int token = (s & 3) + 4 * h + 8 * (s >> 2), slot = __builtin_amdgcn_readlane(of, token), from_page = __builtin_amdgcn_readlane(of_page, token);
            if (slot >= 0) mine |= 1u << s;
            else whole = false;
            const E *from_v = (const E *)(pool_v + kv_block_at(a.pool, from_page >= 0 ? from_page : 0, u.head, slot >= 0 ? slot : 0) * ES) + (size_t)kv_half(slot & 15) * DP * 8 + kv_slot(slot & 15);
#pragma unroll
            for (int i = 0; i < DP / 64; ++i) {
                x[i][s] = 0;
                if (from_page >= 0) x[i][s] = from_v[(lane + 64 * i) * 8];
            }
        }
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) {
            if (whole) {
                Eight y;
                __builtin_memcpy(&y, x[i], sizeof(y));
                *(Eight *)(to_v + (lane + 64 * i) * 8) = y;
            } else
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    if (mine >> s & 1) to_v[(lane + 64 * i) * 8 + s] = x[i][s];
        }
    }
    if (of >= 0)
#pragma unroll
        for (int c = 0; c < NC; ++c) *(u32x4_t *)(pool_k + to_block + (((lane >> 4) + 4 * c) * 16 + key) * 16) = k[c];
    if (FP8 && lane < 32 && of >= 0) scales[kv_scale_at(a.pool, page, u.head, at) + key] = scale;
}

extern "C" int siso_kv_evict(siso_kv *kv, int layer, const siso_kv_batch *batch, long keep, long recent, long early, float *mass, int *born, const int *to,
                             long to_width) {
    if (!kv) return SISO_EINVAL;
    if (layer < -1) return kv_fail(kv, SISO_EINVAL, "siso_kv_evict: layer %d", layer);
    KvEvict a;
    const int rc = kv_batch(kv, "siso_kv_evict", layer < 0 ? 0 : layer, batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (keep < 1 || keep > 1L << 23 || recent < 0 || early < 0 || recent > keep || early > keep - recent)
        return kv_fail(kv, SISO_EINVAL, "siso_kv_evict: %ld positions are kept, %ld recent and %ld early ones", keep, recent, early);
    if (a.batch.n == 0) return SISO_OK;
    if (!mass || (((uintptr_t)mass | (uintptr_t)born) & 3)) return kv_fail(kv, SISO_EINVAL, "siso_kv_evict: masses must be there, aligned to their type");
    if (to && (to_width < 0 || to_width > SISO_KV_MOST / kv->page_tokens)) return kv_fail(kv, SISO_EINVAL, "siso_kv_evict: %ld pages of a sequence", to_width);
    const int at = layer < 0 ? 0 : layer;
    a.pool = kv_pool(kv, at);
    a.keep = (int)keep;
    a.recent = (int)recent;
    a.early = (int)early;
    a.mass = mass + (size_t)at * kv->layer_scales;
    a.born = born ? born + (size_t)at * kv->layer_scales : nullptr;
    a.to = to;
    a.to_width = to ? to_width : 0;
    a.layer_bytes = (long)kv->layer_bytes;
    a.layer_scales = (long)kv->layer_scales;
    a.layers = layer < 0 ? kv->layers : 1;
    // as many units at a time as the workspace has room for, and as a launch has threads for
    const long blocks = (keep + 15) / 16, units = (long)a.batch.n * a.layers * kv->kv_heads;
    long each = (long)SISO_KV_PARTS / (2 * keep);
    if (each > (1L << 23) / blocks) each = (1L << 23) / blocks;
    if (each > 1L << 21) each = 1L << 21;
    if (each < 1) each = 1;
    a.from = (int *)kv->parts;
    long room = batch->max_length > 0 && batch->max_length < a.batch.most ? batch->max_length : a.batch.most;
    room = room < 256 ? 512 : room > KV_CHOOSE_ROOM / 2 ? KV_CHOOSE_ROOM : 2 * ((room + 3) & ~3L);
    const bool few = room <= 2 * KV_CHOOSE_FEW && units > 256;
    if (!few && room * 4 > 32 * 1024) KV_TRY(kv, hipFuncSetAttribute((const void *)k_kv_choose<1024>, hipFuncAttributeMaxDynamicSharedMemorySize, KV_CHOOSE_ROOM * 4));
    for (a.unit0 = 0; a.unit0 < units; a.unit0 += each) {
        a.units = units - a.unit0 < each ? units - a.unit0 : each;
        a.list = a.from + a.units * keep;
        if (few) hipLaunchKernelGGL(k_kv_choose<256>, dim3((unsigned)a.units), dim3(256), (size_t)room * 4, kv->stream, a, (int)room);
        else hipLaunchKernelGGL(k_kv_choose<1024>, dim3((unsigned)a.units), dim3(1024), (size_t)room * 4, kv->stream, a, (int)room);
        KV_TRY(kv, hipGetLastError());
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.units * ((blocks + 3) / 4))), dim3(256), 0, kv->stream, a, (int)blocks); };
        switch (kv->dp / 64 + (kv->dtype == SISO_FP8 ? 4 : 0)) {
            case 1: go(k_kv_move<64, false>); break;
            case 2: go(k_kv_move<128, false>); break;
            case 3: go(k_kv_move<192, false>); break;
            case 4: go(k_kv_move<256, false>); break;
            case 5: go(k_kv_move<64, true>); break;
            case 6: go(k_kv_move<128, true>); break;
            case 7: go(k_kv_move<192, true>); break;
            default: go(k_kv_move<256, true>); break;
        }
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}
