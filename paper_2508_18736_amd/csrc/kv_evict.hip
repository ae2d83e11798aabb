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
// Where a slot's numbers are, of mass and born (of the layer); -1: its page is none.
__device__ __forceinline__ long kv_spot(const KvPool &pool, const int *table, int head, int at) {
    const int page = table[at >> pool.shift];
    return kv_is_page(pool, page) ? (long)kv_scale_at(pool, page, head, at) : -1;
}
// Numbers that are ordered as the masses are; NaN is less than all else (and 0, of positions without a page, is less than that).
__device__ __forceinline__ unsigned kv_order(float mass) {
    const unsigned x = __float_as_uint(mass + 0.f);  // (the two zeros are equal)
    return mass != mass ? 1u : x >> 31 ? ~x : x | 0x80000000u;
}

#define KV_DIGIT 2048

// ---------------------------------------------------------------------------- which positions stay
#define KV_CHOOSE_ROOM 32768  // words of LDS: two for each position (its number and its age), or one; of more positions both are read from memory whenever they are asked for
// Threads of a workgroup: 1,024, or 256 where there are more units than CUs, of at most so many positions each: workgroups of 1,024 that share a CU wait for
// one another at barriers, of few positions longer than the rest takes.  Calls of 48 sequences, 8 heads (us, 256 against 1,024 threads): of 400 positions
// 58.7 and 65.9, of 1,000 127 and 138, of 1,900 245 and 253; of 16 sequences of 1,900 93.1 and 89.9.
#define KV_CHOOSE_FEW 2048
// One workgroup a unit.  Its positions' numbers are brought to LDS once; the `keep`-th largest is found digit by digit (11, 11 and 10 bits), from counts of
// each digit's values.  Each wave then goes over a stretch of the slots, in order: ranks are counts of ballots, so that nothing depends on scheduling.
// Bound by latency: about ten passes over LDS with a barrier each behind two dependent loads (page, then mass and born).
template <int NT>
__global__ __launch_bounds__(NT) void k_kv_choose(KvEvict a, int room) {
    extern __shared__ unsigned numbers[];
    __shared__ unsigned counts[KV_DIGIT];
    constexpr int NW = NT / 64, EACH = KV_DIGIT / NT;
    __shared__ unsigned waves[3][NW];
    __shared__ int newest_of[NW];
    __shared__ unsigned digit, above, same_digit;
    const KvUnit u = kv_unit(a, a.unit0 + blockIdx.x);
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), length = u.s.length, keep = a.keep;
    int *const from = a.from + (long)blockIdx.x * keep, *const list = a.list + (long)blockIdx.x * keep;
    float *const mass = a.mass + u.layer * a.layer_scales;
    int *const born = a.born ? a.born + u.layer * a.layer_scales : nullptr;
    const int *const table = a.batch.pages + (long)u.s.b * a.batch.width, *const to = a.to ? a.to + (long)u.s.b * a.to_width : nullptr;
    const int to_most = a.to_width > (SISO_KV_MOST >> a.pool.shift) ? (int)SISO_KV_MOST : (int)(a.to_width << a.pool.shift);
    const bool all = length <= keep, cached = length <= room;
    if (all && !to) return;
    // Numbers: MANY positions of a thread at a time.
    constexpr int MANY = 8;
    auto each = [&](auto f) __attribute__((always_inline)) {
        for (int i0 = t; i0 < length; i0 += MANY * NT) {
            long at[MANY];
#pragma unroll
            for (int k = 0; k < MANY; ++k) {
                const int i = i0 + k * NT;
                at[k] = kv_spot(a.pool, table, u.head, i < length ? i : i0);
            }
            f(i0, at);
        }
    };
    const bool both = born && 2L * length <= room;  // ages, too, are in LDS
    constexpr int NEVER = -0x7FFFFFFF - 1;
    int newest = length - 1;
    if (!all && born) {
        newest = NEVER;
        each([&](int i0, const long (&at)[MANY]) __attribute__((always_inline)) {
            int when[MANY];
            float weight[MANY];
#pragma unroll
            for (int k = 0; k < MANY; ++k) {
                when[k] = at[k] >= 0 ? born[at[k]] : NEVER;
                weight[k] = both && at[k] >= 0 ? mass[at[k]] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < MANY; ++k) newest = when[k] > newest ? when[k] : newest;
            if (both)
#pragma unroll
                for (int k = 0; k < MANY; ++k)
                    if (i0 + k * NT < length) {
                        numbers[i0 + k * NT] = at[k] >= 0 ? kv_order(weight[k]) : 0u;
                        numbers[length + i0 + k * NT] = (unsigned)when[k];
                    }
        });
        newest = wave_fold(newest, [](int x, int y) __attribute__((always_inline)) { return x > y ? x : y; });
        if (lane == 0) newest_of[w] = newest;
        __syncthreads();
        newest = wave_fold(newest_of[lane & (NW - 1)], [](int x, int y) __attribute__((always_inline)) { return x > y ? x : y; });
    }
    const long recent_from = (long)newest - a.recent;  // above that
    auto safe = [&](int when) { return when > recent_from || when < a.early; };
    auto number_of = [&](long at, int when, float weight) { return at < 0 ? 0u : safe(when) ? 0xFFFFFFFFu : kv_order(weight); };
    if (!all && both) {  // (a thread's own)
#pragma unroll 4
        for (int i = t; i < length; i += NT)
            if (numbers[i] != 0 && safe((int)numbers[length + i])) numbers[i] = 0xFFFFFFFFu;
    } else if (!all && cached)
        each([&](int i0, const long (&at)[MANY]) __attribute__((always_inline)) {
            int when[MANY];
            float weight[MANY];
#pragma unroll
            for (int k = 0; k < MANY; ++k) {
                weight[k] = at[k] >= 0 ? mass[at[k]] : 0.f;
                when[k] = !born ? i0 + k * NT : at[k] >= 0 ? born[at[k]] : 0;
            }
#pragma unroll
            for (int k = 0; k < MANY; ++k)
                if (i0 + k * NT < length) numbers[i0 + k * NT] = number_of(at[k], when[k], weight[k]);
        });
    auto number = [&](int i) -> unsigned {
        if (cached) return numbers[i];
        const long at = kv_spot(a.pool, table, u.head, i);
        return number_of(at, !born ? i : at >= 0 ? born[at] : 0, at >= 0 ? mass[at] : 0.f);
    };
    unsigned bar = 0;  // what is above it stays, and of what is equal the first `ties`
    int ties = 0;
    bool every = true;  // all that is equal
    if (!all) {
        unsigned left = keep;  // of the numbers that have the digits found so far, so many stay
        for (int turn = 0; turn < 3; ++turn) {
            const int shift = turn == 0 ? 21 : turn == 1 ? 10 : 0, bits = turn == 2 ? 10 : 11;
            for (int i = t; i < KV_DIGIT; i += NT) counts[i] = 0;
            __syncthreads();
            for (int i0 = t; i0 < length; i0 += 4 * NT) {
                unsigned x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = i0 + k * NT < length ? number(i0 + k * NT) : 0u;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + k * NT < length && (turn == 0 || (x[k] >> (shift + bits)) == (bar >> (shift + bits))))
                        atomicAdd(&counts[(x[k] >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // from the top: thread t has EACH digits from KV_DIGIT - 1 - EACH t down
            unsigned c[EACH], mine = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                c[k] = counts[KV_DIGIT - 1 - EACH * t - k];
                mine += c[k];
            }
            unsigned upto = mine;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const unsigned x = __shfl_up(upto, off);
                if (lane >= off) upto += x;
            }
            if (lane == 63) waves[0][w] = upto;
            __syncthreads();
            for (int i = 0; i < w; ++i) upto += waves[0][i];
            if (upto - mine < left && upto >= left) {
                unsigned ahead = upto - mine;
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    if (ahead < left && ahead + c[k] >= left) {
                        digit = KV_DIGIT - 1 - EACH * t - k;
                        above = ahead;
                        same_digit = c[k];
                    }
                    ahead += c[k];
                }
            }
            __syncthreads();
            bar |= digit << shift;
            left -= above;
            every = same_digit == left;
            if (every) break;  // (with whatever digits follow)
        }
        ties = (int)left;
    }
    // a wave's slots, 64 at a time
    const int stretch = ((length + NT - 1) / NT) * 64, begin = w * stretch;
    const int end = begin + stretch < length ? begin + stretch : length;
    const u64 below = ((u64)1 << lane) - 1;
    auto first_bits = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : ((u64)1 << n) - 1; };
    constexpr int AHEAD = 4;  // 64 slots, so many times
    auto in_order = [&](auto f) __attribute__((always_inline)) {
        for (int i0 = begin; i0 < end; i0 += 64 * AHEAD) {
            unsigned x[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) x[k] = !all && i0 + 64 * k + lane < end ? number(i0 + 64 * k + lane) : 0u;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) f(i0 + 64 * k, x[k]);
        }
    };
    unsigned equal_before = 0;
    if (!every) {
        unsigned equal = 0;
        in_order([&](int base, unsigned x) __attribute__((always_inline)) { equal += __popcll(__ballot(x == bar) & first_bits(end - base)); });
        if (lane == 0) waves[0][w] = equal;
        __syncthreads();
        for (int i = 0; i < w; ++i) equal_before += waves[0][i];
    }
    unsigned equals = equal_before, hole = 0, mover = 0;
    auto stays = [&](int base, unsigned x) __attribute__((always_inline)) {  // of the wave's next 64 slots
        const u64 in = first_bits(end - base);
        if (every) return (all ? ~0ull : __ballot(x >= bar)) & in;
        const u64 same = __ballot(x == bar) & in;
        const bool early = (same >> lane & 1) && equals + __popcll(same & below) < (unsigned)ties;
        equals += __popcll(same);
        return __ballot(x > bar || early) & in;
    };
    in_order([&](int base, unsigned x) __attribute__((always_inline)) {
        const u64 yes = stays(base, x), low = first_bits(keep - base);
        hole += __popcll(low & first_bits(end - base) & ~yes);
        mover += __popcll(yes & ~low);
    });
    if (lane == 0) {
        waves[1][w] = hole;
        waves[2][w] = mover;
    }
    __syncthreads();
    hole = mover = 0;
    for (int i = 0; i < w; ++i) {
        hole += waves[1][i];
        mover += waves[2][i];
    }
    equals = equal_before;
    in_order([&](int base, unsigned x) __attribute__((always_inline)) {
        const u64 yes = stays(base, x), low = first_bits(keep - base), empties = low & first_bits(end - base) & ~yes, movings = yes & ~low;
        const int i = base + lane;
        if (i < keep && i < end) from[i] = empties >> lane & 1 ? -2 - (int)(hole + __popcll(empties & below)) : to ? i : -1;
        if (movings >> lane & 1) list[mover + __popcll(movings & below)] = i;
        hole += __popcll(empties);
        mover += __popcll(movings);
    });
    __syncthreads();  // (what the workgroup has written to memory its own threads see)
    constexpr int MOVES = 4;
    for (int i0 = t; i0 < u.stay; i0 += MOVES * NT) {
        int of[MOVES];
#pragma unroll
        for (int k = 0; k < MOVES; ++k) of[k] = i0 + k * NT < u.stay ? from[i0 + k * NT] : -1;
#pragma unroll
        for (int k = 0; k < MOVES; ++k)
            if (of[k] <= -2) {
                of[k] = list[-2 - of[k]];
                from[i0 + k * NT] = of[k];
            }
        long at[MOVES], spot[MOVES];
        float weight[MOVES];
        int when[MOVES];
#pragma unroll
        for (int k = 0; k < MOVES; ++k) {
            const int i = i0 + k * NT;
            at[k] = of[k] >= 0 ? kv_spot(a.pool, table, u.head, of[k]) : -1;
            spot[k] = of[k] < 0 || (to && i >= to_most) ? -1 : kv_spot(a.pool, to ? to : table, u.head, i);
        }
#pragma unroll
        for (int k = 0; k < MOVES; ++k) {
            weight[k] = at[k] >= 0 ? mass[at[k]] : 0.f;
            when[k] = born && at[k] >= 0 ? born[at[k]] : 0;
        }
#pragma unroll
        for (int k = 0; k < MOVES; ++k)
            if (spot[k] >= 0) {
                mass[spot[k]] = weight[k];
                if (born) born[spot[k]] = when[k];
            }
    }
}

// ---------------------------------------------------------------------------- what moves
// One wave for a block of 16 slots of a unit.  A lane has every fourth chunk of one slot's key, and of every 64th dimension (in the order in which they lie) the
// eight tokens of each half, from as many places, whose addresses are the wave's.  What is read in place lies behind all that is written.
// Bound by lines that are read for a part: of a token's value every eighth element of its half's lines is its own (10,240 positions of 8 heads out of
// 25,683 in 8 bits).
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
    room = room < 256 ? 512 : room > KV_CHOOSE_ROOM / 2 ? KV_CHOOSE_ROOM : 2 * room;
    const bool few = room <= 2 * KV_CHOOSE_FEW && units > 256;
    if (!few && room * 4 > 48 * 1024) KV_TRY(kv, hipFuncSetAttribute((const void *)k_kv_choose<1024>, hipFuncAttributeMaxDynamicSharedMemorySize, KV_CHOOSE_ROOM * 4));
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
