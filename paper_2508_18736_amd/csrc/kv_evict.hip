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
// Numbers that are ordered as the masses are; what has none is less than all else.
__device__ __forceinline__ unsigned kv_order(float mass) {
    const unsigned x = __float_as_uint(mass + 0.f);  // (the two zeros are equal)
    return mass != mass ? 0u : x >> 31 ? ~x : x | 0x80000000u;
}

#define KV_CHOOSE 1024
#define KV_DIGIT 2048

// ---------------------------------------------------------------------------- which positions stay
// One workgroup a unit.  The `keep`-th largest number is found digit by digit (11, 11 and 10 bits), from counts of each digit's
// values.  Each wave then goes over a stretch of the slots, in order.
__global__ __launch_bounds__(KV_CHOOSE) void k_kv_choose(KvEvict a) {
    __shared__ unsigned counts[KV_DIGIT];
    __shared__ unsigned waves[3][16];
    __shared__ int newest_of[16];
    __shared__ unsigned digit, above;
    const long unit = a.unit0 + blockIdx.x;
    const KvUnit u = kv_unit(a, unit);
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), length = u.s.length, keep = a.keep;
    int *const from = a.from + (long)blockIdx.x * keep, *const list = a.list + (long)blockIdx.x * keep;
    float *const mass = a.mass + u.layer * a.layer_scales;
    int *const born = a.born ? a.born + u.layer * a.layer_scales : nullptr;
    const int *const table = a.batch.pages + (long)u.s.b * a.batch.width, *const to = a.to ? a.to + (long)u.s.b * a.to_width : nullptr;
    const int to_most = a.to_width > (SISO_KV_MOST >> a.pool.shift) ? (int)SISO_KV_MOST : (int)(a.to_width << a.pool.shift);
    const bool all = length <= keep;
    if (all && !to) {
        return;
    }
    int newest = 0;
    if (!all && born) {
        newest = -0x7FFFFFFF - 1;
        for (int i = t; i < length; i += KV_CHOOSE) {
            const long at = kv_spot(a.pool, table, u.head, i);
            if (at >= 0 && born[at] > newest) newest = born[at];
        }
        newest = wave_fold(newest, [](int x, int y) __attribute__((always_inline)) { return x > y ? x : y; });
        if (lane == 0) newest_of[w] = newest;
        __syncthreads();
        newest = wave_fold(newest_of[lane & 15], [](int x, int y) __attribute__((always_inline)) { return x > y ? x : y; });
    } else newest = length - 1;
    const long recent_from = (long)newest - a.recent;  // above that
    auto number = [&](int i) -> unsigned {
        const long at = kv_spot(a.pool, table, u.head, i);
        if (at < 0) return 0u;
        const int when = born ? born[at] : i;
        return when > recent_from || when < a.early ? 0xFFFFFFFFu : kv_order(mass[at]);
    };
    unsigned bar = 0;  // what is above it stays, and of what is equal the first `ties`
    int ties = 0;
    if (!all) {
        unsigned left = keep;  // of the numbers that have the digits found so far, so many stay
        for (int turn = 0; turn < 3; ++turn) {
            const int shift = turn == 0 ? 21 : turn == 1 ? 10 : 0, bits = turn == 2 ? 10 : 11;
            for (int i = t; i < KV_DIGIT; i += KV_CHOOSE) counts[i] = 0;
            __syncthreads();
            for (int i = t; i < length; i += KV_CHOOSE) {
                const unsigned x = number(i);
                if (turn == 0 || (x >> (shift + bits)) == (bar >> (shift + bits))) atomicAdd(&counts[(x >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // from the top: thread t has digits 2047 - 2 t and 2046 - 2 t
            const unsigned c0 = counts[KV_DIGIT - 1 - 2 * t], c1 = counts[KV_DIGIT - 2 - 2 * t];
            unsigned upto = c0 + c1;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const unsigned x = __shfl_up(upto, off);
                if (lane >= off) upto += x;
            }
            if (lane == 63) waves[0][w] = upto;
            __syncthreads();
            for (int i = 0; i < w; ++i) upto += waves[0][i];
            const unsigned before = upto - c0 - c1;
            if (before < left && upto >= left) {
                const bool second = before + c0 < left;
                digit = second ? KV_DIGIT - 2 - 2 * t : KV_DIGIT - 1 - 2 * t;
                above = second ? before + c0 : before;
            }
            __syncthreads();
            bar |= digit << shift;
            left -= above;
        }
        ties = (int)left;
    }
    // a wave's slots, 64 at a time
    const int stretch = ((length + KV_CHOOSE - 1) / KV_CHOOSE) * 64, begin = w * stretch;
    const int end = begin + stretch < length ? begin + stretch : length;
    unsigned equal = 0;
    if (!all)
        for (int i0 = begin; i0 < end; i0 += 64) equal += __popcll(__ballot(i0 + lane < end && number(i0 + lane) == bar));
    if (lane == 0) waves[0][w] = equal;
    __syncthreads();
    unsigned equal_before = 0;
    for (int i = 0; i < w; ++i) equal_before += waves[0][i];
    const u64 below = ((u64)1 << lane) - 1;
    auto stays = [&](int i, unsigned &equals) {  // of the wave's next 64 slots
        const unsigned x = i < end ? number(i) : 0u;
        const u64 same = __ballot(i < end && x == bar);
        const bool yes = all ? i < end : i < end && (x > bar || (x == bar && equals + __popcll(same & below) < (unsigned)ties));
        equals += __popcll(same);
        return yes;
    };
    unsigned holes = 0, movers = 0, equals = equal_before;
    for (int i0 = begin; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const bool yes = stays(i, equals);
        holes += __popcll(__ballot(i < keep && i < end && !yes));
        movers += __popcll(__ballot(i >= keep && yes));
    }
    if (lane == 0) {
        waves[1][w] = holes;
        waves[2][w] = movers;
    }
    __syncthreads();
    unsigned hole = 0, mover = 0;
    for (int i = 0; i < w; ++i) {
        hole += waves[1][i];
        mover += waves[2][i];
    }
    equals = equal_before;
    for (int i0 = begin; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const bool yes = stays(i, equals), empty = i < keep && i < end && !yes, moves = i >= keep && yes;
        const u64 empties = __ballot(empty), movings = __ballot(moves);
        if (i < keep && i < end) from[i] = empty ? -2 - (int)(hole + __popcll(empties & below)) : to ? i : -1;
        if (moves) list[mover + __popcll(movings & below)] = i;
        hole += __popcll(empties);
        mover += __popcll(movings);
    }
    __syncthreads();  // (what the workgroup has written to memory its own threads see)
    for (int i = t; i < u.stay; i += KV_CHOOSE) {
        int of = from[i];
        if (of <= -2) {
            of = list[-2 - of];
            from[i] = of;
        }
        if (of < 0) continue;
        const long at = kv_spot(a.pool, table, u.head, of), spot = to ? (i < to_most ? kv_spot(a.pool, to, u.head, i) : -1) : kv_spot(a.pool, table, u.head, i);
        if (spot < 0) continue;
        mass[spot] = at >= 0 ? mass[at] : 0.f;
        if (born) born[spot] = at >= 0 ? born[at] : 0;
    }
}

// ---------------------------------------------------------------------------- what moves
// One workgroup for a block of 16 slots of a unit: keys a thread for a chunk of 16 bytes, values a thread for a dimension of a half's eight tokens.
// What is read in place lies behind all that is written.
template <bool FP8>
__global__ __launch_bounds__(256) void k_kv_move(KvEvict a, int blocks) {
    constexpr int ES = FP8 ? 1 : 2;
    using E = typename std::conditional<FP8, byte_t, bf16_t>::type;
    using Eight = typename std::conditional<FP8, uint2, u32x4_t>::type;
    __shared__ int from[16], page_of[16];
    const long unit = a.unit0 + blockIdx.x / blocks;
    const int block = (int)(blockIdx.x % blocks), t = threadIdx.x;
    const KvUnit u = kv_unit(a, unit);
    const int at = 16 * block;
    if (at >= u.stay || (!a.to && u.s.length <= a.keep)) return;
    const int *const table = a.batch.pages + (long)u.s.b * a.batch.width;
    if (t < 16) {
        const int of = at + t < u.stay ? a.from[(blockIdx.x / blocks) * (long)a.keep + at + t] : -1;
        from[t] = of;
        int page = of >= 0 ? table[of >> a.pool.shift] : -1;
        if (of >= 0 && !kv_is_page(a.pool, page)) {
            page = -1;
            if (u.head == 0) atomicAdd(a.pool.bad, 1ull);
        }
        page_of[t] = page;
    }
    __syncthreads();
    bool any = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) any = any || from[i] >= 0;
    if (!any) return;
    int page;
    if (a.to) {
        if ((at >> a.pool.shift) >= a.to_width) return;
        page = a.to[(long)u.s.b * a.to_width + (at >> a.pool.shift)];
    } else page = table[at >> a.pool.shift];
    if (!kv_is_page(a.pool, page)) {
        if (t == 0 && u.head == 0) atomicAdd(a.pool.bad, 1ull);
        return;
    }
    const int dp = a.pool.dp, chunks = dp * ES / 16;
    char *const pool_k = a.pool.k + u.layer * a.layer_bytes, *const pool_v = a.pool.v + u.layer * a.layer_bytes;
    char *const kb = pool_k + kv_block_at(a.pool, page, u.head, at) * ES, *const vb = pool_v + kv_block_at(a.pool, page, u.head, at) * ES;
    for (int i = t; i < 16 * chunks; i += 256) {
        const int key = i & 15, c = i >> 4, of = from[key];
        if (of < 0) continue;
        u32x4_t x = u32x4_t{0, 0, 0, 0};
        if (page_of[key] >= 0) x = *(const u32x4_t *)(pool_k + kv_block_at(a.pool, page_of[key], u.head, of) * ES + (c * 16 + (of & 15)) * 16);
        *(u32x4_t *)(kb + (c * 16 + key) * 16) = x;
    }
    for (int i = t; i < 2 * dp; i += 256) {
        const int h = i >= dp, d = i - h * dp;
        auto eight_at = [&](int half) { return FP8 ? kv_v8_at(dp, half, d) : (size_t)(half * dp + d) * 8; };
        E x[8];
        bool whole = true;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int key = (s & 3) + 4 * h + 8 * (s >> 2), of = from[key];
            whole = whole && of >= 0;
            x[s] = 0;
            if (of >= 0 && page_of[key] >= 0)
                x[s] = ((const E *)(pool_v + kv_block_at(a.pool, page_of[key], u.head, of) * ES))[eight_at(kv_half(of & 15)) + kv_slot(of & 15)];
        }
        E *to = (E *)vb + eight_at(h);
        if (whole) {
            Eight y;
            __builtin_memcpy(&y, x, sizeof(y));
            *(Eight *)to = y;
        } else
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (from[(s & 3) + 4 * h + 8 * (s >> 2)] >= 0) to[s] = x[s];
    }
    if (FP8 && t < 32) {
        float *scales = (t < 16 ? a.pool.ks : a.pool.vs) + u.layer * a.layer_scales;
        const int key = t & 15, of = from[key];
        if (of >= 0) scales[kv_scale_at(a.pool, page, u.head, at) + key] = page_of[key] >= 0 ? scales[kv_scale_at(a.pool, page_of[key], u.head, of)] : 0.f;
    }
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
    for (a.unit0 = 0; a.unit0 < units; a.unit0 += each) {
        a.units = units - a.unit0 < each ? units - a.unit0 : each;
        a.list = a.from + a.units * keep;
        hipLaunchKernelGGL(k_kv_choose, dim3((unsigned)a.units), dim3(KV_CHOOSE), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
        const dim3 grid((unsigned)(a.units * blocks));
        if (kv->dtype == SISO_FP8) hipLaunchKernelGGL(k_kv_move<true>, grid, dim3(256), 0, kv->stream, a, (int)blocks);
        else hipLaunchKernelGGL(k_kv_move<false>, grid, dim3(256), 0, kv->stream, a, (int)blocks);
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}
