// Attention over the paged cache (siso_kv_attend).  Layout of the pages: kv_internal.h.
#include <math.h>

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
    float scale;       // times log2(e): the softmax is one of powers of two
    int window;        // 0 = all
    int splits, split_len;  // the axis of positions is cut every split_len (a multiple of 32); the last takes what is left
    bf16_t *out;
    float *lse;
    float *parts;
    long slot0;
};

#define KV_TILE_SHIFT 5  // rows of a tile
#define KV_TILE_EXTRA 1

struct KvTile {
    KvSequence s;
    int row0, rows;    // of the sequence's rows of work: the first one of the tile, how many there are
    int lo, hi;        // positions that some row of the tile sees
    int all_lo, all_hi;  // positions that all rows of the tile see
};

__device__ __forceinline__ bool kv_find_tile(const KvAttend &a, long slot, KvTile &t) {
    const int b = a.batch.single && a.group <= 32 ? (int)slot : kv_sequence_of(a.batch, slot, a.group, KV_TILE_SHIFT, KV_TILE_EXTRA);
    t.s = kv_sequence(a.batch, b);
    const long j = a.batch.single && a.group <= 32 ? 0 : slot - kv_slots_before(t.s.first, b, a.group, KV_TILE_SHIFT, KV_TILE_EXTRA);
    const long work = (long)t.s.rows * a.group;
    if (j < 0 || j * 32 >= work) return false;
    t.row0 = (int)(j * 32);
    t.rows = work - j * 32 < 32 ? (int)(work - j * 32) : 32;
    const int first = t.s.start + t.row0 / a.group, last = t.s.start + (t.row0 + t.rows - 1) / a.group;
    t.hi = last + 1 > 0 ? last + 1 : 0;
    t.lo = a.window > 0 && first - a.window + 1 > 0 ? first - a.window + 1 : 0;
    t.all_hi = first + 1;
    t.all_lo = a.window > 0 && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
    return true;
}
// The part of a tile's positions that split `s` takes: [from, to), from a multiple of 32.
__device__ __forceinline__ void kv_split(const KvAttend &a, const KvTile &t, int s, int &from, int &to) {
    from = s * a.split_len;
    to = s + 1 == a.splits || t.hi < from + a.split_len ? t.hi : from + a.split_len;
    if (from < (t.lo & ~31)) from = t.lo & ~31;
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

// One workgroup for a tile of 32 rows and a split of the positions; its four waves take every fourth 32 of them, each with sums of
// its own, which are joined through LDS in the order of the waves.  Keys and values go straight from memory to
// registers: no wave reads what another does.
template <int DP, bool FP8>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void k_kv_attend_few(KvAttend a) {
    constexpr int ES = FP8 ? 1 : 2;
    constexpr int NF = FP8 ? DP / 32 : DP / 16;  // 16-byte operands of a lane for 32 keys, and for 32 values
    constexpr int NU = DP / 32;
    constexpr int RS = DP + 4;  // floats of a row in LDS
    __shared__ __attribute__((aligned(16))) float sh[4 * 32 * RS + 2 * 4 * 32];  // sums [4][32][RS], then maxima and sums [2][4][32]
    float *sh_m = sh + 4 * 32 * RS, *sh_l = sh_m + 4 * 32;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    const int head = blockIdx.x % a.pool.kv_heads;
    const long item = blockIdx.x / a.pool.kv_heads;
    const long slot = a.slot0 + item / a.splits;
    const int split = (int)(item % a.splits);
    KvTile t;
    if (!kv_find_tile(a, slot, t)) return;
    int from, to;
    kv_split(a, t, split, from, to);
    if (from >= to && a.splits > 1) return;

    // this lane's row (of both halves) as the operand Q^T
    const int row = t.row0 + n, token = row / a.group, qh = head * a.group + row % a.group;
    const bool valid = n < t.rows;
    const int pos = t.s.start + token;
    bf16x8_t qf[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const int d = FP8 ? 16 * (2 * (s >> 1) + h) + 8 * (s & 1) : 16 * s + 8 * h;
        u32x4_t x = {0, 0, 0, 0};
        if (valid && d < a.pool.dim) {
            const bf16_t *from_q = a.q + (long)(t.s.first + token) * a.q_token + (long)qh * a.q_head + d;
            if (a.vec) x = *(const u32x4_t *)from_q;
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = (unsigned)from_q[2 * i] | ((unsigned)from_q[2 * i + 1] << 16);
        }
        qf[s] = kv_as_bf16(x);
    }

    f32x16_t o[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) o[u] = f32x16_t{};
    float m = -INFINITY, l = 0.f;

    u32x4_t kf[NF], vf[NF];
    long page[2], next_page[2];
    // the pages of the two blocks from `at` on; a block beyond what the tile sees takes the other's
    auto find_pages = [&](int at, long (&p)[2]) {
        p[0] = kv_page(a.pool, a.batch, t.s.b, at);
        p[1] = at + 16 < t.hi ? kv_page(a.pool, a.batch, t.s.b, at + 16) : p[0];
    };
    auto load_keys = [&](int at, const long (&p)[2]) {
        const int blk = (lane >> 4) & 1;
        const size_t b0 = kv_block_at(a.pool, p[0] < 0 ? 0 : p[0], head, at), b1 = kv_block_at(a.pool, p[1] < 0 ? 0 : p[1], head, at + 16);
        const char *base = a.pool.k + (blk ? b1 : b0) * ES + h * 256 + (lane & 15) * 16;
#pragma unroll
        for (int s = 0; s < NF; ++s) kf[s] = *(const u32x4_t *)(base + s * 512);
    };
    auto load_values = [&](int at, const long (&p)[2]) {
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const char *base = a.pool.v + kv_block_at(a.pool, p[blk] < 0 ? 0 : p[blk], head, at + 16 * blk) * ES + (h * (NF / 2) * 32 + n) * 16;
#pragma unroll
            for (int u = 0; u < NF / 2; ++u) vf[blk * (NF / 2) + u] = *(const u32x4_t *)(base + u * 512);
        }
    };

    int at = from + 32 * w;
    if (at < to) {
        find_pages(at, page);
        load_keys(at, page);
        load_values(at, page);
    }
    for (; at < to; at += 128) {
        const bool more = at + 128 < to;
        if (more) find_pages(at + 128, next_page);
        float ks[16], vs[16];
        if constexpr (FP8) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const size_t sc = kv_scale_at(a.pool, page[g >> 1] < 0 ? 0 : page[g >> 1], head, at + 16 * (g >> 1)) + 8 * (g & 1) + 4 * h;
                const float4 x = *(const float4 *)(a.pool.ks + sc), y = *(const float4 *)(a.pool.vs + sc);
                ks[4 * g] = x.x, ks[4 * g + 1] = x.y, ks[4 * g + 2] = x.z, ks[4 * g + 3] = x.w;
                vs[4 * g] = y.x, vs[4 * g + 1] = y.y, vs[4 * g + 2] = y.z, vs[4 * g + 3] = y.w;
            }
        }
        f32x16_t s = {};
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(kf[i][0], kf[i][1]), qf[2 * i], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_codes_bf16(kf[i][2], kf[i][3]), qf[2 * i + 1], s, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NF; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_as_bf16(kf[i]), qf[i], s, 0, 0, 0);
        }
        if (more) load_keys(at + 128, next_page);

        // register r holds position at + 8 (r / 4) + 4 h + r % 4 of this lane's row
        const bool edge = at + 32 > t.all_hi || at < t.all_lo || (page[0] | page[1]) < 0;
        unsigned seen = 0xFFFFu;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= FP8 ? ks[r] * a.scale : a.scale;
        if (edge) {
            if (lane == 0 && (page[0] | page[1]) < 0) atomicAdd(a.pool.bad, 1ull);
            seen = 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int p = at + 8 * (r >> 2) + 4 * h + (r & 3);
                if (p <= pos && (a.window == 0 || p > pos - a.window) && page[r >> 3] >= 0) seen |= 1u << r;
                s[r] = seen >> r & 1 ? s[r] : -INFINITY;
            }
        }
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = fmaxf(m, kv_both_halves_max(top));
        if (__ballot(top > m) != 0) {  // (a maximum that stays needs no new sums)
            const float down = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
            l *= down;
#pragma unroll
            for (int u = 0; u < NU; ++u) o[u] *= down;
            m = top;
        }
        const float base = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - base);
            sum += s[r];
        }
        l += sum;
        if constexpr (FP8) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= vs[r];
            if (edge)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = seen >> r & 1 ? s[r] : 0.f;  // (the scale there may be NaN)
        } else if (edge) {
            // Nothing times an infinity is NaN: where some rows do not see a position, its value's infinities and NaN are
            // taken out of the product and added for the rows that see it.
            bool odd = false;
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) odd = odd || kv_not_finite(vf[i][c]);
            if (__ballot(odd) != 0) {
                float *mine = sh + w * 32 * RS;  // [row][32 positions], this wave's own
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[n * 36 + 8 * (r >> 2) + 4 * h + (r & 3)] = seen >> r & 1 ? s[r] : -1.f;
#pragma unroll
                for (int i = 0; i < NF; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if ((vf[i][c] & 0x7F80u) == 0x7F80u) vf[i][c] &= 0xFFFF0000u;
                        if ((vf[i][c] & 0x7F800000u) == 0x7F800000u) vf[i][c] &= 0xFFFFu;
                    }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
                for (int key = 0; key < 32; ++key) {
                    const long from_page = page[key >> 4];
                    if (from_page < 0) continue;
                    const float p = mine[n * 36 + key];
                    const bf16_t *v = (const bf16_t *)a.pool.v + kv_block_at(a.pool, from_page, head, at + (key & 16)) +
                                      (size_t)kv_half(key & 15) * DP * 8 + kv_slot(key & 15);
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const bf16_t x = v[(32 * u + 8 * (r >> 2) + 4 * h + (r & 3)) * 8];
                            if ((x & 0x7F80u) == 0x7F80u && p >= 0.f) o[u][r] += p * bf16_to_f32(x);
                        }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
        bf16x8_t pf[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) pf[r >> 3][r & 7] = (__bf16)s[r];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
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
        if (more) {
            load_values(at + 128, next_page);
            page[0] = next_page[0];
            page[1] = next_page[1];
        }
    }

    l = kv_both_halves_sum(l);
    if (h == 0) {
        sh_m[w * 32 + n] = m;
        sh_l[w * 32 + n] = l;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4 *)(sh + (w * 32 + n) * RS + 32 * u + 8 * g + 4 * h) = make_float4(o[u][4 * g], o[u][4 * g + 1], o[u][4 * g + 2], o[u][4 * g + 3]);
    __syncthreads();
    float *part = a.parts + (item * a.pool.kv_heads + head) * (32 * (DP + 2));
    for (int i = threadIdx.x; i < 32 * (DP / 4); i += 256) {
        const int r = i / (DP / 4), d = i % (DP / 4) * 4;
        if (r >= t.rows) break;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, sh_m[j * 32 + r]);
        float sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float mj = sh_m[j * 32 + r];
            const float f = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj - top);
            sum += sh_l[j * 32 + r] * f;
            const float4 y = *(const float4 *)(sh + (j * 32 + r) * RS + d);
            x.x += y.x * f, x.y += y.y * f, x.z += y.z * f, x.w += y.w * f;
        }
        if (a.splits > 1) {
            *(float4 *)(part + r * DP + d) = x;
            if (d == 0) {
                part[32 * DP + 2 * r] = top;
                part[32 * DP + 2 * r + 1] = sum;
            }
            continue;
        }
        const int work = t.row0 + r, tok = work / a.group, hd = head * a.group + work % a.group;
        const size_t at_out = (size_t)(t.s.first + tok) * a.group * a.pool.kv_heads + hd;
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        if (d < a.pool.dim)
            *(uint2 *)(a.out + at_out * a.pool.dim + d) = make_uint2((unsigned)f32_to_bf16(x.x * inv) | ((unsigned)f32_to_bf16(x.y * inv) << 16),
                                                                    (unsigned)f32_to_bf16(x.z * inv) | ((unsigned)f32_to_bf16(x.w * inv) << 16));
        if (d == 0 && a.lse) a.lse[at_out] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718056f;
    }
}

// Joins the splits of a tile, in their order.
template <int DP>
__global__ __launch_bounds__(256) void k_kv_attend_join(KvAttend a) {
    const int head = blockIdx.x % a.pool.kv_heads;
    const long slot = blockIdx.x / a.pool.kv_heads;
    KvTile t;
    if (!kv_find_tile(a, a.slot0 + slot, t)) return;
    for (int i = threadIdx.x; i < t.rows * (DP / 4); i += 256) {
        const int r = i / (DP / 4), d = i % (DP / 4) * 4;
        float top = -INFINITY, sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < a.splits; ++s) {
            int from, to;
            kv_split(a, t, s, from, to);
            if (from >= to) continue;
            const float *part = a.parts + ((slot * a.splits + s) * a.pool.kv_heads + head) * (32 * (DP + 2));
            const float mj = part[32 * DP + 2 * r], lj = part[32 * DP + 2 * r + 1];
            const float4 y = *(const float4 *)(part + r * DP + d);
            const float both = fmaxf(top, mj);
            const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - both), g = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj - both);
            x.x = x.x * f + y.x * g, x.y = x.y * f + y.y * g, x.z = x.z * f + y.z * g, x.w = x.w * f + y.w * g;
            sum = sum * f + lj * g;
            top = both;
        }
        const int work = t.row0 + r, tok = work / a.group, hd = head * a.group + work % a.group;
        const size_t at_out = (size_t)(t.s.first + tok) * a.group * a.pool.kv_heads + hd;
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        if (d < a.pool.dim)
            *(uint2 *)(a.out + at_out * a.pool.dim + d) = make_uint2((unsigned)f32_to_bf16(x.x * inv) | ((unsigned)f32_to_bf16(x.y * inv) << 16),
                                                                    (unsigned)f32_to_bf16(x.z * inv) | ((unsigned)f32_to_bf16(x.w * inv) << 16));
        if (d == 0 && a.lse) a.lse[at_out] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718056f;
    }
}

// Positions of a split, at least: eight tiles of 32 for each of the four waves cost more to join than they gain when cut further.
#define KV_SPLIT_LEAST 256
#define KV_WORKGROUPS 1024  // what fills the chip: 256 compute units, two workgroups each, twice

template <int DP, bool FP8>
static int attend(siso_kv *kv, KvAttend &a, long max_length) {
    const long slots = a.batch.single && a.group <= 32 ? a.batch.n : kv_slots_before(a.batch.rows, a.batch.n, a.group, KV_TILE_SHIFT, KV_TILE_EXTRA);
    const long tiles = slots * kv->kv_heads, room = (long)(kv->parts_floats / (32 * (DP + 2)));
    long splits = (max_length + KV_SPLIT_LEAST - 1) / KV_SPLIT_LEAST;
    if (splits > KV_WORKGROUPS / tiles) splits = KV_WORKGROUPS / tiles;
    if (splits > room / tiles) splits = room / tiles;
    if (splits < 1) splits = 1;
    a.split_len = (int)((max_length + splits * 128 - 1) / (splits * 128) * 128);
    if (a.split_len < 128) a.split_len = 128;
    a.splits = (int)splits;
    const long piece = (1L << 23) / (kv->kv_heads * splits);  // (a launch has fewer than 2^32 threads)
    for (a.slot0 = 0; a.slot0 < slots; a.slot0 += piece) {
        const long now = slots - a.slot0 < piece ? slots - a.slot0 : piece;
        hipLaunchKernelGGL((k_kv_attend_few<DP, FP8>), dim3((unsigned)(now * splits * kv->kv_heads)), dim3(256), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
        if (splits > 1) {
            hipLaunchKernelGGL(k_kv_attend_join<DP>, dim3((unsigned)(now * kv->kv_heads)), dim3(256), 0, kv->stream, a);
            KV_TRY(kv, hipGetLastError());
        }
    }
    return SISO_OK;
}

extern "C" int siso_kv_attend(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *q, long q_token, long q_head, int heads,
                              float scale, int window, void *out, float *lse) {
    if (!kv) return SISO_EINVAL;
    if (layer < 0) return kv_fail(kv, SISO_EINVAL, "siso_kv_attend: layer %d", layer);
    KvAttend a;
    const int rc = kv_batch(kv, "siso_kv_attend", layer, batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (heads < 1 || heads % kv->kv_heads != 0 || heads / kv->kv_heads > 128)
        return kv_fail(kv, SISO_EINVAL, "siso_kv_attend: %d heads over %d kv heads", heads, kv->kv_heads);
    if (!(fabsf(scale) <= 3.0e38f) || window < 0) return kv_fail(kv, SISO_EINVAL, "siso_kv_attend: scale %g, window %d", (double)scale, window);
    if (a.batch.n == 0 || a.batch.rows == 0) return SISO_OK;
    if (!q || !out || ((uintptr_t)q & 1) || ((uintptr_t)out & 15) || ((uintptr_t)lse & 3))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_attend: queries and outputs must be there, outputs 16-byte aligned");
    a.pool = kv_pool(kv, layer);
    a.q = (const bf16_t *)q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.vec = ((uintptr_t)q & 15) == 0 && q_token % 8 == 0 && q_head % 8 == 0;
    a.group = heads / kv->kv_heads;
    a.scale = scale * 1.44269504089f;
    a.window = window;
    a.out = (bf16_t *)out;
    a.lse = lse;
    a.parts = kv->parts;
    const long max_length = batch->max_length > 0 && batch->max_length < a.batch.most ? batch->max_length : a.batch.most;
    switch (kv->dp / 64 + (kv->dtype == SISO_FP8 ? 4 : 0)) {
        case 1: return attend<64, false>(kv, a, max_length);
        case 2: return attend<128, false>(kv, a, max_length);
        case 3: return attend<192, false>(kv, a, max_length);
        case 4: return attend<256, false>(kv, a, max_length);
        case 5: return attend<64, true>(kv, a, max_length);
        case 6: return attend<128, true>(kv, a, max_length);
        case 7: return attend<192, true>(kv, a, max_length);
        default: return attend<256, true>(kv, a, max_length);
    }
}
