// Attention weights of cached positions, added up (siso_kv_weigh).  Layout of the pages: kv_internal.h.
#include <math.h>

#include "kv_internal.h"

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

struct KvWeigh {
    KvPool pool;
    KvBatch batch;
    const bf16_t *q;
    long q_token, q_head;
    int vec;
    int heads, group;
    float scale;      // its size times log2(e): the weights are powers of two
    unsigned negate;  // a scale below zero: the queries' signs are turned
    int window;
    const float *lse;
    const int *fresh, *newest;
    float decay;
    float *mass;
    int *born;
    int blocks;  // of KV_WEIGH positions, at most
    long item0;
};
#define KV_WEIGH 128  // positions of a workgroup: 32 of each wave

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

// A wave has 32 positions' keys in registers and goes over all rows of work (row = token * group + head in the group) that see one of them, 32 at a
// time: S = Q K^T, in which a lane has one position and 16 rows, so that the sum over rows is one of its own numbers.
template <int DP, bool FP8>
__global__ __launch_bounds__(256) void k_kv_weigh(KvWeigh a) {
    constexpr int ES = FP8 ? 1 : 2;
    constexpr int NF = FP8 ? DP / 32 : DP / 16;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    const long item = a.item0 + blockIdx.x;
    const int head = (int)(item % a.pool.kv_heads), block = (int)(item / a.pool.kv_heads % a.blocks);
    const KvSequence s = kv_sequence(a.batch, (int)(item / a.pool.kv_heads / a.blocks));
    if (s.rows == 0) return;
    for (int at = block * KV_WEIGH + 32 * w; at < s.length; at += a.blocks * KV_WEIGH) {  // (max_length may say less than there is)
        const int pos = at + n;  // this lane's
        int page[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) page[i] = kv_page_entry(a.pool, a.batch, s.b, at + 16 * i < s.length ? at + 16 * i : at);
        const int mine = page[n >> 4];
        const bool held = kv_is_page(a.pool, mine);
        if (lane == 0 || lane == 16)
            if (!held && head == 0 && pos < s.length) atomicAdd(a.pool.bad, 1ull);
        const int pg = held ? mine : 0;
        u32x4_t kf[NF];
        const char *from = a.pool.k + kv_block_at(a.pool, pg, head, at + 16 * (n >> 4)) * ES + h * 256 + (lane & 15) * 16;
#pragma unroll
        for (int i = 0; i < NF; ++i) kf[i] = *(const u32x4_t *)(from + i * 512);
        const size_t spot = kv_scale_at(a.pool, pg, head, pos);
        float scale = a.scale;
        if constexpr (FP8) scale *= a.pool.ks[spot];
        // rows that see some of the 32: from the first at `at` on, up to the last that the window lets see
        int first = at - s.start, last = s.rows - 1;
        first = first > 0 ? first : 0;
        if (a.window > 0) {
            const long end = (long)at + 31 + a.window - 1 - s.start;
            last = end < last ? (int)end : last;
        }
        const int work_end = (last + 1) * a.group;
        float sum = 0.f;
        for (int row0 = first * a.group; row0 < work_end; row0 += 32) {
            const int row = row0 + n, token = row < work_end ? row / a.group : first, qh = head * a.group + (row < work_end ? row % a.group : 0);
            const bf16_t *q = a.q + (long)(s.first + token) * a.q_token + (long)qh * a.q_head;
            f32x16_t acc = f32x16_t{};
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const int e = FP8 ? 16 * (2 * (i >> 1) + h) + 8 * (i & 1) : 16 * i + 8 * h;
                u32x4_t x = u32x4_t{0, 0, 0, 0};
                if (e < a.pool.dim) {
                    if (a.vec) x = *(const u32x4_t *)(q + e);
                    else
#pragma unroll
                        for (int c = 0; c < 4; ++c) x[c] = (unsigned)q[e + 2 * c] | ((unsigned)q[e + 2 * c + 1] << 16);
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[c] ^= a.negate;
                }
                bf16x8_t kx;
                if constexpr (FP8) kx = i & 1 ? kv_codes_bf16(kf[i >> 1][2], kf[i >> 1][3]) : kv_codes_bf16(kf[i >> 1][0], kf[i >> 1][1]);
                else kx = kv_as_bf16(kf[i]);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kv_as_bf16(x), kx, acc, 0, 0, 0);
            }
            float part = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {  // register r: row 8 (r / 4) + 4 h + r % 4 of this lane's position
                const int rr = row0 + 8 * (r >> 2) + 4 * h + (r & 3);
                if (rr < work_end) {
                    const int p = s.start + rr / a.group;
                    const float lse = a.lse[(size_t)(s.first + rr / a.group) * a.heads + head * a.group + rr % a.group];
                    if (pos <= p && (a.window == 0 || pos > p - a.window) && lse != -INFINITY)
                        part += __builtin_amdgcn_exp2f(__fmaf_rn(acc[r], scale, -lse * 1.44269504089f));
                }
            }
            sum += part;
        }
        const LanePair<float> both = lane_pair<32>(sum);
        sum = both.a + both.b;
        if (h == 0 && pos < s.length && held) {
            const int fresh = a.fresh ? a.fresh[s.b] : s.start;
            const float had = pos < fresh ? a.decay * a.mass[spot] : 0.f;
            a.mass[spot] = had + sum;
            if (a.born && pos >= fresh) a.born[spot] = (a.newest ? a.newest[s.b] : s.length - 1) - (s.length - 1 - pos);
        }
    }
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
    a.pool = kv_pool(kv, layer);
    a.q = (const bf16_t *)q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.vec = ((uintptr_t)q & 15) == 0 && q_token % 8 == 0 && q_head % 8 == 0;
    a.heads = heads;
    a.group = heads / kv->kv_heads;
    a.scale = fminf(fmaxf(fabsf(scale) * 1.44269504089f, 1.17549435e-38f), 3.40282347e38f);  // (as siso_kv_attend takes it)
    a.negate = scale < 0.f ? 0x80008000u : 0u;
    a.window = window < a.batch.most ? window : 0;
    a.lse = lse;
    a.fresh = fresh;
    a.newest = newest;
    a.decay = decay;
    a.mass = mass + (size_t)layer * kv->layer_scales;
    a.born = born ? born + (size_t)layer * kv->layer_scales : nullptr;
    const long max_length = batch->max_length > 0 && batch->max_length < a.batch.most ? batch->max_length : a.batch.most;
    a.blocks = (int)((max_length + KV_WEIGH - 1) / KV_WEIGH);
    const long items = (long)a.batch.n * kv->kv_heads * a.blocks, piece = 1L << 23;
    auto go = [&](auto kernel) {
        for (a.item0 = 0; a.item0 < items; a.item0 += piece)
            hipLaunchKernelGGL(kernel, dim3((unsigned)(items - a.item0 < piece ? items - a.item0 : piece)), dim3(256), 0, kv->stream, a);
    };
    switch (kv->dp / 64 + (kv->dtype == SISO_FP8 ? 4 : 0)) {
        case 1: go(k_kv_weigh<64, false>); break;
        case 2: go(k_kv_weigh<128, false>); break;
        case 3: go(k_kv_weigh<192, false>); break;
        case 4: go(k_kv_weigh<256, false>); break;
        case 5: go(k_kv_weigh<64, true>); break;
        case 6: go(k_kv_weigh<128, true>); break;
        case 7: go(k_kv_weigh<192, true>); break;
        default: go(k_kv_weigh<256, true>); break;
    }
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}
