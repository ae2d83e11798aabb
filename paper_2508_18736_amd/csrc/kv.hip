// The paged key/value cache: its handle, writing (quantising) and reading back.  Layout: kv_internal.h.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>
#include <new>
#include <type_traits>

#include "kv_internal.h"

int kv_fail(siso_kv *kv, int code, const char *fmt, ...) {
    if (kv) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(kv->err, sizeof(kv->err), fmt, ap);
        va_end(ap);
    }
    return code;
}

int kv_check_hip(siso_kv *kv, hipError_t e, const char *what) {
    if (e == hipSuccess) return SISO_OK;
    return kv_fail(kv, SISO_EHIP, "%s: %s", what, hipGetErrorString(e));
}

KvPool kv_pool(const siso_kv *kv, int layer) {
    KvPool p;
    p.k = kv->k + (size_t)layer * kv->layer_bytes;
    p.v = kv->v + (size_t)layer * kv->layer_bytes;
    p.ks = kv->ks ? kv->ks + (size_t)layer * kv->layer_scales : nullptr;
    p.vs = kv->vs ? kv->vs + (size_t)layer * kv->layer_scales : nullptr;
    p.bad = kv->counters;
    p.pages = (int)kv->pages;
    p.kv_heads = kv->kv_heads;
    p.shift = __builtin_ctz(kv->page_tokens);
    p.dim = kv->dim;
    p.dp = kv->dp;
    return p;
}

int kv_batch(siso_kv *kv, const char *call, int layer, const siso_kv_batch *batch, KvBatch *out) {
    if (!batch) return kv_fail(kv, SISO_EINVAL, "%s: no batch", call);
    const siso_kv_batch &b = *batch;
    if (b.n < 0 || b.n > 65535 || b.rows < 0 || b.rows > (1L << 24))
        return kv_fail(kv, SISO_EINVAL, "%s: %ld sequences, %ld rows", call, b.n, b.rows);
    if (b.max_new < 0 || b.max_length < 0) return kv_fail(kv, SISO_EINVAL, "%s: max_new %ld, max_length %ld", call, b.max_new, b.max_length);
    if (b.n > 0 && !b.first) return kv_fail(kv, SISO_EINVAL, "%s: no first rows", call);
    memset(out, 0, sizeof(*out));
    if (layer >= 0) {
        if (layer >= kv->layers) return kv_fail(kv, SISO_EINVAL, "%s: layer %d of %d", call, layer, kv->layers);
        if (b.n > 0 && (!b.length || !b.pages)) return kv_fail(kv, SISO_EINVAL, "%s: no lengths or no pages", call);
        if (b.width < 0 || b.width > SISO_KV_MOST / kv->page_tokens) return kv_fail(kv, SISO_EINVAL, "%s: %ld pages of a sequence", call, b.width);
        out->length = b.length;
        out->pages = b.pages;
        out->width = b.width;
        out->most = (int)(b.width * kv->page_tokens);
    }
    out->first = b.first;
    out->n = (int)b.n;
    out->rows = (int)b.rows;
    out->single = b.max_new == 1 && b.rows == b.n ? 1 : 0;
    return SISO_OK;
}

extern "C" int siso_kv_create(int layers, int kv_heads, int head_dim, int page_tokens, long pages, int dtype, siso_kv **out) {
    if (!out) return SISO_EINVAL;
    *out = nullptr;
    if (layers < 1 || kv_heads < 1 || kv_heads > 1024 || head_dim < 8 || head_dim > 256 || head_dim % 8 != 0 || page_tokens < 16 ||
        page_tokens > 1024 || (page_tokens & (page_tokens - 1)) != 0 || pages < 1 || pages > 2147483647L ||
        (dtype != SISO_BF16 && dtype != SISO_FP8))
        return SISO_EINVAL;
    siso_kv *kv = new (std::nothrow) siso_kv();
    if (!kv) return SISO_ENOMEM;
    memset(kv, 0, sizeof(*kv));
    kv->layers = layers;
    kv->kv_heads = kv_heads;
    kv->dim = head_dim;
    kv->dp = (head_dim + 63) / 64 * 64;
    kv->page_tokens = page_tokens;
    kv->pages = pages;
    kv->dtype = dtype;
    // (sizes of 2^63 and more would wrap: no GPU has as much)
    const double all = (double)layers * pages * page_tokens * kv_heads * kv->dp * 2;
    bool ok = all < 1e15;
    if (ok) {
        const size_t vectors = (size_t)pages * page_tokens * kv_heads;
        kv->layer_bytes = vectors * kv->dp * (dtype == SISO_FP8 ? 1 : 2);
        kv->layer_scales = vectors;
        const size_t bytes = kv->layer_bytes * layers, scales = vectors * layers * sizeof(float);
        ok = hipMalloc((void **)&kv->k, bytes) == hipSuccess && hipMalloc((void **)&kv->v, bytes) == hipSuccess;
        ok = ok && hipMemset(kv->k, 0, bytes) == hipSuccess && hipMemset(kv->v, 0, bytes) == hipSuccess;
        if (dtype == SISO_FP8) {
            ok = ok && hipMalloc((void **)&kv->ks, scales) == hipSuccess && hipMalloc((void **)&kv->vs, scales) == hipSuccess;
            ok = ok && hipMemset(kv->ks, 0, scales) == hipSuccess && hipMemset(kv->vs, 0, scales) == hipSuccess;
        }
        const size_t counts = 32 * sizeof(u64) + SISO_KV_JOINS * sizeof(unsigned) + SISO_KV_PLAN_BYTES;
        ok = ok && hipMalloc((void **)&kv->counters, counts) == hipSuccess;
        ok = ok && hipMemset(kv->counters, 0, counts) == hipSuccess;
        kv->arrived = (unsigned *)(kv->counters + 32);
        kv->plan = kv->arrived + SISO_KV_JOINS;
        ok = ok && hipMalloc((void **)&kv->parts, SISO_KV_PARTS * sizeof(float)) == hipSuccess;
        ok = ok && hipDeviceSynchronize() == hipSuccess;
    }
    if (!ok) {
        (void)hipGetLastError();
        siso_kv_destroy(kv);
        return SISO_ENOMEM;
    }
    *out = kv;
    return SISO_OK;
}

extern "C" void siso_kv_destroy(siso_kv *kv) {
    if (!kv) return;
    (void)hipStreamSynchronize(kv->stream);
    if (kv->k) (void)hipFree(kv->k);
    if (kv->v) (void)hipFree(kv->v);
    if (kv->ks) (void)hipFree(kv->ks);
    if (kv->vs) (void)hipFree(kv->vs);
    if (kv->counters) (void)hipFree(kv->counters);
    if (kv->parts) (void)hipFree(kv->parts);
    delete kv;
}

extern "C" int siso_kv_set_stream(siso_kv *kv, void *hip_stream) {
    if (!kv) return SISO_EINVAL;
    kv->stream = (hipStream_t)hip_stream;
    return SISO_OK;
}

extern "C" const char *siso_kv_last_error(const siso_kv *kv) { return kv ? kv->err : "null handle"; }

extern "C" long siso_kv_bad_pages(siso_kv *kv) {
    if (!kv) return SISO_EINVAL;
    u64 bad = 0;
    KV_TRY(kv, hipMemcpyAsync(&bad, kv->counters, sizeof(u64), hipMemcpyDeviceToHost, kv->stream));
    KV_TRY(kv, hipStreamSynchronize(kv->stream));
    return (long)bad;
}

// ---------------------------------------------------------------------------- writing and reading
// One workgroup for a block of 16 positions of one kv head, 16 threads for each of its tokens.  Rows come in and go out whole
// (16 bytes a thread); a block's values change sides, [token][dimension] against [dimension][token], through LDS.  The
// sequence's positions start anywhere in their first block and end anywhere in the last: a block's other tokens stay.
struct KvBlock {
    KvSequence s;
    int at;    // position of the block's first token
    int page;  // what the table says of it
    // Is that a page?  Asked after what does not depend on it has been sent for.
    __device__ __forceinline__ bool held(const KvPool &pool) const {
        const bool is = kv_is_page(pool, page);
        if (!is && threadIdx.x == 0) atomicAdd(pool.bad, 1ull);
        return is;
    }
};

// Slots for siso_kv_write and siso_kv_read: m rows stand in at most m / 16 + 2 blocks.
#define KV_BLOCK_SHIFT 4
#define KV_BLOCK_EXTRA 2
static long kv_block_slots(const KvBatch &b) {
    return b.single ? b.n : kv_slots_before(b.rows, b.n, 1, KV_BLOCK_SHIFT, KV_BLOCK_EXTRA);
}

__device__ __forceinline__ bool kv_find_block(const KvPool &pool, const KvBatch &batch, long slot, KvBlock &k) {
    k.s = batch.single ? kv_sequence(batch, (int)slot) : kv_sequence_of(batch, slot, 1, KV_BLOCK_SHIFT, KV_BLOCK_EXTRA);
    const long j = batch.single ? 0 : slot - kv_slots_before(k.s.first, k.s.b, 1, KV_BLOCK_SHIFT, KV_BLOCK_EXTRA);
    const long at = (long)((k.s.start > 0 ? k.s.start : 0) >> 4) * SISO_KV_BLOCK + j * SISO_KV_BLOCK;
    if (j < 0 || at >= k.s.length || k.s.rows == 0) return false;
    k.at = (int)at;
    k.page = kv_page_entry(pool, batch, k.s.b, k.at);
    return true;
}

__device__ __forceinline__ u32x4_t kv_load8(const bf16_t *row, int vec) {
    if (vec) return *(const u32x4_t *)row;
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (unsigned)row[2 * i] | ((unsigned)row[2 * i + 1] << 16);
    return r;
}
__device__ __forceinline__ float kv_half_of(u32x4_t x, int i) {
    return __uint_as_float(i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16);
}

// Eight elements of a vector that 16 threads hold (each 8 of NC * 128) as codes; the vector's scale.
// Quotients are those of a correctly rounded division: y, 1 / scale rounded, is formed once for the vector, and two steps
// q += (x - q scale) y, whose remainder is exact, end in the number closest to x / scale (Markstein).  Scales for which 1 / scale or a
// remainder could leave the normal range take the division itself.
template <int NC>
__device__ __forceinline__ float kv_quantise(const u32x4_t (&x)[NC], uint2 (&codes)[NC]) {
    float amax = 0.f;
    bool finite = true;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fabsf(kv_half_of(x[c], i));
            finite = finite && a <= 3.4e38f;
            amax = fmaxf(amax, a);
        }
    if (!finite) amax = INFINITY;
    amax = wave_fold<8>(amax, [](float a, float b) __attribute__((always_inline)) { return fmaxf(a, b); });
    const bool bad = !(amax <= 3.4e38f);
    const float scale = amax / 448.0f;
    const bool none = bad || scale == 0.f, plain = !(scale > 1e-25f && scale < 1e25f);
    const float y = __fdiv_rn(1.0f, scale);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = kv_half_of(x[c], i);
            q[i] = v * y;
            q[i] = __fmaf_rn(__fmaf_rn(-q[i], scale, v), y, q[i]);
            q[i] = __fmaf_rn(__fmaf_rn(-q[i], scale, v), y, q[i]);
        }
        if (plain)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = none ? 0.f : __fdiv_rn(kv_half_of(x[c], i), scale);
        // (nearest, ties to even; at most 448 and the rounding of the scale, which is 448)
        int w0 = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), w1 = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
        w0 = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w0, true);
        w1 = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], w1, true);
        codes[c] = make_uint2((unsigned)w0, (unsigned)w1);
    }
    return bad ? __uint_as_float(0x7FC00000u) : scale;
}

// Four dimensions of eight tokens change sides: in[token] = four elements side by side, out[dimension] = eight tokens side by side, and back.
__device__ __forceinline__ void kv_turn(const unsigned (&in)[8], uint2 (&out)[4]) {  // of one byte
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const unsigned a = __builtin_amdgcn_perm(in[4 * half + 1], in[4 * half], 0x05010400u), b = __builtin_amdgcn_perm(in[4 * half + 1], in[4 * half], 0x07030602u);
        const unsigned c = __builtin_amdgcn_perm(in[4 * half + 3], in[4 * half + 2], 0x05010400u), d = __builtin_amdgcn_perm(in[4 * half + 3], in[4 * half + 2], 0x07030602u);
        const unsigned t[4] = {__builtin_amdgcn_perm(c, a, 0x05040100u), __builtin_amdgcn_perm(c, a, 0x07060302u), __builtin_amdgcn_perm(d, b, 0x05040100u),
                               __builtin_amdgcn_perm(d, b, 0x07060302u)};
#pragma unroll
        for (int i = 0; i < 4; ++i) (half ? out[i].y : out[i].x) = t[i];
    }
}
__device__ __forceinline__ void kv_turn_back(const uint2 (&in)[4], unsigned (&out)[8]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        unsigned x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = half ? in[i].y : in[i].x;
        const unsigned a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
        const unsigned c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
        out[4 * half] = __builtin_amdgcn_perm(c, a, 0x05040100u);
        out[4 * half + 1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
        out[4 * half + 2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
        out[4 * half + 3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
    }
}
__device__ __forceinline__ void kv_turn(const uint2 (&in)[8], u32x4_t (&out)[4]) {  // of two bytes
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // two tokens
        out[0][i] = __builtin_amdgcn_perm(in[2 * i + 1].x, in[2 * i].x, 0x05040100u);
        out[1][i] = __builtin_amdgcn_perm(in[2 * i + 1].x, in[2 * i].x, 0x07060302u);
        out[2][i] = __builtin_amdgcn_perm(in[2 * i + 1].y, in[2 * i].y, 0x05040100u);
        out[3][i] = __builtin_amdgcn_perm(in[2 * i + 1].y, in[2 * i].y, 0x07060302u);
    }
}
__device__ __forceinline__ void kv_turn_back(const u32x4_t (&in)[4], uint2 (&out)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[2 * i].x = __builtin_amdgcn_perm(in[1][i], in[0][i], 0x05040100u);
        out[2 * i + 1].x = __builtin_amdgcn_perm(in[1][i], in[0][i], 0x07060302u);
        out[2 * i].y = __builtin_amdgcn_perm(in[3][i], in[2][i], 0x05040100u);
        out[2 * i + 1].y = __builtin_amdgcn_perm(in[3][i], in[2][i], 0x07060302u);
    }
}
__device__ __forceinline__ int kv_token(int half, int s) { return (s & 3) + 4 * half + 8 * (s >> 2); }  // of a half's eight

// Bound by bytes where there are many rows: 21,692 rows of 8 heads of 128 into 8 bits, 135 MB, in 33 us, 4.1 TB/s.  Few rows (8: 5 us, an empty launch
// takes half of that) wait for sequence, page and row, one after the other: a block is 16 tokens so that there are many to wait at a time.
// NC: chunks of 8 elements per thread (dp <= 128: one, else two)
template <int NC, bool FP8>
__global__ __launch_bounds__(256) void k_kv_write(KvPool pool, KvBatch batch, const bf16_t *k, long k_token, long k_head, const bf16_t *v,
                                                  long v_token, long v_head, int vec, long slot0) {
    constexpr int DP = NC * 128;
    constexpr int ES = FP8 ? 1 : 2;
    __shared__ __attribute__((aligned(16))) char turn[SISO_KV_BLOCK * (DP + 8) * ES];
    const int head = blockIdx.x % pool.kv_heads;
    KvBlock blk;
    if (!kv_find_block(pool, batch, slot0 + blockIdx.x / pool.kv_heads, blk)) return;
    const int t = threadIdx.x, key = t >> 4, i = t & 15, dim = pool.dim, dp = pool.dp;
    const int row = blk.at + key - blk.s.start;  // (not below: the first block may begin before the first row)
    const bool in = row >= 0 && row < blk.s.rows;
    u32x4_t kx[NC], vx[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e = 8 * (i + 16 * c);
        const bool take = in && e < dim;
        const long r = blk.s.first + row;
        kx[c] = take ? kv_load8(k + r * k_token + head * k_head + e, vec & 1) : u32x4_t{0, 0, 0, 0};
        vx[c] = take ? kv_load8(v + r * v_token + head * v_head + e, vec & 2) : u32x4_t{0, 0, 0, 0};
    }
    if (!blk.held(pool)) return;
    char *kb = pool.k + kv_block_at(pool, blk.page, head, blk.at) * ES;
    char *vb = pool.v + kv_block_at(pool, blk.page, head, blk.at) * ES;
    if constexpr (FP8) {
        uint2 kc[NC], vc[NC];
        const float ksc = kv_quantise(kx, kc), vsc = kv_quantise(vx, vc);
        if (in && i == 0) {
            const size_t at = kv_scale_at(pool, blk.page, head, blk.at) + key;
            pool.ks[at] = ksc;
            pool.vs[at] = vsc;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e8 = i + 16 * c;
            if (in && e8 * 8 < dim) *(uint2 *)(kb + ((e8 >> 1) * 16 + key) * 16 + (e8 & 1) * 8) = kc[c];
            *(uint2 *)(turn + key * (DP + 8) + e8 * 8) = vc[c];
        }
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e8 = i + 16 * c;
            if (in && e8 * 8 < dim) *(u32x4_t *)(kb + (e8 * 16 + key) * 16) = kx[c];
            *(u32x4_t *)(turn + (key * (DP + 8) + e8 * 8) * 2) = vx[c];
        }
    }
    __syncthreads();
    // which tokens of the block are new
    const int lo = blk.s.start > blk.at ? blk.s.start - blk.at : 0, hi = blk.s.length - blk.at < 16 ? blk.s.length - blk.at : 16;
    for (int j = t; j < dp >> 1; j += 256) {  // a half's eight tokens, four dimensions
        const int h = j >= dp >> 2, d0 = 4 * (j - h * (dp >> 2));
        if (d0 >= dim) continue;
        if constexpr (FP8) {
            unsigned x[8];
            uint2 y[4];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = *(const unsigned *)(turn + kv_token(h, s) * (DP + 8) + d0);
            kv_turn(x, y);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                char *to = vb + kv_v8_at(dp, h, d0 + c);
                if (lo == 0 && hi == 16) *(uint2 *)to = y[c];
                else
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        if (kv_token(h, s) >= lo && kv_token(h, s) < hi) to[s] = (char)((s < 4 ? y[c].x : y[c].y) >> (8 * (s & 3)));
            }
        } else {
            uint2 x[8];
            u32x4_t y[4];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = *(const uint2 *)(turn + (kv_token(h, s) * (DP + 8) + d0) * 2);
            kv_turn(x, y);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                bf16_t *to = (bf16_t *)vb + (h * dp + d0 + c) * 8;
                if (lo == 0 && hi == 16) *(u32x4_t *)to = y[c];
                else
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        if (kv_token(h, s) >= lo && kv_token(h, s) < hi) to[s] = (bf16_t)(s & 1 ? y[c][s >> 1] >> 16 : y[c][s >> 1]);
            }
        }
    }
}

template <class O>
__device__ __forceinline__ void kv_store8(O *to, const float (&x)[8]) {
    if constexpr (sizeof(O) == 4) {
        *(float4 *)to = make_float4(x[0], x[1], x[2], x[3]);
        *(float4 *)(to + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        struct {
            __bf16 v[8];
        } w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = (__bf16)x[i];
        *(u32x4_t *)to = __builtin_bit_cast(u32x4_t, w);
    }
}
__device__ __forceinline__ void kv_decode8(uint2 codes, float scale, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)(i ? codes.y : codes.x), false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)(i ? codes.y : codes.x), true);
        x[4 * i] = a[0] * scale, x[4 * i + 1] = a[1] * scale, x[4 * i + 2] = b[0] * scale, x[4 * i + 3] = b[1] * scale;
    }
}

// The other way round; the same rows into 16 bits in 25 us, 5.4 TB/s.
template <int NC, bool FP8, class O>
__global__ __launch_bounds__(256) void k_kv_read(KvPool pool, KvBatch batch, O *out_k, O *out_v, long slot0) {
    constexpr int DP = NC * 128;
    constexpr int ES = FP8 ? 1 : 2;
    __shared__ __attribute__((aligned(16))) char turn[SISO_KV_BLOCK * (DP + 8) * ES];
    const int head = blockIdx.x % pool.kv_heads, dim = pool.dim, dp = pool.dp;
    const long slot = slot0 + blockIdx.x / pool.kv_heads;
    KvBlock blk;
    const bool some = kv_find_block(pool, batch, slot, blk);
    const int t = threadIdx.x, key = t >> 4, i = t & 15;
    // rows without a position: zeros, by the sequence's first slots, 16 to each (there are at least as many slots)
    if (blk.s.start < 0) {
        const long j = batch.single ? 0 : slot - kv_slots_before(blk.s.first, blk.s.b, 1, KV_BLOCK_SHIFT, KV_BLOCK_EXTRA);
        const long row = j * 16 + key;
        if (j >= 0 && row < blk.s.rows && row < -(long)blk.s.start)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int e = 8 * (i + 16 * c);
                const float zero[8] = {};
                const size_t at = ((size_t)(blk.s.first + row) * pool.kv_heads + head) * dim + e;
                if (e < dim) {
                    kv_store8(out_k + at, zero);
                    kv_store8(out_v + at, zero);
                }
            }
    }
    if (!some) return;
    const int row = blk.at + key - blk.s.start;
    const bool in = row >= 0 && row < blk.s.rows;
    const bool held = blk.held(pool);
    const int page = held ? blk.page : 0;
    using K = typename std::conditional<FP8, uint2, u32x4_t>::type;       // eight elements
    using Four = typename std::conditional<FP8, unsigned, uint2>::type;  // four
    const int vh = t >= dp >> 2, vd = 4 * (t - vh * (dp >> 2));             // the half and the four dimensions that this thread turns
    K kx[NC], vx[4];
    float ksc = 1.f, vsc = 1.f;
    const char *kb = pool.k + kv_block_at(pool, page, head, blk.at) * ES;
    const char *vb = pool.v + kv_block_at(pool, page, head, blk.at) * ES;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e8 = i + 16 * c;
        if (e8 * 8 < dp) kx[c] = *(const K *)(FP8 ? kb + ((e8 >> 1) * 16 + key) * 16 + (e8 & 1) * 8 : kb + (e8 * 16 + key) * 16);
    }
    if (t < dp >> 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) vx[c] = *(const K *)(FP8 ? vb + kv_v8_at(dp, vh, vd + c) : vb + (size_t)(vh * dp + vd + c) * 16);
    if constexpr (FP8) {
        const size_t at = kv_scale_at(pool, page, head, blk.at) + key;
        ksc = pool.ks[at];
        vsc = pool.vs[at];
    }
    if (t < dp >> 1) {
        Four x[8];
        kv_turn_back(vx, x);
#pragma unroll
        for (int s = 0; s < 8; ++s) *(Four *)(turn + (kv_token(vh, s) * (DP + 8) + vd) * ES) = x[s];
    }
    __syncthreads();
    if (!in) return;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e = 8 * (i + 16 * c);
        if (e >= dim) continue;
        float x[8], y[8];
        const K vv = *(const K *)(turn + (key * (DP + 8) + e) * ES);
        if constexpr (FP8) {
            kv_decode8(kx[c], ksc, x);
            kv_decode8(vv, vsc, y);
        } else {
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                x[s] = kv_half_of(kx[c], s);
                y[s] = kv_half_of(vv, s);
            }
        }
        if (!held)
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = y[s] = 0.f;
        const size_t at = ((size_t)(blk.s.first + row) * pool.kv_heads + head) * dim + e;
        kv_store8(out_k + at, x);
        kv_store8(out_v + at, y);
    }
}

// (a launch has fewer than 2^32 threads)
template <class F>
static void kv_in_pieces(const siso_kv *kv, const KvBatch &b, F launch) {
    const long slots = kv_block_slots(b), piece = (1L << 23) / kv->kv_heads;
    for (long slot0 = 0; slot0 < slots; slot0 += piece) {
        const long now = slots - slot0 < piece ? slots - slot0 : piece;
        launch(dim3((unsigned)(now * kv->kv_heads)), slot0);
    }
}

static bool aligned_rows(const void *at, long token, long head) { return ((uintptr_t)at & 15) == 0 && token % 8 == 0 && head % 8 == 0; }

extern "C" int siso_kv_write(siso_kv *kv, int layer, const siso_kv_batch *batch, const void *k, long k_token, long k_head, const void *v,
                             long v_token, long v_head) {
    if (!kv) return SISO_EINVAL;
    if (layer < 0) return kv_fail(kv, SISO_EINVAL, "siso_kv_write: layer %d", layer);
    KvBatch b;
    const int rc = kv_batch(kv, "siso_kv_write", layer, batch, &b);
    if (rc != SISO_OK) return rc;
    if (b.n == 0 || b.rows == 0) return SISO_OK;
    if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 1)) return kv_fail(kv, SISO_EINVAL, "siso_kv_write: keys or values are NULL or at an odd address");
    const KvPool pool = kv_pool(kv, layer);
    const int vec = (aligned_rows(k, k_token, k_head) ? 1 : 0) | (aligned_rows(v, v_token, v_head) ? 2 : 0);
    auto go = [&](auto kernel) {
        kv_in_pieces(kv, b, [&](dim3 grid, long slot0) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, kv->stream, pool, b, (const bf16_t *)k, k_token, k_head, (const bf16_t *)v, v_token, v_head, vec, slot0);
        });
    };
    if (kv->dtype == SISO_FP8) kv->dp <= 128 ? go(k_kv_write<1, true>) : go(k_kv_write<2, true>);
    else kv->dp <= 128 ? go(k_kv_write<1, false>) : go(k_kv_write<2, false>);
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}

extern "C" int siso_kv_read(siso_kv *kv, int layer, const siso_kv_batch *batch, int out_type, void *out_k, void *out_v) {
    if (!kv) return SISO_EINVAL;
    if (layer < 0) return kv_fail(kv, SISO_EINVAL, "siso_kv_read: layer %d", layer);
    KvBatch b;
    const int rc = kv_batch(kv, "siso_kv_read", layer, batch, &b);
    if (rc != SISO_OK) return rc;
    if (out_type != SISO_BF16 && out_type != SISO_F32) return kv_fail(kv, SISO_EINVAL, "siso_kv_read: output type %d", out_type);
    if (b.n == 0 || b.rows == 0) return SISO_OK;
    if (!out_k || !out_v || (((uintptr_t)out_k | (uintptr_t)out_v) & 15))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_read: outputs must be 16-byte aligned");
    const KvPool pool = kv_pool(kv, layer);
    auto go16 = [&](auto kernel) {
        kv_in_pieces(kv, b, [&](dim3 grid, long slot0) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, kv->stream, pool, b, (bf16_t *)out_k, (bf16_t *)out_v, slot0); });
    };
    auto go32 = [&](auto kernel) {
        kv_in_pieces(kv, b, [&](dim3 grid, long slot0) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, kv->stream, pool, b, (float *)out_k, (float *)out_v, slot0); });
    };
    const bool wide = kv->dp > 128;
    if (kv->dtype == SISO_FP8) {
        if (out_type == SISO_F32) wide ? go32(k_kv_read<2, true, float>) : go32(k_kv_read<1, true, float>);
        else wide ? go16(k_kv_read<2, true, bf16_t>) : go16(k_kv_read<1, true, bf16_t>);
    } else {
        if (out_type == SISO_F32) wide ? go32(k_kv_read<2, false, float>) : go32(k_kv_read<1, false, float>);
        else wide ? go16(k_kv_read<2, false, bf16_t>) : go16(k_kv_read<1, false, bf16_t>);
    }
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}
