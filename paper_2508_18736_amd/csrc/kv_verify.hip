// Verification of drafted tokens (siso_kv_verify).
#include "kv_internal.h"

struct KvVerify {
    KvBatch batch;
    const int *tokens;
    int vocab;
    const void *target, *draft;
    long target_stride, draft_stride;
    const float *u_accept, *u_sample;
    int *accepted, *out;
    int slices, slice;  // the vocabulary in slices of `slice` entries, a multiple of KV_SLICE_UNIT
    double *sums;       // [n][slices] sums of the weights
    u64 *best;          // greedy: [rows][slices] largest entry and its place, as keys
    long item0;
};
#define KV_SLICE_UNIT 2048  // 256 threads, eight entries each

// Eight entries from e on of a row that begins anywhere (a row of an odd vocabulary is aligned to its type only).
struct __attribute__((packed, aligned(4))) KvFour32 {
    u32x4_t v;
};
struct __attribute__((packed, aligned(2))) KvFour16 {
    u32x4_t v;
};
__device__ __forceinline__ void kv_entries8(const float *p, float (&x)[8]) {
    const u32x4_t a = ((const KvFour32 *)p)->v, b = ((const KvFour32 *)(p + 4))->v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = __uint_as_float(a[i]);
        x[4 + i] = __uint_as_float(b[i]);
    }
}
__device__ __forceinline__ void kv_entries8(const bf16_t *p, float (&x)[8]) {
    const u32x4_t a = ((const KvFour16 *)p)->v;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? a[i >> 1] & 0xFFFF0000u : a[i >> 1] << 16);
}

// How many of the sequence's drafted tokens are accepted from its own random numbers, the same in every lane of a wave.
template <class T>
__device__ __forceinline__ int kv_accepted(const KvVerify &a, const KvSequence &s) {
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < s.rows - 1; i0 += 64) {
        const int i = i0 + lane;
        bool good = false;
        if (i < s.rows - 1) {
            const int x = a.tokens[s.first + i + 1];
            if ((unsigned)x < (unsigned)a.vocab) {
                const double p = (double)widen(((const T *)a.target)[(long)(s.first + i) * a.target_stride + x]);
                const double q = a.draft ? (double)widen(((const T *)a.draft)[(long)(s.first + i) * a.draft_stride + x]) : 1.0;
                good = (double)a.u_accept[s.first + i] * q < p;  // (two numbers of 24 bits: the product is exact)
            }
        }
        const u64 refused = ~__ballot(good);
        const int at = i0 + (refused ? __ffsll((long long)refused) - 1 : 64);
        if (at >= s.rows - 1) return s.rows - 1;
        if (at < i0 + 64) return at;
    }
    return s.rows - 1;
}

// The weights that the following token is drawn with.
template <class T>
struct KvWeights {
    const T *p, *q;  // q: NULL, or what is subtracted
    int not_this;    // an entry that counts as zero, or -1
    __device__ __forceinline__ double of(float pv, float qv, int e) const {
        const double w = (double)pv - (double)qv;
        return w > 0.0 && e != not_this ? w : 0.0;
    }
    __device__ __forceinline__ void eight(int e, int vocab, double (&w)[8]) const {
        if (e + 8 <= vocab) {
            float x[8], y[8] = {};
            kv_entries8(p + e, x);
            if (q) kv_entries8(q + e, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = of(x[i], y[i], e + i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = e + i < vocab ? of(widen(p[e + i]), q ? widen(q[e + i]) : 0.f, e + i) : 0.0;
        }
    }
};
template <class T>
__device__ __forceinline__ KvWeights<T> kv_weights(const KvVerify &a, const KvSequence &s, int accepted) {
    const bool refused = accepted < s.rows - 1;
    KvWeights<T> w;
    w.p = (const T *)a.target + (long)(s.first + accepted) * a.target_stride;
    w.q = refused && a.draft ? (const T *)a.draft + (long)(s.first + accepted) * a.draft_stride : nullptr;
    w.not_this = refused && !a.draft ? a.tokens[s.first + accepted + 1] : -1;
    return w;
}

__device__ __forceinline__ double kv_wave_sum(double v) {
    return wave_fold(v, [](double a, double b) __attribute__((always_inline)) { return a + b; });
}

// One slice of one sequence's row: the sum of its weights.
template <class T>
__global__ __launch_bounds__(256) void k_kv_sums(KvVerify a) {
    __shared__ double part[4];
    const int b = (int)(blockIdx.x / a.slices), slice = blockIdx.x % a.slices;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0) return;
    const KvWeights<T> weights = kv_weights<T>(a, s, kv_accepted<T>(a, s));
    double sum = 0.0;
    const int end = (slice + 1) * a.slice < a.vocab ? (slice + 1) * a.slice : a.vocab;
    for (int e = slice * a.slice + 8 * threadIdx.x; e < end; e += KV_SLICE_UNIT) {
        double w[8];
        weights.eight(e, a.vocab, w);
        sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
    sum = kv_wave_sum(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(long)b * a.slices + slice] = (part[0] + part[1]) + (part[2] + part[3]);
}

// The first entry of [begin, end) at which the running sum, `before` behind the entries ahead, exceeds `bar`; the last entry with
// weight where rounding leaves none; -1 where nothing has weight.  All 256 threads.  total: the sum of all.
template <class T>
__device__ int kv_find(const KvWeights<T> &weights, int begin, int end, int vocab, double before, double bar, double *total) {
    __shared__ double sh_sum[4];
    __shared__ int sh_found[4], sh_last[4];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int found = 0x7FFFFFFF, last = -1;
    double run = before;
    for (int e0 = begin; e0 < end; e0 += KV_SLICE_UNIT) {
        const int e = e0 + 8 * t;
        double w[8], sum = 0.0;
        if (e < end) {
            weights.eight(e, vocab, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += w[i];
        }
        double upto = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double x = __shfl_up(upto, off);
            if (lane >= off) upto += x;
        }
        if (lane == 63) sh_sum[wave] = upto;
        __syncthreads();
        double at = run + (upto - sum);
        for (int i = 0; i < wave; ++i) at += sh_sum[i];
        run += (sh_sum[0] + sh_sum[1]) + (sh_sum[2] + sh_sum[3]);
        if (e < end)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                at += w[i];
                if (w[i] > 0.0) {
                    last = e + i;
                    if (at > bar && found == 0x7FFFFFFF) found = e + i;
                }
            }
        __syncthreads();
    }
    found = wave_fold(found, [](int a, int b) __attribute__((always_inline)) { return a < b ? a : b; });
    last = wave_fold(last, [](int a, int b) __attribute__((always_inline)) { return a > b ? a : b; });
    if (lane == 0) {
        sh_found[wave] = found;
        sh_last[wave] = last;
    }
    __syncthreads();
    for (int i = 0; i < 4; ++i) {
        found = sh_found[i] < found ? sh_found[i] : found;
        last = sh_last[i] > last ? sh_last[i] : last;
    }
    __syncthreads();
    *total = run;
    return found != 0x7FFFFFFF ? found : last;
}

__device__ __forceinline__ void kv_write_tokens(const KvVerify &a, const KvSequence &s, int accepted, int following) {
    for (int i = threadIdx.x; i < s.rows; i += blockDim.x)
        a.out[s.first + i] = i < accepted ? a.tokens[s.first + i + 1] : i == accepted ? following : -1;
    if (threadIdx.x == 0) a.accepted[s.b] = accepted;
}

template <class T>
__global__ __launch_bounds__(256) void k_kv_choose(KvVerify a) {
    const int b = blockIdx.x;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0) {
        if (threadIdx.x == 0) a.accepted[b] = -1;
        return;
    }
    const int accepted = kv_accepted<T>(a, s);
    KvWeights<T> weights = kv_weights<T>(a, s, accepted);
    const double *sums = a.sums + (long)b * a.slices;
    double total = 0.0;
    for (int i = 0; i < a.slices; ++i) total += sums[i];
    const double u = (double)fminf(fmaxf(a.u_sample[b], 0.f), 0.99999994f);
    int following;
    double ignored;
    if (total > 0.0) {
        const double bar = u * total;
        double before = 0.0;
        int slice = -1;
        for (int i = 0; i < a.slices; ++i) {  // the slice in which the bar is passed, or the last one with weight
            if (!(sums[i] > 0.0)) continue;
            if (slice >= 0) before += sums[slice];
            slice = i;
            if (before + sums[i] > bar) break;
        }
        const int begin = slice * a.slice;
        following = kv_find(weights, begin, begin + a.slice < a.vocab ? begin + a.slice : a.vocab, a.vocab, before, bar, &ignored);
    } else {  // the target's own probabilities, if there are any
        weights.q = nullptr;
        weights.not_this = -1;
        kv_find(weights, 0, a.vocab, a.vocab, 0.0, 0.0, &total);
        following = kv_find(weights, 0, a.vocab, a.vocab, 0.0, u * total, &ignored);
    }
    kv_write_tokens(a, s, accepted, following);
}

// Greedy: one slice of one row, its largest entry as a key that orders equal entries by their place.
template <class T>
__global__ __launch_bounds__(256) void k_kv_largest(KvVerify a) {
    __shared__ u64 part[4];
    const long item = a.item0 + blockIdx.x, row = item / a.slices;
    const int slice = (int)(item % a.slices);
    const T *x = (const T *)a.target + row * a.target_stride;
    const int end = (slice + 1) * a.slice < a.vocab ? (slice + 1) * a.slice : a.vocab;
    float top = -INFINITY;
    int at = -1;
    for (int e = slice * a.slice + 8 * threadIdx.x; e < end; e += KV_SLICE_UNIT) {
        float v[8];
        if (e + 8 <= a.vocab) kv_entries8(x + e, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = e + i < a.vocab ? widen(x[e + i]) : __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (v[i] > top || (at < 0 && v[i] == top)) {
                top = v[i];
                at = e + i;
            }
    }
    u64 key = at < 0 ? 0 : pack_key(top + 0.f, (unsigned)at);  // (+ 0: the two zeros are equal)
    key = wave_max(key);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = key;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 4; ++i) key = part[i] > key ? part[i] : key;
        a.best[row * a.slices + slice] = key;
    }
}

__global__ __launch_bounds__(64) void k_kv_follow_largest(KvVerify a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0) {
        if (lane == 0) a.accepted[b] = -1;
        return;
    }
    int accepted = 0, following = -1;
    for (int i0 = 0; i0 < s.rows; i0 += 64) {
        const int i = i0 + lane;
        int best = -1;
        bool good = false;
        if (i < s.rows) {
            u64 key = 0;
            for (int j = 0; j < a.slices; ++j) {
                const u64 k = a.best[(long)(s.first + i) * a.slices + j];
                key = k > key ? k : key;
            }
            if (key != 0) best = (int)(0xFFFFFFFFu - (unsigned)key);
            good = i < s.rows - 1 && best >= 0 && best == a.tokens[s.first + i + 1];
        }
        const u64 refused = ~__ballot(good);
        const int at = refused ? __ffsll((long long)refused) - 1 : 64;
        accepted = i0 + at;
        following = __shfl(best, at & 63);
        if (at < 64) break;  // (the last row is never `good`: this ends at the latest there)
    }
    kv_write_tokens(a, s, accepted, following);
}

extern "C" int siso_kv_verify(siso_kv *kv, const siso_kv_batch *batch, const int *tokens, int vocab, int type, const void *target,
                              long target_stride, const void *draft, long draft_stride, const float *u_accept, const float *u_sample,
                              int *out_accepted, int *out_tokens) {
    if (!kv) return SISO_EINVAL;
    KvVerify a;
    const int rc = kv_batch(kv, "siso_kv_verify", -1, batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (vocab < 1 || vocab > (1 << 24)) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify: vocabulary of %d", vocab);
    if (type != SISO_F32 && type != SISO_BF16) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify: probabilities of type %d", type);
    if ((u_accept == nullptr) != (u_sample == nullptr) || (!u_accept && draft))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_verify: both random numbers or none, and with none no draft probabilities");
    if (a.batch.n == 0) return SISO_OK;
    if (!out_accepted || (a.batch.rows > 0 && (!tokens || !target || !out_tokens)))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_verify: tokens, target or outputs are NULL");
    const uintptr_t odd = type == SISO_F32 ? 3 : 1;
    if (((uintptr_t)target & odd) || ((uintptr_t)draft & odd)) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify: probabilities are not aligned to their type");
    a.tokens = tokens;
    a.vocab = vocab;
    a.target = target;
    a.draft = draft;
    a.target_stride = target_stride;
    a.draft_stride = draft_stride;
    a.u_accept = u_accept;
    a.u_sample = u_sample;
    a.accepted = out_accepted;
    a.out = out_tokens;
    a.sums = (double *)kv->parts;
    a.best = (u64 *)kv->parts;
    a.item0 = 0;
    // as many slices as fill the chip (2,048 workgroups), of one unit at least; one key or sum each fits the workspace: at most 2,048 or the items
    const long items = u_accept ? a.batch.n : a.batch.rows > 0 ? a.batch.rows : 1;
    const long units = (vocab + KV_SLICE_UNIT - 1) / KV_SLICE_UNIT;
    long slices = 2048 / items;
    slices = slices < 1 ? 1 : slices > units ? units : slices;
    a.slice = (int)((units + slices - 1) / slices * KV_SLICE_UNIT);
    a.slices = (vocab + a.slice - 1) / a.slice;
    const long all = items * a.slices, piece = 1L << 23;
    if (u_accept) {
        const dim3 grid((unsigned)all);
        if (type == SISO_F32) {
            hipLaunchKernelGGL(k_kv_sums<float>, grid, dim3(256), 0, kv->stream, a);
            hipLaunchKernelGGL(k_kv_choose<float>, dim3((unsigned)a.batch.n), dim3(256), 0, kv->stream, a);
        } else {
            hipLaunchKernelGGL(k_kv_sums<bf16_t>, grid, dim3(256), 0, kv->stream, a);
            hipLaunchKernelGGL(k_kv_choose<bf16_t>, dim3((unsigned)a.batch.n), dim3(256), 0, kv->stream, a);
        }
    } else {
        for (a.item0 = 0; a.item0 < all && a.batch.rows > 0; a.item0 += piece) {
            const dim3 grid((unsigned)(all - a.item0 < piece ? all - a.item0 : piece));
            if (type == SISO_F32) hipLaunchKernelGGL(k_kv_largest<float>, grid, dim3(256), 0, kv->stream, a);
            else hipLaunchKernelGGL(k_kv_largest<bf16_t>, grid, dim3(256), 0, kv->stream, a);
            KV_TRY(kv, hipGetLastError());
        }
        hipLaunchKernelGGL(k_kv_follow_largest, dim3((unsigned)a.batch.n), dim3(64), 0, kv->stream, a);
    }
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}
