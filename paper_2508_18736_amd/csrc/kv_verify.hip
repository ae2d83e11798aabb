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
    u64 *parts;         // [n][slices] sums of the weights, as their bits; greedy: [rows][slices] largest entry and its place, as keys
    unsigned *arrived;  // [n] slices of a sequence that are done; zeros between calls
    int lanes;          // greedy: workgroups that share a sequence's rows
    long item0;
};
#define KV_SLICES 256  // of a row, at most: one for each thread of the workgroup that joins them
// Workgroups.  Drawing: as many as are on the chip at once (64 rows of 128,001 with a draft's: 22.2 us; 2,048 come in two turns, 25.5 us; 512:
// 24.5).  Greedy as many, whatever the rows: 64 sequences of 1 to 5 rows of 50,000: 13.3 us, 2,048 16.8; 250 rows of 65,537 in 16 bits 15.4 and 16.3; of
// 5 to 9 rows of 130,000 52.3 and 52.9, in 16 bits 38.6 and 31.4: the largest batches would be served better by twice as many.
#define KV_FILL 1024
// Workgroups of a sequence, greedy: they count themselves at one address, one after the other (8 sequences of 1 to 9 rows of 128,000: 11.7 us; 128:
// 14.0, as many as there are slices and rows: 21.5).
#define KV_ARRIVE 64
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

// Numbers of a workgroup for the one that is done last with a sequence.  They pass the caches of the XCDs (see kv_attend.hip).  All that
// decides how many workgroups come is the same for all of them, whatever the batch's numbers are: the count is always reached.
__device__ __forceinline__ void kv_leave_part(u64 *to, u64 what) { __hip_atomic_store(to, what, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool kv_last(unsigned *arrived, unsigned count) {  // thread 0 has left all numbers; true in the workgroup that is last
    __shared__ int last;
    if (threadIdx.x == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // they are where all workgroups see them
        last = atomicAdd(arrived, 1u) == count - 1;
        if (last) *arrived = 0;  // (for the next call: nobody else comes)
    }
    __syncthreads();
    return last;
}
__device__ __forceinline__ u64 kv_part(const u64 *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

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

// Running sums over the 256 threads of a workgroup; `all`: the sum of all.
__device__ __forceinline__ double kv_running_sum(double v, double *all) {
    __shared__ double waves[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double x = __shfl_up(v, off);
        if (lane >= off) v += x;
    }
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    double before = 0.0;
    for (int i = 0; i < wave; ++i) before += waves[i];
    *all = ((waves[0] + waves[1]) + waves[2]) + waves[3];
    __syncthreads();
    return before + v;
}

// One slice of one sequence's row: the sum of its weights.  The workgroup that is done last with a sequence draws its token.
// Bound by latency more than by bytes: which row is read is known when the draft is judged, and the token when all sums are there.  64
// drafts with their probabilities, 128,001 entries, 66 MB, in 22 us, 2.9 TB/s; one draft of 32,000 entries in 6.7 us.
template <class T>
__global__ __launch_bounds__(256) void k_kv_draw(KvVerify a) {
    __shared__ double part[4], upto[KV_SLICES];
    __shared__ int found[4], has[4];
    const int b = (int)((a.item0 + blockIdx.x) / a.slices), slice = (int)((a.item0 + blockIdx.x) % a.slices), t = threadIdx.x;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0) {
        if (slice == 0 && t == 0) a.accepted[b] = -1;
        return;
    }
    const int accepted = kv_accepted<T>(a, s);
    KvWeights<T> weights = kv_weights<T>(a, s, accepted);
    double sum = 0.0;
    const int end = (slice + 1) * a.slice < a.vocab ? (slice + 1) * a.slice : a.vocab;
    for (int e = slice * a.slice + 8 * t; e < end; e += KV_SLICE_UNIT) {
        double w[8];
        weights.eight(e, a.vocab, w);
        sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
    sum = kv_wave_sum(sum);
    if ((t & 63) == 0) part[t >> 6] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    u64 *parts = a.parts + (long)b * a.slices;
    if (t == 0) kv_leave_part(parts + slice, (u64)__double_as_longlong(sum));
    if (!kv_last(a.arrived + b, a.slices)) return;

    const double mine = t < a.slices ? __longlong_as_double((long long)kv_part(parts + t)) : 0.0;
    double total;
    const double run = kv_running_sum(mine, &total);
    const double u = (double)fminf(fmaxf(a.u_sample[b], 0.f), 0.99999994f);
    int following;
    double ignored;
    if (total > 0.0) {
        // the first slice with weight in which the bar is passed, or the last one with weight
        const double bar = u * total;
        if (t < KV_SLICES) upto[t] = run;
        const u64 over = __ballot(mine > 0.0 && run > bar), some = __ballot(mine > 0.0);
        if ((t & 63) == 0) {
            found[t >> 6] = over ? (t & ~63) + __ffsll((long long)over) - 1 : -1;
            has[t >> 6] = some ? (t & ~63) + 63 - __clzll((long long)some) : -1;
        }
        __syncthreads();
        int at = -1;
        for (int i = 3; i >= 0; --i) at = found[i] >= 0 ? found[i] : at;
        if (at < 0)
            for (int i = 0; i < 4; ++i) at = has[i] >= 0 ? has[i] : at;
        const int begin = at * a.slice;
        following = kv_find(weights, begin, begin + a.slice < a.vocab ? begin + a.slice : a.vocab, a.vocab, at > 0 ? upto[at - 1] : 0.0, bar, &ignored);
    } else {  // the target's own probabilities, if there are any
        weights.q = nullptr;
        weights.not_this = -1;
        kv_find(weights, 0, a.vocab, a.vocab, 0.0, 0.0, &total);
        following = kv_find(weights, 0, a.vocab, a.vocab, 0.0, u * total, &ignored);
    }
    kv_write_tokens(a, s, accepted, following);
}

// Greedy: one slice of every a.lanes-th row of a sequence, the largest entries as keys that order equal ones by their place, four rows
// at a time.  The workgroup that is done last with a sequence compares the draft with them.
// 250 rows of 48 sequences, 65,537 entries of 16 bits, 33 MB, in 15.4 us, 2.1 TB/s: one pass, and the latency of launch and join.
template <class T>
__global__ __launch_bounds__(256) void k_kv_follow(KvVerify a) {
    constexpr int ROWS = 4;
    __shared__ u64 part[ROWS][4];
    const long item = a.item0 + blockIdx.x;
    const int slice = (int)(item % a.slices), lead = (int)(item / a.slices % a.lanes), b = (int)(item / a.slices / a.lanes), t = threadIdx.x;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0) {
        if (slice == 0 && lead == 0 && t == 0) a.accepted[b] = -1;
        return;
    }
    if (lead >= s.rows) return;
    const int end = (slice + 1) * a.slice < a.vocab ? (slice + 1) * a.slice : a.vocab;
    for (int i0 = lead; i0 < s.rows; i0 += ROWS * a.lanes) {
        float top[ROWS];
        int at[ROWS];
        const T *x[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            top[r] = -INFINITY;
            at[r] = -1;
            x[r] = (const T *)a.target + (long)(s.first + (i0 + r * a.lanes < s.rows ? i0 + r * a.lanes : i0)) * a.target_stride;
        }
        for (int e = slice * a.slice + 8 * t; e < end; e += KV_SLICE_UNIT) {
            float v[ROWS][8];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r > 0 && i0 + r * a.lanes >= s.rows) break;
                if (e + 8 <= a.vocab) kv_entries8(x[r] + e, v[r]);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[r][i] = e + i < a.vocab ? widen(x[r][e + i]) : __uint_as_float(0x7FC00000u);
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r > 0 && i0 + r * a.lanes >= s.rows) break;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (v[r][i] > top[r] || (at[r] < 0 && v[r][i] == top[r])) {
                        top[r] = v[r][i];
                        at[r] = e + i;
                    }
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const u64 key = wave_max(at[r] < 0 ? (u64)0 : pack_key(top[r] + 0.f, (unsigned)at[r]));  // (+ 0: the two zeros are equal)
            if ((t & 63) == 0) part[r][t >> 6] = key;
        }
        __syncthreads();
        if (t == 0)
            for (int r = 0; r < ROWS && i0 + r * a.lanes < s.rows; ++r) {
                u64 key = part[r][0];
                for (int i = 1; i < 4; ++i) key = part[r][i] > key ? part[r][i] : key;
                kv_leave_part(a.parts + (long)(s.first + i0 + r * a.lanes) * a.slices + slice, key);
            }
        __syncthreads();
    }
    if (!kv_last(a.arrived + b, (unsigned)(s.rows < a.lanes ? s.rows : a.lanes) * a.slices)) return;

    __shared__ u64 largest[64];
    int accepted = 0, following = -1;
    for (int i0 = 0; i0 < s.rows; i0 += 64) {
        // all parts of 64 rows, side by side in memory, a thread for each
        const int here = s.rows - i0 < 64 ? s.rows - i0 : 64, parts = here * a.slices;
        const u64 *of_rows = a.parts + (long)(s.first + i0) * a.slices;
        if (t < 64) largest[t] = 0;
        __syncthreads();
        for (int j0 = t; j0 < parts; j0 += 4 * 256) {
            u64 k[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) k[c] = kv_part(of_rows + (j0 + 256 * c < parts ? j0 + 256 * c : j0));
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (j0 + 256 * c < parts) atomicMax((unsigned long long *)&largest[(j0 + 256 * c) / a.slices], (unsigned long long)k[c]);
        }
        __syncthreads();
        const int i = i0 + (t & 63);  // (every wave by itself)
        int best = -1;
        bool good = false;
        if (i < s.rows) {
            const u64 most = largest[t & 63];
            if (most != 0) best = (int)(0xFFFFFFFFu - (unsigned)most);
            good = i < s.rows - 1 && best >= 0 && best == a.tokens[s.first + i + 1];
        }
        const u64 refused = ~__ballot(good);
        const int stop = refused ? __ffsll((long long)refused) - 1 : 64;
        accepted = i0 + stop;
        following = __shfl(best, stop & 63);
        if (stop < 64) break;  // (the last row is never `good`: this ends at the latest there; the same in every wave)
        __syncthreads();
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
    a.parts = (u64 *)kv->parts;
    a.arrived = kv->arrived;
    a.item0 = 0;
    // as many slices as fill the chip, of one unit at least (greedy: a part of each for each row; the workspace has room for one of 2^24)
    const long units = (vocab + KV_SLICE_UNIT - 1) / KV_SLICE_UNIT, rows = a.batch.rows > 0 ? a.batch.rows : 1;
    const long max_new = batch->max_new > 0 && batch->max_new < rows ? batch->max_new : rows;
    long lanes = 1, slices;
    if (u_accept) slices = KV_FILL / a.batch.n;
    else {  // four rows keep a workgroup busy
        lanes = KV_FILL / a.batch.n < (max_new + 3) / 4 ? KV_FILL / a.batch.n : (max_new + 3) / 4;
        lanes = lanes < 1 ? 1 : lanes;
        slices = KV_FILL / (a.batch.n * lanes);
        slices = slices * lanes > KV_ARRIVE ? KV_ARRIVE / lanes : slices;
        slices = slices * rows > (long)(SISO_KV_PARTS / 2) ? (long)(SISO_KV_PARTS / 2) / rows : slices;
    }
    slices = slices > KV_SLICES ? KV_SLICES : slices;
    slices = slices < 1 ? 1 : slices > units ? units : slices;
    a.slice = (int)((units + slices - 1) / slices * KV_SLICE_UNIT);
    a.slices = (vocab + a.slice - 1) / a.slice;
    a.lanes = (int)lanes;
    const long all = (long)a.batch.n * a.slices * a.lanes, piece = 1L << 23;
    for (; a.item0 < all; a.item0 += piece) {  // (a launch has fewer than 2^32 threads)
        const dim3 grid((unsigned)(all - a.item0 < piece ? all - a.item0 : piece));
        if (u_accept && type == SISO_F32) hipLaunchKernelGGL(k_kv_draw<float>, grid, dim3(256), 0, kv->stream, a);
        else if (u_accept) hipLaunchKernelGGL(k_kv_draw<bf16_t>, grid, dim3(256), 0, kv->stream, a);
        else if (type == SISO_F32) hipLaunchKernelGGL(k_kv_follow<float>, grid, dim3(256), 0, kv->stream, a);
        else hipLaunchKernelGGL(k_kv_follow<bf16_t>, grid, dim3(256), 0, kv->stream, a);
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}
