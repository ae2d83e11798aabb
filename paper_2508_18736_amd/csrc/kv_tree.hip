// Trees of drafted tokens: who is whose ancestor, which path stands, and where its keys and values go (siso_kv_tree,
// siso_kv_verify_tree, siso_kv_keep).  Their attention is in kv_attend.hip.
#include <type_traits>

#include "kv_entries.h"
#include "kv_internal.h"

#define KV_TREE_WORDS (SISO_KV_TREE / 32)

// The row that row i continues: 0 to i - 1, or -1.
__device__ __forceinline__ int kv_parent(const int *parent, const KvSequence &s, int i) {
    const int p = parent[s.first + i];
    return p >= 0 && p < i ? p : -1;
}

// ---------------------------------------------------------------------------- ancestors
// One workgroup a sequence, one thread a row.  A row knows the ancestors up to some row; with what that one knows it knows twice as many: eight
// turns for any tree, one for each doubling of the depth.  Bound by latency: 5 us are a launch and three loads that wait for each other.
__global__ __launch_bounds__(SISO_KV_TREE) void k_kv_tree(KvBatch batch, const int *parent, unsigned *mask, int *depth) {
    __shared__ unsigned known[SISO_KV_TREE][KV_TREE_WORDS + 1];  // (a word more: rows lie in other banks)
    __shared__ int up[SISO_KV_TREE];
    const KvSequence s = kv_sequence(batch, blockIdx.x);
    if (s.rows > SISO_KV_TREE || s.rows == 0) return;
    const int i = threadIdx.x;
    const bool in = i < s.rows;
    unsigned mine[KV_TREE_WORDS];
    int at = in ? kv_parent(parent, s, i) : -1;
#pragma unroll
    for (int k = 0; k < KV_TREE_WORDS; ++k) mine[k] = i >> 5 == k ? 1u << (i & 31) : 0u;
#pragma unroll
    for (int k = 0; k < KV_TREE_WORDS; ++k) known[i][k] = mine[k];
    up[i] = at;
    while (__syncthreads_or(at >= 0)) {
        if (at >= 0) {
#pragma unroll
            for (int k = 0; k < KV_TREE_WORDS; ++k) mine[k] |= known[at][k];
            at = up[at];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < KV_TREE_WORDS; ++k) known[i][k] = mine[k];
        up[i] = at;
    }
    if (!in) return;
    u32x4_t *to = (u32x4_t *)(mask + (size_t)(s.first + i) * KV_TREE_WORDS);
    to[0] = u32x4_t{mine[0], mine[1], mine[2], mine[3]};
    to[1] = u32x4_t{mine[4], mine[5], mine[6], mine[7]};
    int count = 0;
#pragma unroll
    for (int k = 0; k < KV_TREE_WORDS; ++k) count += __popc(mine[k]);
    if (depth) depth[s.first + i] = count - 1;
}

// ---------------------------------------------------------------------------- verification
struct KvSettle {
    KvBatch batch;
    const int *parent, *tokens;
    int vocab;
    const void *target;
    long target_stride;
    const float *u;
    int *accepted, *rows, *out;
    // greedy, all rows at once, `most` places for each sequence: [places][slices] keys, [places] tokens, [places + n] how many are there (zeros between calls)
    int most;
    u64 *parts;
    int *named;
    unsigned *arrived;
    int slices, slice;
};
#define KV_SETTLE 1024
// Up to so many bytes of them all rows are looked at at once (32 trees of 16 rows of 32,000 entries in 16 bits, 33 MB: 15.5 us a call, row by row 22.6; of 40
// rows, 82 MB: 28.1 and 25.5).
#define KV_SETTLE_ALL (48L << 20)
#define KV_SETTLE_PLACES 4096
static_assert(2 * KV_SETTLE_PLACES <= SISO_KV_JOINS, "a count for each place and sequence");
#define KV_SLICE_UNIT 2048  // entries: eight a thread of 256

__device__ __forceinline__ double kv_sum_up(double v, int lane) {  // running sums over a wave
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double x = __shfl_up(v, off);
        if (lane >= off) v += x;
    }
    return v;
}
__device__ __forceinline__ double kv_weight(float x) { return x > 0.f ? (double)x : 0.0; }
template <class T>
__device__ __forceinline__ void kv_eight(const T *row, int e, int vocab, float beyond, float (&x)[8]) {
    if (e + 8 <= vocab) kv_entries8(row + e, x);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e + i < vocab ? widen(row[e + i]) : beyond;
}

// The largest of the entries begin .. end - 1 of a row, the first of equal ones, as a key; 0 without any.  Of one wave.
template <class T>
__device__ __forceinline__ u64 kv_largest(const T *row, int begin, int end, int vocab, int step) {
    float top = -INFINITY;
    int at = -1;
#pragma unroll 2
    for (int e = begin; e < end; e += step) {
        float x[8];
        kv_eight(row, e, vocab, __uint_as_float(0x7FC00000u), x);
        const float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));  // (NaN only if all are)
        if (most > top || (at < 0 && most == top)) {
            top = most;
#pragma unroll
            for (int i = 7; i >= 0; --i) at = x[i] == most ? e + i : at;
        }
    }
    return wave_max(at < 0 ? (u64)0 : pack_key(top + 0.f, (unsigned)at));  // (+ 0: the two zeros are equal)
}
__device__ __forceinline__ u64 kv_most(const u64 (&keys)[4]) {
    const u64 a = keys[0] > keys[1] ? keys[0] : keys[1], b = keys[2] > keys[3] ? keys[2] : keys[3];
    return a > b ? a : b;
}
__device__ __forceinline__ int kv_key_entry(u64 key) { return key ? (int)(0xFFFFFFFFu - (unsigned)key) : -1; }

// The sum of the weights of every step'th eight entries from begin up to end, of one wave.
template <class T>
__device__ __forceinline__ double kv_sum(const T *row, int begin, int end, int vocab, int step) {
    double sum = 0.0;
#pragma unroll 4
    for (int e = begin; e < end; e += step) {
        float x[8];
        kv_eight(row, e, vocab, 0.f, x);
        sum += ((kv_weight(x[0]) + kv_weight(x[1])) + (kv_weight(x[2]) + kv_weight(x[3]))) + ((kv_weight(x[4]) + kv_weight(x[5])) + (kv_weight(x[6]) + kv_weight(x[7])));
    }
    return wave_fold(sum, [](double a, double b) __attribute__((always_inline)) { return a + b; });
}
// Of up to 64 stretches' sums, one a lane: the first one with weight in which u times the sum of all is passed, or (rounding) the last one with weight;
// -1 without any.  `before`: the sum ahead of it, `bar`: u times the sum.
__device__ __forceinline__ int kv_stretch(double mine, float u, double &before, double &bar) {
    const int lane = threadIdx.x & 63;
    const double upto = kv_sum_up(mine, lane), total = __shfl(upto, 63);
    bar = (double)fminf(fmaxf(u, 0.f), 0.99999994f) * total;
    if (!(total > 0.0)) return -1;
    const u64 over = __ballot(mine > 0.0 && upto > bar), some = __ballot(mine > 0.0);
    const int at = over ? __ffsll((long long)over) - 1 : 63 - __clzll((long long)some);
    before = at > 0 ? __shfl(upto, at - 1) : 0.0;
    return at;
}
// The first of the entries begin .. end - 1 at which the running sum, `before` behind what is ahead of them, exceeds `bar`; the last one with weight
// where rounding leaves none.  All NW waves; sums: NW numbers, found: 2 NW.
template <int NW, class T>
__device__ __forceinline__ int kv_search(const T *row, int begin, int end, int vocab, double before, double bar, double *sums, int *found) {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    int first = 0x7FFFFFFF, last = -1;
    for (int e0 = begin; e0 < end; e0 += 8 * 64 * NW) {
        const int e = e0 + 8 * t;
        float x[8];
        double here = 0.0;
        if (e < end) {
            kv_eight(row, e, vocab, 0.f, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) here += kv_weight(x[i]);
        }
        const double run = kv_sum_up(here, lane);
        if (lane == 63) sums[w] = run;
        __syncthreads();
        double so_far = before + (run - here);
        for (int i = 0; i < NW; ++i) {
            if (i < w) so_far += sums[i];
            before += sums[i];
        }
        if (e < end)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double weight = kv_weight(x[i]);
                so_far += weight;
                if (weight > 0.0) {
                    last = e + i;
                    if (so_far > bar && first == 0x7FFFFFFF) first = e + i;
                }
            }
        __syncthreads();
    }
    first = wave_fold(first, [](int a, int b) __attribute__((always_inline)) { return a < b ? a : b; });
    last = wave_fold(last, [](int a, int b) __attribute__((always_inline)) { return a > b ? a : b; });
    if (lane == 0) {
        found[w] = first;
        found[NW + w] = last;
    }
    __syncthreads();
    first = wave_fold(found[lane & (NW - 1)], [](int a, int b) __attribute__((always_inline)) { return a < b ? a : b; });
    last = wave_fold(found[NW + (lane & (NW - 1))], [](int a, int b) __attribute__((always_inline)) { return a > b ? a : b; });
    __syncthreads();
    return first != 0x7FFFFFFF ? first : last;
}

// The row that continues `row` with token x, the first of several, -1 without any; the same in every lane (and every wave finds the same).
__device__ __forceinline__ int kv_child(const int *parents, const int *tokens, int rows, int row, int x) {
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < rows && x >= 0; i0 += 64) {
        const u64 fits = __ballot(parents[i0 + lane] == row && tokens[i0 + lane] == x);
        if (fits) return i0 + __ffsll((long long)fits) - 1;
    }
    return -1;
}

// One workgroup a sequence: it goes from row to row and reads those alone.  Bound by what one compute unit takes in: rows of 128,001 entries of 32 bits
// at about 110 GB/s each (32 trees of 8 to 40 rows, walks of up to eight: 32 to 45 us, by the card).
template <class T, bool GREEDY>
__global__ __launch_bounds__(KV_SETTLE) void k_kv_settle(KvSettle a) {
    constexpr int NW = KV_SETTLE / 64;
    __shared__ int parents[SISO_KV_TREE], tokens[SISO_KV_TREE];
    __shared__ double sums[NW];
    __shared__ u64 keys[NW];
    __shared__ int found[2 * NW];
    const KvSequence s = kv_sequence(a.batch, blockIdx.x);
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    if (s.rows > SISO_KV_TREE) return;
    if (s.rows == 0) {
        if (t == 0) a.accepted[s.b] = -1;
        return;
    }
    if (t < SISO_KV_TREE) {
        parents[t] = t < s.rows ? kv_parent(a.parent, s, t) : -1;
        tokens[t] = t < s.rows ? a.tokens[s.first + t] : -1;
    }
    __syncthreads();
    int row = 0, count = 0;
    for (;;) {
        const T *p = (const T *)a.target + (long)(s.first + row) * a.target_stride;
        int x;
        if constexpr (GREEDY) {
            const u64 key = kv_largest(p, 8 * t, a.vocab, a.vocab, 8 * KV_SETTLE);
            if (lane == 0) keys[w] = key;
            __syncthreads();
            x = kv_key_entry(wave_max(keys[lane & (NW - 1)]));
            __syncthreads();
        } else {  // every wave sums a stretch; the one that the bar falls into is then searched by all
            const int stretch = ((a.vocab + NW * 512 - 1) / (NW * 512)) * 512, end = (w + 1) * stretch < a.vocab ? (w + 1) * stretch : a.vocab;
            const double sum = kv_sum(p, w * stretch + 8 * lane, end, a.vocab, 512);
            if (lane == 0) sums[w] = sum;
            __syncthreads();
            double before, bar;
            const int at = kv_stretch(lane < NW ? sums[lane & (NW - 1)] : 0.0, a.u[s.first + row], before, bar);
            __syncthreads();
            x = at < 0 ? -1 : kv_search<NW>(p, at * stretch, (at + 1) * stretch < a.vocab ? (at + 1) * stretch : a.vocab, a.vocab, before, bar, sums, found);
        }
        if (t == 0) {
            a.rows[s.first + count] = row;
            a.out[s.first + count] = x;
        }
        ++count;
        const int child = kv_child(parents, tokens, s.rows, row, x);
        if (child < 0) break;
        row = child;  // (it lies behind its parent: this ends)
    }
    for (int i = count + t; i < s.rows; i += KV_SETTLE) a.rows[s.first + i] = a.out[s.first + i] = -1;
    if (t == 0) a.accepted[s.b] = count - 1;
}

// Greedy, where the rows of all trees together are no more than a pass of the whole chip: all rows at once, a slice of one a workgroup; the one that is done last
// with a row names its token, the one that is done last with a sequence walks.  Numbers for them pass the caches of the XCDs.  (Drawn trees go row by row
// whatever they are: a row is searched once more when its sum is known, and all rows of the 32 trees above are 320 MB, 66 us.  Of one tree, or a few, all rows
// at once have not been measured.)
__device__ __forceinline__ bool kv_all_here(unsigned *arrived, unsigned count, int *last) {  // thread 0 has left its number
    if (threadIdx.x == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // it is where all workgroups see it
        *last = atomicAdd(arrived, 1u) == count - 1;
        if (*last) *arrived = 0;  // (for the next call: nobody else comes)
    }
    __syncthreads();
    const bool is = *last;
    __syncthreads();
    return is;
}
template <class T>
__global__ __launch_bounds__(256) void k_kv_settle_all(KvSettle a) {
    __shared__ int parents[SISO_KV_TREE], tokens[SISO_KV_TREE], named[SISO_KV_TREE];
    __shared__ u64 keys[4];
    __shared__ int last;
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    // (which rows there are goes by the sequence alone, whatever the other ones are: every count is reached)
    const int place = (int)(blockIdx.x / a.slices), slice = (int)(blockIdx.x % a.slices), b = place / a.most, in = place % a.most;
    const KvSequence s = kv_sequence(a.batch, b);
    if (s.rows == 0 && in == 0 && slice == 0 && t == 0) a.accepted[b] = -1;
    if (in >= s.rows || s.rows > a.most) return;
    const int row = s.first + in;
    const T *p = (const T *)a.target + (long)row * a.target_stride;
    const int begin = slice * a.slice, end = begin + a.slice < a.vocab ? begin + a.slice : a.vocab;
    u64 *const parts = a.parts + (long)place * a.slices;
    int *const all_named = a.named + b * a.most;
    const u64 key = kv_largest(p, begin + 8 * t, end, a.vocab, 8 * 256);
    if (lane == 0) keys[w] = key;
    __syncthreads();
    if (t == 0) __hip_atomic_store(parts + slice, kv_most(keys), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!kv_all_here(a.arrived + place, a.slices, &last)) return;
    const int x = kv_key_entry(wave_max(lane < a.slices ? __hip_atomic_load(parts + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : (u64)0));
    if (t == 0) __hip_atomic_store(all_named + in, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!kv_all_here(a.arrived + a.batch.n * a.most + b, s.rows, &last)) return;
    if (t < s.rows) {
        parents[t] = kv_parent(a.parent, s, t);
        tokens[t] = a.tokens[s.first + t];
        named[t] = __hip_atomic_load(all_named + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else parents[t] = -1, tokens[t] = -1;
    __syncthreads();
    int at = 0, count = 0;
    for (;;) {  // (every wave by itself)
        const int name = named[at];
        if (t == 0) {
            a.rows[s.first + count] = at;
            a.out[s.first + count] = name;
        }
        ++count;
        const int child = kv_child(parents, tokens, s.rows, at, name);
        if (child < 0) break;
        at = child;
    }
    if (t >= count && t < s.rows) a.rows[s.first + t] = a.out[s.first + t] = -1;
    if (t == 0) a.accepted[s.b] = count - 1;
}

// ---------------------------------------------------------------------------- the path that stands
// One workgroup of dp threads for a sequence, a layer and a kv head.  Its first wave brings 64 rows of the path to LDS, with the pages where they are and where
// they go.  Rows move to lower places, and in order: eight at a time are read before they are written, and what is read later lies behind all that has been
// written.  Bound by latency: loads of the rows' numbers, the path, the page and the row wait for each other (48 paths of 5 to 30 rows, 8 layers of 8 heads in
// 8 bits: 15.3 us; with pages read row by row and 256 threads 21).
#define KV_KEEP_ROWS 8
template <bool FP8>
__global__ __launch_bounds__(256) void k_kv_keep(KvPool pool, KvBatch batch, const int *path, long layer_bytes, long layer_scales, int layers, int b0) {
    constexpr int ES = FP8 ? 1 : 2;
    using E = typename std::conditional<FP8, unsigned char, bf16_t>::type;
    const int head = blockIdx.x % pool.kv_heads, layer = blockIdx.x / pool.kv_heads % layers, t = threadIdx.x;
    const KvSequence s = kv_sequence(batch, b0 + blockIdx.x / pool.kv_heads / layers);
    char *const pool_k = pool.k + layer * layer_bytes, *const pool_v = pool.v + layer * layer_bytes;
    float *const scales = FP8 ? (t & 8 ? pool.vs : pool.ks) + layer * layer_scales : nullptr;
    const int dp = pool.dp, chunks = dp * ES / 16;  // 16-byte chunks of a key
    const int *const table = batch.pages + (long)s.b * batch.width;
    __shared__ int from[64], from_page[64], to_page[64];  // positions; pages or -1
    __shared__ int count, moves;                          // rows of the path of these 64, and from which one on they move
    auto page_of = [&](int at) {
        const int page = at >= 0 && at < batch.most ? table[at >> pool.shift] : -1;
        if (kv_is_page(pool, page)) return page;
        if (head == 0 && at >= 0 && at < batch.most) atomicAdd(pool.bad, 1ull);
        return -1;
    };
    int before = -1;  // the path's last row
    for (int base = 0; base < s.rows; base += 64) {
        if (t < 64) {
            const int j = base + t, p = j < s.rows ? path[s.first + j] : -1, up = __shfl_up(p, 1), prior = t ? up : before;
            const u64 ends = ~__ballot(p >= j && p > prior && p < s.rows), moved = __ballot(p > j);
            const int good = ends ? __ffsll((long long)ends) - 1 : 64, first = moved ? __ffsll((long long)moved) - 1 : 64;
            before = __shfl(p, 63);
            if (t >= first && t < good) {
                from[t] = s.start + p;
                from_page[t] = page_of(s.start + p);
                to_page[t] = page_of(s.start + j);
            }
            if (t == 0) {
                count = good;
                moves = first;
            }
        }
        __syncthreads();
        const int all = count;
        for (int j0 = moves; j0 < all; j0 += KV_KEEP_ROWS) {
            u32x4_t k = u32x4_t{0, 0, 0, 0};
            E v[KV_KEEP_ROWS];
            float scale = 0.f;
            char *k_to = nullptr;
            int page_to[KV_KEEP_ROWS];
            float *scale_to = nullptr;
            // values: a thread for an element of all rows
#pragma unroll
            for (int r = 0; r < KV_KEEP_ROWS; ++r) {
                page_to[r] = -1;
                v[r] = 0;
                if (j0 + r >= all) continue;
                const int at = from[j0 + r], to = s.start + base + j0 + r, page = from_page[j0 + r], key = at & 15;
                page_to[r] = to_page[j0 + r];
                if (page >= 0) {
                    const E *block = (const E *)(pool_v + kv_block_at(pool, page, head, at) * ES);
                    v[r] = block[FP8 ? kv_v8_at(dp, kv_half(key), t) + kv_slot(key) : (kv_half(key) * dp + t) * 8 + kv_slot(key)];
                }
                // keys: a thread for a chunk of a row
                if (t / chunks == r) {
                    if (page >= 0) k = *(const u32x4_t *)(pool_k + kv_block_at(pool, page, head, at) * ES + ((t % chunks) * 16 + key) * 16);
                    if (page_to[r] >= 0) k_to = pool_k + kv_block_at(pool, page_to[r], head, to) * ES + ((t % chunks) * 16 + (to & 15)) * 16;
                }
                if (FP8 && (t & 7) == r && t < 16) {
                    if (page >= 0) scale = scales[kv_scale_at(pool, page, head, at)];
                    if (page_to[r] >= 0) scale_to = scales + kv_scale_at(pool, page_to[r], head, to);
                }
            }
            __syncthreads();
            if (k_to) *(u32x4_t *)k_to = k;
            if (FP8 && scale_to) *scale_to = scale;
#pragma unroll
            for (int r = 0; r < KV_KEEP_ROWS; ++r) {
                if (page_to[r] < 0) continue;
                const int to = s.start + base + j0 + r, key = to & 15;
                E *block = (E *)(pool_v + kv_block_at(pool, page_to[r], head, to) * ES);
                block[FP8 ? kv_v8_at(dp, kv_half(key), t) + kv_slot(key) : (kv_half(key) * dp + t) * 8 + kv_slot(key)] = v[r];
            }
            // (no wait: what the next turn reads nobody has written)
        }
        if (all < 64) return;
        __syncthreads();  // (the 64 rows' places are used again)
    }
}

// ---------------------------------------------------------------------------- calls
static int tree_batch(siso_kv *kv, const char *call, const siso_kv_batch *batch, KvBatch *b) {
    const int rc = kv_batch(kv, call, -1, batch, b);
    if (rc != SISO_OK) return rc;
    if (kv_max_new(batch) > SISO_KV_TREE) return kv_fail(kv, SISO_EINVAL, "%s: trees of %ld rows", call, kv_max_new(batch));
    return SISO_OK;
}

extern "C" int siso_kv_tree(siso_kv *kv, const siso_kv_batch *batch, const int *parent, unsigned *out_mask, int *out_depth) {
    if (!kv) return SISO_EINVAL;
    KvBatch b;
    const int rc = tree_batch(kv, "siso_kv_tree", batch, &b);
    if (rc != SISO_OK) return rc;
    if (b.n == 0 || b.rows == 0) return SISO_OK;
    if (!parent || !out_mask || ((uintptr_t)out_mask & 15)) return kv_fail(kv, SISO_EINVAL, "siso_kv_tree: parents and masks must be there, masks 16-byte aligned");
    hipLaunchKernelGGL(k_kv_tree, dim3(b.n), dim3(SISO_KV_TREE), 0, kv->stream, b, parent, out_mask, out_depth);
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}

extern "C" int siso_kv_verify_tree(siso_kv *kv, const siso_kv_batch *batch, const int *parent, const int *tokens, int vocab, int type,
                                   const void *target, long target_stride, const float *u, int *out_accepted, int *out_rows, int *out_tokens) {
    if (!kv) return SISO_EINVAL;
    KvSettle a;
    const int rc = tree_batch(kv, "siso_kv_verify_tree", batch, &a.batch);
    if (rc != SISO_OK) return rc;
    if (vocab < 1 || vocab > (1 << 24)) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify_tree: vocabulary of %d", vocab);
    if (type != SISO_F32 && type != SISO_BF16) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify_tree: probabilities of type %d", type);
    if (a.batch.n == 0) return SISO_OK;
    if (!out_accepted || (a.batch.rows > 0 && (!parent || !tokens || !target || !out_rows || !out_tokens)))
        return kv_fail(kv, SISO_EINVAL, "siso_kv_verify_tree: parents, tokens, target or outputs are NULL");
    if ((uintptr_t)target & (type == SISO_F32 ? 3 : 1)) return kv_fail(kv, SISO_EINVAL, "siso_kv_verify_tree: probabilities are not aligned to their type");
    a.parent = parent;
    a.tokens = tokens;
    a.vocab = vocab;
    a.target = target;
    a.target_stride = target_stride;
    a.u = u;
    a.accepted = out_accepted;
    a.rows = out_rows;
    a.out = out_tokens;
    const long most = kv_max_new(batch), places = a.batch.n * most;
    if (!u && (long)a.batch.rows * vocab * (type == SISO_F32 ? 4 : 2) <= KV_SETTLE_ALL && most > 0 && places <= KV_SETTLE_PLACES) {
        const long units = (vocab + KV_SLICE_UNIT - 1) / KV_SLICE_UNIT;
        long slices = 1024 / places;
        slices = slices > 64 ? 64 : slices > units ? units : slices;
        slices = slices < 1 ? 1 : slices;
        a.slice = (int)((units + slices - 1) / slices * KV_SLICE_UNIT);
        a.slices = (vocab + a.slice - 1) / a.slice;
        a.most = (int)most;
        a.parts = (u64 *)kv->parts;
        a.named = (int *)(a.parts + places * a.slices);
        a.arrived = kv->arrived;
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(places * a.slices)), dim3(256), 0, kv->stream, a); };
        type == SISO_F32 ? go(k_kv_settle_all<float>) : go(k_kv_settle_all<bf16_t>);
    } else {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.batch.n), dim3(KV_SETTLE), 0, kv->stream, a); };
        if (type == SISO_F32) u ? go(k_kv_settle<float, false>) : go(k_kv_settle<float, true>);
        else u ? go(k_kv_settle<bf16_t, false>) : go(k_kv_settle<bf16_t, true>);
    }
    KV_TRY(kv, hipGetLastError());
    return SISO_OK;
}

extern "C" int siso_kv_keep(siso_kv *kv, int layer, const siso_kv_batch *batch, const int *path) {
    if (!kv) return SISO_EINVAL;
    if (layer < -1) return kv_fail(kv, SISO_EINVAL, "siso_kv_keep: layer %d", layer);
    KvBatch b;
    const int rc = kv_batch(kv, "siso_kv_keep", layer < 0 ? 0 : layer, batch, &b);
    if (rc != SISO_OK) return rc;
    if (b.n == 0 || b.rows == 0) return SISO_OK;
    if (!path) return kv_fail(kv, SISO_EINVAL, "siso_kv_keep: no path");
    const KvPool pool = kv_pool(kv, layer < 0 ? 0 : layer);
    const long layers = layer < 0 ? kv->layers : 1;
    if (layers * kv->kv_heads > 1L << 23) return kv_fail(kv, SISO_EINVAL, "siso_kv_keep: %ld layers of %d kv heads at once", layers, kv->kv_heads);
    const long each = (1L << 23) / (layers * kv->kv_heads);  // sequences of a launch, which has fewer than 2^32 threads
    for (long b0 = 0; b0 < b.n; b0 += each) {
        const dim3 grid((unsigned)((b.n - b0 < each ? b.n - b0 : each) * layers * kv->kv_heads));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kv->dp), 0, kv->stream, pool, b, path, (long)kv->layer_bytes, (long)kv->layer_scales, (int)layers, (int)b0);
        };
        kv->dtype == SISO_FP8 ? go(k_kv_keep<true>) : go(k_kv_keep<false>);
        KV_TRY(kv, hipGetLastError());
    }
    return SISO_OK;
}
