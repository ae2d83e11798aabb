// What the translation units of the paged key/value cache share (siso_kv.h).
#pragma once

#include "siso_internal.h"
#include "siso_kv.h"

// How a page lies in memory.  Attention multiplies 32 x 32 tiles with v_mfma_f32_32x32x16_bf16: S^T = K Q^T, then O^T = V^T P^T.
// Keys and values are kept in the order in which the lanes of these products want them, in blocks of 16 tokens, so that
// a wave loads an operand as whole lines, 16 bytes a lane, straight to registers or LDS, and no product transposes anything.
//   K: 16-byte chunks [chunk of the dimension][token]: lane l of a fragment takes token l % 16 of one of two blocks and every
//      second chunk from l / 32 on.  A chunk is 8 elements of 16 bits or 16 codes: one fragment or two.
//   V: the accumulator of S^T holds, in lane half h, tokens 4 h + j and 8 + 4 h + j (j < 4) of a block: as they are, these
//      eight are an operand of the second product.  V is kept as [h][dimension][these eight tokens] (16 bits: 16 bytes); codes as
//      [h][dimension / 64][32][two 32s of the dimension][eight tokens], again 16 bytes for a lane: two fragments.
// The dimension is rounded up to a multiple of 64; what lies beyond it is zero from siso_kv_create on and never written.
#define SISO_KV_BLOCK 16
__host__ __device__ __forceinline__ int kv_slot(int key) { return (key & 3) + 4 * (key >> 3); }  // of a block's token among the eight of its half
__host__ __device__ __forceinline__ int kv_half(int key) { return (key >> 2) & 1; }

// Pools: [layer][page][kv head][page_tokens * dp * (2 or 1) bytes], blocks one after the other; scales [layer][page][kv head][page_tokens].
struct KvPool {
    char *k, *v;
    float *ks, *vs;  // NULL: 16 bits
    u64 *bad;
    int pages;
    int kv_heads, shift;  // page_tokens = 1 << shift
    int dim, dp;
};

// Positions of a sequence, at most: kernels look up to some thousand positions ahead and up to 2^24 rows and a window back, in 32 bits.
#define SISO_KV_MOST ((1L << 31) - (1L << 25))

struct KvBatch {  // siso_kv_batch as kernels take it
    const int *first, *length, *pages;
    int n, rows;
    long width;
    int most;  // the longest length there can be: width * page_tokens
    int single;  // every sequence has exactly one row
};

// Sequences' rows in groups of 1 << shift, `group` of a row's units each (attention: query heads that share a kv head): group
// number j of sequence b is slot kv_slots_before(b) + j, for every sequence as many slots as it may have groups and `extra`
// more.  Nothing but the rows before a sequence decides where its slots begin: no launch before that one counts them.
__host__ __device__ __forceinline__ long kv_slots_before(long first, long b, int group, int shift, int extra) {
    return ((first * group) >> shift) + b * extra;
}

#ifdef __HIPCC__
struct KvSequence {
    int b, first, rows, length;
    int start;  // position of the first row; may be below zero
};

__device__ __forceinline__ int kv_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ KvSequence kv_sequence(const KvBatch &batch, int b) {
    KvSequence s;
    s.b = b;
    s.first = kv_clamp(batch.first[b], 0, batch.rows);
    s.rows = kv_clamp(batch.first[b + 1], s.first, batch.rows) - s.first;
    s.length = batch.length ? kv_clamp(batch.length[b], 0, batch.most) : 0;
    s.start = s.length - s.rows;
    return s;
}

// The sequence that `slot` belongs to, the same in every lane: the wave looks at 64 sequences at a time.  Of up to 64 the lanes already have
// what is to be known of the one that it is: one wait for memory, not two.
__device__ __forceinline__ KvSequence kv_sequence_of(const KvBatch &batch, long slot, int group, int shift, int extra) {
    const int lane = threadIdx.x & 63;
    if (batch.n <= 64) {
        KvSequence s = kv_sequence(batch, lane < batch.n ? lane : batch.n - 1);
        const int before = __popcll(__ballot(lane < batch.n && kv_slots_before(s.first, lane, group, shift, extra) <= slot));
        const int at = before > 0 ? before - 1 : 0;  // (not decreasing: those before come first)
        s.b = at;
        s.first = __builtin_amdgcn_readlane(s.first, at);
        s.rows = __builtin_amdgcn_readlane(s.rows, at);
        s.length = __builtin_amdgcn_readlane(s.length, at);
        s.start = s.length - s.rows;
        return s;
    }
    int lo = 0, count = batch.n;
    while (count > 1) {
        const int step = (count + 63) / 64, at = lo + lane * step;
        const bool before = lane * step < count && kv_slots_before(kv_clamp(batch.first[at], 0, batch.rows), at, group, shift, extra) <= slot;
        const int k = __popcll(__ballot(before));
        lo += (k > 0 ? k - 1 : 0) * step;
        count = batch.n - lo < step ? batch.n - lo : step;
    }
    return kv_sequence(batch, __builtin_amdgcn_readfirstlane(lo));
}

// What the table says of position `at` (below most, the same in every lane): by a load of the scalar unit, which no vector load
// waits for or is waited for with.
__device__ __forceinline__ int kv_page_entry(const KvPool &pool, const KvBatch &batch, int b, int at) {
    return *(const __attribute__((address_space(4))) int *)(batch.pages + ((long)b * batch.width + (at >> pool.shift)));
}
__device__ __forceinline__ bool kv_is_page(const KvPool &pool, int page) { return (unsigned)page < (unsigned)pool.pages; }
// Where the block of position `at` of a kv head begins, in bytes for elements of one byte (16 bits: twice that).
__device__ __forceinline__ size_t kv_block_at(const KvPool &pool, int page, int head, int at) {
    return ((size_t)((long)page * pool.kv_heads + head) << pool.shift) * pool.dp + (size_t)(((at & ((1 << pool.shift) - 1)) >> 4) * SISO_KV_BLOCK) * pool.dp;
}
// Values in 8 bits: the eight tokens of half h and dimension d, in a block.
__device__ __forceinline__ size_t kv_v8_at(int dp, int h, int d) { return (((h * (dp >> 6) + (d >> 6)) * 32 + (d & 31)) * 2 + ((d >> 5) & 1)) * 8; }
__device__ __forceinline__ size_t kv_scale_at(const KvPool &pool, int page, int head, int at) {
    return ((size_t)((long)page * pool.kv_heads + head) << pool.shift) + (at & ((1 << pool.shift) - 1));
}
#endif

#define SISO_KV_PARTS ((size_t)32 << 20)  // 128 MiB
#define SISO_KV_PLAN_BYTES 16384
#define SISO_KV_JOINS 65536  // sequences of a batch; workgroups of an attention launch that leaves parts to be joined are fewer

struct siso_kv {
    int layers, kv_heads, dim, dp, page_tokens, dtype;
    long pages;
    hipStream_t stream;
    char *k, *v;
    float *ks, *vs;
    size_t layer_bytes, layer_scales;
    u64 *counters;      // [0] page numbers that are none; behind it `arrived`
    unsigned *arrived;  // [SISO_KV_JOINS] how many parts are there of what several workgroups work on; zeros between calls
    void *plan;         // [SISO_KV_PLAN_BYTES], see kv_attend.hip
    float *parts;       // [SISO_KV_PARTS] what splits of a long axis leave for the one that joins them; see kv_attend.hip and kv_verify.hip
    char err[256];
};

int kv_fail(siso_kv *kv, int code, const char *fmt, ...);
int kv_check_hip(siso_kv *kv, hipError_t e, const char *what);
#define KV_TRY(kv, call)                                           \
    do {                                                           \
        const int kv_rc_ = kv_check_hip((kv), (call), #call);      \
        if (kv_rc_ != SISO_OK) return kv_rc_;                      \
    } while (0)
KvPool kv_pool(const siso_kv *kv, int layer);
// Checks a batch for a call that reads the cache (or, layer < 0, does not) and brings it into the kernels' form.
int kv_batch(siso_kv *kv, const char *call, int layer, const siso_kv_batch *batch, KvBatch *out);
// The most rows that a sequence of a checked batch can have.
static inline long kv_max_new(const siso_kv_batch *batch) { return batch->max_new > 0 && batch->max_new < batch->rows ? batch->max_new : batch->rows; }
