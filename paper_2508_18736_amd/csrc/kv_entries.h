// Rows of probabilities or logits, eight entries at a time.
#pragma once

#include "siso_internal.h"

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
