// Rows of at most 64 classes: one lane works on one row, which it holds in registers as
// numbers that order its classes (comp32 of the types with 16-bit keys, comp of fp32).
#pragma once

#include "scores.hpp"
#include "scores_common.hpp"

namespace dscores {

template <dt_dtype XT>
struct Order {
    using T = uint32_t;
    static __device__ __forceinline__ T make(uint32_t key, int c) { return key << 16 | (0xFFFFu - c); }
    static __device__ __forceinline__ uint32_t key(T v) { return v >> 16; }
    static __device__ __forceinline__ int cls(T v) { return int(0xFFFFu - (v & 0xFFFFu)); }
};

template <>
struct Order<DT_F32> {
    using T = uint64_t;
    static __device__ __forceinline__ T make(uint32_t key, int c) { return comp(key, c); }
    static __device__ __forceinline__ uint32_t key(T v) { return comp_key(v); }
    static __device__ __forceinline__ int cls(T v) { return comp_class(v); }
};

// e[i] = element i of the row at p, 0 behind its n elements.  Reads 16 or 4 bytes at a time
// where the rows' alignment allows, and nothing outside the row.
template <dt_dtype XT, int CP>
__device__ __forceinline__ void load_row(const void *x, int64_t row, int64_t ld, int n, int align,
                                         typename Elem<XT>::Raw (&e)[CP]) {
    using Raw = typename Elem<XT>::Raw;
    constexpr int kV = 16 / int(sizeof(Raw)), kW = 4 / int(sizeof(Raw));
    const Raw *p = static_cast<const Raw *>(x) + row * ld;
#pragma unroll
    for (int i = 0; i < CP; ++i) e[i] = Raw(0);
    if constexpr (CP >= kV) {
        if (align >= 16) {
#pragma unroll
            for (int v = 0; v < CP; v += kV) {
                if (v + kV <= n) {
                    struct V { Raw r[kV]; } q =
                        __builtin_bit_cast(V, *reinterpret_cast<const u32x4 *>(p + v));
#pragma unroll
                    for (int i = 0; i < kV; ++i) e[v + i] = q.r[i];
                } else {
#pragma unroll
                    for (int i = 0; i < kV; ++i)
                        if (v + i < n) e[v + i] = p[v + i];
                }
            }
            return;
        }
    }
    if (align >= 4) {
#pragma unroll
        for (int v = 0; v < CP; v += kW) {
            if (v + kW <= n) {
                struct W { Raw r[kW]; } q =
                    __builtin_bit_cast(W, *reinterpret_cast<const uint32_t *>(p + v));
#pragma unroll
                for (int i = 0; i < kW; ++i) e[v + i] = q.r[i];
            } else {
#pragma unroll
                for (int i = 0; i < kW; ++i)
                    if (v + i < n) e[v + i] = p[v + i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < CP; ++i)
            if (i < n) e[i] = p[i];
    }
}

// Descending order by Batcher's odd-even merge network (N = 8, 16, 32, 64: 19, 63, 191, 543
// exchanges, all indexes known to the compiler, so v stays in registers).
template <int N, class T>
__device__ __forceinline__ void sort_registers(T (&v)[N]) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int a = 0; a < N - k; ++a) {
                // a, a + k are exchanged where the merge of blocks of 2p meets them
                const bool on = a >= (k % p) && ((a - (k % p)) % (2 * k)) < k &&
                                (a / (2 * p)) == ((a + k) / (2 * p));
                if (on) {
                    const T x = v[a], y = v[a + k];
                    v[a] = x > y ? x : y;
                    v[a + k] = x > y ? y : x;
                }
            }
}

}  // namespace dscores
