// Rows of class scores: what the score kernels share.  Elements and their ordered keys, the
// walk over a row in 16-byte vectors, teams of wavefronts that work on one row, and the
// weights of the sampler.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dtree_scores.h"

namespace dscores {

// ---- elements ---------------------------------------------------------------------------
//
// key() maps an element to an unsigned number of the same order, 0 for what is never chosen
// (-inf, NaN, no votes, and places outside the row); value() maps it back to the score.

template <dt_dtype XT>
struct Elem;

__device__ __forceinline__ uint32_t float_key(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);                    // -0 becomes +0
    const uint32_t o = b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
    return f > -__builtin_inff() ? o : 0u;                           // false for NaN
}

__device__ __forceinline__ float key_float(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

template <>
struct Elem<DT_F32> {
    using Raw = uint32_t;
    static constexpr int kBytes = 4, kKeyBits = 32;
    static __device__ __forceinline__ float wide(Raw r) { return __uint_as_float(r); }
    static __device__ __forceinline__ uint32_t key(Raw r) { return float_key(wide(r)); }
    static __device__ __forceinline__ float value(uint32_t k) { return key_float(k); }
    static __device__ __forceinline__ Raw narrow(float f) { return __float_as_uint(f); }
};

// The 16-bit types' keys have 16 bits: the ordered bits of the element itself.
__device__ __forceinline__ uint32_t half_order(uint32_t b) {
    return (b & 0x8000u) ? (~b & 0xFFFFu) : (b | 0x8000u);
}

template <>
struct Elem<DT_F16> {
    using Raw = uint16_t;
    static constexpr int kBytes = 2, kKeyBits = 16;
    static __device__ __forceinline__ float wide(Raw r) {
        return float(__builtin_bit_cast(_Float16, r));
    }
    static __device__ __forceinline__ uint32_t key(Raw r) {
        const uint32_t b = r == 0x8000u ? 0u : r;
        // -inf, and NaN of either sign
        return (b == 0xFC00u || (b & 0x7FFFu) > 0x7C00u) ? 0u : half_order(b);
    }
    static __device__ __forceinline__ float value(uint32_t k) {
        return wide(Raw(k & 0x8000u ? k ^ 0x8000u : ~k & 0xFFFFu));
    }
    static __device__ __forceinline__ Raw narrow(float f) {
        return __builtin_bit_cast(Raw, _Float16(f));
    }
};

template <>
struct Elem<DT_BF16> {
    using Raw = uint16_t;
    static constexpr int kBytes = 2, kKeyBits = 16;
    static __device__ __forceinline__ float wide(Raw r) { return __uint_as_float(uint32_t(r) << 16); }
    static __device__ __forceinline__ uint32_t key(Raw r) {
        const uint32_t b = r == 0x8000u ? 0u : r;
        return (b == 0xFF80u || (b & 0x7FFFu) > 0x7F80u) ? 0u : half_order(b);
    }
    static __device__ __forceinline__ float value(uint32_t k) {
        return wide(Raw(k & 0x8000u ? k ^ 0x8000u : ~k & 0xFFFFu));
    }
    // to the nearest, ties to even; a NaN keeps its place
    static __device__ __forceinline__ Raw narrow(float f) {
        const uint32_t b = __float_as_uint(f);
        const uint32_t r = (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16;
        return f != f ? Raw(0x7FC0u) : Raw(r);
    }
};

template <>
struct Elem<DT_U8> {
    using Raw = uint8_t;
    static constexpr int kBytes = 1, kKeyBits = 8;
    static __device__ __forceinline__ float wide(Raw r) { return logf(float(r)); }
    static __device__ __forceinline__ uint32_t key(Raw r) { return r; }
    static __device__ __forceinline__ float value(uint32_t k) { return logf(float(k)); }
};

// ---- rows -------------------------------------------------------------------------------
//
// A row is read in aligned 16-byte vectors.  The first and the last may reach beyond the row:
// of those only the row's own elements are read, one by one.  Vector v holds the classes
// first(v) .. first(v) + kVec - 1.

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <dt_dtype XT>
struct Row {
    using E = Elem<XT>;
    using Raw = typename E::Raw;
    static constexpr int kVec = 16 / E::kBytes;
    static constexpr int kAhead = kVec <= 8 ? 4 : 2;   // vectors in flight on a walk
    const Raw *p;     // class 0
    int n;            // classes
    int skew;         // elements between the 16-byte boundary before the row and the row
    int vecs;

    __device__ __forceinline__ Row(const void *x, int64_t row, int64_t ld, int n_classes) {
        p = static_cast<const Raw *>(x) + row * ld;
        n = n_classes;
        skew = int(reinterpret_cast<uintptr_t>(p) & 15u) / E::kBytes;
        vecs = (n + skew + kVec - 1) / kVec;
    }
    __device__ __forceinline__ int first(int v) const { return v * kVec - skew; }
    __device__ __forceinline__ bool whole(int v) const {
        return first(v) >= 0 && first(v) + kVec <= n;
    }
    static __device__ __forceinline__ Raw at(const u32x4 &a, int i) {
        constexpr int kPerWord = 4 / E::kBytes;
        return Raw(a[i / kPerWord] >> (8 * E::kBytes * (i % kPerWord)));
    }
    __device__ __forceinline__ u32x4 load_whole(int v) const {
        return *reinterpret_cast<const u32x4 *>(p + first(v));
    }
    // Vector v, whose places outside the row are 0.
    __device__ __forceinline__ u32x4 load(int v) const {
        if (whole(v)) return load_whole(v);
        constexpr int kPerWord = 4 / E::kBytes;
        const int c = first(v);
        u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (has(c + i)) r[i / kPerWord] |= uint32_t(p[c + i]) << (8 * E::kBytes * (i % kPerWord));
        return r;
    }
    __device__ __forceinline__ bool has(int c) const { return c >= 0 && c < n; }
    // This thread's share of the vectors [lo, hi), U loads in flight: vector(a, v) for those that
    // lie in the row, single(element, class) for the elements of a first or last one that does not.
    template <int U, class FV, class FE>
    __device__ __forceinline__ void walk(int lo, int hi, int thread, int threads, FV vector,
                                         FE single) const {
        const bool head = lo == 0 && skew > 0 && hi > 0;
        const bool tail = hi == vecs && hi - 1 >= (head ? 1 : lo) && !whole(vecs - 1);
        if (head)
            for (int c = thread; c < kVec - skew && c < n; c += threads) single(p[c], c);
        if (tail)
            for (int c = first(vecs - 1) + thread; c < n; c += threads) single(p[c], c);
        const int end = tail ? hi - 1 : hi;
        int v = (head ? 1 : lo) + thread;
        for (; v + (U - 1) * threads < end; v += U * threads) {
            u32x4 a[U];
#pragma unroll
            for (int u = 0; u < U; ++u) a[u] = load_whole(v + u * threads);
#pragma unroll
            for (int u = 0; u < U; ++u) vector(a[u], v + u * threads);
        }
        for (; v < end; v += threads) vector(load_whole(v), v);
    }
    // f(element, class) for all elements of the share.
    template <int U, class F>
    __device__ __forceinline__ void each(int lo, int hi, int thread, int threads, F f) const {
        walk<U>(lo, hi, thread, threads,
                [&](const u32x4 &a, int v) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) f(at(a, i), first(v) + i);
                },
                f);
    }
    // f(element, class) for the elements of vector v, given as loaded.
    template <class F>
    __device__ __forceinline__ void visit(const u32x4 &a, int v, F f) const {
        const int c = first(v);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (has(c + i)) f(at(a, i), c + i);
    }
};

// ---- teams ------------------------------------------------------------------------------
//
// WAVES wavefronts that work on one row together.  A team of one wavefront shares its
// workgroup with others and never meets a workgroup barrier; a larger one is a workgroup.

template <class T>
__device__ __forceinline__ T xor_lane(T v, int mask) {
    if constexpr (sizeof(T) == 8) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __shfl_xor(int(uint32_t(b)), mask), hi = __shfl_xor(int(uint32_t(b >> 32)), mask);
        return __builtin_bit_cast(T, uint64_t(hi) << 32 | lo);
    } else {
        return __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, v), mask));
    }
}

template <class T>
__device__ __forceinline__ T from_lane(T v, int lane) {
    if constexpr (sizeof(T) == 8) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __shfl(int(uint32_t(b)), lane), hi = __shfl(int(uint32_t(b >> 32)), lane);
        return __builtin_bit_cast(T, uint64_t(hi) << 32 | lo);
    } else {
        return __builtin_bit_cast(T, __shfl(__builtin_bit_cast(int, v), lane));
    }
}

struct Max {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; }
};
struct Min {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a < b ? a : b; }
};
struct Sum {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};

// Over groups of `width` neighbouring lanes (a power of two).
template <class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, Op op, int width = 64) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        if (m < width) v = op(v, xor_lane(v, m));
    return v;
}

// Sum over the lanes before this one; *all gets the wavefront's.
template <class T>
__device__ __forceinline__ T wave_before(T v, int lane, T *all) {
    T s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T o = from_lane(s, lane - d);
        if (lane >= d) s += o;
    }
    *all = from_lane(s, 63);
    return s - v;
}

template <int WAVES>
struct Team {
    static constexpr int kThreads = 64 * WAVES;
    int thread, lane, wave;      // of the team
    uint64_t *box;               // WAVES words of the LDS

    __device__ __forceinline__ void sync() const {
        if constexpr (WAVES == 1) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        } else {
            __syncthreads();
        }
    }
    template <class T, class Op>
    __device__ __forceinline__ T reduce(T v, Op op) const {
        v = wave_reduce(v, op);
        if constexpr (WAVES > 1) {
            T *b = reinterpret_cast<T *>(box);
            sync();                                  // box free
            if (lane == 0) b[wave] = v;
            sync();
            v = b[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v = op(v, b[w]);
        }
        return v;
    }
    // Sum over the threads before this one; *all gets the team's.
    template <class T>
    __device__ __forceinline__ T before(T v, T *all) const {
        T s = wave_before(v, lane, all);
        if constexpr (WAVES > 1) {
            T *b = reinterpret_cast<T *>(box);
            sync();
            if (lane == 0) b[wave] = *all;
            sync();
            T t = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) s += b[w];
                t += b[w];
            }
            *all = t;
        }
        return s;
    }
};

// e^x in fp32 for x <= 0 (and NaN): 2^(x log2 e) by the hardware's 2^y, with the product's
// rounding error put back, since at y = -100 half a step of y alone is 2^-18.
__device__ __forceinline__ float exp_neg(float x) {
    const float y = x * 1.44269504f;
    const float err = fmaf(x, 1.44269504f, -y) + x * 1.92596e-8f;    // log2 e = 1.44269504 + 1.92596e-8
    const float e = __builtin_amdgcn_exp2f(y);
    // below 2^-126 the hardware gives 0; -inf - -inf in err must not reach the result
    return e > 0.0f ? fmaf(e, err * 0.693147181f, e) : e;
}

// ---- the order of a row's classes, best first ---------------------------------------------
//
// comp() makes one number of a key and a class: larger for the larger key, at equal keys for
// the lower class.  No two classes of a row have the same.

__device__ __forceinline__ uint64_t comp(uint32_t key, int c) {
    return uint64_t(key) << 32 | uint32_t(~c);
}
__device__ __forceinline__ uint32_t comp_key(uint64_t v) { return uint32_t(v >> 32); }
__device__ __forceinline__ int comp_class(uint64_t v) { return int(~uint32_t(v)); }

}  // namespace dscores
