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
// rank() maps an element to an unsigned number of the order of scores, NaN of either sign and -inf
// at the bottom (up to kNone): the bits of a float, complemented below zero and with the sign bit
// set above, are in order already, and adding the number of positive NaNs turns these round to
// the bottom.  It takes four operations, on two elements at a time for the 16-bit types, and is
// what walks over long rows look at.  The two zeros are neighbours.
//
// key() is the rank with the zeros made equal and 0 for what is never chosen (also the places
// outside a row); value() maps a key back to the score.

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <dt_dtype XT>
struct Elem;

// Ranks of float types: TURN positive NaNs, ranks of BITS bits.
template <uint32_t TURN, int BITS>
struct FloatRanks {
    static constexpr uint32_t kMask = BITS == 32 ? 0xFFFFFFFFu : 0xFFFFu;
    static constexpr uint32_t kSign = 1u << (BITS - 1);
    static constexpr uint32_t kNone = 2 * TURN;                     // -inf
    static constexpr uint32_t kZero = kSign + TURN;                 // +0; -0 is one below
    static __device__ __forceinline__ uint32_t rank_of_bits(uint32_t b) {
        const uint32_t o = b & kSign ? ~b : b | kSign;
        return (o + TURN) & kMask;
    }
    static __device__ __forceinline__ uint32_t bits_of_key(uint32_t k) {
        const uint32_t o = (k - TURN) & kMask;
        return o & kSign ? o ^ kSign : ~o & kMask;
    }
    static __device__ __forceinline__ uint32_t key_of_rank(uint32_t r) {
        return r <= kNone ? 0u : r == kZero - 1 ? kZero : r;
    }
    // the lowest rank whose key is at least this rank's
    static __device__ __forceinline__ uint32_t from_rank(uint32_t r) { return r == kZero ? r - 1 : r; }
};

template <>
struct Elem<DT_F32> : FloatRanks<0x007FFFFFu, 32> {
    using Raw = uint32_t;
    static constexpr int kBytes = 4;
    static __device__ __forceinline__ float wide(Raw r) { return __uint_as_float(r); }
    static __device__ __forceinline__ uint32_t rank(Raw r) { return rank_of_bits(r); }
    static __device__ __forceinline__ uint32_t key(Raw r) { return key_of_rank(rank(r)); }
    static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(bits_of_key(k)); }
    static __device__ __forceinline__ Raw narrow(float f) { return __float_as_uint(f); }
};

template <>
struct Elem<DT_F16> : FloatRanks<0x03FFu, 16> {
    using Raw = uint16_t;
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float wide(Raw r) {
        return float(__builtin_bit_cast(_Float16, r));
    }
    static __device__ __forceinline__ uint32_t rank(Raw r) { return rank_of_bits(r); }
    static __device__ __forceinline__ uint32_t key(Raw r) { return key_of_rank(rank(r)); }
    static __device__ __forceinline__ float value(uint32_t k) { return wide(Raw(bits_of_key(k))); }
    static __device__ __forceinline__ Raw narrow(float f) {
        return __builtin_bit_cast(Raw, _Float16(f));
    }
};

template <>
struct Elem<DT_BF16> : FloatRanks<0x007Fu, 16> {
    using Raw = uint16_t;
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float wide(Raw r) { return __uint_as_float(uint32_t(r) << 16); }
    static __device__ __forceinline__ uint32_t rank(Raw r) { return rank_of_bits(r); }
    static __device__ __forceinline__ uint32_t key(Raw r) { return key_of_rank(rank(r)); }
    static __device__ __forceinline__ float value(uint32_t k) { return wide(Raw(bits_of_key(k))); }
    // to the nearest, ties to even
    static __device__ __forceinline__ Raw narrow(float f) {
        return __builtin_bit_cast(Raw, __bf16(f));
    }
};

// Votes: the number itself, none at the bottom.
template <>
struct Elem<DT_U8> {
    using Raw = uint8_t;
    static constexpr int kBytes = 1;
    static constexpr uint32_t kNone = 0;
    static __device__ __forceinline__ float wide(Raw r) { return logf(float(r)); }
    static __device__ __forceinline__ uint32_t rank(Raw r) { return r; }
    static __device__ __forceinline__ uint32_t key(Raw r) { return r; }
    static __device__ __forceinline__ uint32_t key_of_rank(uint32_t r) { return r; }
    static __device__ __forceinline__ uint32_t from_rank(uint32_t r) { return r; }
    static __device__ __forceinline__ float value(uint32_t k) { return logf(float(k)); }
};

// The ranks of a vector of 16 bytes, and a running maximum of them.
template <dt_dtype XT>
struct Ranks {
    using E = Elem<XT>;
    // of the four words of a vector: ranks of its elements, in pairs of 16 bits for narrow types
    static constexpr int kWords = XT == DT_U8 ? 8 : 4;
    uint32_t w[kWords];

    __device__ __forceinline__ explicit Ranks(const u32x4 &a) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (XT == DT_F32) {
                w[i] = E::rank(a[i]);
            } else if constexpr (XT == DT_U8) {
                w[i] = a[i] & 0x00FF00FFu;
                w[4 + i] = (a[i] >> 8) & 0x00FF00FFu;
            } else {
                // all ones in the halves below zero, the sign bit in the others (in whole words:
                // of packed 16-bit shifts of a vector's four words the compiler made one)
                const u16x2 turn = {uint16_t(E::kNone / 2), uint16_t(E::kNone / 2)};
                const uint32_t sign = a[i] & 0x80008000u;
                const uint32_t flip = (sign - (sign >> 15)) | 0x80008000u;
                w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2, a[i] ^ flip) + turn);
            }
        }
    }
    // A running maximum, in the words' form
    struct Max {
        uint32_t v = 0;
        __device__ __forceinline__ void add(const Ranks &r) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (XT == DT_F32)
                    v = r.w[i] > v ? r.w[i] : v;
                else
                    v = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
                            __builtin_bit_cast(u16x2, r.w[i]), __builtin_bit_cast(u16x2, v)));
            }
        }
        __device__ __forceinline__ uint32_t rank() const {
            if constexpr (XT == DT_F32) return v;
            return (v & 0xFFFFu) > (v >> 16) ? v & 0xFFFFu : v >> 16;
        }
    };
};

// Whether a vector has elements that reach a bound.  Of the float types the largest of the widened
// elements is compared, three operands an instruction, which costs half an operation an
// element where the ranks cost three.  A NaN is passed over, unless there is nothing else: then it counts
// as reaching the bound, and the elements' ranks tell.  A signalling NaN is passed over as well once
// quiet_max() was called; in the IEEE mode in which kernels start it makes max3 lose what came before it.
__device__ __forceinline__ void quiet_max() {
    constexpr int kMode = 1, kIeee = 9;                // hardware register, bit of it
    __builtin_amdgcn_s_setreg(kMode | kIeee << 6 | (1 - 1) << 11, 0);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

template <dt_dtype XT>
struct Wide {
    using E = Elem<XT>;
    static constexpr int kVec = 16 / E::kBytes, kPerWord = 4 / E::kBytes;
    float x[kVec];
    __device__ __forceinline__ explicit Wide(const u32x4 &a) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            x[i] = E::wide(typename E::Raw(a[i / kPerWord] >> (8 * E::kBytes * (i % kPerWord))));
    }
    __device__ __forceinline__ float max() const {
        float m = max3(x[0], x[1], x[2]);
#pragma unroll
        for (int i = 3; i + 1 < kVec; i += 2) m = max3(m, x[i], x[i + 1]);
        return max3(m, x[kVec - 1], x[kVec - 1]);
    }
};

template <dt_dtype XT>
struct Filter {
    using E = Elem<XT>;
    uint32_t least;        // rank, > kNone
    float bound;
    __device__ __forceinline__ explicit Filter(uint32_t least_rank) : least(least_rank) {
        if constexpr (XT != DT_U8) bound = E::value(E::key_of_rank(least));
    }
    // Whether an element of the vector may reach the bound.
    __device__ __forceinline__ bool maybe(const u32x4 &a) const {
        if constexpr (XT == DT_U8) {
            // what a number has above least - 1, or nothing
            const u16x2 below = {uint16_t(least - 1), uint16_t(least - 1)};
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w = (i < 4 ? a[i & 3] : a[i & 3] >> 8) & 0x00FF00FFu;
                some |= __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(
                            __builtin_bit_cast(u16x2, w), below));
            }
            return some != 0;
        } else {
            return !(Wide<XT>(a).max() < bound);
        }
    }
};

// The largest rank of a part of a row (quiet_max() before it, as for Filter).
template <dt_dtype XT>
struct PartMax {
    using E = Elem<XT>;
    typename Ranks<XT>::Max ranks;
    float m = -__builtin_inff();
    __device__ __forceinline__ void add(const u32x4 &a) {
        if constexpr (XT == DT_U8) {
            ranks.add(Ranks<XT>(a));
        } else {
            const Wide<XT> w(a);
            m = max3(m, w.max(), w.x[0]);
        }
    }
    __device__ __forceinline__ uint32_t rank() const {
        if constexpr (XT == DT_U8)
            return ranks.rank();
        else
            return E::rank(E::narrow(m));                      // exact: it is one of the elements
    }
};

// ---- rows -------------------------------------------------------------------------------
//
// A row is read in aligned 16-byte vectors.  The first and the last may reach beyond the row:
// of those only the row's own elements are read, one by one.  Vector v holds the classes
// first(v) .. first(v) + kVec - 1.

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
        // a row takes less than 2^32 bytes: an offset of 32 bits to an address that, being the same for
        // a whole team, stays in scalar registers
        const char *base = reinterpret_cast<const char *>(p - skew);
        return *reinterpret_cast<const u32x4 *>(base + (uint32_t(v) << 4));
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
    // The vectors that lie in the row as a whole: [inner_lo, inner_hi).
    __device__ __forceinline__ int inner_lo() const { return skew > 0 ? 1 : 0; }
    __device__ __forceinline__ int inner_hi() const {
        const int hi = whole(vecs - 1) ? vecs : vecs - 1;
        return hi > inner_lo() ? hi : inner_lo();
    }
    // This thread's share of the vectors [lo, hi), which lie in the row, U loads in flight.
    template <int U, class FV>
    __device__ __forceinline__ void inner(int lo, int hi, int thread, int threads, FV vector) const {
        int v = lo + thread;
        for (; v + (U - 1) * threads < hi; v += U * threads) {
            u32x4 a[U];
#pragma unroll
            for (int u = 0; u < U; ++u) a[u] = load_whole(v + u * threads);
#pragma unroll
            for (int u = 0; u < U; ++u) vector(a[u], v + u * threads);
        }
        for (; v < hi; v += threads) vector(load_whole(v), v);
    }
    // f(element, class) for the elements outside these, one to a thread: fewer than 32, so a team has
    // a thread for each.
    template <class F>
    __device__ __forceinline__ void ends(int thread, F f) const {
        const int head = inner_lo() == 0 ? 0 : (kVec - skew < n ? kVec - skew : n);
        const int tail = first(inner_hi()) > head ? first(inner_hi()) : head;
        const int c = thread < head ? thread : tail + thread - head;
        if (c < n) f(p[c], c);
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

// A lane's partner in a reduction: by data-parallel moves within rows of 16 lanes, where a
// mirrored lane holds the same as the xor partner once the steps below it are done.
template <int STEP, class T>
__device__ __forceinline__ T partner(T v) {
    if constexpr (STEP >= 16) {
        return xor_lane(v, STEP);
    } else if constexpr (sizeof(T) == 8) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = partner<STEP>(uint32_t(b)), hi = partner<STEP>(uint32_t(b >> 32));
        return __builtin_bit_cast(T, uint64_t(hi) << 32 | lo);
    } else {
        // quad_perm [1,0,3,2], quad_perm [2,3,0,1], row_half_mirror, row_mirror
        constexpr int kControl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
        const int b = __builtin_bit_cast(int, v);
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(b, b, kControl, 0xF, 0xF, true));
    }
}

// Over groups of WIDTH neighbouring lanes (a power of two); every lane gets the result.
template <int WIDTH = 64, class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, Op op) {
    if constexpr (WIDTH > 1) v = op(v, partner<1>(v));
    if constexpr (WIDTH > 2) v = op(v, partner<2>(v));
    if constexpr (WIDTH > 4) v = op(v, partner<4>(v));
    if constexpr (WIDTH > 8) v = op(v, partner<8>(v));
    if constexpr (WIDTH > 16) v = op(v, partner<16>(v));
    if constexpr (WIDTH > 32) v = op(v, partner<32>(v));
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

// Orders a wavefront's accesses of the LDS.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int WAVES>
struct Team {
    static constexpr int kThreads = 64 * WAVES;
    int thread, lane, wave;      // of the team
    uint64_t *box;               // WAVES words of the LDS

    __device__ __forceinline__ void sync() const {
        if constexpr (WAVES == 1) {
            wave_fence();
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
