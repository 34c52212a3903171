// Distillation from a teacher's top scores (ds_distill, ds_distill_backward).  Bound by the memory: the
// backward pass of 4,096 x 65,536 bf16 moves its 1.07 GB in 220 us = 4.9 TB/s (a copy reaches 5.2).
//
// With m the row's largest score and s = sum e^((x - m) / t), q_c = e^((x_c - m) / t) / s.  One
// pass over a row finds m and s together: each thread keeps the largest score it has met and the
// sum relative to it, scaled down when a larger one comes.  The gradient takes a second pass:
// every class gets g t q_c, then the teacher's classes (at most 256 a row) are written again
// with their share of p taken off.  An entry whose class another entry has too adds up all of
// them in the entries' order, so both write the same number.
//
// The loss is t times sum_j p_j ((v_j - top) - (x_j - m) + t (ln s - ln s_v)), with the teacher's
// largest value and its sum: nothing is divided by t, and t^2, which may be no fp32 number, is not
// needed.
#include "scores.hpp"
#include "scores_common.hpp"

namespace dscores {
namespace {

constexpr int kLossOnly = 0, kBoth = 1, kGradOnly = 2;

// G lanes of a wavefront, or a workgroup of G threads, that work on one row.
template <int G>
struct Group {
    static constexpr int kInBlock = G <= 64 ? 256 / G : 1;
    static constexpr int kThreads = G <= 64 ? 256 : G;        // of the workgroup
    int thread;
    float *box;                     // G / 64 words, where G > 64

    __device__ __forceinline__ void sync() const {
        if constexpr (G <= 64) {
            wave_fence();
        } else {
            __syncthreads();
        }
    }
    template <class Op>
    __device__ __forceinline__ float reduce(float v, Op op) const {
        v = wave_reduce<(G < 64 ? G : 64)>(v, op);
        if constexpr (G > 64) {
            sync();
            if ((thread & 63) == 0) box[thread >> 6] = v;
            sync();
            v = box[0];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) v = op(v, box[w]);
        }
        return v;
    }
};

// fmaxf leaves out a NaN, which a sum of exponentials keeps.
struct MaxNum {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// e^((x - m) / t) as 2^((x - m) log2 e / t), c = log2 e / t.  The difference comes first, so that a
// common part of all scores (or a whole row of a type's lowest value) costs nothing; the product's
// rounding is at most 1.5 steps of the exponent, which only small terms have large.  m = -inf: then x
// is too, or NaN.
__device__ __forceinline__ float power(float x, float m, float c) {
    return __builtin_amdgcn_exp2f((x - m) * c);
}
__device__ __forceinline__ float finite(float m) { return m == -__builtin_inff() ? 0.0f : m; }

constexpr float kLog2E = 1.44269504f;

// The largest of some scores, and the sum of e^((x - largest) / t) over them.
struct Stats {
    float m = -__builtin_inff(), s = 0.0f;

    __device__ __forceinline__ void raise(float m1, float c) {
        if (m1 > m) {
            s *= power(m, m1, c);
            m = m1;
        }
    }
    __device__ __forceinline__ void add(float x, float c) {
        raise(x, c);
        s += power(x, finite(m), c);
    }
    template <dt_dtype XT>
    __device__ __forceinline__ void add(const Row<XT> &, const u32x4 &a, float c) {
        // (a NaN may be the largest here: `raise` passes over it, and the sum keeps it; one that
        // hides a larger score from the maximum has made the sum a NaN as well)
        const Wide<XT> w(a);
        raise(w.max(), c);
        const float base = finite(m);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < Row<XT>::kVec; ++i) sum += power(w.x[i], base, c);
        s += sum;
    }
    template <class Gr>
    __device__ __forceinline__ void join(const Gr &g, float c) {
        raise(g.reduce(m, MaxNum()), c);
        s = g.reduce(s, Sum());
    }
    // without any score above -inf (a NaN counts as one)
    __device__ __forceinline__ bool empty() const { return m == -__builtin_inff() && s == 0.0f; }
};

// The teacher's entries of one row: their classes (-1: left out) and weights, in the LDS.
struct Entries {
    int *cls;
    float *p;
};

// Fills them in; returns whether there are any, and the row's loss (the first thread's).
template <dt_dtype XT, int MODE, class Gr>
__device__ __forceinline__ bool teach(const DistillArgs &a, const Gr &g, int threads, int64_t r,
                                      const Row<XT> &row, const Stats &st, const Entries &e,
                                      float *loss) {
    const float c2 = kLog2E / a.temperature;
    const float *values = a.values + r * a.k;
    const int32_t *index = a.index + r * a.k;
    float top = -__builtin_inff();
    for (int j = g.thread; j < a.k; j += threads) {
        const float v = values[j];
        const int c = index[j];
        const bool in = c >= 0 && c < a.in.classes && v != -__builtin_inff();
        e.cls[j] = in ? c : -1;
        e.p[j] = v;
        if (in) top = fmaxf(top, v);
    }
    top = g.reduce(top, MaxNum());
    float sum = 0.0f;
    for (int j = g.thread; j < a.k; j += threads)
        if (e.cls[j] >= 0) sum += power(e.p[j], top, c2);
    sum = g.reduce(sum, Sum());
    const bool any = !(sum == 0.0f);   // the best entry adds 1, a NaN a NaN
    const float per_sum = 1.0f / sum;
    const float log_sums = MODE == kGradOnly ? 0.0f : a.temperature * (logf(st.s) - logf(sum));
    float l = 0.0f;
    for (int j = g.thread; j < a.k; j += threads) {
        float p = 0.0f;
        const int c = e.cls[j];
        if (c >= 0) {
            p = power(e.p[j], top, c2) * per_sum;
            if constexpr (MODE != kGradOnly) {
                // t (ln p - ln q)
                const float x = Elem<XT>::wide(row.p[c]) - finite(st.m);
                if (p != 0.0f) l += p * (((e.p[j] - top) - x) + log_sums);
            }
        }
        e.p[j] = p;
    }
    if constexpr (MODE != kGradOnly) {
        l = g.reduce(l, Sum());
        *loss = any && !st.empty() ? a.temperature * l : 0.0f;
    }
    g.sync();                          // the entries are written
    return any;
}

// A row's gradient: of all its classes, then again of the teacher's.
template <dt_dtype XT>
struct Gradient {
    using E = Elem<XT>;
    using Raw = typename E::Raw;
    const Row<XT> &row;
    Raw *out;
    float c2, base, gt, sum, scale;
    bool some, same;

    __device__ __forceinline__ Gradient(const DistillArgs &a, int64_t r, const Row<XT> &row_of,
                                        const Stats &st, bool taught)
        : row(row_of) {
        out = static_cast<Raw *>(a.grad) + r * a.ld_grad;
        c2 = kLog2E / a.temperature;
        base = finite(st.m);
        gt = a.g[r] * a.temperature;
        sum = st.s;
        scale = gt / st.s;
        some = taught && !st.empty();
        // 16-byte stores where its row lies between 16-byte boundaries as the scores' does
        same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15u) == 0;
    }
    __device__ __forceinline__ float of(float x) const {
        return some ? power(x, base, c2) * scale : 0.0f;
    }
    // Stored past the caches, whose place the next reads need: loss and backward of 4,096 x 65,536
    // bf16 in 340 us, 365 us with ordinary stores.
    __device__ __forceinline__ void vector(const u32x4 &v4, int v) const {
        constexpr int kPerWord = 4 / E::kBytes;
        u32x4 q = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < Row<XT>::kVec; ++i)
            q[i / kPerWord] |= uint32_t(E::narrow(of(E::wide(row.at(v4, i)))))
                               << (8 * E::kBytes * (i % kPerWord));
        Raw *to = out + row.first(v);
        if (same) {
            __builtin_nontemporal_store(q, reinterpret_cast<u32x4 *>(to));
        } else {
#pragma unroll
            for (int i = 0; i < Row<XT>::kVec; ++i) to[i] = row.at(q, i);
        }
    }
    __device__ __forceinline__ void single(Raw x, int c) const { out[c] = E::narrow(of(E::wide(x))); }
    // The teacher's classes of the vectors [lo, hi), once all of these have their first value.
    template <class Gr>
    __device__ __forceinline__ void teacher(const DistillArgs &a, const Gr &g, int threads, int lo,
                                            int hi, const Entries &e) const {
        g.sync();
        if (some)
            for (int j = g.thread; j < a.k; j += threads) {
                const int c = e.cls[j];
                if (c < row.first(lo) || c >= row.first(hi) || c < 0) continue;
                float p = 0.0f;
                for (int i = 0; i < a.k; ++i)
                    if (e.cls[i] == c) p += e.p[i];
                out[c] = E::narrow(gt * (power(E::wide(row.p[c]), base, c2) / sum - p));
            }
    }
};

template <dt_dtype XT, int G, int MODE>
__global__ void __launch_bounds__(Group<G>::kThreads) distill_rows(DistillArgs a) {
    using Gr = Group<G>;
    constexpr int kEntries = G == 8 ? kLaneClasses : DS_MAX_TOP;
    __shared__ int cls[Gr::kInBlock][kEntries];
    __shared__ float p[Gr::kInBlock][kEntries];
    __shared__ float box[G > 64 ? G / 64 : 1];
    const int which = G <= 64 ? int(threadIdx.x) / G : 0;
    const Gr g{G <= 64 ? int(threadIdx.x) % G : int(threadIdx.x), box};
    const Entries e{cls[which], p[which]};
    const float c2 = kLog2E / a.temperature;
    for (int64_t r = int64_t(blockIdx.x) * Gr::kInBlock + which; r < a.in.n;
         r += int64_t(gridDim.x) * Gr::kInBlock) {
        const Row<XT> row(a.in.x, r, a.in.ld, a.in.classes);
        Stats st;
        if constexpr (MODE == kGradOnly) {
            const float2 v = a.stats[r];
            st.m = v.x;
            st.s = v.y;
        } else {
            row.template walk<4>(
                0, row.vecs, g.thread, G, [&](const u32x4 &v, int) { st.add(row, v, c2); },
                [&](auto x, int) { st.add(Elem<XT>::wide(x), c2); });
            st.join(g, c2);
            if (g.thread == 0) a.stats[r] = float2{st.m, st.s};
        }
        float loss = 0.0f;
        const bool taught = teach<XT, MODE>(a, g, G, r, row, st, e, &loss);
        if (MODE != kGradOnly && g.thread == 0) a.loss[r] = loss;
        if constexpr (MODE != kLossOnly) {
            const int per = MODE == kGradOnly ? (row.vecs + a.parts - 1) / a.parts : row.vecs;
            const int lo = MODE == kGradOnly ? int(blockIdx.y) * per : 0;
            const int hi = lo + per < row.vecs ? lo + per : row.vecs;
            if (lo < hi) {
                const Gradient<XT> grad(a, r, row, st, taught);
                row.template walk<2>(
                    lo, hi, g.thread, G, [&](const u32x4 &v4, int v) { grad.vector(v4, v); },
                    [&](auto x, int c) { grad.single(x, c); });
                grad.teacher(a, g, G, lo, hi, e);
            }
        }
        g.sync();
    }
}

// Loss and gradient of rows of at most kHeld vectors a thread, which stay in registers between the
// two: the row crosses the memory once (the second walk of distill_rows finds little of a long
// row in the caches, which all rows in flight share).  1,000 x 50,001 fp16: 56 us = 3.5 TB/s of a row's
// bytes in and out, 64 us with two walks; what bounds it is the memory, and the teacher's part of
// each row, during which its wavefronts load nothing.
constexpr int kHeld = 16;

template <dt_dtype XT, int G>
__global__ void __launch_bounds__(G, 4) distill_held(DistillArgs a) {
    __shared__ int cls[DS_MAX_TOP];
    __shared__ float p[DS_MAX_TOP];
    __shared__ float box[G / 64];
    const Group<G> g{int(threadIdx.x), box};
    const Entries e{cls, p};
    const float c2 = kLog2E / a.temperature;
    for (int64_t r = blockIdx.x; r < a.in.n; r += gridDim.x) {
        const Row<XT> row(a.in.x, r, a.in.ld, a.in.classes);
        u32x4 held[kHeld];
        Stats st;
        // the whole vectors' places; opaque at each use, else all are kept in registers
        const int lo = row.inner_lo(), hi = row.inner_hi();
        auto place = [&](int i) {
            int thread = g.thread;
            asm volatile("" : "+v"(thread));
            return lo + thread + i * G;
        };
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int v = place(i);
            held[i] = row.load_whole(v < hi ? v : lo);       // in any case a place in the row
        }
        row.ends(g.thread, [&](auto x, int) { st.add(Elem<XT>::wide(x), c2); });
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            if (place(i) < hi) st.add(row, held[i], c2);
        }
        st.join(g, c2);
        if (g.thread == 0) a.stats[r] = float2{st.m, st.s};
        float loss = 0.0f;
        const bool taught = teach<XT, kBoth>(a, g, G, r, row, st, e, &loss);
        if (g.thread == 0) a.loss[r] = loss;
        const Gradient<XT> grad(a, r, row, st, taught);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int v = place(i);
            if (v < hi) grad.vector(held[i], v);
        }
        row.ends(g.thread, [&](auto x, int c) { grad.single(x, c); });
        grad.teacher(a, g, G, 0, row.vecs, e);
        g.sync();
    }
}

template <dt_dtype XT, int G>
void run_held(const DistillArgs &a, hipStream_t stream) {
    distill_held<XT, G><<<unsigned(a.in.n < 1048576 ? a.in.n : 1048576), G, 0, stream>>>(a);
}

// Long rows, few of them: a workgroup for each part of a row, and a wavefront to join them.
template <dt_dtype XT>
__global__ void __launch_bounds__(256) distill_part(DistillArgs a) {
    __shared__ float box[4];
    const Group<256> g{int(threadIdx.x), box};
    const float c2 = kLog2E / a.temperature;
    const Row<XT> row(a.in.x, blockIdx.x, a.in.ld, a.in.classes);
    const int per = (row.vecs + a.parts - 1) / a.parts;
    const int lo = int(blockIdx.y) * per < row.vecs ? int(blockIdx.y) * per : row.vecs;
    const int hi = lo + per < row.vecs ? lo + per : row.vecs;
    Stats st;
    if (lo < hi)
        row.template walk<4>(
            lo, hi, g.thread, 256, [&](const u32x4 &v, int) { st.add(row, v, c2); },
            [&](auto x, int) { st.add(Elem<XT>::wide(x), c2); });
    st.join(g, c2);
    if (g.thread == 0) a.part[int64_t(blockIdx.x) * a.parts + blockIdx.y] = float2{st.m, st.s};
}

template <dt_dtype XT>
__global__ void __launch_bounds__(64) distill_join(DistillArgs a) {
    __shared__ int cls[DS_MAX_TOP];
    __shared__ float p[DS_MAX_TOP];
    const Group<64> g{int(threadIdx.x), nullptr};
    const float c2 = kLog2E / a.temperature;
    const int64_t r = blockIdx.x;
    const Row<XT> row(a.in.x, r, a.in.ld, a.in.classes);
    Stats st;
    for (int i = g.thread; i < a.parts; i += 64) {
        const float2 v = a.part[r * a.parts + i];
        st.raise(v.x, c2);
        st.s += v.y * power(v.x, finite(st.m), c2);
    }
    st.join(g, c2);
    if (g.thread == 0) a.stats[r] = float2{st.m, st.s};
    float loss = 0.0f;
    teach<XT, kLossOnly>(a, g, 64, r, row, st, Entries{cls, p}, &loss);
    if (g.thread == 0) a.loss[r] = loss;
}

template <dt_dtype XT, int G, int MODE>
void run_rows(const DistillArgs &a, hipStream_t stream) {
    const int64_t blocks = (a.in.n + Group<G>::kInBlock - 1) / Group<G>::kInBlock;
    distill_rows<XT, G, MODE><<<dim3(unsigned(blocks < 1048576 ? blocks : 1048576), unsigned(a.parts)),
                                Group<G>::kThreads, 0, stream>>>(a);
}

// Rows for 8 lanes: few classes, and no more of the teacher's entries than they have room for
// (1,000,000 x 32 fp32, k = 4, one call: 83 us, 539 with a wavefront a row).
bool small(const DistillArgs &a) { return a.in.classes <= kLaneClasses && a.k <= kLaneClasses; }

// Rows for a wavefront: 30,000 x 2,048 bf16, k = 32, one call: 68 us, 236 with 256 threads a row; on
// longer ones the gain ends with the type (15,000 x 4,096 bf16 73 and 128, fp32 133 and 149, fp32's
// backward pass alone 106 and 97).
constexpr int kWaveClasses = 2048;

template <dt_dtype XT>
void run_backward(DistillArgs a, hipStream_t stream) {
    const int c = a.in.classes;
    a.parts = 1;
    if (small(a)) {
        run_rows<XT, 8, kGradOnly>(a, stream);
    } else if (c <= kWaveClasses) {
        run_rows<XT, 64, kGradOnly>(a, stream);
    } else {
        a.parts = distill_parts(a.in.n, c);
        run_rows<XT, 256, kGradOnly>(a, stream);
    }
}

template <dt_dtype XT>
void run(const DistillArgs &a, hipStream_t stream) {
    const int c = a.in.classes;
    if (a.parts > 1) {
        const dim3 grid(unsigned(a.in.n), unsigned(a.parts));
        distill_part<XT><<<grid, 256, 0, stream>>>(a);
        distill_join<XT><<<unsigned(a.in.n), 64, 0, stream>>>(a);
        if (a.g) run_backward<XT>(a, stream);
    } else if (small(a)) {
        if (a.g) run_rows<XT, 8, kBoth>(a, stream);
        else run_rows<XT, 8, kLossOnly>(a, stream);
    } else if (c <= kWaveClasses) {
        if (a.g) run_rows<XT, 64, kBoth>(a, stream);
        else run_rows<XT, 64, kLossOnly>(a, stream);
    } else if (!a.g) {
        run_rows<XT, 256, kLossOnly>(a, stream);
    } else {
        // one vector more than the row's elements need, for the place of its first one
        const int vecs = (c + Row<XT>::kVec - 1) / Row<XT>::kVec + 1;
        if (vecs <= 256 * kHeld) run_held<XT, 256>(a, stream);
        else if (vecs <= 512 * kHeld) run_held<XT, 512>(a, stream);
        else if (vecs <= 1024 * kHeld) run_held<XT, 1024>(a, stream);
        else run_rows<XT, 256, kBoth>(a, stream);
    }
}

}  // namespace

// Parts of a row: as many as fill the card with workgroups, of 4,096 classes at least.  They cost the loss
// a second launch and save the backward pass its time on few compute units: 100 x 32,768 bf16, k = 64,
// loss 15 us and backward 13, without parts 11 and 17; 256 x 131,072: 18 and 29, 18 and 40; 600 x
// 131,072: 31 and 59 both ways.  Loss and gradient in one call gain on the longest rows (256 x 131,072:
// 47 us, 56 without parts) and lose on others, which then stay in registers (500 x 50,000: 39 and 28).
// Parts of 2,048 to 16,384 classes, and 512 to 2,048 workgroups, take the same within 1 us (1 to 128
// rows of 131,072); of one row of 1,000,000 the backward pass takes 15.3 us with 32 parts at most, 12.6
// with 64 and 12.4 with 128.
int distill_parts(int64_t n, int32_t classes) {
    if (n >= 512 || classes <= 8192) return 1;
    const int64_t want = (1024 + n - 1) / n, most = classes / 4096;
    const int64_t parts = want < most ? want : most;
    return int(parts < 64 ? parts : 64);
}

hipError_t launch_distill(const DistillArgs &a, dt_dtype type, hipStream_t stream) {
    switch (type) {
        case DT_F32: run<DT_F32>(a, stream); break;
        case DT_F16: run<DT_F16>(a, stream); break;
        default: run<DT_BF16>(a, stream); break;
    }
    return hipGetLastError();
}

hipError_t launch_distill_backward(const DistillArgs &a, dt_dtype type, hipStream_t stream) {
    switch (type) {
        case DT_F32: run_backward<DT_F32>(a, stream); break;
        case DT_F16: run_backward<DT_F16>(a, stream); break;
        default: run_backward<DT_BF16>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace dscores
