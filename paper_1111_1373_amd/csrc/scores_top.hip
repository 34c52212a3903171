// The k best classes of each row and the row's log-sum-exp (ds_top_scores).
#include "scores.hpp"
#include "scores_lanes.hpp"
#include "scores_select.hpp"

namespace dscores {
namespace {

template <dt_dtype XT>
__device__ __forceinline__ float log_sum(uint32_t top, float sum) {
    if (top == 0) return -__builtin_inff();
    if constexpr (XT == DT_U8) return logf(sum);           // ln of the votes
    return Elem<XT>::value(top) + logf(sum);
}

// One lane a row.
template <dt_dtype XT, int CP>
__global__ void __launch_bounds__(256) top_lanes(TopArgs a) {
    using O = Order<XT>;
    const int64_t row = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (row >= a.in.n) return;
    typename Elem<XT>::Raw e[CP];
    load_row<XT, CP>(a.in.x, row, a.in.ld, a.in.classes, a.in.align, e);
    typename O::T v[CP];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const uint32_t key = i < a.in.classes ? Elem<XT>::key(e[i]) : 0u;
        top = key > top ? key : top;
        v[i] = i < a.in.classes ? O::make(key, i) : 0;
    }
    const float m = Elem<XT>::value(top);
    // (eight running sums: in one, 64 equal terms that round the same way added up to 30 half steps)
    float part[8] = {};
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const uint32_t key = O::key(v[i]);
        if constexpr (XT == DT_U8)
            part[i & 7] += float(key);
        else if (key > 0)
            part[i & 7] += key == top ? 1.0f : exp_neg(Elem<XT>::value(key) - m);
    }
    const float sum = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
    a.lse[row] = log_sum<XT>(top, sum);
    sort_registers<CP>(v);
    float *values = a.values + row * a.k;
    int32_t *index = a.index + row * a.k;
#pragma unroll
    for (int i = 0; i < CP; ++i)
        if (i < a.k) {
            const uint32_t key = O::key(v[i]);
            values[i] = key > 0 ? Elem<XT>::value(key) : -__builtin_inff();
            index[i] = key > 0 ? O::cls(v[i]) : -1;
        }
}

// e^(x - m) = 2^(x log2 e - m log2 e), whose second product is the same for the whole row.  So is its
// rounding error, up to 0.7 steps of m in the sum's logarithm, which log() puts back.
struct Exponent {
    float base, shift;     // m, -m log2 e
    __device__ __forceinline__ void set(float m) {
        base = m;
        shift = -m * 1.44269504f;
    }
    __device__ __forceinline__ float operator()(float x) const {
        return __builtin_amdgcn_exp2f(fmaf(x, 1.44269504f, shift));
    }
    // of a sum of terms, with e^m
    __device__ __forceinline__ float log(float sum) const {
        return base + fmaf(fmaf(-base, 1.44269504f, -shift), 0.693147181f, logf(sum));
    }
};

// A team a row.
template <dt_dtype XT, int WAVES>
__global__ void __launch_bounds__(WAVES == 1 ? 128 : 64 * WAVES, WAVES >= 4 ? 4 : 2) top_teams(TopArgs a) {
    if constexpr (XT != DT_U8) quiet_max();
    constexpr int kTeams = WAVES == 1 ? 2 : 1;              // of a workgroup
    using E = Elem<XT>;
    __shared__ Collected<WAVES> space[kTeams];
    __shared__ uint64_t box[WAVES];
    const int which = WAVES == 1 ? __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)) : 0;
    const int thread = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const Team<WAVES> t{thread, thread & 63, thread >> 6, box};
    Collected<WAVES> &s = space[which];
    for (int64_t r = int64_t(blockIdx.x) * kTeams + which; r < a.in.n;
         r += int64_t(gridDim.x) * kTeams) {
        const Row<XT> row(a.in.x, r, a.in.ld, a.in.classes);
        // the sum is taken relative to the best of the stretch that is looked at first
        Exponent ex;
        float sum = 0.0f;
        uint32_t votes = 0;
        const int found = best_of_row<XT>(
            t, row, a.k, s,
            [&](const uint32_t *maxima, int parts) {
                uint32_t m = 0;
                for (int i = t.lane; i < parts; i += 64) m = Max()(m, maxima[i]);
                m = E::key_of_rank(wave_reduce(m, Max()));
                ex.set(m > 0 ? E::value(m) : 0.0f);
                sum = 0.0f;
                votes = 0;
            },
            [&](const u32x4 &v4) {
                if constexpr (XT == DT_U8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) votes = __builtin_amdgcn_sad_u8(v4[i], 0u, votes);
                } else {
#pragma unroll
                    for (int i = 0; i < Row<XT>::kVec; ++i) sum += ex(E::wide(row.at(v4, i)));
                }
            },
            [&](auto x) {
                if constexpr (XT == DT_U8)
                    votes += x;
                else
                    sum += ex(E::wide(x));
            });
        const uint32_t top = found > 0 ? comp_key(s.best[0]) : 0u;
        float lse = -__builtin_inff();
        if (top > 0) {
            if constexpr (XT == DT_U8) {
                lse = logf(float(t.reduce(votes, Sum())));
            } else {
                const float best = E::value(top);
                sum = t.reduce(sum, Sum());
                if (best == __builtin_inff()) {
                    lse = best;
                } else if (sum < 1e30f && fabsf(ex.base) <= 1e6f) {
                    lse = ex.log(sum);
                } else {
                    // The best is far above the stretch that the sum is relative to, or so large
                    // that the rounding of m log2 e is, or there is a NaN: again, term by term.
                    sum = 0.0f;
                    row.template each<1>(0, row.vecs, t.thread, t.kThreads, [&](auto x, int) {
                        const float e = exp_neg(E::wide(x) - best);
                        sum += e >= 0.0f ? e : 0.0f;
                    });
                    lse = best + logf(t.reduce(sum, Sum()));
                }
            }
        }
        if (t.thread == 0) a.lse[r] = lse;
        for (int j = t.thread; j < a.k; j += t.kThreads) {
            const uint32_t key = j < found ? comp_key(s.best[j]) : 0u;
            a.values[r * a.k + j] = key > 0 ? E::value(key) : -__builtin_inff();
            a.index[r * a.k + j] = key > 0 ? comp_class(s.best[j]) : -1;
        }
        t.sync();
    }
}

template <dt_dtype XT, int WAVES>
void run_teams(const TopArgs &a, hipStream_t stream) {
    constexpr int kTeams = WAVES == 1 ? 2 : 1;
    const int64_t blocks = (a.in.n + kTeams - 1) / kTeams;
    top_teams<XT, WAVES><<<unsigned(blocks < 65536 ? blocks : 65536), WAVES == 1 ? 128 : 64 * WAVES, 0,
                           stream>>>(a);
}

template <dt_dtype XT>
void run(const TopArgs &a, hipStream_t stream) {
    const int c = a.in.classes;
    if (c <= kLaneClasses) {
        const unsigned blocks = unsigned((a.in.n + 255) / 256);
        if (c <= 8) top_lanes<XT, 8><<<blocks, 256, 0, stream>>>(a);
        else if (c <= 16) top_lanes<XT, 16><<<blocks, 256, 0, stream>>>(a);
        else if (c <= 32) top_lanes<XT, 32><<<blocks, 256, 0, stream>>>(a);
        else top_lanes<XT, 64><<<blocks, 256, 0, stream>>>(a);
    } else if (c <= kCap && a.k <= kSixteenth) {
        run_teams<XT, 1>(a, stream);
    } else if (c <= kCap || (a.k <= kQuarter && (c <= 8192 || a.in.n >= kManyRows))) {
        run_teams<XT, 4>(a, stream);
    } else if (a.in.n > kFewRows) {
        run_teams<XT, 8>(a, stream);
    } else {
        run_teams<XT, 16>(a, stream);
    }
}

}  // namespace

hipError_t launch_top(const TopArgs &a, dt_dtype type, hipStream_t stream) {
    switch (type) {
        case DT_F32: run<DT_F32>(a, stream); break;
        case DT_F16: run<DT_F16>(a, stream); break;
        case DT_BF16: run<DT_BF16>(a, stream); break;
        case DT_U8: run<DT_U8>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace dscores
