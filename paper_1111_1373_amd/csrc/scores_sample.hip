// A class drawn from each row by temperature, top-k, top-p and min-p (ds_sample).
//
// Which class a given random number draws is decided by sums of weights, and so are the
// borders of top-p; with many classes the sums' rounding would decide it.  Weights are
// therefore computed in 64 bits and rounded once to whole multiples of 2^-42 of the largest
// one, and added as 64-bit integers (at most 2^20 of them): every order of summation gives the
// same sum, so the lanes, wavefronts and atomics that share a row cannot change a result.  It is
// fewer bits than a sum in fp64 has (53): a share or a random number within n 2^-41 of a border may
// fall on its other side.
#include "scores.hpp"
#include "scores_lanes.hpp"
#include "scores_select.hpp"

#include <type_traits>

namespace dscores {
namespace {

constexpr double kOne = 4398046511104.0;       // 2^42, the weight of a row's best class
constexpr float kNats = 30.0f;                 // e^-30 rounds to weight 0

// A row's settings, as numbers that mean something.
struct Settings {
    double inv;          // 1 / temperature; 0 for temperature 0
    int k;               // 1 .. n_classes
    double p;
    double min_p;
    bool counts;         // votes at temperature 1
};

template <dt_dtype XT>
__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int64_t row) {
    const float t = a.set.d_temperature ? a.set.d_temperature[row] : a.set.temperature;
    const int k = a.set.d_top_k ? a.set.d_top_k[row] : a.set.top_k;
    const float p = a.set.d_top_p ? a.set.d_top_p[row] : a.set.top_p;
    const float m = a.set.d_min_p ? a.set.d_min_p[row] : a.set.min_p;
    Settings s;
    s.inv = t > 0.0f ? 1.0 / double(t) : 0.0;
    s.k = !(t > 0.0f) ? 1 : (k < 1 || k > a.in.classes) ? a.in.classes : k;
    s.p = p < 1.0f ? double(p) : 1.0;                   // NaN: 1
    s.min_p = m > 0.0f ? double(m < 1.0f ? m : 1.0f) : 0.0;
    s.counts = XT == DT_U8 && t == 1.0f;
    return s;
}

// e^d for -30 <= d <= 0 as a whole multiple of 2^-42.  e^d = 2^n e^r with n the integer next to
// d / ln 2 and |r| <= ln 2 / 2; e^r by the polynomial of degree 9 through its values at the
// Chebyshev nodes of that range, at most 1.9e-14 off (2^-45).  Adding 2^52 leaves the rounded integer in the low
// bits.
__device__ __forceinline__ uint64_t exp_weight(double d) {
    const double n = __builtin_rint(d * 1.4426950408889634);
    const double r = fma(-n, 0.6931471805599453, d);
    double e = 2.7632640194122123e-06;
    e = fma(e, r, 2.488445975018801e-05);
    e = fma(e, r, 0.00019841190648950985);
    e = fma(e, r, 0.0013888801749663156);
    e = fma(e, r, 0.008333333367310203);
    e = fma(e, r, 0.04166666704055183);
    e = fma(e, r, 0.1666666666661565);
    e = fma(e, r, 0.4999999999943859);
    e = fma(e, r, 1.0000000000000013);
    e = fma(e, r, 1.0000000000000135);
    const double w = __builtin_amdgcn_ldexp(e, int(n) + 42) + 4503599627370496.0;
    return __builtin_bit_cast(uint64_t, w) & 0xFFFFFFFFFFFFFull;
}

// Weights of a row's classes, by their keys or as they are read (numbers of votes; scores widened to
// fp32, of which -inf and NaN have weight 0).
template <dt_dtype XT>
struct Weights {
    static constexpr bool kVotes = XT == DT_U8;
    using Read = typename std::conditional<kVotes, uint32_t, float>::type;
    uint32_t top;        // the best key
    Read best;
    double m, inv;       // its score, 1 / temperature
    bool counts;
    const double *ln;    // ln of 0 .. 255 (votes)

    static __device__ __forceinline__ Read read(typename Elem<XT>::Raw e) {
        if constexpr (kVotes)
            return e;
        else
            return Elem<XT>::wide(e);
    }
    template <int N>
    __device__ __forceinline__ Weights(const Settings &s, uint32_t top_key, const double (&ln_table)[N])
        : top(top_key), inv(s.inv), counts(s.counts), ln(ln_table) {
        static_assert(!kVotes || N == 256, "votes look up their logarithms");
        if constexpr (kVotes) {
            best = top;
            m = ln[top];
        } else {
            best = Elem<XT>::value(top);
            m = double(best);
        }
    }
    __device__ __forceinline__ double one() const {
        return counts ? double(top) * 17179869184.0 : kOne;          // 2^34 a vote
    }
    __device__ __forceinline__ uint64_t of(Read x) const {
        if (kVotes && counts) return uint64_t(x) << 34;
        double v;
        if constexpr (kVotes)
            v = ln[x];
        else
            v = double(x);
        const double d = x == best ? 0.0 : (v - m) * inv;            // of +inf too
        return d >= -double(kNats) ? exp_weight(d) : 0;
    }
    __device__ __forceinline__ uint64_t operator()(uint32_t key) const {
        if constexpr (kVotes)
            return of(key);
        else
            return key > 0 ? of(Elem<XT>::value(key)) : 0;
    }
    // the least weight that min_p leaves
    __device__ __forceinline__ uint64_t least(double min_p) const {
        return uint64_t(__builtin_ceil(min_p * one()));
    }
};

// Only as many classes stay as start below this sum of the better ones' weights; the sums are
// whole, so they are below p * sum iff they are below the next whole number.
__device__ __forceinline__ uint64_t share(double p, uint64_t sum) {
    if (p >= 1.0) return ~uint64_t(0);
    const double s = __builtin_ceil(p * double(sum));
    return s >= 1.0 ? uint64_t(s) : 1;                 // the best class always stays
}

// The class is the first whose running sum is larger than this.
__device__ __forceinline__ uint64_t target(float u, uint64_t sum) {
    const float most = 0.99999994f;                    // 1 - 2^-24
    u = u > 0.0f ? (u < most ? u : most) : 0.0f;       // NaN: 0
    return uint64_t(double(u) * double(sum));
}

__device__ __forceinline__ void fill_ln(double *ln) {
    for (int i = threadIdx.x; i < 256; i += blockDim.x) ln[i] = log(double(i));
    __syncthreads();
}

// ---- one lane a row ---------------------------------------------------------------------

// COUNTS: votes at temperature 1 in all rows; their numbers are the weights, and sums of 64 of them
// fit 32 bits (1,000,003 rows of 32 votes by top-p: 34 us, 41 us with 64-bit weights).
template <dt_dtype XT, int CP, bool COUNTS>
__global__ void __launch_bounds__(256) sample_lanes(SampleArgs a) {
    using O = Order<XT>;
    using Sum = typename std::conditional<COUNTS, uint32_t, uint64_t>::type;
    __shared__ double ln[XT == DT_U8 && !COUNTS ? 256 : 1];
    if constexpr (XT == DT_U8 && !COUNTS) fill_ln(ln);
    const int64_t row = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (row >= a.in.n) return;
    const int n = a.in.classes;
    typename Elem<XT>::Raw e[CP];
    load_row<XT, CP>(a.in.x, row, a.in.ld, n, a.in.align, e);
    const Settings set = settings_of<XT>(a, row);
    typename O::T v[CP], first = 0;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        v[i] = i < n ? O::make(Elem<XT>::key(e[i]), i) : 0;
        first = v[i] > first ? v[i] : first;
    }
    if (O::key(first) == 0) {
        a.labels[row] = -1;
        return;
    }
    const auto weights = [&] {
        if constexpr (COUNTS)
            return 0;                      // not needed
        else
            return Weights<XT>(set, O::key(first), ln);
    }();
    auto weight = [&](uint32_t key) -> Sum {
        if constexpr (COUNTS)
            return key;
        else
            return weights(key);
    };
    Sum least;
    if constexpr (COUNTS)
        least = Sum(__builtin_ceil(set.min_p * double(O::key(first))));
    else
        least = weights.least(set.min_p);
    typename O::T cut = 0;                 // classes from here on stay, in their order
    Sum sum = 0;
    if (set.k < n || set.p < 1.0) {
        sort_registers<CP>(v);
        Sum all = 0;
#pragma unroll
        for (int i = 0; i < CP; ++i)
            if (i < set.k) all += weight(O::key(v[i]));
        const uint64_t most = share(set.p, all);
        const Sum end = most > uint64_t(Sum(~Sum(0))) ? Sum(~Sum(0)) : Sum(most);
        Sum before = 0;
#pragma unroll
        for (int i = 0; i < CP; ++i)
            if (i < set.k && before < end) {
                const Sum w = weight(O::key(v[i]));
                cut = v[i];
                before += w;
                if (w >= least) sum += w;
            }
#pragma unroll
        for (int i = 0; i < CP; ++i) v[i] = i < n ? O::make(Elem<XT>::key(e[i]), i) : 0;
    } else {
#pragma unroll
        for (int i = 0; i < CP; ++i) {
            const Sum w = weight(O::key(v[i]));
            if (w >= least) sum += w;
        }
    }
    const Sum goal = Sum(target(a.u[row], sum));
    Sum upto = 0;
    int label = -1;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const Sum w = weight(O::key(v[i]));
        if (v[i] >= cut && w >= least) upto += w;
        if (label < 0 && upto > goal) label = i;
    }
    a.labels[row] = label;
}

template <dt_dtype XT, bool COUNTS>
void run_lanes(const SampleArgs &a, hipStream_t stream) {
    const unsigned blocks = unsigned((a.in.n + 255) / 256);
    const int c = a.in.classes;
    if (c <= 8) sample_lanes<XT, 8, COUNTS><<<blocks, 256, 0, stream>>>(a);
    else if (c <= 16) sample_lanes<XT, 16, COUNTS><<<blocks, 256, 0, stream>>>(a);
    else if (c <= 32) sample_lanes<XT, 32, COUNTS><<<blocks, 256, 0, stream>>>(a);
    else sample_lanes<XT, 64, COUNTS><<<blocks, 256, 0, stream>>>(a);
}

// ---- a team a row -----------------------------------------------------------------------

constexpr int bins_of(int waves) { return waves == 1 ? 256 : 1024; }

template <int WAVES>
struct FewSpace {
    Collected<WAVES> c;
    uint64_t weight[DS_MAX_TOP];
    int label, stay;
    uint64_t goal;
};

constexpr int kQueue = 128;      // keys that a wavefront collects before it weighs 64 of them

template <int WAVES>
struct WideSpace {
    uint64_t mass[bins_of(WAVES)];
    uint32_t number[bins_of(WAVES)];
    uint64_t list[kCap];
    uint32_t queue[WAVES][kQueue];
    uint64_t part[WAVES];
    int count;
    // answers that one thread finds and all read
    int bin, index;
    uint64_t found, before;
};

// A class's place on a scale of kNats / kBins steps below the best: the larger the score the
// lower the bin (each step of the computation keeps the order); kBins for weight 0.  The difference from
// the best is taken of scores times a power of two: 1, but 1/2 where it may pass the largest fp32
// number, and 2^64 where the temperature's reciprocal may, which then counts for small scores
// alone (others are either equal or at least 2^36 apart).
template <dt_dtype XT, int WAVES>
struct Scale {
    using W = Weights<XT>;
    const W &w;
    float unit, base, step;
    __device__ __forceinline__ explicit Scale(const W &weights) : w(weights), unit(1.0f) {
        if constexpr (!W::kVotes) {
            if (w.best >= 0x1p102f)
                unit = 0.5f;
            else if (w.inv > 0x1p100 && fabsf(w.best) < 0x1p60f)
                unit = 0x1p64f;
            base = w.best * unit;
        }
        step = float(w.inv * (bins_of(WAVES) / kNats) / unit);
    }
    __device__ __forceinline__ int bin(typename W::Read x) const {
        constexpr int n = bins_of(WAVES);
        float diff;
        if constexpr (W::kVotes)
            diff = float(w.m) - float(w.ln[x]);
        else
            diff = fmaf(x, -unit, base);
        const float d = x == w.best ? 0.0f : diff * step;
        return d < float(n) ? int(d) : n;                            // n for a NaN
    }
};

// Where the best-first order of a row ends: at the q-th class (BY_WEIGHT false) or at the class
// that makes the sum of weights reach q.  In: the histogram in s.  Out: comp() of the last
// class that stays, and in s.found the weight of all that stay (if not BY_WEIGHT).
template <bool BY_WEIGHT, dt_dtype XT, int WAVES>
__device__ __forceinline__ uint64_t end_of(const Team<WAVES> &t, const Row<XT> &row, const Weights<XT> &weight,
                           const Scale<XT, WAVES> &scale, uint64_t q, WideSpace<WAVES> &s) {
    constexpr int kBins = bins_of(WAVES), kEach = kBins / Team<WAVES>::kThreads;
    static_assert(kEach >= 1, "");
    // the bin in which it lies
    uint64_t w = 0, all_w;
    int n = 0, all_n;
    if (t.thread == 0) s.bin = -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        w += s.mass[t.thread * kEach + i];
        n += int(s.number[t.thread * kEach + i]);
    }
    uint64_t w0 = t.before(w, &all_w);
    int n0 = t.before(n, &all_n);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = t.thread * kEach + i;
        const uint64_t bw = s.mass[b];
        const int bn = int(s.number[b]);
        const bool here = BY_WEIGHT ? (w0 < q && q <= w0 + bw)
                                    : (uint64_t(n0) < q && q <= uint64_t(n0) + uint64_t(bn));
        if (here) {
            s.bin = b;
            s.before = w0;
            s.index = n0;
        }
        w0 += bw;
        n0 += bn;
    }
    t.sync();
    const int bin = s.bin;
    if (bin < 0) {                           // beyond every class with a weight
        if (t.thread == 0) s.found = all_w;
        t.sync();
        return 0;
    }
    const uint64_t before_w = s.before;
    const uint64_t rest = BY_WEIGHT ? q - before_w : q - uint64_t(s.index);
    if (t.thread == 0) s.count = 0;
    t.sync();
    row.template each<2>(0, row.vecs, t.thread, t.kThreads, [&](auto e, int c) {
        if (scale.bin(weight.read(e)) == bin) {
            const int at = atomicAdd(&s.count, 1);
            if (at < kCap) s.list[at] = comp(Elem<XT>::key(e), c);
        }
    });
    t.sync();
    const int members = s.count;
    if (members <= kCap) {
        sort_list(t, s.list, members);
        uint64_t run = 0;
        for (int i0 = 0; i0 < members; i0 += t.kThreads) {
            const int i = i0 + t.thread;
            const uint64_t wi = i < members ? weight(comp_key(s.list[i])) : 0;
            uint64_t all;
            const uint64_t b = run + t.before(wi, &all);
            const bool here = BY_WEIGHT ? (b < rest && rest <= b + wi) : uint64_t(i) + 1 == rest;
            if (i < members && here) {
                s.index = i;
                s.found = before_w + b + wi;
            }
            run += all;
        }
        t.sync();
        return s.list[s.index];
    }
    // Too many to collect: the key at which it lies, by halving, and the place among the
    // classes of that key.
    auto from = [&](uint32_t least, int *count) {
        uint64_t sum = 0;
        int k = 0;
        row.template each<1>(0, row.vecs, t.thread, t.kThreads, [&](auto e, int) {
            const uint32_t key = Elem<XT>::key(e);
            if (key >= least && scale.bin(weight.read(e)) == bin) {
                sum += weight(key);
                ++k;
            }
        });
        *count = t.reduce(k, Sum());
        return t.reduce(sum, Sum());
    };
    // from(lo) >= rest > from(hi), modulo 2^32: the largest key of fp32, +inf, is 2^32 - 1
    uint32_t lo = 1, hi = weight.top + 1;
    int count;
    while (hi - lo > 1) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        const uint64_t sum = from(mid, &count);
        if ((BY_WEIGHT ? sum : uint64_t(count)) >= rest)
            lo = mid;
        else
            hi = mid;
    }
    const uint64_t above = hi - 1 == weight.top ? (count = 0, uint64_t(0)) : from(hi, &count);
    const uint64_t one = weight(lo);
    const uint64_t nth = BY_WEIGHT ? (rest - above + one - 1) / one : rest - uint64_t(count);
    const int c = nth_equal<XT>(t, row, lo, int(nth), &s.index);
    t.sync();
    if (t.thread == 0) s.found = before_w + above + nth * one;
    t.sync();
    return comp(lo, c);
}

// The drawn class among s.c.best[0 .. k), which are in order.
template <dt_dtype XT, int WAVES>
__device__ __forceinline__ int draw_of_few(const Team<WAVES> &t, const Weights<XT> &weight, const Settings &set,
                           int k, float u, FewSpace<WAVES> &s) {
    for (int j = t.thread; j < DS_MAX_TOP; j += t.kThreads)
        s.weight[j] = j < k ? weight(comp_key(s.c.best[j])) : 0;
    t.sync();
    if (t.wave == 0) {
        constexpr int kEach = DS_MAX_TOP / 64;
        uint64_t w[kEach], mine = 0, all;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            w[i] = s.weight[t.lane * kEach + i];
            mine += w[i];
        }
        uint64_t before = wave_before(mine, t.lane, &all);
        const uint64_t end = share(set.p, all), least = weight.least(set.min_p);
        int stay = 0;
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = t.lane * kEach + i;
            if (j < k && before < end && w[i] >= least) {
                ++stay;                      // they are the first ones: both limits are ordered
                sum += w[i];
            }
            before += w[i];
        }
        stay = wave_reduce(stay, Sum());
        sum = wave_reduce(sum, Sum());
        if (t.lane == 0) {
            s.stay = stay;
            s.goal = target(u, sum);
        }
    }
    t.sync();
    const int stay = s.stay;
    const uint64_t goal = s.goal;
    for (int j = t.thread; j < stay; j += t.kThreads) {
        const int c = comp_class(s.c.best[j]);
        uint64_t upto = 0;
#pragma unroll 8
        for (int i = 0; i < stay; ++i)
            upto += comp_class(s.c.best[i]) <= c ? s.weight[i] : 0;
        if (upto > goal && upto - s.weight[j] <= goal) s.label = c;
    }
    t.sync();
    return s.label;
}

// The drawn class among all that stay: those from `cut` on, of weight `least` or more.
template <dt_dtype XT, int WAVES>
__device__ __forceinline__ int draw_of_row(const Team<WAVES> &t, const Row<XT> &row,
                                           const Weights<XT> &weight, uint64_t cut, uint64_t least,
                                           float u, WideSpace<WAVES> &s) {
    using E = Elem<XT>;
    // the last class that stays, by its score and its place; none: all stay
    using Read = typename Weights<XT>::Read;
    Read last = Read(0);
    if constexpr (Weights<XT>::kVotes)
        last = comp_key(cut);
    else
        last = cut == 0 ? -__builtin_inff() : E::value(comp_key(cut));
    const int last_class = cut == 0 ? row.n : comp_class(cut);
    auto within = [&](Read x, int c) { return x > last || (x == last && c <= last_class); };
    auto staying = [&](auto e, int c) {
        const Read x = weight.read(e);
        const uint64_t w = within(x, c) ? weight.of(x) : uint64_t(0);
        return w >= least ? w : uint64_t(0);
    };
    // each wavefront sums a stretch of the row
    const int per = (row.vecs + WAVES - 1) / WAVES;
    auto start = [&](int w) { return w * per < row.vecs ? w * per : row.vecs; };
    const int from = start(t.wave), to = start(t.wave + 1);
    uint64_t sum = 0;
    if (cut == 0) {
        row.template each<1>(from, to, t.lane, 64, [&](auto e, int c) { sum += staying(e, c); });
    } else {
        // Few stay: their keys are queued, and weighed 64 at a time.
        Read *queue = reinterpret_cast<Read *>(s.queue[t.wave]);
        int n = 0;                                           // the same in all lanes
        auto weigh = [&](Read x) {
            const uint64_t w = weight.of(x);
            sum += w >= least ? w : uint64_t(0);
        };
        for (int v0 = from; v0 < to; v0 += 64) {
            const int v = v0 + t.lane;
            const u32x4 a = v < to ? row.load(v) : u32x4{0u, 0u, 0u, 0u};
            const bool whole = v0 > row.inner_lo() && v0 + 64 <= row.inner_hi();
#pragma unroll
            for (int i = 0; i < Row<XT>::kVec; ++i) {
                const int c = row.first(v) + i;
                const Read x = weight.read(row.at(a, i));
                const bool yes = within(x, c) && v < to && (whole || row.has(c));
                const uint64_t mask = __ballot(yes);
                if (mask == 0) continue;
                if (yes) queue[n + __popcll(mask & ((uint64_t(1) << t.lane) - 1))] = x;
                n += __popcll(mask);
                if (n >= 64) {
                    wave_fence();
                    weigh(queue[t.lane]);
                    const Read next = queue[64 + t.lane];
                    wave_fence();
                    n -= 64;
                    if (t.lane < n) queue[t.lane] = next;
                }
            }
        }
        wave_fence();
        if (t.lane < n) weigh(queue[t.lane]);
    }
    sum = wave_reduce(sum, Sum());
    uint64_t all = 0;
    if (t.lane == 0) s.part[t.wave] = sum;
    t.sync();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += s.part[w];
    const uint64_t goal = target(u, all);
    // the stretch, then the vector, then the class at which the sum passes the goal
    uint64_t run = 0;
    int which = 0;
    while (which < WAVES - 1 && run + s.part[which] <= goal) run += s.part[which++];
    const int hi = start(which + 1);
    for (int v0 = start(which); v0 < hi && run <= goal; v0 += t.kThreads) {
        const int v = v0 + t.thread;
        u32x4 a = {0u, 0u, 0u, 0u};
        uint64_t mine = 0, tile;
        if (v < hi) {
            a = row.load(v);
            row.visit(a, v, [&](auto e, int c) { mine += staying(e, c); });
        }
        uint64_t upto = run + t.before(mine, &tile);
        if (upto <= goal && goal < upto + mine)
            row.visit(a, v, [&](auto e, int c) {
                const uint64_t w = staying(e, c);
                if (upto <= goal && goal < upto + w) s.bin = c;
                upto += w;
            });
        run += tile;
    }
    t.sync();
    return s.bin;
}

// Rows of which only few classes stay (FEW: top_k <= 256, or temperature 0), or the others.
__device__ __forceinline__ bool few_stay(const Settings &s, int n) { return s.k <= DS_MAX_TOP && s.k < n; }

template <dt_dtype XT, int WAVES>
__global__ void __launch_bounds__(WAVES == 1 ? 128 : 64 * WAVES, WAVES >= 4 ? 4 : 2)
sample_few(SampleArgs a) {
    if constexpr (XT != DT_U8) quiet_max();
    constexpr int kTeams = WAVES == 1 ? 2 : 1;              // of a workgroup
    __shared__ FewSpace<WAVES> space[kTeams];
    __shared__ uint64_t box[WAVES];
    __shared__ double ln[XT == DT_U8 ? 256 : 1];
    if constexpr (XT == DT_U8) fill_ln(ln);
    const int which = WAVES == 1 ? __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)) : 0;
    const int thread = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const Team<WAVES> t{thread, thread & 63, thread >> 6, box};
    FewSpace<WAVES> &s = space[which];
    const int n = a.in.classes;
    for (int64_t r = int64_t(blockIdx.x) * kTeams + which; r < a.in.n;
         r += int64_t(gridDim.x) * kTeams) {
        const Settings set = settings_of<XT>(a, r);
        if (!few_stay(set, n)) continue;
        const Row<XT> row(a.in.x, r, a.in.ld, n);
        int label = -1;
        const int k = best_of_row<XT>(t, row, set.k, s.c, [](const uint32_t *, int) {},
                                      [](const u32x4 &) {}, [](auto) {});
        if (k > 0) {
            const Weights<XT> weight(set, comp_key(s.c.best[0]), ln);
            label = draw_of_few(t, weight, set, k, a.u[r], s);
        }
        if (t.thread == 0) a.labels[r] = label;
        t.sync();
    }
}

template <dt_dtype XT, int WAVES>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, WAVES >= 4 ? 4 : 2)
sample_wide(SampleArgs a) {
    constexpr int kTeams = WAVES == 1 ? 4 : 1;              // of a workgroup
    __shared__ WideSpace<WAVES> space[kTeams];
    __shared__ uint64_t box[WAVES];
    __shared__ double ln[XT == DT_U8 ? 256 : 1];
    if constexpr (XT == DT_U8) fill_ln(ln);
    const int which = WAVES == 1 ? __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)) : 0;
    const int thread = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const Team<WAVES> t{thread, thread & 63, thread >> 6, box};
    WideSpace<WAVES> &s = space[which];
    const int n = a.in.classes;
    for (int64_t r = int64_t(blockIdx.x) * kTeams + which; r < a.in.n;
         r += int64_t(gridDim.x) * kTeams) {
        const Settings set = settings_of<XT>(a, r);
        if (few_stay(set, n)) continue;
        const Row<XT> row(a.in.x, r, a.in.ld, n);
        typename Ranks<XT>::Max m;
        uint32_t single = 0;
        row.template walk<Row<XT>::kAhead>(
            0, row.vecs, t.thread, t.kThreads,
            [&](const u32x4 &v4, int) { m.add(Ranks<XT>(v4)); },
            [&](auto e, int) { single = Max()(single, Elem<XT>::rank(e)); });
        const uint32_t top = Elem<XT>::key_of_rank(t.reduce(Max()(single, m.rank()), Max()));
        int label = -1;
        if (top > 0) {
            const Weights<XT> weight(set, top, ln);
            uint64_t cut = 0;
            if (set.k < n || set.p < 1.0) {
                const Scale<XT, WAVES> scale(weight);
                constexpr int kBins = bins_of(WAVES);
                for (int b = t.thread; b < kBins; b += t.kThreads) {
                    s.mass[b] = 0;
                    s.number[b] = 0;
                }
                t.sync();
                const bool counted = set.k < n;
                row.template each<1>(0, row.vecs, t.thread, t.kThreads, [&](auto e, int) {
                    const auto x = weight.read(e);
                    const int b = scale.bin(x);
                    const uint64_t w = weight.of(x);
                    if (b < kBins) {
                        atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[b]),
                                  static_cast<unsigned long long>(w));
                        if (counted) atomicAdd(&s.number[b], 1u);
                    }
                });
                t.sync();
                // by number first: of the rest's weight, top-p's share
                cut = end_of<false, XT, WAVES>(
                    t, row, weight, scale, counted ? uint64_t(set.k) : ~uint64_t(0), s);
                const uint64_t all = s.found;
                t.sync();
                if (set.p < 1.0)
                    cut = end_of<true, XT, WAVES>(t, row, weight, scale, share(set.p, all), s);
            }
            label = draw_of_row(t, row, weight, cut, weight.least(set.min_p), a.u[r], s);
        }
        if (t.thread == 0) a.labels[r] = label;
        t.sync();
    }
}

// Settings that only the device sees may ask for either kind of row: then both kernels run, and
// each passes over the other's rows.
// A team of 4 wavefronts finds no good bound for many classes, or for a number that only the
// device knows: one of 8 does.
template <dt_dtype XT, int WAVES>
void run_teams(const SampleArgs &a, hipStream_t stream) {
    constexpr int kFewWaves = WAVES == 4 ? 8 : WAVES == 1 ? 4 : WAVES;
    const bool one = !a.set.d_temperature && a.set.temperature == 0.0f;
    const bool few = one || (!a.set.d_top_k && a.set.top_k >= 1 && a.set.top_k <= DS_MAX_TOP &&
                             a.set.top_k < a.in.classes);        // as few_stay says of a row
    const bool wide = !few && !a.set.d_top_k && !a.set.d_temperature;
    auto blocks = [&](int teams) {
        const int64_t b = (a.in.n + teams - 1) / teams;
        return unsigned(b < 65536 ? b : 65536);
    };
    constexpr int kMost = WAVES == 1 ? kSixteenth : kQuarter;
    const bool quarter = one || (!a.set.d_top_k && a.set.top_k <= kMost);
    if (!wide && quarter)
        sample_few<XT, WAVES><<<blocks(WAVES == 1 ? 2 : 1), WAVES == 1 ? 128 : 64 * WAVES, 0, stream>>>(a);
    else if (!wide)
        sample_few<XT, kFewWaves><<<blocks(1), 64 * kFewWaves, 0, stream>>>(a);
    if (!few)
        sample_wide<XT, WAVES><<<blocks(WAVES == 1 ? 4 : 1), WAVES == 1 ? 256 : 64 * WAVES, 0, stream>>>(a);
}

template <dt_dtype XT>
void run(const SampleArgs &a, hipStream_t stream) {
    const int c = a.in.classes;
    if (c <= kLaneClasses) {
        if (XT == DT_U8 && !a.set.d_temperature && a.set.temperature == 1.0f)
            run_lanes<XT, XT == DT_U8>(a, stream);
        else
            run_lanes<XT, false>(a, stream);
    } else if (c <= kCap) {
        run_teams<XT, 1>(a, stream);       // everything can be collected
    } else if (c <= 8192 || a.in.n > kFewRows) {
        run_teams<XT, 4>(a, stream);
    } else {
        run_teams<XT, 16>(a, stream);
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, dt_dtype type, hipStream_t stream) {
    switch (type) {
        case DT_F32: run<DT_F32>(a, stream); break;
        case DT_F16: run<DT_F16>(a, stream); break;
        case DT_BF16: run<DT_BF16>(a, stream); break;
        case DT_U8: run<DT_U8>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace dscores
