// The best classes of a row, found by a team of wavefronts.
//
// A sort of a whole row would move every element many times; nearly all of them are far from
// the best k.  The largest ranks of parts of the row give a bound: where k parts reach it, k
// classes do, and few more do (of 256 parts and k = 64, about 74).  A walk over the row then
// collects what reaches the bound, and only that is put in order.  The parts may cover a stretch of the
// row alone: with k of its parts' maxima above a bound, the whole row has about (row / stretch)
// times as many classes above it.  So the row is read once from memory, and its first stretch
// again from the cache.
#pragma once

#include "scores_common.hpp"

namespace dscores {

constexpr int kCap = 1024;     // collected classes, in the LDS

template <int WAVES>
struct Collected {
    uint64_t list[kCap];
    uint64_t best[DS_MAX_TOP];
    uint32_t maxima[64 * WAVES];
    int count;
};

// list[0 .. c) in descending order, in place: a bitonic network over the next power of two,
// whose places behind c hold 0 (smaller than any class that is collected).
template <int WAVES>
__device__ __forceinline__ void sort_list(const Team<WAVES> &t, uint64_t *list, int c) {
    int n = 64;
    while (n < c) n <<= 1;
    for (int i = c + t.thread; i < n; i += t.kThreads) list[i] = 0;
    t.sync();
    for (int size = 2; size <= n; size <<= 1)
        for (int d = size >> 1; d > 0; d >>= 1) {
            for (int i = t.thread; i < n >> 1; i += t.kThreads) {
                const int a = 2 * i - (i & (d - 1)), b = a + d;
                const uint64_t x = list[a], y = list[b];
                if ((x < y) == ((a & size) == 0)) {
                    list[a] = y;
                    list[b] = x;
                }
            }
            t.sync();
        }
}

// best[0 .. min(k, c)) = the largest of list[0 .. c), in descending order.  Few are ranked by
// counting the larger ones (every thread reads the whole list, all at the same address).
template <int WAVES>
__device__ __forceinline__ void order_best(const Team<WAVES> &t, Collected<WAVES> &s, int c, int k) {
    if (c <= 256) {
        for (int j = t.thread; j < c; j += t.kThreads) {
            const uint64_t mine = s.list[j];
            int rank = 0;
#pragma unroll 8
            for (int i = 0; i < c; ++i) rank += s.list[i] > mine;
            if (rank < k) s.best[rank] = mine;
        }
    } else {
        sort_list(t, s.list, c);
        for (int j = t.thread; j < k && j < c; j += t.kThreads) s.best[j] = s.list[j];
    }
    t.sync();
}

// The class of the q-th element (q >= 1, in the classes' order) whose key is `key`, at all of
// whose places `in` holds; every thread of the team gets it.
template <dt_dtype XT, int WAVES>
__device__ __forceinline__ int nth_equal(const Team<WAVES> &t, const Row<XT> &row, uint32_t key, int q, int *where) {
    int run = 0;
    for (int v0 = 0; v0 < row.vecs && run < q; v0 += t.kThreads) {
        const int v = v0 + t.thread;
        int n = 0;
        if (v < row.vecs)
            row.visit(row.load(v), v, [&](auto e, int) { n += Elem<XT>::key(e) == key; });
        int all;
        int at = run + t.before(n, &all);
        if (v < row.vecs && at < q && q <= at + n)
            row.visit(row.load(v), v, [&](auto e, int c) {
                if (Elem<XT>::key(e) == key && ++at == q) *where = c;
            });
        run += all;
    }
    t.sync();
    return *where;
}

// Classes of the row whose key is at least `least`.
template <dt_dtype XT, int WAVES>
__device__ __forceinline__ int count_from(const Team<WAVES> &t, const Row<XT> &row, uint32_t least) {
    int n = 0;
    row.template each<Row<XT>::kAhead>(0, row.vecs, t.thread, t.kThreads,
                         [&](auto e, int) { n += Elem<XT>::key(e) >= least; });
    return t.reduce(n, Sum());
}

// The largest rank that at least k of `parts` (<= 64 * PER) maxima in the LDS reach, or one that few
// more than k reach; at least `least`.  Every wavefront finds it by itself, with up to PER
// maxima a lane.
template <int PER>
__device__ __forceinline__ uint32_t bound_of(const uint32_t *maxima, int parts, int lane, int k,
                                             uint32_t least) {
    uint32_t v[PER];
    uint32_t lo = least, top = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = 64 * i < parts ? maxima[64 * i + lane] : 0u;      // parts is a multiple of 64
        top = v[i] > top ? v[i] : top;
    }
    uint32_t hi = wave_reduce(top, Max()) + 1;                   // none reaches hi
    auto reach = [&](uint32_t x) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (64 * i < parts) n += __popcll(__ballot(v[i] >= x));
        return n;
    };
    if (hi <= lo || reach(lo) < k) return lo;
    while (hi - lo > 1) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        const int n = reach(mid);
        if (n < k) {
            hi = mid;
        } else {
            lo = mid;
            if (n <= k + (k >> 3) + 4) break;
        }
    }
    return lo;
}

// s.best[0 .. result) = the row's k best classes, best first (fewer where fewer have a score).
// While it walks over the row, vector(a, v) is called for its vectors and single(e, c) for the
// elements before and behind them; `begin` before that, at each attempt, with the largest rank of
// the stretch.
template <dt_dtype XT, int WAVES, class FB, class FV, class FE>
__device__ __forceinline__ int best_of_row(const Team<WAVES> &t, const Row<XT> &row, int k,
                                           Collected<WAVES> &s, FB begin, FV vector, FE single) {
    using E = Elem<XT>;
    constexpr int kThreads = Team<WAVES>::kThreads;
    // so long a stretch that about 200 classes are collected, which are ordered quickly
    const int64_t want = int64_t(row.vecs) * (k + (k >> 2)) / 200;
    int stretch = want < row.vecs ? int(want) : row.vecs;
    stretch = (stretch + kThreads - 1) / kThreads * kThreads;
    if (stretch > row.vecs) stretch = row.vecs;
    // parts of the maxima: a thread each, or four threads where those are enough
    const bool four = kThreads >= 1024 && k <= 64;
    const int parts = four ? kThreads / 4 : kThreads;
    int c;
    for (;;) {
        typename Ranks<XT>::Max m;
        uint32_t single_max = 0;
        row.template walk<Row<XT>::kAhead>(
            0, stretch, t.thread, kThreads,
            [&](const u32x4 &a, int) { m.add(Ranks<XT>(a)); },
            [&](auto e, int) { single_max = Max()(single_max, E::rank(e)); });
        uint32_t mine = Max()(single_max, m.rank());
        if (four) {
            mine = Max()(mine, xor_lane(mine, 1));
            mine = Max()(mine, xor_lane(mine, 2));
            if ((t.lane & 3) == 0) s.maxima[t.thread >> 2] = mine;
        } else {
            s.maxima[t.thread] = mine;
        }
        if (t.thread == 0) s.count = 0;
        t.sync();
        const uint32_t lo = E::from_rank(bound_of<WAVES>(s.maxima, parts, t.lane, k, E::kNone + 1));
        if (lo == E::kNone + 1 && stretch < row.vecs) {      // a stretch with too few scores
            stretch = row.vecs;
            t.sync();
            continue;
        }
        begin(s.maxima, parts);
        const Filter<XT> filter(lo);
        auto collect = [&](uint32_t rank, int cls) {
            const int at = atomicAdd(&s.count, 1);
            if (at < kCap) s.list[at] = comp(E::key_of_rank(rank), cls);
        };
        row.template walk<Row<XT>::kAhead>(
            0, row.vecs, t.thread, kThreads,
            [&](const u32x4 &a, int v) {
                if (filter.any(a)) {
#pragma unroll
                    for (int i = 0; i < Row<XT>::kVec; ++i) {
                        const uint32_t r = E::rank(row.at(a, i));
                        if (r >= lo) collect(r, row.first(v) + i);
                    }
                }
                vector(a, v);
            },
            [&](auto e, int cls) {
                const uint32_t r = E::rank(e);
                if (r >= lo) collect(r, cls);
                single(e, cls);
            });
        t.sync();
        c = s.count;
        t.sync();                            // read by all before it is written again
        if (c <= kCap || stretch == row.vecs) break;
        stretch = row.vecs;
    }
    if (c > kCap) {
        // Too many equal (or few threads for many classes): the k-th best key itself, by
        // halving, and of the classes that have it the first ones.
        uint32_t kth = 1, over = 0;
        for (int i = t.lane; i < parts; i += 64) over = Max()(over, s.maxima[i]);
        over = E::key_of_rank(wave_reduce(over, Max())) + 1;     // the row's best, and one
        while (over - kth > 1) {
            const uint32_t mid = kth + ((over - kth) >> 1);
            if (count_from(t, row, mid) >= k)
                kth = mid;
            else
                over = mid;
        }
        if (t.thread == 0) s.count = 0;
        t.sync();
        row.template each<Row<XT>::kAhead>(0, row.vecs, t.thread, t.kThreads, [&](auto e, int cls) {
            const uint32_t key = Elem<XT>::key(e);
            if (key > kth) s.list[atomicAdd(&s.count, 1)] = comp(key, cls);   // fewer than k
        });
        t.sync();
        const int above = s.count;
        int run = above;
        for (int v0 = 0; v0 < row.vecs && run < k; v0 += t.kThreads) {
            const int v = v0 + t.thread;
            int n = 0;
            if (v < row.vecs)
                row.visit(row.load(v), v, [&](auto e, int) { n += Elem<XT>::key(e) == kth; });
            int all;
            int at = run + t.before(n, &all);
            if (n > 0)
                row.visit(row.load(v), v, [&](auto e, int cls) {
                    if (Elem<XT>::key(e) == kth) {
                        if (at < k) s.list[at] = comp(kth, cls);
                        ++at;
                    }
                });
            run += all;
        }
        t.sync();
        c = k;
    }
    order_best(t, s, c, k);
    return c < k ? c : k;
}

}  // namespace dscores
