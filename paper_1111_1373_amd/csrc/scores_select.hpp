// The best classes of a row, found by a team of wavefronts.
//
// A sort of a whole row would move every element many times; nearly all of them are far from
// the best k.  Every thread's largest key is known from the first pass over the row.  The k-th
// largest of these is a bound that k classes of the row reach, and few more do (of 1,024
// threads' shares and k = 64, about 66): a second pass collects those, and only they are put
// in order.
#pragma once

#include "scores_common.hpp"

namespace dscores {

constexpr int kCap = 1024;     // collected classes, in the LDS

struct Collected {
    uint64_t list[kCap];
    uint64_t best[DS_MAX_TOP];
    int count;
};

// Number of the team's threads that say yes.
template <int WAVES>
__device__ __forceinline__ int votes_of(const Team<WAVES> &t, bool yes) {
    const int c = __popcll(__ballot(yes));
    if constexpr (WAVES == 1) {
        return c;
    } else {
        int *b = reinterpret_cast<int *>(t.box);
        t.sync();
        if (t.lane == 0) b[t.wave] = c;
        t.sync();
        int s = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += b[w];
        return s;
    }
}

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
__device__ __forceinline__ void order_best(const Team<WAVES> &t, Collected &s, int c, int k) {
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

// s.best[0 .. result) = the row's k best classes, best first (fewer where fewer have a score).
// mine: the thread's largest key (over its share of the walk `each`), top: the row's (> 0).
// `also` is called once for each element.
template <dt_dtype XT, int WAVES, class Also>
__device__ __forceinline__ int best_of_row(const Team<WAVES> &t, const Row<XT> &row, int k, uint32_t mine,
                           uint32_t top, Collected &s, Also also) {
    // the bound: lo, where at least k threads' largest keys reach lo (or lo = 1, every score)
    uint32_t lo = 1, hi = top + 1;      // fewer than k reach hi (unless k = 1)
    if (k == 1) {
        lo = top;
    } else if (votes_of(t, mine > 0) >= k) {
        // any bound with about k above it will do
        while (hi - lo > 1) {
            const uint32_t mid = lo + ((hi - lo) >> 1);
            const int n = votes_of(t, mine >= mid);
            if (n < k) {
                hi = mid;
            } else {
                lo = mid;
                if (n <= k + (k >> 2) + 8) break;
            }
        }
    }
    if (t.thread == 0) s.count = 0;
    t.sync();
    row.template each<Row<XT>::kAhead>(0, row.vecs, t.thread, t.kThreads, [&](auto e, int c) {
        const uint32_t key = Elem<XT>::key(e);
        also(e, key);
        if (key >= lo) {
            const int at = atomicAdd(&s.count, 1);
            if (at < kCap) s.list[at] = comp(key, c);
        }
    });
    t.sync();
    int c = s.count;
    t.sync();                            // read by all before it is written again
    if (c > kCap) {
        // Too many equal (or few threads for many classes): the k-th best key itself, by
        // halving, and of the classes that have it the first ones.
        uint32_t kth = lo, over = top + 1;
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
