// The best classes of a row, found by a team of wavefronts.
//
// A sort of a whole row would move every element many times; nearly all of them are far from
// the best k.  The largest ranks of parts of the row give a bound: where k parts reach it, k
// classes do, and few more do (of 256 parts and k = 64, about 74).  A second walk collects what
// reaches the bound, and only that is put in order.  The parts may cover a stretch of the row alone:
// with k of its maxima above a bound, the whole row has about (row / stretch) times as many
// classes above it.  The stretch stays in the LDS as far as it fits and is read again beyond that: of
// 131,072 bf16 with k = 64 a team of 4 wavefronts looks at 4,369 vectors first and keeps 1,280,
// so 1.2 times the row crosses the memory.  2,048 such rows with their log-sum-exp: 118 us =
// 4.6 TB/s of the rows' bytes (a read alone reaches 6.9); of a row's 52 us with three others on its
// compute unit, 44 are the two walks, bound by loads and by the exponentials' instructions, and 6
// finding the bounds and collecting.
#pragma once

#include "scores_common.hpp"

namespace dscores {

constexpr int kCap = 1024;     // collected classes, in the LDS
constexpr int kSpill = 256;    // queued vectors that a wavefront has no room for

// Vectors of a row's first stretch that are kept in the LDS between the two walks (a compute unit has
// 160 KiB: one team of 16 wavefronts, two of 8), and vectors that a wavefront can queue.
template <int WAVES>
constexpr int kHeldVecs = WAVES == 1 ? 512 : WAVES == 4 ? 1280 : WAVES == 8 ? 3584 : 6144;
template <int WAVES>
constexpr int kShare = WAVES == 1 ? 128 : 64;

// Entries of the list that fewer candidates go to, in the place of the queue, half a vector each:
// sort_list takes the next power of two, and a list has at most kCap.
constexpr int power_of_two_below(int n) {
    int p = 64;
    while (2 * p <= n && 2 * p <= kCap) p *= 2;
    return p;
}
template <int WAVES>
constexpr int kFewerRoom = power_of_two_below(2 * (WAVES * kShare<WAVES> + kSpill));

template <int WAVES>
struct Collected {
    union {
        u32x4 held[kHeldVecs<WAVES>];
        uint64_t list[kCap];   // sorted or ranked, once the walks are over
    };
    uint64_t best[DS_MAX_TOP];
    u32x4 queue[WAVES * kShare<WAVES> + kSpill];     // each wavefront's, then the others
    int place[WAVES * kShare<WAVES> + kSpill];
    uint32_t maxima[64 * WAVES];
    int counts[WAVES];
    int spilt, count;
    uint32_t bound;
};

// list[0 .. c) in descending order, in place: a bitonic network over the next power of two (at
// least 64), for which the list has room, and whose places behind c hold 0 (smaller than any
// class that is collected).
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
// counting the larger ones, with as many neighbouring lanes to one entry as the team has.
template <int LANES, int WAVES>
__device__ __forceinline__ void rank_list(const Team<WAVES> &t, const uint64_t *list, uint64_t *best,
                                          int c, int k) {
    const int part = t.thread & (LANES - 1);
    for (int j0 = 0; j0 < c; j0 += t.kThreads / LANES) {
        const int j = j0 + t.thread / LANES;
        const uint64_t mine = j < c ? list[j] : 0;
        int rank = 0;
#pragma unroll 8
        for (int i = part; i < c; i += LANES) rank += list[i] > mine;
        rank = wave_reduce<LANES>(rank, Sum());
        if (part == 0 && j < c && rank < k) best[rank] = mine;
    }
}

template <int WAVES>
__device__ __forceinline__ void order_best(const Team<WAVES> &t, uint64_t *list, uint64_t *best, int c,
                                           int k) {
    if (8 * c <= t.kThreads) {
        rank_list<8>(t, list, best, c, k);
    } else if (4 * c <= t.kThreads) {
        rank_list<4>(t, list, best, c, k);
    } else if (2 * c <= t.kThreads || c <= 128) {
        rank_list<2>(t, list, best, c, k);
    } else {
        sort_list(t, list, c);
        for (int j = t.thread; j < k && j < c; j += t.kThreads) best[j] = list[j];
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
// more than k reach; at least `least`.  For one wavefront, with up to PER maxima a lane.
template <int PER>
__device__ __forceinline__ uint32_t bound_of(const uint32_t *maxima, int parts, int lane, int k,
                                             uint32_t least) {
    uint32_t v[PER];
    uint32_t lo = ~0u, top = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = 64 * i < parts ? maxima[64 * i + lane] : 0u;      // parts is a multiple of 64
        top = v[i] > top ? v[i] : top;
        if (64 * i < parts) lo = v[i] < lo ? v[i] : lo;
    }
    top = wave_reduce(top, Max());
    uint32_t hi = top + (top != ~0u);                            // none reaches hi (but fp32's +inf)
    lo = wave_reduce(lo, Min());                                 // and all reach lo
    lo = lo > least ? lo : least;
    auto reach = [&](uint32_t x) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (64 * i < parts) n += __popcll(__ballot(v[i] >= x));
        return n;
    };
    if (lo > top || reach(lo) < k) return least;
    while (hi - lo > 1) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        const int n = reach(mid);
        if (n < k) {
            hi = mid;
        } else {
            lo = mid;
            if (n <= k + (k >> 3) + 3) break;
        }
    }
    return lo;
}

// s.best[0 .. result) = the row's k best classes, best first (fewer where fewer have a score).
// begin(maxima, parts) is called with the largest ranks of the parts, then vector(a) for the
// row's whole vectors and single(e) for its other elements; all of it again where the first
// stretch misleads.  Kernels call quiet_max() before.
template <dt_dtype XT, int WAVES, class FB, class FV, class FE>
__device__ __forceinline__ int best_of_row(const Team<WAVES> &t, const Row<XT> &row, int k,
                                           Collected<WAVES> &s, FB begin, FV vector, FE single) {
    using E = Elem<XT>;
    constexpr int kThreads = Team<WAVES>::kThreads, U = 4;
    const int lo_v = row.inner_lo(), hi_v = row.inner_hi();
    // Vectors lo_v + [0, held) are kept, a whole number for each thread.  So long a stretch that about
    // 150 or 230 classes are collected; at least what is kept.
    int held = kHeldVecs<WAVES> / kThreads * kThreads;
    if (held > hi_v - lo_v) held = hi_v - lo_v;
    const int64_t want = int64_t(hi_v - lo_v) * (k + (k >> 2)) / (WAVES == 16 ? 150 : 300);
    int stretch = lo_v + (want > held ? int(want) : held);
    if (stretch > hi_v || k > kThreads / 2) stretch = hi_v;
    // the maxima's parts: a thread each, or four threads where those are enough
    const bool four = kThreads >= 1024 && k <= 64;
    const int parts = four ? kThreads / 4 : kThreads;
    PartMax<XT> m;
    row.template inner<U>(lo_v, lo_v + held, t.thread, kThreads, [&](const u32x4 &a, int v) {
        m.add(a);
        s.held[v - lo_v] = a;
    });
    int seen = lo_v + held;
    uint32_t end_rank = 0;                  // of the element outside the whole vectors that this
    int end_class = 0;                      // thread has, if any
    row.ends(t.thread, [&](auto e, int cls) {
        end_rank = E::rank(e);
        end_class = cls;
    });
    bool fits;
    uint32_t lo;
    for (;;) {
        row.template inner<U>(seen, stretch, t.thread, kThreads,
                              [&](const u32x4 &a, int) { m.add(a); });
        seen = stretch;
        uint32_t mine = Max()(end_rank, lo_v < hi_v ? m.rank() : 0u);
        if (four) {
            mine = Max()(mine, partner<1>(mine));
            mine = Max()(mine, partner<2>(mine));
            if ((t.lane & 3) == 0) s.maxima[t.thread >> 2] = mine;
        } else {
            s.maxima[t.thread] = mine;
        }
        if (t.thread == 0) s.spilt = s.count = 0;
        t.sync();
        // (one wavefront does: eight that did the same would take the others' instructions)
        if (t.wave == 0) {
            lo = four ? bound_of<(WAVES + 3) / 4>(s.maxima, parts, t.lane, k, E::kNone + 1)
                      : bound_of<WAVES>(s.maxima, parts, t.lane, k, E::kNone + 1);
            if (t.lane == 0) s.bound = lo;
        }
        t.sync();
        lo = E::from_rank(s.bound);
        if (lo == E::kNone + 1 && stretch < hi_v) {      // a stretch with too few scores
            stretch = hi_v;
            t.sync();
            continue;
        }
        begin(s.maxima, parts);
        row.ends(t.thread, [&](auto e, int) { single(e); });
        const Filter<XT> filter(lo);
        const int mine_at = t.wave * kShare<WAVES>;
        int met = 0;                                     // the same in all lanes
        // Vector v of each lane (lanes behind the row's end: not `in`).  One of which an element
        // may reach the bound is queued; its elements are looked at later, when every lane has
        // such a vector.
        auto visit = [&](const u32x4 &a, int v, bool in) {
            const bool yes = in && filter.maybe(a);
            const uint64_t mask = __ballot(yes);
            if (mask != 0) {
                int at = met + __popcll(mask & ((uint64_t(1) << t.lane) - 1));
                met += __popcll(mask);
                if (yes) {
                    at = at < kShare<WAVES> ? mine_at + at
                                            : WAVES * kShare<WAVES> + atomicAdd(&s.spilt, 1);
                    if (at < WAVES * kShare<WAVES> + kSpill) {
                        s.queue[at] = a;
                        s.place[at] = v;
                    }
                }
            }
            if (in) vector(a);
        };
        // Wavefronts walk together; a lane behind the end has the last vector again.  Vectors
        // that are kept come from the LDS (each thread reads what it wrote).
        for (int v0 = lo_v + (t.thread & ~63); v0 < hi_v; v0 += U * kThreads) {
            u32x4 a[U];
            if (v0 + (U - 1) * kThreads + 63 < lo_v + held) {
#pragma unroll
                for (int u = 0; u < U; ++u) a[u] = s.held[v0 - lo_v + u * kThreads + t.lane];
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int v = v0 + u * kThreads + t.lane;
                    a[u] = row.load_whole(v < hi_v ? v : hi_v - 1);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = v0 + u * kThreads + t.lane;
                if (v0 + u * kThreads < hi_v) visit(a[u], v, v < hi_v);
            }
        }
        if (t.lane == 0) s.counts[t.wave] = met < kShare<WAVES> ? met : kShare<WAVES>;
        t.sync();
        fits = s.spilt <= kSpill;
        if (fits || stretch == hi_v) break;
        stretch = hi_v;
        t.sync();
    }
    int c = kCap + 1;
    uint64_t *list = s.list;
    if (fits) {
        auto add = [&](uint32_t rank, int cls) {
            const int at = atomicAdd(&s.count, 1);
            if (at < kCap) s.list[at] = comp(E::key_of_rank(rank), cls);
        };
        const int spilt = s.spilt;
        for (int i = t.thread; i < WAVES * kShare<WAVES> + spilt; i += kThreads) {
            if (i < WAVES * kShare<WAVES> && i % kShare<WAVES> >= s.counts[i / kShare<WAVES>]) continue;
            const u32x4 a = s.queue[i];
            const int cls = row.first(s.place[i]);
#pragma unroll
            for (int j = 0; j < Row<XT>::kVec; ++j) {
                const uint32_t r = E::rank(row.at(a, j));
                if (r >= lo) add(r, cls + j);
            }
        }
        if (end_rank >= lo) add(end_rank, end_class);
        t.sync();
        c = s.count;
        t.sync();                            // read by all before it is written again
        if (c > 96 && c <= kCap && k < kThreads) {
            // Ranking takes the square of their number: those that are surely not among the k
            // best are left out by a bound on the ones that are there.
            uint32_t mine = 0;
            for (int i = t.thread; i < c; i += kThreads) mine = Max()(mine, comp_key(s.list[i]));
            s.maxima[t.thread] = mine;
            if (t.thread == 0) s.count = 0;
            t.sync();
            if (t.wave == 0) {
                const uint32_t least = bound_of<WAVES>(s.maxima, kThreads, t.lane, k, 1);
                if (t.lane == 0) s.bound = least;
            }
            t.sync();
            const uint32_t least = s.bound;
            uint64_t *fewer = reinterpret_cast<uint64_t *>(s.queue);     // no longer needed
            constexpr int kRoom = kFewerRoom<WAVES>;
            static_assert(sizeof(s.queue) >= sizeof(uint64_t) * kRoom && (kRoom & (kRoom - 1)) == 0, "");
            for (int i = t.thread; i < c; i += kThreads)
                if (comp_key(s.list[i]) >= least) {
                    const int at = atomicAdd(&s.count, 1);
                    if (at < kRoom) fewer[at] = s.list[i];
                }
            t.sync();
            if (s.count <= kRoom) {              // (equal ones may be many)
                list = fewer;
                c = s.count;
            }
            t.sync();
        }
    }
    if (c > kCap) {
        // Too many equal (or few threads for many classes): the k-th best key itself, by
        // halving, and of the classes that have it the first ones.
        const int have = count_from(t, row, 1);
        k = k < have ? k : have;
        uint32_t kth = 1, over = 1;
        row.template each<2>(0, row.vecs, t.thread, t.kThreads,
                             [&](auto e, int) { over = Max()(over, E::key(e)); });
        over = t.reduce(over, Max()) + 1;
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
    order_best(t, list, s.best, c, k);
    return c < k ? c : k;
}

}  // namespace dscores
