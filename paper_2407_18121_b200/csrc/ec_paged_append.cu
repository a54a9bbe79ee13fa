// What happens to the rows of a paged cache around the attention: the step's probabilities are added to the weights, new
// rows join, and heads that then hold more than `budget` rows give up those of smallest gathered weight.
//  - One new row (a generation step): one launch does all of it. A row's new weight is on hand when the row that leaves is
//    looked for, so the weights are read once; the search is a minimum over (key, row). Bound by latency: a chain of
//    length, page, score and weight reads, which every thread walks for several rows side by side.
//  - More new rows (a prompt): a CTA, or a cluster of them when units are few and long, finds the key of the last row that
//    leaves and lists, in an ordered pass, the holes below the new length and the kept rows that have to move there (kept
//    rows never shift, so only as many rows move as join or sit behind the new length); a second launch moves them with
//    all CTAs of the GPU, bound by the copied bytes. The key is found with histograms of 1024 bins laid over the range the
//    keys really have, so that their counts spread (8-bit digits of float images put most keys into a few bins, whose
//    shared-memory additions then queue up), narrowed to one bin after the other: two or three passes over keys held in
//    shared memory. A list of 16384 costs one SM about 20 us of instructions; over a cluster the histograms are summed and
//    the ordered counts carried on through distributed shared memory.
// Measured per call: one row to 1024 full units of 320 rows 4.6 us; 64 rows onto 256 full units of 2048 14.5 us; prompts of 640 rows
// into 1024 units at budget 320 72 us (the move 57 us, 5.9 TB/s read and written); 16 units of up to 16384 rows 20 us.
// Rows leave in this order: those that cannot be read, then by protection, then by weight (keys are order-preserving unsigned
// images of the weights), and among equals the higher candidate first (cached rows in slot order, then the new rows). For a step that is
// one number per row. A selection gives all protected rows the largest key, which is enough as long as they all stay; where they do not,
// their weights are looked at in a second pass over the candidates, with the others marked as having left.
#include "ec_paged.cuh"

#include <cooperative_groups.h>

namespace ec {

namespace {

constexpr int kThreads = 256;                    // of a move, and of a selection but for long lists
constexpr int kFewRows = 64;                     // up to this many new rows the deciding CTAs move them themselves
constexpr int kMaxSplits = 512;                  // CTAs that share a unit's rows in a step

constexpr uint32_t kKeyProtected = 0xFFFFFFFFu, kKeyNan = 0xFFFFFFFEu;

// Order-preserving image of a weight: -inf lowest (0x007FFFFF, above the 0 of a row that cannot be read), -0 = +0, NaN above +inf.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return kKeyNan;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct Unit {
    int n, h, had, cnt, final, seen;
    size_t u;
};

// What a selection leaves for the launch that moves the rows: by then the lengths have changed.
__device__ __forceinline__ int4 unit_record(const Unit &u, int movers) { return make_int4(movers, u.had, u.cnt, u.seen); }

__device__ __forceinline__ bool is_protected(const AppendArgs &a, const Unit &u, int pos)
{
    return pos < a.sinks || (long long)pos >= (long long)u.seen + u.cnt - a.recent;
}

// What a selection goes by: the weight's image. `among_safe`: of the protected rows, when all others leave; else of the others.
__device__ __forceinline__ uint32_t select_key(bool safe, float w, bool among_safe)
{
    if (safe != among_safe) return safe ? kKeyProtected : 0u;
    return weight_key(w);
}

__device__ __forceinline__ uint32_t candidate_key(const PagedView &c, const AppendArgs &a, const Unit &u, int j, bool among_safe)
{
    float w;
    int pos;
    if (j < u.had) {
        const Slot s = find_slot(c, u.n, j);
        if (s.page < 0) return 0;                // a row that cannot be read leaves first
        const uint32_t m = meta_index(c, u.h, s);
        w = c.weight[m];
        pos = c.pos[m];
    } else {
        const size_t at = u.u * a.T + (j - u.had);
        w = a.w_new ? a.w_new[at] : 0.f;
        pos = a.pos_new ? a.pos_new[at] : u.seen + (j - u.had);
    }
    return select_key(is_protected(a, u, pos), w, among_safe);
}

// Candidate j -> slot `dst`, as lane l of the LPR = D / 8 lanes that copy a row.
__device__ __forceinline__ void move_row(const PagedView &c, const AppendArgs &a, const Unit &u, int dst, int j, int lpr, int l)
{
    const Slot d = look_up_slot(c, u.n, dst);
    const uint4 *k, *v;
    float w;
    int pos;
    if (j < u.had) {
        const Slot s = look_up_slot(c, u.n, j);
        if (!valid_page(c, s)) {
            report_page(c);
            return;
        }
        const size_t from = (size_t)u.h * c.head_step + row_offset(c, s) + l;
        k = c.K + from;
        v = c.V + from;
        const uint32_t m = meta_index(c, u.h, s);
        w = c.weight[m];
        pos = c.pos[m];
    } else {
        const size_t at = u.u * a.T + (j - u.had);
        k = a.K_new + at * lpr + l;
        v = a.V_new + at * lpr + l;
        w = a.w_new ? a.w_new[at] : 0.f;
        pos = a.pos_new ? a.pos_new[at] : u.seen + (j - u.had);
    }
    const uint4 kv = *k, vv = *v;                // a new row's reads do not wait for the page it goes to
    if (!valid_page(c, d)) {
        report_page(c);
        return;
    }
    const size_t to = (size_t)u.h * c.head_step + row_offset(c, d) + l;
    c.K[to] = kv;
    c.V[to] = vv;
    if (l == 0) {
        const uint32_t m = meta_index(c, u.h, d);
        c.weight[m] = w;
        c.pos[m] = pos;
    }
}

constexpr int kUnroll = 2;                       // candidates of a thread side by side in the passes over held keys
constexpr int kBins = 1024;

template <int THREADS> struct SelectSmem {
    int hist[kBins];
    int a[THREADS / 32], b[THREADS / 32];
    uint32_t lo[THREADS / 32], hi[THREADS / 32];
    uint32_t bin;
    int left, here;
    int coarse[32];                              // sums of 32 bins each
    uint32_t all_lo, all_hi;                     // of the CTA, for the others of its cluster
    int all_open, all_equal;
    int2 all_moves;
};

// Exclusive prefix over the warps of x and y, uniform within each warp; the totals come back in `sum`.
template <int THREADS>
__device__ __forceinline__ int2 warps_prefix(int x, int y, SelectSmem<THREADS> &sm, int2 &sum)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                             // the previous use of a and b is over
    if (lane == 0) {
        sm.a[warp] = x;
        sm.b[warp] = y;
    }
    __syncthreads();
    constexpr int kWarps = THREADS / 32;
    const int vx = lane < kWarps ? sm.a[lane] : 0, vy = lane < kWarps ? sm.b[lane] : 0;
    sum = make_int2(__reduce_add_sync(0xFFFFFFFFu, vx), __reduce_add_sync(0xFFFFFFFFu, vy));
    return make_int2(__reduce_add_sync(0xFFFFFFFFu, lane < warp ? vx : 0), __reduce_add_sync(0xFFFFFFFFu, lane < warp ? vy : 0));
}

template <bool AHEAD = false>
__device__ __forceinline__ Unit load_unit(const PagedView &c, const AppendArgs &a, int n, int h)
{
    Unit u;
    u.n = n;
    u.h = h;
    u.u = (size_t)n * c.H + h;
    const int len = read_len<AHEAD>(c, n);
    if (len < 0) {
        u.had = u.cnt = u.final = -1;
        u.seen = 0;
        return u;
    }
    u.had = a.fresh ? 0 : len;
    u.seen = a.fresh ? 0 : read_at<AHEAD>(c.seen + n);
    int cnt = a.counts ? a.counts[n] : a.T;
    u.cnt = min(max(cnt, 0), a.T);
    u.final = (int)min((long long)u.had + u.cnt, (long long)a.budget);
    return u;
}

// The whole CTA, or with SPREAD the whole cluster: lists the moves of unit u (slot to fill, candidate to take) and returns
// their number. `keys` takes the keys of the CTA's candidates when there is room for `room` of them; otherwise they are
// worked out again for every pass.
template <int THREADS, bool SPREAD, bool HELD>
__device__ __forceinline__ int select_body(const PagedView &c, const AppendArgs &a, const Unit &u, SelectSmem<THREADS> &sm,
                                           uint32_t *keys)
{
    namespace cg = cooperative_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kWarps = THREADS / 32;
    const int rank = SPREAD ? (int)cg::this_cluster().block_rank() : 0, ranks = SPREAD ? (int)cg::this_cluster().num_blocks() : 1;
    auto meet = [] {
        if (SPREAD) cg::this_cluster().sync();
        else __syncthreads();
    };
    auto of = [&](int r) { return SPREAD ? cg::this_cluster().map_shared_rank(&sm, r) : &sm; };   // rank r's shared memory
    const int all = u.had + u.cnt, leave = all - u.final;
    int2 *list = a.list + u.u * a.budget;
    if (leave <= 0) {                            // nothing leaves: the new rows go behind the others
        for (int k = rank * THREADS + threadIdx.x; k < u.cnt; k += ranks * THREADS) list[k] = make_int2(u.had + k, u.had + k);
        meet();
        return u.cnt;
    }
    const int share = (all + 32 * ranks - 1) / (32 * ranks) * 32;         // of the candidates, in order
    const int c0 = min(rank * share, all), c1 = min(c0 + share, all);
    const bool held = HELD;
    bool among_safe = false;
    auto key_of = [&](int j) { return held ? keys[j - c0] : candidate_key(c, a, u, j, among_safe); };

    // The range of the keys that the border can lie among, and the number of rows that leave before any other: the
    // protected ones are counted out in the first pass, the others in a second one when protected rows have to leave too.
    uint32_t lo, hi;
    int left = leave, open;
    constexpr int kBatch = 4;                    // candidates of a thread that walk their chain of reads side by side
    const int cached = min(c1, u.had);
    auto scan = [&](auto second_) {
        constexpr bool second = decltype(second_)::value;
        lo = 0xFFFFFFFFu;
        hi = 0;
        open = 0;
        auto take = [&](int j, uint32_t key, bool counts) {
            if (held) keys[j - c0] = key;
            if (counts) {
                lo = min(lo, key);
                hi = max(hi, key);
                ++open;
            }
        };
        for (int base = c0 + threadIdx.x; base < cached; base += kBatch * THREADS) {
            Slot s[kBatch];
            float w[kBatch];
            int pos[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int j = base + i * THREADS;
                s[i].page = -1;
                if (j < cached) s[i] = look_up_slot(c, u.n, j);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (!valid_page(c, s[i])) continue;
                const uint32_t m = meta_index(c, u.h, s[i]);
                w[i] = c.weight[m];
                pos[i] = c.pos[m];
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int j = base + i * THREADS;
                if (j >= cached) continue;
                if (!valid_page(c, s[i])) {      // a row that cannot be read leaves first, protected or not
                    report_page(c);
                    take(j, 0, !second);
                } else {
                    const bool safe = is_protected(a, u, pos[i]);
                    take(j, select_key(safe, w[i], second), safe == second);
                }
            }
        }
        for (int base = max(c0, u.had) + threadIdx.x; base < c1; base += kBatch * THREADS) {
            float w[kBatch];
            int pos[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int j = base + i * THREADS, t = j - u.had;
                if (j >= c1) continue;
                w[i] = a.w_new ? a.w_new[u.u * a.T + t] : 0.f;
                pos[i] = a.pos_new ? a.pos_new[u.u * a.T + t] : u.seen + t;
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int j = base + i * THREADS;
                if (j >= c1) continue;
                const bool safe = is_protected(a, u, pos[i]);
                take(j, select_key(safe, w[i], second), safe == second);
            }
        }
        lo = __reduce_min_sync(0xFFFFFFFFu, lo);
        hi = __reduce_max_sync(0xFFFFFFFFu, hi);
        open = __reduce_add_sync(0xFFFFFFFFu, open);
        if (second) meet();                  // nobody reads what the first pass left here any more
        else __syncthreads();
        if (lane == 0) {
            sm.lo[warp] = lo;
            sm.hi[warp] = hi;
            sm.a[warp] = open;
        }
        __syncthreads();
        lo = __reduce_min_sync(0xFFFFFFFFu, lane < kWarps ? sm.lo[lane] : 0xFFFFFFFFu);
        hi = __reduce_max_sync(0xFFFFFFFFu, lane < kWarps ? sm.hi[lane] : 0u);
        open = __reduce_add_sync(0xFFFFFFFFu, lane < kWarps ? sm.a[lane] : 0);
        if (SPREAD) {
            if (threadIdx.x == 0) {
                sm.all_lo = lo;
                sm.all_hi = hi;
                sm.all_open = open;
            }
            meet();
            const SelectSmem<THREADS> *other = of(lane < ranks ? lane : 0);
            lo = __reduce_min_sync(0xFFFFFFFFu, other->all_lo);
            hi = __reduce_max_sync(0xFFFFFFFFu, other->all_hi);
            open = __reduce_add_sync(0xFFFFFFFFu, lane < ranks ? other->all_open : 0);
        }
    };
    scan(std::false_type{});
    if (left > open) {                           // all of these leave, and some of the protected rows
        left -= open;
        among_safe = true;
        scan(std::true_type{});
    }
    // Of the keys in [lo, hi] `left` leave, and every smaller one. Narrowed until all of the range leaves or it is one key.
    // (At least one row stays, so that among protected rows fewer leave than there are.)
    int equal = 0;                               // > 0: rows at the edge, of which the last `left` leave
    uint32_t edge;                               // rows with a smaller key leave
    if (left == open) {                          // all that are not protected, and nothing else
        left = 0;
        edge = kKeyProtected;
    } else {
        for (;;) {
            const int bits = 32 - __clz(hi - lo), shift = max(0, bits - 10);
            meet();                              // nobody reads the last histogram any more
            for (int i = threadIdx.x; i < kBins; i += THREADS) sm.hist[i] = 0;
            __syncthreads();
#pragma unroll kUnroll
            for (int j = c0 + threadIdx.x; j < c1; j += THREADS) {
                const uint32_t key = key_of(j);
                if (key >= lo && key <= hi) atomicAdd(&sm.hist[(key - lo) >> shift], 1);
            }
            __syncthreads();
            // the bin in which the running count reaches `left`
            if (SPREAD) {                        // first among sums of 32 bins, then within one: little crosses the cluster
                for (int i = warp; i < 32; i += kWarps) {
                    const int group = __reduce_add_sync(0xFFFFFFFFu, sm.hist[i * 32 + lane]);
                    if (lane == 0) sm.coarse[i] = group;
                }
                meet();
                if (warp == 0) {
                    auto find = [&](int mine, int &at) {                  // the lane that passes `left`; at: the count in front of it
                        int incl = mine;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                            if (lane >= o) incl += up;
                        }
                        const int src = __ffs(__ballot_sync(0xFFFFFFFFu, at + incl >= left)) - 1;
                        at += __shfl_sync(0xFFFFFFFFu, incl - mine, src);
                        return src;
                    };
                    int mine = 0, fine = 0, at = 0;
#pragma unroll 8
                    for (int r = 0; r < ranks; ++r) mine += of(r)->coarse[lane];
                    const int group = find(mine, at);
#pragma unroll 8
                    for (int r = 0; r < ranks; ++r) fine += of(r)->hist[group * 32 + lane];
                    const int src = find(fine, at);
                    if (lane == src) {
                        sm.bin = group * 32 + src;
                        sm.left = left - at;
                        sm.here = fine;
                    }
                }
            } else {
                constexpr int kOwn = kBins / THREADS;                     // bins of a thread, in order
                int mine[kOwn], total = 0;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    mine[i] = sm.hist[threadIdx.x * kOwn + i];
                    total += mine[i];
                }
                int incl = total;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                    if (lane >= o) incl += up;
                }
                int2 sum;
                int at = warps_prefix<THREADS>(__shfl_sync(0xFFFFFFFFu, incl, 31), 0, sm, sum).x + incl - total;
                if (at < left && left <= at + total) {
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) {
                        if (at < left && left <= at + mine[i]) {
                            sm.bin = threadIdx.x * kOwn + i;
                            sm.left = left - at;
                            sm.here = mine[i];
                        }
                        at += mine[i];
                    }
                }
            }
            __syncthreads();
            left = sm.left;
            const int here = sm.here;
            lo += sm.bin << shift;
            hi = lo + min(hi - lo, (1u << shift) - 1u);                   // the bin's last key
            if (left == here) {                  // the whole bin leaves (its end is below the protected key)
                edge = hi + 1u;
                left = 0;
                break;
            }
            if (shift == 0) {
                edge = lo;
                equal = here;
                break;
            }
        }
    }
    // Ordered pass, a run of candidates per warp, 32 at a time: k-th hole <- k-th kept row from behind.
    const int span = (share + 32 * kWarps - 1) / (32 * kWarps) * 32;
    const int j0 = min(c0 + warp * span, c1), j1 = min(j0 + span, c1);
    const unsigned below = (1u << lane) - 1u;
    int2 sum;
    int rank_equal = 0;
    const int equal_kept = equal - left;
    if (left > 0) {                              // of the rows at the edge the first ones stay
        int count = 0;
        for (int j = j0 + lane; j - lane < j1; j += 32) count += __popc(__ballot_sync(0xFFFFFFFFu, j < j1 && key_of(j) == edge));
        rank_equal = warps_prefix<THREADS>(count, 0, sm, sum).x;
        if (SPREAD) {
            if (threadIdx.x == 0) sm.all_equal = sum.x;
            meet();
            rank_equal += __reduce_add_sync(0xFFFFFFFFu, lane < rank ? of(lane)->all_equal : 0);
        }
    }
    auto each = [&](auto use) {                  // use(candidate, mask of holes, mask of movers)
        int r = rank_equal;
#pragma unroll kUnroll
        for (int j = j0 + lane; j - lane < j1; j += 32) {
            const uint32_t key = j < j1 ? key_of(j) : 0u;
            bool stay = key >= edge;
            if (left > 0) {
                const unsigned equals = __ballot_sync(0xFFFFFFFFu, j < j1 && key == edge);
                if (key == edge) stay = r + __popc(equals & below) < equal_kept;
                r += __popc(equals);
            }
            const bool low = j < u.had && j < u.final;
            const unsigned holes = __ballot_sync(0xFFFFFFFFu, j < j1 && low && !stay);
            const unsigned movers = __ballot_sync(0xFFFFFFFFu, j < j1 && !low && stay);
            use(j, holes, movers);
        }
    };
    int holes = 0, movers = 0;
    each([&](int, unsigned hm, unsigned mm) {
        holes += __popc(hm);
        movers += __popc(mm);
    });
    int2 at = warps_prefix<THREADS>(holes, movers, sm, sum);
    if (SPREAD) {
        if (threadIdx.x == 0) sm.all_moves = sum;
        meet();
        const int2 other = lane < ranks ? of(lane)->all_moves : make_int2(0, 0);
        at.x += __reduce_add_sync(0xFFFFFFFFu, lane < rank ? other.x : 0);
        at.y += __reduce_add_sync(0xFFFFFFFFu, lane < rank ? other.y : 0);
        sum = make_int2(__reduce_add_sync(0xFFFFFFFFu, other.x), __reduce_add_sync(0xFFFFFFFFu, other.y));
    }
    each([&](int j, unsigned hm, unsigned mm) {
        if (hm >> lane & 1u) list[at.x + __popc(hm & below)].x = j;
        if (mm >> lane & 1u) list[at.y + __popc(mm & below)].y = j;
        at.x += __popc(hm);
        at.y += __popc(mm);
    });
    for (int s = u.had + rank * THREADS + threadIdx.x; s < u.final; s += ranks * THREADS)
        list[sum.x + (s - u.had)].x = s;         // slots behind the old length
    meet();                                      // the list is complete, every key has been read
    return sum.y;
}

template <int THREADS, bool SPREAD>
__device__ __forceinline__ int select_unit(const PagedView &c, const AppendArgs &a, const Unit &u, SelectSmem<THREADS> &sm,
                                           uint32_t *keys, int room)
{
    const int ranks = SPREAD ? (int)cooperative_groups::this_cluster().num_blocks() : 1;
    const int share = (u.had + u.cnt + 32 * ranks - 1) / (32 * ranks) * 32;
    return share <= room ? select_body<THREADS, SPREAD, true>(c, a, u, sm, keys) : select_body<THREADS, SPREAD, false>(c, a, u, sm, keys);
}

// The listed rows of a unit, by `ranks` CTAs of which this is number `rank`.
template <int THREADS>
__device__ __forceinline__ void move_listed(const PagedView &c, const AppendArgs &a, const Unit &u, int movers, int lpr, int rank, int ranks)
{
    const int groups = THREADS / lpr, group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
    const int2 *list = a.list + u.u * a.budget;
    for (int k = rank * groups + group; k < movers; k += ranks * groups) {
        const int2 e = list[k];
        move_row(c, a, u, e.x, e.y, lpr, l);
    }
}

// A CTA or a cluster of `ranks` CTAs per (problem, head). move_here: few rows, moved by those that listed them.
template <int THREADS, bool SPREAD>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) paged_select_kernel(PagedView c, AppendArgs a, int lpr, int move_here, int room, int ranks)
{
    extern __shared__ uint32_t sm_keys[];        // [room]
    __shared__ SelectSmem<THREADS> sm;
    grid_wait();
    grid_release();
    const int unit = SPREAD ? blockIdx.x / ranks : blockIdx.x, rank = SPREAD ? blockIdx.x - unit * ranks : 0;
    const int n = unit / c.H, h = unit - n * c.H;
    const Unit u = load_unit(c, a, n, h);
    if (u.had < 0) {                             // an empty place of the batch
        if (threadIdx.x == 0 && rank == 0) a.moves[u.u] = make_int4(0, 0, 0, 0);
        return;
    }
    const int movers = select_unit<THREADS, SPREAD>(c, a, u, sm, sm_keys, room);
    if (threadIdx.x == 0 && rank == 0) a.moves[u.u] = unit_record(u, movers);
    if (move_here) move_listed<THREADS>(c, a, u, movers, lpr, rank, ranks);
    // of the problem's CTAs, all of which have read its length, the last one changes it
    int *arrived = c.state + kStateAppend + n;
    if (threadIdx.x == 0 && arrive(arrived) == c.H * ranks - 1) {
        *arrived = 0;
        c.lens[n] = u.final;
        c.seen[n] = u.seen + u.cnt;
    }
}

// `parts` CTAs per unit: the listed rows of every unit.
__global__ void __launch_bounds__(kThreads) paged_move_kernel(PagedView c, AppendArgs a, int lpr, int parts)
{
    grid_wait();
    grid_release();
    const int unit = blockIdx.x / parts, part = blockIdx.x - unit * parts;
    const int4 record = a.moves[unit];
    const int movers = record.x;
    Unit u;
    u.n = unit / c.H;
    u.h = unit - u.n * c.H;
    u.u = unit;
    u.had = record.y;
    u.cnt = record.z;
    u.seen = record.w;
    u.final = 0;                                 // not looked at when rows are moved
    // one row per group of lanes at a time: two measured 30% slower, the registers cost more warps than the second
    // row's reads bring
    move_listed<kThreads>(c, a, u, movers, lpr, part, parts);
}

constexpr int kRowThreads = 128;
constexpr int kRowCtas = 8;                      // per SM
constexpr int kRowsHeld = 4;                     // rows a thread has in flight
constexpr int kScoresHeld = 4;                   // query heads whose scores a thread reads side by side

// The row that leaves first has the smallest of these: protected or not (one bit), key (32), then the higher candidate (31 bits:
// the host refuses more candidates).
constexpr uint32_t kLastCandidate = 0x7FFFFFFFu;
__device__ __forceinline__ unsigned long long leave_order(bool safe, uint32_t key, int j)
{
    return ((unsigned long long)(safe ? 1u : 0u) << 63) | ((unsigned long long)key << 31) | (kLastCandidate - (uint32_t)j);
}
__device__ __forceinline__ int row_that_leaves(unsigned long long order) { return (int)(kLastCandidate - ((uint32_t)order & kLastCandidate)); }

// More rows of a unit leave than join, which follows a smaller budget only: a call of its own keeps its registers out of the
// kernel's ordinary way.
__device__ __noinline__ void evict_many(const PagedView &c, const AppendArgs &a, const Unit &u, SelectSmem<kRowThreads> &sm, int lpr)
{
    const int movers = select_unit<kRowThreads, false>(c, a, u, sm, nullptr, 0);
    move_listed<kRowThreads>(c, a, u, movers, lpr, 0, 1);
}

// `splits` CTAs per (problem, head). GATHER: weights <- decay * weights + probabilities of the step. APPEND: at most one
// new row per problem joins; of the problem's CTAs the one that arrives last changes its length, and where a unit's rows
// are shared, decides and moves for all of its heads.
// QUAD: a thread's rows are neighbours in one page, so that one page number and reads of 16 bytes do for the four; else
// they lie kRowThreads apart.
template <bool GATHER, bool APPEND, bool QUAD>
__global__ void __launch_bounds__(kRowThreads, kRowCtas) paged_rows_kernel(const __grid_constant__ PagedView c, GatherArgs ga,
                                                                            const __grid_constant__ AppendArgs ap, int lpr, int splits)
{
    extern __shared__ float2 sm_stat[];          // [G]
    __shared__ unsigned long long sm_low[kRowThreads / 32];
    __shared__ int sm_last;
    __shared__ SelectSmem<kRowThreads> sm_select;
    // With GATHER the launch in front is the attention of the same call, which lets this one in only when everything
    // before it is complete and writes no length, page, weight or position: those are read ahead of the wait.
    if (!GATHER) grid_wait();
    const int unit = blockIdx.x / splits, z = blockIdx.x - unit * splits;
    const int n = unit / c.H, h = unit - n * c.H;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int G = GATHER ? ga.G : 0;
    const size_t head_at = (size_t)unit * G;
    const bool by_row = scores_by_row(c.page_size);
    const int score_rows = by_row ? c.max_pages * c.page_size : c.page_size;
    Unit u;
    if (APPEND) {
        u = load_unit<GATHER>(c, ap, n, h);
    } else {
        u.n = n;
        u.h = h;
        u.u = unit;
        u.had = read_len<GATHER>(c, n);
    }
    if (u.had < 0) {                             // an empty place of the batch
        if (GATHER) grid_wait();
        grid_release();
        if (GATHER && z == 0 && threadIdx.x == 0 && ga.w_new) ga.w_new[unit] = 0.f;
        return;
    }
    // a unit of one CTA: its new row is on its way while the rows that may leave are looked over
    uint4 own_k = make_uint4(0, 0, 0, 0), own_v = own_k;
    const bool carry = APPEND && splits == 1 && warp == 0 && lane < lpr && u.cnt > 0;
    if (carry) {
        own_k = __ldcg(ap.K_new + u.u * lpr + lane);
        own_v = __ldcg(ap.V_new + u.u * lpr + lane);
    }
    const int leave = APPEND ? u.had + u.cnt - u.final : 0;
    const bool simple = leave <= 0 || (leave == 1 && u.cnt == 1);         // else: more rows leave than join
    unsigned long long low = ~0ull;
    bool first = true;
    for (int row0 = z * kRowThreads * kRowsHeld; first || row0 < u.had; row0 += splits * kRowThreads * kRowsHeld) {
        uint32_t m[kRowsHeld];
        const float *score[kRowsHeld];
        float w[kRowsHeld];
        int pos[kRowsHeld];
        bool there[kRowsHeld];
        const int row_step = QUAD ? 1 : kRowThreads, thread_row = row0 + (int)threadIdx.x * (QUAD ? kRowsHeld : 1);
        Slot s = {-1, 0};
#pragma unroll
        for (int r = 0; r < kRowsHeld; ++r) {
            const int row = thread_row + r * row_step;
            there[r] = false;
            if (row >= u.had) continue;
            if (QUAD && r > 0)
                ++s.slot;
            else
                s = GATHER && first ? find_slot<true>(c, n, row) : find_slot(c, n, row);
            there[r] = s.page >= 0;
            m[r] = meta_index(c, h, s);
            if (GATHER)
                score[r] = by_row ? ga.scores + head_at * score_rows + row
                                  : ga.scores + (size_t)((uint32_t)s.page * (uint32_t)c.H + (uint32_t)h) * G * score_rows + s.slot;
            if (APPEND && !there[r]) low = min(low, leave_order(false, 0, row)); // a row that cannot be read leaves first
        }
        if (QUAD) {                              // what lies behind the last row is read with it and not used
            if (there[0]) {
                const float4 x = __ldcg(reinterpret_cast<const float4 *>(c.weight + m[0]));
                w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
                if (APPEND) {
                    const int4 y = __ldcg(reinterpret_cast<const int4 *>(c.pos + m[0]));
                    pos[0] = y.x, pos[1] = y.y, pos[2] = y.z, pos[3] = y.w;
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) {
                if (!there[r]) continue;
                w[r] = __ldcg(c.weight + m[r]);
                if (APPEND) pos[r] = __ldcg(c.pos + m[r]);
            }
        }
        if (GATHER) {
            if (first) {
                grid_wait();
                for (int i = threadIdx.x; i < G; i += kRowThreads) sm_stat[i] = __ldcg(&ga.stat[head_at + i]);
            }
            float p[kRowsHeld], x[kScoresHeld][kRowsHeld];
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) p[r] = 0.f;
            for (int h0 = 0; h0 < G; h0 += kScoresHeld) {
#pragma unroll
                for (int i = 0; i < kScoresHeld; ++i) {
                    if (h0 + i >= G) continue;
                    if (QUAD) {
                        if (!there[0]) continue;
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(score[0] + (size_t)(h0 + i) * score_rows));
                        x[i][0] = y.x, x[i][1] = y.y, x[i][2] = y.z, x[i][3] = y.w;
                    } else {
#pragma unroll
                        for (int r = 0; r < kRowsHeld; ++r)
                            if (there[r]) x[i][r] = __ldcg(score[r] + (size_t)(h0 + i) * score_rows);
                    }
                }
                if (first && h0 == 0) __syncthreads();
#pragma unroll
                for (int i = 0; i < kScoresHeld; ++i) {
                    if (h0 + i >= G) continue;
                    const float2 st = sm_stat[h0 + i];
#pragma unroll
                    for (int r = 0; r < kRowsHeld; ++r)
                        if (there[r]) p[r] = fmaf(fast_exp2((x[i][r] - st.x) * ga.scale_log2e), st.y, p[r]);
                }
            }
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) {
                if (!there[r]) continue;
                w[r] = fmaf(w[r], ga.decay, p[r]);
                if (!QUAD || !there[kRowsHeld - 1]) c.weight[m[r]] = w[r];
            }
            if (QUAD && there[kRowsHeld - 1])
                *reinterpret_cast<float4 *>(c.weight + m[0]) = make_float4(w[0], w[1], w[2], w[3]);
        }
        first = false;
        if (APPEND) {
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) {
                if (!there[r]) continue;
                low = min(low, leave_order(is_protected(ap, u, pos[r]), weight_key(w[r]), thread_row + r * row_step));
            }
        }
    }
    grid_release();
    // the new row's own share
    float w_own = 0.f;
    if (GATHER && ga.w_new && z == 0 && warp == 0) {
        for (int hd = lane; hd < G; hd += 32)
            w_own = fmaf(fast_exp2((ga.score_new[head_at + hd] - sm_stat[hd].x) * ga.scale_log2e), sm_stat[hd].y, w_own);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) w_own += __shfl_xor_sync(0xFFFFFFFFu, w_own, d);
        if (lane == 0) ga.w_new[unit] = w_own;
    }
    if (!APPEND) return;

    if (z == 0 && warp == 0 && u.cnt > 0) {
        if (!GATHER) w_own = ap.w_new ? ap.w_new[unit] : 0.f;
        const bool safe = is_protected(ap, u, ap.pos_new ? ap.pos_new[unit] : u.seen);
        low = min(low, leave_order(safe, weight_key(w_own), u.had));
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) low = min(low, __shfl_xor_sync(0xFFFFFFFFu, low, d));
    if (lane == 0) sm_low[warp] = low;
    __syncthreads();                             // and the weights of this CTA's rows are written
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kRowThreads / 32; ++w) low = min(low, sm_low[w]);
        sm_low[0] = low;
        if (splits > 1) ap.lowest[(size_t)unit * splits + z] = low;
    }
    __syncthreads();
    // One row joins and at most one leaves: the new row goes behind the others or takes the place of the lowest.
    auto place = [&](const Unit &v, unsigned long long lowest, int l) {   // by a warp, of which the first lpr lanes copy
        if (v.cnt == 0) return;
        int dst = v.had;
        if (v.had + v.cnt > v.final) {
            dst = row_that_leaves(lowest);
            if (dst == v.had) return;            // the new row itself is the one that leaves
        }
        if (l < lpr) move_row(c, ap, v, dst, v.had, lpr, l);
    };
    int *arrived = c.state + kStateAppend + n;
    if (splits == 1) {
        // the length has been read: a warp of its own counts the CTA in while the row is placed
        if (threadIdx.x == 32 && arrive(arrived) == c.H - 1) {
            *arrived = 0;
            c.lens[n] = u.final;
            c.seen[n] = u.seen + u.cnt;
        }
        if (!simple) {
            const Unit v = u;
            evict_many(c, ap, v, sm_select, lpr);
        } else if (carry) {
            const int dst = leave <= 0 ? u.had : row_that_leaves(sm_low[0]);
            if (leave > 0 && dst == u.had) return;                        // the new row itself is the one that leaves
            const Slot s = look_up_slot(c, n, dst);
            if (!valid_page(c, s)) {
                report_page(c);
                return;
            }
            const size_t to = (size_t)h * c.head_step + row_offset(c, s) + lane;
            c.K[to] = own_k;
            c.V[to] = own_v;
            if (lane == 0) {
                const uint32_t m = meta_index(c, h, s);
                c.weight[m] = w_own;
                c.pos[m] = ap.pos_new ? ap.pos_new[unit] : u.seen;
            }
        }
        return;
    }
    if (threadIdx.x == 0) sm_last = arrive(arrived) == c.H * splits - 1;
    __syncthreads();
    if (!sm_last) return;
    if (simple) {
        for (int hh = warp; hh < c.H; hh += kRowThreads / 32) {
            Unit v = u;
            v.h = hh;
            v.u = (size_t)n * c.H + hh;
            unsigned long long best = ~0ull;
            for (int i = lane; i < splits; i += 32) best = min(best, __ldcg(&ap.lowest[v.u * splits + i]));
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) best = min(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
            place(v, best, lane);
        }
    } else {
        for (int hh = 0; hh < c.H; ++hh) {
            Unit v = u;
            v.h = hh;
            v.u = (size_t)n * c.H + hh;
            evict_many(c, ap, v, sm_select, lpr);
            __syncthreads();
        }
    }
    if (threadIdx.x == 0) {
        *arrived = 0;
        c.lens[n] = u.final;
        c.seen[n] = u.seen + u.cnt;
    }
}

// CTAs per unit of a rows launch, from the most rows that a unit can hold (the budget, or without an append what the table
// reaches), as the lengths are on the device: as many as fit the GPU at once (a second, partial wave measured 2% of a call of 512
// units of 8192 rows), but no more than two rounds of rows each, so that the longest of a ragged batch are not left to one CTA
// (34 x 32 units of up to 3836 rows: 68 -> 56 us). Sequences far shorter than that pay for CTAs that find nothing to do (64 x 8
// heads x 1000 rows with weights: 58 us under a table of 1024 or 8192 rows, 145 us under one of 131072).
inline int row_splits(long long units, long long rows)
{
    constexpr long long kRound = kRowThreads * kRowsHeld;
    long long z = 148LL * kRowCtas / units;
    const long long least = (rows + 2 * kRound - 1) / (2 * kRound), most = (rows + kRound - 1) / kRound;
    if (z < least) z = least;
    if (z > most) z = most;
    if (z > kMaxSplits) z = kMaxSplits;
    return z < 1 ? 1 : (int)z;
}

constexpr int kKeysHeld = 48 * 1024;             // keys of a CTA in shared memory at most

cudaError_t launch_select(long long units, int ranks, bool wide, int room, cudaStream_t stream, const PagedView &c, const AppendArgs &a, int lpr,
                          int move_here)
{
    auto kernel = ranks > 1 ? paged_select_kernel<kThreads, true> : wide ? paged_select_kernel<1024, false> : paged_select_kernel<kThreads, false>;
    if (room > 10 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeysHeld * (int)sizeof(uint32_t));
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * ranks));
    cfg.blockDim = dim3(wide ? 1024 : kThreads);
    cfg.dynamicSmemBytes = room * sizeof(uint32_t);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, c, a, lpr, move_here, room, ranks);
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t paged_append_workspace_bytes(const ec_paged *c, int T, int budget)
{
    const size_t units = (size_t)c->N * c->H;
    return up256(units * sizeof(int4)) + up256(units * budget * sizeof(int2)) +
           (T <= 1 ? up256(units * row_splits(units, budget) * sizeof(unsigned long long)) : 0);
}

cudaError_t launch_paged_rows(const PagedView &c, int D, const GatherArgs *gather, AppendArgs *append, void *ws, cudaStream_t stream)
{
    const long long units = (long long)c.N * c.H;
    const int lpr = D / 8;
    AppendArgs a = {};
    if (append) {
        a = *append;
        char *p = static_cast<char *>(ws);
        a.moves = reinterpret_cast<int4 *>(p);
        p += up256(units * sizeof(int4));
        a.list = reinterpret_cast<int2 *>(p);
        p += up256(units * a.budget * sizeof(int2));
        a.lowest = reinterpret_cast<unsigned long long *>(p);
    }
    if (gather || a.T <= 1) {
        const int splits = row_splits(units, append ? a.budget : (long long)c.max_pages * c.page_size);
        const GatherArgs g = gather ? *gather : GatherArgs{};
        // Four rows at a time where pages hold whole fours and the arrays lie for it. One by one / by fours: 512 units of 8192
        // rows with weights 377 / 370 us, a step of 384 units of 2048 rows 86.6 / 84.2 us, one row to 1024 units 4.5 / 4.3 us.
        const bool quad = c.page_size % 4 == 0 && ((reinterpret_cast<uintptr_t>(c.weight) | reinterpret_cast<uintptr_t>(c.pos)) & 15) == 0;
        auto pick = [&](auto q) {
            constexpr bool Q = decltype(q)::value;
            return !append ? paged_rows_kernel<true, false, Q> : gather ? paged_rows_kernel<true, true, Q> : paged_rows_kernel<false, true, Q>;
        };
        auto kernel = quad ? pick(std::true_type{}) : pick(std::false_type{});
        return launch_chained(kernel, dim3((unsigned)(splits * units)), kRowThreads, g.G * sizeof(float2), stream, c, g, a, lpr, splits);
    }
    const bool few = a.T <= kFewRows;
    // One CTA of 256 threads per unit; for few units with long lists one of 1024 threads, or a cluster of eight. Measured per
    // call, 256 threads / 1024 threads / cluster: 8 units of 2048 candidates 10.9 / 10.9 / 11.8 us, 64 units of 4096 19 / 12 / -,
    // 16 units of 8192 - / 19 / 19, 16 units of 16384 - / 25 / 21, 8 units of 65536 - / 149 / 46.
    const long long most_keys = (long long)a.budget + a.T;
    const int ranks = most_keys >= 16384 && units * 8 <= 148 * 2 ? 8 : 1;
    const bool wide = ranks == 1 && most_keys >= 4096 && units <= 148;
    const long long share = (most_keys + 32 * ranks - 1) / (32 * ranks) * 32;
    const int room = share <= kKeysHeld ? (int)share : 0;                 // more than that: worked out again for every pass
    cudaError_t e = launch_select(units, ranks, wide, room, stream, c, a, lpr, few ? 1 : 0);
    if (e == cudaSuccess && !few) {
        const int groups = kThreads / lpr;
        long long parts = (148LL * 8 + units - 1) / units;
        const long long most = ((long long)a.budget + groups - 1) / groups;
        if (parts > most) parts = most;
        e = launch_chained(paged_move_kernel, dim3((unsigned)(parts * units)), kThreads, 0, stream, c, a, lpr, (int)parts);
    }
    return e;
}

}  // namespace ec
