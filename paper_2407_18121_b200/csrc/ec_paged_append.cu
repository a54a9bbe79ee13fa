// What happens to the rows of a paged cache around the attention: the step's probabilities are added to the weights, new
// rows join, and heads that then hold more than `budget` rows give up those of smallest gathered weight.
//  - One new row (a generation step): one launch does all of it. A row's new weight is on hand when the row that leaves is
//    looked for, so the weights are read once; the search is a minimum over (key, row). Bound by latency: a chain of
//    length, page, score and weight reads, which every thread walks for several rows side by side.
//  - More new rows (a prompt): a CTA per (problem, head) finds the key of the last row that leaves and lists, in an ordered
//    pass, the holes below the new length and the kept rows that have to move there (kept rows never shift, so only as
//    many rows move as join or sit behind the new length); a second launch moves them with all CTAs of the GPU, bound by
//    the copied bytes. The key is found with histograms of 1024 bins laid over the range the keys really have, so that
//    their counts spread (8-bit digits of float images put most keys into a few bins, whose shared-memory additions then
//    queue up), narrowed to one bin after the other: two or three passes over keys held in shared memory.
// Keys are order-preserving unsigned images of the weights; rows at protected positions get the largest key. Equal keys:
// the higher candidate leaves first (cached rows in slot order, then the new rows).
#include "ec_paged.cuh"

namespace ec {

namespace {

constexpr int kThreads = 256;                    // of a move
constexpr int kFewRows = 16;                     // up to this many new rows the deciding CTA moves them itself
constexpr int kMaxSplits = 512;                  // CTAs that share a unit's rows in a step

constexpr uint32_t kKeyProtected = 0xFFFFFFFFu, kKeyNan = 0xFFFFFFFEu;

// Order-preserving image of a weight: -inf lowest, -0 = +0, NaN above +inf.
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

__device__ __forceinline__ uint32_t candidate_key(const PagedView &c, const AppendArgs &a, const Unit &u, int j)
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
    return is_protected(a, u, pos) ? kKeyProtected : weight_key(w);
}

// Row j of the candidates -> slot `dst`, by LPR = D / 8 lanes of which this is lane l.
__device__ __forceinline__ void move_row(const PagedView &c, const AppendArgs &a, const Unit &u, int dst, int j, int lpr, int l)
{
    const Slot d = find_slot(c, u.n, dst);
    if (d.page < 0) return;
    const size_t to = (size_t)u.h * c.head_step + row_offset(c, d) + l;
    const uint32_t meta_to = meta_index(c, u.h, d);
    const uint4 *k, *v;
    float w;
    int pos;
    if (j < u.had) {
        const Slot s = find_slot(c, u.n, j);
        if (s.page < 0) return;
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
    const uint4 kv = *k, vv = *v;
    c.K[to] = kv;
    c.V[to] = vv;
    if (l == 0) {
        c.weight[meta_to] = w;
        c.pos[meta_to] = pos;
    }
}

constexpr int kBins = 1024;

template <int THREADS> struct SelectSmem {
    int hist[kBins];
    int a[THREADS / 32], b[THREADS / 32];
    uint32_t lo[THREADS / 32], hi[THREADS / 32];
    uint32_t bin;
    int left, here;
};

// Exclusive prefix over the block of x and y; the totals come back in `sum`.
template <int THREADS>
__device__ __forceinline__ int2 block_prefix(int x, int y, SelectSmem<THREADS> &sm, int2 &sum)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int ix = x, iy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int ux = __shfl_up_sync(0xFFFFFFFFu, ix, o), uy = __shfl_up_sync(0xFFFFFFFFu, iy, o);
        if (lane >= o) {
            ix += ux;
            iy += uy;
        }
    }
    __syncthreads();                             // the previous use of a and b is over
    if (lane == 31) {
        sm.a[warp] = ix;
        sm.b[warp] = iy;
    }
    __syncthreads();
    int2 before = make_int2(ix - x, iy - y);
    sum = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) {
            before.x += sm.a[w];
            before.y += sm.b[w];
        }
        sum.x += sm.a[w];
        sum.y += sm.b[w];
    }
    return before;
}

__device__ __forceinline__ Unit load_unit(const PagedView &c, const AppendArgs &a, int n, int h)
{
    Unit u;
    u.n = n;
    u.h = h;
    u.u = (size_t)n * c.H + h;
    const int len = read_len(c, n);
    if (len < 0) {
        u.had = u.cnt = u.final = -1;
        u.seen = 0;
        return u;
    }
    u.had = a.fresh ? 0 : len;
    u.seen = a.fresh ? 0 : c.seen[n];
    int cnt = a.counts ? a.counts[n] : a.T;
    u.cnt = min(max(cnt, 0), a.T);
    u.final = (int)min((long long)u.had + u.cnt, (long long)a.budget);
    return u;
}

// The whole CTA: lists the moves of unit u (slot to fill, candidate to take) and returns their number. `keys` takes the
// candidates' keys when there is room for `room` of them; otherwise they are worked out again for every pass.
template <int THREADS>
__device__ __forceinline__ int select_unit(const PagedView &c, const AppendArgs &a, const Unit &u, SelectSmem<THREADS> &sm,
                                           uint32_t *keys, int room)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int all = u.had + u.cnt, leave = all - u.final;
    int2 *list = a.list + u.u * a.budget;
    if (leave <= 0) {                            // nothing leaves: the new rows go behind the others
        for (int k = threadIdx.x; k < u.cnt; k += THREADS) list[k] = make_int2(u.had + k, u.had + k);
        __syncthreads();
        return u.cnt;
    }
    const bool held = all <= room;
    auto key_of = [&](int j) { return held ? keys[j] : candidate_key(c, a, u, j); };

    // the range of the keys that are not protected, and their number
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    int open = 0;
    for (int j = threadIdx.x; j < all; j += THREADS) {
        const uint32_t key = candidate_key(c, a, u, j);
        if (held) keys[j] = key;
        if (key != kKeyProtected) {
            lo = min(lo, key);
            hi = max(hi, key);
            ++open;
        }
    }
    lo = __reduce_min_sync(0xFFFFFFFFu, lo);
    hi = __reduce_max_sync(0xFFFFFFFFu, hi);
    open = __reduce_add_sync(0xFFFFFFFFu, open);
    __syncthreads();
    if (lane == 0) {
        sm.lo[warp] = lo;
        sm.hi[warp] = hi;
        sm.a[warp] = open;
    }
    __syncthreads();
    open = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        lo = min(lo, sm.lo[w]);
        hi = max(hi, sm.hi[w]);
        open += sm.a[w];
    }
    // Of the keys in [lo, hi] `left` leave, and every smaller one. Narrowed until all of the range leaves or it is one key.
    int left = leave, equal = 0;                 // equal > 0: rows at key lo, of which the last `left` leave
    uint32_t edge;                               // rows with a smaller key leave
    if (left >= open) {                          // protected rows leave too, where they are all that is left
        left -= open;
        equal = all - open;
        edge = kKeyProtected;
    } else {
        for (;;) {
            const int bits = 32 - __clz(hi - lo), shift = max(0, bits - 10);
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += THREADS) sm.hist[i] = 0;
            __syncthreads();
            for (int j = threadIdx.x; j < all; j += THREADS) {
                const uint32_t key = key_of(j);
                if (key >= lo && key <= hi) atomicAdd(&sm.hist[(key - lo) >> shift], 1);
            }
            __syncthreads();
            if (warp == 0) {                     // the bin in which the running count reaches `left`
                int mine = 0;
#pragma unroll
                for (int i = 0; i < kBins / 32; ++i) mine += sm.hist[lane * (kBins / 32) + ((i + lane) & 31)];
                int incl = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                    if (lane >= o) incl += up;
                }
                const unsigned reached = __ballot_sync(0xFFFFFFFFu, incl >= left);
                const int src = __ffs(reached) - 1;
                int at = __shfl_sync(0xFFFFFFFFu, incl - mine, src);
                int bin = sm.hist[src * 32 + lane];
                int run = bin;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xFFFFFFFFu, run, o);
                    if (lane >= o) run += up;
                }
                const int sub = __ffs(__ballot_sync(0xFFFFFFFFu, at + run >= left)) - 1;
                if (lane == sub) {
                    sm.bin = src * 32 + sub;
                    sm.left = left - (at + run - bin);
                    sm.here = bin;
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
    // Ordered pass, a run of candidates per thread (odd, against bank conflicts): k-th hole <- k-th kept row from behind.
    const int span = ((all + THREADS - 1) / THREADS) | 1;
    const int j0 = min((int)threadIdx.x * span, all), j1 = min(j0 + span, all);
    int2 sum;
    int rank = 0;
    const int equal_kept = equal - left;
    if (left > 0) {                              // of the rows at the edge the first ones stay
        int mine = 0;
        for (int j = j0; j < j1; ++j) mine += key_of(j) == edge;
        rank = block_prefix<THREADS>(mine, 0, sm, sum).x;
    }
    int holes = 0, movers = 0;
    auto each = [&](auto hole, auto mover) {
        int r = rank;
        for (int j = j0; j < j1; ++j) {
            const uint32_t key = key_of(j);
            bool stay = key >= edge;
            if (left > 0 && key == edge) stay = r++ < equal_kept;
            if (j < u.had && j < u.final) {
                if (!stay) hole(j);
            } else if (stay) {
                mover(j);
            }
        }
    };
    each([&](int) { ++holes; }, [&](int) { ++movers; });
    int2 at = block_prefix<THREADS>(holes, movers, sm, sum);
    each([&](int j) { list[at.x++].x = j; }, [&](int j) { list[at.y++].y = j; });
    for (int s = u.had + threadIdx.x; s < u.final; s += THREADS) list[sum.x + (s - u.had)].x = s;   // slots behind the old length
    __syncthreads();                             // the list is complete, every key has been read
    return sum.y;
}

// The listed rows of a unit, by the whole CTA.
template <int THREADS>
__device__ __forceinline__ void move_listed(const PagedView &c, const AppendArgs &a, const Unit &u, int movers, int lpr)
{
    const int group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
    const int2 *list = a.list + u.u * a.budget;
    for (int k = group; k < movers; k += THREADS / lpr) {
        const int2 e = list[k];
        move_row(c, a, u, e.x, e.y, lpr, l);
    }
}

// A CTA per (problem, head). move_here: few rows, moved by the CTA that listed them.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) paged_select_kernel(PagedView c, AppendArgs a, int lpr, int move_here, int room)
{
    extern __shared__ uint32_t sm_keys[];        // [room]
    __shared__ SelectSmem<THREADS> sm;
    grid_wait();
    grid_release();
    const int n = blockIdx.x / c.H, h = blockIdx.x - n * c.H;
    const Unit u = load_unit(c, a, n, h);
    if (u.had < 0) {                             // an empty place of the batch
        if (threadIdx.x == 0) a.moves[u.u] = make_int4(0, 0, 0, 0);
        return;
    }
    const int movers = select_unit<THREADS>(c, a, u, sm, sm_keys, room);
    if (threadIdx.x == 0) a.moves[u.u] = unit_record(u, movers);
    if (move_here) move_listed<THREADS>(c, a, u, movers, lpr);
    // of the problem's CTAs, all of which have read its length, the last one changes it
    int *arrived = c.state + kStateAppend + n;
    if (threadIdx.x == 0 && arrive(arrived) == c.H - 1) {
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
    const int groups = kThreads / lpr, group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
    const int2 *list = a.list + u.u * a.budget;
    for (int k = part * groups + group; k < movers; k += parts * groups) {
        const int2 e = list[k];
        move_row(c, a, u, e.x, e.y, lpr, l);
    }
}

constexpr int kRowThreads = 128;
constexpr int kRowCtas = 8;                      // per SM
constexpr int kRowsHeld = 4;                     // rows a thread has in flight
constexpr int kScoresHeld = 4;                   // query heads whose scores a thread reads side by side

// The row that leaves first has the smallest of these: key, then the higher candidate.
__device__ __forceinline__ unsigned long long leave_order(uint32_t key, int j)
{
    return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)j);
}

// `splits` CTAs per (problem, head). GATHER: weights <- decay * weights + probabilities of the step. APPEND: at most one
// new row per problem joins; of the problem's CTAs the one that arrives last changes its length, and where a unit's rows
// are shared, decides and moves for all of its heads.
template <bool GATHER, bool APPEND>
__global__ void __launch_bounds__(kRowThreads, kRowCtas) paged_rows_kernel(PagedView c, GatherArgs ga, AppendArgs ap, int lpr, int splits)
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
    Unit u;
    if (APPEND) {
        u = load_unit(c, ap, n, h);
    } else {
        u.n = n;
        u.h = h;
        u.u = unit;
        u.had = read_len(c, n);
    }
    if (u.had < 0) {                             // an empty place of the batch
        if (GATHER) grid_wait();
        grid_release();
        if (GATHER && z == 0 && threadIdx.x == 0 && ga.w_new) ga.w_new[unit] = 0.f;
        return;
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
#pragma unroll
        for (int r = 0; r < kRowsHeld; ++r) {
            const int row = row0 + r * kRowThreads + threadIdx.x;
            there[r] = false;
            if (row >= u.had) continue;
            const Slot s = find_slot(c, n, row);
            there[r] = s.page >= 0;
            m[r] = meta_index(c, h, s);
            if (GATHER) score[r] = ga.scores + (size_t)((uint32_t)s.page * (uint32_t)c.H + (uint32_t)h) * G * c.page_size + s.slot;
            if (APPEND && !there[r]) low = min(low, leave_order(0, row)); // a row that cannot be read leaves first
        }
#pragma unroll
        for (int r = 0; r < kRowsHeld; ++r) {
            w[r] = 0.f;
            if (!there[r]) continue;
            w[r] = c.weight[m[r]];
            if (APPEND) pos[r] = c.pos[m[r]];
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
#pragma unroll
                    for (int r = 0; r < kRowsHeld; ++r)
                        if (there[r]) x[i][r] = __ldcg(score[r] + (size_t)(h0 + i) * c.page_size);
                }
                if (first && h0 == 0) __syncthreads();
#pragma unroll
                for (int i = 0; i < kScoresHeld; ++i) {
                    if (h0 + i >= G) continue;
                    const float2 st = sm_stat[h0 + i];
#pragma unroll
                    for (int r = 0; r < kRowsHeld; ++r)
                        if (there[r]) p[r] = fmaf(fast_exp2(fmaf(x[i][r], ga.scale_log2e, -st.x)), st.y, p[r]);
                }
            }
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) {
                if (!there[r]) continue;
                w[r] = fmaf(w[r], ga.decay, p[r]);
                c.weight[m[r]] = w[r];
            }
        }
        first = false;
        if (APPEND) {
#pragma unroll
            for (int r = 0; r < kRowsHeld; ++r) {
                if (!there[r]) continue;
                const bool safe = is_protected(ap, u, pos[r]);
                low = min(low, leave_order(safe ? kKeyProtected : weight_key(w[r]), row0 + r * kRowThreads + (int)threadIdx.x));
            }
        }
    }
    grid_release();
    // the new row's own share
    float w_own = 0.f;
    if (GATHER && ga.w_new && z == 0 && warp == 0) {
        for (int hd = lane; hd < G; hd += 32)
            w_own = fmaf(fast_exp2(fmaf(ga.score_new[head_at + hd], ga.scale_log2e, -sm_stat[hd].x)), sm_stat[hd].y, w_own);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) w_own += __shfl_xor_sync(0xFFFFFFFFu, w_own, d);
        if (lane == 0) ga.w_new[unit] = w_own;
    }
    if (!APPEND) return;

    if (z == 0 && warp == 0 && u.cnt > 0) {
        if (!GATHER) w_own = ap.w_new ? ap.w_new[unit] : 0.f;
        const bool safe = is_protected(ap, u, ap.pos_new ? ap.pos_new[unit] : u.seen);
        low = min(low, leave_order(safe ? kKeyProtected : weight_key(w_own), u.had));
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
    auto place = [&](const Unit &v, unsigned long long lowest, int l) {   // by a warp: K on one half, V on the other
        if (v.cnt == 0) return;
        int dst = v.had;
        if (v.had + v.cnt > v.final) {
            dst = (int)(0xFFFFFFFFu - (uint32_t)lowest);
            if (dst == v.had) return;            // the new row itself is the one that leaves
        }
        if (l < lpr) move_row(c, ap, v, dst, v.had, lpr, l);
    };
    int *arrived = c.state + kStateAppend + n;
    if (splits == 1) {
        if (simple) {
            if (warp == 0) place(u, sm_low[0], lane);
        } else {
            const int movers = select_unit<kRowThreads>(c, ap, u, sm_select, nullptr, 0);
            move_listed<kRowThreads>(c, ap, u, movers, lpr);
        }
        if (threadIdx.x == 0 && arrive(arrived) == c.H - 1) {
            *arrived = 0;
            c.lens[n] = u.final;
            c.seen[n] = u.seen + u.cnt;
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
            const int movers = select_unit<kRowThreads>(c, ap, v, sm_select, nullptr, 0);
            move_listed<kRowThreads>(c, ap, v, movers, lpr);
            __syncthreads();
        }
    }
    if (threadIdx.x == 0) {
        *arrived = 0;
        c.lens[n] = u.final;
        c.seen[n] = u.seen + u.cnt;
    }
}

// CTAs per unit of a rows launch: one round of rows each, up to about 16 CTAs per SM in all.
inline int row_splits(long long units, long long rows)
{
    long long z = (148LL * kRowCtas + units - 1) / units;
    const long long most = (rows + kRowThreads * kRowsHeld - 1) / (kRowThreads * kRowsHeld);
    if (z > most) z = most;
    if (z > kMaxSplits) z = kMaxSplits;
    return z < 1 ? 1 : (int)z;
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
        auto kernel = !append ? paged_rows_kernel<true, false> : gather ? paged_rows_kernel<true, true> : paged_rows_kernel<false, true>;
        return launch_chained(kernel, dim3((unsigned)(splits * units)), kRowThreads, g.G * sizeof(float2), stream, c, g, a, lpr, splits);
    }
    const bool few = a.T <= kFewRows;
    // Keys of budget + T candidates are held in shared memory up to 48K of them. Wide CTAs for long lists: one that a CTA of
    // 256 threads walks in 64 steps or more.
    const long long most_keys = (long long)a.budget + a.T;
    const int room = most_keys <= 48 * 1024 ? (int)most_keys : 0;
    const bool wide = most_keys >= 16 * 1024;
    auto kernel = wide ? paged_select_kernel<1024> : paged_select_kernel<256>;
    cudaError_t e = cudaSuccess;
    if (room > 10 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room * (int)sizeof(uint32_t));
    if (e == cudaSuccess)
        e = launch_chained(kernel, dim3((unsigned)units), wide ? 1024u : 256u, room * sizeof(uint32_t), stream, c, a, lpr, few ? 1 : 0, room);
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
