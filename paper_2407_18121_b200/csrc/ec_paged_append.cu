// What happens to the rows of a paged cache around the attention: the step's probabilities are added to the weights, new
// rows join, and heads that then hold more than `budget` rows give up those of smallest gathered weight.
//  - One new row (a generation step): one launch does all of it. A row's new weight is on hand when the row that leaves is
//    looked for, so the weights are read once; the search is a minimum over (key, row). Bound by latency: a chain of
//    length, page, score and weight reads, which every thread walks for several rows side by side.
//  - More new rows (a prompt): a CTA per (problem, head) finds the key of the last row that leaves by radix descent over
//    8-bit digits and lists, in an ordered pass, the holes below the new length and the kept rows that have to move there
//    (kept rows never shift, so only as many rows move as join or sit behind the new length); a second launch moves them
//    with all CTAs of the GPU, bound by the copied bytes.
// Keys are order-preserving unsigned images of the weights; rows at protected positions get the largest key. Equal keys:
// the higher candidate leaves first (cached rows in slot order, then the new rows).
#include "ec_paged.cuh"

namespace ec {

namespace {

constexpr int kThreads = 256;
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

// Exclusive prefix of a flag over the block; returns it and adds the block's count to `total` (uniform).
template <int THREADS>
__device__ __forceinline__ int block_prefix(bool flag, int *warp_counts, int &total)
{
    const unsigned mask = __ballot_sync(0xFFFFFFFFu, flag);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                             // the previous use of warp_counts is over
    if (lane == 0) warp_counts[warp] = __popc(mask);
    __syncthreads();
    int before = total, sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += warp_counts[w];
        sum += warp_counts[w];
    }
    total += sum;
    return before + __popc(mask & ((1u << lane) - 1u));
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

template <int THREADS> struct SelectSmem {
    int hist[256];
    int warp_counts[THREADS / 32];
    uint32_t digit;
    int left;
};

// The whole CTA: lists the moves of unit u (slot to fill, candidate to take) and returns their number.
template <int THREADS>
__device__ __forceinline__ int select_unit(const PagedView &c, const AppendArgs &a, const Unit &u, SelectSmem<THREADS> &sm)
{
    int *hist = sm.hist, *warp_counts = sm.warp_counts;
    const int all = u.had + u.cnt, leave = all - u.final;
    uint32_t edge = 0;                           // rows with a smaller key leave, `left` of those with this key
    int left = 0, equal_kept = 0;
    if (leave > 0) {
        left = leave;
#pragma unroll 1
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += THREADS) hist[i] = 0;
            __syncthreads();
            const uint32_t high = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
            for (int j = threadIdx.x; j < all; j += THREADS) {
                const uint32_t key = candidate_key(c, a, u, j);
                if ((key & high) == edge) atomicAdd(&hist[(key >> shift) & 255u], 1);
            }
            __syncthreads();
            if (threadIdx.x < 32) {              // the digit in which the running count passes `left`
                int sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += hist[threadIdx.x * 8 + i];
                int incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                    if (threadIdx.x >= o) incl += up;
                }
                int at = incl - sum;
                if (at < left && left <= incl) {
                    for (int i = 0; i < 8; ++i) {
                        const int here = hist[threadIdx.x * 8 + i];
                        if (at + here >= left) {
                            sm.digit = threadIdx.x * 8 + i;
                            sm.left = left - at;
                            equal_kept = here;
                            break;
                        }
                        at += here;
                    }
                    hist[0] = equal_kept;        // rows with the edge key, for the last digit
                }
            }
            __syncthreads();
            edge |= sm.digit << shift;
            left = sm.left;
            equal_kept = hist[0] - left;         // after the last digit: of the rows at the edge the first ones stay
            __syncthreads();
        }
    }
    // ordered pass: k-th hole <- k-th kept row from behind
    int equals = 0, holes = 0, movers = 0;
    int2 *list = a.list + u.u * a.budget;
    for (int base = 0; base < all; base += THREADS) {
        const int j = base + threadIdx.x;
        bool stay = j < all, equal = false;
        if (leave > 0 && j < all) {
            const uint32_t key = candidate_key(c, a, u, j);
            equal = key == edge;
            stay = key > edge;
        }
        if (leave > 0) {
            const int rank = block_prefix<THREADS>(equal, warp_counts, equals);
            if (equal) stay = rank < equal_kept;
        }
        const bool low = j < u.had && j < u.final;
        const bool hole = low && !stay, mover = j < all && stay && !low;
        const int hk = block_prefix<THREADS>(hole, warp_counts, holes);
        const int mk = block_prefix<THREADS>(mover, warp_counts, movers);
        if (hole) list[hk].x = j;
        if (mover) list[mk].y = j;
    }
    for (int s = u.had + threadIdx.x; s < u.final; s += THREADS) list[holes + (s - u.had)].x = s;   // slots behind the old length
    __syncthreads();                             // the list is complete, every key has been read
    return movers;
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

__global__ void __launch_bounds__(kThreads) paged_select_kernel(PagedView c, AppendArgs a, int lpr, int move_here)
{
    __shared__ SelectSmem<kThreads> sm;
    grid_wait();
    grid_release();
    const int n = blockIdx.x / c.H, h = blockIdx.x - n * c.H;
    const Unit u = load_unit(c, a, n, h);
    if (u.had < 0) {                             // an empty place of the batch
        if (threadIdx.x == 0) a.moves[u.u] = 0;
        return;
    }
    const int movers = select_unit<kThreads>(c, a, u, sm);
    if (threadIdx.x == 0) a.moves[u.u] = movers;
    if (move_here) move_listed<kThreads>(c, a, u, movers, lpr);
}

// `parts` CTAs per unit: the listed rows of every unit.
__global__ void __launch_bounds__(kThreads) paged_move_kernel(PagedView c, AppendArgs a, int lpr, int parts)
{
    grid_wait();
    grid_release();
    const int unit = blockIdx.x / parts, part = blockIdx.x - unit * parts;
    const int n = unit / c.H, h = unit - n * c.H;
    const Unit u = load_unit(c, a, n, h);
    if (u.had < 0) return;
    const int movers = a.moves[u.u];
    const int groups = kThreads / lpr, group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
    const int2 *list = a.list + u.u * a.budget;
    for (int k = part * groups + group; k < movers; k += parts * groups) {
        const int2 e = list[k];
        move_row(c, a, u, e.x, e.y, lpr, l);
    }
}

// The lengths change when every unit of their problem has been dealt with: a launch of its own.
__global__ void paged_commit_kernel(PagedView c, AppendArgs a)
{
    grid_wait();
    grid_release();
    const int n = blockIdx.x * blockDim.x + threadIdx.x;
    if (n >= c.N) return;
    const Unit u = load_unit(c, a, n, 0);
    if (u.had < 0) return;
    c.lens[n] = u.final;
    c.seen[n] = u.seen + u.cnt;
}

constexpr int kRowThreads = 128;
#ifndef EC_RC
#define EC_RC 8
#endif
constexpr int kRowCtas = EC_RC;                      // per SM
constexpr int kScoresHeld = 4;                   // query heads whose scores a thread reads side by side
constexpr int kRowsHeld = 4;                      // rows a thread has in flight

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
            const int movers = select_unit<kRowThreads>(c, ap, u, sm_select);
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
            const int movers = select_unit<kRowThreads>(c, ap, v, sm_select);
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
    return up256(units * sizeof(int)) + up256(units * budget * sizeof(int2)) +
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
        a.moves = reinterpret_cast<int *>(p);
        p += up256(units * sizeof(int));
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
    cudaError_t e = launch_chained(paged_select_kernel, dim3((unsigned)units), kThreads, 0, stream, c, a, lpr, few ? 1 : 0);
    if (e == cudaSuccess && !few) {
        const int groups = kThreads / lpr;
        long long parts = (148LL * 8 + units - 1) / units;
        const long long most = ((long long)a.budget + groups - 1) / groups;
        if (parts > most) parts = most;
        e = launch_chained(paged_move_kernel, dim3((unsigned)(parts * units)), kThreads, 0, stream, c, a, lpr, (int)parts);
    }
    if (e == cudaSuccess) e = launch_chained(paged_commit_kernel, dim3((unsigned)((c.N + 127) / 128)), 128, 0, stream, c, a);
    return e;
}

}  // namespace ec
