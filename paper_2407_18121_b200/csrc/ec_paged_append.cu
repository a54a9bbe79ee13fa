// New rows join a paged cache; heads that then hold more than `budget` rows give up those of smallest gathered weight.
// One CTA per (problem, head) decides, in three steps:
//   1. keys: order-preserving unsigned image of every candidate's weight (cached rows in slot order, then the new rows);
//      rows at protected positions get the largest key;
//   2. the key of the last row that leaves: radix descent over 8-bit digits with a histogram in shared memory. Equal
//      keys: the higher candidate leaves first;
//   3. an ordered pass that lists the holes below the new length and the kept rows that have to move there (kept rows
//      never shift, so only as many rows move as join or sit behind the new length).
// Bound by latency for a step's single row (8 bytes per cached row are read, one row per head is written) and by the copied
// rows for a prompt, which a second launch moves with all CTAs of the GPU.
#include "ec_paged.cuh"

namespace ec {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kFewRows = 16;                     // up to this many new rows the deciding CTA moves them itself

constexpr uint32_t kKeyProtected = 0xFFFFFFFFu, kKeyNan = 0xFFFFFFFEu;

// Order-preserving image of a weight: -inf lowest, -0 = +0, NaN above +inf.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return kKeyNan;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct AppendArgs {
    PagedView c;
    const uint4 *K_new, *V_new;
    const float *w_new;
    const int *pos_new, *counts;
    int T, fresh, budget, recent, sinks;
    int *moves;                                  // [N * H] rows to move
    int2 *list;                                  // [N * H][budget]: .x = slot to fill, .y = candidate to take
};

struct Unit {
    int n, h, had, cnt, final, seen;
    size_t u;
};

__device__ __forceinline__ uint32_t candidate_key(const AppendArgs &a, const Unit &u, int j)
{
    float w;
    int pos;
    if (j < u.had) {
        const Slot s = find_slot(a.c, u.n, j);
        if (s.page < 0) return 0;                // a row that cannot be read leaves first
        const uint32_t m = meta_index(a.c, u.h, s);
        w = a.c.weight[m];
        pos = a.c.pos[m];
    } else {
        const size_t at = u.u * a.T + (j - u.had);
        w = a.w_new ? a.w_new[at] : 0.f;
        pos = a.pos_new ? a.pos_new[at] : u.seen + (j - u.had);
    }
    const bool safe = pos < a.sinks || (long long)pos >= (long long)u.seen + u.cnt - a.recent;
    return safe ? kKeyProtected : weight_key(w);
}

// Row j of the candidates -> slot `dst`, by LPR = D / 8 lanes of which this is lane l.
__device__ __forceinline__ void move_row(const AppendArgs &a, const Unit &u, int dst, int j, int lpr, int l)
{
    const Slot d = find_slot(a.c, u.n, dst);
    if (d.page < 0) return;
    const size_t to = (size_t)u.h * a.c.head_step + row_offset(a.c, d) + l;
    const uint32_t meta_to = meta_index(a.c, u.h, d);
    const uint4 *k, *v;
    float w;
    int pos;
    if (j < u.had) {
        const Slot s = find_slot(a.c, u.n, j);
        if (s.page < 0) return;
        const size_t from = (size_t)u.h * a.c.head_step + row_offset(a.c, s) + l;
        k = a.c.K + from;
        v = a.c.V + from;
        const uint32_t m = meta_index(a.c, u.h, s);
        w = a.c.weight[m];
        pos = a.c.pos[m];
    } else {
        const size_t at = u.u * a.T + (j - u.had);
        k = a.K_new + at * lpr + l;
        v = a.V_new + at * lpr + l;
        w = a.w_new ? a.w_new[at] : 0.f;
        pos = a.pos_new ? a.pos_new[at] : u.seen + (j - u.had);
    }
    const uint4 kv = *k, vv = *v;
    a.c.K[to] = kv;
    a.c.V[to] = vv;
    if (l == 0) {
        a.c.weight[meta_to] = w;
        a.c.pos[meta_to] = pos;
    }
}

// Exclusive prefix of a flag over the block; returns it and adds the block's count to `total` (uniform).
__device__ __forceinline__ int block_prefix(bool flag, int *warp_counts, int &total)
{
    const unsigned mask = __ballot_sync(0xFFFFFFFFu, flag);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                             // the previous use of warp_counts is over
    if (lane == 0) warp_counts[warp] = __popc(mask);
    __syncthreads();
    int before = total, sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += warp_counts[w];
        sum += warp_counts[w];
    }
    total += sum;
    return before + __popc(mask & ((1u << lane) - 1u));
}

__device__ __forceinline__ Unit load_unit(const AppendArgs &a, int n, int h)
{
    Unit u;
    u.n = n;
    u.h = h;
    u.u = (size_t)n * a.c.H + h;
    const int len = read_len(a.c, n);
    if (len < 0) {
        u.had = u.cnt = u.final = -1;
        u.seen = 0;
        return u;
    }
    u.had = a.fresh ? 0 : len;
    u.seen = a.fresh ? 0 : a.c.seen[n];
    int cnt = a.counts ? a.counts[n] : a.T;
    u.cnt = min(max(cnt, 0), a.T);
    u.final = (int)min((long long)u.had + u.cnt, (long long)a.budget);
    return u;
}

__global__ void __launch_bounds__(kThreads) paged_select_kernel(AppendArgs a, int lpr, int move_here)
{
    __shared__ int hist[256];
    __shared__ int warp_counts[kWarps];
    __shared__ uint32_t sm_digit;
    __shared__ int sm_left;
    grid_wait();
    grid_release();
    const int n = blockIdx.x / a.c.H, h = blockIdx.x - n * a.c.H;
    const Unit u = load_unit(a, n, h);
    if (u.had < 0) {                             // an empty place of the batch
        if (threadIdx.x == 0) a.moves[u.u] = 0;
        return;
    }
    const int all = u.had + u.cnt, leave = all - u.final;
    uint32_t edge = 0;                           // rows with a smaller key leave, `left` of those with this key
    int left = 0, equal_kept = 0;
    if (leave > 0) {
        left = leave;
#pragma unroll 1
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += kThreads) hist[i] = 0;
            __syncthreads();
            const uint32_t high = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
            for (int j = threadIdx.x; j < all; j += kThreads) {
                const uint32_t key = candidate_key(a, u, j);
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
                        const int c = hist[threadIdx.x * 8 + i];
                        if (at + c >= left) {
                            sm_digit = threadIdx.x * 8 + i;
                            sm_left = left - at;
                            equal_kept = c;
                            break;
                        }
                        at += c;
                    }
                    hist[0] = equal_kept;        // rows with the edge key, for the last digit
                }
            }
            __syncthreads();
            edge |= sm_digit << shift;
            left = sm_left;
            equal_kept = hist[0] - left;         // after the last digit: of the rows at the edge the first ones stay
            __syncthreads();
        }
    }
    // ordered pass: k-th hole <- k-th kept row from behind
    int equals = 0, holes = 0, movers = 0;
    int2 *list = a.list + u.u * a.budget;
    for (int base = 0; base < all; base += kThreads) {
        const int j = base + threadIdx.x;
        bool stay = j < all, equal = false;
        if (leave > 0 && j < all) {
            const uint32_t key = candidate_key(a, u, j);
            equal = key == edge;
            stay = key > edge;
        }
        if (leave > 0) {
            const int rank = block_prefix(equal, warp_counts, equals);
            if (equal) stay = rank < equal_kept;
        }
        const bool low = j < u.had && j < u.final;
        const bool hole = low && !stay, mover = j < all && stay && !low;
        const int hk = block_prefix(hole, warp_counts, holes);
        const int mk = block_prefix(mover, warp_counts, movers);
        if (hole) list[hk].x = j;
        if (mover) list[mk].y = j;
    }
    for (int s = u.had + threadIdx.x; s < u.final; s += kThreads) list[holes + (s - u.had)].x = s;   // slots behind the old length
    if (threadIdx.x == 0) a.moves[u.u] = movers;
    if (move_here) {
        __syncthreads();                         // the list is complete, every key has been read
        const int group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
        for (int k = group; k < movers; k += kThreads / lpr) {
            const int2 e = list[k];
            move_row(a, u, e.x, e.y, lpr, l);
        }
    }
}

// `parts` CTAs per unit: the listed rows of every unit.
__global__ void __launch_bounds__(kThreads) paged_move_kernel(AppendArgs a, int lpr, int parts)
{
    grid_wait();
    grid_release();
    const int unit = blockIdx.x / parts, part = blockIdx.x - unit * parts;
    const int n = unit / a.c.H, h = unit - n * a.c.H;
    const Unit u = load_unit(a, n, h);
    if (u.had < 0) return;
    const int movers = a.moves[u.u];
    const int groups = kThreads / lpr, group = threadIdx.x / lpr, l = threadIdx.x - group * lpr;
    const int2 *list = a.list + u.u * a.budget;
    for (int k = part * groups + group; k < movers; k += parts * groups) {
        const int2 e = list[k];
        move_row(a, u, e.x, e.y, lpr, l);
    }
}

// The lengths change when every unit of their problem has been dealt with: a launch of its own.
__global__ void paged_commit_kernel(AppendArgs a)
{
    grid_wait();
    grid_release();
    const int n = blockIdx.x * blockDim.x + threadIdx.x;
    if (n >= a.c.N) return;
    const Unit u = load_unit(a, n, 0);
    if (u.had < 0) return;
    a.c.lens[n] = u.final;
    a.c.seen[n] = u.seen + u.cnt;
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t paged_append_workspace_bytes(const ec_paged *c, int T, int budget)
{
    (void)T;
    const size_t units = (size_t)c->N * c->H;
    return up256(units * sizeof(int)) + up256(units * budget * sizeof(int2));
}

cudaError_t launch_paged_append(const PagedView &c, int D, const void *K_new, const void *V_new, const float *w_new,
                                const int *pos_new, const int *counts, int T, int fresh, int budget, int recent, int sinks,
                                void *ws, cudaStream_t stream)
{
    AppendArgs a;
    a.c = c;
    a.K_new = static_cast<const uint4 *>(K_new);
    a.V_new = static_cast<const uint4 *>(V_new);
    a.w_new = w_new;
    a.pos_new = pos_new;
    a.counts = counts;
    a.T = T;
    a.fresh = fresh;
    a.budget = budget;
    a.recent = recent;
    a.sinks = sinks;
    const size_t units = (size_t)c.N * c.H;
    a.moves = static_cast<int *>(ws);
    a.list = reinterpret_cast<int2 *>(static_cast<char *>(ws) + up256(units * sizeof(int)));
    const int lpr = D / 8;
    const bool few = T <= kFewRows;
    cudaError_t e = launch_chained(paged_select_kernel, dim3((unsigned)units), kThreads, 0, stream, a, lpr, few ? 1 : 0);
    if (e == cudaSuccess && !few) {
        const int groups = kThreads / lpr;
        long long parts = (148LL * 8 + units - 1) / units;
        const long long most = ((long long)budget + groups - 1) / groups;
        if (parts > most) parts = most;
        e = launch_chained(paged_move_kernel, dim3((unsigned)(parts * units)), kThreads, 0, stream, a, lpr, (int)parts);
    }
    if (e == cudaSuccess) e = launch_chained(paged_commit_kernel, dim3((unsigned)((c.N + 127) / 128)), 128, 0, stream, a);
    return e;
}

}  // namespace ec
