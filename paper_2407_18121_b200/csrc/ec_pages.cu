// Pages of a paged cache, handed out from a stack on the device and taken back: block tables, and for every new token the slot of
// its row. Latency is all there is: a handful of dependent reads and two scans over the problems.
//   release   a problem keeps ceil(lens / page_size) pages (none at an empty place); the others go on the stack, problem by problem
//   reserve   problems in order take the pages that their new rows need off the top of the stack, until it holds too few
// Every CTA of a reserve scans all problems itself (1024 at a time), and then writes its part of the tokens and of the table: no
// second launch has to wait for a plan. The arrays that the scan reads change when the last CTA has arrived.
// Eight problems, release and reserve: 8.3 us of the GPU in a graph, 16 called from a program; 512 problems with 12000 tokens 13.4 and
// 17. The bytes (0.1 MB) would take 0.02 us.
#include "ec_rotary.cuh"

namespace ec {

namespace {

constexpr int kThreads = 1024;
constexpr int kStatePages = 32;                  // arrival counter, in the status block; zero between launches

// Inclusive sums over the block of two values; both totals to every thread.
struct Sums {
    long long a;
    int b;
};

__device__ __forceinline__ Sums block_scan(Sums v, Sums &total, Sums *warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xFFFFFFFFu, v.a, o);
        const int b = __shfl_up_sync(0xFFFFFFFFu, v.b, o);
        if (lane >= o) { v.a += a; v.b += b; }
    }
    __syncthreads();                             // the sums of the call before have been read
    if (lane == 31) warps[warp] = v;
    __syncthreads();
    Sums w = warps[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xFFFFFFFFu, w.a, o);
        const int b = __shfl_up_sync(0xFFFFFFFFu, w.b, o);
        if (lane >= o) { w.a += a; w.b += b; }
    }
    total.a = __shfl_sync(0xFFFFFFFFu, w.a, 31);
    total.b = __shfl_sync(0xFFFFFFFFu, w.b, 31);
    const long long pa = __shfl_sync(0xFFFFFFFFu, w.a, (warp + 31) & 31);
    const int pb = __shfl_sync(0xFFFFFFFFu, w.b, (warp + 31) & 31);
    if (warp > 0) { v.a += pa; v.b += pb; }
    return v;
}

// The last of the `many` entries that is not above x (entries ascend, the first is not above x).
__device__ __forceinline__ int owner_of(const int *begin, int many, int x)
{
    int lo = 0, hi = many - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (begin[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ int height_of(const PagedView &c, const PagePool &p)
{
    const int h = *p.n_free;
    if (h < 0 || h > c.n_pages) {
        report_page(c);
        return max(0, min(h, c.n_pages));
    }
    return h;
}

__device__ __forceinline__ int held_of(const PagedView &c, const PagePool &p, int n)
{
    const int h = p.held[n];
    if (h < 0 || h > c.max_pages) {
        report_page(c);
        return -1;
    }
    return h;
}

__device__ __forceinline__ long long rows_wanted(const ReserveArgs &a, int len, int cnt)
{
    const long long rows = (long long)len + cnt;
    return !a.advance && a.limit > 0 ? min(rows, (long long)max(a.limit, len)) : rows;
}

__device__ __forceinline__ int pages_for(const PagedView &c, long long rows) { return (int)((rows + c.page_size - 1) / c.page_size); }

__global__ void __launch_bounds__(kThreads)
reserve_kernel(const PagedView c, const PagePool p, const ReserveArgs a)
{
    __shared__ Sums warps[32];
    __shared__ int s_start[kThreads], s_cnt[kThreads], s_len[kThreads], s_held[kThreads], s_seen[kThreads], s_base[kThreads];
    __shared__ int s_last;
    grid_wait();
    grid_release();
    const int tid = threadIdx.x, height = height_of(c, p);
    const long long cap = (long long)c.max_pages * c.page_size;
    long long tokens = 0;                        // of the problems in front of this tile
    int pages = 0;
    for (int n0 = 0; n0 < c.N; n0 += kThreads) {
        const int n = n0 + tid, many = min(kThreads, c.N - n0);
        int cnt = 0, len = -1, held = -1, seen = 0;
        if (n < c.N) {
            cnt = max(a.counts[n], 0);
            len = c.lens[n];
            held = held_of(c, p, n);
            seen = c.seen[n];
        }
        Sums total, v = {cnt, 0};
        const long long end = tokens + block_scan(v, total, warps).a;
        const long long next_tokens = tokens + total.a;
        const long long rows = rows_wanted(a, len, cnt);
        const bool fits = len >= 0 && held >= 0 && rows <= cap && (!a.advance || end <= a.tokens);
        const int need = fits && cnt > 0 ? max(0, pages_for(c, rows) - held) : 0;
        v = {0, need};
        const int upto = pages + block_scan(v, total, warps).b;
        const int next_pages = pages + total.b;
        const bool ok = fits && (need == 0 || upto <= height);
        s_start[tid] = (int)min(end - cnt, (long long)a.tokens);
        s_cnt[tid] = ok ? cnt : -cnt;            // negative: not granted
        s_len[tid] = len;
        s_held[tid] = held;
        s_seen[tid] = seen;
        s_base[tid] = upto - need;
        if (blockIdx.x == 0 && n < c.N) {
            if (a.starts) a.starts[n] = s_start[tid];
            a.granted[n] = ok ? cnt : 0;
            if (a.starts && n == c.N - 1) a.starts[c.N] = (int)min(end, (long long)a.tokens);
        }
        __syncthreads();
        if (a.slots || a.positions) {
            const int to = (int)min(next_tokens, (long long)a.tokens);
            for (long long t = min(tokens, (long long)a.tokens) + blockIdx.x * kThreads + tid; t < to; t += (long long)gridDim.x * kThreads) {
                const int i = owner_of(s_start, many, (int)t), in = (int)t - s_start[i];
                int slot = -1, pos = -1;
                if (in < s_cnt[i]) {
                    const int row = s_len[i] + in, pg = page_of(c, row);
                    const int page = pg < s_held[i] ? c.table[(size_t)(n0 + i) * c.max_pages + pg] : p.free[height - 1 - (s_base[i] + pg - s_held[i])];
                    if ((unsigned)page < (unsigned)c.n_pages) slot = page * c.page_size + row - pg * c.page_size;
                    else report_page(c);
                    pos = s_seen[i] + in;
                }
                if (a.slots) a.slots[t] = slot;
                if (a.positions) a.positions[t] = pos;
            }
        }
        const int to = min(next_pages, height);
        for (int g = pages + blockIdx.x * kThreads + tid; g < to; g += gridDim.x * kThreads) {
            const int i = owner_of(s_base, many, g);
            if (s_cnt[i] > 0) a.table[(size_t)(n0 + i) * c.max_pages + s_held[i] + g - s_base[i]] = p.free[height - 1 - g];
        }
        tokens = next_tokens;
        pages = next_pages;
        __syncthreads();
    }
    for (long long t = min(tokens, (long long)a.tokens) + blockIdx.x * kThreads + tid; t < a.tokens; t += (long long)gridDim.x * kThreads) {
        if (a.slots) a.slots[t] = -1;
        if (a.positions) a.positions[t] = -1;
    }
    // whoever arrives last brings the problems up to date: nobody reads them any more
    __syncthreads();
    if (tid == 0) {
        s_last = gridDim.x == 1 || arrive(c.state + kStatePages) == (int)gridDim.x - 1;
        if (s_last) c.state[kStatePages] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    int taken = 0;
    for (int n = tid; n < c.N; n += kThreads) {
        const int got = __ldcg(a.granted + n);
        if (got <= 0) continue;
        const int len = c.lens[n], held = p.held[n];
        const int need = max(0, pages_for(c, rows_wanted(a, len, got)) - held);
        taken += need;
        p.held[n] = held + need;
        if (a.advance) {
            a.lens[n] = len + got;
            a.seen[n] += got;
        }
    }
    Sums total, v = {0, taken};
    block_scan(v, total, warps);
    if (tid == 0) *p.n_free = height - total.b;
}

__global__ void __launch_bounds__(kThreads)
release_kernel(const PagedView c, const PagePool p)
{
    __shared__ Sums warps[32];
    __shared__ int s_base[kThreads], s_keep[kThreads];
    grid_wait();
    grid_release();
    const int tid = threadIdx.x, height = height_of(c, p);
    int pages = 0;
    for (int n0 = 0; n0 < c.N; n0 += kThreads) {
        const int n = n0 + tid, many = min(kThreads, c.N - n0);
        int held = 0, keep = 0;
        if (n < c.N) {
            held = held_of(c, p, n);
            keep = held < 0 ? held : min(held, pages_for(c, max(c.lens[n], 0)));
        }
        Sums total, v = {0, held - keep};
        const int base = pages + block_scan(v, total, warps).b - (held - keep);
        s_base[tid] = base;
        s_keep[tid] = keep;
        __syncthreads();
        const int to = pages + total.b;
        for (int g = pages + tid; g < to; g += kThreads) {
            const int i = owner_of(s_base, many, g);
            if (height + g < c.n_pages) p.free[height + g] = c.table[(size_t)(n0 + i) * c.max_pages + s_keep[i] + g - s_base[i]];
            else report_page(c);
        }
        if (n < c.N && keep < held) p.held[n] = keep;
        pages = to;
        __syncthreads();
    }
    if (tid == 0 && pages > 0) *p.n_free = min(height + pages, c.n_pages);
}

}  // namespace

cudaError_t launch_reserve(const PagedView &c, const PagePool &p, const ReserveArgs &a, cudaStream_t stream)
{
    // one CTA until its tokens take longer than the arrival of others
    // a token a thread: its search, table entry and store are a chain (12000 tokens of 512 problems: 13.4 us with the release and a copy
    // of the state in front; 14.5 with two tokens a thread, 20.2 with sixteen)
    const int ctas = a.slots || a.positions ? (a.tokens + kThreads - 1) / kThreads : 1;
    return launch_chained(reserve_kernel, dim3(ctas < 1 ? 1 : ctas > 64 ? 64 : ctas), kThreads, 0, stream, c, p, a);
}

cudaError_t launch_release(const PagedView &c, const PagePool &p, cudaStream_t stream)
{
    return launch_chained(release_kernel, dim3(1), kThreads, 0, stream, c, p);
}

}  // namespace ec
