// What the tensor-core kernels over a paged cache share (attention of a chunk of new tokens, the weights that its
// queries leave behind): the chunk as a kernel argument, tiles of packed query rows, tiles of cached rows fetched page
// by page, and the plan that spreads a ragged batch evenly over one resident wave of CTAs.
//
// Query rows. The G query heads that share a key / value head meet the same rows, so a tile of 128 query rows holds
// floor(128 / G) consecutive tokens with their G heads side by side: row r = token r / G, head r % G. Where G does not
// divide 128 the last rows of a tile stay empty.
//
// Cached rows. A tile of 128 rows arrives in boxes of b rows, b the largest power of two that divides the page size
// (at most 128): a box never crosses a page. Boxes land at multiples of b * 128 bytes; the 128-byte swizzle goes by the
// address in shared memory, so boxes of fewer than 8 rows join the same pattern.
#pragma once

#include "ec_paged.cuh"
#include "ec_tc.cuh"

namespace ec {

struct ChunkArgs {
    PagedView c;
    const int *starts, *counts;                  // packed tokens of problem n: starts[n] .. starts[n] + counts[n]
    int tokens, Hq, G;                           // rows of the packed tensors
    int tile_tokens;                             // tokens of a 128-row query tile: 128 / G
    int box_rows;                                // rows of a copy of cached rows
    float scale_log2e;
    double inv_ctas;                             // 1 / CTAs of the launch
};

// Counters behind the state block's other ones: of the CTAs that share a unit, the first one's are counted up.
constexpr int kChunkMaxCtas = kPagedMaxCtas / 2;
constexpr int kChunkCounters = 4;                // teams of a CTA that finish on their own

cudaError_t launch_chunk_attention(const ChunkArgs &a, int D, int dtype, const void *q, int64_t q_token, int64_t q_head, void *out,
                                   int64_t out_token, int64_t out_head, float *lse, void *ws, cudaStream_t stream);
cudaError_t launch_chunk_weights(const ChunkArgs &a, int D, int dtype, const void *q, int64_t q_token, int64_t q_head, const float *lse,
                                 double decay, void *ws, cudaStream_t stream);
size_t chunk_attention_workspace_bytes(int D);
size_t chunk_weights_workspace_bytes();

namespace {

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}

// One problem of the chunk as the kernels see it; what the device arrays say is checked here and never followed blindly.
struct Problem {
    int start, count, len;
};

template <typename Args>
__device__ __forceinline__ Problem read_problem(const Args &a, int n)
{
    Problem p;
    p.start = a.starts[n];
    p.count = a.counts[n];
    p.len = max(read_len(a.c, n), 0);
    p.count = max(p.count, 0);
    if (p.count > 0 && (p.start < 0 || p.count > a.tokens - p.start)) {
        report_page(a.c);
        p.count = 0;
    }
    return p;
}

// A place in the batch's work. Work is counted in 64 bits (rows for the attention, tokens for the weights); every unit of
// it (a pair of query tiles of a head, a block of cached rows of a head) costs its contraction and a constant for what
// surrounds it. Costs have a closed form, so that no CTA has to walk over the units in front of its own:
//   U::units(a, p)             units of a head of problem p
//   U::before(a, p, units, i)  cost of its units 0 .. i - 1
template <typename U, typename Args>
__device__ __forceinline__ long long head_cost(const Args &a, const Problem &p)
{
    if (p.count == 0) return 0;
    const int units = U::units(a, p);
    return U::before(a, p, units, units);
}

// a / b for a quotient of less than 2^20: an estimate, put right (a division of 64 bits takes ten times as long).
__device__ __forceinline__ int quotient(long long a, long long b)
{
    int q = (int)__fdividef((float)a, (float)b);
    while ((q + 1) * b <= a) ++q;
    while (q * b > a) --q;
    return q;
}

struct Share {
    long long first, last, per;                  // the CTA's run of the work; first >= last: nothing to do
    int n;                                       // problem that holds `first`
    long long before;                            // cost in front of it
};

// Every CTA derives the same division from the lengths; a warp works it out, a lane sums a span of problems.
template <typename U, typename Args>
__device__ __forceinline__ Share make_share(const Args &a, long long least)
{
    const int N = a.c.N, lane = threadIdx.x & 31;
    const int span = (N + 31) >> 5;
    const int n0 = min(lane * span, N), n1 = min(n0 + span, N);
    long long mine = 0;
    for (int n = n0; n < n1; ++n) mine += head_cost<U>(a, read_problem(a, n)) * a.c.H;
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    const long long total = __shfl_sync(0xFFFFFFFFu, incl, 31);
    Share s;
    // any share that covers the work will do: no exact division
    s.per = max(least, (long long)((double)total * a.inv_ctas) + (total >> 50) + 1);
    s.first = s.per * blockIdx.x;
    s.last = min(total, s.first + s.per);
    s.n = 0;
    s.before = 0;
    if (s.first >= total) return s;
    long long at = incl - mine;
    int n = n0;
    const bool here = s.first >= at && s.first < incl;
    if (here) {
        for (; n < n1 - 1; ++n) {
            const long long cost = head_cost<U>(a, read_problem(a, n)) * a.c.H;
            if (s.first < at + cost) break;
            at += cost;
        }
    }
    const int src = __ffs(__ballot_sync(0xFFFFFFFFu, here)) - 1;
    s.n = __shfl_sync(0xFFFFFFFFu, n, src);
    s.before = __shfl_sync(0xFFFFFFFFu, at, src);
    return s;
}

// Walks the units of a CTA's share in order.
template <typename U>
struct Walk {
    Share s;
    Problem p;
    int n, h, i, units;
    long long at;                                // cost in front of the unit

    template <typename Args>
    __device__ __forceinline__ bool begin(const Args &a, long long least)
    {
        s = make_share<U>(a, least);
        if (s.first >= s.last) return false;
        n = s.n;
        p = read_problem(a, n);
        units = U::units(a, p);
        const long long head = U::before(a, p, units, units), in = s.first - s.before;
        h = quotient(in, head);
        const long long rest = in - h * head;
        int lo = 0, hi = units - 1;              // the last unit that does not begin behind `rest`
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (U::before(a, p, units, mid) <= rest) lo = mid;
            else hi = mid - 1;
        }
        i = lo;
        at = s.before + h * head + U::before(a, p, units, i);
        return true;
    }

    // false: the share ends here
    template <typename Args>
    __device__ __forceinline__ bool next(const Args &a, long long cost)
    {
        at += cost;
        if (at >= s.last) return false;
        if (++i < units) return true;
        i = 0;
        if (++h < a.c.H) return true;
        h = 0;
        do {
            if (++n >= a.c.N) return false;
            p = read_problem(a, n);
        } while (head_cost<U>(a, p) == 0);
        units = U::units(a, p);
        return true;
    }
};

// What this CTA has of a unit: its tiles t0 .. t1 - 1 (the unit's are 0 .. tiles - 1), and, where the unit is shared, with whom.
struct Cut {
    bool mine;                                   // false: nothing, another CTA sees to it
    int t0, t1;
    int first, parts;                            // parts > 0: CTAs first .. first + parts - 1 share it
};

// The unit lies at `at` in the work, costs `fixed` and `grain` a tile. Short units are not shared (handing parts over takes as long as
// some tiles do): the CTA that holds their middle has them. Of the others every CTA that takes part has a tile at least.
constexpr int kWholeTiles = 3;

__device__ __forceinline__ Cut cut_unit(const Share &s, long long at, long long cost, int fixed, int grain, int tiles)
{
    const int me = (int)blockIdx.x;
    Cut cut;
    cut.t0 = 0;
    cut.t1 = tiles;
    cut.parts = 0;
    if (tiles <= kWholeTiles) {
        cut.first = quotient(at + min(cost, (long long)fixed + tiles * grain / 2) - 1, s.per);
        cut.mine = cut.first == me;
        return cut;
    }
    cut.first = quotient(at + fixed + grain - 1, s.per);
    const int last = quotient(at + min(cost, fixed + (long long)grain * tiles) - 1, s.per);
    auto tile_at = [&](int cta) {                // the tile that holds the CTA's first place, which is the CTA's own
        const long long x = cta * s.per - at - fixed;
        return x <= 0 ? 0 : min((int)((unsigned)x / (unsigned)grain), tiles);
    };
    cut.mine = me >= cut.first && me <= last;
    if (me > cut.first) cut.t0 = tile_at(me);
    if (me < last) cut.t1 = tile_at(me + 1);
    if (last > cut.first) cut.parts = last - cut.first + 1;
    return cut;
}

inline int box_rows_of(int page_size)
{
    int b = 1;
    while (b < kTileRows && page_size % (2 * b) == 0) b *= 2;
    return b;
}

inline bool encode(CUtensorMap *map, int dtype, const void *ptr, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                   const cuuint32_t *box)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return fn(map, dtype == EC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
              const_cast<void *>(ptr), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Packed queries [tokens, Hq, D] by strides: a box is 64 columns of the G heads of a group of tile_tokens tokens.
// Tokens past the tensor read as zeros.
inline bool make_query_map(CUtensorMap *map, const ChunkArgs &a, int D, int dtype, const void *q, int64_t token, int64_t head)
{
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.Hq, (cuuint64_t)a.tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)head * 2, (cuuint64_t)token * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)a.tile_tokens};
    return encode(map, dtype, q, 3, dims, strides, box);
}

// A pool of pages: a box is 64 columns of box_rows rows of a head in one page.
inline bool make_pool_map(CUtensorMap *map, const ChunkArgs &a, int D, int dtype, const void *pool)
{
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)a.c.page_size, (cuuint64_t)a.c.H, (cuuint64_t)a.c.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)a.c.row_step * 16, (cuuint64_t)a.c.head_step * 16, (cuuint64_t)a.c.page_step * 16};
    const cuuint32_t box[4] = {64, (cuuint32_t)a.box_rows, 1, 1};
    return encode(map, dtype, pool, 4, dims, strides, box);
}

inline int chunk_grid()
{
    const int n = sm_count();
    return n < kChunkMaxCtas ? n : kChunkMaxCtas;
}

// The page of a box of rows: -1 behind the last row that is needed. A box of page -1 is copied like any other: it lies outside of the
// pool, and what arrives is zeros, so that every tile brings the same number of bytes.
__device__ __forceinline__ int box_page(const ChunkArgs &a, int n, int row, int rows) { return row < rows ? look_up_slot(a.c, n, row).page : -1; }

// Turns an entry outside the pool into -1 and reports it. True when there was one.
__device__ __forceinline__ bool bad_page(const ChunkArgs &a, int row, int rows, int &page)
{
    if (row >= rows || (unsigned)page < (unsigned)a.c.n_pages) return false;
    page = -1;
    report_page(a.c);
    return true;
}

// Starts the copies of one box to row `at` of the tile at dst.
template <int D>
__device__ __forceinline__ void copy_box(const ChunkArgs &a, const CUtensorMap *map, int page, int h, int row, int at, uint32_t dst, uint32_t bar)
{
    const int slot = row - page_of(a.c, row) * a.c.page_size;
#pragma unroll
    for (int half = 0; half < D / 64; ++half)
        tma_load_4d(dst + half * (kTileRows * 128) + at * 128, map, half * 64, slot, h, page, bar);
}

// Plain shared-memory stores seen by the tensor cores' reads that a later arrival lets go ahead.
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

}  // namespace

}  // namespace ec
