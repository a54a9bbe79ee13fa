// What the kernels of the paged cache share: the cache as a kernel argument, the address arithmetic of its
// pages and the packed element types.
#pragma once

#include "ec_common.cuh"

#include <cuda_fp16.h>

namespace ec {

namespace {

constexpr uint32_t kRowNone = 0xFFFFFFFFu;   // no row here: not read, no weight
constexpr uint32_t kRowNew = 0xFFFFFFFEu;    // the step's own row, read from the call's inputs

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Kernel launch that may be placed while the previous kernel of the stream drains; every kernel launched
// this way waits (grid_wait) before its first access to memory that an earlier kernel may write.
template <typename... KArgs, typename... Args>
cudaError_t launch_chained(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace

// CTAs of an attention launch at most, and where the arrival counters lie in the state block (in ints behind the
// status word). Every counter is zero between launches: whoever arrives last puts it back.
constexpr int kPagedMaxCtas = 148 * 2;
constexpr int kStateAttention = 64;
constexpr int kStateChunk = kStateAttention + kPagedMaxCtas;       // four per CTA of a chunk's launches, see ec_chunk.cuh
constexpr int kStateAppend = kStateChunk + 2 * kPagedMaxCtas;      // one per problem

// The cache as the kernels take it. Offsets of rows are counted in 16-byte units, in 32 bits: the host refuses
// pools that reach past 2^32 - 2 of them (64 GiB for K and as much for V).
struct PagedView {
    uint4 *K, *V;
    float *weight;
    int *pos;
    const int *table;
    int *lens, *seen;
    int *state;                                  // status word and arrival counters, see kState*
    int N, H, page_size, n_pages, max_pages;
    uint32_t page_step, head_step, row_step;     // strides in 16-byte units
    uint32_t div_mul, div_shift;                 // row / page_size, see page_of
};

// row / page_size for 0 <= row < 2^31 as a multiplication: with 2^(l-1) < d <= 2^l and mul = ceil(2^(31+l) / d), mul * d
// exceeds 2^(31+l) by less than d <= 2^l, so the quotient is off by less than row * 2^l / (2^(31+l) d) < 1 / d: never
// enough to reach the next whole number.
inline void set_page_division(PagedView &c)
{
    uint32_t l = 0;
    while ((1u << l) < (uint32_t)c.page_size) ++l;
    c.div_shift = 31 + l;
    c.div_mul = (uint32_t)(((1ull << c.div_shift) + (uint32_t)c.page_size - 1) / (uint32_t)c.page_size);
}

namespace {

// Counts the CTA in at a counter (to be called by one thread, behind a block barrier): what the CTA wrote before is visible
// to whoever arrives later, what the others wrote before is visible to this CTA behind the next block barrier.
__device__ __forceinline__ int arrive(int *counter)
{
    int before;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
    return before;
}

__device__ __forceinline__ int page_of(const PagedView &c, int row)
{
    return (int)(((unsigned long long)(uint32_t)row * c.div_mul) >> c.div_shift);
}

struct Slot {
    int page, slot;        // page < 0: the table has no valid page here
};

// AHEAD: a read in front of the launch's wait, from the L2: an L1 may still hold what it read for an earlier launch.
template <bool AHEAD, typename T>
__device__ __forceinline__ T read_at(const T *p) { return AHEAD ? __ldcg(p) : *p; }

// The table's entry as it is: to be looked at with valid_page before anything is read through it.
template <bool AHEAD = false>
__device__ __forceinline__ Slot look_up_slot(const PagedView &c, int n, int row)
{
    const int p = page_of(c, row);
    Slot s;
    s.slot = row - p * c.page_size;
    s.page = read_at<AHEAD>(c.table + (size_t)n * c.max_pages + p);
    return s;
}

__device__ __forceinline__ bool valid_page(const PagedView &c, const Slot &s) { return (unsigned)s.page < (unsigned)c.n_pages; }

__device__ __forceinline__ void report_page(const PagedView &c) { atomicExch(c.state, kStatusPage); }

template <bool AHEAD = false>
__device__ __forceinline__ Slot find_slot(const PagedView &c, int n, int row)
{
    Slot s = look_up_slot<AHEAD>(c, n, row);
    if (!valid_page(c, s)) {
        s.page = -1;
        report_page(c);
    }
    return s;
}

// Index of a row's weight and position; fits 32 bits (checked by the host).
__device__ __forceinline__ uint32_t meta_index(const PagedView &c, int h, const Slot &s)
{
    return ((uint32_t)s.page * (uint32_t)c.H + (uint32_t)h) * (uint32_t)c.page_size + (uint32_t)s.slot;
}

// Offset of a row of head 0 in the pools, in 16-byte units.
__device__ __forceinline__ uint32_t row_offset(const PagedView &c, const Slot &s)
{
    return (uint32_t)s.page * c.page_step + (uint32_t)s.slot * c.row_step;
}

// Valid rows of problem n: negative for an empty place; a length past the table's reach is cut and reported.
template <bool AHEAD = false>
__device__ __forceinline__ int read_len(const PagedView &c, int n)
{
    const int len = read_at<AHEAD>(c.lens + n);
    const long long cap = (long long)c.max_pages * c.page_size;
    if (len > cap) {
        atomicExch(c.state, kStatusPage);
        return (int)cap;
    }
    return len;
}

}  // namespace

// Where the scores of an attention call lie: as the pages do, [n_pages, H, G, page_size], or row by row, [N, H, G,
// max_pages * page_size]. The first needs no more room than the pool has rows. Pages of fewer than 8 rows scatter it in
// pieces of less than 32 bytes, which memory takes several times longer to write (27 sequences of up to 20185 rows in
// pages of one row: 81 us a call, 30 us row by row).
inline __host__ __device__ bool scores_by_row(int page_size) { return page_size < 8; }

// What turns an attention call's stored scores into weights: p = 2^((score - .x) * scale_log2e) * .y.
struct GatherArgs {
    const float2 *stat;                          // [N, Hq] (the largest score, factor); the factor is 0 where no row is left
    const float *scores;                         // <q, k>, not scaled, see scores_by_row
    const float *score_new;                      // [N, Hq] the same of the step's own row
    float *w_new;                                // [N, H]; nullptr: the step has no row of its own
    float scale_log2e, decay;
    int G;
};

struct AppendArgs {
    const uint4 *K_new, *V_new;
    const float *w_new;
    const int *pos_new, *counts;
    int T, fresh, budget, recent, sinks;
    int4 *moves;                                 // workspace: [N * H] rows to move, and what the unit was
    int2 *list;                                  // workspace: [N * H][budget]: .x = slot to fill, .y = candidate to take
    unsigned long long *lowest;                  // workspace: [N * H][splits] first row to leave of every part
};

size_t paged_attention_workspace_bytes(const ec_paged *c, int Hq, int accumulate);
// accumulate: *gather is filled for the launch that adds the probabilities to the weights.
cudaError_t launch_paged_attention(const PagedView &c, int D, int dtype, const void *q, const void *k_new, const void *v_new,
                                   int Hq, float scale, int accumulate, float decay, void *out, float *lse, float *w_new,
                                   void *ws, GatherArgs *gather, cudaStream_t stream);
size_t paged_append_workspace_bytes(const ec_paged *c, int T, int budget);
// Either may be nullptr, not both. With both, append->w_new is gather->w_new.
cudaError_t launch_paged_rows(const PagedView &c, int D, const GatherArgs *gather, AppendArgs *append, void *ws_append,
                              cudaStream_t stream);

}  // namespace ec
