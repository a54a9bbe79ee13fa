// Attention of one new token per problem over a paged cache (grouped query heads), with the probability every
// cached row receives added to the row's gathered weight.
//   x[g][j] = scale * <q_g, k_j>,  p = softmax_j(x),  out_g = sum_j p[g][j] v_j,  weight_j <- decay * weight_j + sum_g p[g][j]
// Bound by the K and V rows read from HBM (4 D bytes per row and head); the products ride on mma.sync, whose rate
// (24 instructions per 16 rows and 8 query heads at D = 128) is far above what the loads can feed, so the tcgen05 pipe
// would only add latency here: a tile has 8 to 16 query rows, not 128.
//  - Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that the 16-row side of the instruction
//    is the cache and the 8-column side the group's query heads. P goes from accumulator to operand layout with
//    movmatrix, in two parts, so that the result's own rounding is all that its type costs (one rounding of P
//    measured 1.35 times the error; the second part's products are not seen in the time). fp16 has too few exponents for rows
//    far below the leading one: see Fp16.
//  - Every warp streams its own tiles of 4 KB of K and 4 KB of V through a ring of three asynchronous copies in shared memory
//    (192 KB per SM) and runs ahead over the borders of units, so that the reads never pause while a unit's results are
//    put together. Page numbers are fetched a ring's length before the copies that need them, queries with a unit's
//    first tile. (Fragments straight from global memory to registers, without the ring: 528 us, 338 with it.)
//  - Work is handed out in blocks of a tile per warp, evenly over the CTAs of one resident wave, from the lengths on the
//    device: a ragged batch and one long sequence spread alike. A CTA's share is at most one partial unit at either end and
//    whole units between; of the CTAs that share a unit the one that arrives last joins the parts (nobody waits).
//  - The running maximum is raised only when a tile exceeds it by 2^8 (fp16: 2^4), so that most tiles need no reduction across lanes.
//    It is kept, as the scores are, before the scale: the difference of two scores that are near each other is exact, while the
//    scaled maximum, rounded, may lie 2^128 from its own row (scores of 2^31). Costs one addition per score, not seen in the time.
// Measured per call, all launches, bf16, D = 128: 16 problems x 32 heads x 8192 rows 335 us (6.4 TB/s; 372 us with the weights),
// one problem of 131071 rows, 8 heads for 64 query heads 91 us (5.9 TB/s), 32 problems of 0 .. 8192 rows 27.9 us (4.9 TB/s),
// one problem of 37 rows 4.7 us. What is left at small sizes is a chain of dependent reads (length, page, row), the
// merge of the warps and, for shared units, the arrival and the join: about 6 us beside the streaming.
// Tried and dropped: bringing the weights up to date in this launch, by the CTA that completes a unit (a step of 1024 units
// at budget 320: 61 us instead of 43; the chain of reads stalls the SM for longer than the ring lasts).
#include "ec_paged.cuh"

#include <atomic>

namespace ec {

namespace {

template <int D> constexpr int kTileRows = 2048 / D;                      // rows of a warp's tile: 4 KB of K, 4 KB of V

struct Bf16 {
    static constexpr float kLazy = 8.f;          // the running maximum is raised when exceeded by more than this (log2)
    static constexpr float kTop = 0.f;           // log2 of a probability at the running maximum
    static constexpr float kLeast = -INFINITY;   // parts of this type hold every probability
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b); }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(bf16lo(w), bf16hi(w)); }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

// Parts of P in fp16 are multiples of 2^-24, and rows of a peaked softmax lie further below its maximum than that (a row that
// gathers the attention and has small values, and the output is made of the others). So P is counted from 2^11 at the running
// maximum, which leaves the 2^4 that it may rise under the type's largest number, and is off by 2^-25: 2^-14 of a probability of
// 2^-11, 2^-22 of the maximum's. Tiles with a smaller one take P and V as tf32, where two parts hold 22 bits over all of fp32's
// exponents and V is exact, at twice the products and half the rate. All tiles as tf32 / only these, where there are none: 128 units x 16
// query heads x 8192 rows, D = 64, 58 / 50 us; 1024 units of 640 rows with weights 64 / 60 us (58 without the question).
struct Fp16 {
    static constexpr float kLazy = 4.f;
    static constexpr float kTop = 11.f;
    static constexpr float kLeast = -11.f;       // log2 of the least probability that they hold
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&h);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

// The 22 bits of a probability that two tf32 parts hold, from its fp32 value. The bits that the instruction does not use are cleared.
__device__ __forceinline__ void split_tf32(uint32_t p, uint32_t &hi, uint32_t &lo)
{
    hi = p & 0xFFFFE000u;
    lo = __float_as_uint(__uint_as_float(p) - __uint_as_float(hi)) & 0xFFFFE000u;
}

__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ void copy_piece(uint32_t dst, const uint4 *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// K and V pass through once (once per 16 query heads of a group): marked to leave the L2 first, so that scores and weights stay
// there between their launches (a step of 8 problems x 8 heads of 4096 rows 38 -> 34 us; 32 x 32 x 640 with weights 64 -> 61 us).
__device__ __forceinline__ void stream_piece(uint32_t dst, const uint4 *src, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ uint64_t stream_policy()
{
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_matrices_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <int V> struct Int { static constexpr int value = V; };

struct AttnArgs {
    PagedView c;
    const uint32_t *q;
    const uint4 *k_new, *v_new;                  // k_new == nullptr: the cached rows alone
    int G;                                       // query heads per key / value head
    float scale_log2e, inv_scale;                // inv_scale: 1 / scale_log2e, or a number as large as can be added to
    uint32_t *out;
    float *lse;
    // workspace
    float2 *stat;                                // [N, Hq] (the largest score, what its sum leaves as factor)
    float *score_new;                            // [N, Hq] the score of the step's own row, not scaled
    float *part_o;                               // [2 * CTAs][8 NT][D]
    float2 *part_ml;                             // [2 * CTAs][8 NT]
    float *scores;                               // <q, k>, not scaled, see scores_by_row
    int score_rows;                              // of one query head in a run: page_size or max_pages * page_size
};

// Rows of problem n with its own new row, 0 when there is nothing to attend to. A length past the table's reach is cut.
__device__ __forceinline__ int rows_of(const AttnArgs &a, int n)
{
    const int len = a.c.lens[n];
    return len < 0 ? 0 : min(len, a.c.max_pages * a.c.page_size) + (a.k_new ? 1 : 0);
}

// Every CTA derives the same plan from the lengths. Work is counted in blocks of W tiles, and every unit counts for
// kUnitCost blocks more: putting its results together takes about as long (measured with 8 warps: 2200 clocks for a
// full block, 4200 for a unit of one tile), and without that a CTA whose share is many short units ends last (32 ragged
// problems of 1 .. 8192 rows: 42 us without it).
constexpr int kUnitCost = 1;

struct Plan {
    int per, n, rows, before;                    // n < 0: nothing to do; the count in front of problem n
};

template <int BR>                                // rows of a block
__device__ __forceinline__ int blocks_of(int rows) { return (rows + BR - 1) / BR; }

template <int BR>
__device__ __forceinline__ int cost_of(int rows) { return rows > 0 ? blocks_of<BR>(rows) + kUnitCost : 0; }

// Each warp works it out for itself: a lane sums a span of problems, no barrier.
template <int BR>
__device__ __forceinline__ Plan make_plan(const AttnArgs &a, int units)
{
    const int N = a.c.N, lane = threadIdx.x & 31;
    const int span = (N + 31) >> 5;
    const int n0 = min(lane * span, N), n1 = min(n0 + span, N);
    int mine = 0, rows = 0;
#pragma unroll 8
    for (int n = n0; n < n1; ++n) {
        rows = rows_of(a, n);                    // with one problem a lane this is the one needed below
        mine += cost_of<BR>(rows);
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    const int total = __shfl_sync(0xFFFFFFFFu, incl, 31) * units;
    Plan plan;
    plan.per = (int)(((unsigned)total + gridDim.x - 1) / gridDim.x);
    plan.n = -1;
    plan.rows = plan.before = 0;
    const int first = plan.per * (int)blockIdx.x;
    if (first >= total) return plan;
    // the lane whose span holds the CTA's first block names the problem
    int at = (incl - mine) * units, n = n0;
    const bool here = first >= at && first < incl * units;
    if (here && span > 1) {
        int begin = at;
#pragma unroll 8
        for (int i = n0; i < n1; ++i) {
            const int r = rows_of(a, i), cost = cost_of<BR>(r) * units;
            if (first >= begin && first < begin + cost) {
                n = i;
                rows = r;
                at = begin;
            }
            begin += cost;
        }
    }
    const int src = __ffs(__ballot_sync(0xFFFFFFFFu, here)) - 1;
    plan.n = __shfl_sync(0xFFFFFFFFu, n, src);
    plan.rows = __shfl_sync(0xFFFFFFFFu, rows, src);
    plan.before = __shfl_sync(0xFFFFFFFFu, at, src);
    return plan;
}

// A place in the CTA's run of blocks. Every warp walks it three times: for the page table, S tiles behind for the copies,
// S tiles behind those for the arithmetic.
struct Walk {
    int n, rows, nb;                             // problem, its rows and blocks
    int h, hb, blk;                              // head, block of the group's query heads, block of the unit
    int left;                                    // what is left of the CTA's count, this block included
};

template <int BR>
__device__ __forceinline__ void next_unit(const AttnArgs &a, int head_blocks, Walk &w)
{
    w.blk = 0;
    if (++w.hb < head_blocks) return;
    w.hb = 0;
    if (++w.h < a.c.H) return;
    w.h = 0;
    do {
        if (++w.n >= a.c.N) {
            w.left = 0;
            return;
        }
        w.rows = rows_of(a, w.n);
        w.nb = blocks_of<BR>(w.rows);
    } while (w.nb == 0);
}

template <int BR>
__device__ __forceinline__ void walk_on(const AttnArgs &a, int head_blocks, Walk &w)
{
    --w.left;
    if (++w.blk < w.nb) return;
    w.left -= kUnitCost;
    if (w.left > 0) next_unit<BR>(a, head_blocks, w);
}

// Shared memory of a CTA of W warps that handles 8 NT query heads.
template <int D, int NT, int W> struct Smem {
    static constexpr int kTile = kTileRows<D>;
    static constexpr int kTileBytes = kTile * D * 2;                      // of K, and of V behind it
    static constexpr int kStages = 3;                                     // 24 KB per warp
    static constexpr int kPitch = D + 4;                                  // floats of a head in the merge buffer: no bank conflicts
    static constexpr int kMergeHeads = (W == 8 && NT == 1) || D == 64 ? 4 : 2;
    static constexpr int kMergeSlots = W * kMergeHeads;                   // (warp, head) pairs that fit the merge buffer
    static constexpr int kMergeFloats = kMergeSlots * kPitch;
    static constexpr int kQBytes = 8 * NT * D * 2;
    static constexpr int kQSlots = kStages + 1;                           // the copies run at most kStages units ahead
    static constexpr int kRing = 0;
    static constexpr int kMerge = kRing + W * kStages * 2 * kTileBytes;
    static constexpr int kQ = (kMerge + kMergeFloats * 4 + 255) / 256 * 256;   // fragments are addressed with XORs below 256
    static constexpr int kInfo = kQ + kQSlots * kQBytes;
    static constexpr int kPages = kInfo + W * kStages * kTile * 8;
    static constexpr int kTotal = kPages + W * kStages * kTile * 4;
};

// What is kept of a head beside its output, from its maximum and its sum: exp2((x - .x) * scale_log2e) * .y is the probability
// of a score x.
template <typename E>
__device__ __forceinline__ void keep_normaliser(const AttnArgs &a, size_t at, float M, float L)
{
    const float top = M == -INFINITY ? 0.f : M;
    a.stat[at] = make_float2(top, L == 0.f ? 0.f : exp2f(E::kTop) / L);
    if (a.lse) a.lse[at] = M == -INFINITY ? -INFINITY : fmaf(top, a.scale_log2e, log2f(L) - E::kTop) * 0.6931471805599453f;
}

// Joins the parts of a unit that the CTAs c0 .. c1 hold. A thread owns four dimensions of a head and has several parts in
// flight, the first of them before the parts' factors are known; `buf` (kMergeFloats floats) takes the factors.
template <typename E, int D, int NT, int W>
__device__ __forceinline__ void join_parts(const AttnArgs &a, int c0, int c1, int heads, size_t head_at, float *buf, float *sm_inv)
{
    using M_ = Smem<D, NT, W>;
    constexpr int kThreads = W * 32;
    constexpr int kChunk = M_::kMergeFloats / (8 * NT);
    constexpr int kItems = (8 * NT * (D / 4) + kThreads - 1) / kThreads;
    constexpr int kFlight = NT == 1 ? 8 : 4;      // eight would spill beside the registers of 16 heads
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int parts = c1 - c0 + 1;
    auto part_at = [&](int i) { return (size_t)(2 * (c0 + i) + (i == 0)) * 8 * NT; };
    if (parts <= kFlight) {                      // one round of reads, every thread on its own
#pragma unroll 1
        for (int i = threadIdx.x; i < heads * (D / 4); i += kThreads) {
            const int hd = i / (D / 4), d = 4 * (i - hd * (D / 4));
            float4 v[kFlight];
            float2 ml[kFlight];
#pragma unroll
            for (int c = 0; c < kFlight; ++c) {
                if (c >= parts) continue;
                v[c] = __ldcg(reinterpret_cast<const float4 *>(a.part_o + (part_at(c) + hd) * D + d));
                ml[c] = __ldcg(&a.part_ml[part_at(c) + hd]);
            }
            float M = -INFINITY, L = 0.f;
            float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int c = 0; c < kFlight; ++c)
                if (c < parts) M = fmaxf(M, ml[c].x);
            const float mu = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int c = 0; c < kFlight; ++c) {
                if (c >= parts) continue;
                const float f = fast_exp2((ml[c].x - mu) * a.scale_log2e);
                L = fmaf(ml[c].y, f, L);
                A.x = fmaf(v[c].x, f, A.x);
                A.y = fmaf(v[c].y, f, A.y);
                A.z = fmaf(v[c].z, f, A.z);
                A.w = fmaf(v[c].w, f, A.w);
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            uint2 r;
            r.x = E::pack(A.x * inv, A.y * inv);
            r.y = E::pack(A.z * inv, A.w * inv);
            *reinterpret_cast<uint2 *>(a.out + ((head_at + hd) * D + d) / 2) = r;
            if (d == 0) keep_normaliser<E>(a, head_at + hd, M, L);
        }
        return;
    }
    float4 A[kItems], first[kItems][kFlight];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + k * kThreads, hd = i / (D / 4), d = 4 * (i - hd * (D / 4));
        A[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kFlight; ++c)
            first[k][c] = hd < heads && c < parts ? __ldcg(reinterpret_cast<const float4 *>(a.part_o + (part_at(c) + hd) * D + d))
                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // maximum and sum of every head: a warp per head
    float *sm_m = sm_inv + 8 * NT;
    for (int hd = warp; hd < heads; hd += W) {
        float M = -INFINITY, L = 0.f;
        for (int c = lane; c < parts; c += 32) {
            const float2 v = __ldcg(&a.part_ml[part_at(c) + hd]);
            const float mn = fmaxf(M, v.x);
            if (mn != -INFINITY) L = L * fast_exp2((M - mn) * a.scale_log2e) + v.y * fast_exp2((v.x - mn) * a.scale_log2e);
            M = mn;
            if (c < kChunk) buf[hd * kChunk + c] = v.x;
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const float m2 = __shfl_xor_sync(0xFFFFFFFFu, M, d), l2 = __shfl_xor_sync(0xFFFFFFFFu, L, d);
            const float mn = fmaxf(M, m2);
            if (mn != -INFINITY) L = L * fast_exp2((M - mn) * a.scale_log2e) + l2 * fast_exp2((m2 - mn) * a.scale_log2e);
            M = mn;
        }
        const float mu = M == -INFINITY ? 0.f : M, inv = L == 0.f ? 0.f : 1.f / L;
        if (lane == 0) {
            sm_inv[hd] = inv;
            sm_m[hd] = mu;
            keep_normaliser<E>(a, head_at + hd, M, L);
        }
        for (int c = lane; c < min(parts, kChunk); c += 32) buf[hd * kChunk + c] = fast_exp2((buf[hd * kChunk + c] - mu) * a.scale_log2e);
    }
    __syncthreads();
    for (int cb = 0; cb < parts; cb += kChunk) {
        const int cn = min(kChunk, parts - cb);
        if (cb > 0) {
            __syncthreads();
            for (int i = threadIdx.x; i < heads * cn; i += kThreads) {
                const int hd = i / cn, c = i - hd * cn;
                buf[hd * kChunk + c] = fast_exp2((__ldcg(&a.part_ml[part_at(cb + c) + hd].x) - sm_m[hd]) * a.scale_log2e);
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = threadIdx.x + k * kThreads, hd = i / (D / 4), d = 4 * (i - hd * (D / 4));
            if (hd >= heads) continue;
            const float *f = buf + hd * kChunk;
            auto add = [&](float w, const float4 &v) {
                A[k].x = fmaf(v.x, w, A[k].x);
                A[k].y = fmaf(v.y, w, A[k].y);
                A[k].z = fmaf(v.z, w, A[k].z);
                A[k].w = fmaf(v.w, w, A[k].w);
            };
            int c = 0;
            if (cb == 0) {
#pragma unroll
                for (; c < kFlight; ++c)
                    if (c < parts) add(f[c], first[k][c]);
            }
#pragma unroll 8
            for (; c < cn; ++c) add(f[c], __ldcg(reinterpret_cast<const float4 *>(a.part_o + (part_at(cb + c) + hd) * D + d)));
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + k * kThreads, hd = i / (D / 4), d = 4 * (i - hd * (D / 4));
        if (hd >= heads) continue;
        const float inv = sm_inv[hd];
        uint2 r;
        r.x = E::pack(A[k].x * inv, A[k].y * inv);
        r.y = E::pack(A[k].z * inv, A[k].w * inv);
        *reinterpret_cast<uint2 *>(a.out + ((head_at + hd) * D + d) / 2) = r;
    }
}

// NT: groups of 8 query heads that share a pass over the rows. W: warps of a CTA. GATHER: scores are stored for the weights.
template <typename E, int D, int NT, int W, bool GATHER>
__global__ void __launch_bounds__(W * 32, 8 / W) paged_attention_kernel(AttnArgs a, int head_blocks)
{
    using M_ = Smem<D, NT, W>;
    constexpr int kThreads = W * 32, kTile = M_::kTile, kBlockRows = W * kTile;
    constexpr int RT = kTile / 16;               // 16-row sides of the products in a tile
    constexpr int C = D / 8;                     // 16-byte pieces of a row
    constexpr int KS = D / 16, MT = D / 16;
    constexpr int S = M_::kStages;
    extern __shared__ __align__(1024) unsigned char smem[];
    float *sm_o = reinterpret_cast<float *>(smem + M_::kMerge);
    __shared__ float2 sm_ml[W][8 * NT];
    __shared__ float sm_inv[2 * 8 * NT];
    __shared__ int sm_last;

    // The release stands behind the wait on purpose: a launch that this one lets in early may then read whatever earlier
    // launches wrote before it waits for this one (paged_rows_kernel does).
    grid_wait();
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.G, H = a.c.H, Hq = H * G;
    const int units = H * head_blocks;           // of a problem
    const Plan plan = make_plan<kBlockRows>(a, units);
    // problems without a row to attend to have no block: their outputs are written here
    for (int n = blockIdx.x; n < a.c.N; n += gridDim.x) {
        read_len(a.c, n);                        // reports a length past the table's reach
        if (rows_of(a, n) > 0) continue;
        for (int i = threadIdx.x; i < Hq * (D / 2); i += kThreads) a.out[(size_t)n * Hq * (D / 2) + i] = 0;
        for (int i = threadIdx.x; i < Hq; i += kThreads) {
            a.stat[(size_t)n * Hq + i] = make_float2(0.f, 0.f);
            if (a.lse) a.lse[(size_t)n * Hq + i] = -INFINITY;
        }
    }
    if (plan.n < 0) return;

    Walk use;
    use.n = plan.n;
    use.rows = plan.rows;
    use.nb = blocks_of<kBlockRows>(use.rows);
    use.left = plan.per;
    {
        const unsigned in = (unsigned)(plan.per * (int)blockIdx.x - plan.before);
        const unsigned cost = (unsigned)(use.nb + kUnitCost);
        const int unit = (int)(in / cost);
        use.blk = (int)(in - (unsigned)unit * cost);
        use.h = unit / head_blocks;
        use.hb = unit - use.h * head_blocks;
        if (use.blk >= use.nb) {                 // the share begins behind the unit's blocks
            use.left -= (int)cost - use.blk;
            if (use.left > 0) next_unit<kBlockRows>(a, head_blocks, use);
        }
    }
    Walk ahead = use, scout = use;

    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
    const uint32_t ring = base + M_::kRing + warp * (S * 2 * M_::kTileBytes);
    uint2 *rows_info = reinterpret_cast<uint2 *>(smem + M_::kInfo) + warp * (S * kTile);   // where a row's score lies: (run, row in the run)
    const int *pages = reinterpret_cast<const int *>(smem + M_::kPages) + warp * (S * kTile);
    const uint32_t pages_at = base + M_::kPages + warp * (S * kTile * 4);
    const int tile_row = warp * kTile + lane % kTile;                     // of a block, described by this lane
    const int own_row = a.k_new ? 1 : 0;
    const uint64_t policy = stream_policy();

    // The page of every row of the tile at `scout`, S tiles before the copies need it.
    auto scout_tile = [&](int slot) {
        if (scout.left <= 0) return;
        const int row = scout.blk * kBlockRows + tile_row;
        if (lane < kTile && row < scout.rows - own_row) {
            const int *src = a.c.table + (size_t)scout.n * a.c.max_pages + page_of(a.c, row);
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(pages_at + (slot * kTile + lane) * 4), "l"(src) : "memory");
        }
        walk_on<kBlockRows>(a, head_blocks, scout);
    };
    int q_slot_ahead = 0;
    bool fresh_ahead = true;
    auto copy_tile = [&](int stage) {            // the tile at `ahead`, which then moves on; its pages have arrived
        if (ahead.left > 0) {
            const int h = ahead.h;
            if (fresh_ahead) {                   // the unit's queries, every warp a share of them
                const int head0 = ahead.hb * 8 * NT;
                const size_t head_at = (size_t)ahead.n * Hq + (size_t)h * G + head0;
                for (int i = threadIdx.x; i < 8 * NT * C; i += kThreads) {
                    const int hd = i / C, piece = i - hd * C;
                    const bool there = head0 + hd < G;
                    copy_piece(base + M_::kQ + q_slot_ahead * M_::kQBytes + hd * (D * 2) + ((piece ^ (hd & 7)) << 4),
                               reinterpret_cast<const uint4 *>(a.q) + (there ? (head_at + hd) * C + piece : 0), there ? 16u : 0u);
                }
                q_slot_ahead = q_slot_ahead + 1 == M_::kQSlots ? 0 : q_slot_ahead + 1;
            }
            const int row0 = ahead.blk * kBlockRows + warp * kTile;
            if (row0 < ahead.rows) {
                const int row = row0 + lane % kTile, len = ahead.rows - own_row;
                uint32_t off = kRowNone;
                uint2 info = make_uint2(kRowNone, 0);
                if (row < len) {
                    Slot s;
                    s.page = pages[stage * kTile + lane % kTile];
                    s.slot = row - page_of(a.c, row) * a.c.page_size;
                    if ((unsigned)s.page < (unsigned)a.c.n_pages) {
                        off = row_offset(a.c, s);
                        info = scores_by_row(a.c.page_size) ? make_uint2((uint32_t)ahead.n * (uint32_t)H + (uint32_t)h, (uint32_t)row)
                                                            : make_uint2((uint32_t)s.page * (uint32_t)H + (uint32_t)h, (uint32_t)s.slot);
                    } else {
                        atomicExch(a.c.state, kStatusPage);
                    }
                } else if (row < ahead.rows) {
                    off = info.x = kRowNew;
                }
                if (lane < kTile) rows_info[stage * kTile + lane] = info;
                const uint4 *Kh = a.c.K + (size_t)h * a.c.head_step + lane % C, *Vh = a.c.V + (size_t)h * a.c.head_step + lane % C;
                // rows of one copy instruction lie 32 / C apart from the next one's: their swizzles differ by a constant
                const uint32_t dst0 = (ring + stage * (2 * M_::kTileBytes) + (lane / C) * (D * 2)) + ((lane % C ^ lane / C) << 4);
                const bool plain = __all_sync(0xFFFFFFFFu, off < kRowNew);
                if (plain) {                     // cached rows all through
#pragma unroll
                    for (int i = 0; i < kTile * C / 32; ++i) {
                        const uint32_t o = __shfl_sync(0xFFFFFFFFu, off, i * (32 / C) + lane / C);
                        const uint32_t dst = (dst0 ^ (((i * (32 / C)) & 7) << 4)) + i * 512;
                        stream_piece(dst, Kh + o, policy);
                        stream_piece(dst + M_::kTileBytes, Vh + o, policy);
                    }
                } else {                         // the unit's last rows, or pages that do not exist
                    const size_t own = ((size_t)ahead.n * H + h) * C + lane % C;
#pragma unroll 1
                    for (int i = 0; i < kTile * C / 32; ++i) {
                        const uint32_t o = __shfl_sync(0xFFFFFFFFu, off, i * (32 / C) + lane / C);
                        const uint32_t dst = (dst0 ^ (((i * (32 / C)) & 7) << 4)) + i * 512;
                        const uint32_t bytes = o == kRowNone ? 0u : 16u;  // absent rows are filled with zeros
                        const size_t at = o == kRowNone ? 0 : o;
                        copy_piece(dst, o == kRowNew ? a.k_new + own : Kh + at, bytes);
                        copy_piece(dst + M_::kTileBytes, o == kRowNew ? a.v_new + own : Vh + at, bytes);
                    }
                }
            }
            fresh_ahead = ahead.blk + 1 == ahead.nb;
            walk_on<kBlockRows>(a, head_blocks, ahead);
            __syncwarp();                        // the pages have been read
            scout_tile(stage);
        }
        copies_commit();
    };

#pragma unroll 1
    for (int i = 0; i < S; ++i) scout_tile(i);
    copies_commit();
    copies_wait<0>();
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < S; ++i) copy_tile(i);
    copies_wait<S - 1>();
    __syncthreads();                             // the first unit's queries are here

    // Q's fragments stay in registers for 8 heads; for 16 they would spill, and are read again for every tile
    constexpr bool kHoldQ = NT == 1;
    uint32_t qf[kHoldQ ? NT : 1][kHoldQ ? KS : 1][2], q_at = 0;
    float o[NT][MT][4], m[NT][2], l[NT][2], limit[NT][2], top[NT][2];
    int stage = 0, q_slot = 0, first_block = use.blk;
    auto begin_unit = [&] {                      // the queries of the next unit are here; nothing has been seen of it
        q_at = base + M_::kQ + q_slot * M_::kQBytes + (lane & 7) * (D * 2) + (((lane >> 3) ^ (lane & 7)) << 4);
        q_slot = q_slot + 1 == M_::kQSlots ? 0 : q_slot + 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (kHoldQ) {
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    uint32_t r[4];
                    load_matrices(r, (q_at ^ (ks << 5)) + nt * 8 * (D * 2));
                    qf[nt][ks][0] = r[0];
                    qf[nt][ks][1] = r[1];
                    qf[nt][ks + 1][0] = r[2];
                    qf[nt][ks + 1][1] = r[3];
                }
            }
            m[nt][0] = m[nt][1] = limit[nt][0] = limit[nt][1] = -INFINITY;
            top[nt][0] = top[nt][1] = 0.f;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
        }
    };
    begin_unit();
    while (use.left > 0) {
        const int h = use.h, head0 = use.hb * 8 * NT;                     // first query head of the block within the group
        const int heads = min(G - head0, 8 * NT);
        const size_t head_at = (size_t)use.n * Hq + (size_t)h * G + head0;
        copies_wait<S - 1>();
        __syncwarp();
        if (use.blk * kBlockRows + warp * kTile < use.rows) {
            const uint32_t tile = ring + stage * (2 * M_::kTileBytes);
            // S^T of this tile, even and odd steps in chains of their own
            float s[RT][NT][4], s1[RT][NT][4];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][nt][i] = s1[rt][nt][i] = 0.f;
            {
                const int row = lane & 15;
                const uint32_t at = (tile + row * (D * 2)) + (((lane >> 4) ^ (row & 7)) << 4);
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    uint32_t r[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (kHoldQ) {
                            r[nt][0] = qf[nt][ks][0];
                            r[nt][1] = qf[nt][ks][1];
                            r[nt][2] = qf[nt][ks + 1][0];
                            r[nt][3] = qf[nt][ks + 1][1];
                        } else {
                            load_matrices(r[nt], (q_at ^ (ks << 5)) + nt * 8 * (D * 2));
                        }
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        uint32_t a0[4], a1[4];
                        load_matrices(a0, (at ^ (ks << 5)) + rt * 16 * (D * 2));
                        load_matrices(a1, (at ^ ((ks + 1) << 5)) + rt * 16 * (D * 2));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            E::mma(s[rt][nt], a0, r[nt][0], r[nt][1]);
                            E::mma(s1[rt][nt], a1, r[nt][2], r[nt][3]);
                        }
                    }
                }
            }
            uint2 info[RT][2];                   // rows g and g + 8 of every 16
            bool raise = false;                  // scale > 0: the scores are compared before they are scaled
            float low[NT][2];                    // the lowest of a head; an absent row counts with a score of zero
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                info[rt][0] = rows_info[stage * kTile + rt * 16 + g];
                info[rt][1] = rows_info[stage * kTile + rt * 16 + g + 8];
                const bool there0 = info[rt][0].x != kRowNone, there1 = info[rt][1].x != kRowNone;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float x = s[rt][nt][i] + s1[rt][nt][i], y = s[rt][nt][2 + i] + s1[rt][nt][2 + i];
                        if (E::kLeast > -INFINITY) low[nt][i] = rt == 0 ? fminf(x, y) : fminf(low[nt][i], fminf(x, y));
                        s[rt][nt][i] = there0 ? x : -INFINITY;
                        s[rt][nt][2 + i] = there1 ? y : -INFINITY;
                        raise |= fmaxf(s[rt][nt][i], s[rt][nt][2 + i]) > limit[nt][i];
                    }
            }
            if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float x = fmaxf(s[0][nt][i], s[0][nt][2 + i]);
#pragma unroll
                        for (int rt = 1; rt < RT; ++rt) x = fmaxf(x, fmaxf(s[rt][nt][i], s[rt][nt][2 + i]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
                        const float mn = fmaxf(m[nt][i], x);
                        const float corr = mn == -INFINITY ? 1.f : fast_exp2((m[nt][i] - mn) * a.scale_log2e);   // first tile: 2^-inf = 0
                        m[nt][i] = mn;
                        limit[nt][i] = __fadd_rd(mn, E::kLazy * a.inv_scale);   // rounded up it could let 2^(2 kLazy) pass
                        top[nt][i] = mn == -INFINITY ? 0.f : mn;
                        l[nt][i] *= corr;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            o[nt][mt][i] *= corr;
                            o[nt][mt][2 + i] *= corr;
                        }
                    }
            }
            const int v_row = (lane & 7) + (lane >> 4) * 8;
            const uint32_t v_at = (tile + M_::kTileBytes + v_row * (D * 2)) + ((((lane >> 3) & 1) ^ (v_row & 7)) << 4);
            bool little = false;
            if (E::kLeast > -INFINITY) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) little |= fmaf(low[nt][i] - top[nt][i], a.scale_log2e, E::kTop) < E::kLeast;
            }
            float p[RT][NT][4];                  // rows g, g, g + 8, g + 8 and heads 2t, 2t + 1, 2t, 2t + 1
            auto probabilities = [&] {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[rt][nt][i] = fast_exp2(fmaf(s[rt][nt][i] - top[nt][i & 1], a.scale_log2e, E::kTop));
                        l[nt][0] += p[rt][nt][0] + p[rt][nt][2];
                        l[nt][1] += p[rt][nt][1] + p[rt][nt][3];
                    }
            };
            // decided ahead of the exponentials, which then run between the products (behind them: 3 to 9% of a call)
            if (E::kLeast > -INFINITY && __any_sync(0xFFFFFFFFu, little)) {
                probabilities();
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    // Rows 2t, 2t + 1, 2t + 8, 2t + 9 of head g. V's fragment holds the same rows, two to a register, and the order of
                    // the rows within a product is free: a register's low halves are one k of tf32, its high halves the next.
                    uint32_t hi[NT][4], lo[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const uint32_t x = __float_as_uint(p[rt][nt][2 * r]), y = __float_as_uint(p[rt][nt][2 * r + 1]);
                            const uint32_t low = transpose8x8(__byte_perm(x, y, 0x5410)), high = transpose8x8(__byte_perm(x, y, 0x7632));
                            split_tf32(__byte_perm(low, high, 0x5410), hi[nt][2 * r], lo[nt][2 * r]);
                            split_tf32(__byte_perm(low, high, 0x7632), hi[nt][2 * r + 1], lo[nt][2 * r + 1]);
                        }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        uint32_t av[4];
                        load_matrices_trans(av, (v_at ^ (mt << 5)) + rt * 16 * (D * 2));
#pragma unroll
                        for (int r = 0; r < 2; ++r) {                     // eight rows each: 2t and 2t + 1, then 2t + 8 and 2t + 9
                            const float2 v0 = E::unpack(av[2 * r]), v1 = E::unpack(av[2 * r + 1]);
                            const uint32_t w[4] = {__float_as_uint(v0.x), __float_as_uint(v1.x), __float_as_uint(v0.y), __float_as_uint(v1.y)};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_tf32(o[nt][mt], w, hi[nt][2 * r], hi[nt][2 * r + 1]);
                                mma_tf32(o[nt][mt], w, lo[nt][2 * r], lo[nt][2 * r + 1]);
                            }
                        }
                    }
                }
            } else {
                probabilities();
                uint32_t hi[RT][NT][2], lo[RT][NT][2];   // P as the sum of two rounded parts: 16 bits of it or more meet V (fp16: 14)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const uint32_t x = E::pack(p[rt][nt][2 * r], p[rt][nt][2 * r + 1]);
                            const float2 f = E::unpack(x);
                            hi[rt][nt][r] = transpose8x8(x);
                            lo[rt][nt][r] = transpose8x8(E::pack(p[rt][nt][2 * r] - f.x, p[rt][nt][2 * r + 1] - f.y));
                        }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        uint32_t av[4];
                        load_matrices_trans(av, (v_at ^ (mt << 5)) + rt * 16 * (D * 2));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            E::mma(o[nt][mt], av, hi[rt][nt][0], hi[rt][nt][1]);
                            E::mma(o[nt][mt], av, lo[rt][nt][0], lo[rt][nt][1]);
                        }
                    }
            }
            if (GATHER) {                        // behind the products: the stores' addresses are in nobody's way here
#pragma unroll
                for (int r = 0; r < 2 * RT; ++r) {
                    const uint2 at = info[r >> 1][r & 1];
                    if (at.x == kRowNone) continue;
                    const bool own = at.x == kRowNew;
                    const int step = own ? 1 : a.score_rows;
                    float *dst = (own ? a.score_new + head_at : a.scores + ((size_t)at.x * G + head0) * a.score_rows + at.y) +
                                 (size_t)(2 * t) * step;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int hd = nt * 8 + 2 * t;
                        if (hd < heads) dst[(size_t)(nt * 8) * step] = s[r >> 1][nt][2 * (r & 1)];
                        if (hd + 1 < heads) dst[(size_t)(nt * 8 + 1) * step] = s[r >> 1][nt][2 * (r & 1) + 1];
                    }
                }
            }
        }
        __syncwarp();                            // every lane is done with the stage
        copy_tile(stage);
        stage = stage + 1 == S ? 0 : stage + 1;

        if (use.blk + 1 == use.nb || use.left == 1) {
            const bool whole = first_block == 0 && use.blk + 1 == use.nb;
            const int part = 2 * blockIdx.x + (first_block == 0 ? 1 : 0); // a CTA holds at most one part of each kind
            const int seen_rows = min(use.rows, (use.blk + 1) * kBlockRows) - first_block * kBlockRows;
            const int nw = min(W, (seen_rows + kTile - 1) / kTile);       // warps that had a tile of it
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][i] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][i], d);
            if (warp < nw && g == 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) sm_ml[warp][nt * 8 + 2 * t + i] = make_float2(m[nt][i], l[nt][i]);
            }
            // the warps' results meet in shared memory, `per_round` heads of up to `most` warps at a time
            auto meet = [&](auto per_round_, auto most_) {
                constexpr int per_round = decltype(per_round_)::value, most = decltype(most_)::value;
                for (int h0 = 0; h0 < heads; h0 += per_round) {
                    if (warp < nw) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int at = nt * 8 + 2 * t + i - h0;
                                if (at < 0 || at >= per_round) continue;
                                float *dst = sm_o + (warp * per_round + at) * M_::kPitch + g;
#pragma unroll
                                for (int mt = 0; mt < MT; ++mt) {
                                    dst[mt * 16] = o[nt][mt][i];
                                    dst[mt * 16 + 8] = o[nt][mt][2 + i];
                                }
                            }
                    }
                    __syncthreads();
                    const int items = min(per_round, heads - h0) * (D / 64);   // 64 dimensions of a head, by a warp
                    for (int it = warp; it < items; it += W) {
                        const int at = it / (D / 64), hd = h0 + at, d = (it % (D / 64)) * 64 + 2 * lane;
                        float2 ml[most];
                        float M = -INFINITY, L = 0.f;
#pragma unroll
                        for (int w = 0; w < most; ++w) {
                            ml[w] = w < nw ? sm_ml[w][hd] : make_float2(-INFINITY, 0.f);
                            M = fmaxf(M, ml[w].x);
                        }
                        const float mu = M == -INFINITY ? 0.f : M;
                        float2 A = make_float2(0.f, 0.f);
#pragma unroll
                        for (int w = 0; w < most; ++w) {
                            if (w >= nw) continue;
                            const float f = fast_exp2((ml[w].x - mu) * a.scale_log2e);
                            const float2 v = *reinterpret_cast<const float2 *>(sm_o + (w * per_round + at) * M_::kPitch + d);
                            L = fmaf(ml[w].y, f, L);
                            A.x = fmaf(v.x, f, A.x);
                            A.y = fmaf(v.y, f, A.y);
                        }
                        const float inv = L == 0.f ? 0.f : 1.f / L;       // nothing left by the scores: the output is zero
                        if (whole) a.out[((head_at + hd) * D + d) >> 1] = E::pack(A.x * inv, A.y * inv);
                        else *reinterpret_cast<float2 *>(a.part_o + ((size_t)part * 8 * NT + hd) * D + d) = A;
                        if (d == 0) {
                            if (whole) keep_normaliser<E>(a, head_at + hd, M, L);
                            else a.part_ml[(size_t)part * 8 * NT + hd] = make_float2(M, L);
                        }
                    }
                    copies_wait<S - 1>();        // with the barrier: the next unit's queries are here
                    __syncthreads();
                }
            };
            // sixteen heads leave room for two at a time from eight warps: a unit of one or two tiles takes them in two
            // rounds instead of eight (49 x 40 units of 22 rows: 118 -> 80 us)
            if (NT == 2 && nw <= 2) meet(Int<M_::kMergeSlots / 2>(), Int<2>());
            else meet(Int<M_::kMergeHeads>(), Int<W>());
            if (!whole) {
                // the unit's first and last CTA follow from its first block; the last of them to get here joins the parts
                const int b0 = plan.per * blockIdx.x + (plan.per - use.left) - use.blk;
                const int c0 = b0 / plan.per, c1 = (b0 + use.nb - 1) / plan.per;
                int *arrived = a.c.state + kStateAttention + c0;          // a CTA is the first of one shared unit at most
                if (threadIdx.x == 0) sm_last = arrive(arrived) == c1 - c0;
                __syncthreads();
                if (sm_last) {
                    if (threadIdx.x == 0) *arrived = 0;
                    join_parts<E, D, NT, W>(a, c0, c1, heads, head_at, sm_o, sm_inv);
                    __syncthreads();
                }
            }
            walk_on<kBlockRows>(a, head_blocks, use);
            first_block = use.blk;
            begin_unit();
        } else {
            walk_on<kBlockRows>(a, head_blocks, use);
        }
    }
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct WsLayout {
    size_t stat, score_new, part_o, part_ml, scores, total;
};

WsLayout layout(int N, int H, int D, int n_pages, int page_size, int max_pages, int G, int accumulate)
{
    const int nt = G > 8 ? 2 : 1;
    WsLayout w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    w.stat = take((size_t)N * H * G * sizeof(float2));
    w.score_new = take((size_t)N * H * G * sizeof(float));
    w.part_o = take((size_t)2 * kPagedMaxCtas * 8 * nt * D * sizeof(float));
    w.part_ml = take((size_t)2 * kPagedMaxCtas * 8 * nt * sizeof(float2));
    const size_t rows = scores_by_row(page_size) ? (size_t)N * max_pages * page_size : (size_t)n_pages * page_size;
    w.scores = take(accumulate ? rows * H * G * sizeof(float) : 0);
    w.total = at;
    return w;
}

template <typename E, int D, int NT, int W, bool GATHER>
cudaError_t launch(const AttnArgs &a, cudaStream_t stream)
{
    auto kernel = paged_attention_kernel<E, D, NT, W, GATHER>;
    constexpr int smem = Smem<D, NT, W>::kTotal;
    const int head_blocks = (a.G + 8 * NT - 1) / (8 * NT);
    int dev = 0, ctas = 148;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ctas, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    ctas *= 8 / W;
    if (ctas > kPagedMaxCtas) ctas = kPagedMaxCtas;
    static std::atomic<unsigned long long> allowed{0};                    // devices on which the kernel may use this much
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(allowed.load(std::memory_order_relaxed) & bit) || !bit) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch_chained(kernel, dim3((unsigned)ctas), W * 32, smem, stream, a, head_blocks);
}

// Units from which CTAs have four warps, two to an SM, instead of eight: with many units the barriers of one CTA hide behind
// the other; with few, half as many CTAs leave half as many parts to join. Four / eight warps: 2048 units of 127 rows 33 / 43 us,
// 1024 units of 640 rows with weights 66 / 70 us, 512 units of 8192 rows 340 / 337 us, 8 units of 131071 rows 103 / 92 us.
// Groups of more than eight query heads need the shared memory of eight warps.
constexpr long long kNarrowUnits = 512;

template <typename E, int D, bool GATHER>
cudaError_t launch_g(const AttnArgs &a, cudaStream_t stream)
{
    if (a.G > 8) return launch<E, D, 2, 8, GATHER>(a, stream);
    if ((long long)a.c.N * a.c.H >= kNarrowUnits) return launch<E, D, 1, 4, GATHER>(a, stream);
    return launch<E, D, 1, 8, GATHER>(a, stream);
}

template <typename E, int D>
cudaError_t launch_d(const AttnArgs &a, int accumulate, cudaStream_t stream)
{
    return accumulate ? launch_g<E, D, true>(a, stream) : launch_g<E, D, false>(a, stream);
}

}  // namespace

size_t paged_attention_workspace_bytes(const ec_paged *c, int Hq, int accumulate)
{
    return layout(c->N, c->H, c->D, c->n_pages, c->page_size, c->max_pages, Hq / c->H, accumulate).total;
}

cudaError_t launch_paged_attention(const PagedView &c, int D, int dtype, const void *q, const void *k_new, const void *v_new,
                                   int Hq, float scale, int accumulate, float decay, void *out, float *lse, float *w_new,
                                   void *ws, GatherArgs *gather, cudaStream_t stream)
{
    AttnArgs a;
    a.c = c;
    a.q = static_cast<const uint32_t *>(q);
    a.k_new = static_cast<const uint4 *>(k_new);
    a.v_new = static_cast<const uint4 *>(v_new);
    a.G = Hq / c.H;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.inv_scale = fminf(1.f / a.scale_log2e, 0x1p120f);
    a.out = static_cast<uint32_t *>(out);
    a.lse = lse;
    const WsLayout w = layout(c.N, c.H, D, c.n_pages, c.page_size, c.max_pages, a.G, accumulate);
    char *p = static_cast<char *>(ws);
    a.stat = reinterpret_cast<float2 *>(p + w.stat);
    a.score_new = reinterpret_cast<float *>(p + w.score_new);
    a.part_o = reinterpret_cast<float *>(p + w.part_o);
    a.part_ml = reinterpret_cast<float2 *>(p + w.part_ml);
    a.scores = reinterpret_cast<float *>(p + w.scores);
    a.score_rows = scores_by_row(c.page_size) ? c.max_pages * c.page_size : c.page_size;
    if (accumulate) *gather = {a.stat, a.scores, a.score_new, k_new ? w_new : nullptr, a.scale_log2e, decay, a.G};
    if (dtype == EC_BF16) return D == 128 ? launch_d<Bf16, 128>(a, accumulate, stream) : launch_d<Bf16, 64>(a, accumulate, stream);
    return D == 128 ? launch_d<Fp16, 128>(a, accumulate, stream) : launch_d<Fp16, 64>(a, accumulate, stream);
}

}  // namespace ec
