// Attention of one new token per problem over a paged cache (grouped query heads), with the probability every
// cached row receives added to the row's gathered weight.
//   x[g][j] = scale * <q_g, k_j>,  p = softmax_j(x),  out_g = sum_j p[g][j] v_j,  weight_j <- decay * weight_j + sum_g p[g][j]
// Bound by the K and V rows read from HBM (4 D bytes per row and head); the products ride on mma.sync, whose rate
// (24 instructions per 16 rows and 8 query heads) is far above what the loads can feed, so the tcgen05 pipe would
// only add latency here: a tile has 8 to 16 query rows, not 128.
//  - Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that the 16-row side of the instruction
//    is the cache and the 8-column side the group's query heads. P goes from accumulator to operand layout with
//    movmatrix.
//  - Every warp streams its own 16-row tiles through a ring of asynchronous copies in shared memory (96 KB per CTA, two
//    CTAs per SM) and runs ahead over the borders of units, so that the reads never pause while a unit's results
//    are put together.
//  - Work is handed out in blocks of 64 rows, evenly over the CTAs of one resident wave, from the lengths on the device: a
//    ragged batch and one long sequence spread alike. A CTA's share is at most one partial unit at either end and
//    whole units between; of the CTAs that share a unit the one that arrives last joins the parts (nobody waits).
#include "ec_paged.cuh"

namespace ec {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;                        // rows of a warp's tile
constexpr int kBlockRows = kWarps * kTile;       // rows of a block, the unit of work distribution
constexpr int kCtasPerSm = 2;
constexpr float kLazy = 8.f;                     // the running maximum is raised when exceeded by more than this (log2)

struct Bf16 {
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b); }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(bf16lo(w), bf16hi(w)); }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

struct Fp16 {
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

struct AttnArgs {
    PagedView c;
    const uint32_t *q;
    const uint4 *k_new, *v_new;                  // k_new == nullptr: the cached rows alone
    int G;                                       // query heads per key / value head
    float scale_log2e, decay;
    uint32_t *out;
    float *lse, *w_new;
    // workspace
    float2 *stat;                                // [N, Hq] (maximum in the log2 domain, 1 / sum)
    float *score_new;                            // [N, Hq] score of the step's own row
    float *part_o;                               // [2 * CTAs][8 NT][D]
    float2 *part_ml;                             // [2 * CTAs][8 NT]
    float *scores;                               // [n_pages, H, page_size, G], log2 domain
};

// Rows of problem n with its own new row, 0 when there is nothing to attend to.
__device__ __forceinline__ int rows_of(const AttnArgs &a, int n)
{
    const int len = read_len(a.c, n);
    return len < 0 ? 0 : len + (a.k_new ? 1 : 0);
}

__device__ __forceinline__ int blocks_of(int rows) { return (rows + kBlockRows - 1) / kBlockRows; }

// Every CTA derives the same plan from the lengths: `per` blocks for each CTA, and where its own begin.
struct Plan {
    int per, n;                                  // n < 0: nothing to do
    long long before;                            // blocks in front of problem n
};

__device__ __forceinline__ void make_plan(const AttnArgs &a, int units, int min_per, Plan *plan)
{
    __shared__ long long warp_sum[kWarps];
    const int N = a.c.N;
    const int span = (N + kThreads - 1) / kThreads;
    const int n0 = min((int)threadIdx.x * span, N), n1 = min(n0 + span, N);
    long long mine = 0;
    for (int n = n0; n < n1; ++n) mine += blocks_of(rows_of(a, n));
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if ((threadIdx.x & 31) >= o) incl += up;
    }
    if ((threadIdx.x & 31) == 31) warp_sum[threadIdx.x >> 5] = incl;
    if (threadIdx.x == 0) plan->n = -1;
    __syncthreads();
    long long total = 0, base = incl - mine;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < (int)(threadIdx.x >> 5)) base += warp_sum[w];
        total += warp_sum[w];
    }
    long long per = (total * units + gridDim.x - 1) / gridDim.x;
    if (per < min_per) per = min_per;
    const long long first = per * blockIdx.x;
    if (threadIdx.x == 0) plan->per = (int)per;
    // the thread whose span holds the CTA's first block names the problem
    if (first >= base * units && first < (base + mine) * units) {
        long long at = base * units;
        for (int n = n0; n < n1; ++n) {
            const long long nb = (long long)blocks_of(rows_of(a, n)) * units;
            if (first < at + nb) {
                plan->n = n;
                plan->before = at;
                break;
            }
            at += nb;
        }
    }
    __syncthreads();
}

// A place in the CTA's run of blocks. The loader and the consumer of a warp each walk it, the loader ahead.
struct Walk {
    int n, rows, nb;                             // problem, its rows and blocks
    int unit, blk;                               // (head, head block) of the problem, block of the unit
    int left;                                    // blocks still to do, this one included
};

__device__ __forceinline__ void walk_on(const AttnArgs &a, int units, Walk &w)
{
    --w.left;
    if (++w.blk < w.nb) return;
    w.blk = 0;
    if (++w.unit < units) return;
    w.unit = 0;
    do {
        if (++w.n >= a.c.N) {
            w.left = 0;
            return;
        }
        w.rows = rows_of(a, w.n);
        w.nb = blocks_of(w.rows);
    } while (w.nb == 0);
}

template <int D> struct Ring {
    static constexpr int kTileBytes = kTile * D * 2;                      // of K, and of V behind it
    static constexpr int kStages = D == 128 ? 3 : 6;                      // 24 KB per warp
    static constexpr int kBytes = kWarps * kStages * 2 * kTileBytes;
    static constexpr int kPitch = D + 4;                                  // floats of a head in the merge buffer: no bank conflicts
    static constexpr int kMergeHeads = 4;
    static constexpr int kMergeFloats = kWarps * kMergeHeads * kPitch;
    static constexpr int kSmem = kBytes + kMergeFloats * 4 + kWarps * kStages * kTile * 4;
};

// NT: groups of 8 query heads that share a pass over the rows. GATHER: scores are stored for the weights.
template <typename E, int D, int NT, bool GATHER>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) paged_attention_kernel(AttnArgs a, int head_blocks, int min_per)
{
    using R = Ring<D>;
    constexpr int C = D / 8;                     // 16-byte pieces of a row
    constexpr int KS = D / 16, MT = D / 16;
    constexpr int S = R::kStages;
    extern __shared__ __align__(128) unsigned char smem[];
    float *sm_o = reinterpret_cast<float *>(smem + R::kBytes);
    uint32_t *sm_row = reinterpret_cast<uint32_t *>(smem + R::kBytes + R::kMergeFloats * 4);
    __shared__ float2 sm_ml[kWarps][8 * NT];
    __shared__ float sm_m[8 * NT], sm_inv[8 * NT];
    __shared__ Plan plan;
    __shared__ int sm_last;

    grid_wait();
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.G, H = a.c.H, Hq = H * G;
    const int units = H * head_blocks;           // of a problem
    make_plan(a, units, min_per, &plan);
    // problems without a row to attend to have no block: their outputs are written here
    for (int n = blockIdx.x; n < a.c.N; n += gridDim.x) {
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
    use.rows = rows_of(a, use.n);
    use.nb = blocks_of(use.rows);
    use.left = plan.per;
    {
        const long long in = (long long)plan.per * blockIdx.x - plan.before;
        use.unit = (int)(in / use.nb);
        use.blk = (int)(in - (long long)use.unit * use.nb);
    }
    Walk ahead = use;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S * 2 * R::kTileBytes);
    uint32_t *rows_info = sm_row + warp * (S * kTile);

    // Loader: lane i (and i + 16) looks up row i of a tile, one tile before it is copied, so that the table's latency is
    // not in the way.
    int next_page = -1, next_slot = 0;
    uint32_t next_kind = kRowNone;               // kRowNone, kRowNew, or 0: a cached row
    auto look_up = [&]() {
        next_kind = kRowNone;
        if (ahead.left <= 0) return;
        const int row = ahead.blk * kBlockRows + warp * kTile + (lane & 15);
        const int len = ahead.rows - (a.k_new ? 1 : 0);
        if (row < len) {
            const int p = row / a.c.page_size;
            next_kind = 0;
            next_slot = row - p * a.c.page_size;
            next_page = a.c.table[(size_t)ahead.n * a.c.max_pages + p];
        } else if (row < ahead.rows) {
            next_kind = kRowNew;
        }
    };
    auto copy_tile = [&](int stage) {            // the tile at `ahead`, which then moves on
        if (ahead.left > 0) {
            if (ahead.blk * kBlockRows + warp * kTile < ahead.rows) {
                const int h = ahead.unit / head_blocks;
                uint32_t off = next_kind, info = next_kind;
                if (next_kind == 0) {
                    Slot s;
                    s.page = next_page;
                    s.slot = next_slot;
                    if ((unsigned)next_page >= (unsigned)a.c.n_pages) {
                        atomicExch(a.c.state, kStatusPage);
                        off = info = kRowNone;
                    } else {
                        off = row_offset(a.c, s);
                        info = meta_index(a.c, h, s);
                    }
                }
                if (lane < kTile) rows_info[stage * kTile + lane] = info;
                const uint4 *Kh = a.c.K + (size_t)h * a.c.head_step, *Vh = a.c.V + (size_t)h * a.c.head_step;
                const size_t own = ((size_t)ahead.n * H + h) * C;
                const int piece = lane % C;
                const uint32_t dst0 = ring + stage * (2 * R::kTileBytes);
#pragma unroll
                for (int i = 0; i < kTile * C / 32; ++i) {
                    const int row = i * (32 / C) + lane / C;
                    const uint32_t o = __shfl_sync(0xFFFFFFFFu, off, row);
                    const uint32_t dst = dst0 + row * (D * 2) + ((piece ^ (row & 7)) << 4);
                    const bool is_new = o == kRowNew;
                    const uint32_t bytes = o == kRowNone ? 0u : 16u;      // absent rows are filled with zeros
                    const size_t at = o == kRowNone ? 0 : o;
                    copy_piece(dst, (is_new ? a.k_new + own : Kh + at) + piece, bytes);
                    copy_piece(dst + R::kTileBytes, (is_new ? a.v_new + own : Vh + at) + piece, bytes);
                }
            }
            walk_on(a, units, ahead);
            look_up();
        }
        copies_commit();
    };

    look_up();
#pragma unroll 1
    for (int i = 0; i < S; ++i) copy_tile(i);

    uint32_t qf[NT][KS][2];
    float o[NT][MT][4], m[NT][2], l[NT][2];
    int stage = 0, first_block = 0;
    bool begin = true;
    while (use.left > 0) {
        const int hb = use.unit % head_blocks, h = use.unit / head_blocks;
        const int head0 = hb * 8 * NT;                                    // first query head of the block within the group
        const int heads = min(G - head0, 8 * NT);
        const size_t head_at = (size_t)use.n * Hq + (size_t)h * G + head0;
        if (begin) {
            begin = false;
            first_block = use.blk;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const bool there = nt * 8 + g < heads;
                const uint32_t *q = a.q + (head_at + nt * 8 + g) * (D / 2) + t;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qf[nt][ks][0] = there ? q[ks * 8] : 0u;
                    qf[nt][ks][1] = there ? q[ks * 8 + 4] : 0u;
                }
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
            }
        }
        copies_wait<S - 1>();
        __syncwarp();
        if (use.blk * kBlockRows + warp * kTile < use.rows) {
            const uint32_t base = ring + stage * (2 * R::kTileBytes);
            // S^T of this tile, even and odd steps in chains of their own
            float s[NT][4], s1[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] = s1[nt][i] = 0.f;
            {
                const int row = (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    uint32_t av[4];
                    load_matrices(av, base + row * (D * 2) + (((2 * ks + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) E::mma(ks & 1 ? s1[nt] : s[nt], av, qf[nt][ks][0], qf[nt][ks][1]);
                }
            }
            const uint32_t info0 = rows_info[stage * kTile + g], info1 = rows_info[stage * kTile + g + 8];
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[nt][i] = info0 != kRowNone ? (s[nt][i] + s1[nt][i]) * a.scale_log2e : -INFINITY;
                    s[nt][2 + i] = info1 != kRowNone ? (s[nt][2 + i] + s1[nt][2 + i]) * a.scale_log2e : -INFINITY;
                    raise |= fmaxf(s[nt][i], s[nt][2 + i]) > m[nt][i] + kLazy;
                }
                if (GATHER) {
                    const int hd = nt * 8 + 2 * t;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t info = r ? info1 : info0;
                        if (info == kRowNone) continue;
                        float *dst = info == kRowNew ? a.score_new + head_at : a.scores + (size_t)info * G + head0;
                        if (hd < heads) dst[hd] = s[nt][2 * r];
                        if (hd + 1 < heads) dst[hd + 1] = s[nt][2 * r + 1];
                    }
                }
            }
            if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float x = fmaxf(s[nt][i], s[nt][2 + i]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
                        const float mn = fmaxf(m[nt][i], x);
                        const float corr = mn == -INFINITY ? 1.f : fast_exp2(m[nt][i] - mn);   // first tile: 2^-inf = 0
                        m[nt][i] = mn;
                        l[nt][i] *= corr;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            o[nt][mt][i] *= corr;
                            o[nt][mt][2 + i] *= corr;
                        }
                    }
            }
            uint32_t hi[NT][2], lo[NT][2];       // P as the sum of two rounded parts: 16 bits of it or more meet V
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = fast_exp2(s[nt][i] - (m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1]));
                l[nt][0] += p[0] + p[2];
                l[nt][1] += p[1] + p[3];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t x = E::pack(p[2 * r], p[2 * r + 1]);
                    const float2 f = E::unpack(x);
                    hi[nt][r] = transpose8x8(x);
                    lo[nt][r] = transpose8x8(E::pack(p[2 * r] - f.x, p[2 * r + 1] - f.y));
                }
            }
            {
                const int row = (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    uint32_t av[4];
                    load_matrices_trans(av, base + R::kTileBytes + row * (D * 2) + (((2 * mt + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        E::mma(o[nt][mt], av, hi[nt][0], hi[nt][1]);
                        E::mma(o[nt][mt], av, lo[nt][0], lo[nt][1]);
                    }
                }
            }
        }
        __syncwarp();                            // every lane is done with the stage
        copy_tile(stage);
        stage = stage + 1 == S ? 0 : stage + 1;

        if (use.blk + 1 == use.nb || use.left == 1) {
            // the four warps' results meet in shared memory, four heads at a time
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x = l[nt][i];
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
                    if (g == 0) sm_ml[warp][nt * 8 + 2 * t + i] = make_float2(m[nt][i], x);
                }
            const bool whole = first_block == 0 && use.blk + 1 == use.nb;
            const int part = 2 * blockIdx.x + (first_block == 0 ? 1 : 0); // a CTA holds at most one part of each kind
            for (int hc = 0; hc * R::kMergeHeads < heads; ++hc) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (nt != (hc >> 1) || (t >> 1) != (hc & 1)) continue;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float *dst = sm_o + (warp * R::kMergeHeads + 2 * (t & 1) + i) * R::kPitch + g;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            dst[mt * 16] = o[nt][mt][i];
                            dst[mt * 16 + 8] = o[nt][mt][2 + i];
                        }
                    }
                }
                __syncthreads();
                const int hd = hc * R::kMergeHeads + warp;                // a warp per head
                if (hd < heads) {
                    float M = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm_ml[w][hd].x);
                    const float mu = M == -INFINITY ? 0.f : M;
                    float L = 0.f, f[kWarps];
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        f[w] = fast_exp2(sm_ml[w][hd].x - mu);
                        L = fmaf(sm_ml[w][hd].y, f[w], L);
                    }
                    const float inv = L == 0.f ? 0.f : 1.f / L;           // nothing left by the scores: the output is zero
#pragma unroll
                    for (int d = 0; d < D; d += 64) {
                        float2 A = make_float2(0.f, 0.f);
#pragma unroll
                        for (int w = 0; w < kWarps; ++w) {
                            const float2 v = *reinterpret_cast<const float2 *>(sm_o + (w * R::kMergeHeads + warp) * R::kPitch + d + 2 * lane);
                            A.x = fmaf(v.x, f[w], A.x);
                            A.y = fmaf(v.y, f[w], A.y);
                        }
                        if (whole) a.out[(head_at + hd) * (D / 2) + d / 2 + lane] = E::pack(A.x * inv, A.y * inv);
                        else *reinterpret_cast<float2 *>(a.part_o + ((size_t)part * 8 * NT + hd) * D + d + 2 * lane) = A;
                    }
                    if (lane == 0) {
                        if (whole) {
                            a.stat[head_at + hd] = make_float2(mu, inv);
                            if (a.lse) a.lse[head_at + hd] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
                        } else {
                            a.part_ml[(size_t)part * 8 * NT + hd] = make_float2(M, L);
                        }
                    }
                }
                __syncthreads();
            }
            if (!whole) {
                // the unit's first and last CTA follow from its first block; the last of them to get here joins the parts
                const long long b0 = (long long)plan.per * blockIdx.x + (plan.per - use.left) - use.blk;
                const int c0 = (int)(b0 / plan.per), c1 = (int)((b0 + use.nb - 1) / plan.per);
                int *arrived = a.c.state + kStateAttention + c0;          // a CTA is the first of one shared unit at most
                __threadfence();
                __syncthreads();
                if (threadIdx.x == 0) sm_last = atomicAdd(arrived, 1) == c1 - c0;
                __syncthreads();
                if (sm_last) {
                    __threadfence();
                    if (threadIdx.x == 0) *arrived = 0;
                    for (int hd = warp; hd < heads; hd += kWarps) {
                        float M = -INFINITY, L = 0.f;
                        for (int c = c0 + lane; c <= c1; c += 32) M = fmaxf(M, __ldcg(&a.part_ml[(size_t)(2 * c + (c == c0)) * 8 * NT + hd].x));
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, d));
                        const float mu = M == -INFINITY ? 0.f : M;
                        for (int c = c0 + lane; c <= c1; c += 32) {
                            const float2 v = __ldcg(&a.part_ml[(size_t)(2 * c + (c == c0)) * 8 * NT + hd]);
                            L = fmaf(v.y, fast_exp2(v.x - mu), L);
                        }
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, d);
                        const float inv = L == 0.f ? 0.f : 1.f / L;
                        if (lane == 0) {
                            sm_m[hd] = mu;
                            sm_inv[hd] = inv;
                            a.stat[head_at + hd] = make_float2(mu, inv);
                            if (a.lse) a.lse[head_at + hd] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
                        }
                    }
                    __syncthreads();
                    for (int i = threadIdx.x; i < heads * (D / 2); i += kThreads) {
                        const int hd = i / (D / 2), d = i - hd * (D / 2);
                        float2 A = make_float2(0.f, 0.f);
#pragma unroll 8
                        for (int c = c0; c <= c1; ++c) {
                            const size_t p = (size_t)(2 * c + (c == c0)) * 8 * NT + hd;
                            const float f = fast_exp2(__ldcg(&a.part_ml[p].x) - sm_m[hd]);
                            const float2 v = __ldcg(reinterpret_cast<const float2 *>(a.part_o + p * D + 2 * d));
                            A.x = fmaf(v.x, f, A.x);
                            A.y = fmaf(v.y, f, A.y);
                        }
                        a.out[(head_at + hd) * (D / 2) + d] = E::pack(A.x * sm_inv[hd], A.y * sm_inv[hd]);
                    }
                    __syncthreads();
                }
            }
            begin = true;
        }
        walk_on(a, units, use);
    }
}

// `splits` CTAs per (problem, head) add the probabilities to the weights.
__global__ void __launch_bounds__(kThreads) paged_weights_kernel(AttnArgs a, int splits)
{
    extern __shared__ float2 sm_stat[];          // [G]
    const int at = blockIdx.x / splits, z = blockIdx.x - at * splits;
    const int n = at / a.c.H, h = at - n * a.c.H;
    const int G = a.G;
    grid_wait();
    grid_release();
    const int len = read_len(a.c, n);
    const size_t head_at = ((size_t)n * a.c.H + h) * G;
    if (len < 0) {
        if (z == 0 && threadIdx.x == 0 && a.w_new) a.w_new[at] = 0.f;
        return;
    }
    for (int i = threadIdx.x; i < G; i += kThreads) sm_stat[i] = a.stat[head_at + i];
    __syncthreads();
    for (int row = z * kThreads + threadIdx.x; row < len; row += splits * kThreads) {
        const Slot s = find_slot(a.c, n, row);
        if (s.page < 0) continue;
        const size_t m = meta_index(a.c, h, s);
        float w = 0.f;
        for (int hd = 0; hd < G; ++hd) w = fmaf(fast_exp2(a.scores[m * G + hd] - sm_stat[hd].x), sm_stat[hd].y, w);
        a.c.weight[m] = fmaf(a.c.weight[m], a.decay, w);
    }
    if (z == 0 && threadIdx.x == 0 && a.w_new) {
        float w = 0.f;
        for (int hd = 0; hd < G; ++hd) w = fmaf(fast_exp2(a.score_new[head_at + hd] - sm_stat[hd].x), sm_stat[hd].y, w);
        a.w_new[at] = w;
    }
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

inline int sm_count_here()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 148;
    return n;
}

struct WsLayout {
    size_t stat, score_new, part_o, part_ml, scores, total;
};

WsLayout layout(int N, int H, int D, int n_pages, int page_size, int G, int accumulate)
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
    w.scores = take(accumulate ? (size_t)n_pages * H * page_size * G * sizeof(float) : 0);
    w.total = at;
    return w;
}

template <typename E, int D, int NT, bool GATHER>
cudaError_t launch(const AttnArgs &a, cudaStream_t stream)
{
    const int head_blocks = (a.G + 8 * NT - 1) / (8 * NT);
    int ctas = sm_count_here() * kCtasPerSm;
    if (ctas > kPagedMaxCtas) ctas = kPagedMaxCtas;
    cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<E, D, NT, GATHER>, cudaFuncAttributeMaxDynamicSharedMemorySize, Ring<D>::kSmem);
    if (e != cudaSuccess) return e;
    e = launch_chained(paged_attention_kernel<E, D, NT, GATHER>, dim3((unsigned)ctas), kThreads, Ring<D>::kSmem, stream, a, head_blocks, 2);
    if (e != cudaSuccess || !GATHER) return e;
    // enough CTAs for the GPU, no more than there are rows
    const long long units = (long long)a.c.N * a.c.H;
    long long z = (148LL * 8 + units - 1) / units;
    const long long most = ((long long)a.c.max_pages * a.c.page_size + kThreads - 1) / kThreads;
    if (z > most) z = most;
    return launch_chained(paged_weights_kernel, dim3((unsigned)(z * units)), kThreads, a.G * sizeof(float2), stream, a, (int)z);
}

template <typename E, int D>
cudaError_t launch_d(const AttnArgs &a, int accumulate, cudaStream_t stream)
{
    if (a.G <= 8) return accumulate ? launch<E, D, 1, true>(a, stream) : launch<E, D, 1, false>(a, stream);
    return accumulate ? launch<E, D, 2, true>(a, stream) : launch<E, D, 2, false>(a, stream);
}

}  // namespace

size_t paged_attention_workspace_bytes(const ec_paged *c, int Hq, int accumulate)
{
    return layout(c->N, c->H, c->D, c->n_pages, c->page_size, Hq / c->H, accumulate).total;
}

cudaError_t launch_paged_attention(const PagedView &c, int D, int dtype, const void *q, const void *k_new, const void *v_new,
                                   int Hq, float scale, int accumulate, float decay, void *out, float *lse, float *w_new,
                                   void *ws, cudaStream_t stream)
{
    AttnArgs a;
    a.c = c;
    a.q = static_cast<const uint32_t *>(q);
    a.k_new = static_cast<const uint4 *>(k_new);
    a.v_new = static_cast<const uint4 *>(v_new);
    a.G = Hq / c.H;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.decay = decay;
    a.out = static_cast<uint32_t *>(out);
    a.lse = lse;
    a.w_new = k_new ? w_new : nullptr;
    const WsLayout w = layout(c.N, c.H, D, c.n_pages, c.page_size, a.G, accumulate);
    char *p = static_cast<char *>(ws);
    a.stat = reinterpret_cast<float2 *>(p + w.stat);
    a.score_new = reinterpret_cast<float *>(p + w.score_new);
    a.part_o = reinterpret_cast<float *>(p + w.part_o);
    a.part_ml = reinterpret_cast<float2 *>(p + w.part_ml);
    a.scores = reinterpret_cast<float *>(p + w.scores);
    if (dtype == EC_BF16) return D == 128 ? launch_d<Bf16, 128>(a, accumulate, stream) : launch_d<Bf16, 64>(a, accumulate, stream);
    return D == 128 ? launch_d<Fp16, 128>(a, accumulate, stream) : launch_d<Fp16, 64>(a, accumulate, stream);
}

}  // namespace ec
