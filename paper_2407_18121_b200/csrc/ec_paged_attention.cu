// Attention of one new token per problem over a paged cache (grouped query heads), with the probability every
// cached row receives added to the row's gathered weight.
//   x[g][j] = scale * <q_g, k_j>,  p = softmax_j(x),  out_g = sum_j p[g][j] v_j,  weight_j <- decay * weight_j + sum_g p[g][j]
// Bound by the K and V rows read from HBM (4 D bytes per row and head); the products ride on mma.sync, whose rate
// (16 instructions per 16 rows and 8 query heads) is far above what the loads can feed, so the tcgen05 pipe would
// only add latency here: a tile has 8 to 16 query rows, not 128.
//  - Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that the 16-row side of the instruction
//    is the cache and the 8-column side the group's query heads: a group of 8 or fewer wastes nothing but columns.
//  - The contraction index of S and the row index of O^T may be permuted freely, so a thread takes whole 16-byte pieces
//    of K and V rows straight from global memory as its fragments: no shared memory, no ldmatrix. V's pairs of
//    consecutive rows are formed with byte permutes, P goes from accumulator to operand layout with movmatrix.
//  - Work is handed out in blocks of 64 rows, evenly over the CTAs of one resident wave, from the lengths on the device: a
//    ragged batch and one long sequence spread alike. A CTA's share is at most one partial unit at either end and
//    whole units between; a second launch joins the partial results and, with the final normaliser, turns the stored
//    scores into weights.
#include "ec_paged.cuh"

namespace ec {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;                        // rows of a warp's tile
constexpr int kBlockRows = kWarps * kTile;       // rows of a block, the unit of work distribution
constexpr int kMaxCtas = 148 * 4;
constexpr float kLazy = 8.f;                     // the running maximum is raised when exceeded by more than this (log2)

struct Bf16 {
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b); }
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

__device__ __forceinline__ uint4 load_piece(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

struct AttnArgs {
    PagedView c;
    const uint4 *q, *k_new, *v_new;              // k_new == nullptr: the cached rows alone
    int G;                                       // query heads per key / value head
    float scale_log2e, decay;
    void *out;
    float *lse, *w_new;
    // workspace
    int *plan;                                   // [0]: blocks per CTA, [1 + n]: blocks of a head in front of problem n
    float2 *stat;                                // [N, Hq] (maximum in the log2 domain, sum) of units held by one CTA
    float *score_new;                            // [N, Hq] score of the step's own row
    float *part_o;                               // [2 * CTAs][8 NT][D]
    float2 *part_ml;                             // [2 * CTAs][8 NT]
    float *scores;                               // [n_pages, H, page_size, G], log2 domain
};

// Blocks of one head of problem n: a step's own row rides with the last block.
__device__ __forceinline__ int blocks_of(const AttnArgs &a, int n, int &len)
{
    len = read_len(a.c, n);
    if (len < 0 || (len == 0 && !a.k_new)) return 0;
    return len == 0 ? 1 : (len + kBlockRows - 1) / kBlockRows;
}

// Every CTA derives the same plan from the lengths: `per` blocks for each CTA. Returns the CTA's first problem and the
// number of blocks (of all its heads) in front of that problem through shared memory.
struct Plan {
    int per, n;                                  // n < 0: nothing to do
    long long before;                            // blocks in front of problem n
};

__device__ __forceinline__ void make_plan(const AttnArgs &a, int units_per_problem, int min_per, Plan *shared_plan)
{
    __shared__ long long warp_sum[kWarps];
    const int N = a.c.N;
    const int span = (N + kThreads - 1) / kThreads;
    const int n0 = min((int)threadIdx.x * span, N), n1 = min(n0 + span, N);
    long long mine = 0;
    for (int n = n0; n < n1; ++n) {
        int len;
        mine += blocks_of(a, n, len);
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if ((threadIdx.x & 31) >= o) incl += up;
    }
    if ((threadIdx.x & 31) == 31) warp_sum[threadIdx.x >> 5] = incl;
    if (threadIdx.x == 0) shared_plan->n = -1;
    __syncthreads();
    long long total = 0, base = incl - mine;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < (int)(threadIdx.x >> 5)) base += warp_sum[w];
        total += warp_sum[w];
    }
    const long long all = total * units_per_problem;
    long long per = (all + gridDim.x - 1) / gridDim.x;
    if (per < min_per) per = min_per;
    const long long first = per * blockIdx.x;
    if (threadIdx.x == 0) shared_plan->per = (int)per;
    // the thread whose span holds the CTA's first block names the problem
    const long long b0 = base * units_per_problem, b1 = (base + mine) * units_per_problem;
    const bool publish = blockIdx.x == 0;
    if (publish || (first >= b0 && first < b1)) {
        long long at = base;
        for (int n = n0; n < n1; ++n) {
            int len;
            const int nb = blocks_of(a, n, len);
            if (publish) a.plan[1 + n] = (int)at;
            if (first >= at * units_per_problem && first < (at + nb) * units_per_problem) {
                shared_plan->n = n;
                shared_plan->before = at * units_per_problem;
            }
            at += nb;
        }
    }
    if (publish && threadIdx.x == 0) a.plan[0] = (int)per;
    __syncthreads();
}

// NT: groups of 8 query heads that share a pass over the rows. GATHER: scores are stored for the weights.
template <typename E, int D, int NT, bool GATHER>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 3 : 2) paged_attention_kernel(AttnArgs a, int head_blocks, int min_per)
{
    constexpr int C = D / 8;                     // 16-byte pieces of a row
    constexpr int KI = C / 4, VJ = C / 8, MT = D / 16;
    __shared__ float sm_o[kWarps][8 * NT][D];
    __shared__ float sm_m[kWarps][8 * NT], sm_l[kWarps][8 * NT];
    __shared__ Plan plan;

    grid_wait();
    grid_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.G, H = a.c.H, Hq = H * G;
    const int units_per_problem = H * head_blocks;
    make_plan(a, units_per_problem, min_per, &plan);
    if (plan.n < 0) return;
    const int per = plan.per;
    long long b = (long long)per * blockIdx.x;
    const long long b_end = b + per;
    int n = plan.n;
    long long before = plan.before;

    while (b < b_end) {
        int len;
        const int nb = blocks_of(a, n, len);
        if (b >= before + (long long)nb * units_per_problem) {            // this problem is done (or has no rows)
            before += (long long)nb * units_per_problem;
            if (++n >= a.c.N) break;
            continue;
        }
        const int unit = (int)((b - before) / nb);                        // (head, head block) of the problem
        const int first_block = (int)((b - before) - (long long)unit * nb);
        const int last_block = (int)min((long long)nb, first_block + (b_end - b));
        const int h = unit / head_blocks, hb = unit - h * head_blocks;
        const int head0 = hb * 8 * NT;                                    // first query head of the block within the group
        const int heads = min(G - head0, 8 * NT);
        const int has_new = a.k_new != nullptr;
        const int row_end = last_block == nb ? len + has_new : last_block * kBlockRows;

        const uint4 *Kh = a.c.K + (size_t)h * a.c.head_step, *Vh = a.c.V + (size_t)h * a.c.head_step;
        const uint4 *kn = a.k_new + ((size_t)n * H + h) * C, *vn = a.v_new + ((size_t)n * H + h) * C;

        uint4 qf[NT][KI];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool there = nt * 8 + g < heads;
#pragma unroll
            for (int i = 0; i < KI; ++i)
                qf[nt][i] = there ? a.q[((size_t)n * Hq + (size_t)h * G + head0 + nt * 8 + g) * C + t + 4 * i] : make_uint4(0, 0, 0, 0);
        }

        float o[NT][MT][4];
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
        }

        // Lane i (and i + 16) describes row i of a tile; the others learn it by shuffle.
        uint32_t off_mine, meta_mine;
        auto describe = [&](int row0) {
            const int row = row0 + (lane & 15);
            off_mine = kRowNone;
            meta_mine = 0;
            if (row < row_end) {
                if (row >= len) {
                    off_mine = kRowNew;
                } else {
                    const Slot s = find_slot(a.c, n, row);
                    if (s.page >= 0) {
                        off_mine = row_offset(a.c, s);
                        meta_mine = meta_index(a.c, h, s);
                    }
                }
            }
        };
        uint4 rk[2][KI], rv[4][VJ];
        uint32_t off_k[2];
        auto load_k = [&]() {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint32_t off = __shfl_sync(0xFFFFFFFFu, off_mine, g + 8 * r);
                off_k[r] = off;
                const uint4 *p = off == kRowNew ? kn : Kh + off;
#pragma unroll
                for (int i = 0; i < KI; ++i) rk[r][i] = off != kRowNone ? load_piece(p + t + 4 * i) : make_uint4(0, 0, 0, 0);
            }
        };
        auto load_v = [&](uint32_t off_tile) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t off = __shfl_sync(0xFFFFFFFFu, off_tile, 2 * t + (r & 1) + 8 * (r >> 1));
                const uint4 *p = off == kRowNew ? vn : Vh + off;
#pragma unroll
                for (int j = 0; j < VJ; ++j) rv[r][j] = off != kRowNone ? load_piece(p + g + 8 * j) : make_uint4(0, 0, 0, 0);
            }
        };

        int row0 = first_block * kBlockRows + warp * kTile;
        if (row0 < row_end) {
            describe(row0);
            load_k();
            load_v(off_mine);
        }
        for (; row0 < row_end; row0 += kBlockRows) {
            // S^T of this tile
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] = 0.f;
#pragma unroll
                for (int i = 0; i < KI; ++i) {
                    const uint32_t a0[4] = {rk[0][i].x, rk[1][i].x, rk[0][i].y, rk[1][i].y};
                    E::mma(s[nt], a0, qf[nt][i].x, qf[nt][i].y);
                    const uint32_t a1[4] = {rk[0][i].z, rk[1][i].z, rk[0][i].w, rk[1][i].w};
                    E::mma(s[nt], a1, qf[nt][i].z, qf[nt][i].w);
                }
            }
            const bool there0 = off_k[0] != kRowNone, there1 = off_k[1] != kRowNone;
            uint32_t meta0 = 0, meta1 = 0;
            bool new0 = false, new1 = false;
            if (GATHER) {
                meta0 = __shfl_sync(0xFFFFFFFFu, meta_mine, g);
                meta1 = __shfl_sync(0xFFFFFFFFu, meta_mine, g + 8);
                new0 = off_k[0] == kRowNew;
                new1 = off_k[1] == kRowNew;
            }
            const bool more = row0 + kBlockRows < row_end;                // uniform over the warp
            if (more) {
                describe(row0 + kBlockRows);
                load_k();
            }
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[nt][i] = there0 ? s[nt][i] * a.scale_log2e : -INFINITY;
                    s[nt][2 + i] = there1 ? s[nt][2 + i] * a.scale_log2e : -INFINITY;
                    raise |= fmaxf(s[nt][i], s[nt][2 + i]) > m[nt][i] + kLazy;
                }
                if (GATHER) {
                    const int hd = nt * 8 + 2 * t;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        if (!(r ? there1 : there0)) continue;
                        float *dst = (r ? new1 : new0) ? a.score_new + (size_t)n * Hq + (size_t)h * G + head0
                                                       : a.scores + (size_t)(r ? meta1 : meta0) * G + head0;
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
            uint32_t pb[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float mu = m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1];
                    p[i] = fast_exp2(s[nt][i] - mu);
                }
                l[nt][0] += p[0] + p[2];                                  // the sum takes the weights before they are rounded
                l[nt][1] += p[1] + p[3];
                pb[nt][0] = transpose8x8(E::pack(p[0], p[1]));
                pb[nt][1] = transpose8x8(E::pack(p[2], p[3]));
            }
            // O^T += V^T P^T: the two halves of a packed word are two rows of V^T
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int j = mt >> 2, w = mt & 3;
                const uint32_t x0 = word(rv[0][j], w), x1 = word(rv[1][j], w), x2 = word(rv[2][j], w), x3 = word(rv[3][j], w);
                const uint32_t av[4] = {__byte_perm(x0, x1, 0x5410), __byte_perm(x0, x1, 0x7632), __byte_perm(x2, x3, 0x5410),
                                        __byte_perm(x2, x3, 0x7632)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) E::mma(o[nt][mt], av, pb[nt][0], pb[nt][1]);
            }
            if (more) load_v(off_mine);
        }

        // the four warps' results meet in shared memory
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = l[nt][i];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
                const int hd = nt * 8 + 2 * t + i;
                if (g == 0) {
                    sm_m[warp][hd] = m[nt][i];
                    sm_l[warp][hd] = x;
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const int d0 = 8 * (g + 8 * (mt >> 2)) + 2 * (mt & 3);
                    *reinterpret_cast<float2 *>(&sm_o[warp][hd][d0]) = make_float2(o[nt][mt][i], o[nt][mt][2 + i]);
                }
            }
        __syncthreads();
        const bool whole = first_block == 0 && last_block == nb;
        const int part = 2 * blockIdx.x + (first_block == 0 ? 1 : 0);     // a CTA holds at most one part of each kind
        for (int i = threadIdx.x; i < heads * (D / 2); i += kThreads) {
            const int hd = i / (D / 2), d = 2 * (i - hd * (D / 2));
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm_m[w][hd]);
            const float mu = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            float2 A = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = fast_exp2(sm_m[w][hd] - mu);
                const float2 v = *reinterpret_cast<const float2 *>(&sm_o[w][hd][d]);
                L = fmaf(sm_l[w][hd], f, L);
                A.x = fmaf(v.x, f, A.x);
                A.y = fmaf(v.y, f, A.y);
            }
            if (whole) {
                const size_t at = (size_t)n * Hq + (size_t)h * G + head0 + hd;
                const float inv = L == 0.f ? 0.f : 1.f / L;               // nothing left by the scores: the output is zero
                reinterpret_cast<uint32_t *>(a.out)[(at * D + d) >> 1] = E::pack(A.x * inv, A.y * inv);
                if (d == 0) {
                    a.stat[at] = make_float2(M, L);
                    if (a.lse) a.lse[at] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
                }
            } else {
                *reinterpret_cast<float2 *>(&a.part_o[((size_t)part * 8 * NT + hd) * D + d]) = A;
                if (d == 0) a.part_ml[(size_t)part * 8 * NT + hd] = make_float2(M, L);
            }
        }
        __syncthreads();
        b += last_block - first_block;
    }
}

// `splits` CTAs per (problem, head): joins the parts of units that several CTAs shared, and adds the probabilities to the weights.
template <typename E, int D, int NT, bool GATHER>
__global__ void __launch_bounds__(kThreads) paged_finish_kernel(AttnArgs a, int head_blocks, int splits)
{
    extern __shared__ float sm[];                // [G] maximum, [G] 1 / sum
    const int at = blockIdx.x / splits, z = blockIdx.x - at * splits;
    const int n = at / a.c.H, h = at - n * a.c.H;
    const int G = a.G, H = a.c.H, Hq = H * G;
    float *sm_m = sm, *sm_inv = sm + G;
    grid_wait();
    grid_release();
    int len;
    const int nb = blocks_of(a, n, len);
    const size_t head_at = (size_t)n * Hq + (size_t)h * G;
    if (nb == 0) {
        if (z == 0) {
            for (int i = threadIdx.x; i < G * (D / 2); i += kThreads) reinterpret_cast<uint32_t *>(a.out)[head_at * (D / 2) + i] = 0;
            if (a.lse)
                for (int i = threadIdx.x; i < G; i += kThreads) a.lse[head_at + i] = -INFINITY;
            if (GATHER && a.w_new && threadIdx.x == 0) a.w_new[(size_t)n * H + h] = 0.f;
        }
        return;
    }
    const int per = a.plan[0];
    const long long before = (long long)a.plan[1 + n] * H * head_blocks;
    // normaliser of every query head of the group: a warp per head
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int hd = warp; hd < G; hd += kWarps) {
        const int hb = hd / (8 * NT), in = hd - hb * 8 * NT;
        const long long u0 = before + (long long)(h * head_blocks + hb) * nb;
        const int c0 = (int)(u0 / per), c1 = (int)((u0 + nb - 1) / per);
        float M, L;
        if (c0 == c1) {
            const float2 s = a.stat[head_at + hd];
            M = s.x;
            L = s.y;
        } else {
            M = -INFINITY;
            for (int c = c0 + lane; c <= c1; c += 32) M = fmaxf(M, a.part_ml[(size_t)(2 * c + (c == c0)) * 8 * NT + in].x);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, d));
            const float mu = M == -INFINITY ? 0.f : M;
            L = 0.f;
            for (int c = c0 + lane; c <= c1; c += 32) {
                const float2 s = a.part_ml[(size_t)(2 * c + (c == c0)) * 8 * NT + in];
                L = fmaf(s.y, fast_exp2(s.x - mu), L);
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, d);
            if (z == 0 && lane == 0 && a.lse) a.lse[head_at + hd] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
        }
        if (lane == 0) {
            sm_m[hd] = M == -INFINITY ? 0.f : M;
            sm_inv[hd] = L == 0.f ? 0.f : 1.f / L;
        }
    }
    __syncthreads();
    // outputs of shared units, spread over the row splits by head
    for (int hd = z; hd < G; hd += splits) {
        const int hb = hd / (8 * NT), in = hd - hb * 8 * NT;
        const long long u0 = before + (long long)(h * head_blocks + hb) * nb;
        const int c0 = (int)(u0 / per), c1 = (int)((u0 + nb - 1) / per);
        if (c0 == c1) continue;
        for (int d = threadIdx.x; d < D / 2; d += kThreads) {
            float2 A = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int c = c0; c <= c1; ++c) {
                const size_t part = (size_t)(2 * c + (c == c0)) * 8 * NT + in;
                const float f = fast_exp2(a.part_ml[part].x - sm_m[hd]);
                const float2 v = *reinterpret_cast<const float2 *>(&a.part_o[part * D + 2 * d]);
                A.x = fmaf(v.x, f, A.x);
                A.y = fmaf(v.y, f, A.y);
            }
            reinterpret_cast<uint32_t *>(a.out)[(head_at + hd) * (D / 2) + d] = E::pack(A.x * sm_inv[hd], A.y * sm_inv[hd]);
        }
    }
    if (GATHER) {
        for (int row = z * kThreads + threadIdx.x; row < len; row += splits * kThreads) {
            const Slot s = find_slot(a.c, n, row);
            if (s.page < 0) continue;
            const size_t m = meta_index(a.c, h, s);
            float w = 0.f;
            for (int hd = 0; hd < G; ++hd) w = fmaf(fast_exp2(a.scores[m * G + hd] - sm_m[hd]), sm_inv[hd], w);
            a.c.weight[m] = fmaf(a.c.weight[m], a.decay, w);
        }
        if (z == 0 && threadIdx.x == 0 && a.w_new) {
            float w = 0.f;
            for (int hd = 0; hd < G; ++hd) w = fmaf(fast_exp2(a.score_new[head_at + hd] - sm_m[hd]), sm_inv[hd], w);
            a.w_new[(size_t)n * H + h] = w;
        }
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
    size_t plan, stat, score_new, part_o, part_ml, scores, total;
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
    w.plan = take(((size_t)N + 1) * sizeof(int));
    w.stat = take((size_t)N * H * G * sizeof(float2));
    w.score_new = take((size_t)N * H * G * sizeof(float));
    w.part_o = take((size_t)2 * kMaxCtas * 8 * nt * D * sizeof(float));
    w.part_ml = take((size_t)2 * kMaxCtas * 8 * nt * sizeof(float2));
    w.scores = take(accumulate ? (size_t)n_pages * H * page_size * G * sizeof(float) : 0);
    w.total = at;
    return w;
}

template <typename E, int D, int NT, bool GATHER>
cudaError_t launch(const AttnArgs &a, cudaStream_t stream)
{
    const int head_blocks = (a.G + 8 * NT - 1) / (8 * NT);
    int ctas = sm_count_here() * (NT == 1 ? 3 : 2);
    if (ctas > kMaxCtas) ctas = kMaxCtas;
    cudaError_t e = launch_chained(paged_attention_kernel<E, D, NT, GATHER>, dim3((unsigned)ctas), kThreads, 0, stream, a, head_blocks, 2);
    if (e != cudaSuccess) return e;
    // enough CTAs for the GPU, no more than there are rows (or query heads to join)
    const long long units = (long long)a.c.N * a.c.H;
    long long z = (148LL * 8 + units - 1) / units;
    const long long cap = (long long)a.c.max_pages * a.c.page_size;
    const long long rows = GATHER ? (cap + kThreads - 1) / kThreads : 1;
    const long long most = rows > a.G ? rows : a.G;
    if (z > most) z = most;
    if (z < 1) z = 1;
    return launch_chained(paged_finish_kernel<E, D, NT, GATHER>, dim3((unsigned)(z * units)), kThreads,
                          2 * a.G * sizeof(float), stream, a, head_blocks, (int)z);
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
    a.q = static_cast<const uint4 *>(q);
    a.k_new = static_cast<const uint4 *>(k_new);
    a.v_new = static_cast<const uint4 *>(v_new);
    a.G = Hq / c.H;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.decay = decay;
    a.out = out;
    a.lse = lse;
    a.w_new = k_new ? w_new : nullptr;
    const WsLayout w = layout(c.N, c.H, D, c.n_pages, c.page_size, a.G, accumulate);
    char *p = static_cast<char *>(ws);
    a.plan = reinterpret_cast<int *>(p + w.plan);
    a.stat = reinterpret_cast<float2 *>(p + w.stat);
    a.score_new = reinterpret_cast<float *>(p + w.score_new);
    a.part_o = reinterpret_cast<float *>(p + w.part_o);
    a.part_ml = reinterpret_cast<float2 *>(p + w.part_ml);
    a.scores = reinterpret_cast<float *>(p + w.scores);
    if (dtype == EC_BF16) return D == 128 ? launch_d<Bf16, 128>(a, accumulate, stream) : launch_d<Bf16, 64>(a, accumulate, stream);
    return D == 128 ? launch_d<Fp16, 128>(a, accumulate, stream) : launch_d<Fp16, 64>(a, accumulate, stream);
}

}  // namespace ec
