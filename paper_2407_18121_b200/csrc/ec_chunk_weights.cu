// The attention that the queries of a chunk of new tokens leave on the rows of a paged cache, added to the rows' weights:
//   p[t, g, j] = exp(scale * <q, k_j> - lse[t, g]) for rows j <= lens[n] - counts[n] + t, else 0
//   weight_j <- decay^count * weight_j + sum_t decay^(count - 1 - t) sum_g p[t, g, j]
// which is what `count` steps of one token each would have left.
//
// One contraction, K Q^T with a cached row to a TMEM lane and the queries as columns, so that a thread adds up its row's
// probabilities and nothing has to be exchanged. The decay and the normaliser are one number a column, worked out in 64 bits and
// rounded once to fp32:
//   2^(c S + n),  n = -lse log2(e) + (count - 1 - t) log2(decay)
// Four teams of four warps hold 512 rows of a head, the query tiles (and their numbers) stream past: a query tile is fetched once per
// 512 rows, a row once. A team's S is the only one that it has; while its threads compute, the products fill the other teams'.
// One pair of exponentials in four is a polynomial, 6e-6 off, where a warp's rows are seen by all tokens of a query tile.
// Units are cut over the CTAs along the queries; the parts are added in the order of the tokens by whoever arrives last.
// Bound: the special functions, at 65% of their rate: about 4700 clocks for the four tiles of S that a query tile meets, 3070 of them
// exponentials. 8192 tokens of 32 heads on 8, D = 128: 333 to 339 us by the box, 0.82 PFLOP/s (168 us at the rate of a large library product; 293 in a
// short run, 301 with two warps more that did nothing; S handed back a chunk earlier 299 to 339, with its spills). 32 problems of up to 8 tokens on up to 8192 rows:
// 34 us, of which 8 are the rows' bytes; the rest is starting and one query tile's latency per unit: a unit's rows are asked for when the
// products of the one before are done, its queries before that (behind the rows: 35). Each team's rows let go behind its own last product
// gained nothing there and cost the long prompt 4%. A thread spills 40 bytes.
#include "ec_chunk.cuh"

namespace ec {

namespace {

constexpr int kTeams = 4;                        // of four warps, with a tile of 128 cached rows each
constexpr int kBlockRows = kTeams * kTileRows;   // cached rows of a unit: the query tiles stream past all of them at once
constexpr int kThreads = 64 + kTeams * 128;      // warps: copies, products, teams
constexpr int kItems = 4;
constexpr int kStages = 3;                       // query tiles
constexpr int kTmemCols = 512;                   // S of every team
// Cost of a unit beside its query tiles, and the smallest share of a CTA, in query tiles. 1, 2 and 4 a unit: 32 problems of few tokens 43.2,
// 39.6 and 36.9 us, the odd batch 32.8, 30.7 and 30.7, 8192 tokens 333.1, 334.6 and 336.6. 3, 6 and 12 a share: few tokens 39.7, 39.6 and
// 43.9, the odd batch 26.6, 30.7 and 43.6, 8192 tokens within 0.2%.
constexpr int kUnitTiles = 2;
constexpr int kLeastTiles = 6;
constexpr double kLog2eWide = 1.4426950408889634074;

struct WeightArgs : ChunkArgs {
    const float *lse;                            // [tokens, Hq]
    double log2_decay;
    float *part;                                 // workspace: [2 CTAs][512]
};

struct BlockUnits {                              // a unit: kBlockRows cached rows of a head; its cost is counted in tokens
    static __device__ __forceinline__ int units(const WeightArgs &, const Problem &p) { return (p.len + kBlockRows - 1) / kBlockRows; }
    static __device__ __forceinline__ long long before(const WeightArgs &a, const Problem &p, int, int i)
    {
        // block j is first seen by token max(0, kBlockRows j - base)
        const long long base = p.len - p.count, fixed = (long long)kUnitTiles * a.tile_tokens;
        const long long all = base >= 0 ? base / kBlockRows + 1 : 0;      // blocks that every token sees
        const long long k = min((long long)i, all), m = i - k;
        return k * (p.count + fixed) + m * (p.count + base + fixed) - kBlockRows * (k * m + m * (m - 1) / 2);
    }
};

struct Item {
    int n, h;                                    // n < 0: no work left
    int row0, len;                               // the block's first row, rows of the problem
    int start, count;                            // tokens of the problem
    int qt0, qt1;                                // query tiles of this CTA
    int parts, first, slot;                      // parts > 0: the unit is shared by CTAs first .. first + parts - 1
    int pad;
};

template <int D>
struct Smem {
    static constexpr int kTile = kTileRows * D * 2;
    static constexpr int kK = 0;                                          // a tile per team
    static constexpr int kQ = kTeams * kTile;
    static constexpr int kLse = kQ + kStages * kTile;
    static constexpr int kItem = kLse + kStages * kTileRows * 4;
    static constexpr int kBars = kItem + kItems * (int)sizeof(Item);
    // q_full[stages], q_empty[stages], per team: k_full, k_empty, s_full, s_empty, rdv; item_full, item_empty
    static constexpr int kNumBars = 2 * kStages + 5 * kTeams + 2 * kItems;
    static constexpr int kTmemSlot = kBars + kNumBars * 8;
    static constexpr int kAbort = kTmemSlot + 4;
    static constexpr int kLast = kAbort + 4;
    static constexpr int kOdd = kLast + 4 * kTeams;                       // [stages] whether a normaliser of the tile is not finite
    static constexpr int kTotal = kOdd + 4 * kStages;
    static_assert(kTotal <= 232448, "shared memory of a block");
};

// 2^x for a negative x of any size, in fp32's own accuracy.
__device__ __forceinline__ float exp2_of(double x)
{
    const double whole = rint(x);
    return whole < -160.0 ? 0.f : ldexpf(exp2f((float)(x - whole)), (int)whole);
}

template <int D, int DTYPE>
__global__ void __launch_bounds__(kThreads, 1)
chunk_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const WeightArgs a)
{
    using L = Smem<D>;
    constexpr int kTile = L::kTile;
    constexpr int kBoxBytes = kTileRows * 128;
    constexpr uint32_t kFormat = DTYPE == EC_BF16 ? 1u : 0u;
    // S = K Q^T: M = 128 cached rows, N = 128 query rows, both K-major
    constexpr uint32_t kIdesc = (1u << 4) | (kFormat << 7) | (kFormat << 10) | ((kTileRows >> 3) << 17) | ((kTileRows >> 4) << 24);

    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    auto bar = [&](int i) { return base + (uint32_t)L::kBars + 8u * (uint32_t)i; };
    auto q_full = [&](uint32_t s) { return bar(s); };
    auto q_empty = [&](uint32_t s) { return bar(kStages + s); };
    constexpr int kT0 = 2 * kStages;
    auto k_full = [&](uint32_t x) { return bar(kT0 + 5 * x); };
    auto k_empty = [&](uint32_t x) { return bar(kT0 + 5 * x + 1); };
    auto s_full = [&](uint32_t x) { return bar(kT0 + 5 * x + 2); };
    auto s_empty = [&](uint32_t x) { return bar(kT0 + 5 * x + 3); };
    auto rdv = [&](uint32_t x) { return bar(kT0 + 5 * x + 4); };
    constexpr int kI0 = kT0 + 5 * kTeams;
    auto item_full = [&](uint32_t k) { return bar(kI0 + k); };
    auto item_empty = [&](uint32_t k) { return bar(kI0 + kItems + k); };
    Item *items = reinterpret_cast<Item *>(smem + L::kItem);
    float *lse_s = reinterpret_cast<float *>(smem + L::kLse);
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kTmemSlot);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kAbort);
    volatile int *last_s = reinterpret_cast<volatile int *>(smem + L::kLast);
    volatile int *odd_s = reinterpret_cast<volatile int *>(smem + L::kOdd);
    int *status = a.c.state;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (uint32_t s = 0; s < (uint32_t)kStages; ++s) { mbar_init(q_full(s), 1); mbar_init(q_empty(s), 1 + 4 * kTeams); }
        for (uint32_t x = 0; x < (uint32_t)kTeams; ++x) {
            mbar_init(k_full(x), 1);
            mbar_init(k_empty(x), 1);
            mbar_init(s_full(x), 1);
            mbar_init(s_empty(x), 4);
            mbar_init(rdv(x), 4);
        }
        for (uint32_t k = 0; k < (uint32_t)kItems; ++k) {
            mbar_init(item_full(k), 1);
            mbar_init(item_empty(k), 1 + 4 * kTeams);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_to_async();
    }
    // Rows of a query tile that no copy fills: zeros, so that their scores are finite and the normaliser of -inf hides them.
    for (int i = threadIdx.x; i < kStages * (D / 64) * (kTileRows - a.tile_tokens * a.G) * 8; i += kThreads) {
        const int row = a.tile_tokens * a.G + (i >> 3) % (kTileRows - a.tile_tokens * a.G), tile = (i >> 3) / (kTileRows - a.tile_tokens * a.G);
        *reinterpret_cast<uint4 *>(smem + L::kQ + tile * kBoxBytes + row * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_to_async();
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(base + (uint32_t)L::kTmemSlot), "r"((uint32_t)kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_wait();

    // Whether any token of query tile q sees a row of team x's tile.
    auto meets = [&](const Item &it, uint32_t x, int q) {
        const int row = it.row0 + (int)x * kTileRows, last = min(it.count, (q + 1) * a.tile_tokens) - 1;
        return row < it.len && row <= it.len - it.count + last;
    };
    bool alive = true;

    if (warp == 0) {
        // ------------------------------------------------------------ plan and copies
        Walk<BlockUnits> w;
        bool more = w.begin(a, (long long)kLeastTiles * a.tile_tokens);
        uint32_t nk = 0, asked = 0, nq = 0;       // per team one bit: the parity of its copies, whether there were any; query tiles
        for (uint32_t k = 0; alive; ++k) {
            const uint32_t sl = k % kItems;
            Item it = {};
            it.n = -1;
            long long cost = 0;
            while (more) {                                // the next unit that this CTA has something of
                it.row0 = w.i * kBlockRows;
                it.len = w.p.len;
                it.start = w.p.start;
                it.count = w.p.count;
                const int begin = max(0, it.row0 - (it.len - it.count)) / a.tile_tokens, end = (it.count + a.tile_tokens - 1) / a.tile_tokens;
                cost = BlockUnits::before(a, w.p, w.units, w.i + 1) - BlockUnits::before(a, w.p, w.units, w.i);
                const Cut cut = cut_unit(w.s, w.at, cost, kUnitTiles * a.tile_tokens, a.tile_tokens, end - begin);
                if (cut.mine) {
                    it.n = w.n;
                    it.h = w.h;
                    it.qt0 = begin + cut.t0;
                    it.qt1 = begin + cut.t1;
                    it.first = cut.first;
                    it.parts = cut.parts;
                    it.slot = 2 * (int)blockIdx.x + (cut.first == (int)blockIdx.x);
                    break;
                }
                more = w.next(a, cost);
            }
            if (!mbar_wait(item_empty(sl), ((k / kItems) & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
            if (lane == 0) items[sl] = it;
            __syncwarp();
            if (lane == 0) mbar_arrive(item_full(sl));
            if (!more) break;
            auto copy_queries = [&](int q) {
                const uint32_t s = nq % kStages;
                float nl[4];
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = lane + 32 * i, in = r / a.G, t = q * a.tile_tokens + in;
                    nl[i] = -INFINITY;
                    if (in >= a.tile_tokens || t >= it.count) continue;
                    const float z = a.lse[(size_t)(it.start + t) * a.Hq + (size_t)it.h * a.G + (r - in * a.G)];
                    if (z != -INFINITY) nl[i] = (float)fma(-(double)z, kLog2eWide, a.log2_decay * (double)(it.count - 1 - t));
                    odd |= !(fabsf(nl[i]) < INFINITY);
                }
                if (!mbar_wait(q_empty(s), ((nq / kStages) & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; return; }
#pragma unroll
                for (int i = 0; i < 4; ++i) lse_s[s * kTileRows + lane + 32 * i] = nl[i];
                odd = __any_sync(0xFFFFFFFFu, odd);
                if (lane == 0) odd_s[s] = odd;
                __syncwarp();
                if (lane == 0) {
                    mbar_expect_tx(q_full(s), (uint32_t)(a.tile_tokens * a.G * D * 2));
#pragma unroll
                    for (int half = 0; half < D / 64; ++half)
                        tma_load_3d(base + L::kQ + s * kTile + half * kBoxBytes, &map_q, half * 64, it.h * a.G, it.start + q * a.tile_tokens, q_full(s));
                }
                ++nq;
            };
            if (it.qt0 < it.qt1) copy_queries(it.qt0);    // ahead of the rows, which wait for more
            if (!alive) break;
            if (it.qt0 < it.qt1) {
                // Tile by tile, behind the products of the unit before. Page numbers of all tiles are read at once where they fit a warp.
                const int teams = min(kTeams, (it.len - it.row0 + kTileRows - 1) / kTileRows), per = kTileRows / a.box_rows;
                const bool ahead = teams * per <= 32;
                const int first = ahead && lane < teams * per ? box_page(a, it.n, it.row0 + lane * a.box_rows, it.len) : -1;
#pragma unroll 1
                for (int x = 0; x < teams; ++x) {
                    int page = __shfl_sync(0xFFFFFFFFu, first, (x * per + lane) & 31);
                    if (!mbar_wait(k_empty(x), (nk >> x & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                    if (lane == 0) mbar_expect_tx(k_full(x), kTile);
                    nk ^= 1u << x;
                    asked |= 1u << x;
                    __syncwarp();
#pragma unroll 1
                    for (int box = lane; box < per; box += 32) {
                        const int at = box * a.box_rows, row = it.row0 + x * kTileRows + at;
                        if (!ahead) page = box_page(a, it.n, row, it.len);
                        bad_page(a, row, it.len, page);
                        copy_box<D>(a, &map_k, page, it.h, row, at, base + L::kK + x * kTile, k_full(x));
                    }
                }
                if (!alive) break;
                __syncwarp();
            }
            for (int q = it.qt0 + 1; q < it.qt1 && alive; ++q) copy_queries(q);
            if (!alive) break;
            more = w.next(a, cost);
        }
        if (*abort_flag) {
            // let copies that are still in flight land before the CTA gives its memory back
            for (uint32_t x = 0; x < (uint32_t)kTeams; ++x)
                if (asked >> x & 1u) mbar_drain(k_full(x), (nk >> x & 1u) ^ 1u);
            for (uint32_t t = nq > (uint32_t)kStages ? nq - kStages : 0; t < nq; ++t)
                mbar_drain(q_full(t % kStages), (t / kStages) & 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ products
        if (lane == 0) {
            uint32_t nq = 0, nk[kTeams] = {0, 0, 0, 0}, ns[kTeams] = {0, 0, 0, 0};
            auto wait = [&](uint32_t b, uint32_t phase) {
                if (!mbar_wait(b, phase & 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) alive = false;
                return alive;
            };
            for (uint32_t k = 0; alive; ++k) {
                const uint32_t sl = k % kItems;
                if (!wait(item_full(sl), k / kItems)) break;
                const Item it = items[sl];
                mbar_arrive(item_empty(sl));
                if (it.n < 0) break;
                if (it.qt0 >= it.qt1) continue;
                bool here[kTeams] = {false, false, false, false};
                for (int q = it.qt0; q < it.qt1 && alive; ++q, ++nq) {
                    const uint32_t s = nq % kStages;
                    if (!wait(q_full(s), nq / kStages)) break;
#pragma unroll
                    for (uint32_t x = 0; x < (uint32_t)kTeams; ++x) {
                        if (!alive || !meets(it, x, q)) continue;
                        if (!here[x] && !wait(k_full(x), nk[x])) continue;
                        here[x] = true;
                        if (!wait(s_empty(x), (ns[x] & 1u) ^ 1u)) continue;
                        tc_fence_after();
                        const uint32_t a0 = base + L::kK + x * kTile, b0 = base + L::kQ + s * kTile;
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = (uint32_t)(kk / 4) * kBoxBytes + (uint32_t)(kk % 4) * 32u;
                            umma_bf16(tmem + x * kTileRows, umma_desc(a0 + off), umma_desc(b0 + off), kIdesc, kk > 0 ? 1u : 0u);
                        }
                        umma_commit(s_full(x));
                        ++ns[x];
                    }
                    umma_commit(q_empty(s));
                }
                if (!alive) break;
#pragma unroll
                for (uint32_t x = 0; x < (uint32_t)kTeams; ++x)
                    if (alive && it.row0 + (int)x * kTileRows < it.len) {
                        if (!here[x] && !wait(k_full(x), nk[x])) continue;   // its copy has landed, wanted or not
                        umma_commit(k_empty(x));
                        ++nk[x];
                    }
            }
        }
    } else {
        // ------------------------------------------------------------ sums: a thread owns a cached row
        const uint32_t x = (uint32_t)(warp - 2) >> 2;
        const int q4 = warp & 3, r = q4 * 32 + lane;
        const uint32_t s_addr = tmem + x * kTileRows + ((uint32_t)(q4 * 32) << 16);
        const float2 c2 = make_float2(a.scale_log2e, a.scale_log2e);
        uint32_t nq = 0, ns = 0, nr = 0;
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(rdv(x));
            const bool ok = mbar_wait(rdv(x), nr & 1u, abort_flag, status);
            ++nr;
            return ok;
        };
        for (uint32_t k = 0; alive; ++k) {
            const uint32_t sl = k % kItems;
            if (!mbar_wait(item_full(sl), (k / kItems) & 1u, abort_flag, status)) { alive = false; break; }
            const Item it = items[sl];
            __syncwarp();
            if (lane == 0) mbar_arrive(item_empty(sl));
            if (it.n < 0) break;
            const int row = it.row0 + (int)x * kTileRows + r;
            float *place = nullptr;
            float old = 0.f;
            if (row < it.len) {
                const Slot slot = find_slot(a.c, it.n, row);
                if (slot.page >= 0) {
                    place = a.c.weight + meta_index(a.c, it.h, slot);
                    if (it.parts == 0) old = *place;
                }
            }
            float total = 0.f;
            for (int q = it.qt0; q < it.qt1; ++q, ++nq) {
                const uint32_t s = nq % kStages;
                if (!mbar_wait(q_full(s), (nq / kStages) & 1u, abort_flag, status)) { alive = false; break; }
                if (meets(it, x, q)) {
                    if (!mbar_wait(s_full(x), ns & 1u, abort_flag, status)) { alive = false; break; }
                    ++ns;
                    tc_fence_after();
                    const int token0 = q * a.tile_tokens;
                    const int tokens = min(a.tile_tokens, it.count - token0), columns = tokens * a.G;
                    // columns of tokens that see the row: from here on (rows behind the last one: none). Cut before the product: the
                    // distance to a row of long ago, times the group, passes 32 bits.
                    const int lo = min(max(row - (it.len - it.count) - token0, 0), a.tile_tokens) * a.G;
                    const int lo_warp = __shfl_sync(0xFFFFFFFFu, lo, 0);
                    float2 accA = make_float2(0.f, 0.f), accB = accA;
                    auto chunk = [&](const uint32_t (&raw)[32], int ch, auto mask_tag) {
                        constexpr bool MASKED = decltype(mask_tag)::value;
                        const float4 *ls = reinterpret_cast<const float4 *>(lse_s + s * kTileRows + ch * 32);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 nl = ls[i];
                            float2 e0 = __ffma2_rn(make_float2(__uint_as_float(raw[4 * i]), __uint_as_float(raw[4 * i + 1])), c2, make_float2(nl.x, nl.y));
                            float2 e1 = __ffma2_rn(make_float2(__uint_as_float(raw[4 * i + 2]), __uint_as_float(raw[4 * i + 3])), c2, make_float2(nl.z, nl.w));
                            if (MASKED) {
                                const int c = ch * 32 + 4 * i;
                                // a token without a normaliser takes no part, whatever its query makes of the score
                                e0.x = c >= lo && c < columns && nl.x != -INFINITY ? fast_exp2(e0.x) : 0.f;
                                e0.y = c + 1 >= lo && c + 1 < columns && nl.y != -INFINITY ? fast_exp2(e0.y) : 0.f;
                                e1.x = c + 2 >= lo && c + 2 < columns && nl.z != -INFINITY ? fast_exp2(e1.x) : 0.f;
                                e1.y = c + 3 >= lo && c + 3 < columns && nl.w != -INFINITY ? fast_exp2(e1.y) : 0.f;
                            } else {
                                e0 = exp2_pair(e0, 2 * i);
                                e1 = exp2_pair(e1, 2 * i + 1);
                            }
                            accA = __fadd2_rn(accA, e0);
                            accB = __fadd2_rn(accB, e1);
                        }
                    };
                    auto release = [&]() {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_empty(x));
                    };
                    // The polynomial that takes part in the exponentials knows neither NaN nor an exact zero: normalisers like that go the
                    // careful way too.
                    const bool masked = tokens < a.tile_tokens || odd_s[s] != 0 || __any_sync(0xFFFFFFFFu, lo > 0);
                    if (masked) {
                        // chunks that no row of the warp takes part in are left out
                        const int ch0 = lo_warp / 32, ch1 = (columns + 31) / 32;
                        for (int ch = ch0; ch < ch1; ++ch) {
                            uint32_t raw[32];
                            tmem_ld32_async(s_addr + 32 * ch, raw);
                            tmem_ld_wait(raw);
                            if (ch + 1 == ch1) release();
                            chunk(raw, ch, std::true_type{});
                        }
                        if (ch0 >= ch1) release();
                    } else {
                        uint32_t ra[32], rb[32];
                        tmem_ld32_async(s_addr, ra);
#pragma unroll 1
                        for (int ch = 0; ch < 4; ch += 2) {               // a chunk is under way while the one before is worked on
                            tmem_ld_wait(ra);
                            tmem_ld32_async(s_addr + 32 * ch + 32, rb);
                            chunk(ra, ch, std::false_type{});
                            tmem_ld_wait(rb);
                            if (ch == 0) tmem_ld32_async(s_addr + 64, ra);
                            else release();
                            chunk(rb, ch + 1, std::false_type{});
                        }
                    }
                    total += (accA.x + accA.y) + (accB.x + accB.y);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty(s));
            }
            if (!alive) break;
            const float kept = exp2_of(a.log2_decay * (double)it.count);
            if (it.parts == 0) {
                if (place) *place = fmaf(kept, old, total);
            } else {
                // the CTA that arrives last adds the parts, in the order of the tokens
                const int at = (int)x * kTileRows + r;
                __stcg(a.part + (size_t)it.slot * kBlockRows + at, total);
                if (!meet()) { alive = false; break; }
                int *counter = a.c.state + kStateChunk + it.first * kChunkCounters + (int)x;
                if (q4 == 0 && lane == 0) {
                    const bool last = arrive(counter) == it.parts - 1;
                    if (last) *counter = 0;
                    last_s[x] = last;
                }
                if (!meet()) { alive = false; break; }
                if (last_s[x] && place) {
                    float sum = 0.f;
                    for (int p = 0; p < it.parts; ++p)
                        sum += __ldcg(a.part + (size_t)(2 * (it.first + p) + (p == 0)) * kBlockRows + at);
                    *place = fmaf(kept, *place, sum);
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kTmemCols) : "memory");
    }
}

template <int D, int DTYPE>
cudaError_t launch_t(const WeightArgs &a, const CUtensorMap &mq, const CUtensorMap &mk, cudaStream_t stream)
{
    auto kernel = chunk_weights_kernel<D, DTYPE>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::kTotal);
    if (e != cudaSuccess) return e;
    return launch_chained(kernel, dim3(chunk_grid()), kThreads, Smem<D>::kTotal, stream, mq, mk, a);
}

}  // namespace

size_t chunk_weights_workspace_bytes() { return (size_t)2 * kChunkMaxCtas * kBlockRows * sizeof(float); }

cudaError_t launch_chunk_weights(const ChunkArgs &chunk, int D, int dtype, const void *q, int64_t q_token, int64_t q_head, const float *lse,
                                 double decay, void *ws, cudaStream_t stream)
{
    WeightArgs a;
    static_cast<ChunkArgs &>(a) = chunk;
    a.lse = lse;
    a.log2_decay = log2(decay);
    a.part = static_cast<float *>(ws);
    CUtensorMap mq, mk;
    if (!make_query_map(&mq, a, D, dtype, q, q_token, q_head) || !make_pool_map(&mk, a, D, dtype, a.c.K)) return cudaErrorInvalidValue;
    if (D == 128) return dtype == EC_BF16 ? launch_t<128, EC_BF16>(a, mq, mk, stream) : launch_t<128, EC_FP16>(a, mq, mk, stream);
    return dtype == EC_BF16 ? launch_t<64, EC_BF16>(a, mq, mk, stream) : launch_t<64, EC_FP16>(a, mq, mk, stream);
}

}  // namespace ec
