// Attention of a chunk of new tokens over a paged cache (grouped query heads, ragged batch), with each row's normaliser.
//   token t of problem n sees rows j <= lens[n] - counts[n] + t:
//   x[j] = scale * <q, k_j>,   out = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)
//
// One pass over the rows, 128 at a time, for a tile of 128 query rows (tokens with the heads that share the key head):
//   S = Q K^T      tcgen05.mma from tiles that TMA brought page by page, S in TMEM
//   P = 2^(c S - m2 + top)   a thread owns a query row; P goes over S, as the type of the rows: one rounding of half a step, the
//                  tensor cores take nothing wider. Sums and maxima are fp32 and taken before that rounding. Of the exponentials one
//                  pair in four is a polynomial, 6e-6 off: a hundredth of that rounding, but the normaliser has it too
//   O += P V       P from TMEM, V as it lies in shared memory
// The running maximum is raised when a half of a tile exceeds it by 2^8 (bf16) or 2^4 (fp16), so O is rescaled rarely.
//
// What bounds it. Long prompts: each of two teams of four warps waits for its own S (issued behind its own P V: 512 columns of
// TMEM hold S of both and O of both, with P over S) while the other computes. Per tile and team about 3200 clocks of softmax
// (1800 of them exponentials, where the special functions' rate for both teams is 1540) and 2000 of waiting for S. 8192 tokens of
// 32 heads on 8, D = 128: 680 to 694 us by the box, 0.80 PFLOP/s at the 1.5 GHz that the power limit leaves (610 us in a short run); the
// products alone take 336 us at the rate of a large library product. Few tokens on long caches (32 problems of up to 8 on up to 8192 rows): 37 us,
// of which 15.5 are the rows' bytes; starting (8 thousand clocks to the first S) and joining the parts are the rest. Many short problems: a unit of one to
// three tiles keeps the softmax warps busy for 6 to 7 us whatever it holds; for one token a problem the single-token call is the
// one to use.
//
// Why so.
//  - Two query tiles of a head to a CTA, a team each: rows are fetched once for both. A unit of one query tile has both teams take its
//    tiles in turn and is put together in the CTA: few tokens meet long caches with twice the warps.
//  - The batch's work is cut evenly over one resident CTA per SM by a closed form of its cost, and what a cut leaves of a unit goes
//    through the workspace in fp32, joined in the order of the rows by whoever arrives last. A warp's rows choose together between two
//    ways of computing them, which differ in the last bits; rows that are nobody's have no say. So the bits are the same in every run.
//  - A lazy maximum per half of a tile lets P V of the first half run under the exponentials of the second.
//  - Values of masked rows: a warp looks over the tiles that not every token sees and turns what is not finite into zeros (a
//    product with P = 0 would not hide it); who does see such a row reads it again.
// Registers: at D = 128 nothing is spilt, at D = 64 40 bytes a thread.
// Tried and slower, 8192 tokens (670 us then) and a mixed batch (79 us): sixteen softmax warps with two threads a row (they spill
// and meet once a tile; 732 against 609 in short runs, 98 against 82); a whole row of 128 columns a thread 747 and 94 (spills); the maximum looked at behind the exponentials 686 and 90; teams that
// take turns on a scheduler 705 and 94; S in halves of 64 columns (a product of 64 columns takes as long as one of 128); an item per
// team for short units (no change); the second team helping to put a single query tile together and to join its parts (32 problems of few
// tokens 37.0 and 36.5, the long prompt 608 and 651 in short runs); a masked half that nobody sees as plain zeros (many units of one tile
// 5% faster, the long prompt 666); the next launch let in early (mixed 100 against 89 before other steps). What stands around the loop
// over the tiles moves its time by several per cent, whatever it does.
#include "ec_chunk.cuh"

namespace ec {

namespace {

constexpr int kThreads = 384;                    // warps: copies, products of a team, value check, products of the other, 4 + 4 softmax
constexpr int kHalf = 64;                        // columns of S that a thread holds at a time; P V of the first runs under the second
constexpr int kItems = 4;                        // descriptions of work ahead
constexpr int kInfos = 8;                        // absent rows of the tiles in flight (the rings hold 4 at most)
constexpr int kTmemCols = 512;                   // S of both teams (2 x 128 columns), O of both teams (2 x up to 128)
// Cost of a unit beside its rows, and the smallest share of a CTA. 128, 384 and 768 rows a unit: 32 problems of few tokens 57.0, 36.6 and
// 38.3 us, 16 pieces 113.6, 81.8 and 93.8, the odd batch 35.2, 37.1 and 39.6, 8192 tokens 714, 693 and 710. 256, 640 and 1280 rows a share:
// the odd batch 37.2, 37.1 and 44.9, the others within 1%.
constexpr int kUnitRows = 384;
constexpr int kLeastRows = 640;
constexpr float kLowest = -3.402823466e38f;      // a running maximum that has seen nothing: below every score, and -inf less it is still -inf
constexpr float kLarge = 16777216.f;

template <int DTYPE> struct Elem;
template <> struct Elem<EC_BF16> {
    static constexpr uint32_t kFormat = 1;       // of an operand in the instruction descriptor
    static constexpr float kRaise = 8.f, kTop = 0.f;
    static constexpr uint32_t kExponent = 0x7F807F80u;
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b); }
};
// fp16 has few exponents: P is counted from 2^11 at the running maximum, which leaves the 2^4 that it may rise under the type's
// largest number and takes in rows down to 2^-35 of the maximum's, with all bits down to 2^-25.
template <> struct Elem<EC_FP16> {
    static constexpr uint32_t kFormat = 0;
    static constexpr float kRaise = 4.f, kTop = 11.f;
    static constexpr uint32_t kExponent = 0x7C007C00u;
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&h);
    }
};

struct PairUnits {                               // a unit: two adjacent query tiles of a head
    static __device__ __forceinline__ int units(const ChunkArgs &a, const Problem &p) { return (p.count + 2 * a.tile_tokens - 1) / (2 * a.tile_tokens); }
    static __device__ __forceinline__ long long before(const ChunkArgs &a, const Problem &p, int units, int i)
    {
        const long long base = max(p.len - p.count, 0), step = 2 * a.tile_tokens;
        const int full = units - 1;
        const long long k = i <= full ? i : full;
        long long cost = k * (base + kUnitRows) + step * (k * (k + 1) / 2);
        if (i > full) cost += base + p.count + kUnitRows;
        return cost;
    }
};

struct Item {
    int n, h;                                    // n < 0: no work left
    int token, ntok;                             // first token of the pair (packed), tokens
    int limit;                                   // last row that the first token sees (may be negative)
    int rows;                                    // rows that the pair sees at all
    int kt0, kt1;                                // its tiles in this CTA
    int parts, first, slot;                      // parts > 0: the unit is shared by CTAs first .. first + parts - 1
    int pad;
};

struct Parts {                                   // workspace
    float4 *o;                                   // [2 CTAs][2 teams][D / 4][128]
    float2 *ml;                                  // [2 CTAs][2 teams][128] running maximum (scaled), sum
};

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                   "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
// 64 (32) columns of this thread's TMEM lane, complete when the statement ends: what the load fills is not to be touched before the
// wait, and between two statements the compiler may copy registers.
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[64])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
                 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
                 "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
                 "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
                   "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
                   "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
                   "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
                   "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
                 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// MN-major operand with the 128-byte swizzle: 64 elements of the MN dimension per 128-byte row, 8 steps of the contraction
// index per 1024 bytes; `lbo` bytes to the next 64 elements of the MN dimension, `sbo` to the next 8 steps.
__device__ __forceinline__ uint64_t umma_desc_mn(uint32_t smem_addr, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

// D = A * B, A (two elements of the contraction index per 32-bit column) from TMEM, B from shared memory; M = 128, K = 16.
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

// NaN wins: a score that is not a number makes its row not a number, wherever it stands.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Of 32 columns from `col` on, as bits, those in which one of the rows begin .. end - 1 has a value that is not finite. A slow way
// that healthy values never take.
template <uint32_t EXPONENT>
__device__ __forceinline__ uint32_t spoilt(const ChunkArgs &a, int n, int h, int begin, int end, int col)
{
    uint32_t bits = 0u;
#pragma unroll 1
    for (int row = begin; row < end; ++row) {
        const Slot s = look_up_slot(a.c, n, row);
        if (!valid_page(a.c, s)) continue;
        const uint32_t *v = reinterpret_cast<const uint32_t *>(a.c.V + row_offset(a.c, s) + (size_t)h * a.c.head_step) + col / 2;
#pragma unroll 1
        for (int j = 0; j < 16; ++j) {
            const uint32_t e = v[j] & EXPONENT;
            if ((e & 0xFFFFu) == (EXPONENT & 0xFFFFu)) bits |= 1u << (2 * j);
            if (e >> 16 == EXPONENT >> 16) bits |= 2u << (2 * j);
        }
    }
    return bits;
}

template <int D>
struct Smem {
    static constexpr int kTile = kTileRows * D * 2;
    static constexpr int kKs = D == 128 ? 2 : 4, kVs = D == 128 ? 3 : 4;   // rings of tiles; V stays until its product is done
    static constexpr int kQ = 0;                                          // both query tiles
    static constexpr int kK = 2 * kTile;
    static constexpr int kV = kK + kKs * kTile;
    static constexpr int kOther = kV + kVs * kTile;                       // [128] maximum and sum of the second team
    static constexpr int kBadAny = kOther + kTileRows * 8;                    // [items] whether a value that is not finite became zero
    static constexpr int kItem = kBadAny + kItems * 4;
    static constexpr int kInfo = kItem + kItems * (int)sizeof(Item);
    static constexpr int kBars = kInfo + kInfos * 16;
    // q_full, q_empty, k_full[], k_empty[], v_full[], v_empty[], per team: s_full, p_full[2], pv, o_free, rdv, pv_half; other_done; item_full, item_empty
    static constexpr int kNumBars = 2 + 2 * kKs + 2 * kVs + 2 * 7 + 1 + 2 * kItems;
    static constexpr int kTmemSlot = kBars + kNumBars * 8;
    static constexpr int kAbort = kTmemSlot + 4;
    static constexpr int kLast = kAbort + 4;                              // [2] whether this CTA joins the unit's parts
    static constexpr int kCount = kLast + 8;                              // [3], see where they are used
    static constexpr int kTotal = kCount + 12;
    static_assert(kTotal <= 232448, "shared memory of a block");
};

// Natural log-sum-exp from the maximum (log2) and the sum.
template <typename E>
__device__ __forceinline__ float log_sum(float m2, float l)
{
    return m2 == kLowest && l == l ? -INFINITY : (m2 + (log2f(l) - E::kTop)) * kLn2;
}

// Joins the parts of a unit's query tile, in the order of the rows: a warp of the team takes 32 rows at a time and a quarter of their
// columns, and has two parts in flight.
template <int D, int DTYPE>
__device__ __forceinline__ void join_parts(const Parts parts, int first, int many, int x, int ntok, int G, uint16_t *out, int64_t out_token,
                                        int64_t out_head, float *lse, int Hq)
{
    using E = Elem<DTYPE>;
    const int lane = threadIdx.x & 31, q4 = (threadIdx.x >> 5) & 3;
#pragma unroll 1
    for (int row = lane; row < ntok * G; row += 32) {
        float M = kLowest, sum = 0.f, f[D / 4] = {};
#pragma unroll 1
        for (int p = 0; p < many; p += 2) {
            float2 ml[2] = {make_float2(kLowest, 0.f), make_float2(kLowest, 0.f)};
            float4 o[2][D / 16];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (p + u >= many) continue;
                const size_t from = (size_t)(2 * (first + p + u) + (p + u == 0)) * 2 + x;
                ml[u] = __ldcg(parts.ml + from * kTileRows + row);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[u][i] = __ldcg(parts.o + (from * (D / 4) + q4 * (D / 16) + i) * kTileRows + row);
            }
            const float top = max3(M, ml[0].x, ml[1].x), old = fast_exp2(M - top);
            const float g[2] = {fast_exp2(ml[0].x - top), fast_exp2(ml[1].x - top)};
            M = top;
            sum = fmaf(ml[1].y, g[1], fmaf(ml[0].y, g[0], sum * old));
#pragma unroll
            for (int i = 0; i < D / 4; ++i) f[i] *= old;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (ml[u].x == kLowest) continue;         // nothing was seen, or no such part
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    f[4 * i] = fmaf(o[u][i].x, g[u], f[4 * i]);
                    f[4 * i + 1] = fmaf(o[u][i].y, g[u], f[4 * i + 1]);
                    f[4 * i + 2] = fmaf(o[u][i].z, g[u], f[4 * i + 2]);
                    f[4 * i + 3] = fmaf(o[u][i].w, g[u], f[4 * i + 3]);
                }
            }
        }
        const float scale = M == kLowest && sum == sum ? 0.f : 1.f / sum;
        const int in = row / G, head = row - in * G;
        uint4 *to = reinterpret_cast<uint4 *>(out + in * out_token + head * out_head + q4 * (D / 4));
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
            const float *g = f + 8 * q;
            to[q] = make_uint4(E::pack(g[0] * scale, g[1] * scale), E::pack(g[2] * scale, g[3] * scale), E::pack(g[4] * scale, g[5] * scale),
                               E::pack(g[6] * scale, g[7] * scale));
        }
        if (q4 == 0 && lse) lse[(int64_t)in * Hq + head] = log_sum<E>(M, sum);
    }
}

template <int D, int DTYPE>
__global__ void __launch_bounds__(kThreads, 1)
chunk_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ChunkArgs a, uint16_t *__restrict__ out, int64_t out_token,
                       int64_t out_head, float *__restrict__ lse, const Parts parts)
{
    using L = Smem<D>;
    using E = Elem<DTYPE>;
    constexpr int kTile = L::kTile, kKs = L::kKs, kVs = L::kVs;
    constexpr int kBoxBytes = kTileRows * 128;
    constexpr uint32_t kIdescS = (1u << 4) | (E::kFormat << 7) | (E::kFormat << 10) | ((kTileRows >> 3) << 17) | ((kTileRows >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (E::kFormat << 7) | (E::kFormat << 10) | (1u << 16) | ((D >> 3) << 17) | ((kTileRows >> 4) << 24);

    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    auto bar = [&](int i) { return base + (uint32_t)L::kBars + 8u * (uint32_t)i; };
    const uint32_t q_full = bar(0), q_empty = bar(1);
    auto k_full = [&](uint32_t s) { return bar(2 + s); };
    auto k_empty = [&](uint32_t s) { return bar(2 + kKs + s); };
    auto v_full = [&](uint32_t s) { return bar(2 + 2 * kKs + s); };
    auto v_empty = [&](uint32_t s) { return bar(2 + 2 * kKs + kVs + s); };
    constexpr int kT0 = 2 + 2 * kKs + 2 * kVs;
    auto s_full = [&](uint32_t x) { return bar(kT0 + 7 * x); };
    auto p_full = [&](uint32_t x, uint32_t h) { return bar(kT0 + 7 * x + 1 + h); };
    auto pv = [&](uint32_t x) { return bar(kT0 + 7 * x + 3); };
    auto o_free = [&](uint32_t x) { return bar(kT0 + 7 * x + 4); };
    auto rdv = [&](uint32_t x) { return bar(kT0 + 7 * x + 5); };
    auto pv_half = [&](uint32_t x) { return bar(kT0 + 7 * x + 6); };
    const uint32_t other_done = bar(kT0 + 14);
    auto item_full = [&](uint32_t k) { return bar(kT0 + 15 + k); };
    auto item_empty = [&](uint32_t k) { return bar(kT0 + 15 + kItems + k); };
    Item *items = reinterpret_cast<Item *>(smem + L::kItem);
    float2 *other_s = reinterpret_cast<float2 *>(smem + L::kOther);
    uint2 *infos = reinterpret_cast<uint2 *>(smem + L::kInfo);           // [kInfos][2 halves]
    volatile int *bad_any = reinterpret_cast<volatile int *>(smem + L::kBadAny);
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kTmemSlot);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kAbort);
    volatile int *last_s = reinterpret_cast<volatile int *>(smem + L::kLast);
    // A team does not wait for every copy, and a barrier's parity tells its phase only to who saw the phase before: so a team
    // first waits until the copy that it needs has been asked for (or its values been checked).
    int *counts = reinterpret_cast<int *>(smem + L::kCount);
    int *const k_asked = counts, *const q_asked = counts + 1, *const v_checked = counts + 2;
    int *status = a.c.state;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        counts[0] = counts[1] = counts[2] = 0;
        mbar_init(q_full, 1);
        mbar_init(q_empty, 2);                                           // k, v and queries are released by both teams
        for (uint32_t s = 0; s < (uint32_t)kKs; ++s) { mbar_init(k_full(s), 1); mbar_init(k_empty(s), 2); }
        for (uint32_t s = 0; s < (uint32_t)kVs; ++s) { mbar_init(v_full(s), 1); mbar_init(v_empty(s), 2); }
        for (uint32_t x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            for (uint32_t h = 0; h < 2; ++h) mbar_init(p_full(x, h), 4);
            mbar_init(pv(x), 1);
            mbar_init(pv_half(x), 1);
            mbar_init(o_free(x), 4);
            mbar_init(rdv(x), 4);
        }
        mbar_init(other_done, 4);
        for (uint32_t k = 0; k < (uint32_t)kItems; ++k) {
            mbar_init(item_full(k), 1);
            mbar_init(item_empty(k), 2 + 1 + 8);                         // the products' threads, the value check, the softmax warps
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_to_async();
    }
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
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
    auto tmem_s = [&](uint32_t x) { return tmem + x * (uint32_t)kTileRows; };                 // S, and P over its first half
    auto tmem_o = [&](uint32_t x) { return tmem + 2u * kTileRows + x * (uint32_t)kTileRows; };
    grid_wait();

    // A unit of two query tiles: a team per tile, every tile of rows serves both. A unit of one: both teams work on it and
    // take its tiles of rows in turn; the first team puts the two results together.
    auto is_pair = [&](const Item &it) { return it.ntok > a.tile_tokens; };
    // What team x does of an item: tiles first, first + step, .. below end of the item's, with the rows that its tokens see.
    struct Part { int first, step, end, rows; };
    auto part_of = [&](const Item &it, uint32_t x) {
        const int tiles = it.kt1 - it.kt0;
        if (!is_pair(it)) return Part{(int)x, 2, tiles, it.rows};
        if (x == 1) return Part{0, 1, tiles, it.rows};
        const int sees = max(min(it.rows, it.limit + a.tile_tokens), 0);
        return Part{0, 1, max(min(tiles, (sees + kTileRows - 1) / kTileRows - it.kt0), 0), sees};
    };
    bool alive = true;

    // A thread of the softmax holds 64 scores and as many addresses as the epilogue needs: 4 warps x 88 + 8 x 208 registers are the
    // 12 x 168 of the launch. The four warps of a group change their share by the same instruction, in front of their roles.
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 0) {
            // ------------------------------------------------------------ plan and copies
            Walk<PairUnits> w;
            bool more = w.begin(a, kLeastRows);
            uint32_t tg = 0, nk = 0, nv = 0, nq = 0;           // tiles; copies of K, V and queries started
            for (uint32_t k = 0; alive; ++k) {
                const uint32_t sl = k % kItems;
                Item it = {};
                it.n = -1;
                long long cost = 0;
                while (more) {                                // the next unit that this CTA has something of
                    const int step = 2 * a.tile_tokens;
                    it.ntok = min(step, w.p.count - w.i * step);
                    it.limit = w.p.len - w.p.count + w.i * step;
                    it.rows = max(0, min(w.p.len, it.limit + it.ntok));
                    cost = PairUnits::before(a, w.p, w.units, w.i + 1) - PairUnits::before(a, w.p, w.units, w.i);
                    const Cut cut = cut_unit(w.s, w.at, cost, kUnitRows, kTileRows, (it.rows + kTileRows - 1) / kTileRows);
                    if (cut.mine) {
                        it.n = w.n;
                        it.h = w.h;
                        it.token = w.p.start + w.i * step;
                        it.kt0 = cut.t0;
                        it.kt1 = cut.t1;
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
                auto copy_queries = [&] {
                    if (lane == 0) {
                        const int tiles = it.ntok > a.tile_tokens ? 2 : 1;
                        mbar_expect_tx(q_full, (uint32_t)(tiles * a.tile_tokens * a.G * D * 2));
                        publish(q_asked, (int)nq + 1);
                        for (int x = 0; x < tiles; ++x)
    #pragma unroll
                            for (int half = 0; half < D / 64; ++half)
                                tma_load_3d(base + L::kQ + x * kTile + half * kBoxBytes, &map_q, half * 64, it.h * a.G,
                                            it.token + x * a.tile_tokens, q_full);
                    }
                    ++nq;
                };
                // the queries first when their place is free, else behind the first tile's rows
                bool asked = it.kt0 >= it.kt1 || __all_sync(0xFFFFFFFFu, mbar_try(q_empty, (nq & 1u) ^ 1u));
                if (asked && it.kt0 < it.kt1) copy_queries();
                // page numbers of a lane's first box are read a tile ahead; pages of fewer than 4 rows have more boxes than lanes
                const int boxes = kTileRows / a.box_rows;
                int row = it.kt0 * kTileRows + lane * a.box_rows, next = it.kt0 < it.kt1 ? box_page(a, it.n, row, it.rows) : -1;
                for (int t = it.kt0; t < it.kt1 && alive; ++t, ++tg, row += kTileRows) {
                    int page = next;
                    const uint32_t ks = tg % kKs, vs = tg % kVs;
                    if (!mbar_wait(k_empty(ks), ((tg / kKs) & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                    uint32_t gone[4] = {0u, 0u, 0u, 0u};      // absent rows
                    auto lost = [&](int at) {
                        for (int r = at; r < at + a.box_rows; ++r) {
    #pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (r >> 5 == j) gone[j] |= 1u << (r & 31);
                        }
                    };
                    bool any = lane < boxes && bad_page(a, row, it.rows, page);
                    if (any) lost(lane * a.box_rows);
                    if (lane == 0) {
                        mbar_expect_tx(k_full(ks), kTile);
                    }
                    __syncwarp();
                    const uint32_t k_to = base + L::kK + ks * kTile, v_to = base + L::kV + vs * kTile;
                    if (lane < boxes) copy_box<D>(a, &map_k, page, it.h, row, lane * a.box_rows, k_to, k_full(ks));
    #pragma unroll 1
                    for (int box = lane + 32; box < boxes; box += 32) {
                        const int r = t * kTileRows + box * a.box_rows;
                        int p = box_page(a, it.n, r, it.rows);
                        if (bad_page(a, r, it.rows, p)) {
                            any = true;
                            lost(box * a.box_rows);
                        }
                        copy_box<D>(a, &map_k, p, it.h, r, box * a.box_rows, k_to, k_full(ks));
                    }
                    any = __any_sync(0xFFFFFFFFu, any);
                    if (any) {
    #pragma unroll
                        for (int j = 0; j < 4; ++j) gone[j] = __reduce_or_sync(0xFFFFFFFFu, gone[j]);
                    }
                    if (lane == 0) {
                        infos[2 * (tg % kInfos)] = make_uint2(gone[0], gone[1]);
                        infos[2 * (tg % kInfos) + 1] = make_uint2(gone[2], gone[3]);
                        publish(k_asked, (int)tg + 1);        // S is asked for behind this
                    }
                    ++nk;
                    if (!asked) {
                        if (!mbar_wait(q_empty, (nq & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                        copy_queries();
                        asked = true;
                    }
                    next = t + 1 < it.kt1 ? box_page(a, it.n, row + kTileRows, it.rows) : -1;
                    if (!mbar_wait(v_empty(vs), ((tg / kVs) & 1u) ^ 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                    if (lane == 0) mbar_expect_tx(v_full(vs), kTile);
                    __syncwarp();
                    if (lane < boxes) copy_box<D>(a, &map_v, page, it.h, row, lane * a.box_rows, v_to, v_full(vs));
    #pragma unroll 1
                    for (int box = lane + 32; box < boxes; box += 32) {
                        const int r = t * kTileRows + box * a.box_rows;
                        int p = box_page(a, it.n, r, it.rows);
                        bad_page(a, r, it.rows, p);
                        copy_box<D>(a, &map_v, p, it.h, r, box * a.box_rows, v_to, v_full(vs));
                    }
                    ++nv;
                }
                if (!alive) break;
                more = w.next(a, cost);
            }
            if (*abort_flag) {
                // let copies that are still in flight land before the CTA gives its memory back
                if (nq > 0) mbar_drain(q_full, (nq - 1u) & 1u);
                for (uint32_t t = nk > (uint32_t)kKs ? nk - kKs : 0; t < nk; ++t)
                    mbar_drain(k_full(t % kKs), (t / kKs) & 1u);
                for (uint32_t t = nv > (uint32_t)kVs ? nv - kVs : 0; t < nv; ++t)
                    mbar_drain(v_full(t % kVs), (t / kVs) & 1u);
            }
        } else if (warp == 1 || warp == 3) {
            // ------------------------------------------------------------ products of a team
            if (lane == 0) {
                const uint32_t x = (uint32_t)warp >> 1;
                uint32_t tg0 = 0, nq = 0, np = 0, ni = 0;     // the CTA's tiles and query loads, the team's tiles and items so far
                auto wait = [&](uint32_t b, uint32_t phase) {
                    if (!mbar_wait(b, phase & 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) alive = false;
                    return alive;
                };
                auto wait_count = [&](const int *count, uint32_t least) {
                    if (!reached(count, (int)least, abort_flag, status)) alive = false;
                    return alive;
                };
                // released by both teams: who works alone on it does so twice
                auto release = [&](uint32_t b, bool alone) {
                    umma_commit(b);
                    if (alone) umma_commit(b);
                };
                auto issue_s = [&](uint32_t qt, uint32_t ks) {
                    const uint64_t da = umma_desc(base + L::kQ + qt * kTile), db = umma_desc(base + L::kK + ks * kTile);
    #pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t off = ((uint32_t)(kk / 4) * kBoxBytes + (uint32_t)(kk % 4) * 32u) >> 4;
                        umma_bf16(tmem_s(x), da + off, db + off, kIdescS, kk > 0 ? 1u : 0u);
                    }
                    umma_commit(s_full(x));
                };
                for (uint32_t k = 0; alive; ++k) {
                    const uint32_t sl = k % kItems;
                    if (!wait(item_full(sl), k / kItems)) break;
                    const Item it = items[sl];
                    mbar_arrive(item_empty(sl));
                    if (it.n < 0) break;
                    const int tiles = it.kt1 - it.kt0;
                    if (tiles <= 0) continue;
                    const bool pair = is_pair(it);
                    const uint32_t qt = pair ? x : 0u;
                    const Part mine = part_of(it, x), others = part_of(it, x ^ 1u);
                    auto alone = [&](int t) { return !pair || t >= others.end; };
                    const bool all_mine = others.first >= others.end;          // the other team has nothing in this item
                    const uint32_t tg = tg0;
                    tg0 += (uint32_t)tiles;
                    ++nq;
                    if (mine.first >= mine.end) continue;
                    if (!wait_count(q_asked, nq) || !wait(q_full, nq - 1u)) break;
                    {
                        const uint32_t ks = (tg + mine.first) % kKs;
                        if (!wait_count(k_asked, tg + mine.first + 1) || !wait(k_full(ks), (tg + mine.first) / kKs)) break;
                        tc_fence_after();
                        issue_s(qt, ks);
                        release(k_empty(ks), alone(mine.first));
                        if (mine.first + mine.step >= mine.end) release(q_empty, all_mine);
                    }
                    if (!wait(o_free(x), ni + 1u)) break;
                    ++ni;
    #pragma unroll 1
                    for (int t = mine.first; t < mine.end && alive; t += mine.step) {
                        const int then = t + mine.step;
                        const uint32_t vs = (tg + t) % kVs, ks = (tg + then) % kKs;
                        const int steps = min(kTileRows / 16, (mine.rows - (it.kt0 + t) * kTileRows + 15) / 16);
                        if (!wait_count(v_checked, tg + t + 1)) break;
                        const uint64_t dv = umma_desc_mn(base + L::kV + vs * kTile, kBoxBytes, 1024u);
    #pragma unroll
                        for (uint32_t h = 0; h < 2; ++h) {
                            // O += P V of 64 rows, 16 an instruction
                            if (!wait(p_full(x, h), np)) break;
                            tc_fence_after();
    #pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int kk = 4 * (int)h + i;
                                if (kk < steps) umma_ts(tmem_o(x), tmem_s(x) + h * kHalf + 8u * i, dv + kk * (2048u >> 4), kIdescO, t == mine.first && kk == 0 ? 0u : 1u);
                            }
                            if (h == 0) umma_commit(pv_half(x));
                        }
                        if (!alive) break;
                        ++np;
                        if (then >= mine.end) umma_commit(pv(x));
                        if (then < mine.end) {                // S of the next tile, over this P
                            if (!wait_count(k_asked, tg + then + 1) || !wait(k_full(ks), (tg + then) / kKs)) break;
                            tc_fence_after();
                            issue_s(qt, ks);
                            release(k_empty(ks), alone(then));
                            if (then + mine.step >= mine.end) release(q_empty, all_mine);
                        }
                        release(v_empty(vs), alone(t));
                    }
                }
            }
        } else if (warp == 2) {
            // ------------------------------------------------------------ value check
            // A product with P = 0 does not hide a value that is not finite, so tiles whose rows some token must not see are
            // looked over: such values become zeros, and the item is marked, for the tokens that do see them. Rows behind the last one
            // (memory that holds anything) become zeros too; absent ones are.
            uint32_t tg = 0;
            for (uint32_t k = 0; alive; ++k) {
                const uint32_t sl = k % kItems;
                if (!mbar_wait(item_full(sl), (k / kItems) & 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                const Item it = items[sl];
                if (lane == 0) bad_any[sl] = 0;
                __syncwarp();
                if (it.n < 0) break;
                for (int t = it.kt0; t < it.kt1; ++t, ++tg) {
                    const uint32_t s = tg % kVs;
                    if (!mbar_wait(v_full(s), (tg / kVs) & 1u, abort_flag, status, kWaitLimitNs, kPollBackoffNs)) { alive = false; break; }
                    const int row0 = t * kTileRows, rows = min(kTileRows, it.rows - row0);
                    const int check = max(0, it.limit + 1 - row0);                             // rows before are seen by every token
                    const int end = (rows + 15) & ~15;
                    if (check < end) {
                        uint8_t *tile = smem + L::kV + s * kTile;
                        constexpr int kChunks = D / 8;                                         // 16-byte pieces of a row
                        for (int i = check * kChunks + lane; i < end * kChunks; i += 32) {
                            const int r = i / kChunks, c = i % kChunks;
                            uint4 *at = reinterpret_cast<uint4 *>(tile + (c >> 3) * kBoxBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
                            if (r >= rows) {
                                *at = make_uint4(0u, 0u, 0u, 0u);
                                continue;
                            }
                            uint4 v = *at;
                            uint32_t w[4] = {v.x, v.y, v.z, v.w};
                            bool found = false;
    #pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t e = w[j] & E::kExponent;
                                const bool lo = (e & 0xFFFFu) == (E::kExponent & 0xFFFFu), hi = (e >> 16) == (E::kExponent >> 16);
                                w[j] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
                                found |= lo || hi;
                            }
                            if (found) {
                                *at = make_uint4(w[0], w[1], w[2], w[3]);
                                bad_any[sl] = 1;
                            }
                        }
                        fence_to_async();
                    }
                    __syncwarp();
                    if (lane == 0) publish(v_checked, (int)tg + 1);
                }
                if (lane == 0) mbar_arrive(item_empty(sl));
            }
        }
    } else {
        // ------------------------------------------------------------ softmax: a thread owns a query row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const uint32_t x = (uint32_t)(warp - 4) >> 2;
        const int q4 = warp & 3, r = q4 * 32 + lane;
        const uint32_t lane_sel = (uint32_t)(q4 * 32) << 16;
        const uint32_t s_addr = tmem_s(x) + lane_sel;
        const float c = a.scale_log2e;
        const float2 c2 = make_float2(c, c);
        const int my_token = r / a.G, my_head = r - my_token * a.G;
        uint32_t ns = 0, ni = 0, tg0 = 0, nr = 0, no = 0;  // the team's tiles and items; the CTA's tiles; meetings; results taken over
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
            if (it.n < 0) break;
            const bool pair = is_pair(it);
            const int tiles = it.kt1 - it.kt0;
            const int skip = pair ? (int)x * a.tile_tokens : 0;                             // tokens in front of the team's
            const int ntok = min(a.tile_tokens, it.ntok - skip);
            const int limit = it.limit + skip + my_token;                                   // last row that this row sees
            const bool valid = my_token < ntok, live = q4 * 32 < ntok * a.G;                // live: some row of the warp counts
            const Part part = part_of(it, x);
            float m = -INFINITY, m2 = kLowest, l = 0.f;   // running maximum (not scaled; scaled), sum
            const int plain_to = min(__shfl_sync(0xFFFFFFFFu, limit, 0), it.rows - 1);       // of a warp's rows the first one sees the least
#pragma unroll 1
            for (int i = 2 * part.first; i < 2 * part.end; i += (i & 1) ? 2 * part.step - 1 : 1) {
                const int h = i & 1, t = i >> 1;          // a half of tile t
                if (h == 0) {
                    if (!mbar_wait(s_full(x), ns & 1u, abort_flag, status)) { alive = false; break; }
                    ++ns;
                    tc_fence_after();
                }
                const uint32_t addr = s_addr + kHalf * h;
                const int col0 = (it.kt0 + t) * kTileRows + h * kHalf;
                uint32_t pk[32];
                float2 sum = make_float2(0.f, 0.f);
                if (live) {
                    uint32_t v[kHalf];
                    tmem_load(addr, v);
                    // The running maximum is m; exponents are counted from m2 = m * c, rounded: a rounding that all of the row shares.
                    // Hidden columns make this one too large at most.
                    float mx4[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mx4[j] = __uint_as_float(v[16 * j]);
#pragma unroll
                        for (int k2 = 0; k2 < 16; k2 += 2) mx4[j] = max3(mx4[j], __uint_as_float(v[16 * j + k2]), __uint_as_float(v[16 * j + k2 + 1]));
                    }
                    const float mx = max3(max3(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]);
                    const uint2 gone = infos[2 * ((tg0 + (uint32_t)t) % kInfos) + h];      // absent rows
                    const bool plain = plain_to >= col0 + kHalf - 1 && (gone.x | gone.y) == 0u;
                    if (plain && i == 2 * part.first && fabsf(mx) < INFINITY) {            // the first maximum: nothing to rescale
                        m = mx;
                        m2 = mx * c;
                    }
                    const float from = E::kTop - m2;
                    const float2 from2 = make_float2(from, from);
                    // Rows that are nobody's (the next problem's queries, or what a kernel before left there) have no say: the two ways
                    // differ in the last bits, and a result's bits are its own problem's.
                    if (plain && __all_sync(0xFFFFFFFFu, !valid || (fmaf(mx, c, -m2) <= E::kRaise && fabsf(m2) <= kLarge))) {
                        // almost always: nothing hidden, no new maximum
#pragma unroll
                        for (int k2 = 0; k2 < 32; ++k2) {
                            const float2 e = exp2_pair(__ffma2_rn(make_float2(__uint_as_float(v[2 * k2]), __uint_as_float(v[2 * k2 + 1])), c2, from2), k2);
                            sum = __fadd2_rn(sum, e);
                            pk[k2] = E::pack(e.x, e.y);
                        }
                    } else {
                        // columns of the first and the last 32 that the row sees, as bits
                        const int last = min(limit, it.rows - 1) - col0;
                        const uint32_t see[2] = {(last >= 31 ? 0xFFFFFFFFu : last < 0 ? 0u : (2u << last) - 1u) & ~gone.x,
                                                 (last >= 63 ? 0xFFFFFFFFu : last < 32 ? 0u : (2u << (last - 32)) - 1u) & ~gone.y};
                        float top = -INFINITY;
#pragma unroll
                        for (int k2 = 0; k2 < 32; ++k2) {
                            if (!(see[0] >> k2 & 1u)) v[k2] = 0xFF800000u;
                            if (!(see[1] >> k2 & 1u)) v[32 + k2] = 0xFF800000u;
                            top = max3(top, __uint_as_float(v[k2]), __uint_as_float(v[32 + k2]));
                        }
                        float factor = 1.f;
                        bool raise = false;
                        if (valid && !(fmaf(top, c, -m2) <= E::kRaise)) { // also the first rows that are not all hidden, and NaN
                            const float to = top * c;
                            if (m == -INFINITY) {
                                l = 0.f;                  // what was added before (rows of -inf alone) is nothing
                            } else {
                                raise = true;
                                factor = fast_exp2(m2 - to);
                                l *= factor;
                            }
                            m = top;
                            m2 = to;
                        }
                        // TMEM accesses are warp-wide: the other rows multiply by one
                        if (__any_sync(0xFFFFFFFFu, raise)) {
                            // S was issued behind the previous tile's P V, and the tensor cores complete in issue order: O is at
                            // rest, but for the product with the tile's own first half
                            if (h == 1) {
                                if (!mbar_wait(pv_half(x), (ns & 1u) ^ 1u, abort_flag, status)) { alive = false; break; }
                                tc_fence_after();
                            }
#pragma unroll 1
                            for (int j = 0; j < D / 32; ++j) {
                                tmem_load(tmem_o(x) + lane_sel + 32 * j, pk);
#pragma unroll
                                for (int k2 = 0; k2 < 32; ++k2) pk[k2] = __float_as_uint(__uint_as_float(pk[k2]) * factor);
                                tmem_st32(tmem_o(x) + lane_sel + 32 * j, pk);
                            }
                            tmem_st_wait();
                        }
                        // Scores so large that m2's rounding would show in the exponent (half a step of 2^24 and more): the
                        // difference of two scores that are near each other is exact before the scale.
                        const bool far = fabsf(m2) > kLarge;
                        const float rest = E::kTop + (far ? 0.f : fmaf(m, c, -m2)), use = m == -INFINITY ? 0.f : m;
#pragma unroll
                        for (int k2 = 0; k2 < 32; ++k2) { // an exact zero for -inf
                            const float2 e = make_float2(fast_exp2(fmaf(__uint_as_float(v[2 * k2]) - use, c, rest)),
                                                         fast_exp2(fmaf(__uint_as_float(v[2 * k2 + 1]) - use, c, rest)));
                            sum = __fadd2_rn(sum, e);
                            pk[k2] = E::pack(e.x, e.y);
                        }
                    }
                    tmem_st32(addr, pk);
                    l += sum.x + sum.y;
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(x, h));
            }
            if (!alive) break;
            tg0 += (uint32_t)tiles;
            const bool some = part.first < part.end;      // the team's O holds something
            if (some) {
                if (!mbar_wait(pv(x), ni & 1u, abort_flag, status)) { alive = false; break; }
                ++ni;
                tc_fence_after();
            }
            bool some1 = false;                           // the second team's O of a single query tile does
            float f0 = 1.f, f1 = 0.f;
            if (!pair && tiles > 1) {
                if (x == 1) {
                    other_s[r] = make_float2(m2, l);      // read before o_free(1) lets the team's next product go ahead
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(other_done);
                } else {
                    if (!mbar_wait(other_done, no & 1u, abort_flag, status)) { alive = false; break; }
                    tc_fence_after();
                    const float2 ml = other_s[r];
                    ++no;
                    some1 = true;
                    const float top = max3(m2, ml.x, ml.x);
                    f0 = fast_exp2(m2 - top);
                    f1 = fast_exp2(ml.x - top);
                    l = l * f0 + ml.y * f1;
                    m2 = top;
                }
            }
            if (pair || x == 0) {
                const bool dirty = bad_any[sl] != 0;
                const size_t token = (size_t)it.token + skip + my_token, head = (size_t)it.h * a.G + my_head;
                auto store = [&](uint16_t *row, const float (&f)[32], float inv) {
                    uint4 *to = reinterpret_cast<uint4 *>(row);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float *g = f + 8 * q;
                        to[q] = make_uint4(E::pack(g[0] * inv, g[1] * inv), E::pack(g[2] * inv, g[3] * inv),
                                           E::pack(g[4] * inv, g[5] * inv), E::pack(g[6] * inv, g[7] * inv));
                    }
                };
                const size_t at = (size_t)it.slot * 2 + x;
                const bool none = m2 == kLowest && l == l;               // the row sees nothing, or scores of -inf alone
                const float inv = none ? 0.f : 1.f / l;
                if (live) {
#pragma unroll 1
                    for (int j = 0; j < D / 32; ++j) {
                        const int col = 32 * j;
                        float f[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = 0.f;
                        if (some) {
                            uint32_t ro[32];
                            tmem_load(tmem_o(x) + lane_sel + col, ro);
#pragma unroll
                            for (int i = 0; i < 32; ++i) f[i] = none ? 0.f : __uint_as_float(ro[i]) * f0;
                        }
                        if (some1) {
                            uint32_t ro[32];
                            tmem_load(tmem_o(1) + lane_sel + col, ro);
#pragma unroll
                            for (int i = 0; i < 32; ++i) f[i] = none ? 0.f : fmaf(__uint_as_float(ro[i]), f1, f[i]);
                        }
                        if (dirty && valid && !none) {    // rows of this CTA that not every token of the item sees
                            const uint32_t bits = spoilt<E::kExponent>(a, it.n, it.h, max(max(it.limit + 1, 0), it.kt0 * kTileRows),
                                                                       min(min(limit + 1, it.rows), it.kt1 * kTileRows), col);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (bits >> i & 1u) f[i] = __int_as_float(0x7FFFFFFF);
                        }
                        if (!valid) continue;
                        if (it.parts == 0) {
                            store(out + (int64_t)token * out_token + (int64_t)head * out_head + col, f, inv);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                __stcg(parts.o + (at * (D / 4) + col / 4 + i) * kTileRows + r, make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]));
                        }
                    }
                    if (valid && it.parts == 0 && lse) lse[token * a.Hq + head] = log_sum<E>(m2, l);
                    if (valid && it.parts > 0) __stcg(parts.ml + at * kTileRows + r, make_float2(m2, some ? l : 0.f));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (some) mbar_arrive(o_free(x));
                    if (some1) mbar_arrive(o_free(1));
                }
                if (it.parts > 0) {
                    // the CTA that arrives last puts the parts together, in the order of the rows
                    if (!meet()) { alive = false; break; }
                    int *counter = a.c.state + kStateChunk + it.first * kChunkCounters + (int)x;
                    if (q4 == 0 && lane == 0) {
                        const bool last = arrive(counter) == it.parts - 1;
                        if (last) *counter = 0;
                        last_s[x] = last;
                    }
                    if (!meet()) { alive = false; break; }
                    if (last_s[x]) {
                        join_parts<D, DTYPE>(parts, it.first, it.parts, (int)x, ntok, a.G,
                                             out + ((int64_t)it.token + skip) * out_token + (int64_t)it.h * a.G * out_head, out_token, out_head,
                                             lse ? lse + ((int64_t)it.token + skip) * a.Hq + (int64_t)it.h * a.G : nullptr, a.Hq);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(item_empty(sl));
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
cudaError_t launch_t(const ChunkArgs &a, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, void *out, int64_t out_token,
                     int64_t out_head, float *lse, const Parts &parts, cudaStream_t stream)
{
    auto kernel = chunk_attention_kernel<D, DTYPE>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::kTotal);
    if (e != cudaSuccess) return e;
    return launch_chained(kernel, dim3(chunk_grid()), kThreads, Smem<D>::kTotal, stream, mq, mk, mv, a, static_cast<uint16_t *>(out),
                          out_token, out_head, lse, parts);
}

}  // namespace

size_t chunk_attention_workspace_bytes(int D)
{
    return (size_t)2 * kChunkMaxCtas * 2 * kTileRows * ((size_t)D * sizeof(float) + sizeof(float2));
}

cudaError_t launch_chunk_attention(const ChunkArgs &a, int D, int dtype, const void *q, int64_t q_token, int64_t q_head, void *out,
                                   int64_t out_token, int64_t out_head, float *lse, void *ws, cudaStream_t stream)
{
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, a, D, dtype, q, q_token, q_head) || !make_pool_map(&mk, a, D, dtype, a.c.K) ||
        !make_pool_map(&mv, a, D, dtype, a.c.V))
        return cudaErrorInvalidValue;
    Parts parts;
    parts.o = static_cast<float4 *>(ws);
    parts.ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + (size_t)2 * kChunkMaxCtas * 2 * kTileRows * D * sizeof(float));
    if (D == 128)
        return dtype == EC_BF16 ? launch_t<128, EC_BF16>(a, mq, mk, mv, out, out_token, out_head, lse, parts, stream)
                                : launch_t<128, EC_FP16>(a, mq, mk, mv, out, out_token, out_head, lse, parts, stream);
    return dtype == EC_BF16 ? launch_t<64, EC_BF16>(a, mq, mk, mv, out, out_token, out_head, lse, parts, stream)
                            : launch_t<64, EC_FP16>(a, mq, mk, mv, out, out_token, out_head, lse, parts, stream);
}

}  // namespace ec
