// Rotary positions, alone or on their way into a paged cache.
//   pair i of a head turns by position * freq_i, scaled by `factor`: (a, b) -> (a cos - b sin, a sin + b cos); the inverse turns back
//   (the transposed map, which is the gradient). Pairs are elements (2 i, 2 i + 1) or (i, i + rot / 2) of the first `rot`.
// Bound by HBM: every element is read once and written once. 8192 tokens with 32 + 8 + 8 heads of 128 into their pages (151 MB):
// 29.2 us, 5.2 TB/s (23.1 us at the copy rate); 67 MB turned back 24.6 us against 22.4 of a plain copy of the same tensors. The issue
// slots are as busy as the memory (75%): no division per row, two pairs an instruction (16384 tokens of 8 heads 19.1 -> 17.0 us).
// What the angles cost is shared by the heads of a token: a CTA
// works out the sines and cosines of its tokens once, in shared memory.
//  - An angle is kept as a fraction of a turn in 64 bits of fixed point: freq / 2 pi from the frequency's 64-bit value, times the
//    position as a whole-number product that drops whole turns by itself. What is lost is the rounding of freq / 2 pi, 2^-52 of the
//    angle with the constant's: 5e-7 at a position of 2^31 and a frequency of 1 (in fp32 an angle of 10^6 is off by 0.06). freq / 2 pi
//    in two parts, exact to 2^-64 of a turn, was measured: 24.7 -> 25.2 us for 67 MB, one head of 187 thousand tokens 39 -> 43, for
//    frequencies that no table of angles has.
#include "ec_paged.cuh"
#include "ec_rotary.cuh"
#include "ec_tc.cuh"

#include <algorithm>

namespace ec {

namespace {

constexpr int kRotThreads = 128;
constexpr int kRotCtas = 12;                     // on an SM, by registers: 29.4 and 24.8 us below; 10 and 13 are slower

template <int DTYPE> __device__ __forceinline__ float2 widen2(uint32_t v)
{
    if constexpr (DTYPE == EC_BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
    else return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

template <int DTYPE> __device__ __forceinline__ uint32_t narrow2(float2 f)
{
    if constexpr (DTYPE == EC_BF16) {
        return pack2(f.x, f.y);
    } else {
        const __half2 h = __floats2half2_rn(f.x, f.y);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}

// cos and sin of position * freq, both times factor.
__device__ __forceinline__ float2 turn_of(double freq, int position, float factor, bool inverse)
{
    double turns = freq * 0.15915494309189533577;                         // 1 / 2 pi
    turns -= floor(turns);
    const unsigned long long step = __double2ull_rn(turns * 18446744073709551616.0);
    const unsigned long long phase = step * (unsigned long long)(long long)position;
    float s, c;
    sincospif((float)(int)(phase >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
    return make_float2(c * factor, (inverse ? -s : s) * factor);
}

// Not the read-only path: the output may be the input.
__device__ __forceinline__ uint4 load_once(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// A token's table: for two neighbouring pairs (cos, cos, sin, sin), a piece of a row takes PER pairs. Neighbouring pieces lie next to
// each other, so that a read of a warp meets no bank twice (in the order of the pairs: 32.2 and 29.4 us against 30.5 and 27.6).
template <int PER> __device__ __forceinline__ void put_turn(float *table, int i, int pieces, float2 cs)
{
    const int j = i % PER;
    float *to = table + ((j >> 1) * pieces + i / PER) * 4 + (j & 1);
    to[0] = cs.x;
    to[2] = cs.y;
}

// What one head row of a token becomes: its place in the input and in the output, nullptr: nothing.
struct RowPlace {
    const uint4 *from;
    uint4 *to;
};

// A thread keeps its place in the head (piece `v`) and walks over the rows (token, head) of the CTA; gridDim.y parts of the heads have a
// CTA each. Places(token, head) gives a row's pointers. One row a thread in flight, and as many CTAs as fit: two and four rows a thread are slower (32 -> 37 and 40 us before
// the CTAs were as many).
template <int DTYPE, bool HALF, typename Places>
struct RowTurner {
    const RotaryTurn &r;
    Places places;
    int step, v, lo, hi;                         // lo, hi: pieces of a row, of 16 bytes; hi < 0: there is none
    int token, head, tokens, heads;              // the row in flight, until token = tokens
    bool turns;
    RowPlace at;
    uint4 a, b;

    __device__ __forceinline__ RowTurner(const RotaryTurn &turn, int D, int tokens_, int heads_, Places p) : r(turn), places(p), tokens(tokens_), heads(heads_)
    {
        const int turning = r.rot / (HALF ? 16 : 8), pieces = turning + (D - r.rot) / 8;
        step = kRotThreads / pieces;
        v = threadIdx.x % pieces;
        head = threadIdx.x / pieces;
        token = head < step ? 0 : tokens;        // threads without a piece of a row
        settle();
        turns = v < turning;
        lo = turns ? v : v - turning + r.rot / 8;
        hi = HALF && turns ? v + r.rot / 16 : -1;
    }

    __device__ __forceinline__ void load()
    {
        at = places(token, head);
        if (at.to == nullptr) return;
        a = load_once(at.from + lo);
        if (hi >= 0) b = load_once(at.from + hi);
    }

    __device__ __forceinline__ void settle()
    {
        if (head < heads || token >= tokens) return;
        head -= heads;
        ++token;
        if (head >= heads) {                     // fewer heads than rows at a time
            const int n = head / heads;
            head -= n * heads;
            token += n;
        }
    }

    __device__ __forceinline__ void store(const float2 *table)
    {
        if (at.to == nullptr) return;
        if (turns) {
            const int pieces = r.rot / (HALF ? 16 : 8);
            const float4 *cs = reinterpret_cast<const float4 *>(table + token * (r.rot / 2)) + v;
            uint32_t *xa = reinterpret_cast<uint32_t *>(&a), *xb = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 u = widen2<DTYPE>(xa[i]);
                if (HALF) {                      // two pairs an instruction
                    const float4 t = cs[i * pieces];
                    const float2 c = make_float2(t.x, t.y), s = make_float2(t.z, t.w), w = widen2<DTYPE>(xb[i]);
                    xa[i] = narrow2<DTYPE>(__ffma2_rn(u, c, __fmul2_rn(make_float2(-w.x, -w.y), s)));
                    xb[i] = narrow2<DTYPE>(__ffma2_rn(u, s, __fmul2_rn(w, c)));
                } else {
                    const float4 t = cs[i / 2 * pieces];
                    const float c = i & 1 ? t.y : t.x, s = i & 1 ? t.w : t.z;
                    xa[i] = narrow2<DTYPE>(make_float2(u.x * c - u.y * s, u.x * s + u.y * c));
                }
            }
            if (HALF) at.to[hi] = b;
        }
        at.to[lo] = a;
    }

    // The first rows are under way while `make_table` works out the angles.
    template <typename Table>
    __device__ __forceinline__ void run(const float2 *table, Table make_table)
    {
        if (token < tokens) load();
        make_table();
        __syncthreads();
        while (token < tokens) {
            store(table);
            head += step;
            settle();
            if (token < tokens) load();
        }
    }
};

template <int DTYPE, bool HALF>
__global__ void __launch_bounds__(kRotThreads, kRotCtas)
rotary_kernel(const RotaryTurn r, const RotaryRows x, int D, int per)
{
    extern __shared__ __align__(16) float2 table[];
    const int first = blockIdx.x * per, tokens = min(per, x.N * x.T - first);
    grid_wait();
    grid_release();
    const int n0 = first / x.T, at0 = first - n0 * x.T, share = (x.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * share;
    auto place = [&](int t, int h) {
        int n = n0, at = at0 + t;
        if (at >= x.T) {
            n += at / x.T;
            at %= x.T;
        }
        h += h0;
        return RowPlace{x.x + n * x.x_n + at * x.x_t + h * x.x_h, x.out + n * x.out_n + at * x.out_t + h * x.out_h};
    };
    RowTurner<DTYPE, HALF, decltype(place)> turner(r, D, h0 < x.heads ? tokens : 0, min(share, x.heads - h0), place);
    turner.run(table, [&] {
        const int half = r.rot / 2;
        for (int i = threadIdx.x; i < tokens * half; i += kRotThreads) {
            const int t = i / half, token = first + t, n = token / x.T;
            put_turn<HALF ? 8 : 4>(reinterpret_cast<float *>(table + t * half), i - t * half, r.rot / (HALF ? 16 : 8),
                                   turn_of(r.freqs[i - t * half], x.positions[n * x.pos_n + (token - n * x.T)], r.factor, r.inverse));
        }
    });
}

template <int DTYPE, bool HALF>
__global__ void __launch_bounds__(kRotThreads, kRotCtas)
join_kernel(const RotaryTurn r, const PagedView c, const JoinArgs j, int D, int per)
{
    extern __shared__ __align__(16) float2 table[];
    __shared__ int slot_s[kRotaryMostTokens], pos_s[kRotaryMostTokens];
    __shared__ uint32_t offset_s[kRotaryMostTokens], meta_s[kRotaryMostTokens];    // of head 0, in the pools and in weight and pos
    const int first = blockIdx.x * per, tokens = min(per, j.tokens - first);
    grid_wait();
    grid_release();
    if ((int)threadIdx.x < tokens) {
        int slot = j.slots[first + threadIdx.x];
        if (slot >= c.n_pages * c.page_size) {
            report_page(c);
            slot = -1;
        }
        slot_s[threadIdx.x] = slot;
        pos_s[threadIdx.x] = j.positions[first + threadIdx.x];
        if (slot >= 0) {
            Slot s;
            s.page = page_of(c, slot);
            s.slot = slot - s.page * c.page_size;
            offset_s[threadIdx.x] = row_offset(c, s);
            meta_s[threadIdx.x] = meta_index(c, 0, s);
        }
    }
    __syncthreads();
    const int heads = j.Hq + c.H, share = (heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * share;
    auto row_place = [&](int t, int h) {
        h += h0;
        if (slot_s[t] < 0) return RowPlace{nullptr, nullptr};
        if (h < j.Hq) return RowPlace{j.q + (first + t) * j.q_t + h * j.q_h, j.q_out + (first + t) * j.qo_t + h * j.qo_h};
        h -= j.Hq;
        return RowPlace{j.k + (first + t) * j.k_t + h * j.k_h, c.K + offset_s[t] + (size_t)h * c.head_step};
    };
    RowTurner<DTYPE, HALF, decltype(row_place)> turner(r, D, h0 < heads ? tokens : 0, min(share, heads - h0), row_place);
    turner.run(table, [&] {
        const int half = r.rot / 2;
        for (int i = threadIdx.x; i < tokens * half; i += kRotThreads) {
            const int t = i / half;
            put_turn<HALF ? 8 : 4>(reinterpret_cast<float *>(table + t * half), i - t * half, r.rot / (HALF ? 16 : 8),
                                   turn_of(r.freqs[i - t * half], pos_s[t], r.factor, false));
        }
    });
    // values, weights and positions of the part's share of the key heads
    const int few = (c.H + gridDim.y - 1) / gridDim.y, v0 = blockIdx.y * few, H = min(few, c.H - v0);
    if (H <= 0) return;
    const int pieces = D / 8, v = threadIdx.x % pieces, step = kRotThreads / pieces, rows = tokens * H;
    for (int row = threadIdx.x / pieces; row < rows; row += step) {
        const int t = row / H, h = v0 + row - t * H;
        if (slot_s[t] >= 0) c.V[offset_s[t] + (size_t)h * c.head_step + v] = load_once(j.v + (first + t) * j.v_t + h * j.v_h + v);
    }
    for (int row = threadIdx.x; row < rows; row += kRotThreads) {
        const int t = row / H, h = v0 + row - t * H;
        if (slot_s[t] < 0) continue;
        const uint32_t at = meta_s[t] + (uint32_t)h * (uint32_t)c.page_size;
        c.weight[at] = j.w_new ? j.w_new[(size_t)(first + t) * c.H + h] : 0.f;
        c.pos[at] = pos_s[t];
    }
}

// A CTA has about 72 rows of 256 bytes: tokens of few heads together (one token of 32 and 48 heads: 23.9 and 30.5 us, two 24.8 and 29.4, four
// 27.6 and 30.5), as long as there are twelve CTAs an SM; where there are fewer, many heads of a
// token are split (300 tokens of 288 head rows 29 -> 9 us, 24 of 48 4.6 -> 3.2; 512 of 48 would take 6.0 instead of 4.8). One head, 187
// thousand tokens: 100 us with two tokens a CTA, 36 with sixteen.
struct RotaryShape {
    int per;                                     // tokens of a CTA
    dim3 grid;
};

RotaryShape rotary_shape(int tokens, int heads, int D)
{
    RotaryShape s;
    const int rows = 72 * 128 / D;
    s.per = std::max(1, std::min({(rows + heads / 2) / heads, tokens / (kRotCtas * sm_count()), kRotaryMostTokens}));
    const int ctas = (tokens + s.per - 1) / s.per;
    const int least = ctas < sm_count() ? kRotThreads / (D / 8) : rows;   // rows at once, where there are hardly any
    s.grid = dim3(ctas, std::max(1, std::min(kRotCtas * sm_count() / ctas, (heads + least - 1) / least)));
    return s;
}

}  // namespace

cudaError_t launch_rotary(const RotaryTurn &r, const RotaryRows &x, int D, int dtype, bool half, cudaStream_t stream)
{
    const RotaryShape shape = rotary_shape(x.N * x.T, x.heads, D);
    const int per = shape.per;
    auto go = [&](auto kernel) { return launch_chained(kernel, shape.grid, kRotThreads, (size_t)per * (r.rot / 2) * sizeof(float2), stream, r, x, D, per); };
    if (dtype == EC_BF16) return half ? go(rotary_kernel<EC_BF16, true>) : go(rotary_kernel<EC_BF16, false>);
    return half ? go(rotary_kernel<EC_FP16, true>) : go(rotary_kernel<EC_FP16, false>);
}

cudaError_t launch_join(const RotaryTurn &r, const PagedView &c, const JoinArgs &j, int D, int dtype, bool half, cudaStream_t stream)
{
    const RotaryShape shape = rotary_shape(j.tokens, j.Hq + c.H, D);
    const int per = shape.per;
    auto go = [&](auto kernel) { return launch_chained(kernel, shape.grid, kRotThreads, (size_t)per * (r.rot / 2) * sizeof(float2), stream, r, c, j, D, per); };
    if (dtype == EC_BF16) return half ? go(join_kernel<EC_BF16, true>) : go(join_kernel<EC_BF16, false>);
    return half ? go(join_kernel<EC_FP16, true>) : go(join_kernel<EC_FP16, false>);
}

}  // namespace ec
