// C ABI of a chunk of new tokens on a paged cache (pages, rotary positions, attention, gathered weights) and of the rotary
// positions alone: argument validation, workspace layout and launches.
#include "ec_chunk.cuh"
#include "ec_paged_api.cuh"
#include "ec_rotary.cuh"

#include <math.h>

namespace {

using ec::aligned;

// Packed rows [tokens, heads, D] by strides, in elements: rows of 16-byte pieces, within what a copy's description can hold.
int check_rows(const void *p, int64_t token, int64_t head, int D)
{
    if (!p) return EC_ERR_NULL;
    if (!aligned(p, 16)) return EC_ERR_ALIGN;
    const int64_t most = (int64_t)1 << 38;
    if (token < 1 || head < D || token % 8 || head % 8 || token > most || head > most) return EC_ERR_ARG;
    return EC_OK;
}

int check_turn(const double *freqs, int rot, int interleaved, float factor, int D)
{
    if (rot < 0 || rot > D || rot % (interleaved ? 8 : 16)) return EC_ERR_ARG;
    if (rot > 0 && !freqs) return EC_ERR_NULL;
    if (!aligned(freqs, 8)) return EC_ERR_ALIGN;
    return isfinite(factor) ? EC_OK : EC_ERR_ARG;
}

ec::RotaryTurn turn(const double *freqs, int rot, float factor, int inverse)
{
    ec::RotaryTurn r;
    r.freqs = freqs;
    r.rot = rot;
    r.factor = factor;
    r.inverse = inverse != 0;
    return r;
}

int check_pool(const ec_paged *c, const ec_pages *p)
{
    const int st = ec::check_paged(c);
    if (st != EC_OK) return st;
    if (!p || !p->free_pages || !p->n_free || !p->held) return EC_ERR_NULL;
    return aligned(p->free_pages, 4) && aligned(p->n_free, 4) && aligned(p->held, 4) ? EC_OK : EC_ERR_ALIGN;
}

ec::PagePool pool(const ec_pages *p)
{
    ec::PagePool v;
    v.free = p->free_pages;
    v.n_free = p->n_free;
    v.held = p->held;
    return v;
}

int check_chunk(const ec_paged *c, const int32_t *starts, const int32_t *counts, int tokens, int Hq, float scale)
{
    int st = ec::check_paged(c);
    if (st != EC_OK) return st;
    if (!starts || !counts) return EC_ERR_NULL;
    if (!aligned(starts, 4) || !aligned(counts, 4)) return EC_ERR_ALIGN;
    if (tokens < 0 || Hq < 1 || Hq % c->H || Hq / c->H > 128 || (long long)tokens * Hq >= (1LL << 31)) return EC_ERR_SHAPE;
    if (!(scale > 0.f) || !isfinite(scale * 1.4426950408889634f)) return EC_ERR_ARG;
    return EC_OK;
}

ec::ChunkArgs chunk(const ec_paged *c, const int32_t *starts, const int32_t *counts, int tokens, int Hq, float scale)
{
    ec::ChunkArgs a;
    a.c = ec::view(c);
    a.starts = starts;
    a.counts = counts;
    a.tokens = tokens;
    a.Hq = Hq;
    a.G = Hq / c->H;
    a.tile_tokens = ec::kTileRows / a.G;
    a.box_rows = ec::box_rows_of(c->page_size);
    a.scale_log2e = scale * 1.4426950408889634f;
    a.inv_ctas = 1.0 / ec::chunk_grid();
    return a;
}

int done(cudaError_t e) { return e == cudaSuccess ? EC_OK : EC_ERR_CUDA; }

}  // namespace

extern "C" {

int ec_paged_release(const ec_paged *c, const ec_pages *p, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_release");
    const int st = check_pool(c, p);
    if (st != EC_OK) return st;
    return done(ec::launch_release(ec::view(c), pool(p), (cudaStream_t)stream));
}

int ec_paged_reserve(const ec_paged *c, const ec_pages *p, const int32_t *counts, int tokens, int advance, int limit, int32_t *starts,
                     int32_t *granted, int32_t *slots, int32_t *positions, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_reserve");
    const int st = check_pool(c, p);
    if (st != EC_OK) return st;
    if (!counts || !granted) return EC_ERR_NULL;
    if (tokens < 0 || limit < 0 || (!advance && (slots || positions))) return EC_ERR_ARG;
    if (c->N > 65536) return EC_ERR_SHAPE;
    if (!aligned(counts, 4) || !aligned(starts, 4) || !aligned(granted, 4) || !aligned(slots, 4) || !aligned(positions, 4)) return EC_ERR_ALIGN;
    // several CTAs read the counts while one of them writes the answers
    if (counts == granted || counts == starts || counts == slots || counts == positions) return EC_ERR_ARG;
    ec::ReserveArgs a;
    a.counts = counts;
    a.starts = starts;
    a.granted = granted;
    a.slots = slots;
    a.positions = positions;
    a.table = c->table;
    a.lens = c->lens;
    a.seen = c->seen;
    a.tokens = tokens;
    a.advance = advance != 0;
    a.limit = limit;
    return done(ec::launch_reserve(ec::view(c), pool(p), a, (cudaStream_t)stream));
}

int ec_rotary_frequencies(double *freqs, float *factor, int rot, double base, int scaling, double stretch, double trained, double fast,
                          double slow)
{
    if (!freqs || !factor) return EC_ERR_NULL;
    if (rot < 2 || rot % 2 || rot > 1024) return EC_ERR_SHAPE;
    if (!(base > 1.0) || !isfinite(base) || scaling < EC_ROTARY_PLAIN || scaling > EC_ROTARY_BY_PARTS) return EC_ERR_ARG;
    if (scaling != EC_ROTARY_PLAIN && (!(stretch >= 1.0) || !isfinite(stretch))) return EC_ERR_ARG;
    if (scaling == EC_ROTARY_BY_PARTS && (!(trained > 0.0) || !isfinite(trained) || !(slow > 0.0) || !(fast >= slow) || !isfinite(fast))) return EC_ERR_ARG;
    if (scaling == EC_ROTARY_BASE && rot < 4) return EC_ERR_SHAPE;
    if (scaling == EC_ROTARY_BASE) base *= pow(stretch, (double)rot / (rot - 2));
    double lo = 0.0, hi = 0.0;
    bool all_slow = false;                       // even the fastest pair turns less than `slow` times
    if (scaling == EC_ROTARY_BY_PARTS) {
        // the (fractional) pair that turns x times over the trained length
        auto pair_of = [&](double x) { return rot * log(trained / (x * 2.0 * M_PI)) / (2.0 * log(base)); };
        lo = fmax(floor(pair_of(fast)), 0.0);
        hi = fmin(ceil(pair_of(slow)), rot - 1.0);
        all_slow = pair_of(slow) < 0.0;
    }
    for (int i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot);
        if (scaling == EC_ROTARY_LINEAR) {
            freqs[i] = f / stretch;
        } else if (scaling == EC_ROTARY_BY_PARTS) {
            const double ramp = all_slow ? 1.0 : fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
            freqs[i] = f / stretch * ramp + f * (1.0 - ramp);
        } else {
            freqs[i] = f;
        }
    }
    *factor = scaling == EC_ROTARY_BY_PARTS ? (float)(0.1 * log(stretch) + 1.0) : 1.f;
    return EC_OK;
}

int ec_rotary(const void *x, int64_t x_n, int64_t x_t, int64_t x_h, void *out, int64_t out_n, int64_t out_t, int64_t out_h,
              const int32_t *positions, int64_t pos_n, const double *freqs, int N, int T, int heads, int D, int dtype, int rot,
              int interleaved, float factor, int inverse, void *stream)
{
    ec::NvtxRange nvtx_range("ec_rotary");
    if (N < 0 || T < 0 || heads < 1 || (D != 64 && D != 128)) return EC_ERR_SHAPE;
    if (dtype != EC_BF16 && dtype != EC_FP16) return EC_ERR_ARG;
    if ((long long)N * T >= (1LL << 31) || heads > 65536) return EC_ERR_SHAPE;
    int st = check_turn(freqs, rot, interleaved, factor, D);
    if (st != EC_OK || N == 0 || T == 0) return st;                      // of no rows nothing is looked at
    st = check_rows(x, x_t, x_h, D);
    if (st == EC_OK) st = check_rows(out, out_t, out_h, D);
    if (st != EC_OK) return st;
    if (!positions) return EC_ERR_NULL;
    if (!aligned(positions, 4)) return EC_ERR_ALIGN;
    if (x_n < 0 || out_n < 0 || x_n % 8 || out_n % 8 || pos_n < 0) return EC_ERR_ARG;
    ec::RotaryRows r;
    r.x = static_cast<const uint4 *>(x);
    r.out = static_cast<uint4 *>(out);
    r.positions = positions;
    r.x_n = x_n / 8;
    r.x_t = x_t / 8;
    r.x_h = x_h / 8;
    r.out_n = out_n / 8;
    r.out_t = out_t / 8;
    r.out_h = out_h / 8;
    r.pos_n = pos_n;
    r.N = N;
    r.T = T;
    r.heads = heads;
    return done(ec::launch_rotary(turn(freqs, rot, factor, inverse), r, D, dtype, !interleaved, (cudaStream_t)stream));
}

int ec_paged_join(const void *q, int64_t q_t, int64_t q_h, void *q_out, int64_t qo_t, int64_t qo_h, const void *k, int64_t k_t, int64_t k_h,
                  const void *v, int64_t v_t, int64_t v_h, const float *w_new, const int32_t *slots, const int32_t *positions,
                  const ec_paged *c, int Hq, int tokens, const double *freqs, int rot, int interleaved, float factor, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_join");
    int st = ec::check_paged(c);
    if (st != EC_OK) return st;
    if (tokens < 0 || Hq < 0 || (long long)tokens * (Hq + c->H) >= (1LL << 31) || Hq + c->H > 65536) return EC_ERR_SHAPE;
    st = check_turn(freqs, rot, interleaved, factor, c->D);
    if (st != EC_OK || tokens == 0) return st;
    if ((Hq > 0) != (q != nullptr) || (Hq > 0) != (q_out != nullptr)) return EC_ERR_NULL;
    if (Hq > 0) st = check_rows(q, q_t, q_h, c->D);
    if (st == EC_OK && Hq > 0) st = check_rows(q_out, qo_t, qo_h, c->D);
    if (st == EC_OK) st = check_rows(k, k_t, k_h, c->D);
    if (st == EC_OK) st = check_rows(v, v_t, v_h, c->D);
    if (st != EC_OK) return st;
    if (!slots || !positions) return EC_ERR_NULL;
    if (!aligned(slots, 4) || !aligned(positions, 4) || !aligned(w_new, 4)) return EC_ERR_ALIGN;
    ec::JoinArgs j;
    j.q = static_cast<const uint4 *>(q);
    j.k = static_cast<const uint4 *>(k);
    j.v = static_cast<const uint4 *>(v);
    j.q_out = static_cast<uint4 *>(q_out);
    j.w_new = w_new;
    j.slots = slots;
    j.positions = positions;
    j.q_t = q_t / 8;
    j.q_h = q_h / 8;
    j.qo_t = qo_t / 8;
    j.qo_h = qo_h / 8;
    j.k_t = k_t / 8;
    j.k_h = k_h / 8;
    j.v_t = v_t / 8;
    j.v_h = v_h / 8;
    j.tokens = tokens;
    j.Hq = Hq;
    return done(ec::launch_join(turn(freqs, rot, factor, 0), ec::view(c), j, c->D, c->dtype, !interleaved, (cudaStream_t)stream));
}

size_t ec_paged_chunk_workspace(const ec_paged *c, int Hq)
{
    if (ec::check_paged(c) != EC_OK || Hq < 1 || Hq % c->H || Hq / c->H > 128) return 0;
    const size_t attention = ec::chunk_attention_workspace_bytes(c->D), weights = ec::chunk_weights_workspace_bytes();
    return ec::round256(attention > weights ? attention : weights);
}

int ec_paged_chunk_attention(const void *q, int64_t q_t, int64_t q_h, const int32_t *starts, const int32_t *counts, const ec_paged *c,
                             int Hq, int tokens, float scale, void *out, int64_t out_t, int64_t out_h, float *lse, void *ws,
                             size_t ws_bytes, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_chunk_attention");
    int st = check_chunk(c, starts, counts, tokens, Hq, scale);
    if (st == EC_OK && tokens > 0) st = check_rows(q, q_t, q_h, c->D);
    if (st == EC_OK && tokens > 0) st = check_rows(out, out_t, out_h, c->D);
    if (st != EC_OK) return st;
    if (!aligned(lse, 4)) return EC_ERR_ALIGN;
    st = ec::check_ws(ws, ws_bytes, ec_paged_chunk_workspace(c, Hq));
    if (st != EC_OK || tokens == 0) return st;
    return done(ec::launch_chunk_attention(chunk(c, starts, counts, tokens, Hq, scale), c->D, c->dtype, q, q_t, q_h, out, out_t, out_h, lse, ws,
                                           (cudaStream_t)stream));
}

int ec_paged_chunk_weights(const void *q, int64_t q_t, int64_t q_h, const float *lse, const int32_t *starts, const int32_t *counts,
                           const ec_paged *c, int Hq, int tokens, float scale, double decay, void *ws, size_t ws_bytes, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_chunk_weights");
    int st = check_chunk(c, starts, counts, tokens, Hq, scale);
    if (st == EC_OK && tokens > 0) st = check_rows(q, q_t, q_h, c->D);
    if (st != EC_OK) return st;
    if (!lse && tokens > 0) return EC_ERR_NULL;
    if (!(decay > 0.0 && decay <= 1.0)) return EC_ERR_ARG;
    if (!aligned(lse, 4)) return EC_ERR_ALIGN;
    st = ec::check_ws(ws, ws_bytes, ec_paged_chunk_workspace(c, Hq));
    if (st != EC_OK || tokens == 0) return st;
    return done(ec::launch_chunk_weights(chunk(c, starts, counts, tokens, Hq, scale), c->D, c->dtype, q, q_t, q_h, lse, decay, ws,
                                         (cudaStream_t)stream));
}

}  // extern "C"
