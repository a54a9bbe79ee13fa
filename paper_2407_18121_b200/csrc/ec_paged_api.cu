// C ABI of the paged cache: argument validation, workspace layout and kernel sequencing.
#include "ec_paged.cuh"

#include <math.h>

#include <new>
#include <vector>

namespace {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// The caller owns the struct: every call repeats these checks.
int check_paged(const ec_paged *c)
{
    if (!c) return EC_ERR_NULL;
    if (!c->Kp || !c->Vp || !c->weight || !c->pos || !c->table || !c->lens || !c->seen || !c->state) return EC_ERR_NULL;
    if (c->N < 1 || c->H < 1 || (c->D != 64 && c->D != 128) || c->page_size < 1 || c->n_pages < 1 || c->max_pages < 1)
        return EC_ERR_SHAPE;
    if ((long long)c->N * c->H >= (1LL << 24) || (long long)c->N * c->max_pages >= (1LL << 31)) return EC_ERR_SHAPE;
    if ((long long)c->max_pages * c->page_size >= (1LL << 30)) return EC_ERR_SHAPE;
    if ((long long)c->n_pages * c->H >= (1LL << 31) || (long long)c->n_pages * c->H * c->page_size >= (1LL << 31)) return EC_ERR_SHAPE;
    if (c->dtype != EC_BF16 && c->dtype != EC_FP16) return EC_ERR_ARG;
    const int64_t most = (int64_t)1 << 35;       // 64 GiB of 2-byte elements
    if (c->page_stride < 1 || c->head_stride < 1 || c->row_stride < c->D || c->page_stride % 8 || c->head_stride % 8 ||
        c->row_stride % 8 || c->page_stride > most || c->head_stride > most || c->row_stride > most)
        return EC_ERR_ARG;
    // rows are addressed from their head's row of page 0, in 32-bit counts of 16 bytes
    const double last = (double)(c->n_pages - 1) * (double)c->page_stride + (double)(c->page_size - 1) * (double)c->row_stride +
                        (double)(c->H - 1) * (double)c->head_stride + c->D;
    if (last > (double)most - 16.0) return EC_ERR_SHAPE;
    if (!aligned(c->Kp, 16) || !aligned(c->Vp, 16) || !aligned(c->weight, 4) || !aligned(c->pos, 4) || !aligned(c->table, 4) ||
        !aligned(c->lens, 4) || !aligned(c->seen, 4) || !aligned(c->state, 256))
        return EC_ERR_ALIGN;
    return EC_OK;
}

ec::PagedView view(const ec_paged *c)
{
    ec::PagedView v;
    v.K = static_cast<uint4 *>(c->Kp);
    v.V = static_cast<uint4 *>(c->Vp);
    v.weight = c->weight;
    v.pos = c->pos;
    v.table = c->table;
    v.lens = c->lens;
    v.seen = c->seen;
    v.state = static_cast<int *>(c->state);
    v.N = c->N;
    v.H = c->H;
    v.page_size = c->page_size;
    v.n_pages = c->n_pages;
    v.max_pages = c->max_pages;
    v.page_step = (uint32_t)(c->page_stride / 8);
    v.head_step = (uint32_t)(c->head_stride / 8);
    v.row_step = (uint32_t)(c->row_stride / 8);
    ec::set_page_division(v);
    return v;
}

int check_heads(const ec_paged *c, int Hq)
{
    if (Hq < 1 || Hq % c->H != 0 || Hq / c->H > 128 || (long long)c->N * Hq >= (1LL << 24)) return EC_ERR_SHAPE;
    // work is counted in blocks of 64 rows, in 31 bits
    const long long units = (long long)c->N * c->H * ((Hq / c->H + 7) / 8);
    if (units * ((long long)c->max_pages * c->page_size / 64 + 2) >= (1LL << 31)) return EC_ERR_SHAPE;
    return EC_OK;
}

int check_attention(const void *q, const void *k_new, const void *v_new, const ec_paged *c, int Hq, float scale, int accumulate,
                    float decay, const void *out, const float *lse)
{
    int st = check_paged(c);
    if (st != EC_OK) return st;
    if (!q || !out || (!k_new) != (!v_new)) return EC_ERR_NULL;
    st = check_heads(c, Hq);
    if (st != EC_OK) return st;
    if (!(scale > 0.f) || !isfinite(scale * 1.4426950408889634f)) return EC_ERR_ARG;   // scores are scaled by scale * log2(e)
    if (accumulate && !(decay > 0.f && decay <= 1.f)) return EC_ERR_ARG;
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(lse, 4)) return EC_ERR_ALIGN;
    return EC_OK;
}

int check_budget(const ec_paged *c, int T, int budget, int recent, int sinks)
{
    if (T < 0 || budget < 1 || recent < 0 || sinks < 0 || (long long)recent + sinks > budget) return EC_ERR_ARG;
    if ((long long)budget > (long long)c->max_pages * c->page_size) return EC_ERR_ARG;
    if ((long long)c->N * c->H * T >= (1LL << 31) || (long long)c->max_pages * c->page_size + T >= (1LL << 31)) return EC_ERR_SHAPE;
    if ((long long)c->N * c->H * budget >= (1LL << 31)) return EC_ERR_SHAPE;
    return EC_OK;
}

ec::AppendArgs append_args(const void *K_new, const void *V_new, const float *w_new, const int32_t *pos_new, const int32_t *counts,
                           int T, int fresh, int budget, int recent, int sinks)
{
    ec::AppendArgs a = {};
    a.K_new = static_cast<const uint4 *>(K_new);
    a.V_new = static_cast<const uint4 *>(V_new);
    a.w_new = w_new;
    a.pos_new = pos_new;
    a.counts = counts;
    a.T = T;
    a.fresh = fresh;
    a.budget = budget;
    a.recent = recent;
    a.sinks = sinks;
    return a;
}

int check_ws(const void *ws, size_t have, size_t need)
{
    if (!ws || have < need) return EC_ERR_WORKSPACE;
    return aligned(ws, 256) ? EC_OK : EC_ERR_ALIGN;
}

}  // namespace

extern "C" {

size_t ec_paged_state_bytes(int N) { return N < 1 ? 0 : round256((ec::kStateAppend + (size_t)N) * sizeof(int)); }

int ec_paged_init(ec_paged *c, void *Kp, void *Vp, float *weight, int32_t *pos, int32_t *table, int32_t *lens, int32_t *seen,
                  void *state, int N, int H, int D, int page_size, int n_pages, int max_pages, int dtype, int64_t page_stride,
                  int64_t head_stride, int64_t row_stride, void *stream)
{
    if (!c) return EC_ERR_NULL;
    ec_paged n;
    n.Kp = Kp;
    n.Vp = Vp;
    n.weight = weight;
    n.pos = pos;
    n.table = table;
    n.lens = lens;
    n.seen = seen;
    n.state = state;
    n.N = N;
    n.H = H;
    n.D = D;
    n.page_size = page_size;
    n.n_pages = n_pages;
    n.max_pages = max_pages;
    n.dtype = dtype;
    n.page_stride = page_stride;
    n.head_stride = head_stride;
    n.row_stride = row_stride;
    const int st = check_paged(&n);
    if (st != EC_OK) return st;
    if (cudaMemsetAsync(state, 0, ec_paged_state_bytes(N), (cudaStream_t)stream) != cudaSuccess) return EC_ERR_CUDA;
    *c = n;
    return EC_OK;
}

int ec_paged_check(const ec_paged *c, const int32_t *table, const int32_t *lens, int rows)
{
    const int st = check_paged(c);
    if (st != EC_OK) return st;
    if (!table || !lens) return EC_ERR_NULL;
    const long long cap = (long long)c->max_pages * c->page_size;
    if (rows < 0 || rows > cap) return EC_ERR_ARG;
    try {
        std::vector<bool> used((size_t)c->n_pages, false);
        for (int n = 0; n < c->N; ++n) {
            if (lens[n] < 0) continue;
            if (lens[n] > cap) return EC_ERR_PAGE;
            const long long most = lens[n] > rows ? lens[n] : rows;
            const long long pages = (most + c->page_size - 1) / c->page_size;
            for (long long p = 0; p < pages; ++p) {
                const int id = table[(size_t)n * c->max_pages + p];
                if (id < 0 || id >= c->n_pages || used[(size_t)id]) return EC_ERR_PAGE;
                used[(size_t)id] = true;
            }
        }
    } catch (const std::bad_alloc &) {
        return EC_ERR_TOO_LARGE;
    }
    return EC_OK;
}

size_t ec_paged_attention_workspace(const ec_paged *c, int Hq, int accumulate)
{
    if (check_paged(c) != EC_OK || check_heads(c, Hq) != EC_OK) return 0;
    return ec::paged_attention_workspace_bytes(c, Hq, accumulate);
}

int ec_paged_attention(const void *q, const void *k_new, const void *v_new, const ec_paged *c, int Hq, float scale,
                       int accumulate, float decay, void *out, float *lse, float *w_new, void *ws, size_t ws_bytes, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_attention");
    int st = check_attention(q, k_new, v_new, c, Hq, scale, accumulate, decay, out, lse);
    if (st != EC_OK) return st;
    if (accumulate && k_new && !w_new) return EC_ERR_NULL;
    if (!aligned(w_new, 4)) return EC_ERR_ALIGN;
    st = check_ws(ws, ws_bytes, ec::paged_attention_workspace_bytes(c, Hq, accumulate));
    if (st != EC_OK) return st;
    ec::GatherArgs gather;
    cudaError_t e = ec::launch_paged_attention(view(c), c->D, c->dtype, q, k_new, v_new, Hq, scale, accumulate, decay, out, lse, w_new,
                                               ws, &gather, (cudaStream_t)stream);
    if (e == cudaSuccess && accumulate) e = ec::launch_paged_rows(view(c), c->D, &gather, nullptr, nullptr, (cudaStream_t)stream);
    return e == cudaSuccess ? EC_OK : EC_ERR_CUDA;
}

size_t ec_paged_append_workspace(const ec_paged *c, int T, int budget)
{
    if (check_paged(c) != EC_OK || check_budget(c, T, budget, 0, 0) != EC_OK) return 0;
    return ec::paged_append_workspace_bytes(c, T, budget);
}

int ec_paged_append(const void *K_new, const void *V_new, const float *w_new, const int32_t *pos_new, const int32_t *counts,
                    const ec_paged *c, int T, int fresh, int budget, int recent, int sinks, void *ws, size_t ws_bytes, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_append");
    int st = check_paged(c);
    if (st != EC_OK) return st;
    if (T > 0 && (!K_new || !V_new)) return EC_ERR_NULL;
    st = check_budget(c, T, budget, recent, sinks);
    if (st != EC_OK) return st;
    if (!aligned(K_new, 16) || !aligned(V_new, 16) || !aligned(w_new, 4) || !aligned(pos_new, 4) || !aligned(counts, 4))
        return EC_ERR_ALIGN;
    st = check_ws(ws, ws_bytes, ec::paged_append_workspace_bytes(c, T, budget));
    if (st != EC_OK) return st;
    ec::AppendArgs a = append_args(K_new, V_new, w_new, pos_new, counts, T, fresh, budget, recent, sinks);
    return ec::launch_paged_rows(view(c), c->D, nullptr, &a, ws, (cudaStream_t)stream) == cudaSuccess ? EC_OK : EC_ERR_CUDA;
}

size_t ec_paged_step_workspace(const ec_paged *c, int Hq, int budget)
{
    if (check_paged(c) != EC_OK || check_heads(c, Hq) != EC_OK || check_budget(c, 1, budget, 0, 0) != EC_OK) return 0;
    return ec::paged_attention_workspace_bytes(c, Hq, 1) + round256((size_t)c->N * c->H * sizeof(float)) +
           ec::paged_append_workspace_bytes(c, 1, budget);
}

int ec_paged_decode_step(const void *q, const void *k_new, const void *v_new, const ec_paged *c, int Hq, float scale, float decay,
                         int budget, int recent, int sinks, void *out, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    ec::NvtxRange nvtx_range("ec_paged_decode_step");
    int st = check_attention(q, k_new, v_new, c, Hq, scale, 1, decay, out, lse);
    if (st != EC_OK) return st;
    if (!k_new) return EC_ERR_NULL;
    st = check_budget(c, 1, budget, recent, sinks);
    if (st != EC_OK) return st;
    st = check_ws(ws, ws_bytes, ec_paged_step_workspace(c, Hq, budget));
    if (st != EC_OK) return st;
    char *p = static_cast<char *>(ws);
    float *w_new = reinterpret_cast<float *>(p + ec::paged_attention_workspace_bytes(c, Hq, 1));
    void *ws_append = reinterpret_cast<char *>(w_new) + round256((size_t)c->N * c->H * sizeof(float));
    ec::GatherArgs gather;
    cudaError_t e = ec::launch_paged_attention(view(c), c->D, c->dtype, q, k_new, v_new, Hq, scale, 1, decay, out, lse, w_new, ws,
                                               &gather, (cudaStream_t)stream);
    if (e == cudaSuccess) {
        ec::AppendArgs a = append_args(k_new, v_new, w_new, nullptr, nullptr, 1, 0, budget, recent, sinks);
        e = ec::launch_paged_rows(view(c), c->D, &gather, &a, ws_append, (cudaStream_t)stream);
    }
    return e == cudaSuccess ? EC_OK : EC_ERR_CUDA;
}

}  // extern "C"
