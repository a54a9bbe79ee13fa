"""Buffer management around the C ABI: owns the device tensors and workspaces of one
workload shape and sequences the three calls. No arithmetic happens here.

    s = ElasticCacheSession(N, H, T, D, keep_ratio=0.5, offset=16, scale=1/sqrt(D))
    s.compress(Q, K, V)                  # importance -> select/merge; cache ready, len = budget
    s.compress_with_attention(Q, K, V, out)   # the same, with the prompt's attention output as a by-product
    s.decode(q_all, k_all, v_all, out)   # [steps, N, H, D] each; fixed-point eviction every step

`compress_host` / `decode_host` take pinned host tensors and include the host<->device
copies (on the current stream), for callers whose data starts on the host.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import binding as ec


class ElasticCacheSession:
    def __init__(self, N: int, H: int, T: int, D: int, keep_ratio: float, offset: int, scale: float,
                 population: int = ec.EC_PER_HEAD, protect_ends: bool = True, extra_rows: int = 0,
                 device: Optional[torch.device] = None):
        self.N, self.H, self.T, self.D = N, H, T, D
        self.scale = float(scale)
        self.offset = int(offset)
        self.population = population
        self.protect_ends = protect_ends
        self.n_keep = ec.ec_keep_count(T, keep_ratio)
        if self.n_keep < 1:
            raise ValueError("invalid prompt length or keep ratio")
        self.cap = self.n_keep + extra_rows
        dev = device or torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
        self.scores = torch.empty((N, H, T), dtype=f32, device=dev)
        self.Kc = torch.empty((N, H, self.cap, D), dtype=bf, device=dev)
        self.Vc = torch.empty_like(self.Kc)
        self.anchor_pos = torch.empty((N, H, self.n_keep), dtype=i32, device=dev)
        self.ws_imp = torch.empty(ec.ec_importance_workspace(N, H, T, D), dtype=torch.uint8, device=dev)
        self.ws_sel = torch.empty(ec.ec_select_merge_workspace(N, H, T, D, self.n_keep, population),
                                  dtype=torch.uint8, device=dev)
        self.cache = ec.ec_cache_init(self.Kc, self.Vc, 0, max(self.n_keep, 2), min(self.offset, max(self.n_keep, 2) - 1))
        self.ws_dec = torch.empty(ec.ec_decode_workspace(self.cache), dtype=torch.uint8, device=dev)
        self._stage = None      # device staging for the *_host calls, allocated on first use
        self._dstage = None
        self._up = None         # side streams of decode_host
        self._down = None

    # ---- device-resident inputs ------------------------------------------------------
    def compress(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor) -> None:
        """Prompt call: importance, anchor selection and merge. Resets the cache to `n_keep` rows."""
        ec.ec_importance(Q, K, self.scores, None, self.scale, self.ws_imp)
        ec.ec_select_merge(K, V, self.scores, self.n_keep, self.population, self.protect_ends,
                           self.Kc, self.Vc, self.anchor_pos, None, self.ws_sel)
        self.cache = ec.ec_cache_init(self.Kc, self.Vc, self.n_keep, max(self.n_keep, 2),
                                      min(self.offset, max(self.n_keep, 2) - 1))

    def compress_with_attention(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, out: torch.Tensor,
                                lse: Optional[torch.Tensor] = None) -> None:
        """compress() for callers that also want the prompt's attention output (the model's own forward
        pass): `out` [N,H,T,D] and optionally `lse` [N,H,T] come from ec_prefill_attention, whose
        normaliser also gives the importance by the column-sum pass alone. Same cache afterwards."""
        ec.ec_prefill_attention(Q, K, V, out, lse, self.scores, self.scale, self.ws_imp)
        ec.ec_select_merge(K, V, self.scores, self.n_keep, self.population, self.protect_ends,
                           self.Kc, self.Vc, self.anchor_pos, None, self.ws_sel)
        self.cache = ec.ec_cache_init(self.Kc, self.Vc, self.n_keep, max(self.n_keep, 2),
                                      min(self.offset, max(self.n_keep, 2) - 1))

    def decode(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor,
               want_slots: bool = False):
        """Generation calls for q, k_new, v_new, out of shape [steps, N, H, D]."""
        return ec.ec_decode_steps(q, k_new, v_new, self.cache, self.scale, out, self.ws_dec, want_slots)

    # ---- a new instruction on top of the current cache ---------------------------------
    def logical_slots(self):
        """Physical slots of the cache rows in queue order (oldest first). Fixed budget: the rows
        before the ring never move; the ring holds the `offset` newest rows, oldest at `ring_head`.
        Retention ratio: the list the library maintains (ec_cache_track_order)."""
        c = self.cache
        if c.policy != 0:
            if not c.queue_slots_host:
                raise ValueError("this retention-ratio cache does not track its queue order")
            return [c.queue_slots_host[j] for j in range(c.len)]
        if c.len < c.budget:
            return list(range(c.len))
        base = c.budget - c.offset
        return list(range(base)) + [base + (c.ring_head + i) % c.offset for i in range(c.offset)]

    def recompress(self, Q_new: torch.Tensor, K_new: torch.Tensor, V_new: torch.Tensor, keep_ratio: float):
        """Encode a new instruction of Tq tokens on top of the cache: importance of the cached rows and
        the new rows under the new tokens' queries, then selection and merge over the concatenation.
        Returns a new session holding the compacted result (this one is left untouched)."""
        N, H, Tq, D = Q_new.shape
        P = self.cache.len
        K_all = torch.empty((N, H, P + Tq, D), dtype=torch.bfloat16, device=self.device)
        V_all = torch.empty_like(K_all)
        ec.ec_cache_concat(self.cache, K_new, V_new, K_all, V_all)
        nxt = ElasticCacheSession(N, H, P + Tq, D, keep_ratio, self.offset, self.scale, self.population,
                                  self.protect_ends, device=self.device)
        ws = torch.empty(ec.ec_importance_workspace(N, H, Tq, D), dtype=torch.uint8, device=self.device)
        ec.ec_importance_prefix(Q_new, K_all, nxt.scores, None, self.scale, ws)
        ec.ec_select_merge(K_all, V_all, nxt.scores, nxt.n_keep, nxt.population, nxt.protect_ends,
                           nxt.Kc, nxt.Vc, nxt.anchor_pos, None, nxt.ws_sel)
        nxt.cache = ec.ec_cache_init(nxt.Kc, nxt.Vc, nxt.n_keep, max(nxt.n_keep, 2),
                                     min(nxt.offset, max(nxt.n_keep, 2) - 1))
        return nxt

    # ---- host-resident inputs --------------------------------------------------------
    def _prompt_staging(self):
        if self._stage is None:
            shp = (self.N, self.H, self.T, self.D)
            self._stage = tuple(torch.empty(shp, dtype=torch.bfloat16, device=self.device) for _ in range(3))
        return self._stage

    def _decode_staging(self, steps: int):
        if self._dstage is None or self._dstage[0].shape[0] < steps:
            shp = (steps, self.N, self.H, self.D)
            self._dstage = tuple(torch.empty(shp, dtype=torch.bfloat16, device=self.device) for _ in range(4))
        return self._dstage

    def compress_host(self, Q_host: torch.Tensor, K_host: torch.Tensor, V_host: torch.Tensor,
                      anchor_pos_host: Optional[torch.Tensor] = None) -> int:
        """compress() from pinned host tensors (ec_compress_host). Returns the bytes copied host->device."""
        Q, K, V = self._prompt_staging()
        ec.ec_compress_host(Q_host, K_host, V_host, Q, K, V, self.scores, self.scale, self.n_keep, self.population,
                            self.protect_ends, self.Kc, self.Vc, self.anchor_pos, anchor_pos_host, self.ws_imp,
                            self.ws_sel)
        self.cache = ec.ec_cache_init(self.Kc, self.Vc, self.n_keep, max(self.n_keep, 2),
                                      min(self.offset, max(self.n_keep, 2) - 1))
        return 3 * Q_host.numel() * Q_host.element_size()

    def decode_host(self, q_host: torch.Tensor, k_host: torch.Tensor, v_host: torch.Tensor,
                    out_host: torch.Tensor, chunk: int = 64):
        """decode() from pinned host tensors [steps, N, H, D] (ec_decode_steps_host); writes out_host.
        Returns (h2d, d2h) bytes. Uploads of later chunks and downloads of finished chunks run on two
        side streams while the current chunk decodes."""
        steps = q_host.shape[0]
        chunk = max(chunk, -(-steps // 31))                 # the native call takes at most 31 chunks
        q, k, v, out = (t[:steps] for t in self._decode_staging(steps))
        if self._up is None:
            self._up, self._down = torch.cuda.Stream(), torch.cuda.Stream()
        ec.ec_decode_steps_host(q_host, k_host, v_host, out_host, q, k, v, out, self.cache, self.scale, self.ws_dec,
                                self._up, self._down, chunk)
        nb = q_host.numel() * q_host.element_size()
        return 3 * nb, nb


class PagedCacheSession:
    """Buffers of a paged cache that stays within `budget` rows per problem and evicts by gathered attention weight.

        s = PagedCacheSession(N, H, D, budget=320, recent=16, sinks=4, scale=1/sqrt(D))
        s.prompt(Q, K, V)                    # importance of the prompt's rows, the best `budget` of them into the pages
        s.append(K, V, scores, fresh=True)   # the same with scores from elsewhere (grouped heads, ragged prompts)
        s.decode(q, k_new, v_new, out)       # one token per problem: [N, Hq, D], [N, H, D], [N, H, D] -> [N, Hq, D]

    Every problem owns the pages of its `budget` rows. A problem whose entry of `lens` is negative is an empty place of
    the batch. While the others run on:

        s.end(n)                             # the sequence of place n is over: nothing of it is read or written any more
        s.begin(n)                           # another one begins there, at position 0
        s.append(K, V, scores, counts)       # its prompt: counts [N] is 0 for every other place (prompt() and fresh=True
                                             # begin all of them anew)
    """

    def __init__(self, N: int, H: int, D: int, budget: int, recent: int, sinks: int, scale: float, Hq: Optional[int] = None,
                 page_size: int = 64, dtype: torch.dtype = torch.bfloat16, decay: float = 1.0,
                 device: Optional[torch.device] = None):
        self.N, self.H, self.D, self.Hq = N, H, D, Hq or H
        self.budget, self.recent, self.sinks = int(budget), int(recent), int(sinks)
        self.scale, self.decay = float(scale), float(decay)
        dev = device or torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        pages = -(-self.budget // page_size)
        self.Kp = torch.empty((N * pages, H, page_size, D), dtype=dtype, device=dev)
        self.Vp = torch.empty_like(self.Kp)
        self.weight = torch.zeros((N * pages, H, page_size), dtype=torch.float32, device=dev)
        self.pos = torch.full((N * pages, H, page_size), -1, dtype=torch.int32, device=dev)
        self.table = torch.arange(N * pages, dtype=torch.int32, device=dev).view(N, pages)
        self.lens = torch.zeros(N, dtype=torch.int32, device=dev)
        self.seen = torch.zeros(N, dtype=torch.int32, device=dev)
        self.state = torch.empty(ec.ec_paged_state_bytes(N), dtype=torch.uint8, device=dev)
        self.cache = ec.ec_paged_init(self.Kp, self.Vp, self.weight, self.pos, self.table, self.lens, self.seen, self.state)
        self.ws_step = torch.empty(ec.ec_paged_step_workspace(self.cache, self.Hq, self.budget), dtype=torch.uint8, device=dev)

    def _place(self, t: torch.Tensor, n: int) -> torch.Tensor:
        if not isinstance(n, int) or isinstance(n, bool) or not 0 <= n < self.N:
            raise ValueError(f"a place is a whole number from 0 to {self.N - 1}, got {n!r}")
        return t[n:n + 1]                        # filled by a kernel: an assignment would copy from the host

    def begin(self, n: int) -> None:
        """A sequence begins in place n, without rows and at position 0, whatever was there. In stream order; can be captured."""
        self._place(self.lens, n).zero_()
        self._place(self.seen, n).zero_()

    def end(self, n: int) -> None:
        """Place n is empty from here on. In stream order; can be captured."""
        self._place(self.lens, n).fill_(-1)

    def _scratch(self, size: int) -> torch.Tensor:
        # from the current stream's allocator with every call: a captured prompt keeps its own
        return torch.empty(size, dtype=torch.uint8, device=self.device)

    def append(self, K: torch.Tensor, V: torch.Tensor, scores: Optional[torch.Tensor], counts: Optional[torch.Tensor] = None,
               fresh: bool = False) -> None:
        """Rows [N,H,T,D] with their weights [N,H,T] join the cache; counts [N] when they are not T for every problem."""
        T = K.shape[2]
        ws = self._scratch(ec.ec_paged_append_workspace(self.cache, T, self.budget))
        ec.ec_paged_append(K, V, scores, None, counts, self.cache, fresh, self.budget, self.recent, self.sinks, ws)

    def prompt(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None) -> None:
        """Prompts of T tokens, [N,H,T,D] each (one query head per key head): their rows enter with the importance of
        Eq. 1 as weight; it is left in `scores` (fp32 [N,H,T]) when given. With `out` the prompt's attention output comes from the same call (ec_prefill_attention)."""
        if self.Hq != self.H:
            raise ValueError("grouped query heads: pass the rows' weights to append()")
        if self.Kp.dtype != torch.bfloat16 or K.dim() != 4:
            raise ValueError("the importance of a prompt is computed in bf16, from Q, K and V [N, H, T, D]")
        N, H, T, D = self.N, self.H, K.shape[2], self.D
        ec.check_paged_args(self.cache, (N, H, T, D), Q=Q, K=K, V=V, out=out)
        ec.check_paged_args(self.cache, (N, H, T), torch.float32, lse=lse, scores=scores)
        ws_imp = self._scratch(ec.ec_importance_workspace(N, H, T, D))
        ws_app = self._scratch(ec.ec_paged_append_workspace(self.cache, T, self.budget))
        if scores is None:
            scores = torch.empty((N, H, T), dtype=torch.float32, device=self.device)
        if out is None:
            ec.ec_importance(Q, K, scores, lse, self.scale, ws_imp)
        else:
            ec.ec_prefill_attention(Q, K, V, out, lse, scores, self.scale, ws_imp)
        ec.ec_paged_append(K, V, scores, None, None, self.cache, True, self.budget, self.recent, self.sinks, ws_app)

    def decode(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor,
               lse: Optional[torch.Tensor] = None) -> None:
        """One generation step. May be captured into a CUDA graph and replayed with new values in the same tensors."""
        ec.ec_paged_decode_step(q, k_new, v_new, self.cache, self.scale, self.decay, self.budget, self.recent, self.sinks, out,
                                lse, self.ws_step)

    def status(self) -> int:
        """Synchronises; EC_OK, or EC_ERR_PAGE once a length or a table entry was out of range."""
        return ec.ec_device_status(self.state)


class PagedPoolSession(PagedCacheSession):
    """A paged cache whose problems share one pool of pages and take several new tokens at once.

        s = PagedPoolSession(N, H, D, budget=2048, recent=64, sinks=4, scale=1/sqrt(D), pool_rows=N * 1024, chunk=512)
        s.chunk(q, k, v, counts, out)        # packed tokens [tokens, Hq or H, D] of all problems, counts int32 [N]: a piece of a
                                             # prompt, a whole prompt, drafted tokens; positions follow on, rotary included
        s.decode(q, k_new, v_new, out)       # one token per problem, as before (q and k_new turned by the caller: s.turn)

    A chunk takes pages for its rows from the pool, attends, leaves its attention as weights and evicts down to `budget` rows
    per problem; the pages that eviction or s.end(n) left behind go back with the next call. Where the pool holds too few, problems are
    refused in the order of their numbers: `granted` [N] is 0 for them, nothing of them changes and their part of `out` stays as it
    was. rot elements of every head turn (0: none) by frequencies of ec_rotary_frequencies.
    """

    def __init__(self, N: int, H: int, D: int, budget: int, recent: int, sinks: int, scale: float, pool_rows: int, chunk: int,
                 Hq: Optional[int] = None, page_size: int = 64, dtype: torch.dtype = torch.bfloat16, decay: float = 1.0, rot: int = 0,
                 interleaved: bool = False, freqs: Optional[torch.Tensor] = None, factor: float = 1.0,
                 device: Optional[torch.device] = None):
        self.N, self.H, self.D, self.Hq = N, H, D, Hq or H
        self.budget, self.recent, self.sinks = int(budget), int(recent), int(sinks)
        self.scale, self.decay, self.rot, self.factor = float(scale), float(decay), int(rot), float(factor)
        # what one of a chunk's calls would refuse is refused here: by then the rows have joined
        if min(N, H, self.budget, int(pool_rows), int(chunk), int(page_size)) < 1 or N > 65536:
            raise ValueError(f"N (up to 65536), H, budget, pool_rows, chunk and page_size must be positive, got {N}, {H}, {budget}, {pool_rows}, "
                             f"{chunk}, {page_size}")
        if self.Hq < 1 or self.Hq % H or self.Hq // H > 128 or self.Hq + H > 65536:
            raise ValueError(f"Hq must be a multiple of H = {H}, 128 times it at most, and the heads together 65536 at most, got {self.Hq}")
        if min(self.recent, self.sinks) < 0 or self.recent + self.sinks > self.budget:
            raise ValueError(f"recent and sinks must not be negative nor exceed the budget of {budget} together, got {recent} and {sinks}")
        # the calls take fp32, where a small number may be none and a large one infinite
        scale32, decay32, factor32 = (torch.tensor(x, dtype=torch.float64).float().item() for x in (self.scale, self.decay, self.factor))
        if not 0.0 < scale32 < 1e38 or not 0.0 < decay32 <= 1.0 or self.decay > 1.0:
            raise ValueError(f"scale must be positive and decay in (0, 1], got {scale} and {decay}")
        if not math.isfinite(factor32):
            raise ValueError(f"factor must be finite, got {factor}")
        if not 0 <= rot <= D or rot % (8 if interleaved else 16) or (rot and (freqs is None or tuple(freqs.shape) != (rot // 2,))):
            raise ValueError(f"rot = {rot} must be a multiple of 16 (interleaved: of 8) up to {D}, with {rot // 2} frequencies")
        dev = device or torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        n_pages, max_pages = -(-int(pool_rows) // page_size), -(-(self.budget + int(chunk)) // page_size)
        i32 = dict(dtype=torch.int32, device=dev)
        self.Kp = torch.empty((n_pages, H, page_size, D), dtype=dtype, device=dev)
        self.Vp = torch.empty_like(self.Kp)
        self.weight = torch.zeros((n_pages, H, page_size), dtype=torch.float32, device=dev)
        self.pos = torch.full((n_pages, H, page_size), -1, **i32)
        self.table = torch.full((N, max_pages), -1, **i32)
        self.lens, self.seen = torch.zeros(N, **i32), torch.zeros(N, **i32)
        self.state = torch.empty(ec.ec_paged_state_bytes(N), dtype=torch.uint8, device=dev)
        self.cache = ec.ec_paged_init(self.Kp, self.Vp, self.weight, self.pos, self.table, self.lens, self.seen, self.state)
        self.pages = ec.ec_pages(torch.arange(n_pages, **i32).flip(0).contiguous(), torch.full((1,), n_pages, **i32), torch.zeros(N, **i32))
        self.granted, self.starts = torch.zeros(N, **i32), torch.zeros(N + 1, **i32)
        self.interleaved = bool(interleaved)
        self.freqs = freqs.to(device=dev, dtype=torch.float64).contiguous() if self.rot else None
        sizes = (ec.ec_paged_step_workspace(self.cache, self.Hq, self.budget), ec.ec_paged_chunk_workspace(self.cache, self.Hq),
                 ec.ec_paged_append_workspace(self.cache, 0, self.budget))
        if 0 in sizes:
            raise ValueError("a step, a chunk or an eviction of these sizes would be refused")
        self.ws_step = torch.empty(sizes[0], dtype=torch.uint8, device=dev)

    def turn(self, x: torch.Tensor, out: torch.Tensor) -> None:
        """Rotary positions of the problems' next tokens on x [N, heads, D], for decode()."""
        ec.ec_rotary(x[:, None], out[:, None], self.seen.clamp(min=0)[:, None], self.freqs, self.rot, self.interleaved, self.factor)

    def chunk(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, counts: torch.Tensor, out: torch.Tensor,
              lse: Optional[torch.Tensor] = None) -> None:
        """counts[n] tokens of every problem, packed in order of the problems. Can be captured and replayed with other counts."""
        ec.check_chunk_args(self.cache, self.Hq, counts, lse, q, k, v, out)      # once the rows have joined it is too late
        tokens = q.shape[0]
        i32 = dict(dtype=torch.int32, device=self.device)
        slots, positions = torch.empty(tokens, **i32), torch.empty(tokens, **i32)
        turned = torch.empty((tokens, self.Hq, self.D), dtype=self.Kp.dtype, device=self.device)
        if lse is None:
            lse = torch.empty((tokens, self.Hq), dtype=torch.float32, device=self.device)
        ws = self._scratch(ec.ec_paged_chunk_workspace(self.cache, self.Hq))
        ws_app = self._scratch(ec.ec_paged_append_workspace(self.cache, 0, self.budget))
        ec.ec_paged_release(self.cache, self.pages)
        ec.ec_paged_reserve(self.cache, self.pages, counts, self.starts, self.granted, slots, positions)
        ec.ec_paged_join(q, turned, k, v, None, slots, positions, self.cache, self.freqs, self.rot, self.interleaved, self.factor)
        ec.ec_paged_chunk_attention(turned, self.starts, self.granted, self.cache, self.scale, out, lse, ws)
        ec.ec_paged_chunk_weights(turned, lse, self.starts, self.granted, self.cache, self.scale, self.decay, ws)
        ec.ec_paged_append(None, None, None, None, None, self.cache, False, self.budget, self.recent, self.sinks, ws_app)

    def _rows_for(self, counts: torch.Tensor) -> torch.Tensor:
        """Pages for rows that the next call adds; returns the lengths, with problems that got none marked as empty places."""
        ec.ec_paged_release(self.cache, self.pages)
        ec.ec_paged_reserve(self.cache, self.pages, counts, None, self.granted, advance=False, limit=self.budget)
        kept = self.lens.clone()
        self.lens.masked_fill_((self.granted == 0) & (counts > 0), -1)
        return kept

    def append(self, K: torch.Tensor, V: torch.Tensor, scores: Optional[torch.Tensor], counts: Optional[torch.Tensor] = None,
               fresh: bool = False) -> None:
        if fresh:
            raise ValueError("problems begin with begin(n)")
        if counts is None:
            counts = torch.full((self.N,), K.shape[2], dtype=torch.int32, device=self.device)
        kept = self._rows_for(counts)
        try:
            super().append(K, V, scores, counts)
        finally:
            self.lens.copy_(torch.where((self.granted == 0) & (counts > 0), kept, self.lens))

    def prompt(self, *args, **kwargs) -> None:
        raise ValueError("a prompt is a chunk here: chunk()")

    def decode(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor,
               lse: Optional[torch.Tensor] = None) -> None:
        """One generation step. Problems that get no page are left out: `granted` is 0, their output zero."""
        ones = torch.ones(self.N, dtype=torch.int32, device=self.device)
        kept = self._rows_for(ones)
        try:
            super().decode(q, k_new, v_new, out, lse)
        finally:
            self.lens.copy_(torch.where(self.granted == 0, kept, self.lens))
