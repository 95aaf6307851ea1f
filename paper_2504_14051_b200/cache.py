"""A budgeted KV cache driven through the C ABI: the call a user of the library makes per step.

Holds the caller-owned device buffers (K, V, base, pos, len, scores, ...) and forwards each step to
``caote_step`` (append the new tokens, score, select, compact) or to the whole-step entry point of its variant. No
arithmetic happens here.

method: "caote" (Sec. 3.2 score), "fast" (FastCAOTE, Sec. 3.3), "sum_errors" (the per-row errors added up),
"post_evict" (the "caote" step that also returns the attention output over the retained tokens, Sec. 3.1).

``PagedCache`` is the same for a cache in pages, whose sequences come with prompts and blocks of different lengths and whose
tokens are evicted by the attention weight they have received (H2O, the base score of Sec. 2).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as C


class EvictionCache:
    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, capacity, n_new, dtype, budget,
                 base_mode="last_query", compact_mode="fill", scale: Optional[float] = None,
                 max_evict: Optional[int] = None, device="cuda", method: str = "caote"):
        self.device = torch.device(device)
        scale = head_dim ** -0.5 if scale is None else scale
        self.params = C.make_params(batch, n_q_heads, n_kv_heads, head_dim, capacity, n_new, dtype, scale,
                                    base_mode)
        self.dtype = dtype
        self.compact_mode = C.COMPACT_MODES[compact_mode] if isinstance(compact_mode, str) else compact_mode
        B, Hkv, Hq, d, cap, m = batch, n_kv_heads, n_q_heads, head_dim, capacity, n_new
        dev = self.device
        self.K = torch.zeros((B, Hkv, cap, d), dtype=dtype, device=dev)
        self.V = torch.zeros((B, Hkv, cap, d), dtype=dtype, device=dev)
        self.base = torch.zeros((B, Hkv, cap), dtype=torch.float32, device=dev)
        self.pos = torch.zeros((B, Hkv, cap), dtype=torch.int32, device=dev)
        self.scores = torch.zeros((B, Hkv, cap), dtype=torch.float32, device=dev)
        self.lens = torch.zeros((B,), dtype=torch.int32, device=dev)
        self.n_seen = torch.zeros((B,), dtype=torch.int32, device=dev)
        if isinstance(budget, int):
            budget = torch.full((B,), budget, dtype=torch.int32)
        self.budget = budget.to(device=dev, dtype=torch.int32).contiguous()
        self.max_evict = max_evict if max_evict is not None else max(n_new, 1)
        # what a step hands back (o, evict_idx, n_evict) lives in one buffer, so that a caller who wants it on the
        # host can fetch it with a single copy of `self.results`
        n_o, n_e = B * Hq * m * d, B * Hkv * self.max_evict
        self.results = torch.zeros((n_o + n_e + B,), dtype=torch.float32, device=dev)
        self.o = self.results[:n_o].view(B, Hq, m, d)
        self.evict_idx = self.results[n_o:n_o + n_e].view(torch.int32).view(B, Hkv, self.max_evict)
        self.n_evict = self.results[n_o + n_e:].view(torch.int32)
        self.workspace = C.alloc_workspace(self.params, dev)
        # FastCAOTE (Sec. 3.3) scores against the mean of the cached values: the per-unit sum of V rows is state
        assert method in ("caote", "fast", "sum_errors", "post_evict")
        self.method = method
        self.vsum = torch.zeros((B, Hkv, d), dtype=torch.float32, device=dev) if method == "fast" else None
        self.o_post = torch.zeros_like(self.o) if method == "post_evict" else None

    def load(self, K, V, lens, base=None, pos=None):
        """Install an existing cache state (copied into the owned buffers)."""
        self.K.copy_(K)
        self.V.copy_(V)
        self.lens.copy_(lens)
        self.n_seen.copy_(lens)
        if base is not None:
            self.base.copy_(base)
        if pos is not None:
            self.pos.copy_(pos)
        else:
            cap = self.K.shape[2]
            self.pos.copy_(torch.arange(cap, dtype=torch.int32, device=self.device).expand_as(self.pos))
        if self.vsum is not None:
            C.caote_vsum(self.params, self.V, self.lens, self.vsum)

    def step(self, q, k_new, v_new, stream=None):
        """One eviction step; returns the pre-eviction attention output o [B, Hq, m, d] (method "post_evict":
        the output over the retained tokens)."""
        if self.method == "sum_errors":
            C.caote_step_sum_errors(self.params, q, k_new, v_new, self.K, self.V, self.base, self.pos, self.lens,
                                    self.n_seen, self.budget, self.o, self.scores, self.evict_idx, self.n_evict,
                                    self.compact_mode, self.workspace, stream)
            return self.o
        if self.method == "post_evict":
            C.caote_step_post_evict(self.params, q, k_new, v_new, self.K, self.V, self.base, self.pos, self.lens,
                                    self.n_seen, self.budget, self.o, self.o_post, self.scores, self.evict_idx,
                                    self.n_evict, self.compact_mode, self.workspace, stream)
            return self.o_post
        if self.vsum is not None:
            C.caote_step_fast(self.params, q, k_new, v_new, self.K, self.V, self.base, self.pos, self.lens,
                              self.n_seen, self.budget, self.vsum, self.o, self.scores, self.evict_idx, self.n_evict,
                              self.compact_mode, self.workspace, stream)
            return self.o
        C.caote_step(self.params, q, k_new, v_new, self.K, self.V, self.base, self.pos, self.lens, self.n_seen,
                     self.budget, self.o, self.scores, self.evict_idx, self.n_evict, self.compact_mode,
                     self.workspace, stream)
        return self.o

    def status(self) -> int:
        return C.caote_read_status(self.workspace)


class PagedCache:
    """Sequences in a pool of pages: prompts are attended whole, later tokens in blocks or one at a time, and the lightest
    tokens beyond the budget leave after every call. The host knows every length without asking the device: a call appends
    what it is given and evicts down to the budget.

    A call of `prompt` or `step` takes the new tokens of all sequences packed, q [T, Hq, d], k and v [T, Hkv, d], and how many
    each sequence has (`new`, 0 for none); it returns o [T, Hq, d]. `o` and `lse` of a call are overwritten by the next one. All work
    goes to the current stream. The host's lengths and pages move on with every call, so a captured graph cannot hold one. What is wrong
    with a call's arguments is found before anything of it runs: a refused call may be repeated.
    """

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_tokens, max_total_new, dtype, budget,
                 sinks=4, recent=0, scale: Optional[float] = None, device="cuda"):
        self.device = dev = torch.device(device)
        self.dtype, self.sinks, self.recent = dtype, sinks, recent
        self.page_size, self.n_pages, self.max_pages = page_size, n_pages, -(-max_tokens // page_size)
        self.batch, self.Hq, self.Hkv, self.d = batch, n_q_heads, n_kv_heads, head_dim
        self.scale = head_dim ** -0.5 if scale is None else scale
        if batch * n_kv_heads * -(-self.max_pages * page_size // 16) >= 1 << 31:  # (attention would refuse what append has taken)
            raise ValueError(f"PagedCache: {batch} sequences of up to {self.max_pages * page_size} tokens are more than 2^31 blocks of 16")
        shape = (n_pages, n_kv_heads, page_size)
        self.K = torch.zeros(shape + (head_dim,), dtype=dtype, device=dev)
        self.V = torch.zeros(shape + (head_dim,), dtype=dtype, device=dev)
        self.mass = torch.zeros(shape, dtype=torch.float32, device=dev)
        self.pos = torch.zeros(shape, dtype=torch.int32, device=dev)
        self.page_table = torch.full((batch, self.max_pages), -1, dtype=torch.int32, device=dev)
        self.lens = torch.zeros((batch,), dtype=torch.int32, device=dev)
        self.n_seen = torch.zeros((batch,), dtype=torch.int32, device=dev)
        self.n_evict = torch.zeros((batch,), dtype=torch.int32, device=dev)
        self.budgets = [budget] * batch if isinstance(budget, int) else [int(x) for x in budget]
        if len(self.budgets) != batch or sinks < 0 or recent < 0:
            raise ValueError(f"PagedCache: {batch} budgets, sinks and recent of at least 0 are needed, "
                             f"not {len(self.budgets)}, {sinks} and {recent}")
        self.budget = torch.tensor(self.budgets, dtype=torch.int32, device=dev)
        self.max_total_new = max_total_new
        self.evict_idx = torch.zeros((batch, n_kv_heads, max_total_new), dtype=torch.int32, device=dev)
        self.o = torch.zeros((max_total_new, n_q_heads, head_dim), dtype=dtype, device=dev)
        self.lse = torch.zeros((max_total_new, n_q_heads), dtype=torch.float32, device=dev)
        self.mass_new = torch.zeros((max_total_new, n_kv_heads), dtype=torch.float32, device=dev)
        self.workspace = C.alloc_paged_workspace(self._params(max_total_new, max_total_new), dev)
        self.host_lens = [0] * batch
        self._pages = [[] for _ in range(batch)]
        self._written = [0] * batch  # entries of the device's table that name a page
        self._free = list(range(n_pages - 1, -1, -1))

    def _params(self, total, most):
        return C.make_paged_params(self.batch, self.Hq, self.Hkv, self.d, self.page_size, self.n_pages, self.max_pages, total,
                                   most, self.dtype, self.scale)

    def _begin(self, new, q, k, v):
        """Pages for the new tokens; (lengths, parameters, cu, T). Nothing has changed when it refuses."""
        new = [int(m) for m in new]
        T = sum(new)
        for name, t, heads in (("q", q, self.Hq), ("k", k, self.Hkv), ("v", v, self.Hkv)):
            if t.shape != (T, heads, self.d) or t.dtype is not self.dtype or t.device != self.K.device:
                raise ValueError(f"PagedCache: {name} has to be {(T, heads, self.d)}, {self.dtype} on {self.K.device}, "
                                 f"not {tuple(t.shape)}, {t.dtype} on {t.device}")
        if len(new) != self.batch or min(new) < 0 or not 1 <= T <= self.max_total_new:
            raise ValueError(f"PagedCache: {self.batch} sequences with 1 to {self.max_total_new} new tokens together, not {new}")
        C.check_packed_rows("PagedCache", self.workspace, q, k, v)
        need = [-(-(n + m) // self.page_size) for n, m in zip(self.host_lens, new)]
        if max(need) > self.max_pages:
            raise ValueError(f"PagedCache: a sequence would need {max(need)} pages of at most {self.max_pages}")
        more = [max(0, x - len(p)) for x, p in zip(need, self._pages)]
        if sum(more) > len(self._free):
            raise ValueError(f"PagedCache: {sum(more)} pages are needed, {len(self._free)} are free")
        for b, x in enumerate(more):
            if x:
                self._pages[b] += [self._free.pop() for _ in range(x)]
            held = len(self._pages[b])
            if x or held < self._written[b]:  # (entries of pages that came free go: none may name another sequence's page)
                row = self._pages[b] + [-1] * (self._written[b] - held)
                self.page_table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
                self._written[b] = held
        cu = [0]
        for m in new:
            cu.append(cu[-1] + m)
        return new, self._params(T, max(new)), torch.tensor(cu, dtype=torch.int32).to(self.device), T

    def _end(self, p, new):
        """Eviction down to the budgets; the pages behind the new lengths come free."""
        after = [min(n + m, max(b, 1)) for n, m, b in zip(self.host_lens, new, self.budgets)]
        if any(n + m > a for n, m, a in zip(self.host_lens, new, after)):
            C.caote_paged_evict(p, self.K, self.V, self.mass, self.pos, self.page_table, self.lens, self.n_seen, self.budget,
                                self.sinks, self.recent, self.evict_idx, self.n_evict, self.workspace)
        self.host_lens = after
        for b, n in enumerate(after):
            keep = -(-n // self.page_size)
            self._free += self._pages[b][keep:]
            del self._pages[b][keep:]

    def prompt(self, q, k, v, new):
        """First tokens of sequences that hold none yet: attended among themselves, then put into pages."""
        if any(m and n for m, n in zip(new, self.host_lens)):
            raise ValueError("PagedCache.prompt: a sequence with a prompt already holds tokens")
        new, p, cu, T = self._begin(new, q, k, v)
        o, mass = self.o[:T], self.mass_new[:T]
        C.caote_prompt_attend(p, q, k, v, cu, o, self.lse[:T], mass, self.workspace)
        C.caote_paged_append(p, self.K, self.V, self.mass, self.pos, self.page_table, self.lens, self.n_seen, k, v, mass, cu,
                             self.workspace)
        self._end(p, new)
        return o

    def step(self, q, k, v, new):
        """More tokens of some sequences: into the pages, then attended over everything there."""
        new, p, cu, T = self._begin(new, q, k, v)
        C.caote_paged_append(p, self.K, self.V, self.mass, self.pos, self.page_table, self.lens, self.n_seen, k, v, None, cu,
                             self.workspace)
        o = self.o[:T]
        C.caote_paged_attend(p, q, self.K, self.V, self.mass, self.page_table, self.lens, cu, o, self.lse[:T], self.workspace)
        self._end(p, new)
        return o

    def release(self, b):
        """Sequence b is done: its pages come free and it may start again with a prompt."""
        self._free += self._pages[b]
        self._pages[b] = []
        self.host_lens[b] = 0
        self.lens[b] = 0
        self.n_seen[b] = 0

    def status(self) -> int:
        return C.caote_read_status(self.workspace)
