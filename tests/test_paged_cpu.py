"""Packed prompts and the paged cache without a GPU: the reference against brute force, the library's refusals, the host's
bookkeeping of pages."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_14051_b200 as P
from oracle import paged as ref
from paper_2504_14051_b200 import binding as C


def test_reference_attention_is_masked_softmax():
    g = torch.Generator().manual_seed(0)
    for m, n in [(1, 1), (1, 7), (5, 5), (4, 11)]:
        q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((m, 6), (n, 6), (n, 6)))
        o, lse, w = ref.attend(q.numpy(), k.numpy(), v.numpy(), 0.3)
        s = 0.3 * q @ k.t()
        s[torch.ones(m, n, dtype=torch.bool).triu(n - m + 1)] = -float("inf")
        np.testing.assert_allclose(o, (s.softmax(-1) @ v).numpy(), rtol=1e-12, atol=1e-13)
        np.testing.assert_allclose(lse, s.logsumexp(-1).numpy(), rtol=1e-12)
        np.testing.assert_allclose(w.sum(1), 1.0, rtol=1e-12)


def test_reference_eviction_keeps_what_is_sheltered():
    mass, pos = [5.0, 0.0, 0.0, 3.0, 1.0, 0.5], [0, 1, 2, 3, 4, 5]
    assert ref.evict(mass, pos, 6, 6, 4, 0, 0) == ([1, 2], [(4, 1), (5, 2)])
    assert ref.evict(mass, pos, 6, 6, 4, 2, 0) == ([2, 5], [(4, 2)])
    assert ref.evict(mass, pos, 6, 6, 4, 2, 2) == ([2, 3], [(4, 2), (5, 3)])
    assert ref.evict(mass, pos, 6, 6, 1, 6, 0) == ([0, 1, 2, 3, 4], [(5, 0)])  # all sheltered: the oldest first
    assert ref.evict(mass, pos, 6, 6, 9, 0, 0) == ([], [])


def params(**kw):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, max_pages=4, total_new=6, max_new=5,
             dtype=torch.bfloat16, scale=0.1)
    a.update(kw)
    return C.make_paged_params(**a)


def test_params_struct_matches_header():
    import os
    import re

    text = open(os.path.join(os.path.dirname(P.__file__), "..", "include", "caote_paged.h")).read()
    body = re.search(r"typedef struct \{(.*?)\} caote_paged_params_t;", text, re.S).group(1)
    assert re.findall(r"^\s*(?:int32_t|float)\s+(\w+);", body, re.M) == [f for f, _ in C.PagedParams._fields_]


@pytest.mark.parametrize("bad", [
    dict(batch=0), dict(n_q_heads=7), dict(n_q_heads=34), dict(head_dim=96), dict(page_size=8), dict(page_size=48), dict(page_size=512),
    dict(n_pages=0), dict(max_pages=0), dict(total_new=0), dict(max_new=0), dict(max_new=7), dict(dtype=5), dict(scale=float("nan")),
    dict(n_pages=1 << 26), dict(n_kv_heads=1 << 17, n_q_heads=1 << 17), dict(total_new=1 << 30, max_new=1)])
def test_workspace_size_refuses(bad):
    assert C.caote_paged_workspace_bytes(params(**bad)) == 0


def test_workspace_for_more_rows_serves_fewer():
    for dtype in (torch.bfloat16, torch.float32):
        for heads in [(4, 2), (28, 4), (64, 8)]:
            last = {}
            for T in [1, 2, 7, 16, 64, 100, 500, 2048, 16384]:
                sizes = {m: C.caote_paged_workspace_bytes(params(n_q_heads=heads[0], n_kv_heads=heads[1], total_new=T, max_new=m, dtype=dtype,
                                                                 batch=64, n_pages=4000, max_pages=512))
                         for m in [1, 2, 5, 16, 33, 512, 16384] if m <= T}
                assert list(sizes.values()) == sorted(sizes.values())
                assert all(sizes[m] >= last[m] for m in last)
                last = sizes


def test_refusals_come_before_any_launch():
    lib, before = P.lib(), C.caote_launch_count()
    fake, odd, ws = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(1 << 20)
    p = params()
    need, bp = C.caote_paged_workspace_bytes(p), ctypes.byref(p)

    def prompt(p=bp, q=fake, qs=0, k=fake, v=fake, ks=0, cu=fake, o=fake, ws=ws, n=need):
        return lib.caote_prompt_attend(p, q, qs, k, v, ks, cu, o, None, None, ws, n, None)

    def attend(p=bp, q=fake, qs=0, K=fake, V=fake, table=fake, lens=fake, cu=fake, o=fake, ws=ws, n=need):
        return lib.caote_paged_attend(p, q, qs, K, V, None, table, lens, cu, o, None, ws, n, None)

    def append(p=bp, K=fake, V=fake, table=fake, lens=fake, k=fake, v=fake, ks=0, cu=fake, ws=ws, n=need):
        return lib.caote_paged_append(p, K, V, None, None, table, lens, None, k, v, ks, None, cu, ws, n, None)

    def evict(p=bp, K=fake, V=fake, mass=fake, pos=fake, table=fake, lens=fake, seen=fake, budget=fake, sinks=0, recent=0, out=fake, most=4,
              count=fake, ws=ws, n=need):
        return lib.caote_paged_evict(p, K, V, mass, pos, table, lens, seen, budget, sinks, recent, out, most, count, ws, n, None)

    for f, names in [(prompt, "p q k v cu o ws"), (attend, "p q K V table lens cu o ws"), (append, "p K V table lens k v cu ws"),
                     (evict, "p K V mass pos table lens seen budget out count ws")]:
        for name in names.split():
            assert f(**{name: None}) == C.ERR_INVALID_ARG, (f, name)
        for bad in (dict(batch=0), dict(n_q_heads=7), dict(max_new=7), dict(scale=float("nan"))):
            assert f(p=ctypes.byref(params(**bad))) == C.ERR_INVALID_ARG
        for bad in (dict(head_dim=96), dict(dtype=3)):
            assert f(p=ctypes.byref(params(**bad))) == C.ERR_UNSUPPORTED
        assert f(ws=ctypes.c_void_p((1 << 20) + 8)) == C.ERR_INVALID_ARG
        assert f(n=255) == C.ERR_INVALID_ARG
    for f in (attend, append, evict):
        for bad in (dict(page_size=0), dict(page_size=24), dict(n_pages=0), dict(max_pages=0)):
            assert f(p=ctypes.byref(params(**bad))) == C.ERR_INVALID_ARG
    for f, names in [(prompt, "q k v o"), (attend, "q K V o"), (append, "K V k v"), (evict, "K V")]:
        for name in names.split():
            assert f(**{name: odd}) == C.ERR_INVALID_ARG, (f, name)
    for f, name, dense in [(prompt, "qs", 1024), (prompt, "ks", 256), (attend, "qs", 1024), (append, "ks", 256)]:
        for stride in (dense - 8, dense + 4, -dense, 1 << 31):
            assert f(**{name: stride}) == C.ERR_INVALID_ARG, (f, name, stride)
    assert attend(n=need - 1) == C.ERR_INVALID_ARG
    assert prompt(n=C.caote_paged_workspace_bytes(params(page_size=0, n_pages=0, max_pages=0)) - 1) == C.ERR_INVALID_ARG
    assert evict(sinks=-1) == evict(recent=-1) == evict(most=0) == C.ERR_INVALID_ARG
    assert C.caote_launch_count() == before


@pytest.mark.skipif(torch.cuda.is_available(), reason="only meaningful on a box without a GPU")
def test_calls_fail_loudly_without_a_gpu():
    p = params()
    need, bp = C.caote_paged_workspace_bytes(p), ctypes.byref(p)
    fake, ws = ctypes.c_void_p(4096), ctypes.c_void_p(1 << 20)
    rc = P.lib().caote_paged_attend(bp, fake, 0, fake, fake, None, fake, fake, fake, fake, None, ws, need, None)
    assert rc in (C.ERR_CUDA, C.ERR_UNSUPPORTED)


def test_the_binding_refuses_what_an_address_does_not_show(monkeypatch):
    """Types, sizes, layouts and devices (here everything is on the CPU, which is made to look like the current device)."""
    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a)) or 0

    monkeypatch.setattr(C, "_fn", Lib())
    monkeypatch.setattr(C, "_stream", lambda s: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    io, p = torch.bfloat16, params()
    z = {"q": torch.zeros(6, 8, 128, dtype=io), "k": torch.zeros(6, 2, 128, dtype=io), "cu": torch.zeros(3, dtype=torch.int32),
         "lse": torch.zeros(6, 8), "mass_new": torch.zeros(6, 2), "ws": torch.zeros(256, dtype=torch.uint8),
         "K": torch.zeros(10, 2, 16, 128, dtype=io), "mass": torch.zeros(10, 2, 16), "pos": torch.zeros(10, 2, 16, dtype=torch.int32),
         "table": torch.zeros(2, 4, dtype=torch.int32), "b": torch.zeros(2, dtype=torch.int32),
         "out": torch.zeros(2, 2, 5, dtype=torch.int32)}
    forms = {
        P.caote_prompt_attend: ["q", "k", "k", "cu", "q", "lse", "mass_new", "ws"],
        P.caote_paged_append: ["K", "K", "mass", "pos", "table", "b", "b", "k", "k", "mass_new", "cu", "ws"],
        P.caote_paged_attend: ["q", "K", "K", "mass", "table", "b", "cu", "q", "lse", "ws"],
        P.caote_paged_evict: ["K", "K", "mass", "pos", "table", "b", "b", "b", 4, 64, "out", "b", "ws"]}
    for f, names in forms.items():
        good = [z.get(x, x) if isinstance(x, str) else x for x in names]
        f(p, *good)
        for i, x in enumerate(good):
            if not isinstance(x, torch.Tensor) or names[i] == "ws":
                continue
            wrong = [x.double(), x[:-1].contiguous(), torch.cat([x, x])]
            if names[i] not in ("q", "k"):
                wrong.append(torch.stack([x, x], -1)[..., 0])
            for bad in wrong if names[i] != "out" else wrong[:1] + wrong[3:]:
                with pytest.raises(ValueError):
                    f(p, *good[:i], bad, *good[i + 1:])
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
        with pytest.raises(ValueError, match="device"):
            f(p, *good)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    assert [n for n, _ in calls] == [f.__name__ for f in forms]
    wide = torch.zeros(6, 12, 128, dtype=io)
    P.caote_prompt_attend(p, wide[:, :8], wide[:, 8:10], wide[:, 10:], z["cu"], z["q"], None, None, z["ws"])
    assert calls[-1][1][2] == calls[-1][1][5] == 12 * 128
    for bad in (z["q"].transpose(0, 1).contiguous().transpose(0, 1), z["q"][:1].expand(6, 8, 128),
                torch.zeros(6, 8, 256, dtype=io)[:, :, ::2], torch.zeros(6, 16, 128, dtype=io)[:, ::2]):
        with pytest.raises(ValueError):
            P.caote_paged_attend(p, bad, z["K"], z["K"], None, z["table"], z["b"], z["cu"], z["q"], None, z["ws"])
    with pytest.raises(ValueError, match="stride"):
        P.caote_prompt_attend(p, z["q"], wide[:, 8:10], z["k"], z["cu"], z["q"], None, None, z["ws"])


def test_page_bookkeeping_on_the_host(monkeypatch):
    """Pages are handed out for the new tokens, come back with the eviction, and never serve two sequences."""
    calls = []
    for name in ("caote_prompt_attend", "caote_paged_append", "caote_paged_attend", "caote_paged_evict"):
        monkeypatch.setattr(C, name, lambda *a, name=name: calls.append(name))
    c = P.PagedCache(3, 4, 2, 64, 16, 12, 128, 100, torch.float32, [20, 33, 7], device="cpu")

    def x(T, h):
        return torch.zeros(T, h, 64)

    def check():
        held = [p for s in c._pages for p in s]
        assert sorted(held + c._free) == list(range(12))
        for b in range(3):
            assert len(c._pages[b]) == -(-c.host_lens[b] // 16)
            assert c.page_table[b, :len(c._pages[b])].tolist() == c._pages[b]

    c.prompt(x(60, 4), x(60, 2), x(60, 2), [50, 0, 10])
    assert c.host_lens == [20, 0, 7] and calls == ["caote_prompt_attend", "caote_paged_append", "caote_paged_evict"]
    check()
    calls.clear()
    c.step(x(3, 4), x(3, 2), x(3, 2), [1, 2, 0])
    assert c.host_lens == [20, 2, 7] and calls == ["caote_paged_append", "caote_paged_attend", "caote_paged_evict"]
    check()
    with pytest.raises(ValueError, match="already holds"):
        c.prompt(x(1, 4), x(1, 2), x(1, 2), [1, 0, 0])
    begin = lambda new: c._begin(new, x(sum(new), 4), x(sum(new), 2), x(sum(new), 2))  # noqa: E731
    begin([100, 0, 0])  # 8 of the 12 pages
    with pytest.raises(ValueError, match="are free"):
        begin([0, 90, 0])
    with pytest.raises(ValueError, match="would need"):
        c.host_lens[2] = 120
        begin([0, 0, 9])
    c.host_lens[2] = 7
    for bad in ((x(2, 4), x(3, 2), x(3, 2)), (x(3, 4), x(3, 4), x(3, 2)), (x(3, 4), x(3, 2), x(3, 2).double())):
        with pytest.raises(ValueError, match="has to be"):
            c.step(*bad, [1, 1, 1])
    check_free = len(c._free)
    with pytest.raises(ValueError):
        c.step(x(1, 4), x(1, 2), x(1, 2), [0, 0, 0])
    with pytest.raises(ValueError):
        c.step(x(1, 4), x(1, 2), x(1, 2), [1, -1, 1])
    assert len(c._free) == check_free
    c.release(0)
    c.release(1)
    c.release(2)
    assert sorted(c._free) == list(range(12)) and c.host_lens == [0, 0, 0]
