"""PagedCache without a GPU: a call that is refused has changed nothing, and no entry of the table names a page that its sequence
does not hold. The library is replaced by one that writes down what it was asked for."""
import pytest
import torch

import paper_2504_14051_b200 as P
from paper_2504_14051_b200 import binding as C

Hq, Hkv, D, IO = 4, 2, 64, torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The names of the library's functions that ran. The binding's own checks stay as they are (the CPU is made to look like the
    current device)."""
    made = []

    class Lib:
        def __init__(self, lib):
            self.caote_paged_workspace_bytes = lib.caote_paged_workspace_bytes

        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(C, "_fn", Lib(P.lib()))
    monkeypatch.setattr(C, "_stream", lambda s: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    return made


def cache(**kw):
    a = dict(page_size=16, n_pages=12, max_tokens=128, max_total_new=100, dtype=IO, budget=[20, 33, 7], device="cpu")
    a.update(kw)
    return P.PagedCache(3, Hq, Hkv, D, **a)


def rows(T, heads):
    return torch.zeros(T, heads, D, dtype=IO)


def state(c):
    return (list(c.host_lens), [list(p) for p in c._pages], list(c._free), c.page_table.clone().tolist())


def off_16_bytes(t):
    flat = torch.zeros(t.numel() + 1, dtype=t.dtype)
    return flat[1:].view(t.shape)


LAYOUTS = {
    "heads first, transposed": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1),
    "every other channel": lambda t: t.repeat(1, 1, 2)[:, :, ::2],
    "one row for all": lambda t: t[:1].expand(t.shape),
    "rows that overlap": lambda t: torch.zeros(t.numel(), dtype=t.dtype).as_strided(t.shape, (D, D, 1)),
    "address": off_16_bytes,
    "stride": lambda t: torch.zeros(t.shape[0], t.shape[1] * D + 4, dtype=t.dtype)[:, :-4].view(t.shape[0], t.shape[1], D),
}


@pytest.mark.parametrize("which", ["q", "k", "v", "k and v"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind", ["prompt", "step"])
def test_a_refused_call_has_changed_nothing(calls, kind, layout, which):
    c = cache()
    if kind == "step":
        c.prompt(rows(30, Hq), rows(30, Hkv), rows(30, Hkv), [10, 20, 0])
    calls.clear()
    x = {"q": rows(40, Hq), "k": rows(40, Hkv), "v": rows(40, Hkv)}
    for name in which.split(" and "):
        x[name] = LAYOUTS[layout](x[name])
    before = state(c)
    with pytest.raises(ValueError):
        getattr(c, kind)(**x, new=[17, 20, 3])
    assert calls == [] and state(c) == before
    getattr(c, kind)(*(t.contiguous() if layout != "address" else t.clone() for t in x.values()), [17, 20, 3])  # repeated, in order
    assert "caote_paged_append" in calls and c.host_lens == ([20, 33, 3] if kind == "step" else [17, 20, 3])


def test_what_the_checks_let_through(calls):
    """Slices of one projection's output, single tokens."""
    c = cache()
    wide = torch.zeros(5, Hq + 2 * Hkv, D, dtype=IO)
    for T, new in ((5, [2, 2, 1]), (1, [0, 1, 0])):
        w = wide[:T]
        c.step(w[:, :Hq], w[:, Hq:Hq + Hkv], w[:, Hq + Hkv:], new)
    assert calls == ["caote_paged_append", "caote_paged_attend"] * 2


def test_keys_and_values_of_different_strides_are_refused(calls):
    c = cache()
    with pytest.raises(ValueError, match="same token stride"):
        c.step(rows(3, Hq), rows(3, Hkv), rows(3, 2 * Hkv)[:, :Hkv], [1, 1, 1])
    assert calls == [] and c.host_lens == [0, 0, 0] and len(c._free) == 12


def test_another_device_is_refused(calls):
    c = cache()
    with pytest.raises(ValueError, match="has to be"):
        c.step(rows(3, Hq).to("meta"), rows(3, Hkv), rows(3, Hkv), [1, 1, 1])
    assert calls == []


@pytest.mark.parametrize("bad", [dict(sinks=-1), dict(recent=-1), dict(budget=[20, 33]), dict(budget=[20, 33, 7, 7])])
def test_settings_that_an_eviction_would_refuse(calls, bad):
    """... after the tokens are in the pages."""
    with pytest.raises(ValueError):
        cache(**bad)


def test_more_slots_than_attention_takes(calls):
    """Append takes them: the cache is refused when it is made."""
    with pytest.raises(ValueError, match="blocks of 16"):
        P.PagedCache(1 << 14, Hq, Hkv, D, 256, 1, 1 << 20, 1, IO, 10, device="cpu")


def test_no_entry_names_a_page_of_another_sequence(calls):
    c = cache()
    g = torch.Generator().manual_seed(0)

    def check():
        held = {p: b for b in range(3) for p in c._pages[b]}
        assert sorted(list(held) + c._free) == list(range(12))
        for b, row in enumerate(c.page_table.tolist()):
            assert row[:len(c._pages[b])] == c._pages[b]
            assert all(held.get(p, b) == b for p in row if p >= 0), (b, row)

    c.prompt(rows(100, Hq), rows(100, Hkv), rows(100, Hkv), [60, 30, 10])
    check()
    for i in range(200):
        if i % 20 == 19:
            c.release(i // 20 % 3)
        new = torch.randint(0, 30, (3,), generator=g).tolist()
        T = max(1, sum(new))
        new[0] += T - sum(new)
        c.step(rows(T, Hq), rows(T, Hkv), rows(T, Hkv), new)
        check()
