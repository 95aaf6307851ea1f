"""Packed prompts and the paged cache on the GPU against the definitions in 64 bits (oracle/paged.py).

Bounds, for a row with weights w over values v, e = 2^-24 the rounding of fp32:
  a logit is off by at most D = scale * max_j sum_c |q_c k_jc| * d * 2e (a sum of d products, each addition losing at most 2e of
  the running value); a weight, relative, by R = 2 D + (n + 4) e + 2^-21 (its logit and the statistic, the sum of n terms, the
  exponential, which is good to 2 ulp = 2^-22, or 2^-21 where it is a polynomial);
  o by sum_j w_j |v_j| (R + n 2e), and with bf16 another 2^-8 of that sum (a weight is rounded to bf16 for the product) and
  2^-8 of |o| (the result is); lse by D + (n + 4) e + 2^-21 + 2e |lse|; a key's mass by its R, and e per added row. A weight below
  2^-126 is below what fp32 holds with all its bits: it may come out as anything between 0 and 2^-126, so a key's mass is off by
  2^-126 per added row besides.
"""
import numpy as np
import pytest
import torch

import paper_2504_14051_b200 as P
from oracle import paged as ref
from paper_2504_14051_b200 import binding as C

pytestmark = pytest.mark.gpu
DEV, E = "cuda", 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


class Pages:
    """A pool with the sequences' K and V rows in it; everything else in the pool is NaN."""

    def __init__(self, lens, Hkv, d, page, dtype, seed=0, spare=3, extra=0, fill=float("nan")):
        g = torch.Generator().manual_seed(seed)
        need = [-(-(n + extra) // page) for n in lens]
        self.page, self.lens, self.n_pages, self.max_pages = page, list(lens), sum(need) + spare, max(max(need), 1) + 1
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32)
        self.K = torch.full((self.n_pages, Hkv, page, d), fill).to(dtype)
        self.V = torch.full((self.n_pages, Hkv, page, d), fill).to(dtype)
        self.mass = torch.full((self.n_pages, Hkv, page), float("nan"))
        at = 0
        for b, n in enumerate(lens):
            self.table[b, :need[b]] = order[at:at + need[b]].int()
            at += need[b]
            pg, row = self.at(b, n)
            self.K[pg, :, row] = torch.randn(n, Hkv, d, generator=g).to(dtype)
            self.V[pg, :, row] = torch.randn(n, Hkv, d, generator=g).to(dtype)
            self.mass[pg, :, row] = torch.rand(n, Hkv, generator=g) * 3
        self.g = g

    def at(self, b, n):
        j = torch.arange(n)
        return self.table[b].long()[j // self.page], j % self.page

    def keys_of(self, b, h):
        pg, row = self.at(b, self.lens[b])
        return f64(self.K[pg, h, row]), f64(self.V[pg, h, row])


def check_rows(q, keys_of, cu, Hkv, scale, o, lse, dtype, got_mass=None, mass0=None):
    """o, lse (or None) of every row, and got_mass(b) [Hkv, n] against mass0(b) + the weights received."""
    q, o = f64(q), f64(o)
    T, Hq, d = q.shape
    G = Hq // Hkv
    for b in range(len(cu) - 1):
        for h in range(Hkv if cu[b + 1] > cu[b] else 0):
            k, v = keys_of(b, h)
            n, m = len(k), cu[b + 1] - cu[b]
            mass, slack = np.zeros(n), np.zeros(n)
            for g in range(h * G, (h + 1) * G):
                rows = slice(cu[b], cu[b + 1])
                ro, rl, w = ref.attend(q[rows, g], k, v, scale)
                D = abs(scale) * (np.abs(q[rows, g]) @ np.abs(k).T).max(1) * d * 2 * E
                R = 2 * D + (n + 4) * E + 2.0 ** -21
                A = w @ np.abs(v)
                tol = A * (R + 2 * n * E)[:, None]
                if dtype == BF:
                    tol += 2.0 ** -8 * (A + np.abs(ro) + tol)
                err = np.abs(o[rows, g] - ro)
                assert (err <= tol).all(), f"o of sequence {b}, head {g}: {(err - tol).max()} over, {err.max()}"
                if lse is not None:
                    err = np.abs(f64(lse)[rows, g] - rl)
                    tol = D + (n + 4) * E + 2.0 ** -21 + 2 * E * np.abs(rl)
                    assert (err <= tol).all(), f"lse of sequence {b}, head {g}: {err.max()}"
                mass += w.sum(0)
                slack += (w * (R + G * m * E)[:, None]).sum(0)
            if got_mass is not None:
                m0 = mass0(b)[h] if mass0 else np.zeros(n)
                err = np.abs(got_mass(b)[h] - (m0 + mass))
                tol = slack + 2 * E * (np.abs(m0) + mass) + G * m * 2.0 ** -126
                assert (err <= tol).all(), f"mass of sequence {b}, head {h}: {(err - tol).max()} over at {np.argmax(err - tol)}"


def starts(new):
    return [0] + list(np.cumsum(new))


HEADS = [(4, 2), (7, 1), (8, 8), (16, 1), (6, 2), (12, 4)]


def prompt_case(lengths, heads, d, dtype, seed=0, fused=False, mass=True, scale=None, want_lse=True):
    Hq, Hkv = heads
    g = torch.Generator().manual_seed(seed)
    T, cu, scale = sum(lengths), starts(lengths), d ** -0.5 if scale is None else scale
    qkv = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(dtype)
    qkv[:, :Hq] += 1.0
    dev = qkv.to(DEV)
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    p = P.make_paged_params(len(lengths), Hq, Hkv, d, 0, 0, 0, T, max(lengths), dtype, scale)
    ws = P.alloc_paged_workspace(p, DEV)
    o = torch.full((T, Hq, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((T, Hq), 7.0, device=DEV) if want_lse else None
    m = torch.full((T, Hkv), 7.0, device=DEV) if mass else None
    P.caote_prompt_attend(p, q, k, v, torch.tensor(cu, dtype=torch.int32, device=DEV), o, lse, m, ws)
    torch.cuda.synchronize()
    assert P.caote_read_status(ws) == 0
    kk, vv = f64(k), f64(v)
    check_rows(q, lambda b, h: (kk[cu[b]:cu[b + 1], h], vv[cu[b]:cu[b + 1], h]), cu, Hkv, scale, o, lse, dtype,
               (lambda b: f64(m)[cu[b]:cu[b + 1]].T) if mass else None)
    return o, lse, m


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", [[1], [1, 1, 1], [129], [0, 5, 0, 64, 1], [300, 17], [127, 128, 2], [257]])
def test_prompt(lengths, d, dtype):
    prompt_case(lengths, (8, 2), d, dtype)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_heads(heads, dtype):
    prompt_case([70, 3, 200], heads, 128 if heads != (7, 1) else 64, dtype, seed=1, fused=True)


@pytest.mark.parametrize("mass,want_lse", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_optional_outputs(mass, want_lse, dtype):
    prompt_case([150, 20], (4, 2), 128, dtype, mass=mass, want_lse=want_lse)


@pytest.mark.parametrize("scale", [0.0, -0.05, 0.4])
def test_prompt_scales(scale):
    prompt_case([140, 20], (4, 2), 64, BF, scale=scale)
    prompt_case([140, 20], (4, 2), 64, F32, scale=scale)


@pytest.mark.parametrize("lengths,heads", [([1100, 300], (4, 1)), ([700, 900, 3], (8, 2)), ([513], (28, 4))])
def test_prompt_longer(lengths, heads):
    prompt_case(lengths, heads, 128, BF, seed=3)


def attend_case(lens, new, heads, d, dtype, page=16, seed=0, mass=True, scale=None, want_lse=True, fused=False):
    Hq, Hkv = heads
    T, cu, scale = sum(new), starts(new), d ** -0.5 if scale is None else scale
    pg = Pages(lens, Hkv, d, page, dtype, seed)
    wide = (torch.randn(T, Hq + (2 * Hkv if fused else 0), d, generator=pg.g) + 0.5).to(dtype).to(DEV)
    q = wide[:, :Hq]
    p = P.make_paged_params(len(lens), Hq, Hkv, d, page, pg.n_pages, pg.max_pages, T, max(new), dtype, scale)
    ws = P.alloc_paged_workspace(p, DEV)
    o = torch.full((T, Hq, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((T, Hq), 7.0, device=DEV) if want_lse else None
    m = pg.mass.to(DEV) if mass else None
    cu_t, lens_t = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (cu, lens))
    P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), m, pg.table.to(DEV), lens_t, cu_t, o, lse, ws)
    torch.cuda.synchronize()
    assert P.caote_read_status(ws) == 0
    active = [b for b in range(len(lens)) if new[b]]
    masses = None
    if mass:
        mc = m.cpu()
        masses = lambda b: f64(mc[pg.at(b, lens[b])[0], :, pg.at(b, lens[b])[1]]).T  # noqa: E731
        # what belongs to no attending sequence is as it was
        rest = torch.ones(m.shape, dtype=torch.bool)
        for b in active:
            rest[pg.at(b, lens[b])[0], :, pg.at(b, lens[b])[1]] = False
        assert torch.equal(mc[rest].view(torch.int32), pg.mass[rest].view(torch.int32))
    check_rows(q, pg.keys_of, cu, Hkv, scale, o, lse, dtype, masses,
               (lambda b: f64(pg.mass[pg.at(b, lens[b])[0], :, pg.at(b, lens[b])[1]]).T) if mass else None)
    return o, lse, m


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_single_tokens(page, d, dtype):
    attend_case([1, 16, 17, 300, 255, 128], [1, 1, 1, 1, 1, 1], (8, 2), d, dtype, page)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_single_token_heads(heads, dtype):
    attend_case([130, 33, 1, 513], [1, 1, 1, 0], heads, 128, dtype, 16, seed=2)


@pytest.mark.parametrize("lens", [[5000], [4097, 1, 2500, 900], [64] * 40])
def test_single_tokens_over_many_splits(lens):
    for dtype in (BF, F32):
        attend_case(lens, [1] * len(lens), (8, 2), 128, dtype, 32, seed=3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("lens,new", [([300, 128, 129], [2, 5, 3]), ([200, 77, 500], [33, 77, 1]), ([700, 40], [300, 0]), ([130], [130])])
def test_blocks(lens, new, page, dtype):
    attend_case(lens, new, (8, 2), 128, dtype, page, seed=4)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_block_heads(heads, dtype):
    attend_case([330, 65], [40, 65], heads, 64, dtype, 32, seed=5, fused=True)


@pytest.mark.parametrize("lens,new,heads", [([3000], [128], (8, 2)), ([2500, 1900, 40], [200, 1, 9], (28, 4)), ([1500], [20], (4, 4))])
def test_blocks_longer(lens, new, heads):
    attend_case(lens, new, heads, 128, BF, 16, seed=6)


@pytest.mark.parametrize("new", [[1, 1], [9, 60]])
@pytest.mark.parametrize("scale", [0.0, -0.05, 0.4])
def test_attend_scales_and_optional_outputs(scale, new):
    for dtype in (BF, F32):
        attend_case([140, 90], new, (4, 2), 64, dtype, scale=scale, mass=scale != 0.4, want_lse=scale == 0.0)


def test_a_row_with_a_far_larger_logit():
    """Sinks: the running maximum jumps by hundreds, early and late."""
    for at in (0, 399):
        for new in (1, 64):
            pg = Pages([400], 1, 128, 16, BF, seed=7)
            page, row = pg.at(0, 400)
            pg.K[page[at], :, row[at]] = 8.0
            q = torch.full((new, 4, 128), 1.0, dtype=BF, device=DEV)
            p = P.make_paged_params(1, 4, 1, 128, 16, pg.n_pages, pg.max_pages, new, new, BF, 1.0)
            ws = P.alloc_paged_workspace(p, DEV)
            o, lse = torch.zeros((new, 4, 128), dtype=BF, device=DEV), torch.zeros((new, 4), device=DEV)
            m = pg.mass.to(DEV)
            P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), m, pg.table.to(DEV), torch.tensor([400], dtype=torch.int32, device=DEV),
                                 torch.tensor([0, new], dtype=torch.int32, device=DEV), o, lse, ws)
            mc = m.cpu()
            check_rows(q, pg.keys_of, [0, new], 1, 1.0, o, lse, BF, lambda b: f64(mc[page, :, row]).T, lambda b: f64(pg.mass[page, :, row]).T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_pages_are_read_by_both(dtype):
    pg = Pages([64, 64], 2, 64, 32, dtype, seed=8)
    pg.table[1, 0] = pg.table[0, 0]
    q = torch.randn(6, 4, 64, generator=pg.g).to(dtype).to(DEV)
    p = P.make_paged_params(2, 4, 2, 64, 32, pg.n_pages, pg.max_pages, 6, 5, dtype, 0.125)
    ws = P.alloc_paged_workspace(p, DEV)
    o = torch.zeros((6, 4, 64), dtype=dtype, device=DEV)
    P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), None, pg.table.to(DEV), torch.tensor([64, 64], dtype=torch.int32, device=DEV),
                         torch.tensor([0, 1, 6], dtype=torch.int32, device=DEV), o, None, ws)
    check_rows(q, pg.keys_of, [0, 1, 6], 2, 0.125, o, None, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_bad_lengths_and_pages_are_reported(dtype, new):
    """A sequence whose numbers do not fit is skipped, the others are right; a page outside the pool is never read."""
    pg = Pages([100, 90, 120], 2, 128, 16, dtype, seed=9)
    T = 3 * new
    q = torch.randn(T, 4, 128, generator=pg.g).to(dtype).to(DEV)
    p = P.make_paged_params(3, 4, 2, 128, 16, pg.n_pages, pg.max_pages, T, new, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K, V, cu = pg.K.to(DEV), pg.V.to(DEV), [0, new, 2 * new, 3 * new]
    cap = pg.max_pages * 16

    def call(lens, cu, table=pg.table, mass=None):
        o = torch.full((T, 4, 128), 7.0, dtype=dtype, device=DEV)
        P.caote_paged_attend(p, q, K, V, mass, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                             torch.tensor(cu, dtype=torch.int32, device=DEV), o, None, ws)
        return o, P.caote_read_status(ws)

    good, st = call([100, 90, 120], cu)
    assert st == 0
    for bad in (new - 1, -5, cap + 1, 1 << 30):
        m = pg.mass.to(DEV)
        o, st = call([100, bad, 120], cu, mass=m)
        assert st == C.ERR_BAD_LENGTH, bad
        assert torch.equal(o[:new], good[:new]) and torch.equal(o[2 * new:], good[2 * new:]) and (o[new:2 * new] == 7.0).all()
        page, row = pg.at(1, 90)
        assert torch.equal(m.cpu()[page, :, row], pg.mass[page, :, row])
    for bad_cu in ([0, new, new - 1, 3 * new], [0, new, 2 * new, T + 1], [-1, new, 2 * new, T]):
        assert call([100, 90, 120], bad_cu)[1] == C.ERR_BAD_LENGTH
    for bad in (-1, pg.n_pages, 1 << 30):
        table = pg.table.clone()
        table[1, 2] = bad
        o, st = call([100, 90, 120], cu, table, mass=pg.mass.to(DEV))
        assert st == C.ERR_BAD_PAGE
        assert torch.equal(o[:new], good[:new]) and torch.equal(o[2 * new:], good[2 * new:])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append(dtype):
    lens, new, page, Hkv, d = [0, 15, 33, 40], [20, 1, 0, 8], 16, 3, 64
    pg = Pages(lens, Hkv, d, page, dtype, seed=10, extra=20)
    T, cu = sum(new), starts(new)
    wide = torch.randn(T, 2 * Hkv + 1, d, generator=pg.g).to(dtype).to(DEV)
    k, v = wide[:, :Hkv], wide[:, Hkv:2 * Hkv]
    mass_new = torch.rand(T, Hkv, generator=pg.g).to(DEV)
    p = P.make_paged_params(4, 6, Hkv, d, page, pg.n_pages, pg.max_pages, T, 20, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    for first in (mass_new, None):
        K, V, mass, table = pg.K.to(DEV), pg.V.to(DEV), pg.mass.to(DEV), pg.table.to(DEV)
        pos = torch.full(mass.shape, -3, dtype=torch.int32, device=DEV)
        lens_t, seen = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, [0, 115, 133, 140]))
        P.caote_paged_append(p, K, V, mass, pos, table, lens_t, seen, k, v, first, torch.tensor(cu, dtype=torch.int32, device=DEV), ws)
        assert P.caote_read_status(ws) == 0
        assert lens_t.tolist() == [20, 16, 33, 48] and seen.tolist() == [20, 116, 133, 148]
        wK, wV, wm, wp = pg.K.clone(), pg.V.clone(), pg.mass.clone(), torch.full(mass.shape, -3, dtype=torch.int32)
        for b in range(4):
            at, row = pg.at(b, lens[b] + new[b])
            at, row, rows = at[lens[b]:], row[lens[b]:], slice(cu[b], cu[b + 1])
            wK[at, :, row], wV[at, :, row] = k[rows].cpu(), v[rows].cpu()
            wm[at, :, row] = first[rows].cpu() if first is not None else 0.0
            wp[at, :, row] = ([0, 115, 133, 140][b] + torch.arange(new[b], dtype=torch.int32))[:, None].expand(-1, Hkv)
        bits = torch.int16 if dtype == BF else torch.int32
        assert torch.equal(K.cpu().view(bits), wK.view(bits)) and torch.equal(V.cpu().view(bits), wV.view(bits))
        assert torch.equal(mass.cpu().view(torch.int32), wm.view(torch.int32)) and torch.equal(pos.cpu(), wp)


def test_append_refuses_on_the_device():
    lens, page = [10, 10, 10], 16
    pg = Pages(lens, 2, 64, page, F32, seed=11, extra=30)
    p = P.make_paged_params(3, 4, 2, 64, page, pg.n_pages, pg.max_pages, 60, 20, F32, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    k = torch.randn(60, 2, 64, device=DEV)

    def call(lens, cu, table):
        K, V, lens_t = pg.K.to(DEV), pg.V.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
        P.caote_paged_append(p, K, V, None, None, table.to(DEV), lens_t, None, k, k, None, torch.tensor(cu, dtype=torch.int32, device=DEV), ws)
        return K.cpu(), lens_t.tolist(), P.caote_read_status(ws)

    cap = pg.max_pages * page
    K, got, st = call([10, cap - 19, 10], [0, 20, 40, 60], pg.table)
    assert st == C.ERR_OVERFLOW and got == [30, cap - 19, 30]
    for cu in ([0, 21, 40, 60], [0, 20, 10, 60], [0, 20, 40, 61], [-1, 20, 40, 60]):
        assert call([10, 10, 10], cu, pg.table)[2] == C.ERR_BAD_LENGTH
    table = pg.table.clone()
    table[1, 1] = pg.n_pages
    K, got, st = call([10, 10, 10], [0, 20, 40, 60], table)
    assert st == C.ERR_BAD_PAGE and got == [30, 10, 30]
    at, row = pg.at(2, 30)
    assert torch.equal(K[at[10:], :, row[10:]], k[40:60].cpu())


def evict_case(lens, budgets, Hkv=2, d=64, page=16, dtype=F32, seed=0, sinks=0, recent=0, mass_of=None, pos_of=None, max_evict=None):
    pg = Pages(lens, Hkv, d, page, dtype, seed)
    B = len(lens)
    pos = torch.full(pg.mass.shape, -3, dtype=torch.int32)
    seen = [n + 5 for n in lens]
    for b, n in enumerate(lens):
        at, row = pg.at(b, n)
        for h in range(Hkv):
            if mass_of:
                pg.mass[at, h, row] = mass_of(torch.rand(n, generator=pg.g))
            pos[at, h, row] = (pos_of(n) if pos_of else torch.randperm(n + 5, generator=pg.g)[:n]).int()
    ks = [max(0, n - max(1, x)) for n, x in zip(lens, budgets)]
    most = max_evict or max(max(ks), 1)
    p = P.make_paged_params(B, 2 * Hkv, Hkv, d, page, pg.n_pages, pg.max_pages, 1, 1, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K, V, m, po, table = (x.to(DEV) for x in (pg.K, pg.V, pg.mass, pos, pg.table))
    lens_t, seen_t, bud = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, seen, budgets))
    out = torch.full((B, Hkv, most), -9, dtype=torch.int32, device=DEV)
    cnt = torch.full((B,), -9, dtype=torch.int32, device=DEV)
    P.caote_paged_evict(p, K, V, m, po, table, lens_t, seen_t, bud, sinks, recent, out, cnt, ws)
    assert P.caote_read_status(ws) == 0
    assert lens_t.tolist() == [n - k for n, k in zip(lens, ks)] and cnt.tolist() == ks
    wK, wV, wm, wp = pg.K.clone(), pg.V.clone(), pg.mass.clone(), pos.clone()
    for b, n in enumerate(lens):
        at, row = pg.at(b, n)
        for h in range(Hkv):
            gone, moves = ref.evict(pg.mass[at, h, row].numpy(), pos[at, h, row].tolist(), n, seen[b], budgets[b], sinks, recent)
            assert out[b, h].tolist() == gone + [-9] * (most - ks[b]), (b, h)
            for x, y in zip((wK, wV, wm, wp), (pg.K, pg.V, pg.mass, pos)):
                for s, t in moves:
                    x[at[t], h, row[t]] = y[at[s], h, row[s]]
    bits = torch.int16 if dtype == BF else torch.int32
    for x, y, t in ((K, wK, bits), (V, wV, bits), (m, wm, torch.int32), (po, wp, torch.int32)):
        assert torch.equal(x.cpu().view(t), y.view(t))


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F32, 128), (BF, 64), (BF, 128)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_evict(page, dtype, d):
    evict_case([300, 17, 1, 0, 64], [260, 17, 1, 5, 3], d=d, page=page, dtype=dtype)


@pytest.mark.parametrize("sinks,recent", [(4, 0), (0, 50), (4, 50), (1000, 0), (0, 1 << 30)])
def test_evict_sheltered(sinks, recent):
    evict_case([300, 120, 57], [299, 60, 56], sinks=sinks, recent=recent)
    evict_case([300, 120, 57], [250, 1, 20], sinks=sinks, recent=recent, pos_of=torch.arange)


@pytest.mark.parametrize("mass_of", [lambda r: r * 0, lambda r: (r * 4).floor(), lambda r: torch.where(r < 0.3, float("inf"), r),
                                     lambda r: torch.where(r < 0.3, float("nan"), r), lambda r: r - 0.5, lambda r: r * 1e-42])
def test_evict_ties_and_odd_weights(mass_of):
    evict_case([400, 33], [399, 32], mass_of=mass_of, sinks=2, recent=5)
    evict_case([400, 33], [150, 2], mass_of=mass_of, sinks=2, recent=5)


@pytest.mark.parametrize("n,budget", [(8193, 8192), (9000, 8000), (9000, 6000), (25000, 24999), (25000, 24000), (25000, 22000)])
def test_evict_long(n, budget):
    evict_case([n], [budget], Hkv=1, page=64, mass_of=lambda r: (r * 3000).floor(), sinks=4, recent=n // 8)


def test_evict_refuses_on_the_device():
    pg = Pages([100, 100, 100], 2, 64, 16, F32, seed=12)
    p = P.make_paged_params(3, 4, 2, 64, 16, pg.n_pages, pg.max_pages, 1, 1, F32, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)

    def call(lens, table, most=50):
        K, m = pg.K.to(DEV), pg.mass.to(DEV)
        pos = torch.zeros(m.shape, dtype=torch.int32, device=DEV)
        lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
        cnt = torch.zeros(3, dtype=torch.int32, device=DEV)
        P.caote_paged_evict(p, K, K.clone(), m, pos, table.to(DEV), lens_t, torch.tensor([100] * 3, dtype=torch.int32, device=DEV),
                            torch.tensor([90, 90, 60], dtype=torch.int32, device=DEV), 0, 0,
                            torch.zeros((3, 2, most), dtype=torch.int32, device=DEV), cnt, ws)
        return lens_t.tolist(), cnt.tolist(), P.caote_read_status(ws)

    assert call([100] * 3, pg.table) == ([90, 90, 60], [10, 10, 40], 0)
    assert call([100] * 3, pg.table, most=39) == ([90, 90, 100], [10, 10, 0], C.ERR_OVERFLOW)
    cap = pg.max_pages * 16
    assert call([100, cap + 1, 100], pg.table) == ([90, cap + 1, 60], [10, 0, 40], C.ERR_BAD_LENGTH)
    for bad in (-1, pg.n_pages):
        table = pg.table.clone()
        table[1, 3] = bad
        assert call([100] * 3, table) == ([90, 100, 60], [10, 0, 40], C.ERR_BAD_PAGE)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_run_of_prompts_blocks_and_single_tokens(dtype):
    """PagedCache through prompts, blocks, single tokens and evictions, against dense per-head lists of tokens in 64 bits."""
    B, Hq, Hkv, d, page, budgets, sinks, recent = 3, 8, 2, 64, 16, [60, 45, 200], 2, 8
    c = P.PagedCache(B, Hq, Hkv, d, page, 60, 400, 300, dtype, budgets, sinks=sinks, recent=recent)
    g = torch.Generator().manual_seed(13)
    keep = [[{"k": [], "v": [], "pos": []} for _ in range(Hkv)] for _ in range(B)]
    seen = [0] * B
    for kind, new in [("prompt", [100, 0, 131]), ("step", [1, 0, 1]), ("prompt", [0, 7, 0]), ("step", [40, 3, 90]), ("step", [1, 1, 1]),
                      ("step", [0, 70, 1]), ("step", [1, 1, 1]), ("step", [17, 1, 1])]:
        T, cu = sum(new), starts(new)
        q, k, v = ((torch.randn(T, h, d, generator=g) + (0.5 if h == Hq else 0)).to(dtype) for h in (Hq, Hkv, Hkv))
        o = getattr(c, kind)(q.to(DEV), k.to(DEV), v.to(DEV), new)
        assert c.status() == 0
        for b in range(B):
            for h in range(Hkv):
                u = keep[b][h]
                u["k"] += list(f64(k[cu[b]:cu[b + 1], h]))
                u["v"] += list(f64(v[cu[b]:cu[b + 1], h]))
                u["pos"] += list(range(seen[b], seen[b] + new[b]))
            seen[b] += new[b]
        check_rows(q, lambda b, h: (np.array(keep[b][h]["k"]), np.array(keep[b][h]["v"])), cu, Hkv, d ** -0.5, o, c.lse[:T], dtype)
        # the evictions themselves are whole numbers from the device's own weights: followed, their order checked elsewhere
        table, lens, pos = c.page_table.cpu().numpy(), c.lens.tolist(), c.pos.cpu().numpy()
        assert lens == c.host_lens == [min(n, x) if n else 0 for n, x in zip([len(keep[b][0]["k"]) for b in range(B)], budgets)]
        for b in range(B):
            for h in range(Hkv):
                u = keep[b][h]
                pg, row = ref.slots(table[b], page, lens[b])
                held = pos[pg, h, row].tolist()
                where = {x: i for i, x in enumerate(u["pos"])}
                assert len(set(held)) == len(held) and set(held) <= set(where)
                if lens[b] < len(u["pos"]):
                    assert set(range(sinks)) <= set(held) and set(range(seen[b] - recent, seen[b])) <= set(held)
                keep[b][h] = {"k": [u["k"][where[x]] for x in held], "v": [u["v"][where[x]] for x in held], "pos": held}
    c.release(1)
    assert c.host_lens[1] == 0 and c.lens.tolist()[1] == 0


@pytest.mark.parametrize("new", [1, 40])
def test_another_stream_and_a_captured_graph(new):
    """The calls go to the stream that they are given; captured and replayed they give what the eager calls give."""
    lens, page, Hkv, d = [200, 77], 16, 2, 128
    pg = Pages(lens, Hkv, d, page, BF, seed=14, extra=200)
    T = 2 * new
    q = torch.randn(T, 4, d, generator=pg.g).to(BF).to(DEV)
    k, v = (torch.randn(T, Hkv, d, generator=pg.g).to(BF).to(DEV) for _ in range(2))
    p = P.make_paged_params(2, 4, Hkv, d, page, pg.n_pages, pg.max_pages, T, new, BF, d ** -0.5)
    cu = torch.tensor([0, new, T], dtype=torch.int32, device=DEV)

    def state():
        mass = torch.nan_to_num(pg.mass, nan=0.25).to(DEV)
        return dict(K=pg.K.to(DEV), V=pg.V.to(DEV), mass=mass, pos=torch.arange(mass.numel(), dtype=torch.int32, device=DEV).view(mass.shape),
                    lens=torch.tensor(lens, dtype=torch.int32, device=DEV), seen=torch.tensor([300, 300], dtype=torch.int32, device=DEV),
                    out=torch.full((2, Hkv, new), -1, dtype=torch.int32, device=DEV), cnt=torch.zeros(2, dtype=torch.int32, device=DEV),
                    o=torch.zeros((T, 4, d), dtype=BF, device=DEV), lse=torch.zeros((T, 4), device=DEV), ws=P.alloc_paged_workspace(p, DEV))

    table, budget = pg.table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)

    def step(s, stream=None):
        P.caote_paged_append(p, s["K"], s["V"], s["mass"], s["pos"], table, s["lens"], s["seen"], k, v, None, cu, s["ws"], stream)
        P.caote_paged_attend(p, q, s["K"], s["V"], s["mass"], table, s["lens"], cu, s["o"], s["lse"], s["ws"], stream)
        P.caote_paged_evict(p, s["K"], s["V"], s["mass"], s["pos"], table, s["lens"], s["seen"], budget, 2, 4, s["out"], s["cnt"], s["ws"], stream)

    eager, other, graphed = state(), state(), state()
    for _ in range(3):
        step(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        step(other, side)
    side.synchronize()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for x in eager:
        if x != "ws":
            a = eager[x].view(torch.int16 if eager[x].dtype == BF else torch.int32)
            for s in (other, graphed):
                assert torch.equal(a, s[x].view(a.dtype)), x
    assert eager["lens"].tolist() == lens and P.caote_read_status(graphed["ws"]) == 0


def test_equal_calls_give_equal_bits():
    a = attend_case([900, 300, 40], [30, 1, 9], (28, 4), 128, BF, 32, seed=15)
    b = attend_case([900, 300, 40], [30, 1, 9], (28, 4), 128, BF, 32, seed=15)
    for x, y in zip(a, b):
        assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))
