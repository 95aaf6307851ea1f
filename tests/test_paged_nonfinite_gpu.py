"""Infinities, NaN and very large values in attention over prompts and pages: a row that sees a NaN or a logit of +inf is NaN, with its
log-sum-exp and the weights it gives; a logit of -inf is a weight of 0; everything else is what the definition gives in 64 bits. Whichever
kernel a call takes, whichever slot the value is in.

Bounds as in test_paged_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2504_14051_b200 as P
from oracle import paged as ref
from test_paged_gpu import BF, DEV, E, F32, Pages, f64, starts

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def check(q, keys_of, cu, Hkv, scale, o, lse, mass, dtype, mass0=None):
    """o [T, Hq, d], lse [T, Hq] and mass(b) [Hkv, n] against the definition; where that is NaN they have to be."""
    q, o, lse = f64(q), f64(o), f64(lse)
    d, G = q.shape[2], q.shape[1] // Hkv
    for b in range(len(cu) - 1):
        rows = slice(cu[b], cu[b + 1])
        m = cu[b + 1] - cu[b]
        for h in range(Hkv if m else 0):
            k, v = keys_of(b, h)
            n = len(k)
            want, slack = np.zeros(n), np.zeros(n)
            finite = np.where(np.isfinite(k), k, 0.0)
            for g in range(h * G, (h + 1) * G):
                with np.errstate(all="ignore"):
                    ro, rl, w = ref.attend(q[rows, g], k, v, scale)
                lost = np.isnan(rl)
                assert (np.isnan(o[rows, g]).all(1) == lost).all() and (np.isnan(o[rows, g]).any(1) == lost).all(), f"o, {b}, {g}"
                assert (np.isnan(lse[rows, g]) == lost).all(), f"lse of sequence {b}, head {g}: {lse[rows, g][lost]}"
                see = ~lost
                qq = np.where(np.isfinite(q[rows, g]), q[rows, g], 0.0)
                D = abs(scale) * (np.abs(qq) @ np.abs(finite).T).max(1) * d * 2 * E
                R = 2 * D + (n + 4) * E + 2.0 ** -21
                A = w @ np.abs(v)
                tol = A * (R + 2 * n * E)[:, None]
                if dtype == BF:
                    tol += 2.0 ** -8 * (A + np.abs(ro) + tol)
                assert (np.abs(o[rows, g] - ro)[see] <= tol[see]).all(), f"o of sequence {b}, head {g}"
                err = np.abs(lse[rows, g] - rl)
                assert (err <= D + (n + 4) * E + 2.0 ** -21 + 2 * E * np.abs(rl))[see].all(), f"lse of sequence {b}, head {g}"
                want += w.sum(0)
                slack += (np.where(see[:, None], w, 0.0) * (R + G * m * E)[:, None]).sum(0)
            if mass is None:
                continue
            m0 = mass0(b)[h] if mass0 else np.zeros(n)
            got, lost = mass(b)[h], np.isnan(want)
            assert (np.isnan(got) == lost).all(), f"mass of sequence {b}, head {h}: NaN at {np.nonzero(np.isnan(got) != lost)[0][:9]}"
            err, tol = np.abs(got - (m0 + want)), slack + 2 * E * (np.abs(m0) + want) + G * m * 2.0 ** -126
            assert (err <= tol)[~lost].all(), f"mass of sequence {b}, head {h}"


def prompt(q, k, v, lengths, dtype, scale):
    T, Hq, d = q.shape
    Hkv, cu = k.shape[1], starts(lengths)
    p = P.make_paged_params(len(lengths), Hq, Hkv, d, 0, 0, 0, T, max(lengths), dtype, scale)
    ws = P.alloc_paged_workspace(p, DEV)
    o, lse, m = (torch.full(s, 7.0, dtype=t, device=DEV) for s, t in (((T, Hq, d), dtype), ((T, Hq), F32), ((T, Hkv), F32)))
    P.caote_prompt_attend(p, q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(cu, dtype=torch.int32, device=DEV), o, lse, m, ws)
    assert P.caote_read_status(ws) == 0
    kk, vv, mm = f64(k), f64(v), f64(m)
    check(q, lambda b, h: (kk[cu[b]:cu[b + 1], h], vv[cu[b]:cu[b + 1], h]), cu, Hkv, scale, o, lse, lambda b: mm[cu[b]:cu[b + 1]].T, dtype)
    return o, lse, m


def attend(pg, q, new, dtype, scale):
    T, Hq, d = q.shape
    Hkv, cu, B = pg.K.shape[1], starts(new), len(new)
    p = P.make_paged_params(B, Hq, Hkv, d, pg.page, pg.n_pages, pg.max_pages, T, max(new), dtype, scale)
    ws = P.alloc_paged_workspace(p, DEV)
    K, V, table = pg.K.to(DEV), pg.V.to(DEV), pg.table.to(DEV)
    lens, cu_t = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (pg.lens, cu))
    outs = []
    for m in (pg.mass.to(DEV), None):
        o, lse = torch.full((T, Hq, d), 7.0, dtype=dtype, device=DEV), torch.full((T, Hq), 7.0, device=DEV)
        P.caote_paged_attend(p, q.to(DEV), K, V, m, table, lens, cu_t, o, lse, ws)
        assert P.caote_read_status(ws) == 0
        mc = None if m is None else m.cpu()
        mass = None if m is None else lambda b: f64(mc[pg.at(b, pg.lens[b])[0], :, pg.at(b, pg.lens[b])[1]]).T  # noqa: B023,E731
        check(q, pg.keys_of, cu, Hkv, scale, o, lse, mass, dtype,
              lambda b: f64(pg.mass[pg.at(b, pg.lens[b])[0], :, pg.at(b, pg.lens[b])[1]]).T)
        outs.append((o, lse, m))
    return outs


KEYS = {"nan": NAN, "+inf": INF, "-inf": -INF}
FORMS = [(BF, 128), (BF, 64), (F32, 64)]


def poison(x, value):
    """A row whose product with rows of positive first channels is `value`."""
    if np.isnan(value):
        x[:] = value
    else:
        x[..., 0] = value


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("value", KEYS)
def test_a_key_of_a_prompt(value, dtype, d):
    """In each slot of eight; the other KV head and the other prompt do not see it."""
    g = torch.Generator().manual_seed(1)
    for at in (0, 31, *range(136, 144), 299):
        q, k, v = (torch.randn(350, h, d, generator=g) for h in (4, 2, 2))
        q[..., 0] = q[..., 0].abs() + 0.1
        poison(k[at, 1], KEYS[value])
        if value == "-inf" and at == 0:
            continue  # (the first row would see nothing else)
        prompt(q.to(dtype), k.to(dtype), v.to(dtype), [300, 50], dtype, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", KEYS)
@pytest.mark.parametrize("at", [5, 390, 600, 1031, 1098])
def test_a_key_of_a_prompt_whose_keys_are_split(at, value, d):
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(1100, h, d, generator=g) for h in (2, 1, 1))
    q[..., 0] = q[..., 0].abs() + 0.1
    poison(k[at, 0], KEYS[value])
    prompt(q.to(BF), k.to(BF), v.to(BF), [1100], BF, d ** -0.5)


@pytest.mark.parametrize("dtype,d", FORMS)
def test_a_query_of_a_prompt(dtype, d):
    """One head of one token: the keys behind it have nothing of it."""
    g = torch.Generator().manual_seed(3)
    for at in (*range(8), 131, 270):
        q, k, v = (torch.randn(300, h, d, generator=g) for h in (2, 2, 2))
        q[at, 1] = NAN
        prompt(q.to(dtype), k.to(dtype), v.to(dtype), [300], dtype, d ** -0.5)


def key_in_the_pages(lens, new, value, dtype, d):
    for at in (0, 6, 127, lens[0] - new[0] - 1, lens[0] - 1):
        pg = Pages(lens, 2, d, 16, dtype, seed=at)
        page, row = pg.at(0, lens[0])
        x = pg.K[page[at], 1, row[at]]
        poison(x, value)
        pg.K[page[at], 1, row[at]] = x
        q = torch.randn(sum(new), 4, d, generator=pg.g)
        q[..., 0] = q[..., 0].abs() + 0.1
        attend(pg, q.to(dtype), new, dtype, d ** -0.5)


def query_over_the_pages(lens, new, dtype, d):
    """The new tokens behind it are not seen by it and have nothing of it."""
    for at in range(min(new[0], 8)):
        pg = Pages(lens, 2, d, 32, dtype, seed=at)
        q = torch.randn(sum(new), 4, d, generator=pg.g)
        q[at, 3] = NAN
        attend(pg, q.to(dtype), new, dtype, d ** -0.5)


BLOCKS = [([700, 90], [40, 9]), ([3000, 100], [70, 1])]


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("value", KEYS)
@pytest.mark.parametrize("lens,new", BLOCKS)
def test_a_key_in_the_pages(lens, new, value, dtype, d):
    key_in_the_pages(lens, new, KEYS[value], dtype, d)


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("lens,new", BLOCKS)
def test_a_query_over_the_pages(lens, new, dtype, d):
    query_over_the_pages(lens, new, dtype, d)


FEW = [([700, 90], [1, 1]), ([700, 90], [3, 2]), ([3000], [1]), ([1200], [8])]


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("value", KEYS)
@pytest.mark.parametrize("lens,new", FEW)
def test_a_key_in_the_pages_of_few_rows(lens, new, value, dtype, d):
    key_in_the_pages(lens, new, KEYS[value], dtype, d)


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("lens,new", FEW)
def test_a_query_of_few_rows(lens, new, dtype, d):
    query_over_the_pages(lens, new, dtype, d)


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("n,m", [(300, 1), (3000, 1), (300, 300), (3000, 70)])
def test_logits_of_minus_infinity_alone(n, m, dtype, d):
    """A softmax over nothing but -inf is no number (nor is one over NaN: the second head, 0 times an infinity)."""
    pg = Pages([n], 1, d, 16, dtype, seed=4)
    pg.K[:, :, :, 0] = -INF
    q = torch.randn(m, 2, d, generator=pg.g)
    q[:, 0, 0], q[:, 1, 0] = 1.0, 0.0
    q[:, 1] = 0.0
    o, lse = torch.zeros((m, 2, d), dtype=dtype, device=DEV), torch.zeros((m, 2), device=DEV)
    p = P.make_paged_params(1, 2, 1, d, 16, pg.n_pages, pg.max_pages, m, m, dtype, 0.1)
    P.caote_paged_attend(p, q.to(dtype).to(DEV), pg.K.to(DEV), pg.V.to(DEV), None, pg.table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV),
                         torch.tensor([0, m], dtype=torch.int32, device=DEV), o, lse, P.alloc_paged_workspace(p, DEV))
    assert torch.isnan(o).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [40, 70, 110, 130, 200, 250])
def test_large_values_behind_rising_logits(at, d):
    """Numerators are formed against a reference that may lag: values of up to 2^80 times these are still in range."""
    g = torch.Generator().manual_seed(5)
    T = 300
    q = torch.ones(T, 4, d).to(BF)
    k, v = (0.05 * torch.randn(T, 2, d, generator=g)).to(BF), (2.0 ** 80 * (torch.rand(T, 2, d, generator=g) * 2 - 1)).to(BF)
    for rise in (10.0, 14.5, 20.0, 40.0, 60.0):  # (nats)
        x = k.clone()
        x[at] = rise / d
        x[at + 20] = 1.4 * rise / d
        prompt(q, x, v, [T], BF, 1.0)


@pytest.mark.parametrize("dtype,d", FORMS)
def test_large_values_of_tokens_that_a_row_does_not_see(dtype, d):
    """A masked weight is exactly 0."""
    g = torch.Generator().manual_seed(6)
    T, at = 300, 200
    q, k, v = (torch.randn(T, h, d, generator=g) for h in (4, 2, 2))
    v[at:] *= 2.0 ** 120
    prompt(q[:at].to(dtype), k[:at].to(dtype), v[:at].to(dtype), [at], dtype, d ** -0.5)
    p = P.make_paged_params(1, 4, 2, d, 0, 0, 0, T, T, dtype, d ** -0.5)
    o = torch.zeros((T, 4, d), dtype=dtype, device=DEV)
    P.caote_prompt_attend(p, q.to(dtype).to(DEV), k.to(dtype).to(DEV), v.to(dtype).to(DEV), torch.tensor([0, T], dtype=torch.int32, device=DEV), o,
                          None, None, P.alloc_paged_workspace(p, DEV))
    qq, kk, vv = (f64(x[:at].to(dtype)) for x in (q, k, v))
    for hq in range(4):
        ro, _, w = ref.attend(qq[:, hq], kk[:, hq // 2], vv[:, hq // 2], d ** -0.5)
        D = d ** -0.5 * (np.abs(qq[:, hq]) @ np.abs(kk[:, hq // 2]).T).max(1) * d * 2 * E
        A = w @ np.abs(vv[:, hq // 2])
        tol = A * (2 * D + (at + 4) * E + 2.0 ** -21 + 2 * T * E)[:, None]
        if dtype == BF:
            tol += 2.0 ** -8 * (A + np.abs(ro) + tol)
        assert (np.abs(f64(o)[:at, hq] - ro) <= tol).all()
