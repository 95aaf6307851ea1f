"""Packed prompts and the paged cache where they could go wrong: many sequences, rows behind the last one, other sequences' NaN,
large groups, pools past 32-bit offsets, calls beside one another, sequences that evict nothing or one token among others."""
import numpy as np
import pytest
import torch

import paper_2504_14051_b200 as P
from paper_2504_14051_b200 import binding as C
from test_paged_gpu import BF, DEV, F32, Pages, attend_case, check_rows, evict_case, f64, prompt_case, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_sequences(dtype):
    """More than the 32 that a scan holds at a time, some without new tokens."""
    g = np.random.default_rng(0)
    lengths = [int(x) for x in g.integers(0, 40, 70)]
    lengths[33] = 200
    prompt_case(lengths, (4, 2), 64, dtype, seed=1)
    lens = [int(x) for x in g.integers(1, 300, 70)]
    for most in (1, 3, 30):
        new = [min(n, int(x)) for n, x in zip(lens, g.integers(0, most + 1, 70))]
        new[69] = min(most, lens[69])
        attend_case(lens, new, (4, 2), 64, dtype, 16, seed=2)


@pytest.mark.parametrize("heads", [(16, 1), (32, 2), (13, 1), (5, 1), (10, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_large_and_odd_groups(heads, d):
    prompt_case([150, 40], heads, d, BF, seed=3)
    attend_case([700, 90, 33], [1, 1, 1], heads, d, BF, 32, seed=4)
    attend_case([700, 90, 33], [2, 1, 2], heads, d, BF, 32, seed=4, mass=False)
    attend_case([1300, 90, 33], [40, 1, 9], heads, d, BF, 64, seed=5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [(8, 1, 3), (8, 2, 4), (4, 1, 7), (4, 1, 8), (16, 2, 3)])
def test_drafted_tokens_without_weights(rows, d):
    """Up to 32 rows of a pair take the streaming kernel where no weights are wanted."""
    Hq, Hkv, m = rows
    attend_case([513, 40, 1000, m], [m, 1, m, m], (Hq, Hkv), d, BF, 16, seed=6, mass=False)


@pytest.mark.parametrize("new", [[70], [128], [256, 3]])
@pytest.mark.parametrize("d", [64, 128])
def test_split_keys(new, d):
    """Few row blocks and many keys: the last round's items are cut, down to splits in which some rows see nothing."""
    lens = [4000, 2000][:len(new)]
    attend_case(lens, new, (4, 1), d, BF, 64, seed=7)


def test_split_keys_where_the_block_spans_splits():
    attend_case([1500], [1400], (2, 1), 128, BF, 32, seed=8)
    attend_case([1100, 30], [1100, 30], (4, 1), 64, BF, 128, seed=8)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_outside_the_sequences_are_left_alone(dtype):
    """cu that begins behind row 0 and ends before row T."""
    T, cu, Hq, Hkv, d = 90, [7, 40, 40, 73], 4, 2, 64
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(T, h, d, generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    for x in (q, k, v):
        x[:7] = float("nan")
        x[73:] = float("nan")
    p = P.make_paged_params(3, Hq, Hkv, d, 0, 0, 0, T, 40, dtype, 0.125)
    ws = P.alloc_paged_workspace(p, DEV)
    o, lse, mass = torch.full((T, Hq, d), 7.0, dtype=dtype, device=DEV), torch.full((T, Hq), 7.0, device=DEV), torch.full((T, Hkv), 7.0, device=DEV)
    P.caote_prompt_attend(p, q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(cu, dtype=torch.int32, device=DEV), o, lse, mass, ws)
    assert P.caote_read_status(ws) == 0
    for x in (o, lse, mass):
        assert (x[:7] == 7.0).all() and (x[73:] == 7.0).all()
    kk, vv = f64(k), f64(v)
    check_rows(q, lambda b, h: (kk[cu[b]:cu[b + 1], h], vv[cu[b]:cu[b + 1], h]), cu, Hkv, 0.125, o, lse, dtype,
               lambda b: f64(mass)[cu[b]:cu[b + 1]].T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_of_one_sequence_stays_there(dtype):
    cu, Hq, Hkv, d = [0, 50, 131, 200], 4, 2, 128
    g = torch.Generator().manual_seed(10)
    q, k, v = (torch.randn(200, h, d, generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    for x in (q, k, v):
        x[50:131] = float("nan")
    p = P.make_paged_params(3, Hq, Hkv, d, 0, 0, 0, 200, 81, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    o, lse, mass = torch.zeros((200, Hq, d), dtype=dtype, device=DEV), torch.zeros((200, Hq), device=DEV), torch.zeros((200, Hkv), device=DEV)
    P.caote_prompt_attend(p, q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(cu, dtype=torch.int32, device=DEV), o, lse, mass, ws)
    kk, vv = f64(k), f64(v)
    for lo, hi in ((0, 50), (131, 200)):
        check_rows(q[lo:hi], lambda b, h: (kk[lo:hi, h], vv[lo:hi, h]), [0, hi - lo], Hkv, 0.1, o[lo:hi], lse[lo:hi], dtype,
                   lambda b: f64(mass)[lo:hi].T)


def test_infinite_queries_and_keys_end():
    """Nothing is said about their results, but the call returns and other sequences are right."""
    for bad in (float("inf"), float("-inf"), float("nan"), 3e38):
        pg = Pages([300, 200], 2, 128, 16, BF, seed=11)
        at, row = pg.at(0, 300)
        pg.K[at[::7], :, row[::7]] = bad
        for new in (1, 20):
            q = torch.randn(2 * new, 4, 128, generator=pg.g).to(BF).to(DEV)
            q[0] = bad
            p = P.make_paged_params(2, 4, 2, 128, 16, pg.n_pages, pg.max_pages, 2 * new, new, BF, 0.1)
            ws = P.alloc_paged_workspace(p, DEV)
            o = torch.zeros((2 * new, 4, 128), dtype=BF, device=DEV)
            P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), pg.mass.to(DEV), pg.table.to(DEV),
                                 torch.tensor([300, 200], dtype=torch.int32, device=DEV),
                                 torch.tensor([0, new, 2 * new], dtype=torch.int32, device=DEV), o, None, ws)
            assert P.caote_read_status(ws) == 0
            check_rows(q[new:], lambda b, h: pg.keys_of(1, h), [0, new], 2, 0.1, o[new:], None, BF)


def test_a_later_tile_with_far_larger_logits():
    """The reference moves in the middle of a walk, in either half of a tile and in either part of a half, by little and by far."""
    for at in (130, 170, 200, 240):
        for size in (0.25, 1.0, 8.0):
            g = torch.Generator().manual_seed(12)
            T = 300
            q = torch.ones(T, 4, 128, dtype=BF)
            k, v = (0.1 * torch.randn(T, 2, 128, generator=g)).to(BF), torch.randn(T, 2, 128, generator=g).to(BF)
            k[at] = size
            p = P.make_paged_params(1, 4, 2, 128, 0, 0, 0, T, T, BF, 1.0)
            ws = P.alloc_paged_workspace(p, DEV)
            o, lse, mass = torch.zeros((T, 4, 128), dtype=BF, device=DEV), torch.zeros((T, 4), device=DEV), torch.zeros((T, 2), device=DEV)
            P.caote_prompt_attend(p, q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor([0, T], dtype=torch.int32, device=DEV), o, lse, mass, ws)
            kk, vv = f64(k), f64(v)
            check_rows(q, lambda b, h: (kk[:, h], vv[:, h]), [0, T], 2, 1.0, o, lse, BF, lambda b: f64(mass).T)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
def test_offsets_past_32_bits(dtype, d):
    """Pages near the end of a pool whose elements do not fit 32 bits: append, attend, evict."""
    page, Hkv = 256, 4
    n_pages = (1 << 32) // (Hkv * page * d) + 8
    K = torch.empty((n_pages, Hkv, page, d), dtype=dtype, device=DEV)
    V = torch.empty_like(K)
    mass, pos = torch.empty((n_pages, Hkv, page), device=DEV), torch.empty((n_pages, Hkv, page), dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(13)
    lengths = [300, 200]
    T, cu = 500, [0, 300, 500]
    table = torch.tensor([[n_pages - 1, n_pages - 3], [n_pages - 2, -1]], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn(T, h, d, generator=g).to(dtype) for h in (8, Hkv, Hkv))
    p = P.make_paged_params(2, 8, Hkv, d, page, n_pages, 2, T, 300, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    lens, seen = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    cu_t = torch.tensor(cu, dtype=torch.int32, device=DEV)
    P.caote_paged_append(p, K, V, mass, pos, table, lens, seen, k.to(DEV), v.to(DEV), None, cu_t, ws)
    o = torch.zeros((T, 8, d), dtype=dtype, device=DEV)
    P.caote_paged_attend(p, q.to(DEV), K, V, mass, table, lens, cu_t, o, None, ws)
    kk, vv = f64(k), f64(v)
    check_rows(q, lambda b, h: (kk[cu[b]:cu[b + 1], h], vv[cu[b]:cu[b + 1], h]), cu, Hkv, 0.1, o, None, dtype)
    p1 = P.make_paged_params(2, 8, Hkv, d, page, n_pages, 2, 2, 1, dtype, 0.1)
    o1 = torch.zeros((2, 8, d), dtype=dtype, device=DEV)
    P.caote_paged_attend(p1, q[[299, 499]].to(DEV), K, V, None, table, lens, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), o1, None, ws)
    check_rows(q[[299, 499]], lambda b, h: (kk[cu[b]:cu[b + 1], h], vv[cu[b]:cu[b + 1], h]), [0, 1, 2], Hkv, 0.1, o1, None, dtype)
    out, cnt = torch.zeros((2, Hkv, 40), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    P.caote_paged_evict(p, K, V, mass, pos, table, lens, seen, torch.tensor([260, 199], dtype=torch.int32, device=DEV), 4, 16, out, cnt, ws)
    assert P.caote_read_status(ws) == 0 and lens.tolist() == [260, 199] and cnt.tolist() == [40, 1]
    for b, (n, total) in enumerate(((260, 300), (199, 200))):
        held = torch.cat([pos[table[b, i]] for i in range(2) if table[b, i] >= 0], dim=1)[:, :n].cpu()
        keys = torch.cat([K[table[b, i]] for i in range(2) if table[b, i] >= 0], dim=1)[:, :n].cpu()
        for h in range(Hkv):
            assert len(set(held[h].tolist())) == n
            assert torch.equal(keys[h].view(torch.int16 if dtype == BF else torch.int32),
                               k[cu[b] + held[h].long(), h].contiguous().view(torch.int16 if dtype == BF else torch.int32))


def test_calls_beside_one_another():
    """Two streams with workspaces of their own."""
    cases = []
    for seed in (14, 15):
        pg = Pages([2000, 900, 77], 2, 128, 16, BF, seed=seed)
        for new in (1, 50):
            q = torch.randn(3 * new, 8, 128, generator=pg.g).to(BF).to(DEV)
            p = P.make_paged_params(3, 8, 2, 128, 16, pg.n_pages, pg.max_pages, 3 * new, new, BF, 0.1)
            cases.append((p, q, pg.K.to(DEV), pg.V.to(DEV), pg.mass.to(DEV), pg.table.to(DEV), torch.tensor([2000, 900, 77], dtype=torch.int32, device=DEV),
                          torch.tensor([0, new, 2 * new, 3 * new], dtype=torch.int32, device=DEV)))

    def run(c, mass, ws, stream=None):
        o = torch.zeros_like(c[1])
        P.caote_paged_attend(c[0], c[1], c[2], c[3], mass, c[5], c[6], c[7], o, None, ws, stream)
        return o

    want = []
    for c in cases:
        m = c[4].clone()
        want.append((run(c, m, P.alloc_paged_workspace(c[0], DEV)), m))
    streams = [torch.cuda.Stream() for _ in cases]
    spaces, masses = [P.alloc_paged_workspace(c[0], DEV) for c in cases], [c[4].clone() for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for m, c in zip(masses, cases):
            m.copy_(c[4])
        torch.cuda.synchronize()
        for s, ws, m, c in zip(streams, spaces, masses, cases):
            with torch.cuda.stream(s):
                got.append(run(c, m, ws, s))
        torch.cuda.synchronize()
        for (o, m), x, y in zip(want, got, masses):
            assert torch.equal(o, x) and torch.equal(torch.nan_to_num(m), torch.nan_to_num(y))


def test_one_workspace_serves_smaller_calls_in_any_order():
    pg = Pages([600, 90, 300], 2, 64, 32, BF, seed=16)
    big = P.make_paged_params(3, 8, 2, 64, 32, pg.n_pages, pg.max_pages, 300, 100, BF, 0.1)
    shared = P.alloc_paged_workspace(big, DEV)
    K, V, table = pg.K.to(DEV), pg.V.to(DEV), pg.table.to(DEV)
    lens = torch.tensor([600, 90, 300], dtype=torch.int32, device=DEV)
    for new in ([90, 90, 90], [1, 1, 1], [3, 0, 2], [0, 1, 0], [17, 64, 1], [1, 1, 1]):
        T, cu = sum(new), starts(new)
        p = P.make_paged_params(3, 8, 2, 64, 32, pg.n_pages, pg.max_pages, T, max(new), BF, 0.1)
        q = torch.randn(T, 8, 64, generator=pg.g).to(BF).to(DEV)
        outs = []
        for ws in (shared, P.alloc_paged_workspace(p, DEV)):
            o, m = torch.zeros((T, 8, 64), dtype=BF, device=DEV), pg.mass.to(DEV)
            P.caote_paged_attend(p, q, K, V, m, table, lens, torch.tensor(cu, dtype=torch.int32, device=DEV), o, None, ws)
            assert P.caote_read_status(ws) == 0
            outs.append((o, torch.nan_to_num(m)))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("Hkv", [1, 3, 5, 8, 9, 12])
def test_evict_one_token_for_any_number_of_heads(Hkv):
    evict_case([64, 300, 1, 0, 17], [63, 299, 1, 1, 17], Hkv=Hkv, d=64, page=16, sinks=2, recent=5, max_evict=1)
    evict_case([64, 300, 1, 0, 17], [63, 290, 1, 1, 17], Hkv=Hkv, d=64, page=16, sinks=2, recent=5)


def test_evict_where_room_for_many_is_given():
    """Several CTAs per pair, and sequences that evict none, one or two."""
    evict_case([400, 300, 200, 50], [400, 299, 198, 10], max_evict=100, sinks=1, recent=3)
    evict_case([2000, 700], [1800, 400], max_evict=300, page=64, d=128, dtype=BF)


def test_evict_more_than_are_not_sheltered():
    evict_case([500, 500], [30, 400], sinks=40, recent=300, pos_of=torch.arange)
    evict_case([500, 500], [200, 205], sinks=0, recent=300, pos_of=torch.arange)


def test_append_to_many_sequences():
    """More sequences than starts are kept in shared memory."""
    B, Hkv, d, page = 1500, 1, 64, 16
    new = [b % 3 for b in range(B)]
    T, cu = sum(new), starts(new)
    p = P.make_paged_params(B, 2, Hkv, d, page, B, 1, T, 2, F32, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K, V = torch.zeros((B, Hkv, page, d), device=DEV), torch.zeros((B, Hkv, page, d), device=DEV)
    pos = torch.full((B, Hkv, page), -1, dtype=torch.int32, device=DEV)
    table = torch.arange(B - 1, -1, -1, dtype=torch.int32, device=DEV).view(B, 1)
    lens = torch.full((B,), 5, dtype=torch.int32, device=DEV)
    k = torch.randn(T, Hkv, d, device=DEV)
    P.caote_paged_append(p, K, V, None, pos, table, lens, None, k, 2 * k, None, torch.tensor(cu, dtype=torch.int32, device=DEV), ws)
    assert P.caote_read_status(ws) == 0 and lens.tolist() == [5 + m for m in new]
    for b in (0, 1, 2, 700, 1498, 1499):
        rows = slice(cu[b], cu[b + 1])
        assert torch.equal(K[B - 1 - b, 0, 5:5 + new[b]], k[rows, 0]) and torch.equal(V[B - 1 - b, 0, 5:5 + new[b]], 2 * k[rows, 0])
        assert pos[B - 1 - b, 0].tolist() == [-1] * 5 + list(range(5, 5 + new[b])) + [-1] * (11 - new[b])


def test_empty_calls():
    """No sequence has a new token in it: T rows are packed, none is any sequence's."""
    pg = Pages([30, 40], 2, 64, 16, BF, seed=17)
    p = P.make_paged_params(2, 4, 2, 64, 16, pg.n_pages, pg.max_pages, 3, 3, BF, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    o, m = torch.full((3, 4, 64), 7.0, dtype=BF, device=DEV), pg.mass.to(DEV)
    lens = torch.tensor([30, 40], dtype=torch.int32, device=DEV)
    cu = torch.tensor([1, 1, 1], dtype=torch.int32, device=DEV)
    q = torch.zeros(3, 4, 64, dtype=BF, device=DEV)
    P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), m, pg.table.to(DEV), lens, cu, o, None, ws)
    P.caote_paged_append(p, pg.K.to(DEV), pg.V.to(DEV), m, None, pg.table.to(DEV), lens, None, q[:, :2], q[:, 2:], None, cu, ws)
    assert P.caote_read_status(ws) == 0 and (o == 7.0).all() and lens.tolist() == [30, 40]
    assert torch.equal(m.cpu().view(torch.int32), pg.mass.view(torch.int32))


def test_budget_and_counts_are_checked_before_anything_moves():
    assert C.ERR_BAD_PAGE == -8
    pg = Pages([40], 1, 64, 16, F32, seed=18)
    p = P.make_paged_params(1, 1, 1, 64, 16, pg.n_pages, pg.max_pages, 1, 1, F32, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K, m = pg.K.to(DEV), pg.mass.to(DEV)
    pos = torch.arange(m.numel(), dtype=torch.int32, device=DEV).view(m.shape)
    for budget in (0, -7):  # counts as 1
        lens = torch.tensor([3], dtype=torch.int32, device=DEV)
        cnt = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.caote_paged_evict(p, K.clone(), K.clone(), m.clone(), pos.clone(), pg.table.to(DEV), lens, lens.clone(),
                            torch.tensor([budget], dtype=torch.int32, device=DEV), 0, 0, torch.zeros((1, 1, 4), dtype=torch.int32, device=DEV), cnt, ws)
        assert lens.tolist() == [1] and cnt.tolist() == [2]


@pytest.mark.parametrize("B,new", [(3, 700), (20, 100), (300, 20)])
def test_append_where_some_sequences_have_a_bad_page(B, new):
    """The last page of two sequences is none: they keep their lengths, all others get their rows."""
    old, page, Hkv, d = 10, 16, 2, 64
    pages = (old + new + page - 1) // page
    p = P.make_paged_params(B, 4, Hkv, d, page, B * pages, pages, B * new, new, F32, 0.1)
    table = torch.randperm(B * pages, generator=torch.Generator().manual_seed(B), dtype=torch.int64).to(torch.int32).view(B, pages)
    bad = {1: -1, B - 1: B * pages}
    given = table.clone()
    for b, x in bad.items():
        given[b, pages - 1] = x
    K = torch.full((B * pages, Hkv, page, d), 5.0, device=DEV)
    V, k, v = K.clone(), torch.randn(B * new, Hkv, d, device=DEV), torch.randn(B * new, Hkv, d, device=DEV)
    lens = torch.full((B,), old, dtype=torch.int32, device=DEV)
    seen = lens.clone()
    ws = P.alloc_paged_workspace(p, DEV)
    cu = torch.arange(0, B * new + 1, new, dtype=torch.int32, device=DEV)
    P.caote_paged_append(p, K, V, None, None, given.to(DEV), lens, seen, k, v, None, cu, ws)
    assert P.caote_read_status(ws) == C.ERR_BAD_PAGE
    want = [old if b in bad else old + new for b in range(B)]
    assert lens.tolist() == want and seen.tolist() == want
    for pool, rows in ((K, k), (V, v)):
        # [B, slots, Hkv, d]
        got = pool[table.long().to(DEV)].permute(0, 1, 3, 2, 4).reshape(B, pages * page, Hkv, d)
        assert (got[:, :old] == 5.0).all() and (got[:, old + new:] == 5.0).all()
        good = [b for b in range(B) if b not in bad]
        assert torch.equal(got[good, old:old + new], rows.view(B, new, Hkv, d)[good])
