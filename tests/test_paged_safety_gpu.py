"""Calls with page tables or starts that do not fit: what belongs to other sequences stays as it is."""
import pytest
import torch

import paper_2504_14051_b200 as P
from paper_2504_14051_b200 import binding as C
from test_paged_gpu import BF, DEV, F32, Pages

pytestmark = pytest.mark.gpu


def pages_with_page_0_in(b, *args, **kw):
    """Pages whose page 0, where a bad index might end up, holds the first tokens of sequence b."""
    pg = Pages(*args, **kw)
    x = int(pg.table[b, 0])
    for pool in (pg.K, pg.V, pg.mass):
        pool[[0, x]] = pool[[x, 0]].clone()
    zero = pg.table == 0
    pg.table[pg.table == x] = 0
    pg.table[zero] = x
    return pg


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_a_bad_page_adds_no_weight_to_other_sequences(new, d, dtype):
    lens = [100, 390, 120]
    pg = pages_with_page_0_in(0, lens, 2, d, 16, dtype, seed=1)
    T = 3 * new
    q = torch.randn(T, 4, d, generator=pg.g).to(dtype).to(DEV)
    p = P.make_paged_params(3, 4, 2, d, 16, pg.n_pages, pg.max_pages, T, new, dtype, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K, V, lens_t = pg.K.to(DEV), pg.V.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, new, 2 * new, T], dtype=torch.int32, device=DEV)

    def call(table):
        m, o = pg.mass.to(DEV), torch.zeros((T, 4, d), dtype=dtype, device=DEV)
        P.caote_paged_attend(p, q, K, V, m, table.to(DEV), lens_t, cu, o, None, ws)
        return m.cpu().view(torch.int32), o, P.caote_read_status(ws)

    want, o0, st = call(pg.table)
    assert st == 0
    own = torch.zeros(pg.n_pages, dtype=torch.bool)
    own[pg.table[1, :-(-390 // 16)].long()] = True
    for at in ([2], [0], [24], [3, 7, 20], list(range(25))):
        for bad in (-1, pg.n_pages, 1 << 30, -(1 << 31)):
            table = pg.table.clone()
            table[1, at] = bad
            got, o, st = call(table)
            assert st == C.ERR_BAD_PAGE
            assert torch.equal(got[~own], want[~own]), (at, bad)
            lost = pg.table[1, at].long()  # the pages whose place the bad index has
            assert torch.equal(got[lost], pg.mass[lost].view(torch.int32))
            assert torch.equal(o[:new], o0[:new]) and torch.equal(o[2 * new:], o0[2 * new:])


@pytest.mark.parametrize("many", [0, 1100])
@pytest.mark.parametrize("cu", [[0, 5, 3, 8], [4, 8, 0, 4], [0, 0, 4, 2, 8], [0, 8, 7]])
def test_append_with_starts_that_do_not_ascend(cu, many):
    """Which sequence a row belongs to is not clear then: no length moves on (with more sequences than fit shared memory, too)."""
    cu = cu + [8] * many
    B, T = len(cu) - 1, 8
    p = P.make_paged_params(B, 2, 1, 64, 16, 2 * B, 2, T, T, F32, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    K = torch.full((2 * B, 1, 16, 64), 5.0, device=DEV)
    V, k = K.clone(), torch.randn(T, 1, 64, device=DEV)
    table = torch.arange(2 * B, dtype=torch.int32, device=DEV).view(B, 2)
    lens = torch.full((B,), 3, dtype=torch.int32, device=DEV)
    seen = torch.full((B,), 9, dtype=torch.int32, device=DEV)
    P.caote_paged_append(p, K, V, None, None, table, lens, seen, k, k, None, torch.tensor(cu, dtype=torch.int32, device=DEV), ws)
    assert P.caote_read_status(ws) == C.ERR_BAD_LENGTH
    assert (lens == 3).all() and (seen == 9).all()
    assert (K[:, :, :3] == 5.0).view(B, 2, -1)[:, 0].all() and (V[:, :, :3] == 5.0).view(B, 2, -1)[:, 0].all()  # the tokens that are there
    cu = torch.tensor([0, 5, 8] + [8] * (B - 2), dtype=torch.int32, device=DEV)
    P.caote_paged_append(p, K, V, None, None, table, lens, seen, k, k, None, cu, ws)  # (the workspace is as good as before)
    assert P.caote_read_status(ws) == 0 and lens[:2].tolist() == [8, 6] and (lens[2:] == 3).all()
    assert torch.equal(K[0, 0, 3:8], k[:5, 0]) and torch.equal(V[2, 0, 3:6], k[5:, 0])


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64)])
@pytest.mark.parametrize("m", [1, 3, 60])
def test_sequences_that_overlap_are_reported_and_nothing_else_is_touched(m, dtype, d):
    """cu that goes back and forth: every second sequence has all rows, more row blocks than the call has room for."""
    B, guard = 66, 7.0
    cu = torch.tensor([0, m] * (B // 2) + [0], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(3)

    def guarded(*shape, dtype):
        """A tensor in the middle of a larger one."""
        n = 1
        for x in shape:
            n *= x
        whole = torch.full((n + 2 * 4096,), guard, dtype=dtype, device=DEV)
        return whole, whole[4096:4096 + n].view(shape)

    q, k, v = (torch.randn(m, h, d, generator=g).to(dtype).to(DEV) for h in (4, 2, 2))
    pg = Pages([200] * B, 2, d, 16, dtype, seed=3)
    for pages in (False, True):
        p = P.make_paged_params(B, 4, 2, d, *((16, pg.n_pages, pg.max_pages) if pages else (0, 0, 0)), m, m, dtype, 0.1)
        size = C.caote_paged_workspace_bytes(p)
        space, ws = guarded(size, dtype=torch.uint8)
        ws.zero_()
        all_o, o = guarded(m, 4, d, dtype=dtype)
        all_lse, lse = guarded(m, 4, dtype=F32)
        if pages:
            all_mass, mass = guarded(pg.n_pages, 2, 16, dtype=F32)
            mass.copy_(pg.mass)
            P.caote_paged_attend(p, q, pg.K.to(DEV), pg.V.to(DEV), mass, pg.table.to(DEV), torch.full((B,), 200, dtype=torch.int32, device=DEV), cu, o, lse, ws)
        else:
            all_mass, mass = guarded(m, 2, dtype=F32)
            P.caote_prompt_attend(p, q, k, v, cu, o, lse, mass, ws)
        assert P.caote_read_status(ws) == C.ERR_BAD_LENGTH
        for x in (space, all_o, all_lse, all_mass):
            assert (x[:4096] == guard).all() and (x[-4096:] == guard).all()


def test_weights_in_a_cache_of_more_than_2_27_tokens():
    """Groups of 16: the first row that sees a key, counted from the key's end of the cache, passes 32 bits. All keys are equal, so that
    sums are whole numbers up to 2^23 and every weight is 16 / (n - 1) + 16 / n: off by the log-sum-exp, 27 in the log2 domain (2^-19
    there, twice, times ln 2), and the exponential (2^-21)."""
    n, page, d = (1 << 27) + 1024, 256, 64
    pages = n // page
    K = torch.zeros((pages, 1, page, d), dtype=BF, device=DEV)
    V, mass = torch.zeros_like(K), torch.zeros((pages, 1, page), device=DEV)
    p = P.make_paged_params(1, 16, 1, d, page, pages, pages, 2, 2, BF, 0.1)
    ws = P.alloc_paged_workspace(p, DEV)
    q, o = torch.ones((2, 16, d), dtype=BF, device=DEV), torch.zeros((2, 16, d), dtype=BF, device=DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).view(1, pages)
    P.caote_paged_attend(p, q, K, V, mass, table, torch.tensor([n], dtype=torch.int32, device=DEV), torch.tensor([0, 2], dtype=torch.int32, device=DEV),
                         o, None, ws)
    assert P.caote_read_status(ws) == 0
    flat = mass.view(-1)
    want, tol = 16 / (n - 1) + 16 / n, 2 * 0.7 * 2.0 ** -19 + 2.0 ** -21 + 32 * 2.0 ** -24
    assert ((flat[:-1] - want).abs() <= tol * want).all(), (flat[:-1] - want).abs().argmax()
    assert abs(float(flat[-1]) - 16 / n) <= tol * 16 / n


@pytest.mark.filterwarnings("ignore:The CUDA Graph is empty")
def test_a_cache_refuses_to_be_captured_and_goes_on():
    c = P.PagedCache(1, 4, 2, 64, 16, 8, 100, 40, BF, 30)
    q, k, v = (torch.randn(40, h, 64, device=DEV).to(BF) for h in (4, 2, 2))
    c.prompt(q, k, v, [40])
    before = (list(c.host_lens), [list(p) for p in c._pages], c.lens.tolist())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.capture_begin()
        try:
            with pytest.raises(ValueError, match="captured"):
                c.step(q[:1], k[:1], v[:1], [1])
        finally:
            graph.capture_end()
    torch.cuda.synchronize()
    assert (list(c.host_lens), [list(p) for p in c._pages], c.lens.tolist()) == before
    c.step(q[:1], k[:1], v[:1], [1])
    assert c.lens.tolist() == c.host_lens == [30] and c.status() == 0
