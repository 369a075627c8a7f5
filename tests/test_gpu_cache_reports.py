"""What the calls of the paged cache report: a refused reservation, seen by the append behind it; faults that one launch of several meets."""
import numpy as np
import pytest
import torch

from paper_2601_15305_b200 import binding as gsa
from test_gpu_cache import BF16, F32, GEOMETRIES, I32, Pair, i32

pytestmark = pytest.mark.gpu


def _reserve(p, n_new):
    start = torch.full((p.plain.B,), -7, dtype=I32, device="cuda")
    gsa.gsa_cache_reserve(p.c, i32(n_new), start, p.ws)
    return start


def _put(p, n_new, start, L, ws=None):
    K, V, g2, kI = [t.cuda() for t in p.tokens(L)]
    gsa.gsa_cache_append(p.c, K, V, g2, kI, i32(n_new), start, p.ws if ws is None else ws)


# ---- a refused reservation ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("why,n_new,status", [("pages", [1, 90, 0], 7), ("row", [1, 0, 2000], 6), ("negative", [-1, 3, 1], 6)])
def test_an_append_behind_a_refused_reservation_says_so(why, n_new, status):
    p = Pair(3, 8, 10, **GEOMETRIES[1], seed=50)
    p.append([20, 16, 5])
    before = p.pool.clone()
    start = _reserve(p, n_new)
    assert (start == -1).all()
    _put(p, n_new, start, 90)                                            # (no look at the status in between, as in a captured step)
    assert p.status() == status
    _put(p, n_new, start, 90)                                            # and again: still nothing stored
    assert p.status() == status
    assert torch.equal(p.pool, before) and p.lens.tolist() == [20, 16, 5]
    # a reservation that goes through ends it
    p.append([1, 0, 2])
    p.same_pages()


def test_only_lost_tokens_are_reported():
    """A refusal is reported where tokens were given that it kept out, by an append on its workspace."""
    p = Pair(3, 8, 10, **GEOMETRIES[1], seed=51)
    p.append([20, 16, 5])
    other = torch.full_like(p.ws, 0xFF)
    for stale in (7, 6):                                                 # bytes that look like a refused call's status are none
        start = _reserve(p, [0, 500, 0])
        assert p.status() == 6                                           # (its row holds 160)
        _put(p, [0, 0, 0], start, 1)                                     # nothing given
        assert p.status() == 0
        _put(p, [1, 1, 1], start, 1)                                     # left out by the caller: that call's head is not a refusal any more
        assert p.status() == 0
        other[:4].view(I32).fill_(stale)
        _put(p, [1, 1, 1], start, 1, other)
        assert gsa.gsa_device_status(other) == 0
    start = _reserve(p, [0, 90, 0])
    assert p.status() == 7
    p.lens += 1                                                          # (places that the caller made by itself: 20, 16 begins a page, 5)
    _put(p, [1, 0, 1], i32([20, -1, 5]), 1)
    assert p.status() == 0
    p.lens -= 1
    # in a batch of 4096 sequences the one whose tokens are lost is found
    B = 4096
    q = Pair(B, 8, 2, **GEOMETRIES[1], seed=52)
    n = np.zeros(B, np.int32)
    n[4077] = 33                                                         # its row holds 32
    start = _reserve(q, n)
    kv, kI = torch.zeros(B, 1, 1, 64, dtype=BF16, device="cuda"), torch.zeros(B, 1, 32, dtype=BF16, device="cuda")
    gsa.gsa_cache_append(q.c, kv, kv, None, kI, i32(n), start, q.ws)
    assert q.status() == 6


def test_a_captured_step_on_a_full_pool_reports_every_time():
    """Reservation and append as one graph on one workspace, the stages on another, as a program runs them."""
    p = Pair(2, 4, 6, n_kv=1, d_h=64, dI=32, T=16, seed=53)
    p.append([30, 15])                                                   # 2 + 1 pages, one is free
    gp = gsa.make_params(B=2, Lq=1, Lk=96, n_h=4, n_kv=1, d_h=64, HI=2, dI=32, k_base=8, k_min=4, k_max=16, k_mode=2)
    one, start = i32([1, 1]), torch.zeros(2, dtype=I32, device="cuda")
    K, V, g2, kI = [t.cuda() for t in p.tokens(1)]
    qI, w = torch.randn(2, 1, 2, 32, generator=p.gen).to(BF16).cuda(), torch.ones(2, 1, 2, device="cuda")
    sc, idx, kt = (torch.zeros(2, 1, 96, device="cuda"), torch.zeros(2, 1, 16, dtype=I32, device="cuda"), torch.zeros(2, 1, dtype=I32, device="cuda"))
    ws = torch.zeros_like(p.ws)

    def step():
        gsa.gsa_cache_reserve(p.c, one, start, p.ws)
        gsa.gsa_cache_append(p.c, K, V, g2, kI, one, start, p.ws)
        gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, None, sc, 96, ws)
        gsa.gsa_cache_topk(p.c, gp, sc, 96, idx, kt, None, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                                           # 31, 16
    side.synchronize()
    assert p.status() == 0
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    want = [([32, 17], 0)] + [([32, 17], 7)] * 3                         # the fourth page, then none
    for lens, status in want:
        g.replay()
        torch.cuda.synchronize()
        assert p.lens.tolist() == lens and p.status() == status and gsa.gsa_device_status(ws) == 0
    gsa.gsa_cache_release(p.c, i32([1, 0]), p.ws)
    g.replay()
    torch.cuda.synchronize()
    assert p.lens.tolist() == [1, 18] and p.status() == 0


@pytest.mark.parametrize("pages", [12, 9])
def test_prompts_outlive_a_refused_fork(pages):
    """Prompts to beams in one go, without a look at the status between fork and release: the release takes from the lengths on the device
    whether the copies are there."""
    p = Pair(6, pages, 4, **GEOMETRIES[1], seed=54)
    p.append([40, 33, 0, 0, 0, 0])                                       # 3 + 3 pages; four copies take four more
    before = p.pool.clone()
    src = i32([-1, -1, 0, 0, 1, 1])
    gsa.gsa_cache_fork(p.c, src, True, p.ws)
    drop = (p.lens[2] > 0).to(I32) * i32([1, 1, 0, 0, 0, 0])
    ws = torch.zeros_like(p.ws)
    gsa.gsa_cache_release(p.c, drop, ws)
    assert gsa.gsa_device_status(ws) == 0
    if pages == 12:
        assert p.status() == 0 and p.lens.tolist() == [0, 0, 40, 40, 33, 33]
    else:
        assert p.status() == 7 and p.lens.tolist() == [40, 33, 0, 0, 0, 0]
        p.same_tables()
        assert torch.equal(p.pool, before)


# ---- calls of several launches -----------------------------------------------------------------------------------------------
def _keys_only(lens, T, dI, max_pages, seed, n_pages=None):
    """A cache that holds k^I alone, its pages scattered: the handle, its arrays, the keys [B][n, dI] as fp64."""
    geo = dict(page_tokens=T, n_kv=1, d_h=64, dI=dI)
    need = [-(-max(n, 0) // T) for n in lens]
    n_pages = n_pages or sum(need) + 3
    page = gsa.gsa_cache_page_bytes(gsa.cache_geometry(B=len(lens), n_pages=n_pages, max_pages=max_pages, **geo))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.zeros(n_pages * page, dtype=torch.uint8, device="cuda")
    rec = (page - T * 2 * dI) // T
    keys = pool.view(BF16).as_strided((n_pages, T, dI), (page // 2, dI, 1), T * rec // 2)
    keys.copy_(torch.randn(n_pages, T, dI, generator=gen, device="cuda") * dI ** -0.5)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(I32)
    table, at = torch.full((len(lens), max_pages), -1, dtype=I32, device="cuda"), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(n_pages, dtype=I32, device="cuda")
    refs[order[:at].long()] = 1
    c = gsa.make_cache(pool, table, i32(lens), refs, **geo)
    held = [keys[table[b, :m].long()].flatten(0, 1)[:max(n, 0)].double() for b, (n, m) in enumerate(zip(lens, need))]
    return c, held


def _score_case(c, held, lens, Lq, Lk, HI, dI, act, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = len(lens)
    gp = gsa.make_params(B=B, Lq=Lq, Lk=Lk, n_h=1, n_kv=1, d_h=64, HI=HI, dI=dI, act=act)
    qI = torch.randn(B, Lq, HI, dI, generator=gen, device="cuda").to(BF16)
    w, bI = torch.rand(B, Lq, HI, generator=gen, device="cuda"), torch.randn(HI, generator=gen, device="cuda") * 0.2
    stride = (Lk + 3) // 4 * 4
    sc = torch.full((B, Lq, stride), float("nan"), device="cuda")
    ws = torch.full((gsa.gsa_cache_workspace_bytes(c),), 0xFF, dtype=torch.uint8, device="cuda")
    run = lambda: gsa.gsa_cache_indexer_scores(c, gp, qI, w, bI, sc, stride, ws)  # noqa: E731

    def check(rows):
        for b, t in rows:
            n = max(0, lens[b] - Lq + t + 1)
            z = qI[b, t].double() @ held[b][:n].T + bI.double()[:, None]
            f = z.clamp(min=0) if act else torch.sigmoid(z)
            # products are exact, their sum is fp32: a matrix instruction cuts each of 16 and what they are added to by 2^-23 of the
            # magnitudes' sum at most (17 / 16 dI in all, bias and scaling 4 more); a sigmoid's slope is at most 1/4, its own error 2^-20;
            # the sum over the heads is fp32 again
            terms = qI[b, t].double().abs() @ held[b][:n].abs().T + bI.double().abs()[:, None]
            wt = w[b, t].double()
            tol = wt @ (terms * (dI + 8) * 2.0 ** -23 * (1.0 if act else 0.25) + 2.0 ** -20 + f * HI * 2.0 ** -23)
            assert ((sc[b, t, :n].double() - wt @ f).abs() <= tol).all(), (b, t)
            assert sc[b, t, n:].isnan().all(), (b, t)

    return run, check, ws


@pytest.mark.parametrize("act", [0, 1])
def test_scores_of_more_rows_than_a_launch_takes(act):
    """2304 rows; lengths and pages that only the first, or only the second launch (rows from 2048 on: the last sequence) finds out of range."""
    Lq, T = 256, 16
    lens = [300, 256, 0, 700, 90, 1, 511, 260, 333]
    c, held = _keys_only(lens, T, 32, 50, 60)
    run, check, ws = _score_case(c, held, lens, Lq, 800, 4, 32, act, 61)
    run()
    assert gsa.gsa_device_status(ws) == 0
    check([(b, t) for b in range(9) for t in list(range(0, Lq, 31)) + [Lq - 1]])
    table, kept = c.tensors[1], c.tensors[2].clone()
    for b in (8, 0, 3):
        for bad in (-1, 801, 2 ** 31 - 1):
            c.tensors[2][b] = bad
            run()
            assert gsa.gsa_device_status(ws) == 6, (b, bad)
            c.tensors[2].copy_(kept)
            run()
            assert gsa.gsa_device_status(ws) == 0
        page = int(table[b, 1])
        table[b, 1] = -1
        run()
        assert gsa.gsa_device_status(ws) == 6, b
        table[b, 1] = page
    run()
    assert gsa.gsa_device_status(ws) == 0


@pytest.mark.parametrize("row", [5, 2047, 2048, 4500])
def test_an_attention_launch_keeps_what_an_earlier_one_found(row):
    """4600 rows are three launches; an index out of range in one of them."""
    p = Pair(1, 20, 300, **GEOMETRIES[1], seed=62)
    p.append([200])
    rows, k_max = 4600, 16
    gp = gsa.make_params(B=1, Lq=rows, Lk=4800, n_h=2, n_kv=1, d_h=64, HI=1, dI=32, k_base=1, k_min=1, k_max=k_max)
    Q = torch.randn(1, rows, 2, 64, generator=p.gen).to(BF16).cuda()
    idx = torch.randint(0, 200, (1, rows, k_max), dtype=I32, generator=p.gen).cuda()
    kt = torch.full((1, rows), k_max, dtype=I32, device="cuda")
    out, ws = torch.zeros_like(Q), torch.full((gsa.gsa_cache_attn_workspace_bytes(gp),), 0xFF, dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, ws)
    assert gsa.gsa_device_status(ws) == 0
    good = out.clone()
    idx[0, row, 3] = 200
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, ws)
    assert gsa.gsa_device_status(ws) == 6
    others = torch.arange(rows, device="cuda") != row
    assert torch.equal(out[0, others], good[0, others])
    idx[0, row, 3] = 199
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, ws)
    assert gsa.gsa_device_status(ws) == 0


def test_calls_allocate_nothing():
    """Device memory stays as it is over calls of every kind (the first ones load their kernels)."""
    p = Pair(2, 60, 12, **GEOMETRIES[2], seed=63)
    gp = gsa.make_params(B=2, Lq=1, Lk=300, n_h=4, n_kv=2, d_h=64, HI=2, dI=64, k_base=300, k_min=4, k_max=300, k_mode=2)
    K, V, g2, kI = [t.cuda() for t in p.tokens(150)]
    n_new, none = i32([150, 3]), i32([0, 1])
    start, live = torch.zeros(2, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    K2, V2, kI2 = torch.zeros_like(K), torch.zeros_like(K), torch.zeros_like(kI)
    qI, w, Q = torch.randn(2, 1, 2, 64, device="cuda").to(BF16), torch.ones(2, 1, 2, device="cuda"), torch.randn(2, 1, 4, 64, device="cuda").to(BF16)
    sc, idx, kt, out = (torch.zeros(2, 1, 300, device="cuda", dtype=F32), torch.zeros(2, 1, 300, dtype=I32, device="cuda"),
                        torch.zeros(2, 1, dtype=I32, device="cuda"), torch.zeros_like(Q))
    wa, src, both = torch.zeros(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda"), i32([-1, 0]), i32([1, 1])

    def turn():
        gsa.gsa_cache_reserve(p.c, n_new, start, p.ws)
        gsa.gsa_cache_append(p.c, K, V, g2, kI, n_new, start, p.ws)
        gsa.gsa_cache_read(p.c, K2, V2, kI2, p.ws)
        gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, None, sc, 300, p.ws)
        gsa.gsa_cache_topk(p.c, gp, sc, 300, idx, kt, None, p.ws)
        gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, wa)
        gsa.gsa_cache_release(p.c, none, p.ws)
        for share in (True, False):
            gsa.gsa_cache_fork(p.c, src, share, p.ws)
            gsa.gsa_cache_release(p.c, none, p.ws)
        gsa.gsa_cache_compact(p.c, live, p.ws)
        gsa.gsa_cache_release(p.c, both, p.ws)

    for _ in range(2):
        turn()
    torch.cuda.synchronize()
    held, free = torch.cuda.memory_allocated(), torch.cuda.mem_get_info()[0]
    n0 = gsa.gsa_launch_count()
    for _ in range(25):
        turn()
    torch.cuda.synchronize()
    assert gsa.gsa_launch_count() - n0 >= 25 * 14
    assert torch.cuda.memory_allocated() == held and torch.cuda.mem_get_info()[0] == free
    assert int(live) == 5 and p.lens.tolist() == [0, 0] and (p.refs == 0).all()
