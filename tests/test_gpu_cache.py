"""The paged 4-bit cache on the GPU against its plain 64-bit form (cache_plain.py).

Stored values, page tables, counts and copied bytes have to be equal: the format is defined to the bit.  Tolerances of the two stages
that compute in floating point, derived:
  * attention: the softmax numerators are rounded to fp16, at a scale where a row's largest is at least 2^7: half a step is 2^-11 of one
    (2^-11 sum_j a_j |v_j| of the sum), or 2^-25 below fp16's normal range, 2^-32 of the row's sum (2^-32 sum_j |v_j|); the output is
    rounded to bf16 (2^-8 of it); scores are fp32 sums of at most 128 exact products, within 128 * 2^-24 of sum_d |q_d k_d|, which
    the exponential turns into as large a relative error of a probability, and its own is 2^-21.
  * indexer: fp32 sums of exact products; the sigmoid's slope is at most 1/4, its approximation within 2^-20; eight heads.
"""
import numpy as np
import pytest
import torch

from cache_plain import PlainCache, bf16
from paper_2601_15305_b200 import binding as gsa

pytestmark = pytest.mark.gpu

I32, BF16, F32 = torch.int32, torch.bfloat16, torch.float32
GEOMETRIES = [dict(n_kv=8, d_h=128, dI=64, T=64), dict(n_kv=1, d_h=64, dI=32, T=16), dict(n_kv=2, d_h=64, dI=64, T=32),
              dict(n_kv=4, d_h=128, dI=32, T=128), dict(n_kv=1, d_h=128, dI=64, T=16), dict(n_kv=8, d_h=64, dI=32, T=64)]


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


class Pair:
    """A cache on the GPU and its plain twin."""

    def __init__(self, B, n_pages, max_pages, n_kv, d_h, dI, T, seed=0):
        self.plain = PlainCache(B, n_pages, T, max_pages, n_kv, d_h, dI)
        self.gen = torch.Generator().manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.pool = torch.zeros(self.plain.pool.size, dtype=torch.uint8, device="cuda")
        self.table, self.lens, self.refs = (torch.full((B, max_pages), -1, dtype=I32, device="cuda"),
                                            torch.zeros(B, dtype=I32, device="cuda"), torch.zeros(n_pages, dtype=I32, device="cuda"))
        self.c = gsa.make_cache(self.pool, self.table, self.lens, self.refs, page_tokens=T, n_kv=n_kv, d_h=d_h, dI=dI)
        assert gsa.gsa_cache_page_bytes(self.c) == self.plain.page_bytes
        self.ws = torch.full((gsa.gsa_cache_workspace_bytes(self.c),), 0xFF, dtype=torch.uint8, device="cuda")

    def status(self):
        return gsa.gsa_device_status(self.ws)

    def same_tables(self):
        assert np.array_equal(self.table.cpu().numpy(), self.plain.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.plain.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.plain.refs)

    def same_pages(self):
        """The records and keys of every token held (bytes behind a sequence's end are nobody's)."""
        pool = self.pool.cpu().numpy().reshape(self.plain.pool.shape)
        P = self.plain
        for b in range(P.B):
            for j in range(P.pages_of(P.lens[b])):
                n, page = min(P.T, int(P.lens[b]) - j * P.T), P.table[b, j]
                D = P.D + P.D // 8
                got, want = (x[page, :P.T * P.rec].reshape(P.T, P.rec)[:n, :D] for x in (pool, P.pool))
                assert np.array_equal(got, want), (b, j, np.argwhere(got != want)[:4])
                got, want = (x[page, P.T * P.rec:].reshape(P.T, -1)[:n] for x in (pool, P.pool))
                assert np.array_equal(got, want), (b, j)

    def reserve(self, n_new):
        start = torch.full((self.plain.B,), -7, dtype=I32, device="cuda")
        gsa.gsa_cache_reserve(self.c, i32(n_new), start, self.ws)
        want, want_start = self.plain.reserve(n_new)
        assert self.status() == want
        assert np.array_equal(start.cpu().numpy(), want_start)
        self.same_tables()
        return start

    def tokens(self, L, outliers=True, gate=True):
        P = self.plain
        K = torch.randn(P.B, L, P.n_kv, P.d_h, generator=self.gen)
        if outliers:
            K[..., 3::P.d_h // 4] *= 5
        V = torch.randn(P.B, L, P.n_kv, P.d_h, generator=self.gen)
        g2 = 2 * torch.randn(P.B, L, P.n_kv, P.d_h, generator=self.gen) if gate else None
        kI = torch.randn(P.B, L, P.dI, generator=self.gen) * P.dI ** -0.5
        return [x if x is None else x.to(BF16) for x in (K, V, g2, kI)]

    def append(self, n_new, x=None, gate=True):
        start = self.reserve(n_new)
        K, V, g2, kI = x if x is not None else self.tokens(max(1, int(max(n_new))), gate=gate)
        gsa.gsa_cache_append(self.c, *[t if t is None else t.cuda() for t in (K, V, g2, kI)], i32(n_new), start, self.ws)
        assert self.status() == 0
        self.plain.append(f64(K), f64(V), None if g2 is None else f64(g2), kI.view(torch.int16).numpy().view(np.uint16), n_new,
                          start.cpu().numpy())


# ---- storing and reading ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "-".join(map(str, g.values())))
def test_stored_tokens_equal_the_definition(geo, gate):
    B, L = 3, 2 * geo["T"] + 7
    p = Pair(B, 16, 5, **geo, seed=3)
    p.append([geo["T"] + 1, 1, 0], gate=gate)
    p.append([L - geo["T"] - 1, 2, 5], gate=gate)                        # behind a partly filled page, into a fresh one
    p.same_tables()
    p.same_pages()
    # read back: exact values, nothing behind a sequence's end touched
    n = L + 9
    K = torch.full((B, n, geo["n_kv"], geo["d_h"]), 7.0, dtype=BF16, device="cuda")
    V, kI = K.clone(), torch.full((B, n, geo["dI"]), 7.0, dtype=BF16, device="cuda")
    gsa.gsa_cache_read(p.c, K, V, kI, p.ws)
    assert p.status() == 0
    for b in range(B):
        m = int(p.plain.lens[b])
        for got, want in zip((K, V, kI), p.plain.tokens(b, np.arange(m))):
            assert np.array_equal(f64(got[b, :m]), want)
            assert (got[b, m:] == 7.0).all()
    # any of the three alone, and fewer positions than a sequence has
    V2 = torch.full((B, 5, geo["n_kv"], geo["d_h"]), 7.0, dtype=BF16, device="cuda")
    gsa.gsa_cache_read(p.c, None, V2, None, p.ws)
    assert torch.equal(V2, V[:, :5])


def test_values_at_the_borders_of_the_format():
    """Halves between codes and between scales, zeros, the smallest and largest scales, infinities and NaN, gates that close."""
    geo = GEOMETRIES[1]
    p = Pair(1, 64, 64, **geo, seed=4)
    rows = []
    g = np.zeros(64)
    rows.append(g.copy())                                                # zeros: the smallest scale, code 0
    for scale in (1.0, 1.125, 1.875 * 2.0 ** 11, 1.75 * 2.0 ** 11, 2.0 ** -20, 2.0 ** -21, 2.0 ** -30, 3e38, 2.0 ** 40):
        x = np.tile(np.arange(-7.5, 8.0, 1.0), 4) * scale                # every half step; 7.5 sets the scale
        x[::16] = 7 * scale
        rows.append(x)
        rows.append(np.tile(np.linspace(-7, 7, 16), 4) * scale)
    for m in range(8):                                                   # max / 7 halfway between two scales
        x = np.linspace(-1, 1, 64)
        x[::16] = 7 * (17 + 2 * m) / 16
        rows.append(x)
    for bad in (np.inf, -np.inf, np.nan):
        x = np.linspace(-1, 1, 64)
        x[20] = bad
        rows.append(x)
    x = torch.tensor(np.stack(rows)).to(BF16).view(1, -1, 1, 64)
    n = x.shape[1]
    kI = torch.zeros(1, n, geo["dI"], dtype=BF16)
    g2 = torch.tensor([0.0, 90.0, -90.0, 30.0, -30.0, 200.0, -200.0, float("inf"), float("-inf"), float("nan")] * 20).to(BF16)
    g2 = g2[:64].repeat(n, 1).view(1, n, 1, 64)
    p.append([n], x=(x, x, None, kI))
    p.append([n], x=(x, x, g2, kI))
    p.same_pages()


def test_gated_values_are_rounded_correctly():
    """4 million gated values: the codes are those of the 64-bit product rounded to bf16, also next to a border."""
    geo = dict(n_kv=8, d_h=128, dI=64, T=128)
    p = Pair(1, 40, 40, **geo, seed=5)
    n = 512
    K, V, _, kI = p.tokens(n, gate=False)
    # every finite bf16 logit between -88 and 88 in turn
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16)
    every = every[every.isfinite() & (every.abs() <= 88)]
    for i in range(8):
        at = (torch.arange(V.numel()) + i * V.numel()) % every.numel()
        p.append([n], x=(K, V, every[at].view(V.shape), kI))
        V = (V.float() * 1.37).to(BF16)
    p.same_pages()


def test_append_skips_what_it_must_not_write():
    geo = GEOMETRIES[1]
    p = Pair(3, 12, 4, **geo, seed=6)
    p.append([20, 16, 5])
    before = p.pool.clone()
    K, V, g2, kI = [t.cuda() for t in p.tokens(3)]
    one = i32([1, 1, 1])

    def put(start, n_new=one):
        gsa.gsa_cache_append(p.c, K, V, g2, kI, n_new, i32(start), p.ws)
        return p.status()

    assert put([-1, -1, -1]) == 0 and torch.equal(p.pool, before)        # refused by the reservation: left out
    assert put([20, 16, 5]) == 6 and torch.equal(p.pool, before)         # behind the ends
    assert put([2 ** 31 - 1, 2 ** 24, 100000]) == 6 and torch.equal(p.pool, before)
    assert put([-1, -1, -1], i32([0, -5, 2 ** 31 - 1])) == 0 and torch.equal(p.pool, before)
    assert put([19, 15, 4], i32([0, -5, 0])) == 0 and torch.equal(p.pool, before)
    gsa.gsa_cache_release(p.c, i32([0, 0, 1]), p.ws)
    p.plain.release([0, 0, 1])
    src = [-1, -1, 0]
    gsa.gsa_cache_fork(p.c, i32(src), True, p.ws)
    assert p.status() == p.plain.fork(src, True) == 0
    p.same_tables()
    before = p.pool.clone()
    assert put([3, -1, -1]) == 6 and torch.equal(p.pool, before)         # a shared page
    p.table[1, 0] = 12                                                   # no page of the pool
    assert put([-1, 3, -1]) == 6 and torch.equal(p.pool, before)
    p.table[1, 0] = -1
    assert put([-1, 3, -1]) == 6 and torch.equal(p.pool, before)


# ---- pages -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("seed", range(6))
def test_runs_of_page_calls_follow_the_plain_tables(seed):
    """Reservations, forks (shared and copied), releases and compactions in random order, refused ones among them."""
    rng = np.random.default_rng(seed)
    geo = GEOMETRIES[[1, 2, 5][seed % 3]]
    B, n_pages, max_pages = int(rng.integers(2, 40)), int(rng.integers(20, 300)), int(rng.integers(4, 30))
    p = Pair(B, n_pages, max_pages, **geo, seed=seed)
    live = torch.full((1,), -7, dtype=I32, device="cuda")
    seen = set()
    for step in range(40):
        kind = ["append", "append", "fork", "release", "compact"][int(rng.integers(5))]
        if kind == "append":
            n = rng.integers(0, geo["T"] * 2, B) * (rng.random(B) < 0.4)
            if rng.random() < 0.7:
                n = np.minimum(n, max_pages * geo["T"] - p.plain.lens)
            start = p.reserve(n)
            seen.add(("reserve", p.status()))
            if (start.cpu().numpy() >= 0).all() and n.max() > 0:
                x = p.tokens(int(n.max()))
                gsa.gsa_cache_append(p.c, *[t.cuda() for t in x], i32(n), start, p.ws)
                assert p.status() == 0
                p.plain.append(f64(x[0]), f64(x[1]), f64(x[2]), x[3].view(torch.int16).numpy().view(np.uint16), n, start.cpu().numpy())
        elif kind == "fork":
            src = np.full(B, -1)
            empty, full = np.flatnonzero(p.plain.lens == 0), np.flatnonzero(p.plain.lens > 0)
            if len(full) and len(empty):
                for b in empty[:int(rng.integers(1, 5))]:
                    src[b] = rng.choice(full)
            if rng.random() < 0.15:
                src[int(rng.integers(B))] = int(rng.integers(-3, B + 3))         # often not allowed
            share = bool(rng.random() < 0.6)
            gsa.gsa_cache_fork(p.c, i32(src), share, p.ws)
            want = p.plain.fork(src, share)
            assert p.status() == want
            seen.add(("fork", want))
        elif kind == "release":
            drop = (rng.random(B) < 0.25).astype(np.int32) * 5
            gsa.gsa_cache_release(p.c, i32(drop), p.ws)
            assert p.status() == p.plain.release(drop)
        else:
            gsa.gsa_cache_compact(p.c, live, p.ws)
            assert p.status() == 0
            assert int(live) == p.plain.compact()
        p.same_tables()
        p.same_pages()
    assert ("reserve", 0) in seen


def test_refused_calls_change_nothing():
    geo = GEOMETRIES[1]
    p = Pair(4, 10, 6, **geo, seed=8)
    p.append([40, 16, 0, 0])                                             # 3 + 1 pages, 6 are free
    for n in ([0, 0, 96, 1], [1, 0, -1, 0], [57, 0, 0, 0], [2 ** 31 - 1, 0, 0, 0], [-2 ** 31, 0, 0, 0]):
        p.reserve(n)                                                     # compares status, start and tables
    # onto a sequence that has tokens, onto itself, from no sequence, from a copy of this call
    for src, share in (([-1, 0, -1, -1], True), ([-1, -1, 2, -1], True), ([-1, -1, 4, -1], True), ([-1, -1, 3, 0], True),
                       ([-1, -1, 2 ** 31 - 1, -1], False)):
        gsa.gsa_cache_fork(p.c, i32(src), share, p.ws)
        assert p.status() == p.plain.fork(src, share) == 6
        p.same_tables()
    # two copies of three pages take all six
    gsa.gsa_cache_fork(p.c, i32([-1, -1, 0, 0]), False, p.ws)
    assert p.status() == p.plain.fork([-1, -1, 0, 0], False) == 0
    p.same_tables()
    gsa.gsa_cache_release(p.c, i32([0, 0, 1, 1]), p.ws)
    p.plain.release([0, 0, 1, 1])
    p.reserve([0, 80, 0, 0])                                             # 5 of the 6
    gsa.gsa_cache_fork(p.c, i32([-1, -1, 0, -1]), False, p.ws)
    assert p.status() == p.plain.fork([-1, -1, 0, -1], False) == 7
    p.same_tables()
    assert gsa.lib().gsa_device_status(gsa._dp(p.ws), gsa._stream(None), None) == -8


def test_large_pools_and_batches():
    """As many sequences and pages as a call takes: every thread and word of the plan has work."""
    B, n_pages, T = 4096, 1 << 20, 16
    table = torch.full((B, 300), -1, dtype=I32, device="cuda")
    lens, refs = torch.zeros(B, dtype=I32, device="cuda"), torch.zeros(n_pages, dtype=I32, device="cuda")
    geo = dict(page_tokens=T, n_kv=1, d_h=64, dI=32)
    bytes_ = gsa.gsa_cache_page_bytes(gsa.cache_geometry(B=B, n_pages=n_pages, max_pages=300, **geo))
    pool = torch.zeros(n_pages * bytes_, dtype=torch.uint8, device="cuda")
    c = gsa.make_cache(pool, table, lens, refs, **geo)
    ws = torch.empty(gsa.gsa_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    start, live = torch.empty(B, dtype=I32, device="cuda"), torch.empty(1, dtype=I32, device="cuda")
    rng = np.random.default_rng(10)
    n1 = rng.integers(0, 255 * T, B).astype(np.int32)
    gsa.gsa_cache_reserve(c, i32(n1), start, ws)
    assert gsa.gsa_device_status(ws) == 0
    need = -(-n1 // T)
    off = np.cumsum(need) - need
    t = table.cpu().numpy()
    for b in range(0, B, 97):
        assert np.array_equal(t[b, :need[b]], off[b] + np.arange(need[b])) and (t[b, need[b]:] == -1).all()
    r = refs.cpu().numpy()
    assert (r[:need.sum()] == 1).all() and (r[need.sum():] == 0).all()
    # more than there is: 4096 times 1400 pages behind what a row of a wider table holds
    wide = torch.full((B, 1700), -1, dtype=I32, device="cuda")
    wide[:, :300] = table
    cw = gsa.make_cache(pool, wide, lens, refs, **geo)
    gsa.gsa_cache_reserve(cw, i32(np.full(B, 1400 * T)), start, ws)
    assert gsa.gsa_device_status(ws) == 7 and (start == -1).all() and torch.equal(refs.cpu(), torch.from_numpy(r))
    assert torch.equal(wide[:, :300], table) and (wide[:, 300:] == -1).all() and np.array_equal(lens.cpu().numpy(), n1)
    # every third ends; the rest moves to the front
    mark = pool.view(n_pages, -1)[:, :4].view(torch.int32)
    mark.copy_(torch.arange(n_pages, device="cuda", dtype=I32)[:, None])
    drop = (np.arange(B) % 3 == 0).astype(np.int32)
    gsa.gsa_cache_release(c, i32(drop), ws)
    gsa.gsa_cache_compact(c, live, ws)
    assert gsa.gsa_device_status(ws) == 0
    n = int(need[drop == 0].sum())
    assert int(live) == n
    t2, r2, m = table.cpu().numpy(), refs.cpu().numpy(), mark.cpu().numpy()[:, 0]
    assert (r2[:n] == 1).all() and (r2[n:] == 0).all()
    for b in range(1, B, 97):
        if not drop[b]:
            assert np.array_equal(m[t2[b, :need[b]]], t[b, :need[b]])    # the page's bytes went with it
    assert sorted(t2[t2 >= 0].tolist()) == list(range(n))


# ---- indexer and selection ---------------------------------------------------------------------------------------------------
def _filled(geo, lens, seed, n_pages=None, extra=0):
    pages = sum(-(-n // geo["T"]) for n in lens)
    p = Pair(len(lens), (n_pages or pages + 5) + extra, max(1, max(-(-n // geo["T"]) for n in lens)), **geo, seed=seed)
    # pages scattered over the pool: reserve in two turns, the second behind the first of all sequences
    first = [n // 2 for n in lens]
    if max(first):
        p.append(first)
    p.append([n - f for n, f in zip(lens, first)])
    return p


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("geo,HI,Lq,lens", [(GEOMETRIES[0], 8, 1, [700, 0, 1, 64, 65]), (GEOMETRIES[1], 4, 2, [300, 1, 2, 0]),
                                            (GEOMETRIES[2], 1, 4, [130, 3, 4]), (GEOMETRIES[3], 2, 7, [513, 6])])
def test_indexer_scores_over_pages(geo, HI, Lq, lens, act):
    p = _filled(geo, lens, 11)
    B, Lk = len(lens), max(lens) + 3 if max(lens) + 3 <= p.plain.max_pages * geo["T"] else max(lens)
    gp = gsa.make_params(B=B, Lq=Lq, Lk=Lk, n_h=geo["n_kv"], n_kv=geo["n_kv"], d_h=geo["d_h"], HI=HI, dI=geo["dI"], act=act)
    qI = torch.randn(B, Lq, HI, geo["dI"], generator=p.gen).to(BF16)
    w, bI = torch.rand(B, Lq, HI, generator=p.gen), torch.randn(HI, generator=p.gen) * 0.2
    stride = (Lk + 35) // 4 * 4
    sc = torch.full((B, Lq, stride), float("nan"), device="cuda")
    gsa.gsa_cache_indexer_scores(p.c, gp, qI.cuda(), w.cuda(), bI.cuda(), sc, stride, p.ws)
    assert p.status() == 0
    got = sc.cpu().numpy()
    for b in range(B):
        for t in range(Lq):
            want = p.plain.scores(b, t, Lq, f64(qI[b, t]), f64(w[b, t]), f64(bI), act)
            n = len(want)
            assert np.isnan(got[b, t, n:]).all()
            # sum_i w_i: at most HI; a product sum of at most 64 terms: 64 * 2^-24 * sum |q k|, below 64 here; sigmoid 2^-20
            tol = HI * (64 * 2.0 ** -24 * 64 * (1.0 if act else 0.25) + 2.0 ** -20)
            assert np.abs(got[b, t, :n] - want).max(initial=0) <= tol


def test_scores_equal_those_over_the_contiguous_keys():
    """Sequences of one length: bit for bit what gsa_indexer_scores gives on the keys read out."""
    geo = GEOMETRIES[0]
    p = _filled(geo, [1000] * 3, 12)
    B, Lq, Lk = 3, 2, 1000
    gp = gsa.make_params(B=B, Lq=Lq, Lk=Lk, n_h=16, n_kv=8, d_h=128, HI=8, dI=64)
    kI = torch.empty(B, Lk, 64, dtype=BF16, device="cuda")
    gsa.gsa_cache_read(p.c, None, None, kI, p.ws)
    qI, w = torch.randn(B, Lq, 8, 64, generator=p.gen).to(BF16).cuda(), torch.rand(B, Lq, 8, generator=p.gen).cuda()
    a, b = torch.zeros(B, Lq, Lk, device="cuda"), torch.zeros(B, Lq, Lk, device="cuda")
    gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, None, a, Lk, p.ws)
    gsa.gsa_indexer_scores(gp, qI, kI, w, None, b, Lk, p.ws)
    assert torch.equal(a, b)


def _plain_topk(row, n, p):
    x = row[:n].astype(np.float64)
    if n <= 0:
        return [], 0, 0.0
    var = max(0.0, (x * x).mean() - x.mean() ** 2)
    r = {0: p.k_base * var / p.v_bar, 1: p.k_base * p.v_bar / var if var > 0 else 1e300, 2: p.k_base}[p.k_mode]
    k = min(n, int(min(max(np.floor(r), p.k_min), p.k_max)))
    order = np.lexsort((np.arange(n), -x))[:k]
    return np.sort(order).tolist(), k, var


@pytest.mark.parametrize("k_mode", [0, 2])
@pytest.mark.parametrize("B,Lq,lens", [(4, 1, [3000, 0, 1, 17]), (3, 4, [5000, 3, 8000]), (2, 2, [16384, 9000]), (5, 1, [40000, 16385, 100, 0, 16384]),
                                       (60, 1, [20000 if b % 3 else 900 * (b % 7) for b in range(60)]), (1, 1, [131072 + 500])])
def test_topk_with_lengths_of_its_own(B, Lq, lens, k_mode):
    """Every launch shape: rows in registers of 128, 256 and 512 threads, clusters, rows split between two launches by length."""
    T = 128
    Lk = max(lens)
    geo = dict(page_tokens=T, n_kv=1, d_h=64, dI=32)
    table = torch.full((B, -(-Lk // T)), -1, dtype=I32, device="cuda")
    refs = torch.zeros(1, dtype=I32, device="cuda")
    pool = torch.zeros(gsa.gsa_cache_page_bytes(gsa.cache_geometry(B=B, n_pages=1, max_pages=1, **geo)), dtype=torch.uint8, device="cuda")
    c = gsa.make_cache(pool, table, i32(lens), refs, **geo)              # (the selection looks at the lengths alone)
    gen = torch.Generator().manual_seed(B * 7 + Lq)
    stride = (Lk + 3) // 4 * 4
    sc = torch.rand(B, Lq, stride, generator=gen)
    sc[:, :, ::5] = (sc[:, :, ::5] * 8).round() / 8                      # ties
    for b, n in enumerate(lens):
        for t in range(Lq):
            sc[b, t, max(0, n - Lq + t + 1):] = float("nan")             # nothing behind a row's end may count
    gp = gsa.make_params(B=B, Lq=Lq, Lk=Lk, n_h=1, n_kv=1, d_h=64, HI=1, dI=32, k_base=700, k_min=5, k_max=1000, v_bar=0.09, k_mode=k_mode)
    idx = torch.full((B, Lq, gp.k_max), -7, dtype=I32, device="cuda")
    kt, var = torch.full((B, Lq), -7, dtype=I32, device="cuda"), torch.full((B, Lq), -7.0, device="cuda")
    ws = torch.empty(gsa.gsa_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_topk(c, gp, sc.cuda(), stride, idx, kt, var, ws)
    torch.cuda.synchronize()
    idx, kt, var = idx.cpu().numpy(), kt.cpu().numpy(), var.cpu().numpy()
    for b, n in enumerate(lens):
        for t in range(Lq):
            want, k, v = _plain_topk(sc[b, t].numpy(), n - Lq + t + 1, gp)
            # (k_base * var / v_bar is never this close to an integer here: the sums differ by 1e-12)
            assert kt[b, t] == k, (b, t, kt[b, t], k)
            assert idx[b, t, :k].tolist() == want and (idx[b, t, k:] == -1).all(), (b, t)
            assert abs(var[b, t] - v) <= 2.0 ** -23 * v


# ---- attention ---------------------------------------------------------------------------------------------------------------
def _attend(p, G, Lq, sets, k_max, sm_scale=0.0, qscale=1.0, Lk=None, seed=0):
    """sets[b][t]: positions.  Runs the kernel and compares every row."""
    P = p.plain
    B, n_h = P.B, P.n_kv * G
    gen = torch.Generator().manual_seed(seed)
    Q = (torch.randn(B, Lq, n_h, P.d_h, generator=gen) * qscale).to(BF16)
    g1 = torch.randn(B, Lq, n_h, P.d_h, generator=gen).to(BF16)
    idx = np.full((B, Lq, k_max), -1, np.int32)
    kt = np.zeros((B, Lq), np.int32)
    for b in range(B):
        for t in range(Lq):
            kt[b, t] = len(sets[b][t])
            idx[b, t, :kt[b, t]] = sets[b][t]
    gp = gsa.make_params(B=B, Lq=Lq, Lk=Lk or max(Lq, int(P.lens.max())), n_h=n_h, n_kv=P.n_kv, d_h=P.d_h, HI=1, dI=P.dI, k_base=1, k_min=1,
                         k_max=k_max, sm_scale=sm_scale)
    out = torch.full((B, Lq, n_h, P.d_h), float("nan"), dtype=BF16, device="cuda")
    ws = torch.full((gsa.gsa_cache_attn_workspace_bytes(gp),), 0xFF, dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, Q.cuda(), g1.cuda(), i32(idx), i32(kt), out, ws)
    status = gsa.gsa_device_status(ws)
    return Q, g1, out, status, gp


def _check_rows(p, Q, g1, out, sets, Lq, sm_scale, rows=None):
    P = p.plain
    got = f64(out)
    for b in range(P.B):
        for t in range(Lq):
            if rows is not None and (b, t) not in rows:
                continue
            q = f64(Q[b, t])
            want, mag = P.attn(b, q, f64(g1[b, t]), sets[b][t], sm_scale)
            if len(sets[b][t]):
                K, V, _ = [np.abs(x) for x in P.tokens(b, np.asarray(sets[b][t]))]
                tiny = 2.0 ** -32 * np.repeat(V.sum(0), q.shape[0] // P.n_kv, 0)
                z = max(np.abs(q[h]) @ K[:, h // (q.shape[0] // P.n_kv)].T.max(1) for h in range(q.shape[0])) * sm_scale
            else:
                z = tiny = 0.0
            tol = (2.0 ** -11 * mag + 2.0 ** -8 * np.abs(want)) * 1.01 + mag * (2 * (128 * 2.0 ** -24 * z + 2.0 ** -21)) + tiny + 1e-30
            assert (np.abs(got[b, t] - want) <= tol).all(), (b, t, (np.abs(got[b, t] - want) / tol).max())


def _random_sets(rng, lens, Lq, sizes, sort=True):
    out = []
    i = 0
    for n in lens:
        row = []
        for t in range(Lq):
            vis = max(0, n - Lq + t + 1)
            k = min(vis, sizes[i % len(sizes)])
            i += 1
            s = rng.choice(vis, k, replace=False) if k else np.zeros(0, np.int64)
            row.append(np.sort(s) if sort else s)
        out.append(row)
    return out


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "-".join(map(str, g.values())))
def test_attention_of_every_head_layout(geo, G):
    lens = [200, 0, 1, 77]
    p = _filled(geo, lens, 13)
    sets = _random_sets(np.random.default_rng(1), lens, 1, [90, 1, 1, 33])
    Q, g1, out, status, _ = _attend(p, G, 1, sets, 96)
    assert status == 0
    _check_rows(p, Q, g1, out, sets, 1, geo["d_h"] ** -0.5)


@pytest.mark.parametrize("Lq", [1, 3])
@pytest.mark.parametrize("size", [1, 15, 16, 17, 31, 32, 33, 64, 300, 1000])
def test_attention_of_every_set_size(size, Lq):
    geo = GEOMETRIES[2]
    lens = [1100, 40, 700]
    p = _filled(geo, lens, 14)
    sets = _random_sets(np.random.default_rng(size), lens, Lq, [size, max(1, size // 2), size], sort=size % 2 == 0)
    Q, g1, out, status, _ = _attend(p, 2, Lq, sets, max(size, 4))
    assert status == 0
    _check_rows(p, Q, g1, out, sets, Lq, geo["d_h"] ** -0.5)


def test_attention_of_a_long_set_and_of_empty_rows():
    geo = GEOMETRIES[0]
    lens = [4500, 0, 10, 4500, 0]
    p = _filled(geo, lens, 15)
    rng = np.random.default_rng(2)
    sets = [[np.arange(4096)], [[]], [[]], [np.sort(rng.choice(4500, 2500, replace=False))], [[]]]
    Q, g1, out, status, _ = _attend(p, 2, 1, sets, 4096)
    assert status == 0
    _check_rows(p, Q, g1, out, sets, 1, 128 ** -0.5)
    assert (out[1] == 0).all() and (out[2] == 0).all() and (out[4] == 0).all()
    # every set empty
    Q, g1, out, status, _ = _attend(p, 2, 1, [[[]]] * 5, 16)
    assert status == 0 and (out == 0).all()


def test_attention_where_one_key_dominates_and_keys_repeat():
    geo = GEOMETRIES[4]
    p = _filled(geo, [500], 16)
    rng = np.random.default_rng(3)
    s = rng.choice(500, 300)                                             # repeats, in any order: each counts
    Q, g1, out, status, _ = _attend(p, 4, 1, [[s]], 300, sm_scale=2.0, qscale=3.0)
    assert status == 0
    _check_rows(p, Q, g1, out, [[s]], 1, 2.0)


@pytest.mark.parametrize("rows", [1300, 4096, 5000])
def test_attention_of_many_rows(rows):
    """Rows that are dealt out as tiles (many of them whole in one unit's run) and, beyond 4096, as whole rows."""
    geo = GEOMETRIES[1]
    lens = [700]
    p = _filled(geo, lens, 17)
    rng = np.random.default_rng(4)
    sets = [[np.sort(rng.choice(700, int(rng.integers(0, 50)), replace=False)) for _ in range(rows)]]
    Q, g1, out, status, _ = _attend_many(p, 4, rows, sets, 64)
    assert status == 0
    _check_rows(p, Q, g1, out, sets, rows, 64 ** -0.5, rows={(0, t) for t in list(range(0, rows, 37)) + [rows - 1]})


def _attend_many(p, G, rows, sets, k_max):
    """More rows than the sequence has tokens cannot be asked for as one sequence's rows (Lq <= Lk): the cache's table is widened."""
    P = p.plain
    wide = -(-rows // P.T)
    p.table = torch.cat([p.table, torch.full((P.B, wide), -1, dtype=I32, device="cuda")], 1).contiguous()
    p.c = gsa.make_cache(p.pool, p.table, p.lens, p.refs, page_tokens=P.T, n_kv=P.n_kv, d_h=P.d_h, dI=P.dI)
    return _attend(p, G, rows, sets, k_max, Lk=rows)


def test_nan_shows_where_it_is_selected_and_only_there():
    geo = GEOMETRIES[0]
    p = _filled(geo, [100, 100], 18)
    K, V, g2, kI = p.tokens(1, gate=False)
    K[0, 0, 3, 20] = float("nan")
    V[1, 0, 2, 100] = float("inf")
    p.append([1, 1], x=(K, V, None, kI))
    with_, without = [[np.array([5, 100, 7])], [np.array([100, 3, 4])]], [[np.array([5, 7])], [np.array([99, 3, 4])]]
    _, _, out, status, _ = _attend(p, 2, 1, with_, 8)
    o = out.float().cpu()
    assert status == 0
    assert o[0, 0, 6:8].isnan().all() and o[0, 0, :6].isfinite().all() and o[0, 0, 8:].isfinite().all()
    assert o[1, 0, 4:6, 96:112].isnan().all()                            # the 16 values that share the infinity's scale
    assert o[1, 0, 4:6, :96].isfinite().all() and o[1, 0, 4:6, 112:].isfinite().all() and o[1, 0, :4].isfinite().all()
    Q, g1, out, status, _ = _attend(p, 2, 1, without, 8)
    assert status == 0
    _check_rows(p, Q, g1, out, without, 1, 128 ** -0.5)


@pytest.mark.parametrize("damage", ["too_large", "negative", "budget", "page", "no_page", "length"])
def test_corrupt_sets_and_tables_are_reported_not_followed(damage):
    geo = GEOMETRIES[1]
    p = _filled(geo, [100, 60], 19)
    sets = [[np.arange(40)], [np.arange(20)]]
    if damage == "too_large":
        sets[1][0][7] = 2 ** 31 - 1
    if damage == "negative":
        sets[1][0][7] = -2 ** 31
    if damage == "page":
        p.table[1, 1] = 2 ** 31 - 1
    if damage == "no_page":
        p.table[1, 0] = -1
    if damage == "length":
        p.lens[1] = 2 ** 31 - 1
    P = p.plain
    Q, g1, out, status, gp = _attend(p, 4, 1, sets, 40)
    if damage == "budget":
        ws = torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
        idx = torch.zeros(2, 1, 40, dtype=I32, device="cuda")
        gsa.gsa_cache_attn_fwd(p.c, gp, Q.cuda(), g1.cuda(), idx, i32([[41], [-5]]), out, ws)
        status = gsa.gsa_device_status(ws)
        assert (out[1] == 0).all()
    else:
        _check_rows(p, Q, g1, out, sets, 1, 64 ** -0.5, rows={(0, 0)})   # the other row is as it was
    assert status == 6
    assert out.float().isfinite().all()
    if damage in ("page", "no_page", "length"):
        x = [torch.empty(2, 64, 1, 64, dtype=BF16, device="cuda"), torch.empty(2, 64, 1, 64, dtype=BF16, device="cuda"),
             torch.empty(2, 64, 32, dtype=BF16, device="cuda")]
        gsa.gsa_cache_read(p.c, *x, p.ws)
        assert p.status() == 6
        sc = torch.zeros(2, 1, 104, device="cuda")
        gsa.gsa_cache_indexer_scores(p.c, gp, torch.ones(2, 1, 1, 32, dtype=BF16, device="cuda"), torch.ones(2, 1, 1, device="cuda"),
                                     None, sc, 104, p.ws)
        assert p.status() == 6


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "-".join(map(str, g.values())))
def test_attention_of_large_sets_of_every_head_layout(geo, G):
    """Sets too large for a CTA of their own: runs of tiles over all SMs, rows cut anywhere, empty rows between them."""
    lens = [1300, 0, 5, 900, 0, 0, 401, 1300]
    p = _filled(geo, lens, 40 + G)
    sets = _random_sets(np.random.default_rng(G), lens, 2, [1200, 700, 1, 1, 3, 16, 899, 17, 1, 1, 0, 9, 400, 33, 1111, 1200], sort=G > 2)
    Q, g1, out, status, _ = _attend(p, G, 2, sets, 1200)
    assert status == 0
    _check_rows(p, Q, g1, out, sets, 2, geo["d_h"] ** -0.5)
    assert all((out[b, t] == 0).all() for b in range(8) for t in range(2) if len(sets[b][t]) == 0)


@pytest.mark.parametrize("rows", [30, 73, 74, 148, 149])
@pytest.mark.parametrize("k_max", [32, 33, 64, 65, 128, 129])
def test_attention_on_both_sides_of_the_row_split(rows, k_max):
    """Eight KV heads: two units a CTA, so that sets of 32 keys (128, where rows fill half the SMs) end the form with a CTA for each row."""
    geo = GEOMETRIES[5]
    p = _filled(geo, [rows + 150], 41)
    sets = _random_sets(np.random.default_rng(k_max), [rows + 150], rows, [k_max, k_max, 1, 0, k_max - 15, min(k_max, 33)])
    Q, g1, out, status, _ = _attend(p, 2, rows, sets, k_max)
    assert status == 0
    _check_rows(p, Q, g1, out, sets, rows, 64 ** -0.5, rows={(0, t) for t in list(range(0, rows, 11)) + [rows - 2, rows - 1]})
    assert not out.isnan().any()


@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("k_max", [24, 600])
def test_queries_that_are_not_finite_stay_in_their_head(G, k_max):
    geo = GEOMETRIES[3]
    p = _filled(geo, [700, 650], 42)
    sets = _random_sets(np.random.default_rng(G), [700, 650], 1, [k_max, k_max - 3])
    n_h = 4 * G
    Q = torch.randn(2, 1, n_h, 128, generator=p.gen).to(BF16)
    spoilt = Q.clone()
    spoilt[0, 0, 1, 5], spoilt[0, 0, n_h - 1, 127], spoilt[1, 0, 0, 64] = float("inf"), float("nan"), -float("inf")
    g1 = torch.randn(2, 1, n_h, 128, generator=p.gen).to(BF16)
    idx, kt = np.full((2, 1, k_max), -1, np.int32), np.zeros((2, 1), np.int32)
    for b in range(2):
        kt[b, 0] = len(sets[b][0])
        idx[b, 0, :kt[b, 0]] = sets[b][0]
    gp = gsa.make_params(B=2, Lq=1, Lk=700, n_h=n_h, n_kv=4, d_h=128, HI=1, dI=32, k_base=1, k_min=1, k_max=k_max)
    ws = torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
    out = torch.zeros(2, 1, n_h, 128, dtype=BF16, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, spoilt.cuda(), g1.cuda(), i32(idx), i32(kt), out, ws)
    assert gsa.gsa_device_status(ws) == 0
    for b, h in ((0, 1), (0, n_h - 1), (1, 0)):
        assert out[b, 0, h].isnan().all()
        out[b, 0, h], Q[b, 0, h] = 0.0, 0.0
        g1[b, 0, h] = -float("inf")                                      # (its row of the plain form: zeros)
    _check_rows(p, Q, g1, out, sets, 1, 128 ** -0.5)


@pytest.mark.parametrize("exponent", [-100, -20, 20, 40])
def test_queries_of_any_magnitude(exponent):
    """Scores are formed from Q times a power of two: very small and very large ones, heads of one group far apart, as exactly as others."""
    geo = GEOMETRIES[4]
    p = _filled(geo, [300], 43)
    Q = torch.randn(1, 1, 4, 128, generator=p.gen) * 2.0 ** exponent
    Q[0, 0, 1] *= 2.0 ** -10
    g1 = torch.randn(1, 1, 4, 128, generator=p.gen).to(BF16)
    gp = gsa.make_params(B=1, Lq=1, Lk=300, n_h=4, n_kv=1, d_h=128, HI=1, dI=64, k_base=1, k_min=1, k_max=300, sm_scale=2.0 ** -(exponent + 4))
    out, ws = torch.zeros(1, 1, 4, 128, dtype=BF16, device="cuda"), torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
    Q, s = Q.to(BF16), np.arange(0, 300, 2)
    idx = np.full((1, 1, 300), -1, np.int32)
    idx[0, 0, :150] = s
    gsa.gsa_cache_attn_fwd(p.c, gp, Q.cuda(), g1.cuda(), i32(idx), i32([[150]]), out, ws)
    assert gsa.gsa_device_status(ws) == 0
    _check_rows(p, Q, g1, out, [[s]], 1, 2.0 ** -(exponent + 4))


def test_a_sequence_longer_than_the_bound_is_reported_and_cut():
    geo = GEOMETRIES[1]
    p = _filled(geo, [100, 60], 44)
    gp = gsa.make_params(B=2, Lq=1, Lk=64, n_h=1, n_kv=1, d_h=64, HI=1, dI=32, k_base=8, k_min=8, k_max=8, k_mode=2)
    qI, w = torch.randn(2, 1, 1, 32, generator=p.gen).to(BF16).cuda(), torch.ones(2, 1, 1, device="cuda")
    sc = torch.full((2, 1, 68), float("nan"), device="cuda")
    gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, None, sc, 68, p.ws)
    assert p.status() == 6
    assert sc[0, 0, :64].isfinite().all() and sc[0, 0, 64:].isnan().all() and sc[1, 0, :60].isfinite().all() and sc[1, 0, 60:].isnan().all()
    idx, kt = torch.full((2, 1, 8), -7, dtype=I32, device="cuda"), torch.zeros(2, 1, dtype=I32, device="cuda")
    gsa.gsa_cache_topk(p.c, gp, sc, 68, idx, kt, None, p.ws)
    assert p.status() == 6 and (kt == 8).all() and int(idx.max()) < 64 and int(idx.min()) >= 0
    for b, n in ((0, 64), (1, 60)):
        assert idx[b, 0].tolist() == torch.sort(torch.sort(sc[b, 0, :n], descending=True, stable=True).indices[:8]).values.tolist()
    Q = torch.randn(2, 1, 1, 64, generator=p.gen).to(BF16).cuda()
    out, ws = torch.zeros_like(Q), torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, ws)
    assert gsa.gsa_device_status(ws) == 6 and out.isfinite().all()
    # and a negative length: nothing visible, reported by all three
    p.lens[0] = -3
    gsa.gsa_cache_topk(p.c, gp, sc, 68, idx, kt, None, p.ws)
    assert p.status() == 6 and kt.flatten().tolist() == [0, 8] and (idx[0] == -1).all()
    gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, None, sc, 68, p.ws)
    assert p.status() == 6
    # the next call that finds nothing wrong says so
    p.lens[0] = 64
    gsa.gsa_cache_topk(p.c, gp, sc, 68, idx, kt, None, p.ws)
    assert p.status() == 0
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, out, ws)
    assert gsa.gsa_device_status(ws) == 0


@pytest.mark.parametrize("k_mode", [1, 3])
def test_topk_of_the_other_budget_rules(k_mode):
    B, lens, T = 5, [900, 0, 1, 60, 1000], 128
    geo = dict(page_tokens=T, n_kv=1, d_h=64, dI=32)
    table, refs = torch.full((B, 8), -1, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    pool = torch.zeros(gsa.gsa_cache_page_bytes(gsa.cache_geometry(B=B, n_pages=1, max_pages=1, **geo)), dtype=torch.uint8, device="cuda")
    c = gsa.make_cache(pool, table, i32(lens), refs, **geo)
    sc = torch.rand(B, 1, 1000, generator=torch.Generator().manual_seed(5))
    gp = gsa.make_params(B=B, Lq=1, Lk=1000, n_h=1, n_kv=1, d_h=64, HI=1, dI=32, k_base=50, k_min=5, k_max=1000, v_bar=0.09, k_mode=k_mode)
    idx, kt = torch.full((B, 1, 1000), -7, dtype=I32, device="cuda"), torch.zeros(B, 1, dtype=I32, device="cuda")
    ws = torch.empty(gsa.gsa_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_topk(c, gp, sc.cuda(), 1000, idx, kt, None, ws)
    assert gsa.gsa_device_status(ws) == 0
    for b, n in enumerate(lens):
        want, k, _ = (list(range(n)), n, 0.0) if k_mode == 3 else _plain_topk(sc[b, 0].numpy(), n, gp)
        assert int(kt[b, 0]) == k and idx[b, 0, :k].tolist() == want and (idx[b, 0, k:] == -1).all()


def test_workspaces_of_the_size_asked_for_are_enough():
    """Nothing is written behind the bytes that the size queries name."""
    geo = GEOMETRIES[2]
    lens = [500, 40, 0]
    p = _filled(geo, lens, 45)
    n = p.ws.numel()
    guarded = torch.full((n + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
    p.ws = guarded[:n]
    p.append([3, 0, 40])
    # (503 tokens are 16 of 23 pages, 40 are 2: behind the release 5 are free, too few for a copy, enough for one that shares)
    for call, want in ((lambda: gsa.gsa_cache_fork(p.c, i32([-1, -1, -1]), True, p.ws), 0), (lambda: gsa.gsa_cache_release(p.c, i32([0, 1, 0]), p.ws), 0),
                       (lambda: gsa.gsa_cache_fork(p.c, i32([-1, 0, -1]), False, p.ws), 7), (lambda: gsa.gsa_cache_compact(p.c, i32([0]), p.ws), 0),
                       (lambda: gsa.gsa_cache_fork(p.c, i32([-1, 0, -1]), True, p.ws), 0)):
        call()
        assert p.status() == want
    assert (guarded[n:] == 0x5A).all()
    for Lq, k_max, G in ((1, 16, 8), (1, 400, 8), (39, 400, 1), (3, 37, 4)):
        gp = gsa.make_params(B=3, Lq=Lq, Lk=500, n_h=2 * G, n_kv=2, d_h=64, HI=2, dI=64, k_base=30, k_min=1, k_max=k_max, v_bar=0.03)
        n = gsa.gsa_cache_attn_workspace_bytes(gp)
        guarded = torch.full((n + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        Q = torch.randn(3, Lq, 2 * G, 64, generator=p.gen).to(BF16).cuda()
        idx = torch.randint(0, 40, (3, Lq, k_max), dtype=I32, generator=p.gen).cuda()
        kt = torch.full((3, Lq), k_max, dtype=I32, device="cuda")
        gsa.gsa_cache_attn_fwd(p.c, gp, Q, Q, idx, kt, torch.empty_like(Q), guarded[:n])
        torch.cuda.synchronize()
        assert (guarded[n:] == 0x5A).all()


def test_pages_whose_bytes_lie_behind_four_gigabytes():
    """The same tokens in a small pool and at the end of one of 5 GB: the same bits from every call."""
    geo = GEOMETRIES[3]                                                  # 81920 bytes a page
    lens, n_pages = [700, 300], 60000
    small = _filled(geo, lens, 46)
    B, Lq = 2, 1
    K, V = (torch.zeros(B, 700, 4, 128, dtype=BF16, device="cuda") for _ in range(2))
    kI = torch.zeros(B, 700, 32, dtype=BF16, device="cuda")
    gsa.gsa_cache_read(small.c, K, V, kI, small.ws)
    per = gsa.gsa_cache_page_bytes(small.c)
    pool = torch.zeros(n_pages * per, dtype=torch.uint8, device="cuda")
    refs = torch.ones(n_pages, dtype=I32, device="cuda")
    refs[-40:] = 0
    assert (n_pages - 40) * per > 1 << 32
    table, lens_ = torch.full((B, 6), -1, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    c = gsa.make_cache(pool, table, lens_, refs, page_tokens=128, n_kv=4, d_h=128, dI=32)
    ws = torch.empty(gsa.gsa_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    start = torch.zeros(B, dtype=I32, device="cuda")
    gsa.gsa_cache_reserve(c, i32(lens), start, ws)
    gsa.gsa_cache_append(c, K, V, None, kI, i32(lens), start, ws)        # (what was read is stored without loss)
    assert gsa.gsa_device_status(ws) == 0 and int(table.max()) >= n_pages - 40 and int(table[0, 0]) == n_pages - 40
    gp = gsa.make_params(B=B, Lq=Lq, Lk=700, n_h=8, n_kv=4, d_h=128, HI=4, dI=32, k_base=200, k_min=10, k_max=400, v_bar=0.03)
    r = lambda *s: torch.randn(*s, generator=small.gen).to(BF16).cuda()  # noqa: E731
    qI, w, Q, g1 = r(B, 1, 4, 32), torch.rand(B, 1, 4, generator=small.gen).cuda(), r(B, 1, 8, 128), r(B, 1, 8, 128)
    got = []
    for cache, w_ in ((small.c, small.ws), (c, ws)):
        K2, V2, k2 = torch.zeros_like(K), torch.zeros_like(V), torch.zeros_like(kI)
        gsa.gsa_cache_read(cache, K2, V2, k2, w_)
        sc = torch.zeros(B, 1, 704, device="cuda")
        gsa.gsa_cache_indexer_scores(cache, gp, qI, w, None, sc, 704, w_)
        idx, kt = torch.zeros(B, 1, 400, dtype=I32, device="cuda"), torch.zeros(B, 1, dtype=I32, device="cuda")
        gsa.gsa_cache_topk(cache, gp, sc, 704, idx, kt, None, w_)
        out, wa = torch.zeros_like(Q), torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
        gsa.gsa_cache_attn_fwd(cache, gp, Q, g1, idx, kt, out, wa)
        assert gsa.gsa_device_status(wa) == 0
        got.append((K2, V2, k2, sc, idx, kt, out))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.equal(got[0][0], K) and (got[0][5] > 0).all()
    # a copy of a page there, and its way to the front
    gsa.gsa_cache_release(c, i32([0, 1]), ws)
    gsa.gsa_cache_fork(c, i32([-1, 0]), False, ws)
    assert gsa.gsa_device_status(ws) == 0
    K2 = torch.zeros_like(K)
    gsa.gsa_cache_read(c, K2, None, None, ws)
    assert torch.equal(K2[1], K2[0]) and torch.equal(K2[0], K[0])
    refs[:100] = 0
    live = torch.zeros(1, dtype=I32, device="cuda")
    gsa.gsa_cache_compact(c, live, ws)
    assert gsa.gsa_device_status(ws) == 0 and int(live) == n_pages - 40 - 100 + 12 and int(table.max()) < 100
    gsa.gsa_cache_read(c, K2, None, None, ws)
    assert torch.equal(K2[1], K2[0]) and torch.equal(K2[0], K[0])


# ---- as it is used -----------------------------------------------------------------------------------------------------------
def _step(p, gp, x, buf):
    """One decode step: new tokens in, scores, sets, attention."""
    gsa.gsa_cache_reserve(p.c, buf["n_new"], buf["start"], p.ws)
    gsa.gsa_cache_append(p.c, x["K"], x["V"], x["g2"], x["kI"], buf["n_new"], buf["start"], p.ws)
    gsa.gsa_cache_indexer_scores(p.c, gp, x["qI"], x["w"], None, buf["scores"], buf["scores"].shape[-1], p.ws)
    gsa.gsa_cache_topk(p.c, gp, buf["scores"], buf["scores"].shape[-1], buf["idx"], buf["kt"], None, p.ws)
    gsa.gsa_cache_attn_fwd(p.c, gp, x["Q"], x["g1"], buf["idx"], buf["kt"], buf["out"], buf["ws"])


def _step_inputs(p, gp, gen):
    B, P = gp.B, p.plain
    K, V, g2, kI = p.tokens(1)
    n = lambda *s: torch.randn(*s, generator=gen).to(BF16)  # noqa: E731
    return dict(K=K, V=V, g2=g2, kI=kI, qI=n(B, 1, gp.HI, P.dI), w=torch.rand(B, 1, gp.HI, generator=gen), Q=n(B, 1, gp.n_h, P.d_h),
                g1=n(B, 1, gp.n_h, P.d_h))


def _step_buffers(gp):
    new = lambda *s, dtype=I32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    return dict(n_new=torch.ones(gp.B, dtype=I32, device="cuda"), start=new(gp.B), scores=new(gp.B, 1, (gp.Lk + 31) // 32 * 32, dtype=F32),
                idx=new(gp.B, 1, gp.k_max), kt=new(gp.B, 1), out=new(gp.B, 1, gp.n_h, gp.d_h, dtype=BF16),
                ws=new(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8))


def _plain_step(p, gp, x, buf):
    """The plain cache takes the step, then judges what the GPU left in the buffers."""
    P = p.plain
    status, start = P.reserve([1] * gp.B)
    assert status == 0 and np.array_equal(start, buf["start"].cpu().numpy())
    P.append(f64(x["K"]), f64(x["V"]), f64(x["g2"]), x["kI"].cpu().view(torch.int16).numpy().view(np.uint16), [1] * gp.B, start)
    p.same_tables()
    sc, idx, kt = buf["scores"].cpu().numpy(), buf["idx"].cpu().numpy(), buf["kt"].cpu().numpy()
    sets = []
    for b in range(gp.B):
        n = int(P.lens[b])
        want = P.scores(b, 0, 1, f64(x["qI"][b, 0]), f64(x["w"][b, 0]), np.zeros(gp.HI), 0)
        assert np.abs(sc[b, 0, :n] - want).max() <= gp.HI * (64 * 2.0 ** -24 * 16 + 2.0 ** -20)
        s, k, _ = _plain_topk(sc[b, 0], n, gp)
        assert kt[b, 0] == k and idx[b, 0, :k].tolist() == s
        sets.append([np.array(s)])
    _check_rows(p, x["Q"], x["g1"], buf["out"], sets, 1, P.d_h ** -0.5)


def test_decode_steps_with_forks_releases_and_compaction():
    geo = dict(n_kv=2, d_h=64, dI=32, T=16)
    p = Pair(6, 120, 20, **geo, seed=20)
    p.append([100, 33, 0, 7, 0, 160])
    gen = torch.Generator().manual_seed(21)
    gp = gsa.make_params(B=6, Lq=1, Lk=20 * 16, n_h=8, n_kv=2, d_h=64, HI=4, dI=32, k_base=40, k_min=8, k_max=64, v_bar=0.03)
    buf = _step_buffers(gp)
    live = torch.zeros(1, dtype=I32, device="cuda")
    for step in range(12):
        if step == 3:                                                    # a beam that shares, and one that copies
            gsa.gsa_cache_release(p.c, i32([0, 0, 1, 0, 1, 0]), p.ws)
            p.plain.release([0, 0, 1, 0, 1, 0])
            for src, share in (([-1, -1, 0, -1, -1, -1], True), ([-1, -1, -1, -1, 5, -1], False)):
                gsa.gsa_cache_fork(p.c, i32(src), share, p.ws)
                assert p.status() == p.plain.fork(src, share) == 0
        if step == 6:                                                    # the first prompt ends; its pages stay with the beam
            gsa.gsa_cache_release(p.c, i32([1, 0, 0, 0, 0, 0]), p.ws)
            p.plain.release([1, 0, 0, 0, 0, 0])
        if step == 8:
            gsa.gsa_cache_compact(p.c, live, p.ws)
            assert int(live) == p.plain.compact()
        x = {k: v.cuda() for k, v in _step_inputs(p, gp, gen).items()}
        _step(p, gp, x, buf)
        _plain_step(p, gp, x, buf)
    p.same_pages()


def test_captured_steps_share_a_workspace_and_follow_new_inputs():
    """Two captured graphs on one workspace, replayed in turn on another stream, against the plain cache."""
    geo = dict(n_kv=1, d_h=128, dI=64, T=16)
    pairs = [Pair(2, 40, 12, **geo, seed=30), Pair(3, 60, 12, **geo, seed=31)]
    pairs[0].append([50, 3])
    pairs[1].append([70, 20, 0])
    gen = torch.Generator().manual_seed(32)
    ws = torch.zeros(max(p.ws.numel() for p in pairs), dtype=torch.uint8, device="cuda")
    gps = [gsa.make_params(B=p.plain.B, Lq=1, Lk=12 * 16, n_h=4, n_kv=1, d_h=128, HI=8, dI=64, k_base=30, k_min=8, k_max=48, v_bar=0.03) for p in pairs]
    bufs = [_step_buffers(gp) for gp in gps]
    shared = torch.zeros(max(b["ws"].numel() for b in bufs), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    graphs, inputs = [], []
    for p, gp, buf in zip(pairs, gps, bufs):
        p.ws, buf["ws"] = ws, shared
        x = {k: v.cuda() for k, v in _step_inputs(p, gp, gen).items()}
        torch.cuda.synchronize()
        with torch.cuda.stream(side):                                    # one step outside: module loading is no part of a graph
            _step(p, gp, x, buf)
        side.synchronize()
        _plain_step(p, gp, x, buf)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            _step(p, gp, x, buf)
        graphs.append(g)
        inputs.append(x)
    for step in range(4):
        fresh = [_step_inputs(p, gp, gen) for p, gp in zip(pairs, gps)]
        with torch.cuda.stream(side):
            for g, x, f in zip(graphs, inputs, fresh):
                for k in x:
                    x[k].copy_(f[k])
                g.replay()
        side.synchronize()
        for p, gp, x, buf in zip(pairs, gps, inputs, bufs):
            _plain_step(p, gp, x, buf)


def test_same_bits_again():
    geo = GEOMETRIES[0]
    p = _filled(geo, [3000, 1000], 33)
    rng = np.random.default_rng(5)
    sets = [[rng.choice(3000, 2000, replace=False)], [rng.choice(1000, 900, replace=False)]]
    runs = [_attend(p, 2, 1, sets, 2048)[2] for _ in range(4)]
    assert all(torch.equal(runs[0], r) for r in runs[1:])


def test_chunked_prefill_reads_the_cache_back():
    """A chunk of rows against the cache: read out, then the existing path on contiguous tensors; the 4-bit attention on the same sets
    differs from it by the two kernels' roundings alone (the other rounds its probabilities to bf16: 2^-8 of sum a |v|)."""
    geo = GEOMETRIES[0]
    Lk, Lq = 600, 40
    p = _filled(geo, [Lk], 34)
    gp = gsa.make_params(B=1, Lq=Lq, Lk=Lk, n_h=16, n_kv=8, d_h=128, HI=8, dI=64, k_base=100, k_min=20, k_max=200, v_bar=0.03)
    gen = torch.Generator().manual_seed(35)
    n = lambda *s: torch.randn(*s, generator=gen).to(BF16).cuda()  # noqa: E731
    K, V, kI = (torch.empty(1, Lk, 8, 128, dtype=BF16, device="cuda"), torch.empty(1, Lk, 8, 128, dtype=BF16, device="cuda"),
                torch.empty(1, Lk, 64, dtype=BF16, device="cuda"))
    gsa.gsa_cache_read(p.c, K, V, kI, p.ws)
    Q, g1, qI, w = n(1, Lq, 16, 128), n(1, Lq, 16, 128), n(1, Lq, 8, 64), torch.rand(1, Lq, 8, generator=gen).cuda()
    out, idx, kt = torch.empty_like(Q), torch.zeros(1, Lq, 200, dtype=I32, device="cuda"), torch.zeros(1, Lq, dtype=I32, device="cuda")
    ws = torch.empty(gsa.gsa_workspace_bytes(gp, 0), dtype=torch.uint8, device="cuda")
    gsa.gsa_forward(gp, Q, K, V, qI, kI, w, None, g1, None, out, idx, kt, None, 0, ws)
    assert gsa.gsa_device_status(ws) == 0
    out4 = torch.empty_like(Q)
    ws4 = torch.empty(gsa.gsa_cache_attn_workspace_bytes(gp), dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, Q, g1, idx, kt, out4, ws4)
    assert gsa.gsa_device_status(ws4) == 0
    sets = [[idx[0, t, :int(kt[0, t])].cpu().numpy() for t in range(Lq)]]
    _check_rows(p, Q.cpu(), g1.cpu(), out4, sets, Lq, 128 ** -0.5)
    for t in range(0, Lq, 7):
        want, mag = p.plain.attn(0, f64(Q[0, t]), f64(g1[0, t]), sets[0][t], 128 ** -0.5)
        assert (np.abs(f64(out[0, t]) - f64(out4[0, t])) <= 2 * 2.0 ** -8 * (mag + np.abs(want)) * 1.05 + 1e-6).all()


def test_binding_refuses_tensors_that_do_not_fit():
    geo = GEOMETRIES[2]
    p = _filled(geo, [100, 60], 47)
    c, ws = p.c, p.ws
    gp = gsa.make_params(B=2, Lq=1, Lk=100, n_h=4, n_kv=2, d_h=64, HI=2, dI=64, k_base=8, k_min=1, k_max=16)
    new = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    n2, kv, k3 = new(2, dtype=I32), new(2, 3, 2, 64), new(2, 3, 64)
    good = {
        "gsa_cache_reserve": [n2, new(2, dtype=I32)], "gsa_cache_append": [kv, kv, kv, k3, n2, n2], "gsa_cache_read": [kv, kv, k3],
        "gsa_cache_release": [n2], "gsa_cache_compact": [new(1, dtype=I32)],
        "gsa_cache_indexer_scores": [gp, new(2, 1, 2, 64), new(2, 1, 2, dtype=F32), new(2, dtype=F32), new(2, 1, 100, dtype=F32), 100],
        "gsa_cache_topk": [gp, new(2, 1, 100, dtype=F32), 100, new(2, 1, 16, dtype=I32), new(2, 1, dtype=I32), new(2, 1, dtype=F32)],
        "gsa_cache_attn_fwd": [gp, new(2, 1, 4, 64), new(2, 1, 4, 64), new(2, 1, 16, dtype=I32), new(2, 1, dtype=I32), new(2, 1, 4, 64)],
    }
    n0, before = gsa.gsa_launch_count(), p.lens.clone()
    for name, args in good.items():
        f = getattr(gsa, name)
        for i, a in enumerate(args):
            if not isinstance(a, torch.Tensor):
                continue
            wide = torch.zeros(tuple(a.shape) + (2,), dtype=a.dtype, device="cuda")[..., 0]        # the right shape, strided
            others = [a.cpu(), a.to(torch.float16), torch.zeros(tuple(a.shape)[:-1] + (a.shape[-1] + 1,), dtype=a.dtype, device="cuda"), [1, 2]]
            for bad in others + ([wide] if a.numel() > 1 else []):
                with pytest.raises(gsa.GsaError):
                    f(c, *args[:i], bad, *args[i + 1:], ws)
        for bad_ws in (None, ws.cpu(), ws[:8], ws[::2], ws.data_ptr()):
            with pytest.raises(gsa.GsaError):
                f(c, *args, bad_ws)
    with pytest.raises(gsa.GsaError):
        gsa.gsa_cache_fork(c, n2.float(), True, ws)
    assert gsa.gsa_launch_count() == n0 and torch.equal(p.lens, before)


def test_calls_on_a_stream_that_is_not_the_current_one():
    geo = GEOMETRIES[0]
    p = _filled(geo, [300, 200], 48)
    gp = gsa.make_params(B=2, Lq=1, Lk=320, n_h=16, n_kv=8, d_h=128, HI=8, dI=64, k_base=40, k_min=8, k_max=64, v_bar=0.03)
    gen = torch.Generator().manual_seed(49)
    x = {k: v.cuda() for k, v in _step_inputs(p, gp, gen).items()}
    buf, side = _step_buffers(gp), torch.cuda.Stream()
    torch.cuda.synchronize()
    late = torch.zeros(64 << 20, device="cuda")
    with torch.cuda.stream(side):                                        # work ahead of the step on its stream, none on the current one
        for _ in range(20):
            late += 1
        x["Q"].mul_(0.5)
    gsa.gsa_cache_reserve(p.c, buf["n_new"], buf["start"], p.ws, stream=side)
    gsa.gsa_cache_append(p.c, x["K"], x["V"], x["g2"], x["kI"], buf["n_new"], buf["start"], p.ws, stream=side)
    gsa.gsa_cache_indexer_scores(p.c, gp, x["qI"], x["w"], None, buf["scores"], buf["scores"].shape[-1], p.ws, stream=side)
    gsa.gsa_cache_topk(p.c, gp, buf["scores"], buf["scores"].shape[-1], buf["idx"], buf["kt"], None, p.ws, stream=side)
    gsa.gsa_cache_attn_fwd(p.c, gp, x["Q"], x["g1"], buf["idx"], buf["kt"], buf["out"], buf["ws"], stream=side)
    side.synchronize()
    _plain_step(p, gp, x, buf)
