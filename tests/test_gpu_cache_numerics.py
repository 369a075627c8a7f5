"""Values that the cache's kernels must not lose: NaN and infinities in what the indexer's scores are made of."""
import numpy as np
import pytest
import torch

from paper_2601_15305_b200 import binding as gsa
from test_gpu_cache import BF16, GEOMETRIES, I32, _filled, f64

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _scores(p, Lq, HI, act, qI, w, bI, Lk):
    gp = gsa.make_params(B=p.plain.B, Lq=Lq, Lk=Lk, n_h=p.plain.n_kv, n_kv=p.plain.n_kv, d_h=p.plain.d_h, HI=HI, dI=p.plain.dI, act=act,
                         k_base=4, k_min=4, k_max=4, k_mode=2)
    sc = torch.full((p.plain.B, Lq, Lk), -5.0, device="cuda")
    gsa.gsa_cache_indexer_scores(p.c, gp, qI, w, bI, sc, Lk, p.ws)
    assert p.status() == 0
    return sc, gp


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("where", ["query", "key", "bias", "weight"])
@pytest.mark.parametrize("geo,HI", [(GEOMETRIES[0], 8), (GEOMETRIES[1], 4), (GEOMETRIES[2], 1)])
def test_a_nan_shows_in_the_scores_it_belongs_to(geo, HI, where, act):
    p = _filled(geo, [99, 40], 70)
    K, V, g2, kI = p.tokens(1)
    if where == "key":
        kI[0, 0, 5] = NAN
    p.append([1, 1], x=(K, V, g2, kI))
    gen = torch.Generator().manual_seed(71)
    Lq, Lk = 2, 100
    qI, w, bI = torch.randn(2, Lq, HI, geo["dI"], generator=gen).to(BF16), torch.rand(2, Lq, HI, generator=gen), torch.zeros(HI)
    clean, gp = _scores(p, Lq, HI, act, qI.cuda(), w.cuda(), bI.cuda(), Lk)
    expect = torch.zeros(2, Lq, Lk, dtype=torch.bool)
    if where == "query":
        qI[1, 1, HI - 1, 3] = NAN
        expect[1, 1, :41] = True
    elif where == "weight":
        w[0, 0, HI // 2] = NAN
        expect[0, 0, :99] = True
    elif where == "bias":
        bI[HI - 1] = NAN
        expect[0, 0, :99] = expect[0, 1, :100] = expect[1, 0, :40] = expect[1, 1, :41] = True
    else:
        expect[0, 1, 99] = True                                          # the first row does not see the last key
    sc, _ = _scores(p, Lq, HI, act, qI.cuda(), w.cuda(), bI.cuda(), Lk)
    assert torch.equal(sc.isnan().cpu(), expect)
    if where != "key":
        assert torch.equal(sc[~expect.cuda()], clean[~expect.cuda()])
    # the selection puts a NaN above every score: such a key is taken, not lost
    idx, kt = torch.zeros(2, Lq, 4, dtype=I32, device="cuda"), torch.zeros(2, Lq, dtype=I32, device="cuda")
    gsa.gsa_cache_topk(p.c, gp, sc, Lk, idx, kt, None, p.ws)
    assert p.status() == 0
    if where == "key":
        assert 99 in idx[0, 1].tolist() and 99 not in idx[0, 0].tolist()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("HI", [1, 2, 4, 8])
def test_infinities_in_the_scores(HI, act):
    """An infinite pre-activation is a gate of 0 or 1, or an infinite or closed ReLU: no NaN, from a key or from a bias."""
    p = _filled(GEOMETRIES[0], [63], 72)
    K, V, g2, kI = p.tokens(1)
    kI[0, 0, 9] = INF
    p.append([1], x=(K, V, g2, kI))
    qI, w, bI = torch.randn(1, 1, HI, 64, generator=p.gen).to(BF16), torch.ones(1, 1, HI), torch.zeros(HI)
    for sign in (0, 1, -1):
        if sign:
            bI[HI - 1] = sign * INF
        sc, _ = _scores(p, 1, HI, act, qI.cuda(), w.cuda(), bI.cuda(), 64)
        keys = p.plain.tokens(0, np.arange(64))[2]
        with np.errstate(all="ignore"):
            z = f64(qI[0, 0]) @ keys.T + f64(bI)[:, None]
            want = (np.maximum(z, 0) if act else 1 / (1 + np.exp(-z))).sum(0)
        clash = np.isnan(want)                                           # (an infinite key against an infinite bias of the other sign)
        assert not clash[:63].any()
        got = f64(sc[0, 0])
        assert np.array_equal(np.isnan(got), clash)
        assert np.array_equal(np.isinf(got), np.isinf(want))
        fin = np.isfinite(want)
        # (the terms of a score: 64 products of which the sum is below 64, see the other tests)
        assert np.abs(got[fin] - want[fin]).max(initial=0) <= HI * (72 * 2.0 ** -23 * 64 * (1.0 if act else 0.25) + 2.0 ** -20 + 64 * 2.0 ** -23)
