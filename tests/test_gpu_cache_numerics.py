"""Values that the cache's kernels must not lose: NaN in queries, keys, biases and gates; heads of one group far apart; keys with outliers."""
import numpy as np
import pytest
import torch

from cache_check import check_attention, score_error
from paper_2601_15305_b200 import binding as gsa
from test_gpu_cache import BF16, GEOMETRIES, I32, Pair, _filled, _random_sets, f64, i32

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


def _attention(p, G, Lq, sets, k_max, Q, g1, sm_scale=0.0):
    P = p.plain
    idx, kt = np.full((P.B, Lq, k_max), -1, np.int32), np.zeros((P.B, Lq), np.int32)
    for b in range(P.B):
        for t in range(Lq):
            kt[b, t] = len(sets[b][t])
            idx[b, t, :kt[b, t]] = sets[b][t]
    gp = gsa.make_params(B=P.B, Lq=Lq, Lk=int(P.lens.max()), n_h=P.n_kv * G, n_kv=P.n_kv, d_h=P.d_h, HI=1, dI=P.dI, k_base=1, k_min=1, k_max=k_max,
                         sm_scale=sm_scale)
    out = torch.full((P.B, Lq, P.n_kv * G, P.d_h), -3.0, dtype=BF16, device="cuda")
    ws = torch.full((gsa.gsa_cache_attn_workspace_bytes(gp),), 0xFF, dtype=torch.uint8, device="cuda")
    gsa.gsa_cache_attn_fwd(p.c, gp, Q.cuda(), g1.cuda(), i32(idx), i32(kt), out, ws)
    assert gsa.gsa_device_status(ws) == 0
    return out


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("geo,sizes,k_max,Lq", [(GEOMETRIES[0], [16, 9], 16, 1), (GEOMETRIES[1], [200, 150], 200, 1), (GEOMETRIES[4], [700, 690], 700, 1),
                                                (GEOMETRIES[5], [30, 700], 700, 1), (GEOMETRIES[5], [700, 16, 650], 700, 40)])
def test_a_nan_in_the_output_gate_shows(geo, sizes, k_max, Lq, G):
    """Rows finished by one unit, by a CTA of their own, and by the merge kernel, with eight warps a row and with one."""
    lens = [750, 750]
    p = _filled(geo, lens, 73)
    sets = _random_sets(np.random.default_rng(G), lens, Lq, sizes)
    n_h, d = geo["n_kv"] * G, geo["d_h"]
    gen = torch.Generator().manual_seed(74)
    Q, g1 = torch.randn(2, Lq, n_h, d, generator=gen).to(BF16), torch.randn(2, Lq, n_h, d, generator=gen).to(BF16)
    clean = _attention(p, G, Lq, sets, k_max, Q, g1)
    spoilt, expect = g1.clone(), torch.zeros(g1.shape, dtype=torch.bool)
    for b in range(2):
        for t in range(Lq):
            for h, i in ((0, 0), (n_h - 1, d - 1), (n_h // 2, 17), (0, d - 2)):
                spoilt[b, t, h, i], expect[b, t, h, i] = NAN, True
    spoilt[0, 0, 0, 1], spoilt[0, 0, 0, 2] = INF, -INF                   # gates of 1 and 0
    out = _attention(p, G, Lq, sets, k_max, Q, spoilt).cpu()
    assert torch.equal(out.isnan(), expect)
    kept = ~expect
    kept[0, 0, 0, 1:3] = False
    assert torch.equal(out[kept], clean.cpu()[kept])
    want, mag = p.plain.attn(0, f64(Q[0, 0]), np.full((n_h, d), 60.0), np.asarray(sets[0][0]), d ** -0.5)
    assert abs(float(out[0, 0, 0, 1]) - want[0, 1]) <= 2.0 ** -8 * abs(want[0, 1]) + 2.0 ** -10 * mag[0, 1] and abs(float(out[0, 0, 0, 2])) <= 2.0 ** -100


@pytest.mark.parametrize("exponent", [24, 27, 28, 29, 32, 40, 80, 110])
@pytest.mark.parametrize("k_max", [40, 700])
@pytest.mark.parametrize("geo", [GEOMETRIES[2], GEOMETRIES[4], GEOMETRIES[0]], ids=lambda g: "-".join(map(str, g.values())))
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_scores_of_any_finite_magnitude(geo, G, k_max, exponent):
    """Scores of 2^24 .. 2^110: far above the distance of neighbouring fp32 numbers there, the first key of a row takes it; keys that are alike share it."""
    lens = [720, 730]
    p = Pair(2, 2 * 740 // geo["T"] + 2, 740 // geo["T"] + 1, **geo, seed=80)
    p.append([700, 710])
    K, V, g2, kI = p.tokens(20, gate=False)
    K[:, 10:] = K[:, :10]                                                # ten pairs of equal keys with values of their own
    p.append([20, 20], x=(K, V, g2, kI))
    sets = _random_sets(np.random.default_rng(G), [700, 710], 1, [k_max - 20, k_max - 21])
    sets = [[np.concatenate([s[0], np.arange(n - 20, n)])] for s, n in zip(sets, lens)]
    n_h, d = geo["n_kv"] * G, geo["d_h"]
    gen = torch.Generator().manual_seed(81)
    Q = (torch.randn(2, 1, n_h, d, generator=gen) * 2.0 ** exponent).to(BF16)
    Q[0, 0, 0] = K[0, 4, 0] * 2.0 ** exponent                            # (one head's largest score is a pair's)
    g1 = torch.randn(2, 1, n_h, d, generator=gen).to(BF16)
    out = f64(_attention(p, G, 1, sets, k_max, Q, g1))
    assert np.isfinite(out).all()
    for b in range(2):
        K64, V64, _ = p.plain.tokens(b, sets[b][0])
        gate = 1 / (1 + np.exp(-f64(g1[b, 0])))
        for h in range(n_h):
            z = K64[:, h // G] @ f64(Q[b, 0, h]) * d ** -0.5
            top = np.flatnonzero(z == z.max())
            rest = np.delete(z, top)
            # (scores are within 2^-14 of sum s |q|, below 2^-10 of the largest here; at a distance of 64 and more a key's part is below 2^-90)
            if rest.max() > z.max() * (1 - 2.0 ** -9) - 64:
                continue
            want = V64[top, h // G].mean(0) * gate[h]
            mag = np.abs(V64[top, h // G]).mean(0) * gate[h]
            assert (np.abs(out[b, 0, h] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -18 + 2.0 ** -11) * mag + 1e-25).all(), (b, h)
            if (b, h) == (0, 0):
                assert len(top) == 2


@pytest.mark.parametrize("far", [-36, -60, 36])
@pytest.mark.parametrize("k_max", [40, 700])
@pytest.mark.parametrize("geo", [GEOMETRIES[2], GEOMETRIES[3], GEOMETRIES[0]], ids=lambda g: "-".join(map(str, g.values())))
@pytest.mark.parametrize("G", [2, 4, 8])
def test_heads_of_a_group_however_far_apart(geo, G, k_max, far):
    """One query head of a KV head's group is 2^36 or 2^60 times as large as the others, or they as it: each is as exact as alone."""
    lens = [720, 730]
    p = _filled(geo, lens, 75)
    sets = _random_sets(np.random.default_rng(G), lens, 1, [k_max, k_max - 1])
    n_h, d = geo["n_kv"] * G, geo["d_h"]
    gen = torch.Generator().manual_seed(76)
    Q, g1 = torch.randn(2, 1, n_h, d, generator=gen), torch.randn(2, 1, n_h, d, generator=gen).to(BF16)
    odd = [kv * G + (kv + 1) % G for kv in range(geo["n_kv"])]           # one head of each group, not always the same
    rest = [h for h in range(n_h) if h not in odd]
    Q[:, :, odd] *= 2.0 ** -far
    Q = Q.to(BF16)
    out = _attention(p, G, 1, sets, k_max, Q, g1)
    assert out.isfinite().all()
    check_attention(p.plain, Q, g1, out, sets, 1, d ** -0.5, heads=rest if far < 0 else range(n_h))


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("geo", [GEOMETRIES[0], GEOMETRIES[1], GEOMETRIES[4], GEOMETRIES[5]], ids=lambda g: "-".join(map(str, g.values())))
def test_outliers_that_the_queries_do_not_look_at(geo, G):
    """Every group of 16 has a channel 64 times as wide as the others, where Q is 0: scores far smaller than what they are summed up from."""
    d, n = geo["d_h"], 400
    p = Pair(1, n // geo["T"] + 2, n // geo["T"] + 1, **geo, seed=77)
    gen = torch.Generator().manual_seed(78)
    K, V = (torch.randn(1, n, geo["n_kv"], d, generator=gen) for _ in range(2))
    K[..., 7::16] = 64 * K[..., 7::16].sign()
    p.append([n], x=(K.to(BF16), V.to(BF16), None, torch.zeros(1, n, geo["dI"], dtype=BF16)))
    Q = torch.randn(1, 1, geo["n_kv"] * G, d, generator=gen) * 4
    Q[..., 7::16] = 0
    Q, g1 = Q.to(BF16), torch.randn(1, 1, geo["n_kv"] * G, d, generator=gen).to(BF16)
    sets = [[np.arange(n)]]
    err, _ = score_error(p.plain, 0, f64(Q[0, 0]), sets[0][0], d ** -0.5)
    assert err.max() < 0.05                                              # (the check below still tells something)
    out = _attention(p, G, 1, sets, n, Q, g1)
    check_attention(p.plain, Q, g1, out, sets, 1, d ** -0.5)
