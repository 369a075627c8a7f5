"""The loops that carry the large calls on the paged 4-bit cache: units with many tiles, warps with many steps of keys, runs of several rounds.

An attention unit (a warp for each KV head) has at least two tiles of 16 keys and one SM sixteen warps: below some 600 tiles for eight KV heads, 4700
for one, no unit has more.  The ring of a warp has four stages, the addresses of its records four blocks of four or eight tiles, which the CTA's units pass
together: the sets below give every unit 20 to 42 tiles, so that both come round, and totals that the units do not divide.
"""
import numpy as np
import pytest
import torch

from cache_check import check_attention
from cache_plain import PlainCache
from paper_2601_15305_b200 import binding as gsa
from test_gpu_cache import BF16, GEOMETRIES, I32, Pair, _attend, f64, i32
from test_gpu_cache_reports import _keys_only, _score_case

pytestmark = pytest.mark.gpu


# ---- attention ---------------------------------------------------------------------------------------------------------------
def _long_sets(rng, lens, Lq, most):
    """Ragged sets of every row, some of them empty or of one key, in any order in every third row."""
    out = []
    for b, n in enumerate(lens):
        rows = []
        for t in range(Lq):
            vis = max(0, n - Lq + t + 1)
            k = (0, 1, most, most - 7, most // 2 + t, most, 16, most - 1, 33, most)[(b * 3 + t) % 10]
            s = rng.permutation(vis)[:k]
            rows.append(s if t % 3 == 0 else np.sort(s))
        out.append(rows)
    return out


@pytest.fixture(scope="module")
def caches():
    """Filled once for each layout: the plain twin takes its tokens one by one."""
    made = {}

    def get(i):
        if i not in made:
            geo = GEOMETRIES[i]
            lens = [4350, 0, 4200]
            p = Pair(3, sum(-(-n // geo["T"]) for n in lens) + 3, -(-4350 // geo["T"]), **geo, seed=80 + i)
            p.append([2000, 0, 1999])
            p.append([2350, 0, 2201])
            made[i] = p
        return made[i]

    return get


# rows a sequence: tiles of all rows over the units of 148 SMs (296 for eight KV heads .. 2368 for one) make 20 to 42 a unit
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("i,Lq,most", [(5, 60, 3001), (0, 61, 3107), (3, 100, 3501), (2, 100, 4001), (1, 170, 4090), (4, 171, 4011)])
def test_attention_where_every_unit_has_many_tiles(caches, i, Lq, most, G):
    p = caches(i)
    P = p.plain
    rng = np.random.default_rng(i * 10 + G)
    sets = _long_sets(rng, P.lens, Lq, most)
    tiles, units = sum(-(-len(s) // 16) for r in sets for s in r), torch.cuda.get_device_properties(0).multi_processor_count * (16 // P.n_kv)
    per = -(-tiles // units)
    assert per > 4 * (8 if P.n_kv >= 4 else 4) and tiles % units != 0    # (all four blocks of addresses are used again, some units have a tile less)
    Q, g1, out, status, _ = _attend(p, G, Lq, sets, most, seed=G)
    assert status == 0 and not out.isnan().any()
    rows = {(b, t) for b in (0, 2) for t in list(range(0, Lq, 23)) + [1, Lq - 2, Lq - 1]} | {(1, 0), (1, Lq - 1)}
    check_attention(P, Q, g1, out, sets, Lq, P.d_h ** -0.5, rows=rows, run_tiles=per + 1)
    # the rows that are not compared: the same bits in a call of their own order of work
    again = _attend(p, G, Lq, sets, most, seed=G)[2]
    assert torch.equal(out, again)


def test_large_calls_give_the_same_bits_every_time(caches):
    """Work is dealt by the sets' sizes alone: repeated, on another stream, behind other work and on a workspace that another call has used."""
    p = caches(0)
    sets = _long_sets(np.random.default_rng(7), p.plain.lens, 33, 2900)
    first = _attend(p, 2, 33, sets, 2900, seed=3)[2]
    side = torch.cuda.Stream()
    late = torch.zeros(32 << 20, device="cuda")
    for turn in range(6):
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            late += turn
            again = _attend(p, 2, 33, sets, 2900, seed=3)[2]
            torch.cuda.current_stream().synchronize()
        assert torch.equal(first, again)


# ---- indexer -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("HI,dI,T", [(8, 64, 64), (4, 32, 16), (1, 64, 128)])
def test_scores_where_every_warp_has_many_steps(HI, dI, T, act):
    """50 thousand steps of 32 keys over 2368 warps: 21 each, from row to row, their pages looked up again within a row."""
    lens = [40000, 0, 33333, 1, 40001, 25000, 39999, 20017]
    c, held = _keys_only(lens, T, dI, -(-40001 // T), 90)
    run, check, ws = _score_case(c, held, lens, 8, 40001, HI, dI, act, 91)
    run()
    assert gsa.gsa_device_status(ws) == 0
    check([(b, t) for b in range(8) for t in range(8)])


# ---- tokens in and out -------------------------------------------------------------------------------------------------------
def _codes(P, x):
    from cache_plain import encode
    return encode(x.reshape(-1, P.n_kv, P.d_h))


@pytest.mark.parametrize("geo,lens,first", [(dict(n_kv=8, d_h=128, dI=64, T=64), [3001, 0, 1203], [130, 0, 77]),
                                            (dict(n_kv=1, d_h=64, dI=32, T=16), [40013, 39990], [3, 21]),
                                            (dict(n_kv=2, d_h=128, dI=32, T=128), [9000, 1, 8197], [129, 0, 128])])
def test_tokens_stored_and_read_in_runs_of_several_rounds(geo, lens, first):
    """Bit for bit; more groups than a wave of warps takes in a round or two, runs that begin inside a token, sequences that end inside a run."""
    B, T = len(lens), geo["T"]
    P = PlainCache(B, sum(-(-n // T) for n in lens) + 2, T, -(-max(lens) // T), geo["n_kv"], geo["d_h"], geo["dI"])
    table, refs = torch.full((B, P.max_pages), -1, dtype=I32, device="cuda"), torch.zeros(P.n_pages, dtype=I32, device="cuda")
    pool = torch.zeros(P.pool.size, dtype=torch.uint8, device="cuda")
    c = gsa.make_cache(pool, table, i32(np.zeros(B)), refs, page_tokens=T, n_kv=geo["n_kv"], d_h=geo["d_h"], dI=geo["dI"])
    ws = torch.full((gsa.gsa_cache_workspace_bytes(c),), 0xFF, dtype=torch.uint8, device="cuda")
    gen, start = torch.Generator().manual_seed(92), torch.zeros(B, dtype=I32, device="cuda")
    kept = [[] for _ in lens]
    for n_new in (first, [n - f for n, f in zip(lens, first)]):
        L = max(n_new)
        K, V = (torch.randn(B, L, geo["n_kv"], geo["d_h"], generator=gen).to(BF16) for _ in range(2))
        kI = torch.randn(B, L, geo["dI"], generator=gen).to(BF16)
        for x in (K, V, kI):                                             # what nobody asked for must not matter
            for b, n in enumerate(n_new):
                x[b, n:] = float("nan")
        gsa.gsa_cache_reserve(c, i32(n_new), start, ws)
        assert gsa.gsa_device_status(ws) == 0
        gsa.gsa_cache_append(c, K.cuda(), V.cuda(), None, kI.cuda(), i32(n_new), start, ws)
        assert gsa.gsa_device_status(ws) == 0
        for b, n in enumerate(n_new):
            kept[b].append((K[b, :n], V[b, :n], kI[b, :n]))
    L = max(lens) + 5 if (max(lens) + 5) <= P.max_pages * T else max(lens)
    K, V, kI = (torch.full((B, L, geo["n_kv"], geo["d_h"]), 7.0, dtype=BF16, device="cuda"), torch.full((B, L, geo["n_kv"], geo["d_h"]), 7.0, dtype=BF16, device="cuda"),
                torch.full((B, L, geo["dI"]), 7.0, dtype=BF16, device="cuda"))
    gsa.gsa_cache_read(c, K, V, kI, ws)
    assert gsa.gsa_device_status(ws) == 0
    from cache_plain import decode
    by = pool.cpu().numpy().reshape(P.pool.shape)
    tab = table.cpu().numpy()
    for b, n in enumerate(lens):
        if n:
            k, v, ki = [torch.cat([part[i] for part in kept[b]]) for i in range(3)]
            pos = np.arange(n)
            page, slot = tab[b, pos // T], pos % T
            r = by[page[:, None], (slot * P.rec)[:, None] + np.arange(P.D + P.D // 8)]
            for i, (x, got) in enumerate(((k, K), (v, V))):
                u, scale = _codes(P, f64(x))
                flat = u.reshape(n, -1)
                assert np.array_equal(r[:, i * P.D // 2:(i + 1) * P.D // 2], flat[:, 0::2] | (flat[:, 1::2] << 4))
                assert np.array_equal(r[:, P.D:].reshape(n, P.n_kv, 2, -1)[:, :, i], scale)
                assert np.array_equal(f64(got[b, :n]), decode(u, scale).reshape(n, P.n_kv, P.d_h))
            assert torch.equal(kI[b, :n].cpu(), ki)
        assert (K[b, n:] == 7.0).all() and (V[b, n:] == 7.0).all() and (kI[b, n:] == 7.0).all()


def test_one_sequence_of_a_cache_as_a_cache():
    """One table row and its length, as views, with the cache's pool and counts: that sequence alone, for its prompt."""
    geo = GEOMETRIES[2]
    p = Pair(3, 80, 20, **geo, seed=93)
    p.append([300, 5, 0])
    view = gsa.make_cache(p.pool, p.table[1:2], p.lens[1:2], p.refs, page_tokens=geo["T"], n_kv=geo["n_kv"], d_h=geo["d_h"], dI=geo["dI"])
    n = 170
    K, V, g2, kI = p.tokens(n)
    start = torch.zeros(1, dtype=I32, device="cuda")
    gsa.gsa_cache_reserve(view, i32([n]), start, p.ws)
    gsa.gsa_cache_append(view, *[x[1:2].contiguous().cuda() for x in (K, V, g2, kI)], i32([n]), start, p.ws)
    assert p.status() == 0
    status, at = p.plain.reserve([0, n, 0])
    assert status == 0 and int(start) == at[1] == 5
    p.plain.append(f64(K), f64(V), f64(g2), kI.view(torch.int16).numpy().view(np.uint16), [0, n, 0], at)
    p.same_tables()
    p.same_pages()
    out = [torch.zeros(1, n + 5, 2, 64, dtype=BF16, device="cuda"), torch.zeros(1, n + 5, 2, 64, dtype=BF16, device="cuda"),
           torch.zeros(1, n + 5, 64, dtype=BF16, device="cuda")]
    gsa.gsa_cache_read(view, *out, p.ws)
    assert p.status() == 0
    for got, want in zip(out, p.plain.tokens(1, np.arange(n + 5))):
        assert np.array_equal(f64(got[0]), want)
