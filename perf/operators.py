"""The paged 4-bit cache and the operators that work on it, as cases that a timing program can run.

    listed()              the named cases
    draw(rng)             one more case of the same ranges
    prepare(case, seed)   the cache, the inputs and the buffers a caller has in hand before the call
    run(state)            one pass: in plain torch operations (own = False) or through the library's entry points (own = True)
    work(case)            bytes and flops a pass cannot do without
    exact(case, seed)     the outputs in 64 bits, from the operators' definition

Four operations:
  * attn: sparse gated attention over index sets, K and V' in the cache's pages (decode, a few drafted tokens, a chunk of rows).
  * scores: the gated lightning indexer for decode rows, k^I in the cache's pages, every sequence with a length of its own.
  * append: pages for new tokens, their K, V * sigmoid(g2) and k^I into the cache, and the whole cache read back as the
    contiguous tensors that chunked prefill takes.
  * fork / compact: page tables, reference counts and page copies (beams that share their prompt's pages or copy them, freed
    prompts; a pool whose live pages move to its front).

The cache.  A pool of pages of T tokens; table[b, s // T] names the page of position s of sequence b.  A token's record holds
4-bit codes of K, 4-bit codes of V', one scale byte for each 16 values (for each KV head d_h / 16 of K, then of V'), padded to
16 bytes; behind a page's records stand its tokens' k^I in bf16.  A scale byte n stands for (1 + n % 8 / 8) * 2^(n // 8 - 20),
255 for NaN; a code u for (u - 8) * scale.
"""
import math

import torch

own = False

BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8

# the layer that the benchmark's decode and prefill configurations use, the `tiny` configuration's, and the parity tests' head layouts
LAYER = dict(n_h=16, n_kv=8, d_h=128, HI=8, dI=64)
SMALL = dict(n_h=4, n_kv=1, d_h=64, HI=4, dI=32)
LAYOUTS = (dict(n_h=8, n_kv=8, d_h=128, HI=4, dI=64), dict(n_h=16, n_kv=2, d_h=128, HI=8, dI=64),
           dict(n_h=32, n_kv=8, d_h=64, HI=4, dI=32), dict(n_h=8, n_kv=2, d_h=64, HI=2, dI=32))


def _case(op, B, Lq, Lk, layer=LAYER, **opt):
    c = dict(op=op, B=B, Lq=Lq, Lk=Lk, T=64, ragged=False, k_base=2048, k_max=4096, gate=True, share=True, act=0)
    c.update(layer)
    c.update(opt)
    return c


def listed():
    named = {
        # the smallest call: one stream of the small layer, where launches and latency are all there is
        "attn_1x2051_small": _case("attn", 1, 1, 2051, SMALL, T=16, k_base=64, k_max=128),
        # one stream of the benchmark's layer, its usual budget
        "attn_1x32771": _case("attn", 1, 1, 32771),
        # a full decode batch: 32 slots of different lengths, one of them empty, budgets from 512 to 4096
        "attn_32x128k_ragged": _case("attn", 32, 1, 131072, ragged=True),
        # four drafted tokens a stream, wide groups of query heads
        "attn_8x4_of_9001": _case("attn", 8, 4, 9001, LAYOUTS[1], ragged=True, k_base=768, k_max=1500),
        # a chunk of rows against a cache, narrow heads
        "attn_chunk_257_of_20011": _case("attn", 1, 257, 20011, LAYOUTS[2], k_base=1000, k_max=1500),
        # the indexer of a decode step: the whole batch, and one stream
        "scores_32x128k_ragged": _case("scores", 32, 1, 131072, ragged=True),
        "scores_1x32771": _case("scores", 1, 1, 32771),
        # new tokens: one for each of 32 streams with short caches, a chunk of 8192 behind 4099, odd lengths through narrow heads
        "append_32x1": _case("append", 32, 1, 160, ragged=True),
        "append_8192_behind_4099": _case("append", 1, 8192, 12291),
        "append_5x777_narrow": _case("append", 5, 777, 2001, LAYOUTS[3], T=32, ragged=True),
        # eight prompts become four beams each that share their pages, and are freed
        "fork_8_prompts_to_32_beams": _case("fork", 40, 1, 4099),
        # a pool of 5600 pages, half of them freed by sequences that ended
        "compact_5600_pages": _case("compact", 56, 1, 6400),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn", "attn", "attn", "scores", "scores", "append", "append", "append", "fork", "compact"))
    layer = LAYER if rng.random() < 0.5 else rng.choice((SMALL,) + LAYOUTS)
    opt = dict(T=rng.choice((16, 32, 64, 64, 128)), ragged=rng.random() < 0.6)
    if op == "attn":
        B, Lq = _log_uniform(rng, 1, 32), rng.choice((1, 1, 1, 2, 4))
        Lk = _log_uniform(rng, 40, 131072)
        if rng.random() < 0.2:
            B, Lq, Lk = 1, _log_uniform(rng, 5, 200), _log_uniform(rng, 400, 20000)
        k_max = min(4096 if Lq <= 4 else 1500, _log_uniform(rng, 16, 8192))
        if B * Lq > 32:
            k_max = min(k_max, 1500)
        return _case(op, B, Lq, Lk, layer, k_base=max(1, k_max // rng.choice((1, 2, 3))), k_max=k_max, **opt)
    if op == "scores":
        return _case(op, _log_uniform(rng, 1, 32), rng.choice((1, 1, 2, 4)), _log_uniform(rng, 40, 131072 // 4), layer,
                     act=rng.choice((0, 0, 1)), **opt)
    if op == "append":
        B = _log_uniform(rng, 1, 32)
        Lq = rng.choice((1, 1, _log_uniform(rng, 2, 8192 // B)))
        return _case(op, B, Lq, Lq + _log_uniform(rng, 40, max(41, 12000 // B)), layer, gate=rng.random() < 0.7, **opt)
    if op == "fork":
        return _case(op, 5 * _log_uniform(rng, 1, 8), 1, _log_uniform(rng, 40, 4099), layer, share=rng.random() < 0.6, **opt)
    return _case(op, _log_uniform(rng, 2, 56), 1, _log_uniform(rng, 100, 6400), layer, **opt)


# ---- sizes that follow from a case ------------------------------------------------------------------------------------
def _lens(c):
    """Tokens of every sequence at the end of the pass."""
    B, L, Lq = c["B"], c["Lk"], c["Lq"]
    if c["op"] == "fork":                        # the first fifth of the slots are prompts, the others wait for beams
        return [max(1, L - 61 * b) if b < B // 5 else 0 for b in range(B)]
    if not c["ragged"]:
        return [L] * B
    lens = [max(Lq, L * ((5 * b + 3) % 8 + 1) // 8 - 7 * b) for b in range(B)]
    if B >= 4:
        lens[-1] = 0                             # a padded batch
    return lens


def _new(c, lens):
    """Tokens that an append brings, for every sequence."""
    return [min(n, max(1, c["Lq"] - (3 * b if c["ragged"] else 0))) for b, n in enumerate(lens)]


def _sizes(c):
    D = c["n_kv"] * c["d_h"]
    rec = (D + D // 8 + 15) // 16 * 16
    return D, rec, c["T"] * (rec + 2 * c["dI"])


def _rows(c, lens):
    """(visible keys, selected keys) of every query row."""
    out = []
    for b, n in enumerate(lens):
        for t in range(c["Lq"]):
            vis = max(0, n - c["Lq"] + t + 1)
            out.append((vis, min(vis, c["k_max"], max(1, int(c["k_base"] * (1, 0.5, 2, 0.25)[(b + t) % 4])))))
    return out


# ---- the cache's format in plain torch ---------------------------------------------------------------------------------
def _quantize(x):
    """x [..., d_h] fp32 -> codes [..., d_h] (0 .. 15) and scale bytes [..., d_h / 16]."""
    g = x.unflatten(-1, (-1, 16))
    amax = g.abs().amax(-1)
    fine = amax.isfinite()                       # (amax of a NaN is NaN)
    bits = (torch.where(fine, amax, torch.zeros_like(amax)) / 7).view(I32)
    byte = (((bits + (1 << 19)) >> 20) - 856).clamp(0, 254)
    s = ((byte + 856) << 20).view(F32)
    u = torch.where(fine[..., None], (g / s[..., None]).round().clamp(-7, 7), torch.zeros_like(g)) + 8
    return u.to(U8).flatten(-2), torch.where(fine, byte, torch.full_like(byte, 255)).to(U8)


def _records(c, K, V):
    """K, V [N, n_kv, d_h] fp32 -> [N, record bytes] uint8."""
    (ku, ks), (vu, vs) = _quantize(K), _quantize(V)
    pair = lambda u: (u[..., 0::2] | (u[..., 1::2] << 4)).flatten(1)  # noqa: E731
    r = torch.cat([pair(ku), pair(vu), torch.stack((ks, vs), 2).flatten(1)], 1)
    return torch.nn.functional.pad(r, (0, _sizes(c)[1] - r.shape[1]))


def _values(c, r):
    """Records [..., record bytes] -> K, V [..., n_kv, d_h] fp32."""
    D, n_kv, d_h = _sizes(c)[0], c["n_kv"], c["d_h"]
    byte = r[..., D:D + D // 8].to(I32).unflatten(-1, (n_kv, 2, d_h // 16))
    s = torch.where(byte == 255, torch.nan, ((byte + 856) << 20).view(F32))
    out = []
    for i in range(2):
        b = r[..., i * D // 2:(i + 1) * D // 2]
        u = torch.stack((b & 15, b >> 4), -1).flatten(-2).unflatten(-1, (n_kv, d_h // 16, 16))
        out.append(((u.to(F32) - 8) * s[..., i, :, None]).flatten(-2))
    return out


def _tokens(c, pool):
    """The records and the indexer keys of a pool as [page, slot, ...]."""
    _, rec, page = _sizes(c)
    n = pool.numel() // page
    return pool.as_strided((n, c["T"], rec), (page, rec, 1)), pool.view(BF16).as_strided((n, c["T"], c["dI"]), (page // 2, c["dI"], 1), c["T"] * rec // 2)


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _normal(gen, *shape, scale=1.0):
    x = torch.randn(*shape, generator=gen, dtype=BF16, device="cuda")
    return x.mul_(scale) if scale != 1.0 else x


def _keys(c, gen, *shape):
    """Keys as a layer makes them: normal, four channels of every head several times as wide."""
    k = _normal(gen, *shape, c["n_kv"], c["d_h"])
    k[..., 5::c["d_h"] // 4] *= 4
    return k


def _cache(c, gen, lens, fill, spare=8):
    """A cache that holds lens[b] tokens, its pages scattered over the pool as after some hours of service."""
    D, rec, page = _sizes(c)
    T, B = c["T"], c["B"]
    need = [-(-n // T) for n in lens]
    used = sum(need)
    n_pages = used + spare
    perm = torch.randperm(n_pages, generator=gen, device="cuda")
    max_pages = max(1, -(-c["Lk"] // T))
    s = dict(pool=torch.zeros(n_pages * page, dtype=U8, device="cuda"))
    host = torch.full((B, max_pages), -1, dtype=torch.int64)
    at = 0
    for b, n in enumerate(need):
        host[b, :n] = torch.arange(at, at + n)
        at += n
    host = host.cuda()
    # table, lengths and counts side by side, so that one copy puts them back
    ints = torch.zeros(B * max_pages + B + n_pages, dtype=I32, device="cuda")
    s["table"], s["lens"], s["refs"] = ints[:B * max_pages].view(B, max_pages), ints[B * max_pages:B * max_pages + B], ints[B * max_pages + B:]
    s["table"].copy_(torch.where(host >= 0, perm[host.clamp(min=0)], host))
    s["lens"].copy_(torch.tensor(lens, dtype=I32))
    s["refs"][perm[:used]] = 1
    s["ints"] = ints
    recs, kI = _tokens(c, s["pool"])
    step = max(1, (1 << 26) // (T * D))
    for i in range(0, used, step):
        pages = perm[i:min(used, i + step)]
        n = pages.numel() * T
        if fill != "kI":
            K = _keys(c, gen, n).float()
            V = _normal(gen, n, c["n_kv"], c["d_h"]).float() * torch.sigmoid(_normal(gen, n, c["n_kv"], c["d_h"]).float())
            recs[pages] = _records(c, K, V).view(-1, T, rec)
        kI[pages] = _normal(gen, n, c["dI"], scale=c["dI"] ** -0.5).view(-1, T, c["dI"])
    return s


def _sets(c, gen, lens):
    """Ascending index sets of the sizes of _rows, spread over the visible keys: one key of each of k even stretches."""
    rows = torch.tensor(_rows(c, lens), device="cuda")
    vis, k = rows[:, :1].double(), rows[:, 1:].double()
    j = torch.arange(c["k_max"], device="cuda")[None]
    lo, hi = (j * vis / k.clamp(min=1)).long(), ((j + 1) * vis / k.clamp(min=1)).long()
    pos = lo + (torch.rand(lo.shape, generator=gen, device="cuda") * (hi - lo)).long()
    idx = torch.where(j < k, torch.minimum(pos, hi - 1).clamp(min=0), -1)
    return idx.to(I32).view(c["B"], c["Lq"], c["k_max"]), rows[:, 1].to(I32).view(c["B"], c["Lq"])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Lq, Lk, op = c["B"], c["Lq"], c["Lk"], c["op"]
    new = lambda *shape, dtype=BF16: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
    lens = _lens(c)
    s = dict(c=c)
    if op == "attn":
        s.update(_cache(c, gen, lens, "all"))
        s["Q"], s["g1"] = _normal(gen, B, Lq, c["n_h"], c["d_h"]), _normal(gen, B, Lq, c["n_h"], c["d_h"])
        s["idx"], s["kt"] = _sets(c, gen, lens)
        s["out"] = new(B, Lq, c["n_h"], c["d_h"])
    elif op == "scores":
        s.update(_cache(c, gen, lens, "kI"))
        s["qI"] = _normal(gen, B, Lq, c["HI"], c["dI"])
        s["w"] = torch.sigmoid(torch.randn(B, Lq, c["HI"], generator=gen, device="cuda"))
        s["bI"] = torch.randn(c["HI"], generator=gen, device="cuda") * 0.1
        s["scores"] = new(B, Lq, (Lk + 31) // 32 * 32, dtype=F32)
    elif op == "append":
        n_new = _new(c, lens)
        s.update(_cache(c, gen, [a - n for a, n in zip(lens, n_new)], "all", spare=8 + sum(-(-a // c["T"]) for a in lens)))
        s["K"], s["V"], s["kI"] = _keys(c, gen, B, Lq), _normal(gen, B, Lq, c["n_kv"], c["d_h"]), _normal(gen, B, Lq, c["dI"], scale=c["dI"] ** -0.5)
        s["g2"] = _normal(gen, B, Lq, c["n_kv"], c["d_h"]) if c["gate"] else None
        s["n_new"] = torch.tensor(n_new, dtype=I32, device="cuda")
        s["start"] = new(B, dtype=I32)
        s["K_all"], s["V_all"], s["kI_all"] = new(B, Lk, c["n_kv"], c["d_h"]), new(B, Lk, c["n_kv"], c["d_h"]), new(B, Lk, c["dI"])
    elif op == "fork":
        P = B // 5
        s.update(_cache(c, gen, lens, "all", spare=8 + 4 * sum(1 if c["share"] else -(-n // c["T"]) for n in lens)))
        s["src_of"] = torch.tensor([-1] * P + [i % P for i in range(B - P)], dtype=I32, device="cuda")
        s["drop"] = torch.tensor([1] * P + [0] * (B - P), dtype=I32, device="cuda")
    else:
        s.update(_cache(c, gen, lens, "all"))
        ended = torch.rand(B, generator=gen, device="cuda") < 0.5
        s["refs"][s["table"][ended][s["table"][ended] >= 0].long()] = 0
        s["table"][ended] = -1
        s["lens"][ended] = 0
        s["live"] = new(1, dtype=I32)
    s["start_ints"] = s["ints"].clone()          # (the program's own copy of where a repeated step starts from)
    s["ws"] = new(64 << 20, dtype=U8)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(state):
    s = state
    c = s["c"]
    if own:
        return _run_own(c, s)
    return dict(attn=_plain_attn, scores=_plain_scores, append=_plain_append, fork=_plain_fork, compact=_plain_compact)[c["op"]](c, s)


def _run_own(c, s):
    from paper_2601_15305_b200 import binding as gsa
    op = c["op"]
    if "cache" not in s:                         # (a program makes these once, next to its buffers)
        s["cache"] = gsa.make_cache(s["pool"], s["table"], s["lens"], s["refs"], page_tokens=c["T"], n_kv=c["n_kv"], d_h=c["d_h"], dI=c["dI"])
        s["p"] = gsa.make_params(B=c["B"], Lq=c["Lq"], Lk=c["Lk"], n_h=c["n_h"], n_kv=c["n_kv"], d_h=c["d_h"], HI=c["HI"], dI=c["dI"],
                                 k_base=c["k_base"], k_min=1, k_max=c["k_max"], act=c["act"])
    cache, p, ws = s["cache"], s["p"], s["ws"]
    if op == "attn":
        gsa.gsa_cache_attn_fwd(cache, p, s["Q"], s["g1"], s["idx"], s["kt"], s["out"], ws)
        return s["out"]
    if op == "scores":
        gsa.gsa_cache_indexer_scores(cache, p, s["qI"], s["w"], s["bI"], s["scores"], s["scores"].shape[-1], ws)
        return s["scores"]
    s["ints"].copy_(s["start_ints"])
    if op == "append":
        gsa.gsa_cache_reserve(cache, s["n_new"], s["start"], ws)
        gsa.gsa_cache_append(cache, s["K"], s["V"], s["g2"], s["kI"], s["n_new"], s["start"], ws)
        gsa.gsa_cache_read(cache, s["K_all"], s["V_all"], s["kI_all"], ws)
        return dict(K=s["K_all"], V=s["V_all"], kI=s["kI_all"], table=s["table"], lens=s["lens"], refs=s["refs"], start=s["start"])
    if op == "fork":
        gsa.gsa_cache_fork(cache, s["src_of"], c["share"], ws)
        gsa.gsa_cache_release(cache, s["drop"], ws)
        return dict(pool=s["pool"], table=s["table"], lens=s["lens"], refs=s["refs"])
    gsa.gsa_cache_compact(cache, s["live"], ws)
    return dict(pool=s["pool"], table=s["table"], refs=s["refs"], live=s["live"])


def _plain_attn(c, s):
    n_kv, G = c["n_kv"], c["n_h"] // c["n_kv"]
    pos = s["idx"].long().clamp(min=0)
    page = s["table"].long().gather(1, (pos // c["T"]).flatten(1)).view_as(pos).clamp(min=0)
    K, V = _values(c, _tokens(c, s["pool"])[0][page, pos % c["T"]])               # [B, Lq, k, n_kv, d_h]
    Q = s["Q"].float().unflatten(2, (n_kv, G))
    z = torch.einsum("bqhgd,bqkhd->bqhgk", Q, K) * c["d_h"] ** -0.5
    on = torch.arange(c["k_max"], device="cuda") < s["kt"][:, :, None, None, None]
    z = torch.where(on, z, -torch.inf)
    e = torch.where(on, torch.exp(z - z.amax(-1, keepdim=True)), 0.0)
    o = torch.einsum("bqhgk,bqkhd->bqhgd", e, V) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return (o.flatten(2, 3) / (1 + torch.exp(-s["g1"].float()))).to(BF16)


def _plain_scores(c, s):
    T, Lk = c["T"], c["Lk"]
    kI = _tokens(c, s["pool"])[1][s["table"].long().clamp(min=0)].flatten(1, 2)[:, :Lk].float()
    z = torch.einsum("bqhd,bkd->bqhk", s["qI"].float(), kI) + s["bI"][:, None]
    f = z.clamp(min=0) if c["act"] == 1 else 1 / (1 + torch.exp(-z))
    I = (f * s["w"][..., None]).sum(2)
    vis = s["lens"][:, None] - c["Lq"] + 1 + torch.arange(c["Lq"], device="cuda")
    out = s["scores"].clone()
    out[..., :Lk] = torch.where(torch.arange(Lk, device="cuda") < vis[..., None], I, out[..., :Lk])
    return out


def _free_pages(refs):
    """Page numbers, the free ones first, each part ascending."""
    return torch.argsort((refs != 0).to(U8), stable=True)


def _plain_append(c, s):
    T, B, Lq, Lk = c["T"], c["B"], c["Lq"], c["Lk"]
    s["ints"].copy_(s["start_ints"])
    table, lens, refs = s["table"], s["lens"].long(), s["refs"]
    n_new = s["n_new"].long()
    have, want = (lens + T - 1) // T, (lens + n_new + T - 1) // T
    first = torch.cumsum(want - have, 0) - (want - have)
    j = torch.arange(table.shape[1], device="cuda")
    fresh = (j >= have[:, None]) & (j < want[:, None])
    rank = (first[:, None] + j - have[:, None]).clamp(0, refs.numel() - 1)
    page = torch.where(fresh, _free_pages(refs)[rank], table.long())
    refs.index_add_(0, page.clamp(min=0).flatten(), fresh.to(I32).flatten())
    table.copy_(page)
    start = lens.to(I32)
    lens = lens + n_new
    s["lens"].copy_(lens)
    # the new tokens, by the position they take; a value's gate next to a border of bf16 needs 64 bits
    V = s["V"] if s["g2"] is None else (s["V"].double() / (1 + torch.exp(-s["g2"].double()))).to(BF16)
    r = _records(c, s["K"].float().flatten(0, 1), V.float().flatten(0, 1)).view(B, Lq, -1)
    recs, kI = _tokens(c, s["pool"])
    i = torch.arange(Lq, device="cuda")
    live = i < n_new[:, None]
    pos = (start.long()[:, None] + i).clamp(max=table.shape[1] * T - 1)
    at = page.gather(1, pos // T).clamp(min=0)
    spare = _free_pages(refs)[0]                 # (rows behind a sequence's new tokens go to a page that nothing names)
    at = torch.where(live, at, spare)
    recs[at, pos % T], kI[at, pos % T] = r, s["kI"]
    # the whole cache, contiguous
    all_pages = page.clamp(min=0)
    K, V = _values(c, recs[all_pages].flatten(1, 2)[:, :Lk])
    on = (torch.arange(Lk, device="cuda") < lens[:, None])[..., None]
    put = lambda x, old: torch.where(on.view(on.shape + (1,) * (x.dim() - 3)), x.to(BF16), old)  # noqa: E731
    return dict(K=put(K, s["K_all"]), V=put(V, s["V_all"]), kI=put(kI[all_pages].flatten(1, 2)[:, :Lk], s["kI_all"]), table=table,
                lens=s["lens"], refs=refs, start=start)


def _plain_fork(c, s):
    T = c["T"]
    s["ints"].copy_(s["start_ints"])
    table, lens, refs, src_of = s["table"], s["lens"].long(), s["refs"], s["src_of"].long()
    page_bytes = _sizes(c)[2]
    takes = src_of >= 0
    src = src_of.clamp(min=0)
    n = torch.where(takes, lens[src], torch.zeros_like(lens))
    shared = n // T if c["share"] else torch.zeros_like(n)
    want = (n + T - 1) // T
    first = torch.cumsum(want - shared, 0) - (want - shared)
    j = torch.arange(table.shape[1], device="cuda")
    fresh = (j >= shared[:, None]) & (j < want[:, None])
    joint = j < shared[:, None]
    free = _free_pages(refs)
    theirs = table.long()[src]
    mine = torch.where(fresh, free[(first[:, None] + j - shared[:, None]).clamp(0, refs.numel() - 1)], theirs)
    page = torch.where(fresh | joint, mine, table.long())
    # copies: every page's source, itself where nothing is copied to it
    source = torch.arange(refs.numel(), device="cuda")
    source[torch.where(fresh, mine, free[-1]).flatten()] = torch.where(fresh, theirs, free[-1]).flatten()
    pool = s["pool"].view(-1, page_bytes)[source].flatten()
    refs.index_add_(0, page.clamp(min=0).flatten(), (fresh | joint).to(I32).flatten())
    lens = torch.where(takes, n, lens)
    # the prompts' slots are given up
    drop = (s["drop"] != 0)[:, None] & (page >= 0)
    refs.index_add_(0, page.clamp(min=0).flatten(), -drop.to(I32).flatten())
    table.copy_(torch.where(drop, -1, page))
    s["lens"].copy_(torch.where(s["drop"] != 0, 0, lens))
    return dict(pool=pool, table=table, lens=s["lens"], refs=refs)


def _plain_compact(c, s):
    s["ints"].copy_(s["start_ints"])
    table, refs = s["table"], s["refs"]
    i = torch.arange(refs.numel(), device="cuda")
    live = refs > 0
    n = live.sum()
    moves, hole = live & (i >= n), ~live & (i < n)
    rank = torch.cumsum(moves, 0) - 1
    holes, movers = torch.argsort((~hole).to(U8), stable=True), torch.argsort((~moves).to(U8), stable=True)
    to = torch.where(moves, holes[rank.clamp(min=0)], i)                          # where a page goes
    hole_rank = (torch.cumsum(hole, 0) - 1).clamp(min=0)
    source = torch.where(hole, movers[hole_rank], i)                              # what a page holds afterwards
    pool = s["pool"].view(-1, _sizes(c)[2])[source].flatten()
    new_refs = torch.where(hole, refs[source], torch.where(moves, 0, refs))
    refs.copy_(new_refs)
    table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)], -1))
    return dict(pool=pool, table=table, refs=refs, live=n.to(I32).view(1))


# ---- the outputs in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] in ("fork", "compact"):
        return None                              # whole numbers and copied bytes
    lens = _lens(c)
    return dict(attn=_exact_attn, scores=_exact_scores, append=_exact_append)[c["op"]](c, s, lens)


def _scale64(byte):
    t = torch.tensor([(8 + n % 8) * 2.0 ** (n // 8 - 23) for n in range(255)] + [math.nan], dtype=F64, device="cuda")
    return t[byte.long()]


def _exact_attn(c, s, lens):
    D, rec, page_bytes = _sizes(c)
    T, d_h, G = c["T"], c["d_h"], c["n_h"] // c["n_kv"]
    pool = s["pool"].view(-1, page_bytes)
    out = torch.zeros(s["Q"].shape, dtype=F64, device="cuda")
    for b in range(c["B"]):
        for t in range(c["Lq"]):
            k = int(s["kt"][b, t])
            if not k:
                continue
            pos = s["idx"][b, t, :k].long()
            at = s["table"][b].long()[pos // T] * page_bytes + (pos % T) * rec
            r = pool.view(-1)[at[:, None] + torch.arange(rec, device="cuda")]
            scale = _scale64(r[:, D:D + D // 8]).view(k, c["n_kv"], 2, d_h // 16)

            def half(i):
                by = r[:, i * (D // 2):(i + 1) * (D // 2)].to(F64)
                code = torch.empty(k, D, dtype=F64, device="cuda")
                code[:, 1::2] = torch.floor(by / 16)
                code[:, 0::2] = by - 16 * code[:, 1::2]
                return (code.view(k, c["n_kv"], d_h // 16, 16) - 8) * scale[:, :, i, :, None]

            K, V = half(0).reshape(k, c["n_kv"], d_h), half(1).reshape(k, c["n_kv"], d_h)
            a = torch.softmax(torch.einsum("hgd,khd->hgk", s["Q"][b, t].double().view(-1, G, d_h), K) / math.sqrt(d_h), -1)
            out[b, t] = torch.einsum("hgk,khd->hgd", a, V).reshape(c["n_h"], d_h) * torch.sigmoid(s["g1"][b, t].double())
    return out


def _exact_scores(c, s, lens):
    T, page_bytes, rec = c["T"], _sizes(c)[2], _sizes(c)[1]
    out = s["scores"].double()
    for b, n in enumerate(lens):
        if not n:
            continue
        pos = torch.arange(n, device="cuda")
        at = s["table"][b].long()[pos // T] * (page_bytes // 2) + (T * rec // 2) + (pos % T) * c["dI"]
        k = s["pool"].view(BF16)[at[:, None] + torch.arange(c["dI"], device="cuda")].double()
        for t in range(c["Lq"]):
            vis = n - c["Lq"] + t + 1
            z = s["qI"][b, t].double() @ k[:vis].T + s["bI"].double()[:, None]
            out[b, t, :vis] = s["w"][b, t].double() @ (z.clamp(min=0) if c["act"] == 1 else torch.sigmoid(z))
    return out


def _exact_append(c, s, lens):
    D, rec, page_bytes = _sizes(c)
    T, d_h, n_kv = c["T"], c["d_h"], c["n_kv"]
    half = torch.arange(D // 2, device="cuda")

    def stored(x):                               # what 4 bits keep of x [N, n_kv, d_h]
        g = x.reshape(x.shape[0], n_kv, d_h // 16, 16)
        y = g.abs().amax(-1, keepdim=True) / 7
        m, e = torch.frexp(y)                    # y = m * 2^e, 0.5 <= m < 1: three more bits of m, halves up
        sc = torch.floor(m * 16 + 0.5) / 16 * torch.exp2(e.double())
        sc = sc.clamp(2.0 ** -20, 1.75 * 2.0 ** 11)
        return ((g / sc).round().clamp(-7, 7) * sc).reshape(x.shape)

    K, V, kI = s["K_all"].double(), s["V_all"].double(), s["kI_all"].double()
    old = [n - m for n, m in zip(lens, _new(c, lens))]
    for b, n in enumerate(old):
        if n:
            pos = torch.arange(n, device="cuda")
            page = s["table"][b].long()[pos // T]
            at = page * page_bytes + (pos % T) * rec
            by = s["pool"]
            sc = _scale64(by[at[:, None] + D + torch.arange(D // 8, device="cuda")]).view(n, n_kv, 2, d_h // 16)
            for i, x in enumerate((K, V)):
                v = by[at[:, None] + i * (D // 2) + half].to(F64)
                hi = torch.floor(v / 16)
                code = torch.stack((v - 16 * hi, hi), -1).view(n, n_kv, d_h // 16, 16) - 8
                x[b, :n] = (code * sc[:, :, i, :, None]).view(n, n_kv, d_h)
            ki = page * (page_bytes // 2) + T * rec // 2 + (pos % T) * c["dI"]
            kI[b, :n] = by.view(BF16)[ki[:, None] + torch.arange(c["dI"], device="cuda")].double()
        m = lens[b] - n
        if m:
            v = s["V"][b, :m].double()
            if s["g2"] is not None:
                v = (v * torch.sigmoid(s["g2"][b, :m].double())).to(BF16).double()
            K[b, n:n + m], V[b, n:n + m], kI[b, n:n + m] = stored(s["K"][b, :m].double()), stored(v), s["kI"][b, :m].double()
    return dict(K=K, V=V, kI=kI, table=None, lens=None, refs=None, start=None)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    c = case
    D, rec, page = _sizes(c)
    B, Lq, lens = c["B"], c["Lq"], _lens(c)
    token = D + D // 8
    if c["op"] == "attn":
        rows = _rows(c, lens)
        pairs = sum(k for _, k in rows)
        # a sequence's tokens are read once, however many of its rows select them
        read = sum(min(n, sum(k for _, k in rows[b * Lq:(b + 1) * Lq])) for b, n in enumerate(lens))
        return {"bytes": read * token + 4 * pairs + 6 * B * Lq * c["n_h"] * c["d_h"], "flops": 4 * pairs * c["n_h"] * c["d_h"]}
    if c["op"] == "scores":
        pairs = sum(v for v, _ in _rows(c, lens))
        return {"bytes": 2 * c["dI"] * sum(lens) + 4 * pairs + B * Lq * c["HI"] * (2 * c["dI"] + 4), "flops": 2 * pairs * c["HI"] * c["dI"]}
    if c["op"] == "append":
        n = sum(_new(c, lens))
        return {"bytes": n * (2 * D * (3 if c["gate"] else 2) + token + 4 * c["dI"]) + sum(lens) * (token + 4 * D + 4 * c["dI"]), "flops": 0}
    pages = sum(-(-n // c["T"]) for n in lens)
    if c["op"] == "fork":
        moved = 4 * sum((1 if n % c["T"] else 0) if c["share"] else -(-n // c["T"]) for n in lens)
        return {"bytes": 2 * moved * page + 4 * (12 * pages), "flops": 0}
    return {"bytes": 2 * (pages // 4) * page + 4 * (6 * pages), "flops": 0}
