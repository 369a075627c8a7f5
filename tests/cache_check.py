"""The attention over a paged 4-bit cache against its plain 64-bit form, every rounding of the kernel counted.

For one row, head h, with a = softmax(z), z = sm_scale K q, over keys whose K codes have the scales s (one for 16 values):
  scores      Up to four query heads a KV head: 16 values of one scale are summed up as sum u q, u = 0 .. 15, from -8 sum q on, in fp32, by
              four matrix instructions of four products each.  Partial sums stay within 8 sum |q|, products within 15 sum |q|; an instruction cuts each
              of its five addends by at most 2^-23 of the largest and the result by 2^-23 of its own: 4 (5 * 15 + 8) 2^-23 sum |q|; the start is
              15 sums in fp32, 8 * 15 * 2^-24.  Together below 2^-14 s sum |q|.  (Q as fp16 adds 2^-35 max|q| of its head for a value, which is less.)
              Eight heads: products of bf16 are exact, eight instructions of 17 addends: 136 * 2^-23 < 2^-15 of sum |q k|.
              The scaled score and its distance from the reference: within 2^-21 of the row's largest |z|.
  numerators  2^x within 2^-21, then e of the scores' error dz in all: exp(dz) - 1 + 2^-21, in numerator and denominator alike: twice that.
              Rounded to fp16 for the product with V', the row's largest being at least 2^7: 2^-11 of each, or 2^-32 of the row's sum.
  sums        fp32: a matrix instruction of 17 addends for each tile of a unit's run, merges of a row's parts and the sum of the numerators in fp32.
  out         normalised and gated in fp32 (2^-20), rounded to bf16 (2^-8).
"""
import numpy as np

from test_gpu_cache import f64


def key_scales(P, b, pos):
    """Scales of K's codes [n, n_kv, d_h / 16] of the listed positions, NaN where the byte is 255."""
    pos = np.asarray(pos, np.int64)
    page, slot = P.table[b, pos // P.T], pos % P.T
    byte = P.pool[page[:, None], (slot * P.rec + P.D)[:, None] + np.arange(P.D // 8)].reshape(-1, P.n_kv, 2, P.d_h // 16)[:, :, 0].astype(np.int64)
    return np.where(byte == 255, np.nan, (8 + byte % 8) * 2.0 ** (byte // 8 - 23))


def score_error(P, b, q, pos, sm_scale, K=None):
    """(bound of a score's error, largest |score|) of every head."""
    n_h = q.shape[0]
    G = n_h // P.n_kv
    K = P.tokens(b, pos)[0] if K is None else K
    err, top = np.zeros(n_h), np.zeros(n_h)
    s = key_scales(P, b, pos)
    for h in range(n_h):
        kv = h // G
        if G <= 4:
            e = 2.0 ** -14 * (s[:, kv] @ np.abs(q[h]).reshape(-1, 16).sum(1)) + 2.0 ** -35 * np.abs(q[h]).max() * np.abs(K[:, kv]).sum(1)
        else:
            e = 2.0 ** -15 * (np.abs(K[:, kv]) @ np.abs(q[h]))
        top[h] = np.abs(K[:, kv] @ q[h]).max() * sm_scale
        err[h] = e.max() * sm_scale + 2.0 ** -21 * top[h]
    return err, top


def check_attention(P, Q, g1, out, sets, Lq, sm_scale, rows=None, run_tiles=8, heads=None):
    """sets[b][t]: positions; rows: those that are compared (all); run_tiles: at least as many as a unit has tiles; heads: those compared."""
    got = f64(out)
    seen = 0
    for b in range(P.B):
        for t in range(Lq):
            if rows is not None and (b, t) not in rows:
                continue
            pos = np.asarray(sets[b][t], np.int64)
            if len(pos) == 0:
                assert (got[b, t] == 0).all(), (b, t)
                continue
            q = f64(Q[b, t])
            n_h = q.shape[0]
            want, mag = P.attn(b, q, f64(g1[b, t]), pos, sm_scale)
            K, V, _ = P.tokens(b, pos)
            with np.errstate(over="ignore"):
                e = np.minimum(np.expm1(score_error(P, b, q, pos, sm_scale, K)[0])[:, None] + 2.0 ** -21, 1e9)
            tiny = 2.0 ** -32 * np.repeat(np.abs(V).sum(0), n_h // P.n_kv, 0)
            sums = (17 * run_tiles + 128) * 2.0 ** -23 + 2.0 ** -20
            tol = mag * (2.0 ** -11 + 2 * e * (1 + e) + sums) * 1.01 + tiny
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 1e-30
            bad = np.abs(got[b, t] - want) > tol
            bad |= ~np.isfinite(got[b, t])
            if heads is not None:
                bad = bad[list(heads)]
            assert not bad.any(), (b, t, np.argwhere(bad)[:4], (np.abs(got[b, t] - want) / tol).max())
            seen += 1
    assert seen or rows is None
