"""The paged 4-bit cache in plain numpy, in 64 bits and loops: what include/gsa.h says, without the library's code."""
from __future__ import annotations

import math

import numpy as np
import torch


def bf16(x: np.ndarray) -> np.ndarray:
    """fp64 -> fp32 -> bf16 (each to nearest, halves to even), as fp64."""
    with np.errstate(all="ignore"):
        f = np.asarray(x, np.float64).astype(np.float32)
    return torch.from_numpy(f).to(torch.bfloat16).double().numpy()


def scale_of(byte: int) -> float:
    return math.nan if byte == 255 else (8 + byte % 8) * 2.0 ** (byte // 8 - 23)


SCALES = np.array([scale_of(n) for n in range(255)])


def encode(x: np.ndarray):
    """x [..., 16 m] fp64 -> (codes [..., 16 m] uint8, scale bytes [..., m] uint8)."""
    g = x.reshape(*x.shape[:-1], -1, 16)
    amax = np.abs(g).max(-1)
    fine = np.isfinite(g).all(-1)
    y = np.where(fine, amax, 0.0) / 7
    # the scale that y rounds to, halves up: the number of midpoints at or below y
    byte = np.searchsorted((SCALES[:-1] + SCALES[1:]) / 2, y, side="right")
    s = SCALES[byte]
    with np.errstate(all="ignore"):
        c = np.clip(np.rint(np.where(fine[..., None], g, 0.0) / s[..., None]), -7, 7)
    return (c + 8).astype(np.uint8).reshape(x.shape), np.where(fine, byte, 255).astype(np.uint8)


def decode(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    s = np.append(SCALES, math.nan)[byte]
    g = codes.reshape(*codes.shape[:-1], -1, 16).astype(np.float64) - 8
    return (g * s[..., None]).reshape(codes.shape)


class PlainCache:
    """Tables and pages as the library keeps them; a page's bytes in the library's layout."""

    def __init__(self, B, n_pages, T, max_pages, n_kv, d_h, dI):
        self.B, self.n_pages, self.T, self.max_pages, self.n_kv, self.d_h, self.dI = B, n_pages, T, max_pages, n_kv, d_h, dI
        D = n_kv * d_h
        self.D, self.rec = D, (D + D // 8 + 15) // 16 * 16
        self.page_bytes = T * (self.rec + 2 * dI)
        self.pool = np.zeros((n_pages, self.page_bytes), np.uint8)
        self.table = np.full((B, max_pages), -1, np.int32)
        self.lens = np.zeros(B, np.int32)
        self.refs = np.zeros(n_pages, np.int32)

    def pages_of(self, n):
        return -(-int(n) // self.T)

    # ---- pages: each returns the status word ----
    def _take(self, requests):
        """requests: [(b, slot)] in order; the page numbers, or None if there are too few."""
        free = np.flatnonzero(self.refs == 0)
        if len(free) < len(requests):
            return None
        for (b, j), page in zip(requests, free):
            self.table[b, j] = page
            self.refs[page] = 1
        return free[:len(requests)]

    def reserve(self, n_new):
        n_new = np.asarray(n_new)
        if (n_new < 0).any() or (self.lens + n_new.astype(np.int64) > self.max_pages * self.T).any():
            return 6, np.full(self.B, -1, np.int32)
        req = [(b, j) for b in range(self.B) for j in range(self.pages_of(self.lens[b]), self.pages_of(self.lens[b] + n_new[b]))]
        if self._take(req) is None:
            return 7, np.full(self.B, -1, np.int32)
        start = self.lens.copy()
        self.lens = (self.lens + n_new).astype(np.int32)
        return 0, start

    def fork(self, src_of, share):
        src_of = np.asarray(src_of)
        for b, s in enumerate(src_of):
            if s >= 0 and (s >= self.B or s == b or self.lens[b] != 0 or src_of[s] >= 0):
                return 6
        req, copies = [], []
        for b, s in enumerate(src_of):
            if s < 0:
                continue
            first = self.lens[s] // self.T if share else 0
            for j in range(first, self.pages_of(self.lens[s])):
                req.append((b, j))
                copies.append(self.table[s, j])
        new = self._take(req)
        if new is None:
            return 7
        for a, p in zip(copies, new):
            self.pool[p] = self.pool[a]
        for b, s in enumerate(src_of):
            if s >= 0:
                if share:
                    for j in range(self.lens[s] // self.T):
                        self.table[b, j] = self.table[s, j]
                        self.refs[self.table[s, j]] += 1
                self.lens[b] = self.lens[s]
        return 0

    def release(self, drop):
        for b, d in enumerate(drop):
            if d:
                for j in range(self.pages_of(self.lens[b])):
                    self.refs[self.table[b, j]] -= 1
                self.table[b] = -1
                self.lens[b] = 0
        return 0

    def compact(self):
        live = np.flatnonzero(self.refs)
        n = len(live)
        for p, hole in zip(live[live >= n], np.flatnonzero(self.refs[:n] == 0)):
            self.pool[hole] = self.pool[p]
            self.table[self.table == p] = hole
            self.refs[hole], self.refs[p] = self.refs[p], 0
        return n

    # ---- tokens ----
    def append(self, K, V, g2, kI, n_new, start):
        """K, V, g2 [B, L, n_kv, d_h] fp64 (bf16 values), kI [B, L, dI] uint16 (bf16 bits)."""
        with np.errstate(all="ignore"):
            Vg = V if g2 is None else bf16(V / (1 + np.exp(-g2)))
        for b in range(self.B):
            for i in range(int(n_new[b]) if start[b] >= 0 else 0):
                s = int(start[b]) + i
                page, slot = self.table[b, s // self.T], s % self.T
                r = self.pool[page, slot * self.rec:(slot + 1) * self.rec]
                scales = np.empty((self.n_kv, 2, self.d_h // 16), np.uint8)
                for k, x in enumerate((K[b, i], Vg[b, i])):
                    u, byte = encode(x)
                    u = u.reshape(-1)
                    r[k * self.D // 2:(k + 1) * self.D // 2] = u[0::2] | (u[1::2] << 4)
                    scales[:, k] = byte
                r[self.D:self.D + self.D // 8] = scales.reshape(-1)
                at = self.T * self.rec + slot * 2 * self.dI
                self.pool[page, at:at + 2 * self.dI] = kI[b, i].view(np.uint8)

    def tokens(self, b, pos):
        """K, V' [n, n_kv, d_h] fp64 and kI [n, dI] fp64 of the listed positions."""
        pos = np.asarray(pos, np.int64)
        page, slot = self.table[b, pos // self.T], pos % self.T
        r = self.pool[page[:, None], (slot * self.rec)[:, None] + np.arange(self.rec)]
        scales = r[:, self.D:self.D + self.D // 8].reshape(-1, self.n_kv, 2, self.d_h // 16)
        out = []
        for k in range(2):
            by = r[:, k * self.D // 2:(k + 1) * self.D // 2]
            u = np.stack((by & 15, by >> 4), -1).reshape(-1, self.n_kv, self.d_h)
            out.append(decode(u, scales[:, :, k]))
        ki = self.pool[page[:, None], (self.T * self.rec + slot * 2 * self.dI)[:, None] + np.arange(2 * self.dI)]
        ki = (np.ascontiguousarray(ki).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        return out[0], out[1], ki.reshape(len(pos), self.dI)

    # ---- stages ----
    def scores(self, b, t, Lq, qI, w, bI, act):
        """Row t of sequence b: I over its visible keys."""
        n = max(0, int(self.lens[b]) - Lq + t + 1)
        if n == 0:
            return np.zeros(0)
        z = qI @ self.tokens(b, np.arange(n))[2].T + bI[:, None]
        return w @ (np.maximum(z, 0) if act else 1 / (1 + np.exp(-z)))

    def attn(self, b, Q, g1, pos, sm_scale):
        """One row: (out [n_h, d_h], sigmoid(g1) * sum_j a_j |v_j|: the scale of its roundings)."""
        n_h = Q.shape[0]
        if len(pos) == 0:
            return np.zeros_like(Q), np.zeros_like(Q)
        K, V, _ = self.tokens(b, pos)
        G = n_h // self.n_kv
        out, mag = np.empty_like(Q), np.empty_like(Q)
        gate = 1 / (1 + np.exp(-g1))
        for h in range(n_h):
            z = K[:, h // G] @ Q[h] * sm_scale
            e = np.exp(z - z.max())
            a = e / e.sum()
            out[h], mag[h] = (a @ V[:, h // G]) * gate[h], (a @ np.abs(V[:, h // G])) * gate[h]
        return out, mag
