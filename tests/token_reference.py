"""Small caches and plain 64-bit forms for the tests of drafted tokens and of token eviction."""
import math

import numpy as np
import torch

import paper_2502_15294_amd as ra

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


class Cache:
    """A layer's history in the library's layout, beside its rounds as dense arrays: k[b][r], v[b][r] are float64
    [Hkv, len, d].  Padding of the value tiles is 7, storage that belongs to no round NaN."""

    def __init__(self, lens, Hkv, d, dtype, paged, seed=0, R_max=None, device="cuda", values=True):
        rng = np.random.default_rng(seed)
        self.B, self.R, self.Hkv, self.d, self.dtype, self.paged = len(lens), R_max or max([len(l) for l in lens] + [1]), Hkv, d, dtype, paged
        self.lens = np.zeros((self.B, self.R), dtype=np.int32)
        for b, l in enumerate(lens):
            self.lens[b, :len(l)] = l
        self.n = np.array([len(l) for l in lens], dtype=np.int32)
        self.k = [[self.draw(rng, (Hkv, n, d)) for n in l] for l in lens]
        self.v = [[self.draw(rng, (Hkv, n, d)) for n in l] for l in lens]
        self.place(rng)
        nk, nv = self.pool
        k, v = np.full((nk * Hkv + 1, d), np.nan), np.full(nv * Hkv * d + 16, np.nan)
        for b, l in enumerate(lens):
            for r, n in enumerate(l):
                rows, elems, pad = self.where(b, r)
                k[rows], v[elems], v[pad] = self.k[b][r], self.v[b][r], 7.0
        up = lambda x: torch.from_numpy(x).to(TORCH[dtype]).to(device)  # noqa: E731
        self.dk, self.dv = up(k), up(v) if values else None
        t = lambda x: torch.from_numpy(x).to(device)  # noqa: E731
        self.seg_len, self.n_rounds = t(self.lens), t(self.n)
        self.view = ra.KVView(self.dk, self.dv, t(self.off), self.seg_len, self.n_rounds, Hkv, d, int(self.lens.sum(1).max()),
                              block_table=t(self.table) if paged else None, block_size=16 if paged else 0,
                              seg_off_v=None if paged else t(self.off_v))

    def draw(self, rng, shape):
        return torch.from_numpy(rng.standard_normal(shape)).to(TORCH[self.dtype]).double().numpy()

    def place(self, rng):
        l16 = (self.lens.astype(np.int64) + 15) // 16 * 16
        if self.paged:
            slots = l16 // 16
            self.off = np.cumsum(slots, 1) - slots
            self.off_v = None
            total = int(slots.sum())
            ids = rng.permutation(total + 3).astype(np.int32)  # some blocks belong to nobody
            self.table = np.full((self.B, max(1, int(slots.sum(1).max()))), 0, dtype=np.int32)
            at = 0
            for b in range(self.B):
                m = int(slots[b].sum())
                self.table[b, :m] = ids[at:at + m]
                at += m
            self.pool = ((total + 3) * 16,) * 2
        else:
            flat = self.lens.astype(np.int64).ravel()
            self.off = (np.cumsum(flat) - flat).reshape(self.lens.shape) + 2
            self.off_v = (np.cumsum(l16.ravel()) - l16.ravel()).reshape(self.lens.shape) + 16
            self.table = None
            self.pool = (int(flat.sum()) + 2, int(l16.sum()) + 16)

    def where(self, b, r):
        """Rows of the keys [Hkv, len], elements of the values [Hkv, len, d], elements of the last value tile's padding."""
        n, Hkv, d = int(self.lens[b, r]), self.Hkv, self.d
        g, t = np.arange(Hkv)[:, None], np.arange((n + 15) // 16 * 16)[None]
        if self.paged:
            block = self.table[b, self.off[b, r] + t // 16].astype(np.int64) if n else t
            rows = (block * Hkv + g) * 16 + t % 16
            elems = (block * Hkv + g) * d * 16 + t % 16
        else:
            rows = self.off[b, r] * Hkv + g * n + t
            elems = (self.off_v[b, r] * Hkv + g * ((n + 15) // 16 * 16) + t // 16 * 16) * d + t % 16
        elems = elems[..., None] + 16 * np.arange(d)
        return rows[:, :n], elems[:, :n], elems[:, n:]

    def history(self, b, sel):
        """Keys and values [Hkv, tokens, d] of the listed rounds (None: all), one after the other."""
        rounds = range(self.n[b]) if sel is None else [r for r in sel[b] if 0 <= r < self.n[b]]
        empty = np.zeros((self.Hkv, 0, self.d))
        return (np.concatenate([empty] + [self.k[b][r] for r in rounds], 1), np.concatenate([empty] + [self.v[b][r] for r in rounds], 1))


def context(cache, Hq, q_len, cur_cap=0):
    """A context and its workspace, as large as the library asks for."""
    ctx = ra.ra_create(0)
    n = ra.ra_workspace_bytes(cache.B, cache.R, Hq, cache.Hkv, cache.d, q_len, ra.RA_BF16 if cache.dtype == "bf16" else ra.RA_F32,
                              int(cache.lens.sum(1).max()) + cur_cap)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")  # (as a number: NaN)
    ra.ra_set_workspace(ctx, ws)
    return ctx, ws


def selection(cache, sel, device="cuda"):
    idx = np.full((cache.B, cache.R), -1, dtype=np.int32)
    for b, s in enumerate(sel):
        idx[b, :len(s)] = s
    return torch.from_numpy(idx).to(device), torch.tensor([len(s) for s in sel], dtype=torch.int32, device=device)


def softmax_rows(s):
    """Weights and log-sum-exp of logits [rows, tokens]; a row without tokens: zeros and -inf."""
    top = np.maximum(s.max(1, initial=-np.inf, keepdims=True), -1e300)
    e = np.exp(s - top)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.log(total) + top
    return e / np.maximum(total, 1e-300), np.where(total > 0, lse, -np.inf)[:, 0]


def unit_roundoff_sum(n):
    """Largest relative error of a sum of n products in fp32, in any order: n halves of a step, 2^-24 each."""
    return n * 2.0 ** -24


def logit_error(q, k, scale):
    """Bound of what a logit computed in fp32 is off by, for the whole set: the sum of |q k| times the error of a sum of d
    products, and its product with the scale."""
    d = q.shape[-1]
    largest = float((np.abs(q).reshape(-1, d) @ np.abs(k).reshape(-1, d).T).max(initial=0.0)) * scale
    return largest * (unit_roundoff_sum(d) + 4 * 2.0 ** -24)


def scale_of(d):
    return 1.0 / math.sqrt(d)
