"""Inputs, tolerances and checks of the tests of the paged cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged_oracle as O
from paper_2412_04757_amd import LtriPagedCache, paged_config

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """A cache on the device and the same in numpy (64 bits). Places that hold no token are NaN, tables name no page there."""

    def __init__(self, device, lens, *, hq=8, hkv=2, dim=128, dtype="bf16", page=16, rows=1, weights=True, seed=0, spare=3, room=0, token_major=False,
                 seen=None, max_rows=None):
        self.device, self.dtype, self.rows, self.dim, self.hq, self.hkv, self.page = device, dtype, rows, dim, hq, hkv, page
        self.gen = torch.Generator().manual_seed(seed)
        S, width = len(lens), max(1, -(-(max(lens) + room) // page))
        need = [-(-(n + room) // page) for n in lens]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=self.gen).tolist()
        self.table = np.full((S, width), -1, np.int32)
        for s in range(S):
            for p in range(need[s]):
                self.table[s, p] = order.pop()
        self.lens = np.array(lens, np.int32)
        self.seen = np.array(lens if seen is None else seen, np.int32)
        shape = (n_pages, hkv, page, dim)
        self.k, self.v = np.full(shape, np.nan), np.full(shape, np.nan)
        self.weight = np.full(shape[:3], np.nan, np.float32).astype(np.float64) if weights else None
        self.pos = np.full(shape[:3], -7, np.int64) if weights else None
        for s in range(S):
            T = int(lens[s])
            if not T:
                continue
            i = np.arange(T)
            pg, sl = self.table[s][i // page], i % page
            mean = self.values((T // 24 + 1, hkv, dim))[i // 24]
            self.k[pg, :, sl] = self.round(mean + 0.3 * self.values((T, hkv, dim)))
            self.v[pg, :, sl] = self.values((T, hkv, dim))
            if weights:
                self.weight[pg, :, sl] = torch.rand((T, hkv), generator=self.gen).double().numpy()
                self.pos[pg, :, sl] = i[:, None]
        self.q = self.values((S, rows, hq, dim))
        self.k_new, self.v_new = self.values((S, hkv, rows, dim)), self.values((S, hkv, rows, dim))
        cfg = paged_config(hq, hkv, dim, dtype, page_tokens=page, n_pages=n_pages, table_pages=width, max_seqs=S,
                           rows_max=rows if max_rows is None else max_rows, weights=weights)
        pools = [self.on(x) for x in (self.k, self.v)]
        if token_major:
            pools = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in pools]
        self.cache = LtriPagedCache(cfg, device, k_pages=pools[0], v_pages=pools[1],
                                    weight=torch.from_numpy(self.weight).float().to(device) if weights else None,
                                    pos=torch.from_numpy(self.pos).int().to(device) if weights else None)
        self.cache.scratch.fill_(0xFF)                    # NaN wherever something is read that no launch wrote
        self.push()

    def values(self, shape):
        return self.round(torch.randn(shape, generator=self.gen).numpy())

    def round(self, x):
        return torch.as_tensor(x).to(TYPES[self.dtype]).double().numpy()

    def on(self, x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(TYPES[self.dtype]).to(self.device)

    def push(self):
        self.d_table, self.d_lens, self.d_seen = (torch.from_numpy(x.copy()).to(self.device) for x in (self.table, self.lens, self.seen))

    def args(self, seen=True):
        return (self.d_table, self.d_lens, self.d_seen) if seen else (self.d_table, self.d_lens)

    def new_lse(self):
        return torch.full(self.q.shape[:3], float("nan"), dtype=torch.float32, device=self.device)

    def tolerances(self, n_sum=None):
        """Bounds by arithmetic. A score is a sum of d products in 32 bits (each addition off by at most 2^-23 of the sum of
        magnitudes, whatever its rounding), scaled and its exponential taken (a few 2^-23 each, and as much for scores of up to 32);
        sums over n tokens are off by at most n 2^-24 where they are formed one by one. The result and the weights are quotients of two such sums."""
        n = int(self.lens.max()) if n_sum is None else n_sum
        there = np.isfinite(self.k)
        size = np.sqrt(np.nanmax((np.where(there, self.k, 0.0) ** 2).sum(-1))) * np.sqrt((self.q ** 2).sum(-1).max()) / np.sqrt(self.dim)
        score = (self.dim + 4) * 2.0 ** -23 * size + 8 * 2.0 ** -23
        rel = 2 * score + 2 * n * 2.0 ** -24 + 8 * 2.0 ** -23
        split = 2.0 ** -16 if self.dtype == "bf16" else 0.0          # probabilities as two bf16 parts
        v = np.nanmax(np.abs(np.where(np.isfinite(self.v), self.v, 0.0)))
        return {"out_abs": (rel + split) * v, "out_rel": torch.finfo(TYPES[self.dtype]).eps / 2, "lse": rel + 2.0 ** -23 * (size + 16), "weight": rel}

    def check_attend(self, out, lse, want, want_lse):
        t = self.tolerances()
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= t["out_abs"] + t["out_rel"] * 1.01 * np.abs(want)).all(), np.abs(got - want).max()
        if lse is not None:
            got = lse.double().cpu().numpy()
            there = ~np.isneginf(want_lse)
            assert np.array_equal(~np.isneginf(got), there)
            off = np.abs(got[there] - want_lse[there])
            assert (off <= t["lse"]).all(), off.max()

    def check_weight(self):
        """Weights against the oracle's, which has run on self.weight; places without a token as they were."""
        got, want = self.cache.weight.double().cpu().numpy(), self.weight
        assert np.array_equal(np.isnan(got), np.isnan(want))
        there = ~np.isnan(want)
        # a weight has at most rows x group shares of 1 each, one more rounding or two
        t = self.tolerances()["weight"] * 1.0 + 4 * 2.0 ** -23
        assert (np.abs(got - want)[there] <= t * np.abs(want[there]) + 2.0 ** -30).all(), (np.abs(got - want)[there] / want[there]).max()

    def check_pools(self):
        """Rows, to the bit, and positions."""
        for got, want in ((self.cache.k_pages, self.k), (self.cache.v_pages, self.v)):
            assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
        if self.pos is not None:
            assert np.array_equal(self.cache.pos.cpu().numpy(), self.pos)

    def oracle_attend(self, decay=None):
        return O.attend(self.k, self.v, self.weight, self.table, self.lens, self.q, decay)

    def oracle_append(self, w_new=None):
        O.append(self.k, self.v, self.weight, self.pos, self.table, self.lens, self.seen, self.k_new, self.v_new, w_new)
