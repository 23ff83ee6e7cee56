"""Paged-cache test states: pools, tables and lengths in numpy, and their contiguous copies for the 64-bit oracle."""
from __future__ import annotations

import numpy as np

from paper_2603_30033_b200 import workloads as W
from tests import helpers as H

U_BF16, U_FP32 = 2.0 ** -8, 2.0 ** -24        # half a step, relative


def half_step(dtype):
    return U_BF16 if dtype == "bf16" else U_FP32


# Slots that a state's table has room for at least.  A step chooses its kernels by what the table can hold, not by lengths it cannot see:
# with room for 32768 the kernels for long contexts run, with just enough the one-launch form wherever it is built for the shape.
ROOM = 32768


class PagedState:
    """Random paged caches of `lens` own slots per sequence behind a prefix of P slots.  Everything that no call may use
    (unused slots, unowned pages, table entries past a sequence's last page) holds NaN, infinities and bad page numbers."""

    def __init__(self, w, lens, page, *, P=0, new=1, seed=5, spare=2, core_gain=1.0):
        self.w, self.lens, self.page, self.P = w, list(lens), page, P
        rng = np.random.default_rng(seed)
        B, r3, t3 = len(lens), w.r[2], w.t[2]
        new = [new] * B if np.isscalar(new) else list(new)
        need = [-(-(n + m) // page) for n, m in zip(lens, new)]
        pre = -(-P // page)
        self.n_pages = sum(need) + pre + spare
        self.max_pages = max(max(max(need), 1) + 1, -(-ROOM // page))
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((B, self.max_pages), -7, np.int32)
        self.table[:, -1] = 1 << 30
        o = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[o:o + n]
            o += n
        self.prefix_table = order[o:o + pre].copy()
        bad = np.array([np.nan, np.inf, -np.inf, 3e38], np.float32)
        self.K = bad[rng.integers(0, 4, (self.n_pages, page, r3))]
        self.V = bad[rng.integers(0, 4, (self.n_pages, page, t3))]
        self.shared = w.shared_kv
        if self.shared:
            self.V = self.K
        # own rows and prefix rows, rounded to the storage type
        rows = lambda n, r: W.round_to_storage(rng.standard_normal((n, r)), w.dtype)
        self.own_k = [rows(n, r3) for n in lens]
        self.own_v = self.own_k if self.shared else [rows(n, t3) for n in lens]
        self.pre_k = rows(P, r3)
        self.pre_v = self.pre_k if self.shared else rows(P, t3)
        for b, n in enumerate(lens):
            self.scatter(self.K, self.table[b], self.own_k[b])
            self.scatter(self.V, self.table[b], self.own_v[b])
        self.scatter(self.K, self.prefix_table, self.pre_k)
        self.scatter(self.V, self.prefix_table, self.pre_v)
        self.x = W.round_to_storage(rng.standard_normal((B, w.d_model)), w.dtype)
        wt = {k: W.round_to_storage(v, w.dtype) for k, v in W.make_weights(w, core_gain=core_gain).items()}
        if self.shared:
            wt["Ut3"] = wt["U3"]
        self.wt = wt

    def scatter(self, pool, pages, rows, first=0):
        for i, row in enumerate(rows, start=first):
            pool[pages[i // self.page], i % self.page] = row

    def contiguous(self):
        """[B, P + max len + 1, r] copies of the keys and values as one sequence holds them, and their lengths."""
        B, cap = len(self.lens), self.P + max(self.lens) + 1
        Kc = np.zeros((B, cap, self.w.r[2]))
        Vc = np.zeros((B, cap, self.w.t[2]))
        for b, n in enumerate(self.lens):
            Kc[b, :self.P], Vc[b, :self.P] = self.pre_k, self.pre_v
            Kc[b, self.P:self.P + n], Vc[b, self.P:self.P + n] = self.own_k[b], self.own_v[b]
        return Kc, Vc, np.array([self.P + n for n in self.lens], np.int32)

    def device(self):
        """Device tensors: x, weights, K, V, table, lengths, prefix table."""
        import torch
        w = self.w
        dw = H.weights_to_device(self.wt, w.dtype)
        K = H.to_device(self.K, w.dtype)
        V = K if self.shared else H.to_device(self.V, w.dtype)
        if self.shared:
            dw[7] = dw[3]
        i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
        return H.to_device(self.x, w.dtype), dw, K, V, i32(self.table), i32(self.lens), i32(self.prefix_table)

    def oracle_step(self):
        """(y, new key rows as cached, new value rows) of one decode step in 64 bits."""
        from oracle import tucker_oracle as O
        w, wt = self.w, self.wt
        Kc, Vc, lens = self.contiguous()
        if self.shared and w.rope:
            y, l = O.tucker_attn_decode_shared_rope(self.x, wt["C"], wt["U1"], wt["U2"], wt["U3"], wt["Ct"], wt["Ut1"],
                                                    wt["Ut2"], Kc, lens, rope_base=w.rope_base)
            return y, l, l
        return O.tucker_attn_decode(self.x, *[wt[k] for k in H.WEIGHT_KEYS], Kc, Vc, lens, rope=w.rope, rope_base=w.rope_base)

    def expect_pool(self, before, slot_rows, r):
        """`before` (a pool as numpy) with rows written: slot_rows = [(sequence, slot, row)]; and the mask of those rows."""
        out, mask = before.copy(), np.zeros(before.shape[:2], bool)
        for b, slot, row in slot_rows:
            pg = self.table[b, slot // self.page]
            out[pg, slot % self.page], mask[pg, slot % self.page] = row, True
        return out, mask


def check_rows(got, ref, dtype, what):
    """Output rows against 64 bits, row by row in the 2-norm.

    fp32: sums of a few thousand terms in fp32 give about sqrt(n) 2^-24 of the terms' size, each step of the chain
    (projection, core, scores, softmax, values, core, output) again: below 1e-5 of the row.
    bf16 storage: the tensor-core path rounds the query, the probabilities, z and y to bf16, each off by at most 2^-8 and by
    2^-8 / sqrt(3) = 2.3e-3 in the mean square; the query's rounding reaches the probabilities times the scores' standard
    deviation (about 1 here).  Four independent such roundings: 4.5e-3 in the mean square; 1e-2 leaves a factor of two."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert np.isfinite(got).all(), what
    err = np.linalg.norm(got - ref, axis=-1) / np.linalg.norm(ref, axis=-1)
    assert err.max() <= (1e-2 if dtype == "bf16" else 1e-5), f"{what}: relative row errors up to {err.max():.3e}"


def check_pool(got, before, ref, mask, dtype, what):
    """A pool after a call: rows outside `mask` are untouched bit for bit; rows inside are the 64-bit rows rounded once
    (half a step) after an fp32 sum over d (at most 2^-24 sqrt(d) of the row's scale, 5e-5 with a wide margin for d <= 4096
    and the accumulation order of the tensor cores; 1e-5 for the FMA path) and an fp32 rotation (2^-22 or so)."""
    a, b = np.ascontiguousarray(got).view(np.uint32), np.ascontiguousarray(before).view(np.uint32)
    assert np.array_equal(a[~mask], b[~mask]), f"{what}: rows of nobody were written"
    g, r = got[mask].astype(np.float64), ref[mask]
    assert np.isfinite(g).all(), what
    bound = half_step(dtype) * np.abs(r) + (5e-5 if dtype == "bf16" else 1e-5)
    assert (np.abs(g - r) <= bound).all(), f"{what}: {np.max(np.abs(g - r) - bound):.3e} over the bound"
