"""The 8-bit cache in numpy, 64 bits: rows to codes and scales and back, and states of paged caches that hold them."""
from __future__ import annotations

import numpy as np

from tests import helpers as H
from tests import paged_helpers as P

U_E4M3 = 2.0 ** -4                   # half a step, relative; 2^-10 absolute below 2^-6 (in units of the scale)


def exponents(v):
    """k of each row: the least integer, at least -96, with max |v| <= 448 2^k; 0 for a row of zeros."""
    a = np.abs(v).max(-1)
    k = np.ceil(np.log2(np.where(a > 0, a, 448.0) / 448.0)).astype(np.int64)
    k = np.where(a > 448.0 * 2.0 ** k.astype(np.float64), k + 1, k)                    # log2 is rounded
    k = np.where(a <= 448.0 * 2.0 ** (k - 1).astype(np.float64), k - 1, k)
    return np.where(a > 0, np.maximum(k, -96), 0)


def nearest(x):
    """e4m3 numbers nearest to x (|x| <= 448), ties to even."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.round(x / step) * step


def quantise(v):
    """(code values, scales) of the rows v."""
    s = 2.0 ** exponents(v).astype(np.float64)
    return nearest(v / s[..., None]), s


def encode(c):
    """Bytes of code values (all of them e4m3 numbers)."""
    a = np.abs(c)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    m = np.where(a < 2.0 ** -6, a * 2.0 ** 9, a / 2.0 ** e * 8 - 8)
    b = np.where(a < 2.0 ** -6, m, (e + 7) * 8 + m).astype(np.uint8)
    return b | np.where(np.signbit(c), np.uint8(128), np.uint8(0))


def decode(b):
    """Values of code bytes."""
    b = np.asarray(b, np.uint8)
    e, m, s = (b >> 3) & 15, b & 7, np.where(b & 128, -1.0, 1.0)
    v = np.where(e == 0, m * 2.0 ** -9, (8.0 + m) * 2.0 ** (e.astype(np.float64) - 10))
    return np.where((b & 127) == 127, np.nan, s * v)


class Q8State(P.PagedState):
    """PagedState whose rows are held in 8 bits.  Whatever no call may use holds NaN codes and any scale byte."""

    def __init__(self, w, lens, page, *, seed=5, row_scale=3.0, **kw):
        super().__init__(w, lens, page, seed=seed, **kw)
        rng = np.random.default_rng(seed + 1000)
        n, r3, t3 = self.n_pages, w.r[2], w.t[2]
        junk = np.array([0x7F, 0xFF, 0x7E, 0xFE, 0x00], np.uint8)
        mk = lambda r: junk[rng.integers(0, 5, (n, page, r))]
        self.Kb, self.Ksb = mk(r3), rng.integers(0, 256, (n, page)).astype(np.uint8)
        self.Vb, self.Vsb = (self.Kb, self.Ksb) if self.shared else (mk(t3), rng.integers(0, 256, (n, page)).astype(np.uint8))
        # rows whose sizes differ by up to 2^row_scale
        size = lambda m: 2.0 ** (row_scale * (rng.random((m, 1)) - 0.5))
        parts = [(self.table[b], "own_k", "own_v", b) for b in range(len(lens))] + [(self.prefix_table, "pre_k", "pre_v", None)]
        for pages, kn, vn, b in parts:
            for name, codes, scales in ((kn, self.Kb, self.Ksb), (vn, self.Vb, self.Vsb)):
                if name == vn and self.shared:
                    continue
                rows = getattr(self, name)[b] if b is not None else getattr(self, name)
                if not len(rows):
                    continue
                c, s = quantise(rows * size(len(rows)))
                i = np.arange(len(rows))
                codes[pages[i // page], i % page] = encode(c)
                scales[pages[i // page], i % page] = np.log2(s).astype(np.int64) + 127
                if b is not None:
                    getattr(self, name)[b] = c * s[:, None]
                else:
                    setattr(self, name, c * s[:, None])
            if self.shared:
                if b is not None:
                    self.own_v[b] = self.own_k[b]
                else:
                    self.pre_v = self.pre_k

    def device(self):
        """Device tensors: x, weights, (K, Ks, V, Vs), table, lengths, prefix table."""
        import torch
        w = self.w
        dw = H.weights_to_device(self.wt, w.dtype)
        if self.shared:
            dw[7] = dw[3]
        K, Ks = pool_to_device(self.Kb, self.Ksb)
        V, Vs = (K, Ks) if self.shared else pool_to_device(self.Vb, self.Vsb)
        i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
        return H.to_device(self.x, w.dtype), dw, (K, Ks, V, Vs), i32(self.table), i32(self.lens), i32(self.prefix_table)

    def new_rows(self):
        """The new tokens' key rows (rotated, except with one pool) and value rows in 64 bits, before they are quantised."""
        x = np.asarray(self.x, np.float64)
        k, v = x @ np.asarray(self.wt["U3"], np.float64), x @ np.asarray(self.wt["Ut3"], np.float64)
        if self.w.rope and not self.shared:
            pos = np.array([self.P + n for n in self.lens])
            k = rotate(k, pos, self.w.rope_base)
        return k, v

    def oracle_step(self, kn, vn):
        """y of one decode step in 64 bits: every key and value as the cache holds it, the new tokens' (kn, vn) too."""
        w = self.w
        f = lambda n: np.asarray(self.wt[n], np.float64)
        x = np.asarray(self.x, np.float64)
        G = np.einsum("ha,aqc->hqc", f("U1"), f("C"))
        Gt = np.einsum("ha,ajc->hjc", f("Ut1"), f("Ct"))
        scale = (w.d_model / w.n_H) ** -0.5
        turned = self.shared and w.rope
        y = []
        for b, n in enumerate(self.lens):
            q = np.einsum("q,hqc->hc", x[b] @ f("U2"), G)
            if w.rope:
                q = rotate(q, np.full(w.n_H, self.P + n), w.rope_base)
            k = np.concatenate([self.pre_k, self.own_k[b], kn[b:b + 1]])
            v = np.concatenate([self.pre_v, self.own_v[b], vn[b:b + 1]])
            if turned:
                k = rotate(k, np.arange(len(k)), w.rope_base)
            s = (q @ k.T) * scale
            p = np.exp(s - s.max(1, keepdims=True))
            o = (p @ v) / p.sum(1, keepdims=True)
            y.append(f("Ut2") @ np.einsum("hjc,hc->j", Gt, o))
        return np.stack(y)


def pool_to_device(codes, scales):
    import torch
    return (torch.from_numpy(codes.copy()).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales.copy()).cuda().view(torch.float8_e8m0fnu))


def rotate(x, pos, base):
    """Rows x [n, r] rotated at positions pos [n] (interleaved pairs)."""
    r = x.shape[-1]
    a = np.asarray(pos, np.float64)[:, None] * float(base) ** (-np.arange(0, r, 2) / r)
    e, o = x[:, 0::2], x[:, 1::2]
    out = np.empty_like(x, dtype=np.float64)
    out[:, 0::2], out[:, 1::2] = e * np.cos(a) - o * np.sin(a), e * np.sin(a) + o * np.cos(a)
    return out


def bytes_of(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def check_pool(pool, scales, before, scales_before, at, rows, what, slack=5e-5):
    """A pool after a call.  `at` = (pages, rows in the page) of the rows written, `rows` = what they are in 64 bits.

    Everything else is untouched bit for bit.  A written row stands for numbers within half a step of the 64-bit ones: 2^-4 of
    the number, or 2^-10 of the scale where it is small; `slack` (of the row's largest number) is the fp32 sum's and rotation's
    own error, as for the bf16 pools, which can move a number past a rounding border, and past a scale's: the step is then that of
    the larger scale."""
    got, gs = bytes_of(pool), bytes_of(scales)
    mask = np.zeros(before.shape[:2], bool)
    mask[at] = True
    assert np.array_equal(got[~mask], before[~mask]) and np.array_equal(gs[~mask], scales_before[~mask]), f"{what}: rows of nobody were written"
    value = decode(got[at]) * 2.0 ** (gs[at].astype(np.float64) - 127)[:, None]
    assert np.isfinite(value).all(), what
    k = exponents(rows * (1 + slack))
    byte = gs[at].astype(np.int64) - 127
    assert ((byte <= k) & (byte >= exponents(rows * (1 - slack)))).all(), f"{what}: scales"
    top = np.abs(rows).max(-1, keepdims=True)
    bound = np.maximum(U_E4M3 * np.abs(rows), 2.0 ** -10 * 2.0 ** k.astype(np.float64)[:, None]) + 2 * slack * top
    over = np.abs(value - rows) - bound
    assert (over <= 0).all(), f"{what}: {over.max():.3e} over the bound"
