"""Paged latent cache held in 8 bits: append, store, read, decode, decode behind a shared prefix, against 64 bits.

Whatever no call may use (slots past a length, pages of nobody, table entries past a sequence's last page) holds NaN codes, any
scale bytes and bad page numbers in every state here."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2603_30033_b200 import binding as Bd
from paper_2603_30033_b200 import workloads as W
from tests import helpers as H
from tests import paged_helpers as P
from tests import q8_helpers as Q

pytestmark = pytest.mark.gpu

SMALL = dict(d_model=64, n_H=4, r=(2, 16, 12), t=(3, 10, 20))
SMALL16 = dict(d_model=64, n_H=4, r=(2, 16, 16), t=(3, 16, 32))
TC64 = dict(d_model=256, n_H=8, r=(4, 64, 64), t=(4, 64, 64))
TC128 = dict(d_model=512, n_H=32, r=(8, 96, 128), t=(8, 32, 128))
TC96 = dict(d_model=192, n_H=6, r=(3, 96, 96), t=(2, 32, 96))
TC_KV = dict(d_model=128, n_H=2, r=(2, 32, 128), t=(1, 64, 64))
TC_VK = dict(d_model=320, n_H=5, r=(5, 32, 64), t=(5, 96, 128))
ODD = dict(d_model=60, n_H=3, r=(2, 7, 6), t=(1, 5, 9))
WIDE = dict(d_model=128, n_H=2, r=(2, 16, 600), t=(2, 16, 300))


def workload(shape, dtype, rope=True, shared=False, seed=91, **kw):
    return H.custom_workload(kind="decode", dtype=dtype, rope=rope, rope_base=500000.0, shared_kv=shared, seed=seed, **{**shape, **kw})


def pytest_generate_tests(metafunc):
    # decode steps run twice: with tables that have room for long contexts, and with tables just large enough, for which small
    # shapes take the one-launch form
    if "room" in metafunc.fixturenames and metafunc.function.__name__.startswith("test_decode"):
        metafunc.parametrize("room", ["wide", "narrow"], indirect=True)


@pytest.fixture(autouse=True)
def room(request, monkeypatch):
    monkeypatch.setattr(P, "ROOM", P.ROOM if getattr(request, "param", "narrow") == "wide" else 0)


def host(t):
    return t.float().cpu().numpy()


def expected_path(st, flags=0):
    """2 (tensor-core kernels) for the bf16 shapes of the bf16 cache's tensor-core step, else 1."""
    w = st.w
    ranks = (w.r[2], w.t[2]) in [(128, 128), (64, 64), (96, 96), (128, 64), (64, 128)] and w.r[1] % 32 == 0 and w.t[1] % 32 == 0
    tc = w.dtype == "bf16" and ranks and w.d_model % 64 == 0 and (st.page in (16, 32, 64) or st.page % 128 == 0)
    return 2 if tc and not flags & Bd.TA_FLAG_FORCE_GENERIC else 1


def step(st, dev=None, append=True, flags=0, prefix_call=None, **kw):
    """(y, pools after the step)"""
    x, dw, pools, table, lens, ptab = dev or st.device()
    w = st.w
    args = dict(n_H=w.n_H, rope=w.rope, rope_base=w.rope_base, append=append, flags=flags, **kw)
    if prefix_call if prefix_call is not None else st.P > 0:
        y = Bd.tucker_attn_decode_prefix_q8(x, *dw, *pools, table, lens, ptab if st.P else None, st.P, **args)
    else:
        y = Bd.tucker_attn_decode_paged_q8(x, *dw, *pools, table, lens, **args)
    assert Bd.last_path() == expected_path(st, flags) or (Bd.last_path() == 3 and not flags)
    assert Bd.last_device_error() == 0
    return y, pools


def slots(st):
    """(pages, rows in them) of the slots that new tokens go to."""
    n = np.array(st.lens)
    return st.table[np.arange(len(n)), n // st.page], n % st.page


def stored_rows(codes, scales, at):
    return Q.decode(Q.bytes_of(codes)[at]) * 2.0 ** (Q.bytes_of(scales)[at].astype(np.float64) - 127)[:, None]


@pytest.mark.parametrize("shape", [SMALL16, TC64, dict(d_model=768, n_H=12, r=(12, 64, 64), t=(12, 64, 64))], ids=str)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_short_contexts_run_in_one_launch(dtype, shape):
    for prefix in (0, 100):
        check_step(Q.Q8State(workload(shape, dtype), [37, 0], 16, P=prefix), what="one launch")
        assert Bd.last_path() == 3 and Bd.last_launch_count() == 1


def check_step(st, flags=0, what="", tol=None, **kw):
    """A step that appends, and one that does not: pools, y against 64 bits on the rows that the cache then holds."""
    y, (K, Ks, V, Vs) = step(st, flags=flags, **kw)
    at = slots(st)
    kn, vn = st.new_rows()
    Q.check_pool(K, Ks, st.Kb, st.Ksb, at, kn, what + " K")
    Q.check_pool(V, Vs, st.Vb, st.Vsb, at, vn, what + " V")
    ref = st.oracle_step(stored_rows(K, Ks, at), stored_rows(V, Vs, at))
    P.check_rows(host(y), ref, st.w.dtype, what + " y")
    y2, (K, Ks, V, Vs) = step(st, flags=flags, append=False, **kw)
    assert torch.equal(y, y2), what + ": y without appending"
    for t, b in ((K, st.Kb), (Ks, st.Ksb), (V, st.Vb), (Vs, st.Vsb)):
        assert np.array_equal(Q.bytes_of(t), b), what + ": pools without appending"


SHAPES = [("fp32", SMALL), ("fp32", ODD), ("fp32", SMALL16), ("bf16", SMALL), ("bf16", TC64), ("bf16", TC128), ("bf16", TC96),
          ("bf16", TC_KV), ("bf16", TC_VK)]


# ---- decode ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1, 48, 7])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64), ("bf16", TC_KV)])
def test_decode_page_sizes(dtype, shape, page):
    check_step(Q.Q8State(workload(shape, dtype), [0, 1, 15, 16, 127, 128, 129, 300, 511], page), what=f"page {page}")


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("dtype,shape", SHAPES)
def test_decode_shapes(dtype, shape, rope, shared):
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    check_step(Q.Q8State(workload(shape, dtype, rope, shared), [0, 5, 700, 131, 64], 16), what=f"{dtype} {shape} rope {rope} shared {shared}")


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("prefix", [1, 16, 129, 1000])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128), ("bf16", TC_VK)])
def test_decode_prefix(dtype, shape, prefix, shared):
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    check_step(Q.Q8State(workload(shape, dtype, shared=shared), [0, 40, 129, 3], 32, P=prefix), what=f"prefix {prefix}")


def test_decode_without_a_prefix_through_the_prefix_call():
    st = Q.Q8State(workload(TC64, "bf16"), [3, 200], 16)
    assert torch.equal(step(st, prefix_call=True)[0], step(st, prefix_call=False)[0])


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128)])
def test_decode_generic_and_other_forms_agree(dtype, shape):
    st = Q.Q8State(workload(shape, dtype), [0, 77, 400], 16, P=50)
    check_step(st, flags=Bd.TA_FLAG_FORCE_GENERIC, what="generic")
    assert Bd.last_path() == 1
    check_step(st, what="chosen")


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC128)])
def test_decode_large_and_growing_scores(dtype, shape):
    """Scores of a standard deviation of about 8, growing along the sequence: the running maximum moves again and again.  An
    output that a few keys decide carries their scores' errors: 8 * 2^-9 of the output per rounded query would be 1.6e-2; the
    queries are carried to 2^-12 or better, which leaves the check's ordinary bound."""
    st = Q.Q8State(workload(shape, dtype), [1500, 3, 260], 32, core_gain=8.0)
    for b, rows in enumerate(st.own_k):
        n = len(rows)
        grown, s = Q.quantise(rows * np.linspace(0.05, 1.0, n)[:, None])
        st.own_k[b] = grown * s[:, None]
        i = np.arange(n)
        st.Kb[st.table[b, i // 32], i % 32] = Q.encode(grown)
        st.Ksb[st.table[b, i // 32], i % 32] = np.log2(s).astype(int) + 127
    check_step(st, what="growing")


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128)])
def test_decode_scales_far_apart(dtype, shape):
    """Value rows of sizes 2^-30 .. 2^30 and rows of zeros, key rows of sizes 2^-20 .. 2^2: the output is the few largest rows'."""
    st = Q.Q8State(workload(shape, dtype), [300, 40, 1], 16)
    rng = np.random.default_rng(8)
    for b in range(3):
        n = st.lens[b]
        i = np.arange(n)
        at = (st.table[b, i // 16], i % 16)
        for name, codes, scales, lo, hi in (("own_k", st.Kb, st.Ksb, -20, 2), ("own_v", st.Vb, st.Vsb, -30, 30)):
            rows = getattr(st, name)[b] * 2.0 ** rng.integers(lo, hi + 1, (n, 1))
            rows[::7] = 0.0
            c, s = Q.quantise(rows)
            getattr(st, name)[b] = c * s[:, None]
            codes[at], scales[at] = Q.encode(c), np.log2(s).astype(int) + 127
    check_step(st, what="scales")


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128)])
def test_decode_rows_that_are_not_finite(dtype, shape):
    """A cached NaN row (scale 255) makes its own sequence's output NaN and no other's."""
    st = Q.Q8State(workload(shape, dtype), [200, 200, 33], 16)
    st.Kb[st.table[1, 3], 5], st.Ksb[st.table[1, 3], 5] = 0x7F, 255
    y, (K, Ks, V, Vs) = step(st)
    at = slots(st)
    ref = st.oracle_step(stored_rows(K, Ks, at), stored_rows(V, Vs, at))
    y = host(y)
    assert np.isnan(y[1]).all()
    P.check_rows(y[[0, 2]], ref[[0, 2]], dtype, "others")
    st.x[2, 0] = np.inf
    y, (K, Ks, V, Vs) = step(st)
    assert np.isnan(host(y)[1:]).all() and np.isfinite(host(y)[0]).all()
    assert Q.bytes_of(Ks)[at][2] == 255 and Q.bytes_of(Vs)[at][2] == 255 and (Q.bytes_of(V)[at][2] == 0x7F).all()


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("fp32", SMALL16), ("bf16", TC64)])
def test_decode_bad_tables_and_lengths(dtype, shape):
    """Rows behind a bad page number count as zeros with weight; nothing is written through one; a bad length is clamped, flagged,
    and appends nothing."""
    st = Q.Q8State(workload(shape, dtype), [50, 20], 16)
    st.table[0, 1] = st.n_pages
    x, dw, pools, table, lens, _ = st.device()
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, *pools, table, lens, n_H=st.w.n_H, rope=True, rope_base=st.w.rope_base)
    assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_PAGE
    st.own_k[0][16:32], st.own_v[0][16:32] = 0.0, 0.0
    at = slots(st)
    P.check_rows(host(y), st.oracle_step(stored_rows(pools[0], pools[1], at), stored_rows(pools[2], pools[3], at)), dtype, "zeros")
    st.table[0, 1], st.table[1, 1] = 0, -1                   # the new token of sequence 1 has no page
    dev = st.device()
    Bd.tucker_attn_decode_paged_q8(x, *dw, *dev[2], dev[3], dev[4], n_H=st.w.n_H, rope=True, rope_base=st.w.rope_base)
    assert Bd.last_device_error() & Bd.TA_DEVERR_BAD_PAGE
    changed = (Q.bytes_of(dev[2][0]) != st.Kb).any(-1)
    assert changed.sum() <= 1 and not changed[np.arange(st.n_pages) != at[0][0]].any()
    for bad in (-1, st.max_pages * 16):
        dev = st.device()
        Bd.tucker_attn_decode_paged_q8(x, *dw, *dev[2], dev[3], torch.tensor([bad, 5], dtype=torch.int32, device="cuda"), n_H=st.w.n_H,
                                       rope=True, rope_base=st.w.rope_base)
        assert Bd.last_device_error() & Bd.TA_DEVERR_BAD_CACHE_LEN
        assert (Q.bytes_of(dev[2][0]) != st.Kb).any(-1).sum() <= 1


# ---- append, store, read ---------------------------------------------------------------------------------------------

def ragged(st, new, pad, lead=0):
    """Token rows: `lead` of nobody, those of the sequences, `pad` of nobody; (T, tok_start, (pages, rows), positions)."""
    start = np.concatenate([[0], np.cumsum(new)]) + lead
    pos = np.concatenate([np.arange(n, n + m) for n, m in zip(st.lens, new)] + [np.zeros(0, int)]).astype(int)
    seq = np.repeat(np.arange(len(new)), new)
    return start[-1] + pad, start, (st.table[seq, pos // st.page], pos % st.page), pos


def i32(a):
    return torch.from_numpy(np.asarray(a, np.int32)).cuda()


APPENDS = [("fp32", SMALL, 16), ("fp32", ODD, 7), ("fp32", WIDE, 16), ("bf16", SMALL, 1), ("bf16", TC64, 16), ("bf16", TC128, 64), ("bf16", TC96, 48),
           ("bf16", TC_KV, 128), ("bf16", TC_VK, 32)]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("new", [[1, 1, 1], [0, 0, 1], [130, 0, 257], [5, 700, 64]], ids=str)
@pytest.mark.parametrize("dtype,shape,page", APPENDS)
def test_append(dtype, shape, page, new, shared):
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    w = workload(shape, dtype, shared=shared)
    st = Q.Q8State(w, [0, 33, 260], page, new=new)
    T, start, at, pos = ragged(st, new, pad=7, lead=2)
    rng = np.random.default_rng(1)
    X = W.round_to_storage(rng.standard_normal((T, w.d_model)), dtype)
    X[:2], X[start[-1]:] = np.nan, np.inf
    _, dw, (K, Ks, V, Vs), table, lens, _ = st.device()
    pos0 = 0 if shared else 11
    Bd.tucker_cache_append_paged_q8(H.to_device(X, dtype), dw[3], dw[7], K, Ks, V, Vs, table, lens, i32(start), rope=True,
                                    rope_base=w.rope_base, pos0=pos0)
    assert Bd.last_device_error() == 0
    x = np.asarray(X[2:start[-1]], np.float64)
    v = x @ np.asarray(st.wt["Ut3"], np.float64)
    k = v if shared else Q.rotate(x @ np.asarray(st.wt["U3"], np.float64), pos + pos0, w.rope_base)
    Q.check_pool(K, Ks, st.Kb, st.Ksb, at, k, "K")
    Q.check_pool(V, Vs, st.Vb, st.Vsb, at, v, "V")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape,page", [(SMALL, 16), (ODD, 7), (WIDE, 16), (TC64, 16), (TC128, 64), (TC96, 48), (TC_VK, 32)])
@pytest.mark.parametrize("shared", [False, True])
def test_store_and_read(dtype, shape, page, shared):
    """Rows of every size, of zeros and with numbers that are not finite: codes and scales bit for bit (the rows are exact inputs);
    read back, exact values, everything else in the buffers left as it was."""
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    w = workload(shape, dtype, shared=shared)
    new = [5, 300, 0, 77]
    st = Q.Q8State(w, [0, 33, 7, 260], page, new=new)
    T, start, at, _ = ragged(st, new, pad=3, lead=2)
    rng = np.random.default_rng(2)
    def rows(r):
        a = rng.standard_normal((T, r)) * 2.0 ** rng.integers(-100, 100, (T, 1))
        a[3] = 0.0
        a[4, 0], a[6, r - 1] = np.inf, np.nan
        a[8] = 448.0                                          # borders of the scale and of the codes
        a[9] = np.nextafter(np.float32(448.0), np.float32(500.0))
        a[10] = rng.integers(0, 120, r) * 4.0
        return W.round_to_storage(a, dtype)
    kr = rows(w.r[2])
    vr = kr if shared else rows(w.t[2])
    _, _, (K, Ks, V, Vs), table, lens, _ = st.device()
    dk = H.to_device(kr, dtype)
    dv = dk if shared else H.to_device(vr, dtype)
    Bd.tucker_cache_store_paged_q8(dk, dv, K, Ks, V, Vs, table, lens, i32(start))
    assert Bd.last_device_error() == 0
    part = slice(2, start[-1])
    expect = {}
    for name, codes, scales, before, sbefore, r in (("K", K, Ks, st.Kb, st.Ksb, kr), ("V", V, Vs, st.Vb, st.Vsb, vr)):
        r = np.asarray(r[part], np.float64)
        ok = np.isfinite(r).all(-1)
        c, s = Q.quantise(np.where(ok[:, None], r, 1.0))
        want, swant = before.copy(), sbefore.copy()
        want[at] = np.where(ok[:, None], Q.encode(c), 0x7F)
        swant[at] = np.where(ok, np.log2(s).astype(int) + 127, 255)
        got = Q.bytes_of(codes)
        same = (got == want) | ((got | want) == 128) & (got & 127 == 0) & (want & 127 == 0)       # a zero's sign is not checked
        assert same.all(), name
        assert np.array_equal(Q.bytes_of(scales), swant), name + " scales"
        expect[name] = np.where(ok[:, None], c * s[:, None], np.nan)
    outs = [torch.full((T, r), 7.0, dtype=dk.dtype, device="cuda") for r in ((w.r[2],) if shared else (w.r[2], w.t[2]))]
    Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, table, lens, i32(start), outs[0], outs[-1])
    assert Bd.last_device_error() == 0
    for o, name in zip(outs, "KV"):
        o = host(o)
        assert (o[:2] == 7).all() and (o[start[-1]:] == 7).all()
        assert np.array_equal(o[part].astype(np.float64), expect[name], equal_nan=True), name


def test_store_and_read_bad_tables_and_lengths():
    st = Q.Q8State(workload(TC64, "bf16"), [10, 20], 16, new=[30, 5])
    T, start, at, _ = ragged(st, [30, 5], pad=0)
    st.table[0, 1] = -3
    _, _, (K, Ks, V, Vs), table, lens, _ = st.device()
    rows = torch.ones(T, 64, dtype=torch.bfloat16, device="cuda")
    Bd.tucker_cache_store_paged_q8(rows, rows, K, Ks, V, Vs, table, lens, i32(start))
    assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_PAGE
    a, b = torch.full_like(rows, 7.0), torch.full_like(rows, 7.0)
    Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, table, lens, i32(start), a, b)
    assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_PAGE
    want = np.ones(T)
    want[6:22] = 0.0                                          # slots 16 .. 31
    assert (host(a) == want[:, None]).all() and (host(b) == want[:, None]).all()
    last = i32([st.max_pages * 16 - 2, -1])                   # two of the rows exist; no sequence starts at -1
    a.fill_(7.0)
    Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, table, last, i32(start), a, b)
    assert Bd.last_device_error() & Bd.TA_DEVERR_BAD_CACHE_LEN
    assert (host(a)[2:] == 7).all() and (host(a)[:2] == 0).all()
    before = Q.bytes_of(K).copy()
    Bd.tucker_cache_store_paged_q8(rows, rows, K, Ks, V, Vs, table, last, i32(start))
    assert Bd.last_device_error() & Bd.TA_DEVERR_BAD_CACHE_LEN and np.array_equal(Q.bytes_of(K), before)


def test_no_tokens():
    st = Q.Q8State(workload(TC64, "bf16"), [10, 20], 16)
    _, dw, pools, table, lens, _ = st.device()
    none = torch.zeros(0, 256, dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    Bd.tucker_cache_append_paged_q8(none, dw[3], dw[7], *pools, table, lens, zero, rope=True)
    Bd.tucker_cache_store_paged_q8(rows, rows, *pools, table, lens, zero)
    Bd.tucker_cache_read_paged_q8(*pools, table, lens, zero, rows, torch.zeros_like(rows))
    assert Bd.last_device_error() == 0 and np.array_equal(Q.bytes_of(pools[0]), st.Kb)


# ---- together --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128)])
def test_prefill_store_steps_and_read(dtype, shape, shared):
    """A prefill's cache stored in 8 bits, a second prompt appended, three steps, everything read back: every step against 64 bits
    on the cache as it then is."""
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    w = workload(shape, dtype, shared=shared)
    B, N, page = 2, 70, 16
    st = Q.Q8State(w, [N, N], page, new=[30, 30])
    x0, dw, pools, table, _, _ = st.device()
    K, Ks, V, Vs = pools
    rng = np.random.default_rng(4)
    X = H.to_device(W.round_to_storage(rng.standard_normal((B, N, w.d_model)), dtype), dtype)
    kc = torch.zeros(B, N, w.r[2], dtype=X.dtype, device="cuda")
    vc = kc if shared else torch.zeros(B, N, w.t[2], dtype=X.dtype, device="cuda")
    Bd.tucker_attn_fwd(X, *dw, n_H=w.n_H, causal=True, rope=True, rope_base=w.rope_base, Kcache=kc, Vcache=vc)
    rows = lambda t: t.view(B * N, -1)
    Bd.tucker_cache_store_paged_q8(rows(kc), rows(vc), K, Ks, V, Vs, table, i32([0, 0]), i32([0, N, 2 * N]))
    more = H.to_device(W.round_to_storage(rng.standard_normal((20, w.d_model)), dtype), dtype)
    lens = np.array([N, N])
    Bd.tucker_cache_append_paged_q8(more, dw[3], dw[7], *pools, table, i32(lens), i32([0, 20, 20]), rope=True, rope_base=w.rope_base)
    lens = lens + [20, 0]
    for i in range(3):
        x = W.round_to_storage(rng.standard_normal((B, w.d_model)), dtype)
        y = Bd.tucker_attn_decode_paged_q8(H.to_device(x, dtype), *dw, *pools, table, i32(lens), n_H=w.n_H, rope=True, rope_base=w.rope_base)
        lens = lens + 1
        start = np.concatenate([[0], np.cumsum(lens)])
        outs = [torch.zeros(start[-1], r, device="cuda") for r in ((w.r[2],) if shared else (w.r[2], w.t[2]))]
        Bd.tucker_cache_read_paged_q8(*pools, table, i32([0, 0]), i32(start), outs[0], outs[-1])
        assert Bd.last_device_error() == 0
        k, v = (o.double().cpu().numpy() for o in (outs[0], outs[-1]))
        st.x, st.lens = x, list(lens - 1)
        st.own_k = [k[start[b]:start[b + 1] - 1] for b in range(B)]
        st.own_v = [v[start[b]:start[b + 1] - 1] for b in range(B)]
        ref = st.oracle_step(k[start[1:] - 1], v[start[1:] - 1])
        P.check_rows(host(y), ref, dtype, f"step {i}")


@pytest.mark.parametrize("prefix", [0, 300])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL16), ("bf16", TC64), ("bf16", TC128)])
def test_captured_calls_replay_on_new_contents(dtype, shape, prefix):
    """Append, store, read and a step in one graph, on another stream, replayed after every buffer has new contents; two graphs
    with workspaces of their own in turn."""
    w = workload(shape, dtype)
    states = [Q.Q8State(w, [20, 150, 5], 16, P=prefix, new=[9, 2, 3], seed=s) for s in (5, 6)]
    rng = np.random.default_rng(9)
    X = [H.to_device(W.round_to_storage(rng.standard_normal((11, w.d_model)), dtype), dtype) for _ in range(2)]
    start = i32([0, 8, 9, 11])

    def buffers(st):
        return [t.clone() for t in [st.device()[0], *st.device()[2], *st.device()[3:]]]

    def calls(b, X, dw, ws, outs):
        x, K, Ks, V, Vs, table, lens, ptab = b
        Bd.tucker_cache_append_paged_q8(X, dw[3], dw[7], K, Ks, V, Vs, table, lens, start, rope=True, rope_base=w.rope_base, workspace=ws)
        Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, table, lens, start, outs[0], outs[1])
        Bd.tucker_cache_store_paged_q8(outs[0], outs[1], K, Ks, V, Vs, table, lens, start)
        Bd.tucker_attn_decode_prefix_q8(x, *dw, K, Ks, V, Vs, table, lens, ptab if prefix else None, prefix, n_H=w.n_H, rope=True,
                                        rope_base=w.rope_base, workspace=ws, out=outs[2])

    dw = states[0].device()[1]
    new_outs = lambda: [torch.zeros(11, w.r[2], dtype=X[0].dtype, device="cuda"), torch.zeros(11, w.t[2], dtype=X[0].dtype, device="cuda"),
                        torch.zeros(3, w.d_model, dtype=X[0].dtype, device="cuda")]
    direct = []
    for st, Xi in zip(states, X):
        b, o = buffers(st), new_outs()
        calls(b, Xi, dw, Bd.alloc_workspace(64 << 20, Xi.device), o)
        direct.append((b, o))
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        b, o, Xb = buffers(states[0]), new_outs(), X[0].clone()
        ws = Bd.alloc_workspace(64 << 20, Xb.device)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls(b, Xb, dw, ws, o)
        graphs.append((g, b, o, Xb, ws))                      # a graph's workspace lives as long as the graph
    for order in ((0, 1), (1, 0)):
        for (g, b, o, Xb, _), i in zip(graphs, order):
            for dst, src in zip(b, buffers(states[i])):
                if dst.numel():
                    dst.view(torch.uint8).copy_(src.view(torch.uint8))
            Xb.copy_(X[i])
        for g, *_ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (g, b, o, Xb, _), i in zip(graphs, order):
            for got, want in zip(b + o, direct[i][0] + direct[i][1]):
                assert not got.numel() or torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    assert Bd.last_device_error() == 0


def test_calls_on_another_stream():
    st = Q.Q8State(workload(TC64, "bf16"), [300, 20], 16)
    want = step(st)[0]
    dev = st.device()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = step(st, dev)[0]
    s.synchronize()
    assert torch.equal(y, want)


def test_binding_refusals():
    st = Q.Q8State(workload(TC64, "bf16"), [10, 20], 16)
    x, dw, (K, Ks, V, Vs), table, lens, _ = st.device()
    kw = dict(n_H=st.w.n_H, rope=True)
    with pytest.raises(TypeError):
        Bd.tucker_attn_decode_paged_q8(x, *dw, K.view(torch.uint8), Ks, V, Vs, table, lens, **kw)
    with pytest.raises(TypeError):
        Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks.view(torch.uint8), V, Vs, table, lens, **kw)
    with pytest.raises(ValueError):
        Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks[:-1], V, Vs, table, lens, **kw)
    with pytest.raises(ValueError):
        Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table[:1], lens, **kw)
    with pytest.raises(ValueError):
        Bd.tucker_attn_decode_paged_q8(x, *dw, K.transpose(0, 1).contiguous().transpose(0, 1), Ks, V, Vs, table, lens, **kw)
    with pytest.raises(ValueError):
        Bd.tucker_attn_decode_prefix_q8(x, *dw, K, Ks, V, Vs, table, lens, None, 5, **kw)
    rows = torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        Bd.tucker_cache_store_paged_q8(rows, rows.float(), K, Ks, V, Vs, table, lens, i32([0, 1, 2]))
    with pytest.raises(Bd.TuckerAttnError):
        Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, table, lens, i32([0, 1, 2]), rows, rows)
    with pytest.raises(ValueError):
        Bd.tucker_cache_store_paged_q8(rows, rows, K, Ks, V, Vs, table, lens, i32([0, 1]))


# ---- many tiles per CTA ----------------------------------------------------------------------------------------------

def big_state(shape, lens, page, P=0, rope=True, shared=False, seed=3, gain=1.0, ramp=None):
    """A state whose pools are made on the device: (x, weights, pools, table, lengths, prefix table), workload."""
    w = workload(shape, "bf16", rope=rope, shared=shared)
    wt = {k: W.round_to_storage(v, "bf16") for k, v in W.make_weights(w, core_gain=gain).items()}
    dw = H.weights_to_device(wt, "bf16")
    if shared:
        dw[7] = dw[3]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-(n + 1) // page) for n in lens]
    pre = -(-P // page)
    n = sum(need) + pre + 1
    order = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(max(need) + 1, -(-32768 // page))), -1, dtype=torch.int32, device="cuda")
    o = 0
    for b, m in enumerate(need):
        table[b, :m] = order[o:o + m]
        o += m
    def pool(r):
        codes = torch.randn(n, page, r, generator=g, device="cuda").mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn)
        scales = (torch.randint(-2, 3, (n, page), generator=g, device="cuda") + 120).to(torch.uint8)
        return codes, scales.view(torch.float8_e8m0fnu)
    K, Ks = pool(w.r[2])
    V, Vs = (K, Ks) if shared else pool(w.t[2])
    if ramp is not None:                             # key sizes grow along every sequence
        for b, m in enumerate(lens):
            i = torch.arange(m, device="cuda")
            e = (ramp[0] + (ramp[1] - ramp[0]) * i.double() / max(m, 1)).round().to(torch.uint8) + 0
            Ks.view(torch.uint8)[table[b, i // page].long(), i % page] = (e + 120).to(torch.uint8)
    x = torch.randn(len(lens), w.d_model, generator=g, device="cuda").bfloat16()
    return (x, dw, (K, Ks, V, Vs), table, i32(lens), order[o:o + pre].contiguous()), w


def reference64(state, w, P, stored_k, stored_v):
    """y in 64 bits on the device; stored_k, stored_v: the new rows as the cache holds them."""
    x, dw, (K, Ks, V, Vs), table, lens, ptab = state
    C, U1, U2, U3, Ct, Ut1, Ut2, Ut3 = (t.double() for t in dw)
    page = K.shape[1]
    G, Gt = torch.einsum("ha,aqc->hqc", U1, C), torch.einsum("ha,ajc->hjc", Ut1, Ct)
    def rows(codes, scales, pages, m):
        i = torch.arange(m, device="cuda")
        pg = pages[i // page].long()
        return codes.view(torch.uint8)[pg, i % page].view(torch.float8_e4m3fn).double() * torch.exp2(scales.view(torch.uint8)[pg, i % page].double() - 127)[:, None]
    def rot(t, pos):
        r = t.shape[-1]
        a = pos.double()[:, None] * w.rope_base ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
        e, o = t[:, 0::2], t[:, 1::2]
        return torch.stack((e * a.cos() - o * a.sin(), e * a.sin() + o * a.cos()), -1).flatten(-2)
    out = []
    for b, m in enumerate(lens.tolist()):
        q = torch.einsum("q,hqc->hc", x[b].double() @ U2, G)
        k = torch.cat((rows(K, Ks, ptab, P), rows(K, Ks, table[b], m), stored_k[b:b + 1]))
        v = torch.cat((rows(V, Vs, ptab, P), rows(V, Vs, table[b], m), stored_v[b:b + 1]))
        if w.rope:
            q = rot(q, torch.full((w.n_H,), P + m, device="cuda"))
            if w.shared_kv:
                k = rot(k, torch.arange(len(k), device="cuda"))
        p = torch.softmax(q @ k.T * (w.d_model / w.n_H) ** -0.5, -1)
        out.append(Ut2 @ torch.einsum("hjc,hc->j", Gt, p @ v))
    return torch.stack(out).cpu().numpy()


LONG = [("one sequence over all CTAs", TC128, [60000], 64),
        ("odd numbers of tiles, ends inside pages", TC64, [20011, 127, 128, 129, 0, 40000, 255, 256, 9999], 16),
        ("many short sequences per CTA", TC96, [(37 * i) % 300 for i in range(1500)], 16),
        ("one tile each, several per CTA", TC_KV, [(11 * i) % 128 for i in range(900)], 128),
        ("two tiles each", TC_VK, [128 + (7 * i) % 100 for i in range(500)], 32),
        ("ragged batch", TC128, [1000 * (i % 13) + 77 * i for i in range(64)], 256),
        ("pages that a step straddles", TC64, [383, 384, 385, 6000, 767, 129, 9001], 384),
        ("one head, pages of 640", dict(d_model=64, n_H=1, r=(1, 32, 96), t=(1, 32, 96)), [641, 639, 1280, 5000, 0], 640)]


@pytest.mark.parametrize("shared", ["two pools", "one pool", "one pool, rotated"])
@pytest.mark.parametrize("what,shape,lens,page", LONG, ids=[c[0] for c in LONG])
def test_many_tiles(what, shape, lens, page, shared):
    rope, shared = shared != "one pool", shared != "two pools"
    if shared:
        shape = {**shape, "t": (shape["t"][0], shape["t"][1], shape["r"][2])}
    state, w = big_state(shape, lens, page, rope=rope, shared=shared)
    x, dw, pools, table, dl, _ = state
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, *pools, table, dl, n_H=w.n_H, rope=w.rope, rope_base=w.rope_base)
    assert Bd.last_path() == 2 and Bd.last_device_error() == 0
    check_against_64(state, w, 0, y, what)


def check_against_64(state, w, P_len, y, what):
    x, dw, pools, table, dl, _ = state
    n, page = dl.cpu().numpy(), pools[0].shape[1]
    at = (table.cpu().numpy()[np.arange(len(n)), n // page], n % page)
    sk, sv = (torch.from_numpy(stored_rows(pools[i], pools[i + 1], at)).cuda() for i in (0, 2))
    P.check_rows(host(y), reference64(state, w, P_len, sk, sv), "bf16", what)


@pytest.mark.parametrize("ramp", [(0, 6), (6, 0)], ids=str)
def test_many_tiles_scores_that_grow_or_fall(ramp):
    """Key sizes that change by 2^6 along 20000 tokens: references move late in a segment, accumulators are rescaled, parts of a
    sequence with maxima far apart are joined."""
    state, w = big_state(TC128, [20000, 777, 20000], 64, gain=0.25, ramp=ramp)
    x, dw, pools, table, dl, _ = state
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, *pools, table, dl, n_H=w.n_H, rope=True, rope_base=w.rope_base)
    assert Bd.last_device_error() == 0
    check_against_64(state, w, 0, y, f"ramp {ramp}")


@pytest.mark.parametrize("nats", [9.5, 11, 12, 13, 14])
def test_one_key_outweighs_thousands_of_equal_ones(nats):
    """Weights e^-9.5 .. e^-14 of the largest, 12000 of them in one segment, and the largest's value row is zeros: all are rounded
    alike, and y is off by as much.  To 2^-28 of the largest each: 0.5% at 14."""
    B, m, page = 150, 12000, 64
    state, w = big_state({**TC128, "n_H": 8}, [m] + [0] * (B - 1), page, rope=False)      # (as many heads as core slices: queries independent)
    x, dw, (K, Ks, V, Vs), table, dl, _ = state
    x[1:] = x[0]                                              # every sequence the same, on the same pages
    table[1:] = table[0]
    dl[1:] = m
    C, U1, U2 = (t.double() for t in dw[:3])
    q = torch.einsum("q,ha,aqc->hc", x[0].double() @ U2, U1, C) * (w.d_model / w.n_H) ** -0.5
    top = q.T @ torch.linalg.solve(q @ q.T, torch.full((w.n_H,), float(nats), device="cuda", dtype=torch.float64))
    g = torch.Generator(device="cuda").manual_seed(5)
    value = torch.randn(V.shape[2], generator=g, device="cuda")
    kb, vb = K.view(torch.uint8), V.view(torch.uint8)
    kb[:] = 0
    vb[:] = value.to(torch.float8_e4m3fn).view(torch.uint8)
    Ks.view(torch.uint8)[:] = 127
    Vs.view(torch.uint8)[:] = 127
    k = torch.frexp(top.abs().amax() / 448).exponent
    first = int(table[0, 0])
    kb[first, 7] = (top * torch.exp2(-k.double())).float().to(torch.float8_e4m3fn).view(torch.uint8)
    Ks.view(torch.uint8)[first, 7] = 127 + k
    vb[first, 7] = 0
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, dl, n_H=w.n_H, rope=False, append=False)
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2
    u3, ut3 = (x[:1].double() @ dw[i].double() for i in (3, 7))
    def stored(t):
        c, sc = Q.quantise(t.cpu().numpy())
        return torch.from_numpy(c * sc[:, None]).cuda()
    one = ((x[:1], dw, (K, Ks, V, Vs), table[:1], dl[:1], state[5]), w)
    P.check_rows(host(y), np.repeat(reference64(*one, 0, stored(u3), stored(ut3)), B, 0), "bf16", f"{nats} nats")


@pytest.mark.parametrize("scale", [-30, -12, 0, 30])
@pytest.mark.parametrize("shared", [False, True])
def test_value_rows_of_zeros_among_small_and_large_ones(scale, shared):
    """Rows of zeros have the scale 1 whatever the others have; some of them get most of the weight (a key that many queries like,
    whose value row is nothing)."""
    state, w = big_state({**TC64, "n_H": 4}, [3000, 500, 129], 64, rope=False, shared=shared)
    x, dw, (K, Ks, V, Vs), table, dl, _ = state
    dw[7] *= 2.0 ** (scale // 5 if shared else scale)           # the new tokens' value rows of the others' size (one pool: dw[3] too)
    if not shared:
        Vs.view(torch.uint8)[:] = 120 + scale
        V.view(torch.uint8)[:, ::5] = 0
        Vs.view(torch.uint8)[:, ::5] = 127
        Ks.view(torch.uint8)[:, 10] += 3
    else:
        Ks.view(torch.uint8)[:] = 120 + scale // 5
        K.view(torch.uint8)[:, ::5] = 0
        Ks.view(torch.uint8)[:, ::5] = 127
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, dl, n_H=w.n_H, rope=False, append=False)
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2
    u3, ut3 = (x.double() @ dw[i].double() for i in (3, 7))
    def stored(t):
        c, sc = Q.quantise(t.cpu().numpy())
        return torch.from_numpy(c * sc[:, None]).cuda()
    ref = reference64(state, w, 0, stored(u3), stored(ut3))
    P.check_rows(host(y), ref, "bf16", f"scale {scale}")


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("rope", [True, False])
def test_long_prefix(shared, rope):
    state, w = big_state(TC128 if not shared else {**TC128, "t": (8, 32, 128)}, [0, 300, 4000, 127] * 4, 64, P=20001, rope=rope, shared=shared)
    x, dw, pools, table, dl, ptab = state
    y = Bd.tucker_attn_decode_prefix_q8(x, *dw, *pools, table, dl, ptab, 20001, n_H=w.n_H, rope=rope, rope_base=w.rope_base)
    assert Bd.last_device_error() == 0
    check_against_64(state, w, 20001, y, "long prefix")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("r3,t3,one_pool", [(128, 128, False), (64, 40, False), (256, 136, False), (96, 96, True)])
def test_store_and_read_many_rows(r3, t3, one_pool, dtype):
    """More rows than the GPU has threads for; sequences that begin and end anywhere."""
    g, page = torch.Generator(device="cuda").manual_seed(r3), 48
    new, lens = [17001, 0, 1, 22222, 31], [100, 7, 47, 0, 48]
    need = [-(-(n + m) // page) for n, m in zip(lens, new)]
    n_pages, T = sum(need) + 3, sum(new)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((5, max(need)), -3, dtype=torch.int32, device="cuda")
    for b in range(5):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    start = [3] + [3 + sum(new[:b + 1]) for b in range(5)]
    def rows_of(r):
        x = torch.randn(T + 10, r, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (T + 10, 1), generator=g, device="cuda").float())
        x[::1001] = 0
        return x.to(dtype)
    pool = lambda r: (torch.randint(0, 255, (n_pages, page, r), generator=g, device="cuda", dtype=torch.uint8),
                      torch.randint(0, 255, (n_pages, page), generator=g, device="cuda", dtype=torch.uint8))
    K, V = pool(r3), pool(t3)
    rk, rv = rows_of(r3), rows_of(t3)
    if one_pool:
        V, rv = K, rk
    before = [t.clone() for t in K + V]
    as8 = lambda c, s: (c.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu))
    Bd.tucker_cache_store_paged_q8(rk, rv, *as8(*K), *as8(*V), table, i32(lens), i32(start))
    assert Bd.last_device_error() == 0
    seq = torch.repeat_interleave(torch.arange(5, device="cuda"), torch.tensor(new, device="cuda"))
    slot = torch.cat([torch.arange(n, n + m, device="cuda") for n, m in zip(lens, new)])
    at = table[seq, slot // page].long() * page + slot % page
    for (codes, scales), rows, c0, s0 in ((K, rk, *before[:2]), (V, rv, *before[2:])):
        want_c, want_s = Q.quantise(rows[3:3 + T].double().cpu().numpy())
        want = c0.view(-1, rows.shape[1]).clone(), s0.view(-1).clone()
        want[0][at] = torch.from_numpy(Q.encode(want_c)).cuda()
        want[1][at] = torch.from_numpy((np.log2(want_s) + 127).astype(np.uint8)).cuda()
        assert torch.equal(scales.view(-1), want[1])
        assert torch.equal(codes.view(-1, rows.shape[1]) & 127, want[0] & 127)                   # (the sign of zero is free)
    out = [torch.full((T + 10, r), 7.0, device="cuda").to(dtype) for r in (r3, t3)]
    Bd.tucker_cache_read_paged_q8(*as8(*K), *as8(*V), table, i32(lens), i32(start), out[0], out[0] if one_pool else out[1])
    assert Bd.last_device_error() == 0
    for (codes, scales), o in ((K, out[0]),) if one_pool else ((K, out[0]), (V, out[1])):
        c = codes.view(-1, o.shape[1])[at].view(torch.float8_e4m3fn).double()
        assert torch.equal(o[3:3 + T].double(), c * torch.exp2(scales.view(-1)[at].double() - 127)[:, None])
        assert (o[:3] == 7).all() and (o[3 + T:] == 7).all()


# ---- long appends ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,r3,t3,T,one_pool", [(64, 128, 128, 19000, False), (64, 96, 128, 19400, False), (64, 256, 256, 9600, False),
                                                (64, 224, 224, 19000, True), (64, 32, 256, 5000, False), (1024, 64, 64, 6000, False),
                                                (4096, 128, 128, 16384, False), (4096, 160, 96, 700, False)])
@pytest.mark.parametrize("rope", [True, False])
def test_append_of_long_prompts(d, r3, t3, T, one_pool, rope):
    """Every division of the work: one CTA for all columns of one or two row tiles, d split over 2, 4 and 8 CTAs, factors apart."""
    g, base, page = torch.Generator(device="cuda"), 500000.0, 64
    g.manual_seed(T + r3)
    lens, new = [70, 0, 5], [T // 3, 1, T - T // 3 - 1]
    need = [-(-(n + m) // page) for n, m in zip(lens, new)]
    n_pages = sum(need) + 2
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((3, max(need)), -3, dtype=torch.int32, device="cuda")
    for b in range(3):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    normal = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
    X, U3 = normal(T + 40, d), normal(d, r3, std=d ** -0.5)
    X[T:] = float("nan")                                     # rows of nobody behind the last sequence
    Ut3 = U3 if one_pool else normal(d, t3, std=d ** -0.5)
    pool = lambda r: (torch.randint(0, 255, (n_pages, page, r), generator=g, device="cuda", dtype=torch.uint8),
                      torch.randint(0, 255, (n_pages, page), generator=g, device="cuda", dtype=torch.uint8))
    K, Ks = pool(r3)
    V, Vs = (K, Ks) if one_pool else pool(t3)
    before = [t.clone() for t in (K, Ks, V, Vs)]
    as8 = lambda c, s: (c.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu))
    start = [0, new[0], new[0] + 1, T]
    Bd.tucker_cache_append_paged_q8(X, U3, Ut3, *as8(K, Ks), *as8(V, Vs), table, i32(lens), i32(start), rope=rope, rope_base=base)
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2
    pos = torch.cat([torch.arange(n, n + m, device="cuda") for n, m in zip(lens, new)])
    seq = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(new, device="cuda"))
    rows = table[seq, pos // page].long() * page + pos % page
    x = X[:T].double()
    v64, k64 = x @ Ut3.double(), x @ U3.double()
    if rope and not one_pool:
        a = pos.double()[:, None] * base ** (-torch.arange(0, r3, 2, device="cuda", dtype=torch.float64) / r3)
        e, o = k64[:, 0::2], k64[:, 1::2]
        k64 = torch.stack((e * a.cos() - o * a.sin(), e * a.sin() + o * a.cos()), -1).flatten(-2)
    for codes, scales, c0, s0, want in ((K, Ks, *before[:2], v64 if one_pool else k64), (V, Vs, *before[2:], v64)):
        codes, scales, c0, s0 = codes.view(-1, codes.shape[-1]), scales.view(-1), c0.view(-1, codes.shape[-1]), s0.view(-1)
        rest = torch.ones(len(s0), dtype=torch.bool, device="cuda")
        rest[rows] = False
        assert torch.equal(codes[rest], c0[rest]) and torch.equal(scales[rest], s0[rest])
        s = torch.exp2(scales[rows].double() - 127)[:, None]
        got = codes[rows].view(torch.float8_e4m3fn).double() * s
        top = want.abs().amax(1, keepdim=True)
        assert (top <= 448 * s * (1 + 5e-5)).all() and ((top >= 224 * s * (1 - 5e-5))).all()
        bound = torch.maximum(Q.U_E4M3 * want.abs(), 2.0 ** -10 * s) + 1e-4 * top        # see check_pool
        assert ((got - want).abs() <= bound).all()


# ---- the bounds-checking build ---------------------------------------------------------------------------------------

CHILD = "TA_BOUNDS_CHECK_CHILD"


@pytest.mark.skipif(os.environ.get(CHILD) == "1", reason="already inside the bounds-checking run")
def test_under_the_bounds_checking_build():
    """Every global index that the kernels form lies in its tensor: the tests that assert a device error word of zero, once more in a
    child process that loads the build which checks."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, TUCKER_ATTN_LIB="checked")
    env[CHILD] = "1"
    sel = "decode_shapes or decode_prefix or page_sizes or many_tiles or long_prefix or append or store or read or one_launch or q8_library"
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-v", "-m", "gpu", "-k", sel, "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       env=env, cwd=root, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert "test_q8_library_checks PASSED" in r.stdout


@pytest.mark.skipif(os.environ.get(CHILD) != "1", reason="runs only inside the bounds-checking run")
def test_q8_library_checks():
    assert Bd.bounds_checked()
