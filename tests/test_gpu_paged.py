"""Paged latent cache: append, decode, decode behind a shared prefix, against the 64-bit oracle.

Whatever no call may use (slots past a length, pages of nobody, table entries past a sequence's last page) holds NaN,
infinities, the type's largest values or bad page numbers in every state here."""
import numpy as np
import pytest

from paper_2603_30033_b200 import binding as Bd
from paper_2603_30033_b200 import workloads as W
from tests import helpers as H
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu

SMALL = dict(d_model=64, n_H=4, r=(2, 16, 12), t=(3, 10, 20))
TC64 = dict(d_model=256, n_H=8, r=(4, 64, 64), t=(4, 64, 64))
TC128 = dict(d_model=512, n_H=32, r=(8, 96, 128), t=(8, 32, 128))
TC96 = dict(d_model=192, n_H=6, r=(3, 96, 96), t=(2, 32, 96))
TC_KV = dict(d_model=128, n_H=2, r=(2, 32, 128), t=(1, 64, 64))
TC_VK = dict(d_model=320, n_H=5, r=(5, 32, 64), t=(5, 96, 128))
ODD = dict(d_model=60, n_H=3, r=(2, 7, 6), t=(1, 5, 9))


def host(t):
    return t.float().cpu().numpy()


def workload(shape, dtype, rope=True, shared=False, seed=91, **kw):
    return H.custom_workload(kind="decode", dtype=dtype, rope=rope, rope_base=500000.0, shared_kv=shared, seed=seed, **{**shape, **kw})


def pytest_generate_tests(metafunc):
    # decode steps run twice: with tables that have room for long contexts, and with tables just large enough, for which small
    # shapes take the one-launch form
    if "room" in metafunc.fixturenames and not metafunc.function.__name__.startswith(("test_append", "test_far_positions", "test_step_in_one_launch", "test_paged_calls_under")):
        metafunc.parametrize("room", ["wide", "narrow"], indirect=True)


@pytest.fixture(autouse=True)
def room(request, monkeypatch):
    monkeypatch.setattr(P, "ROOM", P.ROOM if getattr(request, "param", "narrow") == "wide" else 0)


def expected_path(st, flags=0):
    """2 (tensor-core kernels) for the bf16 shapes of the contiguous tensor-core decode step with pages of 16, 32, 64 or a
    multiple of 128 rows, else 1."""
    w = st.w
    ranks = (w.r[2], w.t[2]) in [(128, 128), (64, 64), (96, 96), (128, 64), (64, 128)] and w.r[1] % 32 == 0 and w.t[1] % 32 == 0
    tc = w.dtype == "bf16" and ranks and w.d_model % 64 == 0 and (st.page in (16, 32, 64) or st.page % 128 == 0)
    return 2 if tc and not flags & Bd.TA_FLAG_FORCE_GENERIC else 1


def run_step(st, append=True, flags=0, prefix_call=None, **kw):
    x, dw, K, V, table, lens, ptab = st.device()
    w = st.w
    args = dict(n_H=w.n_H, rope=w.rope, rope_base=w.rope_base, append=append, flags=flags, **kw)
    if prefix_call if prefix_call is not None else st.P > 0:
        y = Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, lens, ptab if st.P else None, st.P, **args)
    else:
        y = Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, **args)
    expected = expected_path(st, flags)
    assert Bd.last_path() == expected or (Bd.last_path() == 3 and not flags and (P.ROOM == 0 or expected == 1))
    assert Bd.last_device_error() == 0
    return y, K, V


def check_step(st, append=True, flags=0, what="", **kw):
    k0 = host(st.device()[2]) if not st.shared else host(H.to_device(st.K, st.w.dtype))
    v0 = k0 if st.shared else host(H.to_device(st.V, st.w.dtype))
    y, K, V = run_step(st, append, flags, **kw)
    ref, kn, vn = st.oracle_step()
    P.check_rows(host(y), ref, st.w.dtype, what + " y")
    rows = lambda new: [(b, n, new[b]) for b, n in enumerate(st.lens)] if append else []
    for name, pool, before, new in (("K", K, k0, vn if st.shared else kn), ("V", V, v0, vn)):
        want, mask = st.expect_pool(before.astype(np.float64), rows(new), 0)
        P.check_pool(host(pool), before, want, mask, st.w.dtype, f"{what} {name}")


STEP_SHAPES = [("fp32", SMALL), ("fp32", ODD), ("bf16", SMALL), ("bf16", TC64), ("bf16", TC128), ("bf16", TC96),
               ("bf16", TC_KV), ("bf16", TC_VK)]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1, 48, 7])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64), ("bf16", TC_KV)])
def test_decode_paged_page_sizes(dtype, shape, page):
    st = P.PagedState(workload(shape, dtype), [0, 1, 15, 16, 127, 128, 129, 300, 511], page)
    check_step(st, what=f"page {page}")


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("dtype,shape", STEP_SHAPES)
def test_decode_paged_shapes(dtype, shape, rope, append):
    st = P.PagedState(workload(shape, dtype, rope=rope), [37, 0, 1, 255, 256, 700], 32, new=1 if append else 0)
    check_step(st, append=append, what=f"{shape}")


@pytest.mark.parametrize("dtype,shape", [("fp32", dict(d_model=96, n_H=24, r=(24, 16, 8), t=(24, 40, 500))),
                                         ("bf16", dict(d_model=128, n_H=32, r=(32, 160, 64), t=(32, 224, 128))),
                                         ("bf16", dict(d_model=256, n_H=2, r=(2, 256, 128), t=(2, 256, 128)))])
def test_large_core_ranks(dtype, shape):
    """Head and output ranks at the limits of the shared-memory tables (and, fp32, past them)."""
    for pre in (0, 70):
        check_step(P.PagedState(workload(shape, dtype), [20, 0, 150], 16, P=pre), what=f"{shape}")


@pytest.mark.parametrize("B,n", [(1, 0), (1, 1), (1, 2500), (200, 3), (3, 1023)])
def test_decode_paged_batches(B, n):
    st = P.PagedState(workload(TC64, "bf16"), [max(0, n - 7 * (b % 5)) for b in range(B)], 16)
    check_step(st, what=f"B {B} n {n}")


@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("dtype,shape", [("fp32", dict(SMALL, t=(3, 10, 12))), ("bf16", TC64), ("bf16", TC96),
                                         ("bf16", dict(TC128, t=(8, 32, 128)))])
def test_decode_paged_shared_latent_pool(dtype, shape, rope):
    st = P.PagedState(workload(shape, dtype, rope=rope, shared=True), [0, 1, 16, 127, 130, 413], 16)
    check_step(st, what=f"shared {shape}")


@pytest.mark.parametrize("prefix", [1, 15, 16, 127, 128, 129, 255, 500, 1000])
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64), ("bf16", TC128)])
def test_prefix_lengths(dtype, shape, prefix):
    st = P.PagedState(workload(shape, dtype), [0, 1, 40, 129, 17], 16, P=prefix)
    check_step(st, what=f"prefix {prefix}")


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 5])
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("dtype,shape", STEP_SHAPES)
def test_prefix_shapes(dtype, shape, append, page):
    st = P.PagedState(workload(shape, dtype), [0, 33, 200], page, P=301, new=1 if append else 0)
    check_step(st, append=append, what=f"prefix {shape}")


@pytest.mark.parametrize("dtype,shape", STEP_SHAPES)
def test_prefix_without_rope(dtype, shape):
    st = P.PagedState(workload(shape, dtype, rope=False), [3, 0, 90, 17], 64, P=520)
    check_step(st, what=f"prefix, no rope {shape}")


@pytest.mark.parametrize("B,n_H", [(1, 1), (1, 32), (2, 2), (9, 8), (40, 16), (130, 4)])
def test_prefix_batches(B, n_H):
    shape = dict(TC64, n_H=n_H, r=(min(4, n_H), 64, 64), t=(min(4, n_H), 64, 64))
    st = P.PagedState(workload(shape, "bf16"), [(13 * b) % 50 for b in range(B)], 32, P=777)
    check_step(st, what=f"B {B} n_H {n_H}")


@pytest.mark.parametrize("dtype,shape", [("fp32", dict(SMALL, t=(3, 10, 12))), ("bf16", TC64), ("bf16", TC96)])
@pytest.mark.parametrize("rope", [True, False])
def test_prefix_shared_latent_pool(dtype, shape, rope):
    st = P.PagedState(workload(shape, dtype, rope=rope, shared=True), [0, 21, 140], 16, P=205)
    check_step(st, what=f"prefix shared {shape}")


def test_prefix_of_length_zero_is_the_paged_step():
    import torch
    st = P.PagedState(workload(TC64, "bf16"), [5, 0, 300], 32)
    a, b = run_step(st, prefix_call=False), run_step(st, prefix_call=True)
    assert all(torch.equal(p.view(torch.int16), q.view(torch.int16)) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_scores(dtype):
    """Scores of a standard deviation of about 20, growing along the sequence: nearly one key per head remains."""
    shape = SMALL if dtype == "fp32" else TC64
    for pre in (0, 400):
        st = P.PagedState(workload(shape, dtype), [600, 3, 131], 16, P=pre, core_gain=1.0)
        ramp = lambda a, n0: W.round_to_storage(a * (1.0 + 20.0 * (n0 + np.arange(len(a)))[:, None] / 1100.0), dtype)
        st.own_k = [ramp(a, pre) for a in st.own_k]
        st.pre_k = ramp(st.pre_k, 0)
        for b in range(len(st.lens)):
            st.scatter(st.K, st.table[b], st.own_k[b])
        st.scatter(st.K, st.prefix_table, st.pre_k)
        y, _, _ = run_step(st)
        ref, _, _ = st.oracle_step()
        err = np.linalg.norm(host(y) - ref, axis=-1) / np.linalg.norm(ref, axis=-1)
        # the query's rounding (2^-8 / sqrt(3) of each product's size in the mean square) reaches the scores times their standard
        # deviation, here about 8 for the larger keys: 2.3e-3 * 8, and the largest of a few rows three times that
        assert err.max() <= (6e-2 if dtype == "bf16" else 1e-4), err


def test_far_positions():
    """Angles of positions near 2^31: the rotation must not lose them (64-bit angles); a long prefix is only claimed, not
    stored: its slots are read through a one-page table, so prefix_len stays small and pos0 of the append carries the offset."""
    w = workload(TC64, "bf16")
    st = P.PagedState(w, [3, 0], 16, new=[5, 2])
    pos0 = 2 ** 31 - 1 - 8192
    check_append(st, [5, 2], pos0=pos0)


# ---- append ----------------------------------------------------------------------------------------------------------

def check_append(st, new, pad=0, front=0, pos0=0, flags=0, seed=3):
    """Appends new[b] tokens to sequence b; `front` / `pad` rows of nobody before and behind."""
    import torch
    from oracle import tucker_oracle as O
    w, B = st.w, len(st.lens)
    rng = np.random.default_rng(seed)
    T = front + sum(new) + pad
    X = W.round_to_storage(rng.standard_normal((T, w.d_model)), w.dtype)
    start = front + np.concatenate(([0], np.cumsum(new)))
    Xd = H.to_device(X, w.dtype)
    if T:
        Xd[:front] = float("nan")
        Xd[front + sum(new):] = float("inf")
    x, dw, K, V, table, lens, _ = st.device()
    k0, v0 = host(K), host(V)
    Bd.tucker_cache_append_paged(Xd, dw[3], dw[7], K, V, table, lens, torch.from_numpy(start.astype(np.int32)).cuda(),
                                 rope=w.rope, rope_base=w.rope_base, pos0=pos0, flags=flags)
    tc = w.dtype == "bf16" and w.d_model % 64 == 0 and all(32 <= r <= 256 and r % 32 == 0 for r in (w.r[2], w.t[2]))
    assert Bd.last_path() == (2 if tc else 1)
    assert Bd.last_device_error() == 0
    kr, vr = [], []
    for b in range(B):
        xb = X[start[b]:start[b + 1]]
        k, v = xb @ st.wt["U3"], xb @ st.wt["Ut3"]
        if w.rope and not st.shared:
            k = O.rope_rotate(k, pos0 + st.lens[b] + np.arange(new[b]), w.rope_base)
        kr += [(b, st.lens[b] + i, k[i]) for i in range(new[b])]
        vr += [(b, st.lens[b] + i, v[i]) for i in range(new[b])]
    for name, pool, before, rows in (("K", K, k0, vr if st.shared else kr), ("V", V, v0, vr)):
        want, mask = st.expect_pool(before.astype(np.float64), rows, 0)
        P.check_pool(host(pool), before, want, mask, w.dtype, f"append {name} {new}")


@pytest.mark.parametrize("r3,t3", [(32, 32), (32, 256), (160, 64), (256, 256), (96, 224)])
@pytest.mark.parametrize("rope", [True, False])
def test_append_rank_widths(r3, t3, rope):
    new = [70, 1, 140]
    shape = dict(d_model=640, n_H=4, r=(2, 32, r3), t=(2, 32, t3))
    check_append(P.PagedState(workload(shape, "bf16", rope=rope), [3, 0, 90], 16, new=new), new, pad=9)


APPENDS = [[1], [0, 1], [3, 0, 0, 7], [1] * 9, [127], [128], [129], [40, 0, 300, 1], [0, 0, 2]]


@pytest.mark.parametrize("new", APPENDS, ids=str)
@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("fp32", ODD), ("bf16", ODD), ("bf16", TC64), ("bf16", TC128),
                                         ("bf16", TC96), ("bf16", TC_VK)])
def test_append(dtype, shape, new):
    lens = [(31 * b + 5) % 70 for b in range(len(new))]
    check_append(P.PagedState(workload(shape, dtype), lens, 16, new=new), new, pad=3)


@pytest.mark.parametrize("page", [1, 7, 16, 32, 64, 128, 384])
@pytest.mark.parametrize("rope", [True, False])
def test_append_page_sizes(page, rope):
    new = [150, 1, 0, 33]
    check_append(P.PagedState(workload(TC64, "bf16", rope=rope), [0, 15, 16, 100], page, new=new), new, front=2, pad=130)


@pytest.mark.parametrize("dtype,shape", [("fp32", dict(SMALL, t=(3, 10, 12))), ("bf16", TC64)])
@pytest.mark.parametrize("rope", [True, False])
def test_append_shared_latent_pool(dtype, shape, rope):
    new = [9, 64, 1]
    check_append(P.PagedState(workload(shape, dtype, rope=rope, shared=True), [0, 7, 30], 16, new=new), new, pad=1)


@pytest.mark.parametrize("d_model,total", [(64, 700), (1024, 5000), (4096, 1500), (4096, 16)])
def test_append_many_tokens(d_model, total):
    B = 7
    new = [total // B + (b % 3) - 1 for b in range(B)]
    shape = dict(TC128, d_model=d_model)
    check_append(P.PagedState(workload(shape, "bf16"), [11 * b for b in range(B)], 64, new=new), new, pad=5, pos0=1000)


def test_append_of_nothing():
    check_append(P.PagedState(workload(TC64, "bf16"), [4, 0], 16), [0, 0])
    check_append(P.PagedState(workload(TC64, "bf16"), [4, 0], 16), [0, 0], pad=4)


# ---- what a call must refuse or flag -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64)])
def test_bad_pages_are_flagged_and_nothing_is_written_through_them(dtype, shape):
    import torch
    for where, bad in (("own", -1), ("own", 1 << 30), ("new", -5), ("prefix", 1 << 20)):
        st = P.PagedState(workload(shape, dtype), [40, 16], 16, P=33)
        if where == "own":
            st.table[0, 1] = bad
        elif where == "new":
            st.table[1, 1] = bad                        # the page of sequence 1's new token
        else:
            st.prefix_table[1] = bad
        x, dw, K, V, table, lens, ptab = st.device()
        k0 = K.clone()
        y = Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, lens, ptab, st.P, n_H=st.w.n_H, rope=True, rope_base=st.w.rope_base)
        assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_PAGE, where
        assert torch.isfinite(y.float()).all()
        changed = (K != k0).any(-1) & ~(torch.isnan(K).any(-1) & torch.isnan(k0).any(-1))
        assert int(changed.sum()) <= 2


def test_bad_lengths_are_flagged():
    import torch
    st = P.PagedState(workload(TC64, "bf16"), [5, 20], 16)
    x, dw, K, V, table, lens, _ = st.device()
    table[:] = torch.arange(table.numel(), device="cuda", dtype=torch.int32).view(table.shape) % st.n_pages
    K.zero_(), V.zero_()
    for bad in (-3, table.shape[1] * 16):
        lens[1] = bad
        y = Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, n_H=st.w.n_H, rope=True)
        assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_CACHE_LEN and torch.isfinite(y.float()).all()
        X = torch.ones(4, st.w.d_model, device="cuda", dtype=torch.bfloat16)
        K.zero_()
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, V, table, lens, torch.tensor([0, 0, 4], dtype=torch.int32, device="cuda"), rope=True)
        assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_CACHE_LEN and not K.any()


def test_append_past_the_table_drops_only_the_tokens_concerned():
    import torch
    w = workload(TC64, "bf16")
    K = torch.zeros(4, 16, 64, device="cuda", dtype=torch.bfloat16)
    V = torch.zeros_like(K)
    table = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda")
    dw = H.weights_to_device({k: W.round_to_storage(v, w.dtype) for k, v in W.make_weights(w).items()}, w.dtype)
    X = torch.randn(20, w.d_model, device="cuda").bfloat16()
    Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, V, table, torch.tensor([20], dtype=torch.int32, device="cuda"),
                                 torch.tensor([0, 20], dtype=torch.int32, device="cuda"), rope=True)
    assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_CACHE_LEN          # slots 32 .. 39 do not exist
    used = K.ne(0).any(-1)
    assert used[0, 4:].all() and int(used.sum()) == 12


def test_binding_refuses():
    import torch
    st = P.PagedState(workload(TC64, "bf16"), [5, 20], 16, P=40)
    x, dw, K, V, table, lens, ptab = st.device()
    kw = dict(n_H=st.w.n_H, rope=True)
    ok = lambda **o: {**dict(K=K, V=V, table=table, lens=lens, ptab=ptab, n=40), **o}
    for o, exc in [(ok(K=K[:, ::2]), ValueError), (ok(V=V[:-1].contiguous()), ValueError), (ok(table=table.long()), TypeError),
                   (ok(table=table[:, ::2]), ValueError), (ok(lens=lens[:1]), ValueError), (ok(ptab=ptab[:2]), ValueError),
                   (ok(ptab=None), ValueError), (ok(n=-1), ValueError), (ok(K=K.float(), V=V.float()), TypeError),
                   (ok(V=K), Bd.TuckerAttnError), (ok(table=table.cpu()), ValueError)]:
        with pytest.raises(exc):
            Bd.tucker_attn_decode_prefix(x, *dw, o["K"], o["V"], o["table"], o["lens"], o["ptab"], o["n"], **kw)
    with pytest.raises(ValueError):
        Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, workspace=torch.empty(1 << 20, dtype=torch.uint8), **kw)
    small = dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"), **kw)
    if P.ROOM:
        with pytest.raises(Bd.TuckerAttnError) as e:
            Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, **small)
        assert e.value.status == -3
    else:                                                     # one launch, no workspace: the tensor is not looked at
        small["workspace"][:] = 7
        Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, **small)
        assert Bd.last_path() == 3 and small["workspace"].eq(7).all()
    k0 = K.clone()
    for bad in (ok(lens=lens.float()), ok(ptab=ptab[None])):
        with pytest.raises((TypeError, ValueError)):
            Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, bad["lens"], bad["ptab"], 40, **kw)
    assert torch.equal(k0.view(torch.int16), K.view(torch.int16))
    X = torch.zeros(3, st.w.d_model, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(Bd.TuckerAttnError):                   # one pool, two projections
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, K, table, lens, torch.zeros(3, dtype=torch.int32, device="cuda"), rope=True)
    with pytest.raises(ValueError):
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, V, table, lens, torch.zeros(2, dtype=torch.int32, device="cuda"), rope=True)
    with pytest.raises(Bd.TuckerAttnError):
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, V, table, lens, torch.zeros(3, dtype=torch.int32, device="cuda"), rope=True, pos0=-1)
    assert Bd.last_device_error() == 0


def test_pages_past_32_bit_offsets():
    """Pages whose rows lie past 2^32 bytes and past 2^31 elements of the pool: the same rows, and the same results bit for bit, as
    in a small pool.  One pool serves keys and values (half the memory); both ways of appending, both attention kernels."""
    import torch
    shape = dict(d_model=256, n_H=8, r=(4, 64, 128), t=(4, 64, 128))
    w = workload(shape, "bf16", rope=False, shared=True)
    st = P.PagedState(w, [300, 0, 129], 128, P=260, new=5)
    x, dw, K, _, table, lens, ptab = st.device()
    big_pages = 2 ** 31 // (128 * 128) + 64
    free, _ = torch.cuda.mem_get_info()
    if free < 3 * big_pages * 128 * 128 * 2:
        pytest.skip("needs 13 GB of device memory")
    big = torch.empty(big_pages, 128, 128, device="cuda", dtype=torch.bfloat16)
    shift = big_pages - st.n_pages
    big[shift:] = K
    X = torch.randn(6, 256, device="cuda").bfloat16()
    start = torch.tensor([0, 4, 4, 6], dtype=torch.int32, device="cuda")
    up = lambda t: torch.where((t >= 0) & (t < st.n_pages), t + shift, t).int()
    out = []
    for pool, tb, pt in ((K, table, ptab), (big, up(table), up(ptab))):
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], pool, pool, tb, lens, start, rope=False)
        n = lens + torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
        out.append(Bd.tucker_attn_decode_prefix(x, *dw, pool, pool, tb, n, pt, 260, n_H=8, rope=False))
        out.append(Bd.tucker_attn_decode_paged(x, *dw, pool, pool, tb, n, n_H=8, rope=False, flags=Bd.TA_FLAG_FORCE_GENERIC))
        assert Bd.last_device_error() == 0
    bits = lambda t: t.view(torch.int16)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    assert torch.equal(bits(big[shift:]), bits(K))


def test_bad_length_appends_nothing():
    import torch
    for dtype, shape in (("fp32", SMALL), ("bf16", TC64)):
        st = P.PagedState(workload(shape, dtype), [5, 20], 16)
        x, dw, K, V, table, lens, _ = st.device()
        lens[1] = -1
        K0, V0 = K.clone(), V.clone()
        Bd.tucker_attn_decode_paged(x, *dw, K, V, table, lens, n_H=st.w.n_H, rope=True)
        assert Bd.last_device_error() == Bd.TA_DEVERR_BAD_CACHE_LEN
        pg = int(table[1, 0])
        bits = torch.int16 if dtype == "bf16" else torch.int32
        assert torch.equal(K[pg].view(bits), K0[pg].view(bits)) and torch.equal(V[pg].view(bits), V0[pg].view(bits))


def test_flagged_generic_path_agrees():
    """TA_FLAG_FORCE_GENERIC runs bf16 on the FMA kernels: within the roundings of the tensor-core path of it."""
    st = P.PagedState(workload(TC128, "bf16"), [700, 0, 33], 16, P=150)
    a, Ka, Va = run_step(st)
    b, Kb, Vb = run_step(st, flags=Bd.TA_FLAG_FORCE_GENERIC)
    P.check_rows(host(a), host(b).astype(np.float64), "bf16", "generic against tensor-core")


# ---- together --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64)])
def test_prefix_prompts_and_steps_together(dtype, shape):
    """A shared prompt appended once, the sequences' own prompts appended behind it, then decode steps that append: every
    step's output is the last row of the causal forward over the whole sequence."""
    import torch
    from oracle import tucker_oracle as O
    w = workload(shape, dtype)
    P0, own, steps, page = 37, [0, 5, 33, 1], 4, 16
    B = len(own)
    st = P.PagedState(w, [0] * B, page, P=P0, new=[n + steps for n in own])
    rng = np.random.default_rng(17)
    rnd = lambda *s: W.round_to_storage(rng.standard_normal(s), dtype)
    Xp, Xo, Xs = rnd(P0, w.d_model), [rnd(n, w.d_model) for n in own], rnd(steps, B, w.d_model)
    _, dw, K, V, table, lens, ptab = st.device()
    K.fill_(float("nan")), V.fill_(float("nan"))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    kw = dict(rope=True, rope_base=w.rope_base)
    Bd.tucker_cache_append_paged(H.to_device(Xp, dtype), dw[3], dw[7], K, V, ptab[None], i32(0), i32(0, P0), **kw)
    Bd.tucker_cache_append_paged(H.to_device(np.concatenate(Xo), dtype), dw[3], dw[7], K, V, table, lens,
                                 i32(*np.concatenate(([0], np.cumsum(own))).tolist()), pos0=P0, **kw)
    lens += i32(*own)
    for s in range(steps):
        y = Bd.tucker_attn_decode_prefix(H.to_device(Xs[s], dtype), *dw, K, V, table, lens, ptab, P0, n_H=w.n_H, **kw)
        lens += 1
        assert Bd.last_device_error() == 0
        for b in range(B):
            full = np.concatenate([Xp, Xo[b], Xs[:s + 1, b]])
            ref = O.tucker_attn_fwd(full, *[st.wt[k] for k in H.WEIGHT_KEYS], causal=True, rope=True, rope_base=w.rope_base,
                                    rows=[len(full) - 1])[0]
            err = np.linalg.norm(host(y)[b] - ref) / np.linalg.norm(ref)
            # as check_rows, and the cached rows are rounded too: two more roundings of 2.3e-3 in the mean square
            assert err <= (1.5e-2 if dtype == "bf16" else 1e-5), (s, b, err)


def test_append_then_contiguous_prefill_agree():
    """The rows an append writes are those the prefill forward writes to its contiguous caches (up to one rounding step)."""
    import torch
    w = workload(TC64, "bf16")
    N = 150
    st = P.PagedState(w, [0, 0], 32, new=N)
    X = torch.randn(2, N, w.d_model, device="cuda").bfloat16()
    _, dw, K, V, table, lens, _ = st.device()
    Kc = torch.zeros(2, N, 64, device="cuda", dtype=torch.bfloat16)
    Vc = torch.zeros_like(Kc)
    Bd.tucker_attn_fwd(X, *dw, n_H=w.n_H, causal=True, rope=True, rope_base=w.rope_base, Kcache=Kc, Vcache=Vc)
    Bd.tucker_cache_append_paged(X.view(2 * N, -1), dw[3], dw[7], K, V, table, lens,
                                 torch.tensor([0, N, 2 * N], dtype=torch.int32, device="cuda"), rope=True, rope_base=w.rope_base)
    assert Bd.last_device_error() == 0
    slot = torch.arange(N, device="cuda")
    for pool, cache in ((K, Kc), (V, Vc)):
        rows = pool[table[:, slot // 32].long(), slot % 32].float()
        # both round the same sums, formed in another order: at most one step of bf16 apart, or tiny
        assert ((rows - cache.float()).abs() <= 2 * P.U_BF16 * cache.float().abs() + 1e-4).all()


@pytest.mark.parametrize("dtype,shape", [("fp32", SMALL), ("bf16", TC64)])
def test_captured_calls_replay_on_new_contents(dtype, shape):
    import torch
    st = P.PagedState(workload(shape, dtype), [40, 7, 300], 16, P=200, new=3)
    x, dw, K, V, table, lens, ptab = st.device()
    w = st.w
    kw = dict(rope=True, rope_base=w.rope_base)
    X = x.clone()
    start = torch.arange(4, dtype=torch.int32, device="cuda")

    def both(K, V, lens, y):
        Bd.tucker_cache_append_paged(X, dw[3], dw[7], K, V, table, lens, start, pos0=200, **kw)
        return Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, lens + 1, ptab, 200, n_H=w.n_H, out=y, **kw)

    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    K0, V0 = K.clone(), V.clone()
    both(K0, V0, lens, y0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    Kg, Vg, lg = K.clone(), V.clone(), lens.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        both(Kg, Vg, lg, y1)
    for turn in range(3):
        Kg.copy_(K), Vg.copy_(V), lg.copy_(lens)
        if turn:
            x.copy_(torch.randn_like(x)), X.copy_(torch.randn_like(X)), lg.sub_(2 * turn)
            lg.clamp_(min=0)
        K0.copy_(K), V0.copy_(V)
        both(K0, V0, lg, y0)
        graph.replay()
        torch.cuda.synchronize()
        assert Bd.last_device_error() == 0
        assert torch.equal(y0, y1)
        bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
        assert torch.equal(bits(Kg), bits(K0)) and torch.equal(bits(Vg), bits(V0))


def test_two_streams_at_once():
    """Two steps on two streams, each with its own workspace and pools, give what they give alone, bit for bit."""
    import torch
    sts = [P.PagedState(workload(TC64, "bf16"), [900, 31, 400, 2], 16, P=513, seed=s) for s in (1, 2)]
    devs = [s.device() for s in sts]
    pools = [(d[2].clone(), d[3].clone()) for d in devs]
    call = lambda d, K, V: Bd.tucker_attn_decode_prefix(d[0], *d[1], K, V, d[4], d[5], d[6], 513, n_H=8, rope=True)
    alone = [call(d, d[2], d[3]).clone() for d in devs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, d, (K, V) in zip(streams, devs, pools):
            with torch.cuda.stream(s):
                got.append(call(d, K, V))
        torch.cuda.synchronize()
        assert Bd.last_device_error() == 0
        for a, g in zip(alone, got):
            assert torch.equal(a, g)


# ---- the one-launch form ------------------------------------------------------------------------------------------------

ONE_LAUNCH = [dict(d_model=64, n_H=1, r=(1, 8, 8), t=(1, 8, 8)), dict(d_model=72, n_H=3, r=(2, 24, 40), t=(5, 40, 24)),
              dict(d_model=200, n_H=5, r=(7, 64, 128), t=(3, 256, 8)), dict(d_model=512, n_H=32, r=(8, 96, 128), t=(8, 32, 128)),
              dict(d_model=1088, n_H=17, r=(17, 256, 64), t=(16, 56, 96)), dict(d_model=768, n_H=12, r=(12, 64, 64), t=(12, 64, 64))]


@pytest.mark.parametrize("prefix", [0, 1, 77, 700])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", ONE_LAUNCH, ids=lambda s: f"d{s['d_model']}h{s['n_H']}")
def test_step_in_one_launch(shape, dtype, prefix, monkeypatch):
    """Head counts, ranks and d at the edges of what the one-launch form takes; no keys at all, fewer keys than CTAs, full and
    partial tiles, pages that end inside a tile."""
    monkeypatch.setattr(P, "ROOM", 0)
    for page, lens in ((7, [0, 1, 5, 8, 63]), (16, [513, 64, 0]), (128, [129])):
        st = P.PagedState(workload(shape, dtype), lens, page, P=prefix)
        check_step(st, what=f"{shape} page {page} prefix {prefix}")
        if Bd.last_path() != 3:      # 32 heads over 700 keys and more: the tensor cores are faster
            assert dtype == "bf16" and shape["n_H"] == 32 and prefix == 700 and Bd.last_path() == 2
        else:
            assert Bd.last_launch_count() == 1


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_step_in_one_launch_of_one_pool(dtype, monkeypatch):
    """One un-rotated pool: without rope the one-launch form reads it once for keys and values; with rope it does not apply."""
    monkeypatch.setattr(P, "ROOM", 0)
    shape = dict(d_model=768, n_H=12, r=(12, 64, 64), t=(12, 64, 64))
    for rope, path in ((False, 3), (True, 2 if dtype == "bf16" else 1)):
        check_step(P.PagedState(workload(shape, dtype, rope=rope, shared=True), [130, 0, 7], 16, P=90), what=f"rope {rope}")
        assert Bd.last_path() == path


def test_step_in_one_launch_takes_no_workspace(monkeypatch):
    """The C entry points: NULL for the workspace where the query says so, refused where it does not."""
    import ctypes
    lib = Bd.load_library()
    ask = lib.tucker_attn_decode_prefix_workspace_bytes
    w = workload(TC64, "bf16")
    for rooms, none in ((0, True), (32768, False)):
        monkeypatch.setattr(P, "ROOM", rooms)
        st = P.PagedState(w, [5, 20], 16, P=40)
        x, dw, K, V, table, lens, ptab = st.device()
        desc = Bd.make_desc(B=2, N=1, d_model=w.d_model, n_H=w.n_H, r=w.r, t=w.t, causal=True, rope=True, rope_base=w.rope_base)
        cache = Bd.TuckerPagedCache(K.data_ptr(), V.data_ptr(), table.data_ptr(), st.n_pages, st.page, st.max_pages)
        d, c = bytes(desc), bytes(cache)
        assert (ask(d, c, 40) == Bd.TA_WORKSPACE_NONE) == none
        y = __import__("torch").empty_like(x)
        rc = lib.tucker_attn_decode_prefix(d, x.data_ptr(), *[t.data_ptr() for t in dw], c, lens.data_ptr(), ptab.data_ptr(), 40, 1,
                                           y.data_ptr(), None, 0, 0)
        assert rc == (0 if none else -1)
    assert Bd.last_device_error() == 0


def test_step_in_one_launch_more_sequences_than_clusters(monkeypatch):
    """Clusters of a second wave."""
    monkeypatch.setattr(P, "ROOM", 0)
    shape = dict(d_model=128, n_H=4, r=(2, 16, 16), t=(2, 16, 16))
    check_step(P.PagedState(workload(shape, "fp32"), [(37 * b) % 300 for b in range(40)], 16), what="40 sequences")
    assert Bd.last_path() in (1, 3)
    check_step(P.PagedState(workload(shape, "fp32"), [(37 * b) % 30 for b in range(17)], 16), what="17 sequences")
    assert Bd.last_path() == 3


def test_step_in_one_launch_extreme_scores(monkeypatch):
    """Scores of the order of +-500: the maximum is taken before any exponential, across tiles and CTAs."""
    monkeypatch.setattr(P, "ROOM", 0)
    import torch
    for dtype in ("fp32", "bf16"):
        w = workload(dict(d_model=256, n_H=4, r=(4, 64, 64), t=(4, 64, 64)), dtype)
        st = P.PagedState(w, [300, 3, 0], 16, P=200, core_gain=60.0)
        y, _, _ = run_step(st)
        assert Bd.last_path() == 3 and torch.isfinite(y.float()).all()


# ---- bounds-checking build ---------------------------------------------------------------------------------------------------

@pytest.mark.skipif(__import__("os").environ.get("TA_BOUNDS_CHECK_CHILD") == "1", reason="already inside a bounds-checking run")
def test_paged_calls_under_the_bounds_checking_build():
    """The paged tests once more in a child process that loads the library built with -DTA_BOUNDS_CHECK: every global index that the
    kernels form for a store, or for a load from the workspace, is compared with its tensor's extent; each test asserts a clean
    error word."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, TUCKER_ATTN_LIB="checked", TA_BOUNDS_CHECK_CHILD="1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "-k",
                        "one_launch or page_sizes or paged_shapes or prefix_lengths or prefix_batches or append or shared_latent_pool or together",
                        os.path.abspath(__file__)], env=env, cwd=root, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
