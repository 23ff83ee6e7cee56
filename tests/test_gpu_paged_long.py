"""Paged latent cache at lengths where a CTA works on many tiles: long appends, long sequences, long prefixes.  Inputs and
64-bit references live on the GPU (the sizes are too large for the numpy oracle of the other paged tests)."""
import pytest

from paper_2603_30033_b200 import binding as Bd
from tests import paged_helpers as P

pytestmark = pytest.mark.gpu


def generator(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rotate(x, pos, base):
    """Rows x [..., r] (64 bits) rotated by the angles of positions pos [...]."""
    import torch
    r = x.shape[-1]
    a = pos.double()[..., None] * float(base) ** (torch.arange(0, r, 2, device=x.device, dtype=torch.float64) / -r)
    co, si = a.cos(), a.sin()
    xe, xo = x[..., 0::2], x[..., 1::2]
    return torch.stack((xe * co - xo * si, xe * si + xo * co), dim=-1).flatten(-2)


# ---- append ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,r3,t3,T,one_pool", [(64, 128, 128, 19000, False), (64, 96, 128, 19400, False), (64, 256, 256, 9600, False),
                                                (64, 224, 224, 19000, True), (4096, 128, 128, 32768, False)])
@pytest.mark.parametrize("rope", [True, False])
def test_append_of_long_prompts(d, r3, t3, T, one_pool, rope):
    """Prompts so long that a CTA finishes all columns of two row tiles by itself (up to 16 units of 32 columns): every
    row of the pools against 64 bits, and the rows of nobody unchanged."""
    import torch
    g, base, page = generator(T + r3), 500000.0, 64
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
    K = normal(n_pages, page, r3)
    V = K if one_pool else normal(n_pages, page, t3)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    start = [0, new[0], new[0] + 1, T]
    before = [K.clone(), V.clone()]
    lib = Bd.load_library()
    desc = Bd.make_desc(B=3, N=1, d_model=d, n_H=1, r=(1, 1, r3), t=(1, 1, t3), causal=True, rope=rope, rope_base=base, dtype=Bd.TA_DTYPE_BF16)
    cache = Bd.TuckerPagedCache(K.data_ptr(), V.data_ptr(), table.data_ptr(), n_pages, page, max(need))
    # no partial sums: d is not split, one CTA finishes all columns of its rows
    assert lib.tucker_cache_append_paged_workspace_bytes(bytes(desc), bytes(cache), T + 40) == 256
    Bd.tucker_cache_append_paged(X, U3, Ut3, K, V, table, i32(*lens), i32(*start), rope=rope, rope_base=base)
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2
    seq = torch.cat([torch.full((m,), b, device="cuda") for b, m in enumerate(new)])
    pos = torch.cat([torch.arange(n, n + m, device="cuda") for n, m in zip(lens, new)])
    at = table[seq, pos // page].long() * page + pos % page
    k, v = X[:T].double() @ U3.double(), X[:T].double() @ Ut3.double()
    if rope and not one_pool:
        k = rotate(k, pos, base)
    for pool, was, rows in zip((K, V), before, (k, v)):
        flat, old = pool.view(-1, rows.shape[1]), was.view(-1, rows.shape[1])
        # one rounding to bf16 after an fp32 sum over d and a rotation: as paged_helpers.check_pool
        assert ((flat[at].double() - rows).abs() <= P.U_BF16 * rows.abs() + 5e-5).all()
        others = torch.ones(len(flat), dtype=torch.bool, device="cuda")
        others[at] = False
        assert torch.equal(flat[others], old[others])


# ---- waits that run out ------------------------------------------------------------------------------------------------

def test_block_whose_wait_ran_out_stays_until_the_late_bytes_have_come():
    """Between the blocks of a cluster: the wait gives up and is flagged, the block does not end before its peer has sent."""
    assert Bd.last_device_error() == 0
    for budget_us in (500, 5000):
        out = Bd.selftest_cluster_wait(budget_us)
        assert Bd.last_device_error() == Bd.TA_DEVERR_WAIT_TIMEOUT
        assert out.tolist() == [0, 1]
    assert Bd.last_device_error() == 0
    for bad in (0, -1, 100001):
        with pytest.raises(Bd.TuckerAttnError):
            Bd.selftest_cluster_wait(bad)


# ---- steps whose CTAs work on many tiles and several sequences -----------------------------------------------------------

class LongState:
    """A bf16 step of `lens` own slots behind a prefix of P, on the GPU.  Rows grow along a sequence (prefix first) by `growth`,
    so that the running maximum of the scores keeps moving; unused rows and pages hold NaN and infinities, unused table entries
    bad page numbers."""

    def __init__(self, d, h, r, t, lens, page, *, P=0, rope=True, one_pool=False, growth=7.0, seed=1):
        import torch
        g, dev, B = generator(seed), "cuda", len(lens)
        normal = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=dev) * std).bfloat16()
        self.h, self.rope, self.one_pool, self.page, self.P, self.lens, self.base = h, rope, one_pool, page, P, lens, 500000.0
        need, pre = [n // page + 1 for n in lens], -(-P // page)
        n_pages, room = sum(need) + pre + 3, max(max(need) + 1, -(-32768 // page))
        order = torch.randperm(n_pages, generator=g, device=dev).int()
        table = torch.full((B, room), -9, dtype=torch.int32)
        first = 0
        for b, n in enumerate(need):
            table[b, :n] = order[first:first + n].cpu()
            first += n
        table[:, -1] = 1 << 30
        self.table, self.ptab = table.cuda(), order[first:first + pre].contiguous()
        self.len = torch.tensor(lens, dtype=torch.int32, device=dev)
        top = float(P + max(lens) + 1)
        grow = lambda pos: 1.0 + growth * pos.double() / top
        seq = torch.cat([torch.full((n,), b, device=dev) for b, n in enumerate(lens)])
        slot = torch.cat([torch.arange(n, device=dev) for n in lens])
        self.own_rows = self.table[seq, slot // page].long() * page + slot % page
        at = torch.arange(P, device=dev)
        self.pre_rows = self.ptab[at // page].long() * page + at % page if P else at
        junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device=dev).bfloat16()

        def pool(rank):
            m = junk[torch.randint(0, 4, (n_pages * page, rank), generator=g, device=dev)]
            m[self.own_rows] = (torch.randn(len(slot), rank, generator=g, device=dev) * grow(P + slot)[:, None]).bfloat16()
            m[self.pre_rows] = (torch.randn(P, rank, generator=g, device=dev) * grow(at)[:, None]).bfloat16()
            return m.view(n_pages, page, rank)

        self.K = pool(r[2])
        self.V = self.K if one_pool else pool(t[2])
        self.x = normal(B, d)
        C, U1, U2, U3 = normal(*r, std=(d / (r[0] * r[1] * r[2])) ** 0.5), normal(h, r[0], std=h ** -0.5), normal(d, r[1], std=d ** -0.5), normal(d, r[2], std=d ** -0.5)
        Ct, Ut1, Ut2 = normal(*t, std=(t[1] * t[2]) ** -0.25), normal(h, t[0], std=h ** -0.5), normal(d, t[1], std=d ** -0.5)
        self.w = [C, U1, U2, U3, Ct, Ut1, Ut2, U3 if one_pool else normal(d, t[2], std=d ** -0.5)]

    def reference(self):
        """y [B, d] and the new token's rows of K and V as the cache takes them, in 64 bits."""
        import torch
        C, U1, U2, U3, Ct, Ut1, Ut2, Ut3 = [a.double() for a in self.w]
        x, B, P, n = self.x.double(), len(self.lens), self.P, self.len.long()
        turn = (lambda a, pos: rotate(a, pos, self.base)) if self.rope else (lambda a, pos: a)
        late = turn if self.one_pool else (lambda a, pos: a)            # one pool: keys are rotated when they are read
        flat = lambda pool, rows: pool.view(-1, pool.shape[2])[rows].double()
        scale = (x.shape[1] / self.h) ** -0.5
        q = torch.einsum("ha,bac->bhc", U1, torch.einsum("bq,aqc->bac", x @ U2, C)) * scale
        q = turn(q, (P + n)[:, None].expand(B, self.h))
        new_k, new_v = x @ U3, x @ Ut3
        kn = turn(new_k, P + n)
        kp, vp = late(flat(self.K, self.pre_rows), torch.arange(P, device="cuda")), flat(self.V, self.pre_rows)
        o, end = [], 0
        for b, m in enumerate(self.lens):
            rows = self.own_rows[end:end + m]
            end += m
            k = torch.cat((kp, late(flat(self.K, rows), P + torch.arange(m, device="cuda")), kn[b:b + 1]))
            o.append((q[b] @ k.t()).softmax(1) @ torch.cat((vp, flat(self.V, rows), new_v[b:b + 1])))
        z = torch.einsum("ha,ajc,bhc->bj", Ut1, Ct, torch.stack(o))
        return z @ Ut2.t(), new_v if self.one_pool else kn, new_v

    def check(self, what):
        import torch
        before = [self.K.clone(), self.V.clone()]
        y_ref, kn, vn = self.reference()
        kw = dict(n_H=self.h, rope=self.rope, rope_base=self.base)
        y = Bd.tucker_attn_decode_prefix(self.x, *self.w, self.K, self.V, self.table, self.len, self.ptab if self.P else None, self.P, **kw)
        assert Bd.last_device_error() == 0 and Bd.last_path() == 2
        P.check_rows(y.double().cpu().numpy(), y_ref.cpu().numpy(), "bf16", what)
        b = torch.arange(len(self.lens), device="cuda")
        at = self.table[b, self.len.long() // self.page].long() * self.page + self.len.long() % self.page
        for pool, was, rows in zip((self.K, self.V), before, (kn, vn)):
            flat, old = pool.view(-1, pool.shape[2]), was.view(-1, pool.shape[2])
            assert ((flat[at].double() - rows).abs() <= P.U_BF16 * rows.abs() + 5e-5).all(), what
            keep = torch.ones(len(flat), dtype=torch.bool, device="cuda")
            keep[at] = False
            assert torch.equal(flat[keep].view(torch.int16), old[keep].view(torch.int16)), what


RANKS = {"64": ((4, 64, 64), (4, 64, 64)), "96": ((3, 96, 96), (2, 32, 96)), "128": ((8, 96, 128), (8, 32, 128)),
         "128/64": ((2, 32, 128), (1, 64, 64)), "64/128": ((5, 32, 64), (5, 96, 128))}


# The tolerance of paged_helpers.check_rows holds with growing scores too: query and rotated keys are carried to 2^-17 (scores of up
# to 50: 4e-4), cached rows are exact, and P, z and y are rounded whatever the scores.
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("pools", ["two", "one", "one, no rope"])
@pytest.mark.parametrize("ranks", RANKS)
def test_streaming_many_tiles_and_sequences_per_cta(ranks, pools, page):
    """More tiles per CTA than its ring has stages, long and short sequences mixed: stages used again and again, the accumulator
    rescaled, the rotation's base carried from tile to tile, several sequences in one CTA."""
    r, t = RANKS[ranks]
    if pools != "two" and r[2] != t[2]:
        pytest.skip("one pool has one rank")
    lens = [(b * b * 37 + 5 * b) % 4000 for b in range(100)]
    for at, n in ((3, 0), (10, 1), (11, 127), (12, 128), (13, 0), (30, 129), (50, 0), (51, 0), (52, 16)):
        lens[at] = n
    tiles = sum(n // 128 + 1 for n in lens)
    assert tiles > 148 * 7                                             # the deepest ring has six stages
    LongState(256, 8, r, t, lens, page, rope=pools != "one, no rope", one_pool=pools != "two").check(f"{ranks} {pools} {page}")


@pytest.mark.parametrize("pools", ["two", "one"])
@pytest.mark.parametrize("lens", [[100003], [70000, 0, 50001]], ids=str)
def test_streaming_one_sequence_over_many_ctas(lens, pools):
    LongState(128, 32, (4, 64, 128), (4, 64, 128), lens, 64, one_pool=pools == "one").check(f"{lens} {pools}")


@pytest.mark.parametrize("pools", ["two", "one", "one, no rope"])
@pytest.mark.parametrize("ranks", RANKS)
@pytest.mark.parametrize("B,h,prefix,page", [(20, 32, 30001, 64), (41, 16, 29952, 128), (1200, 32, 500, 16)])
def test_prefix_many_units_and_row_blocks_per_cta(B, h, prefix, page, ranks, pools):
    """Several key tiles per CTA (ring and accumulator used again, rescaled), CTAs that end one block of 256 rows and begin the next, a last
    block of 128 rows or fewer, a last key tile that is full or not."""
    r, t = RANKS[ranks]
    if pools != "two" and r[2] != t[2]:
        pytest.skip("one pool has one rank")
    units = -(-B * h // 256) * -(-prefix // 128)
    assert units > 148 * 4                                             # three or six buffers, two a unit
    lens = [(13 * b) % (300 if B < 100 else 3) for b in range(B)]
    LongState(512, h, r, t, lens, page, P=prefix, rope=pools != "one, no rope", one_pool=pools != "two").check(f"{B} {ranks} {pools}")


# ---- long sequences ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("pair", [0, 1, 2, 5])
def test_rotation_late_in_a_long_share_of_one_sequence(pair):
    """One un-rotated pool with latent RoPE, 2^27 keys: every CTA rotates about seven thousand tiles of one sequence.  All rows are
    zero (one page, read again and again) but two, one near the start and one near the end of the first CTA's share, whose rotated keys
    are the same multiple of the query's coordinate pair `pair` up to their rounding to bf16: they share the softmax, at
    scores of S = 2000, so that an error e of the late row's rotation moves the shares by S e.

    Tolerance: a rotated key is carried as two bf16 numbers, off by 2^-18 of its size at most in each coordinate, the angle addition by
    2^-22 or so, and the tile's base by 64 steps of at most 2^-23: S (2 * 2^-18 + 64 * 2^-23 + 2^-22) = 0.031 in the difference of the two
    scores, a quarter of that in a share (p (1 - p)), where the two rows may point in opposite directions: twice that.  With the
    roundings of P, z and y (2^-8 each, the last two relative to the row): 0.016 + 3 * 2^-8 = 0.028.  fp32 sums of products of size S: 2^-23 S = 2.4e-4."""
    import torch
    g, S, L, page, base = generator(pair), 2000.0, 1 << 27, 128, 500000.0
    d, h, r1, r = 128, 2, 2, 64
    normal = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
    x, C, U1, U2, U3 = normal(1, d), normal(r1, 32, r, std=0.2), normal(h, r1), normal(d, 32, std=d ** -0.5), normal(d, r, std=d ** -0.5)
    Ct, Ut1, Ut2 = normal(r1, 32, r, std=0.2), normal(h, r1), normal(d, 32)
    D = lambda t: t.double()
    q = torch.einsum("ha,aqc,q->hc", D(U1), D(C), D(x)[0] @ D(U2)) * (d / h) ** -0.5
    q = rotate(q, torch.full((h,), L, device="cuda"), base)
    v = torch.zeros(r, dtype=torch.float64, device="cuda")
    v[2 * pair:2 * pair + 2] = q[0, 2 * pair:2 * pair + 2]
    v *= S / v.dot(q[0])
    tiles = L // page + 1
    early, late = 2, tiles // 148 - 10
    pool = torch.zeros(3, page, r, device="cuda", dtype=torch.bfloat16)
    table = torch.zeros(1, tiles, dtype=torch.int32, device="cuda")
    table[0, early], table[0, late] = 1, 2
    # of the 128 places in either page the two whose scores are closest, the rows themselves pointing well apart
    at = torch.stack((early * page + torch.arange(page), late * page + torch.arange(page))).cuda()
    cand = rotate(v.expand(2, page, r), -at, base).bfloat16()
    sc = rotate(D(cand), at, base) @ q[0]
    apart = torch.nn.functional.cosine_similarity(D(cand[0])[:, None], D(cand[1])[None], dim=-1) < 0.5
    best = int((sc[0][:, None] - sc[1][None]).abs().masked_fill(~apart, 1e9).argmin())
    slot = torch.tensor([best // page, best % page], device="cuda")
    pos, rows = at[[0, 1], slot], cand[[0, 1], slot]
    pool[1, slot[0]], pool[2, slot[1]] = rows[0], rows[1]
    y = Bd.tucker_attn_decode_paged(x, C, U1, U2, U3, Ct, Ut1, Ut2, U3, pool, pool, table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                                    n_H=h, rope=True, rope_base=base, append=False)
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2
    new = D(x)[0] @ D(U3)
    keys = torch.cat((rotate(D(rows), pos, base), rotate(new[None], torch.tensor([L], device="cuda"), base), torch.zeros(1, r, device="cuda").double()))
    vals = torch.cat((D(rows), new[None], torch.zeros(1, r, device="cuda").double()))
    s = q @ keys.t() + torch.tensor([0, 0, 0, float(L - 2)], device="cuda").double().log().clamp(min=0)
    o = s.softmax(1) @ vals
    assert 0.01 < float(s.softmax(1)[0, 0]) < 0.99                  # both rows matter
    ref = D(Ut2) @ torch.einsum("ha,ajc,hc->j", D(Ut1), D(Ct), o)
    err = float((D(y)[0] - ref).norm() / ref.norm())
    print(f"pair {pair}: share {float(s.softmax(1)[0, 0]):.3f} error {err:.2e}")
    assert err <= 0.028, err


# ---- large scores in the one-launch form --------------------------------------------------------------------------------

@pytest.mark.parametrize("gain", [8.0, 60.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_step_in_one_launch_large_scores_against_the_oracle(dtype, gain, monkeypatch):
    """Scores up to the order of 60 and 500: few keys carry a head, in any tile of any CTA, and running maxima, rescaled sums and the
    join of the CTAs' parts decide the values.

    Tolerance: all arithmetic is fp32 from the stored values on.  The query (sums over 256, 64 and 4 terms, a rotation) and the
    score (64 terms) are off by about sqrt(256) 2^-24 + 2 sqrt(64) 2^-24 = 2e-6 of |q| |k| at most, which counts twice in a quotient
    of exponentials, and the rows of values that share the weight may be twice as long as their mean: 8e-6 |q| |k|.  On top of it what
    small scores leave (1e-5, paged_helpers.check_rows) and, in bf16, the rounding of y: 2^-8 of each element."""
    import numpy as np
    from paper_2603_30033_b200 import workloads as W
    from tests import helpers as H
    monkeypatch.setattr(P, "ROOM", 0)
    w = H.custom_workload(kind="decode", dtype=dtype, rope=True, rope_base=500000.0, seed=91, d_model=256, n_H=4, r=(4, 64, 64), t=(4, 64, 64))
    for lens, pre in (([300, 3, 0], 200), ([1000, 77], 0), ([0, 1], 1100)):
        st = P.PagedState(w, lens, 16, P=pre, core_gain=gain)
        q = np.einsum("ha,bac->bhc", st.wt["U1"], np.einsum("bq,aqc->bac", st.x @ st.wt["U2"], st.wt["C"])) * (256 / 4) ** -0.5
        keys = np.concatenate([st.pre_k, st.x @ st.wt["U3"], *st.own_k])
        size = np.linalg.norm(q, axis=-1).max() * np.linalg.norm(keys, axis=-1).max()
        x, dw, K, V, table, n, ptab = st.device()
        y = Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, n, ptab if pre else None, pre, n_H=4, rope=True, rope_base=w.rope_base)
        assert Bd.last_path() == 3 and Bd.last_device_error() == 0
        got, ref = y.double().cpu().numpy(), st.oracle_step()[0]
        err = np.linalg.norm(got - ref, axis=-1) / np.linalg.norm(ref, axis=-1)
        print(f"{dtype} gain {gain} |q||k| {size:.0f} errors {err}")
        assert (err <= 8e-6 * size + 1e-5 + (P.U_BF16 if dtype == "bf16" else 0.0)).all(), (size, err)


# ---- arguments and uses that the other tests leave out -------------------------------------------------------------------

@pytest.mark.parametrize("room", [0, 32768])
@pytest.mark.parametrize("flags", [0, Bd.TA_FLAG_FORCE_GENERIC])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_explicit_scale(dtype, flags, room, monkeypatch):
    """Four times the default scale gives, bit for bit, what a core of four times the size gives: a power of two passes through
    every rounding unchanged."""
    import torch
    from tests import helpers as H
    monkeypatch.setattr(P, "ROOM", room)
    w = H.custom_workload(kind="decode", dtype=dtype, rope=True, rope_base=500000.0, seed=5, d_model=256, n_H=4, r=(4, 64, 64), t=(4, 64, 64))
    st = P.PagedState(w, [300, 3, 0], 16, P=200, core_gain=0.5)
    x, dw, K, V, table, n, ptab = st.device()
    kw = dict(n_H=4, rope=True, rope_base=w.rope_base, append=False, flags=flags)
    a = Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, n, ptab, 200, scale=4 * (256 / 4) ** -0.5, **kw)
    b = Bd.tucker_attn_decode_prefix(x, dw[0] * 4, *dw[1:], K, V, table, n, ptab, 200, **kw)
    c = Bd.tucker_attn_decode_prefix(x, *dw, K, V, table, n, ptab, 200, **kw)
    assert Bd.last_device_error() == 0 and torch.equal(a, b) and not torch.equal(a, c)


@pytest.mark.parametrize("pools", ["two", "one"])
def test_captured_prefix_step_replays_while_another_graph_runs(pools):
    """Two graphs of the same step on different states, each with its own workspace, replayed on two streams at once: what the calls give
    alone, bit for bit."""
    import torch
    r, t = RANKS["128"]
    sts = [LongState(512, 16, r, t, [90, 0, 1500, 7, 300], 64, P=3001, one_pool=pools == "one", seed=k) for k in (3, 4)]
    step = lambda s, K, V, y: Bd.tucker_attn_decode_prefix(s.x, *s.w, K, V, s.table, s.len, s.ptab, s.P, n_H=s.h, rope=True, rope_base=s.base, out=y)
    alone, graphs, out = [], [], []
    for s in sts:
        K = s.K.clone()
        alone.append((step(s, K, K if s.one_pool else s.V.clone(), torch.empty_like(s.x)), K))
    torch.cuda.synchronize()
    for s in sts:
        g, K, y = torch.cuda.CUDAGraph(), s.K.clone(), torch.empty_like(s.x)
        V = K if s.one_pool else s.V.clone()
        with torch.cuda.graph(g):
            step(s, K, V, y)
        graphs.append(g)
        out.append((y, K))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert Bd.last_device_error() == 0
    for (y0, k0), (y1, k1) in zip(alone, out):
        assert torch.equal(y0, y1) and torch.equal(k0.view(torch.int16), k1.view(torch.int16))
