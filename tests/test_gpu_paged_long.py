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
