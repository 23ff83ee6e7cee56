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
