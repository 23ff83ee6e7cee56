"""8-bit paged cache at the ends of its range: scores of thousands, value rows of zeros among rows of any size, weights far below the
largest.  Against 64 bits on the rows as the cache holds them."""
import numpy as np
import pytest
import torch

from paper_2603_30033_b200 import binding as Bd
from tests import paged_helpers as P
from tests import q8_helpers as Q
from tests.test_gpu_q8 import TC64, TC96, TC128, big_state, host, reference64

pytestmark = pytest.mark.gpu


def stored(rows):
    """Rows (64 bits, on the device) as the cache holds them."""
    c, s = Q.quantise(rows.cpu().numpy())
    return torch.from_numpy(c * s[:, None]).cuda()


def check(state, w, y, what, same=False):
    """y of a step without a prefix and without RoPE; same: all sequences are the first."""
    x, dw, pools, table, lens, ptab = state
    assert Bd.last_device_error() == 0 and Bd.last_path() == 2, what
    n = 1 if same else len(lens)
    one = ((x[:n], dw, pools, table[:n], lens[:n], ptab), w)
    new = [stored(x[:n].double() @ dw[i].double()) for i in (3, 7)]
    ref = reference64(*one, 0, *new)
    P.check_rows(host(y), np.repeat(ref, len(lens), 0) if same else ref, "bf16", what)


def repeated(m, page=64):
    """A state of 150 sequences that are the first one, m cached tokens each: every CTA has several steps, segments begin and end at
    every place.  As many heads as core slices, so that the heads' queries [heads, r3] (64 bits, scaled) are independent."""
    state, w = big_state({**TC128, "n_H": 8}, [m] + [0] * 149, page, rope=False)
    x, dw, _, table, lens, _ = state
    x[1:], table[1:], lens[1:] = x[0].clone(), table[0].clone(), m
    C, U1, U2 = (t.double() for t in dw[:3])
    q = torch.einsum("q,ha,aqc->hc", x[0].double() @ U2, U1, C) * (w.d_model / w.n_H) ** -0.5
    return state, w, q


def towards(q, target):
    """The shortest key that every query gives the score `target`."""
    return q.T @ torch.linalg.solve(q @ q.T, torch.full((len(q),), float(target), device=q.device, dtype=q.dtype))


@pytest.mark.parametrize("nats", [1400, 5700, 11500])
@pytest.mark.parametrize("since", [0, 1000])
def test_scores_with_a_large_common_part(nats, since):
    """All keys from slot `since` on share a part that adds `nats` (to a few percent) to every score, besides scores of a
    standard deviation of 2.  A softmax does not see a common part.

    Tolerance: the common part's codes are the same bytes in every row, and so is what the queries' rounding does to it.  Left is
    fp32: eight roundings (four products of 32 coordinates, three pieces, a multiply-add) of at most 2^-23 of 16600 (11500 nats
    in log2 units) are 0.016 at worst and 0.003 in the mean square, 0.2% of a weight, and independent from key to key; the bound of a step
    with small scores holds as it is."""
    m, split = 3000, 96
    state, w, q = repeated(m)
    x, dw, (K, Ks, V, Vs), table, lens, _ = state
    top = towards(q[:, :split], nats)
    k = int(torch.frexp(top.abs().amax() / 448).exponent)      # the codes' scale: the common part fills their range
    g = torch.Generator(device="cuda").manual_seed(7)
    kb = K.view(torch.uint8)
    code = lambda v: (v * 2.0 ** -k).float().to(torch.float8_e4m3fn).view(torch.uint8)
    kb[:, :, :split] = code(top)
    noise = torch.randn(*K.shape[:2], K.shape[2] - split, generator=g, device="cuda") * (2.0 / q[:, split:].norm(dim=1).mean())
    kb[:, :, split:] = code(noise)
    Ks.view(torch.uint8)[:] = 127 + k
    early = torch.arange(since, device="cuda")
    kb[table[0, early // 64].long(), early % 64, :split] = 0
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, lens, n_H=w.n_H, rope=False, append=False)
    check(state, w, y, f"{nats} nats since {since}", same=True)


@pytest.mark.parametrize("shape", [TC64, {**TC96, "n_H": 8}], ids=["64", "96"])
@pytest.mark.parametrize("cached", [64, 256])
def test_new_value_row_of_zeros_in_a_fresh_tile(shape, cached):
    """The new token's value row is zeros (x = 0) and lies where nothing was requested from the pools, among rows of 2^-30.  The row is
    narrower than a line of the tile, whose rest is the kernel's to fill: a larger step before leaves other bytes there."""
    before, wb = big_state(TC128, [5000] * 40, 64, rope=False)
    state, w = big_state(shape, [cached] * 300, 64, rope=False)
    x, dw, (K, Ks, V, Vs), table, lens, _ = state
    x.zero_()
    Vs.view(torch.uint8)[:] = 90
    for _ in range(3):
        Bd.tucker_attn_decode_paged_q8(before[0], *before[1], *before[2], *before[3:5], n_H=wb.n_H, rope=False, append=False)
        y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, lens, n_H=w.n_H, rope=False, append=False)
        check(state, w, y, f"{cached} cached")


@pytest.mark.parametrize("scale", [-89, -60, 12, 30, 60, 100])
@pytest.mark.parametrize("run", [0, 700])
def test_value_rows_of_zeros_among_rows_of_any_size(scale, run):
    """Every fifth value row, and the first `run` of a sequence, are zeros (whose scale is 1 whatever the others' is); some of them have
    keys that get most of the weight.  A row of zeros adds nothing to the output and its weight to the sum.  Whole steps of nothing but
    such rows are joined with others."""
    state, w = big_state({**TC64, "n_H": 4}, [3000, 700, 129], 64, rope=False)
    x, dw, (K, Ks, V, Vs), table, lens, _ = state
    dw[7] *= 2.0 ** scale                                       # the new tokens' value rows of the others' size
    vb, vs = V.view(torch.uint8), Vs.view(torch.uint8)
    vs[:] = 120 + scale
    vb[:, ::5] = 0
    vs[:, ::5] = 127
    Ks.view(torch.uint8)[:, 10] += 3
    i = torch.arange(run, device="cuda")
    for b in (0, 1):
        at = (table[b, i // 64].long(), i % 64)
        vb[at], vs[at] = 0, 127
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, lens, n_H=w.n_H, rope=False, append=False)
    check(state, w, y, f"scale {scale}")


@pytest.mark.parametrize("nats", [9.5, 11, 12, 13, 14])
def test_weights_far_below_the_largest_keep_their_bits(nats):
    """12000 equal weights e^-9.5 .. e^-14 of the largest in one segment: all are rounded alike, and y is off by as much.  The largest's
    value row has one number, in a coordinate that the output core ignores, and the same scale as the others'.

    Tolerance: weights are held to 2^-27 of the largest, which is 0.9% of e^-14 at worst and a third of that in the mean square of
    where the weight falls; the other roundings as in every step."""
    state, w, q = repeated(12000)
    x, dw, (K, Ks, V, Vs), table, lens, _ = state
    ignored = 5
    dw[4][:, :, ignored] = 0
    top = towards(q, nats)
    g = torch.Generator(device="cuda").manual_seed(5)
    kb, vb = K.view(torch.uint8), V.view(torch.uint8)
    kb[:] = 0
    vb[:] = torch.randn(V.shape[2], generator=g, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    Ks.view(torch.uint8)[:] = 127
    Vs.view(torch.uint8)[:] = 127
    k = int(torch.frexp(top.abs().amax() / 448).exponent)
    first = int(table[0, 0])
    kb[first, 7] = (top * 2.0 ** -k).float().to(torch.float8_e4m3fn).view(torch.uint8)
    Ks.view(torch.uint8)[first, 7] = 127 + k
    vb[first, 7] = 0
    vb[first, 7, ignored] = 0x7E
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, lens, n_H=w.n_H, rope=False, append=False)
    check(state, w, y, f"{nats} nats", same=True)


def test_value_rows_of_sizes_far_apart():
    """Scales 2^90 apart in one sequence, at random: the large rows are the output, all rows are the sum."""
    state, w = big_state({**TC64, "n_H": 4}, [3000, 700, 129], 64, rope=False)
    x, dw, (K, Ks, V, Vs), table, lens, _ = state
    g = torch.Generator(device="cuda").manual_seed(9)
    small = torch.rand(Vs.shape, generator=g, device="cuda") < 0.5
    Vs.view(torch.uint8)[:] = torch.where(small, 70, 160).to(torch.uint8)
    y = Bd.tucker_attn_decode_paged_q8(x, *dw, K, Ks, V, Vs, table, lens, n_H=w.n_H, rope=False, append=False)
    check(state, w, y, "2^90")
