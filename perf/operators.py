"""Measured cases of the serving operators over a paged latent KV cache.

  append   tokens appended to the paged cache: latent keys and values projected from X, keys rotated by latent RoPE
           on the way, rows scattered to the pages of their sequences
  decode   one decode step of a layer for a batch whose latent caches are paged
  prefix   one decode step for a batch whose sequences share a long prefix that is stored, and attended to, once

`run` computes each in its plain form (elementary torch operations in 32 bits), or, with `own` set, through the
framework's entry points.  `exact` is the operators' definition in 64 bits, written apart from the plain form.

Paged cache: pools K [n_pages, page, r3] and V [n_pages, page, t3]; the row of slot i of sequence b is row i % page
of page block_table[b, i // page].  Entries past a sequence's last page, and slots past its length, hold anything.
With `shared` one pool of latent rows serves keys and values; together with RoPE it holds un-rotated rows.
"""
import math

import torch

own = False


# ---- cases -----------------------------------------------------------------------------------------------------------

def _case(op, name=None, **kw):
    c = dict(op=op, dtype="bf16", B=1, d=4096, heads=32, r1=8, r2=128, r3=128, t1=8, t2=128, t3=128, page=64, rope=True,
             base=500000.0, shared=False, ragged=True)
    c.update(kw)
    if name is not None:
        c = {"name": name, **c}
    return c


_SMALL = dict(d=768, heads=12, r1=12, r2=64, r3=64, t1=12, t2=64, t3=64, base=10000.0)


def listed():
    return [
        # --- append: L = cached tokens of the longest sequence before the call, new = most new tokens of a sequence
        # every sequence of a serving batch brings one token
        _case("append", "append_one_each", B=64, L=4000, new=1, pad=0),
        # a batch of prompts of mixed lengths, the small model's shape, small pages, rows of padding behind the last one
        _case("append", "append_prompts", B=8, L=0, new=1024, pad=37, page=16, **_SMALL),
        # two long prompts: the largest call
        _case("append", "append_long_prompts", B=2, L=0, new=8192, pad=0, page=128, ragged=False),
        # single precision, a few prompts that continue cached ones
        _case("append", "append_fp32", B=3, L=200, new=150, pad=5, page=16, dtype="fp32", **_SMALL),
        # --- decode: L = cached tokens of the longest sequence
        # one user, a few tokens in: latency
        _case("decode", "decode_first_tokens", B=1, L=37, page=16, **_SMALL),
        # a medium batch of one shared latent cache (keys rotated when read), odd rank
        _case("decode", "decode_shared_rope", B=24, L=3001, page=32, d=768, heads=12, r1=4, r2=96, r3=96, t1=4, t2=96, t3=96,
              shared=True),
        # the long-context serving batch, every sequence of another length
        _case("decode", "decode_long_batch", B=64, L=32768, page=64),
        # single precision
        _case("decode", "decode_fp32", B=4, L=1500, page=16, dtype="fp32", **_SMALL),
        # --- prefix: P = tokens of the shared prefix, L = own cached tokens of the longest sequence
        # a few samples of one prompt, small model
        _case("prefix", "prefix_samples", B=6, P=999, L=100, page=16, **_SMALL),
        # a system prompt in front of a medium batch
        _case("prefix", "prefix_system_prompt", B=32, P=4097, L=700, page=64),
        # a long document that a large batch asks about: the largest call
        _case("prefix", "prefix_document", B=64, P=32768, L=1024, page=128),
        # single precision
        _case("prefix", "prefix_fp32", B=4, P=801, L=60, page=16, dtype="fp32", **_SMALL),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "decode", "prefix"])
    fp32 = rng.random() < 0.2
    d, heads = rng.choice([(768, 12)] if fp32 else [(768, 12), (1024, 8), (2048, 16), (4096, 32)])
    rank = rng.choice([64] if fp32 else [64, 96, 128])
    kw = dict(d=d, heads=heads, r1=rng.choice([4, 8]), r2=rank, r3=rank, t1=rng.choice([4, 8]), t2=rank, t3=rank,
              page=rng.choice([16, 32, 64, 128]), rope=rng.random() < 0.8, base=rng.choice([10000.0, 500000.0]),
              ragged=rng.random() < 0.8, dtype="fp32" if fp32 else "bf16")
    if not fp32 and rank != 96 and rng.random() < 0.25:
        kw["t3"] = kw["t2"] = 192 - rank                     # value rank other than the key rank
    if op == "append":
        B = _log(rng, 1, 4 if fp32 else 64)
        most = 150 if fp32 else 16384 // B
        return _case(op, B=B, new=_log(rng, 1, most), L=rng.randrange(0, 5000), pad=rng.choice([0, 0, 3, 50]), **kw)
    if op == "decode":
        B = _log(rng, 1, 4 if fp32 else 64)
        shared = not fp32 and kw["t3"] == kw["r3"] and rng.random() < 0.25
        return _case(op, B=B, L=_log(rng, 1, 1500 if fp32 else 16384), shared=shared, **kw)
    B = _log(rng, 1, 4 if fp32 else 64)
    return _case(op, B=B, P=_log(rng, 1, 801 if fp32 else 32768), L=_log(rng, 1, 60 if fp32 else 1024), **kw)


def _spread(most, B, ragged):
    """Lengths of B sequences, the longest `most`; ragged: spread over a quarter of it to all of it, in no order."""
    if not ragged or B == 1:
        return [most] * B
    return [most - (most * 3 // 4) * ((5 * b + 3) % B) // B if b else most for b in range(B)]


def _sizes(c):
    """Per sequence: cached tokens before the call, new tokens."""
    lens = _spread(c["L"], c["B"], c["ragged"])
    new = _spread(c["new"], c["B"], c["ragged"]) if c["op"] == "append" else [1] * c["B"]
    return lens, [max(1, n) for n in new]


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 13)
    dt = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    lens, new = _sizes(c)
    B, page, d = c["B"], c["page"], c["d"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dt)

    s = dict(c)
    # pages: every sequence owns those of its slots, the prefix its own, in no order; a few belong to nobody
    need = [(lens[b] + new[b] + page - 1) // page for b in range(B)]
    pre = (c.get("P", 0) + page - 1) // page
    n_pages = sum(need) + pre + 3
    max_pages = max(need) + 1
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    # entry (b, j) of the table is page number (pages of the sequences before b) + j of that order
    first = torch.tensor([sum(need[:b]) for b in range(B)], device=dev)[:, None]
    cols = torch.arange(max_pages, device=dev)[None, :]
    have = torch.tensor(need, device=dev)[:, None]
    table = torch.where(cols < have, order[(first + cols).clamp(max=n_pages - 1)], torch.full((), -1, device=dev, dtype=torch.int32))
    s["table"] = table.contiguous()
    if c["op"] == "prefix":
        s["prefix_table"] = order[sum(need):sum(need) + pre].contiguous()
    s["K"] = normal(n_pages, page, c["r3"])
    s["V"] = s["K"] if c["shared"] else normal(n_pages, page, c["t3"])
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["max_len"] = max(lens)
    # factors with columns of length one; cores that give scores of standard deviation 2
    s["U3"] = normal(d, c["r3"], std=d ** -0.5)
    s["Ut3"] = s["U3"] if c["shared"] else normal(d, c["t3"], std=d ** -0.5)
    if c["op"] == "append":
        tokens = sum(new)
        s["tokens"] = tokens
        s["X"] = normal(tokens + c["pad"], d)
        s["start"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
        return s
    h = c["heads"]
    s["x"] = normal(B, d)
    s["C"] = normal(c["r1"], c["r2"], c["r3"], std=2.0 * (d / (c["r1"] * c["r2"] * c["r3"])) ** 0.5)
    s["U1"] = normal(h, c["r1"], std=h ** -0.5)
    s["U2"] = normal(d, c["r2"], std=d ** -0.5)
    s["Ct"] = normal(c["t1"], c["t2"], c["t3"], std=(c["t2"] * c["t3"]) ** -0.25)
    s["Ut1"] = normal(h, c["t1"], std=h ** -0.5)
    s["Ut2"] = normal(d, c["t2"], std=d ** -0.5)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _rotate(x, pos, base):
    """Rows x [..., r] (float) rotated by the angles of positions pos [...]: pairs (2 i, 2 i + 1), base^(-2 i / r)."""
    r = x.shape[-1]
    theta = float(base) ** (torch.arange(0, r, 2, device=x.device, dtype=torch.float64) / -r)
    a = pos.double()[..., None] * theta
    co, si = a.cos().float(), a.sin().float()
    xe, xo = x[..., 0::2], x[..., 1::2]
    return torch.stack((xe * co - xo * si, xe * si + xo * co), dim=-1).flatten(-2)


def _slots(s, seq, pos):
    """Row numbers, in a pool seen as [n_pages * page, rank], of slots `pos` of sequences `seq`."""
    return s["table"][seq, pos // s["page"]].long() * s["page"] + pos % s["page"]


def _put(pool, rows, values):
    pool.view(-1, pool.shape[-1])[rows] = values.to(pool.dtype)


def _plain_append(s):
    n = s["tokens"]
    X = s["X"][:n].float()
    row = torch.arange(n, device=X.device)
    seq = torch.searchsorted(s["start"][1:], row.int(), right=True)
    pos = s["len"][seq].long() + row - s["start"][seq].long()
    at = _slots(s, seq, pos)
    k = X @ s["U3"].float()
    if s["rope"]:
        k = _rotate(k, pos, s["base"])
    _put(s["K"], at, k)
    _put(s["V"], at, X @ s["Ut3"].float())
    return {"K": s["K"], "V": s["V"]}


def _plain_step(s):
    B, h, L, P = s["B"], s["heads"], s["max_len"], s.get("P", 0)
    x, n = s["x"].float(), s["len"].long()
    k_new, v_new = x @ s["U3"].float(), x @ s["Ut3"].float()
    l_new = v_new
    q = torch.einsum("ha,bac->bhc", s["U1"].float(), torch.einsum("bq,aqc->bac", x @ s["U2"].float(), s["C"].float()))
    if s["rope"]:
        k_new, q = _rotate(k_new, P + n, s["base"]), _rotate(q, (P + n)[:, None].expand(B, h), s["base"])
    # the cached rows of every sequence, up to the longest; what lies past a sequence's end is masked
    pos = torch.arange(L, device=x.device)
    at = (s["table"].clamp(min=0)[:, pos // s["page"]].long() * s["page"] + pos % s["page"])
    there = pos[None, :] < n[:, None]
    rows = s["K"].view(-1, s["r3"])[at].float()
    v = rows if s["shared"] else s["V"].view(-1, s["t3"])[at].float()
    k = _rotate(rows, pos[None, :].expand(B, L), s["base"]) if s["shared"] and s["rope"] else rows
    v = torch.where(there[:, :, None], v, 0.0)
    score = (q @ k.transpose(1, 2)).masked_fill(~there[:, None, :], -math.inf)
    score = torch.cat((score, (q * k_new[:, None, :]).sum(-1, keepdim=True)), dim=2)
    if P:
        at = s["prefix_table"].long()
        kp = s["K"][at].view(-1, s["r3"])[:P].float()
        vp = s["V"][at].view(-1, s["t3"])[:P].float()
        score = torch.cat((score, (q.view(B * h, -1) @ kp.t()).view(B, h, P)), dim=2)
    score = score * (s["d"] / h) ** -0.5
    p = (score - score.amax(dim=2, keepdim=True)).exp()
    p = p / p.sum(dim=2, keepdim=True)
    o = p[:, :, :L] @ v + p[:, :, L:L + 1] * v_new[:, None, :]
    if P:
        o = o + (p[:, :, L + 1:].reshape(B * h, P) @ vp).view(B, h, -1)
    z = torch.einsum("bac,ajc->bj", torch.einsum("ha,bhc->bac", s["Ut1"].float(), o), s["Ct"].float())
    y = z @ s["Ut2"].float().t()
    at = _slots(s, torch.arange(B, device=x.device), n)
    if s["shared"]:
        _put(s["K"], at, l_new)
    else:
        _put(s["K"], at, k_new)
        _put(s["V"], at, v_new)
    return {"y": y.to(s["x"].dtype), "K": s["K"], "V": s["V"]}


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _own(s):
    from paper_2603_30033_b200 import binding
    if s["op"] == "append":
        binding.tucker_cache_append_paged(s["X"], s["U3"], s["Ut3"], s["K"], s["V"], s["table"], s["len"], s["start"],
                                          rope=s["rope"], rope_base=s["base"])
        return {"K": s["K"], "V": s["V"]}
    weights = [s[k] for k in ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")]
    kw = dict(n_H=s["heads"], rope=s["rope"], rope_base=s["base"], append=True)
    if s["op"] == "decode":
        y = binding.tucker_attn_decode_paged(s["x"], *weights, s["K"], s["V"], s["table"], s["len"], **kw)
    else:
        y = binding.tucker_attn_decode_prefix(s["x"], *weights, s["K"], s["V"], s["table"], s["len"], s["prefix_table"],
                                              s["P"], **kw)
    return {"y": y, "K": s["K"], "V": s["V"]}


def run(state):
    if own:
        return _own(state)
    return _plain_append(state) if state["op"] == "append" else _plain_step(state)


# ---- work ------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    lens, new = _sizes(c)
    B, d, h = c["B"], c["d"], c["heads"]
    width = c["r3"] if c["shared"] else c["r3"] + c["t3"]
    if c["op"] == "append":
        n = sum(new)
        entries = sum((m + c["page"] - 1) // c["page"] for m in new)
        return {"bytes": e * (n * d + d * width + n * width) + 4 * (2 * B + 1 + entries), "flops": 2 * n * d * width}
    P = c.get("P", 0)
    cached = sum(lens) + P
    core = c["r1"] * c["r2"] * c["r3"] + c["t1"] * c["t2"] * c["t3"] + h * (c["r1"] + c["t1"])
    weights = core + d * (c["r2"] + c["t2"] + width)
    entries = sum(m // c["page"] + 1 for m in lens) + (P + c["page"] - 1) // c["page"]
    keys = sum(m + 1 + P for m in lens)                       # key rows that a head of a sequence attends to, over the batch
    per_token = d * (c["r2"] + c["t2"] + width) + c["r1"] * c["r3"] * (c["r2"] + h) + c["t1"] * c["t3"] * (c["t2"] + h)
    return {"bytes": e * (cached * width + weights + 2 * B * d + B * width) + 4 * (B + entries),
            "flops": 2 * h * keys * (c["r3"] + c["t3"]) + 2 * B * per_token}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _turn(x, pos, base):
    """Latent RoPE by complex numbers: coordinate pair i of a row at position pos times exp(i pos base^(-2 i / r))."""
    r = x.shape[-1]
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], r // 2, 2).contiguous())
    w = torch.exp(-math.log(base) * 2.0 / r * torch.arange(r // 2, device=x.device, dtype=torch.float64))
    a = torch.as_tensor(pos, device=x.device, dtype=torch.float64).unsqueeze(-1) * w
    return torch.view_as_real(z * torch.polar(torch.ones_like(a), a)).reshape(x.shape)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    lens, new = _sizes(c)
    page, P = c["page"], c.get("P", 0)
    Kx = s["K"].double()
    Vx = Kx if c["shared"] else s["V"].double()
    table = s["table"].cpu().tolist()
    U3, Ut3 = s["U3"].double(), s["Ut3"].double()

    def rows_of(pool, pages, n):
        """The first n rows of the pages listed, in order."""
        idx = torch.tensor(pages[:(n + page - 1) // page], dtype=torch.int64, device=pool.device)
        return pool[idx].reshape(-1, pool.shape[-1])[:n]

    if c["op"] == "append":
        t0 = 0
        for b, n in enumerate(new):
            xb = s["X"][t0:t0 + n].double()
            t0 += n
            i = torch.arange(lens[b], lens[b] + n, device=xb.device)
            pages = torch.tensor(table[b], device=xb.device)[i // page]
            k = xb @ U3
            Kx[pages, i % page] = _turn(k, i, c["base"]) if c["rope"] else k
            Vx[pages, i % page] = xb @ Ut3
        return {"K": Kx, "V": Vx}
    heads, scale = c["heads"], 1.0 / math.sqrt(c["d"] / c["heads"])
    G = torch.tensordot(s["U1"].double(), s["C"].double(), dims=1)             # one r2 x r3 matrix per head
    Gt = torch.tensordot(s["Ut1"].double(), s["Ct"].double(), dims=1)          # one t2 x t3 matrix per head
    turned = c["shared"] and c["rope"]                                          # the cache holds un-rotated rows
    out, fresh = [], []
    if P:
        pt = s["prefix_table"].cpu().tolist()
        kp, vp = rows_of(Kx, pt, P), rows_of(Vx, pt, P)
    for b in range(c["B"]):
        n = lens[b]
        xb = s["x"][b].double()
        k, v = rows_of(Kx, table[b], n), rows_of(Vx, table[b], n)
        if turned:
            k = _turn(k, torch.arange(n, device=k.device), c["base"])
        kn, vn = xb @ U3, xb @ Ut3
        q = torch.stack([(xb @ s["U2"].double()) @ G[i] for i in range(heads)])
        if c["rope"]:
            kn, q = _turn(kn, P + n, c["base"]), _turn(q, torch.full((heads,), P + n), c["base"])
        keys, values = torch.cat((k, kn[None])), torch.cat((v, vn[None]))
        score = q @ keys.t()
        o_max = score.amax(1)
        if P:
            sp = q @ kp.t()
            o_max = torch.maximum(o_max, sp.amax(1))
        e = torch.exp((score - o_max[:, None]) * scale)
        total, o = e.sum(1), e @ values
        if P:
            e = torch.exp((sp - o_max[:, None]) * scale)
            total, o = total + e.sum(1), o + e @ vp
        o = o / total[:, None]
        z = sum(Gt[i] @ o[i] for i in range(heads))
        out.append(s["Ut2"].double() @ z)
        fresh.append((table[b][n // page], n % page, vn if turned else kn, vn))
    for pg, row, kn, vn in fresh:
        Kx[pg, row] = kn
        if not c["shared"]:
            Vx[pg, row] = vn
    return {"y": torch.stack(out), "K": Kx, "V": Vx}
