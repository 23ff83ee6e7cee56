"""Measured cases of the serving operators over a paged latent KV cache that is held in 8 bits.

  append   tokens appended to the cache: latent keys and values projected from X, keys rotated by latent RoPE, each row
           quantised on its way to its page
  store    latent rows that are there already (a prefill wrote them) quantised into the pages
  read     cached rows read back
  decode   one decode step of a layer for a batch whose latent caches are paged and in 8 bits
  prefix   one decode step for a batch whose sequences share a long prefix that is stored, and attended to, once

`run` computes each in its plain form (elementary torch operations in 32 bits), or, with `own` set, through the
framework's entry points.  `exact` is the operators' definition in 64 bits, written apart from the plain form.

Cache: pools of e4m3 codes K [n_pages, page, r3] and V [n_pages, page, t3], and a scale 2^k for every row (an 8-bit
exponent) Ks, Vs [n_pages, page]; a row stands for its codes times its scale.  A row v is written with the least k, but
no less than -96, for which max |v| <= 448 * 2^k (a row of zeros: k = 0).  The row of slot i of sequence b is row
i % page of page block_table[b, i // page].  Entries past a sequence's last page, and slots past its length, hold
anything.  With `shared` one pool of latent rows serves keys and values; together with RoPE it holds un-rotated rows.
A decode step's new row takes part in its own attention as the cache stores it.
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
        # every sequence of a serving batch brings one token: latency
        _case("append", "append_one_each", B=64, L=4000, new=1, pad=0),
        # two long prompts
        _case("append", "append_long_prompts", B=2, L=0, new=8192, pad=0, page=128, ragged=False),
        # single precision, a few prompts that continue cached ones, rows of padding behind the last
        _case("append", "append_fp32", B=3, L=200, new=150, pad=5, page=16, dtype="fp32", **_SMALL),
        # --- store: the rows of a prefill of several prompts of mixed lengths go to their pages
        _case("store", "store_prompts", B=8, L=0, new=4096, pad=37),
        # single precision, a short continuation, small pages
        _case("store", "store_fp32", B=3, L=77, new=150, pad=5, page=16, dtype="fp32", **_SMALL),
        # --- read: the caches of a few long sequences as rows, to be moved or attended to by a prefill
        _case("read", "read_long", B=4, L=0, new=32768, pad=0),
        # a few rows from the middle of short ones
        _case("read", "read_rows", B=5, L=33, new=100, pad=3, page=16, **_SMALL),
        # --- decode: L = cached tokens of the longest sequence
        # one user, a few tokens in: latency
        _case("decode", "decode_first_tokens", B=1, L=37, page=16, **_SMALL),
        # a medium batch of one shared latent cache (keys rotated when read), odd rank
        _case("decode", "decode_shared_rope", B=24, L=3001, page=32, d=768, heads=12, r1=4, r2=96, r3=96, t1=4, t2=96, t3=96,
              shared=True),
        # the long-context serving batch, every sequence of another length: the largest call
        _case("decode", "decode_long_batch", B=64, L=32768, page=64),
        # --- prefix: P = tokens of the shared prefix, L = own cached tokens of the longest sequence
        # a few samples of one prompt, small model
        _case("prefix", "prefix_samples", B=6, P=999, L=100, page=16, **_SMALL),
        # a long document that a large batch asks about
        _case("prefix", "prefix_document", B=64, P=32768, L=1024, page=128),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "store", "read", "decode", "decode", "prefix"])
    fp32 = rng.random() < 0.2
    d, heads = rng.choice([(768, 12)] if fp32 else [(768, 12), (1024, 8), (2048, 16), (4096, 32)])
    rank = rng.choice([64] if fp32 else [64, 96, 128])
    kw = dict(d=d, heads=heads, r1=rng.choice([4, 8]), r2=rank, r3=rank, t1=rng.choice([4, 8]), t2=rank, t3=rank,
              page=rng.choice([16, 32, 64, 128]), rope=rng.random() < 0.8, base=rng.choice([10000.0, 500000.0]),
              ragged=rng.random() < 0.8, dtype="fp32" if fp32 else "bf16")
    if not fp32 and rank != 96 and rng.random() < 0.25:
        kw["t3"] = kw["t2"] = 192 - rank                     # value rank other than the key rank
    if op in ("append", "store", "read"):
        B = _log(rng, 1, 4 if fp32 and op == "append" else 64)
        most = 150 if fp32 and op == "append" else (16384 if op == "append" else 32768) // B
        return _case(op, B=B, new=_log(rng, 1, most), L=rng.randrange(0, 5000), pad=rng.choice([0, 0, 3, 50]), **kw)
    if op == "decode":
        B = _log(rng, 1, 4 if fp32 else 64)
        kw["shared"] = not fp32 and kw["t3"] == kw["r3"] and rng.random() < 0.25
        most = 1500 if fp32 else (3001 if kw["shared"] and kw["rope"] else 16384)
        return _case(op, B=min(B, 24) if kw["shared"] and kw["rope"] else B, L=_log(rng, 1, most), **kw)
    B = _log(rng, 1, 4 if fp32 else 64)
    return _case(op, B=B, P=_log(rng, 1, 801 if fp32 else 32768), L=_log(rng, 1, 60 if fp32 else 1024), **kw)


def _spread(most, B, ragged):
    """Lengths of B sequences, the longest `most`; ragged: spread over a quarter of it to all of it, in no order."""
    if not ragged or B == 1:
        return [most] * B
    return [most - (most * 3 // 4) * ((5 * b + 3) % B) // B if b else most for b in range(B)]


def _sizes(c):
    """Per sequence: cached tokens before the call (read: the first slot that is read), rows that are written or read."""
    lens = _spread(c["L"], c["B"], c["ragged"])
    new = _spread(c["new"], c["B"], c["ragged"]) if "new" in c else [1] * c["B"]
    return lens, [max(1, n) for n in new]


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 29)
    dt = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    lens, new = _sizes(c)
    B, page, d = c["B"], c["page"], c["d"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dt)

    def rows(*shape):
        """Latent rows: normal, the sizes of the rows within a factor of four of each other."""
        size = torch.exp2(torch.rand(*shape[:-1], 1, generator=g, device=dev) * 2 - 1)
        return torch.randn(*shape, generator=g, device=dev) * size

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
    s["K"], s["Ks"] = _quantise(rows(n_pages, page, c["r3"]))
    s["V"], s["Vs"] = (s["K"], s["Ks"]) if c["shared"] else _quantise(rows(n_pages, page, c["t3"]))
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["max_len"] = max(lens)
    if "new" in c:
        s["tokens"] = sum(new)
        s["start"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    total = sum(new) + c.get("pad", 0)
    if c["op"] == "store":
        s["Krows"], s["Vrows"] = rows(total, c["r3"]).to(dt), rows(total, c["t3"]).to(dt)
        return s
    if c["op"] == "read":
        # the buffers that the rows go to; what lies behind the last sequence's rows stays
        s["Krows"], s["Vrows"] = torch.zeros(total, c["r3"], dtype=dt, device=dev), torch.zeros(total, c["t3"], dtype=dt, device=dev)
        return s
    # factors with columns of length one; cores that give scores of standard deviation 2
    s["U3"] = normal(d, c["r3"], std=d ** -0.5)
    s["Ut3"] = s["U3"] if c["shared"] else normal(d, c["t3"], std=d ** -0.5)
    if c["op"] == "append":
        s["X"] = normal(total, d)
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

def _quantise(v):
    """Codes and scales of the rows v [..., r] (float)."""
    a = v.abs().amax(dim=-1)
    m, e = torch.frexp(a)                                    # a = m 2^e, m in [1/2, 1): a <= 7/8 2^(k + 9)
    k = torch.where(a > 0, e - 9 + (m > 0.875).to(e.dtype), torch.zeros_like(e)).clamp(min=-96)
    codes = torch.ldexp(v, -k[..., None]).to(torch.float8_e4m3fn)
    return codes, (k + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _scale(s):
    """Scales as floats."""
    return torch.exp2(s.view(torch.uint8).float() - 127)


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


def _put(s, which, at, v):
    """Rows v (float) quantised to rows `at` of the pool."""
    codes, scale = _quantise(v)
    s[which].view(torch.uint8).view(-1, v.shape[-1])[at] = codes.view(torch.uint8)
    s[which + "s"].view(torch.uint8).view(-1)[at] = scale.view(torch.uint8)
    return codes.float() * _scale(scale)[..., None]


def _get(s, which, at):
    """Rows `at` of the pool, as floats."""
    pool = s[which].view(torch.uint8)
    codes = pool.view(-1, pool.shape[-1])[at].view(torch.float8_e4m3fn).float()
    return codes * _scale(s[which + "s"].view(torch.uint8).view(-1)[at])[..., None]


def _cache(s):
    return {"K": s["K"], "Ks": s["Ks"], "V": s["V"], "Vs": s["Vs"]}


def _plain_rows(s):
    """Sequence, slot and pool row of each row of a ragged batch."""
    row = torch.arange(s["tokens"], device=s["table"].device)
    seq = torch.searchsorted(s["start"][1:], row.int(), right=True)
    pos = s["len"][seq].long() + row - s["start"][seq].long()
    return pos, _slots(s, seq, pos)


def _plain_append(s):
    pos, at = _plain_rows(s)
    X = s["X"][:s["tokens"]].float()
    k = X @ s["U3"].float()
    _put(s, "K", at, _rotate(k, pos, s["base"]) if s["rope"] else k)
    _put(s, "V", at, X @ s["Ut3"].float())
    return _cache(s)


def _plain_store(s):
    _, at = _plain_rows(s)
    _put(s, "K", at, s["Krows"][:s["tokens"]].float())
    _put(s, "V", at, s["Vrows"][:s["tokens"]].float())
    return _cache(s)


def _plain_read(s):
    _, at = _plain_rows(s)
    s["Krows"][:s["tokens"]] = _get(s, "K", at).to(s["Krows"].dtype)
    s["Vrows"][:s["tokens"]] = _get(s, "V", at).to(s["Vrows"].dtype)
    return {"Krows": s["Krows"], "Vrows": s["Vrows"]}


def _plain_step(s):
    B, h, L, P = s["B"], s["heads"], s["max_len"], s.get("P", 0)
    x, n = s["x"].float(), s["len"].long()
    k_new, v_new = x @ s["U3"].float(), x @ s["Ut3"].float()
    q = torch.einsum("ha,bac->bhc", s["U1"].float(), torch.einsum("bq,aqc->bac", x @ s["U2"].float(), s["C"].float()))
    if s["rope"]:
        q = _rotate(q, (P + n)[:, None].expand(B, h), s["base"])
    # the cached rows of every sequence, up to the longest; what lies past a sequence's end is masked
    pos = torch.arange(L, device=x.device)
    at = s["table"].clamp(min=0)[:, pos // s["page"]].long() * s["page"] + pos % s["page"]
    there = pos[None, :] < n[:, None]
    k = _get(s, "K", at)
    v = k if s["shared"] else _get(s, "V", at)
    if s["shared"] and s["rope"]:
        k = _rotate(k, pos[None, :].expand(B, L), s["base"])
    v = torch.where(there[:, :, None], v, 0.0)
    score = (q @ k.transpose(1, 2)).masked_fill(~there[:, None, :], -math.inf)
    # the new row as the cache stores it
    at = _slots(s, torch.arange(B, device=x.device), n)
    if s["shared"]:
        v_new = _put(s, "K", at, v_new)
        k_new = _rotate(v_new, P + n, s["base"]) if s["rope"] else v_new
    else:
        k_new = _put(s, "K", at, _rotate(k_new, P + n, s["base"]) if s["rope"] else k_new)
        v_new = _put(s, "V", at, v_new)
    score = torch.cat((score, (q * k_new[:, None, :]).sum(-1, keepdim=True)), dim=2)
    if P:
        i = torch.arange(P, device=x.device)
        at = s["prefix_table"][i // s["page"]].long() * s["page"] + i % s["page"]
        kp, vp = _get(s, "K", at), _get(s, "V", at)
        score = torch.cat((score, (q.reshape(B * h, -1) @ kp.t()).view(B, h, P)), dim=2)
    score = score * (s["d"] / h) ** -0.5
    p = (score - score.amax(dim=2, keepdim=True)).exp()
    p = p / p.sum(dim=2, keepdim=True)
    o = p[:, :, :L] @ v + p[:, :, L:L + 1] * v_new[:, None, :]
    if P:
        o = o + (p[:, :, L + 1:].reshape(B * h, P) @ vp).view(B, h, -1)
    z = torch.einsum("bac,ajc->bj", torch.einsum("ha,bhc->bac", s["Ut1"].float(), o), s["Ct"].float())
    y = z @ s["Ut2"].float().t()
    return {"y": y.to(s["x"].dtype), **_cache(s)}


# ---- the framework's operators ---------------------------------------------------------------------------------------

def _own(s):
    from paper_2603_30033_b200 import binding
    pools = (s["K"], s["Ks"], s["V"], s["Vs"], s["table"])
    if s["op"] == "append":
        binding.tucker_cache_append_paged_q8(s["X"], s["U3"], s["Ut3"], *pools, s["len"], s["start"], rope=s["rope"], rope_base=s["base"])
        return _cache(s)
    if s["op"] == "store":
        binding.tucker_cache_store_paged_q8(s["Krows"], s["Vrows"], *pools, s["len"], s["start"])
        return _cache(s)
    if s["op"] == "read":
        binding.tucker_cache_read_paged_q8(*pools, s["len"], s["start"], s["Krows"], s["Vrows"])
        return {"Krows": s["Krows"], "Vrows": s["Vrows"]}
    weights = [s[k] for k in ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")]
    kw = dict(n_H=s["heads"], rope=s["rope"], rope_base=s["base"], append=True)
    if s["op"] == "decode":
        y = binding.tucker_attn_decode_paged_q8(s["x"], *weights, *pools, s["len"], **kw)
    else:
        y = binding.tucker_attn_decode_prefix_q8(s["x"], *weights, *pools, s["len"], s["prefix_table"], s["P"], **kw)
    return {"y": y, **_cache(s)}


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "store": _plain_store, "read": _plain_read}.get(state["op"], _plain_step)(state)


# ---- work ------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    lens, new = _sizes(c)
    B, d, h = c["B"], c["d"], c["heads"]
    width = c["r3"] if c["shared"] else c["r3"] + c["t3"]
    row = width + (1 if c["shared"] else 2)                   # bytes of a cached token
    if "new" in c:
        n = sum(new)
        entries = sum((m + c["page"] - 1) // c["page"] for m in new)
        if c["op"] != "append":
            return {"bytes": n * (e * width + row) + 4 * (2 * B + 1 + entries), "flops": n * width}
        return {"bytes": e * (n * d + d * width) + n * row + 4 * (2 * B + 1 + entries), "flops": 2 * n * d * width}
    P = c.get("P", 0)
    cached = sum(lens) + P
    core = c["r1"] * c["r2"] * c["r3"] + c["t1"] * c["t2"] * c["t3"] + h * (c["r1"] + c["t1"])
    weights = core + d * (c["r2"] + c["t2"] + width)
    entries = sum(m // c["page"] + 1 for m in lens) + (P + c["page"] - 1) // c["page"]
    keys = sum(m + 1 + P for m in lens)                       # key rows that a head of a sequence attends to, over the batch
    per_token = d * (c["r2"] + c["t2"] + width) + c["r1"] * c["r3"] * (c["r2"] + h) + c["t1"] * c["t3"] * (c["t2"] + h)
    return {"bytes": (cached + B) * row + e * (weights + 2 * B * d) + 4 * (B + entries),
            "flops": 2 * h * keys * (c["r3"] + c["t3"]) + 2 * B * per_token}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _turn(x, pos, base):
    """Latent RoPE by complex numbers: coordinate pair i of a row at position pos times exp(i pos base^(-2 i / r))."""
    r = x.shape[-1]
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], r // 2, 2).contiguous())
    w = torch.exp(-math.log(base) * 2.0 / r * torch.arange(r // 2, device=x.device, dtype=torch.float64))
    a = torch.as_tensor(pos, device=x.device, dtype=torch.float64).unsqueeze(-1) * w
    return torch.view_as_real(z * torch.polar(torch.ones_like(a), a)).reshape(x.shape)


def _fit(v):
    """The scale of each row of v, by trying the powers of two upwards."""
    a = v.abs().amax(-1)
    two_k = torch.full_like(a, 2.0 ** -96)
    for k in range(-96, 128):
        two_k = torch.where(a > 448 * two_k, torch.full_like(a, 2.0 ** (k + 1)), two_k)
    return torch.where(a == 0, torch.ones_like(a), two_k)


def _nearest(v):
    """The e4m3 number nearest to each v (|v| <= 448): steps of 2^(e - 3) in the binade 2^e, of 2^-9 below 2^-6."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(v / step) * step


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    lens, new = _sizes(c)
    page, P = c["page"], c.get("P", 0)
    pools = {}                                                # codes and scales; both names of a shared pool are one
    for w in ("K", "V"):
        pools[w] = pools["K"] if w == "V" and c["shared"] else (s[w].double(), s[w + "s"].float().double())
    table = s["table"].cpu().tolist()

    def rows_of(w, pages, beg, end):
        """Rows beg .. end - 1 of the pages listed, in order."""
        i = torch.arange(beg, end, device=s["table"].device)
        pg = torch.tensor(pages, dtype=torch.int64, device=i.device)[i // page] if end > beg else i
        codes, scale = pools[w]
        return codes[pg, i % page] * scale[pg, i % page][:, None]

    def write(w, pages, beg, v):
        """The rows v to slots beg ..: as the numbers that the codes are the nearest to."""
        i = torch.arange(beg, beg + len(v), device=v.device)
        pg = torch.tensor(pages, dtype=torch.int64, device=v.device)[i // page]
        scale = _fit(v)
        pools[w][0][pg, i % page] = v / scale[:, None]
        pools[w][1][pg, i % page] = scale

    def cache():
        return {"K": pools["K"][0], "Ks": pools["K"][1], "V": pools["V"][0], "Vs": pools["V"][1]}

    if "new" in c:
        t0 = 0
        out = {"Krows": s["Krows"].double(), "Vrows": s["Vrows"].double()} if c["op"] == "read" else None
        for b, n in enumerate(new):
            part = slice(t0, t0 + n)
            t0 += n
            if c["op"] == "read":
                for w in ("K", "V"):
                    out[w + "rows"][part] = rows_of(w, table[b], lens[b], lens[b] + n)
            elif c["op"] == "store":
                for w in ("K", "V"):
                    write(w, table[b], lens[b], s[w + "rows"][part].double())
            else:
                xb = s["X"][part].double()
                k = xb @ s["U3"].double()
                write("K", table[b], lens[b], _turn(k, torch.arange(lens[b], lens[b] + n), c["base"]) if c["rope"] else k)
                write("V", table[b], lens[b], xb @ s["Ut3"].double())
        return out or cache()
    heads, scale = c["heads"], 1.0 / math.sqrt(c["d"] / c["heads"])
    U3, Ut3 = s["U3"].double(), s["Ut3"].double()
    G = torch.tensordot(s["U1"].double(), s["C"].double(), dims=1)             # one r2 x r3 matrix per head
    Gt = torch.tensordot(s["Ut1"].double(), s["Ct"].double(), dims=1)          # one t2 x t3 matrix per head
    turned = c["shared"] and c["rope"]                                          # the cache holds un-rotated rows
    out, fresh = [], []
    if P:
        pt = s["prefix_table"].cpu().tolist()
        kp, vp = rows_of("K", pt, 0, P), rows_of("V", pt, 0, P)

    def stored(v):
        f = _fit(v[None])[0]
        return _nearest(v / f) * f

    for b in range(c["B"]):
        n = lens[b]
        xb = s["x"][b].double()
        k, v = rows_of("K", table[b], 0, n), rows_of("V", table[b], 0, n)
        kn, vn = xb @ U3, xb @ Ut3
        if turned:
            k = _turn(k, torch.arange(n, device=k.device), c["base"])
        elif c["rope"]:
            kn = _turn(kn, P + n, c["base"])
        fresh.append((kn, vn))
        kn, vn = stored(kn), stored(vn)
        if turned:
            kn = _turn(kn, P + n, c["base"])
        q = torch.stack([(xb @ s["U2"].double()) @ G[i] for i in range(heads)])
        if c["rope"]:
            q = _turn(q, torch.full((heads,), P + n), c["base"])
        keys, values = torch.cat((k, kn[None])), torch.cat((v, vn[None]))
        if P:
            keys, values = torch.cat((kp, keys)), torch.cat((vp, values))
        score = q @ keys.t()
        e = torch.exp((score - score.amax(1, keepdim=True)) * scale)
        o = (e @ values) / e.sum(1)[:, None]
        z = sum(Gt[i] @ o[i] for i in range(heads))
        out.append(s["Ut2"].double() @ z)
    for b, (kn, vn) in enumerate(fresh):
        write("K", table[b], lens[b], kn[None])
        if not c["shared"]:
            write("V", table[b], lens[b], vn[None])
    return {"y": torch.stack(out), **cache()}
