"""Exact attention for serving, beside the quantized attention of this library: what its users have it compute.

A case names an operator (``kind``) and a problem:

  prompt   ``binding.ExactAttention``: attention over packed sequences, grouped heads, causal or not
  append   ``binding.PagedCache.append`` and ``.read``: keys rotated by their positions and stored with the values in a
           paged cache, in the tensors' own type or in 4 bits, then read back; the queries are rotated in the same call
  prefix   ``PagedCache.read``, then ``ExactAttention``: a further piece of prompts whose earlier part is cached
  cached   ``PagedCache.attend``: the last one or few queries of every sequence over its pages
  step     ``PagedCache.append``, then ``.attend``: one generation step of a layer

Sequence lengths of a case follow from its numbers alone (``_lengths``), and with them its work.

Storage in 4 bits: a group is 32 neighbouring head dimensions of one token and head.  It is kept as its smallest value
``lo`` and a step ``(largest - lo) / 15``, both bfloat16, and 32 codes 0..15; it stands for ``lo + code * step``.  A
page of one head holds the codes of all its tokens (d/2 bytes each), then their (lo, step) pairs (d/8 bytes each).
The 8 codes of dimensions 32 g + 8 t .. + 7 fill, lowest first, the 4 bytes at t * d/8 + 4 g of the token's code row.
"""
import math
import random

import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16


# ---------------------------------------------------------------- cases
def _case(kind, **kw):
    base = dict(kind=kind, B=1, H=8, Hk=8, d=128, dtype="bf16", n=1, longest=1, ragged=True, mix=1)
    base.update(kw)
    return base


def listed():
    return [
        # five short packed prompts, one of them empty: a call that is all launch and latency
        dict(_case("prompt", B=5, H=12, Hk=4, d=64, longest=201, causal=True, mix=5), name="prompt_short"),
        # a batch of prompts of different lengths, four query heads to a key head
        dict(_case("prompt", B=16, H=32, Hk=8, d=128, longest=2048, causal=True, mix=6), name="prompt_batch"),
        # one long prompt at the sizes of the repository's largest configuration
        dict(_case("prompt", B=1, H=16, Hk=4, d=128, longest=16384, ragged=False, causal=True), name="prompt_long"),
        # images of 785 tokens, every token seeing every other, in float32 (checking a bfloat16 deployment)
        dict(_case("prompt", B=8, H=12, Hk=12, d=64, longest=785, ragged=False, causal=False, dtype="f32"),
             name="images_f32"),
        # one new token of each of 48 sequences into a bfloat16 cache: latency
        dict(_case("append", B=48, H=32, Hk=8, d=128, page=16, bits=16, rot=128, adjacent=True, longest=8192),
             name="append_tokens"),
        # a long prompt's keys and values into a 4-bit cache
        dict(_case("append", B=1, n=16384, H=16, Hk=8, d=128, page=64, bits=4, rot=128, adjacent=False, longest=16384),
             name="append_prompt_4bit"),
        # 256 further tokens of four prompts over what a 4-bit cache holds of them
        dict(_case("prefix", B=4, n=256, H=16, Hk=4, d=128, page=64, bits=4, longest=8192, causal=True, mix=9),
             name="prefix_4bit"),
        # a single short sequence, one query: latency
        dict(_case("cached", B=1, H=12, Hk=12, d=64, page=16, bits=16, longest=901, ragged=False), name="one_sequence"),
        # a serving batch over a bfloat16 cache
        dict(_case("cached", B=64, H=32, Hk=8, d=128, page=16, bits=16, longest=4096, mix=11), name="batch"),
        # one generation step of a layer over a 4-bit cache: the new tokens are appended, then attended to
        dict(_case("step", B=64, H=32, Hk=8, d=128, page=32, bits=4, rot=128, adjacent=False, longest=8192, mix=12),
             name="step_4bit"),
        # two sequences at the longest context: few rows, a long axis to split
        dict(_case("cached", B=2, H=32, Hk=4, d=128, page=64, bits=4, longest=131072, mix=13), name="long_4bit"),
        # four drafted tokens of each sequence checked in one call, float32
        dict(_case("cached", B=6, n=4, H=8, Hk=4, d=64, page=16, bits=32, longest=16384, dtype="f32", mix=14),
             name="draft_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    most_f32 = {"bytes": most["bytes"] / 2, "flops": most["flops"] / 16}
    while True:
        kind = rng.choice(["prompt", "prompt", "append", "prefix", "cached", "cached", "step"])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        d = rng.choice([64, 128])
        Hk = rng.choice([1, 2, 4, 5, 8, 12])
        c = _case(kind, H=Hk * rng.choice([1, 1, 2, 3, 4, 6, 8]), Hk=Hk, d=d, dtype=dtype, mix=rng.randrange(1, 10 ** 6),
                  ragged=rng.random() < 0.8)
        if kind == "prompt":
            c.update(B=_log(rng, 1, 64), longest=_log(rng, 1, 16384), causal=rng.random() < 0.7)
        else:
            c.update(page=rng.choice([16, 32, 64, 128]), bits=rng.choice([4, 32 if dtype == "f32" else 16]))
        if kind in ("append", "step"):
            c.update(rot=rng.choice([d, d // 2, 0]), adjacent=rng.random() < 0.5)
        if kind == "append":
            c.update(B=_log(rng, 1, 256), n=1, longest=_log(rng, 16, 131072))
            if rng.random() < 0.5:
                c.update(B=_log(rng, 1, 4), n=_log(rng, 16, 16384))
            c["longest"] = max(c["longest"], c["n"])
        if kind == "prefix":
            c.update(B=_log(rng, 1, 8), n=_log(rng, 2, 1024), causal=True)
            c["longest"] = _log(rng, c["n"], 16384)
        if kind in ("cached", "step"):
            c.update(B=_log(rng, 1, 128), n=1 if kind == "step" else rng.choice([1, 1, 1, 2, 4, 5]), longest=_log(rng, 8, 131072))
        cap = most if dtype == "bf16" else most_f32
        w = work(c)
        if w["flops"] <= cap["flops"] and w["bytes"] <= cap["bytes"] and _padded(c) <= 2 ** 31:
            return c


def _padded(c):
    """Elements of the largest intermediate of the plain form: every sequence padded to the longest."""
    if c["kind"] == "append":
        return 0
    scores = c["B"] * (c["H"] // c["Hk"]) * c["longest"] * (c["longest"] if c["kind"] == "prompt" else c["n"])
    return max(scores, c["B"] * c["Hk"] * c["longest"] * c["d"] if c["kind"] != "prompt" else 0)


def _lengths(c):
    """Keys of every sequence.  Ragged: spread over their logarithm from one token on, the first one the longest; a
    packed batch of prompts ends with an empty one."""
    rng = random.Random(c["mix"])
    lens = [c["longest"]] + [_log(rng, max(1, c["longest"] // 8), c["longest"]) if c["ragged"] else c["longest"]
                             for _ in range(c["B"] - 1)]
    if c["ragged"] and c["B"] > 2:
        lens[1] = min(c["longest"], c["n"])
        if c["kind"] == "prompt":
            lens[-1] = 0
    return lens if c["kind"] == "prompt" else [max(x, c["n"]) for x in lens]


def _scale(c):
    return 1.0 / math.sqrt(c["d"])


def _row_bytes(c):
    """Bytes of one token of one head in the cache, keys or values."""
    return 5 * c["d"] // 8 if c["bits"] == 4 else c["d"] * c["bits"] // 8


def work(c):
    es, d, H, Hk, lens = (4 if c["dtype"] == "f32" else 2), c["d"], c["H"], c["Hk"], _lengths(c)
    T, n = sum(lens), c["n"]
    new = c["B"] * n
    if c["kind"] == "prompt":
        pairs = sum(x * (x + 1) // 2 if c["causal"] else x * x for x in lens)
        return {"bytes": es * d * T * (2 * H + 2 * Hk) + 4 * H * T, "flops": 4 * d * H * pairs}
    seen = sum(n * x - n * (n - 1) // 2 for x in lens)
    attend = {"bytes": 2 * Hk * T * _row_bytes(c) + 2 * es * d * H * new + 4 * H * new, "flops": 4 * d * H * seen}
    if c["kind"] == "cached":
        return attend
    if c["kind"] == "prefix":                              # the rows are written in the tensors' type and read once
        return {"bytes": attend["bytes"] + 4 * es * d * Hk * T, "flops": attend["flops"]}
    put = es * d * new * (2 * Hk + 2 * H) + 2 * Hk * new * _row_bytes(c) + 4 * new * c["rot"]
    turn = 3 * c["rot"] * new * (H + Hk) + (8 * d * new * Hk if c["bits"] == 4 else 0)
    if c["kind"] == "append":                              # the stored rows come back in the tensors' type
        return {"bytes": put + 2 * Hk * new * _row_bytes(c) + 2 * es * d * Hk * new, "flops": turn}
    return {"bytes": put + attend["bytes"], "flops": turn + attend["flops"]}


# ---------------------------------------------------------------- storage in 4 bits
def _encode(x):
    """float32 [..., d] -> (codes uint8 [..., d/2], (lo, step) bfloat16 [..., d/32, 2])."""
    d = x.shape[-1]
    g = x.unflatten(-1, (d // 32, 32))
    lo = g.amin(-1).to(BF16)
    step = ((g.amax(-1) - lo.float()) * (1.0 / 15.0)).to(BF16)
    by = step.float().unsqueeze(-1)
    q = torch.where(by > 0, (g - lo.float().unsqueeze(-1)) / by, torch.zeros_like(g)).round().clamp(0, 15).to(torch.uint8)
    q = q.unflatten(-1, (4, 4, 2)).transpose(-4, -3)       # [..., t, g, byte, nibble]
    codes = (q[..., 0] | (q[..., 1] << 4)).flatten(-3)
    return codes, torch.stack([lo, step], -1)


def _decode(codes, par):
    """What (codes, pairs) stand for: float32 [..., d]."""
    groups = par.shape[-2]
    b = codes.unflatten(-1, (4, groups, 4)).transpose(-3, -2)
    q = torch.stack([b & 15, b >> 4], -1).flatten(-3).float()
    return (par[..., 0:1].float() + q * par[..., 1:2].float()).flatten(-2)


def _split(buf, page, d):
    """Views of a 4-bit cache [pages, Hk, page * 5 d / 8] bytes: codes and (lo, step) pairs."""
    cut = page * d // 2
    codes = buf[..., :cut].unflatten(-1, (page, d // 2))
    par = buf[..., cut:].view(BF16).unflatten(-1, (page, d // 32, 2))
    return codes, par


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + c["mix"])
    dt = F32 if c["dtype"] == "f32" else BF16
    B, H, Hk, d, n, lens = c["B"], c["H"], c["Hk"], c["d"], c["n"], _lengths(c)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)

    def rows(T, heads, spread=1.0):
        return (spread * torch.randn(T, heads, d, device=dev, generator=g)).to(dt)

    st = {"case": c, "lens": ints(lens)}
    ends = [0]
    for x in lens:
        ends.append(ends[-1] + x)
    if c["kind"] == "prompt":
        # queries, keys and values as views of one projection's output, as a layer has them
        wide = (torch.randn(max(ends[-1], 1), (H + 2 * Hk), d, device=dev, generator=g)).to(dt)[:ends[-1]]
        st.update(Q=wide[:, :H], K=wide[:, H:H + Hk], V=wide[:, H + Hk:], cu=ints(ends))
    else:
        page, bits = c["page"], c["bits"]
        per = [-(-x // page) for x in lens]
        pages = sum(per) + 3                                 # a few that belong to nobody
        order = torch.randperm(pages, device=dev, generator=g).to(torch.int32)
        table = torch.zeros(B, max(per), dtype=torch.int32, device=dev)
        at = 0
        for b, k in enumerate(per):
            table[b, :k] = order[at:at + k]
            at += k
        seq = torch.repeat_interleave(torch.arange(B, device=dev), st["lens"].long(), output_size=ends[-1])
        pos = torch.arange(ends[-1], device=dev) - ints(ends)[:-1].long()[seq]
        slot = table[seq, pos // page].long() * page + pos % page
        new = pos >= st["lens"].long()[seq] - n              # the last n tokens of each sequence are this pass's
        keys = torch.zeros(pages, Hk, page * 5 * d // 8, dtype=torch.uint8, device=dev) if bits == 4 else \
            torch.zeros(pages, Hk, page, d, dtype=dt, device=dev)
        st.update(keys=keys, values=torch.zeros_like(keys), table=table)
        # keys have a few wide dimensions, as learned ones do
        spread = 1.0 + 3.0 * (torch.rand(Hk, d, device=dev, generator=g) < 0.05)
        fill = torch.randn(pages, Hk, page, d, device=dev, generator=g) if c["kind"] != "append" else None
        for name in ("keys", "values") if fill is not None else ():
            x = (fill * spread[:, None]).to(dt) if name == "keys" else fill.roll(1, 0).to(dt)
            if bits == 4:
                for part in range(0, pages, 4096):
                    codes, par = _split(st[name][part:part + 4096], page, d)
                    a, b = _encode(x[part:part + 4096].float())
                    codes.copy_(a)
                    par.copy_(b)
            else:
                st[name].copy_(x)
        del fill
        st["Q"] = rows(B * n, H)
        if c["kind"] in ("append", "step"):
            wide = torch.randn(B * n, 2 * Hk, d, device=dev, generator=g)
            wide[:, :Hk] *= spread
            wide = wide.to(dt)
            st.update(K=wide[:, :Hk], V=wide[:, Hk:], slots=slot[new].to(torch.int32), pos=pos[new].to(torch.int32))
            rot = c["rot"]
            if rot:
                rate = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
                angle = torch.arange(c["longest"], device=dev, dtype=torch.float64)[:, None] * rate
                st.update(cos=angle.cos().float(), sin=angle.sin().float())
        if c["kind"] == "prefix":
            st.update(slots=slot.to(torch.int32), cu_q=ints([n * b for b in range(B + 1)]), cu_k=ints(ends))
    if own:
        from paper_2607_12789_b200 import binding
        if c["kind"] in ("prompt", "prefix"):
            st["attention"] = binding.ExactAttention(H, Hk, d, dtype=dt, causal=c["causal"])
        if c["kind"] != "prompt":
            st["cache"] = binding.PagedCache(st["keys"], st["values"], c["page"], d, dtype=dt, bits=c["bits"])
        if c["kind"] in ("cached", "step"):
            st["plan"] = st["cache"].plan(H, B, n)
    return st


# ---------------------------------------------------------------- plain forms
def _softmax_product(S, seen, V):
    """Rows of S over the columns that `seen` leaves: (weights V, log of the sum); a row without any gives 0 and -inf."""
    S = S.masked_fill(~seen, -math.inf)
    top = S.amax(-1, keepdim=True)
    P = (S - torch.where(top.isinf(), torch.zeros_like(top), top)).exp()
    total = P.sum(-1, keepdim=True)
    Y = (P @ V) / torch.where(total > 0, total, torch.ones_like(total))
    return Y, (total.log() + top).squeeze(-1)


def _prompt_plain(Q, K, V, len_q, len_k, cu_q, cu_k, most_q, most_k, c):
    """Every sequence padded to the longest, one key head at a time."""
    H, Hk, dev = c["H"], c["Hk"], Q.device
    G = H // Hk
    i, j = torch.arange(most_q, device=dev), torch.arange(most_k, device=dev)
    in_q, in_k = i < len_q[:, None], j < len_k[:, None]
    at_q = (cu_q[:-1, None] + i).clamp(max=max(Q.shape[0] - 1, 0)).long()
    at_k = (cu_k[:-1, None] + j).clamp(max=max(K.shape[0] - 1, 0)).long()
    seen = in_k[:, None, :].expand(-1, most_q, -1)
    if c["causal"]:
        seen = seen & (j <= i[:, None] + (len_k - len_q)[:, None, None])
    Y = torch.zeros(Q.shape[0] + 1, H, c["d"], device=dev)
    L = torch.zeros(Q.shape[0] + 1, H, device=dev)
    to = torch.where(in_q, at_q, torch.full_like(at_q, Q.shape[0]))
    for h in range(Hk):
        q = Q[:, h * G:(h + 1) * G].float()[at_q].transpose(1, 2)          # [B, G, nq, d]
        k, v = K[:, h].float()[at_k][:, None], V[:, h].float()[at_k][:, None]
        y, l = _softmax_product((q * _scale(c)) @ k.transpose(-1, -2), seen[:, None], v)
        Y[to, h * G:(h + 1) * G] = y.transpose(1, 2)
        L[to, h * G:(h + 1) * G] = l.transpose(1, 2)
    return Y[:-1].to(Q.dtype), L[:-1]


def _rotate(x, st):
    """Rotation of the leading `rot` dimensions by the positions' angles: float32, rounded once to the tensors' type."""
    c = st["case"]
    rot = c["rot"]
    if not rot:
        return x
    cos, sin = (st[k][st["pos"].long()][:, None] for k in ("cos", "sin"))
    f = x.float()
    a, b = (f[..., 0:rot:2], f[..., 1:rot:2]) if c["adjacent"] else (f[..., :rot // 2], f[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if c["adjacent"] else torch.cat([u, v], -1)
    return torch.cat([turned.to(x.dtype), x[..., rot:]], -1)


def _append_plain(st):
    c = st["case"]
    page, d = c["page"], c["d"]
    p, r = st["slots"].long() // page, st["slots"].long() % page
    for buf, x in ((st["keys"], _rotate(st["K"], st)), (st["values"], st["V"])):
        if c["bits"] == 4:
            codes, par = _split(buf, page, d)
            codes[p, :, r], par[p, :, r] = _encode(x.float())
        else:
            buf[p, :, r] = x
    return _rotate(st["Q"], st)


def _read_plain(st):
    c = st["case"]
    page, d, dt = c["page"], c["d"], st["Q"].dtype
    p, r = st["slots"].long() // page, st["slots"].long() % page
    out = []
    for buf in (st["keys"], st["values"]):
        if c["bits"] == 4:
            codes, par = _split(buf, page, d)
            out.append(_decode(codes[p, :, r], par[p, :, r]).to(dt))
        else:
            out.append(buf[p, :, r])
    return out


def _cached_plain(st, Q):
    c, table, lens = st["case"], st["table"].long(), st["lens"]
    B, H, Hk, d, n, page = c["B"], c["H"], c["Hk"], c["d"], c["n"], c["page"]

    def pages(buf):
        x = _decode(*(v[table] for v in _split(buf, page, d))) if c["bits"] == 4 else buf[table].float()
        return x.transpose(1, 2).flatten(2, 3)                              # [B, Hk, tokens, d]

    L = table.shape[1] * page
    j = torch.arange(L, device=Q.device)
    seen = j < (lens[:, None] - n + 1 + torch.arange(n, device=Q.device))[..., None]      # [B, n, tokens]
    q = Q.float().view(B, n, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).flatten(2, 3) * _scale(c)
    y, l = _softmax_product(q @ pages(st["keys"]).transpose(-1, -2), seen[:, None].repeat(1, 1, H // Hk, 1), pages(st["values"]))
    back = lambda t: t.unflatten(2, (H // Hk, n)).movedim(3, 1).flatten(2, 3).flatten(0, 1)
    return back(y).to(Q.dtype), back(l)


def run(state):
    st, c = state, state["case"]
    kind = c["kind"]
    if own:
        if kind == "prompt":
            return st["attention"](st["Q"], st["K"], st["V"], st["cu"], lse=True)
        if kind in ("append", "step"):
            turn = dict(pos=st["pos"], cos=st["cos"], sin=st["sin"], adjacent=c["adjacent"]) if c["rot"] else {}
            Q = st["cache"].append(st["K"], st["V"], st["slots"], Q=st["Q"], **turn)
            if kind == "append":
                return (Q, *st["cache"].read(st["slots"]))
            return (Q, *st["cache"].attend(Q, st["table"], st["lens"], lse=True, plan=st["plan"]))
        if kind == "prefix":
            K, V = st["cache"].read(st["slots"])
            return st["attention"](st["Q"], K, V, st["cu_q"], st["cu_k"], lse=True)
        return st["cache"].attend(st["Q"], st["table"], st["lens"], lse=True, plan=st["plan"])
    if kind == "prompt":
        return _prompt_plain(st["Q"], st["K"], st["V"], st["lens"], st["lens"], st["cu"], st["cu"], c["longest"], c["longest"], c)
    if kind in ("append", "step"):
        Q = _append_plain(st)
        return (Q, *_read_plain(st)) if kind == "append" else (Q, *_cached_plain(st, Q))
    if kind == "prefix":
        K, V = _read_plain(st)
        n = torch.full_like(st["lens"], c["n"])
        return _prompt_plain(st["Q"], K, V, n, st["lens"], st["cu_q"], st["cu_k"], c["n"], c["longest"], c)
    return _cached_plain(st, st["Q"])


# ---------------------------------------------------------------- the operators' definitions in 64 bits
def _one_head(q, k, v, first, scale):
    """Queries [n, d] of one head over keys [m, d]; query i sees keys 0 .. first + i (first None: all of them)."""
    n, m = q.shape[0], k.shape[0]
    y, l = q.new_zeros(n, q.shape[1]), q.new_full((n,), -math.inf)
    if not m:
        return y, l
    for at in range(0, n, 4096):
        s = scale * (q[at:at + 4096] @ k.T)
        if first is not None:
            rows = torch.arange(at, at + s.shape[0], device=q.device)[:, None] + first
            s = torch.where(torch.arange(m, device=q.device) <= rows, s, -math.inf)
        l[at:at + 4096] = torch.logsumexp(s, -1)
        w = torch.exp(s - l[at:at + 4096, None])
        y[at:at + 4096] = torch.where(torch.isinf(l[at:at + 4096, None]), 0.0, w) @ v
    return y, l


def _turn64(x, cos, sin, rot, adjacent, dt):
    out = x.double().clone()
    for k in range(rot // 2):
        a, b = (2 * k, 2 * k + 1) if adjacent else (k, k + rot // 2)
        c, s = cos[:, k, None].double(), sin[:, k, None].double()
        out[..., a] = x[..., a].double() * c - x[..., b].double() * s
        out[..., b] = x[..., b].double() * c + x[..., a].double() * s
    return out.to(dt).double()                             # stored and handed on in the tensors' type


def _stored64(x, bits):
    """What the cache holds of x [..., d] (float64): x itself, or its groups' nearest of 16 values."""
    if bits != 4:
        return x
    out = torch.empty_like(x)
    for a in range(0, x.shape[-1], 32):
        v = x[..., a:a + 32]
        lo = v.min(-1, keepdim=True).values.to(BF16).double()
        step = ((v.max(-1, keepdim=True).values - lo) / 15).to(BF16).double()
        out[..., a:a + 32] = lo + step * ((v - lo) / step.clamp(min=1e-300)).round().clamp(0, 15)
    return out


def _held64(buf, slots, c):
    """Rows of the cache at `slots`, [T, Hk, d] in float64, code by code from the bytes."""
    page, d, Hk = c["page"], c["d"], c["Hk"]
    p, r = torch.div(slots, page, rounding_mode="floor"), slots % page
    if c["bits"] != 4:
        return buf[p, :, r].double()
    raw = buf[p]                                           # [T, Hk, bytes]
    at = torch.arange(d, device=buf.device)
    g, t, e = at // 32, at % 32 // 8, at % 8
    byte = r[:, None] * (d // 2) + t * (d // 8) + 4 * g + e // 2
    q = raw.gather(2, byte[:, None].expand(-1, Hk, -1)) >> (4 * (e % 2)).to(torch.uint8) & 15
    par = raw[..., page * d // 2:].contiguous().view(BF16).view(len(p), Hk, page, d // 32, 2)
    par = par[torch.arange(len(p), device=buf.device), :, r].double()
    return par[..., 0][..., g] + q.double() * par[..., 1][..., g]


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    H, Hk, d, n, lens = c["H"], c["Hk"], c["d"], c["n"], _lengths(c)
    dev, G = st["Q"].device, H // Hk
    if work(c)["flops"] > 6e12:
        return None
    ends = [sum(lens[:b]) for b in range(len(lens) + 1)]
    if c["kind"] == "prompt":
        Y = torch.zeros(ends[-1], H, d, dtype=torch.float64, device=dev)
        L = torch.zeros(ends[-1], H, dtype=torch.float64, device=dev)
        for b in range(c["B"]):
            part = slice(ends[b], ends[b + 1])
            for h in range(H):
                q, k, v = (st[x][part, y].double() for x, y in (("Q", h), ("K", h // G), ("V", h // G)))
                Y[part, h], L[part, h] = _one_head(q, k, v, 0 if c["causal"] else None, _scale(c))
        return Y, L
    dt = st["Q"].dtype
    if c["kind"] in ("append", "step"):
        turned = [st["Q"].double(), st["K"].double()]
        if c["rot"]:
            cos, sin = st["cos"][st["pos"].long()], st["sin"][st["pos"].long()]
            turned = [_turn64(st[x], cos, sin, c["rot"], c["adjacent"], dt) for x in ("Q", "K")]
        Q, new = turned[0], [_stored64(turned[1], c["bits"]), _stored64(st["V"].double(), c["bits"])]
        if c["kind"] == "append":
            return (Q, *(x.to(dt).double() for x in new))
    else:
        Q, new = st["Q"].double(), None
    Y = torch.zeros(c["B"] * n, H, d, dtype=torch.float64, device=dev)
    L = torch.zeros(c["B"] * n, H, dtype=torch.float64, device=dev)
    for b, x in enumerate(lens):
        at = torch.arange(x, device=dev)
        slots = st["table"][b, at // c["page"]].long() * c["page"] + at % c["page"]
        part = slice(b * n, (b + 1) * n)
        kv = []
        for i, name in enumerate(("keys", "values")):
            parts = [_held64(st[name], s, c) for s in slots.split(2048)]
            rows = torch.cat(parts)
            if new is not None:
                rows[x - n:] = new[i][part]
            kv.append(rows.to(dt).double() if c["kind"] == "prefix" else rows)
        for h in range(H):
            y, l = _one_head(Q[part, h], kv[0][:, h // G], kv[1][:, h // G], x - n, _scale(c))
            Y[part, h], L[part, h] = y, l
    return (Q, Y, L) if c["kind"] == "step" else (Y, L)
