"""The 4-bit key / value cache: writing rows into it, reading them back, attention over it; each in its plain form and as the framework's
call, with the cases they are measured on.

Three kinds of case:
  append  new keys and values [B, rows, Hkv, D] -> (keys turned by their positions) 4-bit codes with a scale and a zero point per group, in pages;
          the answer is the values that then stand in the cache
  read    positions of a paged cache -> the values that they stand for
  attend  query rows [B, rows, H, D] of a draft step, a verification pass or a tree over the cached positions they see

Storage of the cache, [n_pages][Hkv][page / 16] tiles of 16 tokens, each: 16 x D / 2 bytes of keys, token by token: byte t * D / 8 + 4 j + i / 2 of a
token holds dimension 32 j + 8 t + i (i = 0..7, low nibble first); as many bytes of values: word ((w * 8 + g) * 4 + t) * 4 + 2 h + e holds token
8 h + 2 t + e, dimension 64 w + 8 i + g at nibble i; [group][token] scale words (key's bf16 low, value's high); [group][token] zero points of the
keys, then of the values, a byte each.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of the tiny configuration (4 heads of 64): all latency
        dict(name="append tiny step", op="append", B=1, rows=1, Hkv=4, D=64, group=32, page=16, at=37, ragged=False, a="f32", rope=True),
        # a verification round of the batch mode at the 13B shape: eight sequences, one draft each
        dict(name="append 13b batch round", op="append", B=8, rows=2, Hkv=40, D=128, group=64, page=16, at=1055, ragged=False, a="f32", rope=True),
        # four prompts of unlike lengths at the 70B shape, as a prompt pass leaves its keys and values
        dict(name="append 70b prompts", op="append", B=4, rows=2047, Hkv=8, D=128, group=128, page=64, at=0, ragged=True, a="bf16", rope=True),
        # a short text of the tiny configuration, read back
        dict(name="read tiny", op="read", B=1, ctx=101, Hkv=4, D=64, group=64, page=16, out="f32"),
        # two long contexts handed to a step that wants 16 bits
        dict(name="read 70b long", op="read", B=2, ctx=16385, Hkv=8, D=128, group=32, page=128, out="bf16"),
        # draft step of the tiny configuration: all latency
        dict(name="attend tiny step", op="attend", B=1, rows=1, H=4, Hkv=4, D=64, group=32, page=16, ctx=101, ragged=False, a="f32", rope=True, tree=False),
        # verification pass after four drafts at the 13B shape, the benchmark's context
        dict(name="attend 13b verify m5", op="attend", B=1, rows=5, H=40, Hkv=40, D=128, group=64, page=16, ctx=1056, ragged=False, a="f32", rope=True, tree=False),
        # draft step at the 70B shape over a longer text
        dict(name="attend 70b draft step", op="attend", B=1, rows=1, H=64, Hkv=8, D=128, group=128, page=16, ctx=4097, ragged=False, a="f32", rope=True, tree=False),
        # tree verification: a chain of six with a sibling each, at the 13B shape
        dict(name="attend 13b tree m13", op="attend", B=1, rows=13, H=40, Hkv=40, D=128, group=32, page=64, ctx=2000, ragged=False, a="f32", rope=True, tree=True),
        # batch round: eight sequences of unlike lengths, one draft each
        dict(name="attend 70b batch round", op="attend", B=8, rows=2, H=64, Hkv=8, D=128, group=64, page=16, ctx=8191, ragged=True, a="bf16", rope=True, tree=False),
        # one draft step of a large batch
        dict(name="attend 70b batch of 32", op="attend", B=32, rows=1, H=64, Hkv=8, D=128, group=128, page=64, ctx=8192, ragged=True, a="bf16", rope=False, tree=False),
        # verification pass after four drafts over a very long text
        dict(name="attend 70b long m5", op="attend", B=1, rows=5, H=64, Hkv=8, D=128, group=64, page=128, ctx=130001, ragged=False, a="f32", rope=True, tree=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    D = rng.choice([64, 128, 128])
    c = dict(op=op, D=D, group=rng.choice([g for g in (32, 64, 128) if g <= D]), page=rng.choice([16, 32, 64, 128]), B=_log(rng, 1, 32), Hkv=rng.choice([1, 2, 4, 5, 8, 8, 40]))
    if op == "append":
        c["rows"] = rng.choice([rng.randint(1, 16), _log(rng, 1, 2048)])
        while c["B"] * c["rows"] * c["Hkv"] * D > 4 * 2047 * 8 * 128:
            c["rows"] = (c["rows"] + 1) // 2
        return dict(c, at=rng.choice([0, _log(rng, 1, 4000)]), ragged=rng.random() < 0.5, a=rng.choice(["f32", "bf16"]), rope=rng.random() < 0.7)
    c["ctx"] = _log(rng, 1, 130000)
    if op == "read":
        while c["B"] * c["ctx"] * c["Hkv"] * D > 2 * 16385 * 8 * 128:
            c["ctx"] = (c["ctx"] + 1) // 2
        return dict(c, out=rng.choice(["f32", "bf16"]))
    rows, heads = rng.choice([1, 1, rng.randint(2, 6), rng.randint(1, 16)]), rng.choice([1, 1, 2, 4, 8, 8, 7])
    while c["Hkv"] * heads > 64:
        heads = (heads + 1) // 2
    while c["B"] * c["ctx"] * c["Hkv"] > 130001 * 8 or c["B"] * c["ctx"] * c["Hkv"] * heads * rows > 130001 * 64 * 5:
        c["ctx"] = (c["ctx"] + 1) // 2
        if c["ctx"] == 1:
            c["B"] = (c["B"] + 1) // 2
    return dict(c, rows=rows, H=c["Hkv"] * heads, ragged=rng.random() < 0.5, a=rng.choice(["f32", "f32", "bf16"]), rope=rng.random() < 0.6, tree=rows > 1 and rng.random() < 0.3)


def _lengths(case):
    """Tokens of each sequence (append: rows of each): the first has all of them, the others, where they are ragged, some share."""
    n = case["rows"] if case["op"] == "append" else case["ctx"]
    if not case.get("ragged"):
        return [n] * case["B"]
    return [n] + [max(1, int(n * (0.25 + 0.75 * (b * 0.6180339887 % 1)))) for b in range(1, case["B"])]


def work(case):
    c = case
    D, Hkv, tokens = c["D"], c["Hkv"], sum(_lengths(c))
    packed = tokens * Hkv * 2 * (D // 2 + 3 * (D // c["group"]))
    if c["op"] == "append":
        return {"bytes": packed + tokens * Hkv * 2 * D * (4 if c["a"] == "f32" else 2), "flops": 8 * tokens * Hkv * D}
    if c["op"] == "read":
        return {"bytes": packed + tokens * Hkv * 2 * D * (4 if c["out"] == "f32" else 2), "flops": 4 * tokens * Hkv * D}
    return {"bytes": packed + 2 * c["B"] * c["rows"] * c["H"] * D * (4 if c["a"] == "f32" else 2), "flops": 4 * tokens * c["H"] * c["rows"] * D}


# ------------------------------------------------------------------------------------------------ inputs
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _tokens(g, dev, B, n, Hkv, D):
    """Keys and values as models have them: some channels of the keys carry an offset and more spread, values are near normal."""
    k = torch.randn(B, n, Hkv, D, generator=g, device=dev)
    loud = (torch.rand(1, 1, Hkv, D, generator=g, device=dev) < 0.06).float()
    k = k * (1 + 2 * loud) + 3 * loud * torch.randn(1, 1, Hkv, D, generator=g, device=dev)
    v = torch.randn(B, n, Hkv, D, generator=g, device=dev) * torch.exp(0.3 * torch.randn(B, n, Hkv, 1, generator=g, device=dev))
    return k, v


def _tile_bytes(case):
    return 16 * case["D"] + 96 * (case["D"] // case["group"])


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    c = case
    B, D, Hkv, T = c["B"], c["D"], c["Hkv"], c["page"]
    lengths = _lengths(c)
    most = (c["at"] + c["rows"] if c["op"] == "append" else c["ctx"])
    P = -(-most // T)
    n_pages = B * P + 3
    st = dict(case=c, n_pages=n_pages)
    st["table"] = torch.randperm(n_pages, generator=g, device=dev)[:B * P].to(torch.int32).view(B, P)  # pages of a sequence lie anywhere in the pool
    st["pool"] = torch.zeros(n_pages * Hkv * (T // 16) * _tile_bytes(c), dtype=torch.uint8, device=dev)
    st["rope"] = None
    if c.get("rope"):
        turn = torch.arange(most, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device=dev, dtype=torch.float64) / D)
        st["rope"] = torch.stack([turn.cos(), turn.sin()], -1).float()
    if c["op"] == "append":
        k, v = _tokens(g, dev, B, c["rows"], Hkv, D)
        st["k"], st["v"] = k.to(_TYPES[c["a"]]), v.to(_TYPES[c["a"]])
        st["start"] = torch.full((B,), c["at"], dtype=torch.int32, device=dev)
        st["n_rows"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        st["n_ctx"] = st["start"] + st["n_rows"]
    else:
        # the cache as earlier steps left it
        k, v = _tokens(g, dev, B, P * T, Hkv, D)
        tiles = st["pool"].view(n_pages, Hkv, T // 16, -1)
        tiles[st["table"].view(-1).long()] = _pack(k, v, c).view(B, P, T // 16, Hkv, -1).transpose(2, 3).reshape(B * P, Hkv, T // 16, -1)
        del k, v
        st["n_ctx"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
    if c["op"] == "attend":
        R = c["rows"]
        st["q"] = (torch.randn(B, R, c["H"], D, generator=g, device=dev) * 1.2).to(_TYPES[c["a"]])
        st["visible"] = st["positions"] = None
        if c["tree"]:  # a chain (rows 0, 1, 3, 5, ..) with a sibling of each of its later rows (2, 4, 6, ..)
            m = torch.arange(R, device=dev)
            chain = (m[:, None] >= m) & ((m % 2 == 1) | (m == 0))
            on = torch.where(((m % 2 == 1) | (m == 0))[:, None], chain, (chain & (m < m[:, None] - 1)) | (m == m[:, None]))
            st["visible"] = (on.long() << m).sum(-1).to(torch.int32)[None].expand(B, R).contiguous()
            st["positions"] = (st["n_ctx"][:, None] - R + ((m + 1) // 2)[None]).clamp(min=0).to(torch.int32).contiguous()
    if own:
        import paper_2406_03853_b200 as eesd
        st["cache"] = eesd.KV4Cache(n_pages, Hkv, D, page_tokens=T, group=c["group"], buffer=st["pool"])
    return st


def _quantize(w, group):
    """[.., D] fp32 -> codes (float), scales bf16, zero points; a value next to a rounding border needs 64 bits"""
    w = w.unflatten(-1, (-1, group)).double()
    lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
    s = _to_bf16((hi - lo) / 15)
    d = torch.where(s > 0, s.double(), 1.0)
    z = torch.round(-lo / d).clamp(0, 15)
    return ((w / d[..., None]).round_() + z[..., None]).clamp_(0, 15).float(), s, z.float()


def _to_bf16(x):
    """float64 >= 0 -> bf16, rounded once to nearest even"""
    f = x.float()
    down = torch.where(f.double() > x, f.view(torch.int32) - 1, f.view(torch.int32))
    odd = torch.where(down.view(torch.float32).double() != x, down | 1, down)  # to odd first, so that the second rounding sees which side the rest lies on
    return odd.view(torch.float32).to(torch.bfloat16)


def _pack(k, v, case):
    """[B, n, Hkv, D] keys and values, n whole tiles -> bytes [B, n / 16, Hkv, tile] (fp32 quotients do here: this makes inputs)"""
    B, n, Hkv, D = k.shape
    W, J, G = D // 64, D // 32, D // case["group"]

    def codes(x):
        x = x.unflatten(-1, (G, -1))
        lo, hi = x.amin(-1).clamp_(max=0), x.amax(-1).clamp_(min=0)
        s = ((hi - lo) / 15).to(torch.bfloat16)
        z = (-lo / s.float()).round_().clamp_(0, 15)
        return ((x / s.float()[..., None]).round_() + z[..., None]).clamp_(0, 15).to(torch.uint8).flatten(-2), s.view(torch.int16), z.to(torch.uint8)

    def by_tile(x):  # [B, n, Hkv, G, ..] -> [B, n / 16, Hkv, G, 16]
        return x.unflatten(1, (-1, 16)).permute(0, 1, 3, 4, 2)

    ck, sk, zk = codes(k)
    ck = ck.view(B, n // 16, 16, Hkv, J, 4, 8).permute(0, 1, 3, 2, 5, 4, 6)
    ck = (ck[..., ::2] | ck[..., 1::2] << 4).reshape(B, n // 16, Hkv, -1)
    cv, sv, zv = codes(v)
    cv = cv.view(B, n // 16, 2, 4, 2, Hkv, W, 8, 8).permute(0, 1, 5, 6, 8, 3, 2, 4, 7)  # h t e Hkv w i g -> Hkv w g t h e i
    cv = (cv[..., ::2] | cv[..., 1::2] << 4).reshape(B, n // 16, Hkv, -1)
    scales = torch.stack([by_tile(sk), by_tile(sv)], -1).contiguous().view(torch.uint8).reshape(B, n // 16, Hkv, -1)
    return torch.cat([ck, cv, scales, by_tile(zk).reshape(B, n // 16, Hkv, -1), by_tile(zv).reshape(B, n // 16, Hkv, -1)], -1)


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return {"append": _append, "read": _read, "attend": _attend}[state["case"]["op"]](state)


def _append(st):
    c = st["case"]
    if own:
        cache = st["cache"]
        cache.append(st["k"], st["v"], st["table"], st["start"], n_rows=st["n_rows"], rope=st["rope"])
        k, v = cache.read(st["table"], c["rows"], start=st["start"], n_ctx=st["n_ctx"])
        return {"k": k, "v": v}
    k, v = st["k"].float(), st["v"].float()
    at = st["start"][:, None] + torch.arange(c["rows"], device=k.device)
    if st["rope"] is not None:
        k = _turn(k, st["rope"], at)
    there = (at < st["n_ctx"][:, None])[..., None, None]

    def held(x):
        q, s, z = _quantize(x, c["group"])
        return torch.where(there, ((q - z[..., None]) * s.float()[..., None]).flatten(-2), 0.0)

    return {"k": held(k), "v": held(v)}


def _turn(x, rope, at):
    """Pairs (2 i, 2 i + 1) of [B, rows, heads, D] turned by their rows' angles; each product and each sum is rounded to fp32"""
    cos, sin = rope[at.long()].unbind(-1)
    cos, sin = cos[:, :, None], sin[:, :, None]
    a, b = x[..., ::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _values(st):
    """keys and values of all positions, fp32 [B, Hkv, n, D]"""
    c = st["case"]
    B, D, Hkv, T = c["B"], c["D"], c["Hkv"], c["page"]
    G, half = D // c["group"], 8 * D
    t = st["pool"].view(st["n_pages"], Hkv, T // 16, -1)[st["table"].long()].transpose(1, 2).reshape(B, Hkv, -1, _tile_bytes(c))  # [B, Hkv, tiles, bytes]

    def nibbles(x):
        return torch.stack([x & 15, x >> 4], -1).flatten(-2)

    k = nibbles(t[..., :half]).unflatten(-1, (16, 4, D // 32, 8)).transpose(-3, -2).reshape(B, Hkv, -1, G, c["group"])
    v = nibbles(t[..., half:2 * half]).unflatten(-1, (D // 64, 8, 4, 2, 2, 8)).permute(0, 1, 2, 6, 5, 7, 3, 8, 4).reshape(B, Hkv, -1, G, c["group"])
    meta = t[..., 2 * half:].contiguous()
    s = meta[..., :64 * G].contiguous().view(torch.bfloat16).unflatten(-1, (G, 16, 2)).transpose(-3, -2).reshape(B, Hkv, -1, G, 2).float()
    z = meta[..., 64 * G:].unflatten(-1, (2, G, 16)).permute(0, 1, 2, 5, 4, 3).reshape(B, Hkv, -1, G, 2).float()
    return [((x - z[..., i, None]) * s[..., i, None]).flatten(-2) for i, x in enumerate((k, v))]


def _read(st):
    c = st["case"]
    if own:
        k, v = st["cache"].read(st["table"], c["ctx"], n_ctx=st["n_ctx"], dtype=_TYPES[c["out"]])
        return {"k": k, "v": v}
    k, v = (x[:, :, :c["ctx"]].transpose(1, 2).to(_TYPES[c["out"]]).contiguous() for x in _values(st))
    return {"k": k, "v": v}


def _attend(st):
    c = st["case"]
    if own:
        import paper_2406_03853_b200 as eesd
        return eesd.attend_rows(st["q"], st["cache"], st["table"], st["n_ctx"], visible=st["visible"], rope=st["rope"], positions=st["positions"])
    B, R, H, D, Hkv = c["B"], c["rows"], c["H"], c["D"], c["Hkv"]
    q = st["q"].float()
    n = st["n_ctx"].long()
    old = n[:, None] - R  # positions before the new rows
    m = torch.arange(R, device=q.device)
    if st["rope"] is not None:
        q = _turn(q, st["rope"], (old + m).clamp(min=0) if st["positions"] is None else st["positions"])
    k, v = _values(st)
    p = torch.arange(k.shape[2], device=q.device)
    if st["visible"] is None:
        seen = p <= (old + m)[..., None]
    else:
        new = p - old[..., None]
        seen = (new < 0) | ((st["visible"].long()[..., None] >> new.clamp(0, 31) & 1).bool() & (new < R))
    seen = seen[:, None, :, None]  # [B, 1, R, 1, n]
    q = q.view(B, R, Hkv, H // Hkv, D).transpose(1, 2).reshape(B, Hkv, -1, D)
    x = (q @ k.transpose(-1, -2)).view(B, Hkv, R, H // Hkv, -1) * D ** -0.5
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
    total = e.sum(-1, keepdim=True)
    out = (e.view(B, Hkv, -1, e.shape[-1]) @ v).view(B, Hkv, R, H // Hkv, D) / torch.where(total > 0, total, 1.0)
    return out.transpose(1, 2).reshape(B, R, H, D).to(st["q"].dtype)


# ------------------------------------------------------------------------------------------------ exact values
def exact(case, seed):
    """From the definition in 64 bits: every stored value by its own byte, sequence by sequence and head by head."""
    st = prepare(case, seed)
    c = case
    B, D, Hkv = c["B"], c["D"], c["Hkv"]
    if c["op"] == "append":
        return _exact_append(st)
    if c["op"] == "read":
        out = {n: torch.zeros(B, c["ctx"], Hkv, D, dtype=torch.float64, device="cuda") for n in "kv"}
        for b in range(B):
            for h in range(Hkv):
                out["k"][b, :, h], out["v"][b, :, h] = _exact_values(st, b, h, c["ctx"])
        return out
    R, share = c["rows"], c["H"] // Hkv
    out = torch.zeros(B, R, c["H"], D, dtype=torch.float64, device="cuda")
    for b in range(B):
        L = int(st["n_ctx"][b])
        for h in range(Hkv):
            k, v = _exact_values(st, b, h, L)
            for m in range(R):
                at = L - R + m
                seen = torch.arange(L, device="cuda") <= at
                if st["visible"] is not None:
                    bits = int(st["visible"][b, m])
                    seen = torch.tensor([p < L - R or bits >> (p - L + R) & 1 == 1 for p in range(max(0, L - 40), L)], device="cuda")
                    seen = torch.cat([torch.ones(L - len(seen), dtype=torch.bool, device="cuda"), seen])
                    at = int(st["positions"][b, m])
                if not bool(seen.any()):
                    continue
                q = st["q"][b, m, h * share:(h + 1) * share]
                if st["rope"] is not None:
                    q = _exact_turn(q, st["rope"][max(at, 0)])
                w = torch.softmax((q.double() @ k[seen].t()) / math.sqrt(D), -1)
                out[b, m, h * share:(h + 1) * share] = w @ v[seen]
    return out


def _exact_turn(x, angles):
    """x [.., D], angles [D / 2, 2] (or with leading axes): products and sums rounded to fp32, as the definition has them"""
    c, s = angles[..., 0].double(), angles[..., 1].double()
    x = x.double()
    r = torch.empty_like(x)
    r[..., 0::2] = (x[..., 0::2] * c).float().double() - (x[..., 1::2] * s).float().double()
    r[..., 1::2] = (x[..., 0::2] * s).float().double() + (x[..., 1::2] * c).float().double()
    return r.float()


def _exact_values(st, b, h, n):
    c = st["case"]
    D, T, G = c["D"], c["page"], c["D"] // c["group"]
    size = _tile_bytes(c)
    p, d = torch.arange(n, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    tile = (st["table"][b][p // T].long() * c["Hkv"] + h) * (T // 16) + p % T // 16
    t, pool = p % 16, st["pool"]
    scale_words = pool.view(torch.int32)
    found = []
    for which in range(2):
        if which == 0:
            at, nib = t * (D // 2) + d % 32 // 8 * (D // 8) + d // 32 * 4 + d % 8 // 2, d % 2
        else:
            at, nib = 8 * D + (((d // 64 * 8 + d % 8) * 4 + t % 8 // 2) * 4 + t // 8 * 2 + t % 2) * 4 + d % 64 // 16, d % 16 // 8
        code = pool[tile * size + at].long() >> 4 * nib & 15
        zero = pool[tile * size + 16 * D + 64 * G + (which * G + d // c["group"]) * 16 + t].long()
        word = scale_words[(tile * size + 16 * D) // 4 + d // c["group"] * 16 + t]
        scale = ((word << 16) if which == 0 else (word & -65536)).view(torch.float32).double()
        found.append((code - zero).double() * scale)
    return found


def _exact_append(st):
    c = st["case"]
    out = {}
    for name in "kv":
        x = st[name]
        if name == "k" and st["rope"] is not None:
            x = _exact_turn(x, st["rope"][c["at"]:c["at"] + c["rows"]][None, :, None])
        x = x.double()
        y = torch.empty_like(x)
        for a in range(0, c["D"], c["group"]):
            w = x[..., a:a + c["group"]]
            lo = torch.minimum(w.min(-1).values, torch.zeros((), device="cuda", dtype=torch.float64))
            hi = torch.maximum(w.max(-1).values, torch.zeros((), device="cuda", dtype=torch.float64))
            frac, power = torch.frexp((hi - lo) / 15)
            s = torch.ldexp(torch.round(frac * 256), power - 8)
            safe = s.clamp(min=1e-300)
            z = torch.round(-lo / safe).clamp(0, 15)
            y[..., a:a + c["group"]] = ((torch.round(w / safe[..., None]) + z[..., None]).clamp(0, 15) - z[..., None]) * s[..., None]
        for b, n in enumerate(_lengths(c)):
            y[b, n:] = 0
        out[name] = y
    return out
