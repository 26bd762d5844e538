"""The 4-bit projections and the logit rules, each in its plain form and as the framework's call, with the cases they are measured on.

Three kinds of case:
  quantize  weights [R, K] -> 4-bit codes with a scale (and a zero point) per group of K-neighbours, and the values they stand for
  project   M token rows [M, K] times a 4-bit matrix [R, K]^T (the skinny projection of a decode or verification pass)
  logits    repetition / frequency / presence penalties, biases and a grammar mask on the logit rows of a decode or verification round
"""
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # gate rows of the tiny configuration (d 256, F 688): one small matrix, latency counts
        dict(name="quantize tiny ffn", op="quantize", R=688, K=256, group=32, w="f32", scale="f32", zero=False),
        # a ragged matrix: neither dimension fits a tile, the last group is short
        dict(name="quantize ragged", op="quantize", R=1025, K=1000, group=64, w="bf16", scale="bf16", zero=True),
        # the down projection of the 13B shape, as a user quantises a model layer by layer
        dict(name="quantize 13b down", op="quantize", R=5120, K=13824, group=128, w="bf16", scale="bf16", zero=False),
        # vocabulary head of the tiny configuration for one draft row: all latency
        dict(name="project tiny head m1", op="project", M=1, R=1024, K=256, group=32, a="f32", scale="f32", zero=False),
        # QKV of a 13B draft step: one row
        dict(name="project 13b qkv m1", op="project", M=1, R=15360, K=5120, group=128, a="f32", scale="bf16", zero=False),
        # gate and up of a 13B verification pass after four drafts
        dict(name="project 13b gate up m5", op="project", M=5, R=27648, K=5120, group=64, a="f32", scale="bf16", zero=True),
        # down projection of a full pass at the 70B shape: the longest sums, the most rows
        dict(name="project 70b down m16", op="project", M=16, R=8192, K=28672, group=128, a="f32", scale="bf16", zero=True),
        # ragged shape with bf16 rows and the smallest groups
        dict(name="project ragged m11", op="project", M=11, R=4099, K=5000, group=32, a="bf16", scale="f32", zero=False),
        # one draft step of one sequence: penalties over a 512-token prompt and some output, no mask
        dict(name="logits draft step", op="logits", B=1, rows=1, V=32000, pad=0, history=600, prompt=512, bias=16, mask=False, penalties=True),
        # a verification round of the batch mode: eight sequences, one draft each, everything on
        dict(name="logits batch round", op="logits", B=8, rows=2, V=32000, pad=0, history=1024, prompt=512, bias=64, mask=True, penalties=True),
        # a wider odd vocabulary, biases and grammar mask only (constrained decoding without penalties)
        dict(name="logits odd vocabulary", op="logits", B=16, rows=5, V=50257, pad=0, history=0, prompt=0, bias=300, mask=True, penalties=False),
        # the largest acceptance round of the sweep: 64 sequences, 16 drafts each
        dict(name="logits sweep", op="logits", B=64, rows=17, V=32000, pad=0, history=2048, prompt=1024, bias=64, mask=True, penalties=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "project", "project", "logits", "logits"])
    if op == "quantize":
        R, K = _log(rng, 16, 16000), _log(rng, 32, 30000)
        while R * K > 5120 * 13824:
            R, K = (R + 1) // 2, K
        return dict(op=op, R=R, K=K, group=rng.choice([32, 64, 128]), w=rng.choice(["f32", "bf16"]), scale=rng.choice(["f32", "bf16"]), zero=rng.random() < 0.5)
    if op == "project":
        R, K = _log(rng, 64, 60000), _log(rng, 128, 30000)
        if rng.random() < 0.6:  # most models' widths are whole tiles
            R, K = max(128, R // 128 * 128), max(128, K // 128 * 128)
        while R * K > 8192 * 28672:
            R = (R + 1) // 2
        return dict(op=op, M=rng.randint(1, 16), R=R, K=K, group=rng.choice([32, 64, 128]), a=rng.choice(["f32", "f32", "bf16"]),
                    scale=rng.choice(["f32", "bf16"]), zero=rng.random() < 0.5)
    B, rows, V = _log(rng, 1, 64), rng.randint(1, 17), _log(rng, 1000, 130000)
    if rng.random() < 0.5:
        V = max(1024, V // 128 * 128)
    while B * rows * V > 64 * 17 * 32000:
        B = (B + 1) // 2
    history = rng.choice([0, _log(rng, 1, 4096), _log(rng, 64, 4096)])
    penalties = rng.random() < 0.7
    return dict(op=op, B=B, rows=rows, V=V, pad=rng.choice([0, 0, (-V) % 64, 3]), history=history, prompt=rng.randint(0, history),
                bias=rng.choice([0, _log(rng, 1, 1000)]), mask=not penalties or rng.random() < 0.6, penalties=penalties)


def work(case):
    c = case
    if c["op"] == "logits":
        n = c["B"] * c["rows"] * c["V"]
        b = 8 * n + (n // 8 if c["mask"] else 0) + 8 * c["B"] * c["bias"] + (4 * c["B"] * (c["history"] + c["rows"] - 1) if c["penalties"] else 0)
        return {"bytes": b, "flops": n * (4 if c["penalties"] else 1)}
    R, K = c["R"], c["K"]
    groups = -(-K // c["group"])
    packed = R * K / 2 + R * groups * ((4 if c["scale"] == "f32" else 2) + (0.5 if c["zero"] else 0))
    if c["op"] == "quantize":
        return {"bytes": packed + R * K * ((4 if c["w"] == "f32" else 2) + 4), "flops": 4 * R * K}
    return {"bytes": packed + c["M"] * K * (4 if c["a"] == "f32" else 2) + 4 * c["M"] * R, "flops": 2 * c["M"] * R * K}


# ------------------------------------------------------------------------------------------------ inputs
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _weights(case, g, device):
    """Projection weights as models have them: near normal, a spread of sizes over the rows, a few large columns."""
    R, K = case["R"], case["K"]
    w = torch.randn(R, K, generator=g, device=device, dtype=torch.float32)
    w *= 0.02 * torch.exp(0.3 * torch.randn(R, 1, generator=g, device=device))
    w *= 1 + 4 * (torch.rand(1, K, generator=g, device=device) < 0.005)
    return w


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    c = case
    st = dict(case=c)
    if c["op"] == "quantize":
        st["w"] = _weights(c, g, dev).to(_TYPES[c["w"]])
    elif c["op"] == "project":
        R, K, G = c["R"], c["K"], -(-c["K"] // c["group"])
        # codes and scales as they come with a quantised model
        st["codes"] = (torch.randn(R, K, generator=g, device=dev) * 2.6 + 7.7).round_().clamp_(0, 15).to(torch.uint8)
        st["scales"] = (0.006 * torch.exp(0.4 * torch.randn(R, G, generator=g, device=dev))).to(_TYPES[c["scale"]])
        st["zeros"] = (7.5 + 1.5 * torch.randn(R, G, generator=g, device=dev)).round_().clamp_(0, 15).to(torch.uint8) if c["zero"] else None
        a = torch.randn(c["M"], K, generator=g, device=dev) * (1 + 20 * (torch.rand(1, K, generator=g, device=dev) < 0.002))  # normalised rows with outliers
        st["a"] = a.to(_TYPES[c["a"]])
        if own:
            import paper_2406_03853_b200 as eesd
            st["w4"] = eesd.W4Matrix.from_codes(st["codes"], st["scales"], st["zeros"], group=c["group"])
    else:
        B, rows, V, H = c["B"], c["rows"], c["V"], c["history"]
        full = torch.randn(B, rows, V + c["pad"], generator=g, device=dev) * 3
        st["logits"] = full[:, :, :V]

        def tokens(*shape):  # texts repeat themselves: low ids more often
            u = torch.rand(*shape, generator=g, device=dev)
            return (u * u * u * V).to(torch.int32).clamp_(max=V - 1)

        st["history"] = st["drafted"] = None
        if c["penalties"]:
            st["repetition"] = 1 + 0.3 * torch.rand(B, generator=g, device=dev)
            st["frequency"] = 0.5 * torch.rand(B, generator=g, device=dev)
            st["presence"] = 0.5 * torch.rand(B, generator=g, device=dev)
            if H:
                st["history"] = tokens(B, H)
                # sequences are of unlike lengths; the prompt of each comes first
                n = H - (torch.rand(B, generator=g, device=dev) * 0.3 * H).to(torch.int32)
                st["n_history"] = n
                st["n_prompt"] = torch.minimum(n, torch.full_like(n, c["prompt"]))
            if rows > 1:
                st["drafted"] = tokens(B, rows - 1)
        st["bias_start"] = None
        if c["bias"]:
            st["bias_start"] = torch.arange(B + 1, device=dev, dtype=torch.int32) * c["bias"]
            st["bias_ids"] = tokens(B * c["bias"])
            st["bias_values"] = 4 * torch.randn(B * c["bias"], generator=g, device=dev)
        st["mask"] = None
        if c["mask"]:  # a grammar allows anything from a handful of tokens to most of them
            words = -(-V // 32)
            keep = torch.rand(B, rows, 1, generator=g, device=dev)
            bits = (torch.rand(B, rows, words * 32, generator=g, device=dev) < keep).view(B, rows, words, 32)
            st["mask"] = (bits.to(torch.int64) << torch.arange(32, device=dev)).sum(-1).to(torch.int32)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if c["op"] == "quantize":
        return _quantize_own(state) if own else _quantize_plain(state)
    if c["op"] == "project":
        return _project_own(state) if own else _project_plain(state)
    return _logits_own(state) if own else _logits_plain(state)


def _quantize_own(st):
    import paper_2406_03853_b200 as eesd
    c = st["case"]
    m = eesd.W4Matrix.quantize(st["w"], group=c["group"], scale_dtype=_TYPES[c["scale"]], zero_point=c["zero"])
    return {"values": m.dense(), "scales": m.scales()}


def _project_own(st):
    import paper_2406_03853_b200 as eesd
    return eesd.project_rows(st["a"], st["w4"])


def _logits_own(st):
    import paper_2406_03853_b200 as eesd
    keys = ("history", "n_history", "n_prompt", "drafted", "repetition", "frequency", "presence", "bias_start", "bias_ids", "bias_values", "mask")
    return eesd.process_logits(st["logits"], eesd.LogitRules(**{k: st[k] for k in keys if st.get(k) is not None}))


def _quantize_plain(st):
    c = st["case"]
    R, K, g = c["R"], c["K"], c["group"]
    G = -(-K // g)
    w = torch.nn.functional.pad(st["w"].double(), (0, G * g - K)).view(R, G, g)  # a value next to a rounding border needs 64 bits
    if c["zero"]:
        lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
        s = _to_scale((hi - lo) / 15, c["scale"])
        d = torch.where(s > 0, s.double(), 1.0)
        z = torch.round(-lo / d).clamp(0, 15)
        q = (torch.round(w / d[..., None]) + z[..., None]).clamp(0, 15) - z[..., None]
    else:
        s = _to_scale(w.abs().amax(-1) / 7, c["scale"])
        d = torch.where(s > 0, s.double(), 1.0)
        q = torch.round(w / d[..., None]).clamp(-8, 7)
    v = q.float() * s.float()[..., None]
    return {"values": v.view(R, G * g)[:, :K].contiguous(), "scales": s}


def _to_scale(x, kind):
    """float64 -> f32 or bf16, rounded once to nearest even"""
    if kind == "f32":
        return x.float()
    f = x.float()
    odd = f.view(torch.int32)  # round to odd in 32 bits first, so that the second rounding sees which side the rest lies on
    down = torch.where(f.double() > x, odd - 1, odd)  # towards zero (x >= 0)
    odd = torch.where(down.view(torch.float32).double() != x, down | 1, down)
    return odd.view(torch.float32).to(torch.bfloat16)


def _project_plain(st):
    c = st["case"]
    g = c["group"]
    z = 8.0 if st["zeros"] is None else st["zeros"].float().repeat_interleave(g, 1)[:, :c["K"]]
    w = (st["codes"].float() - z) * st["scales"].float().repeat_interleave(g, 1)[:, :c["K"]]
    return st["a"].float() @ w.t()


def _logits_plain(st):
    c = st["case"]
    l = st["logits"]
    B, rows, V = l.shape
    if c["penalties"]:
        count = torch.zeros(B, rows, V, device=l.device, dtype=torch.int32)
        prompt = torch.zeros(B, V, device=l.device, dtype=torch.int32)
        if st["history"] is not None:
            h = st["history"].long()
            at = torch.arange(h.shape[1], device=l.device)[None]
            mine = at < st["n_history"][:, None]
            given = at < st["n_prompt"][:, None]
            prompt.scatter_add_(1, h, (mine & given).int())
            count[:, 0].scatter_add_(1, h, (mine & ~given).int())
        if st["drafted"] is not None:
            x = st["drafted"].long()
            count[:, 1:].scatter_add_(2, x[:, :, None], torch.ones_like(x, dtype=torch.int32)[:, :, None])
        count = count.cumsum(1, dtype=torch.int32)
        rep, freq, pres = (st[k][:, None, None] for k in ("repetition", "frequency", "presence"))
        seen = (count > 0) | (prompt > 0)[:, None]
        l = torch.where(seen, torch.where(l > 0, l / rep, l * rep), l)
        l = l - (freq * count.float() + pres * (count > 0).float())
    if st["bias_start"] is not None:
        n = st["bias_ids"].numel()
        b = torch.repeat_interleave(torch.arange(B, device=l.device), n // B)
        last = torch.full((B * V,), -1, device=l.device, dtype=torch.int64)  # an id given twice takes its last value
        last.scatter_reduce_(0, b * V + st["bias_ids"].long(), torch.arange(n, device=l.device), "amax")
        bias = torch.where(last >= 0, st["bias_values"][last.clamp(min=0)], 0.0)
        l = l + bias.view(B, 1, V)
    if st["mask"] is not None:
        bits = (st["mask"][..., None] >> torch.arange(32, device=l.device, dtype=torch.int32)) & 1
        l = torch.where(bits.flatten(2)[..., :V] != 0, l, float("-inf"))
    return l


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    c = case
    if c["op"] == "quantize":
        R, K, g = c["R"], c["K"], c["group"]
        vals, scales = [], []
        for k in range(0, K, g):
            w = st["w"][:, k:k + g].double()
            if c["zero"]:
                lo = torch.minimum(w.min(1).values, torch.zeros((), device=w.device, dtype=w.dtype))
                hi = torch.maximum(w.max(1).values, torch.zeros((), device=w.device, dtype=w.dtype))
                s = _nearest((hi - lo) / 15, c["scale"])
                z = (-lo / s.clamp(min=1e-300)).round()
                q = ((w / s.clamp(min=1e-300)[:, None]).round() + z[:, None]).clamp(0, 15) - z[:, None]
            else:
                s = _nearest(torch.maximum(w.max(1).values, -w.min(1).values) / 7, c["scale"])
                q = (w / s.clamp(min=1e-300)[:, None]).round().clamp(-8, 7)
            vals.append(q * s[:, None])
            scales.append(s)
        return {"values": torch.cat(vals, 1), "scales": torch.stack(scales, 1)}
    if c["op"] == "project":
        out = torch.zeros(c["M"], c["R"], device="cuda", dtype=torch.float64)
        a = st["a"].double()
        for i in range(st["scales"].shape[1]):  # group by group
            k = slice(i * c["group"], min(c["K"], (i + 1) * c["group"]))
            z = 8 if st["zeros"] is None else st["zeros"][:, i:i + 1].double()
            out += (a[:, k] @ (st["codes"][:, k].double() - z).t()) * st["scales"][:, i].double()
        return out
    l = st["logits"].double().cpu().numpy().copy()
    B, rows, V = l.shape
    host = {k: v.cpu().numpy() for k, v in st.items() if isinstance(v, torch.Tensor)}
    for b in range(B):
        bias = np.zeros(V)
        if c["bias"]:
            s = slice(host["bias_start"][b], host["bias_start"][b + 1])
            bias[host["bias_ids"][s]] = host["bias_values"][s]  # numpy: the last of equal indices stays
        text = host["history"][b, :host["n_history"][b]] if "history" in host else np.zeros(0, np.int64)
        split = int(host["n_prompt"][b]) if "history" in host else 0
        for i in range(rows):
            if c["penalties"]:
                gen = np.concatenate([text[split:], host["drafted"][b, :i]]) if "drafted" in host else text[split:]
                n = np.bincount(gen, minlength=V)
                hit = np.unique(np.concatenate([text[:split], gen])).astype(np.int64)
                rho, x = float(host["repetition"][b]), l[b, i, hit]
                l[b, i, hit] = np.where(x > 0, x / rho, x * rho)
                l[b, i] -= float(host["frequency"][b]) * n + float(host["presence"][b]) * (n > 0)
            l[b, i] += bias
            if c["mask"]:
                allowed = np.unpackbits(host["mask"][b, i].view(np.uint8), bitorder="little")[:V]
                l[b, i, allowed == 0] = -np.inf
    return torch.from_numpy(l)


def _nearest(x, kind):
    """The nearest value of the scale's type (ties to even), as float64: by its significand's bits, 24 or 8"""
    m, e = torch.frexp(x)
    p = 24 if kind == "f32" else 8
    return torch.ldexp(torch.round(m * 2.0 ** p), e - p)
