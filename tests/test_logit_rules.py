"""Logit rules (penalties, biases, grammar masks) on the GPU against a plain 64-bit implementation.

Bound per entry: the kernel rounds each operation once to fp32, so it is off by at most 2^-24 of each intermediate
result: |l1|, |frequency n|, |frequency n + presence|, |l2|, |l3|."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b


def rules_ref(l, history=None, n_history=None, n_prompt=None, drafted=None, repetition=None, frequency=None, presence=None, bias=None, mask=None):
    """float64 [B, rows, V] results and the bound of the fp32 ones; arguments are host arrays, bias a list of (id, value) lists"""
    l = l.astype(np.float64)
    B, rows, V = l.shape
    out, bound = np.empty_like(l), np.zeros_like(l)
    for s in range(B):
        text = [] if history is None else list(history[s][:max(0, min(len(history[s]), n_history[s] if n_history is not None else len(history[s])))])
        split = 0 if n_prompt is None else max(0, min(int(n_prompt[s]), len(text)))
        for i in range(rows):
            gen = text[split:] + ([] if drafted is None else list(drafted[s][:i]))
            n = np.zeros(V)
            seen = np.zeros(V, bool)
            for t in gen:
                if 0 <= t < V:
                    n[t] += 1
                    seen[t] = True
            for t in text[:split]:
                if 0 <= t < V:
                    seen[t] = True
            x = l[s, i]
            rho = 1.0 if repetition is None else float(repetition[s])
            l1 = np.where(seen, np.where(x > 0, x / rho, x * rho), x)
            f = (0.0 if frequency is None else float(frequency[s])) * n
            p = f + (0.0 if presence is None else float(presence[s])) * (n > 0)
            l2 = l1 - p
            add = np.zeros(V)
            for t, v in ([] if bias is None else bias[s]):
                if 0 <= t < V:
                    add[t] = v
            l3 = l2 + add
            out[s, i] = l3
            with np.errstate(invalid="ignore"):
                bound[s, i] = 2.0 ** -24 * 1.001 * np.nan_to_num(abs(l1) + abs(f) + abs(p) + abs(l2) + abs(l3), nan=0, posinf=0, neginf=0) + 1e-44
            if mask is not None:
                allowed = np.unpackbits(np.ascontiguousarray(mask[s, i]).view(np.uint8), bitorder="little")[:V] != 0
                out[s, i][~allowed] = -np.inf
    return out, bound


def close(got, want, bound):
    got = got.double().cpu().numpy()
    fin = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    off = np.abs(got[fin] - want[fin])
    assert (off <= bound[fin]).all(), np.max(off / bound[fin])


def make(B, rows, V, H, n_bias, mask, seed, penalties=True):
    g = np.random.default_rng(seed)
    d = dict(l=(g.standard_normal((B, rows, V)) * 3).astype(np.float32))
    kw = {}
    if penalties:
        d["repetition"] = (1 + g.random(B)).astype(np.float32)
        d["frequency"] = (g.random(B) - 0.3).astype(np.float32)
        d["presence"] = (g.random(B) - 0.3).astype(np.float32)
        if H:
            d["history"] = g.integers(-2, V + 2, (B, H)).astype(np.int32)   # a few ids outside the vocabulary
            d["history"][:, ::3] = g.integers(0, min(V, 7), d["history"][:, ::3].shape)
            d["n_history"] = g.integers(-1, H + 2, B).astype(np.int32)
            d["n_prompt"] = g.integers(-1, H + 2, B).astype(np.int32)
        if rows > 1:
            d["drafted"] = g.integers(-1, V + 1, (B, rows - 1)).astype(np.int32)
            d["drafted"][:, 1:] = np.where(g.random((B, rows - 2)) < 0.5, d["drafted"][:, :1], d["drafted"][:, 1:])
    kw = {k: torch.from_numpy(v).cuda() for k, v in d.items() if k != "l"}
    if n_bias:
        lens = g.integers(0, n_bias + 1, B)
        lens[0] = n_bias
        ids = g.integers(-1, V + 1, lens.sum()).astype(np.int32)
        ids[::4] = g.integers(0, V, ids[::4].shape) % 5          # ids given twice
        vals = (4 * g.standard_normal(lens.sum())).astype(np.float32)
        start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        d["bias"] = [list(zip(ids[start[s]:start[s + 1]], vals[start[s]:start[s + 1]])) for s in range(B)]
        kw.update(bias_start=torch.from_numpy(start).cuda(), bias_ids=torch.from_numpy(ids).cuda(), bias_values=torch.from_numpy(vals).cuda())
    if mask:
        words = (V + 31) // 32
        m = g.integers(0, 2 ** 32, (B, rows, words), dtype=np.uint64).astype(np.uint32).view(np.int32)
        m[0, 0] = 0                                              # nothing left
        m[-1, -1] = -1                                           # everything
        d["mask"] = m
        kw["mask"] = torch.from_numpy(m).cuda()
    return d, eesd.LogitRules(**kw)


@pytest.mark.gpu
@pytest.mark.parametrize("B,rows,V", [(1, 1, 1), (1, 1, 31), (2, 3, 32), (3, 2, 33), (1, 17, 1024), (2, 5, 1025), (5, 2, 4100), (1, 1, 32000), (8, 2, 32000),
                                      (3, 4, 50257), (64, 17, 2000), (2, 256, 130), (40, 1, 128256)])
def test_against_64_bits(B, rows, V):
    for i, (H, nb, mask, pen) in enumerate([(0, 0, True, False), (1, 0, False, True), (700, 40, True, True), (5000 if V < 40000 else 600, 0, True, True), (0, 9, False, False), (0, 0, False, True)]):
        d, r = make(B, rows, V, H, nb, mask, 7 * i + V + B, pen)
        logits = torch.from_numpy(d["l"]).cuda()
        want, bound = rules_ref(**d)
        out = eesd.process_logits(logits, r)
        close(out, want, bound)
        assert torch.equal(logits.cpu(), torch.from_numpy(d["l"]))
        again = eesd.process_logits(logits, r, out=logits)       # in place
        assert again.data_ptr() == logits.data_ptr() and torch.equal(again.view(torch.int32), out.view(torch.int32))


@pytest.mark.gpu
def test_strides_alignment_and_untouched_padding():
    B, rows, V = 3, 4, 4096
    d, r = make(B, rows, V, 50, 8, True, 3)
    want, bound = rules_ref(**d)
    for pad, off in ((0, 0), (4, 0), (5, 0), (8, 1), (64, 4), (7, 3)):
        src = torch.full((B, rows, V + pad), 9.0, device="cuda")
        dst = torch.full((B, rows, V + pad), 5.0, device="cuda")
        view, to = src[:, :, off:off + V], dst[:, :, off:off + V]
        view.copy_(torch.from_numpy(d["l"]))
        assert eesd.process_logits(view, r, out=to) is to
        close(to, want, bound)
        keep = torch.ones(V + pad, dtype=torch.bool, device="cuda")
        keep[off:off + V] = False
        assert (dst[:, :, keep] == 5.0).all() and (src[:, :, keep] == 9.0).all()
        close(eesd.process_logits(view, r), want, bound)
    # strided token lists and masks
    wide = torch.zeros(B, 100, dtype=torch.int32, device="cuda")
    wide[:, 3:53] = torch.from_numpy(d["history"]).cuda()
    m = torch.zeros(B, rows, V // 32 + 3, dtype=torch.int32, device="cuda")
    m[:, :, :V // 32] = torch.from_numpy(d["mask"]).cuda()
    kw = {k: torch.from_numpy(d[k]).cuda() for k in ("n_history", "n_prompt", "drafted", "repetition", "frequency", "presence")}
    d2 = {k: v for k, v in d.items() if k != "bias"}
    want, bound = rules_ref(**d2)
    close(eesd.process_logits(torch.from_numpy(d["l"]).cuda(), eesd.LogitRules(history=wide[:, 3:53], mask=m, **kw)), want, bound)


@pytest.mark.gpu
def test_not_finite_logits_and_rows_without_anything():
    B, rows, V = 2, 2, 200
    d, r = make(B, rows, V, 30, 0, True, 11)
    d["l"][0, 0, :] = np.nan                                     # this row is masked throughout
    d["l"][0, 1, 3:9] = [np.inf, -np.inf, np.nan, 0.0, -0.0, 1e38]
    d["l"][1, 1, :6] = [np.inf, -np.inf, np.nan, 0.0, -0.0, 3e38]   # and this one not at all
    want, bound = rules_ref(**d)
    out = eesd.process_logits(torch.from_numpy(d["l"]).cuda(), r)
    assert (out[0, 0] == float("-inf")).all()
    close(out, want, bound)


@pytest.mark.gpu
def test_two_dimensional_form_streams_and_graph():
    B, V = 6, 5000
    d, _ = make(B, 1, V, 300, 20, True, 5)
    words = torch.from_numpy(d["mask"][:, 0].copy()).cuda()
    hist = torch.from_numpy(d["history"]).cuda()
    n = torch.full((B,), 10, dtype=torch.int32, device="cuda")
    rep = torch.from_numpy(d["repetition"]).cuda()
    r = eesd.LogitRules(history=hist, n_history=n, repetition=rep, mask=words)
    logits = torch.from_numpy(d["l"][:, 0].copy()).cuda()

    def want():
        return rules_ref(d["l"], history=d["history"], n_history=n.cpu().numpy(), repetition=d["repetition"], mask=d["mask"])

    w, bound = want()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out = eesd.process_logits(logits, r)
    torch.cuda.synchronize()
    assert out.shape == (B, V)
    close(out[:, None], w, bound)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = eesd.process_logits(logits, r)
    for k in (0, 1, 50, 300):                                    # the history grows under the captured call
        n.fill_(k)
        g.replay()
        torch.cuda.synchronize()
        close(out[:, None], *want())


@pytest.mark.gpu
def test_refusals():
    f = lambda *s: torch.zeros(*s, device="cuda")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    for kw in (dict(history=f(2, 3)), dict(history=i(3)), dict(history=i(2, 4)[:, ::2]), dict(n_history=i(2)), dict(history=i(2, 3), n_prompt=i(3)),
               dict(repetition=f(2), frequency=f(3)), dict(bias_ids=i(3)), dict(bias_start=i(3), bias_ids=i(4), bias_values=f(3)), dict(drafted=i(2, 3), mask=i(2, 3, 4)),
               dict(repetition=f(4)[::2]), dict(repetition=torch.zeros(2)), dict(mask=f(2, 3, 4))):
        with pytest.raises(ValueError):
            eesd.LogitRules(**kw)
    r = eesd.LogitRules(history=i(2, 3), drafted=i(2, 2), repetition=f(2) + 1, mask=i(2, 3, 4))
    assert eesd.process_logits(f(2, 3, 128), r).shape == (2, 3, 128)
    for bad in (f(2, 2, 128), f(1, 3, 128), f(2, 3, 129), f(2, 128), f(2, 3, 128).double(), f(2, 3, 256)[:, :, ::2], f(2, 6, 128)[:, :3], torch.zeros(2, 3, 128)):
        with pytest.raises(ValueError):
            eesd.process_logits(bad, r)
    with pytest.raises(ValueError):
        eesd.process_logits(f(2, 3, 128), r, out=f(2, 3, 127))
    buf = f(2 * 3 * 128 + 128)
    a, o = buf[:768].view(2, 3, 128), buf[128:].view(2, 3, 128)
    with pytest.raises(eesd.EesdError):
        eesd.process_logits(a, r, out=o)                         # overlapping, but not in place
    with pytest.raises(eesd.EesdError):
        eesd.process_logits(f(1, 257, 8), eesd.LogitRules())     # too many rows a sequence


def test_null_and_sizes_are_refused_without_a_device():
    L, r = eesd.lib(), b.RulesStruct()
    p = C.addressof(r)
    x = 1 << 20   # a non-null address that is never dereferenced: every call below is refused on the host
    call = lambda **k: (lambda a: L.eesd_process_logits(None, a["l"], a["li"], a["o"], a["lo"], a["B"], a["rows"], a["V"], a["r"]))(
        {**dict(l=x, li=8, o=2 * x, lo=8, B=1, rows=1, V=8, r=p), **k})
    for kw in (dict(l=None), dict(o=None), dict(r=None), dict(B=0), dict(rows=0), dict(rows=257), dict(V=0), dict(li=7), dict(lo=7), dict(l=x + 2), dict(o=x + 4), dict(lo=9, o=x)):
        assert call(**kw) == -1, kw
    r.n_bias = 3
    assert call() == -1
    r.n_bias = -1
    assert call() == -1
    r.n_bias = 0
    r.mask, r.mask_stride = x, 0
    assert call() == -1
    r.mask = None
    r.history, r.history_len, r.history_stride = x, 5, 4
    assert call() == -1
    r.history = None
    r.drafted, r.drafted_stride = x, 1
    assert call(rows=3) == -1
    assert call(B=2 ** 31 - 1, rows=2, V=1) == -8      # more rows than a grid counts


def test_w4_layout_and_its_refusals_without_a_device():
    L, l = eesd.lib(), b.W4Layout()
    for R, K, g, sd, zp in ((1, 1, 32, 0, 0), (17, 65, 64, 1, 1), (27648, 5120, 128, 1, 0), (8192, 28672, 32, 0, 1)):
        assert L.eesd_w4_layout_of(C.byref(b.W4Desc(R, K, g, sd, zp)), C.byref(l)) == 0
        n = 128 // g * 16
        assert (l.row_blocks, l.k_blocks, l.groups) == (-(-R // 16), -(-K // 128), -(-K // g))
        assert (l.scales, l.zeros, l.block_bytes) == (1024, 1024 + n * (4, 2)[sd], 1024 + n * (4, 2)[sd] + n * zp)
        assert l.block_bytes % 16 == 0 and l.total_bytes == l.row_blocks * l.k_blocks * l.block_bytes
    for bad, st in (((0, 8, 32, 0, 0), -1), ((8, 0, 32, 0, 0), -1), ((8, 8, 16, 0, 0), -8), ((8, 8, 32, 2, 0), -1), ((8, 8, 32, 0, 2), -1), ((2 ** 29, 8, 32, 0, 0), -1)):
        assert L.eesd_w4_layout_of(C.byref(b.W4Desc(*bad)), C.byref(l)) == st
    assert L.eesd_w4_layout_of(None, C.byref(l)) == -1
    d = b.W4Desc(8, 8, 32, 0, 0)
    assert L.eesd_w4_layout_of(C.byref(d), None) == -1
    p = C.addressof(d)
    assert L.eesd_w4_project_rows(None, p, None, 1 << 20, 0, 1 << 20, 8, 1 << 20, 8, 1, None, 0) == -1
    assert L.eesd_w4_project_rows(None, p, 1 << 20, 10, 0, 1 << 20, 8, 1 << 20, 8, 1, None, 0) == -2
    assert L.eesd_w4_quantize(None, p, 0, None, 8, 1 << 20, 1 << 20) == -1
