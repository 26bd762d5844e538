"""Logit rules: the repetition penalty over the whole range of fp32.  One rounding of a quotient or product of two fp32 numbers, so results are
compared for equality with numpy's."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b


@pytest.mark.gpu
@pytest.mark.parametrize("V", [4096, 4099])
def test_quotients_of_every_size_are_rounded_once(V):
    g = np.random.default_rng(V)
    top = np.finfo(np.float32).max
    rhos = np.array([1.0, 1.2, 1.7, 3.3, 10.0, 0.5, 0.7, np.nextafter(np.float32(1), np.float32(0)), np.nextafter(np.float32(1), np.float32(2)), 1e-30, 1e30, 2.0 ** -130,
                     top], np.float32)
    with np.errstate(all="ignore"):
        x = np.ldexp(1 + g.random((len(rhos), 3, V)), g.integers(-149, 128, (len(rhos), 3, V))).astype(np.float32)
        x[:, 1] *= np.where(g.random((len(rhos), V)) < 0.5, -1, 1).astype(np.float32)
        x[:, 2] = np.ldexp(1 + g.random((len(rhos), V)), g.integers(-2, 4, (len(rhos), V)))          # ordinary logits
        x[:, 0, :16] = np.nextafter(top, np.float32(0)) * np.float32(2.0) ** -np.arange(16, dtype=np.float32)
        x[:, 0, 16:32] = top * np.float32(2.0) ** -np.arange(16, dtype=np.float32)
        x[:, 0, 32:40] = [0.0, -0.0, np.inf, -np.inf, 2.0 ** -149, 2.0 ** -126, -(2.0 ** -149), np.nan]
        rho = rhos[:, None, None]
        want = np.where(x > 0, x / rho, x * rho).astype(np.float32)
    seen = torch.arange(V, dtype=torch.int32, device="cuda").repeat(len(rhos), 1)
    r = eesd.LogitRules(history=seen, n_prompt=torch.full((len(rhos),), V, dtype=torch.int32, device="cuda"), repetition=torch.from_numpy(rhos).cuda())
    got = eesd.process_logits(torch.from_numpy(x).cuda(), r).cpu().numpy()
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same.all(), [(x[tuple(i)], rhos[i[0]], got[tuple(i)], want[tuple(i)]) for i in np.argwhere(~same)[:5]]


def refused(**kw):
    """eesd_process_logits with addresses that are never dereferenced: what it answers on the host"""
    r = b.RulesStruct()
    a = dict(V=8, li=None, B=1, rows=1)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            setattr(r, k, v)
    ld = a["V"] if a["li"] is None else a["li"]
    return eesd.lib().eesd_process_logits(None, 1 << 20, ld, 1 << 45, ld, a["B"], a["rows"], a["V"], C.addressof(r))


def test_lengths_that_32_bits_do_not_count_past_are_refused():
    # a block's column, token and bias indices go a few thousand past the end
    far = 2 ** 31 - 1
    for n in (2 ** 30 + 1, far - 4096, far):
        assert refused(V=n) == -8
        assert refused(history=1 << 20, history_len=n, history_stride=n, repetition=1 << 20) == -8
        assert refused(bias_start=1 << 20, bias_ids=1 << 20, bias_values=1 << 20, n_bias=n) == -8


def test_misaligned_lists_are_refused():
    at = (1 << 20) + 2
    assert refused(history=at, history_len=4, history_stride=4, repetition=1 << 20) == -1
    for name in ("n_history", "n_prompt"):
        assert refused(history=1 << 20, history_len=4, history_stride=4, repetition=1 << 20, **{name: at}) == -1
    for name in ("repetition", "frequency", "presence"):
        assert refused(history=1 << 20, history_len=4, history_stride=4, **{name: at}) == -1
    assert refused(rows=3, drafted=at, drafted_stride=2, repetition=1 << 20) == -1
    for name in ("bias_start", "bias_ids", "bias_values"):
        assert refused(n_bias=3, **{**dict(bias_start=1 << 20, bias_ids=1 << 20, bias_values=1 << 20), name: at}) == -1
    assert refused(mask=at, mask_stride=1) == -1
