"""Attention over the 4-bit cache at inputs that show lost bits: long even sums, numerators that cancel, queries with loud channels, the ends of the range."""
import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from tests import kv4_ref as ref
from tests.test_gpu_kv4 import DT, gen, ints, new_cache, rope_table, rows

pytestmark = pytest.mark.gpu


def pad(table, room):
    """room: entries to spare; with many of them the call is shared out by runs"""
    return torch.nn.functional.pad(table, (0, room), value=-1)


def half_step(dtype):
    """the largest rounding of a result, relative to it"""
    return 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8


@pytest.mark.parametrize("a", ["bf16", "f32"])
def test_long_even_sums(a):
    """Equal scores over 2^18 positions, 32768 of them a warp: the sums are of what the codes stand for, and nothing larger beside it.  Values of -1, 0 and 1 times a
    token's factor (8 bits: a numerator times its scale is exact), with 8 and -7 in two dimensions so that the scale is the factor; 300 sequences on the same
    pages, so that a block has whole segments."""
    B, Hkv, D, page, n = 300, 2, 64, 128, 1 << 18
    c, table = new_cache(1, n, Hkv, D, page, 64)
    g = gen(1)
    v = torch.randint(-1, 2, (1, n, Hkv, D), generator=g, device="cuda").float()
    v[..., 0], v[..., 1] = 8, -7
    v *= 1 + torch.randint(0, 128, (1, n, Hkv, 1), generator=g, device="cuda") / 128
    c.append(torch.zeros_like(v), v, table, ints([0]))
    held = c.read(table, n)[1][0].double()
    assert torch.equal(held, v[0].double())
    del v
    q = torch.randn(B, 1, Hkv, D, generator=g, device="cuda").to(DT[a])
    out = eesd.attend_rows(q, c, table.expand(B, -1).contiguous(), ints([n] * B))[:, 0].double()
    want = held.mean(0)
    # a warp has the pairs of tiles 8 i + w: its sums are at most twice the largest that begins at the start, and every one of its 2048 (or, where a segment is
    # cut, fewer) steps rounds one (or a product of at most 16) by 2^-23, twice that where a step is two additions; one rounding of 2^-22 at the end
    parts = held.view(-1, 8, 32, Hkv, D).sum(2).cumsum(0).abs().amax((0, 1))
    tol = 8 * 2048 * 2.0 ** -22 * (2 * parts + 16) / n + (half_step(DT[a]) + 2.0 ** -20) * want.abs()
    off = (out - want).abs()
    assert (off <= tol).all(), float((off / tol).max())
