"""Attention over the 4-bit cache: every part that a segment is cut into counts, seen without a tolerance that grows with the text."""
import pytest
import torch

import paper_2406_03853_b200 as eesd
from tests.test_gpu_kv4 import DT, gen, ints, new_cache

pytestmark = pytest.mark.gpu


def pad(table, room):
    """room: entries to spare; with many of them the call is shared out by runs"""
    return torch.nn.functional.pad(table, (0, room), value=-1)


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("room", [0, 1000])
@pytest.mark.parametrize("R,H", [(1, 3), (3, 4), (16, 3)])
@pytest.mark.parametrize("share", ["ranges", "in turn"])
def test_every_part_counts(share, R, H, room, a):
    """Equal scores and values that are 1 in one dimension: each dimension's result is its share of the positions.  Dimensions take 64 ranges of 1094 positions (a
    block's part is a quarter of one or more), or tiles in turn (a part is one in 68 of a dimension's)"""
    D, n = 64, 70001
    c, table = new_cache(1, n, 1, D, 128, 64)
    p = torch.arange(n, device="cuda")
    dim = p * D // n if share == "ranges" else p // 16 % D
    v = torch.nn.functional.one_hot(dim, D).float()[None, :, None]
    c.append(torch.zeros_like(v), v, table, ints([0]))
    q = torch.randn(1, R, H, D, generator=gen(6), device="cuda").to(DT[a])
    out = eesd.attend_rows(q, c, pad(table, room), ints([n]))[0].double()
    held = c.read(table, n)[1][0, :, 0].double()
    for m in range(R):
        want = held[:n - R + m + 1].mean(0)
        # (numerators are powers of two times scales: exact; whole multiples of one scale below 2^24: sums exact; joined in fp32)
        tol = ((2.0 ** -24 if a == "f32" else 2.0 ** -8) + 2.0 ** -19) * want
        assert ((out[m] - want).abs() <= tol).all(), m


def test_every_part_of_many_segments_counts():
    """runs that hold whole segments and pieces of two, lengths from one tile to many"""
    D, B, Hkv, H = 64, 40, 5, 10
    lengths = [(977 * i) % 4000 + 1 for i in range(B)]
    c, table = new_cache(1, 4000, Hkv, D, 16, 64)
    p = torch.arange(4000, device="cuda")
    v = torch.nn.functional.one_hot(p // 16 % D, D).float()[None, :, None].repeat(1, 1, Hkv, 1)
    c.append(torch.zeros_like(v), v, table, ints([0]))
    held = c.read(table, 4000)[1][0, :, 0].double()
    for a in ("f32", "bf16"):
        q = torch.randn(B, 1, H, D, generator=gen(6), device="cuda").to(DT[a])
        for room in (0, 4000):
            out = eesd.attend_rows(q, c, pad(table.expand(B, -1), room), ints(lengths))[:, 0].double()
            for i, n in enumerate(lengths):
                want = held[:n].mean(0)
                assert ((out[i] - want).abs() <= ((2.0 ** -24 if a == "f32" else 2.0 ** -8) + 2.0 ** -19) * want).all(), (i, n)
