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


def bound(out, A, of_rows, n, dtype):
    """How far a result may be when nothing is dearer than fp32.  A = sum p |v|, S = scale sum |q k|, Q = scale max |q| sum |k|.
    Scores: two fp16 terms of a query leave 2^-22 of it, or 2^-25 where the largest is at least 2^14 (2^-39 of it); up to 4 groups' sums of 32 to 128 products and
    their scales, at most 16 roundings of 2^-24.  Exponentials 2^-22, numerators' two terms 2^-22 and the product before them 2^-23, each by 2^-28 of the largest
    product with a value.  Sums of n positions, at least 8 warps: two roundings of 2^-24 per 16 positions and 64 for joining."""
    S, most, Q, _ = of_rows
    dx = S * (2.0 ** -22 + 2.0 ** -20) + Q * 2.0 ** -39
    rel = 2 * dx + 3 * 2.0 ** -22 + (n / 64 + 64) * 2.0 ** -24
    return A * rel[..., None] * (1 + 1e-3) + (n * 2.0 ** -28 * most)[..., None] + half_step(dtype) * out.abs() + 1e-37


def check(cache, table, q, n_ctx, room=0, scale=None, **kw):
    D = q.shape[-1]
    n = table.shape[1] * cache.page_tokens
    k, v = cache.read(table, n)
    out = eesd.attend_rows(q, cache, pad(table, room), ints(n_ctx), scale=scale, **{i: x for i, x in kw.items()})
    qq = q.float()
    if kw.get("rope") is not None:
        R = q.shape[1]
        where = kw["positions"].cpu().numpy() if kw.get("positions") is not None else np.array([[L - R + m for m in range(R)] for L in n_ctx])
        qq = torch.from_numpy(ref.turn(qq.cpu().numpy(), kw["rope"], where)).cuda()
    want, A, of_rows = ref.attend(qq, k.double(), v.double(), n_ctx, None, scale or D ** -0.5, kw.get("visible"))
    tol = bound(want, A, of_rows, max(n_ctx), q.dtype)
    off = (out.double() - want).abs()
    assert (off <= tol).all(), (float((off / tol).nan_to_num(1e30).max()), float(off.max()))
    return out


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


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("room", [0, 30000])
@pytest.mark.parametrize("D,group", [(64, 64), (128, 32), (128, 128)])
def test_numerators_that_cancel(D, group, room, a):
    """pairs of positions with opposite values and nearly equal scores: what is left of them is far below either"""
    B, R, H, Hkv, n = 1, 3, 4, 2, 192
    c, table = new_cache(B, n, Hkv, D, 16, group)
    g = gen(2)
    v = torch.randint(-7, 8, (B, n, Hkv, D), generator=g, device="cuda").float()
    v[..., ::32], v[..., 1::32] = 8, -7                    # (a scale of 1, and zero points that keep every value, and its opposite, as it is)
    v[:, 1::2] = -v[:, ::2]
    k = torch.randn(B, n, Hkv, D, generator=g, device="cuda") * 2.0 ** -13
    c.append(k, v, table, ints([0]))
    assert torch.equal(c.read(table, n)[1], v)
    q = torch.randn(B, R, H, D, generator=g, device="cuda").to(DT[a])
    out = check(c, table, q, [n], room)
    assert out[:, -1].float().abs().mean() < 2.0 ** -10


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("room", [0, 30000])
@pytest.mark.parametrize("D,group,R,H", [(64, 32, 1, 2), (128, 32, 5, 8), (128, 64, 16, 2), (128, 128, 3, 4)])
def test_queries_with_a_loud_channel(D, group, R, H, room, a):
    """one channel of the queries far above the others, where the keys are nothing (or little): the others keep their own bits"""
    Hkv, n = 2, 500
    k, v = rows(1, n, Hkv, D, torch.float32, 5)
    for loud, there in ((100.0, 0.0), (2.0 ** 14, 0.0), (1000.0, 1e-4), (2.0 ** 17, 0.0)):
        k2 = k.clone()
        k2[..., 5] *= there
        c, table = new_cache(1, n, Hkv, D, 16, group)
        c.append(k2, v, table, ints([0]))
        q = torch.randn(1, R, H, D, generator=gen(6), device="cuda")
        q[..., 5] *= loud
        check(c, table, q.to(DT[a]), [n], room)


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("room", [0, 30000])
def test_loud_channels_turned(a, room):
    """a pair of loud channels under rotary angles, plain queries beside it"""
    D, n, R, H, Hkv = 128, 700, 4, 8, 2
    rope = rope_table(n, D)
    k, v = rows(1, n, Hkv, D, torch.float32, 7)
    k[..., 64:66] = 0
    c, table = new_cache(1, n, Hkv, D, 16, 64)
    c.append(k, v, table, ints([0]), rope=rope)
    q = torch.randn(1, R, H, D, generator=gen(8), device="cuda")
    q[..., 64:66] *= 3000
    check(c, table, q.to(DT[a]), [n], room, rope=rope)


@pytest.mark.parametrize("a", ["bf16", "f32"])
@pytest.mark.parametrize("room", [0, 30000])
@pytest.mark.parametrize("ek,eq", [(100, -100), (124, -124), (123, -140), (-100, 100), (-115, 118), (60, -58), (-130, 110)])
def test_keys_over_the_whole_range(ek, eq, room, a):
    """keys that the cache holds have scores wherever queries times keys are numbers"""
    R, H, Hkv, D, n = 3, 4, 2, 128, 300
    k, v = rows(1, n, Hkv, D, torch.float32, 9)
    c, table = new_cache(1, n, Hkv, D, 16, 64)
    c.append((k.double() * 2.0 ** (ek - 4)).float(), v, table, ints([0]))
    q = (torch.randn(1, R, H, D, generator=gen(10), device="cuda").double() * 2.0 ** (eq + 4)).to(DT[a])
    out = check(c, table, q, [n], room)
    assert out.isfinite().all()


@pytest.mark.parametrize("room", [0, 30000])
@pytest.mark.parametrize("es", [-120, -60, 60, 120])
def test_scales_over_the_whole_range(es, room):
    """a scale far from 1 with queries that bring the scores back"""
    R, H, Hkv, D, n = 3, 4, 2, 64, 300
    k, v = rows(1, n, Hkv, D, torch.float32, 11)
    c, table = new_cache(1, n, Hkv, D, 16, 64)
    c.append(k, v, table, ints([0]))
    q = torch.randn(1, R, H, D, generator=gen(12), device="cuda") * 2.0 ** -es
    check(c, table, q, [n], room, scale=2.0 ** es / 8)


@pytest.mark.parametrize("room", [0, 30000])
@pytest.mark.parametrize("R,H,Hkv", [(13, 8, 8), (16, 64, 8), (2, 3, 1)])
def test_trees_of_bf16_rows(R, H, Hkv, room):
    """a chain with a sibling each, turned by their depths"""
    B, D, n = 2, 128, 260
    c, table = new_cache(B, n, Hkv, D, 32, 64)
    rope = rope_table(n, D)
    k, v = rows(B, n, Hkv, D, torch.bfloat16, 3)
    depth = [(m + 1) // 2 for m in range(R)]
    n_ctx = [n, 200]
    positions = ints([[L - R + d for d in depth] for L in n_ctx])
    chain = lambda m: sum(1 << j for j in range(m) if (j % 2 == 1 or j == 0) and depth[j] < depth[m]) | 1 << m
    visible = ints([[chain(m) for m in range(R)]] * B)
    c.append(k, v, table, ints([0] * B), rope=rope)
    c.append(k[:, :R], v[:, :R], table, ints([L - R for L in n_ctx]), rope=rope, positions=positions)
    q = torch.randn(B, R, H, D, generator=gen(4), device="cuda").to(torch.bfloat16)
    check(c, table, q, n_ctx, room, visible=visible, rope=rope, positions=positions)
