"""The 4-bit key / value cache: what stands in it after append, what read gives back, attention over it, against a plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from tests import kv4_ref as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rope_table(n, D, theta=10000.0):
    a = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    return torch.stack([a.cos(), a.sin()], -1).float().cuda()


def new_cache(B, n, Hkv, D, page, group, seed=0, spare=2, garbage=False):
    """a cache with room for n tokens of B sequences, their pages anywhere in the pool"""
    P = -(-n // page)
    c = eesd.KV4Cache(B * P + spare, Hkv, D, page_tokens=page, group=group)
    if garbage:
        c.buffer.copy_(torch.randint(0, 256, c.buffer.shape, generator=gen(seed + 9), device="cuda", dtype=torch.uint8))
    table = torch.randperm(B * P + spare, generator=gen(seed), device="cuda")[:B * P].to(torch.int32).view(B, P)
    return c, table


def rows(B, n, Hkv, D, dtype, seed):
    g = gen(seed)
    k = torch.randn(B, n, Hkv, D, generator=g, device="cuda") * (1 + 3 * (torch.rand(1, 1, Hkv, D, generator=g, device="cuda") < 0.05)) + 0.3
    v = torch.randn(B, n, Hkv, D, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(B, n, Hkv, 1, generator=g, device="cuda"))
    return k.to(dtype), v.to(dtype)


def check_held(cache, table, k, v, at, rope=None, positions=None, n_rows=None):
    """the pool holds exactly the codes, scales and zero points of k, v at positions at[b] + m; returns which bytes of the pool that says nothing of"""
    B, R, Hkv, D = k.shape
    page, group = cache.page_tokens, cache.group
    n = table.shape[1] * page
    codes, scales, zeros = ref.held(cache.buffer, table, n, Hkv, D, page, group)
    kk = k.float().cpu().numpy()
    if rope is not None:
        where = np.asarray(at)[:, None] + np.arange(R) if positions is None else positions.cpu().numpy()
        kk = ref.turn(kk, rope, where)
    for i, x in enumerate((kk, v.float().cpu().numpy())):
        c, s, z = ref.quantize(x, group)
        for b in range(B):
            for m in range(R if n_rows is None else n_rows[b]):
                p = at[b] + m
                if 0 <= p < n:
                    np.testing.assert_array_equal(scales[i, b, p], s[b, m])
                    ok = ~np.isnan(s[b, m])
                    np.testing.assert_array_equal(zeros[i, b, p][ok], z[b, m][ok])
                    np.testing.assert_array_equal(codes[i, b, p][ok.repeat(group, -1)], c[b, m][ok.repeat(group, -1)])


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("B,R,Hkv,page,at", [(1, 1, 1, 16, 0), (1, 1, 3, 16, 37), (2, 5, 2, 32, 13), (1, 40, 2, 64, 7), (3, 16, 1, 128, 112)])
def test_append_is_exact(B, R, Hkv, page, at, D, group, a):
    c, table = new_cache(B, at + R, Hkv, D, page, group, seed=R)
    k, v = rows(B, R, Hkv, D, DT[a], R + D)
    rope = rope_table(at + R, D) if R % 2 else None
    c.append(k, v, table, ints([at] * B), rope=rope)
    check_held(c, table, k, v, [at] * B, rope)
    # what is read back is what stands there
    got = c.read(table, R, start=ints([at] * B))
    low = c.read(table, R, start=ints([at] * B), dtype=torch.bfloat16)
    want = ref.values(*(x[:, :, at:at + R] for x in ref.held(c.buffer, table, at + R, Hkv, D, page, group)), group)
    for i in range(2):
        assert torch.equal(got[i].cpu(), torch.from_numpy(want[i]).float())      # (a product of an integer below 16 and a bf16: exact)
        assert torch.equal(low[i], got[i].to(torch.bfloat16))


def test_append_ties_borders_and_odd_groups():
    D, group = 128, 32
    w = torch.zeros(16, D)
    half = torch.arange(D).float() % 31 / 2
    w[0] = (half - 7.5).clamp(-7, 8)                          # scale 1: every quotient is a tie or an integer
    w[1] = half.clamp(0, 15)
    w[2] = -half.clamp(0, 15)
    w[3] = half * (1 + 2.0 ** -8)                             # scale halfway between two bf16
    w[4] = half * (1 + 2.0 ** -8 + 2.0 ** -20)
    w[5] = torch.nextafter(half, torch.full((D,), 99.0))
    w[6] = torch.nextafter(half, torch.full((D,), -99.0))
    w[7] = 1e-40
    w[8, 5], w[8, 6] = 3e38, -3e38                            # the range passes the largest fp32
    w[9] = 1e-45
    w[10, 3] = float("nan")
    w[11, 40], w[11, 70] = float("inf"), float("-inf")
    w[12] = torch.rand(D, generator=torch.Generator().manual_seed(1)) + 100
    w[13] = -torch.rand(D, generator=torch.Generator().manual_seed(2)) - 100
    w[14] = torch.randn(D, generator=torch.Generator().manual_seed(3)) * 1e30
    w[15] = torch.randn(D, generator=torch.Generator().manual_seed(4)) * 1e-30
    w = w.cuda()
    k, v = w[None, :, None], w.flip(0)[None, :, None]
    for c, table in (new_cache(1, 16, 1, D, 16, group), new_cache(1, 16, 1, D, 16, 128)):
        c.append(k, v, table, ints([0]))
        check_held(c, table, k, v, [0])
        got = c.read(table, 16)[0][0, :, 0]
        assert got[10, :32].isnan().all() and (c.group == 128 or not got[10, 32:].isnan().any())
        assert got[9].eq(0).all() and got[11, 32:64].isnan().all()


@pytest.mark.parametrize("D,group,page", [(64, 32, 16), (128, 128, 32), (128, 32, 16)])
def test_append_leaves_the_rest_of_the_pool(D, group, page):
    """pages that end inside the rows, ragged rows, positions and pages that do not exist: only the rows' own bytes change"""
    B, R, Hkv = 6, 21, 2
    c, table = new_cache(B, 3 * 16 + 5, Hkv, D, page, group, seed=4, garbage=True)
    n = table.shape[1] * page
    at = [11, -4, n - 9, 0, 5, 2147483640]                    # inside; before the first position; past the table; ..; past everything
    n_rows = [21, 21, 21, 0, -3, 21]
    table[4, 0] = 2 ** 30
    k, v = rows(B, R, Hkv, D, torch.float32, 5)
    before = c.buffer.clone()
    c.append(k, v, table, ints(at), n_rows=ints(n_rows))
    torch.cuda.synchronize()
    table_ok = table.clone()
    table_ok[4, 0] = 0
    old = ref.held(before, table_ok, n, Hkv, D, page, group)
    now = ref.held(c.buffer, table_ok, n, Hkv, D, page, group)
    check_held(c, table_ok, k, v, at, n_rows=[max(x, 0) for x in n_rows])
    mine = np.zeros((B, n), bool)
    for b in range(B):
        for m in range(n_rows[b]):
            if 0 <= at[b] + m < n:
                mine[b, at[b] + m] = True
    assert mine[0].sum() == 21 and mine[1].sum() == 17 and mine[2].sum() == 9 and not mine[3:].any()
    for x, y in zip(old, now):
        np.testing.assert_array_equal(x[:, ~mine], y[:, ~mine])
    # pages of nobody
    used = set(table.cpu().view(-1).tolist())
    pool0, pool1 = (t.view(c.n_pages, -1) for t in (before, c.buffer))
    for p in range(c.n_pages):
        if p not in used:
            assert torch.equal(pool0[p], pool1[p])


def test_pages_that_do_not_exist():
    D, Hkv, page = 64, 2, 16
    for bad in (-1, 4, 2147483647, -2147483648):
        c = eesd.KV4Cache(4, Hkv, D, page_tokens=page, group=32)
        table = ints([[2, bad, 0]])
        k, v = rows(1, 48, Hkv, D, torch.float32, 6)
        c.append(k, v, table, ints([0]))
        gk, gv = c.read(table, 64)
        assert gk[0, 16:32].eq(0).all() and gv[0, 16:32].eq(0).all() and gk[0, 48:].eq(0).all()
        assert gk[0, :16].ne(0).any() and gk[0, 32:48].ne(0).any()
        q = torch.randn(1, 2, 4, D, generator=gen(1), device="cuda")
        out = eesd.attend_rows(q, c, table, ints([47]))
        # the same with the page's positions left out
        keep = list(range(16)) + list(range(32, 47))
        want, A, S = ref.attend(q.double(), gk[:, keep].double(), gv[:, keep].double(), [31], None, D ** -0.5)
        assert ((out.double() - want).abs() <= ref.bound(want, A, S, 48, D, torch.float32)).all()
        assert eesd.attend_rows(q, c, ints([[bad, bad, bad]]), ints([47])).eq(0).all()


def test_strided_unaligned_and_broadcast_rows():
    B, R, H, Hkv, D = 2, 3, 4, 2, 128
    c, table = new_cache(B, 40, Hkv, D, 16, 64)
    fused = torch.randn(B, R, (H + 2 * Hkv) * D + 3, generator=gen(2), device="cuda")
    for off in (0, 1):   # a projection's rows as they come, and beside every alignment
        k = fused[..., off + H * D:off + (H + Hkv) * D].unflatten(-1, (Hkv, D))
        v = fused[..., off + (H + Hkv) * D:off + (H + 2 * Hkv) * D].unflatten(-1, (Hkv, D))
        q = fused[..., off:off + H * D].unflatten(-1, (H, D))
        for x, y, z in ((k, v, q), (k.to(torch.bfloat16), v.to(torch.bfloat16), q.to(torch.bfloat16)), (k.transpose(0, 1).contiguous().transpose(0, 1), v, q)):
            c.append(x, y, table, ints([9, 30]))
            check_held(c, table, x, y, [9, 30])
            a, b = eesd.attend_rows(z, c, table, ints([12, 33])), eesd.attend_rows(z.contiguous(), c, table, ints([12, 33]))
            assert torch.equal(a, b)
    one = torch.randn(1, 1, 1, D, generator=gen(3), device="cuda").expand(B, R, Hkv, D)
    c.append(one, one, table, ints([0, 16]))
    check_held(c, table, one, one, [0, 16])
    wide = torch.zeros(B, 64, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table                       # a table with room to spare, one row of it apart
    got = c.read(wide[:, :table.shape[1]], 40)
    assert torch.equal(got[0], c.read(table, 40)[0])


def test_read_bounds():
    D, Hkv = 64, 3
    c, table = new_cache(2, 50, Hkv, D, 16, 64)
    k, v = rows(2, 50, Hkv, D, torch.float32, 8)
    c.append(k, v, table, ints([0, 0]))
    full = c.read(table, 64)
    for start, n_ctx in (([0, 5], [50, 0]), ([-7, 60], [10, 62]), ([63, 2147483647], [64, 2147483647]), ([-2147483648, 33], [-1, 40])):
        got = c.read(table, 20, start=ints(start), n_ctx=ints(n_ctx))
        for x, y in zip(got, full):
            want = torch.zeros(2, 20, Hkv, D, device="cuda")
            for b in range(2):
                for m in range(20):
                    p = start[b] + m
                    if 0 <= p < min(64, n_ctx[b]):
                        want[b, m] = y[b, p]
            assert torch.equal(x, want)


def check_attend(c, table, q, n_ctx, n_rows=None, visible=None, rope=None, positions=None, scale=None, room=0):
    """room: entries that the call's page table has to spare (what a call may hold decides how it is shared out)"""
    B, R, H, D = q.shape
    n = table.shape[1] * c.page_tokens
    k, v = c.read(table, n)
    table = torch.nn.functional.pad(table, (0, room), value=-1)
    out = eesd.attend_rows(q, c, table, ints(n_ctx), n_rows=None if n_rows is None else ints(n_rows), scale=scale, visible=visible, rope=rope, positions=positions)
    assert out.dtype == q.dtype and out.shape == q.shape
    qq = q.float()
    if rope is not None:
        own = [R if n_rows is None else min(max(x, 0), R) for x in n_rows or [R] * B]
        where = np.array([[n_ctx[b] - own[b] + m for m in range(R)] for b in range(B)]) if positions is None else positions.cpu().numpy()
        qq = torch.from_numpy(ref.turn(qq.cpu().numpy(), rope, where)).cuda()
    want, A, S = ref.attend(qq, k.double(), v.double(), n_ctx, n_rows, scale or D ** -0.5, visible)
    tol = ref.bound(want, A, S, n, D, q.dtype)
    off = (out.double() - want).abs()
    assert (off <= tol).all(), (float((off / tol.clamp(min=1e-300)).nan_to_num().max()), float(off.max()))
    again = eesd.attend_rows(q, c, table, ints(n_ctx), n_rows=None if n_rows is None else ints(n_rows), scale=scale, visible=visible, rope=rope, positions=positions)
    assert torch.equal(out, again)                        # the same bits every time
    return out


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("B,R,H,Hkv,page,n", [(1, 1, 1, 1, 16, 1), (1, 1, 4, 4, 16, 17), (2, 3, 8, 2, 32, 130), (1, 16, 7, 1, 64, 333), (3, 5, 16, 2, 16, 700),
                                              (1, 2, 40, 40, 128, 1056), (1, 9, 16, 1, 16, 2049)])
def test_attend(B, R, H, Hkv, page, n, D, group, a):
    c, table = new_cache(B, n, Hkv, D, page, group, seed=n, garbage=True)
    k, v = rows(B, n, Hkv, D, torch.float32, n)
    rope = rope_table(n, D) if n % 2 else None
    c.append(k, v, table, ints([0] * B), rope=rope)
    q = torch.randn(B, R, H, D, generator=gen(n + 1), device="cuda").to(DT[a])
    n_ctx = [max(1, n - 11 * b) for b in range(B)]
    for room in (0, 30000):
        check_attend(c, table, q, n_ctx, rope=rope, room=room)


@pytest.mark.parametrize("a", ["f32", "bf16"])
def test_attend_rows_that_see_little_or_nothing(a):
    B, R, H, Hkv, D = 7, 6, 4, 2, 128
    c, table = new_cache(B, 100, Hkv, D, 16, 64, garbage=True)
    k, v = rows(B, 100, Hkv, D, torch.float32, 1)
    n_ctx, n_rows = [0, 1, 3, 100, 50, 33, -5], [6, 6, 6, 1, 0, -2, 3]
    c.append(k, v, table, ints([0] * B))
    q = torch.randn(B, R, H, D, generator=gen(2), device="cuda").to(DT[a])
    out = check_attend(c, table, q, n_ctx, n_rows)
    assert out[0].eq(0).all() and out[1, :5].eq(0).all() and out[2, :3].eq(0).all() and out[3, 1:].eq(0).all() and out[4:].eq(0).all()
    assert out[1, 5].ne(0).any() and out[2, 3].ne(0).any() and out[3, 0].ne(0).any()
    # a tree whose rows see: themselves alone; nothing new; an earlier and a later row; nothing at all where there is nothing old
    visible = ints([[1 << m for m in range(R)], [0] * R, [0x2a] * R, [-1] * R, [0] * R, [1] * R, [7] * R])
    out = check_attend(c, table, q, [6, 6, 6, 40, 100, 1, 3], [6, 6, 6, 6, 6, 1, 3], visible)
    assert out[1].eq(0).all() and out[4].ne(0).any()
    kk, vv = c.read(table, 6)
    assert (out[0].float() - vv[0].repeat_interleave(2, 1)).abs().max() <= 2.0 ** -8 * vv[0].abs().max()   # one position: its value


@pytest.mark.parametrize("R,H,Hkv", [(13, 8, 8), (16, 64, 8), (2, 3, 1)])
def test_attend_tree(R, H, Hkv):
    B, D, n = 2, 128, 260
    c, table = new_cache(B, n, Hkv, D, 32, 64)
    rope = rope_table(n, D)
    k, v = rows(B, n, Hkv, D, torch.float32, 3)
    depth = [(m + 1) // 2 for m in range(R)]
    n_ctx = [n, 200]
    positions = ints([[L - R + d for d in depth] for L in n_ctx])
    chain = lambda m: sum(1 << j for j in range(m) if (j % 2 == 1 or j == 0) and depth[j] < depth[m]) | 1 << m
    visible = ints([[chain(m) for m in range(R)]] * B)
    c.append(k, v, table, ints([0] * B), rope=rope)
    c.append(k[:, :R], v[:, :R], table, ints([L - R for L in n_ctx]), rope=rope, positions=positions)
    check_held(c, table, k[:, :R], v[:, :R], [L - R for L in n_ctx], rope, positions)
    q = torch.randn(B, R, H, D, generator=gen(4), device="cuda")
    check_attend(c, table, q, n_ctx, visible=visible, rope=rope, positions=positions)


@pytest.mark.parametrize("D,group", [(64, 64), (128, 32)])
def test_what_is_not_seen_has_no_effect(D, group):
    """NaN, infinite and huge scales behind a row's last position, and in the new rows that a tree's row does not see"""
    B, R, H, Hkv, n = 1, 4, 4, 2, 77
    c, table = new_cache(B, n + 30, Hkv, D, 16, group)
    k, v = rows(B, n + 30, Hkv, D, torch.float32, 5)
    c.append(k, v, table, ints([0]))
    q = torch.randn(B, R, H, D, generator=gen(6), device="cuda")
    tree = ints([[1, 1, 5, 8]])
    clean, clean_tree = check_attend(c, table, q, [n]), check_attend(c, table, q, [n], visible=tree)
    for bad in (float("nan"), 3e38, -1e30):
        k2, v2 = k.clone(), v.clone()
        k2[:, n - 1:] = bad                                # rows 0..2 do not see row 3, nobody what comes after
        v2[:, n - 1:] = bad
        c.append(k2, v2, table, ints([0]))
        assert torch.equal(eesd.attend_rows(q, c, table, ints([n]))[:, :3], clean[:, :3])
        assert torch.equal(eesd.attend_rows(q, c, table, ints([n]), visible=tree)[:, :3], clean_tree[:, :3])
    # a row of queries that is not finite, or huge, leaves the others
    c.append(k, v, table, ints([0]))
    for bad in (float("nan"), float("inf"), 1e30):
        q2 = q.clone()
        q2[:, 1] = bad
        out = eesd.attend_rows(q2, c, table, ints([n]))
        assert torch.equal(out[:, [0, 2, 3]], clean[:, [0, 2, 3]])
        assert bad == 1e30 or out[:, 1].isnan().all()
    # one that is seen
    v2 = v.clone()
    v2[:, 3, 0, :group] = float("nan")
    c.append(k, v2, table, ints([0]))
    out = eesd.attend_rows(q, c, table, ints([n]))
    assert out[..., :2, :group].isnan().all() and not out[..., 2:, :].isnan().any() and not out[..., :2, group:].isnan().any()


@pytest.mark.parametrize("a", ["f32", "bf16"])
def test_ranges(a):
    """scores from all equal to one position alone, values whose scales run over 2^80, queries of unlike sizes"""
    B, R, H, Hkv, D, n = 1, 4, 8, 2, 128, 500
    c, table = new_cache(B, n, Hkv, D, 16, 32)
    k, v = rows(B, n, Hkv, D, torch.float32, 7)
    v = v * torch.exp2(torch.linspace(-40, 40, n, device="cuda")[torch.randperm(n, generator=gen(8), device="cuda")])[None, :, None, None]
    c.append(k, v, table, ints([0]))
    q = torch.randn(B, R, H, D, generator=gen(9), device="cuda")
    q = (q * torch.tensor([0.0, 1e-6, 1.0, 30.0], device="cuda")[None, :, None, None]).to(DT[a])
    check_attend(c, table, q, [n])
    check_attend(c, table, q, [n], scale=2.0)
    c.append(k, torch.zeros_like(v), table, ints([0]))
    assert check_attend(c, table, q, [n]).eq(0).all()
    c.append(torch.zeros_like(k), v, table, ints([0]))
    check_attend(c, table, q, [n])


def test_one_position_decides_after_a_long_text():
    """the running maximum rises late, by little and by much, once in a while"""
    D, n = 64, 3000
    c, table = new_cache(1, n, 1, D, 16, 64)
    q = torch.ones(1, 1, 2, D, device="cuda")
    q[:, :, 1] = -0.25
    k = torch.randn(1, n, 1, D, generator=gen(1), device="cuda") * 0.1
    for i in range(10, n, 211):
        k[:, i] += i / 150                                 # scores up to 160
    v = torch.randn(1, n, 1, D, generator=gen(2), device="cuda")
    c.append(k, v, table, ints([0]))
    check_attend(c, table, q, [n])
    c.append(k.flip(1), v, table, ints([0]))
    check_attend(c, table, q, [n])


def test_ragged_batch_and_long_contexts():
    B, R, H, Hkv, D = 9, 2, 8, 1, 128
    lengths = [5000, 1, 17, 20000, 300, 0, 4096, 129, 2500]
    c, table = new_cache(B, max(lengths), Hkv, D, 128, 128)
    k, v = rows(B, max(lengths), Hkv, D, torch.bfloat16, 3)
    c.append(k, v, table, ints([0] * B), n_rows=ints(lengths))
    q = torch.randn(B, R, H, D, generator=gen(4), device="cuda")
    out = check_attend(c, table, q, lengths)
    check_attend(c, table, q, lengths, n_rows=[2, 1, 0, 2, 1, 2, 1, 2, 1])
    # a sequence by itself: within rounding, since it is cut up otherwise
    alone = eesd.attend_rows(q[3:4], c, table[3:4], ints(lengths[3:4]))
    assert (alone - out[3:4]).abs().max() <= 1e-5 * out[3].abs().max()


def test_offsets_past_32_bits():
    """a pool of over 4 GB, its last pages in use"""
    Hkv, D, page = 8, 128, 128
    per = ref.tile_bytes(D, 128) * 8 * Hkv
    pages = (1 << 32) // per + 40
    c = eesd.KV4Cache(pages, Hkv, D, page_tokens=page, group=128, buffer=torch.empty(pages * per, dtype=torch.uint8, device="cuda"))
    table = ints([[pages - 1, pages - 2, 0], [pages - 3, 1, pages - 4]])
    k, v = rows(2, 300, Hkv, D, torch.float32, 5)
    c.append(k, v, table, ints([0, 0]))
    small, t2 = new_cache(2, 384, Hkv, D, page, 128)
    small.append(k, v, t2, ints([0, 0]))
    for x, y in zip(c.read(table, 300), small.read(t2, 300)):
        assert torch.equal(x, y)
    q = torch.randn(2, 1, 64, D, generator=gen(4), device="cuda")
    assert torch.equal(eesd.attend_rows(q, c, table, ints([300, 290])), eesd.attend_rows(q, small, t2, ints([300, 290])))


def test_streams_graphs_and_given_buffers():
    B, R, H, Hkv, D, n = 2, 3, 16, 2, 128, 900
    c, table = new_cache(B, n + 8, Hkv, D, 16, 64)
    k, v = rows(B, n, Hkv, D, torch.float32, 5)
    c.append(k, v, table, ints([0, 0]))
    q = torch.randn(B, R, H, D, generator=gen(6), device="cuda")
    L = ints([n, n - 100])
    want = eesd.attend_rows(q, c, table, L)
    # two streams at once
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(eesd.attend_rows(q, c, table, L))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    # a graph of a step, replayed as the text grows: lengths are read on the device
    length = ints([n, n - 100])
    kn, vn = rows(B, 1, Hkv, D, torch.float32, 7)
    step = lambda: (c.append(kn, vn, table, length - 1), eesd.attend_rows(q[:, :1], c, table, length))[1]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        length.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, eesd.attend_rows(q[:, :1], c, table, length))
    # the caller's own memory
    from paper_2406_03853_b200 import binding as b
    out = torch.full_like(q, float("nan"))
    scratch = torch.randint(0, 255, (1 << 23,), device="cuda", dtype=torch.uint8)
    L2 = ints([n, n - 100])
    again = eesd.attend_rows(q, c, table, L2, out=out, scratch=scratch)
    assert again.data_ptr() == out.data_ptr() and torch.equal(out, eesd.attend_rows(q, c, table, L2))
    assert b.lib() is not None


def test_refusals():
    c, table = new_cache(2, 32, 2, 64, 16, 32)
    k, v = rows(2, 3, 2, 64, torch.float32, 1)
    q = torch.zeros(2, 3, 4, 64, device="cuda")
    at, L = ints([0, 0]), ints([3, 3])
    bad = [lambda: c.append(k.cpu(), v, table, at), lambda: c.append(k, v.to(torch.bfloat16), table, at), lambda: c.append(k.half(), v.half(), table, at),
           lambda: c.append(k[:, :, :1], v, table, at), lambda: c.append(k, v[:, :2], table, at), lambda: c.append(k[..., :32], v[..., :32], table, at),
           lambda: c.append(k.transpose(2, 3), v, table, at), lambda: c.append(k, v, table.long(), at), lambda: c.append(k, v, table[:1], at),
           lambda: c.append(k, v, table, at.long()), lambda: c.append(k, v, table, at[:1]), lambda: c.append(k, v, table, None),
           lambda: c.append(k, v, table, at, n_rows=at[:1]), lambda: c.append(k, v, table, at, rope=torch.zeros(5, 64, 2, device="cuda")),
           lambda: c.append(k, v, table, at, rope=torch.zeros(5, 32, 2, device="cuda", dtype=torch.float64)), lambda: c.append(k, v, table, at, positions=at),
           lambda: c.append(k, v, table.t().contiguous().t(), at), lambda: c.read(table, 0), lambda: c.read(table, 4, dtype=torch.float16),
           lambda: c.read(table[0], 4), lambda: c.read(table, 4, n_ctx=at[:1]),
           lambda: eesd.attend_rows(q, None, table, L), lambda: eesd.attend_rows(q.double(), c, table, L), lambda: eesd.attend_rows(q[:, :, :3], c, table, L),
           lambda: eesd.attend_rows(torch.zeros(2, 17, 4, 64, device="cuda"), c, table, L), lambda: eesd.attend_rows(q, c, table, None),
           lambda: eesd.attend_rows(q, c, table, L, visible=L), lambda: eesd.attend_rows(q, c, table, L, out=q[:, :2]),
           lambda: eesd.attend_rows(q, c, table, L, out=torch.zeros_like(q, dtype=torch.bfloat16)), lambda: eesd.attend_rows(q[:, :0], c, table, L),
           lambda: eesd.KV4Cache(4, 2, 64, buffer=torch.zeros(8, dtype=torch.uint8, device="cuda"))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} went through")
    for f in (lambda: eesd.KV4Cache(4, 2, 96), lambda: eesd.KV4Cache(4, 2, 64, page_tokens=8), lambda: eesd.KV4Cache(4, 2, 64, group=128), lambda: eesd.KV4Cache(0, 2, 64),
              lambda: eesd.attend_rows(q, c, table, L, scale=0.0), lambda: eesd.attend_rows(q, c, table, L, scale=math.nan),
              lambda: eesd.attend_rows(torch.zeros(2, 1, 4, 64, device="cuda"), c, torch.zeros(2, 99999, dtype=torch.int32, device="cuda"), L,
                                       scratch=torch.zeros(16, dtype=torch.uint8, device="cuda")),
              lambda: c.read(torch.zeros(1025, 1, dtype=torch.int32, device="cuda"), 1)):
        with pytest.raises(eesd.EesdError):
            f()


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("room", [0, 30000])
def test_largest_and_smallest_keys_and_values(a, room):
    """values of 2^87 and 2^-100, keys of 2^80 and 2^-80 with queries that bring the scores back"""
    B, R, H, Hkv, D, n = 1, 3, 4, 2, 128, 700
    k, v = rows(B, n, Hkv, D, torch.float32, 3)
    v = v / v.abs().max()
    q = torch.randn(B, R, H, D, generator=gen(4), device="cuda")
    for ek, ev in ((80, 87), (-80, -100), (0, 87), (0, -100)):
        c, table = new_cache(B, n, Hkv, D, 16, 64, garbage=True)
        c.append(k * 2.0 ** ek, v * 2.0 ** ev, table, ints([0]))
        out = check_attend(c, table, (q * 2.0 ** -ek).to(DT[a]), [n], room=room)
        assert out.abs().max() > 2.0 ** (ev - 8)


def test_more_segments_than_blocks_and_one_of_many_parts():
    """runs that hold many whole segments and pieces of two; one segment that every block has a part of"""
    D = 64
    B, R, H, Hkv = 40, 2, 10, 5
    lengths = [(37 * b) % 300 + 1 for b in range(B)]
    c, table = new_cache(B, 304, Hkv, D, 16, 32)
    k, v = rows(B, 304, Hkv, D, torch.bfloat16, 3)
    c.append(k, v, table, ints([0] * B))
    q = torch.randn(B, R, H, D, generator=gen(4), device="cuda")
    check_attend(c, table, q, lengths, room=4000)
    check_attend(c, table, q, lengths, n_rows=[b % 3 for b in range(B)], visible=ints([[1, 3]] * B), room=4000)
    c, table = new_cache(1, 70001, 1, D, 128, 64)
    k, v = rows(1, 70001, 1, D, torch.bfloat16, 5)
    c.append(k, v, table, ints([0]))
    for a in ("f32", "bf16"):
        for rows_, heads in ((1, 3), (3, 4), (16, 3)):
            check_attend(c, table, torch.randn(1, rows_, heads, D, generator=gen(6), device="cuda").to(DT[a]), [70001], room=1000)


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("n", [16, 200, 3000])
@pytest.mark.parametrize("room", [0, 30000])
def test_a_large_value_leaves_what_it_does_not_touch(a, n, room):
    """a token whose scale is far above the others', with a code that stands for 0 (and is not 0): its dimensions are the other tokens' alone"""
    D = 128
    k, v = rows(1, n, 1, D, torch.float32, 11)
    q = torch.randn(1, 1, 2, D, generator=gen(12), device="cuda").to(DT[a])
    for big in (1e2, 1e3, 1e4, 1e5):
        v2 = v.clone()
        v2[:, 5] *= big
        v2[:, 5, :, :96] = 0
        v2[:, 5, :, 96], v2[:, 5, :, 97] = 3 * big, -3 * big
        c, table = new_cache(1, n, 1, D, 16, 128)
        c.append(k * 0.1, v2, table, ints([0]))
        assert c.read(table, n)[1][0, 5, 0, :96].eq(0).all()
        check_attend(c, table, q, [n], room=room)


def test_tables_of_16_million_pages():
    """more tiles than 31 bits count, most of them in pages that do not exist: the same bits as with a narrow table, and a context of 2^31 - 1 tokens"""
    D, Hkv, page, n = 64, 2, 128, 700
    c, table = new_cache(1, n, Hkv, D, page, 64)
    k, v = rows(1, n, Hkv, D, torch.float32, 3)
    c.append(k, v, table, ints([0]))
    wide = torch.full((1, 1 << 24), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    narrow = torch.nn.functional.pad(table, (0, 30000), value=-1)
    for a in ("f32", "bf16"):
        q = torch.randn(1, 16, 16, D, generator=gen(4), device="cuda").to(DT[a])
        assert torch.equal(eesd.attend_rows(q, c, wide, ints([n])), eesd.attend_rows(q, c, narrow, ints([n])))
    # the same heads eight times: 2^31 tiles to look for
    c16 = eesd.KV4Cache(8, 16, D, page_tokens=page, group=64)
    t16 = ints([[5, 0, 3, 7, 1]])
    c16.append(k.repeat(1, 1, 8, 1)[:, :640], v.repeat(1, 1, 8, 1)[:, :640], t16, ints([0]))
    wide[:, :6] = -1
    wide[:, :5] = t16
    q = torch.randn(1, 1, 16, D, generator=gen(5), device="cuda")
    got = eesd.attend_rows(q, c16, wide, ints([2 ** 31 - 1]))
    kk, vv = c16.read(t16, 640)
    want, A, S = ref.attend(q, kk.double(), vv.double(), [640], None, D ** -0.5)
    assert ((got.double() - want).abs() <= ref.bound(want, A, S, 640, D, torch.float32)).all()
    assert c16.read(wide, 3, start=ints([2 ** 31 - 4]))[0].eq(0).all()


def test_binding_refusals():
    c, table = new_cache(2, 64, 2, 64, 16, 32)
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    k, q, at = z(2, 3, 2, 64), z(2, 3, 4, 64), ints([0, 0])
    rope = z(80, 32, 2)
    for kw in (dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=96), dict(page_tokens=8), dict(group=128)):
        with pytest.raises(eesd.EesdError):
            eesd.KV4Cache(**{**dict(n_pages=2, n_kv_heads=2, head_dim=64), **kw})
    for bad in (z(10, dtype=torch.uint8), z(c.layout.total_bytes), z(2, c.layout.total_bytes, dtype=torch.uint8), torch.zeros(c.layout.total_bytes, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            eesd.KV4Cache(c.n_pages, 2, 64, group=32, buffer=bad)
    shared = (dict(page_table=table.long()), dict(page_table=table.cpu()), dict(page_table=table[:1]), dict(page_table=table[0]), dict(page_table=table[:, :0]), dict(page_table=table[:1].expand(2, -1)),
              dict(page_table=table.t().contiguous().t()), dict(page_table=None), dict(rope=rope.double()), dict(rope=rope[:, :16]), dict(rope=rope[0]), dict(rope=rope[::2]), dict(rope=rope.cpu()),
              dict(positions=z(2, 3)), dict(positions=z(2, 2, dtype=torch.int32)), dict(n_rows=z(3, dtype=torch.int32)), dict(n_rows=[1, 1]), dict(n_rows=at.long()))
    call = dict(k=k, v=k, page_table=table, start=at, n_rows=None, rope=None, positions=None)
    for kw in shared + (dict(k=k.half()), dict(k=k.bfloat16()), dict(k=q), dict(v=q), dict(k=k[:, :0]), dict(k=k[..., ::2]), dict(k=k.cpu()), dict(k=k[0]), dict(v=k[:, :2]), dict(v=k[:1]), dict(v=None),
                        dict(start=None), dict(start=at[:1]), dict(start=at.float())):
        with pytest.raises(ValueError):
            c.append(**{**call, **kw})
    call = dict(q=q, cache=c, page_table=table, n_ctx=at, n_rows=None, scale=None, visible=None, rope=None, positions=None, out=None, scratch=None)
    for kw in shared + (dict(q=q.half()), dict(q=q[:, :, :3]), dict(q=z(2, 17, 4, 64)), dict(q=z(2, 3, 4, 32)), dict(q=q.cpu()), dict(q=None), dict(cache=table), dict(n_ctx=None), dict(n_ctx=at[:1]),
                        dict(visible=z(2, 3)), dict(visible=ints([[1, 1]] * 2)), dict(out=q.bfloat16()), dict(out=q[:1]), dict(out=z(2, 3, 64, 4).transpose(2, 3)), dict(out=q.cpu()), dict(scratch=z(64)),
                        dict(scratch=z(64, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            eesd.attend_rows(**{**call, **kw})
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(out=z(2 * 3 * 4 * 64 + 1)[1:].view(2, 3, 4, 64)),
               dict(page_table=torch.nn.functional.pad(table, (0, 99999)), scratch=z(64, dtype=torch.uint8))):
        with pytest.raises(eesd.EesdError):
            eesd.attend_rows(**{**call, **kw})
    for kw in (dict(page_table=table[0]), dict(page_table=None), dict(count=0), dict(start=at[:1]), dict(n_ctx=at.long()), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            c.read(**{**dict(page_table=table, count=4), **kw})
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,group", [(64, 64), (128, 32)])
def test_long_reads_are_those_of_their_parts(D, group, dtype):
    """many tiles, of which a block takes several: the same values as in short reads, starts inside tiles, before the first position and past the context"""
    B, Hkv, n = 9, 2, 9000
    c, table = new_cache(B, n, Hkv, D, 32, group, garbage=True)
    k, v = rows(B, n, Hkv, D, torch.bfloat16, 3)
    c.append(k, v, table, ints([0] * B))
    table[3, 7] = -1
    start, n_ctx = ints([0, 5, -300, 16, 4000, 8999, 15, -1, 40]), ints([9000, 8000, 777, 9000, 0, 9000, 16, 9008, 31])
    bits = torch.int32 if dtype == torch.float32 else torch.int16   # (positions never written hold anything, NaN included)
    for bound in (None, n_ctx):
        got = c.read(table, n, start=start, n_ctx=bound, dtype=dtype)
        for i in range(0, n, 500):
            for x, y in zip(got, c.read(table, 500, start=start + i, n_ctx=bound, dtype=dtype)):
                assert torch.equal(x[:, i:i + 500].view(bits), y.view(bits))
