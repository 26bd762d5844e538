"""The 4-bit projection over the whole range of its activations, against 64-bit sums.

Bounds, per output, with S = sum |A| |value| over the row.  An activation is two fp16 terms of 11 bits, together off by at most 2^-23 of itself
(2 units of 2^-24) while it is at least 2^-27 of the largest of its row's 128 columns, and by at most 2^-50 of that largest below.  In a group
where a single product is not 0 the tensor core's sums are exact, so what is left are fp32 roundings of 2^-24 of at most S each: one
for joining the two terms of a group, one for its scale, one for adding it to the sum, and 26 for the parts of 8 slices of K and 16
warps.  Where many products meet, the tensor core aligns the 16 products of an instruction and the
running sum to the largest of them and cuts off what lies below 2^-23 of it: 17 addends, 34 units of 2^-24, for each 16 columns of a
group, of which the two terms' sums take (1 + 2^-11) of them."""
import pytest
import torch

import paper_2406_03853_b200 as eesd

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def matrix(codes, scales, zeros, group):
    K = codes.shape[1]
    z = 8.0 if zeros is None else zeros.double().repeat_interleave(group, 1)[:, :K]
    value = (codes.double() - z) * scales.double().repeat_interleave(group, 1)[:, :K]
    return eesd.W4Matrix.from_codes(codes, scales, zeros, group=group), value


def bound_of(A, value, group, dense):
    """The bound above; a piece's floor of 2^-50 of its largest included"""
    a = A.double()
    M, K = a.shape
    pieces, groups = -(-K // 128), -(-K // group)
    largest = torch.nn.functional.pad(a.abs(), (0, pieces * 128 - K)).view(M, pieces, 128).amax(-1).repeat_interleave(128, 1)[:, :K]
    units = 2 + 3 * groups + 26 + (35 * (group // 16) if dense else 0)
    floor = torch.where(a.abs() < largest * 2.0 ** -27, largest * 2.0 ** -50, torch.zeros_like(a))
    return units * U * (a.abs() @ value.abs().t()) + floor @ value.abs().t() + 1e-44


def outliers(group, zp, factor, dense, K=384, R=64, seed=1):
    """Weights whose codes stand for 0 at one column of each 128, where the activations are `factor` times their neighbours; sparse: and
    everywhere else but at one column of each group."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = -(-K // group)
    zeros = torch.randint(0, 16, (R, G), generator=g, device="cuda", dtype=torch.uint8) if zp else None
    z = (zeros if zp else torch.full((R, G), 8, device="cuda", dtype=torch.uint8)).repeat_interleave(group, 1)[:, :K]
    big = torch.arange(0, K, 128, device="cuda") + torch.randint(0, 128, (-(-K // 128),), generator=g, device="cuda")
    codes = torch.randint(0, 16, (R, K), generator=g, device="cuda", dtype=torch.uint8)
    if not dense:
        at = torch.arange(0, K, group, device="cuda") + torch.randint(0, group, (G,), generator=g, device="cuda")
        keep = torch.zeros(K, dtype=torch.bool, device="cuda")
        keep[at] = True
        codes = torch.where(keep[None], codes, z)
    codes[:, big] = z[:, big]
    scales = 0.01 * torch.exp(torch.randn(R, G, generator=g, device="cuda"))
    A = torch.randn(16, K, generator=g, device="cuda")
    A[:, big] *= factor
    return (*matrix(codes.contiguous(), scales, zeros, group), A)


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("factor", [1.0, 1e3, 1e5, 1e7])
def test_a_large_activation_does_not_erase_its_neighbours(factor, group, zp):
    for dense in (False, True):
        m, value, A = outliers(group, zp, factor, dense)
        for M in (1, 3, 4, 5, 8, 9, 16):
            out, a = eesd.project_rows(A[:M], m), A[:M].double()
            off = (out.double() - a @ value.t()).abs() / bound_of(A[:M], value, group, dense)
            assert float(off.max()) <= 1, (M, dense, float(off.max()))


def extremes():
    """(name, activations of a row [128 + 40], code - 8 at the same columns, scales of its groups of 64): results that stay in range although
    sums before the scale, or their terms, do not"""
    n = 168
    zero = lambda: torch.zeros(n)
    out = []
    a, c = zero(), zero()
    a[5], c[5] = 3e38, 7
    out.append(("one large activation", a, c, 0.01))
    a, c = zero(), zero()
    a[3:40], c[3:40] = 2e38, 7
    a[40:60], c[40:60] = -2e38, 5
    out.append(("sums beyond the range on either side", a, c, 1e-4))
    a, c = torch.full((n,), 1e30), torch.full((n,), -3.0)
    a[[17, 140]], c[[17, 140]] = -3.4e38, 0
    out.append(("the largest where the code stands for 0", a, c, 1e3))
    a, c = zero(), torch.full((n,), 5.0)
    a[[17, 140]], c[[17, 140]] = 3.4e38, 0
    out.append(("nothing but that, and large scales", a, c, 1e38))
    a, c = torch.linspace(-1, 1, n) * 1e-30, torch.arange(n) % 15 - 7.0
    out.append(("small activations, large scales", a, c, 3e38))
    a, c = torch.linspace(-1, 1, n) * 1e37, torch.arange(n) % 15 - 7.0
    out.append(("large activations, small scales", a, c, 1e-37))
    a, c = torch.linspace(-1, 1, n) * 1e-41, torch.arange(n) % 15 - 7.0
    out.append(("subnormal activations", a, c, 1e30))
    return out


def test_nothing_overflows_before_the_scale():
    cases = extremes()
    A = torch.stack([a for _, a, _, _ in cases]).cuda()
    for i, (name, a, c, s) in enumerate(cases):
        R = 24
        codes = (c + 8).to(torch.uint8).expand(R, -1).contiguous().cuda()
        for group in (32, 64, 128):
            scales = torch.full((R, -(-len(c) // group)), s, device="cuda")
            m, value = matrix(codes, scales, None, group)
            for rows in ([i], [i] * 4, list(range(i, -1, -1)) + [i] * 6, [i] * 16):
                out = eesd.project_rows(A[rows], m)[0].double()
                ref = (A[i:i + 1].double() @ value.t())[0]
                bound = bound_of(A[i:i + 1], value, group, True)[0] + scales.double().sum(1) * 2.0 ** -149   # (a group's sum below 2^-126)
                assert bool(out.isfinite().all()), (name, group, len(rows))
                assert bool(((out - ref).abs() <= bound).all()), (name, group, len(rows), float(((out - ref).abs() / bound).max()))


@pytest.mark.parametrize("R,K,group", [(40, 300, 32), (300, 9000, 32), (4100, 5120, 64), (1000, 13824, 128), (64, 28672, 128), (8192, 28672, 128)])
def test_a_row_does_not_depend_on_the_rows_beside_it(R, K, group):
    g = torch.Generator(device="cuda").manual_seed(R)
    G = -(-K // group)
    m, _ = matrix(torch.randint(0, 16, (R, K), generator=g, device="cuda", dtype=torch.uint8), 0.01 * torch.exp(torch.randn(R, G, generator=g, device="cuda")),
                  torch.randint(0, 16, (R, G), generator=g, device="cuda", dtype=torch.uint8), group)
    A = torch.randn(16, K, generator=g, device="cuda")
    alone = torch.cat([eesd.project_rows(A[i:i + 1], m) for i in range(16)])
    for M in range(2, 17):
        assert torch.equal(eesd.project_rows(A[:M], m), alone[:M]), M
        assert torch.equal(eesd.project_rows(A[16 - M:], m), alone[16 - M:]), M
    order = torch.randperm(16, generator=g, device="cuda")
    assert torch.equal(eesd.project_rows(A[order], m), alone[order])


@pytest.mark.parametrize("R,K,group", [(80011, 200, 32), (200000, 64, 64)])
def test_more_row_blocks_than_one_round_of_blocks_takes(R, K, group):
    g = torch.Generator(device="cuda").manual_seed(K)
    G = -(-K // group)
    m, value = matrix(torch.randint(0, 16, (R, K), generator=g, device="cuda", dtype=torch.uint8), 0.01 * torch.exp(torch.randn(R, G, generator=g, device="cuda")), None, group)
    A = torch.randn(16, K, generator=g, device="cuda")
    for M in (1, 4, 7, 16):
        out = eesd.project_rows(A[:M], m)
        off = (out.double() - A[:M].double() @ value.t()).abs() / bound_of(A[:M], value, group, True)
        assert float(off.max()) <= 1, (M, float(off.max()))
