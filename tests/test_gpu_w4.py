"""4-bit weights on the GPU: quantisation, storage, dequantisation and the skinny projection against plain 64-bit
implementations.

Quantisation is integer work on exactly rounded quotients, so codes, scales, zero points and values are compared for
equality.  The projection's bound, per output, with S = sum |A| |value| over the row: an activation is rounded to a multiple of a
power of two 2^-f, the smallest (f <= 126) with the largest of its row's 128 columns at most 8355711 (up to 4 rows 2139062016) of them, so
it is off by at most half a multiple: 1 / 8355711 (1 / 2139062016) of that largest, or 2^-127; sums of products within a group are exact integers; joining up to four digits, the scale and the addition to the total round
once each, 6 * 2^-24 of at most S for each of the row's groups; 8 slices of K, 16 warps' parts and their joins: 26 * 2^-24 S."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def quantize_ref(w, group, scale_dtype, zp):
    """codes, scales, zeros (int arrays and float64) of w (float64 [R, K]) by the definition"""
    R, K = w.shape
    codes, scales, zeros = np.zeros((R, K), np.int64), [], []
    for k in range(0, K, group):
        p = w[:, k:k + group]
        lo, hi = np.minimum(p.min(1), 0), np.maximum(p.max(1), 0)
        x = (hi - lo) / 15 if zp else np.maximum(hi, -lo) / 7
        m, e = np.frexp(x)
        bits = np.where(e < -125, (24 if scale_dtype == "f32" else 8) - (-125 - e), 24 if scale_dtype == "f32" else 8)   # subnormals have fewer
        s = np.ldexp(np.round(m * 2.0 ** bits), e - bits)
        d = np.where(s > 0, s, 1)[:, None]
        z = np.clip(np.round(-lo[:, None] / d), 0, 15) if zp else np.full((R, 1), 8.0)
        z = np.where(s[:, None] > 0, z, 0 if zp else 8)
        q = np.clip(np.round(p / d) + z, 0, 15) if zp else np.clip(np.round(p / d), -8, 7) + 8
        codes[:, k:k + group] = np.where(s[:, None] > 0, q, z)
        scales.append(s)
        zeros.append(z[:, 0])
    return codes, np.stack(scales, 1), np.stack(zeros, 1)


def weights(R, K, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(R, K, generator=g, device="cuda") * 0.02).to(dtype)


def check_quantize(w, group, scale, zp):
    m = eesd.W4Matrix.quantize(w, group=group, scale_dtype=DT[scale], zero_point=zp)
    codes, scales, zeros = quantize_ref(w.double().cpu().numpy(), group, scale, zp)
    np.testing.assert_array_equal(m.scales().double().cpu().numpy(), scales)
    if zp:
        np.testing.assert_array_equal(m.zeros().cpu().numpy(), zeros)
    np.testing.assert_array_equal(m.codes().cpu().numpy(), codes)
    K = w.shape[1]
    v64 = (codes - np.repeat(zeros, group, 1)[:, :K]) * np.repeat(scales, group, 1)[:, :K]
    v = torch.from_numpy(v64).float()   # one rounding
    assert torch.equal(m.dense().cpu(), v)
    assert torch.equal(m.dense(torch.bfloat16).cpu(), v.to(torch.bfloat16))
    return m


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("scale", ["f32", "bf16"])
@pytest.mark.parametrize("w", ["f32", "bf16"])
@pytest.mark.parametrize("R,K,group", [(16, 64, 32), (1, 1, 32), (1, 129, 128), (17, 63, 64), (33, 65, 64), (40, 1000, 128), (688, 256, 32), (129, 2050, 32)])
def test_quantize_is_exact(R, K, group, w, scale, zp):
    check_quantize(weights(R, K, DT[w], seed=R + K), group, scale, zp)


@pytest.mark.parametrize("zp", [False, True])
@pytest.mark.parametrize("scale", ["f32", "bf16"])
def test_quantize_ties_borders_and_odd_groups(scale, zp):
    R, K = 32, 128
    w = torch.zeros(R, K)
    half = torch.arange(K).float() % 29 / 2 - 7           # halves: every quotient is a tie or an integer when the scale is 1
    w[0] = half.clamp(-7, 7)
    w[1] = (half + 7).clamp(0, 15) * 1.0
    w[1, 5] = 15.0
    w[2] = half.clamp(-7, 7) * (1 + 2 ** -8)              # scale not representable in bf16
    w[3] = torch.nextafter(half.clamp(-7, 7), torch.full((K,), 9.0))    # one step beside the ties
    w[4] = torch.nextafter(half.clamp(-7, 7), torch.full((K,), -9.0))
    w[5] = 1e-40                                          # subnormal scale
    w[6, 7] = 3e38
    w[6, 8] = -3e38                                       # the range passes the largest fp32
    w[7] = 1e-45
    w[8] = -torch.rand(K, generator=torch.Generator().manual_seed(1))     # one sign only
    w[9] = torch.rand(K, generator=torch.Generator().manual_seed(2))
    w[10, 127] = -8.0
    w[12:] = torch.randn(R - 12, K, generator=torch.Generator().manual_seed(3)) * torch.exp(torch.linspace(-60, 60, R - 12))[:, None]
    if zp:
        w[6, 8] = -1.0   # (hi - lo fits)
    check_quantize(w.cuda(), 32, scale, zp)
    check_quantize(w.cuda(), 128, scale, zp)


def test_quantize_strided_unaligned_and_not_finite():
    big = weights(40, 515, torch.float32, 5)
    for view in (big[:, 3:300], big[:, 4:260], big[::2, :129], big.to(torch.bfloat16)[:, 1:200], big.to(torch.bfloat16)[3:5, 8:136]):
        check_quantize(view, 64, "bf16", True)
    w = weights(20, 256, torch.float32, 6)
    ref = eesd.W4Matrix.quantize(w, group=64).dense()
    w[3, 70], w[5, 200], w[7, 0] = float("nan"), float("inf"), float("-inf")
    for zp in (False, True):
        d = eesd.W4Matrix.quantize(w, group=64, zero_point=zp).dense()
        bad = torch.zeros(20, 256, dtype=torch.bool, device="cuda")
        bad[3, 64:128], bad[5, 192:], bad[7, :64] = True, True, True
        assert torch.equal(d.isnan(), bad)
        if not zp:
            assert torch.equal(d[~bad], ref[~bad])


def random_matrix(R, K, group, scale, zp, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = -(-K // group)
    codes = torch.randint(0, 16, (R, K), generator=g, device="cuda", dtype=torch.uint8)
    scales = (0.01 * torch.exp(torch.randn(R, G, generator=g, device="cuda"))).to(DT[scale])
    zeros = torch.randint(0, 16, (R, G), generator=g, device="cuda", dtype=torch.uint8) if zp else None
    z = 8.0 if zeros is None else zeros.double().repeat_interleave(group, 1)[:, :K]
    value = (codes.double() - z) * scales.double().repeat_interleave(group, 1)[:, :K]
    return eesd.W4Matrix.from_codes(codes, scales, zeros, group=group), value, codes, scales, zeros


def check_project(m, value, A, group):
    out = eesd.project_rows(A, m)
    a = A.double()
    ref, S = a @ value.t(), a.abs() @ value.abs().t()
    M, K = A.shape
    pad = torch.nn.functional.pad(a.abs(), (0, -K % 128)).view(M, -1, 128)
    step = (pad.amax(-1) * (1 / 2139062016 if M <= 4 else 1 / 8355711) + 2.0 ** -127).repeat_interleave(128, 1)[:, :K]
    bound = step @ value.abs().t() + (6 * -(-K // group) + 26) * 2.0 ** -24 * S + 1e-44
    assert out.dtype == torch.float32 and out.shape == ref.shape
    assert bool(((out.double() - ref).abs() <= bound).all()), float(((out.double() - ref).abs() / bound).max())
    return out


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("R,K,group,scale,zp", [
    (128, 64, 32, "f32", False), (1, 1, 32, "bf16", True), (16, 63, 64, "f32", True), (130, 65, 128, "bf16", False), (1024, 256, 32, "f32", True),
    (257, 1000, 64, "bf16", True), (515, 4096, 128, "bf16", True), (100, 9000, 32, "f32", False), (4100, 1344, 64, "f32", False)])
def test_project_every_row_count(R, K, group, scale, zp, a):
    m, value, codes, scales, zeros = random_matrix(R, K, group, scale, zp, R + K)
    assert torch.equal(m.codes(), codes) and torch.equal(m.scales(), scales) and (zeros is None or torch.equal(m.zeros(), zeros))
    g = torch.Generator(device="cuda").manual_seed(K)
    for M in range(1, 17):
        A = (torch.randn(M, K, generator=g, device="cuda") * (1 + 30 * (torch.rand(1, K, generator=g, device="cuda") < 0.01))).to(DT[a])
        out = check_project(m, value, A, group)
        assert torch.equal(out, eesd.project_rows(A, m))   # the same bits every time


@pytest.mark.parametrize("R,K,group", [(15360, 5120, 128), (27648, 5120, 32), (5120, 13824, 64), (8192, 28672, 128), (32000, 8192, 128)])
def test_project_layer_shapes(R, K, group):
    m, value, *_ = random_matrix(R, K, group, "bf16", True, 1)
    for M, a in ((1, "f32"), (5, "f32"), (16, "f32"), (8, "bf16"), (11, "bf16")):
        A = torch.randn(M, K, generator=torch.Generator(device="cuda").manual_seed(M), device="cuda").to(DT[a])
        check_project(m, value, A, group)


def test_project_range_of_activations():
    # magnitudes that change along the row: later columns far larger or far smaller than the first, and from row to row
    m, value, *_ = random_matrix(96, 6000, 64, "f32", True, 9)
    for a in ("f32", "bf16"):
        A = torch.randn(6, 6000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        A[0] *= torch.exp(torch.linspace(-60, 60, 6000, device="cuda"))
        A[1] *= torch.exp(torch.linspace(60, -60, 6000, device="cuda"))
        A[2] *= 1e-37
        A[3, :5990] = 0
        A[4] = 0
        A[5] *= 1e30
        A[5, 100:] *= 1e-35
        out = check_project(m, value, A.to(DT[a]), 64)
        assert (out[4] == 0).all()


def test_project_not_finite_rows_keep_to_themselves():
    m, value, *_ = random_matrix(200, 700, 32, "bf16", False, 3)
    A = torch.randn(7, 700, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    clean = eesd.project_rows(A, m)
    A[1, 650], A[3, 0], A[6, 333] = float("nan"), float("inf"), float("-inf")
    out = eesd.project_rows(A, m)
    for i in range(7):
        if i in (1, 3, 6):
            assert out[i].isnan().all()
        else:
            assert torch.equal(out[i], clean[i])


def test_project_strided_rows_and_untouched_neighbours():
    R, K = 300, 520
    m, value, *_ = random_matrix(R, K, 128, "f32", True, 4)
    for a in ("f32", "bf16"):
        wide = torch.randn(9, 2 * K + 3, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(DT[a])
        for off in (0, 1, 2, 3, 4, 8):
            check_project(m, value, wide[:, off:off + K], 128)
        check_project(m, value, wide[::2, :K], 128)
        A = wide[:4, :K]
        out = torch.full((4, R + 5), 7.0, device="cuda")
        st = eesd.lib().eesd_w4_project_rows(torch.cuda.current_stream().cuda_stream, C.addressof(m.desc), m.buffer.data_ptr(), m.buffer.numel(),
                                             b._DTYPES[A.dtype], A.data_ptr(), A.stride(0), out.data_ptr(), R + 5, 4, None, 0)
        assert st == 0
        assert torch.equal(out[:, :R], eesd.project_rows(A, m)) and (out[:, R:] == 7.0).all()


def test_streams_and_graph_replay():
    R, K = 1024, 2048
    m, value, *_ = random_matrix(R, K, 64, "bf16", True, 8)
    w = weights(R, K, torch.bfloat16, 3)
    A = [torch.randn(5, K, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(3)]
    want = [eesd.project_rows(x, m) for x in A]
    dense = eesd.W4Matrix.quantize(w).dense()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for x, y in zip(A, want):
            assert torch.equal(eesd.project_rows(x, m), y)
    torch.cuda.synchronize()
    x, ww, g = A[0].clone(), w.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = eesd.project_rows(x, m)
        q = eesd.W4Matrix.quantize(ww)
        d, yq = q.dense(), eesd.project_rows(x, q)
    for i in range(3):
        x.copy_(A[i])
        ww.copy_(w * (i + 1))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
        if i == 0:
            assert torch.equal(d, dense)
        assert torch.equal(yq, eesd.project_rows(x, eesd.W4Matrix.quantize(ww)))


def test_refusals():
    L = eesd.lib()
    m, value, *_ = random_matrix(64, 128, 64, "f32", False, 8)
    A = torch.zeros(2, 128, device="cuda")
    out = torch.zeros(2, 64, device="cuda")
    p, n, d = m.buffer.data_ptr(), m.buffer.numel(), C.addressof(m.desc)
    s = torch.cuda.current_stream().cuda_stream
    good = dict(m=d, p=p, n=n, dt=0, A=A.data_ptr(), lda=128, out=out.data_ptr(), ldo=64, M=2, s=None, sn=0)

    def call(**kw):
        a = {**good, **kw}
        return L.eesd_w4_project_rows(s, a["m"], a["p"], a["n"], a["dt"], a["A"], a["lda"], a["out"], a["ldo"], a["M"], a["s"], a["sn"])

    assert call() == 0
    for kw in (dict(m=None), dict(p=None), dict(p=p + 4), dict(A=None), dict(A=A.data_ptr() + 2), dict(out=None), dict(M=0), dict(M=17), dict(lda=127), dict(ldo=63), dict(dt=2)):
        assert call(**kw) == -1, kw
    assert call(n=n - 1) == -2
    big, *_ = random_matrix(64, 1024, 64, "f32", False, 9)   # (5 rows x 8 blocks of 128 columns: staged in scratch)
    A5, out5, db = torch.zeros(5, 1024, device="cuda"), torch.zeros(5, 64, device="cuda"), C.addressof(big.desc)
    need = L.eesd_w4_project_scratch_bytes(db, 5)
    sc = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
    assert need > 0 and L.eesd_w4_project_scratch_bytes(db, 17) == 0 and L.eesd_w4_project_scratch_bytes(d, 5) == 0
    five = dict(m=db, p=big.buffer.data_ptr(), n=big.buffer.numel(), A=A5.data_ptr(), lda=1024, out=out5.data_ptr(), M=5)
    assert call(**five, s=sc.data_ptr(), sn=need) == 0
    assert call(**five) == -1 and call(**five, s=sc.data_ptr() + 8, sn=need) == -1 and call(**five, s=sc.data_ptr(), sn=need - 1) == -2
    assert torch.equal(eesd.project_rows(A5, big, scratch=sc), out5)
    with pytest.raises(ValueError):
        eesd.project_rows(A5, big, scratch=sc.float())
    w = torch.zeros(64, 128, device="cuda")
    assert L.eesd_w4_quantize(s, d, 0, w.data_ptr(), 127, p, n) == -1
    assert L.eesd_w4_quantize(s, d, 5, w.data_ptr(), 128, p, n) == -1
    assert L.eesd_w4_quantize(s, d, 0, None, 128, p, n) == -1
    assert L.eesd_w4_quantize(s, d, 0, w.data_ptr(), 128, p, n - 1) == -2
    assert L.eesd_w4_dequantize(s, d, p, n, 0, w.data_ptr(), 127) == -1
    assert L.eesd_w4_dequantize(s, d, p, n, 0, None, 128) == -1
    assert L.eesd_w4_pack(s, d, w.data_ptr(), w.data_ptr(), w.data_ptr(), p, n) == -1     # zero points for a symmetric matrix
    assert L.eesd_w4_pack(s, d, w.data_ptr(), None, None, p, n) == -1
    for bad in (A.double(), A[0], torch.zeros(2, 127, device="cuda"), torch.zeros(17, 128, device="cuda"), torch.zeros(0, 128, device="cuda"),
                torch.zeros(128, 2, device="cuda").t(), A.cpu()):
        with pytest.raises(ValueError):
            eesd.project_rows(bad, m)
    for bad in (w.half(), w[0], w.t()[:, :3], w.cpu(), w[:, :0]):
        with pytest.raises(ValueError):
            eesd.W4Matrix.quantize(bad)
    with pytest.raises(eesd.EesdError):
        eesd.W4Matrix.quantize(w, group=48)
    with pytest.raises(ValueError):
        eesd.W4Matrix.quantize(w, scale_dtype=torch.float16)
    with pytest.raises(ValueError):
        eesd.W4Matrix.from_codes(torch.zeros(64, 128, device="cuda", dtype=torch.uint8), torch.zeros(64, 3, device="cuda"), group=64)
    with pytest.raises(ValueError):
        eesd.W4Matrix.from_codes(torch.zeros(64, 128, device="cuda", dtype=torch.uint8), torch.zeros(64, 2, device="cuda"),
                                 torch.zeros(64, 1, device="cuda", dtype=torch.uint8), group=64)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scale", ["f32", "bf16"])
@pytest.mark.parametrize("zp", [False, True])
def test_quantize_bf16_borders(group, scale, zp):
    """bf16 weights take their extremes in pairs: every row and column decides once, and ties, subnormals and the largest values"""
    g = torch.Generator().manual_seed(7)
    w = torch.randn(64, 256, generator=g) * 0.02
    for i in range(256):                                  # each column is the largest of some row's group, with either sign
        w[i % 64, i] = (1 if i % 3 else -1) * (1 + i / 256)
    w[0] = (torch.arange(256) % 29 / 2 - 7).clamp(-7, 7)  # ties
    w[1] = 0.0
    w[2] = 1e-40
    w[3, 7], w[3, 9] = 3e38, -3e38 if not zp else -1.0
    w[4] = -w[4].abs()
    w[5] = w[5].abs()
    w[6] = torch.randn(256, generator=g) * 1e-38
    w[7] = -0.0
    check_quantize(w.to(torch.bfloat16).cuda(), group, scale, zp)
    check_quantize(w.to(torch.bfloat16).cuda()[:61, :200], group, scale, zp)


def test_two_projections_at_once_and_one_scratch_for_two_graphs():
    m, value, *_ = random_matrix(4096, 4096, 128, "bf16", True, 21)
    rows = [torch.randn(9, 4096, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(2)]
    alone = [eesd.project_rows(a, m) for a in rows]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in rows]
    for _ in range(20):
        outs = []
        for a, s in zip(rows, streams):
            with torch.cuda.stream(s):
                outs.append(eesd.project_rows(a, m))
        torch.cuda.synchronize()
        assert all(torch.equal(o, x) for o, x in zip(outs, alone))
    # the scratch's contents are irrelevant: graphs replayed one after the other can share it
    sc = torch.empty(b.lib().eesd_w4_project_scratch_bytes(m._desc_ptr, 9), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for a in rows:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(eesd.project_rows(a, m, scratch=sc))
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1):
        outs[i].zero_()
        graphs[i].replay()
        assert torch.equal(outs[i], alone[i])
    with pytest.raises(ValueError):   # one byte seen many times
        eesd.project_rows(rows[0], m, scratch=sc[:1].expand(sc.numel()))
    with pytest.raises(eesd.EesdError):   # rows that lie on one another
        eesd.project_rows(rows[0][:1].expand(3, 4096), m)
    with pytest.raises(eesd.EesdError):
        eesd.W4Matrix.quantize(rows[0][:1].expand(3, 4096))
