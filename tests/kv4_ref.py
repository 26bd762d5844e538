"""The 4-bit key / value cache in 64 bits, from the storage and the formulas that include/eesd.h states: the tests' plain implementation."""
import numpy as np
import torch


def tile_bytes(D, group):
    return 16 * D + 96 * (D // group)


def decode_tile(tile, D, group):
    """bytes of a tile -> (codes, scales, zero points) of keys and values: codes [2, 16, D], scales [2, 16, G] float64, zeros [2, 16, G]"""
    G = D // group
    words = tile.view(np.uint32)
    codes = np.zeros((2, 16, D), np.int64)
    for tok in range(16):
        h, t, e = tok // 8, tok % 8 // 2, tok % 2
        for d in range(D):
            codes[0, tok, d] = words[(tok * (D // 2) + d % 32 // 8 * (D // 8) + d // 32 * 4) // 4] >> 4 * (d % 8) & 15
            codes[1, tok, d] = words[2 * D + ((d // 64 * 8 + d % 8) * 4 + t) * 4 + 2 * h + e] >> 4 * (d % 64 // 8) & 15
    w = words[4 * D:4 * D + 16 * G].reshape(G, 16)
    bits = np.stack([w << 16, w & np.uint32(0xffff0000)]).astype(np.uint32)
    scales = bits.view(np.float32).astype(np.float64).transpose(0, 2, 1)
    zeros = tile[16 * D + 64 * G:].reshape(2, G, 16).transpose(0, 2, 1).astype(np.int64)
    return codes, scales, zeros


def held(pool, table, n, Hkv, D, page, group):
    """(codes, scales, zeros) that stand at positions 0..n-1 of every sequence: [2, B, n, Hkv, D or G]"""
    pool, table = pool.cpu().numpy().reshape(-1, Hkv, page // 16, tile_bytes(D, group)), table.cpu().numpy()
    B, G = table.shape[0], D // group
    out = np.zeros((2, B, n, Hkv, D), np.int64), np.zeros((2, B, n, Hkv, G)), np.zeros((2, B, n, Hkv, G), np.int64)
    for b in range(B):
        for h in range(Hkv):
            for i in range(0, n, 16):
                tile = pool[table[b, i // page], h, i % page // 16]
                for o, x in zip(out, decode_tile(tile, D, group)):
                    o[:, b, i:i + 16, h] = x[:, :n - i]
    return out


def turn(x, rope, positions):
    """[B, rows, heads, D] fp32 turned by rope[positions[b, m]], each operation rounded to fp32"""
    cs = rope.cpu().numpy()[np.clip(positions, 0, rope.shape[0] - 1)][:, :, None]
    x = x.astype(np.float32)
    a, b, c, s = x[..., ::2], x[..., 1::2], cs[..., 0], cs[..., 1]
    out = np.empty_like(x)
    out[..., ::2], out[..., 1::2] = a * c - b * s, a * s + b * c
    return out


def quantize(w, group):
    """[.., D] fp32 -> (codes, scales, zeros), exactly (integers and fractions where it matters)"""
    from fractions import Fraction
    w = np.asarray(w, np.float32)
    shape = w.shape[:-1] + (w.shape[-1] // group, group)
    w = w.reshape(shape)
    codes, scales, zeros = np.zeros(shape, np.int64), np.zeros(shape[:-1]), np.zeros(shape[:-1], np.int64)

    def rn(f):   # nearest integer, ties to even
        return round(f)

    for i in np.ndindex(*shape[:-1]):
        g = w[i]
        if not np.isfinite(g).all():
            scales[i] = np.nan
            continue
        lo, hi = Fraction(float(min(g.min(), 0))), Fraction(float(max(g.max(), 0)))
        s = bf16_nearest((hi - lo) / 15)
        scales[i] = float(s)
        if s:
            z = min(max(rn(-lo / s), 0), 15)
            zeros[i] = z
            codes[i] = [min(max(rn(Fraction(float(x)) / s) + z, 0), 15) for x in g]
    return codes.reshape(codes.shape[:-2] + (-1,)), scales, zeros


def bf16_nearest(f):
    """the bf16 nearest to a fraction >= 0 (ties to even), as a fraction"""
    from fractions import Fraction
    if f == 0:
        return f
    e = -133   # the step of subnormals
    while f / Fraction(2) ** e >= 256:
        e += 1
    return round(f / Fraction(2) ** e) * Fraction(2) ** e


def values(codes, scales, zeros, group):
    with np.errstate(invalid="ignore"):
        return (codes - zeros.repeat(group, -1)) * scales.repeat(group, -1)


def attend(q, k, v, n_ctx, n_rows, scale, visible=None):
    """q [B, R, H, D] (turned), k, v [B, n, Hkv, D] float64 on any device, -> out and what tolerances are made of: A = sum p |v| [B, R, H, D], and of
    each row and head [B, R, H] the largest sum |q k| scale, the largest p |v|, the largest (max |q|) sum |k| scale, and sum p max |v|"""
    B, R, H, D = q.shape
    share = H // k.shape[2]
    out, A = (torch.zeros(B, R, H, D, dtype=torch.float64, device=k.device) for _ in range(2))
    S, most, Q, M = (torch.zeros(B, R, H, dtype=torch.float64, device=k.device) for _ in range(4))
    for b in range(B):
        n = R if n_rows is None else min(max(int(n_rows[b]), 0), R)
        L = int(n_ctx[b])
        p = torch.arange(k.shape[1], device=k.device)
        for m in range(n):
            if visible is None:
                seen = p <= L - n + m
            else:
                bits = int(visible[b, m]) & 0xffffffff
                own = torch.tensor([bits >> j & 1 for j in range(n)], dtype=torch.bool, device=k.device)
                new = p - (L - n)
                seen = (new < 0) | ((new >= 0) & (new < n) & own[new.clamp(0, n - 1)])
            if not bool(seen.any()):
                continue
            kk, vv = k[b, seen].repeat_interleave(share, 1), v[b, seen].repeat_interleave(share, 1)
            qq = q[b, m].double()
            x = scale * torch.einsum("hd,phd->hp", qq, kk)
            w = torch.softmax(x, -1)
            out[b, m], A[b, m] = torch.einsum("hp,phd->hd", w, vv), torch.einsum("hp,phd->hd", w, vv.abs())
            S[b, m] = scale * torch.einsum("hd,phd->hp", qq.abs(), kk.abs()).amax(-1)
            Q[b, m] = scale * qq.abs().amax(-1) * kk.abs().sum(-1).amax(0)
            most[b, m], M[b, m] = (w.t()[..., None] * vv.abs()).amax((0, 2)), (w.t() * vv.abs().amax(-1)).sum(0)
    return out, A, (S, most, Q, M)


def bound(out, A, of_rows, n, D, dtype):
    """How far attend_rows may be.  Scores: whole numbers up to the scales; queries are off by half a step of 2^-22 (bf16: 2^-14) of their row's largest at most (the largest
    is at least half of 127 * 65536, or 127 * 256, steps), and up to 4 groups' sums, two conversions and products are rounded to fp32: 16 * 2^-24.  Exponentials by
    2^-22, numerators by 2^-21 (bf16: 2^-11) and each by 2^-28 of the largest product with a value (a group's largest value is at least 7.5 scales, a
    code at most 15).  Sums over n positions take two steps per 16 of them, and 64 for joining.  bf16 sums 64 + c and 64 + z, at most 79 where the largest value is at least 7.5 scales: two
    sums of 10.5 of it, each of n / 128 + 1 steps (eight warps or more share the positions), 21 (n / 128 + 1) <= 1.1 (n / 8 + 64) up to 1800 positions, and
    more blocks share them beyond; the result is rounded to its type."""
    S, most, Q, M = of_rows
    f32 = dtype == torch.float32
    dx = S * 2.0 ** -20 + Q * 2.0 ** (-22 if f32 else -14)
    steps = (n / 8 + 64) * 2.0 ** -23
    rel = 2 * dx + 2.0 ** -22 + (2.0 ** -21 if f32 else 2.0 ** -11) + steps
    return A * rel[..., None] * (1 + 1e-3) + (n * 2.0 ** -28 * most + (0 if f32 else steps * 1.1 * M))[..., None] + (2.0 ** -24 if f32 else 2.0 ** -8) * out.abs() + 1e-37
