"""The C entries of the 4-bit key / value cache refuse what they cannot do before anything reaches a device."""
import ctypes as C
import struct

import pytest

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b

OK, BADARG, NOMEM, UNSUPPORTED = 0, -1, -2, -8
AT = 1 << 20      # an address that nobody follows


def desc(n_pages=4, heads=2, D=64, page=16, group=32):
    return b.KV4Desc(n_pages, heads, D, page, group)


def rows(table=AT, stride=4, pages=4, B=2, rows=3, n_rope=0, at=AT, n_rows=0, rope=0, positions=0):
    return b._kv4_rows(table, stride, pages, B, rows, n_rope, at, n_rows, rope, positions)


def tensor(data=AT, sb=384, sr=128, sh=64):
    return b._kv4_tensor(data, sb, sr, sh)


def attention(r, dt, q, H, scale, vis, out, s, sn):
    return None if r is None else r + q + struct.pack("PPPNiif4x", vis, out, s, sn, dt, H, scale)


def size(d):
    l = b.KV4Layout()
    assert eesd.lib().eesd_kv4_layout_of(C.addressof(d), C.addressof(l)) == OK
    return l


@pytest.mark.parametrize("D,group,page,tile", [(64, 32, 16, 1216), (64, 64, 32, 1120), (128, 32, 64, 2432), (128, 64, 128, 2240), (128, 128, 16, 2144)])
def test_layout(D, group, page, tile):
    l = size(desc(5, 3, D, page, group))
    G = D // group
    assert (l.v_codes, l.scales, l.k_zeros, l.v_zeros, l.tile_bytes) == (8 * D, 16 * D, 16 * D + 64 * G, 16 * D + 80 * G, tile)
    assert l.page_bytes == tile * page // 16 * 3 and l.total_bytes == 5 * l.page_bytes


def test_layout_refusals():
    f, l = eesd.lib().eesd_kv4_layout_of, b.KV4Layout()
    assert f(None, C.addressof(l)) == BADARG
    for kw, want in ((dict(n_pages=0), BADARG), (dict(heads=0), BADARG), (dict(heads=65536), BADARG), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
                     (dict(page=48), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=128), UNSUPPORTED)):
        d = desc(**kw)
        assert f(C.addressof(d), C.addressof(l)) == want, kw
    assert f(C.addressof(desc(2 ** 31 - 1, 65535, 128, 128, 32)), C.addressof(l)) == OK and l.total_bytes > 1 << 60


def calls():
    L, d = eesd.lib(), desc()
    n = size(d).total_bytes
    p = C.addressof(d)
    need = L.eesd_kv4_attend_scratch_bytes(p, rows(), 4)
    assert need == 0
    append = lambda d=p, pool=AT, n=n, r=rows(), dt=0, k=tensor(), v=tensor(): L.eesd_kv4_append(None, d, pool, n, r, dt, k, v)
    read = lambda d=p, pool=AT, n=n, r=rows(), ctx=None, dt=0, k=AT, v=AT: L.eesd_kv4_read(None, d, pool, n, r, ctx, dt, k, v)
    attend = lambda d=p, pool=AT, n=n, r=rows(), dt=0, q=tensor(), H=4, scale=0.125, vis=0, out=AT, s=0, sn=0: L.eesd_kv4_attend(
        None, d, pool, n, attention(r, dt, q, H, scale, vis, out, s, sn))
    return append, read, attend, n, d


def test_entry_refusals():
    append, read, attend, n, keep = calls()
    for f in (append, read, attend):
        for kw, want in ((dict(d=None), BADARG), (dict(pool=None), BADARG), (dict(pool=AT + 8), BADARG), (dict(n=n - 1), NOMEM), (dict(r=None), BADARG), (dict(r=rows(table=0)), BADARG),
                         (dict(r=rows(table=AT + 2)), BADARG), (dict(r=rows(stride=3)), BADARG), (dict(r=rows(pages=0)), BADARG), (dict(r=rows(B=0)), BADARG),
                         (dict(r=rows(rows=0)), BADARG), (dict(r=rows(at=AT + 1)), BADARG), (dict(r=rows(B=1025)), UNSUPPORTED), (dict(dt=2), BADARG), (dict(dt=-1), BADARG),
                         (dict(r=rows(rope=AT, n_rope=0)), BADARG), (dict(r=rows(rope=AT + 4, n_rope=9)), BADARG), (dict(r=rows(n_rows=AT + 3)), BADARG), (dict(r=rows(positions=AT + 3)), BADARG)):
            assert f(**kw) == want, kw
    for kw in (dict(k=None), dict(v=None), dict(k=tensor(data=0)), dict(k=tensor(data=AT + 2)), dict(v=tensor(sb=-1)), dict(k=tensor(sr=-1)), dict(v=tensor(sh=-64)), dict(r=rows(at=0)),
               dict(dt=1, k=tensor(data=AT + 1))):
        assert append(**kw) == BADARG, kw
    assert append(r=rows(rows=2 ** 31 - 1, B=1024)) == UNSUPPORTED and read(r=rows(rows=2 ** 31 - 1, B=1024)) == UNSUPPORTED
    for kw in (dict(k=None, v=None), dict(k=AT + 4), dict(v=AT + 8), dict(ctx=AT + 2)):
        assert read(**kw) == BADARG, kw
    for kw in (dict(q=tensor(data=0)), dict(q=tensor(sr=-1)), dict(r=rows(rows=17)), dict(H=0), dict(H=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(vis=AT + 1), dict(out=0), dict(out=AT + 8), dict(r=rows(at=0))):
        assert attend(**kw) == BADARG, kw


def test_scratch():
    L, d = eesd.lib(), desc(400, 2, 128, 16, 64)
    p, n = C.addressof(d), size(d).total_bytes
    long = rows(stride=99999, pages=99999)
    need = L.eesd_kv4_attend_scratch_bytes(p, long, 4)
    assert need > 0 and need % 16 == 0
    for bad in (dict(H=3), dict(H=0), dict(r=rows(stride=99999, pages=99999, rows=17)), dict(r=None)):
        assert L.eesd_kv4_attend_scratch_bytes(p, bad.get("r", long), bad.get("H", 4)) == 0
    f = lambda s, sn: L.eesd_kv4_attend(None, p, AT, n, attention(long, 0, tensor(), 4, 0.125, 0, AT, s, sn))
    assert f(0, need) == BADARG and f(AT + 8, need) == BADARG and f(AT, need - 1) == NOMEM


def test_attend_refuses_what_its_integers_do_not_hold():
    append, read, attend, n, keep = calls()
    wide = desc(heads=1)
    big = dict(d=C.addressof(wide), n=size(wide).total_bytes)
    assert attend(r=rows(rows=16, B=1), H=1 << 27, **big) == UNSUPPORTED            # 2^31 columns
    assert attend(r=rows(rows=16, B=1024, pages=2 ** 31 - 1, stride=2 ** 31 - 1), H=1 << 20, **big) == UNSUPPORTED
    assert eesd.lib().eesd_kv4_attend_scratch_bytes(big["d"], rows(rows=16, B=1), 1 << 27) == 0
    # the largest ranges of tokens that a table may name are not refused (no scratch memory is given)
    assert attend(r=rows(rows=1, B=1024, pages=2 ** 27, stride=2 ** 27), H=8, **big) == BADARG
