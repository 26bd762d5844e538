"""Attention over the 4-bit cache: the scratch memory of a call, on streams, in graphs, from call to call."""
import ctypes as C

import pytest
import torch

import paper_2406_03853_b200 as eesd
from paper_2406_03853_b200 import binding as b
from tests.test_gpu_kv4 import DT, gen, ints, new_cache, rows

pytestmark = pytest.mark.gpu

ROOM = 30000   # entries of a page table to spare: the call is shared out by runs, which take scratch memory


def pad(table, room=ROOM):
    return torch.nn.functional.pad(table, (0, room), value=-1)


def scratch_bytes(cache, B, R, H, pages):
    return b.lib().eesd_kv4_attend_scratch_bytes(C.addressof(cache._desc), b._kv4_rows(1 << 20, pages, pages, B, R, 0, 1 << 20, 0, 0, 0), H)


class Scratch:
    """exactly the bytes that a call asks for, full of garbage, with more of it behind that has to stay"""

    def __init__(self, size, seed):
        self.all = torch.randint(0, 256, (size + 4096,), generator=gen(seed), device="cuda", dtype=torch.uint8)
        self.size, self.behind = size, self.all[size:].clone()

    def __call__(self):
        return self.all[:self.size]

    def check(self):
        assert torch.equal(self.all[self.size:], self.behind)


def filled(B, n, Hkv, D, group, seed):
    c, table = new_cache(B, n, Hkv, D, 16, group, seed=seed)
    k, v = rows(B, n, Hkv, D, torch.float32, seed)
    c.append(k, v, table, ints([0] * B))
    return c, pad(table)


@pytest.mark.parametrize("a", ["f32", "bf16"])
@pytest.mark.parametrize("D,group", [(64, 64), (128, 64)])
def test_scratch_of_exactly_its_size(D, group, a):
    """calls of unlike shapes on one scratch, one after the other: each the bits of a call that makes its own"""
    B, Hkv, n = 3, 2, 900
    c, table = filled(B, n, Hkv, D, group, 1)
    shapes = [(3, 1, 2), (3, 16, 16), (1, 5, 4), (2, 2, 10), (3, 16, 2), (1, 1, 2)]
    sizes = [scratch_bytes(c, B_, R, H, table.shape[1]) for B_, R, H in shapes]
    assert min(sizes) > 0 and len(set(sizes)) > 1
    shared, calls = Scratch(max(sizes), 3), []
    for i, ((B_, R, H), size) in enumerate(zip(shapes, sizes)):
        q = torch.randn(B_, R, H, D, generator=gen(10 + i), device="cuda").to(DT[a])
        L = ints([n - 100 * j - i for j in range(B_)])
        own = Scratch(size, 5 + i)
        want = eesd.attend_rows(q, c, table[:B_], L)
        assert torch.equal(eesd.attend_rows(q, c, table[:B_], L, scratch=own()), want)
        own.check()
        with pytest.raises(eesd.EesdError):
            eesd.attend_rows(q, c, table[:B_], L, scratch=own()[:-1])
        calls.append((q, table[:B_], L, want))
    got = [eesd.attend_rows(q, c, t, L, scratch=shared()) for _ in range(3) for q, t, L, _ in calls]   # (no synchronisation between them)
    for i, x in enumerate(got):
        assert torch.equal(x, calls[i % len(calls)][3]), i
    shared.check()


@pytest.mark.parametrize("a", ["f32", "bf16"])
def test_two_streams_with_their_own_scratch(a):
    D, Hkv, n, H = 128, 2, 1500, 16
    c, table = filled(2, n, Hkv, D, 64, 2)
    qs = [torch.randn(2, 3, H, D, generator=gen(i), device="cuda").to(DT[a]) for i in range(2)]
    L = ints([n, n - 333])
    size = scratch_bytes(c, 2, 3, H, table.shape[1])
    assert size > 0
    want = [eesd.attend_rows(q, c, table, L) for q in qs]
    scratch = [Scratch(size, 20 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(eesd.attend_rows(qs[i], c, table, L, scratch=scratch[i]()))
                got[i].append(eesd.attend_rows(qs[i], c, table, L))
    torch.cuda.synchronize()
    for i in range(2):
        scratch[i].check()
        assert all(torch.equal(x, want[i]) for x in got[i])


@pytest.mark.parametrize("given", [False, True])
def test_captured_steps_with_scratch(given):
    """a step (append, attention) of the form that takes scratch memory, captured twice and replayed in turn as the texts grow, other calls between"""
    D, Hkv, H, n = 64, 2, 8, 600
    worlds = []
    for i in range(2):
        c, table = filled(1, n + 40, Hkv, D, 32, 30 + i)
        kn, vn = rows(1, 2, Hkv, D, torch.float32, 40 + i)
        q = torch.randn(1, 2, H, D, generator=gen(50 + i), device="cuda")
        length = ints([n])
        size = scratch_bytes(c, 1, 2, H, table.shape[1])
        assert size > 0
        worlds.append((c, table, kn, vn, q, length, Scratch(size, 60 + i)))

    def step(w):
        c, table, kn, vn, q, length, s = w
        c.append(kn, vn, table, length - 2)
        return eesd.attend_rows(q, c, table, length, scratch=s() if given else None)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for w in worlds:
            step(w)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for w in worlds:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(w))
        graphs.append(g)
    for i in range(17):
        for w in worlds:
            w[5].add_(2)
        for g in graphs:
            g.replay()
        between = [eesd.attend_rows(torch.cat([w[4], w[4]], 1), w[0], w[1], w[5]) for w in worlds]   # (another shape, its own memory)
        for g in reversed(graphs):
            g.replay()
        torch.cuda.synchronize()
        for w, out in zip(worlds, outs):
            c, table, _, _, q, length, s = w
            assert torch.equal(out, eesd.attend_rows(q, c, table, length)), i
            s.check()
        assert all(x.isfinite().all() for x in between)
