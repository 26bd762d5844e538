"""A decode round put together from the 4-bit operators: projections, the cache they write into, attention over it, logit rules and acceptance."""
import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd
from tests import kv4_ref as ref
from tests.test_gpu_kv4 import check_held, gen, ints, new_cache, rope_table

pytestmark = pytest.mark.gpu

H, HKV, D, GROUP, PAGE, HIDDEN, VOCAB = 8, 2, 64, 32, 16, 256, 96
LAYERS = 2


class Model:
    """embedding, layers of (projection, attention, projection, residual), head: 4-bit matrices, a cache a layer"""

    def __init__(self, seed, B, tokens):
        g = gen(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.embed = r(VOCAB, HIDDEN)
        self.qkv = [eesd.W4Matrix.quantize(r((H + 2 * HKV) * D, HIDDEN) / 16, group=64) for _ in range(LAYERS)]
        self.o = [eesd.W4Matrix.quantize(r(HIDDEN, H * D) / 16, group=64) for _ in range(LAYERS)]
        self.head = eesd.W4Matrix.quantize(r(VOCAB, HIDDEN) / 8, group=64)
        self.caches, self.tables = zip(*(new_cache(B, tokens, HKV, D, PAGE, GROUP, seed=i, garbage=True) for i in range(LAYERS)))
        self.rope = rope_table(tokens, D)

    def rows(self, tokens, at, visible=None, positions=None, seen=None):
        """tokens [B, R] at places at .. at + R - 1 of their sequences -> logits [B, R, VOCAB]; seen(layer, q, k, v, attention) looks on"""
        B, R = tokens.shape
        x = self.embed[tokens.long()]
        for l in range(LAYERS):
            qkv = eesd.project_rows(x.reshape(B * R, HIDDEN), self.qkv[l]).view(B, R, -1)
            q, k, v = (t.unflatten(-1, (-1, D)) for t in qkv.split([H * D, HKV * D, HKV * D], -1))
            self.caches[l].append(k, v, self.tables[l], at, rope=self.rope, positions=positions)
            y = eesd.attend_rows(q, self.caches[l], self.tables[l], at + R, rope=self.rope, visible=visible, positions=positions)
            if seen:
                seen(l, q, k, v, y)
            x = x + eesd.project_rows(y.reshape(B * R, H * D), self.o[l]).view(B, R, HIDDEN)
        return eesd.project_rows(x.reshape(B * R, HIDDEN), self.head).view(B, R, VOCAB)


def checker(m, at, R, visible=None, positions=None):
    """each layer's cache against exact quantisation, its attention against 64 bits over what stands there"""
    where = np.array([[a + i for i in range(R)] for a in at]) if positions is None else positions.cpu().numpy()

    def seen(l, q, k, v, y):
        check_held(m.caches[l], m.tables[l], k, v, at, m.rope, ints(where.tolist()))
        n = max(at) + R
        kk, vv = m.caches[l].read(m.tables[l], n)
        qq = torch.from_numpy(ref.turn(q.cpu().numpy(), m.rope, where)).cuda()
        want, A, S = ref.attend(qq, kk.double(), vv.double(), [a + R for a in at], None, D ** -0.5, visible)
        assert ((y.double() - want).abs() <= ref.bound(want, A, S, n, D, torch.float32)).all(), l

    return seen


def test_rounds_of_two_sequences():
    """a text in passes of 8, 5 and 1 rows, the last ones rewritten after a refusal; the first layer's cache is that of one pass"""
    B, n = 2, 40
    m, once = Model(1, B, 64), Model(1, B, 64)
    text = torch.randint(0, VOCAB, (B, n), generator=gen(2), device="cuda")
    place = 0
    while place < n:
        R = 8 if place < 24 else 5 if place + 5 <= n else 1
        if place == 29:   # a guess that is refused: its rows are written over
            m.rows((text[:, place:place + R] + 1) % VOCAB, ints([place, place]))
        logits = m.rows(text[:, place:place + R], ints([place, place]), seen=checker(m, [place] * B, R))
        assert logits.isfinite().all()
        place += R
    for i in range(0, n, 8):
        once.rows(text[:, i:i + 8], ints([i, i]))
    for x, y in zip(m.caches[0].read(m.tables[0], n), once.caches[0].read(once.tables[0], n)):
        assert torch.equal(x, y)   # (a projected row does not depend on the rows beside it, nor a quantised one)


def test_tree_then_its_accepted_path():
    """a tree of 7 rows (two candidates a position), then its accepted path written again as a chain: the next row's logits agree with those of the tree"""
    B, n = 2, 19
    m = Model(3, B, 48)
    text = torch.randint(0, VOCAB, (B, n), generator=gen(4), device="cuda")
    for i in (0, 8, 16):
        m.rows(text[:, i:i + 8], ints([i, i]))
    depth = [0, 1, 1, 2, 2, 3, 3]
    parent = [None, 0, 0, 1, 1, 3, 3]

    def path(i):
        return ([] if parent[i] is None else path(parent[i])) + [i]

    visible = ints([[sum(1 << j for j in path(i)) for i in range(7)]] * B)
    positions = ints([[n + d for d in depth]] * B)
    tokens = torch.randint(0, VOCAB, (B, 7), generator=gen(5), device="cuda")
    logits = m.rows(tokens, ints([n, n]), visible, positions, checker(m, [n, n], 7, visible, positions))
    taken = path(6)
    again = m.rows(tokens[:, taken], ints([n, n]), seen=checker(m, [n, n], len(taken)))
    # what both read is the same but for the second layer's codes of rows whose attention was summed in another order: fp32 rounding, or a code's step
    off = (again - logits[:, taken]).abs().max() / logits.abs().max()
    assert torch.equal(again.argmax(-1), logits[:, taken].argmax(-1)) and off < 0.05
    # logit rules and greedy acceptance go on from here
    rules = eesd.LogitRules(mask=ints([[[-1, -1, 0x7fffffff]] * 4] * B))
    out = eesd.process_logits(again.contiguous(), rules)
    assert out[..., 95].eq(float("-inf")).all() and out[..., :95].eq(again[..., :95]).all()


def test_captured_round_goes_on():
    """a captured round of 3 rows, replayed as the text grows over pages' ends, has the bits of the same round called; two graphs at once on their own caches"""
    models = [Model(6, 1, 96) for _ in range(3)]
    at, tokens = [ints([20]) for _ in models], [torch.zeros(1, 3, dtype=torch.int32, device="cuda") for _ in models]
    text = torch.randint(0, VOCAB, (1, 96), generator=gen(7), device="cuda", dtype=torch.int32)
    for m in models:
        m.rows(text[:, :10], ints([0]))
        m.rows(text[:, 10:20], ints([10]))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for m, a, t in zip(models, at, tokens):
            m.rows(t, a)
    torch.cuda.synchronize()
    graphs, got = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(models[i].rows(tokens[i], at[i]))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for place in range(20, 90, 3):
        for a, t in zip(at, tokens):
            a.fill_(place)
            t.copy_(text[:, place:place + 3])
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        want = models[2].rows(tokens[2], at[2])
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1], want), place
