"""Attention over the 4-bit cache: results and scratch memory that lie on what the call reads are refused."""
import pytest
import torch

import paper_2406_03853_b200 as eesd
from tests.test_gpu_kv4 import gen, ints
from tests.test_gpu_kv4_workspace import filled, scratch_bytes

pytestmark = pytest.mark.gpu


def test_results_that_lie_on_what_is_read_are_refused():
    """blocks read queries after others have written results: out and scratch lie apart from what the call reads and from each other"""
    D, Hkv, H, n = 64, 2, 4, 100
    c, table = filled(2, n, Hkv, D, 64, 7)
    L = ints([n, n - 3])
    q = torch.randn(2, 3, H, D, generator=gen(1), device="cuda")
    size = scratch_bytes(c, 2, 3, H, table.shape[1])
    want = eesd.attend_rows(q, c, table, L)
    both = torch.zeros(2 * q.numel(), device="cuda")
    inside = both[:q.numel()].view_as(q).copy_(q)
    over = both[16:16 + q.numel()].view_as(q)
    work = torch.zeros(size + q.nbytes, dtype=torch.uint8, device="cuda")
    at = work[size - 16:size - 16 + q.nbytes].view(torch.float32).view_as(q)
    in_pool = c.buffer[:q.nbytes].view(torch.float32).view_as(q)
    for kw in (dict(q=q, out=q), dict(q=inside, out=over), dict(q=q, out=in_pool), dict(q=q, scratch=work[:size], out=at), dict(q=at.copy_(q), scratch=work[:size]),
               dict(q=q, scratch=c.buffer[:size] if c.buffer.numel() >= size else c.buffer)):
        with pytest.raises(ValueError):
            eesd.attend_rows(**{**dict(cache=c, page_table=table, n_ctx=L), **kw})
    # side by side is fine
    after = both[q.numel():].view_as(q)
    assert torch.equal(eesd.attend_rows(inside, c, table, L, out=after), want)
    behind = work[size:].view(torch.float32).view_as(q)
    assert torch.equal(eesd.attend_rows(q, c, table, L, out=behind, scratch=work[:size]), want)
