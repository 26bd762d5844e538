"""4-bit cache: numbers that the C records do not hold are refused, not cut to 32 bits."""
import pytest
import torch

import paper_2406_03853_b200 as eesd


@pytest.mark.parametrize("kw", [dict(n_pages=(1 << 32) + 4), dict(n_kv_heads=(1 << 32) + 2), dict(head_dim=(1 << 32) + 64), dict(page_tokens=(1 << 32) + 16), dict(group=(1 << 32) + 64),
                                dict(n_pages=1 << 31), dict(n_pages=-(1 << 32) + 4)])
def test_descriptions(kw):
    with pytest.raises(ValueError):
        eesd.KV4Cache(**{**dict(n_pages=4, n_kv_heads=2, head_dim=64), **kw})


@pytest.mark.gpu
def test_counts_and_scales():
    c = eesd.KV4Cache(4, 2, 64)
    table, L = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, 2, 64, device="cuda")
    for count in (1 << 31, 1 << 40):
        with pytest.raises(ValueError):
            c.read(table, count)
    for scale in (1e39, float("inf"), 1e300):
        with pytest.raises(eesd.EesdError):
            eesd.attend_rows(q, c, table, L, scale=scale)
    assert eesd.attend_rows(q, c, table, L, scale=3.4e38).eq(0).all()
