"""Acceptance of more drafts than a pass has rows, on masked rows: an id outside the vocabulary is rejected where it stands."""
import pytest
import torch

import paper_2406_03853_b200 as eesd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [3, 16, 17, 40])
@pytest.mark.parametrize("token", [2 ** 31 - 1, -1, 500])
def test_a_token_outside_the_vocabulary_on_a_row_without_any(K, token):
    V = 500
    p = torch.randn(1, K + 1, V, generator=torch.Generator(device="cuda").manual_seed(K), device="cuda")
    x = p[:, :K].argmax(-1).int()
    p[0, 1] = float("-inf")
    x[0, 1] = token
    n, y = eesd.accept_resample(p, p[:, :K].contiguous(), x.contiguous(), torch.zeros(1, K, device="cuda"), torch.zeros(1, device="cuda"), 0.0)
    assert n.tolist() == [1] and y.tolist() == [-1]
