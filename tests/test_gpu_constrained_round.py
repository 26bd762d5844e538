"""A decode round on 4-bit heads under logit rules, put together as a caller would: project the rows with the draft's and the
target's 4-bit heads, process both sides' logits with the same rules, draft, accept.  Each step is checked against its plain form, the
decisions against the CPU oracle on the processed logits (bit-exact), and no emitted token is one the mask forbids."""
import numpy as np
import pytest
import torch

import eesd_synth as synth
import oracle
import paper_2406_03853_b200 as eesd
from tests.helpers import engine_from_spec, oracle_from_spec
from tests.test_gpu_w4 import check_project
from tests.test_logit_rules import close, rules_ref

pytestmark = pytest.mark.gpu


def masks(B, rows, V, seed, keep=0.3):
    g = np.random.default_rng(seed)
    words = (V + 31) // 32
    bits = np.zeros((B, rows, words * 32), np.uint8)
    bits[:, :, :V] = g.random((B, rows, V)) < keep
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32), bits[:, :, :V]


@pytest.mark.parametrize("T", [0.0, 0.8])
def test_round_on_four_bit_heads(T):
    B, K, V, d, H = 3, 4, 4001, 640, 40
    rows = K + 1
    g = torch.Generator(device="cuda").manual_seed(7)
    target = eesd.W4Matrix.quantize(torch.randn(V, d, generator=g, device="cuda") * 0.05, group=64, zero_point=True)
    draft = eesd.W4Matrix.quantize(target.dense() + 0.01 * torch.randn(V, d, generator=g, device="cuda"), group=128)
    hidden = torch.randn(B * rows, d, generator=g, device="cuda")
    p = check_project(target, target.dense().double(), hidden, 64).view(B, rows, V)
    q = eesd.project_rows(hidden + 0.05, draft).view(B, rows, V)[:, :K].contiguous()

    history = torch.randint(0, V, (B, H), generator=g, device="cuda", dtype=torch.int32)
    n_prompt = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    rep = torch.tensor([1.0, 1.3, 2.0], device="cuda")
    freq = torch.tensor([0.0, 0.2, 0.5], device="cuda")
    pres = torch.tensor([0.3, 0.0, 0.1], device="cuda")
    words, allowed = masks(B, rows, V, 3)
    mask = torch.from_numpy(words).cuda()
    common = dict(history=history, n_prompt=n_prompt, repetition=rep, frequency=freq, presence=pres)
    ua, ur, ud = (torch.rand(s, generator=g, device="cuda").mul(2 ** 24).floor() / 2 ** 24 for s in ((B, K), (B,), (B, K)))

    # drafts, one step at a time: row i counts the drafts before it
    x = torch.zeros(B, K, dtype=torch.int32, device="cuda")
    qp = torch.empty_like(q)
    for i in range(K):
        step = eesd.process_logits(q[:, :i + 1].contiguous(), eesd.LogitRules(drafted=x[:, :i].contiguous(), mask=mask[:, :i + 1].contiguous(), **common))
        qp[:, i] = step[:, i]
        x[:, i] = eesd.sample_rows(step[:, i].contiguous(), None if T == 0 else ud[:, i].contiguous(), T)
    assert torch.equal(eesd.process_logits(q, eesd.LogitRules(drafted=x[:, :K - 1].contiguous(), mask=mask[:, :K].contiguous(), **common)), qp)   # all rows at once
    pp = eesd.process_logits(p, eesd.LogitRules(drafted=x, mask=mask, **common))
    host = dict(history=history.cpu().numpy(), n_prompt=n_prompt.cpu().numpy(), drafted=x.cpu().numpy(), repetition=rep.cpu().numpy(),
                frequency=freq.cpu().numpy(), presence=pres.cpu().numpy(), mask=words)
    close(pp, *rules_ref(p.cpu().numpy(), **host))

    n, y = eesd.accept_resample(pp, qp, x, ua, ur, T)
    n_ref, y_ref = oracle.accept_resample_batch(pp.cpu().numpy(), qp.cpu().numpy(), x.cpu().numpy(), ua.cpu().numpy(), ur.cpu().numpy(), T)
    np.testing.assert_array_equal(n.cpu().numpy(), n_ref)
    np.testing.assert_array_equal(y.cpu().numpy(), y_ref)
    for b in range(B):
        assert all(allowed[b, i, x[b, i]] for i in range(K)) and allowed[b, n_ref[b], y_ref[b]]


@pytest.mark.parametrize("V", [40, 1000, 32000, 40001])
def test_a_row_without_any_token_is_answered_with_minus_one(V):
    g = torch.Generator(device="cuda").manual_seed(1)
    B, K = 3, 3
    p = torch.randn(B, K + 1, V, generator=g, device="cuda")
    q = p[:, :K].clone()
    none = torch.zeros(B, K + 1, (V + 31) // 32, dtype=torch.int32, device="cuda")
    none[0], none[1, :1], none[2, :3] = -1, -1, -1          # sequence 0: all allowed; 1: row 1 and on nothing; 2: the last row nothing
    pp = eesd.process_logits(p, eesd.LogitRules(mask=none))
    x = q.argmax(-1).int().contiguous()
    ua, ur = torch.zeros(B, K, device="cuda"), torch.full((B,), 0.5, device="cuda")
    for T in (0.0, 1.0):
        rows = eesd.sample_rows(pp.view(-1, V), torch.full((B * (K + 1),), 0.25, device="cuda"), T).view(B, K + 1).cpu()
        empty = (none == 0).all(-1).cpu()
        assert (rows[empty] == -1).all() and ((rows[~empty] >= 0) & (rows[~empty] < V)).all()
        n, y = eesd.accept_resample(pp, q, x, ua, ur, T)
        assert n.tolist() == [3, 1, 3] and y[1].item() == -1 and y[2].item() == -1 and 0 <= y[0].item() < V
        # a draft row that was masked to nothing drafts -1: rejected where it stands, the next token comes from the target's row
        bad = x.clone()
        bad[0, 1] = -1
        q2 = q.clone()
        q2[0, 1] = float("-inf")
        n, y = eesd.accept_resample(pp, q2, bad, ua, ur, T)
        assert n[0].item() == 1 and 0 <= y[0].item() < V


def test_rules_on_the_engines_logits():
    # verification logits of the tiny model, processed in place where the engine left them, against the oracle's logits
    spec = synth.TINY
    eng, m = engine_from_spec(spec, max_ctx=96), oracle_from_spec(spec, 96)
    prompt = synth.prompt_tokens(3, 20, spec.vocab).numpy()
    eng.prefill(prompt)
    m.target_rows(prompt[:-1], 0, want_logits=False)
    rows = np.concatenate([prompt[-1:], synth.prompt_tokens(4, 3, spec.vocab).numpy()]).astype(np.int32)
    eng.verify_only(rows)
    _, want = m.target_rows(rows, len(prompt) - 1)
    words, allowed = masks(1, 4, spec.vocab, 9, 0.5)
    history = torch.from_numpy(prompt[None].astype(np.int32)).cuda()
    rep = torch.tensor([1.5], device="cuda")
    lg = eng.logits(0, 4)
    r = eesd.LogitRules(history=history, drafted=torch.from_numpy(rows[None, 1:]).cuda(), repetition=rep, mask=torch.from_numpy(words).cuda())
    out = eesd.process_logits(lg.view(1, 4, -1), r, out=lg.view(1, 4, -1))
    assert out.data_ptr() == lg.data_ptr()
    ref, _ = rules_ref(want[None].astype(np.float32), history=prompt[None], drafted=rows[None, 1:], repetition=np.array([1.5]), mask=words)
    got = lg.cpu().numpy()
    fin = np.isfinite(ref[0])
    assert (fin == (allowed[0] != 0)).all() and (np.isneginf(got) == ~fin).all()
    assert np.abs(got[fin] - ref[0][fin]).max() < 1.5 * 2e-2   # (the engine's own tolerance, times the largest factor of the rules)
    tok = eesd.sample_rows(lg.clone(), None, 0.0).cpu().numpy()
    assert all(allowed[0, i, t] for i, t in enumerate(tok))
    eng.close()
