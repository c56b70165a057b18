"""The example that runs the operators together: a speculative step and a
tuning step (examples/draft_step.py), against the same steps in float64."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("draft_step", os.path.join(ROOT, "examples", "draft_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def test_greedy_drafts_of_the_whole_decoder_are_all_accepted(ex):
    """With one block the drafter is the decoder: at temperature 0 every draft is the target's own choice."""
    d = ex.Decoder(vocab=700, width=128, blocks=1)
    last = torch.arange(9, device="cuda")
    tokens, accepted = d.verify(last, torch.zeros(9, device="cuda"), 3, generator(2))
    assert (accepted == 3).all() and (tokens >= 0).all()
    rows = torch.cat([last[:, None], tokens[:, :3].long()], dim=1)
    assert torch.equal(tokens.long(), d.logits(rows).argmax(dim=1).view(9, 4))


def test_sampled_step(ex):
    d = ex.Decoder(vocab=900, width=128, blocks=2)
    tokens, accepted = d.verify(torch.arange(40, device="cuda"), torch.full((40,), 0.9, device="cuda"), 4, generator(3))
    tokens, accepted = tokens.cpu().numpy(), accepted.cpu().numpy()
    assert ((accepted >= 0) & (accepted <= 4)).all()
    for t, n in zip(tokens, accepted):
        assert ((t[:n + 1] >= 0) & (t[:n + 1] < 900)).all() and (t[n + 1:] == -1).all()


def test_tuning_follows_the_gradient(ex):
    """20 steps in float64 from the same start: the loss falls alike.  FP32
    keeps each step's parameters within about 1e-6 of their size, and a step's
    map stretches differences by at most 1 + rate * curvature, below 2 for the
    few steps that matter; 1e-3 relative on the loss is far outside that."""
    g = generator(4)
    Q, scale = ex.export(g, 200, 64)
    up = ex.sp.dense_fused_create(Q, scale, backward=True)
    table, bias = torch.randn((50, 64), device="cuda", generator=g), torch.zeros(200, device="cuda")
    ids = torch.randint(-1, 50, (120,), device="cuda", generator=g)
    wanted = torch.randn((120, 200), device="cuda", generator=g).abs()
    t64, b64 = table.double().cpu().numpy(), np.zeros(200)
    losses = ex.tune(table, up, bias, ids, wanted)
    Qh, sh, ih, wh = Q.cpu().numpy(), scale.double().cpu().numpy(), ids.cpu().numpy(), wanted.double().cpu().numpy()
    want = []
    for _ in range(20):
        x = so.embed_forward(t64, ih, 1.0)
        z = so.fused_pre(Qh, sh, x, b64)
        diff = so.act(z, "gelu") - wh
        want.append(0.5 * (diff ** 2).sum() / 120)
        dx, db, _ = so.fused_backward(Qh, sh, diff / 120, z, "gelu")
        t64 = t64 - 0.5 * so.embed_backward(dx, ih, 50, 1.0)
        b64 = b64 - 0.5 * db
    assert want[-1] < 0.97 * want[0]
    assert np.allclose(losses, want, rtol=1e-3)
