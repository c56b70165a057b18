"""How many bits of an operand the fused projection keeps (dense_fused.h).

Every output here has one code that is not zero, so it is a single product and
nothing of a sum's rounding hides what an operand lost.  With u = 2^-24 and q
the code:

    rows of up to FUSED_FEW_ROWS: every bit of an FP32 operand takes part; its
    parts' products (exact) are added and scaled: 4 u of the result
    more rows: an FP32 operand enters to 2^-23 of itself or 2^-39 of its row's
    largest, whichever is more; then 4 u as above

In the gradient g * scale is the operand, rounded once: 1 u more.  2^-149 (1 + |q|)
is for values that are subnormal.
"""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from tests.launches import launches
from tests.test_fused_gpu import TYPES, act_code, dev, handle, host, problem

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FEW = 32


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def one_code(r, outputs, inputs):
    """Codes [outputs][inputs] of which one in each row is not zero."""
    Q = np.zeros((outputs, inputs), np.int8)
    Q[np.arange(outputs), r.integers(0, inputs, outputs)] = r.choice([-127, -90, -3, 1, 2, 55, 100, 127], outputs)
    return Q


def columns(Q):
    return np.ascontiguousarray(Q.T)


def limit(want, operand, Q, rows, extra, scale=1.0):
    """operand: [B][n] as it enters, Q: [outputs][n] with one code a row, scale: of the outputs."""
    q = np.abs(Q.astype(np.float64)).sum(axis=1)
    lim = (4 + extra) * U * np.abs(want) + 2.0 ** -149 * (1 + q) * np.maximum(scale, 1)
    if rows > FEW:
        lim = lim + 2.0 ** -23 * np.abs(want) + 2.0 ** -39 * np.abs(operand).max(axis=1, keepdims=True) * q * scale
    return lim


SIZES = [(200, 200, 0, 0), (200, 1000, 0, 0), (96, 2100, 3, 1), (64, 8200, 0, 0), (101, 90, 0, 0)]


@pytest.mark.parametrize("B", [1, 20, 32, 33, 70, 600])
@pytest.mark.parametrize("K,M,pad,offset", SIZES)
@pytest.mark.parametrize("yk", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_gradient_operand(sp, B, K, M, pad, offset, yk, act):
    """g * scale is an FP32 value whatever the type of dy, and dx may be FP32."""
    r = np.random.default_rng([41, B, K, M])
    p = {"Q": columns(one_code(r, K, M)), "scale": r.uniform(0.5, 1.5, M).astype(np.float32)}
    dy, z = dev(r.normal(size=(B, M)), yk, pad, offset), dev(r.normal(size=(B, M)), yk, pad, offset)
    dx = torch.full((B, K), float("nan"), device="cuda")
    h = handle(sp, p, backward=True)
    sp.dense_fused_backward(h, dy, dx=dx, pre=z if act != "none" else None, act=act_code(sp, act))
    torch.cuda.synchronize()
    want, _, g = so.fused_backward(p["Q"], np.ones(M), host(dy) * p["scale"].astype(np.float64), host(z), act)
    lim = limit(want, g, columns(p["Q"]), B, 1)
    got = host(dx)
    assert (np.abs(got - want) <= lim).all(), np.nanmax(np.abs(got - want) / lim)
    h.close()


def wide(r, B, n):
    """FP32 values of every size up to 1e34, subnormal ones among them."""
    x = r.uniform(1, 2, (B, n)) * r.choice([-1, 1], (B, n)) * 10.0 ** r.uniform(-44, 33, (B, n))
    return x.astype(np.float32)


@pytest.mark.parametrize("B", [1, 16, 20, 32, 33, 300])
@pytest.mark.parametrize("K,M", [(130, 130), (300, 5000), (64, 33000)])
def test_wide_activations(sp, B, K, M):
    """FP32 activations of any size beside each other: up to FUSED_FEW_ROWS rows keep all of their bits."""
    r = np.random.default_rng([42, B, K, M])
    p = {"Q": one_code(r, M, K), "scale": r.uniform(0.5, 1.5, M).astype(np.float32)}
    x, y = dev(wide(r, B, K)), torch.full((B, M), float("nan"), device="cuda")
    h = handle(sp, p)
    sp.dense_fused_forward(h, x, y)
    torch.cuda.synchronize()
    want = so.fused_pre(p["Q"], p["scale"], host(x))
    lim = limit(want, host(x), p["Q"], B, 0, p["scale"].astype(np.float64))
    got = host(y)
    assert (np.abs(got - want) <= lim).all(), np.nanmax(np.abs(got - want) / lim)
    h.close()


@pytest.mark.parametrize("B", [1, 32, 33, 300])
def test_wide_gradients(sp, B):
    r = np.random.default_rng([43, B])
    p = {"Q": columns(one_code(r, 150, 150)), "scale": (2.0 ** r.integers(-3, 3, 150)).astype(np.float32)}
    dy, dx = dev(wide(r, B, 150)), torch.full((B, 150), float("nan"), device="cuda")
    h = handle(sp, p, backward=True)
    sp.dense_fused_backward(h, dy, dx=dx)
    torch.cuda.synchronize()
    want, _, _ = so.fused_backward(p["Q"], p["scale"], host(dy))
    # (g * scale rounds to a multiple of 2^-149 where it is subnormal)
    lim = limit(want, host(dy) * p["scale"], columns(p["Q"]), B, 1) + 2.0 ** -149 * 127
    got = host(dx)
    assert (np.abs(got - want) <= lim).all(), np.nanmax(np.abs(got - want) / lim)
    h.close()


@pytest.mark.parametrize("B", [33, 63, 64, 200, 700])
@pytest.mark.parametrize("K,M,pad,offset", [(1024, 1280, 0, 0), (1100, 1300, 3, 1), (1023, 1280, 0, 0), (1024, 1279, 0, 0), (2100, 8300, 0, 0)])
@pytest.mark.parametrize("xk", ["f32", "bf16"])
def test_bf16_gradient_in_both_forms(sp, B, K, M, pad, offset, xk):
    """Planes apart and side by side, at the sizes where one follows the other: integers exactly, each operand's bits."""
    r = np.random.default_rng([44, B, K, M])
    p = problem(K, M, B, integer=True)
    h = handle(sp, p, backward=True)
    dy, dx = dev(p["dy"], "bf16", pad, offset), dev(np.full((B, K), np.nan), xk, pad, offset)
    db = torch.full((M,), float("nan"), device="cuda")
    ws = torch.full((sp.dense_fused_workspace_bytes(h, B, torch.bfloat16),), 255, dtype=torch.uint8, device="cuda")  # (NaN)
    names = [n for n, _, _ in launches(lambda st: sp.dense_fused_backward(h, dy, dx=dx, dbias=db, workspace=ws, stream=st))]
    planes = 2 if M >= 1280 and K >= 1024 and B >= 64 else 1
    assert any(f"k_fused_tileIDF16_Li{planes}E" in n for n in names), names
    sp.dense_fused_backward(h, dy, dx=dx, dbias=db, workspace=ws)
    torch.cuda.synchronize()
    want, wb, _ = so.fused_backward(p["Q"], p["scale"], host(dy))
    assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[xk])) and (db.cpu().numpy() == wb).all()
    h.close()
    p = {"Q": columns(one_code(r, K, M)), "scale": r.uniform(0.5, 1.5, M).astype(np.float32)}
    h = handle(sp, p, backward=True)
    dy, dx = dev(r.normal(size=(B, M)), "bf16", pad, offset), torch.full((B, K), float("nan"), device="cuda")
    sp.dense_fused_backward(h, dy, dx=dx)
    torch.cuda.synchronize()
    want, _, g = so.fused_backward(p["Q"], np.ones(M), host(dy) * p["scale"].astype(np.float64))
    lim = limit(want, g, columns(p["Q"]), B, 1)
    assert (np.abs(host(dx) - want) <= lim).all()
    h.close()
