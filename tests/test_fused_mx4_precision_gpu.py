"""GPU checks of the digits that the gradient of four-bit weights keeps of g * scale (dense_fused.h): outputs whose
sums are small differences of large terms show what a term was rounded to."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from oracle import step_oracle as step
from tests.test_fused_gpu import HALF_UNIT, TYPES, U, act_code, dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def pairs(K, M):
    """Codes and exponents of weights [M][K] in which outputs 2 i and 2 i + 1 are the only ones of inputs i mod (M / 2), with 1 and -1."""
    codes = np.zeros((M, K), np.uint8)
    k = np.arange(K)
    codes[2 * (k % (M // 2)), k], codes[2 * (k % (M // 2)) + 1, k] = 2, 10
    return codes, np.full((M, (K + 31) // 32), 127, np.uint8)


def handle(sp, codes, scales):
    t = [torch.from_numpy(a).cuda() for a in (so.mx4_pack(codes), scales)]
    return sp.dense_fused_create_mx4(*t, codes.shape[1], backward=True)


SHAPES = [(64, 60, 40), (1030, 1300, 70), (96, 2600, 33), (72, 8200, 50)]


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("xk", ["bf16", "f32"])
def test_slopes_of_bf16_outputs_keep_their_digits(sp, K, M, B, act, xk):
    """dx[k] = g[m] - g[m + 1], both of one dy and of values before the activation that lie close together: some 2^-5 of either.
    A term is held to 2^-23 of itself or 2^-39 of its row's largest, its slope to 1e-6; dx is rounded to its type.  Two terms in
    two parts each are added, and zeros: 6 u sqrt(4) of the sum of sizes, as elsewhere for n = 4."""
    r = np.random.default_rng([41, K, M, B])
    codes, scales = pairs(K, M)
    W = so.mx4_values(codes, scales)
    dy = np.repeat(r.normal(size=(B, M // 2)), 2, axis=1)
    z = np.repeat(r.normal(size=(B, M // 2)), 2, axis=1)
    z[:, 1::2] += 1 / 16
    dy, pre = dev(dy, "bf16"), dev(z, "bf16")
    h = handle(sp, codes, scales)
    dx = torch.full((B, K), float("nan"), dtype=TYPES[xk], device="cuda")
    sp.dense_fused_backward(h, dy, dx=dx, pre=pre, act=act_code(sp, act))
    torch.cuda.synchronize()
    want, _, g = step.fused_backward(W, np.ones(M), host(dy), host(pre), act)
    mass, slopes = np.abs(g) @ np.abs(W), 1e-6 * np.abs(host(dy)) @ np.abs(W)
    lim = ((2.0 ** -23 + 12 * U) * (mass + slopes) + slopes + 2 * 2.0 ** -39 * np.abs(g).max(axis=1, keepdims=True)
           + HALF_UNIT[xk] * np.abs(want) * 1.01)
    bad = np.abs(host(dx) - want) > lim
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(host(dx) - want) / lim)))
    h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("xk", ["bf16", "f32"])
def test_bf16_outputs_of_any_size_enter_exactly(sp, K, M, B, act, xk):
    """Without a slope g is dy or 0, of 8 bits, and so is g * scale.  Elements from 2^-30 to 1 times their row's largest, outputs' scales
    between 2^-20 and 2^20: the differences of two of one size, to the bit."""
    r = np.random.default_rng([42, K, M, B])
    codes, scales = pairs(K, M)
    power = r.integers(-20, 21, M // 2)
    scales = np.repeat((127 + power).astype(np.uint8), 2)[:, None] + np.zeros_like(scales)
    W = so.mx4_values(codes, scales)
    size = np.repeat(2.0 ** (r.integers(-30, 1, (B, M // 2)) - power), 2, axis=1)
    dy = size * (1 + r.integers(0, 128, (B, M)) / 128)
    z = r.normal(size=(B, M))
    dy, pre = dev(dy, "bf16"), dev(z, "bf16")
    h = handle(sp, codes, scales)
    dx = torch.full((B, K), float("nan"), dtype=TYPES[xk], device="cuda")
    sp.dense_fused_backward(h, dy, dx=dx, pre=pre if act == "relu" else None, act=act_code(sp, act))
    torch.cuda.synchronize()
    want, _, _ = step.fused_backward(W, np.ones(M), host(dy), host(pre), act)
    assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[xk]))
    h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("yk", ["bf16", "f32"])
def test_rows_of_elements_of_unlike_sizes(sp, K, M, B, yk):
    """Elements of a row from 2^-50 to 1 times its largest: each is held to 2^-23 of itself or 2^-39 of that, whichever is more."""
    r = np.random.default_rng([43, K, M, B])
    codes, scales = pairs(K, M)
    W = so.mx4_values(codes, scales)
    dy = dev(r.normal(size=(B, M)) * np.repeat(2.0 ** r.integers(-50, 1, (B, M // 2)), 2, axis=1), yk)
    pre = dev(r.normal(size=(B, M)), yk)
    h = handle(sp, codes, scales)
    dx = torch.full((B, K), float("nan"), device="cuda")
    sp.dense_fused_backward(h, dy, dx=dx, pre=pre, act=sp.DENSE_ACT_SILU)
    torch.cuda.synchronize()
    want, _, g = step.fused_backward(W, np.ones(M), host(dy), host(pre), "silu")
    mass, slopes = np.abs(g) @ np.abs(W), 1e-6 * np.abs(host(dy)) @ np.abs(W)
    lim = (2.0 ** -23 + 12 * U) * (mass + slopes) + slopes + 2 * 2.0 ** -39 * np.abs(g).max(axis=1, keepdims=True) + U * np.abs(want)
    assert (np.abs(host(dx) - want) <= lim).all(), float(np.max(np.abs(host(dx) - want) / lim))
    h.close()
