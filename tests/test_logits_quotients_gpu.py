"""GPU check of the repetition penalty's quotient and product (head_logits.h): FP32's, to the bit, over all of its range."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

V = 3000


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def penalised(sp, x, r):
    """x [S, V] with every token in the prompt, r [S]."""
    S = x.shape[0]
    ids = torch.arange(V, dtype=torch.int32, device="cuda").repeat(S, 1)
    logits = torch.from_numpy(x[:, None, :].copy()).cuda()
    out = torch.empty_like(logits)
    sp.head_logits_adjust(logits, out, ids=ids, n_prompt=torch.full((S,), V, dtype=torch.int32, device="cuda"),
                          repetition=torch.from_numpy(r).cuda())
    torch.cuda.synchronize()
    return out[:, 0].cpu().numpy()


def check(sp, x, r):
    with np.errstate(all="ignore"):
        want = np.where(x > 0, x / r[:, None], x * r[:, None])
    got = penalised(sp, x, r)
    same = (got.view(np.int32) == want.view(np.int32)) | (np.isnan(got) & np.isnan(want))
    assert same.all(), [tuple(float(v).hex() for v in (x[i, j], r[i], got[i, j], want[i, j])) for i, j in np.argwhere(~same)[:3]]


def floats(r, shape, lo, hi):
    """FP32 values with exponents in [lo, hi), subnormals rounded."""
    return np.ldexp(r.integers(1 << 23, 1 << 24, shape).astype(np.float64), r.integers(lo, hi, shape) - 23).astype(np.float32)


@pytest.mark.parametrize("lo,hi", [(-149, -120), (-126, -100), (-60, 60), (-3, 8), (100, 128)])
@pytest.mark.parametrize("near", [(-1, 1), (-20, 20), (-149, -100), (100, 128)])
def test_every_size(sp, lo, hi, near):
    """Logits of these sizes, either sign, penalties near 1 and far from it, quotients and products down to 2^-149 and past the largest."""
    r = np.random.default_rng([51, lo + 200, near[0] + 200])
    x = floats(r, (20, V), lo, hi) * r.choice([-1, 1], (20, V)).astype(np.float32)
    check(sp, x, floats(r, 20, *near))


def test_the_ends_of_the_range(sp):
    """The largest numbers with penalties just below and above 1, zeros, infinities, NaN, and penalties that are none."""
    r = np.random.default_rng(52)
    top = np.float32(np.finfo(np.float32).max)
    x = np.empty((24, V), np.float32)
    x[:] = (top.view(np.int32) - np.arange(V, dtype=np.int32)).view(np.float32)
    x[:, -8:] = [0.0, -0.0, np.inf, -np.inf, np.nan, 2.0 ** -149, -2.0 ** -149, 2.0 ** -126]
    x[:, 100:] *= np.where(r.random((24, V - 100)) < 0.5, 1, -1).astype(np.float32)
    p = np.concatenate([1 - np.arange(1, 9) * 2.0 ** -24, 1 + np.arange(1, 9) * 2.0 ** -23,
                        [1.0, 0.0, -1.3, 2.0 ** -149, float(top), np.inf, np.nan, 2.0]]).astype(np.float32)
    check(sp, x, p)
