"""GPU parity of the microscaled four-bit quantizer (quantize.h): codes, scales and values bit for bit."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def rows(a, dtype, pad, offset, fill):
    """Rows of an array in a buffer with `pad` elements between them, the first `offset` elements into it."""
    a = torch.as_tensor(a).to(dtype)
    buf = torch.full((a.shape[0] * (a.shape[1] + pad) + offset,), fill, dtype=dtype, device="cuda")
    view = buf[offset:].view(a.shape[0], a.shape[1] + pad)[:, :a.shape[1]]
    view.copy_(a)
    return view, buf


def check(sp, x, kind, pad=0, offset=0, with_values=True, code_pad=0):
    """x: float32 array; everything that is not an output stays as it was."""
    M, K = x.shape
    xd, _ = rows(x, TYPES[kind], pad, offset, 7.0)
    codes, c_buf = rows(np.zeros((M, (K + 1) // 2), np.uint8), torch.uint8, code_pad, offset, 77)
    scales, s_buf = rows(np.zeros((M, (K + 31) // 32), np.uint8), torch.uint8, code_pad, offset, 78)
    values, v_buf = rows(np.zeros((M, K), np.float32), TYPES[kind], pad, offset, 79.0)
    before = [t.clone() for t in (c_buf, s_buf, v_buf)]
    sp.spike_quantize_mx4(xd, codes, scales, values=values if with_values else None)
    torch.cuda.synchronize()
    want, want_s, want_v = so.mx4_quantize(xd.float().cpu().numpy())
    assert (scales.cpu().numpy() == want_s).all()
    assert (codes.cpu().numpy() == so.mx4_pack(want)).all()
    if with_values:
        got = values.cpu().double().numpy()
        assert ((got == want_v) | (np.isnan(got) & np.isnan(want_v))).all()
    for view, buf, old in ((codes, c_buf, before[0]), (scales, s_buf, before[1]), (values, v_buf, before[2])):
        view.zero_()
        assert torch.equal(buf, old), "bytes between rows were written"


SHAPES = [(1, 1), (3, 2), (2, 31), (5, 32), (4, 33), (7, 64), (3, 100), (2, 257), (40, 96), (9, 1536), (300, 40), (2, 6144), (1, 20001)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_shapes(sp, kind, M, K):
    r = np.random.default_rng([1, M, K])
    x = (r.normal(size=(M, K)) * np.exp(r.normal(size=(M, 1)) * 3)).astype(np.float32)
    x[r.random((M, K)) < 0.05] = 0.0
    check(sp, x, kind)
    check(sp, x, kind, with_values=False)
    check(sp, x, kind, pad=3, offset=1, code_pad=1)
    check(sp, x, kind, pad=8, offset=8, code_pad=4)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_every_midpoint(sp, kind):
    """All multiples of 1/16 up to 8 with both signs, blocks led by 4 to 7.9, at several powers of two."""
    steps = np.arange(0, 128) / 16.0
    x = np.zeros((14, 2 * 128 // 31 * 32 + 64), np.float32)
    vals = np.concatenate([steps, -steps])
    k = 0
    for v in vals:
        if k % 32 == 0:
            x[:, k] = 4.0 + (k // 32 % 8) * 0.5
            k += 1
        x[:, k] = v
        k += 1
    x *= 2.0 ** np.array([-8, -3, -1, 0, 1, 2, 3, 4, 5, 7, 9, 10, 11, 12])[:, None].astype(np.float32)
    check(sp, x, kind)


def test_range_ends(sp):
    """Subnormal and largest values, blocks with NaN and infinities beside whole ones, negative zeros."""
    r = np.random.default_rng(5)
    x = r.uniform(-8, 8, (12, 96)).astype(np.float32)
    for m, p in enumerate((-149, -148, -140, -130, -128, -127, -126, -125, -124, 100, 125)):
        x[m] = (x[m].astype(np.float64) * 2.0 ** p).clip(-3.4e38, 3.4e38).astype(np.float32)
    x[11, 40], x[11, 41], x[11, 70], x[11, 0] = np.inf, np.nan, -np.inf, -0.0
    for kind in ("f32", "bf16"):
        check(sp, x, kind)
    y = r.uniform(-8, 8, (6, 64)).astype(np.float32) * 2.0 ** np.array([-27, -26, -24, -16, 0, 12])[:, None].astype(np.float32)
    y[4, 3], y[5, 40] = np.inf, np.nan
    check(sp, y, "f16")


def test_in_place_values_and_streams(sp):
    """values may be x: what a tuned weight is rounded to."""
    x = torch.randn((70, 200), device="cuda")
    want, _, want_v = so.mx4_quantize(x.cpu().numpy())
    codes = torch.zeros((70, 100), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((70, 7), dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    sp.spike_quantize_mx4(x, codes, scales, values=x, stream=st)
    st.synchronize()
    assert (codes.cpu().numpy() == so.mx4_pack(want)).all() and (x.cpu().double().numpy() == want_v).all()


def test_long_rows_and_many(sp):
    """More units than one launch's first workgroups; rows longer than a wave's stretch; nothing for no rows."""
    for M, K in ((20000, 33), (3, 100000)):
        r = np.random.default_rng(M)
        x = r.normal(size=(M, K)).astype(np.float32)
        xd = torch.from_numpy(x).cuda()
        codes = torch.zeros((M, (K + 1) // 2), dtype=torch.uint8, device="cuda")
        scales = torch.zeros((M, (K + 31) // 32), dtype=torch.uint8, device="cuda")
        values = torch.zeros_like(xd)
        sp.spike_quantize_mx4(xd, codes, scales, values=values)
        torch.cuda.synchronize()
        pick = r.integers(0, M, 3)
        want, want_s, want_v = so.mx4_quantize(x[pick][:, :3000])
        assert (scales.cpu().numpy()[pick][:, :93] == want_s[:, :93]).all()
        n = min(1500, codes.shape[1])
        assert (codes.cpu().numpy()[pick][:, :n - 12] == so.mx4_pack(want)[:, :n - 12]).all()
        unpacked = torch.stack([codes & 15, codes >> 4], dim=2).view(M, -1)[:, :K].cpu().numpy()
        assert (so.mx4_values(unpacked, scales.cpu().numpy()) == values.cpu().double().numpy()).all()
        # every value is within the block's bound of its element
        power = np.repeat(np.ldexp(1.0, scales.cpu().numpy().astype(int) - 127), 32, axis=1)[:, :K]
        assert (np.abs(values.cpu().double().numpy() - x) <= 2.0 * power).all()
    empty = lambda n, t=torch.uint8: torch.empty((0, n), dtype=t, device="cuda")  # noqa: E731
    sp.spike_quantize_mx4(empty(40, torch.float32), empty(20), empty(2))


def test_graph_replays(sp):
    x = torch.randn((50, 320), device="cuda", dtype=torch.bfloat16)
    codes = torch.zeros((50, 160), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((50, 10), dtype=torch.uint8, device="cuda")
    values = torch.zeros_like(x)
    sp.spike_quantize_mx4(x, codes, scales, values=values)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.spike_quantize_mx4(x, codes, scales, values=values)
    for _ in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        sp.spike_quantize_mx4(x, codes, scales, values=values)
        torch.cuda.synchronize()
        want = [t.clone() for t in (codes, scales, values)]
        for t in (codes, scales, values):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip((codes, scales, values), want))
