"""GPU parity of the fused projection with four-bit weights, of rows in any type
and in four bits, and of its gradient (dense_fused.h) against the float64 definition.

Where weights are multiples of 1/4 and rows small integers the sums are exact in
FP32 and outputs match bit for bit.  Elsewhere, as for INT8 weights, n additions of rounding u =
2^-24 each, taken as independent, stay within

    lim = 6 u sqrt(n) sum_k |W x|,  n = parts * K + 32

(parts: three BF16 parts of an FP32 row or gradient at most, one of four-bit rows, whose products are
exact); the activation adds at most 1e-6 + 4e-7 |y|, its slope is at most 1.13 in size, and storing rounds by
half a unit of the type.  Gradients enter the product to 2^-11 or better.  Weights whose blocks are within
2^28 of their output's largest are exact in every operand.
"""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from oracle import step_oracle as step
from tests.launches import launches
from tests.test_fused_gpu import HALF_UNIT, SHAPES, TYPES, U, act_code, dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def coded(r, rows, K, lo, hi):
    """Random codes [rows][K] and exponents in [lo, hi)."""
    return r.integers(0, 16, (rows, K)).astype(np.uint8), r.integers(lo, hi, (rows, (K + 31) // 32)).astype(np.uint8)


def problem(K, M, B, seed=0, integer=False):
    """integer: weights multiples of 1/4 up to 12, rows of integers (four-bit rows: of halves up to 12)."""
    r = np.random.default_rng([21, K, M, B, seed])
    p = dict(zip(("codes", "scales"), coded(r, M, K, 126, 129) if integer else coded(r, M, K, 115, 120)))
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    p["x_codes"], p["x_scales"] = coded(r, B, K, 127, 129) if integer else coded(r, B, K, 120, 130)
    if integer:
        p.update(bias=r.integers(-4, 5, M).astype(np.float32), x=r.integers(-3, 4, (B, K)).astype(np.float32),
                 residual=r.integers(-8, 9, (B, M)).astype(np.float32), dy=r.integers(-3, 4, (B, M)).astype(np.float32))
    else:
        p.update(bias=r.normal(0, 0.5, M).astype(np.float32), x=r.normal(size=(B, K)).astype(np.float32),
                 residual=r.normal(size=(B, M)).astype(np.float32), dy=r.normal(size=(B, M)).astype(np.float32))
    return p


def bytes_dev(a, pad=0, offset=0):
    """uint8 rows on the device, `pad` bytes of 0xff (NaN exponents, full codes) between them."""
    buf = torch.full((a.shape[0] * (a.shape[1] + pad) + offset,), 255, dtype=torch.uint8, device="cuda")
    view = buf[offset:].view(a.shape[0], a.shape[1] + pad)[:, :a.shape[1]]
    view.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return view


def packed(codes, junk=True):
    """Codes two to a byte; where K is odd the last byte's upper half is junk that belongs to nothing."""
    b = so.mx4_pack(codes)
    if junk and codes.shape[1] % 2:
        b[:, -1] |= 0x70
    return b


def handle(sp, p, backward=False, pad=0, offset=0):
    return sp.dense_fused_create_mx4(bytes_dev(packed(p["codes"]), pad, offset), bytes_dev(p["scales"], pad, offset),
                                     p["codes"].shape[1], backward=backward)


def rows_of(p):
    return so.mx4_values(p["x_codes"], p["x_scales"])


def forward(sp, h, p, xk, yk, act="none", bias=True, residual=True, pre=False, pad=0, offset=0, stream=None):
    """((y, z), expected y, expected z, the rows in 64 bits); xk "mx4": rows of codes."""
    B, M = p["x"].shape[0], p["W"].shape[0]
    y = dev(np.full((B, M), np.nan), yk, pad, offset)
    z = dev(np.full((B, M), np.nan), yk, pad, offset) if pre else None
    res = dev(p["residual"], yk, pad, offset) if residual else None
    kw = dict(bias=torch.from_numpy(p["bias"]).cuda() if bias else None, act=act_code(sp, act), residual=res, pre=z, stream=stream)
    if xk == "mx4":
        x64 = rows_of(p)
        args = bytes_dev(packed(p["x_codes"]), pad, offset), bytes_dev(p["x_scales"], pad, offset)
        torch.cuda.synchronize()
        sp.dense_fused_forward_mx4(h, *args, y, **kw)
    else:
        x = dev(p["x"], xk, pad, offset)
        x64 = host(x)
        torch.cuda.synchronize()
        sp.dense_fused_forward(h, x, y, **kw)
    torch.cuda.synchronize()
    want_z = x64 @ p["W"].T + (p["bias"].astype(np.float64) if bias else 0.0)
    want = step.act(want_z, act) + (host(res) if residual else 0.0)
    return (y, z), want, want_z, x64


def check_forward(p, xk, yk, out, want, want_z, x64, residual=None):
    y, z = out
    parts = 3 if xk == "f32" else 1
    mass = np.abs(x64) @ np.abs(p["W"]).T
    lim_z = 6 * U * np.sqrt(parts * x64.shape[1] + 32) * (mass + np.abs(want_z))
    lim = 1.13 * lim_z + 1e-6 + 4e-7 * np.abs(want) + HALF_UNIT[yk] * np.abs(want) * 1.01 + 2.0 ** -25
    if residual is not None:
        lim += 2 * U * np.abs(residual)
    got = host(y)
    assert np.isfinite(got).all(), "outputs left unwritten"
    bad = np.abs(got - want) > lim
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], lim[bad][0])
    if z is not None:
        assert (np.abs(host(z) - want_z) <= lim_z + HALF_UNIT[yk] * np.abs(want_z) * 1.01 + 2.0 ** -25).all()


TYPE_PAIRS = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("mx4", "f32"), ("mx4", "bf16"), ("mx4", "f16")]
MORE_SHAPES = [(31, 33, 40), (32, 16, 50), (128, 64, 33), (256, 300, 64), (384, 1040, 200), (96, 4100, 9), (160, 33000, 3), (150, 33000, 20)]


@pytest.mark.parametrize("K,M,B", SHAPES + MORE_SHAPES)
@pytest.mark.parametrize("xk,yk", TYPE_PAIRS)
def test_integers_are_exact(sp, K, M, B, xk, yk):
    p = problem(K, M, B, integer=True)
    for pad, offset, act in ((0, 0, "none"), (5, 1, "relu"), (16, 16, "none")):
        h = handle(sp, p, pad=pad, offset=offset)
        (y, z), want, want_z, _ = forward(sp, h, p, xk, yk, act=act, pre=True, pad=pad, offset=offset)
        assert torch.equal(y.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[yk])), (act, pad)
        assert torch.equal(z.cpu(), torch.from_numpy(want_z.astype(np.float32)).to(TYPES[yk])), (act, pad)
        h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk,act", [("f32", "f32", "gelu"), ("bf16", "bf16", "gelu"), ("f16", "f16", "silu"),
                                       ("f32", "f32", "none"), ("mx4", "f32", "none"), ("mx4", "bf16", "gelu")])
def test_forward(sp, K, M, B, xk, yk, act):
    p = problem(K, M, B)
    h = handle(sp, p)
    out, want, want_z, x64 = forward(sp, h, p, xk, yk, act=act, pre=True, pad=8 if K % 2 else 0)
    check_forward(p, xk, yk, out, want, want_z, x64, np.abs(p["residual"]))
    out, want, want_z, x64 = forward(sp, h, p, xk, yk, act=act, bias=False, residual=False)
    check_forward(p, xk, yk, out, want, want_z, x64)
    h.close()


def test_long_inputs(sp):
    """16,500 inputs and 20,000 outputs: long sums, sums split over workgroups, many tiles."""
    for K, M, B, xk in ((16500, 40, 3, "f32"), (16500, 40, 70, "bf16"), (16500, 40, 70, "mx4"), (16512, 72, 300, "mx4"),
                        (16500, 40, 5, "mx4"), (33, 20000, 2, "bf16"), (40, 20000, 100, "f32"), (40, 20000, 100, "mx4")):
        p = problem(K, M, B)
        h = handle(sp, p)
        out, want, want_z, x64 = forward(sp, h, p, xk, "f32", act="gelu", residual=False)
        check_forward(p, xk, "f32", out, want, want_z, x64)
        h.close()


def kernel_names(sp, h, p, xk, B, M):
    y = torch.empty((B, M), device="cuda")
    if xk == "mx4":
        c, s = bytes_dev(packed(p["x_codes"])), bytes_dev(p["x_scales"])
        ws = torch.empty(max(16, sp.dense_fused_forward_mx4_workspace_bytes(h, c, s)), dtype=torch.uint8, device="cuda")
        call = lambda st: sp.dense_fused_forward_mx4(h, c, s, y, workspace=ws, stream=st)  # noqa: E731
    else:
        x = dev(p["x"], xk)
        ws = torch.empty(max(16, sp.dense_fused_forward_workspace_bytes(h, x)), dtype=torch.uint8, device="cuda")
        call = lambda st: sp.dense_fused_forward(h, x, y, workspace=ws, stream=st)  # noqa: E731
    return [name for name, _, _ in launches(call)]


# single products: an output whose weights are one code of one block, an input at a time
@pytest.mark.parametrize("xk", ["f32", "bf16", "f16", "mx4"])
@pytest.mark.parametrize("B", [1, 40])
def test_single_products_of_any_exponent(sp, xk, B):
    """One weight an output, exponents from 0 to 254 from output to output: a power of two changes nothing but the result's."""
    K, M = 70, 255
    p = problem(K, M, B)
    r = np.random.default_rng([22, B])
    p["codes"][:] = 0
    at = r.integers(0, K, M)
    p["codes"][np.arange(M), at] = r.integers(1, 8, M)
    p["scales"][:] = np.arange(M)[:, None]
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    h = handle(sp, p)
    (y, _), want, _, _ = forward(sp, h, p, xk, "f32", bias=False, residual=False)
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)
    got = y.cpu().numpy()
    # FP32 rows of many go as two planes, 2^-23 of an element.  A 24-bit element times 1.5 has 25 bits, which FP32
    # does not hold: adding its parts' products rounds twice, u each.  16-bit and four-bit elements (11 bits at most,
    # 13 with the code's) are exact.  Subnormal results round once more
    lim = ((2.0 ** -23 if B > 32 else 0.0) + 2 * U if xk == "f32" else 0.0) * np.abs(want) + 2.0 ** -149
    fine = np.abs(want) < 2.0 ** 127
    assert (np.abs(got.astype(np.float64) - want) <= lim)[fine].all()
    assert np.isfinite(got[fine]).all() and np.isfinite(want32[fine]).all()
    h.close()


@pytest.mark.parametrize("xk", ["f32", "bf16", "f16", "mx4"])
@pytest.mark.parametrize("B", [3, 40])
def test_blocks_of_unlike_exponents(sp, xk, B):
    """Blocks of one output up to 2^100 apart, the row without the large ones: what is far below its output's largest
    is held to 2^-37 of that (F16 operands), or exactly down to 2^-127 of it (BF16 operands, four-bit rows)."""
    K, M = 256, 64
    p = problem(K, M, B)
    r = np.random.default_rng([23, B])
    p["scales"] = r.integers(40, 141, p["scales"].shape).astype(np.uint8)
    p["scales"][:, 3] = 140
    p["codes"][:, 96] = 7
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    p["x"][:, 96:128] = 0.0
    p["x_codes"][:, 96:128] = 0
    h = handle(sp, p)
    (y, _), want, want_z, x64 = forward(sp, h, p, xk, "f32", bias=False, residual=False)
    mass = np.abs(x64) @ np.abs(p["W"]).T
    lim = 6 * U * np.sqrt(3 * K + 32) * (mass + np.abs(want)) + 2.0 ** -140
    if xk == "f16" or (xk == "f32" and B > 32):
        lim += 2.0 ** -37 * np.abs(x64).sum(axis=1, keepdims=True) * np.abs(p["W"]).max(axis=1)
    assert (np.abs(host(y) - want) <= lim).all(), np.max(np.abs(host(y) - want) / lim)
    h.close()


@pytest.mark.parametrize("xk", ["f32", "bf16", "f16", "mx4"])
@pytest.mark.parametrize("B", [3, 40])
def test_nan_blocks_stay_in_their_outputs(sp, xk, B):
    """A weight's block of exponent 255 is NaN for its output, a row's for its row; an output of zeros is its bias."""
    p = problem(200, 50, B, integer=True)
    p["scales"][7, 6] = 255
    p["codes"][9], p["scales"][9] = 0, 200
    p["codes"][10] = 8  # negative zeros
    if xk == "mx4":
        p["x_scales"][1, 2] = 255
    else:
        p["x"][1, 70] = np.nan
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    h = handle(sp, p, backward=True)
    (y, _), _, _, x64 = forward(sp, h, p, xk, "f32", residual=False)
    got = host(y)
    assert np.isnan(got[:, 7]).all() and np.isnan(got[1]).all()
    W, rest = p["W"].copy(), np.delete(np.arange(B), 1)
    W[7] = 0
    want = x64[rest] @ W.T + p["bias"]
    keep = np.arange(50) != 7
    assert (got[rest][:, keep] == want[:, keep]).all() and (got[rest, 9] == p["bias"][9]).all()
    # in the gradient, the inputs of that block; the output's others count
    W = np.where(np.isnan(p["W"]), 0.0, p["W"])
    dy, dx = dev(p["dy"], "f32"), torch.empty((B, 200), device="cuda")
    sp.dense_fused_backward(h, dy, dx=dx)
    got = host(dx)
    assert np.isnan(got[:, 192:200]).all() and (got[:, :192] == (p["dy"].astype(np.float64) @ W)[:, :192]).all()
    h.close()


def backward(sp, h, p, xk, yk, act, pad=0, offset=0, z=None, want_dx=True, want_bias=True):
    B, M = p["dy"].shape
    K = p["W"].shape[1]
    dy = dev(p["dy"], yk, pad, offset)
    pre = dev(z, yk, pad, offset) if act != "none" else None
    dx = dev(np.full((B, K), np.nan), xk, pad, offset) if want_dx else None
    db = torch.full((M,), float("nan"), device="cuda") if want_bias else None
    sp.dense_fused_backward(h, dy, dx=dx, dbias=db, pre=pre, act=act_code(sp, act))
    torch.cuda.synchronize()
    return dx, db, step.fused_backward(p["W"], np.ones(M), host(dy), None if pre is None else host(pre), act)


@pytest.mark.parametrize("K,M,B", SHAPES + [(96, 4100, 40), (520, 2100, 700)])
@pytest.mark.parametrize("xk,yk", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
def test_backward_of_integers_is_exact(sp, K, M, B, xk, yk):
    p = problem(K, M, B, integer=True)
    z = np.random.default_rng([24, K, M, B]).integers(-3, 4, (B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    for act, pad, offset in (("none", 0, 0), ("relu", 3, 1)):
        dx, db, (want, wb, _) = backward(sp, h, p, xk, yk, act, pad, offset, z)
        assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[xk])), act
        assert (db.cpu().numpy() == wb).all(), act
    h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk,act", [("f32", "f32", "gelu"), ("bf16", "bf16", "gelu"), ("f16", "f16", "silu")])
def test_backward(sp, K, M, B, xk, yk, act):
    p = problem(K, M, B)
    z = np.random.default_rng([25, K, M, B]).normal(size=(B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    dx, db, (want, wb, g) = backward(sp, h, p, xk, yk, act, pad=8 if K % 2 else 0, z=z)
    w = np.abs(p["W"])
    parts = {"f32": 3, "bf16": 1, "f16": 2}[yk]
    entry = {"f32": 0.0, "bf16": HALF_UNIT["bf16"], "f16": 2.0 ** -15}[yk]
    g_err = np.abs(host(torch.from_numpy(p["dy"]).to(TYPES[yk]))) * 1e-6
    lim = (6 * U * np.sqrt(parts * M + 32) * (np.abs(g) @ w) + 6 * entry * np.sqrt((g * g) @ (w * w)) + g_err @ w
           + HALF_UNIT[xk] * np.abs(want) * 1.01 + 2.0 ** -25)
    assert (np.abs(host(dx) - want) <= lim).all(), np.max(np.abs(host(dx) - want) / lim)
    blim = 6 * U * np.sqrt(B + 8) * np.abs(g).sum(axis=0) + g_err.sum(axis=0) + 1e-30
    assert (np.abs(host(db) - wb) <= blim).all()
    h.close()


@pytest.mark.parametrize("K,M,B", [(70, 60, 40), (300, 700, 90), (520, 2100, 700)])
@pytest.mark.parametrize("xk,entry", [("bf16", 2.0 ** -12), ("f32", 2.0 ** -23)])
def test_gradient_of_bf16_outputs_keeps_its_digits(sp, K, M, B, xk, entry):
    """A BF16 dy whose slopes give it more digits: to a BF16 dx they enter with 11 bits (2^-12 of an element), to an FP32 one
    with 2^-23 of it; the slope is off by 1e-6, and dx is rounded to its type."""
    p = problem(K, M, B)
    z = np.random.default_rng([27, K, M, B]).normal(size=(B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    dx, _, (want, _, g) = backward(sp, h, p, xk, "bf16", "silu", z=z, want_bias=False)
    w = np.abs(p["W"])
    g_err = np.abs(host(torch.from_numpy(p["dy"]).bfloat16())) * 1e-6
    lim = (6 * U * np.sqrt(2 * M + 32) * (np.abs(g) @ w) + 6 * entry * np.sqrt((g * g) @ (w * w)) + g_err @ w
           + HALF_UNIT[xk] * np.abs(want) * 1.01 + 2.0 ** -25)
    assert (np.abs(host(dx) - want) <= lim).all(), np.max(np.abs(host(dx) - want) / lim)
    h.close()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(sp, act):
    """dx and dbias along a direction against central differences of the definition in 64 bits."""
    p = problem(150, 90, 37)
    h = handle(sp, p, backward=True)
    r = np.random.default_rng(8)
    v, vb = r.normal(size=p["x"].shape), r.normal(size=90)
    z = p["x"].astype(np.float64) @ p["W"].T + p["bias"]
    p["dy"] = r.normal(size=z.shape).astype(np.float32)
    dx, db, _ = backward(sp, h, p, "f32", "f32", act, z=z)
    f = lambda t: (step.act((p["x"] + t * v) @ p["W"].T + p["bias"] + t * vb, act) * p["dy"]).sum()  # noqa: E731
    num = (f(1e-5) - f(-1e-5)) / 2e-5
    got = (host(dx) * v).sum() + (host(db) * vb).sum()
    assert abs(num - got) <= 2e-6 * (np.abs(host(dx) * v).sum() + np.abs(host(db) * vb).sum())
    h.close()


@pytest.mark.parametrize("B", [3, 90, 700])
def test_graph_replays(sp, B):
    """Captured forwards (rows in BF16 and in codes) and backward, replayed with eager work between."""
    p = problem(320, 192, B)
    h = handle(sp, p, backward=True)
    x, dy = dev(p["x"], "bf16"), dev(p["dy"], "bf16")
    codes = torch.empty((B, 160), dtype=torch.uint8, device="cuda")
    scales = torch.empty((B, 10), dtype=torch.uint8, device="cuda")
    y, z, y4, dx = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x)
    db, bias = torch.empty(192, device="cuda"), torch.from_numpy(p["bias"]).cuda()

    def run():
        sp.dense_fused_forward(h, x, y, bias=bias, act=sp.DENSE_ACT_GELU, pre=z)
        sp.spike_quantize_mx4(x, codes, scales)
        sp.dense_fused_forward_mx4(h, codes, scales, y4, bias=bias, act=sp.DENSE_ACT_GELU)
        sp.dense_fused_backward(h, dy, dx=dx, dbias=db, pre=z, act=sp.DENSE_ACT_GELU)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        dy.copy_(torch.randn(dy.shape, device="cuda"))
        run()
        torch.cuda.synchronize()
        outs = (y, z, y4, dx, db)
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert torch.equal(t, w), i
    h.close()


def test_streams_and_residual_in_place(sp):
    p = problem(200, 96, 40)
    h = handle(sp, p)
    c, s = bytes_dev(packed(p["x_codes"])), bytes_dev(p["x_scales"])
    r = dev(p["residual"], "bf16")
    y = torch.empty_like(r)
    sp.dense_fused_forward_mx4(h, c, s, y, residual=r)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    sp.dense_fused_forward_mx4(h, c, s, r, residual=r, stream=st)
    st.synchronize()
    assert torch.equal(r, y)
    h.close()


def test_no_rows_and_refusals(sp):
    p = problem(40, 24, 6)
    h = handle(sp, p)
    u8 = lambda *shape: torch.empty(shape, dtype=torch.uint8, device="cuda")  # noqa: E731
    y = torch.empty((6, 24), device="cuda")
    sp.dense_fused_forward_mx4(h, u8(0, 20), u8(0, 2), torch.empty((0, 24), device="cuda"))
    with pytest.raises(ValueError, match="must be"):
        sp.dense_fused_forward_mx4(h, u8(6, 19), u8(6, 2), y)
    with pytest.raises(ValueError, match="must be"):
        sp.dense_fused_forward_mx4(h, u8(6, 20), u8(6, 1), y)
    with pytest.raises(TypeError, match="uint8"):
        sp.dense_fused_forward_mx4(h, u8(6, 20).to(torch.int8), u8(6, 2), y)
    with pytest.raises(TypeError, match="y's type"):
        sp.dense_fused_forward_mx4(h, u8(6, 20), u8(6, 2), y, residual=y.bfloat16())
    with pytest.raises(sp.SpikeError, match="BACKWARD"):
        sp.dense_fused_backward(h, y, dx=torch.empty((6, 40), device="cuda"))
    i8 = sp.dense_fused_create(torch.zeros((24, 40), dtype=torch.int8, device="cuda"), torch.ones(24, device="cuda"))
    with pytest.raises(sp.SpikeError, match="four-bit"):
        sp.dense_fused_forward_mx4(i8, u8(6, 20), u8(6, 2), y)
    with pytest.raises(sp.SpikeError, match="four-bit"):
        sp.dense_fused_forward_mx4(i8, u8(60, 20), u8(60, 2), torch.empty((60, 24), device="cuda"))
    i8.close()
    h.close()
    with pytest.raises(sp.SpikeError, match="null handle"):
        sp.dense_fused_forward_mx4(h, u8(6, 20), u8(6, 2), y)


def test_forward_workspace_is_what_the_query_says(sp):
    """Whole rows of 128 need none where sums are not split; others are copied."""
    for K, M, B, off, some in ((1536, 1600, 1100, 0, False), (1536, 1600, 1100, 1, True), (1568, 1600, 1100, 0, True), (6100, 70, 32, 0, False)):
        p = problem(K, M, 1)
        h = handle(sp, p)
        c, s = bytes_dev(np.zeros((B, (K + 1) // 2), np.uint8), 0, off), bytes_dev(np.zeros((B, (K + 31) // 32), np.uint8))
        y = torch.empty((B, M), device="cuda")
        n = sp.dense_fused_forward_mx4_workspace_bytes(h, c, s)
        assert (n > 0) == some
        sp.dense_fused_forward_mx4(h, c, s, y, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
        if n > 0:
            with pytest.raises(sp.SpikeError, match="workspace"):
                sp.dense_fused_forward_mx4(h, c, s, y, workspace=torch.empty(n - 16, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert (y == 0).all()
        h.close()


# sizes that take each kernel form: few rows by 1, 2 and 4 tiles of outputs (and two of rows), FP32 rows as columns
# and in parts, every tile shape of four-bit rows with the steps in one part and in several
@pytest.mark.parametrize("xk,K,M,B,name", [("f32", 200, 100, 5, "k_fused_spread"), ("f32", 100, 4200, 1, "k_fused_spread"),
                                           ("f32", 72, 17000, 4, "k_fused_spread"), ("f32", 8192, 4200, 1, "k_fused_spread"),
                                           ("f32", 4096, 17000, 2, "k_fused_spread"), ("f32", 72, 17000, 6, "k_fused_rows"),
                                           ("f32", 9000, 40, 2, "k_fused_rows"), ("bf16", 72, 33000, 20, "k_fused_rows"),
                                           ("mx4", 200, 100, 9, "k_mx4_rows"), ("mx4", 100, 4200, 9, "k_mx4_rows"),
                                           ("mx4", 72, 33000, 16, "k_mx4_rows"), ("mx4", 72, 33000, 20, "k_mx4_rows"),
                                           ("mx4", 1100, 4100, 3000, "k_mx4_tileILi4ELi8E"), ("mx4", 1100, 2100, 1500, "k_mx4_tileILi2ELi4E"),
                                           ("mx4", 520, 200, 100, "k_mx4_tileILi1ELi4E"), ("mx4", 6200, 200, 100, "k_fused_join")])
def test_every_form(sp, xk, K, M, B, name):
    p = problem(K, M, B, integer=True)
    h = handle(sp, p)
    names = kernel_names(sp, h, p, xk, B, M)
    assert any(name in n for n in names), names
    for pad, offset in ((0, 0), (1, 1)):
        (y, z), want, want_z, _ = forward(sp, h, p, xk, "f32", act="relu", pre=True, pad=pad, offset=offset)
        assert torch.equal(y.cpu(), torch.from_numpy(want.astype(np.float32))) and torch.equal(z.cpu(), torch.from_numpy(want_z.astype(np.float32)))
    h.close()


@pytest.mark.parametrize("B", [1, 5])
@pytest.mark.parametrize("K", [130, 1536])
def test_columns_of_few_fp32_rows(sp, K, B):
    """Rows as parts in columns: subnormals, values whose lowest bits lie below BF16's steps, infinities, beside ordinary rows."""
    M = 70
    p = problem(K, M, B)
    r = np.random.default_rng([26, K, B])
    p["scales"] = r.integers(125, 129, p["scales"].shape).astype(np.uint8)
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    p["x"] = (r.normal(size=(B, K)) * 10.0 ** r.uniform(-44, -34, (B, K))).astype(np.float32)
    h = handle(sp, p)
    (y, _), want, _, x64 = forward(sp, h, p, "f32", "f32", bias=False, residual=False)
    # a sum of multiples of 2^-150 (weights of 1/8 at least times steps of 2^-149), each addition off by u, stored to 2^-149
    lim = 6 * U * np.sqrt(3 * K + 32) * (np.abs(x64) @ np.abs(p["W"]).T) + 2.0 ** -149
    assert (np.abs(host(y) - want) <= lim).all(), np.max(np.abs(host(y) - want) / lim)
    p["x"] = r.normal(size=(B, K)).astype(np.float32)
    p["x"][0, 3] = np.inf
    p["codes"][:, 3] = np.where(np.arange(M) % 2, 2, 10)
    p["W"] = so.mx4_values(p["codes"], p["scales"])
    h2 = handle(sp, p)
    with np.errstate(invalid="ignore"):
        (y, _), want, _, x64 = forward(sp, h2, p, "f32", "f32", bias=False, residual=False)
    got = host(y)
    assert (got[0] == np.where(np.arange(M) % 2, np.inf, -np.inf)).all()
    lim = 6 * U * np.sqrt(3 * K + 32) * (np.abs(x64[1:]) @ np.abs(p["W"]).T)
    assert (np.abs(got[1:] - want[1:]) <= lim).all()
    h.close()
    h2.close()


@pytest.mark.parametrize("B", [3, 40, 600])
def test_nothing_is_left_from_the_call_before(sp, B):
    """A call whose rows are all NaN, then one of integers: nothing of the first is in the second."""
    p = problem(136, 520, B, integer=True)
    h = handle(sp, p)
    nan = torch.full((B, 5), 255, dtype=torch.uint8, device="cuda")
    y = torch.empty((B, 520), device="cuda")
    sp.dense_fused_forward_mx4(h, torch.full((B, 68), 0x77, dtype=torch.uint8, device="cuda"), nan, y)
    sp.dense_fused_forward_mx4(h, bytes_dev(packed(p["x_codes"])), bytes_dev(p["x_scales"]), y)
    torch.cuda.synchronize()
    assert torch.equal(y.cpu(), torch.from_numpy((rows_of(p) @ p["W"].T).astype(np.float32)))
    h.close()


def test_quantised_weights_give_the_product_of_their_values(sp):
    """Export, product with rows in BF16 and in four bits, gradient: each as with the values that the export returns."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    W, x, dy = (torch.randn(s, device="cuda", generator=g) for s in ((300, 200), (90, 200), (90, 300)))
    codes, scales = torch.empty((300, 100), dtype=torch.uint8, device="cuda"), torch.empty((300, 7), dtype=torch.uint8, device="cuda")
    values = torch.empty_like(W)
    sp.spike_quantize_mx4(W, codes, scales, values=values)
    h = sp.dense_fused_create_mx4(codes, scales, 200, backward=True)
    xb = x.bfloat16()
    xc, xs = torch.empty((90, 100), dtype=torch.uint8, device="cuda"), torch.empty((90, 7), dtype=torch.uint8, device="cuda")
    xv = torch.empty_like(xb)
    sp.spike_quantize_mx4(xb, xc, xs, values=xv)
    y, y4, dx = torch.empty((90, 300), device="cuda"), torch.empty((90, 300), device="cuda"), torch.empty((90, 200), device="cuda")
    sp.dense_fused_forward(h, xb, y)
    sp.dense_fused_forward_mx4(h, xc, xs, y4)
    sp.dense_fused_backward(h, dy, dx=dx)
    torch.cuda.synchronize()
    v64 = host(values)
    for got, rows, K in ((y, host(xb) @ v64.T, 200), (y4, host(xv) @ v64.T, 200), (dx, host(dy) @ v64, 300)):
        mass = np.sqrt((host(dy if K == 300 else xb) ** 2).sum(axis=1, keepdims=True) * (v64 ** 2).sum(axis=0 if K == 300 else 1))
        # (mass bounds the sum of the products' sizes by no less than its K-th root of K: Cauchy; four-bit rows may be a quarter larger)
        assert (np.abs(host(got) - rows) <= 6 * U * np.sqrt(2 * K + 32) * 1.25 * np.sqrt(K) * mass + 2.0 ** -23 * mass).all()
    h.close()
