"""GPU parity of the fused INT8 projection and its gradient (dense_fused.h)
against the float64 definition.

Where every value is a small integer the sums are exact in FP32, so the
outputs must match bit for bit (padding, tails, strides, layouts).  Elsewhere
the sums carry rounding: n additions of rounding u = 2^-24 each, taken as
independent, stay within

    lim = 6 u sqrt(n) sum_k |scale Q x|,  n = parts * K + 32

(parts: three BF16 parts of an FP32 activation or gradient at most; 32: waves, scale, bias).  The
activation adds at most 1e-6 + 4e-7 |y| (its polynomial's 1.7e-7 and ten FP32
operations), its slope is at most 1.13 in size, and storing rounds by half a
unit of the type.  In the backward pass each g * scale enters with 11
bits or more for BF16 dy (the bound allows 8) and with 16 or more for F16.
"""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from tests.launches import launches

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_UNIT = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}
ACTS = ["none", "relu", "gelu", "silu"]


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def dev(a, kind="f32", pad=0, offset=0):
    """Device tensor of array [B, n] in rows of n + pad elements, its first `offset` elements into the memory."""
    a = torch.as_tensor(np.ascontiguousarray(a)).to(TYPES[kind])
    B, n = a.shape
    buf = torch.full((B * (n + pad) + offset,), float("nan"), dtype=TYPES[kind], device="cuda")
    view = buf[offset:].view(B, n + pad)[:, :n]
    view.copy_(a)
    return view


def host(t):
    return t.detach().double().cpu().numpy()


def problem(K, M, B, seed=0, integer=False):
    r = np.random.default_rng([11, K, M, B, seed])
    if integer:
        return {"Q": r.integers(-8, 9, (M, K)).astype(np.int8), "scale": (2.0 ** r.integers(-2, 3, M)).astype(np.float32),
                "bias": r.integers(-4, 5, M).astype(np.float32), "x": r.integers(-3, 4, (B, K)).astype(np.float32),
                "residual": r.integers(-8, 9, (B, M)).astype(np.float32), "dy": r.integers(-3, 4, (B, M)).astype(np.float32)}
    return {"Q": np.clip(np.rint(r.normal(0, 30, (M, K))), -128, 127).astype(np.int8),
            "scale": (r.uniform(0.5, 1.5, M) / (30 * np.sqrt(K))).astype(np.float32),
            "bias": r.normal(0, 0.5, M).astype(np.float32), "x": r.normal(size=(B, K)).astype(np.float32),
            "residual": r.normal(size=(B, M)).astype(np.float32), "dy": r.normal(size=(B, M)).astype(np.float32)}


def handle(sp, p, backward=False):
    return sp.dense_fused_create(torch.from_numpy(p["Q"]).cuda(), torch.from_numpy(p["scale"]).cuda(), backward=backward)


def act_code(sp, act):
    return {"none": sp.DENSE_ACT_NONE, "relu": sp.DENSE_ACT_RELU, "gelu": sp.DENSE_ACT_GELU, "silu": sp.DENSE_ACT_SILU}[act]


def forward(sp, h, p, xk, yk, act="none", bias=True, residual=True, pre=False, pad=0, offset=0, stream=None):
    B, M = p["x"].shape[0], p["Q"].shape[0]
    x = dev(p["x"], xk, pad, offset)
    y = dev(np.full((B, M), np.nan), yk, pad, offset)
    z = dev(np.full((B, M), np.nan), yk, pad, offset) if pre else None
    res = dev(p["residual"], yk, pad, offset) if residual else None
    torch.cuda.synchronize()
    sp.dense_fused_forward(h, x, y, bias=torch.from_numpy(p["bias"]).cuda() if bias else None, act=act_code(sp, act),
                           residual=res, pre=z, stream=stream)
    torch.cuda.synchronize()
    want_z = so.fused_pre(p["Q"], p["scale"], host(x), p["bias"] if bias else None)
    want = so.act(want_z, act) + (host(res) if residual else 0.0)
    return (x, y, z), want, want_z


def check_forward(sp, p, xk, yk, act, out, want, want_z, residual=None):
    x, y, z = out
    K = p["Q"].shape[1]
    parts = 3 if xk == "f32" else 1
    mass = (np.abs(host(x)) @ np.abs(p["Q"].astype(np.float64)).T) * p["scale"].astype(np.float64)
    lim_z = 6 * U * np.sqrt(parts * K + 32) * (mass + np.abs(want_z))
    lim = 1.13 * lim_z + 1e-6 + 4e-7 * np.abs(want) + HALF_UNIT[yk] * np.abs(want) * 1.01 + 2.0 ** -25
    if residual is not None:
        lim += 2 * U * np.abs(residual)
    got = host(y)
    assert np.isfinite(got).all(), "outputs left unwritten"
    bad = np.abs(got - want) > lim
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], lim[bad][0])
    if z is not None:
        zlim = lim_z + HALF_UNIT[yk] * np.abs(want_z) * 1.01 + 2.0 ** -25
        assert (np.abs(host(z) - want_z) <= zlim).all()


# rows on both sides of every kernel's range, sizes that fill no tile, one input, one output
SHAPES = [(1, 1, 1), (7, 3, 2), (64, 16, 16), (65, 17, 17), (63, 15, 33), (100, 257, 5), (257, 100, 64), (1536, 130, 1),
          (1536, 384, 7), (640, 300, 65), (200, 520, 130), (129, 1040, 31), (1000, 257, 300), (320, 768, 513), (192, 1600, 1100)]


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
def test_integers_are_exact(sp, K, M, B, xk, yk):
    """Sums below 2^24 in steps of 1/4: the FP32 value is exact, so y is the correctly rounded result."""
    p = problem(K, M, B, integer=True)
    h = handle(sp, p)
    for act, pad, offset in (("none", 0, 0), ("relu", 5, 1)):
        (x, y, z), want, want_z = forward(sp, h, p, xk, yk, act=act, pre=True, pad=pad, offset=offset)
        assert torch.equal(y.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[yk])), (act, pad)
        assert torch.equal(z.cpu(), torch.from_numpy(want_z.astype(np.float32)).to(TYPES[yk])), (act, pad)
    h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk,act", [("f32", "f32", "gelu"), ("bf16", "bf16", "gelu"), ("f16", "f16", "silu"),
                                       ("bf16", "f32", "silu"), ("f32", "f32", "none")])
def test_forward(sp, K, M, B, xk, yk, act):
    p = problem(K, M, B)
    h = handle(sp, p)
    out, want, want_z = forward(sp, h, p, xk, yk, act=act, pre=True, pad=8 if K % 2 else 0)
    check_forward(sp, p, xk, yk, act, out, want, want_z, np.abs(p["residual"]))
    out, want, want_z = forward(sp, h, p, xk, yk, act=act, bias=False, residual=False)
    check_forward(sp, p, xk, yk, act, out, want, want_z)
    h.close()


def test_long_inputs(sp):
    """16,500 inputs and 20,000 outputs: long sums, many tiles."""
    for K, M, B, xk in ((16500, 40, 3, "f32"), (16500, 40, 70, "bf16"), (33, 20000, 2, "bf16"), (40, 20000, 100, "f32")):
        p = problem(K, M, B)
        h = handle(sp, p)
        out, want, want_z = forward(sp, h, p, xk, "f32", act="gelu", residual=False)
        check_forward(sp, p, xk, "f32", "gelu", out, want, want_z)
        h.close()


def test_wide_values(sp):
    """Large, tiny, subnormal activations keep their digits: FP32 parts cover the whole range."""
    p = problem(96, 32, 40)
    r = np.random.default_rng(5)
    p["x"] = (p["x"] * 10.0 ** r.uniform(-30, 30, p["x"].shape)).astype(np.float32)
    h = handle(sp, p)
    out, want, want_z = forward(sp, h, p, "f32", "f32", bias=False, residual=False)
    check_forward(sp, p, "f32", "f32", "none", out, want, want_z)
    h.close()


@pytest.mark.parametrize("xk", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B", [1, 20, 70])
def test_non_finite_inputs_stay_in_their_row(sp, xk, B):
    """An infinite activation gives infinities of the codes' signs (NaN where the code is 0), a NaN gives NaN; other rows are untouched."""
    p = problem(130, 50, B)
    p["Q"][:, 3] = np.where(np.arange(50) % 3 == 0, 0, np.where(np.arange(50) % 3 == 1, 5, -5)).astype(np.int8)
    p["x"][0, 3] = np.inf
    if B > 1:
        p["x"][1, 129] = np.nan
    h = handle(sp, p)
    with np.errstate(invalid="ignore"):
        (x, y, _), want, _ = forward(sp, h, p, xk, "f32", residual=False)
    got = host(y)
    assert np.isnan(got[0][0::3]).all() and (got[0][1::3] == np.inf).all() and (got[0][2::3] == -np.inf).all()
    if B > 1:
        assert np.isnan(got[1]).all()
    assert np.isfinite(got[2:]).all() and np.allclose(got[2:], want[2:], rtol=1e-3, atol=1e-3)
    h.close()


def test_activation_extremes(sp):
    """z far out on both sides, and 0: K = 1, scale 1, code 1."""
    z = np.array([[-200.0, -40.0, -13.0, -8.0, -3.0, -1e-30, 0.0, 1e-30, 3.0, 8.0, 40.0, 200.0]], np.float32).T
    p = {"Q": np.ones((1, 1), np.int8), "scale": np.ones(1, np.float32), "bias": np.zeros(1, np.float32), "x": z}
    h = handle(sp, p)
    for act in ACTS:
        (x, y, _), want, _ = forward(sp, h, p, "f32", "f32", act=act, residual=False)
        assert (np.abs(host(y) - want) <= 1e-6 + 4e-7 * np.abs(want)).all(), act
    h.close()


def test_residual_in_place_and_streams(sp):
    p = problem(200, 96, 40)
    h = handle(sp, p)
    x, r = dev(p["x"], "bf16"), dev(p["residual"], "bf16")
    y = torch.empty_like(r)
    sp.dense_fused_forward(h, x, y, residual=r)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    sp.dense_fused_forward(h, x, r, residual=r, stream=st)
    st.synchronize()
    assert torch.equal(r, y)
    h.close()


def backward(sp, h, p, xk, yk, act, pad=0, offset=0, z=None, want_dx=True, want_bias=True):
    B, M = p["dy"].shape
    K = p["Q"].shape[1]
    dy = dev(p["dy"], yk, pad, offset)
    pre = dev(z, yk, pad, offset) if act != "none" else None
    dx = dev(np.full((B, K), np.nan), xk, pad, offset) if want_dx else None
    db = torch.full((M,), float("nan"), device="cuda") if want_bias else None
    sp.dense_fused_backward(h, dy, dx=dx, dbias=db, pre=pre, act=act_code(sp, act))
    torch.cuda.synchronize()
    want = so.fused_backward(p["Q"], p["scale"], host(dy), None if pre is None else host(pre), act)
    return dx, db, want


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("bf16", "f32")])
def test_backward_of_integers_is_exact(sp, K, M, B, xk, yk):
    p = problem(K, M, B, integer=True)
    z = np.random.default_rng([12, K, M, B]).integers(-3, 4, (B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    for act, pad, offset in (("none", 0, 0), ("relu", 3, 1)):
        dx, db, (want, wb, _) = backward(sp, h, p, xk, yk, act, pad, offset, z)
        # dx of the narrow types is exact in FP32 first, then rounded once
        assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[xk])), act
        assert (db.cpu().numpy() == wb).all(), act
    h.close()


@pytest.mark.parametrize("K,M,B", SHAPES)
@pytest.mark.parametrize("xk,yk,act", [("f32", "f32", "gelu"), ("bf16", "bf16", "gelu"), ("f16", "f16", "silu"),
                                       ("bf16", "f32", "none"), ("f16", "f16", "none")])
def test_backward(sp, K, M, B, xk, yk, act):
    p = problem(K, M, B)
    z = np.random.default_rng([13, K, M, B]).normal(size=(B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    dx, db, (want, wb, g) = backward(sp, h, p, xk, yk, act, pad=8 if K % 2 else 0, z=z)
    w = np.abs(p["Q"].astype(np.float64)) * p["scale"].astype(np.float64)[:, None]
    parts = {"f32": 3, "bf16": 1, "f16": 2}[yk]
    entry = {"f32": 0.0, "bf16": HALF_UNIT["bf16"], "f16": 2.0 ** -15}[yk]  # cut at 16 bits: one sign, so twice 2^-16
    g_err = np.abs(host(torch.from_numpy(p["dy"]).to(TYPES[yk]))) * 1e-6 if act != "none" else 0.0
    lim = (6 * U * np.sqrt(parts * M + 32) * (np.abs(g) @ w) + 6 * entry * np.sqrt((g * g) @ (w * w))
           + (g_err @ w if act != "none" else 0.0) + HALF_UNIT[xk] * np.abs(want) * 1.01 + 2.0 ** -25)
    got = host(dx)
    assert (np.abs(got - want) <= lim).all(), np.max(np.abs(got - want) / lim)
    blim = 6 * U * np.sqrt(B + 8) * np.abs(g).sum(axis=0) + (g_err.sum(axis=0) if act != "none" else 0.0) + 1e-30
    assert (np.abs(host(db) - wb) <= blim).all()
    # one without the other
    _, db2, _ = backward(sp, h, p, xk, yk, act, pad=8 if K % 2 else 0, z=z, want_dx=False)
    dx2, _, _ = backward(sp, h, p, xk, yk, act, pad=8 if K % 2 else 0, z=z, want_bias=False)
    assert torch.equal(db, db2) and torch.equal(dx, dx2)
    h.close()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(sp, act):
    """dx and dbias along a direction against central differences of the definition in 64 bits."""
    p = problem(150, 90, 37)
    h = handle(sp, p, backward=True)
    r = np.random.default_rng(8)
    v, vb = r.normal(size=p["x"].shape), r.normal(size=90)
    z = so.fused_pre(p["Q"], p["scale"], p["x"], p["bias"])
    p["dy"] = r.normal(size=z.shape).astype(np.float32)
    dx, db, _ = backward(sp, h, p, "f32", "f32", act, z=z)
    f = lambda t: (so.fused_forward(p["Q"], p["scale"], p["x"] + t * v, p["bias"] + t * vb, act) * p["dy"]).sum()  # noqa: E731
    num = (f(1e-5) - f(-1e-5)) / 2e-5
    got = (host(dx) * v).sum() + (host(db) * vb).sum()
    # FP32 z (2^-24) and dx: each term within 1e-6 of its size
    assert abs(num - got) <= 2e-6 * (np.abs(host(dx) * v).sum() + np.abs(host(db) * vb).sum())
    h.close()


def test_no_rows(sp):
    p = problem(40, 24, 1)
    h = handle(sp, p, backward=True)
    empty = lambda n: torch.empty((0, n), device="cuda")  # noqa: E731
    sp.dense_fused_forward(h, empty(40), empty(24))
    db = torch.full((24,), 7.0, device="cuda")
    sp.dense_fused_backward(h, empty(24), dx=empty(40), dbias=db)
    torch.cuda.synchronize()
    assert (db == 0).all()
    h.close()


@pytest.mark.parametrize("B", [3, 90, 700])
def test_graph_replays(sp, B):
    """Captured forward and backward, replayed with eager work between: every replay gives the eager bits."""
    p = problem(320, 192, B)
    h = handle(sp, p, backward=True)
    x, dy = dev(p["x"], "bf16"), dev(p["dy"], "bf16")
    y, z, dx = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x)
    db, bias = torch.empty(192, device="cuda"), torch.from_numpy(p["bias"]).cuda()
    ws = torch.empty(sp.dense_fused_workspace_bytes(h, B, torch.bfloat16), dtype=torch.uint8, device="cuda")

    def step():
        sp.dense_fused_forward(h, x, y, bias=bias, act=sp.DENSE_ACT_GELU, pre=z)
        sp.dense_fused_backward(h, dy, dx=dx, dbias=db, pre=z, act=sp.DENSE_ACT_GELU, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        dy.copy_(torch.randn(dy.shape, device="cuda"))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, z, dx, db)]
        for t in (y, z, dx, db, ws):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((y, z, dx, db), want):
            assert torch.equal(t, w), i
    h.close()


def test_refusals(sp):
    p = problem(40, 24, 6)
    h = handle(sp, p)
    x, y = dev(p["x"]), torch.empty((6, 24), device="cuda")
    with pytest.raises(ValueError, match="must be"):
        sp.dense_fused_forward(h, x[:, :39], y)
    with pytest.raises(ValueError, match="must be"):
        sp.dense_fused_forward(h, x, y[:5])
    with pytest.raises(ValueError, match="contiguous rows"):
        sp.dense_fused_forward(h, x, torch.empty((24, 6), device="cuda").t())
    with pytest.raises(TypeError):
        sp.dense_fused_forward(h, x.double(), y)
    with pytest.raises(TypeError, match="residual"):
        sp.dense_fused_forward(h, x, y, residual=y.bfloat16())
    with pytest.raises(TypeError, match="bias"):
        sp.dense_fused_forward(h, x, y, bias=torch.zeros(23, device="cuda"))
    with pytest.raises(TypeError, match="device tensor"):
        sp.dense_fused_forward(h, x.cpu(), y)
    with pytest.raises(sp.SpikeError, match="activation"):
        sp.dense_fused_forward(h, x, y, act=9)
    with pytest.raises(sp.SpikeError, match="DENSE_FUSED_BACKWARD"):
        sp.dense_fused_backward(h, y, dx=torch.empty_like(x))
    with pytest.raises(sp.SpikeError, match="neither"):
        sp.dense_fused_backward(h, y)
    with pytest.raises(sp.SpikeError, match="pre"):
        sp.dense_fused_backward(h, y, dbias=torch.empty(24, device="cuda"), act=sp.DENSE_ACT_GELU)
    with pytest.raises(sp.SpikeError, match="workspace"):
        sp.dense_fused_backward(h, y, dbias=torch.empty(24, device="cuda"),
                                workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    h.close()


@pytest.mark.parametrize("xk", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("K,B", [(72, 40), (72, 600), (8, 70), (136, 300), (1000, 513)])
def test_nothing_is_left_from_the_call_before(sp, xk, K, B):
    """A call whose inputs are all NaN, then one of integers whose last step is short: nothing of the first is in the second."""
    p = problem(K, 520, B, integer=True)
    h = handle(sp, p)
    y = torch.empty((B, 520), device="cuda")
    x = dev(p["x"], xk)
    for n in (B, 2048):
        sp.dense_fused_forward(h, torch.full((n, K), float("nan"), device="cuda", dtype=TYPES[xk]), torch.empty((n, 520), device="cuda"))
    sp.dense_fused_forward(h, x, y)
    torch.cuda.synchronize()
    assert torch.equal(y.cpu(), torch.from_numpy(so.fused_pre(p["Q"], p["scale"], p["x"]).astype(np.float32)))
    h.close()


# sizes that take each kernel form: few rows by 1, 2 and 4 tiles of outputs (and two of
# rows); every tile shape (the template's tiles per wave, waves, stages and teams), with
# the steps in one part and in several
FEW = [(200, 100, 9), (100, 4200, 9), (72, 33000, 16), (72, 33000, 20)]
ONE_PLANE = [((4, 8, 4, 1, 2, 1), 1104, 4100, 3800, False), ((2, 8, 4, 1, 2, 1), 72, 4100, 1300, False),
             ((2, 4, 4, 1, 4, 1), 456, 384, 2752, False), ((1, 4, 4, 1, 4, 1), 72, 4100, 100, False),
             ((1, 4, 4, 1, 4, 1), 6000, 2100, 40, True), ((2, 4, 4, 1, 4, 2), 1000, 2100, 520, False),
             ((1, 2, 4, 1, 4, 2), 72, 70, 40, False), ((1, 2, 4, 1, 4, 2), 6000, 70, 40, True),
             ((1, 2, 4, 1, 4, 4), 2000, 70, 40, False), ((1, 2, 4, 1, 4, 4), 6000, 70, 1300, True)]
TWO_PLANES = [((4, 4, 4, 1, 2, 1), 1000, 4100, 2600, False), ((2, 2, 4, 1, 4, 1), 136, 1000, 2600, False),
              ((2, 2, 4, 1, 4, 1), 6000, 70, 1300, True), ((1, 2, 4, 1, 4, 1), 72, 70, 40, False),
              ((1, 2, 4, 1, 4, 1), 6000, 2100, 40, True), ((1, 2, 4, 1, 4, 2), 1000, 70, 40, False),
              ((1, 2, 4, 1, 4, 2), 2000, 70, 40, True), ((2, 4, 4, 1, 2, 1), 72, 4100, 1300, False),
              ((2, 4, 4, 1, 2, 1), 2000, 2100, 520, True)]


def kernel_names(sp, h, x, y):
    ws = torch.empty(max(1, sp.dense_fused_forward_workspace_bytes(h, x)), dtype=torch.uint8, device="cuda")
    return [name for name, _, _ in launches(lambda st: sp.dense_fused_forward(h, x, y, workspace=ws, stream=st))]


def check_integers(sp, h, p, xk, yk):
    for pad, offset in ((0, 0), (1, 1)):
        (x, y, z), want, want_z = forward(sp, h, p, xk, yk, act="relu", pre=True, pad=pad, offset=offset)
        assert torch.equal(y.cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[yk]))
        assert torch.equal(z.cpu(), torch.from_numpy(want_z.astype(np.float32)).to(TYPES[yk]))


@pytest.mark.parametrize("K,M,B", FEW)
@pytest.mark.parametrize("xk,yk", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_few_rows(sp, K, M, B, xk, yk):
    p = problem(K, M, B, integer=True)
    h = handle(sp, p)
    names = kernel_names(sp, h, dev(p["x"], xk), torch.empty((B, M), device="cuda"))
    assert len(names) == 1 and "k_fused_rows" in names[0]
    check_integers(sp, h, p, xk, yk)
    h.close()


@pytest.mark.parametrize("xk,shape,K,M,B,split", [(xk, *c) for xk in ("bf16", "f16") for c in ONE_PLANE if xk == "bf16" or c[3] < 3000]
                         + [("f32", *c) for c in TWO_PLANES])
def test_every_tile_shape(sp, xk, shape, K, M, B, split):
    p = problem(K, M, B, integer=True)
    h = handle(sp, p)
    names = kernel_names(sp, h, dev(p["x"], xk), torch.empty((B, M), device="cuda"))
    planes = 2 if xk == "f32" else 1
    assert any("k_fused_tile" in n and "".join(f"Li{v}E" for v in (planes, *shape)) in n for n in names), names
    assert any("k_fused_join" in n for n in names) == split
    assert any("k_fused_cut" in n for n in names) == (xk == "f32")
    check_integers(sp, h, p, xk, "f32")
    h.close()


@pytest.mark.parametrize("yk,shape,K,M,B,split", [("f32", *c) for c in TWO_PLANES] + [("bf16", *c) for c in ONE_PLANE])
def test_every_tile_shape_of_the_gradient(sp, yk, shape, K, M, B, split):
    p = problem(M, K, B, integer=True)
    h = handle(sp, p, backward=True)
    dy, dx = dev(p["dy"], yk), torch.empty((B, M), device="cuda")
    ws = torch.empty(sp.dense_fused_workspace_bytes(h, B, TYPES[yk]), dtype=torch.uint8, device="cuda")
    planes = 1 if yk == "bf16" else 2
    names = [n for n, _, _ in launches(lambda st: sp.dense_fused_backward(h, dy, dx=dx, workspace=ws, stream=st))]
    assert any("k_fused_tile" in n and "".join(f"Li{v}E" for v in (planes, *shape)) in n for n in names), names
    assert any("k_fused_join" in n for n in names) == split
    dx, _, (want, _, _) = backward(sp, h, p, "f32", yk, "none", want_bias=False)
    assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)))
    h.close()


# outputs on both sides of what a workgroup's threads hold, rows that the vectors do not fit
@pytest.mark.parametrize("M", [40, 2048, 2056, 4100, 8192, 8200, 14000, 33000])
@pytest.mark.parametrize("yk", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B", [33, 1100])
def test_gate_forms(sp, yk, M, B):
    """Every form of the gate: dx and dbias of integers, rows whole or at odd strides, one without the other."""
    p = problem(64, M, B, integer=True)
    z = np.random.default_rng([18, M, B]).integers(-3, 4, (B, M)).astype(np.float32)
    h = handle(sp, p, backward=True)
    for pad, offset in ((0, 0), (3, 1)):
        dx, db, (want, wb, _) = backward(sp, h, p, "f32", yk, "relu", pad, offset, z)
        assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32))) and (db.cpu().numpy() == wb).all()
    dx2, _, _ = backward(sp, h, p, "f32", yk, "relu", z=z, want_bias=False)
    _, db2, _ = backward(sp, h, p, "f32", yk, "relu", z=z, want_dx=False)
    assert torch.equal(dx, dx2) and torch.equal(db, db2)
    h.close()


@pytest.mark.parametrize("yk,entry", [("f32", 2.0 ** -23), ("bf16", 2.0 ** -11)])
@pytest.mark.parametrize("B", [50, 600])
def test_gradients_of_any_size(sp, yk, entry, B):
    """Rows of dy between 1e-34 and 1e30, one all zero, one infinite: each keeps its digits, none touches another."""
    p = problem(96, 200, B)
    r = np.random.default_rng([19, B])
    rows = 10.0 ** r.uniform(-34, 30, (B, 1))
    rows[0] = 0.0
    p["dy"] = (p["dy"] * rows).astype(np.float32)
    p["dy"][1, 7] = np.inf
    p["Q"][7, :] = np.where(np.arange(96) % 2, 5, -5).astype(np.int8)
    h = handle(sp, p, backward=True)
    dx, db, (want, _, g) = backward(sp, h, p, "f32", yk, "none")
    got = host(dx)
    assert (got[1] == np.where(np.arange(96) % 2, np.inf, -np.inf)).all() and (got[0] == 0).all()
    got, want, g = np.delete(got, 1, 0), np.delete(want, 1, 0), np.delete(g, 1, 0)
    w = np.abs(p["Q"].astype(np.float64)) * p["scale"].astype(np.float64)[:, None]
    lim = ((6 * U * np.sqrt(2 * 200 + 32) + 2 * U) * (np.abs(g) @ w) + 6 * entry * np.sqrt((g * g) @ (w * w))
           + 2.0 ** -39 * np.abs(g * p["scale"]).max(axis=1, keepdims=True) * np.abs(p["Q"].astype(np.float64)).sum(axis=0) + 2.0 ** -140)
    assert (np.abs(got - want) <= lim).all(), np.max(np.abs(got - want) / lim)
    h.close()


@pytest.mark.parametrize("K", [300, 2060, 5000])
def test_scaled_rows(sp, K):
    """FP32 rows of many sizes next to each other, and elements far below their row's largest.

    An element enters the product to 2^-23 of itself or to 2^-40 of its row's largest,
    whichever is more; the sums' rounding is as above.  The largest meets the code 0
    in every other output, so that the small ones have to carry those.
    """
    p = problem(K, 64, 100)
    r = np.random.default_rng([17, K])
    rows = 10.0 ** r.uniform(-36, 30, (100, 1))
    rows[:6, 0] = 1e-44, 1e-40, 1e-38, 3e-38, 1e30, 0.0
    below = 2.0 ** -r.uniform(0, 30, (100, 1))
    at = r.integers(0, K, 100)
    x = r.uniform(-1, 1, (100, K)) * rows * below
    x[np.arange(100), at] = rows[:, 0]
    p["x"] = x.astype(np.float32)
    p["Q"][::2, :] *= (np.bincount(at, minlength=K) == 0).astype(np.int8)
    h = handle(sp, p)
    (xd, y, _), want, want_z = forward(sp, h, p, "f32", "f32", bias=False, residual=False)
    w = np.abs(p["Q"].astype(np.float64)) * p["scale"].astype(np.float64)[:, None]
    x64 = np.abs(host(xd))
    top = x64.max(axis=1, keepdims=True)
    lim = (6 * U * np.sqrt(2 * K + 32) * (x64 @ w.T) + 2.0 ** -23 * (x64 @ w.T) + 2.0 ** -40 * top * w.sum(axis=1)
           + U * np.abs(want) + 2.0 ** -149 * 128)
    got = host(y)
    assert (np.abs(got - want) <= lim).all(), np.max(np.abs(got - want) / lim)
    h.close()


def test_rows_that_fill_no_chunk_are_cut_too(sp):
    """16-bit rows of an odd length, or off 16-byte boundaries, go through a plane."""
    for K, pad, offset in ((101, 0, 0), (96, 1, 0), (96, 0, 1)):
        p = problem(K, 64, 50, integer=True)
        h = handle(sp, p)
        x = dev(p["x"], "bf16", pad, offset)
        y = torch.empty((50, 64), device="cuda")
        assert any("k_fused_align" in n for n in kernel_names(sp, h, x, y))
        sp.dense_fused_forward(h, x, y)
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), torch.from_numpy(so.fused_pre(p["Q"], p["scale"], p["x"]).astype(np.float32)))
        h.close()


@pytest.mark.parametrize("yk", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K,M,B", [(70, 72, 40), (2000, 300, 90), (300, 6000, 333), (520, 2100, 700)])
def test_backward_forms(sp, yk, K, M, B):
    """Products of one and two planes in several shapes, split and not, the bias gradient summed beside them."""
    p = problem(K, M, B, integer=True)
    h = handle(sp, p, backward=True)
    dx, db, (want, wb, _) = backward(sp, h, p, "f32", yk, "none")
    assert torch.equal(dx.cpu(), torch.from_numpy(want.astype(np.float32)))
    assert (db.cpu().numpy() == wb).all()
    h.close()


@pytest.mark.parametrize("xk,yk", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("K,M,B", [(6000, 70, 40), (2000, 72, 40), (1000, 520, 300), (200, 96, 9)])
def test_residual_in_place_of_every_form(sp, xk, yk, K, M, B):
    """y is the residual: the sums in one part, split over workgroups and joined, and few rows, give the same as apart."""
    p = problem(K, M, B)
    h = handle(sp, p)
    x, r = dev(p["x"], xk), dev(p["residual"], yk)
    y = torch.empty_like(r)
    sp.dense_fused_forward(h, x, y, act=sp.DENSE_ACT_GELU, residual=r)
    sp.dense_fused_forward(h, x, r, act=sp.DENSE_ACT_GELU, residual=r)
    torch.cuda.synchronize()
    assert torch.isfinite(y.float()).all() and torch.equal(r, y)
    h.close()


def test_refusals_of_the_gradient_name_their_cause(sp):
    """A closed handle and too many rows have no workspace size: the call itself refuses them."""
    h = handle(sp, problem(8, 1, 1), backward=True)
    n = sp.FUSED_MAX_B + 1
    with pytest.raises(sp.SpikeError, match="B = "):
        sp.dense_fused_backward(h, torch.empty((n, 1), device="cuda"), dbias=torch.empty(1, device="cuda"))
    with pytest.raises(sp.SpikeError, match="B = "):
        sp.dense_fused_forward(h, torch.empty((n, 8), dtype=torch.bfloat16, device="cuda"), torch.empty((n, 1), device="cuda"))
    h.close()
    for B in (3, 40):
        with pytest.raises(sp.SpikeError, match="null handle"):
            sp.dense_fused_backward(h, torch.empty((B, 1), device="cuda"), dx=torch.empty((B, 8), device="cuda"))
        with pytest.raises(sp.SpikeError, match="null handle"):
            sp.dense_fused_forward(h, torch.empty((B, 8), device="cuda"), torch.empty((B, 1), device="cuda"))


def test_forward_workspace_is_what_the_query_says(sp):
    """Aligned 16-bit rows need none, except where the sums are split; FP32 rows and others need some."""
    for K, M, B, xk, some in ((192, 1600, 1100, "bf16", False), (6000, 70, 40, "bf16", True), (192, 1600, 1100, "f32", True), (6000, 70, 32, "f32", False)):
        h = handle(sp, problem(K, M, 1))
        x, y = torch.zeros((B, K), dtype=TYPES[xk], device="cuda"), torch.empty((B, M), device="cuda")
        n = sp.dense_fused_forward_workspace_bytes(h, x)
        assert (n > 0) == some
        sp.dense_fused_forward(h, x, y, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
        if n > 0:
            with pytest.raises(sp.SpikeError, match="workspace"):
                sp.dense_fused_forward(h, x, y, workspace=torch.empty(n - 16, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert (y == 0).all()
        h.close()
