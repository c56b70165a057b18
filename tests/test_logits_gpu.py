"""GPU parity of the penalties, biases and masks on logits (head_logits.h) against the float64 definition.

A value goes through a division or product, two subtractions (one of a product) and an addition in FP32, each off by at most
half a unit of what it gives, u = 2^-24; then it is rounded to its type.  With t the largest of the sizes on the way,
that is at most 5 u t and half a unit of the type.
"""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_UNIT = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def strided(a, dtype, pad=0, offset=0, fill=0):
    """[S][n] evenly spaced rows (or [S] rows) with `pad` elements between them."""
    a = torch.as_tensor(np.ascontiguousarray(a)).to(dtype)
    rows, cols = math.prod(a.shape[:-1]), a.shape[-1]
    buf = torch.full((rows * (cols + pad) + offset,), fill, dtype=dtype, device="cuda")
    view = buf[offset:].view(*a.shape[:-1], cols + pad)[..., :cols]
    view.copy_(a)
    return view, buf


def inputs(S, n, V, L, n_bias, seed=0):
    r = np.random.default_rng([31, S, n, V, L, seed])
    few = max(1, min(V, 40))  # ids often repeat, and a few lie outside
    ids = np.where(r.random((S, L)) < 0.5, r.integers(0, few, (S, L)), r.integers(-3, V + 3, (S, L))).astype(np.int32)
    return {"ids": ids, "n_ids": r.integers(-1, L + 2, S).astype(np.int32), "n_prompt": r.integers(-1, L + 2, S).astype(np.int32),
            "drafts": r.integers(-1, min(V, 10) + 1, (S, n - 1)).astype(np.int32),
            "repetition": r.uniform(0.7, 1.5, S).astype(np.float32), "presence": r.uniform(-1, 1, S).astype(np.float32),
            "frequency": r.uniform(-0.5, 0.5, S).astype(np.float32),
            "bias_ids": r.integers(-1, min(V, 60) + 1, (S, n_bias)).astype(np.int32),
            "bias": r.normal(size=(S, n_bias)).astype(np.float32) * 3, "mask": r.random((S, n, V)) < 0.7}


def call(sp, logits, out, i, pad=0, offset=0, stream=None, **leave):
    """head_logits_adjust with device copies of `i`; leave: keys that are None."""
    d = {k: None if leave.get(k, 1) is None or i[k] is None else torch.from_numpy(np.ascontiguousarray(i[k])).cuda()
         for k in ("ids", "n_ids", "n_prompt", "drafts", "repetition", "presence", "frequency", "bias_ids", "bias")}
    if d["ids"] is not None and pad:
        d["ids"] = strided(i["ids"], torch.int32, pad, offset, 3)[0]
    if leave.get("mask", 1) is not None:
        d["mask"] = strided(so.pack_mask(i["mask"]).view(np.int32), torch.int32, pad, offset, -1)[0]
    torch.cuda.synchronize()
    sp.head_logits_adjust(logits, out, stream=stream, **d)
    torch.cuda.synchronize()


def check(x64, out, i, kind, **leave):
    arg = {k: (None if leave.get(k, 1) is None else i[k]) for k in i}
    want = so.logits_adjust(x64, **arg)
    got = out.double().cpu().numpy()
    assert (np.isneginf(got) == np.isneginf(want)).all()
    fine = ~np.isneginf(want)
    count = 64 + i["ids"].shape[1]
    biggest = np.abs(x64) * 1.5 + 0.5 * count + 1 + 12
    touched = want != x64
    lim = HALF_UNIT[kind] * 1.01 * np.abs(want) + np.where(touched, 5 * U * biggest, 0.0) + 2.0 ** -25 * touched
    assert (np.abs(got - want) <= lim)[fine].all(), np.max((np.abs(got - want) / lim)[fine])
    same = fine & ~touched
    assert (got[same] == x64[same]).all()


SHAPES = [(1, 1, 1, 1, 1), (2, 1, 33, 5, 3), (3, 5, 100, 40, 0), (1, 2, 2047, 300, 64), (2, 3, 2048, 17, 1), (2, 3, 2049, 1000, 5),
          (3, 32, 5000, 64, 9), (1, 5, 57344, 1500, 16), (5, 1, 4100, 0, 2), (2, 2, 1000, 9001, 300)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("S,n,V,L,n_bias", SHAPES)
def test_against_the_definition(sp, kind, S, n, V, L, n_bias):
    i = inputs(S, n, V, L, n_bias)
    r = np.random.default_rng([32, V])
    x = r.normal(size=(S, n, V)) * 4
    x[0, 0, 0] = -np.inf
    for pad, offset in ((0, 0), (3, 1), (8, 8)):
        logits, _ = strided(x, TYPES[kind], pad, offset, 5.0)
        out, buf = strided(np.zeros_like(x), TYPES[kind], pad, offset, 6.0)
        before = buf.clone()
        call(sp, logits, out, i, pad, offset)
        x64 = logits.double().cpu().numpy()
        check(x64, out, i, kind)
        out.zero_()
        before_rows = before.clone()
        assert torch.equal(buf, before_rows), "elements between rows were written"
    # in place, the same bits
    call(sp, logits, out, i, pad, offset)
    want = out.clone()
    call(sp, logits, logits, i, pad, offset)
    assert torch.equal(logits, want)


@pytest.mark.parametrize("without", [("ids",), ("n_ids",), ("n_prompt",), ("drafts",), ("repetition",), ("presence",), ("frequency",),
                                     ("bias_ids", "bias"), ("mask",), ("ids", "drafts"),
                                     ("ids", "n_ids", "n_prompt", "drafts", "repetition", "presence", "frequency", "bias_ids", "bias", "mask")])
def test_inputs_left_out(sp, without):
    i = inputs(3, 4, 3000, 90, 12)
    x = np.random.default_rng(33).normal(size=(3, 4, 3000)) * 4
    logits, out = strided(x, torch.float32)[0], torch.empty((3, 4, 3000), device="cuda")
    leave = {k: None for k in without}
    call(sp, logits, out, i, **leave)
    check(logits.double().cpu().numpy(), out, i, "f32", **leave)


def test_masks_that_leave_nothing_and_values_that_are_not_finite(sp):
    """An empty mask gives -inf throughout, whatever was there; NaN and +inf stay where they are allowed."""
    i = inputs(2, 2, 100, 20, 4)
    i["mask"][0, 0] = False
    i["mask"][1] = True
    x = np.random.default_rng(34).normal(size=(2, 2, 100))
    x[0, 0, :50], x[1, 1, 70], x[1, 1, 71], x[1, 0, 72] = np.nan, np.nan, np.inf, -np.inf
    i["ids"][:] = 5
    logits, out = strided(x, torch.float32)[0], torch.empty((2, 2, 100), device="cuda")
    call(sp, logits, out, i, bias_ids=None, bias=None)
    got = out.cpu().numpy()
    assert np.isneginf(got[0, 0]).all() and np.isnan(got[1, 1, 70]) and got[1, 1, 71] == np.inf and got[1, 0, 72] == -np.inf


def test_the_last_bias_counts_and_calls_repeat(sp):
    """The same token named many times: its last entry, every time."""
    i = inputs(1, 1, 500, 3000, 5000)
    i["bias_ids"][:] = np.random.default_rng(35).integers(0, 20, i["bias_ids"].shape)
    x = np.random.default_rng(36).normal(size=(1, 1, 500))
    logits, out = strided(x, torch.float32)[0], torch.empty((1, 1, 500), device="cuda")
    call(sp, logits, out, i)
    check(logits.double().cpu().numpy(), out, i, "f32")
    first = out.clone()
    for _ in range(3):
        call(sp, logits, out, i)
        assert torch.equal(out, first)


def test_streams_graphs_and_no_sequences(sp):
    i = inputs(4, 3, 2500, 200, 8)
    x = torch.randn((4, 3, 2500), device="cuda")
    out = torch.empty_like(x)
    d = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in i.items() if k != "mask"}
    d["mask"] = torch.from_numpy(so.pack_mask(i["mask"]).view(np.int32)).cuda()
    st = torch.cuda.Stream()
    sp.head_logits_adjust(x, out, **d)
    torch.cuda.synchronize()
    want = out.clone()
    out.zero_()
    st.wait_stream(torch.cuda.current_stream())
    sp.head_logits_adjust(x, out, stream=st, **d)
    st.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.head_logits_adjust(x, out, **d)
    for _ in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        d["ids"].copy_(torch.randint(0, 2500, d["ids"].shape, device="cuda"))
        sp.head_logits_adjust(x, out, **d)
        torch.cuda.synchronize()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    sp.head_logits_adjust(x[:0], out[:0])


def test_quotients_are_rounded_once(sp):
    """Every token seen once in the prompt: x / r and x * r bit for bit as FP32 gives them, for penalties near 1 and far from it."""
    r = torch.cat([torch.rand(60) * 1.5 + 0.5, torch.tensor([1.0, 0.0, 1e-40, 1e-20, 3.0, 1e20, 1e38, float("inf")])]).cuda()
    S, V = r.numel(), 3000
    x = (torch.randn((S, 1, V), device="cuda") * torch.exp(torch.randn((S, 1, V), device="cuda") * 8)).clamp(-1e30, 1e30)
    x[:, 0, :4] = torch.tensor([float("inf"), -float("inf"), 3e38, 1e-30], device="cuda")
    ids = torch.arange(V, dtype=torch.int32, device="cuda").repeat(S, 1)
    out = torch.empty_like(x)
    sp.head_logits_adjust(x, out, ids=ids, n_prompt=torch.full((S,), V, dtype=torch.int32, device="cuda"), repetition=r)
    torch.cuda.synchronize()
    rc, xc = r.cpu().numpy()[:, None, None], x.cpu().numpy()
    with np.errstate(all="ignore"):
        want = np.where(xc > 0, xc / rc, xc * rc)
    got = out.cpu().numpy()
    # (a quotient below 2^-126 may be a step of 2^-149 off)
    small = np.abs(want) < 2.0 ** -120
    assert ((got == want) | (np.isnan(got) & np.isnan(want)))[~small].all()
    assert (np.abs(got.astype(np.float64) - want) <= 2.0 ** -149)[small].all()


def test_refusals_of_the_binding(sp):
    x = torch.zeros((2, 3, 50), device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    for error, kw in ((TypeError, dict(out=x.bfloat16())), (ValueError, dict(out=torch.zeros((2, 3, 49), device="cuda"))),
                      (TypeError, dict(ids=i32(2, 4).long())), (ValueError, dict(ids=i32(3, 4))), (TypeError, dict(n_ids=i32(3))),
                      (TypeError, dict(drafts=i32(2, 3))), (TypeError, dict(bias_ids=i32(2, 4))),
                      (TypeError, dict(bias_ids=i32(2, 4), bias=torch.zeros(7, device="cuda"))), (ValueError, dict(mask=i32(2, 3, 1))),
                      (TypeError, dict(repetition=torch.zeros(2, device="cuda").double()))):
        kw = {"out": x, **kw}
        with pytest.raises(error):
            sp.head_logits_adjust(x, **kw)
