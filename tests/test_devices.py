"""Tensors of another device than the current one are refused by the bindings, whichever argument they are: the library would
read them from the current device's kernels.  On the CPU, with tensors that say where they are and a library that takes down calls."""
import pytest
import torch


class Placed(torch.Tensor):
    """A tensor that claims to lie on a device."""
    place = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.place


def on(place, *shape, dtype=torch.float32):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Placed)
    t.place = place
    return t


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 64 if name.endswith("workspace_bytes") else 0
        return call


@pytest.fixture
def sp(monkeypatch):
    from paper_2606_03026_amd import _binding
    monkeypatch.setattr(_binding, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return _binding


B, K, M, S, N, V = 40, 64, 96, 3, 2, 100
U8, I32 = torch.uint8, torch.int32
# entry point: {argument: (shape, type)}
CALLS = {
    "spike_quantize_mx4": dict(x=((M, K), None), codes=((M, K // 2), U8), scales=((M, 2), U8), values=((M, K), None)),
    "dense_fused_create_mx4": dict(codes=((M, K // 2), U8), scales=((M, 2), U8)),
    "dense_fused_forward": dict(x=((B, K), None), y=((B, M), None), bias=((M,), None), residual=((B, M), None), pre=((B, M), None),
                                workspace=((64,), U8)),
    "dense_fused_forward_mx4": dict(codes=((B, K // 2), U8), scales=((B, 2), U8), y=((B, M), None), bias=((M,), None),
                                    residual=((B, M), None), pre=((B, M), None), workspace=((64,), U8)),
    "dense_fused_backward": dict(dy=((B, M), None), dx=((B, K), None), dbias=((M,), None), pre=((B, M), None), workspace=((64,), U8)),
    "head_logits_adjust": dict(logits=((S, N, V), None), out=((S, N, V), None), ids=((S, 8), I32), n_ids=((S,), I32), n_prompt=((S,), I32),
                               drafts=((S, N - 1), I32), repetition=((S,), None), presence=((S,), None), frequency=((S,), None),
                               bias_ids=((S, 4), I32), bias=((S, 4), None), mask=((S, N, 4), I32)),
    "spike_clip_forward": dict(result=((2,), None), workspace=((64,), U8)),
}


def call(sp, name, places):
    args = {k: on(places.get(k, 0), *shape, dtype=dtype or torch.float32) for k, (shape, dtype) in CALLS[name].items()}
    extra = {}
    if name.startswith("dense_fused"):
        extra = {"K": K} if "create" in name else {"h": sp.DenseFused(1, K, M)}
    elif name == "spike_clip_forward":
        extra = {"h": sp.SpikeClip(1, (), torch.device("cuda", 0)), "max_norm": 1.0}
    if "create" not in name:
        extra["stream"] = 0
    return getattr(sp, name)(**args, **extra)


@pytest.mark.parametrize("name", CALLS)
def test_every_argument_is_looked_at(sp, name):
    call(sp, name, {})
    assert name in sp._lib.calls
    for k in CALLS[name]:
        sp._lib.calls.clear()
        with pytest.raises(ValueError, match=f"{k} is on .*current device"):
            call(sp, name, {k: 1})
        assert name not in sp._lib.calls


@pytest.mark.parametrize("where", ["grad", "out"])
def test_gradients_and_their_outputs(sp, where):
    grads, outs = [on(0, 8), on(0, 3)], [on(0, 8), None]
    sp.spike_clip_create(grads, outs)
    assert "spike_clip_create" in sp._lib.calls
    sp._lib.calls.clear()
    (grads if where == "grad" else outs)[0 if where == "out" else 1] = on(1, 8 if where == "out" else 3)
    with pytest.raises(ValueError, match="is on .*current device"):
        sp.spike_clip_create(grads, outs)
    assert "spike_clip_create" not in sp._lib.calls
    with pytest.raises(TypeError, match="device tensor"):
        sp.spike_clip_create([torch.zeros(8)])


def test_host_tensors_stay_refused_by_their_type(sp):
    with pytest.raises(TypeError, match="x must be a device tensor"):
        sp.dense_fused_forward(sp.DenseFused(1, K, M), torch.zeros(B, K), on(0, B, M), stream=0)
    with pytest.raises(TypeError, match="bias must be a device tensor"):
        sp.dense_fused_forward(sp.DenseFused(1, K, M), on(0, B, K), on(0, B, M), bias=torch.zeros(M),
                               workspace=on(0, 64, dtype=U8), stream=0)
    with pytest.raises(TypeError, match="logits must be a device tensor"):
        sp.head_logits_adjust(torch.zeros(S, N, V), on(0, S, N, V), stream=0)
