"""Refusals of the C entry points of four-bit weights, logits and clipping: bad arguments return a code and a
message before anything reaches the GPU; and what the calls launch, recorded on the CPU."""
import ctypes

import pytest

from tests.test_launch_limits import record  # noqa: F401  (the fixture)

D = 0x1000  # an address that is never used: validation fails first
P = 1 << 40  # one that no recorded launch reads


@pytest.fixture(scope="module")
def sp():
    from paper_2606_03026_amd import _binding
    return _binding


def test_quantizer(sp):
    lib = sp.raw_library()

    def call(x=D, t=0, ldx=64, M=3, K=64, c=D, ldc=32, s=D, lds=2, v=None, ldv=0):
        return lib.spike_quantize_mx4(x, t, ldx, M, K, c, ldc, s, lds, v, ldv, None)

    for bad in (dict(x=None), dict(t=3), dict(ldx=63), dict(M=-1), dict(M=(1 << 24) + 1), dict(K=0), dict(K=(1 << 24) + 1), dict(c=None),
                dict(ldc=31), dict(s=None), dict(lds=1), dict(v=D, ldv=63), dict(x=D + 2), dict(v=D + 2, ldv=64), dict(v=D, ldv=65),
                dict(M=1 << 16, K=1 << 16, ldx=1 << 16, ldc=1 << 15, lds=1 << 11), dict(K=65, ldx=65), dict(K=65, ldx=65, ldc=33)):
        assert call(**bad) == sp.SPIKE_EINVAL, bad
        assert sp.spike_proj_last_error()
    assert call(M=0, x=None, c=None, s=None) == sp.SPIKE_OK


def test_four_bit_handles(sp):
    lib = sp.raw_library()
    out = ctypes.c_void_p()
    create = lambda c=D, ldc=32, s=D, lds=2, K=64, M=32, f=0, o=ctypes.byref(out): lib.dense_fused_create_mx4(c, ldc, s, lds, K, M, f, o)  # noqa: E731
    for bad in (dict(c=None), dict(s=None), dict(ldc=31), dict(lds=1), dict(K=0), dict(M=0), dict(K=sp.FUSED_MAX_DIM + 1), dict(f=2), dict(o=None),
                dict(K=65), dict(K=65, ldc=33)):
        assert create(**bad) == sp.SPIKE_EINVAL, bad
        assert out.value is None and sp.spike_proj_last_error()
    assert create(K=1 << 16, M=1 << 15) == sp.SPIKE_EUNSUPPORTED
    assert lib.dense_fused_forward_mx4(None, D, 32, D, 2, 1, None, 0, None, 0, D, 0, 32, None, 0, None, 0, None) == sp.SPIKE_EINVAL
    assert "handle" in sp.spike_proj_last_error()
    assert lib.dense_fused_forward_mx4_workspace_bytes(None, D, 32, D, 2, 40) == -1


def test_logits(sp):
    lib = sp.raw_library()

    def call(x=D, ldx=100, t=0, S=2, n=3, V=100, ids=D, ldi=8, L=8, n_ids=None, n_prompt=None, drafts=D, r=None, p=None, f=None, bi=None, b=None,
             nb=0, m=None, ldm=4, out=D, ldo=100):
        return lib.head_logits_adjust(x, ldx, t, S, n, V, ids, ldi, L, n_ids, n_prompt, drafts, r, p, f, bi, b, nb, m, ldm, out, ldo, None)

    for bad in (dict(x=None), dict(out=None), dict(ldx=99), dict(ldo=99), dict(t=4), dict(S=-1), dict(S=sp.LOGITS_MAX_S + 1), dict(n=0),
                dict(n=sp.LOGITS_MAX_N + 1), dict(V=0), dict(V=sp.LOGITS_MAX_V + 1), dict(L=-1), dict(L=sp.LOGITS_MAX_L + 1), dict(ldi=7),
                dict(nb=-1), dict(nb=sp.LOGITS_MAX_BIAS + 1), dict(nb=2), dict(nb=2, bi=D), dict(nb=2, b=D), dict(m=D, ldm=3), dict(x=D + 2),
                dict(ids=D + 1), dict(r=D + 2), dict(p=D + 1), dict(f=D + 3), dict(drafts=D + 2), dict(m=D + 1), dict(n_ids=D + 2),
                dict(n_prompt=D + 1), dict(out=D, ldo=101)):
        assert call(**bad) == sp.SPIKE_EINVAL, bad
        assert sp.spike_proj_last_error()
    assert call(S=0, x=None, out=None) == sp.SPIKE_OK


def test_clipping(sp):
    lib = sp.raw_library()
    out = ctypes.c_void_p()

    def create(grads=(P, P + 4096), outs=None, types=(0, 1), sizes=(8, 8), n=2, o=ctypes.byref(out)):
        g = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
        q = None if outs is None else (ctypes.c_void_p * len(outs))(*outs)
        return lib.spike_clip_create(g, q, None if types is None else (ctypes.c_int32 * len(types))(*types),
                                     None if sizes is None else (ctypes.c_int64 * len(sizes))(*sizes), n, o)

    for bad in (dict(grads=None), dict(types=None), dict(sizes=None), dict(n=-1), dict(n=sp.CLIP_MAX_TENSORS + 1), dict(o=None),
                dict(types=(0, 3)), dict(sizes=(8, -1)), dict(sizes=(8, (1 << 40) + 1)), dict(sizes=(1 << 40, 1)), dict(grads=(P, None)),
                dict(grads=(P + 2, P + 4096)), dict(grads=(P, P + 4097)), dict(grads=(P, P + 30)), dict(outs=(P + 4, None)), dict(outs=(P + 8192, P + 8192)),
                dict(outs=(P + 4096, None)), dict(outs=(P + 4096, P)), dict(outs=(P + 8192, P + 8193))):
        assert create(**bad) == sp.SPIKE_EINVAL, bad
        assert out.value is None and sp.spike_proj_last_error()
    assert lib.spike_clip_destroy(None) == sp.SPIKE_OK and lib.spike_clip_workspace_bytes(None) == -1
    assert lib.spike_clip_forward(None, 1.0, D, D, 1 << 20, None) == sp.SPIKE_EINVAL


def test_launches_of_the_largest_sizes(record):  # noqa: F811
    """Fewer than 2^32 threads a launch, whatever the sizes."""
    logits = [["head_logits_adjust", "pliiiiplippppppppiplplp",
               [P, V, t, S, n, V, P, 1 << 22, 1 << 22, None, None, P, P, P, P, P, P, 1 << 16, P, (V + 31) // 32, P, V, None], -1]
              for t in (0, 1) for S, n, V in ((4096, 32, 1 << 30), (4096, 1, 57344), (1, 1, 1), (64, 5, 57344))]
    quant = [["spike_quantize_mx4", "piliiplplplp", [P, t, K, M, K, P, (K + 1) // 2, P, (K + 31) // 32, P, K, None], -1]
             for t in (0, 2) for M, K in ((1 << 24, 1), (1 << 24, 128), (1 << 7, 1 << 24), ((1 << 24) - 1, 127), (57344, 1536))]
    for c, (rc, launches) in zip(logits + quant, record(logits + quant)):
        assert rc == 0 and len(launches) == 1 and all(0 < g * b < 1 << 32 for g, b in launches), (c[2][:6], launches)


def test_a_refused_launch_is_reported(record):  # noqa: F811
    logits = ["head_logits_adjust", "pliiiiplippppppppiplplp", [P, 100, 0, 2, 1, 100] + [None, 0, 0] + [None] * 8 + [0, None, 0, P, 100, None], 0]
    quant = ["spike_quantize_mx4", "piliiplplplp", [P, 0, 64, 2, 64, P, 32, P, 2, None, 0, None], 0]
    for rc, launches in record([logits, quant]):
        assert rc == -2 and len(launches) == 1
