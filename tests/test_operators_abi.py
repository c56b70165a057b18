"""Refusals of the C entry points of the operators around the projections: bad
arguments return a code and a message before anything reaches the GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def sp():
    from paper_2606_03026_amd import _binding
    return _binding


D = 0x1000  # an address that is never used: validation fails first


def test_fused(sp):
    lib = sp.raw_library()
    out = ctypes.c_void_p()
    create = lambda Q=D, s=D, K=64, M=32, f=0, o=ctypes.byref(out): lib.dense_fused_create(Q, s, K, M, f, o)  # noqa: E731
    for bad in (dict(Q=None), dict(s=None), dict(s=D + 2), dict(K=0), dict(M=0), dict(K=sp.FUSED_MAX_DIM + 1), dict(f=2), dict(o=None)):
        assert create(**bad) == sp.SPIKE_EINVAL, bad
        assert out.value is None and sp.spike_proj_last_error()
    assert create(K=1 << 16, M=1 << 15) == sp.SPIKE_EUNSUPPORTED
    assert lib.dense_fused_destroy(None) == sp.SPIKE_OK
    assert lib.dense_fused_forward(None, D, 0, 64, 1, None, 0, None, 0, D, 0, 32, None, 0, None, 0, None) == sp.SPIKE_EINVAL
    assert "handle" in sp.spike_proj_last_error()
    assert lib.dense_fused_backward(None, D, 0, 32, None, 0, 0, 1, D, 0, 64, D, D, 1 << 20, None) == sp.SPIKE_EINVAL
    assert lib.dense_fused_workspace_bytes(None, 4, 0) == -1


def test_embedding(sp):
    lib = sp.raw_library()
    f32, i8, i32 = sp.SPIKE_TYPE_F32, sp.SPIKE_TYPE_I8, sp.SPIKE_TYPE_I32

    def forward(table=D, tt=f32, rs=None, V=10, dim=8, ld=8, ids=D, it=i32, T=4, scale=1.0, out=D, ot=f32, ldo=8):
        return lib.spike_embed_forward(table, tt, rs, V, dim, ld, ids, it, T, scale, out, ot, ldo, None)

    for bad in (dict(table=None), dict(tt=i32), dict(tt=i8), dict(rs=D), dict(V=0), dict(V=sp.EMBED_MAX_V + 1), dict(dim=0),
                dict(dim=sp.EMBED_MAX_D + 1), dict(ld=7), dict(ids=None), dict(it=f32), dict(T=-1), dict(T=sp.EMBED_MAX_T + 1),
                dict(scale=float("inf")), dict(out=None), dict(ot=i8), dict(ldo=7), dict(table=D + 2), dict(ids=D + 2)):
        assert forward(**bad) == sp.SPIKE_EINVAL, bad
        assert sp.spike_proj_last_error()
    assert forward(T=0, table=None, ids=None, out=None) == sp.SPIKE_OK
    ws = lib.spike_embed_workspace_bytes(4, 8)
    assert ws > 0 and lib.spike_embed_workspace_bytes(-1, 8) == -1 and lib.spike_embed_workspace_bytes(4, 0) == -1
    assert lib.spike_embed_workspace_bytes(sp.EMBED_MAX_T, 65536) == -1

    def backward(grad=D, gt=f32, ldg=8, ids=D, it=i32, T=4, V=10, dim=8, scale=1.0, acc=0, dt=D, tt=f32, ld=8, w=D, n=ws):
        return lib.spike_embed_backward(grad, gt, ldg, ids, it, T, V, dim, scale, acc, dt, tt, ld, w, n, None)

    for bad in (dict(grad=None), dict(gt=i8), dict(ldg=7), dict(ids=None), dict(it=9), dict(T=-1), dict(V=0), dict(dim=0),
                dict(scale=float("nan")), dict(acc=2), dict(dt=None), dict(tt=i8), dict(ld=7), dict(w=None), dict(n=ws - 1),
                dict(w=D + 8), dict(grad=D + 1), dict(dt=D + 2)):
        assert backward(**bad) == sp.SPIKE_EINVAL, bad
    assert backward(T=sp.EMBED_MAX_T, dim=65536, ldg=65536, ld=65536) == sp.SPIKE_EUNSUPPORTED
    assert backward(T=0, acc=1, grad=None, ids=None, w=None, n=0) == sp.SPIKE_OK


def test_drafts(sp):
    lib = sp.raw_library()
    ws = lib.head_draft_workspace_bytes(2, 3, 100)
    assert ws > 0 and lib.head_draft_workspace_bytes(2, sp.DRAFT_MAX_G + 1, 100) == -1
    assert lib.head_draft_workspace_bytes(2, 3, 0) == -1

    def verify(target=D, ldt=100, draft=D, ldd=100, t=0, drafts=D, n_draft=None, u=D, noise=D, ldn=100, temp=None, S=2, G=3,
               V=100, tokens=D, n=D, accept=None, prob=None, w=D, nw=ws):
        return lib.head_draft_verify(target, ldt, draft, ldd, t, drafts, n_draft, u, noise, ldn, temp, S, G, V, tokens, n,
                                     accept, prob, w, nw, None)

    for bad in (dict(target=None), dict(ldt=99), dict(ldd=99), dict(t=3), dict(drafts=None), dict(u=None), dict(noise=None),
                dict(ldn=99), dict(S=-1), dict(G=-1), dict(V=0), dict(S=sp.DRAFT_MAX_S + 1), dict(G=sp.DRAFT_MAX_G + 1),
                dict(tokens=None), dict(n=None), dict(w=None), dict(nw=ws - 1), dict(w=D + 8), dict(target=D + 2),
                dict(accept=D + 1), dict(prob=D + 2), dict(temp=D + 1), dict(n_draft=D + 3)):
        assert verify(**bad) == sp.SPIKE_EINVAL, bad
        assert sp.spike_proj_last_error()
    assert verify(S=0, target=None, noise=None, tokens=None, n=None, w=None) == sp.SPIKE_OK
