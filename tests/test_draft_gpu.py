"""GPU parity of the verification of drafted tokens (head_draft.h).

Tokens and counts equal the float64 definition's wherever no decision is
closer than 1e-5 (relative) to falling the other way: p and q carry FP32
rounding, u = 2^-24 times the size of the exponent (at most 60 here: 3.6e-6)
and a few more for the sum and the quotient; accept and prob are held to
4 u (60 + 32) = 2.2e-5 relative.
"""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NEAR, REL = 1e-5, 2.2e-5


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03026_amd import _binding
    return _binding


def problem(S, G, V, seed=0, ragged=True, banned=0.1):
    r = np.random.default_rng([31, S, G, V, seed])
    target = r.normal(0, 2.5, (S, G + 1, V))
    draft = target[:, :G] + r.normal(0, 0.7, (S, G, V))
    if banned:
        off = r.random(V) < banned
        off[r.integers(V)] = False
        target[:, :, off] = -np.inf
        draft[:, :, off] = -np.inf
    p = {"target": target, "draft": draft, "uniform": r.random((S, G)).astype(np.float32),
         "noise": r.exponential(size=(S, V)).astype(np.float32) + np.float32(1e-20),
         "temperature": np.where(r.random(S) < 0.2, 0.0, r.uniform(0.5, 1.5, S)).astype(np.float32),
         "n_draft": r.integers(0, G + 1, S).astype(np.int32) if ragged else None}
    hot = np.maximum(p["temperature"], 1e-3)[:, None, None]
    with np.errstate(invalid="ignore"):
        p["drafts"] = (draft / hot + r.gumbel(size=(S, G, V))).argmax(axis=2).astype(np.int32) if G else np.zeros((S, 0), np.int32)
    return p


def run(sp, p, kind="f32", pad=0, offset=0, dist=True, temperature=True, outputs=True, workspace=None, stream=None):
    S, G1, V = p["target"].shape
    G = G1 - 1

    def logits(a, n):
        buf = torch.full((S * n * (V + pad) + offset,), float("nan"), dtype=TYPES[kind], device="cuda")
        v = buf[offset:].view(S, n, V + pad)[:, :, :V]
        v.copy_(torch.from_numpy(a))
        return v

    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    target = logits(p["target"], G1)
    draft = logits(p["draft"], G) if dist and G else None
    noise = torch.full((S, V + pad), float("nan"), device="cuda")[:, :V]
    noise.copy_(torch.from_numpy(p["noise"]))
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    tokens, n = i32(S, G1), i32(S)
    accept = torch.full((S, G), -1.0, device="cuda") if outputs else None
    prob = torch.full((S, G1), -1.0, device="cuda") if outputs else None
    temp = p["temperature"] if temperature else None
    torch.cuda.synchronize()
    sp.head_draft_verify(target, draft, dev(p["drafts"]), dev(p["uniform"]), noise, tokens, n, accept=accept, prob=prob,
                         n_draft=dev(p["n_draft"]), temperature=dev(temp), workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    cpu = lambda t: None if t is None else t.float().cpu().numpy()  # noqa: E731
    want = so.draft_verify(cpu(target), cpu(draft), p["drafts"], p["uniform"], p["noise"], p["n_draft"], temp)
    return (tokens.cpu().numpy(), n.cpu().numpy(), cpu(accept), cpu(prob)), want


def check(got, want, near_allowed=True):
    tokens, n, accept, prob = got
    wt, wn, wa, wp, margin = want
    sure = margin > NEAR if near_allowed else np.ones(len(margin), bool)
    assert sure.mean() > 0.9
    assert (tokens[sure] == wt[sure]).all() and (n[sure] == wn[sure]).all(), np.argwhere((tokens != wt).any(axis=1) & sure)
    if accept is not None:
        assert (np.abs(accept - wa) <= REL * wa).all()
        assert (np.abs(prob - wp)[sure] <= REL * wp[sure]).all()


SHAPES = [(1, 0, 1), (1, 4, 1), (3, 1, 2), (2, 5, 33), (5, 3, 257), (1, 4, 5000), (2, 8, 2048), (7, 2, 2049), (40, 3, 1000), (3, 31, 130)]


@pytest.mark.parametrize("S,G,V", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dist", [True, False])
def test_against_definition(sp, S, G, V, kind, dist):
    for ragged, pad, offset in ((False, 0, 0), (True, 5, 1)):
        p = problem(S, G, V, ragged=ragged)
        check(*run(sp, p, kind, pad, offset, dist, temperature=ragged))


def test_vocabulary(sp):
    """The decoder's 57,344 slots, and rows that end inside a part."""
    for S, G, V in ((1, 4, 57344), (6, 4, 57344), (2, 2, 50001)):
        p = problem(S, G, V)
        check(*run(sp, p))
        check(*run(sp, p, dist=False, outputs=False))


def test_each_refusal_position(sp):
    """uniform forces acceptance (0) or refusal (1) at each place in turn."""
    G = 5
    p = problem(G + 1, G, 700, ragged=False)
    p["temperature"][:] = 1.0
    p["uniform"][:] = 0.0
    for j in range(G):
        p["target"][j, j, p["drafts"][j, j]] = -np.inf
    got, want = run(sp, p)
    assert got[1].tolist() == list(range(G + 1))
    check(got, want)
    for s in range(G + 1):
        assert (got[0][s, :s] == p["drafts"][s, :s]).all() and (got[0][s, s + 1:] == -1).all()


def test_equal_distributions(sp):
    """p = q: every draft of probability above 0 is accepted (u < 1); with u = 1 forced, r is zero and the target is raced instead."""
    p = problem(4, 3, 600, ragged=False, banned=0)
    p["draft"] = p["target"][:, :3].copy()
    p["temperature"][:] = 0.8
    check(*run(sp, p), near_allowed=False)
    assert (run(sp, p)[0][1] == 3).all()
    p["uniform"][:] = 1.0
    got, want = run(sp, p)
    assert (got[1] == 0).all() and (want[1] == 0).all()
    score = np.stack([so.probabilities(p["target"][s, 0], 0.8) for s in range(4)]) / p["noise"]
    assert (got[0][:, 0] == score.argmax(axis=1)).all()


def test_masked_rows(sp):
    """Rows that allow nothing: the draft is refused, the next token is -1; with NaN, -inf and the type's lowest value in masked places."""
    p = problem(4, 2, 300, ragged=False, banned=0)
    p["temperature"][:] = 1.0
    p["uniform"][:] = 0.0
    p["target"][0, 0] = -np.inf           # first row of the target
    p["target"][1, 0, ::2] = np.nan
    p["target"][1, 2] = np.nan            # the row after the last draft
    p["draft"][2, 0] = -np.inf            # the draft's own: accepted where the target allows the token
    p["target"][3, :, 5:] = np.finfo(np.float32).min
    p["drafts"][1, 0] = 1
    p["drafts"][3] = [0, 7]
    got, want = run(sp, p)
    check(got, want, near_allowed=False)
    assert got[1][0] == 0 and got[0][0].tolist() == [-1, -1, -1]
    assert got[1][1] == 2 and got[0][1, 2] == -1 and got[3][1, 2] == 0
    assert got[1][2] >= 1 and got[2][2, 0] == 1
    assert got[1][3] == 1 and 0 <= got[0][3, 1] < 5


def test_infinite_logits_share(sp):
    p = problem(1, 1, 100, ragged=False, banned=0)
    p["temperature"][:] = 0.7
    p["target"][0, :, [3, 60]] = np.inf
    p["drafts"][0, 0] = 60
    p["uniform"][:] = 0.0
    got, want = run(sp, p)
    check(got, want, near_allowed=False)
    assert got[3][0].tolist() == [0.5, 0.5] and got[0][0, 1] in (3, 60)


def test_greedy_ties_take_the_lowest(sp):
    for V in (9, 5000):
        p = problem(2, 2, V, ragged=False, banned=0)
        p["temperature"] = np.array([0.0, -1.0], np.float32)  # not positive: greedy too
        p["target"][:] = 0.0
        p["target"][:, :, [4, 7]] = 1.0
        p["drafts"][:] = [[4, 7], [7, 4]]
        got, want = run(sp, p, dist=False)
        check(got, want, near_allowed=False)
        assert got[0].tolist() == [[4, 4, -1], [4, -1, -1]]


def test_extreme_temperatures(sp):
    p = problem(4, 2, 400, ragged=False)
    p["temperature"] = np.array([1e-30, 1e30, np.inf, 0.01], np.float32)
    got, want = run(sp, p)
    n_allowed = np.isfinite(p["target"][0, 0]).sum()
    assert got[1][2] <= 2 and np.allclose(got[3][2][got[0][2] >= 0], 1.0 / n_allowed, rtol=1e-5)
    assert got[0][0, 0] == p["target"][0, 0].argmax()
    assert (got[0][:, 0] >= 0).all()


def test_bad_drafts_and_noise(sp):
    """Drafts outside the vocabulary are refused; noise that is not positive never wins; counts are clamped."""
    p = problem(4, 2, 50, ragged=False)
    p["drafts"][0, 0], p["drafts"][1, 0], p["drafts"][2, 0] = -1, 50, 2 ** 31 - 1
    p["noise"][:, ::2] = 0.0
    p["noise"][:, 1::4] = np.nan
    p["n_draft"] = np.array([9, 2, 2, -5], np.int32)
    for dist in (True, False):
        got, want = run(sp, p, dist=dist)
        check(got, want, near_allowed=False)
        assert (got[1][:3] == 0).all() and got[1][3] == 0
        assert all(t < 0 or t % 4 == 3 for t in got[0][:, 0])
    p["noise"][:] = 0.0
    assert (run(sp, p)[0][0][:, 0] == -1).all()


def test_law_of_the_tokens(sp):
    """4,000 sequences of 5 tokens: the first emitted token follows the target, within 5 standard deviations."""
    n, V = 4000, 5
    r = np.random.default_rng(32)
    pt, qt = np.array([0.4, 0.3, 0.15, 0.1, 0.05]), np.array([0.05, 0.1, 0.15, 0.3, 0.4])
    p = {"target": np.log(np.broadcast_to(pt, (n, 2, V))).copy(), "draft": np.log(np.broadcast_to(qt, (n, 1, V))).copy(),
         "drafts": r.choice(V, (n, 1), p=qt).astype(np.int32), "uniform": r.random((n, 1)).astype(np.float32),
         "noise": r.exponential(size=(n, V)).astype(np.float32), "temperature": None, "n_draft": None}
    got, want = run(sp, p, temperature=False)
    check(got, want)
    freq = np.bincount(got[0][:, 0], minlength=V) / n
    assert (np.abs(freq - pt) < 5 * np.sqrt(pt * (1 - pt) / n)).all()


def test_graph_replays_and_streams(sp):
    S, G, V = 5, 3, 3000
    p = problem(S, G, V)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    target, draft = dev(p["target"]).float(), dev(p["draft"]).float()
    drafts, uniform, noise, temp = (dev(p[k]) for k in ("drafts", "uniform", "noise", "temperature"))
    out = [torch.zeros((S, G + 1), dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda"),
           torch.zeros((S, G), device="cuda"), torch.zeros((S, G + 1), device="cuda")]
    ws = torch.full((sp.head_draft_workspace_bytes(S, G, V),), 255, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        sp.head_draft_verify(target, draft, drafts, uniform, noise, out[0], out[1], accept=out[2], prob=out[3],
                             temperature=temp, workspace=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        uniform.copy_(torch.rand(S, G))
        noise.exponential_()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        for t in out:
            t.zero_()
        ws.fill_(255)
        if i % 2:
            st = torch.cuda.Stream()
            st.wait_stream(torch.cuda.current_stream())
            step(st)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(out, want):
            assert torch.equal(t, w)


def test_no_sequences_and_refusals(sp):
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i32 = torch.int32
    sp.head_draft_verify(z(0, 3, 10), None, z(0, 2, t=i32), z(0, 2), z(0, 10), z(0, 3, t=i32), z(0, t=i32))
    args = dict(target=z(2, 3, 10), draft=z(2, 2, 10), drafts=z(2, 2, t=i32), uniform=z(2, 2), noise=z(2, 10),
                tokens=z(2, 3, t=i32), n_accepted=z(2, t=i32))
    for key, bad, err in (("draft", z(2, 3, 10), "draft"), ("drafts", z(2, 2, t=torch.int64), "drafts"),
                          ("uniform", z(2, 3), "uniform"), ("noise", z(2, 9), "noise"), ("tokens", z(2, 2, t=i32), "tokens"),
                          ("target", z(2, 3, 10, t=torch.float64), "type"), ("draft", z(2, 2, 10).bfloat16(), "draft"),
                          ("target", z(2, 10, 3).transpose(1, 2), "target")):
        with pytest.raises((TypeError, ValueError), match=err):
            sp.head_draft_verify(**{**args, key: bad})
    with pytest.raises(sp.SpikeError, match="workspace"):
        sp.head_draft_verify(**args, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="no workspace"):
        sp.head_draft_verify(z(1, 33, 4), None, z(1, 32, t=i32), z(1, 32), z(1, 4), z(1, 33, t=i32), z(1, t=i32))


@pytest.mark.parametrize("V", [50, 5000, 30000])
@pytest.mark.parametrize("dist", [True, False])
@pytest.mark.parametrize("bad", [0.0, -1.0, float("nan"), float("inf")])
def test_residual_without_usable_noise(sp, V, dist, bad):
    """r is max(p - q, 0) as soon as that is positive anywhere: where none of its tokens has noise that
    can win, nothing else wins in their place.  Sequence 1 has one such token left, sequence 2's draft is
    accepted (p itself is raced)."""
    p = problem(3, 1, V, ragged=False, banned=0)
    p["temperature"][:] = 1.0
    p["uniform"][:] = [[1.0], [1.0], [0.0]]
    few = np.arange(V) % 7 == 3  # with a distribution: p > q on these alone
    for s in range(3):
        p["draft"][s, 0] = p["target"][s, 0] + np.where(few & (np.arange(V) != p["drafts"][s, 0]), 0.0, 4.0)
    q = [so.probabilities(p["draft"][s, 0].astype(np.float32), 1.0) if dist else (np.arange(V) == p["drafts"][s, 0]) * 1.0
         for s in range(3)]
    for s in range(3):
        left = so.probabilities(p["target"][s, 0].astype(np.float32), 1.0) - q[s] > 0
        assert left.any() and not left.all()
        if s == 1:
            left[np.argmax(left)] = False  # the lowest keeps its noise
        p["noise"][s, left] = bad
    got, want = run(sp, p, dist=dist)
    assert want[0][0].tolist() == [-1, -1] and want[0][1, 0] >= 0 and want[1].tolist() == [0, 0, 1]
    assert (got[0] == want[0]).all() and (got[1] == want[1]).all()
    assert got[3][0, 0] == 0
