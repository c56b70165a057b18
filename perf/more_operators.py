"""Four-bit weights and activations, logits on their way to a token, and the norm of a step's gradients, as timed cases.

Next to the INT8 export and its projections stand the same ones in microscaled
four-bit floating point: blocks of 32 values of a row share a power of two, a
value is one of 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with a sign.  Beside the check of
drafted tokens stands what a serving loop does to logits before it (penalties
for tokens that were there, biases, a grammar's mask), and behind the gradients
their common norm and its clipping.  `listed()` holds the cases at the sizes of
the 22-block, 1536-wide decoder that `workloads.py` describes; `draw(rng)` gives
more of the same ranges.  With `own` false, `run` computes the plain forms; with
`own` true it calls the library.  All inputs are seeded and made on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

WIDTH, HIDDEN, VOCAB, BLOCKS = 1536, 6144, 57344, 22
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# a drawn case stays below the listed ones
MAX_FLOPS = 3e11
MAX_WEIGHTS = WIDTH * VOCAB
MAX_LOGITS = 64 * 5 * VOCAB


def _quant(name, M, K, x, pad=0):
    return {"name": name, "kind": "quant", "M": M, "K": K, "x": x, "pad": pad}


def _proj(name, K, M, B, x, y, act, bias=True, residual=False, pre=False, pad=0):
    """x: the input's type, "mx4" for rows of four-bit codes; y: the output's; pre: the values before the activation
    are kept for the backward pass; pad: extra elements of a row."""
    return {"name": name, "kind": "proj", "K": K, "M": M, "B": B, "x": x, "y": y, "act": act, "bias": bias,
            "residual": residual, "pre": pre, "pad": pad}


def listed():
    return [
        # the head's weights exported, and what the codes stand for kept to tune against
        _quant("quant_head", VOCAB, WIDTH, "f32"),
        # the activations of 64 sequences with four drafted tokens each, on their way to a four-bit product
        _quant("quant_b320", 320, WIDTH, "bf16"),
        # one token through a head of four-bit weights
        _proj("w4_head_b1", WIDTH, VOCAB, 1, "f32", "f32", "none", bias=False),
        # 64 sequences with four drafted tokens each through the FFN up projection
        _proj("w4_up_b320", WIDTH, HIDDEN, 320, "bf16", "bf16", "gelu"),
        # prefill of a long prompt in FP32, a length that fills no tile
        _proj("w4_up_b2500", WIDTH, HIDDEN, 2500, "f32", "f32", "gelu"),
        # a small serving batch through the attention output projection, rows and weights in four bits
        _proj("mx4_out_b7", WIDTH, WIDTH, 7, "mx4", "bf16", "none", residual=True),
        # a large batch of prompts through the FFN up projection, rows and weights in four bits
        _proj("mx4_up_b16384", WIDTH, HIDDEN, 16384, "mx4", "bf16", "gelu"),
        # the backward pass of a tuning step through frozen four-bit weights
        {"name": "w4_up_grad_b8192", "kind": "proj_grad", "K": WIDTH, "M": HIDDEN, "B": 8192, "x": "bf16", "y": "bf16",
         "act": "gelu", "bias": True, "pad": 0},
        # one sequence's next token: 1,500 tokens of history, no drafts
        {"name": "logits_s1", "kind": "logits", "S": 1, "n": 1, "V": VOCAB, "L": 1500, "logits": "f32", "mask": True,
         "biases": 16, "pad": 0},
        # four drafted tokens of each of 64 sequences, verified next
        {"name": "logits_s64", "kind": "logits", "S": 64, "n": 5, "V": VOCAB, "L": 4096, "logits": "f32", "mask": True,
         "biases": 64, "pad": 0},
        # the gradients of a tuning step of all biases
        {"name": "clip_biases", "kind": "clip", "table": 0, "blocks": BLOCKS, "D": WIDTH, "grad": "f32", "clips": True},
        # the same with the embedding table's
        {"name": "clip_table", "kind": "clip", "table": VOCAB, "blocks": BLOCKS, "D": WIDTH, "grad": "f32", "clips": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, wide):
    """A size between lo and hi: a multiple of 80 (of 16, and now and then of 64 or more) where `wide`, else odd."""
    n = _log_int(rng, lo, hi)
    return max(80, n // 80 * 80) if wide else n | 1


def draw(rng):
    kind = rng.choice(["quant", "proj", "proj", "proj", "proj_grad", "logits", "clip"])
    if kind == "quant":
        K = _size(rng, 33, HIDDEN, rng.random() < 0.7)
        M = max(1, min(_log_int(rng, 1, VOCAB), MAX_WEIGHTS // K))
        return {"kind": kind, "M": M, "K": K, "x": rng.choice(["f32", "bf16", "f16"]), "pad": rng.choice([0, 0, 8, 5])}
    if kind in ("proj", "proj_grad"):
        wide = rng.random() < 0.7  # a model's widths; else any
        K, M, B = _size(rng, 100, HIDDEN, wide), _size(rng, 100, VOCAB, wide), _log_int(rng, 1, 16384)
        M = M if M * K <= MAX_WEIGHTS else _size(rng, 100, MAX_WEIGHTS // K, wide)
        B = max(1, min(B, int(MAX_FLOPS / (2.0 * K * M))))
        case = {"kind": kind, "K": K, "M": M, "B": B, "act": rng.choice(["none", "relu", "gelu", "silu"]),
                "bias": rng.random() < 0.7, "pad": rng.choice([0, 0, 8, 5])}
        x = rng.choice(["f32", "bf16", "bf16", "f16", "mx4", "mx4"] if kind == "proj" else ["f32", "bf16", "bf16", "f16"])
        case["x"] = x
        case["y"] = rng.choice(["f32", "bf16", "bf16", "f16"]) if x == "mx4" else x if rng.random() < 0.7 else "f32"
        if kind == "proj":
            case.update(residual=rng.random() < 0.4, pre=rng.random() < 0.3)
        return case
    if kind == "logits":
        S, n, V = _log_int(rng, 1, 64), rng.choice([1, 1, 3, 5]), _size(rng, 1000, VOCAB, rng.random() < 0.5)
        S = max(1, min(S, MAX_LOGITS // (n * V)))
        return {"kind": kind, "S": S, "n": n, "V": V, "L": _log_int(rng, 8, 8192),
                "logits": rng.choice(["f32", "f32", "bf16", "f16"]), "mask": rng.random() < 0.7,
                "biases": rng.choice([0, 5, 64]), "pad": rng.choice([0, 0, 8, 3])}
    D = _size(rng, 64, 4096, rng.random() < 0.7)
    return {"kind": kind, "table": rng.choice([0, min(_log_int(rng, 100, VOCAB), MAX_WEIGHTS // D)]),
            "blocks": rng.randint(1, BLOCKS), "D": D, "grad": rng.choice(["f32", "f32", "bf16", "f16"]),
            "clips": rng.random() < 0.7}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rows(g, B, n, kind, pad, std=1.0):
    """[B, n] values ~ N(0, std) as a view of rows of n + pad elements."""
    return (torch.randn((B, n + pad), device="cuda", generator=g) * std).to(TYPES[kind])[:, :n]


def _encode(x):
    """Codes (two to a byte, the first in the low half), exponent bytes and values of FP32 rows [R, K]."""
    R, K = x.shape
    blocks = torch.zeros((R, (K + 31) // 32 * 32), device="cuda")
    blocks[:, :K] = x
    blocks = blocks.view(R, -1, 32)
    byte = ((blocks.abs().amax(dim=2).view(torch.int32) >> 23) - 2).clamp_min(0)
    size = blocks.abs() * ((254 - byte) << 23).view(torch.float32)[:, :, None]
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    size = (torch.round(size / step) * step).clamp_max(6.0)
    level = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size * 0.5 + 4)).to(torch.int32)
    code = (level + 8 * torch.signbit(blocks).to(torch.int32)).view(R, -1)
    scale = torch.where(byte == 0, 2.0 ** -127, (byte << 23).view(torch.float32))
    values = (torch.copysign(size, blocks) * scale[:, :, None]).view(R, -1)[:, :K]
    code = code[:, :(K + 1) // 2 * 2].view(R, -1, 2)  # (codes past K are zero)
    return (code[:, :, 0] + 16 * code[:, :, 1]).to(torch.uint8), byte.to(torch.uint8), values


def _padded(t, pad):
    """The same rows in a buffer of `pad` more elements a row."""
    if not pad:
        return t
    full = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    full[:, :t.shape[1]] = t
    return full[:, :t.shape[1]]


def _inputs(case, seed):
    """The case's plain inputs, from the seed alone."""
    g = _generator(seed)
    kind = case["kind"]
    if kind == "quant":
        # rows of unlike sizes, as outputs' weights and tokens' activations have
        x = torch.randn((case["M"], case["K"] + case["pad"]), device="cuda", generator=g)
        x *= torch.exp(torch.randn((case["M"], 1), device="cuda", generator=g)) * 0.02
        return {"x": x.to(TYPES[case["x"]])[:, :case["K"]]}
    if kind in ("proj", "proj_grad"):
        K, M, B, pad = case["K"], case["M"], case["B"], case["pad"]
        W = torch.randn((M, K), device="cuda", generator=g)
        W *= torch.empty((M, 1), device="cuda").uniform_(0.5, 1.5, generator=g) / math.sqrt(K)
        i = dict(zip(("codes", "scales"), _encode(W)))
        if kind == "proj":
            if case["x"] == "mx4":
                rows = _encode(torch.randn((B, K), device="cuda", generator=g))
                i["x_codes"], i["x_scales"] = _padded(rows[0], pad), _padded(rows[1], pad)
            else:
                i["x"] = _rows(g, B, K, case["x"], pad)
            i["residual"] = _rows(g, B, M, case["y"], pad) if case["residual"] else None
            i["bias"] = torch.randn(M, device="cuda", generator=g) * 0.1 if case["bias"] else None
        else:
            i["dy"] = _rows(g, B, M, case["y"], pad)
            i["pre"] = _rows(g, B, M, case["y"], pad) if case["act"] != "none" else None
        return i
    if kind == "logits":
        S, n, V, L = case["S"], case["n"], case["V"], case["L"]
        i = {"logits": (torch.randn((S, n, V + case["pad"]), device="cuda", generator=g) * 3.0).to(TYPES[case["logits"]])[:, :, :V]}
        # histories with the frequencies of text (rank r with weight 1 / (r + 2)), the ranks spread over the vocabulary
        u = torch.rand((S, L + n - 1), device="cuda", generator=g, dtype=torch.float64)
        rank = (2.0 * ((V + 2) / 2.0) ** u - 2.0).long().clamp_(0, V - 1)
        ids = (rank * (7919 if V % 7919 else 7907) % V).to(torch.int32)
        i["ids"], i["drafts"] = ids[:, :L].contiguous(), ids[:, L:].contiguous()
        i["n_ids"] = torch.randint(L // 2, L + 1, (S,), device="cuda", generator=g, dtype=torch.int32)
        i["n_prompt"] = (i["n_ids"] * torch.rand(S, device="cuda", generator=g)).to(torch.int32)
        spread = lambda lo, hi: torch.empty(S, device="cuda").uniform_(lo, hi, generator=g)  # noqa: E731
        i["repetition"], i["presence"], i["frequency"] = spread(1.0, 1.3), spread(0.0, 1.0), spread(0.0, 0.5)
        i["bias_ids"] = i["bias"] = None
        if case["biases"]:
            i["bias_ids"] = torch.randint(0, V, (S, case["biases"]), device="cuda", generator=g, dtype=torch.int32)
            # (what a token is named with again is what it had: its id decides)
            i["bias"] = (i["bias_ids"] % 17 - 8).float() * 0.75
        # a grammar allows a tenth of the words of a mask in full, and half of the bits of the others
        i["mask"] = None
        if case["mask"]:
            words = torch.randint(-2 ** 31, 2 ** 31, (S, n, (V + 31) // 32), device="cuda", generator=g)
            words[torch.rand(words.shape, device="cuda", generator=g) < 0.1] = -1
            i["mask"] = words.to(torch.int32)
        return i
    D = case["D"]
    sizes = ([case["table"] * D] if case["table"] else []) + [4 * D, D] * case["blocks"]
    grads = [(torch.randn(k, device="cuda", generator=g) * 0.01).to(TYPES[case["grad"]]) for k in sizes]
    norm = 0.01 * math.sqrt(sum(sizes))
    return {"grads": grads, "max_norm": norm * (0.3 if case["clips"] else 3.0)}


def prepare(case, seed):
    """Inputs, output buffers, and the handle of the weights laid out once or of the list of gradients."""
    s = dict(_inputs(case, seed), case=case)
    if not own:
        return s
    from paper_2606_03026_amd import _binding as sp

    kind = case["kind"]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "quant":
        M, K = case["M"], case["K"]
        s.update(codes=new(M, (K + 1) // 2, dtype=torch.uint8), scales=new(M, (K + 31) // 32, dtype=torch.uint8),
                 values=new(M, K, dtype=TYPES[case["x"]]))
    elif kind in ("proj", "proj_grad"):
        K, M, B = case["K"], case["M"], case["B"]
        s["act"] = {"none": sp.DENSE_ACT_NONE, "relu": sp.DENSE_ACT_RELU, "gelu": sp.DENSE_ACT_GELU,
                    "silu": sp.DENSE_ACT_SILU}[case["act"]]
        s["handle"] = sp.dense_fused_create_mx4(s["codes"], s["scales"], K, backward=kind == "proj_grad")
        if kind == "proj":
            s["out"] = new(B, M, dtype=TYPES[case["y"]])
            s["kept"] = new(B, M, dtype=TYPES[case["y"]]) if case["pre"] else None
        else:
            s["dx"] = new(B, K, dtype=TYPES[case["x"]])
            s["dbias"] = new(M) if case["bias"] else None
    elif kind == "logits":
        s["out"] = new(case["S"], case["n"], case["V"], dtype=TYPES[case["logits"]])
    else:
        s["outs"] = [torch.empty_like(t) for t in s["grads"]]
        s["handle"] = sp.spike_clip_create(s["grads"], s["outs"])
        s["result"] = new(2)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _decode(codes, scales, K):
    """FP32 rows [R, K] of codes and exponent bytes."""
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
    pairs = torch.stack([codes & 15, codes >> 4], dim=2).view(codes.shape[0], -1)[:, :K]
    byte = scales.to(torch.int32)
    scale = torch.where(byte == 0, 2.0 ** -127, (byte << 23).view(torch.float32))
    return levels[pairs.to(torch.int32)] * scale.repeat_interleave(32, dim=1)[:, :K]


def _plain_logits(s):
    case = s["case"]
    S, n, V, L = case["S"], case["n"], case["V"], case["L"]
    x = s["logits"].float()
    place = torch.arange(L, device="cuda")
    ids = s["ids"].long()
    said = ((place >= s["n_prompt"][:, None]) & (place < s["n_ids"][:, None])).float()
    prompt = (place < torch.minimum(s["n_prompt"], s["n_ids"])[:, None]).float()
    count = torch.zeros((S, V), device="cuda").scatter_add_(1, ids, said)[:, None, :].repeat(1, n, 1)
    seen = torch.zeros((S, V), device="cuda").scatter_add_(1, ids, prompt)[:, None, :]
    if n > 1:  # row j has the first j drafts behind its history
        j = torch.arange(n, device="cuda")
        ahead = (j[None, :-1] < j[:, None]).float().expand(S, n, n - 1)
        count.scatter_add_(2, s["drafts"].long()[:, None, :].expand(S, n, n - 1), ahead)
    r, p, f = (s[k][:, None, None] for k in ("repetition", "presence", "frequency"))
    y = torch.where((count > 0) | (seen > 0), torch.where(x > 0, x / r, x * r), x)
    y = y - f * count
    y = torch.where(count > 0, y - p, y)
    if s["bias"] is not None:
        bias = torch.zeros((S, V), device="cuda").scatter_(1, s["bias_ids"].long(), s["bias"])
        y = y + bias[:, None, :]
    if s["mask"] is not None:
        bit = (s["mask"][:, :, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        y = torch.where(bit.view(S, n, -1)[:, :, :V] != 0, y, -math.inf)
    return y.to(TYPES[case["logits"]])


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quant":
        codes, byte, values = _encode(s["x"].float())
        return codes, byte, values.to(TYPES[case["x"]])
    if kind == "proj":
        x = _decode(s["x_codes"], s["x_scales"], case["K"]) if case["x"] == "mx4" else s["x"].float()
        z = x @ _decode(s["codes"], s["scales"], case["K"]).t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        y = y.to(TYPES[case["y"]])
        return (y, z.to(TYPES[case["y"]])) if case["pre"] else y
    if kind == "proj_grad":
        g = s["dy"].float()
        if s["pre"] is not None:
            g = g * _act_grad(s["pre"].float(), case["act"])
        dx = (g @ _decode(s["codes"], s["scales"], case["K"])).to(TYPES[case["x"]])
        return (dx, g.sum(dim=0)) if case["bias"] else dx
    if kind == "logits":
        return _plain_logits(s)
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / norm).clamp_max(1.0)
    return [torch.stack([norm, factor])] + [(t.float() * factor).to(t.dtype) for t in s["grads"]]


def _own(s):
    from paper_2606_03026_amd import _binding as sp

    kind = s["case"]["kind"]
    if kind == "quant":
        sp.spike_quantize_mx4(s["x"], s["codes"], s["scales"], values=s["values"])
        return s["codes"], s["scales"], s["values"]
    if kind == "proj":
        if s["case"]["x"] == "mx4":
            sp.dense_fused_forward_mx4(s["handle"], s["x_codes"], s["x_scales"], s["out"], bias=s["bias"], act=s["act"],
                                       residual=s["residual"], pre=s["kept"])
        else:
            sp.dense_fused_forward(s["handle"], s["x"], s["out"], bias=s["bias"], act=s["act"], residual=s["residual"],
                                   pre=s["kept"])
        return s["out"] if s["kept"] is None else (s["out"], s["kept"])
    if kind == "proj_grad":
        sp.dense_fused_backward(s["handle"], s["dy"], dx=s["dx"], dbias=s["dbias"], act=s["act"], pre=s["pre"])
        return s["dx"] if s["dbias"] is None else (s["dx"], s["dbias"])
    if kind == "logits":
        sp.head_logits_adjust(s["logits"], s["out"], ids=s["ids"], n_ids=s["n_ids"], n_prompt=s["n_prompt"],
                              drafts=s["drafts"], repetition=s["repetition"], presence=s["presence"],
                              frequency=s["frequency"], bias_ids=s["bias_ids"], bias=s["bias"], mask=s["mask"])
        return s["out"]
    sp.spike_clip_forward(s["handle"], s["max_norm"], s["result"])
    return [s["result"]] + s["outs"]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------

def _coded(rows, K):
    """Bytes of rows of K four-bit values and their exponents."""
    return rows * ((K + 1) // 2 + (K + 31) // 32)


def work(case):
    kind = case["kind"]
    if kind == "quant":
        M, K = case["M"], case["K"]
        return {"bytes": 2 * M * K * BYTES[case["x"]] + _coded(M, K), "flops": 2.0 * M * K}
    if kind in ("proj", "proj_grad"):
        K, M, B = case["K"], case["M"], case["B"]
        ty = BYTES[case["y"]]
        wide = 1 + case["residual"] + case["pre"] if kind == "proj" else 1 + (case["act"] != "none")
        x = _coded(B, K) if case["x"] == "mx4" else B * K * BYTES[case["x"]]
        return {"bytes": _coded(M, K) + 4 * M * case["bias"] + x + B * M * ty * wide, "flops": 2.0 * B * M * K}
    if kind == "logits":
        S, n, V = case["S"], case["n"], case["V"]
        b = 2 * S * n * V * BYTES[case["logits"]] + S * (3 * case["L"] + 8 * case["biases"]) + S * n * V / 8 * case["mask"]
        return {"bytes": b, "flops": 4.0 * S * n * V}
    size = case["D"] * (case["table"] + 5 * case["blocks"])
    return {"bytes": 2 * size * BYTES[case["grad"]], "flops": 3.0 * size}


def _power(e):
    """2 ** e in 64 bits, exactly (a power function's last bit would move what lies between two levels)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(codes, scales, K):
    out = torch.zeros((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (codes.long() >> (4 * half)) & 15
        e, m = (c & 7) >> 1, (c & 1).double()
        size = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * _power(e - 1))
        out[:, half::2] = torch.where(c >= 8, -size, size)
    out = out[:, :K]
    power = _power(scales.long() - 127)
    return out * power[:, torch.arange(K, device="cuda") // 32]


def _exact_quant(x):
    """Nearest level by distance, ties to the one whose code is even; blocks by the exponent of their largest."""
    M, K = x.shape
    at = torch.arange(K, device="cuda") // 32
    top = torch.zeros((M, int(at[-1]) + 1), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(1, at.expand(M, K), x.abs(), "amax")
    power = _power((torch.frexp(top.clamp_min(2.0 ** -125)).exponent - 3).clamp_min(-127))[:, at]
    size, best, off = x.abs() / power, torch.zeros_like(x), torch.full_like(x, math.inf)
    for k in (0, 2, 4, 6, 1, 3, 5, 7):  # (an equal distance does not replace an even code)
        d = (size - LEVELS[k]).abs()
        best, off = torch.where(d < off, LEVELS[k], best), torch.minimum(d, off)
    return torch.where(x < 0, -best, best) * power


def exact(case, seed):
    i = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quant":
        return None, None, _exact_quant(i["x"].double())
    if kind == "proj":
        K = case["K"]
        x = _exact_rows(i["x_codes"], i["x_scales"], K) if case["x"] == "mx4" else i["x"].double()
        z = torch.mm(x, _exact_rows(i["codes"], i["scales"], K).t().contiguous())
        z = z if i["bias"] is None else z + i["bias"].double()
        y = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
             "silu": torch.nn.functional.silu}[case["act"]](z)
        y = y if i["residual"] is None else y + i["residual"].double()
        return (y, z) if case["pre"] else y
    if kind == "proj_grad":
        g = i["dy"].double()
        if i["pre"] is not None:
            z = i["pre"].double().requires_grad_(True)
            y = {"relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](z)
            g, = torch.autograd.grad(y, z, g)
        dx = torch.mm(g, _exact_rows(i["codes"], i["scales"], case["K"]))
        return (dx, g.sum(dim=0)) if case["bias"] else dx
    if kind == "logits":
        S, n, V = case["S"], case["n"], case["V"]
        out = torch.empty((S, n, V), dtype=torch.float64, device="cuda")
        for s in range(S):
            end = int(i["n_ids"][s])
            start = min(int(i["n_prompt"][s]), end)
            prompt = torch.bincount(i["ids"][s, :start].long(), minlength=V)
            r, p, f = (float(i[k][s]) for k in ("repetition", "presence", "frequency"))
            for j in range(n):
                said = torch.cat([i["ids"][s, start:end], i["drafts"][s, :j]]).long()
                c = torch.bincount(said, minlength=V)
                x = i["logits"][s, j].double()
                y = torch.where(c + prompt > 0, torch.where(x > 0, x / r, x * r), x) - f * c - p * (c > 0)
                if i["bias"] is not None:
                    extra = torch.zeros(V, dtype=torch.float64, device="cuda")
                    extra[i["bias_ids"][s].long()] = i["bias"][s].double()
                    y = y + extra
                if i["mask"] is not None:
                    at = torch.arange(V, device="cuda")
                    y = torch.where((i["mask"][s, j].long()[at // 32] >> (at % 32)) & 1 == 1, y, -math.inf)
                out[s, j] = y
        return out
    norm = math.sqrt(sum(float(t.double().pow(2).sum()) for t in i["grads"]))
    factor = min(1.0, i["max_norm"] / norm)
    return [torch.tensor([norm, factor], dtype=torch.float64, device="cuda")] + [t.double() * factor for t in i["grads"]]
