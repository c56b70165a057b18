"""Pins of the definitions in oracle/serve_oracle.py, on paper and by laws."""
import math

import numpy as np
import pytest

from oracle import serve_oracle as so


def test_levels_by_hand():
    """Every midpoint goes to the even code, what lies beside it to its side."""
    for size, code in ((0.0, 0), (0.25, 0), (0.2501, 1), (0.5, 1), (0.75, 2), (0.7499, 1), (1.25, 2), (1.26, 3), (1.75, 4),
                       (1.74, 3), (2.5, 4), (2.51, 5), (3.5, 6), (3.49, 5), (5.0, 6), (5.01, 7), (6.0, 7), (7.99, 7), (1e30, 7)):
        assert so.mx4_level(size) == code, size


def test_block_by_hand():
    """Largest size 5 in [4, 8): p = 2, e = 127, scale 1.  Largest 20: p = 4, e = 129, scale 4."""
    x = np.zeros((1, 40), np.float32)
    x[0, :5] = 5.0, -0.75, 0.2, -0.0, 2.5
    x[0, 32:35] = 20.0, -6.0, 1.0
    codes, scales, values = so.mx4_quantize(x)
    assert scales.tolist() == [[127, 129]]
    assert codes[0, :5].tolist() == [6, 10, 0, 8, 4] and codes[0, 32:35].tolist() == [6, 11, 0]
    assert values[0, :5].tolist() == [4.0, -1.0, 0.0, 0.0, 2.0] and values[0, 32:35].tolist() == [16.0, -6.0, 0.0]
    assert so.mx4_pack(codes)[0, :3].tolist() == [6 + 10 * 16, 0 + 8 * 16, 4]
    assert (so.mx4_values(codes, scales) == values).all()


def test_ends_of_the_range():
    """The largest FP32 exponent, subnormals (e stays 0), zeros, and what is not finite."""
    x = np.array([[np.finfo(np.float32).max], [2.0 ** -124], [2.0 ** -125], [2.0 ** -149], [0.0], [np.inf], [np.nan]], np.float32)
    codes, scales, values = so.mx4_quantize(x)
    assert scales[:, 0].tolist() == [252, 1, 0, 0, 0, 255, 255]
    assert codes[:, 0].tolist() == [7, 6, 6, 0, 0, 0, 0]
    assert values[0, 0] == 6 * 2.0 ** 125 and values[1, 0] == 2.0 ** -124 and values[2, 0] == 2.0 ** -125 and np.isnan(values[5:]).all()


def test_error_and_scaling():
    """Off by at most 1/8 of the block's largest up to 6 scales and 1/4 above, less than that elsewhere; powers of two go through."""
    r = np.random.default_rng(3)
    x = r.normal(size=(20, 70)).astype(np.float32)
    codes, scales, values = so.mx4_quantize(x)
    power = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)[:, :70]
    size = np.abs(x) / power
    step = np.where(size < 2, 0.25, np.where(size < 4, 0.5, 1.0))
    assert (np.abs(values - x) <= np.where(size > 6, size - 6, step) * power).all()
    c2, s2, v2 = so.mx4_quantize(x * np.float32(2.0 ** 9))
    assert (c2 == codes).all() and (s2 == scales + 9).all()


@pytest.mark.parametrize("mistake", ["ties_up", "no_saturation", "floor_scale", "block_16"])
def test_planted_mistakes_in_the_quantizer(mistake):
    x = np.zeros((1, 64), np.float32)
    x[0, :4] = 7.0, 2.5, 0.25, 5.0
    x[0, 20] = 0.3
    want = so.mx4_quantize(x)
    level, block = so.mx4_level, 32
    size = lambda v, e: abs(v) / 2.0 ** (e - 127)  # noqa: E731
    e = 127
    if mistake == "floor_scale":
        e = 126
    if mistake == "block_16":
        block = 16
    if mistake == "ties_up":
        level = lambda s: int(np.flatnonzero(np.abs(so.LEVELS - min(s, 6)) == np.abs(so.LEVELS - min(s, 6)).min())[-1])  # noqa: E731
    if mistake == "no_saturation":
        level = lambda s: so.mx4_level(s) if s <= 6 else 0  # noqa: E731
    got = [level(size(v, e if i < block else 123)) for i, v in enumerate(x[0, :32].astype(float))]
    assert got != want[0][0, :32].tolist()


def test_logits_by_hand():
    """V = 4, history 0 (prompt), 2, 2; then the draft 3: r = 2, f = 0.5, p = 0.25, bias 1 on token 1."""
    x = np.array([[[4.0, 1.0, -2.0, 3.0], [4.0, 1.0, -2.0, 3.0]]])
    ids = np.array([[0, 2, 2, 9]], np.int32)
    out = so.logits_adjust(x, ids=ids, n_ids=[3], n_prompt=[1], drafts=np.array([[3]]), repetition=[2.0], presence=[0.25],
                           frequency=[0.5], bias_ids=np.array([[1, 1]]), bias=np.array([[7.0, 1.0]]),
                           mask=np.array([[[1, 1, 1, 1], [0, 1, 1, 1]]], bool))
    assert out[0, 0].tolist() == [2.0, 2.0, -5.25, 3.0]
    assert out[0, 1].tolist() == [-np.inf, 2.0, -5.25, 0.75]


def test_logits_without_anything_are_themselves():
    x = np.random.default_rng(1).normal(size=(2, 3, 5))
    assert (so.logits_adjust(x) == x).all()
    assert (so.logits_adjust(x, ids=np.full((2, 4), -1), repetition=[2.0, 3.0], presence=[1, 1], frequency=[1, 1]) == x).all()


def test_mask_words():
    m = np.zeros((1, 1, 40), bool)
    m[0, 0, [0, 5, 31, 33]] = True
    assert so.pack_mask(m)[0, 0].tolist() == [1 + 32 + 2 ** 31, 2]


def test_clip_by_hand():
    norm, factor, out = so.clip([np.array([3.0, 0.0]), np.array([-4.0])], 2.5)
    assert norm == 5.0 and factor == 0.5 and out[0].tolist() == [1.5, 0.0] and out[1].tolist() == [-2.0]
    assert so.clip([np.array([3.0, 4.0])], 5.0)[1] == 1.0
    assert so.clip([np.zeros(3)], 1.0)[:2] == (0.0, 1.0)
    norm, factor, out = so.clip([np.array([np.inf, 1.0])], 1.0)
    assert math.isinf(norm) and factor == 1.0 and out[0].tolist() == [np.inf, 1.0]
