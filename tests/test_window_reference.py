"""The plain implementations that the tests of the masked attention and of the 4-bit rows compare with: their own checks."""

import numpy as np
import pytest

import window_reference as R


def test_the_grid_and_its_ties():
    x = np.zeros((1, 64), dtype=np.float32)
    x[0, :17] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, 0.2500001, 0.7499999, 4.9999, 5.0001, -6, 6.9, 0.5]
    codes, scales = R.pack(x)
    assert scales.tolist() == [[127, 2]]                     # 6.9 rounds to 6; a block of zeros has the least scale
    got = R.unpack(codes, scales)[0, :17]
    assert got.tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, 0.5, 0.5, 4, 6, -6, 6, 0.5]
    x[0, 15] = 7                                             # would be 8: the next power of two
    codes, scales = R.pack(x)
    assert scales[0, 0] == 128 and R.unpack(codes, scales)[0, 15] == 8


def test_every_value_is_within_half_a_step_of_the_grid():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 128)) * np.exp2(rng.integers(-60, 60, (200, 1)))).astype(np.float32)
    got = R.unpack(*R.pack(x))
    top = np.abs(x.reshape(200, 4, 32)).max(-1).repeat(32, axis=1)
    # steps of the scale's binade: at most 2 * scale, and the scale is at most top / 3.5
    assert (np.abs(got - x) <= top / 3.5 + 1e-300).all()
    assert (R.unpack(*R.pack(got.astype(np.float32))) == got).all()


@pytest.mark.parametrize("n,W,causal,span,sinks,want", [
    (3, 2, True, 0, 0, ["110", "111"]),
    (5, 2, True, 2, 1, ["10110", "10011"]),
    (5, 1, False, 1, 0, ["00001"]),
    (2, 3, True, 0, 0, ["00", "10", "11"]),                  # one query before the first row
    (0, 2, True, 4, 4, ["", ""]),
    (4, 2, False, 2, 9, ["1111", "1111"]),
])
def test_visible_rows(n, W, causal, span, sinks, want):
    got = ["".join("01"[int(x)] for x in row) for row in R.visible(n, W, causal, span, sinks)]
    assert got == want


def test_attention_is_attention_over_the_tokens_that_slots_stand_for():
    rng = np.random.default_rng(2)
    Q, K, V = rng.standard_normal((2, 3, 64)), rng.standard_normal((9, 64)), rng.standard_normal((9, 64))
    c = rng.integers(1, 4, 9)
    a, off = R.attention(Q, K, V * c[:, None], causal=False, span=0, sinks=0, counts=c)
    b, _ = R.attention(Q, K.repeat(c, 0), V.repeat(c, 0), causal=False, span=0, sinks=0)
    assert np.abs(a - b).max() < 1e-12 and (off > 0).all() and off.max() < 1e-3
