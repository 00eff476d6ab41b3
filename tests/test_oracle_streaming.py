"""The 64-bit definitions of the streaming operators against hand-computed values and properties."""
import numpy as np
import pytest

from oracle import streaming as so


def test_rope_turns_pairs_and_keeps_the_rest():
    x = np.arange(8.0).reshape(1, 1, 8) + 1  # 1 .. 8
    ang = np.array([[np.pi / 2, np.pi]])
    half = so.rope(x, ang)[0, 0]
    # pairs (1, 3) by a quarter turn -> (-3, 1), (2, 4) by half a turn -> (-2, -4); 5 .. 8 kept
    assert np.allclose(half, [-3, -2, 1, -4, 5, 6, 7, 8])
    inter = so.rope(x, ang, interleaved=True, scale=2.0)[0, 0]
    assert np.allclose(inter, [-4, 2, -6, -8, 5, 6, 7, 8])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_scores_depend_on_the_distance_alone(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(1, 1, 32)), rng.normal(size=(1, 1, 32))
    f = 100.0 ** (-np.arange(16) / 16)

    def score(p, r):
        a = so.rope(q, so.rope_angles([p], f), interleaved)
        b = so.rope(k, so.rope_angles([r], f), interleaved)
        return float((a * b).sum())

    assert abs(score(5, 3) - score(1005, 1003)) < 1e-9
    assert abs(score(5, 3) - score(6, 3)) > 1e-3


def test_row_limits():
    assert so.row_limits(3, 3, 1).tolist() == [1, 2, 3]
    assert so.row_limits(3, 10, 1).tolist() == [8, 9, 10]
    assert so.row_limits(5, 5, 2).tolist() == [2, 2, 4, 4, 5]
    assert so.row_limits(4, 9, 0).tolist() == [9] * 4
    assert so.row_limits(4, 2, 1).tolist() == [-1, 0, 1, 2]  # more new tokens than the sequence holds
    assert so.row_limits(0, 7, 1).size == 0


def test_attention_of_chunks_equals_the_whole_prompt():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(21, 4, 8)), rng.normal(size=(21, 2, 8)), rng.normal(size=(21, 2, 8))
    whole = so.seq_attention(q, k, v, so.row_limits(21, 21, 7), 0.3)
    at = 0
    for n in (14, 7):  # whole blocks of 7
        part = so.seq_attention(q[at:at + n], k[:at + n], v[:at + n], so.row_limits(n, at + n, 7), 0.3)
        for a, b in zip(part, whole):
            assert np.allclose(a, b[at:at + n], atol=1e-12)
        at += n


def test_attention_leaves_out_what_a_row_does_not_see():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 1, 4)), rng.normal(size=(3, 1, 4)), rng.normal(size=(3, 1, 4))
    k[2], v[2] = np.nan, np.inf
    out, lse, _ = so.seq_attention(q, k, v, [0, 1, 2], 0.5)
    assert np.all(out[0] == 0) and lse[0, 0] == -np.inf
    assert np.allclose(out[1, 0], v[0, 0]) and np.isfinite(out[2]).all()
