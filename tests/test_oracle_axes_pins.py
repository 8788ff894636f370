"""The oracle of positions with axes and of the embedding by them."""
import numpy as np

from oracle import axes as A
from paper_2602_24082_b200 import binding as B


def test_without_spans_all_axes_are_the_packed_positions():
    rows = [[(3, (4, 1, 2))], [(1, (5,)), (6, (1, 1))]]
    pos = A.position_ids(rows, [], np.zeros((0, 3)))
    want = [0, 1, 2, 3, 4, 5, 6, 3, 3, 4, 0, 1, 2, 3, 4, 5, 0, 1, 2, 3, 4, 5, 6, 6]
    assert (pos == want).all()


def test_spans_count_with_their_longest_side():
    # text, a 1 x 2 x 3 image, text | response | response that begins with a 2 x 1 x 2 video
    pos = A.position_ids([[(9, (2, 5))]], [1, 11], [(1, 2, 3), (2, 1, 2)])
    assert pos.T.tolist() == [[0, 0, 0], [1, 1, 1], [1, 1, 2], [1, 1, 3], [1, 2, 1], [1, 2, 2], [1, 2, 3], [4, 4, 4],
                              [5, 5, 5], [6, 6, 6], [7, 7, 7], [6, 6, 6], [6, 6, 7], [7, 6, 6], [7, 6, 7], [8, 8, 8]]


def test_embedding_by_one_axis_is_the_plain_one_and_the_inverse_undoes_it():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(7, 2, 64))
    pos = rng.integers(0, 5000, 7)
    got = A.rope(x, pos[None], [0] * 32, 10000.0)
    i = np.arange(32)
    turn = np.exp(1j * pos[:, None] * 10000.0 ** (-i / 32))[:, None]
    z = (x[..., :32] + 1j * x[..., 32:]) * turn
    assert np.abs(got - np.concatenate([z.real, z.imag], -1)).max() < 1e-12
    assert np.abs(A.rope(got, pos[None], [0] * 32, 10000.0, True) - x).max() < 1e-12
    three = np.stack([pos, pos, pos])
    assert np.array_equal(got, A.rope(x, three, [0, 1, 2, 2] * 8, 10000.0))


def test_sections():
    assert list(B.axis_of_frequency((2, 3, 1))) == [0, 0, 1, 1, 1, 2]
    assert list(B.axis_of_frequency((2, 3, 1), True)) == [0, 1, 2, 0, 1, 1]
    assert list(B.axis_of_frequency((0, 2), True)) == [1, 1]
