"""The tests' reference of the operators of a block with experts, held to what is known of them by other means."""
import numpy as np

import mx_experts_reference as E


def test_the_generator_gives_the_published_words():
    """The known answers that its authors publish for ten rounds: counter and key of zeros, of ones, and of digits of pi."""
    def words(counter, key):
        low, high = counter[0] | counter[1] << 32, counter[2] | counter[3] << 32
        return [int(w) for w in E.random_words([low], key[0] | key[1] << 32, high)[0]]

    ones = 0xFFFFFFFF
    assert words([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_sort_by_hand():
    offsets, place, order = E.sort([2, 0, 5, 2, -1, 0], 4)
    assert offsets.tolist() == [0, 2, 2, 4, 4]
    assert place.tolist() == [2, 0, -1, 3, -1, 1]
    assert order.tolist() == [1, 5, 0, 3, -1, -1]


def test_back_and_forth():
    """Gather and combine are each other's transpose, and the gradients are the differences."""
    g = np.random.default_rng(5)
    place = np.array([[3, -1], [0, 5], [-1, 9], [2, 1]])
    x, rows, w, r = g.standard_normal((4, 6)), g.standard_normal((7, 6)), g.standard_normal((4, 2)), g.standard_normal((4, 6))
    y, has = E.gather(x, place, 7)
    assert has.tolist() == [True, True, True, True, False, True, False]
    assert np.isclose((y * rows * has[:, None]).sum(), (x * E.combine(rows, place)[0]).sum())
    dx, _, dw, _ = E.combine_grad(r, place, w, rows)
    f = lambda rows, w: (E.combine(rows, place, w)[0] * r).sum()      # noqa: E731
    d = 1e-3 * g.standard_normal(rows.shape)
    assert np.isclose(f(rows + d, w) - f(rows - d, w), 2 * (dx * d).sum())
    d = 1e-3 * g.standard_normal(w.shape)
    assert np.isclose(f(rows, w + d) - f(rows, w - d), 2 * (dw * d).sum())


def test_ranges_are_cut_off():
    assert E.ranges([0, 3, 2, 9, 12], 10) == [(0, 3), (3, 3), (2, 9), (9, 10)]
