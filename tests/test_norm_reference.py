"""The 64-bit reference of layer norm and dropout (norm_reference.py) against what is known of both: the generator's published
words, gradients by differences, the generator's two forms against each other."""
import numpy as np
import pytest

import norm_reference as ref

# counter, key, words: the test vectors published with the generator
KNOWN = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
         ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
         ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
          (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]


@pytest.mark.parametrize("counter, key, words", KNOWN)
def test_generator_gives_its_published_words(counter, key, words):
    assert tuple(ref.philox(counter, key)) == words


@pytest.mark.parametrize("first, n", [(0, 9), (3, 1), (5, 12), (2 ** 34 + 1, 7), (2 ** 32 * 4 - 2, 5)])
def test_vectorised_generator_is_the_scalar_one(first, n):
    seed, sequence = 0x123456789ABCDEF0, 0xFEDCBA9876543210
    key = (seed & 0xFFFFFFFF, seed >> 32)
    want = [ref.philox(((e // 4) & 0xFFFFFFFF, (e // 4) >> 32, sequence & 0xFFFFFFFF, sequence >> 32), key)[e % 4]
            for e in range(first, first + n)]
    assert ref.words(n, seed, sequence, first).tolist() == want


def test_kept_share_is_what_p_says():
    n = 200000
    for p in (0.1, 0.5, 0.9):
        share = 1 - ref.kept((n,), p, 7, 8).mean()
        assert abs(share - p) < 5 * np.sqrt(p * (1 - p) / n)  # five standard deviations, of a fixed draw
    assert ref.kept((n,), 0.0, 7, 8).all() and not ref.kept((n,), 1.0, 7, 8).any()


@pytest.mark.parametrize("shape", [(3, 5, 1), (2, 7, 4), (4, 1, 1), (1, 2, 3)])
def test_gradient_formula_against_differences(shape):
    """Central differences of L = sum(dy * y) in 64 bits: off by h^2 times a third derivative and by the rounding of L over h,
    1e-10 and some 1e-11 here (values of about one, h = 1e-5; rstd < 30 makes the derivative's factors some 1e4 at most)."""
    rng = np.random.default_rng(11)
    z, dy = rng.standard_normal(shape), rng.standard_normal(shape)
    gamma, beta, eps = rng.standard_normal(shape[1]), rng.standard_normal(shape[1]), 1e-2
    _, mean, rstd = ref.norm(z, gamma, beta, eps)
    dx, dgamma, dbeta = ref.norm_backward(dy, z, gamma, mean, rstd)

    def loss(z, gamma, beta):
        return (dy * ref.norm(z, gamma, beta, eps)[0]).sum()

    h = 1e-5
    for at in np.ndindex(shape):
        step = np.zeros(shape)
        step[at] = h
        assert abs((loss(z + step, gamma, beta) - loss(z - step, gamma, beta)) / (2 * h) - dx[at]) < 1e-5
    for c in range(shape[1]):
        step = np.zeros(shape[1])
        step[c] = h
        assert abs((loss(z, gamma + step, beta) - loss(z, gamma - step, beta)) / (2 * h) - dgamma[c]) < 1e-5
        assert abs((loss(z, gamma, beta + step) - loss(z, gamma, beta - step)) / (2 * h) - dbeta[c]) < 1e-5
