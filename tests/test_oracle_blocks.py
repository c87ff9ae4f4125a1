"""Pins of oracle/blocks.py: the generator's published known answers, chances
and layout of the bits, closed forms, and gradients by differences."""
import numpy as np
import pytest

from oracle import blocks as B


@pytest.mark.parametrize("ctr,key,want", [
    ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])])
def test_philox_known_answers(ctr, key, want):
    """The generator's own published test vectors for ten rounds."""
    assert [int(v) for v in B.philox(ctr, key)] == want


def test_kept_takes_its_bits_in_order():
    # counter (0, 0, 0, 0), key 0: halves e8d5.. of the first known answer, the lowest first
    halves = [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00]
    for t in sorted(halves):
        p = t / 65536.0
        got = B.kept(1, 8, p, 0, 0, 0)[0]
        assert got.tolist() == [65536.0 / (65536 - t) if h >= t else 0.0 for h in halves]
    # row, step and site are the counter's other words, the key is the seed's two
    ctr, key = [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]
    words = B.philox(ctr, key)
    want = [int(w) >> s & 0xFFFF for w in words for s in (0, 16)]
    seed = key[0] + (key[1] << 32)
    wide = B.philox([0] + ctr[1:], key)
    got = B.kept(1, 9, 0.5, seed, ctr[2] + (7 << 32), ctr[3], row0=ctr[1])[0]
    first = [int(w) >> s & 0xFFFF for w in wide for s in (0, 16)]
    assert (got[:8] > 0).tolist() == [h >= 32768 for h in first]
    assert len(want) == 8


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.05, 0.1, 0.25, 0.5, 0.9, 1.0])
def test_chances(p):
    k = B.kept(256, 1001, p, 12345, 6, 7)
    t = round(p * 65536)
    share = np.mean(k == 0)
    # five standard deviations of a share of 256256 draws
    assert abs(share - t / 65536) <= 5 * np.sqrt(t / 65536 * (1 - t / 65536) / k.size) + 1e-12
    assert abs(k.mean() - (1.0 if t < 65536 else 0.0)) <= 5 * np.sqrt((t / 65536) / max(1e-9, 1 - t / 65536) / k.size) + 1e-12


def test_draws_differ_by_seed_step_site_and_place():
    base = B.kept(64, 64, 0.5, 1, 2, 3)
    for other in ((2, 2, 3), (1 + 2 ** 32, 2, 3), (1, 3, 3), (1, 2, 4)):
        assert 0.4 < np.mean(B.kept(64, 64, 0.5, *other) == base) < 0.6
    assert (B.kept(64, 64, 0.5, 1, 2 + 2 ** 32, 3) == base).all()  # (a step's lowest 32 bits count)
    assert (B.kept(8, 64, 0.5, 1, 2, 3, row0=8) == base[8:16]).all()
    assert (B.kept(64, 13, 0.5, 1, 2, 3) == base[:, :13]).all()


def test_layernorm_closed_forms():
    y = B.layernorm([[1.0, 3.0]], [1.0, 2.0], [10.0, 20.0], 0.0)
    assert y.tolist() == [[9.0, 22.0]]
    assert B.layernorm([[5.0, 5.0, 5.0]], np.ones(3), np.ones(3), 1e-5).tolist() == [[1.0, 1.0, 1.0]]
    h = np.random.default_rng(0).standard_normal((5, 33))
    y = B.layernorm(h, np.ones(33), np.zeros(33), 0.0)
    assert np.allclose(y.mean(axis=1), 0, atol=1e-14) and np.allclose((y * y).mean(axis=1), 1, rtol=1e-13)
    assert np.allclose(B.layernorm(3 * h + 7, np.ones(33), np.zeros(33), 0.0), y, atol=1e-13)  # shift and scale


def test_layernorm_gradients_by_differences():
    g = np.random.default_rng(1)
    h, dy, dres = (g.standard_normal((3, 7)) for _ in range(3))
    gamma, beta = g.standard_normal(7), g.standard_normal(7)
    dh, dg, db = B.layernorm_bwd(dy, h, gamma, 1e-3, dres)
    loss = lambda a, b, c: np.sum(dy * B.layernorm(a, b, c, 1e-3)) + np.sum(dres * a)
    e = 1e-6
    for got, arg in ((dh, 0), (dg, 1), (db, 2)):
        args = [h, gamma, beta]
        for at in np.ndindex(got.shape):
            d = np.zeros_like(args[arg])
            d[at] = e
            up, down = ([a + (s * d if i == arg else 0) for i, a in enumerate(args)] for s in (1, -1))
            assert abs((loss(*up) - loss(*down)) / (2 * e) - got[at]) <= 1e-7


def test_cross_entropy_closed_forms():
    labels = np.array([0, 3, -1, 2])
    loss, row, lse, z = B.linear_xent(np.zeros((4, 2)), np.ones((2, 10)), None, labels, -1)
    assert np.allclose(row, [np.log(10)] * 2 + [0] + [np.log(10)], rtol=1e-15) and np.isclose(loss, np.log(10))
    # a bias of -Inf takes a class out
    bias = np.zeros(10)
    bias[5:] = -np.inf
    assert np.allclose(B.linear_xent(np.zeros((4, 2)), np.ones((2, 10)), bias, labels, -1)[2], np.log(5))
    assert B.linear_xent(np.zeros((2, 2)), np.ones((2, 4)), None, np.array([7, 7]), 7)[0] == 0.0
    assert np.isnan(B.linear_xent(np.zeros((2, 2)), np.ones((2, 4)), None, np.array([4, 1]), -1)[0])


def test_cross_entropy_gradients_by_differences():
    g = np.random.default_rng(2)
    x, w, bias = g.standard_normal((5, 4)), g.standard_normal((4, 6)), g.standard_normal(6)
    labels = np.array([1, 5, -1, 0, 1])
    _, _, lse, z = B.linear_xent(x, w, bias, labels, -1)
    grads = B.linear_xent_bwd(x, w, B.linear_xent_grad(z, lse, labels, -1), labels, -1, 3.0)
    e = 1e-6
    for arg, got in enumerate(grads):
        for at in np.ndindex(got.shape):
            args = [x, w, bias]
            d = np.zeros_like(args[arg])
            d[at] = e
            up, down = (B.linear_xent(*[a + (s * d if i == arg else 0) for i, a in enumerate(args)], labels, -1)[0]
                        for s in (1, -1))
            assert abs(3.0 * (up - down) / (2 * e) - got[at]) <= 1e-7
