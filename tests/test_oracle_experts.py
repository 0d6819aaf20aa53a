"""Pins of the oracle's expert products, gated unit, gradients and four-bit rows: closed forms, double loops and central differences."""
import numpy as np
import pytest

from oracle import experts as ox


def case(seed, E=3, C=4, K=5, N=6):
    rng = np.random.default_rng(seed)
    counts = np.array([2, 0, 4])[:E]
    off = np.concatenate([[0], np.cumsum(counts)])
    x = rng.normal(size=(E, C, K))
    return rng, off, counts, x, rng.normal(size=(E, K, N))


def test_products_are_double_loops_over_the_filled_rows():
    rng, off, counts, x, W = case(0)
    y, size = ox.expert_matmul(x, W, off)
    for j in range(3):
        for s in range(4):
            for n in range(6):
                want = sum(x[j, s, k] * W[j, k, n] for k in range(5)) if s < counts[j] else 0.0
                assert np.isclose(y[j, s, n], want, rtol=1e-13, atol=1e-14)
    assert np.array_equal(ox.expert_matmul(x, W.transpose(0, 2, 1), off, transposed=True)[0], y)
    assert (size >= np.abs(y)).all()


def central(f, at, d, h=1e-6):
    return (f(at + h * d) - f(at - h * d)) / (2 * h)


def test_gradients_are_central_differences():
    rng, off, counts, x, W = case(1)
    dy = rng.normal(size=(3, 4, 6))
    keep = (np.arange(4)[None, :] < counts[:, None])[..., None]
    loss = lambda x_, W_: (ox.expert_matmul(x_, W_, off)[0] * dy).sum()     # noqa: E731
    d = rng.normal(size=x.shape)
    assert np.isclose(central(lambda a: loss(a, W), x, d), (ox.expert_matmul(dy, W, off, transposed=True)[0] * d * keep).sum(), rtol=1e-7)
    d = rng.normal(size=W.shape)
    assert np.isclose(central(lambda a: loss(x, a), W, d), (ox.expert_matmul_wgrad(x, dy, off)[0] * d).sum(), rtol=1e-7)
    gate_up, dh = rng.normal(size=(3, 4, 6)), rng.normal(size=(3, 4, 3))
    d = rng.normal(size=gate_up.shape)
    got, h = ox.swiglu_backward(gate_up, dh, off)
    assert np.isclose(central(lambda a: (ox.swiglu(a) * dh * keep).sum(), gate_up, d), (got * d).sum(), rtol=1e-7)
    assert np.allclose(h, ox.swiglu(gate_up) * keep)


def test_combine_backward_is_central_differences_of_combine():
    import oracle
    rng = np.random.default_rng(2)
    assign = np.array([[0, 1], [1, -1], [2, 0]])
    pos = np.array([[0, 0], [1, 0], [0, 1]])
    gates, eo, dy = rng.random((3, 2)), rng.normal(size=(3, 2, 5)), rng.normal(size=(3, 5))
    de, dg, _ = ox.combine_backward(dy, eo, assign, pos, gates)
    d = rng.normal(size=eo.shape)
    assert np.isclose(central(lambda a: (oracle.combine(a, assign, pos, gates) * dy).sum(), eo, d), (de * d).sum(), rtol=1e-7)
    d = rng.normal(size=gates.shape)
    assert np.isclose(central(lambda a: (oracle.combine(eo, assign, pos, a) * dy).sum(), gates, d), (dg * d).sum(), rtol=1e-7)


def test_silu_at_its_ends():
    v = ox.swiglu(np.array([[-1e4, -30.0, 0.0, 30.0, 1e4] + [1.0] * 5]))
    assert np.allclose(v, [[0.0, -30.0 * np.exp(-30.0), 0.0, 30.0, 1e4]], rtol=1e-12, atol=0)


def test_four_bit_numbers_ties_ends_and_blocks():
    block = np.zeros(32)
    block[:9] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9]
    codes, scales = ox.mxfp4_quantise(block)
    assert scales.tolist() == [127] and codes[:9].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 7]
    assert ox.mxfp4_values(codes, scales)[:9].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6]
    codes, scales = ox.mxfp4_quantise(-block * 2.0 ** 10)
    assert scales.tolist() == [137] and codes[:9].tolist() == [14, 8, 10, 10, 12, 12, 14, 14, 15]
    assert ox.mxfp4_quantise(np.zeros(32))[1].tolist() == [0]
    assert ox.mxfp4_quantise(np.full(32, 2.0 ** -140))[1].tolist() == [0]
    assert ox.mxfp4_quantise(np.where(np.arange(64) == 40, np.inf, 1.0))[1].tolist() == [125, 255]
    assert np.array_equal(ox.mxfp4_unpack(ox.mxfp4_pack(codes)), codes)


@pytest.mark.parametrize("seed", range(3))
def test_four_bit_rounding_is_within_half_a_step(seed):
    x = np.random.default_rng(seed).normal(size=(5, 96)) * 10.0 ** np.random.default_rng(seed).integers(-3, 3, size=(5, 1))
    codes, scales = ox.mxfp4_quantise(x)
    v = ox.mxfp4_values(codes, scales)
    unit = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=-1)
    m = np.abs(x) / unit
    step = np.where(m < 2, 0.5, np.where(m < 4, 1.0, 2.0))
    assert (np.abs(v - x) <= step / 2 * unit)[m <= 6].all() and (np.abs(v)[m > 6] == 6 * unit[m > 6]).all() and m.max() < 8
