"""The bounds of sum_error.py hold for sums in f32 (rounded, or cut at every step) and not for operands or partial sums in fewer
bits; no device."""
import numpy as np
import pytest

from tests.sum_error import fma_bound, off, tensor_bound


def keep(a, bits, cut=False):
    """a with `bits` significant bits, rounded or cut."""
    m, e = np.frexp(a)
    return np.ldexp((np.trunc if cut else np.rint)(m * 2.0 ** bits), e - bits)


def operands(R, N, K, bits):
    rng = np.random.default_rng(K + R)
    return keep(rng.standard_normal((R, K)), bits), keep(0.05 * rng.standard_normal((N, K)), bits)


@pytest.mark.parametrize("K", [512, 2048, 8192])
def test_fma_bound(K):
    x, w = operands(24, 32, K, 24)
    exact = x @ w.T
    chain = np.zeros((24, 32), np.float32)
    for k in range(K):                                     # (the product's own rounding too: more than a fused one's)
        chain += x[:, k, None].astype(np.float32) * w[None, :, k].astype(np.float32)
    rms, top = off(chain, exact, x, w)
    assert fma_bound(K) / 8 < rms <= 1.25 * fma_bound(K) and top <= 8 * fma_bound(K)
    rms, _ = off(keep(x, 11) @ keep(w, 11).T, exact, x, w)
    assert rms > 8 * fma_bound(K), "operands of 11 bits pass"
    rms, _ = off(sum(keep(x[:, k::4] @ w[:, k::4].T, 11) for k in range(4)), exact, x, w)
    assert rms > 2 * fma_bound(K), "partial sums of 11 bits pass"


@pytest.mark.parametrize("products", [16, 32])
@pytest.mark.parametrize("K", [512, 2048, 8192])
def test_tensor_bound(K, products):
    x, w = operands(24, 32, K, 8 if products == 16 else 4)
    exact = x @ w.T
    acc = np.zeros((24, 32))
    for k in range(0, K, products):
        acc = keep(acc + x[:, k:k + products] @ w[:, k:k + products].T, 24, cut=True)
    rms, top = off(acc, exact, x, w)
    assert rms <= tensor_bound(K, products) and top <= 8 * tensor_bound(K, products)
    for bits in (8, 11):                                   # bf16, fp16
        rms, _ = off(sum(keep(x[:, k::4] @ w[:, k::4].T, bits) for k in range(4)), exact, x, w)
        assert rms > 1.5 * tensor_bound(K, products), f"partial sums of {bits} bits pass"
        rms, _ = off(keep(exact, bits), exact, x, w)
        assert rms > tensor_bound(K, products), f"a sum of {bits} bits passes"
