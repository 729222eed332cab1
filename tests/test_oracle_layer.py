"""Pins of the layer steps' 64-bit model: brute force, closed forms and loops."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as lo


def all_e4m3():
    v = [m / 8.0 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8.0) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array([x for x in v if x <= 448.0])


def test_e4m3_is_the_nearest_of_the_grid():
    grid = all_e4m3()
    assert grid.size == 127 and grid[-1] == 448.0
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(0, 448, 500), np.exp2(rng.uniform(-12, 9, 500)), grid, (grid[1:] + grid[:-1]) / 2])
    x = x[x <= 464.0]
    got = lo.e4m3(x)
    for xi, gi in zip(x, got):
        d = np.abs(grid - xi)
        near = np.flatnonzero(d == d.min())
        assert gi in grid[near]
        if len(near) == 2:                       # a tie: the even code
            assert gi == grid[[n for n in near if n % 2 == 0][0]]
    assert np.array_equal(lo.e4m3(-x), -got)
    assert lo.e4m3(np.inf) == 448.0 and lo.e4m3(-1e9) == -448.0 and np.isnan(lo.e4m3(np.nan))


def test_scale_is_the_smallest_that_holds_the_block():
    rng = np.random.default_rng(1)
    y = rng.standard_normal((6, 96)) * np.exp2(rng.integers(-20, 60, (6, 3)).repeat(32, 1).astype(float))
    y[0, :32] = 0.0
    y[1, :32] = 448.0
    y[2, :32] = np.nextafter(448.0, 1000.0)
    y[3, 4], y[3, 5] = np.inf, np.nan
    e = lo.scale_exponents(y)
    assert e[0, 0] == -32 and e[1, 0] == 0 and e[2, 0] == 1
    m = np.where(np.isfinite(y), np.abs(y), 0).reshape(6, 3, 32).max(2)
    assert np.all(m <= 448.0 * np.exp2(e))
    assert np.all((m > 448.0 * np.exp2(e - 1)) | (e == -32))


@pytest.mark.parametrize("rows,n", [(1, 32), (130, 160), (257, 256)])
def test_tiles_are_a_permutation(rows, n):
    at = lo.tile_index(rows, n).reshape(-1)
    assert len(set(at)) == at.size and at.min() == 0 and at.max() < -(-rows // 128) * -(-n // 128) * 512
    if rows > 32:
        assert lo.tile_index(rows, n)[32, 0] == 4 and lo.tile_index(rows, n)[1, 0] == 16


def test_norm_closed_forms():
    s, y = lo.add_norm(np.full((1, 8), 2.0), np.full((1, 8), 1.0), None, 16.0)
    assert np.allclose(s, 3.0) and np.allclose(y, 3.0 / 5.0)
    x = np.random.default_rng(2).standard_normal((3, 40))
    _, y = lo.add_norm(x, None, None, 0.0)
    assert np.allclose(np.mean(y * y, axis=1), 1.0)
    _, z = lo.add_norm(7 * x, None, np.full(40, 2.0), 0.0)
    assert np.allclose(z, 2 * y)


def test_linear_against_loops():
    rng = np.random.default_rng(3)
    x, w, u = rng.standard_normal((3, 5)), rng.standard_normal((4, 5)), rng.standard_normal((4, 5))
    b, c, r = rng.standard_normal(4), rng.standard_normal(4), rng.standard_normal((3, 4))
    got = lo.linear(x, w, b, "silu", u, c, r)
    gel = lo.linear(x, w, None, "gelu")
    for i in range(3):
        for j in range(4):
            z = sum(x[i, k] * w[j, k] for k in range(5))
            v = sum(x[i, k] * u[j, k] for k in range(5)) + c[j]
            assert math.isclose(got[i, j], (z + b[j]) / (1 + math.exp(-z - b[j])) * v + r[i, j], rel_tol=1e-12)
            assert math.isclose(gel[i, j], z * 0.5 * (1 + math.erf(z / math.sqrt(2))), rel_tol=1e-12)


def test_rope_axes():
    rng = np.random.default_rng(4)
    B, M, Hq, Hkv, d = 2, 3, 2, 1, 8
    x = rng.standard_normal((B, M, (Hq + 2 * Hkv) * d))
    pos = rng.integers(0, 50, (B, M, 3))
    q, k, v = lo.rope(x, pos, (1, 2, 1), 100.0, Hq, Hkv, d)
    heads = x.reshape(B, M, 4, d)
    assert np.array_equal(v[:, 0], heads[:, :, 3])
    for i, a in enumerate((0, 1, 1, 2)):                 # as a product of complex numbers
        turn = np.exp(1j * pos[..., a] * 100.0 ** (-2 * i / d))
        z = (heads[:, :, 1, i] + 1j * heads[:, :, 1, i + 4]) * turn
        assert np.allclose(q[:, :, 1, i], z.real) and np.allclose(q[:, :, 1, i + 4], z.imag)
    # the same position on every axis is the ordinary rotation; scores depend on the distance alone
    one = lo.rope(x, np.repeat(pos[..., :1], 3, 2), (1, 2, 1), 100.0, Hq, Hkv, d)
    two = lo.rope(x, pos[..., :1], (4,), 100.0, Hq, Hkv, d)
    assert all(np.allclose(a, b) for a, b in zip(one, two))
    far = lo.rope(x, pos + 11, (1, 2, 1), 100.0, Hq, Hkv, d)
    s1 = np.einsum("bid,bjd->bij", q[:, :, 0], k[:, 0])
    s2 = np.einsum("bid,bjd->bij", far[0][:, :, 0], far[1][:, 0])
    assert np.allclose(s1, s2)
