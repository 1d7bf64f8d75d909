"""The 64-bit form of the update with orthogonalised steps: against the singular value decomposition, and its bound."""
import numpy as np
import pytest

from oracle import muon


@pytest.mark.parametrize("shape", [(1, 1), (5, 9), (9, 5), (16, 16)])
@pytest.mark.parametrize("iterations", [1, 5])
def test_singular_vectors_stay(shape, iterations):
    u = np.random.default_rng(0).standard_normal(shape)
    x, off = muon.orthogonalise(u, 0.0, iterations)
    U, s, V = np.linalg.svd(u, full_matrices=False)
    s = s / np.linalg.norm(u)
    a, b, c = muon.COEFFICIENTS
    for _ in range(iterations):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(x, U * s @ V, atol=1e-10)
    assert 0 < off < 0.02 * np.linalg.norm(x)


@pytest.mark.parametrize("shape,decay", [((24, 24), 0.0), ((24, 60), 0.0), ((40, 40), 1.0), ((60, 24), 1.5), ((100, 300), 0.5), ((200, 200), 2.0)])
def test_distance_of_rounded_operands(shape, decay):
    """X, A and B rounded to fp16 times 2^10 between products: as far off as is expected."""
    u = np.random.default_rng(1).standard_normal(shape)
    if decay:
        U, s, V = np.linalg.svd(u, full_matrices=False)
        u = U * (1.0 / (1 + np.arange(len(s))) ** decay) @ V
    held = lambda m: (m * 1024).astype(np.float16).astype(np.float64) / 1024  # noqa: E731
    x = u.T if shape[0] > shape[1] else u
    x = held(x / np.linalg.norm(u))
    a, b, c = muon.COEFFICIENTS
    for _ in range(5):
        A = held(x @ x.T)
        B = held(a * np.eye(len(A)) + b * A + c * A @ A)
        x = held(B @ x)
    want, off = muon.orthogonalise(u, 0.0, 5)
    got = np.linalg.norm((x.T if shape[0] > shape[1] else x) - want)
    assert off / 3 <= got <= 2 * off


def test_step():
    rng = np.random.default_rng(2)
    w, g, m = (rng.standard_normal((6, 4)) for _ in range(3))
    new, buf, off = muon.step(w, g, m, 0.1, 0.9, 0.01, 0.2, 1e-7, 1, 5)
    x, _ = muon.orthogonalise(g + 0.9 * (0.9 * m + g), 1e-7, 5)
    assert np.allclose(buf, 0.9 * m + g) and np.allclose(new, w - 0.1 * (0.2 * np.sqrt(6) * x + 0.01 * w)) and off > 0
