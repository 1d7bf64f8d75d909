"""The update with orthogonalised steps in 64 bits, from its definition, and how far one with operands in fp16 may be from it."""
import numpy as np

COEFFICIENTS = tuple(float(np.float32(x)) for x in (3.4445, -4.7750, 2.0315))   # as the library holds them
F32 = 2.0 ** -24                       # half a step, relative
F16_NOISE = 2.0 ** -20 / 12            # mean square of an fp16 rounding, relative to the value's square, at most (steps of 2^-10, even)


def orthogonalise(u, eps, iterations):
    """X of the definition, and the root of the expected squared distance (2-norm of all elements) of one whose X, A and B
    are rounded to fp16 between products.

    Roundings are noise of F16_NOISE times a matrix' squared norm, taken to be spread evenly over its elements, and so over the
    elements of its form in any orthogonal basis.  In that of X's singular vectors, which no iteration turns, the derivative of
    p(X) = a X + b X X'X + c X X'X X'X is diagonal: it scales the symmetric part of element (i, j) by the divided difference
    (p(s_i) - p(s_j)) / (s_i - s_j), the antisymmetric one by (p(s_i) + p(s_j)) / (s_i + s_j), and elements outside the square
    by p(s_i) / s_i.  What an iteration adds is therefore carried to the end exactly, to first order."""
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    x = (u.T if tall else u) / (np.linalg.norm(u) + eps)
    m, n = x.shape
    xs = [x]
    for _ in range(iterations):
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
        xs.append(x)
    s = np.linalg.svd(xs[0], compute_uv=False)
    values = [s]
    for _ in range(iterations):
        s = a * s + b * s ** 3 + c * s ** 5
        values.append(s)
    # from the last X backwards: what the iterations that follow make of an element
    minus, plus, outside = np.ones((m, m)), np.ones((m, m)), np.ones(m)
    energy = F16_NOISE * (xs[-1] ** 2).sum()
    for k in reversed(range(iterations)):
        s, p, X = values[k], values[k + 1], xs[k]
        A = X @ X.T
        B = a * np.eye(m) + b * A + c * A @ A                            # what is held of the factor
        i, j = s[:, None], s[None, :]
        for noise, part in ((F16_NOISE * (B ** 2).sum(), j + 0 * i), (F16_NOISE * (A ** 2).sum(), (b + c * (i * i + j * j)) * j)):
            sym, anti = (part + part.T) / 2, (part - part.T) / 2         # of symmetric noise times X
            energy += noise / m ** 2 * ((sym * minus) ** 2 + (anti * plus) ** 2).sum()
        slope = a + 3 * b * s ** 2 + 5 * c * s ** 4
        near = np.abs(i - j) < 1e-6 * (i + j) + 1e-300
        with np.errstate(divide="ignore", invalid="ignore"):
            minus = minus * np.where(near, (slope[:, None] + slope) / 2, (p[:, None] - p) / np.where(near, 1.0, i - j))
            plus = plus * np.where(i + j > 1e-300, (p[:, None] + p) / np.where(i + j > 1e-300, i + j, 1.0), a)
        outside = outside * (a + b * s ** 2 + c * s ** 4)
        energy += F16_NOISE * (X ** 2).sum() / (m * n) * (((minus ** 2 + plus ** 2) / 2).sum() + (n - m) * (outside ** 2).sum())
    return (xs[-1].T if tall else xs[-1]), float(np.sqrt(energy))


def step(w, g, m, lr, momentum, weight_decay, rms, eps, nesterov, iterations):
    """New weights, new momentum, and how far (2-norm) weights may be: three times what is expected of fp16's roundings, and fp32's."""
    m = momentum * m + g
    u = g + momentum * m if nesterov else m
    x, off = orthogonalise(u, eps, iterations)
    size = rms * np.sqrt(max(w.shape))
    new = w - lr * (size * x + weight_decay * w)
    return new, m, lr * size * (3 * off + 64 * F32 * np.linalg.norm(x)) + 4 * F32 * (np.linalg.norm(w) + np.linalg.norm(new))
