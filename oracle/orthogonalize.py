"""Newton-Schulz orthogonalisation and the Muon step in 64 bits.

  X = U / (|U| + eps);  steps times:  A = X X^T,  X = k0 X + (k1 A + k2 A A) X

through the singular values: the products change nothing else, so U = L diag(s) R^T becomes L diag(p(...p(s / |U|))) R^T
with p(s) = k0 s + k1 s^3 + k2 s^5.
"""
import numpy as np


def polynomial(s, coef):
    for k0, k1, k2 in coef:
        s = s * (k0 + k1 * s ** 2 + k2 * s ** 4)
    return s


def orthogonalize(u, coef, eps):
    """u [count, rows, cols]; coef: one triple per step."""
    u = np.asarray(u, np.float64)
    left, s, right = np.linalg.svd(u, full_matrices=False)
    norm = np.sqrt((u ** 2).sum((1, 2)))[:, None] + eps
    return np.einsum("nik,nk,nkj->nij", left, polynomial(s / norm, coef), right)


def products(u, coef, eps):
    """The same from the products themselves."""
    x = np.asarray(u, np.float64)
    x = x / (np.sqrt((x ** 2).sum((1, 2), keepdims=True)) + eps)
    for k0, k1, k2 in coef:
        a = x @ x.transpose(0, 2, 1)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    return x


def rounding_bound(u, coef, eps):
    """How far, in the Frobenius norm, fp32-grade arithmetic may be from `orthogonalize`, for every matrix of u.

    A product over K terms from operands of 22 bits: 2^-21 for the operands and what their product leaves out, and K / 8
    roundings of the running sum by 2^-24 each; term errors are independent, so |d(XY)| = e_K |X|_F |Y|_2.  A step's own
    error is enlarged by the steps behind it by at most the largest slope of their composed polynomial (an odd function
    of the singular values: its difference quotients, of sums too, are slopes somewhere between)."""
    u = np.asarray(u, np.float64)
    m, n = sorted(u.shape[1:])
    s = np.linalg.svd(u, compute_uv=False) / (np.sqrt((u ** 2).sum((1, 2)))[:, None] + eps)
    e = lambda K: 2.0 ** -21 + K / 8 * 2.0 ** -24
    fro, two = lambda v: np.sqrt((v ** 2).sum(1)), lambda v: np.abs(v).max(1)

    def slope(r, rest):
        grid = np.linspace(0, r, 20001)
        return np.abs(np.diff(polynomial(grid, rest)) / np.diff(grid)).max() if len(rest) else 1.0

    total = slope(1.0, coef) * 2.0 ** -21 * fro(s)                      # X itself: momentum, norm, halves
    top = 1.0
    for k, (k0, k1, k2) in enumerate(coef):
        a, b, new = s ** 2, k1 * s ** 2 + k2 * s ** 4, polynomial(s, coef[k:k + 1])
        da = e(n) * fro(s) * two(s) + 2.0 ** -21 * fro(a)
        daa = e(m) * fro(a) * two(a) + 2 * two(a) * da
        db = abs(k1) * da + abs(k2) * daa + 2.0 ** -21 * fro(b)
        dx = two(s) * db + e(m) * two(b) * fro(s) + 2.0 ** -21 * (abs(k0) * fro(s) + fro(new))
        top = np.abs(polynomial(np.linspace(0, top, 20001), coef[k:k + 1])).max()
        total = total + slope(top, coef[k + 1:]) * dx
        s = new
    return total


def muon(w, m, g, lr, mu, wd, scale, coef, eps, nesterov):
    """New weights and momenta of one layer; lr, mu, wd [P]."""
    w, m, g = (np.asarray(v, np.float64) for v in (w, m, g))
    lr, mu, wd = (np.asarray(v, np.float64)[:, None, None] for v in (lr, mu, wd))
    m = mu * m + g
    return (1 - lr * wd) * w - lr * scale * orthogonalize(g + mu * m if nesterov else m, coef, eps), m
