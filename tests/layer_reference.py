"""The layers' operators by their definitions in 64 bits, on the CPU, with the magnitudes that bounds of their errors are made of."""
import math

import torch

K = math.sqrt(2 / math.pi)
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def parts(name, z):
    """(act(z), the two terms of act'(z), size of the argument that an exponential is taken of)."""
    one, zero = torch.ones_like(z), torch.zeros_like(z)
    if name == "relu":
        return torch.where(z <= 0, zero, z), (z > 0).double(), zero, zero
    if name == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * phi, phi, z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), z * z
    if name == "gelu_tanh":
        u = K * (z + 0.044715 * z ** 3)
        p, rest = torch.sigmoid(2 * u), torch.sigmoid(-2 * u)
        return z * p, p, 2 * z * p * rest * K * (1 + 0.134145 * z * z), 2 * u.abs()
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p, z * p * torch.sigmoid(-z), z.abs()
    return z, one, zero, zero


def orthogonal(g, steps, coefficients=None):
    """(X, bound of the error's Frobenius norm) for one matrix; coefficients: one triple a step.

    The map of a step is an odd function of the singular values, so an error's Frobenius norm grows by at most the largest of its slope and of its value
    over its argument, on 0 .. |X|.  What a step adds: X, A and b A + c A A are held within 2^-22 of their magnitudes, and a sum of n products
    is off by 8 sqrt(n) U of the sum of their magnitudes (n roundings of either sign); |X| |X|' has at most the norm |X|_F^2."""
    x = g.double()
    norm = x.norm()
    x = x / norm if norm > 0 else x
    if x.shape[0] > x.shape[1]:
        x = x.T
    r, n = x.shape
    u, held = 2.0 ** -24, 2.0 ** -22
    e = held * float(x.norm())
    for i in range(steps):
        a, b, c = coefficients[i] if coefficients else COEFFICIENTS
        gram = x @ x.T
        s2, f = float(torch.linalg.matrix_norm(x, 2)), float(x.norm())
        grid = torch.linspace(0, s2, 2001, dtype=torch.float64)
        slope = float((a + 3 * b * grid ** 2 + 5 * c * grid ** 4).abs().max())
        ratio = float((a + b * grid ** 2 + c * grid ** 4).abs().max())
        poly = b * gram + c * gram @ gram + a * torch.eye(r, dtype=torch.float64)
        e_gram = (held + 8 * n ** 0.5 * u) * f * f
        e_poly = (abs(b) + 2 * abs(c) * s2 ** 2) * e_gram + abs(c) * 8 * r ** 0.5 * u * float(gram.norm()) ** 2 + 4 * u * float(poly.norm())
        e_poly += held * float(poly.norm())
        out = poly @ x
        e = max(slope, ratio) * e + e_poly * s2 + held * ratio * f + 8 * r ** 0.5 * u * float(poly.norm()) * f + held * float(out.norm())
        x = out
    return (x.T if g.shape[0] > g.shape[1] else x), e
