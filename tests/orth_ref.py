"""Orthogonal updates from their definition, on the CPU, in the inputs' own precision."""
import torch

MUON = [(3.4445, -4.7750, 2.0315)] * 5
CUBIC = [(1.5, -0.5, 0.0)] * 12                # converges to singular values of 1
QUINTIC = [(15 / 8, -10 / 8, 3 / 8)] * 9


def steps(g, coefs, eps):
    """The definition: the steps one by one."""
    coefs = [tuple(float(torch.tensor(v, dtype=torch.float32)) for v in s) for s in coefs]   # as the descriptor holds them
    x = g / (g.double().square().sum().sqrt().to(g.dtype) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for a, b, c in coefs:
        A = x @ x.t()
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.t() if tall else x


def by_singular_values(g, coefs, eps):
    """The same on the singular values alone."""
    u, s, vt = torch.linalg.svd(g.double(), full_matrices=False)
    s = s / (s.square().sum().sqrt() + eps)
    for a, b, c in coefs:
        s = s * (a + b * s ** 2 + c * s ** 4)
    return (u * s) @ vt


def gradient(gen, rows, cols):
    """A few strong directions under noise."""
    k = min(8, rows, cols)
    rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return 1e-3 * ((rn(rows, k) * torch.tensor([10.0, 5, 3, 2, 1, 1, 0.5, 0.5])[:k]) @ rn(k, cols) + rn(rows, cols))
