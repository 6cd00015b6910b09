"""Layer norm from its definition, in 64 bits on the CPU."""
import torch


def forward(x, gamma, beta, eps):
    mean = x.mean(1)
    v = x - mean[:, None]
    rstd = (v.square().mean(1) + eps) ** -0.5
    return v * rstd[:, None] * gamma + beta, mean, rstd


def gradients(dy, x, gamma, mean, rstd):
    """dx without a residual path's part, dgamma, dbeta."""
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def case(g, M, C, T):
    """Rows with a mean and spread per channel, parameters, gradients."""
    rn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = (rn(M, C) * (0.5 + rn(C).abs()) + 0.5 * rn(C)).to(T)
    return x, 1 + 0.2 * rn(C), 0.2 * rn(C), rn(M, C).to(T), rn(M, C).to(T)
