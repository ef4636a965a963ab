"""The orthogonalised update in 64 bits on the very u that the kernels form, with a bound that what S = u^T u and the steps are held in shows in."""
import math

import torch

U = torch.finfo(torch.float32).eps / 2          # a rounding to fp32: 2^-24
COEFFICIENTS = (3.4445, -4.775, 2.0315)


def graded(L, r, seed, device, weak=1e-3, middle=0.05):
    """[L, r] fp32 with one strong direction (1) and three weak ones mixed into four columns, the others between; columns in any order.  The square of a weak direction is 1e-6 of S: rounded to
    fp32 it is off by percents, and the steps, which lift that direction four hundredfold, bring it to the size of the others."""
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(L, r, generator=gen, dtype=torch.float64)
    if L >= r:
        q, _ = torch.linalg.qr(q)
    s = torch.full((r,), middle, dtype=torch.float64)
    s[0], s[1:4] = 1.0, weak
    v = torch.eye(r, dtype=torch.float64)
    v[:4, :4] = torch.tensor([[1, 1, 1, 1], [1, -1, 1, -1], [1, 1, -1, -1], [1, -1, -1, 1]]) / 2
    return (((q * s) @ v)[:, torch.randperm(r, generator=gen)] * 1e-3).float().to(device)


def iterate(S, steps=5, eps=1e-7, coefficients=COEFFICIENTS):
    """Q of X = u Q, from S, in S's own precision."""
    a, b, c = coefficients
    eye = torch.eye(S.shape[0], dtype=S.dtype, device=S.device)
    norm = S.diagonal().sum().sqrt() + eps
    G, Q = S / norm ** 2, eye
    for _ in range(steps):
        P = a * eye + b * G + c * G @ G
        Q, G = Q @ P, G @ P @ P
    return Q / norm


def momentum_of(m, g, mu=0.95, nesterov=True):
    """m' and u with the roundings of two fp32 multiply-adds.  (Each is formed in 64 bits and rounded: the same but for one value in 2^28.)"""
    mu = torch.tensor(mu, dtype=torch.float32).item()
    new = (mu * m.double() + g.double()).float()
    return new, (g.double() + mu * new.double()).float() if nesterov else new


def update(u, tall, steps=5):
    """X for u [L, r] (tall) or [r, L], one step after the other in 64 bits, and how far r multiply-adds in fp32 of u and a Q rounded to fp32 may be off (sums in 64 bits: a
    hundredth more)."""
    a, b, c = COEFFICIENTS
    x = u.double() if tall else u.double().t()
    r = x.shape[1]
    x = x / (torch.linalg.norm(x) + 1e-7)
    for _ in range(steps):
        G = x.t() @ x
        x = a * x + x @ (b * G + c * G @ G)
    v = u.double() if tall else u.double().t()
    off = 1.01 * (r + 2) * U * (v.abs() @ iterate(v.t() @ v, steps).abs())
    return (x, off) if tall else (x.t(), off.t())
