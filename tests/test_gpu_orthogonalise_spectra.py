"""Orthogonalised updates of matrices whose singular values differ by far more than float16's 11 bits, as a gradient's that all rows have in common do:
what is small comes up by its 3.4445-fold an iteration, and with it whatever was rounded off beside it.

An iteration X' = a X + (b A + c A A) X knows X to 22 bits in its first part, and to 11, an error of H = 2^-11 of X at most, in the second, where
|b t + c t^2| <= 2.81 for the t = s^2 of up to 1.3^2 that come up and next to nothing for small ones.  Roundings of A and of B, H of each, count with
|b + 2 c t| (0.7 where t is one) and |a + b t + c t^2| (0.7 there).  That is 4.2 H of X' an iteration where they all were alike; the slope that carries them
on is between -1.6 and 1.7 for s of 0.68 to 1.14 and of either sign, and half of them are below half of H: 4 H for each iteration are allowed.
Rests of 22 bits grow to 2^-23 3.4445^n, below that."""
import math

import pytest
import torch

from .test_gpu_expert_training import COEFFICIENTS, H

pytestmark = pytest.mark.gpu


def spectrum(m, n, values, g):
    u, v = (torch.linalg.qr(torch.randn(d, min(m, n), generator=g, dtype=torch.float64))[0] for d in (m, n))
    return ((u * values) @ v.t()).float()


def matrices(m, n):
    g, few = torch.Generator().manual_seed(m * 1000 + n), min(m, n)
    i = torch.arange(1, few + 1, dtype=torch.float64)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    yield "random", rand(m, n)
    yield "two directions over noise", 0.01 * rand(m, n) + rand(m, 2) @ rand(2, n)
    yield "one direction over noise", 0.003 * rand(m, n) + rand(m, 1) @ rand(1, n)
    for power in (1, 2, 3):
        yield f"1 / i^{power}", spectrum(m, n, i ** -power, g)
    yield "two and the others a thousandth", spectrum(m, n, torch.where(i <= 2, 1.0, 1e-3), g)
    yield "flat", spectrum(m, n, torch.ones_like(i), g)


def update(v, iterations):
    """O(v) in float, as a Muon step that does nothing else has it."""
    from paper_2603_19289_amd import training as T
    p = torch.zeros_like(v, device="cuda")
    T.Muon([p], lr=1.0, momentum=0.0, nesterov=False, weight_decay=0.0, update_rms=1.0, iterations=iterations).step([v.to("cuda")])
    return -p.double() / math.sqrt(max(v.shape))


@pytest.mark.parametrize("iterations", [1, 2, 5, 10])
@pytest.mark.parametrize("m,n", [(256, 256), (130, 300), (300, 129), (600, 1000)])
def test_what_is_small_is_not_rounding(m, n, iterations):
    a, b, c = COEFFICIENTS
    for name, v in matrices(m, n):
        x = v.cuda().double()
        x = x / x.norm()
        for _ in range(iterations):
            q = x @ x.t()
            x = a * x + (b * q + c * q @ q) @ x
        off = ((update(v, iterations) - x).norm() / x.norm()).item()
        print(m, n, iterations, name, f"{off:.2e}")
        assert off <= 4 * H * iterations, (name, off)
