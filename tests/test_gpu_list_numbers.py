"""GPU: numbers of the AdamW and Lion steps where fp32 is at its end: decay rates near one, sums of the smallest values.

u = 2^-24 is the relative error of one fp32 rounding."""
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402
from test_gpu_list_ops import gen, opt, scalar  # noqa: E402, F401


@pytest.mark.parametrize("n", [100003, 1500000])
@pytest.mark.parametrize("beta", [0.9, 0.95, 0.999, 0.9999, 0.99999, 1 - 2.0 ** -20])
def test_moments_decay_by_the_given_beta(opt, beta, n):  # noqa: F811
    # Without a gradient a moment is multiplied by beta.  A beta rounded to fp32 is u / 2 off, which is as much as the rounding
    # of the product and the same in every step.  With beta's remainder carried along, the error beyond the product's half step
    # is the remainder's rounding and that of its product, u each of at most 2 u of the moment: 4 u^2, and a half step is u / 2
    # of the result or more.
    M = torch.randn(n, generator=gen(1), device="cuda")
    V = torch.rand(n, generator=gen(2), device="cuda") + 0.01
    G, X = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")

    def decayed(before, after):
        want = before.double() * beta
        size = after.abs()
        half = (torch.nextafter(size, torch.full_like(size, 1e9)).double() - size.double()) / 2
        return bool(((after.double() - want).abs() <= half * (1 + 2.0 ** -19)).all())

    for adamw in (True, False):
        m, v = M.clone(), V.clone()
        if adamw:
            opt.adamw_step(binding.param_list([binding.param_desc(X, G, m, v)]), 0.0, 5, beta, beta)
            assert decayed(V, v)
        else:
            opt.lion_step(binding.param_list([binding.param_desc(X, G, m)]), 0.0, 0.9, beta)
        assert decayed(M, m)


@pytest.mark.parametrize("beta", [0.0, 0.5, 0.9, 0.9999])
def test_infinite_moments_stay_what_they_are(opt, beta):  # noqa: F811
    # a square beyond fp32's range makes V infinite, and from then on the step is zero, not NaN
    inf = float("inf")
    X, G = torch.tensor([1.0, 2.0, 3.0, 4.0], device="cuda"), torch.tensor([2e25, 0.5, 0.5, 0.0], device="cuda")
    M, V = torch.tensor([0.0, 0.0, 0.1, 0.1], device="cuda"), torch.tensor([0.0, inf, inf, inf], device="cuda")
    before = X.clone()
    for t in range(1, 5):
        opt.adamw_step(binding.param_list([binding.param_desc(X, G, M, V)]), 0.01, t, 0.9, max(beta, 0.5))
        assert bool((V == inf).all()) and torch.equal(X, before) and bool(torch.isfinite(M).all())
    for sign in (inf, -inf):
        X, M = torch.zeros(3, device="cuda"), torch.full((3,), sign, device="cuda")
        G = torch.tensor([1.0, 0.0, -1.0], device="cuda")
        opt.lion_step(binding.param_list([binding.param_desc(X, G, M)]), 0.5, 0.9, max(beta, 0.5))
        assert bool((M == sign).all()) and bool((X == (-0.5 if sign > 0 else 0.5)).all())
    # beta = 0 keeps nothing of the moments
    X, G, M, V = (torch.full((5,), x, device="cuda") for x in (1.0, 0.25, 7.0, 9.0))
    opt.adamw_step(binding.param_list([binding.param_desc(X, G, M, V)]), 0.0, 1, 0.0, 0.0)
    assert bool((M == 0.25).all()) and bool((V == 0.0625).all())


@pytest.mark.parametrize("b1,s", [(0.95, 1.0), (0.95, 0.678), (0.9, 0.4438), (0.7, 0.2169), (0.4, 1.2073), (0.3, 1.367), (0.2, 0.413)])
@pytest.mark.parametrize("n", [1, 3000])
def test_lion_sign_of_the_smallest_values(opt, b1, s, n):  # noqa: F811
    # moments and gradients of a few times 2^-149, where every product loses what is below that: the sign is still that of
    # the exact sum (of a sum that float64 tells from zero)
    f = Fraction(float(np.float32(s)))
    near = [(m, round(-Fraction(b1) * m / ((1 - Fraction(b1)) * f)) + d) for m in range(-40, 41) for d in range(-2, 3)]
    total = [Fraction(b1) * m + (1 - Fraction(b1)) * f * g for m, g in near]
    kept = [k for k, c in enumerate(total) if abs(c) > Fraction(1, 2 ** 40)]
    unit = 2.0 ** -149
    m = torch.tensor(np.array([near[k][0] * unit for k in kept], np.float32)).repeat(n).cuda()
    g = torch.tensor(np.array([near[k][1] * unit for k in kept], np.float32)).repeat(n).cuda()
    want = torch.tensor([1.0 if total[k] > 0 else -1.0 for k in kept]).repeat(n).cuda()
    X = torch.zeros_like(m)
    opt.lion_step(binding.param_list([binding.param_desc(X, g, m)]), 1.0, b1, 0.98, grad_scale=None if s == 1.0 else scalar(s))
    assert torch.equal(X, -want)
