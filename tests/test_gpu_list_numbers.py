"""GPU: numbers of the AdamW and Lion steps where fp32 is at its end: sums of the smallest values."""
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402
from test_gpu_list_ops import opt, scalar  # noqa: E402, F401


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
