"""GPU: arrays of one list that lie inside one another's span without sharing an element: rows and columns of one matrix, numbers
between two rows."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402
from test_gpu_list_ops import COEF, NORM, check_clipped, check_step, f32, gen, norm64, opt  # noqa: E402, F401

CUTS = {"rows of three": lambda t: [t[0:3:2], t[1:2], t[3:]], "a row beside columns": lambda t: [t[:, :100], t[4:5, 100:], t[:4, 100:], t[5:, 100:]],
        "two distances": lambda t: [t[:, :133], t[0::2, 133:], t[1::2, 133:]], "three rows apart": lambda t: [t[0::3], t[1::3], t[2::3]]}


@pytest.mark.parametrize("shape", [(7, 200), (97, 300), (64, 4096)])
@pytest.mark.parametrize("cut", list(CUTS))
def test_parts_of_one_matrix(opt, cut, shape):  # noqa: F811
    parts = CUTS[cut]
    r = lambda k: torch.randn(shape, generator=gen(k), device="cuda")  # noqa: E731
    for dtype in (torch.float32, torch.bfloat16):
        t = r(1).to(dtype)
        before = t.clone()
        opt.clip_grads(binding.grad_list(parts(t)), 0.5 * norm64([before]))
        check_clipped([t], [t], [before], 0.5)
    new = dict(X=r(2), G=r(3), M=r(4), V=r(5).abs(), X16=torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))
    for adamw in (True, False):
        old = {k: t.clone() for k, t in new.items()}
        V = parts(new["V"]) if adamw else [None] * len(parts(new["V"]))
        params = binding.param_list([binding.param_desc(*p) for p in zip(parts(new["X"]), parts(new["G"]), parts(new["M"]), V, parts(new["X16"]))])
        if adamw:
            opt.adamw_step(params, 0.01, 1)
        else:
            opt.lion_step(params, 0.01, 0.9, 0.95)
        check_step(old, new, adamw, f32(0.01), 0.9, 0.95, 1e-8, 1, 1.0, 1.0, 0.0)
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("rows", [5, 300])
def test_outputs_between_the_rows(opt, rows):  # noqa: F811
    wide = torch.randn((rows, 1040), generator=gen(1), device="cuda")
    G, norm, coef = wide[:, :1000], wide[0, 1003:1004], wide[1, 1039:1040]
    before = wide.clone()
    want = norm64([G])
    opt.grad_norm(binding.grad_list([G]), norm_out=norm, max_norm=0.25 * want, coef_out=coef)
    assert abs(float(norm) - want) <= NORM * want and abs(float(coef) - 0.25) <= (COEF + 2.0 ** -24) * 0.25
    opt.clip_grads(binding.grad_list([G]), 0.25 * want, norm_out=norm, coef_out=coef)
    check_clipped([G], [G], [before[:, :1000]], 0.25)
    before[0, 1003], before[1, 1039] = norm[0], coef[0]
    assert torch.equal(wide[:, 1000:], before[:, 1000:])
