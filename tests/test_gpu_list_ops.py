"""GPU: the global norm, clipping, AdamW and Lion steps over lists of arrays against their formulas in float64.

u = 2^-24 is the relative error of one fp32 rounding, U = 2^-8 that of a rounding to bf16 (half of each type's eps)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402

u, U, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -149
# A norm: groups of up to 16 squares are summed in fp32 (one rounding per term: 16 u of the sum, half of that in its root), the
# groups in 64 bits; then one rounding.
NORM = 9 * u
# A coefficient: the norm's error and the division's.
COEF = NORM + u
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def opt():
    with binding.Dion() as o:
        yield o


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# How a tensor lies in memory: (elements before it, distance of its rows beyond its columns)
PLAIN, SHIFTED, SLICED, ALIGNED_SLICES = (0, 0), (3, 0), (5, 3), (0, 16)
SHAPES = [(1, 1), (1, 7), (1, 8), (3, 5), (1, 31), (1, 255), (2, 512), (1, 1023), (1, 1024), (1, 1025), (17, 61), (1, 4097), (64, 128),
          (257, 63), (40, 8), (333, 1), (1, 100003), (130, 2048)]


def place(shape, dtype, lie, value=None, seed=0, fill=7.0):
    """A tensor of this shape inside a larger buffer that holds `fill` around it; returns (tensor, buffer)."""
    rows, cols = shape
    shift, pad = lie
    buf = torch.full((shift + rows * (cols + pad) + 9,), fill, dtype=dtype, device="cuda")
    t = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.randn(t.shape, generator=gen(seed), device="cuda") if value is None else torch.as_tensor(value))
    return t, buf


def surroundings_kept(t, buf, fill=7.0):
    """Whatever of the buffer is not the tensor still holds `fill`."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(t.shape, t.stride(), t.storage_offset() - buf.storage_offset()).fill_(False)
    return bool((buf[mask] == fill).all())


def scalar(x=0.0):
    return torch.full((1,), float(x), device="cuda")


def norm64(tensors, kind=2):
    each = [float(t.double().abs().max()) if kind == "inf" else float(torch.linalg.vector_norm(t.double())) for t in tensors if t.numel()]
    return max(each, default=0.0) if kind == "inf" else math.sqrt(math.fsum(e * e for e in each))


# ---- the norm ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", [2, "inf"])
@pytest.mark.parametrize("lie", [PLAIN, SHIFTED, SLICED, ALIGNED_SLICES])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_one(opt, dtype, lie, kind):
    for k, shape in enumerate(SHAPES):
        t, _ = place(shape, DT[dtype], lie, seed=k, fill=1e9)
        out = scalar(-1)
        opt.grad_norm(binding.grad_list([t]), kind, norm_out=out)
        want = norm64([t], kind)
        assert abs(float(out) - want) <= (NORM * want if kind == 2 else 0.0), shape


@pytest.mark.parametrize("kind", [2, "inf"])
def test_norm_of_a_mixed_list(opt, kind):
    lies = [PLAIN, SHIFTED, SLICED, ALIGNED_SLICES]
    ts = [place(s, DT["bf16" if k % 3 == 0 else "f32"], lies[k % 4], seed=k, fill=1e9)[0] for k, s in enumerate(SHAPES)]
    empty = torch.zeros(0, device="cuda")
    ts = [empty, empty] + ts[:5] + [empty] + ts[5:] + [empty]
    total, each, coef = scalar(-1), torch.full((len(ts) + 1,), -1.0, device="cuda"), scalar(-1)
    items = binding.grad_list(ts)
    opt.grad_norm(items, kind, norm_out=total, each_out=each, max_norm=0.5, coef_out=coef)
    want = norm64(ts, kind)
    tol = NORM if kind == 2 else 0.0
    assert abs(float(total) - want) <= tol * want
    assert abs(float(coef) - 0.5 / want) <= (COEF if kind == 2 else u) * 0.5 / want
    for t, got in zip(ts, each.tolist()):
        assert abs(got - norm64([t], kind)) <= tol * norm64([t], kind)
    assert float(each[-1]) == -1.0
    # without the norms of each the total may take other sums, but the same on every call
    first, again = scalar(), scalar()
    opt.grad_norm(items, kind, norm_out=first)
    opt.grad_norm(items, kind, norm_out=again)
    assert abs(float(first) - want) <= tol * want and torch.equal(first, again)
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("count", [0, 1, 24, 25, 80, 81, 96, 97, 180, 181, 500, 501, 1234])
def test_norm_of_long_lists(opt, count):
    flat = torch.randn(count * 37 + 1, generator=gen(count), device="cuda")
    ts = [flat[37 * k:37 * k + 1 + k % 37] for k in range(count)]
    total, each = scalar(-1), torch.full((count,), -1.0, device="cuda")
    opt.grad_norm(binding.grad_list(ts), norm_out=total, each_out=each if count else None)
    want = norm64(ts)
    assert abs(float(total) - want) <= NORM * want
    assert all(abs(g - norm64([t])) <= NORM * norm64([t]) for t, g in zip(ts, each.tolist()))
    opt.grad_norm(binding.grad_list(ts), "inf", norm_out=total)
    assert float(total) == norm64(ts, "inf")


def test_norm_of_nothing(opt):
    empty, out, each, coef = torch.zeros(0, device="cuda"), scalar(-1), torch.full((40,), -1.0, device="cuda"), scalar(-1)
    for kind in (2, "inf"):
        opt.grad_norm(binding.grad_list([empty] * 40), kind, norm_out=out, each_out=each, max_norm=1.0, coef_out=coef)
        assert float(out) == 0.0 and float(coef) == 1.0 and not bool(each.any())
        opt.clip_grads(binding.grad_list([empty] * 140), 1.0, norm_type=kind, norm_out=out, coef_out=coef)
        assert float(out) == 0.0 and float(coef) == 1.0
        opt.clip_grads(binding.grad_list([empty] * 140), 1.0, norms=torch.full((3,), 2.0, device="cuda"), norm_type=kind, coef_out=coef)
        assert abs(float(coef) - (0.5 if kind == "inf" else 0.5 / math.sqrt(3))) <= COEF
    none = binding.param_list([binding.param_desc(empty, empty, empty, empty)] * 30)
    opt.adamw_step(none, 0.1, 1)
    opt.lion_step(none, 0.1)
    assert opt.get_status() == (0, 0)


def test_norm_counts_an_array_twice(opt):
    t, out = torch.randn(1000, generator=gen(0), device="cuda"), scalar()
    opt.grad_norm(binding.grad_list([t, t]), norm_out=out)
    assert abs(float(out) - math.sqrt(2) * norm64([t])) <= NORM * float(out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-20, 1e18, 1e19, 1e30, 1e36])
def test_norm_of_extreme_values(opt, dtype, size):
    # squares beyond fp32's range on either side, alone, beside zeros and beside ordinary values
    t = (torch.randn(5000, generator=gen(1), device="cuda") * size).to(DT[dtype])
    z = torch.zeros(5000, dtype=DT[dtype], device="cuda")
    z[::7] = t[::7]
    for ts in ([t], [z], [t, torch.ones(77, device="cuda")]):
        out, each = scalar(), torch.zeros(len(ts), device="cuda")
        opt.grad_norm(binding.grad_list(ts), norm_out=out, each_out=each)
        # (a norm below 2^-126 has fewer bits)
        assert abs(float(out) - norm64(ts)) <= NORM * norm64(ts) + TINY
        assert abs(float(each[0]) - norm64(ts[:1])) <= NORM * norm64(ts[:1]) + TINY
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("kind", [2, "inf"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 4097, 99999])
def test_norm_that_is_not_finite(opt, kind, bad, at):
    t = torch.randn(100000, generator=gen(2), device="cuda")
    t[at] = bad
    for ts in ([t], [t.bfloat16()], [torch.ones(3, device="cuda"), t]):
        out, coef, each = scalar(), scalar(), torch.zeros(len(ts), device="cuda")
        opt.grad_norm(binding.grad_list(ts), kind, norm_out=out, each_out=each, max_norm=1.0, coef_out=coef)
        want = float("nan") if bad != bad else float("inf")
        assert str(float(out)) == str(want) == str(float(each[-1])) and math.isnan(float(coef))
        assert opt.get_status() == (binding.STATUS_NONFINITE, 0)
    assert opt.get_status() == (0, 0)


def test_norm_beyond_32_bit_offsets(opt):
    n = 2 ** 32 + 1234567
    t = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    out = scalar()
    opt.grad_norm(binding.grad_list([t]), norm_out=out)
    assert abs(float(out) - math.sqrt(n)) <= NORM * math.sqrt(n)
    t[-1] = 2.0 ** 20
    opt.grad_norm(binding.grad_list([t]), "inf", norm_out=out)
    assert float(out) == 2.0 ** 20
    rows = t[:2 ** 32].view(2 ** 20, 4096)[:, :8]      # the last row of the slice lies beyond 2^32 elements less one row
    opt.grad_norm(binding.grad_list([rows]), norm_out=out)
    assert abs(float(out) - math.sqrt(rows.numel())) <= NORM * math.sqrt(rows.numel())
    # in place, the far end included
    coef = scalar()
    opt.clip_grads(binding.grad_list([t[:-1]]), 0.5 * math.sqrt(n - 1), coef_out=coef)
    assert abs(float(coef) - 0.5) <= COEF * 0.5 * 2
    assert bool((t[:-1][-1000:] == 0.5).all()) and bool((t[:1000] == 0.5).all()) and float(t[-1]) == 2.0 ** 20
    assert float(t[2 ** 31 - 3:2 ** 31 + 3].sum()) == 3.0 and float(t[2 ** 32 - 3:2 ** 32 + 3].sum()) == 3.0


# ---- clipping ----------------------------------------------------------------------------------------------------

def check_clipped(ts, outs, before, coef):
    for t, o, b in zip(ts, outs, before):
        want = b.double() * coef
        half = u if o.dtype == torch.float32 else U
        # the product's rounding, the coefficient's error, the rounding to the result's type
        tol = (COEF + u + half) * want.abs() + (TINY if o.dtype == torch.float32 else 2.0 ** -134)
        assert bool(((o.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("lie", [PLAIN, SHIFTED, SLICED, ALIGNED_SLICES])
@pytest.mark.parametrize("types", ["f32 f32", "f32 bf16", "bf16 f32", "bf16 bf16", "f32 in place", "bf16 in place"])
def test_clip(opt, types, lie):
    src, dst = types.split(" ", 1)
    ts = [place(s, DT[src], lie, seed=k) for k, s in enumerate(SHAPES)]
    grads = [t for t, _ in ts]
    before = [g.clone() for g in grads]
    outs = ts if dst == "in place" else [place(s, DT[dst], PLAIN if k % 2 else lie, value=3.0, seed=k) for k, s in enumerate(SHAPES)]
    want = norm64(grads)
    norm, coef = scalar(), scalar()
    items = binding.grad_list(grads, None if dst == "in place" else [o for o, _ in outs])
    opt.clip_grads(items, 0.37, norm_out=norm, coef_out=coef)
    assert abs(float(norm) - want) <= NORM * want and abs(float(coef) - 0.37 / want) <= COEF * 0.37 / want
    check_clipped(grads, [o for o, _ in outs], before, 0.37 / want)
    for o, buf in outs + ts:
        assert surroundings_kept(o, buf)
    if dst != "in place":
        assert all(torch.equal(g, b) for g, b in zip(grads, before))
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("kind", [2, "inf"])
@pytest.mark.parametrize("lie", [PLAIN, SHIFTED, SLICED, ALIGNED_SLICES])
@pytest.mark.parametrize("types", ["f32 bf16", "bf16 f32", "f32 in place", "bf16 in place"])
def test_clip_short_lists(opt, types, lie, kind):
    # lists that one launch clips, up to its last tile and just beyond
    src, dst = types.split(" ", 1)
    for shapes in ([(1, 1)], SHAPES[:16], [(1, 262144)], [(64, 2048), (64, 2048)], [(1, 262145)], [(3, 40)] * 60, [(2, 40)] * 90, [(0, 5), (1, 3)]):
        ts = [place(s, DT[src], lie, seed=k) for k, s in enumerate(shapes)]
        grads = [t for t, _ in ts]
        before = [g.clone() for g in grads]
        outs = ts if dst == "in place" else [place(s, DT[dst], lie, value=3.0, seed=k) for k, s in enumerate(shapes)]
        want = norm64(grads, kind)
        norm, coef, alone = scalar(), scalar(), scalar()
        items = binding.grad_list(grads, None if dst == "in place" else [o for o, _ in outs])
        opt.grad_norm(items, kind, norm_out=alone)
        opt.clip_grads(items, 0.25 * want, norm_type=kind, norm_out=norm, coef_out=coef)
        tol = NORM if kind == 2 else 0.0
        assert abs(float(norm) - want) <= tol * want and abs(float(alone) - want) <= tol * want
        assert abs(float(coef) - 0.25) <= (COEF + u) * 0.25
        check_clipped(grads, [o for o, _ in outs], before, 0.25)
        for o, buf in outs + ts:
            assert surroundings_kept(o, buf)
    assert opt.get_status() == (0, 0)


def test_neighbours_in_memory(opt):
    # views of flat buffers, one behind the other, with what must not be walked as one: a gap, another type, another
    # rate, another decay, a slice, an empty array
    sizes = [5, 8, 4096, 1, 333, 64, 0, 77, 2048, 9, 1000]
    total = sum(sizes)
    flat = {k: torch.randn(total + 1, generator=gen(i), device="cuda") for i, k in enumerate(("X", "G", "M"))}
    flat["V"] = torch.rand(total + 1, generator=gen(9), device="cuda")
    flat["X16"] = torch.zeros(total + 1, dtype=torch.bfloat16, device="cuda")
    at, views = 0, []
    for n in sizes:
        views.append({k: f[at:at + n] for k, f in flat.items()})
        at += n
    views[3]["G"] = views[3]["G"].bfloat16()
    scales = [1.0] * 4 + [0.5] * 7
    decays = [0.0] * 8 + [0.25] * 3
    for adamw in (True, False):
        before = [{k: t.clone() for k, t in v.items()} for v in views]
        tail = {k: f[-1].clone() for k, f in flat.items()}
        params = binding.param_list([binding.param_desc(v["X"], v["G"], v["M"], v["V"] if adamw else None, v["X16"], s, d)
                                     for v, s, d in zip(views, scales, decays)])
        if adamw:
            opt.adamw_step(params, 0.01, 2)
        else:
            opt.lion_step(params, 0.01, 0.9, 0.95)
        for b, v, s, d in zip(before, views, scales, decays):
            check_step(b, v, adamw, f32(0.01), 0.9, 0.95, 1e-8, 2, 1.0, s, d)
        assert all(torch.equal(f[-1], tail[k]) for k, f in flat.items())
    # the norm and the scaling of the same views, some left out
    for left_out in ([], [2], [0, 5]):
        gs = [v["G"] for k, v in enumerate(views) if k not in left_out]
        G = flat["G"].clone()
        outs = [torch.zeros_like(g) for g in gs]
        norm, coef = scalar(), scalar()
        opt.clip_grads(binding.grad_list(gs, outs), 1.0, norm_out=norm, coef_out=coef)
        want = norm64(gs)
        assert abs(float(norm) - want) <= NORM * want
        check_clipped(gs, outs, gs, 1.0 / want)
        opt.clip_grads(binding.grad_list(gs), 1e9, norm_out=norm)
        assert abs(float(norm) - want) <= NORM * want and torch.equal(G, flat["G"])
    opt.clip_grads(binding.grad_list([v["G"] for k, v in enumerate(views) if k not in (2, 3)]), 0.0)
    assert not any(bool(v["G"].any()) for k, v in enumerate(views) if k not in (2, 3))
    assert torch.equal(flat["G"][13:13 + 4097], G[13:13 + 4097]) and torch.equal(flat["G"][-1], G[-1])


def test_clip_below_the_threshold(opt):
    ts = [torch.randn(s, generator=gen(3), device="cuda") for s in ((100, 33), (4097,))]
    before = [t.clone() for t in ts]
    coef = scalar()
    for top in (norm64(ts) * 1.001, float("inf")):
        opt.clip_grads(binding.grad_list(ts), top, coef_out=coef)
        assert float(coef) == 1.0 and all(torch.equal(t, b) for t, b in zip(ts, before))
        outs = [torch.zeros_like(t, dtype=torch.bfloat16) for t in ts]
        opt.clip_grads(binding.grad_list(ts, outs), top)
        assert all(torch.equal(o, b.bfloat16()) for o, b in zip(outs, before))
    opt.clip_grads(binding.grad_list(ts), 0.0, coef_out=coef)
    assert float(coef) == 0.0 and not any(bool(t.any()) for t in ts)
    opt.clip_grads(binding.grad_list(ts), 0.0, coef_out=coef)      # zeros have norm zero, which is not above zero
    assert float(coef) == 1.0 and not any(bool(t.any()) for t in ts)


@pytest.mark.parametrize("kind", [2, "inf"])
def test_clip_by_given_norms(opt, kind):
    # two lists and the norms of other ranks, clipped by the norm of the whole
    a, b = [torch.randn(4097, generator=gen(4), device="cuda")], [torch.randn((65, 40), generator=gen(5), device="cuda").bfloat16()]
    others = torch.tensor([3.0, 0.0, 41.0], device="cuda")
    norms = torch.cat([torch.zeros(2, device="cuda"), others])
    opt.grad_norm(binding.grad_list(a), kind, norm_out=norms[0:1])
    opt.grad_norm(binding.grad_list(b), kind, norm_out=norms[1:2])
    parts = [norm64(a, kind), norm64(b, kind)] + others.tolist()
    want = max(parts) if kind == "inf" else math.sqrt(math.fsum(p * p for p in parts))
    before = [a[0].clone(), b[0].clone()]
    norm, coef = scalar(), scalar()
    opt.clip_grads(binding.grad_list(a), 1.5, norms=norms, norm_type=kind, norm_out=norm, coef_out=coef)
    assert abs(float(norm) - want) <= NORM * want and abs(float(coef) - 1.5 / want) <= COEF * 1.5 / want
    opt.clip_grads(binding.grad_list(b), 1.5, norms=norms, norm_type=kind)
    check_clipped(a + b, a + b, before, 1.5 / want)
    # no arrays at all: the coefficient alone
    norm2, coef2 = scalar(), scalar()
    opt.clip_grads(binding.grad_list([]), 1.5, norms=norms, norm_type=kind, norm_out=norm2, coef_out=coef2)
    assert torch.equal(norm, norm2) and torch.equal(coef, coef2)
    opt.clip_grads(binding.grad_list([]), 1.5, norm_out=norm2, coef_out=coef2)
    assert float(norm2) == 0.0 and float(coef2) == 1.0
    many = torch.full((1000,), 2.0, device="cuda")
    opt.clip_grads(binding.grad_list([]), 1.0, norms=many, norm_out=norm2)
    assert abs(float(norm2) - 2.0 * math.sqrt(1000)) <= NORM * float(norm2)


@pytest.mark.parametrize("count", [25, 81, 181, 401, 1000])
def test_clip_long_lists(opt, count):
    flat = torch.randn(count * 41, generator=gen(count), device="cuda")
    before = flat.clone()
    ts = [flat[41 * k:41 * k + 41 - k % 3] for k in range(count)]
    want = norm64(ts)
    norm = scalar()
    opt.clip_grads(binding.grad_list(ts), 1.0, norm_out=norm)
    assert abs(float(norm) - want) <= NORM * want
    check_clipped(ts, ts, [before[41 * k:41 * k + 41 - k % 3] for k in range(count)], 1.0 / want)
    gaps = torch.ones(count * 41, dtype=torch.bool, device="cuda")
    for k in range(count):
        gaps[41 * k:41 * k + 41 - k % 3] = False
    assert torch.equal(flat[gaps], before[gaps])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_clip_spoils_gradients_of_no_norm(opt, bad):
    ts = [torch.randn(5000, generator=gen(6), device="cuda"), torch.randn((30, 30), generator=gen(7), device="cuda").bfloat16()]
    ts[1][3, 3] = bad
    coef = scalar()
    opt.clip_grads(binding.grad_list(ts), 1.0, coef_out=coef)
    assert math.isnan(float(coef)) and all(bool(torch.isnan(t).all()) for t in ts)
    assert opt.get_status() == (binding.STATUS_NONFINITE, 0)
    # every step that reads them is cancelled
    X, M, Q = (torch.randn(s, generator=gen(8), device="cuda") for s in ((30, 30), (30, 30), (30, 4)))
    kept = [t.clone() for t in (X, M, Q)]
    opt.step(X, M, ts[1], Q, 0.01)
    status, skipped = opt.get_status()
    assert status & binding.STATUS_NONFINITE and skipped == 1
    assert all(torch.equal(a, b) for a, b in zip((X, M, Q), kept))


# ---- AdamW and Lion ----------------------------------------------------------------------------------------------

def make_params(shapes, g, m, lies, copy, seed, adamw=True):
    """Parameters whose moments are those of a run; [(tensors by name, buffers by name)]"""
    made = []
    for k, shape in enumerate(shapes):
        r = lambda: torch.randn(shape, generator=gen(seed + 10 * k), device="cuda")  # noqa: B023, E731
        value = {"X": r() * 0.5, "G": torch.randn(shape, generator=gen(seed + 10 * k + 1), device="cuda") * 0.1,
                 "M": torch.randn(shape, generator=gen(seed + 10 * k + 2), device="cuda") * 0.03}
        if adamw:
            value["V"] = torch.rand(shape, generator=gen(seed + 10 * k + 3), device="cuda") * 0.01
        if copy:
            value["X16"] = torch.zeros(shape, device="cuda")
        types = {"X": torch.float32, "G": DT[g], "M": DT[m], "V": torch.float32, "X16": torch.bfloat16}
        ts, bufs = {}, {}
        for j, (name, v) in enumerate(value.items()):
            ts[name], bufs[name] = place(shape, types[name], lies[j % len(lies)], value=v, seed=0)
        made.append((ts, bufs))
    return made


def describe(made, lr_scale=1.0, wd=0.0):
    return binding.param_list([binding.param_desc(ts["X"], ts["G"], ts["M"], ts.get("V"), ts.get("X16"), lr_scale, wd) for ts, _ in made])


def f32(x):
    return float(np.float32(x))


def check_step(before, after, adamw, lr, b1, b2, eps, t, s, lr_scale, wd):
    """One step in float64 from `before`, and how far fp32 may be from it."""
    g, x, m = before["G"].double() * s, before["X"].double(), before["M"].double()
    size_m = None
    if adamw:
        new_m = b1 * m + (1 - b1) * g
        new_v = b2 * before["V"].double() + (1 - b2) * g * g
        den = torch.sqrt(new_v / (1 - b2 ** t)) + eps
        step = new_m / (1 - b1 ** t) / den
        size_m = b1 * m.abs() + (1 - b1) * g.abs()
        # M: beta, 1 - beta, s g, the product and the sum, one rounding each.  V: those of the square too, all its terms
        # positive; squares below 2^-126 lose what is below 2^-149.  The step: M's error and, relative to the step, V's
        # 6 u halved by the root (3), V's correction and its product halved (1), the root 2^-23 (2), eps and the sum (2), M's
        # correction and its product (2), the quotient 2^-22 (4): 14 u.
        tol_m, tol_v = 5 * u * size_m + TINY, 8 * u * new_v + 4 * TINY
        # (sqrt(V + tiny) - sqrt(V) <= sqrt(tiny): counts where V itself is that small)
        tol_step = 5 * u * size_m / (1 - b1 ** t) / den + 14 * u * step.abs() + step.abs() * torch.sqrt(torch.full_like(den, 4 * TINY)) / den
        assert bool(((after["V"].double() - new_v).abs() <= tol_v).all())
    else:
        c = b1 * m + (1 - b1) * g
        step, tol_step = torch.sign(c), torch.zeros_like(c)
        new_m = b2 * m + (1 - b2) * g
        size_m = b2 * m.abs() + (1 - b2) * g.abs()
        tol_m = 5 * u * size_m + TINY
    new_x = x * (1 - lr * lr_scale * wd) - lr * lr_scale * step
    # X: the factor 1 - lr wd and its product, lr and its scale (three roundings), the sum
    rate = lr * lr_scale
    tol_x = 2 * u * x.abs() + rate * (tol_step + 4 * u * step.abs()) + u * new_x.abs() + TINY
    assert bool(((after["X"].double() - new_x).abs() <= tol_x).all()), float(((after["X"].double() - new_x).abs() / tol_x).max())
    if after["M"].dtype == torch.bfloat16:
        tol_m = tol_m + U * (new_m.abs() + tol_m)
    assert bool(((after["M"].double() - new_m).abs() <= tol_m).all())
    if "X16" in after:
        assert torch.equal(after["X16"], after["X"].bfloat16())
    assert torch.equal(after["G"], before["G"])


@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "lion"])
@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("lies", [[PLAIN], [SHIFTED], [SLICED], [ALIGNED_SLICES], [PLAIN, SHIFTED], [PLAIN, ALIGNED_SLICES, SLICED],
                                  [PLAIN, SHIFTED, PLAIN, PLAIN, PLAIN], [SLICED, PLAIN, SLICED, SLICED, SLICED], [SHIFTED, ALIGNED_SLICES, SHIFTED, SHIFTED, SHIFTED]])
@pytest.mark.parametrize("g,m", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_step(opt, adamw, g, m, lies, copy):
    made = make_params(SHAPES, g, m, lies, copy, 100, adamw)
    before = [{k: t.clone() for k, t in ts.items()} for ts, _ in made]
    lr, b1, b2, eps, t, lr_scale, wd = 0.02, 0.9, 0.95, 1e-8, 3, 0.75, 0.1
    scale = scalar(0.625) if copy else None
    params = describe(made, lr_scale, wd)
    if adamw:
        opt.adamw_step(params, lr, t, b1, b2, eps, grad_scale=scale)
    else:
        opt.lion_step(params, lr, b1, b2, grad_scale=scale)
    for b, (ts, bufs) in zip(before, made):
        check_step(b, ts, adamw, f32(lr), b1, b2, eps, t, 0.625 if copy else 1.0, lr_scale, f32(wd))
        for name in ts:
            assert surroundings_kept(ts[name], bufs[name]), name
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "lion"])
@pytest.mark.parametrize("count", [0, 24, 25, 81, 181, 250, 251, 700])
def test_step_on_long_lists(opt, adamw, count):
    made = make_params([(1, 1 + k % 50) for k in range(count)], "bf16", "f32", [PLAIN], True, 7, adamw)
    before = [{k: t.clone() for k, t in ts.items()} for ts, _ in made]
    empty = torch.zeros(0, device="cuda")
    none = binding.param_desc(empty, empty, empty, empty)
    params = binding.param_list([none] + [binding.param_desc(ts["X"], ts["G"], ts["M"], ts.get("V"), ts["X16"]) for ts, _ in made] + [none])
    if adamw:
        opt.adamw_step(params, 0.01, 1)
    else:
        opt.lion_step(params, 0.01, 0.9, 0.95)
    for b, (ts, _) in zip(before, made):
        check_step(b, ts, adamw, f32(0.01), 0.9, 0.95, 1e-8, 1, 1.0, 1.0, 0.0)


@pytest.mark.parametrize("size", [0.0, 1e-30, 1e-12, 1e12])
@pytest.mark.parametrize("t", [1, 2, 100000])
def test_adamw_of_extreme_gradients(opt, size, t):
    # a first step from empty moments, gradients of zero, squares that vanish: no NaN, the formula's values
    n = 3000
    X, G = torch.randn(n, generator=gen(1), device="cuda"), torch.randn(n, generator=gen(2), device="cuda") * size
    M, V = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    before = dict(X=X.clone(), G=G.clone(), M=M.clone(), V=V.clone())
    opt.adamw_step(binding.param_list([binding.param_desc(X, G, M, V)]), 0.01, t, 0.9, 0.95, 1e-8)
    assert bool(torch.isfinite(X).all())
    check_step(before, dict(X=X, G=G, M=M, V=V), True, f32(0.01), 0.9, 0.95, 1e-8, t, 1.0, 1.0, 0.0)


def test_adamw_of_zeros_without_eps(opt):
    # 0 / 0 is NaN in the formula as it is in fp32; one parameter with a gradient keeps its value
    X, G = torch.ones(2, device="cuda"), torch.tensor([0.0, 1.0], device="cuda")
    M, V = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    opt.adamw_step(binding.param_list([binding.param_desc(X, G, M, V)]), 0.5, 1, 0.9, 0.95, 0.0)
    assert math.isnan(float(X[0])) and abs(float(X[1]) - 0.5) <= 20 * u


def test_lion_sign_where_the_sum_cancels(opt):
    # gradients that are the moment's negative to within a rounding: the sign is that of the exact sum
    n, b1, b2 = 200000, 0.95, 0.98
    M = torch.randn(n, generator=gen(1), device="cuda")
    G = (-M.double() * b1 / (1 - b1)).float()
    G[::5] = torch.nextafter(G[::5], torch.full_like(G[::5], 1e9))
    M[:100], G[:100] = 0.0, 0.0
    M[100:200] = 0.0
    G[100:200] *= 1e-38
    for s in (1.0, 0.7):
        X = torch.zeros(n, device="cuda")
        scale = scalar(s)
        g = (G / scale).clone() if s != 1.0 else G.clone()
        before = dict(X=X.clone(), G=g.clone(), M=M.clone())
        m = M.clone()
        opt.lion_step(binding.param_list([binding.param_desc(X, g, m)]), 1.0, b1, b2, grad_scale=scale)
        want = torch.sign(b1 * M.double() + (1 - b1) * (g.double() * scale.double()))
        assert torch.equal(X.double(), -want)
        assert bool((X[:100] == 0).all())
        check_step(before, dict(X=X, G=g, M=m), False, 1.0, b1, b2, 0.0, 1, float(scale.double()), 1.0, 0.0)


@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "lion"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_step_is_cancelled_by_its_scale(opt, adamw, bad):
    made = make_params(SHAPES[:9] * 30, "f32", "f32", [PLAIN], True, 3, adamw)      # (two launches, one step)
    before = [{k: t.clone() for k, t in ts.items()} for ts, _ in made]
    if adamw:
        opt.adamw_step(describe(made), 0.01, 1, grad_scale=scalar(bad))
    else:
        opt.lion_step(describe(made), 0.01, grad_scale=scalar(bad))
    assert all(torch.equal(b[k], ts[k]) for b, (ts, _) in zip(before, made) for k in b)
    assert opt.get_status() == (binding.STATUS_NONFINITE, 1)


@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "lion"])
def test_nan_stays_in_its_element(opt, adamw):
    made = make_params([(1, 4097)], "f32", "f32", [PLAIN], False, 4, adamw)
    ts = made[0][0]
    ts["G"].view(-1)[1234] = float("nan")
    if adamw:
        opt.adamw_step(describe(made), 0.01, 1)
    else:
        opt.lion_step(describe(made), 0.01)
    for name in ("X", "M") + (("V",) if adamw else ()):
        assert torch.isnan(ts[name].view(-1)).nonzero().view(-1).tolist() == [1234], name


def test_step_number_on_the_device(opt):
    for t in (1, 2, 5000):
        a, b = make_params(SHAPES[:8], "f32", "f32", [PLAIN], False, 5), make_params(SHAPES[:8], "f32", "f32", [PLAIN], False, 5)
        opt.adamw_step(describe(a), 0.01, t)
        opt.adamw_step(describe(b), 0.01, torch.tensor([t], device="cuda"))
        for (x, _), (y, _) in zip(a, b):      # (the two pow's may round differently: one step of the corrections)
            assert torch.equal(x["M"], y["M"]) and torch.equal(x["V"], y["V"])
            assert bool(((x["X"] - y["X"]).abs() <= 0.01 * 10 * 4 * u + 2 * u * x["X"].abs()).all())
    c = make_params(SHAPES[:8], "f32", "f32", [PLAIN], False, 5)
    kept = [{k: t.clone() for k, t in ts.items()} for ts, _ in c]
    opt.get_status()
    opt.adamw_step(describe(c), 0.01, torch.tensor([0], device="cuda"))
    assert all(torch.equal(k[n], ts[n]) for k, (ts, _) in zip(kept, c) for n in k)
    assert opt.get_status() == (0, 1)


def test_step_beyond_32_bit_offsets(opt):
    n = 2 ** 31 + 12345
    X = torch.zeros(n, device="cuda")
    G, M = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    opt.lion_step(binding.param_list([binding.param_desc(X, G, M)]), 0.25, 0.5, 0.5)
    assert bool((X == -0.25).all()) and bool((M == 0.25).all())


# ---- streams, graphs, devices ------------------------------------------------------------------------------------

def test_on_another_stream(opt):
    side = torch.cuda.Stream()
    t = torch.randn(1 << 22, generator=gen(9), device="cuda")
    want = norm64([t])
    torch.cuda.synchronize()
    out, coef, norm = scalar(), scalar(), scalar()
    with torch.cuda.stream(side):
        t.mul_(2.0)
        items = binding.grad_list([t])
        opt.grad_norm(items, norm_out=out)                  # the current stream
        opt.clip_grads(items, 1.0, norm_out=norm, coef_out=coef)
    opt.grad_norm(items, norm_out=coef, stream=side)        # a given one
    side.synchronize()
    assert abs(float(out) - 2 * want) <= NORM * 2 * want and torch.equal(out, norm)
    assert abs(float(coef) - 1.0) <= COEF + 2 * u


def test_captured_and_replayed(opt):
    # clipping and both steps in a graph; what changes from step to step lies on the device
    n = 5000
    grads = [torch.randn(n, generator=gen(k), device="cuda") for k in range(4)]
    X, G, M, V = (torch.zeros(n, device="cuda") for _ in range(4))
    Y, N = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    t, coef, norm = torch.zeros(1, dtype=torch.int64, device="cuda"), scalar(), scalar()
    items = binding.grad_list([G])
    params, others = binding.param_list([binding.param_desc(X, G, M, V)]), binding.param_list([binding.param_desc(Y, G, N)])

    def one():
        t.add_(1)
        opt.clip_grads(items, 1.0, norm_out=norm)
        opt.grad_norm(items, max_norm=0.5, coef_out=coef)
        opt.adamw_step(params, 0.01, t, grad_scale=coef)
        opt.lion_step(others, 0.01, grad_scale=coef)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    assert not bool(X.any()) and int(t) == 0
    seen = []
    for g in grads:
        G.copy_(g)
        graph.replay()
        seen.append((X.clone(), M.clone(), V.clone(), Y.clone(), N.clone(), norm.clone()))
    for s in (X, M, V, Y, N, t):
        s.zero_()
    for g, want in zip(grads, seen):
        G.copy_(g)
        one()
        assert all(torch.equal(a, b) for a, b in zip((X, M, V, Y, N, norm), want))
        assert abs(float(norm) - norm64([g])) <= NORM * norm64([g])
    assert opt.get_status() == (0, 0)


def test_binding_checks(opt):
    t, half = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.float16)
    items = binding.grad_list([t])
    with pytest.raises(ValueError):
        binding.grad_list([half])
    with pytest.raises(ValueError):
        binding.grad_list([t], [half])
    with pytest.raises(ValueError):
        binding.param_desc(t, t, t, half)
    with pytest.raises(ValueError):
        binding.param_desc(t, t, t, t, X16=t)
    with pytest.raises(ValueError):
        opt.grad_norm(items, norm_out=torch.zeros(1))
    with pytest.raises(ValueError):
        opt.grad_norm(items, norm_out=torch.zeros(1, device="cuda", dtype=torch.float64))
    with pytest.raises(ValueError):
        opt.grad_norm(items, each_out=torch.zeros(0, device="cuda"))
    with pytest.raises(TypeError):
        opt.grad_norm([t], norm_out=t)
    with pytest.raises(TypeError):
        opt.adamw_step(items, 0.1, 1)
    with pytest.raises(ValueError):
        opt.adamw_step(binding.param_list([]), 0.1, torch.ones(1, device="cuda"))
    with pytest.raises(binding.DionError):
        opt.grad_norm(items)                                   # nothing to write
    with pytest.raises(binding.DionError):
        opt.clip_grads(binding.grad_list([t, t]), 1.0)          # the same array twice
    with pytest.raises(binding.DionError):
        opt.clip_grads(items, -1.0)
    with pytest.raises(binding.DionError):                     # AdamW without V
        opt.adamw_step(binding.param_list([binding.param_desc(t, t.clone(), t.clone())]), 0.1, 1)
    with pytest.raises(binding.DionError):
        opt.adamw_step(binding.param_list([]), 0.1, 0)
    assert opt.get_status() == (0, 0)


# ---- calls at the edges of what the documentation allows ---------------------------------------------------------

def test_slices_of_one_matrix_in_one_call(opt):
    # columns, and every other row, of one matrix as entries of one list: each element is scaled once
    for cut in (lambda t: [t[:, :100], t[:, 100:133], t[:, 133:]], lambda t: [t[0::2], t[1::2]], lambda t: [t[:50], t[50:51], t[51:]]):
        t = torch.randn((97, 300), generator=gen(1), device="cuda")
        before, parts = t.clone(), None
        parts = cut(t)
        opt.clip_grads(binding.grad_list(parts), 0.5 * norm64([before]))
        check_clipped([t], [t], [before], 0.5)
        X, M, V = torch.randn((97, 300), generator=gen(2), device="cuda"), torch.zeros(97, 300, device="cuda"), torch.zeros(97, 300, device="cuda")
        old = dict(X=X.clone(), G=t.clone(), M=M.clone(), V=V.clone())
        opt.adamw_step(binding.param_list([binding.param_desc(*p) for p in zip(cut(X), cut(t), cut(M), cut(V))]), 0.01, 1)
        check_step(old, dict(X=X, G=t, M=M, V=V), True, f32(0.01), 0.9, 0.95, 1e-8, 1, 1.0, 1.0, 0.0)


def test_one_gradient_into_two_results(opt):
    for n in (1000, 700000):
        g = torch.randn(n, generator=gen(1), device="cuda")
        before = g.clone()
        outs = [torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
        opt.clip_grads(binding.grad_list([g, g], outs), 0.1)
        check_clipped([g, g], outs, [before, before], 0.1 / (math.sqrt(2) * norm64([before])))
        assert torch.equal(g, before)


def test_shapes_of_any_rank(opt):
    ts = [torch.randn(s, generator=gen(k), device="cuda") for k, s in enumerate([(), (3,), (2, 3, 5), (1, 1, 1, 7), (4, 0, 2), (64, 3, 3, 3)])]
    out, each = scalar(), torch.full((len(ts),), -1.0, device="cuda")
    opt.grad_norm(binding.grad_list(ts), norm_out=out, each_out=each)
    assert abs(float(out) - norm64(ts)) <= NORM * norm64(ts)
    assert all(abs(e - norm64([t])) <= NORM * norm64([t]) for e, t in zip(each.tolist(), ts))
    M = [torch.zeros_like(t) for t in ts]
    X = [torch.zeros_like(t) for t in ts]
    opt.lion_step(binding.param_list([binding.param_desc(x, g, m) for x, g, m in zip(X, ts, M)]), 0.5)
    assert all(torch.equal(x, -0.5 * torch.sign(t)) for x, t in zip(X, ts))


def test_two_contexts_at_once(opt):
    # one context per stream; long lists, so that the launches overlap
    streams, ts, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    with binding.Dion() as other:
        for k in range(2):
            ts.append(torch.randn(30000000 + 12345 * k, generator=gen(k), device="cuda"))
            outs.append((scalar(), scalar(), torch.zeros(1, device="cuda")))
        want = [norm64([t]) for t in ts]
        torch.cuda.synchronize()
        for rep in range(20):
            for o, st, t, (norm, inf, each) in zip((opt, other), streams, ts, outs):
                items = binding.grad_list([t])
                o.grad_norm(items, norm_out=norm, each_out=each, stream=st)
                o.clip_grads(items, 1e9, norm_type="inf", norm_out=inf, stream=st)
        torch.cuda.synchronize()
        for t, w, (norm, inf, each) in zip(ts, want, outs):
            assert abs(float(norm) - w) <= NORM * w and torch.equal(norm, each) and float(inf) == norm64([t], "inf")
        assert opt.get_status() == other.get_status() == (0, 0)


def test_graphs_that_share_a_context(opt):
    # two graphs of one context, replayed in turn: neither leaves anything that the other trips over
    ts = [torch.randn(n, generator=gen(n), device="cuda") for n in (5000000, 4000000)]
    outs = [scalar() for _ in ts]
    graphs = []
    for t, out in zip(ts, outs):
        items, each = binding.grad_list([t[:1000], t[1001:]]), torch.zeros(2, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            opt.grad_norm(items, norm_out=out, each_out=each)
        graphs.append((g, norm64([t[:1000], t[1001:]]), out, each, items))
    # ... and replayed side by side on two streams, with direct calls beside them
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    direct = scalar()
    for _ in range(200):
        for st, (g, want, out, each, items) in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        opt.grad_norm(binding.grad_list([ts[0]]), norm_out=direct)
    torch.cuda.synchronize()
    for g, want, out, each, items in graphs:
        assert abs(float(out) - want) <= NORM * want and abs(float(each.double().square().sum().sqrt()) - want) <= 2 * NORM * want
    assert abs(float(direct) - norm64([ts[0]])) <= NORM * float(direct)
    eager = scalar()
    for _ in range(5):
        for g, want, out, each, items in graphs:
            g.replay()
            opt.grad_norm(items, norm_out=eager, each_out=each)
            assert abs(float(out) - want) <= NORM * want and torch.equal(out, eager)


# ---- together, as a training step uses them ----------------------------------------------------------------------

def test_training_steps_of_a_small_model(opt):
    # matrices by Dion, embedding and gains by AdamW, biases by Lion, all clipped by one norm: every state
    # against float64, step by step from the states that the device holds
    from oracle import dion_oracle as orc
    r = lambda *shape: torch.randn(*shape, generator=gen(sum(shape)), device="cuda")  # noqa: E731
    E, gain, bias = r(50, 48) * 0.5, torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
    W1, W2 = r(64, 48) * 0.2, r(96, 64) * 0.2
    leaves = {"E": E, "gain": gain, "bias": bias, "W1": W1, "W2": W2}
    params = {k: t.clone().requires_grad_() for k, t in leaves.items()}
    M = {k: torch.zeros_like(t) for k, t in leaves.items()}
    V = {k: torch.zeros_like(leaves[k]) for k in ("E", "gain")}
    E16 = torch.zeros_like(E, dtype=torch.bfloat16)
    Q = {k: torch.linalg.qr(r(leaves[k].shape[1], 8))[0].contiguous() for k in ("W1", "W2")}
    tokens = torch.arange(32, device="cuda") % 50
    target = r(32, 96)
    lr, mu = 0.01, 0.95
    for t in range(1, 4):
        h = torch.relu(params["E"][tokens] @ params["W1"].t()) * params["gain"] + params["bias"]
        loss = ((h @ params["W2"].t() - target) ** 2).mean() * 10.0
        grads = dict(zip(params, torch.autograd.grad(loss, list(params.values()))))
        before = {k: p.detach().clone() for k, p in params.items()}
        kept = {"M": {k: v.clone() for k, v in M.items()}, "V": {k: v.clone() for k, v in V.items()}, "G": {k: g.clone() for k, g in grads.items()},
                "Q": {k: v.clone() for k, v in Q.items()}}
        X = {k: p.data for k, p in params.items()}
        matrices, others = binding.grad_list([grads["W1"], grads["W2"]]), binding.grad_list([grads[k] for k in ("E", "gain", "bias")])
        norms, norm, coef = torch.zeros(2, device="cuda"), scalar(), scalar()
        opt.grad_norm(matrices, norm_out=norms[:1])
        opt.grad_norm(others, norm_out=norms[1:])
        max_norm = 0.5 * norm64(list(kept["G"].values()))
        opt.clip_grads(matrices, max_norm, norms=norms, norm_out=norm, coef_out=coef)
        opt.step_grouped([(X[k], M[k], grads[k], Q[k]) for k in ("W1", "W2")], lr)
        opt.adamw_step(binding.param_list([binding.param_desc(X["E"], grads["E"], M["E"], V["E"], E16, weight_decay=0.1),
                                           binding.param_desc(X["gain"], grads["gain"], M["gain"], V["gain"])]), lr, t, grad_scale=coef)
        opt.lion_step(binding.param_list([binding.param_desc(X["bias"], grads["bias"], M["bias"])]), lr, 0.9, 0.95, grad_scale=coef)
        assert opt.get_status() == (0, 0)
        s = 0.5
        assert abs(float(norm) - 2 * max_norm) <= (NORM + 2 * u) * 2 * max_norm and abs(float(coef) - s) <= (COEF + 4 * u) * s
        check_clipped([grads[k] for k in ("W1", "W2")], [grads[k] for k in ("W1", "W2")], [kept["G"][k] for k in ("W1", "W2")], s)
        for k in ("W1", "W2"):
            d = lambda x: x.double().cpu().numpy()  # noqa: E731
            want = orc.step(d(before[k]), d(kept["M"][k]), d(kept["G"][k]) * s, d(kept["Q"][k]), mu, lr, 1e-8)
            for name, got in (("X", X[k]), ("M", M[k]), ("Q", Q[k])):      # (the library's stated bound)
                assert np.linalg.norm(d(got) - getattr(want, name)) <= 1e-4 * np.linalg.norm(getattr(want, name)), (t, k, name)
        c = float(coef.double())
        for k, decay in (("E", f32(0.1)), ("gain", 0.0)):
            after = {"X": X[k], "G": grads[k], "M": M[k], "V": V[k]}
            if k == "E":
                after["X16"] = E16
            check_step({"X": before[k], "G": kept["G"][k], "M": kept["M"][k], "V": kept["V"][k]}, after, True, f32(lr), 0.9, 0.95, 1e-8, t, c, 1.0, decay)
        check_step({"X": before["bias"], "G": kept["G"]["bias"], "M": kept["M"]["bias"]}, {"X": X["bias"], "G": grads["bias"], "M": M["bias"]},
                   False, f32(lr), 0.9, 0.95, 0.0, t, c, 1.0, 0.0)


def test_sharded_clipper_on_one_rank(opt):
    from paper_2504_05295_b200 import sharded
    shards, whole = torch.randn((300, 77), generator=gen(1), device="cuda"), torch.randn(4096, generator=gen(2), device="cuda")
    both = [shards.clone(), whole.clone()]
    want = norm64(both)
    clipper = sharded.ShardedClipper(opt, binding.grad_list([shards]), binding.grad_list([whole]), "cuda")
    clipper.clip(1.0, scale_whole=False)
    assert abs(float(clipper.norm) - want) <= (NORM + NORM) * want
    check_clipped([shards], [shards], both[:1], float(clipper.coef.double()))
    assert torch.equal(whole, both[1])
    shards.copy_(both[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    clipper.clip(1.0, stream=side)
    side.synchronize()
    check_clipped([shards, whole], [shards, whole], both, float(clipper.coef.double()))
