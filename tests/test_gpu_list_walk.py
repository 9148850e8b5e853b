"""GPU: blocks that walk several tiles and go from array to array, groups of four rounds, the sizes at which the launches change
their form; every element against float64."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402
from test_gpu_list_ops import (ALIGNED_SLICES, DT, PLAIN, SHIFTED, SLICED, check_clipped, check_step, f32, gen, norm64, opt, place,  # noqa: E402, F401
                               scalar, surroundings_kept)

u = 2.0 ** -24
# A norm: each of a group's 8 squares is added with one fp32 rounding (8 u of the sum, 4 u of its root), the groups in 64 bits;
# one rounding of the result.
NORM = 5 * u
TILE = 2048      # elements of a tile (256 groups of 8); of an array that goes element by element 1024

# Arrays of uneven sizes, some empty, some narrow, some of long rows; about 3.3 million elements, and each lies differently
UNEVEN = [(1, 700001), (0, 5), (1, 3), (300, 2500), (2000, 7), (1, 1), (1, 400000), (64, 40), (3, 0), (17, 61), (500, 999), (1, 8), (1, 300007),
          (5000, 33), (2, 70001), (1, 2047), (1, 2049), (9, 4100), (40, 2048), (4, 9)]
LIES = [[PLAIN], [SHIFTED], [SLICED], [ALIGNED_SLICES], [PLAIN, SHIFTED, PLAIN, PLAIN, PLAIN], [PLAIN, SHIFTED], [SLICED, PLAIN, SLICED, SLICED, SLICED]]
# longer: two arrays beside them that are many tiles each
LONG = UNEVEN[:7] + [(1, 5000011)] + UNEVEN[7:] + [(1200, 4099)]


def more_tiles_than(blocks_per_sm, tiles_per_block, shapes):
    """Every block of one wave has so many tiles or more."""
    tiles = sum(r * c for r, c in shapes) // TILE
    return tiles >= tiles_per_block * blocks_per_sm * torch.cuda.get_device_properties(0).multi_processor_count


def build(shapes, g, m, copy, adamw, zero_weights=False):
    made = []
    for k, shape in enumerate(shapes):
        r = lambda j: torch.randn(shape, generator=gen(100 * k + j), device="cuda")  # noqa: B023, E731
        value = {"X": r(0) * 0.5 * (not zero_weights), "G": r(1) * 0.1, "M": r(2) * 0.03}
        if adamw:
            value["V"] = torch.rand(shape, generator=gen(100 * k + 3), device="cuda") * 0.01
        if copy:
            value["X16"] = torch.zeros(shape, device="cuda")
        types = {"X": torch.float32, "G": DT[g], "M": DT[m], "V": torch.float32, "X16": torch.bfloat16}
        lies = LIES[k % len(LIES)]
        made.append({name: place(shape, types[name], lies[j % len(lies)], value=v) for j, (name, v) in enumerate(value.items())})
    return made


@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "lion"])
@pytest.mark.parametrize("g,m,copy", [("f32", "f32", False), ("bf16", "f32", True), ("f32", "bf16", True), ("bf16", "bf16", False)])
@pytest.mark.parametrize("shapes", [UNEVEN, LONG], ids=["uneven", "long"])
def test_step(opt, shapes, g, m, copy, adamw):  # noqa: F811
    # one wave of blocks with two or more tiles each; and (of the long list) more blocks than a wave
    assert more_tiles_than(3 if adamw else 4, 2, shapes) and (shapes is UNEVEN or more_tiles_than(3 if adamw else 4, 5, shapes))
    made = build(shapes, g, m, copy, adamw, zero_weights=copy and m == "bf16")
    before = [{k: t.clone() for k, (t, _) in one.items()} for one in made]
    lr, b1, b2, t, wd = 0.02, 0.9, 0.95, 7, 0.1
    params = binding.param_list([binding.param_desc(*(one[k][0] if k in one else None for k in ("X", "G", "M", "V", "X16")), 0.75, wd) for one in made])
    if adamw:
        opt.adamw_step(params, lr, torch.tensor([t], device="cuda") if copy else t, b1, b2, 1e-8, grad_scale=scalar(0.625))
    else:
        opt.lion_step(params, lr, b1, b2, grad_scale=scalar(0.625))
    for b, one in zip(before, made):
        if b["X"].numel():
            check_step(b, {k: t for k, (t, _) in one.items()}, adamw, f32(lr), b1, b2, 1e-8, t, 0.625, 0.75, f32(wd))
        for name, (tensor, buf) in one.items():
            assert surroundings_kept(tensor, buf), name
    assert opt.get_status() == (0, 0)


@pytest.mark.parametrize("types", ["f32 f32", "f32 bf16", "bf16 f32", "bf16 bf16", "f32 in place", "bf16 in place"])
@pytest.mark.parametrize("shapes", [UNEVEN, LONG], ids=["uneven", "long"])
@pytest.mark.parametrize("kind", [2, "inf"])
def test_clip(opt, shapes, types, kind):  # noqa: F811
    assert more_tiles_than(4, 2, shapes)
    src, dst = types.split(" ", 1)
    ts = [place(s, DT[src], LIES[k % len(LIES)][0], seed=k) for k, s in enumerate(shapes)]
    grads = [t for t, _ in ts]
    before = [t.clone() for t in grads]
    # (every fourth result is cut differently from its gradient)
    outs = ts if dst == "in place" else [place(s, DT[dst], SHIFTED if k % 4 == 3 else LIES[k % len(LIES)][0], value=3.0) for k, s in enumerate(shapes)]
    want = norm64(grads, kind)
    norm, coef, alone, each = scalar(), scalar(), scalar(), torch.full((len(ts),), -1.0, device="cuda")
    items = binding.grad_list(grads, None if dst == "in place" else [o for o, _ in outs])
    opt.grad_norm(items, kind, norm_out=alone, each_out=each)
    tol = NORM if kind == 2 else 0.0
    assert abs(float(alone) - want) <= tol * want
    for t, got in zip(grads, each.tolist()):
        assert abs(got - norm64([t], kind)) <= tol * norm64([t], kind)
    opt.clip_grads(items, 0.37 * want, norm_type=kind, norm_out=norm, coef_out=coef)
    assert abs(float(norm) - want) <= tol * want and abs(float(coef) - 0.37) <= (tol + 2 * u) * 0.37
    check_clipped(grads, [o for o, _ in outs], before, 0.37)
    for t, buf in outs + ts:
        assert surroundings_kept(t, buf)
    if dst != "in place":
        assert all(torch.equal(t, b) for t, b in zip(grads, before))
    assert opt.get_status() == (0, 0)


# gradients and results that lie at different places; four rounds at once from 1024 groups of one row in a block's share
@pytest.mark.parametrize("lie,out_lie", [(PLAIN, PLAIN), (SHIFTED, SHIFTED), (SHIFTED, PLAIN)])
@pytest.mark.parametrize("types", ["f32 f32", "f32 bf16", "bf16 f32", "bf16 bf16", "f32 in place"])
def test_clip_of_long_rows(opt, types, lie, out_lie):  # noqa: F811
    src, dst = types.split(" ", 1)
    for shape in ((1, 12345679), (2, 6200003)):
        assert more_tiles_than(4, 5, [shape])
        G, buf = place(shape, DT[src], lie, seed=1)
        before = G.clone()
        out, out_buf = (G, buf) if dst == "in place" else place(shape, DT[dst], out_lie, value=3.0)
        want, coef = norm64([G]), scalar()
        opt.clip_grads(binding.grad_list([G], [out]), 0.25 * want, coef_out=coef)
        assert abs(float(coef) - 0.25) <= (NORM + 2 * u) * 0.25
        check_clipped([G], [out], [before], 0.25)
        assert surroundings_kept(out, out_buf) and surroundings_kept(G, buf)


@pytest.mark.parametrize("types", ["f32 bf16", "bf16 bf16", "bf16 in place"])
def test_clip_by_many_blocks(opt, types):  # noqa: F811
    # more than 64 tiles for every block of a wave, uneven arrays between two long ones
    src, dst = types.split(" ", 1)
    shapes = [(1, 40000003)] + UNEVEN + [(9001, 4500)]
    assert more_tiles_than(4, 65, shapes)
    ts = [place(s, DT[src], LIES[k % 4][0], seed=k) for k, s in enumerate(shapes)]
    grads = [t for t, _ in ts]
    before = [t.clone() for t in grads]
    outs = ts if dst == "in place" else [place(s, DT[dst], SHIFTED if k % 4 == 3 else LIES[k % 4][0], value=3.0) for k, s in enumerate(shapes)]
    want, norm = norm64(grads), scalar()
    opt.clip_grads(binding.grad_list(grads, [o for o, _ in outs]), 0.5 * want, norm_out=norm)
    assert abs(float(norm) - want) <= NORM * want
    for t, o, b in zip(grads, outs, before):
        check_clipped([t], [o[0]], [b], 0.5)
        assert surroundings_kept(*o)


@pytest.mark.parametrize("types", ["f32 bf16", "bf16 f32", "f32 in place"])
@pytest.mark.parametrize("kind", [2, "inf"])
def test_the_last_list_of_one_launch(opt, types, kind):  # noqa: F811
    # 96 tiles of 2048 elements, cut in any way, are clipped by one launch; one more takes two
    src, dst = types.split(" ", 1)
    for shapes, launches in (([(1, 96 * TILE)], 1), ([(1, 96 * TILE + 1)], 2), ([(1, 40 * TILE), (1, 56 * TILE)], 1), ([(1, 40 * TILE), (1, 56 * TILE), (1, 1)], 2),
                             ([(1, TILE + 1)] * 48, 1), ([(1, TILE + 1)] * 49, 2), ([(1, 5)] * 96, 1), ([(1, 5)] * 97, 2), ([(96 * 64, 16)], 1)):
        ts = [place(s, DT[src], (0, 1) if s[0] > 1 else PLAIN, seed=k) for k, s in enumerate(shapes)]
        grads = [t for t, _ in ts]
        before = [t.clone() for t in grads]
        outs = ts if dst == "in place" else [place(s, DT[dst], PLAIN, value=3.0) for s in shapes]
        want, norm, coef, alone = norm64(grads, kind), scalar(), scalar(), scalar()
        items = binding.grad_list(grads, [o for o, _ in outs])
        count = opt.launch_count()
        opt.grad_norm(items, kind, norm_out=alone)
        assert opt.launch_count() - count == 1
        opt.clip_grads(items, 0.25 * want, norm_type=kind, norm_out=norm, coef_out=coef)
        assert opt.launch_count() - count == 1 + launches, shapes[:1]
        tol = NORM if kind == 2 else 0.0
        assert abs(float(norm) - want) <= tol * want and abs(float(alone) - want) <= tol * want and abs(float(coef) - 0.25) <= (tol + 2 * u) * 0.25
        check_clipped(grads, [o for o, _ in outs], before, 0.25)
        for o, buf in outs:
            assert surroundings_kept(o, buf)


@pytest.mark.parametrize("value", [1.0, 1.5, 1.9999999, 0.7])
@pytest.mark.parametrize("n", [8, 1000, 2000003])
def test_norm_of_equal_values(opt, value, n):  # noqa: F811
    # every group rounds alike: the bound of a group is that of the whole
    t, out = torch.full((n,), value, device="cuda"), scalar()
    opt.grad_norm(binding.grad_list([t]), norm_out=out)
    want = float(t[0].double()) * math.sqrt(n)
    assert abs(float(out) - want) <= NORM * want
