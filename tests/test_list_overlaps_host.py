"""CPU: which arrays of a list overlap.  Whatever is in order reaches the missing context (no device is touched, the pointers are
numbers)."""
import random

import pytest

from test_list_host import ALIAS, BASE, BF16, F32, INVALID, clip, grad, lib, norm, param, rule, step  # noqa: F401

DISJOINT = INVALID


def piece(matrix_ld, rows, cols, size=4):
    """The part of a matrix that two slices name, as an array of its own."""
    r0, r1, rstep = rows.indices(1 << 20)
    c0, c1, _ = cols.indices(matrix_ld)
    n = len(range(r0, r1, rstep))
    return dict(rows=n, cols=c1 - c0, G=BASE + (r0 * matrix_ld + c0) * size, ldg=matrix_ld * rstep if n > 1 else c1 - c0)


# two parts of one matrix of 24 columns that share no element
APART = [
    ((slice(0, 3, 2), slice(0, 24)), (slice(1, 2), slice(0, 24))),           # even rows, the odd one
    ((slice(0, 5, 2), slice(0, 24)), (slice(1, 4, 2), slice(0, 24))),
    ((slice(0, 4), slice(0, 8)), (slice(1, 2), slice(8, 16))),               # columns, a row beside them
    ((slice(0, 4), slice(8, 16)), (slice(2, 3), slice(0, 8))),
    ((slice(0, 4), slice(8, 16)), (slice(1, 2), slice(16, 24))),
    ((slice(0, 8), slice(0, 8)), (slice(0, 8, 2), slice(8, 24))),            # every row, every other row
    ((slice(0, 9, 2), slice(0, 24)), (slice(1, 8, 4), slice(0, 24))),
    ((slice(0, 9, 3), slice(0, 12)), (slice(0, 8, 2), slice(12, 24))),
]
# ... and that share one
TOGETHER = [
    ((slice(0, 5, 2), slice(0, 24)), (slice(2, 3), slice(0, 24))),
    ((slice(0, 4), slice(0, 9)), (slice(1, 2), slice(8, 16))),
    ((slice(0, 4), slice(8, 16)), (slice(3, 4), slice(0, 9))),
    ((slice(0, 8), slice(0, 9)), (slice(0, 8, 2), slice(8, 24))),
    ((slice(0, 9, 2), slice(0, 24)), (slice(1, 9, 3), slice(0, 1))),         # rows 0 2 4 6 8 and 1 4 7
    ((slice(0, 9, 2), slice(23, 24)), (slice(1, 9, 7), slice(0, 24))),       # rows 1 and 8
]


@pytest.mark.parametrize("pair,want", [(p, DISJOINT) for p in APART] + [(p, ALIAS) for p in TOGETHER])
def test_parts_of_one_matrix(lib, pair, want):  # noqa: F811
    a, b = (piece(24, *p) for p in pair)
    for x, y in ((a, b), (b, a)):
        assert clip(lib, grad(**x), grad(**y)) == want
        # written parameters, and a gradient that lies beside a parameter
        at = lambda d: dict(rows=d["rows"], cols=d["cols"], X=d["G"], ldx=d["ldg"])  # noqa: E731
        assert step(lib, param(**at(x)), param(at=1 << 16, **at(y))) == want
        one = {k: x[k] for k in ("rows", "cols")}
        if (x["rows"], x["cols"]) == (y["rows"], y["cols"]):
            assert step(lib, param(X=x["G"], ldx=x["ldg"], G=y["G"], ldg=y["ldg"], **one)) == want
    # arrays that are only read may overlap
    assert norm(lib, grad(**a), grad(**b)) == DISJOINT


def test_three_parts_of_one_matrix(lib):  # noqa: F811
    t = [piece(300, slice(0, 50), slice(0, 300)), piece(300, slice(50, 51), slice(0, 100)), piece(300, slice(50, 97), slice(100, 300)),
         piece(300, slice(51, 97), slice(0, 100))]
    assert clip(lib, *[grad(**x) for x in t]) == DISJOINT
    assert clip(lib, *[grad(**x) for x in t + [piece(300, slice(96, 97), slice(299, 300))]]) == ALIAS


def test_numbers_in_the_gaps_of_an_array(lib):  # noqa: F811
    # rows of 8 fp32 numbers, 16 apart: a number of the caller's between two rows is no part of the array
    a = grad(rows=4, cols=8, ldg=16)
    for row in range(3):
        for col in range(16):
            at, want = BASE + (16 * row + col) * 4, ALIAS if col < 8 else DISJOINT
            assert norm(lib, a, norm_out=at) == want and norm(lib, a, norm_out=None, coef=at) == want
            assert clip(lib, a, norm_out=at) == want and clip(lib, a, coef=at) == want and clip(lib, a, norms=at, num=1) == want
            p = param(rows=4, cols=8, ldx=16)
            assert step(lib, p, r=rule(grad_scale=at)) == want and step(lib, p, r=rule(grad_scale=at), adamw=False) == want
    assert norm(lib, a, norm_out=None, each=BASE + 15 * 4) == DISJOINT
    assert norm(lib, a, grad(G=BASE + 0x1000), norm_out=None, each=BASE + 15 * 4) == ALIAS      # two numbers, one of them in row 1
    assert step(lib, param(rows=4, cols=8, ldx=16), r=rule(step_dev=BASE + 8 * 4)) == DISJOINT
    assert step(lib, param(rows=4, cols=8, ldx=16), r=rule(step_dev=BASE + 6 * 4)) == ALIAS


def test_drawn_pairs(lib):  # noqa: F811
    # against the set of their bytes
    rng = random.Random(5)
    seen = {DISJOINT: 0, ALIAS: 0}
    for _ in range(3000):
        arrays, bytes_of = [], []
        for k in range(2):
            size = rng.choice([2, 4])
            rows, cols = rng.randint(1, 9), rng.randint(1, 9)
            ld = cols + rng.choice([0, 1, 3, 9, 20])
            if k and rng.random() < 0.4:
                ld = max(cols, ld0 * rng.choice([1, 2, 3]))  # noqa: F821
            ld0 = ld  # noqa: F841
            at = rng.randint(0, 60) * 4
            arrays.append(grad(rows=rows, cols=cols, G=BASE + at, ldg=ld, g=BF16 if size == 2 else F32))
            bytes_of.append({at + (i * ld + j) * size + b for i in range(rows) for j in range(cols) for b in range(size)})
        want = ALIAS if bytes_of[0] & bytes_of[1] else DISJOINT
        seen[want] += 1
        assert clip(lib, *arrays) == want and clip(lib, *arrays[::-1]) == want
    assert min(seen.values()) > 500


def test_long_arrays_are_compared_quickly(lib):  # noqa: F811
    # a million rows each, side by side: few of them have to be looked at
    a = grad(rows=1 << 20, cols=4000, ldg=4096 * 2)
    b = grad(rows=1 << 20, cols=90, G=BASE + 4000 * 4, ldg=4096)
    assert clip(lib, a, b) == DISJOINT
    b.ldg = b.ldo = 4095
    assert clip(lib, a, b) == ALIAS
