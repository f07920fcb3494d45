"""The sizes at which the linear layers are tested take every way that there is, and the tests' bounds see a lost part of a sum (CPU)."""
import math
import os
import random

import pytest
import torch

from tests._ways import OPS, WAYS, sum_error, way_class


@pytest.fixture(scope="module")
def lib():
    import paper_2602_01872_amd as g
    if not os.path.exists(g.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return g.load()


@pytest.mark.parametrize("op", OPS)
def test_every_way_is_among_the_tested(lib, op):
    tested = {way_class(lib, op, *e) for e in WAYS[op]}
    r = random.Random(OPS.index(op))

    def size(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))

    for _ in range(20_000):
        i, j, s = (size(1, 8192), size(1, 8192), size(1, 300_000)) if op == "dw" else (size(1, 300_000), size(1, 8192), size(1, 20_000))
        i = max(8, i // 8 * 8) if op == "dw" and r.random() < 0.6 else i
        j = max(8, j // 8 * 8) if r.random() < 0.6 else j
        s = max(16, s // 16 * 16) if r.random() < 0.6 else s
        pad, off = r.choice([(0, 0), (0, 0), (8, 0), (16, 0), (1, 0), (3, 1)])
        if i * j * s < 1 << 37:
            assert way_class(lib, op, i, j, s, pad, off) in tested, (i, j, s, pad, off)


@pytest.mark.parametrize("op,step", [("bf16", 64), ("dx", 64), ("dw", 64), ("e4m3", 128), ("e4m3 to fp32", 128)])
def test_the_largest_tile_is_tested_at_odd_and_even_numbers_of_steps(lib, op, step):
    seen = set()
    for i, j, s, pad, off in WAYS[op]:
        if way_class(lib, op, i, j, s, pad, off)[1:4] == ("tiles", 2, "one"):
            assert i % 256 and j % 256
            seen.add((min(-(-s // step), 6 - -(-s // step) % 2), s % step == 0))
    assert {n for n, _ in seen} >= {1, 2, 3, 4, 5} and {whole for _, whole in seen} == {True, False}


@pytest.mark.parametrize("i,j,s,splits", [(16, 24, 20_001, 64), (130, 70, 40_000, 128)])
def test_the_bound_sees_a_lost_split(i, j, s, splits):
    r = torch.Generator().manual_seed(3)
    a, b = (torch.randn(s, n, generator=r).to(torch.bfloat16).double() for n in (i, j))
    want, size = a.t() @ b, (a.square().t() @ b.square()).sqrt()
    each = -(-s // splits)
    parts = [(a[k:k + each].float().t() @ b[k:k + each].float()).double() for k in range(0, s, each)]
    bound = sum_error(s) * float(size.norm())
    assert float((sum(parts) - want).norm()) <= bound
    for wrong in (sum(parts[:-1]), sum(parts) + parts[0], torch.zeros_like(want)):
        assert float((wrong - want).norm()) > 20 * bound
