"""Tiles and slices that the products of the INT8 linear layers and of the orthogonalised updates take at the sizes of
the GPU tests (csrc/mm_plan.h, host arithmetic): the kernels that those sizes are named for, and together every kernel
that any size takes."""
import math
import os
import random
import re
import subprocess

import pytest

import test_gpu_linear_i8
import test_gpu_ortho
import test_gpu_tiles
import test_gpu_weight_steps

HERE = os.path.dirname(os.path.abspath(__file__))
# kTileKinds in its order: the tile's sides, and whether two groups of waves share it
KINDS = [(256, 256, ""), (192, 192, ""), (192, 128, ""), (128, 128, ""), (96, 96, ""), (64, 64, ""), (64, 64, "2"),
         (128, 128, "2"), (96, 96, "2")]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """Plans of lines of mm_plan_query.cpp."""
    exe = str(tmp_path_factory.mktemp("plan") / "mm_plan_query")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", os.path.join(HERE, "..", "paper_1802_00930_amd", "csrc"),
                           os.path.join(HERE, "helpers", "mm_plan_query.cpp"), "-o", exe])

    def run(lines):
        res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120,
                             check=True)
        out = [tuple(map(int, line.split())) for line in res.stdout.splitlines()]
        assert len(out) == len(lines)
        return out
    return run


def i8(rows):
    return ["i8 %d %d %d" % r for r in rows]


def ortho(rows, split):
    return ["ortho %d %d %d %d" % (*r, split) for r in rows]


def tile(kind, slices=1):
    if kind < 0:
        return "few"
    a, b, groups = KINDS[kind]
    return "%d x %d%s%s" % (a, b, " (2)" if groups else "", ", %d slices" % slices if slices > 1 else "")


def comments(name):
    """The comment behind every row of a list of test_gpu_tiles."""
    text = open(os.path.join(HERE, "test_gpu_tiles.py")).read()
    body = text[text.index("\n%s = [" % name):]
    return re.findall(r"\),\s+# (.*)", body[:body.index("\n]")])


def test_products_take_the_tiles_that_they_are_named_for(plan):
    named = comments("PRODUCTS")
    assert len(named) == len(test_gpu_tiles.PRODUCTS)
    got = [tile(*p) for p in plan(i8(test_gpu_tiles.PRODUCTS))]
    want = [c.replace("rows of a batch", "few").replace(" by two groups", " (2)") for c in named]
    assert got == want


def test_updates_take_the_tiles_that_they_are_named_for(plan):
    named = comments("ORTHO")
    assert len(named) == len(test_gpu_tiles.ORTHO)
    for row, name in zip(test_gpu_tiles.ORTHO, named):
        g, s, p, x, _ = plan(ortho([row[1:]], row[0] == "f32"))[0]
        assert "%s; %s; %s" % (tile(g, s), tile(p), tile(x)) == name, row


def test_weight_steps_take_the_tiles_that_they_are_named_for(plan):
    rows = test_gpu_weight_steps.TILES
    for (b, r, c, name), (g, s, p, x, grouped) in zip(rows, plan(ortho([row[:3] for row in rows], 1))):
        assert "%s; %s%s; %s" % (tile(g, s), tile(p), " together" if grouped else "", tile(x)) == name, (b, r, c)
    for row in test_gpu_weight_steps.TOGETHER:
        assert plan(ortho([row], 1))[0][4] == 1, row
    # every size of the lists that are meant for it
    assert all(p[4] for p in plan(ortho([(1, 51, 8000), (1, 8000, 51)], 1)))


def log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def test_every_product_kernel_that_sizes_take_is_tested(plan):
    def kernel(row, p):
        return ("few", min(row[0], 17), min(row[0], 33)) if p[0] < 0 else (p[0], p[1] > 1)
    rows = test_gpu_tiles.PRODUCTS + test_gpu_linear_i8.PRODUCTS + test_gpu_weight_steps.PRODUCTS
    tested = {kernel((16 if r[0] <= 16 else 32 if r[0] <= 32 else 64,), p) if p[0] < 0 else kernel(r, p)
              for r, p in zip(rows, plan(i8(rows)))}
    rng = random.Random(1)
    sweep = [(log(rng, 1, 60000), log(rng, 1, 60000), log(rng, 1, 131071)) for _ in range(60000)]
    taken = {kernel((16 if r[0] <= 16 else 32 if r[0] <= 32 else 64,), p) if p[0] < 0 else kernel(r, p)
             for r, p in zip(sweep, plan(i8(sweep)))}
    assert len(taken) > 15 and taken <= tested


def instances(p):
    g, s, y, x, grouped = p
    return {("gram", g, s > 1), ("poly", y), ("step", x)}


@pytest.mark.parametrize("split", [0, 1])
def test_every_update_kernel_that_sizes_take_is_tested(plan, split):
    t = ("f32" if split else "bf16",)
    rows = [r[1:] for r in test_gpu_tiles.ORTHO + test_gpu_weight_steps.UPDATES if r[:1] == t] + test_gpu_ortho.SHAPES
    tested = set().union(*map(instances, plan(ortho(rows, split))))
    rng = random.Random(2)
    sweep = [(rng.choice([1, 1, 1, 2, 4, 9, 16]), log(rng, 1, 16384), log(rng, 1, 16384)) for _ in range(60000)]
    taken = set().union(*map(instances, plan(ortho(sweep, split))))
    assert len(taken) > 15 and taken <= tested
    if split:
        rows = test_gpu_tiles.MUON + [r[:3] for r in test_gpu_weight_steps.TILES]
        with_group = lambda p: instances(p) | {("poly", p[2], p[4])}  # noqa: E731
        tested = set().union(*map(with_group, plan(ortho(rows, 1))))
        assert set().union(*map(with_group, plan(ortho(sweep, 1)))) <= tested
