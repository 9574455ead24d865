"""The rules of the 8-bit product on the host: every form of tiles is reached, and by a size that the GPU tests run; every tile is taken once; the
pieces of a stage fill their place in LDS without overlap and are read without bank conflicts."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2506_19852_amd import build as hip_build
from test_gpu_product import MORE_SIZES, SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if not os.path.exists(hip_build.HIPCC) and shutil.which(hip_build.HIPCC) is None:
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("host") / "product_rule"
    r = subprocess.run([hip_build.HIPCC, *hip_build.FLAGS, "--cuda-host-only", os.path.join(ROOT, "tests", "host", "product_rule.hip"), "-o", str(exe)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]

    def run(lines):
        r = subprocess.run([str(exe)], input="\n".join(lines), stdout=subprocess.PIPE, text=True, timeout=120)
        assert r.returncode == 0
        return [[int(v) for v in line.split()] for line in r.stdout.strip().split("\n")]
    return run


def test_every_form_is_reached_by_a_tested_size(rule):
    tested = [s for s in SIZES if s[0] > 16]
    forms = {f[0] for f in rule([f"form {m} {n} {-(-k // 128)}" for m, n, k in tested])}
    assert forms == set(range(8)), forms


def test_large_products_take_large_tiles_and_few_tiles_split_the_groups(rule):
    large, few, one = rule(["form 32760 5120 40", "form 64 512 64", "form 17 1 1"])
    assert large[1:4] == [256, 256, 1] and few[3] > 1 and max(one[1:3]) <= 128


def test_rows_left_over_take_a_form_of_their_own(rule):
    shapes = [(m, n, g) for m in (300, 2000, 5120, 5121, 9999, 14040, 32760) for n in (1500, 5120, 8192) for g in (3, 40, 110)]
    got = rule([f"form {m} {n} {g}" for m, n, g in shapes])
    for (m, n, g), (form, rows, columns, _, of_form, rest) in zip(shapes, got):
        assert of_form == m or (0 < of_form < m and of_form % rows == 0 and form < 2), (m, n, g)
    assert any(r[4] != m for (m, _, _), r in zip(shapes, got)) and any(r[4] == m for (m, _, _), r in zip(shapes, got))
    tested = [s for s in SIZES if s[0] > 16]
    assert any(r[4] != s[0] for s, r in zip(tested, rule([f"form {m} {n} {-(-k // 128)}" for m, n, k in tested])))


@pytest.mark.parametrize("shape", [(1, 1), (1, 20), (20, 1), (7, 3), (8, 8), (9, 5), (128, 20), (17, 33)], ids=str)
def test_every_tile_is_taken_once(rule, shape):
    (flat,) = rule([f"tiles {shape[0]} {shape[1]}"])
    got = {(flat[i], flat[i + 1]) for i in range(0, len(flat), 2)}
    assert len(flat) == 2 * shape[0] * shape[1] and got == {(m, n) for m in range(shape[0]) for n in range(shape[1])}


@pytest.mark.parametrize("operand", [0, 1])
def test_pieces(rule, operand):
    at, conflicts = rule([f"pieces {operand}"])
    at = np.array(at).reshape(256, 8)
    assert np.array_equal(np.sort(at.ravel()), np.arange(256 * 8) * 16) and (at // 256 == np.arange(256)[:, None] // 2).all()
    # fragments of a lane lie at constant distances: rows 16 apart of A, 4 apart (within 16) of B
    step = 4 if operand else 16
    rows = [r for r in range(64) if r % 16 < 4] if operand else range(240)
    for r in rows:
        assert (at[r + step] - at[r] == step * 128).all()
    assert conflicts == [0]


def test_every_form_is_reached_by_a_tested_size_that_is_not_small(rule):
    small = [r[0] for r in rule([f"small {m} {n}" for m, n, _ in SIZES])]
    assert {0, 1} == set(small)
    tested = [s for s, is_small in zip(SIZES, small) if not is_small]
    forms = {f[0] for f in rule([f"form {m} {n} {-(-k // 128)}" for m, n, k in tested + MORE_SIZES])}
    assert forms == set(range(8)), forms
    assert [r[0] for r in rule(["small 16 100000", "small 17 2048", "small 17 2064", "small 512 128", "small 1000 1000"])] == [1, 1, 0, 1, 0]


def test_the_tiles_of_every_launch_are_those_of_a_tested_size(rule):
    """Of sizes that take tiles: each form for all rows, and pairs of forms that share the rows, large ones for the rest among them."""
    from test_gpu_product import TWO_LAUNCHES

    def tiled(sizes):
        small = rule([f"small {m} {n}" for m, n, _ in sizes])
        return [(m, n, k) for (m, n, k), (is_small,) in zip(sizes, small) if not is_small]

    sizes = tiled(SIZES + MORE_SIZES + TWO_LAUNCHES)
    assert len(tiled(MORE_SIZES)) == 3 and len(tiled(TWO_LAUNCHES)) == len(TWO_LAUNCHES)
    alone, shared = set(), set()
    for (m, _, _), (form, _, _, _, of_form, rest) in zip(sizes, rule([f"form {m} {n} {-(-k // 128)}" for m, n, k in sizes])):
        alone.add(form) if of_form == m else shared.add((form, rest))
    assert alone == set(range(8)), alone
    assert shared == {(0, 6), (0, 1), (0, 2), (0, 3), (1, 3), (1, 7)}, shared
