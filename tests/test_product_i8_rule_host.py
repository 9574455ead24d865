"""The rules of the 8-bit integer product on the host: every form of tiles is reached, by a size that the GPU tests run too, and rows left over are whole tiles'."""
import os
import shutil
import subprocess

import pytest

from paper_2506_19852_amd import build as hip_build
from test_gpu_linear_i8 import SIZES
from test_gpu_linear_i8_long import LONG

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if not os.path.exists(hip_build.HIPCC) and shutil.which(hip_build.HIPCC) is None:
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("host") / "product_i8_rule"
    r = subprocess.run([hip_build.HIPCC, *hip_build.FLAGS, "--cuda-host-only", os.path.join(ROOT, "tests", "host", "product_i8_rule.hip"), "-o", str(exe)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]

    def run(lines):
        r = subprocess.run([str(exe)], input="\n".join(lines), stdout=subprocess.PIPE, text=True, timeout=120)
        assert r.returncode == 0
        return [[int(v) for v in line.split()] for line in r.stdout.strip().split("\n")]
    return run


def _of(rule, sizes):
    small = rule([f"small {m} {n}" for m, n, _ in sizes])
    large = [s for s, (p,) in zip(sizes, small) if not p]
    return small, large, rule([f"form {m} {n} {-(-k // 128)}" for m, n, k in large])


def test_every_form_is_reached_by_a_tested_size(rule):
    small, large, plans = _of(rule, SIZES)
    forms = {p[0] for p in plans} | {p[5] for p, s in zip(plans, large) if p[4] != s[0]}
    assert forms == set(range(10)), (forms, [(s, p) for s, p in zip(large, plans)])
    assert {p for (p,) in small} == {0, 1}


def test_rows_left_over_are_behind_whole_tiles(rule):
    sizes = [(m, n, k) for m in (5, 64, 300, 2000, 5120, 5121, 9999, 14040, 32760) for n in (70, 1500, 5120, 8192) for k in (100, 5120, 14040)] + [(2500, 8192, 4096), (6000, 3000, 4096)]
    _, large, plans = _of(rule, sizes)
    for (m, n, k), (form, rows, columns, _, of_form, rest) in zip(large, plans):
        assert of_form == m or (0 < of_form < m and of_form % rows == 0 and form < 2), (m, n, k)
    assert any(p[4] != s[0] for s, p in zip(large, plans)) and any(p[4] == s[0] for s, p in zip(large, plans))
    _, large, plans = _of(rule, SIZES)
    assert any(p[4] != s[0] for s, p in zip(large, plans))


def test_large_products_take_large_tiles_and_few_rows_parts_of_the_groups(rule):
    large, few = rule(["form 32760 5120 40", "form 64 5120 40"])
    assert large[1:4] == [256, 256, 1] and few[1:3] == [32, 64] and few[3] > 1


@pytest.mark.parametrize("shape", [(1, 1), (1, 20), (20, 1), (5, 3), (6, 6), (7, 5), (12, 7), (128, 20), (17, 33)], ids=str)
def test_every_tile_is_taken_once(rule, shape):
    (flat,) = rule([f"tiles {shape[0]} {shape[1]}"])
    got = {(flat[i], flat[i + 1]) for i in range(0, len(flat), 2)}
    assert len(flat) == 2 * shape[0] * shape[1] and got == {(m, n) for m in range(shape[0]) for n in range(shape[1])}


def test_long_gradients_leave_rows_over_in_either_product(rule):
    _, _, dx = _of(rule, [(m, k, n) for m, n, k in LONG])
    _, _, dw = _of(rule, [(n, k, m) for m, n, k in LONG])
    assert [p[4] < m for p, (m, _, _) in zip(dx, LONG)] == [True, False] and [p[4] < n for p, (_, n, _) in zip(dw, LONG)] == [False, True]
