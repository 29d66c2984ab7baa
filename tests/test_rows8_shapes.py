"""The rules that choose tiles and pieces for the operators on rows in 8 bits (csrc/ops/rows8_shapes.h), compiled by themselves on the host: every
tile is chosen for sizes that the GPU tests compute."""
import itertools
import os
import shutil
import subprocess

import pytest

import rows8_tiles as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not shutil.which("g++"), reason="no g++")


def evaluate(tmp_path, expressions, each):
    """`each` numbers for every C++ expression over the header, printed as a list of integers."""
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    lines = "\n".join(f"    {{ const auto s = {e}; for (long long v : {{{each}}}) std::printf(\"%lld \", v); std::printf(\"\\n\"); }}" for e in expressions)
    src.write_text('#include <cstdio>\n#include "rows8_shapes.h"\nusing namespace cams_ops;\nint main()\n{\n' + lines + "\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2111_00705_amd", "csrc", "ops"), "-o", str(exe), str(src)],
                   check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout
    return [tuple(int(x) for x in line.split()) for line in out.splitlines()]


def test_products_of_the_gpu_tests_take_every_tile(tmp_path):
    got = evaluate(tmp_path, [f"product_shape({r}, {c}, {o}, true, true)" for r, c, o in T.PRODUCTS], "(long long)s.high, (long long)s.wide, (long long)(s.splits > 1)")
    assert got == [tuple(int(v) for v in want) for want in T.PRODUCTS.values()]
    tiles = {(64, 64, True), (64, 64, False), (64, 128, False), (128, 128, True), (128, 128, False), (256, 128, False), (256, 256, False)}
    assert tiles < set(T.PRODUCTS.values())


def test_weight_gradients_of_the_gpu_tests_take_every_tile(tmp_path):
    calls, want = [], []
    for (n, per, cols, outs), tile in T.WEIGHTS.items():
        for binary, dtype, lies, wide in itertools.product((0, 1), (0, 1, 2), (0, 1), (0, 1)):
            calls.append(f"weight_shape({n * per}, {cols}, {outs}, {n}, {binary}, {dtype}, {lies}, {wide})")
            want.append((tile[0], int(tile[1])))
    assert evaluate(tmp_path, calls, "(long long)s.tile, (long long)(s.splits > 1)") == want
    assert set(T.WEIGHTS.values()) == {(64, True), (64, False), (128, True), (128, False), (256, False)}


def test_planes(tmp_path):
    """(planes of q, of dy, dy written anew) for fp32, bfloat16, half precision."""
    call = lambda cols, outs, binary, dtype, wide, lies=1: f"weight_shape(640, {cols}, {outs}, 2, {binary}, {dtype}, {lies}, {wide})"
    cases = {
        call(64, 64, 0, 0, 0): (1, 3, 1), call(64, 64, 1, 0, 1): (1, 3, 1),
        call(64, 64, 1, 1, 1): (1, 1, 0), call(64, 64, 1, 1, 1, 0): (1, 1, 1), call(64, 60, 1, 1, 1): (1, 1, 1),
        call(64, 640, 0, 1, 1): (3, 1, 0), call(64, 640, 0, 1, 0): (2, 1, 0), call(640, 64, 0, 1, 1): (1, 3, 1), call(640, 64, 0, 1, 0): (1, 2, 1),
        call(64, 64, 1, 2, 1): (1, 2, 1), call(64, 64, 1, 2, 0): (1, 2, 1), call(64, 64, 0, 2, 0): (1, 2, 1), call(64, 64, 0, 2, 1): (1, 3, 1),
    }
    assert evaluate(tmp_path, list(cases), "(long long)s.q_planes, (long long)s.dy_planes, (long long)s.copied") == list(cases.values())
