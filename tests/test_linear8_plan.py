"""The rules that choose the kernels of products in 8 bits (csrc/ob_linear8_plan.h), without a device: the sizes of
tests/test_gpu_linear8.py reach every kind, and parts stay within the workspace."""
import os
import random
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "linear8_plan")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "paper_2104_06069_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "linear8_plan.cpp"), "-o", exe], check=True)

    def ask(questions):
        lines = "".join(" ".join(str(int(v)) for v in q) + "\n" for q in questions)
        return [tuple(line.split()) for line in subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout.splitlines()]
    return ask


def sizes(name):
    text = open(os.path.join(ROOT, "tests", "test_gpu_linear8.py")).read()
    at = text.index(f"def {name}(")
    return [tuple(map(int, m)) for m in re.findall(r"\((\d+), (\d+), (\d+)\)", text[text.rindex("parametrize(\"rows,k,n\"", 0, at):at])]


def test_the_sizes_of_the_tests_reach_every_kind(ask):
    found = set()
    for name in ("test_many_tiles", "test_few_rows"):
        cases = sizes(name)
        assert len(cases) >= 8
        for wide in (False, True):
            for (rows, k, n), plan in zip(cases, ask([(rows, n, (k + 127) // 128, wide, False) for rows, k, n in cases])):
                found.add((wide,) + (plan if plan[0] == "few" else (plan[0], plan[1] != "1")))
            # (into rows of n + 8 results, of any address: never FLOW256; into a new tensor:)
            for (rows, k, n), plan in zip(cases, ask([(rows, n, (k + 127) // 128, wide, n % 8 == 0) for rows, k, n in cases])):
                found.add((wide,) + (plan if plan[0] == "few" else (plan[0], plan[1] != "1")))
    for wide in (False, True):
        assert {(wide, kind, False) for kind in ("W256", "W128", "W64", "TEAMS64")} <= found, found
        assert (wide, "W64", True) in found and (wide, "TEAMS64", True) in found
        assert {(wide, "few", "32", "8"), (wide, "few", "16", "8"), (wide, "few", "16", "16")} <= found, found
        assert (wide, "FLOW256", False) in found


def test_any_size(ask):
    """The program itself ends where parts are more than the slabs or the workspace has room for."""
    rng = random.Random(0)
    size = lambda most: int(2 ** rng.uniform(0, most))  # noqa: E731
    questions = [(size(22), size(20), rng.choice([0, 1, size(15)]), rng.random() < 0.5, rng.random() < 0.5) for _ in range(20000)]
    assert len(ask(questions)) == len(questions)
    small = [(size(10), size(10), size(15), rng.random() < 0.5, 1) for _ in range(20000)]
    assert any(int(a[1]) > 1 for a in ask(small) if a[0] != "few")


def test_the_products_of_both_formats_reach_every_kind(ask):
    """Each size of tests/test_gpu_linear8_tiles.py goes through forward and both gradients, in both formats, into 16 and 32 bits."""
    pytest.importorskip("torch")
    from tests.test_gpu_linear8_tiles import TILES
    found = set()
    for wide in (False, True):
        for (rows, depth, cols), plan in zip(TILES, ask([(rows, cols, (depth + 127) // 128, wide, cols % 8 == 0) for rows, depth, cols in TILES])):
            found.add((wide, plan[0], plan[1] != "1"))
            if plan[0] == "FLOW256":      # (several tiles for a workgroup, of two slabs and of more)
                found.add((wide, plan[0], "two" if depth <= 256 else "more") if -(-rows // 256) * -(-cols // 256) > 2 * 256 else None)
    for wide in (False, True):
        assert {(wide, kind, False) for kind in ("W256", "W128", "FLOW256")} <= found, found
        assert {(wide, "FLOW256", "two"), (wide, "FLOW256", "more")} <= found, found
        assert any((wide, kind, True) in found for kind in ("W64", "TEAMS64"))
    assert {kind for _, kind, _ in found - {None}} == {"W256", "W128", "W64", "TEAMS64", "FLOW256"}, found
