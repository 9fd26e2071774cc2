"""The rules that choose the matrix operators' kernels (csrc/ob_matrix_plan.h), without a device: the sizes of
tests/test_gpu_matrix_tiles.py reach every kind of tile, for every order of the operands and number of terms, and the tables of tiles
hold each tile once."""
import itertools

import pytest

pytest.importorskip("torch")
from tests import matrixplan  # noqa: E402
from tests.test_gpu_matrix_tiles import APART, EXPERTS, LISTS, QUINTIC, SMALL  # noqa: E402


def test_experts_cases_reach_every_kind():
    rows, weights = set(), set()
    for (groups, count, k, n, direct), layout in itertools.product(EXPERTS, ("kn", "nk")):
        forward, input_grad, (kind, parts) = matrixplan.of_experts(groups, count, k, n, layout, direct)
        rows |= {(forward, layout == "kn", direct), (input_grad, layout == "nk", direct)}      # (W read across its rows, or along)
        weights.add((kind, parts != "1", direct))
    for strided in (False, True):
        assert {(kind, strided, True) for kind in ("T256", "T128", "T64", "DEEP", "few")} <= rows
        assert {(kind, strided, False) for kind in ("T128", "T64", "few")} <= rows
    assert {(kind, False, True) for kind in ("T256", "T128", "T64", "DEEP")} | {("T128", False, False), ("T64", False, False)} <= weights
    assert {("T64", True, True), ("T64", True, False)} <= weights


def test_lists_reach_every_kind():
    sides = lambda list_: [(m, n) for count, m, n in list_ for _ in range(count)]  # noqa: E731
    symmetric, full = set(), set()
    for list_, fine in LISTS:
        for way, terms, sym, apply in matrixplan.of_list(sides(list_), fine, QUINTIC, 5):
            symmetric.add((terms, sym))
            full.add((terms, apply))
            symmetric.add((way, sym))
            full.add((way, apply))
    for found in (symmetric, full):
        assert found >= {(what, kind) for what in ("1", "2", "step", "follow") for kind in ("T256", "T128", "T64", "DEEP")}
    for list_, fine in APART:
        ways = [(p[0], p[1]) for p in matrixplan.of_list(sides(list_), fine, QUINTIC, 5)]
        assert sorted(ways) == [("follow", "2"), ("step", "2")] if fine else sorted(ways) == [("follow", "2"), ("step", "1")], ways
    assert matrixplan.of_list(SMALL, True, QUINTIC, 5) == "small"
