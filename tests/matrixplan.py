"""Asks the library's own rules (csrc/ob_matrix_plan.h) which kernels a call of the matrix operators takes, without a device."""
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@functools.lru_cache(maxsize=None)
def program():
    exe = os.path.join(tempfile.mkdtemp(prefix="matrix_plan_"), "matrix_plan")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "paper_2104_06069_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "matrix_plan.cpp"), "-o", exe], check=True)
    return exe


def ask(*questions):
    lines = "".join(" ".join(str(int(v) if isinstance(v, bool) else v) for v in q) + "\n" for q in questions)
    r = subprocess.run([program()], input=lines, capture_output=True, text=True, check=True)
    return [line.split() for line in r.stdout.splitlines()]


def of_list(shapes, fine, coefficients, steps):
    """shapes: (rows, columns) of the matrices -> [(way, terms, kind of the symmetric products, of the full ones)] or "small" """
    coefficients = list(coefficients) + list(coefficients[-3:]) * steps
    sides = [s for r, c in shapes if r for s in (min(r, c), max(r, c))]
    words, = ask(("list", fine, steps, *coefficients[:3 * steps], len(sides) // 2, *sides))
    return "small" if words == ["small"] else [tuple(words[i:i + 4]) for i in range(0, len(words), 4)]


def of_experts(groups, rows, k, n, layout, direct, max_rows=None):
    """-> (forward, input_grad, weight_grad: kind and parts)"""
    h, w = (k, n) if layout == "kn" else (n, k)
    f, i, g = ask(("rows", groups, rows, k, n, direct), ("rows", groups, rows, n, k, direct), ("weights", groups, rows, h, w, max_rows or rows, direct))
    return f[0], i[0], tuple(g)
