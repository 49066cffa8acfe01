"""Sizes that the MXFP4 products refuse, asked of the library on the host.

The queries run in a process of their own: one that divides by a tile count of
zero ends the process that asks.
"""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def ask(expression):
    code = f"from paper_2411_12692_amd import _lib; lib = _lib.load(); A = 1 << 20; print({expression})"
    p = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, text=True, timeout=120)
    assert p.returncode == 0, f"the process ended with {p.returncode}"
    return eval(p.stdout)


@pytest.mark.parametrize("x", ["A", "None"])
def test_workspace_of_no_rows(x):
    """No rows of W: nothing is needed, for any number of tokens and a sum of any
    length."""
    got = ask(f"[lib.si_linear_mxfp4_workspace_bytes({x}, 256, m, 0, n, g) "
              "for m in (1, 4, 5, 64, 65, 5000) for n in (100, 128, 16384) for g in (0, 1)]")
    assert got == [0] * 36


def test_workspace_of_unsupported_shapes():
    """0 where the product itself is refused: more than a launch can hold, and
    lengths outside the products' range."""
    got = ask("[lib.si_linear_mxfp4_workspace_bytes(A, n, m, rows, n, g) for m, rows, n, g in "
              "((1 << 24, 1 << 24, 100, 0), (1 << 24, 64, 1 << 20, 1), (5, -1, 128, 0), (-1, 5, 128, 0), (5, 5, 0, 0), "
              "(5, 5, (1 << 20) + 1, 0), ((1 << 24) + 1, 5, 128, 0), (5, (1 << 24) + 1, 128, 0))]")
    assert got == [0] * 8


def test_refusal_of_no_rows():
    """The product of no rows is refused by its own check."""
    status, text = ask("(lib.si_linear_mxfp4(A, 0, 128, 5, 128, A, A, 0, A, 2, None, 0, None) == _lib.SI_ERR_SHAPE, "
                       "lib.si_last_error().decode())")
    assert status and "rows=0" in text


def test_the_copy_of_x_limits_only_calls_that_make_one():
    """2^24 tokens of 4096 values: x that can be read in place needs no launch for
    its copy (2^33 threads), which is refused where x has to be copied."""
    m, rows, n = 1 << 24, 3, 4096
    got = ask(f"[lib.si_linear_mxfp4_tile(1, {m}, {rows}, {n}, 0), lib.si_linear_mxfp4_tile(0, {m}, {rows}, {n}, 0), "
              f"lib.si_linear_mxfp4(A + 2, 0, {n}, {m}, {n}, A, A, {rows}, A, 2, A, 1 << 60, None) == _lib.SI_ERR_SHAPE]")
    assert got[0] >= 0 and got[1] >= 0 and got[2]
