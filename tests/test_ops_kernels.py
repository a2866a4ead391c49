"""Which kernels of the row operators the library holds: every one that some width asks for, and no other."""
import re
import shutil
import subprocess

import pytest

from paper_2607_19539_b200 import binding as B, ops


def packs_of(vec, rows, width, values, most_threads, ragged):
    """row_shape of csrc/rowops.cu: packs of `vec` elements per thread."""
    packs = (width + 2 * (vec - 1)) // vec if ragged else -(-width // vec)
    want = 8 if rows <= 296 else values
    threads = lambda n: -(-(-(-packs // n)) // 32) * 32  # noqa: E731
    after = lambda n: 2 * n if vec >= 4 or n >= 32 else 4 * n  # noqa: E731
    n = 1 if vec >= 4 else 2
    while (after(n) * vec <= want and packs > 32 * n) or threads(n) > most_threads(vec * n):
        n = after(n)
    return n


def reached():
    norm_threads = lambda v: 1024 if v <= 8 else 512  # noqa: E731
    swiglu_threads = lambda v: 1024 if v <= 16 else 512  # noqa: E731
    norm, back, swiglu = set(), set(), set()
    # the number of packs changes only where the number of warps does
    widths = sorted({w for w in range(1, ops.MAX_ROW + 1) if w < 600 or w % 64 in (0, 1, 7, 8, 63) or w > ops.MAX_ROW - 32})
    for rows in (1, 296, 297, 100000):
        for w in widths:
            for vec in (8, 4, 1):
                for ragged in (False, True):
                    if (ragged and (vec == 1 or (w + 2 * (vec - 1)) // vec * vec > ops.MAX_ROW)) or (not ragged and w % vec):
                        continue
                    norm.add((vec, packs_of(vec, rows, w, vec if vec >= 4 else 8, norm_threads, ragged), ragged))
                    back.add((vec, packs_of(vec, rows, w, 8, norm_threads, ragged), ragged))
            for vec in (8, 4, 2, 1):
                if w % vec == 0:
                    swiglu.add((vec, packs_of(vec, rows, w, 16, swiglu_threads, False)))
    return norm, back, swiglu


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm to list the library's kernels with")
def test_every_row_kernel_is_reached_and_every_reached_one_is_there():
    B.load()
    names = subprocess.run(["nm", "-C", B.library_path()], capture_output=True, text=True, check=True).stdout
    have = lambda kernel: {tuple(m.split(", ")) for m in re.findall(rf"::{kernel}<([^<>]*)>\(", names)}  # noqa: E731
    norm, back, swiglu = reached()
    T = {8: ["__nv_bfloat16", "__half"], 4: ["float"], 2: ["__nv_bfloat16", "__half"], 1: ["__nv_bfloat16", "__half", "float"]}
    weights = lambda t: {t, "float"}  # noqa: E731
    flag = lambda r: "true" if r else "false"  # noqa: E731
    norms = {(t, w, str(v), str(n), flag(r)) for v, n, r in norm for t in T[v] for w in weights(t)}
    assert have("add_norm_kernel") == norms and have("add_norm_lean_kernel") == norms
    for kernel, ragged in (("add_norm_backward_kernel", False), ("add_norm_backward_ragged_kernel", True)):
        assert have(kernel) == {(t, w, str(v), str(n)) for v, n, r in back if r == ragged for t in T[v] for w in weights(t)}
    assert have("swiglu_quant_kernel") == {(t, str(v), str(n)) for v, n in swiglu for t in T[v]}
