"""The digest that says whether a captured figure still belongs to the GEMM kernel covers all of the kernel's source."""
import os
import re
import shutil

import pytest

import bench
from paper_2607_19539_b200 import build


def headers_behind(name):
    """Every project header that a file includes, directly or not."""
    found = set()
    with open(os.path.join(build.CSRC, name)) as f:
        for h in re.findall(r'#\s*include\s+"([^"]+)"', f.read()):
            found |= {h} | headers_behind(h)
    return found


def test_the_kernel_has_headers():
    assert {"ptx.cuh", "common.cuh", "mover.cuh"} <= headers_behind("producer.cuh")


@pytest.fixture
def copy(tmp_path, monkeypatch):
    """The kernels' source once more, where it can be changed, and the digest before the change."""
    before = bench.kernel_sha1()
    csrc = tmp_path / os.path.relpath(build.CSRC, bench.ROOT)
    shutil.copytree(build.CSRC, csrc)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_sha1() == before
    return csrc, before


@pytest.mark.parametrize("name", sorted(headers_behind("producer.cuh") | {"producer.cuh"}))
def test_digest_follows_every_header(copy, name):
    csrc, before = copy
    with open(csrc / name, "a") as f:
        f.write("\n// changed\n")
    assert bench.kernel_sha1() != before


def test_digest_does_not_follow_other_kernels(copy):
    csrc, before = copy
    with open(csrc / "rowops.cu", "a") as f:
        f.write("\n// changed\n")
    assert bench.kernel_sha1() == before
