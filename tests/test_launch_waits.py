"""Programmatic dependent launches: a kernel is set up while the one before it still runs, so it must wait for that one before it
touches memory, every CTA of it.  What a kernel that releases its dependents early has written is promised to them only behind that
wait.  The sources are read; no GPU needed."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_1804_08066_b200" / "csrc"
AROUND_CODEC = ["mqg_clip.cu", "mqg_embedding.cu", "mqg_embedding_grad.cu", "mqg_token_sort.cu"]
KERNEL = re.compile(r"__global__\s+void\s*(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\s*\(")


def _bodies(source):
    for m in KERNEL.finditer(source):
        start = source.index("{", m.end())
        yield m.group(1), source[start:re.compile(r"^}", re.M).search(source, start).start()]


@pytest.mark.parametrize("path", sorted(CSRC.glob("*.cu*")), ids=lambda p: p.name)
def test_no_kernel_releases_its_dependents_before_it_ends(path):
    code = re.sub(r"//[^\n]*", "", path.read_text())
    assert "launch_dependents" not in code


@pytest.mark.parametrize("name", AROUND_CODEC)
def test_every_kernel_waits_under_no_condition(name):
    source = (CSRC / name).read_text()
    bodies = dict(_bodies(source))
    assert len(bodies) == source.count("__global__") > 0
    for kernel, body in bodies.items():
        assert re.search(r"^    grid_dependency_wait\(\);", body, re.M), kernel
        # before it, parameters only: no access to global memory
        before = body[:re.search(r"^ *grid_dependency_wait\(\);", body, re.M).start()]
        assert not re.search(r"__ld\w+\(|atomic\w+\(|\.load\(|\.store\(|\bmemcpy", before), kernel
