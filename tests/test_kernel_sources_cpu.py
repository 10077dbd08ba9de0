"""Rules that every kernel's source keeps, because breaking them shows on a device only now and then (no device here)."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2607_01844_b200" / "csrc"
SOURCES = sorted(p for p in CSRC.iterdir() if p.suffix in (".cuh", ".cu"))


def code(path):
    """The file without its comments."""
    text = re.sub(r"/\*.*?\*/", lambda m: "\n" * m.group().count("\n"), path.read_text(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def functions(path):
    """Bodies of the top-level functions: from a line that starts in the first column to the closing brace in the first column."""
    return re.findall(r"^(?:template|__global__|__device__|inline|static).*?^\}", code(path), flags=re.S | re.M)


@pytest.mark.parametrize("path", SOURCES, ids=lambda p: p.name)
def test_another_ctas_shared_memory_is_used_only_after_a_cluster_barrier(path):
    """A CTA of a cluster may be started after its peers: its shared memory is there only once a barrier of the cluster has been passed."""
    bodies = functions(path)
    remote = [r"mapa\."]
    for body in bodies:                 # helpers that map an address leave the barrier to the kernels that call them
        if "__global__" not in body and "mapa." in body and "cluster_sync_all()" not in body[:body.index("mapa.")]:
            remote.append(r"\b" + re.search(r"(\w+)\(", body[body.index("void") if "void" in body else 0:]).group(1) + r"\(")
    for body in bodies:
        if "__global__" in body:
            uses = [m.start() for r in remote for m in re.finditer(r, body)]
            assert not uses or "cluster_sync_all()" in body[:min(uses)], body[:160]


@pytest.mark.parametrize("path", SOURCES, ids=lambda p: p.name)
def test_nothing_is_read_through_the_read_only_path(path):
    """A kernel that programmatic launches bring up early lives while the one before it still writes, and a read-only load (__ldg, or a
    kernel's `const ... * __restrict__` parameter, which the compiler may turn into one) is defined only for memory that nobody writes
    in the reader's lifetime; nor does the compiler have to keep such a load behind the wait for the grid before."""
    text = code(path)
    assert "__ldg" not in text and "ld.global.nc" not in text and not re.search(r"const\s+\w+\s*\*\s*__restrict__", text)
