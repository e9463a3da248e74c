"""What no result of a kernel shows, checked in the kernels' source: barriers that have to stand before an access
and the alignment of what is accessed by wider words."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2108_02416_gb300", "csrc")


def kernels():
    """(file, name, text) of every kernel, without comments."""
    out = []
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for part in re.split(r"(?m)^__global__", src)[1:]:
            part = part[: part.index("\n}") + 2]
            out.append((name, re.search(r"(\w+_kernel)\s*\(", part).group(1), part))
    return out


KERNELS = kernels()
REMOTE = re.compile(r"map_shared_rank|\b\w+_peer\(|\bpeer\(")


def test_kernels_are_found():
    names = {k[1] for k in KERNELS}
    assert {"hold_kernel", "few_kernel", "scatter_kernel", "detect_wide_kernel"} <= names


@pytest.mark.parametrize("file,name,text", [k for k in KERNELS if REMOTE.search(k[2])], ids=lambda x: x if "_kernel" in x and len(x) < 40 else "")
def test_blocks_of_a_cluster_have_begun_before_their_memory_is_touched(file, name, text):
    """A block's shared memory is there for the others only once it has begun, which being scheduled together does not
    say: a barrier of the cluster does."""
    before = text[: REMOTE.search(text).start()]
    arrived, waited = before.find("cluster_begin()"), before.find("cluster_begun()")
    assert 0 <= arrived < waited or "cluster_sync_all()" in before or "cluster.sync()" in before


@pytest.mark.parametrize("file,name,text", KERNELS, ids=[f"{k[0]}-{k[1]}" for k in KERNELS])
def test_shared_arrays_read_by_wider_words_are_aligned(file, name, text):
    """An array of 16-bit or 8-bit elements in shared memory is aligned to its element alone unless it says more."""
    for line in re.findall(r"__shared__[^;]*\buint(?:8|16)_t[^;]*;", text):
        aligned = re.search(r"__align__\((\d+)\)", line)
        for array in re.findall(r"(\w+)(?:\[[^\]]*\])+", line):
            for wide in re.findall(r"reinterpret_cast<(?:const )?(\w+) \*>\(\s*&?" + array + r"\b", text):
                need = {"uint32_t": 4, "uint2": 8, "uint4": 16, "float4": 16}[wide]
                assert aligned and int(aligned.group(1)) >= need, (array, wide)
