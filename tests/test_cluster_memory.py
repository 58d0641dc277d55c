"""Shared memory of another CTA of a cluster may be touched only once that CTA is known to have begun, that is, behind a barrier of the whole
cluster.  Read from the sources: no device."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2502_07861_b200", "csrc")


def _kernels(text):
    """Name and body of every kernel, comments taken out."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    for at in re.finditer(r"__global__", text):
        open_brace = text.index("{", at.end())
        name = next(n for n in re.findall(r"(\w+)\s*\(", text[at.end():open_brace]) if n.endswith("_kernel"))
        depth, end = 1, open_brace + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield name, text[open_brace:end]


def _unguarded(body):
    """Accesses that no barrier of the cluster comes before in a block that encloses them."""
    blocks, bad = [], []
    for token in re.finditer(r"[{}]|map_shared_rank|cluster\.sync\(\)|barrier_wait|sums_before", body):
        what = token.group()
        if what == "{":
            blocks.append(False)
        elif what == "}":
            blocks.pop()
        elif what == "map_shared_rank":
            if not any(blocks):
                bad.append(body[:token.start()].count("\n"))
        else:
            blocks[-1] = True
    return bad


def _clustered():
    for file in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, file)) as f:
            for name, body in _kernels(f.read()):
                if "map_shared_rank" in body:
                    yield file, name, body


def test_kernels_that_use_distributed_shared_memory_are_found():
    assert {"attn_few_cluster_kernel", "evict_select_kernel", "score_tc_kernel"} <= {name for _, name, _ in _clustered()}


@pytest.mark.parametrize("file,name,body", [pytest.param(*k, id=k[1]) for k in _clustered()])
def test_a_cluster_barrier_comes_first(file, name, body):
    assert not _unguarded(body), (file, name)


def test_an_access_behind_a_barrier_that_is_not_always_taken_is_found():
    assert _unguarded("{ if (a) { cluster.sync(); } cluster.map_shared_rank(p, 0); }")
    assert not _unguarded("{ if (a) { cluster.sync(); cluster.map_shared_rank(p, 0); } }")


@pytest.mark.parametrize("streams,rows,bf16,clusters", [
    (148, 120, 0, True), (74, 200, 0, True), (149, 120, 0, False), (200, 100, 0, False), (256, 60, 0, False), (80, 300, 0, False), (200, 100, 1, True), (256, 100, 1, True),
])
def test_clusters_serve_no_more_ctas_than_run_at_once(streams, rows, bf16, clusters):
    """One query of up to eight heads over rows of 128 dims: the clusters need no workspace, two launches do.  A CTA of fp32 rows has an SM to itself."""
    import ctypes as C

    import paper_2502_07861_b200 as bk

    size = C.c_size_t(0)
    assert bk.load().balancekv_attn_scored_workspace(streams, rows, 1, 4, 128, bf16, 1, C.byref(size)) == 0
    assert (size.value == 0) == clusters
