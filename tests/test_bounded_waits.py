"""Kernels with roles for warps (one asks for tiles, one multiplies, the others use the products): whichever of them gives up a wait, copies and
products on their way are waited for before the CTA's memory is used for something else or the CTA ends.  Giving up cannot be brought
about without breaking a kernel, so this is read from the sources: the last waits hang on no warp's own success."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2502_07861_b200", "csrc")
KERNELS = [("kernels_attn_tc.cu", "attn_tc_kernel"), ("kernels_score_tc.cu", "score_tc_kernel"), ("kernels_score_tc.cu", "score_stream_kernel")]


def _body(file, name):
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = text.index("{", text.index(name + "("))
    depth, end = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[at:end]


def _conditions(body, at):
    """What the blocks and the statement that hold body[at] hang on."""
    heads, start = [], 0
    for i, c in enumerate(body[:at]):
        if c == "{":
            heads.append(body[start:i])
        elif c == "}":
            heads.pop()
        if c in "{};":
            start = i + 1
    return [*heads, body[start:at]]


@pytest.mark.parametrize("file,name", KERNELS)
@pytest.mark.parametrize("call", ["copy_landed(&", "copies_landed(", "products_done("])
def test_the_last_waits_are_everybodys(file, name, call):
    body = _body(file, name)
    places = [_conditions(body, m.start()) for m in re.finditer(re.escape(call), body)]
    free = [c for c in places if not any(re.search(r"\bok\b|abort|\bi < n\b", head) for head in c if "for (" not in head and "while (" not in head)]
    assert free, (name, call, places)
    assert all("n > 0" in " ".join(c) for c in free)       # and no CTA waits for what it never asked for


def test_results_do_not_take_the_place_of_query_tiles_on_their_way():
    body = _body("kernels_attn_tc.cu", "attn_tc_kernel")
    gave_up = re.search(r"if \(!ok\) \{\s*l = NAN;\s*copy_landed\(&q_full\);", body)
    assert gave_up and gave_up.start() < body.index("stage")
