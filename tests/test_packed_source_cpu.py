"""What a GPU run of the packed forward cannot be relied on to show, because it holds by chance, is read in its source."""
import os
import re

from paper_2507_01652_b200 import build


def body(name, of):
    """The text of a function, by its braces."""
    at = of.index("{", re.search(r"\b%s\(" % name, of).end())
    depth, i = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(of[i], 0)
        i += 1
        if depth == 0:
            return of[at:i]


def test_a_second_store_of_p_waits_for_the_first():
    """tcgen05.st is asynchronous: two stores to the same columns are ordered by a wait between them only.  Where a row's
    maximum moves, P is formed and stored again."""
    with open(os.path.join(build.CSRC, "lasad_packed_tc.cu")) as f:
        text = body("softmax_rows", f.read())
    stores = [m.start() for m in re.finditer(r"\bexponentials\(", text)]
    assert len(stores) == 2
    assert "tmem_wait_st();" in text[stores[0]:stores[1]]
    assert "tmem_wait_st();" in text[stores[1]:]                       # and the products start after the last
