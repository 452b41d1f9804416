"""Shared memory that the cache's attention writes by ordinary stores and by
asynchronous copies in turn.  The memory model orders a thread's stores before
its later copies to the same bytes only by a proxy fence; on the GPU the
barriers between them hide a missing one, so the sources are read here.  The
bytes are the query rows of the few-query kernel: cleared by ordinary stores
where an item has no query, filled by copies where the next one has."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_14782_gb300", "csrc")


def loading_warp():
    with open(os.path.join(CSRC, "cache_attend.cu")) as f:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    start = code.index("if (warp == kWarps) {")
    depth, i = 0, start
    while True:
        depth += {"{": 1, "}": -1}.get(code[i], 0)
        i += 1
        if depth == 0 and code[i - 1] == "}":
            return code[start:i]


def test_cleared_query_rows_are_fenced_before_copies_may_fill_them():
    code = loading_warp()
    stores = [m.start() for m in re.finditer(r"\*reinterpret_cast<uint4\*>\(smem \+ row", code)]
    copies = [m.start() for m in re.finditer(r"\bload_bytes\(base \+ row", code)]
    assert len(stores) == 1 and len(copies) == 1  # what this test knows of
    published = code.index("mbar_arrive(full)", stores[0])
    assert "fence_proxy_async_smem();" in code[stores[0]:published]
