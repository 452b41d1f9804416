"""Roles of the many-query kernel in which a warp's lanes go on together after a
wait.  Lanes that gave up one by one would leave the others at a warp barrier, or
in an instruction of the whole warp, for good: the wait has to give the warp one
answer.  On the GPU its lanes run out of time together as a rule, so the sources
are read here."""

import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_14782_gb300", "csrc")


def body(name, path="cache_prompt.cu"):
    with open(os.path.join(CSRC, path)) as f:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    at = code.index("{", re.search(rf"__forceinline__ \w+ {name}\(", code).end())
    depth = 0
    for i in range(at, len(code)):
        depth += {"{": 1, "}": -1}.get(code[i], 0)
        if depth == 0:
            return code[at:i + 1]


@pytest.mark.parametrize("role", ["load", "convert_keys", "convert_values"])
def test_waits_of_a_warp_give_one_answer(role):
    code = body(role)
    assert "__syncwarp" in code
    assert len(re.findall(r"\bwait_all\(", code)) >= 2
    assert not re.findall(r"\bwait\(", code)
    # what a lane waits for alone decides nothing
    for line in re.findall(r"[^\n;{}]*\bmbar_wait\([^\n;]*", code):
        assert re.match(r"\s*(if \([\w +]+\) )?mbar_wait\(", line), line


def test_the_answer_is_a_vote():
    assert re.search(r"return __all_sync\(0xFFFFFFFFu, wait\(", body("wait_all"))


def test_the_few_query_kernels_loading_warp_votes():
    with open(os.path.join(CSRC, "cache_attend.cu")) as f:
        code = f.read()
    gone = code[code.index("auto gone ="):]
    assert "return !__all_sync(0xFFFFFFFFu, there);" in gone[:gone.index("};")]
    load = gone[:gone.index("// ---------------------------------------------------------- products")]
    assert len(re.findall(r"if \(gone\(", load)) == 2
