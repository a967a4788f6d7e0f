"""mmasim_matvec4.cu as it is written: orders between the lanes of a warp that no output can be relied on to show."""
import os
import re

from paper_2511_10909_b200.build import CSRC


def body(text, head):
    """The braces behind `head`."""
    start = text.index("{", text.index(head))
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if not depth:
            return text[start:i + 1]


def test_a_stage_is_read_by_all_lanes_before_it_is_filled_again():
    """A lane reads scale codes that another lane copied, so both ways the lanes have to meet: between the copies' end and the reads (await),
    and between the reads and the next copies into that stage (in front of fetch, which fills what the step before has read)."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "mmasim_matvec4.cu")).read())
    wait = body(text, "void await() const")
    assert wait.rindex("__syncwarp();") > wait.rindex("cp.async.wait_group")
    steps = body(text, "template <bool GENERAL> __device__ __forceinline__ void run()")
    loop = body(steps, "while (now.done < tiles)")
    assert re.match(r"\{\s*__syncwarp\(\);\s*fetch<GENERAL>\(\);\s*await\(\);", loop)
    assert loop.count("fetch<GENERAL>()") == 1 and text.count("__syncwarp();") == 2
