"""After a wait of pldp_attend_prompt's kernel has run out its warps leave their loops.  That a warp leaves is decided by a vote:
lanes that each looked for themselves could decide differently, and those that went on would wait for the others at the next
instruction that takes a whole warp.  (No run shows it but one that hangs, so the source is read.)"""
import os
import re

from paper_2412_01447_gb300 import _build


def _source(name):
    text = open(os.path.join(_build.CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def test_leaving_is_voted_on():
    text = _source("pldp_prompt.cuh")
    looks = [line.strip() for line in text.splitlines() if "dead" in line and not re.search(r"wait_(for|more)\(.*&sh\.dead\)", line)]
    vote = "auto given_up = [&] { return __any_sync(0xFFFFFFFFu, *static_cast<volatile int*>(&sh.dead)); };"
    assert vote in looks
    for line in looks:
        assert line in (vote, "int dead, zeros;", "sh.dead = 0;",
                        "*static_cast<volatile int*>(&sh.dead) = 1;",
                        "if (sh.dead && a.status)"), line
    # the last look, for the status, is behind every loop and has no vote behind it but the CTA's barrier
    tail = text[text.index("if (sh.dead && a.status)"):]
    assert not re.search(r"__(any|all|ballot|shfl\w*|reduce\w*)_sync|__syncwarp|tmem_(load|store)", tail[: tail.index("__syncthreads")])
