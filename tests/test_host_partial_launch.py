"""The partial launch of the decode kernel (a shared decode's own keys) starts beside the kernel ahead of it, and the merge
behind it relies on its end for that kernel's end too: every way out of the device code waits for it.  Read from the
source, since the way out that matters is the one after a wait that ran out of time."""
import os
import re

from paper_2409_15012_b200 import build as mbuild

WAIT = re.compile(r'if \(CL == 1 && p\.partial\) asm volatile\("griddepcontrol\.wait;" ::: "memory"\);')


def ways_out():
    """(text in front of it in its block, conditions of the blocks around it) of every return of the kernel and of its end."""
    with open(os.path.join(mbuild.CSRC, "decode_bf16.cu")) as f:
        text = f.read()
    text = re.sub(r"//[^\n]*", "", text)
    begin = text.index("{", text.index("decode_split_bf16_kernel("))
    found, opened = [], []
    for at in range(begin, len(text)):
        if text[at] == "{":
            opened.append(at)
        elif text[at] == "}":
            first = opened.pop()
            if not opened:
                found.append((text[first:at].strip(), []))
                return found
        elif text.startswith("return;", at):
            around = [re.split(r"[;{}]", text[:o].strip())[-1] for o in opened]
            found.append((text[opened[-1]:at].strip(), around))


def test_every_way_out_of_a_partial_launch_waits():
    ways = ways_out()
    assert len(ways) >= 3
    for before, around in ways:
        paired = any("if constexpr (CL > 1)" in a for a in around)      # (clusters are never partial)
        last = before.rsplit("\n", 1)[-1].strip()
        assert paired or WAIT.fullmatch(last), before[-200:]


def test_clusters_are_never_partial():
    with open(os.path.join(mbuild.CSRC, "decode_bf16.cu")) as f:
        text = f.read()
    assert re.search(r"const bool paired = !p\.partial &&", text) and re.search(r"const int cl = paired \? 2 : 1;", text)
