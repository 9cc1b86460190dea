"""Rules of the device code that no run can show to be broken without a hang or a wrong read: checked on the sources."""
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2601_12347_b200", "csrc")


def source(name):
    """A source without its comments and strings of assembly."""
    text = open(os.path.join(CSRC, name)).read()
    text = re.sub(r"//[^\n]*", "", text)
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return re.sub(r'"(?:[^"\\\n]|\\.)*"', '""', text)


def heads_around(text, at):
    """What stands in front of every brace that is open at a position, the innermost last."""
    heads, last = [], 0
    for i, c in enumerate(text[:at]):
        if c == "{":
            heads.append(text[last:i].strip())
        elif c == "}":
            heads.pop()
        if c in "{};":
            last = i + 1
    return heads


@pytest.mark.parametrize("name", ["row_project.cu", "layer_update_tc.cu"])
def test_lanes_of_a_warp_give_up_together(name):
    """A wait that runs out for some lanes of a warp only leaves them at another barrier than the rest, for good: what polls
    for itself is the role of one thread, and a warp that waits has one verdict."""
    text = source(name)
    alone = [m.start() for m in re.finditer(r"\bmbar_wait_bounded\s*\(", text)]
    assert alone and re.search(r"\bmbar_wait_warp\s*\(", text)
    for at in alone:
        assert any(re.search(r"\blead\b|\blane == 0\b", h) for h in heads_around(text, at)), text[max(0, at - 200):at + 60]


@pytest.mark.parametrize("name", ["row_project.cu", "row_norms.cu", "requests.cuh"])
def test_only_the_bank_is_read_past_coherence(name):
    """Kernels start while the one before still runs: what that one may write (rows, t, a plan) is read by ordinary loads, or out of L2;
    never as memory that stays as it is."""
    text = source(name)
    assert not re.search(r"__restrict__|ld\.global\.nc", open(os.path.join(CSRC, name)).read())
    for m in re.finditer(r"\b__ldg\s*\(", text):
        assert any(re.search(r"\bbank_word\b", h) for h in heads_around(text, m.start())), text[m.start() - 100:m.end() + 60]
    for m in re.finditer(r"\bbank(?:_word|8)\s*\(([^;]*);", text):
        assert not re.search(r"\bp\.(t|x|y|base|plan|plain|bias|ids|slots)\b|\bat\[", m.group(1)), m.group(0)
