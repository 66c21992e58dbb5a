"""The set-up of mbarriers in the kernels' sources (nothing is compiled or launched).

fence.mbarrier_init orders the executing thread's own earlier mbarrier.init before other
accesses, those of TMA among them; a barrier that another thread has set up is not covered
by it.  So each kernel sets its barriers up and fences them in the same branch of one thread."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_04895_gb300", "csrc")


def code(path):
    text = open(path).read()
    text = re.sub(r"/\*.*?\*/", lambda m: " " * len(m.group()), text, flags=re.S)
    return re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), text)


def blocks(text):
    """(first, last) of every pair of braces."""
    open_, out = [], []
    for i, c in enumerate(text):
        if c == "{":
            open_.append(i)
        elif c == "}":
            out.append((open_.pop(), i))
    return out


def setups(path):
    """For each mbar_init of a file: the head of the innermost block that also fences behind it."""
    text = code(path)
    pairs = blocks(text)
    for m in re.finditer(r"\bmbar_init\(", text):
        if re.search(r"void\s+$", text[:m.start()]):     # the definition
            continue
        around = [b for b in pairs if b[0] < m.start() < b[1]
                  and "fence_mbar_init()" in text[m.start():b[1]]]
        if not around:
            yield None
            continue
        first = max(around)[0]
        head = text[:first].rstrip()
        yield head[max(head.rfind(c) for c in ";{}") + 1:].strip()


# (probe.cu's kernel goes on with one thread alone, before any barrier)
FILES = [f for pat in ("*.cu", "*.cuh") for f in sorted(glob.glob(os.path.join(CSRC, pat)))
         if "mbar_init(" in code(f) and os.path.basename(f) != "probe.cu"]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_one_thread_sets_barriers_up_and_fences_them(path):
    for head in setups(path):
        assert head and re.fullmatch(r"if \((?:threadIdx\.x|team\.thread|lane) == 0\)", head), head


def test_files_are_found():
    assert any(f.endswith("matvec4.cu") for f in FILES) and len(FILES) > 5
