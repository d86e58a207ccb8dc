"""tcgen05.alloc waits without a limit, so the order of allocation, dependency wait and early start of the next kernel decides whether
two kernels of a stream can wait for each other: checked in the kernels' sources."""
import os
import re

import pytest

from paper_2502_20727_b200 import build as spd_build

STEPS = {"signal": "pdl_launch_dependents()", "alloc": "tcgen05.alloc.", "wait": "pdl_wait()"}


def kernels():
    """(file, kernel, first position of every step in its body) of the kernels that allocate tensor memory."""
    found = []
    for path in spd_build.sources():
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__", text):
            name = re.compile(r"(\w+_kernel)\(").search(text, m.end())
            at = text.index("{", text.index(")", text.index("(", name.end() - 1)))
            depth, end = 0, at
            while True:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
                if not depth:
                    break
            body = text[at:end]
            if STEPS["alloc"] in body:
                found.append((os.path.basename(path), name.group(1), {k: body.find(s) for k, s in STEPS.items()}))
    return found


def test_the_kernels_are_found():
    assert len(kernels()) >= 5


@pytest.mark.parametrize("file,kernel,at", kernels())
def test_columns_are_owned_before_the_next_kernel_may_take_them(file, kernel, at):
    """The next kernel may allocate before its own wait and holds the columns until this one has ended.  It starts once every block of
    this one has signalled: a block that then still waits for its predecessor, and allocates after that, can be left without."""
    assert min(at.values()) >= 0
    if at["wait"] < at["alloc"]:
        assert at["alloc"] < at["signal"], f"{file}: {kernel} lets the next kernel start before it owns its tensor memory"


@pytest.mark.parametrize("path", spd_build.sources())
def test_a_warp_takes_one_way_past_the_abort_flag(path):
    """Any warp may raise the flag at any time, so lanes that read it for themselves can differ: where a warp-wide instruction
    (tcgen05.commit by an elected lane) hangs on it, the warp has to have one answer."""
    for m in re.finditer(r"if \(([^{;]*\babort_flag\b[^{;]*)\) \{([^}]*)\}", re.sub(r"//[^\n]*", "", open(path).read())):
        if re.search(r"\bcommit\(|elect\.sync", m.group(2)):
            assert re.search(r"__(any|all)_sync\(0xffffffffu, \*abort_flag\)", m.group(1)), m.group(0)
