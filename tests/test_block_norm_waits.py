"""Rows that come by DMA into LDS are read behind a wait that takes them by itself.

The compiler does not know of the DMA's loads (they are written in assembly), so nothing but the kernel's own
wait keeps a read of LDS behind them.  A wait that lets n newer operations pass is right only where n of
them are issued behind the DMA in every form of the norm, at every depth of the ring and in the first round
too; there are as few as two (a norm's two statistics), and none of them need be a store.
"""
import os
import re

from paper_2606_19025_amd import build


def kernels():
    """(name, body) of the kernels of block_norm.hip that fetch rows by DMA."""
    with open(os.path.join(build.CSRC, "block_norm.hip")) as f:
        text = f.read()
    parts = re.split(r"__global__ [^\n]*\bvoid (\w+)\(", text)
    return [(n, b) for n, b in zip(parts[1::2], parts[2::2]) if "fetch(" in b]


def test_row_kernels_wait_for_all_of_their_rows():
    found = kernels()
    assert {n for n, _ in found} == {"block_norm_fwd_kernel", "block_norm_bwd_kernel"}
    for name, body in found:
        loop = body[body.index("for (int t0 = first"):]
        waits = [(m.start(), m.group(1)) for m in re.finditer(r"s_waitcnt vmcnt\(([^)]*)\)", loop)]
        assert waits and all(n == "0" for _, n in waits), (name, waits)
        # and it comes ahead of what a round reads and fetches, under no condition
        first = min(loop.index("read(src"), loop.index("fetch("))
        line = loop[loop.rindex("\n", 0, waits[0][0]):waits[0][0]]
        assert waits[0][0] < first and not re.search(r"\b(if|else)\b", line), name
