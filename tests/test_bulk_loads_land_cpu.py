"""A block must not end while copies into its shared memory, or products into its tensor memory, are on their way: whoever asks for them waits
for them before the block's end, whether or not a wait of the block has run out before.  The roles of the kernels are read, as source."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2503_06671_b200" / "csrc"
ROLE = re.compile(r"\n    (?:if|\} else if) \((?=[^\n]*\bwarp\b)[^\n]*\{\n")   # a branch on the warp, at the kernel's own level


def roles(name):
    """The kernel's branches on the warp, without the setup in front of them."""
    text = (CSRC / name).read_text()
    text = text[text.index("bool alive = true;"):]
    text = text[:text.index("\n}\n")]
    cuts = [m.start() for m in ROLE.finditer(text)]
    end = text.index("\n    pdl_launch_dependents();", cuts[-2])
    return [text[a:b] for a, b in zip(cuts, [c for c in cuts[1:] if c < end] + [end])]


def tail(role):
    """What a role does once it is through, or has given up."""
    return "\n".join(role.splitlines()[-6:])


@pytest.mark.parametrize("name,loaders", [("linear_umma.cuh", 2), ("linear_backward_small.cuh", 1)])
def test_loads_and_products_end_before_the_block(name, loaders):
    parts = roles(name)
    assert len(parts) >= 4
    ring = [p for p in parts if "tma_load_2d(" in p]
    assert len(ring) == loaders
    for part in ring:
        end = tail(part)
        assert re.search(r"landed\(full, p\.stages, \w+(\.r)?\);", end), "the ring's loads"
        assert re.search(r"wait_lane\((b|w)_full, 0,", end), "the operand that stays"
        assert "alive" not in end, "it may be another role that has given up"
    issue = [p for p in parts if re.search(r"\bmma\(", p)]
    assert len(issue) == 1 and "finish(finished);" in tail(issue[0])
    for part in parts:
        if "tma_load_3d(" in part:                                        # a residual: asked for one unit ahead
            assert re.search(r"!alive && lane == 0\) wait_lane\(res_bar, units & 1,", tail(part))
        if "tma_store_3d(" in part:
            assert "bulk_wait_read<0>()" in tail(part)
