"""No forward of a linear begins beside the kernel before it, which may be writing its input: held by the host's code, as no call shows it."""
import os
import re

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2305_14152_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_few_tokens():
    text = source("split_sm100.cu")
    launch = text[text.index("int launch_split(const"):]
    sides = re.findall(r"\bp\.side = ([^;]+);", launch)
    # the call's own, without kBeside for a forward, and the two launches of a gated block, of which the first waits
    assert sides == ["!trans && side == kBeside ? kInOrder : side", "kFollowed", "kBeside"]
    at = [launch.index(part) for part in ("plan_glu(", "p.side = kFollowed", "PEQA_TRY(launch(cut.head))", "p.side = kBeside", "return launch(cut.rest)")]
    assert at == sorted(at)
    assert "p.side" not in text[text.index("size_t fit_split"):text.index("int launch_split(const")]


def test_many_tokens():
    text = source("fwd_pair_sm100.cu")
    kernel = text[text.index("qfwd_pair_kernel("):]
    assert "kBeside" not in text and kernel.index("griddepcontrol.wait") < kernel.index("warp == 0")
