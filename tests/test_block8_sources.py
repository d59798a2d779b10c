"""Sources of the 8-bit block operators (no GPU): barriers that a warp has to reach as one are reached as one.

PTX leaves an `.aligned` barrier (bar.sync is one) undefined for a warp whose lanes are apart, and a compiler may leave them apart behind loops of
unlike lengths or a branch of one lane.  Nothing that runs shows it reliably, so the sources are looked at."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_08524_b200", "csrc")
FILES = [p for name in ("d3_block8*", "d3_mm8_*", "d3_logits*") for p in sorted(glob.glob(os.path.join(CSRC, name)))]


def without_comments(text):
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_warps_come_together_in_front_of_barriers():
    found = 0
    for path in FILES:
        text = without_comments(open(path).read())
        for m in re.finditer(r'asm volatile\("(bar\.sync|barrier\.cluster\.(arrive|wait))', text):
            found += 1
            line = text.count("\n", 0, m.start()) + 1
            assert text[: m.start()].rstrip().endswith("__syncwarp();"), f"{os.path.basename(path)}, line {line} without comments: {m.group(1)}"
    assert len(FILES) >= 5 and found >= 3


def test_warps_come_together_in_front_of_waits_for_tensor_memory():
    """Between what one lane does alone and a tcgen05 load or the wait for it stands a __syncwarp."""
    found = 0
    for path in FILES:
        text = without_comments(open(path).read())
        for m in re.finditer(r"\btc_ld(_wait)?\(", text):
            before = text[: m.start()]
            if re.search(r"void\s*$", before):                 # its definition
                continue
            apart = max((x.end() for x in re.finditer(r"if \(lane == 0\)", before)), default=-1)
            started = max((x.end() for x in re.finditer(r"__global__|\[&\]\(\)", before)), default=-1)
            if apart > started:
                found += 1
                assert "__syncwarp();" in before[apart:], f"{os.path.basename(path)}: {before[apart:][-200:]}"
    assert found >= 2
