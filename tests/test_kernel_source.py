"""What PTX leaves undefined and no result shows: instructions for whole warps or warpgroups (.sync.aligned) have to be reached by all of
their lanes together.  Read off the kernels' source, since a run only shows what one compiler made of it."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_19427_b200", "csrc")
TMEM = re.compile(r"\btmem_(?:ld|st)\d+\w*\(")
TOGETHER = re.compile(r"__syncwarp\(\)|__(?:all|any)_sync\(|\bwarp_wait\w*\(|\bwait_acc\(\)|__syncthreads\(\)")
# control flow in which lanes part: rows, tokens and channels that do not exist, and the functions that store under such conditions
PARTS = re.compile(r"if \(!?(?:there|valid|cv|exists|mine\.in|tb \+ k < T && cv|b < B && exists|m >= p\.M)\b|\bfinish\(|\bwalk_segment<")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", lambda m: re.sub(r"[^\n]", " ", m.group()), text, flags=re.S)


def blocks(text):
    """(start, end, header) of every brace block; the header is what stands between the last ; { } and the opening brace"""
    stack, out = [], []
    for i, c in enumerate(text):
        if c == "{":
            at, depth = i - 1, 0
            while at >= 0 and (depth or text[at] not in ";{}"):   # (a ; inside the parentheses of a for does not end it)
                depth += {")": 1, "(": -1}.get(text[at], 0)
                at -= 1
            stack.append((i, " ".join(text[at + 1:i].split())))
        elif c == "}":
            start, header = stack.pop()
            out.append((start, i, header))
    return out


def is_loop(header):
    return re.search(r"(?:^|\s)(?:for|while) ?\(", header) is not None


def reached_apart(text):
    """Lines of accesses to tensor memory inside a loop that follow, with nothing that brings the warp together in between, a place where its lanes part"""
    found, all_blocks = [], blocks(text)
    for m in TMEM.finditer(text):
        around = [b for b in all_blocks if b[0] < m.start() < b[1] and is_loop(b[2])]
        if not around:
            continue
        start, end, _ = max(around)
        before = text[m.end():end] + text[start:m.start()]   # what ran since this access, once around the loop
        apart = [p.end() for p in PARTS.finditer(before)]
        together = [p.start() for p in TOGETHER.finditer(before)]
        if apart and not (together and together[-1] > apart[-1]):
            found.append(text[:m.start()].count("\n") + 1)
    return found


def test_the_reader_sees_what_it_should():
    loop = "for (int c = 0; c < n; ++c) {\n tmem_ld16(a + c, x);\n if (there) {\n *p = x[0];\n }\n%s}\n"
    assert reached_apart(loop % "") == [2] and reached_apart(loop % "__syncwarp();\n") == []
    assert reached_apart("for (;;) { tmem_ld16(a, x); if (last) f(); }") == []


@pytest.mark.parametrize("name", ["rglru_sm100_linattn.cu"])
def test_tensor_memory_is_read_by_whole_warps(name):
    assert reached_apart(source(name)) == []
