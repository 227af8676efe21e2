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
    """(start, end, header, before) of every brace block; the header is what stands between the last ; { } (at `before`) and the opening brace"""
    stack, out = [], []
    for i, c in enumerate(text):
        if c == "{":
            at, depth = i - 1, 0
            while at >= 0 and (depth or text[at] not in ";{}"):   # (a ; inside the parentheses of a for does not end it)
                depth += {")": 1, "(": -1}.get(text[at], 0)
                at -= 1
            stack.append((i, " ".join(text[at + 1:i].split()), at))
        elif c == "}":
            start, header, before = stack.pop()
            out.append((start, i, header, before))
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
        start, end = max(around)[:2]
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


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.startswith("rglru_sm100")))
def test_tensor_memory_is_read_by_whole_warps(name):
    assert reached_apart(source(name)) == []


def conditions(text, at):
    """The conditions on `warp` under which the code at `at` runs: of its own branch, and the negated ones of the branches before it"""
    out, all_blocks = [], blocks(text)
    for start, end, header, before in all_blocks:
        if not start < at < end:
            continue
        chain = []   # this branch's and those of the branches before it
        while (m := re.fullmatch(r"(else )?if \((.*)\)|(else)", header)):
            chain.append(m.group(2) or "True")
            if not (m.group(1) or m.group(3)):
                break
            start, _, header, before = next(b for b in all_blocks if b[1] == before)
        if "warp" in " ".join(chain):
            out.append(chain)
    return out


def warps_that_run(text, at, names, warps):
    ran = []
    for w in range(warps):
        value = dict(names, warp=w, true=True)
        if all(eval(c[0], {}, value) and not any(eval(e, {}, value) for e in c[1:]) for c in conditions(text, at)):
            ran.append(w)
    return ran


def test_register_budgets_are_set_by_whole_warpgroups():
    """setmaxnreg: all warps of a warpgroup execute the same one"""
    text = source("rglru_sm100_linattn.cu")
    names = {}
    for m in re.finditer(r"constexpr int ([^;]*);", text):
        for part in m.group(1).split(","):
            name, value = part.split("=")
            try:
                names[name.strip()] = eval(value, {}, names)
            except (NameError, SyntaxError):
                pass
    warps, seen = names["THREADS"] // 32, []
    for m in re.finditer(r"\breg_(?:dec|inc)<", text):
        ran = warps_that_run(text, m.start(), names, warps)
        assert ran and len(ran) % 4 == 0 and all(ran[i] == ran[0] + i for i in range(len(ran))) and ran[0] % 4 == 0, (text[:m.start()].count("\n") + 1, ran)
        seen += ran
    assert sorted(seen) == list(range(warps))


@pytest.mark.parametrize("name", ["rglru_norm.cu", "rglru_linear.cu", "rglru_linattn.cu", "rglru_sm100_linear.cu", "rglru_sm100_linattn.cu"])
def test_shared_arrays_that_are_read_16_bytes_at_a_time_are_aligned(name):
    """A shared array of floats starts at a multiple of four bytes unless it says more"""
    text = source(name)
    assert [m.group() for m in re.finditer(r"__shared__ float \w+", text)] == []
