"""What lanes of one wavefront hand each other through shared memory, read in the compiler's own form of the kernels: between a word's store and
its load by another lane, and between that load and the next store, stands something that the compiler moves no access across. Without it the
order holds only as long as the compiler cannot tell the two addresses apart, which no run shows."""
import os
import re
import subprocess

import pytest

from paper_2411_01830_amd import build

# arrays that lanes of a wavefront share without a barrier of the workgroup, by the kernel whose they are
SHARED = {
    "ft_linear4.hip": {"ft_linear4_narrow_kernel": ["codes_lds", "x_lds"], "ft_linear4_wide_kernel": ["codes_lds"]},
    "ft_verify.hip": {"ft_verify_kernel": ["chunk"]},
}
_cache = {}


def code(tmp_path_factory, source):
    if source not in _cache:
        out = tmp_path_factory.mktemp("code") / (source + ".ll")
        subprocess.run([build.hipcc(), "-x", "hip", *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, source), "-o", str(out)],
                       check=True, capture_output=True)
        _cache[source] = out.read_text()
    return _cache[source]


def kernels(text):
    """(name, blocks) of every kernel: a block is its label, its lines and the labels that it goes on to."""
    for m in re.finditer(r"^define [^\n]*amdgpu_kernel[^\n]*@(\S+?)\([^\n]*\{\n(.*?)^\}", text, re.S | re.M):
        blocks, label, lines = [], "entry", []
        for line in m.group(2).split("\n"):
            head = re.match(r"^([\w.$\"-]+):", line)
            if head:
                blocks.append((label, lines))
                label, lines = head.group(1), []
            elif line.strip():
                lines.append(line.strip())
        blocks.append((label, lines))
        yield m.group(1), [(b, l, re.findall(r"label %([\w.$\"-]+)", "\n".join(l))) for b, l in blocks if l]


def out_of_order(name, blocks, array):
    """Accesses of the array that nothing keeps behind those of another kind before them."""
    names = {m for _, lines, _ in blocks for line in lines for m in re.findall(r"@[\w.$]+", line) if re.search(rf"\d{array}$", m)}
    assert names, (name, array)
    derived = set(names)
    grown = True
    while grown:                                             # pointers that come of the array's
        grown = False
        for _, lines, _ in blocks:
            for line in lines:
                m = re.match(r"(%[\w.]+) = (getelementptr|phi ptr|select|bitcast|addrspacecast)\b(.*)", line)
                if m and m.group(1) not in derived and any(re.search(re.escape(d) + r"(?![\w.$])", m.group(3)) for d in derived):
                    derived.add(m.group(1))
                    grown = True

    def kind(line):
        if line.startswith("fence ") or re.search(r"asm sideeffect [^\n]*~\{memory\}", line):
            return "fence"
        m = re.match(r"store .* ptr addrspace\(3\) ([%@][\w.$]+|getelementptr .*?)(, align|$)", line) or \
            re.match(r"%[\w.]+ = load .* ptr addrspace\(3\) ([%@][\w.$]+|getelementptr .*?)(, align|$)", line)
        if m and any(re.search(re.escape(d) + r"(?![\w.$])", m.group(1)) for d in derived):
            return "store" if line.startswith("store") else "load"
        return None

    steps = {b: [k for k in map(kind, lines) if k] for b, lines, _ in blocks}
    assert {"store", "load"} <= {k for s in steps.values() for k in s}, (name, array)
    before = {b: set() for b, _, _ in blocks}                # what may have been since the last fence where a block begins
    bad, changed = set(), True
    while changed:
        changed = False
        for b, _, on in blocks:
            since = set(before[b])
            for i, k in enumerate(steps[b]):
                if k == "fence":
                    since = set()
                else:
                    if {"store": "load", "load": "store"}[k] in since:
                        bad.add((b, i, k))
                    since.add(k)
            for t in on:
                if not since <= before[t]:
                    before[t] |= since
                    changed = True
    return bad


@pytest.mark.parametrize("source,kernel,array", [(s, k, a) for s, of in SHARED.items() for k, arrays in of.items() for a in arrays])
def test_lanes_that_share_words_are_kept_in_order(tmp_path_factory, source, kernel, array):
    seen = 0
    for name, blocks in kernels(code(tmp_path_factory, source)):
        if kernel in name:
            seen += 1
            bad = out_of_order(name, blocks, array)
            assert not bad, (name, array, sorted(bad)[:5])
    assert seen >= 3


def test_shared_memory_is_aligned_as_it_is_read(tmp_path_factory):
    """Scales and zeros are bytes to the compiler and are read in words of two and four."""
    arrays = re.findall(r"^(@\S*(?:scales|zeros)_lds\S*) = .*addrspace\(3\) global .* align (\d+)", code(tmp_path_factory, "ft_linear4.hip"), re.M)
    assert len(arrays) > 10
    assert [name for name, align in arrays if int(align) < 16] == []
