"""Static check of the machine code of the paged attention kernels: the waits for loads in the tile loop of few rows are those
that the source writes, one by one, and no kernel spills vector registers or moves sums into accumulation registers."""
import os
import re
import shutil
import subprocess
from collections import Counter

import pytest

from paper_2510_10129_amd import build
from test_isa_audit import HIPCC


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("isa_waits") / "paged.s"
    cmd = [HIPCC, *build.FLAGS, "-S", "--cuda-device-only", "-o", str(out), os.path.join(build.CSRC, "paged_attention.hip")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return re.findall(r"^(_ZN\S*(?:few|chunk)_attn_kernel\S*):[^\n]*\n(.*?)\.end_amdhsa_kernel", out.read_text(), flags=re.S | re.M)


def tile_loop(body):
    """The text of the basic blocks that can be reached from the first LDS read written by hand and reach it again without a barrier:
    between two blocks of columns there is one, so what is left is the loop over tiles."""
    blocks, at = [[]], {}
    for n, line in enumerate(body.split("\n")):
        label = re.match(r"(\.LBB\d+_\d+):", line)
        if label:
            blocks.append([])
            at[label.group(1)] = len(blocks) - 1
        blocks[-1].append(line)
        if re.match(r"\ts_(?:c?branch|endpgm|setpc)", line):
            blocks.append([])
    after, before = {}, {}
    for n, lines in enumerate(blocks):
        to, last = set(), next((l for l in reversed(lines) if l.startswith("\ts_")), "")
        if last.startswith("\ts_cbranch") or last.startswith("\ts_branch"):
            to.add(at[last.split()[1]])
        if not re.match(r"\ts_(?:branch|endpgm|setpc)", last) and n + 1 < len(blocks):
            to.add(n + 1)
        if any(l.startswith("\ts_barrier") for l in lines):
            to = set()
        after[n] = to
        for t in to:
            before.setdefault(t, set()).add(n)

    def reach(n, edges):
        seen, todo = set(), [n]
        while todo:
            for t in edges.get(todo.pop(), ()):
                if t not in seen:
                    seen.add(t)
                    todo.append(t)
        return seen

    read = next(n for n, lines in enumerate(blocks) if re.search(r"#ASMSTART\n\tds_read_b128", "\n".join(lines)))
    loop = reach(read, after) & reach(read, before)
    assert read in loop
    return "\n".join("\n".join(blocks[n]) for n in sorted(loop))


def load_waits(text):
    return Counter(int(n) for n in re.findall(r"^\ts_waitcnt[^\n]*vmcnt\((\d+)\)", text, flags=re.M))


def by_hand(name):
    """wait_k and wait_v of the source, for a ring of `ns` tiles of `nl` loads each."""
    nl, ns = (8, 2) if "ILi128E" in name else (4, 4)
    return Counter([nl * (1 + 2 * j) for j in range(ns)] + [nl * 2 * j for j in range(ns)] + [nl * (2 * ns - 1)])


def test_few_rows_wait_in_the_tile_loop_only_by_hand(kernels):
    found = [k for k in kernels if "few_attn_kernel" in k[0]]
    assert len(found) == 3
    for name, body in found:
        loop = tile_loop(body)
        assert loop.count("v_mfma") >= 12 and load_waits(loop) == by_hand(name), (name, load_waits(loop))
        # one more, as the compiler would put it in front of a matrix instruction, is seen
        at = loop.index("\tv_mfma")
        planted = loop[:at] + "\ts_waitcnt vmcnt(0)\n" + loop[at:]
        assert load_waits(planted) != by_hand(name)


def test_no_vector_register_is_spilled(kernels):
    assert len(kernels) == 9
    for name, body in kernels:
        assert "v_accvgpr" not in body and "scratch_" not in body.split(".amdhsa_kernel")[0], name
