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
    """The lines of the shortest cycle that the first LDS read written by hand lies in and a matrix instruction too: from the label that a
    branch goes back to, to that branch, and the blocks behind it that end with a branch back into it."""
    lines = body.split("\n")
    at = {m.group(1): n for n, l in enumerate(lines) for m in [re.match(r"(\.LBB\d+_\d+):", l)] if m}
    back = [(at[m.group(1)], n) for n, l in enumerate(lines) for m in [re.match(r"\ts_c?branch\S* (\.LBB\d+_\d+)", l)]
            if m and m.group(1) in at and at[m.group(1)] <= n]
    read = next(n for n, l in enumerate(lines) if l.startswith("\tds_read_b128") and "#ASMSTART" in lines[n - 1])
    lo, hi = min(((t, b) for t, b in back if t <= read <= b and any("v_mfma" in l for l in lines[t:b])), key=lambda x: x[1] - x[0])
    keep = list(range(lo, hi + 1))
    for t, b in back:
        if lo <= t <= hi < b:
            block = max(n for n in at.values() if n <= b)
            keep += [n for n in range(block, b + 1) if n not in keep]
    return "\n".join(lines[n] for n in keep)


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
