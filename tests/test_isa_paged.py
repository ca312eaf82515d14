"""Static check of the machine code of the paged attention kernels: as for the other kernels with hand-written LDS reads,
nothing touches a read's registers before a wait that covers it, and none is in flight across control flow."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2510_10129_amd import build
from test_isa_audit import HIPCC, audit


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("isa") / "paged.s"
    cmd = [HIPCC, *build.FLAGS, "-S", "--cuda-device-only", "-o", str(out), os.path.join(build.CSRC, "paged_attention.hip")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    text = out.read_text()
    return lambda name: re.findall(r"^(_ZN\S*%s\S*):[^\n]*\n(.*?)\.end_amdhsa_kernel" % name, text, flags=re.S | re.M)


def test_reads_of_few_rows_are_waited_for(kernels):
    found = kernels("few_attn_kernel")
    assert len(found) == 3, [k[0] for k in found]          # 16 columns at either head dim, 32 at 64
    for name, body in found:
        seen, bad = audit(body)
        # K: two halves of 16 keys, V: the same of every 16 rows of O^T
        assert seen == (24 if "ILi128E" in name else 12), (name, seen)
        assert not bad, (name, bad[:5])


def test_reads_of_many_rows_are_waited_for(kernels):
    found = kernels("chunk_attn_kernel")
    assert len(found) == 6, [k[0] for k in found]          # two head dims, wide and narrow pages; few rows of 128
    for name, body in found:
        seen, bad = audit(body)
        assert seen >= 40, (name, seen)
        assert not bad, (name, bad[:5])


def test_paged_kernels_keep_to_vector_registers(kernels):
    """No spills, no sums moved between vector and accumulation registers."""
    for name, body in kernels("(?:few|chunk)_attn_kernel"):
        assert "v_accvgpr" not in body and "scratch_store" not in body, name


def test_few_rows_wait_for_tiles_by_hand_alone(kernels):
    """Between the loop's first LDS read and its last MFMA no wait for loads is the compiler's: it would be for all tiles on their
    way."""
    for name, body in kernels("few_attn_kernel"):
        lines = body.split("\n")
        first = [n for n, l in enumerate(lines) if l.strip().startswith("ds_read_b128")][0]
        last = [n for n, l in enumerate(lines) if "v_mfma" in l][-1]
        waits = [l.strip() for l in lines[first:last] if "s_waitcnt" in l and "vmcnt" in l]
        by_hand = {4 * n for n in range(1, 16)} | {0}
        assert waits and all(int(re.search(r"vmcnt\((\d+)\)", l).group(1)) in by_hand for l in waits), (name, waits)
