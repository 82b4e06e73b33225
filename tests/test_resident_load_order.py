"""The order of the loads of the resident objectives against top lists (CPU: the assembly that
hipcc makes of them).  A row's first vectors are loaded straight into LDS, and the wait before
they are read lets the NV - NS youngest memory instructions be outstanding.  It covers the loads into LDS
only if all of them are issued before the others of that row."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2609_24150_amd import build as B

SOURCES = sorted(f for f in os.listdir(B.CSRC) if re.fullmatch(r"aal_topk_loss_fused_\w+\.hip", f))


def kernels(source, folder):
    out = os.path.join(folder, source + ".s")
    cmd = [B.hipcc(), *B.COMMON_FLAGS, "-S", "--cuda-device-only", os.path.join(B.CSRC, source), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        text = f.read()
    return re.findall(r"^(\S*k_top_fused\S*):(.*?)s_endpgm", text, re.S | re.M)


def test_loads_into_lds_come_first(tmp_path):
    try:
        B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not found")
    assert SOURCES
    with cf.ThreadPoolExecutor(len(SOURCES)) as ex:
        found = list(ex.map(lambda s: kernels(s, str(tmp_path)), SOURCES))
    wrong, staged = [], 0
    for name, body in (k for ks in found for k in ks):
        for part in re.split(r"^\s*s_barrier.*$", body, flags=re.M):  # the barriers keep loads where they are
            plain = False
            for load in re.findall(r"^\s*buffer_load_dwordx4 [^;\n]*", part, flags=re.M):
                into_lds = load.rstrip().endswith("lds")
                staged += into_lds
                plain = plain or not into_lds
                if into_lds and plain:
                    wrong.append(name)
    assert staged > 0
    assert not wrong, (len(wrong), wrong[:4])
