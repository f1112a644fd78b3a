"""The update kernels of plain caches run five CTAs an SM at 48 registers a
thread. The compiler says whether they still fit without spilling to memory."""
import os
import re
import subprocess
import sys

from conftest import ROOT


def test_update_kernels_do_not_spill(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import build as B
    r = subprocess.run([B.nvcc(), *B.ARCH, *B.FLAGS, "-Xptxas", "-v", "-c",
                        os.path.join(B.CSRC, "hkv_update.cu"), "-o", str(tmp_path / "u.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = re.findall(r"entry function '(\S+)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads"
                       r".*?Used (\d+) registers", r.stderr, re.S)
    kernels = [x for x in found if re.search(r"\d(evict|append_evict|repack)_kernel", x[0])]
    assert len(kernels) == 12          # three kernels, two head sizes, two types
    for name, stores, loads, registers in kernels:
        assert (int(stores), int(loads)) == (0, 0) and int(registers) <= 48, (name, stores, loads)
