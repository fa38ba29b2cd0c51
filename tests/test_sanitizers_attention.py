"""CPU builds under AddressSanitizer + UndefinedBehaviorSanitizer (no GPU involved): the comparison of places in memory against brute force, and the host side of attention
between whole sequences and of the norms and rotation before it, their workspaces and shares over the whole range of shapes, and their refusals."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

from test_sanitizers import ENV, HERE, ROOT

SANITIZE = ["-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined"]


def run(exe):
    r = subprocess.run([exe], env=ENV, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr


def test_places_against_brute_force(tmp_path):
    exe = str(tmp_path / "overlap_driver")
    subprocess.run(["g++"] + SANITIZE + ["-static-libasan", os.path.join(HERE, "overlap_driver.cpp"), "-o", exe], check=True)
    run(exe)


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not found")
def test_attention_host_code_under_sanitizers(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2303_08810_amd import build as bra_build
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    # the objects that test_sanitizers.py has compiled, where they are newer than the sources
    objs = [os.path.join(bra_build.OBJ_DIR, "host_sanitize", os.path.basename(f)[:-4] + ".o") for f in bra_build.sources()]
    sources = glob.glob(os.path.join(bra_build.CSRC, "*")) + [os.path.join(ROOT, "include", "bra.h"), bra_build.__file__]
    if not all(map(os.path.exists, objs)) or min(map(os.path.getmtime, objs)) <= max(map(os.path.getmtime, sources)):
        objs = bra_build.compile_objects(tag="host_sanitize", extra_flags=["-g"] + host, opt="-O1")
    exe, drv = str(tmp_path / "attention_driver"), str(tmp_path / "attention_driver.o")
    subprocess.run(["g++"] + SANITIZE + ["-c", os.path.join(HERE, "attention_driver.cpp"), "-o", drv], check=True)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", drv] + objs + ["-fsanitize=address,undefined", "-o", exe],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    run(exe)
