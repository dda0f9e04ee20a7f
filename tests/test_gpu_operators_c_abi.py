"""The rotary, 8-bit and cross-attention calls from a plain C program (tests/c_abi/operators_check.c), and the binding's structures against
the header's, member by member."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2511_16047_amd as amskv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2511_16047_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def _run(tmp_path, *args):
    """A one-second host compile of a C file; the library itself was built beforehand."""
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    exe = str(tmp_path / "operators_check")
    cmd = ["gcc", "-std=c11", "-O2", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(ROCM, "include"),
           "-I" + os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "c_abi", "operators_check.c"), "-o", exe,
           "-L" + PKG, "-lamskv", "-L" + os.path.join(ROCM, "lib"), "-lamdhip64", "-lm",
           "-Wl,-rpath," + PKG, "-Wl,-rpath," + os.path.join(ROCM, "lib")]
    b = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert b.returncode == 0, b.stdout[-4000:]
    r = subprocess.run([exe, *args], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-4000:]
    return r.stdout


def test_structures_of_the_binding(tmp_path):
    want = {k: int(v) for k, v in (line.split() for line in _run(tmp_path, "layout").splitlines())}
    got = {}
    for name, of in (("amskv_rope", amskv.Rope), ("amskv_strides", amskv.Strides), ("amskv_cross", amskv.Cross)):
        got[name] = ctypes.sizeof(of)
        got.update({"%s.%s" % (name, m): getattr(of, m).offset for m, *_ in of._fields_})
    assert got == want


@pytest.mark.gpu
def test_c_program_runs(tmp_path):
    out = _run(tmp_path)
    print(out)
    assert "operators_check: ok" in out
