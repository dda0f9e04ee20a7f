"""The library as it is shipped: the host layer's calls of the kernels' files are ordinary references, and one that nothing defines
stops the build."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_16047_amd import build

CSRC = build.CSRC


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm")
def test_no_launcher_is_weak():
    """A weak one may be missing: the library would load, and the call would jump to address 0."""
    assert os.path.exists(build.LIB), "libamskv.so is not built (python -m paper_2511_16047_amd.build)"
    with open(os.path.join(CSRC, "amskv_internal.hpp")) as f:
        declared = set(re.findall(r"\b(launch_\w+|cross_workspace_bytes)\(", f.read()))
    out = subprocess.run(["nm", "-DC", build.LIB], stdout=subprocess.PIPE, text=True, check=True).stdout
    kinds = {m.group(2): m.group(1) for m in re.finditer(r"(\w) amskv::(\w+)\(", out)}
    assert len(declared) >= 15
    assert {n: kinds.get(n) for n in declared} == {n: "T" for n in declared}


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_a_missing_function_fails_the_link(tmp_path):
    src, obj = str(tmp_path / "caller.cpp"), str(tmp_path / "caller.o")
    with open(src, "w") as f:
        f.write("int defined_nowhere();\nextern \"C\" int caller() { return defined_nowhere(); }\n")
    subprocess.run(["g++", "-fPIC", "-c", src, "-o", obj], check=True)
    with pytest.raises(RuntimeError) as e:
        build.link([obj], str(tmp_path / "lib.so"))
    assert "defined_nowhere" in str(e.value)
