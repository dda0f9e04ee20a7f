"""The rules that divide the launches over an 8-bit cache's codes (csrc/take_choice.hpp, the code the dispatch runs) built for the CPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "take_choice.hpp"
using namespace amskv;
int main() {
  char what;
  long long a, b, c, d;
  while (std::scanf(" %c %lld %lld %lld %lld", &what, &a, &b, &c, &d) == 5) {
    if (what == 's') std::printf("%d\n", slides_at_once((int)a, b, c, (int)d));
    if (what == 'm') std::printf("%d\n", move_threads(a, (int)b, (int)c));
    if (what == 'e') {
      const ExportGrid g = export_grid((int)c, a, (int)b);
      std::printf("%lld %lld %lld\n", g.parts, g.units, g.layers);
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("choice")
    src, exe = str(d / "choice.cpp"), str(d / "choice")
    with open(src, "w") as f:
        f.write(PROGRAM)
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                        "-I" + os.path.join(ROOT, "paper_2511_16047_amd", "csrc"), src, "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert b.returncode == 0, b.stdout[-4000:]

    def run(what, launches):
        r = subprocess.run([exe], input="".join("%s %d %d %d %d\n" % (what, *x, *(0,) * (4 - len(x))) for x in launches), stdout=subprocess.PIPE, text=True, timeout=120, check=True)
        return [tuple(int(y) for y in line.split()) for line in r.stdout.splitlines()]

    return run


MANY = (1, 100, 128, 4000, (1 << 22) - 1, 1 << 22, 1 << 23, (1 << 24) - 1, 1 << 24)    # (b,h)


def test_a_slide_is_a_launch(ask):
    """Whole waves, as many as a workgroup may have, fewer than 2^32 threads in all."""
    launches = [(blocks, d, bh) for blocks in (1, 8, 16, 17, 300) for d in (64, 128) for bh in MANY]
    for (blocks, d, bh), (threads,) in zip(launches, ask("m", launches)):
        assert threads in (128, 256, 512, 1024) and threads * bh < 1 << 32
        assert bh >= 1 << 22 or threads == (256 if blocks * d <= 1024 and bh >= 128 else 1024)


def test_a_read_back_is_a_launch(ask):
    """Every (b,h) has its workgroups, fewer than 2^32 threads along an axis, and none beyond 2^31 workgroups or 65535 layers."""
    launches = [(rows, d, bh) for rows in (1, 16, 33, 64, 65, 300, 5000, 1 << 22) for d in (64, 128) for bh in MANY if rows * bh < 1 << 33]
    for (rows, d, bh), (parts, units, layers) in zip(launches, ask("e", launches)):
        assert (parts - 1) * 256 < rows * d // 16 <= parts * 256
        assert parts * units * 256 < 1 << 32 and 1 <= layers <= 65535
        assert (layers - 1) * units < bh <= layers * units
        assert layers == 1 or parts * bh * 256 >= 1 << 32


# (b,h), tokens of the new scale, blocks of 16 that slide, head dim; as timed, at once or in two launches
@pytest.mark.parametrize("bh,tokens,blocks,d,at_once", [
    (16, 16, 1, 64, 1), (16, 256, 16, 64, 1), (16, 512, 16, 64, 0), (256, 256, 16, 64, 1), (16, 128, 8, 128, 1), (16, 256, 16, 128, 0),
    (960, 16, 1, 64, 0), (16, 16, 32, 64, 1), (16, 16, 64, 64, 0), (1, 1, 256, 64, 0), (256, 16, 256, 64, 0), (16, 16, 16, 128, 1),
    (16, 16, 32, 128, 0), (256, 1, 256, 128, 0)])
def test_a_short_scale_behind_long_survivors_has_a_launch_of_its_own(ask, bh, tokens, blocks, d, at_once):
    assert ask("s", [(bh, tokens, blocks, d)]) == [(at_once,)]
