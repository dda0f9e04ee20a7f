"""The rules that divide the launches of 8-bit and cross attention (csrc/attend_rows_choice.hpp, the code the dispatch runs) built for the CPU:
which form the launches of the GPU tests take, that every form that is built is taken by some launch, that none is taken that is not
built, and that the workspace a caller is asked for is what the division writes."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2511_16047_amd as amskv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_16047_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "attend_rows_choice.hpp"
using namespace amskv::rows;
int main() {
  int cross, d, keys;
  long long units, n;
  while (std::scanf("%d %d %lld %lld %d", &cross, &d, &units, &n, &keys) == 5) {
    if (cross) {
      const Division x = divide(d, units, n, keys);
      std::printf("%d %d %d\n", x.team_waves, x.teams, x.splits);
    } else {
      const Form f = choose_codes(d, units, n, keys);
      std::printf("%d %d %d\n", f.team_waves, f.teams, 1);
    }
  }
}
"""


def _built(file, kernel):
    """{head dim: {(waves of a team, teams)}} from the dispatch's own lines."""
    with open(os.path.join(CSRC, file)) as f:
        text = f.read()
    text = text[text.index(kernel):]
    out = {64: set(), 128: set()}
    for d, waves, teams in re.findall(r"go<(64|128), (\d), (\d), \d>", text):
        out[int(d)].add((int(waves), int(teams)))
    return out


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("choice")
    src, exe = str(d / "choice.cpp"), str(d / "choice")
    with open(src, "w") as f:
        f.write(PROGRAM)
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + CSRC, src, "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert b.returncode == 0, b.stdout[-4000:]

    def ask(cross, launches):
        r = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % (cross, *x) for x in launches), stdout=subprocess.PIPE, text=True, timeout=120,
                           check=True)
        return [tuple(int(y) for y in line.split()) for line in r.stdout.splitlines()]

    return ask


SHAPES = [(d, units, n, keys) for d in (64, 128) for units in (1, 2, 7, 16, 64, 150, 256, 481, 960, 3840, 20000)
          for n in (1, 4, 25, 32, 33, 64, 65, 100, 128, 129, 256, 400, 700, 1600, 4096) for keys in (1, 32, 33, 96, 97, 250, 600, 1100, 2500, 6000, 16000)]


@pytest.mark.parametrize("cross", [0, 1], ids=["codes", "cross"])
def test_every_form_that_is_built_and_no_other(choose, cross):
    built = _built("cross.hip", "launch_cross(") if cross else _built("attend_codes.hip", "launch_attend_codes(")
    taken = {64: set(), 128: set()}
    for x, f in zip(SHAPES, choose(cross, SHAPES)):
        taken[x[0]].add(f[:2])
        assert f[2] >= 1
    assert taken == built


# (b,h), queries, keys of the step, as the tests of test_gpu_cache_in_8_bits.py and test_gpu_operators_reach.py drive them, and the forms they are there for
@pytest.mark.parametrize("launch,form", [
    ((64, 3, 300, 800), (1, 8)), ((128, 3, 300, 1600), (1, 8)), ((64, 3, 257, 290), (1, 4)), ((128, 3, 257, 290), (1, 4)),
    ((64, 6, 1, 1), (1, 1)), ((64, 2080, 169, 205), (1, 1)), ((128, 2080, 100, 104), (4, 1)), ((64, 150, 256, 456), (8, 1)),
    ((128, 150, 256, 456), (8, 1)), ((128, 150, 225, 425), (8, 1)), ((128, 272, 225, 1056), (4, 1)), ((64, 150, 128, 328), (4, 1)),
    ((128, 150, 128, 328), (4, 1)), ((64, 75, 500, 700), (8, 1)), ((128, 75, 500, 700), (8, 1)), ((128, 130, 257, 457), (4, 1)),
    ((64, 150, 256, 2756), (8, 1)), ((128, 150, 256, 2756), (8, 1)), ((64, 150, 256, 2816), (8, 1)), ((128, 150, 256, 2816), (8, 1))])
def test_launches_of_the_gpu_tests_over_codes(choose, launch, form):
    assert choose(0, [launch]) == [form + (1,)]


# (b, kv head), rows, states of test_gpu_cross_attention.py
@pytest.mark.parametrize("launch,form", [
    ((64, 27, 1, 77), (1, 1)), ((64, 4, 256, 1000), (1, 4)), ((128, 4, 256, 1000), (1, 4)), ((64, 160, 250, 200), (8, 1)),
    ((128, 160, 250, 200), (4, 1)), ((64, 160, 100, 200), (4, 1)), ((64, 512, 20, 4100), (8, 1)), ((128, 160, 20, 4100), (4, 1)),
    ((64, 272, 260, 1100), (4, 1)), ((128, 272, 260, 1100), (4, 1)), ((64, 128, 500, 1100), (8, 1)), ((64, 112, 700, 200), (8, 1))])
def test_launches_of_the_gpu_tests_over_states(choose, launch, form):
    assert choose(1, [launch])[0][:2] == form


def test_workspaces_hold_what_a_division_writes(choose):
    split = 0
    for x, (waves, teams, splits) in zip(SHAPES, choose(1, SHAPES)):
        d, units, n, keys = x
        s = amskv.Strides(n * d, n * d, d)
        k = amskv.Strides(keys * d, keys * d, d)
        need = amskv.amskv_cross_workspace_bytes(amskv.Cross(batch=units, heads=1, kv_heads=1, head_dim=d, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=n,
                                                             kv_tokens=keys, q=s, k=k, v=k, o=s))
        rows = 32 * waves
        tiles = (n + rows - 1) // rows
        assert need == (0 if splits == 1 else units * tiles * splits * rows * (d + 2) * 4)
        assert splits == 1 or (units * tiles < 256 and splits * 4 * (64 if waves == 8 else 32) * teams <= keys + 63)
        split += splits > 1
    assert split > 100


# the most (b, kv head) there may be, with the rows of a unit that memory has room for: calls that the checks let through
MOST = [(d, units, n, keys) for d in (64, 128) for units in (1 << 22, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24) for n in (1, 32, 64, 96, 120)
        for keys in (1, 33, 96, 300, 2017, 2048, 1 << 26) if units * ((n + 31) // 32) <= (1 << 26) - 8] + [(64, 1, 1 << 26, 70), (128, 2, 1 << 26, 3000)]


def test_launches_stay_below_the_threads_a_grid_may_have(choose):
    """2^32 along an axis."""
    for x, (waves, teams, splits) in zip(MOST, choose(1, MOST)):
        d, units, n, keys = x
        groups = (units * -(-n // (32 * waves)) + 7) * splits
        assert groups * 64 * waves * teams < 1 << 32, x
