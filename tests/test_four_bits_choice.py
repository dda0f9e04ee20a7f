"""The estimate that divides the launches over keys in 4 bits (csrc/attend_rows_choice.hpp, the code the dispatch runs) built for the CPU: that
every form that is built is taken by some launch and none that is not, that launches stay within a grid's threads, that a workspace is
what the division writes, and what the launches of the GPU tests reach."""
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
int main() {
  int d, most;
  long long units, n, keys;
  while (std::scanf("%d %lld %lld %lld %d", &d, &units, &n, &keys, &most) == 5) {
    const amskv::rows::Division x = amskv::rows::divide4(d, units, n, keys, most);
    std::printf("%d %d %d\n", x.team_waves, x.teams, x.splits);
  }
}
"""
FORMS = {(1, 1), (1, 4), (1, 8), (4, 1), (8, 1)}


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("choice4")
    src, exe = str(d / "choice.cpp"), str(d / "choice")
    with open(src, "w") as f:
        f.write(PROGRAM)
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + CSRC, src, "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert b.returncode == 0, b.stdout[-4000:]

    def ask(launches, most):
        r = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % (*x, most) for x in launches), stdout=subprocess.PIPE, text=True, timeout=120,
                           check=True)
        return [tuple(int(y) for y in line.split()) for line in r.stdout.splitlines()]

    return ask


SHAPES = [(d, units, n, keys) for d in (64, 128) for units in (1, 2, 7, 16, 64, 150, 256, 481, 960, 3840, 20000)
          for n in (1, 4, 25, 32, 33, 64, 65, 100, 128, 129, 256, 400, 700, 1600, 4096) for keys in (0, 1, 32, 33, 96, 97, 250, 600, 1100, 2500, 6000, 16000)]


@pytest.mark.parametrize("file,most", [("attend_codes.hip", 1), ("cross.hip", 48)])
def test_every_form_that_is_built_and_no_other(choose, file, most):
    with open(os.path.join(CSRC, file)) as f:
        text = f.read()
    built = {64: set(), 128: set()}
    for d, waves, teams in re.findall(r"go<(64|128), (\d), (\d), \d, 4(?:, false)?>", text):
        built[int(d)].add((int(waves), int(teams)))
    taken = {64: set(), 128: set()}
    for x, f in zip(SHAPES, choose(SHAPES, most)):
        taken[x[0]].add(f[:2])
        assert 1 <= f[2] <= most
    assert taken == built == {64: FORMS, 128: FORMS}


def test_workspaces_hold_what_a_division_writes(choose):
    split = 0
    shapes = [x for x in SHAPES if x[3] > 0]
    for x, (waves, teams, splits) in zip(shapes, choose(shapes, 48)):
        d, units, n, keys = x
        s = amskv.Strides(n * d, n * d, d)
        need = amskv.amskv_cross_workspace_bytes(amskv.Cross(batch=units, heads=1, kv_heads=1, head_dim=d, dtype=amskv.AMSKV_DTYPE_BF16_KV4, q_tokens=n,
                                                             kv_tokens=keys, q=s, o=s))
        rows = 32 * waves
        tiles = (n + rows - 1) // rows
        assert need == (0 if splits == 1 else units * tiles * splits * rows * (d + 2) * 4)
        # each wave of a split has two blocks of keys at least
        assert splits == 1 or (units * tiles <= 1200 and splits * 2 * (64 if waves == 8 else 32) * teams <= keys + 63 * teams)
        split += splits > 1
    assert split > 100


MOST = [(d, units, n, keys) for d in (64, 128) for units in (1 << 22, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24) for n in (1, 32, 64, 96, 120)
        for keys in (1, 33, 96, 300, 2017, 2048, 1 << 26) if units * ((n + 31) // 32) <= (1 << 26) - 8] + [(64, 1, 1 << 26, 70), (128, 2, 1 << 26, 3000)]


def test_launches_stay_below_the_threads_a_grid_may_have(choose):
    """2^32 along an axis."""
    for most in (1, 48):
        for x, (waves, teams, splits) in zip(MOST, choose(MOST, most)):
            d, units, n, keys = x
            groups = (units * -(-n // (32 * waves)) + 7) * splits
            assert groups * 64 * waves * teams < 1 << 32, x


# (b,h), queries, keys of steps that test_gpu_cache_in_4_bits.py drives
def test_the_gpu_tests_reach_every_form(choose):
    for d in (64, 128):
        cache = [(d, 3, q, q + b) for q in (1, 7, 31, 32, 33, 63, 64, 65, 128, 129, 255, 256, 257, 300, 520) for b in (0, 1, 15, 16, 31, 33, 64, 500)]
        cache += [(d, u, q, q + b) for u, q in ((150, 65), (150, 128), (150, 225), (150, 256), (130, 257), (75, 500)) for b in (0, 1, 16, 30, 33, 64, 95, 200)]
        cache += [(d, 272, 225, 225 + b) for b in (799, 831, 840)]
        cache += [(d, 64, q, q + b) for q, b in ((576, 500), (512, 705), (505, 551), (576, 0), (551, 449))]
        assert {x[:2] for x in choose(cache, 1)} == FORMS
        # (b, kv head), rows, states of test_gpu_held_states.py
        cross = [(d, u, n, 77) for u in (27, 18, 9) for n in (1, 2, 8, 5, 40, 33, 264, 100, 300, 800, 129, 1032, 387, 900, 2400)]
        cross += [(d, 4, n, k) for n in (1, 32, 64, 128, 256) for k in (1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000)]
        cross += [(d, u, n, k) for k in (5000, 4096) for u, n in ((4, 1), (2, 4), (2, 24), (10, 40), (5, 260), (20, 1))]
        cross += [(d, u, n, 200) for u, n in ((160, 100), (160, 129), (160, 300), (192, 250), (224, 257), (112, 700))]
        cross += [(d, 272, 260, 1100), (d, 128, 500, 1100)]
        got = choose(cross, 48)
        assert {x[:2] for x in got} == FORMS and any(x[2] > 1 for x in got)
