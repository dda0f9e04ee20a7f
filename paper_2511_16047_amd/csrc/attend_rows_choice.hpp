// How the launches of attend_rows.hpp's and attend_four.hpp's kernels are divided: plain host code.
#pragma once
#include <algorithm>
#include <cmath>

namespace amskv {
namespace rows {

// Which form a launch takes: waves to a team, teams to a workgroup.
struct Form {
  int team_waves, teams;
};

// Of waves by themselves and teams of four and eight for n rows: the fewest rows, of whole blocks of 32, whole 128 and whole 256, where a
// row of a team costs four (eight) of a lone wave's.
inline Form cheapest(long long n, double four, double eight) {
  const double alone = (double)((n + 31) / 32 * 32), team4 = four * (double)((n + 127) / 128 * 128), team8 = eight * (double)((n + 255) / 256 * 256);
  return alone <= team4 && alone <= team8 ? Form{1, 1} : team4 <= team8 ? Form{4, 1} : Form{8, 1};
}

// ---- attention over codes (attend_codes.hip)
// Which form: waves to a team, teams to a workgroup.  `units` (b,h) of `n` query rows over `keys` keys.  One key block: waves by
// themselves.  Few waves of 32 rows: the keys of a row block are shared by 4 or 8 of them.  Otherwise teams, which read K and V
// once for 128 or 256 rows, where that pays for the rows they are padded to: a row of a team costs 0.70 to 0.95 of a lone
// wave's, less the longer the keys.  us a launch, <1,1> / <1,4> / <1,8> / <4,1> / <8,1>.  Head dim 64: 16 units 256 x 530 14.5 / 7.3 / 6.6 / 14.1 /
// 15.5, 64 units 400 x 1400 36.9 / 24.9 / 26.5 / 31.9 / 32.5, 256 units 100 x 205 9.2 / 9.4 / 12.5 / 9.1 / 8.6, 560 units 260 x 265 27.9 / 37.4 / 54.6 /
// 30.9 / 37.3, 1360 units 355 x 359 98 / 126 / 165 / 84 / 94, 3840 units 25 x 55 11.1 / 18.7 / 28.7 / 20.1 / 30.8, 256 x 530 259 / 320 / 400 / 218 / 214.
// Head dim 128: 16 units 256 x 530 17.4 / 9.4 / 9.9 / 17.3 / 21.2, 15 units 1344 x 5136 148 / 101 / 103 / 121 / 143, 304 units 354 x 1179 132 / 151 /
// 183 / 101 / 122, 64 units 1844 x 2324 229 / 239 / - / 185 / 173, 2160 units 120 x 122 52 / 95 / - / 56 / 68.  (263 shapes, half of them drawn; the
// choice takes 1.008 of the best on average.)
inline Form choose_codes(int head_dim, long long units, long long n, long long keys) {
  const long long waves = units * ((n + 31) / 32), wide = units * ((n + 255) / 256), blocks = (keys + 31) / 32;
  if (blocks <= 1) return {1, 1};
  if (head_dim == 64) {
    if (waves <= 256 && blocks >= 16) return {1, 8};
    if (waves <= 512 || (waves <= 1024 && (wide <= 128 || blocks >= (n <= 32 ? 32 : 12)))) return {1, 4};
  } else {
    if (waves <= 208 && blocks >= 40) return {1, 8};
    if (waves <= (blocks >= 50 ? 800 : blocks >= 8 ? 512 : blocks >= 3 ? 256 : 0)) return {1, 4};
  }
  Form f;
  if (head_dim == 64)
    f = keys < 256 ? cheapest(n, 0.85, 0.78) : cheapest(n, 0.77, 0.69);
  else
    f = keys < 256 ? cheapest(n, 0.92, 0.95) : keys < 1024 ? cheapest(n, 0.74, 0.78) : cheapest(n, 0.76, 0.70);
  // Large teams where the fullest CU then has about as few rows (the keys of a tile are read for twice as many).  us, large / small, head
  // dim 128: 64 units 4096 x 6421 776 / 831, 576 x 997 34 / 38, 80 units 1024 x 2000 (512 rows on a CU or 384) 124 / 114, 16 units 1344 x 5136 (256
  // or 128) 143 / 121; head dim 64: 40 units 1444 x 3700 73 / 90, 100 units 700 x 1500 (512 or 384) 55 / 50.
  if (f.team_waves > 1) {
    const long long small = (units * ((n + 127) / 128) + 255) / 256 * 128, large = (wide + 255) / 256 * 256;
    f = (head_dim == 64 || keys >= 1024 ? 0.86 : 0.97) * large <= small ? Form{8, 1} : Form{4, 1};
  }
  return f;
}

// ---- cross attention (cross.hip)
// what a workgroup leaves for the second launch: O^T of its rows, then (reference, sum) of each
constexpr int partial_floats(int rows, int head_dim) { return rows * (head_dim + 2); }

// How a call is divided: the form, and workgroups that share the keys of a row tile.
struct Division {
  int team_waves, teams, splits;
};
// `units` (b, kv head) of `n` query rows over up to `keys` states.  Waves by themselves where there are at most 96 states and not
// many rows; few waves of 32 rows: four to a row block; otherwise teams that read K and V once for 128 or 256 rows where that
// pays for the rows they are padded to -- a row of a team costs 0.58 to 0.95 of a lone wave's, less the longer the keys, as K
// and V are better brought by a team, whole rows at a time, than by lanes that follow a key each; for the same reason up to 64
// rows too where K and V are large.  Teams of eight at head dim 128 are left out: 6% shorter at best, mostly longer, as they were when this was
// measured, without the step of one basic block that codes have there.  us a launch, <1,1> / <1,4> / <4,1> / <8,1> (16 heads, batch B).  Head dim 64: B 8, 36 x 77 4.9 / 4.9 / 5.4 /
// 5.2, B 32 256 x 512 32 / 39 / 24 / 27, 1024 x 512 100 / 128 / 67 / 67, 589 units 1 x 1999 62 / 57 / 54 / 69, 481 units 2432 x 231 231 / 300 / 162 / 164, 230
// units 358 x 19 7.7 / 14.9 / 7.5 / 8.4.  Head dim 128: B 2 256 x 64 5.3 / 6.2 / 6.7 / 8.2, B 8 4096 x 77 72 / 166 / 65 / 79, 146 units 272 x 2063 127 / 126 /
// 77 / 121, 10 units 1053 x 4446 124 / 90 / 47 / 58, 722 units 424 x 10 35 / 94 / 37 / 47, 12 units 2812 x 1530 81 / 84 / 53 / 50.  (247 shapes, 110 of them
// drawn; the choice takes 1.008 of the best of those on average.)
inline Division divide(int head_dim, long long units, long long n, int keys) {
  const long long waves = units * ((n + 31) / 32), wide = units * ((n + 255) / 256), blocks = ((long long)keys + 31) / 32;
  const long long bytes = units * keys * head_dim * 4;
  Form f;
  if (blocks <= 3 && (n <= 64 || waves <= 1024))
    f = {1, 1};
  else if (n <= 64 && blocks >= 64 && bytes >= (head_dim == 64 ? 400000000 : 250000000))
    f = head_dim == 64 ? Form{8, 1} : Form{4, 1};
  else if (head_dim == 64 ? waves <= 512 || (waves <= 1024 && wide <= 128) : waves <= 256 || (waves <= 512 && n <= 64))
    f = {1, 4};
  else if (head_dim == 64)
    f = keys <= 96 ? cheapest(n, 0.92, 0.95) : keys < 256 ? cheapest(n, 0.85, 0.81) : cheapest(n, 0.73, 0.66);
  else
    f = cheapest(n, keys <= 32 ? 1.0 : keys <= 128 ? 0.88 : 0.58, HUGE_VAL);  // (no eight waves: one workgroup to a CU)
  // (a launch has fewer than 2^32 threads; waves by themselves have the fewest, 64 to 32 rows, and the caller sees to it that they fit)
  if ((units * ((n + 32 * f.team_waves - 1) / (32 * f.team_waves)) + 7) * 64 * f.team_waves * f.teams > 0xffffffffll) f = {1, 1};
  Division d{f.team_waves, f.teams, 1};
  const int tile = d.team_waves == 8 ? 64 : 32;
  const long long groups = units * ((n + 32 * d.team_waves - 1) / (32 * d.team_waves));
  const int trips = (int)(((long long)keys + tile * d.teams - 1) / (tile * d.teams));
  // The keys of a row tile are shared by `splits` workgroups, each with 4 tiles for a team at least and 2 to a CU at most, where
  // that is estimated to be shorter (us): a tile takes 0.6 (a block of 32 keys at head dim 128 by one wave 1.1, a tile of 64 by
  // eight waves 0.8), longer where a CU has several workgroups, beside what K and V take to arrive; splitting costs a launch and the
  // way of its sums through the workspace.  us with / without:  Head dim 64: 8 x 1 query x 2000
  // states 8.4 / 12.2, 16000 12.7 / 71.5, 64 x 1 x 16000 49 / 110, 150 x 128 x 2000 31 / 40, 16000 174 / 302 (with 4 instead of 3 to a row tile
  // 167, with 2 195).  Head dim 128: 16 x 256 x 4000 29 / 40, 230 row tiles of 128 x 16000 270 / 303, x 2000 not split 43 (in two 55).
  if (groups >= 256 || trips < 8) return d;
  const double tile_us = d.team_waves == 8 ? 0.8 : d.team_waves == 1 && head_dim == 128 ? 1.1 : 0.6, arrive = bytes / 5.5e6;
  const double share = d.team_waves == 1 ? 1.15 : d.team_waves == 4 ? 0.65 : 0.75;
  const double sums = 2e-6 / 2.5 * groups * partial_floats(32 * d.team_waves, head_dim) * 4;
  double least = 0;
  for (int s = 1; s <= std::min((512 + groups - 1) / groups, trips / 4ll); s += s < 16 ? 1 : s / 8) {
    const long long per_cu = (groups * s + 255) / 256;
    const double walk = (double)trips / s * tile_us * (per_cu == 1 ? 1.0 : std::fmax(1.0, share * per_cu));
    const double us = std::hypot(walk, arrive) + (s == 1 ? 0 : 3 + 0.1 * s + sums * s);
    if (s == 1 || us < least) {
      least = us;
      d.splits = s;
    }
  }
  return d;
}

// ---- keys in 4 bits (attend_codes.hip, cross.hip)
// us that a launch of form f is estimated to take, whose workgroups share the keys of a row tile by `splits`.  A wave walks its blocks of 32
// keys in rounds, a block taking a wave by itself `alone`, and waves that share a SIMD `shared` each once that is longer, `around` a workgroup:
// arguments, Q and its parts, first tiles, O.  Beside it K, V, Q and O come from memory (5 TB/s) and K and V from the L2s again for every row
// tile (lone waves 10 TB/s, teams 6.5); the three are added in squares.  Splits cost a launch and the way of their sums.
// The constants are a fit to 322 shapes, 310 of them drawn, 1 to 25 forms and splits each (MI355X), but for those of teams at head dim 128, which
// were set by hand from later kernels, 64 units 4096 x 6421 and the steps before it.  With the kernels as they are the estimate is off by
// 0.16 of the time (rms) over 272 other shapes, 260 of them drawn, and the choice takes 1.017 of the best on average, 1.36 at most (head
// dim 64, 32 units, 315 x 15916); constants fitted to these anew would take 1.014.  The rule of 16-bit keys took 1.078 (up to 2.97).  us, that
// rule / this: head dim 128, 64 units, 4 rows x 14400 48 / 25; head dim 64, 1024 x 1 x 4000 115 / 45, 288 x 1 x 9266 101 / 42, 143 x 8 x 214 x 35 38 / 30.
inline double estimate4(int head_dim, double units, double n, double keys, Form f, int splits) {
  struct Times {
    double alone, shared, around;
  };
  const bool wide = head_dim == 128;
  const int w = f.team_waves, which = w == 1 ? (f.teams == 1 ? 0 : f.teams == 4 ? 1 : 2) : w == 4 ? 3 : 4;
  static const Times times[2][5] = {{{0.52, 0.27, 1.5}, {0.48, 0.26, 2.2}, {0.42, 0.28, 1.5}, {0.40, 0.23, 2.6}, {0.32, 0.21, 2.9}},
                                    {{0.68, 0.27, 1.6}, {0.65, 0.18, 3.3}, {0.50, 0.47, 3.4}, {0.48, 0.35, 2.6}, {0.38, 0.345, 3.7}}};
  const Times& t = times[wide][which];
  const int waves = w * f.teams, fit = (w == 1 ? (wide ? 8 : 12) : w == 4 ? (wide ? 12 : 16) : (wide ? 8 : 16)) / waves;
  const double tiles = std::ceil(n / (32 * w)), groups = units * tiles, blocks = std::ceil(keys / 32), tile = w == 8 ? 2 : 1;
  const double mine = w == 1 ? std::ceil(blocks / (f.teams * splits)) : std::ceil(std::ceil(blocks / tile) / splits) * tile;
  const double to_a_cu = std::ceil(groups * splits / 256), places = fit < 1 ? 1 : fit, together = std::fmin(to_a_cu, places) * waves / 4;
  const double busy = std::ceil(n / 32) / (tiles * w);  // waves of a team that have rows; the others bring keys
  const double block = std::fmax(t.alone, together * (t.shared * busy + (w > 1 ? 0.01 : 0)));
  const double walk = std::fmax(1, to_a_cu / places) * (mine * block + t.around);
  const double kv = keys * head_dim * 1.0625, memory = units * (kv + 4 * n * head_dim) / 5e6, l2 = groups * kv / (w == 1 ? 10e6 : 6.5e6);
  const double sums = splits == 1 ? 0 : 1.9 + 0.07 * splits + units * n * splits * (head_dim + 2) * 8 / 3e6;
  return 2.4 + std::sqrt(walk * walk + memory * memory + l2 * l2) + sums;
}

// The form and the splits, up to `most`, that are estimated to be shortest.  Each team has a block, each wave of a split two.
inline Division divide4(int head_dim, long long units, long long n, long long keys, int most) {
  static const Form forms[5] = {{1, 1}, {1, 4}, {1, 8}, {4, 1}, {8, 1}};
  static const int runs[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48};
  Division best{1, 1, 1};
  double least = 0;
  const long long blocks = (keys + 31) / 32;
  for (const Form& f : forms) {
    const int w = f.team_waves, waves = w * f.teams;
    const long long groups = units * ((n + 32 * w - 1) / (32 * w)), trips = (keys + (w == 8 ? 64 : 32) * f.teams - 1) / ((w == 8 ? 64 : 32) * f.teams);
    if (f.teams > 1 && f.teams > blocks) continue;
    // (a launch has fewer than 2^32 threads; waves by themselves have the fewest, and the caller sees to it that they fit)
    if (waves > 1 && (groups + 7) * 64 * waves > 0xffffffffll) continue;
    for (const int s : runs) {
      if (s > 1 && (s > most || trips / s < 2 || groups > 1200 || groups * s > (waves == 1 ? 4096 : 2048))) break;
      const double us = estimate4(head_dim, (double)units, (double)n, (double)keys, f, s);
      if (least == 0 || us < least) {
        least = us;
        best = {w, f.teams, s};
      }
    }
  }
  return best;
}

}  // namespace rows
}  // namespace amskv
