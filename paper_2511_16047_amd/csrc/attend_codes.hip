// Attention of a step over a cache in 8 bits (Section 3.1's per-scale attention; the kept scales are e4m3 codes with a power
// of two per 16 tokens, the current scale codes too or, read in place, the caller's bf16 rows).  attend_rows.hpp has the
// formulation; here is how a launch is divided.
#include "attend_rows.hpp"

namespace amskv {
namespace {

constexpr int kMostWhole = 8;  // query tiles on the fullest XCD up to which a (b,h) stays on one (place())

template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd>
__global__ __launch_bounds__(64 * kTeamWaves* kTeams, kMinWavesPerSimd) void attend_codes_kernel(
    const char* __restrict__ q, char* __restrict__ o, Codes codes, int t_q, long long cap_tokens, SegTable seg, ExtKV ext, CallerIo io,
    float scale_log2e, int n_bh, int n_qtiles, int n_whole) {
  fetch_arguments<6 * 8 + 16 + sizeof(SegTable) + sizeof(ExtKV) + sizeof(CallerIo)>();
  using U = rows::Unit<D, kTeamWaves, kTeams, true>;
  __shared__ __align__(1024) char lds[U::kLds];
  Place at{(int)blockIdx.x, 0};
  if (n_qtiles > 1) at = place<true>(blockIdx.x, n_bh, n_qtiles, n_whole);
  const long long bh = at.bh;
  if (bh >= n_bh) return;  // the whole workgroup
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const int base = at.tile * U::kRows + 32 * (wave % kTeamWaves);
  const bool active = base < t_q;

  rows::bf16x8 qf[U::KS];
  const char* q_row = q + unit_offset(io.q, bh, io.heads) + min(base + r, t_q - 1) * io.q.tok;
#pragma unroll
  for (int t = 0; t < U::KS; ++t) qf[t] = *reinterpret_cast<const rows::bf16x8*>(q_row + U::q_at(t, h));

  const long long x_unit = unit_offset(io.kv, bh, io.heads), blocks = cap_tokens / AMSKV_KV8_BLOCK;
  const rows::Keys keys{codes.k + bh * cap_tokens * D, codes.v + bh * cap_tokens * D, codes.k_scale + bh * blocks, codes.v_scale + bh * blocks,
                        (const char*)ext.k + x_unit, (const char*)ext.v + x_unit, io.kv.tok, io.kv.tok, seg.ext_start,
                        seg.total - seg.ext_start};
  typename U::Result x;
  U::clear(x);
  U::walk(x, qf, lds, keys, seg, 0, U::tiles(keys), scale_log2e, active);
  U::meet(x, lds);
  const int row = base + (U::fresh(threadIdx.x) & 31);  // (not kept over the walk)
  U::put(x, reinterpret_cast<__bf16*>(o + unit_offset(io.o, bh, io.heads) + min(row, t_q - 1) * io.o.tok), active && row < t_q);
}

template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd>
hipError_t go(const void* q, void* o, const Codes& c, int bh, int t_q, int64_t cap, const SegTable& seg, const ExtKV& ext,
              const CallerIo& io, float scale_log2e, hipStream_t st) {
  constexpr int kRows = 32 * kTeamWaves;
  const int n_qtiles = (t_q + kRows - 1) / kRows, n_whole = whole_units(bh, n_qtiles, kMostWhole);
  hipLaunchKernelGGL((attend_codes_kernel<D, kTeamWaves, kTeams, kMinWavesPerSimd>), dim3(n_qtiles == 1 ? bh : placed_grid(bh, n_qtiles, n_whole)),
                     dim3(64 * kTeamWaves * kTeams), 0, st, (const char*)q, (char*)o, c, t_q, (long long)cap, seg, ext, io, scale_log2e, bh,
                     n_qtiles, n_whole);
  return hipGetLastError();
}

// Which form: waves to a team, teams to a workgroup.  `units` (b,h) of `n` query rows over `keys` keys.  One key block: waves by
// themselves.  Few waves of 32 rows: the keys of a row block are shared by 4 or 8 of them.  Otherwise teams, which read K and V
// once for 128 or 256 rows, where that pays for the rows they are padded to: a row of a team costs 0.70 to 0.95 of a lone
// wave's, less the longer the keys.  us a launch, <1,1> / <1,4> / <1,8> / <4,1> / <8,1>.  Head dim 64: 16 units 256 x 530 14.5 / 7.3 / 6.6 / 14.1 /
// 15.5, 64 units 400 x 1400 36.9 / 24.9 / 26.5 / 31.9 / 32.5, 256 units 100 x 205 9.2 / 9.4 / 12.5 / 9.1 / 8.6, 560 units 260 x 265 27.9 / 37.4 / 54.6 /
// 30.9 / 37.3, 1360 units 355 x 359 98 / 126 / 165 / 84 / 94, 3840 units 25 x 55 11.1 / 18.7 / 28.7 / 20.1 / 30.8, 256 x 530 259 / 320 / 400 / 218 / 214.
// Head dim 128: 16 units 256 x 530 17.4 / 9.4 / 9.9 / 17.3 / 21.2, 15 units 1344 x 5136 148 / 101 / 103 / 121 / 143, 304 units 354 x 1179 132 / 151 /
// 183 / 101 / 122, 64 units 1844 x 2324 229 / 239 / - / 185 / 173, 2160 units 120 x 122 52 / 95 / - / 56 / 68.  (263 shapes, half of them drawn; the
// choice takes 1.008 of the best on average.)
rows::Form choose(int head_dim, long long units, long long n, long long keys) {
  const long long waves = units * ((n + 31) / 32), wide = units * ((n + 255) / 256), blocks = (keys + 31) / 32;
  if (blocks <= 1) return {1, 1};
  if (head_dim == 64) {
    if (waves <= 256 && blocks >= 16) return {1, 8};
    if (waves <= 512 || (waves <= 1024 && (wide <= 128 || blocks >= (n <= 32 ? 32 : 12)))) return {1, 4};
  } else {
    if (waves <= 208 && blocks >= 40) return {1, 8};
    if (waves <= (blocks >= 50 ? 800 : blocks >= 8 ? 512 : blocks >= 3 ? 256 : 0)) return {1, 4};
  }
  rows::Form f;
  if (head_dim == 64)
    f = keys < 256 ? rows::cheapest(n, 0.85, 0.78) : rows::cheapest(n, 0.77, 0.69);
  else
    f = keys < 256 ? rows::cheapest(n, 0.92, 0.95) : keys < 1024 ? rows::cheapest(n, 0.74, 0.78) : rows::cheapest(n, 0.76, 0.70);
  // Large teams where the fullest CU then has about as few rows (the keys of a tile are read for twice as many).  us, large / small, head
  // dim 128: 64 units 4096 x 6421 776 / 831, 576 x 997 34 / 38, 80 units 1024 x 2000 (512 rows on a CU or 384) 124 / 114, 16 units 1344 x 5136 (256
  // or 128) 143 / 121; head dim 64: 40 units 1444 x 3700 73 / 90, 100 units 700 x 1500 (512 or 384) 55 / 50.
  if (f.team_waves > 1) {
    const long long small = (units * ((n + 127) / 128) + 255) / 256 * 128, large = (wide + 255) / 256 * 256;
    f = (head_dim == 64 || keys >= 1024 ? 0.86 : 0.97) * large <= small ? rows::Form{8, 1} : rows::Form{4, 1};
  }
  return f;
}

}  // namespace

hipError_t launch_attend_codes(const void* q, void* o, const Codes& c, int bh, int t_q, int head_dim, int64_t cap_tokens,
                               const SegTable& seg, const ExtKV& ext, const CallerIo& io, float softmax_scale, hipStream_t st) {
  const float s = softmax_scale * 1.4426950408889634f;
  auto run = [&](auto f) { return f(q, o, c, bh, t_q, cap_tokens, seg, ext, io, s, st); };
  const rows::Form f = choose(head_dim, bh, t_q, seg.total);
  if (head_dim == 64) {
    if (f.team_waves == 1) return f.teams == 1 ? run(go<64, 1, 1, 3>) : f.teams == 4 ? run(go<64, 1, 4, 3>) : run(go<64, 1, 8, 2>);
    return f.team_waves == 4 ? run(go<64, 4, 1, 4>) : run(go<64, 8, 1, 4>);
  }
  if (f.team_waves == 1) return f.teams == 1 ? run(go<128, 1, 1, 2>) : f.teams == 4 ? run(go<128, 1, 4, 2>) : run(go<128, 1, 8, 2>);
  return f.team_waves == 4 ? run(go<128, 4, 1, 2>) : run(go<128, 8, 1, 2>);
}

}  // namespace amskv
