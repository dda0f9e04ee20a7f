// Attention of a step over a cache in 8 bits (Section 3.1's per-scale attention; the kept scales are e4m3 codes with a power
// of two per 16 tokens, the current scale codes too or, read in place, the caller's bf16 rows).  attend_rows.hpp has the
// formulation; here is how a launch is divided.
#include "attend_rows.hpp"
#include "attend_rows_choice.hpp"

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

}  // namespace

hipError_t launch_attend_codes(const void* q, void* o, const Codes& c, int bh, int t_q, int head_dim, int64_t cap_tokens,
                               const SegTable& seg, const ExtKV& ext, const CallerIo& io, float softmax_scale, hipStream_t st) {
  const float s = softmax_scale * 1.4426950408889634f;
  auto run = [&](auto f) { return f(q, o, c, bh, t_q, cap_tokens, seg, ext, io, s, st); };
  const rows::Form f = rows::choose_codes(head_dim, bh, t_q, seg.total);
  if (head_dim == 64) {
    if (f.team_waves == 1) return f.teams == 1 ? run(go<64, 1, 1, 3>) : f.teams == 4 ? run(go<64, 1, 4, 3>) : run(go<64, 1, 8, 2>);
    return f.team_waves == 4 ? run(go<64, 4, 1, 4>) : run(go<64, 8, 1, 4>);
  }
  if (f.team_waves == 1) return f.teams == 1 ? run(go<128, 1, 1, 2>) : f.teams == 4 ? run(go<128, 1, 4, 2>) : run(go<128, 1, 8, 2>);
  return f.team_waves == 4 ? run(go<128, 4, 1, 2>) : run(go<128, 8, 1, 2>);
}

}  // namespace amskv
