// Attention of a step over a cache in 8 or 4 bits (Section 3.1's per-scale attention; the kept scales are e4m3 codes with a power
// of two per 16 tokens, or e2m1 codes with one per 32 channels of a token, the current scale codes too or, read in place, the
// caller's bf16 rows).  attend_rows.hpp has the formulation; here is how a launch is divided.
#include "attend_four.hpp"
#include "attend_rows_choice.hpp"

namespace amskv {
namespace {

constexpr int kMostWhole = 8;  // query tiles on the fullest XCD up to which a (b,h) stays on one (place())

// kMixed (4 bits): rows read in place may follow the codes
template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd, int kBits, bool kMixed>
__global__ __launch_bounds__(64 * kTeamWaves* kTeams, kMinWavesPerSimd) void attend_codes_kernel(
    const char* __restrict__ q, char* __restrict__ o, CodesOf<kBits> codes, int t_q, long long cap_tokens, SegTable seg, ExtKV ext, CallerIo io,
    float scale_log2e, int n_bh, int n_qtiles, int n_whole) {
  fetch_arguments<6 * 8 + 16 + sizeof(SegTable) + sizeof(ExtKV) + sizeof(CallerIo)>();
  using U = rows::Unit<D, kTeamWaves, kTeams, kBits>;
  constexpr bool kFour = kBits == 4 && kTeamWaves > 1 && !(kMixed && D == 64);  // K goes to the matrix cores in 4 bits
  using Team = rows::FourBitTeam<D, kTeamWaves == 1 ? 4 : kTeamWaves, kMixed>;
  __shared__ __align__(1024) char lds[kFour ? Team::kLds : U::kLds];
  Place at{(int)blockIdx.x, 0};
  if (n_qtiles > 1) at = place<true>(blockIdx.x, n_bh, n_qtiles, n_whole);
  const long long bh = at.bh;
  if (bh >= n_bh) return;  // the whole workgroup
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int base = at.tile * U::kRows + 32 * (wave % kTeamWaves);
  const bool active = base < t_q;

  auto q_row = [&](int of_lane) { return q + unit_offset(io.q, bh, io.heads) + min(base + (of_lane & 31), t_q - 1) * io.q.tok; };
  rows::bf16x8 qf[U::KS];
  u32x4 raw[D / 64][4];
  if constexpr (kFour) {
    rows::load_query<D>(raw, q_row(lane), h);
  } else {
    const char* row = q_row(lane);
#pragma unroll
    for (int t = 0; t < U::KS; ++t) qf[t] = *reinterpret_cast<const rows::bf16x8*>(row + U::q_at(t, h));
  }

  const long long x_unit = unit_offset(io.kv, bh, io.heads), blocks = cap_tokens / AMSKV_KV8_BLOCK;
  rows::Keys keys{nullptr, nullptr, nullptr, nullptr, (const char*)ext.k + x_unit, (const char*)ext.v + x_unit, io.kv.tok, io.kv.tok, seg.ext_start,
                  seg.total - seg.ext_start, nullptr, nullptr};
  keys.k_codes = codes.k + bh * cap_tokens * (D * kBits / 8);
  keys.v_codes = codes.v + bh * cap_tokens * (D * kBits / 8);
  if constexpr (kBits == 8) {
    keys.k_scale = codes.k_scale + bh * blocks;
    keys.v_scale = codes.v_scale + bh * blocks;
  } else {
    keys.k_group = codes.k_group + bh * cap_tokens * (D / AMSKV_KV4_GROUP);
    keys.v_group = codes.v_group + bh * cap_tokens * (D / AMSKV_KV4_GROUP);
  }
  typename U::Result x;
  U::clear(x);
  if constexpr (kFour) {
    typename Team::Query parts;
    rows::split_query(parts, raw);
    Team::walk(x, parts, [&]() { return q_row(U::fresh(threadIdx.x)); }, lds, keys, seg, 0, Team::tiles(keys), scale_log2e, active);
  } else {
    U::walk(x, qf, lds, keys, seg, 0, U::tiles(keys), scale_log2e, active);
  }
  U::meet(x, lds);
  const int row = base + (U::fresh(threadIdx.x) & 31);  // (not kept over the walk)
  int heads = io.heads;
  if constexpr (kFour) asm volatile("" : "+s"(heads));  // (nor what divides by them)
  U::put(x, reinterpret_cast<__bf16*>(o + unit_offset(io.o, bh, heads) + min(row, t_q - 1) * io.o.tok), active && row < t_q);
}

template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd, int kBits = 8, bool kMixed = true>
hipError_t go(const void* q, void* o, const CodesOf<kBits>& c, int bh, int t_q, int64_t cap, const SegTable& seg, const ExtKV& ext,
              const CallerIo& io, float scale_log2e, hipStream_t st) {
  constexpr int kRows = 32 * kTeamWaves;
  const int n_qtiles = (t_q + kRows - 1) / kRows, n_whole = whole_units(bh, n_qtiles, kMostWhole);
  hipLaunchKernelGGL((attend_codes_kernel<D, kTeamWaves, kTeams, kMinWavesPerSimd, kBits, kMixed>), dim3(n_qtiles == 1 ? bh : placed_grid(bh, n_qtiles, n_whole)),
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

hipError_t launch_attend_codes4(const void* q, void* o, const Codes4& c, int bh, int t_q, int head_dim, int64_t cap_tokens,
                                const SegTable& seg, const ExtKV& ext, const CallerIo& io, float softmax_scale, hipStream_t st) {
  const float s = softmax_scale * 1.4426950408889634f;
  auto run = [&](auto f) { return f(q, o, c, bh, t_q, cap_tokens, seg, ext, io, s, st); };
  const rows::Division f = rows::divide4(head_dim, bh, t_q, seg.total, 1);
  const bool mixed = seg.ext_start < seg.total;
  if (head_dim == 64) {
    if (f.team_waves == 1) return f.teams == 1 ? run(go<64, 1, 1, 3, 4>) : f.teams == 4 ? run(go<64, 1, 4, 3, 4>) : run(go<64, 1, 8, 2, 4>);
    if (mixed) return f.team_waves == 4 ? run(go<64, 4, 1, 4, 4>) : run(go<64, 8, 1, 4, 4>);
    return f.team_waves == 4 ? run(go<64, 4, 1, 4, 4, false>) : run(go<64, 8, 1, 4, 4, false>);
  }
  if (f.team_waves == 1) return f.teams == 1 ? run(go<128, 1, 1, 2, 4>) : f.teams == 4 ? run(go<128, 1, 4, 2, 4>) : run(go<128, 1, 8, 2, 4>);
  if (mixed) return f.team_waves == 4 ? run(go<128, 4, 1, 2, 4>) : run(go<128, 8, 1, 2, 4>);
  return f.team_waves == 4 ? run(go<128, 4, 1, 3, 4, false>) : run(go<128, 8, 1, 2, 4, false>);
}

}  // namespace amskv
