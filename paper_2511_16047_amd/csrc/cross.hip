// Cross attention: the queries of a step over an encoder's states, whose number differs from batch element to batch element
// and is known on the device only.  attend_rows.hpp has the formulation.
//
// A unit is a (b, kv head).  Its query rows are the queries of all heads that read this kv head -- row r is query r % T of the
// head's r / T -- so shared heads read K and V once, and a single token of 8 heads is one block of 8 rows, not 8 of one.
// Bound: K and V from HBM where rows are few (8 x 8 kv heads, 4 rows, up to 16000 states, head dim 128: 472 MB in 89 us and 5 for the second
// launch); the matrix pipe and, with short states, the time to Q and the first tiles, which only the other workgroup of the CU
// hides (8 x 16 heads, 4096 x up to 512, head dim 128: 120 us, 0.57 PFLOP/s and 2.4 TB/s).
// A launch over few rows and many states does not fill the chip with one workgroup to 32 or 128 rows; then `splits` workgroups
// take equal runs of key tiles each, leave their sums unnormalised in the workspace, and a second launch puts them together.
#include "attend_four.hpp"
#include "attend_rows_choice.hpp"

namespace amskv {
namespace {

constexpr int kMostWhole = 8;  // row tiles on the fullest XCD up to which a unit stays on one (place())

struct CrossArgs {
  const char *q, *k, *v;
  char* o;
  RowMap q_map, k_map, v_map, o_map;
  const int *lengths, *offsets;
  long long kv_rows;
  float* workspace;
  float scale_log2e;
  long long held_rows;  // 4 bits: rows of a unit of the held tensors, and where the bytes of their groups begin
  long long groups_at;
  int kv_heads, group, q_tokens, kv_tokens, n_units, row_tiles, splits, n_whole;
};

// the states of batch element b: first row (of the packed axis) and how many; whatever the device arrays hold, rows exist
__device__ __forceinline__ int states(const CrossArgs& a, unsigned b, long long& first) {
  first = 0;
  if (a.offsets != nullptr) {
    const long long from = min(max((long long)a.offsets[b], 0ll), a.kv_rows), to = min(max((long long)a.offsets[b + 1], 0ll), a.kv_rows);
    first = from;
    return (int)min(max(to - from, 0ll), (long long)a.kv_tokens);
  }
  return a.lengths != nullptr ? min(max(a.lengths[b], 0), a.kv_tokens) : a.kv_tokens;
}

template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd, int kBits>
__global__ __launch_bounds__(64 * kTeamWaves* kTeams, kMinWavesPerSimd) void cross_kernel(CrossArgs a) {
  fetch_arguments<sizeof(CrossArgs)>();
  using U = rows::Unit<D, kTeamWaves, kTeams, kBits>;
  constexpr bool kFour = kBits == 4 && kTeamWaves > 1;  // K goes to the matrix cores in 4 bits
  using Team = rows::FourBitTeam<D, kTeamWaves == 1 ? 4 : kTeamWaves, false>;
  __shared__ __align__(1024) char lds[kFour ? Team::kLds : U::kLds];
  const int tiles = a.row_tiles * a.splits;
  Place at{(int)blockIdx.x, 0};
  if (tiles > 1) at = place<true>(blockIdx.x, a.n_units, tiles, a.n_whole);
  if (at.bh >= a.n_units) return;  // the whole workgroup
  const unsigned b = (unsigned)at.bh / (unsigned)a.kv_heads, g = (unsigned)at.bh - b * a.kv_heads;
  const int tile = a.splits == 1 ? at.tile : at.tile / a.splits, split = at.tile - tile * a.splits;
  long long first;
  const int n = states(a, b, first);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int n_rows = a.group * a.q_tokens, base = tile * U::kRows + 32 * (wave % kTeamWaves);
  const bool active = base < n_rows;
  // byte offset of the lane's row in Q or O (found twice, not kept over the walk)
  auto row_at = [&](const RowMap& m, int of_lane, int q_tokens) {
    const int row = min(base + (of_lane & 31), n_rows - 1);
    const int head = a.group == 1 ? 0 : row / q_tokens, token = row - head * q_tokens;
    return b * m.batch + ((long long)g * a.group + head) * m.head + token * m.tok;
  };

  const char* q_row = a.q + row_at(a.q_map, lane, a.q_tokens);
  // (asked for before the number of states is waited for)
  rows::bf16x8 qf[U::KS];
  u32x4 raw[D / 64][4];
  if constexpr (kFour) {
    rows::load_query<D>(raw, q_row, h);
  } else {
#pragma unroll
    for (int t = 0; t < U::KS; ++t) qf[t] = *reinterpret_cast<const rows::bf16x8*>(q_row + U::q_at(t, h));
  }

  rows::Keys keys{};
  if constexpr (kBits == 16) {
    const long long kb = a.offsets ? first * a.k_map.tok : b * a.k_map.batch, vb = a.offsets ? first * a.v_map.tok : b * a.v_map.batch;
    keys.kx = a.k + kb + g * a.k_map.head;
    keys.vx = a.v + vb + g * a.v_map.head;
    keys.k_tok = a.k_map.tok;
    keys.v_tok = a.v_map.tok;
    keys.n_rows = n;
  } else {
    const long long row = a.offsets ? g * a.held_rows + first : (long long)at.bh * a.held_rows;
    keys.k_codes = (const unsigned char*)a.k + row * (D / 2);
    keys.v_codes = (const unsigned char*)a.v + row * (D / 2);
    keys.k_group = (const unsigned char*)a.k + a.groups_at + row * (D / AMSKV_KV4_GROUP);
    keys.v_group = (const unsigned char*)a.v + a.groups_at + row * (D / AMSKV_KV4_GROUP);
    keys.n_codes = n;
  }
  const int n_tiles = U::tiles(keys), each = (n_tiles + a.splits - 1) / a.splits;
  const int from = min(split * each, n_tiles), to = min(from + each, n_tiles);
  typename U::Result x;
  U::clear(x);
  SegTable none;
  none.n = 0;
  if constexpr (kFour) {
    typename Team::Query parts;
    rows::split_query(parts, raw);
    Team::walk(x, parts, [&]() { return q_row; }, lds, keys, none, from, to, a.scale_log2e, active);
  } else {
    U::walk(x, qf, lds, keys, none, from, to, a.scale_log2e, active);
  }
  U::meet(x, lds);
  const int late = U::fresh(threadIdx.x) & 63;
  if (a.splits == 1) {
    int q_tokens = a.q_tokens;
    if constexpr (kFour) asm volatile("" : "+s"(q_tokens));
    U::put(x, reinterpret_cast<__bf16*>(a.o + row_at(a.o_map, late, q_tokens)), active && base + (late & 31) < n_rows);
    return;
  }
  float* mine = a.workspace + (((long long)at.bh * a.row_tiles + tile) * a.splits + split) * rows::partial_floats(U::kRows, D);
  const int local = 32 * (wave % kTeamWaves) + (late & 31);
  if (active && base + (late & 31) < n_rows) U::put_partial(x, mine + local * D);
  if (wave < kTeamWaves && late < 32) *reinterpret_cast<float2*>(mine + U::kRows * D + 2 * local) = make_float2(x.ref, x.sum);
}

// A lane has 4 channels of a row.
template <int D>
__global__ __launch_bounds__(256) void cross_meet_kernel(CrossArgs a, int rows_of_tile) {
  const int n_rows = a.group * a.q_tokens;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, per_unit = (long long)n_rows * (D / 4);
  const long long unit = i / per_unit;
  if (unit >= a.n_units) return;
  const int rest = (int)(i - unit * per_unit), row = rest / (D / 4), c = rest % (D / 4);
  const int tile = row / rows_of_tile, local = row - tile * rows_of_tile;
  const float* from = a.workspace + (unit * a.row_tiles + tile) * a.splits * (long long)rows::partial_floats(rows_of_tile, D);
  // (a few runs at a time, their loads under way together)
  constexpr int kAtOnce = 8;
  float top = -INFINITY, total = 0.f;
  rows::f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.splits; s0 += kAtOnce) {
    float2 st[kAtOnce];
    rows::f32x4 y[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float* p = from + (long long)min(s0 + i, a.splits - 1) * rows::partial_floats(rows_of_tile, D);
      st[i] = *reinterpret_cast<const float2*>(p + rows_of_tile * D + 2 * local);
      y[i] = *reinterpret_cast<const rows::f32x4*>(p + local * D + 4 * c);
      if (s0 + i >= a.splits) st[i].x = -INFINITY;
    }
    float new_top = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) new_top = fmaxf(new_top, st[i].x);
    const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - new_top);
    total *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] *= old;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float w = st[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[i].x - new_top);  // (a run without keys: 0)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(w, y[i][e], sum[e]);
      total = fmaf(w, st[i].y, total);
    }
    top = new_top;
  }
  const float inv = total > 0.f ? 1.0f / total : 0.f;
  rows::bf16x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (__bf16)(sum[e] * inv);
  const unsigned b = (unsigned)unit / (unsigned)a.kv_heads, g = (unsigned)unit - b * a.kv_heads;
  const int head = row / a.q_tokens, token = row - head * a.q_tokens;
  *reinterpret_cast<rows::bf16x4*>(a.o + b * a.o_map.batch + ((long long)g * a.group + head) * a.o_map.head + token * a.o_map.tok + 8 * c) = w;
}

template <int D, int kTeamWaves, int kTeams, int kMinWavesPerSimd, int kBits = 16>
hipError_t go(CrossArgs& a, hipStream_t st) {
  const int n_rows = a.group * a.q_tokens;
  a.row_tiles = (n_rows + 32 * kTeamWaves - 1) / (32 * kTeamWaves);
  const int tiles = a.row_tiles * a.splits;
  a.n_whole = whole_units(a.n_units, tiles, kMostWhole);
  hipLaunchKernelGGL((cross_kernel<D, kTeamWaves, kTeams, kMinWavesPerSimd, kBits>), dim3(tiles == 1 ? a.n_units : placed_grid(a.n_units, tiles, a.n_whole)),
                     dim3(64 * kTeamWaves * kTeams), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const long long lanes = (long long)a.n_units * n_rows * (D / 4);
  hipLaunchKernelGGL(cross_meet_kernel<D>, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, st, a, 32 * kTeamWaves);
  return hipGetLastError();
}

}  // namespace

static rows::Division division(bool four_bits, int head_dim, int units, int rows, int kv_tokens) {
  return four_bits ? rows::divide4(head_dim, units, rows, kv_tokens, 48) : rows::divide(head_dim, units, rows, kv_tokens);
}

static uint64_t workspace_bytes(bool four_bits, int batch, int heads, int kv_heads, int head_dim, int q_tokens, int kv_tokens) {
  const int units = batch * kv_heads, rows = heads / kv_heads * q_tokens;
  if (units == 0 || rows == 0 || kv_tokens == 0) return 0;
  const rows::Division d = division(four_bits, head_dim, units, rows, kv_tokens);
  if (d.splits == 1) return 0;
  const uint64_t row_tiles = (rows + 32 * d.team_waves - 1) / (32 * d.team_waves);
  return (uint64_t)units * row_tiles * d.splits * rows::partial_floats(32 * d.team_waves, head_dim) * sizeof(float);
}

uint64_t cross_workspace_bytes(int batch, int heads, int kv_heads, int head_dim, int q_tokens, int kv_tokens) {
  return workspace_bytes(false, batch, heads, kv_heads, head_dim, q_tokens, kv_tokens);
}
uint64_t cross_workspace_bytes4(int batch, int heads, int kv_heads, int head_dim, int q_tokens, int kv_tokens) {
  return workspace_bytes(true, batch, heads, kv_heads, head_dim, q_tokens, kv_tokens);
}

hipError_t launch_cross(const CrossCall& c, hipStream_t st) {
  CrossArgs a{};
  a.q = (const char*)c.q;
  a.k = (const char*)c.k;
  a.v = (const char*)c.v;
  a.o = (char*)c.o;
  a.q_map = c.q_map;
  a.k_map = c.k_map;
  a.v_map = c.v_map;
  a.o_map = c.o_map;
  a.lengths = c.lengths;
  a.offsets = c.offsets;
  a.kv_rows = c.kv_rows;
  a.workspace = c.workspace;
  a.scale_log2e = c.softmax_scale * 1.4426950408889634f;
  a.kv_heads = c.kv_heads;
  a.group = c.heads / c.kv_heads;
  a.q_tokens = c.q_tokens;
  a.kv_tokens = c.kv_tokens;
  a.n_units = c.batch * c.kv_heads;
  if (c.four_bits) {
    const long long units = c.offsets ? c.kv_heads : a.n_units;
    a.held_rows = c.offsets ? c.kv_rows : c.kv_tokens;
    a.groups_at = units * a.held_rows * (c.head_dim / 2);
  }
  if (a.n_units == 0 || a.group * a.q_tokens == 0) return hipSuccess;
  const rows::Division d = division(c.four_bits, c.head_dim, a.n_units, a.group * a.q_tokens, a.kv_tokens);
  a.splits = a.workspace ? d.splits : 1;
  if (c.four_bits) {
    if (c.head_dim == 64) {
      if (d.team_waves == 1) return d.teams == 1 ? go<64, 1, 1, 3, 4>(a, st) : d.teams == 4 ? go<64, 1, 4, 3, 4>(a, st) : go<64, 1, 8, 2, 4>(a, st);
      return d.team_waves == 4 ? go<64, 4, 1, 4, 4>(a, st) : go<64, 8, 1, 4, 4>(a, st);
    }
    if (d.team_waves == 1) return d.teams == 1 ? go<128, 1, 1, 2, 4>(a, st) : d.teams == 4 ? go<128, 1, 4, 2, 4>(a, st) : go<128, 1, 8, 2, 4>(a, st);
    return d.team_waves == 4 ? go<128, 4, 1, 3, 4>(a, st) : go<128, 8, 1, 2, 4>(a, st);
  }
  if (c.head_dim == 64) {
    if (d.team_waves == 1) return d.teams == 1 ? go<64, 1, 1, 4>(a, st) : go<64, 1, 4, 4>(a, st);
    return d.team_waves == 4 ? go<64, 4, 1, 4>(a, st) : go<64, 8, 1, 4>(a, st);
  }
  if (d.team_waves == 1) return d.teams == 1 ? go<128, 1, 1, 2>(a, st) : go<128, 1, 4, 2>(a, st);
  return go<128, 4, 1, 2>(a, st);
}

}  // namespace amskv
