// An encoder's K and V put into 4 bits, and read back (codes.hpp has the format; the attention over them is cross.hip).
//
// A lane has 8 channels of a row: 16 bytes of bf16, 4 bytes of codes, and a group's 4 lanes are a quad, so its largest element takes two
// steps on the vector ALU.  A wave's lanes follow the rows of one unit, whose codes lie back to back; a lane has kRows of them under way.
// Bound: HBM and, at the smallest, a launch.  K and V of 96 packed prompts of up to 512 states, 16 heads, head dim 128: written 45 to 56 us (4.5 to
// 5.7 TB/s read + write), read back 41 (6.2); 8 documents of up to 16000, 8 heads, 101 to 113 (5.3 to 5.9) and 92 (6.5); 77 states of a short prompt
// 2.9 and 2.6.  A workgroup has 512 bytes of a row, of heads side by side in a token-major tensor, and the heads of a block of rows go to
// neighbouring workgroups: with one head to a workgroup 63 to 71, 135 to 140 us.  What is read back goes past the caches: 8 x 16000 states of 8
// heads 126 -> 93 us, 96 x 250 of 16, head dim 64, 19.2 -> 17.6.  With a kernel behind that reads it the two differ by a tenth either way: K and V of
// 8 MB both kernels 11.1 us past the caches and 11.9 through them, 34 MB 26.9 and 24.6, 201 MB 121.8 and 118.5, 524 MB 303 both.  (Loads past
// them: 42.7 us for 35.8 where a projection has just made the states.)
#include "codes.hpp"

namespace amskv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kRows = 4;               // rows of a lane under way
constexpr int kSideBySide = 512;       // bytes of a row that a workgroup has of several heads
constexpr unsigned kMostGroups = 1 << 20;  // workgroups; beyond that they take several blocks of rows

struct HoldArgs {
  char *x[2];
  unsigned char* held[2];
  RowMap map[2];
  const int *lengths, *offsets;
  long long rows, groups_at;  // rows of a unit, bytes of codes
  unsigned blocks, all_blocks;  // blocks of rows to a unit, of all groups of heads
  int kv_heads, batch, kv_tokens;
  int side;  // 2^side heads side by side in a workgroup, a divisor of kv_heads
};

// rows [first, end) of a unit that hold states
__device__ __forceinline__ void live_rows(const HoldArgs& a, unsigned b, long long& first, long long& end) {
  first = 0;
  end = a.rows;
  if (a.offsets != nullptr) {
    first = min(max((long long)a.offsets[0], 0ll), a.rows);
    end = min(max((long long)a.offsets[a.batch], 0ll), a.rows);
  } else if (a.lengths != nullptr) {
    end = min(max(a.lengths[b], 0), a.kv_tokens);
  }
}

// the largest of a quad's four values
__device__ __forceinline__ float quad_max(float m) {
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0xB1, 0xf, 0xf, true)));  // quad_perm 1 0 3 2
  return fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x4E, 0xf, 0xf, true)));  // 2 3 0 1
}

template <int D, bool kBack>
__global__ __launch_bounds__(256) void hold_kernel(HoldArgs a) {
  fetch_arguments<sizeof(HoldArgs)>();
  constexpr int kLanes = D / 8;               // of a row
  const int at_once = 256 / kLanes >> a.side;  // rows of a workgroup at a time
  const int tensor = blockIdx.y;
  if (a.x[tensor] == nullptr) return;
  const int c = threadIdx.x % kLanes, of_all = threadIdx.x / kLanes, r = of_all >> a.side;
  const unsigned head = of_all & ((1 << a.side) - 1), groups_of_heads = (unsigned)a.kv_heads >> a.side;
  const RowMap& m = a.map[tensor];
  for (unsigned block = blockIdx.x; block < a.all_blocks; block += gridDim.x) {
    // the heads of a block of rows, which lie side by side in a token-major tensor, go to workgroups of one time
    const unsigned rest = block / groups_of_heads, g = ((block - rest * groups_of_heads) << a.side) + head, b = rest / a.blocks;
    const long long row0 = (long long)(rest - b * a.blocks) * (at_once * kRows) + r, unit = (long long)b * a.kv_heads + g;
    long long first, end;
    live_rows(a, b, first, end);
    char* x = a.x[tensor] + b * m.batch + g * m.head + 16 * c;
    unsigned char* codes = a.held[tensor] + unit * a.rows * (D / 2) + 4 * c;
    unsigned char* groups = a.held[tensor] + a.groups_at + unit * a.rows * (D / AMSKV_KV4_GROUP) + c / 4;
    auto live = [&](int i) {
      const long long row = row0 + i * at_once;
      return row >= first && row < end;
    };
    if constexpr (kBack) {
      unsigned in[kRows], byte[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (live(i)) {
          const long long row = row0 + i * at_once;
          in[i] = *reinterpret_cast<const unsigned*>(codes + row * (D / 2));
          byte[i] = groups[row * (D / AMSKV_KV4_GROUP)];
        }
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (live(i)) __builtin_nontemporal_store(values4(in[i], power_of_byte(byte[i])), reinterpret_cast<u32x4*>(x + (row0 + i * at_once) * m.tok));
    } else {
      bf16x8 in[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        in[i] = {};
        if (live(i)) in[i] = *reinterpret_cast<const bf16x8*>(x + (row0 + i * at_once) * m.tok);
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        float y[8], largest = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] = (float)in[i][e];
          largest = fmaxf(largest, fabsf(y[e]));
        }
        const unsigned byte = group_exponent(quad_max(largest)) + 127;
        if (live(i)) {
          const long long row = row0 + i * at_once;
          *reinterpret_cast<unsigned*>(codes + row * (D / 2)) = codes4(y, power_of_byte(byte));
          if (c % 4 == 0) groups[row * (D / AMSKV_KV4_GROUP)] = (unsigned char)byte;
        }
      }
    }
  }
}

template <bool kBack>
hipError_t go(const HoldCall& c, hipStream_t st) {
  HoldArgs a{};
  a.x[0] = (char*)c.k;
  a.x[1] = (char*)c.v;
  a.held[0] = c.k_held;
  a.held[1] = c.v_held;
  a.map[0] = c.k_map;
  a.map[1] = c.v_map;
  a.lengths = c.lengths;
  a.offsets = c.offsets;
  a.rows = c.offsets ? c.kv_rows : c.kv_tokens;
  const long long units = c.offsets ? c.kv_heads : (long long)c.batch * c.kv_heads;
  a.groups_at = units * a.rows * (c.head_dim / 2);
  a.kv_heads = c.kv_heads;
  a.batch = c.batch;
  a.kv_tokens = c.kv_tokens;
  while ((c.head_dim * 2 << a.side) < kSideBySide && c.kv_heads % (2 << a.side) == 0) ++a.side;
  const int per = (256 / (c.head_dim / 8) >> a.side) * kRows;
  const long long blocks = (a.rows + per - 1) / per, all = (units >> a.side) * blocks;
  if (all > 0x7fffffffll) return hipErrorInvalidValue;  // (the loop's counter)
  a.blocks = (unsigned)blocks;
  a.all_blocks = (unsigned)all;
  if (a.all_blocks == 0) return hipSuccess;
  const dim3 grid(a.all_blocks < kMostGroups ? a.all_blocks : kMostGroups, 2);
  auto kernel = c.head_dim == 64 ? hold_kernel<64, kBack> : hold_kernel<128, kBack>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_hold(const HoldCall& c, hipStream_t st) { return go<false>(c, st); }
hipError_t launch_unhold(const HoldCall& c, hipStream_t st) { return go<true>(c, st); }

}  // namespace amskv
