// What happens to the tensors of a scale between the projection and the attention (the step that Section 3.1's attention takes
// as given): queries and keys turned by their tokens' positions, keys and values put into the cache, in its own type or in 8
// bits.  And the other two kernels of an 8-bit cache that only move data: compaction and read-back.
//
// Turn.  Pair (x, y) -> (x c - y s, y c + x s), c and s from a table of the scale's tokens.  Both channels of a pair belong to one
// lane: an item is 16 channels of a row -- 8 pairs -- held as two pieces of 8, which are pieces j and j + rot_dim/16 of the
// row with AMSKV_ROPE_HALF and pieces 2j and 2j + 1 otherwise (pairs inside the pieces, channels that do not turn, tensors that do
// not).  Every product is rounded by itself: the result does not hang on where a compiler fuses, and an 8-bit code, which
// jumps by 2^-4 where fp32 differs in its last bit, is the same wherever the formula is evaluated in fp32.
//
// 8 bits.  A block of 16 tokens x D shares the least power of two 2^e, e >= -100, with max |x| <= 448 * 2^e; x is held as the e4m3
// number next to x * 2^-e (v_cvt_pk_fp8_f32 rounds to nearest, ties to even; nothing is beyond 448).  A power of two because a
// code times it is a bf16 number: the attention gets exactly the held values, and e4m3, a floating format over 2^17, would gain
// nothing from a finer scale.  A wave owns the 16 tokens of a block, 4 lanes to a row, so the block's maximum is one
// reduction over its lanes; scales of 8 tokens and fewer put 2 to 16 heads into a wave.
//
// Bound: HBM at the fine scales, 4.5 to 5.1 TB/s read + write (a device copy 4.9): 8 x 4096 rows of 16 heads out of a fused projection, head
// dim 128 59 us (270 MB); K and V of 3840 (b,h), 169 tokens, head dim 64, to codes 48.6 us (249 MB); Q and K turned, K and V to codes,
// 960 (b,h), 256 tokens 31.8 us (157 MB).  Launch and the latency of arguments, rows and stores at the coarse ones: 2.4 to 5 us.
#include "codes.hpp"
#include "take_choice.hpp"

namespace amskv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kOwners = 8;

struct Piece {
  float x[8];
};

__device__ __forceinline__ Piece load8(const __bf16* p) {
  const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
  Piece r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.x[i] = (float)v[i];
  return r;
}
__device__ __forceinline__ Piece load8(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
  return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void store8(__bf16* p, const Piece& v) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)v.x[i];
  *reinterpret_cast<bf16x8*>(p) = r;
}
__device__ __forceinline__ void store8(float* p, const Piece& v) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v.x[0], v.x[1], v.x[2], v.x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v.x[4], v.x[5], v.x[6], v.x[7]};
}

__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
  const float xc = x * c, ys = y * s, yc = y * c, xs = x * s;
  x = xc - ys;
  y = yc + xs;
}

// the 8 pairs of an item; t: their (c, s); back: the sign bit to turn by the other angle, or 0
__device__ __forceinline__ void turn_item(Piece& a, Piece& b, const float* t, bool half, int back) {
  auto s = [&](int i) { return __int_as_float(__float_as_int(t[2 * i + 1]) ^ back); };
  if (half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(a.x[i], b.x[i], t[2 * i], s(i));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn(a.x[2 * i], a.x[2 * i + 1], t[2 * i], s(i));
      turn(b.x[2 * i], b.x[2 * i + 1], t[8 + 2 * i], s(4 + i));
    }
  }
}

__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// e of a block whose largest magnitude is m (finite): the least e >= -100 with m <= 448 * 2^e = 1.75 * 2^(e + 8)
__device__ __forceinline__ int block_exponent(float m) {
  const int bits = __float_as_int(m);
  const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return max(e, -100);
}

__device__ __forceinline__ u32x2 codes8(const Piece& p, float by) {
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(p.x[4 * w] * by, p.x[4 * w + 1] * by, 0, false);
    r[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(p.x[4 * w + 2] * by, p.x[4 * w + 3] * by, c, true);
  }
  return r;
}

struct TakeArgs {
  int which[3];        // tensor of each blockIdx.y
  const char* src[3];  // K, V, Q
  char* dst[3];
  RowMap from[3], to[3];
  float* scales[2];
  const float* table;
  long long table_batch, cap_tokens;
  int dst_new, pieces_turned, half, inverse;
  int batch, heads, tokens, blocks, row_shift, groups, heads_per_wave;
};

// One wave: a block of 16 tokens of heads [first, end) of batch element b, in 16 row slots of 4 lanes.  A slot is a token of one
// head (T > 8) or of one of 16 / 2^row_shift heads at once.
template <typename T, int D, bool kEight>
__device__ __forceinline__ void take_block(const TakeArgs& a, int tensor, unsigned b, int block, int first, int end) {
  constexpr int kItems = D / 64;  // per lane
  const int lane = threadIdx.x & 63;
  const int slot = lane >> 2, rows = 1 << a.row_shift, together = 16 >> a.row_shift;
  const int t = block * 16 + (slot & (rows - 1));
  const bool turns = a.table != nullptr && tensor != 1;

  int at[kItems][2];  // first channels of the item's two pieces
  float tab[kItems][16];
  bool turned[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int j = (lane & 3) + 4 * i;
    turned[i] = turns && 2 * j < a.pieces_turned;
    at[i][0] = 8 * (turned[i] && a.half ? j : 2 * j);
    at[i][1] = 8 * (turned[i] && a.half ? j + (a.pieces_turned >> 1) : 2 * j + 1);
    if (turned[i] && t < a.tokens) {
      const float* p = a.table + b * a.table_batch + ((long long)t * (a.pieces_turned * 4) + 8 * j) * 2;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(p + 4 * v);
#pragma unroll
        for (int e = 0; e < 4; ++e) tab[i][4 * v + e] = x[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) tab[i][e] = 0.f;
    }
  }
  for (int h0 = first; h0 < end; h0 += together) {
    const int h = h0 + (slot >> a.row_shift);
    const bool live = t < a.tokens && h < end;
    Piece x[kItems][2];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][p].x[e] = 0.f;
      if (live) {
        const T* row = reinterpret_cast<const T*>(a.src[tensor] + b * a.from[tensor].batch + h * a.from[tensor].head + t * a.from[tensor].tok);
        x[i][0] = load8(row + at[i][0]);
        x[i][1] = load8(row + at[i][1]);
      }
    }
    int back = 0;
    if constexpr (!kEight) {
      back = a.inverse ? (int)0x80000000 : 0;
      asm volatile("" : "+v"(back));  // (formed here, so that the rows are asked for before the table is waited for)
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (turned[i]) turn_item(x[i][0], x[i][1], tab[i], a.half, back);
    if (kEight && tensor < 2) {
#pragma unroll
      for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[i][p].x[e]));
      for (int step = 1; step < 4 * rows; step <<= 1) m = fmaxf(m, __shfl_xor(m, step, 64));
      const int e = block_exponent(m);
      const float by = power_of_two(-e);
      if (e == 120) {  // 256 * 2^120, where the largest bf16 numbers would be rounded to, is none
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int c = 0; c < 8; ++c) x[i][p].x[c] = fminf(fmaxf(x[i][p].x[c], -0x1.ep127f), 0x1.ep127f);
      }
      if (live) {
        const long long bh = (long long)b * a.heads + h;
        const long long token = a.dst_new + t;
        char* row = a.dst[tensor] + (bh * a.cap_tokens + token) * D;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          *reinterpret_cast<u32x2*>(row + at[i][0]) = codes8(x[i][0], by);
          *reinterpret_cast<u32x2*>(row + at[i][1]) = codes8(x[i][1], by);
        }
        if ((lane & (4 * rows - 1)) == 0) a.scales[tensor][bh * (a.cap_tokens / AMSKV_KV8_BLOCK) + token / AMSKV_KV8_BLOCK] = power_of_two(e);
      }
    } else if (live) {
      T* row = reinterpret_cast<T*>(a.dst[tensor] + b * a.to[tensor].batch + h * a.to[tensor].head + t * a.to[tensor].tok);
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        store8(row + at[i][0], x[i][0]);
        store8(row + at[i][1], x[i][1]);
      }
    }
  }
}

template <typename T, int D, bool kEight>
__global__ __launch_bounds__(64 * kWaves) void take_kernel(TakeArgs a) {
  fetch_arguments<sizeof(TakeArgs)>();
  const unsigned wave = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = wave / (unsigned)a.groups, group = wave - unit * a.groups;
  const unsigned b = unit / (unsigned)a.blocks, block = unit - b * a.blocks;
  if (b >= (unsigned)a.batch) return;
  const int first = group * a.heads_per_wave;
  take_block<T, D, kEight>(a, a.which[blockIdx.y], b, block, first, min(first + a.heads_per_wave, a.heads));
}

// Blocks that slide to lower places, in the order of their offsets: begin[i] .. begin[i+1] of the list come from src[i] and go to
// dst[i] (all in blocks).
struct BlockList {
  int32_t n, total;
  int32_t begin[AMSKV_MAX_SCALES], src[AMSKV_MAX_SCALES], dst[AMSKV_MAX_SCALES];
};
// The codes and scales of one (b,h) of one tensor slide, a pass at a time, by all threads of the workgroup: everything a pass reads
// has arrived before any of it is written, and it is written below where it and all that follows is read.  Behind the last
// barrier nothing is left to read.  Bound: HBM where the (b,h) are many, else one workgroup's passes, a trip to memory each: 3 to 7 us
// at the coarse scales, 21.6 us at the last of ten scales, 960 (b,h), head dim 64.
template <int D>
__device__ __forceinline__ void slide(unsigned char* rows, float* scales, const BlockList& list) {
  constexpr int kChunks = 4;  // of 16 bytes a thread and pass; a block of 16 tokens is D of them
  auto place = [&](int i, int& src, int& dst) {
    src = dst = 0;
    for (int r = 0; r < list.n; ++r)
      if (i >= list.begin[r]) {
        src = list.src[r] + i - list.begin[r];
        dst = list.dst[r] + i - list.begin[r];
      }
  };
  const long long total = (long long)list.total * D;
  for (long long c0 = 0; c0 < total; c0 += (long long)blockDim.x * kChunks) {
    u32x4 buf[kChunks];
    long long to[kChunks];
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      const long long i = c0 + u * (int)blockDim.x + (int)threadIdx.x;
      to[u] = -1;
      if (i < total) {
        int src, dst;
        place((int)(i / D), src, dst);
        buf[u] = *reinterpret_cast<const u32x4*>(rows + ((long long)src * D + i % D) * 16);
        to[u] = ((long long)dst * D + i % D) * 16;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kChunks; ++u)
      if (to[u] >= 0) *reinterpret_cast<u32x4*>(rows + to[u]) = buf[u];
  }
  for (int c0 = 0; c0 < list.total; c0 += (int)blockDim.x) {
    const int i = c0 + (int)threadIdx.x;
    int src = 0, dst = 0;
    float x = 0.f;
    if (i < list.total) {
      place(i, src, dst);
      x = scales[src];
    }
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(x) : : "memory");
    __syncthreads();
    if (i < list.total) scales[dst] = x;
  }
}

template <int D>
__global__ __launch_bounds__(1024) void move_codes_kernel(Codes c, long long cap_tokens, BlockList list) {
  fetch_arguments<sizeof(Codes) + 8 + sizeof(BlockList)>();
  const long long bh = blockIdx.x;
  slide<D>((blockIdx.y ? c.v : c.k) + bh * cap_tokens * D, (blockIdx.y ? c.v_scale : c.k_scale) + bh * (cap_tokens / AMSKV_KV8_BLOCK), list);
}

// Both in one launch: the workgroup that owns a (b,h) of a tensor slides what stays of it, then its waves take the blocks of the
// new scale, whose place may be where the survivors lay.
template <int D>
__global__ __launch_bounds__(64 * kOwners) void slide_and_take_kernel(TakeArgs a, BlockList list) {
  fetch_arguments<sizeof(TakeArgs) + sizeof(BlockList)>();
  const int tensor = a.which[blockIdx.y];
  const long long bh = blockIdx.x;
  const unsigned b = (unsigned)bh / (unsigned)a.heads;
  const int h = (int)(bh - (long long)b * a.heads);
  if (tensor < 2) slide<D>((unsigned char*)a.dst[tensor] + bh * a.cap_tokens * D, a.scales[tensor] + bh * (a.cap_tokens / AMSKV_KV8_BLOCK), list);
  for (int block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); block < a.blocks; block += kOwners)
    take_block<__bf16, D, true>(a, tensor, b, block, h, h + 1);
}

BlockList block_list(const MoveList& mv) {
  BlockList list{};
  for (int i = 0; i < mv.n; ++i) {
    list.begin[list.n] = list.total;
    list.src[list.n] = mv.src[i] / AMSKV_KV8_BLOCK;
    list.dst[list.n] = mv.dst[i] / AMSKV_KV8_BLOCK;
    list.total += mv.len[i] / AMSKV_KV8_BLOCK;
    ++list.n;
  }
  return list;
}

template <typename T, int D>
hipError_t take(const Take& t, hipStream_t st) {
  TakeArgs a{};
  const void* src[3] = {t.k, t.v, t.q};
  int n = 0;
  for (int i = 0; i < 3; ++i)
    if (src[i]) a.which[n++] = i;
  if (n == 0 || t.batch == 0 || t.heads == 0 || t.tokens == 0) return hipSuccess;
  for (int i = 0; i < 3; ++i) {
    a.src[i] = (const char*)src[i];
    a.from[i] = i == 2 ? t.q_map : t.kv_map;
    a.to[i] = i == 2 ? t.q_out_map : t.out_map;
  }
  a.dst[0] = t.eight_bits ? (char*)t.codes.k : (char*)t.k_out;
  a.dst[1] = t.eight_bits ? (char*)t.codes.v : (char*)t.v_out;
  a.dst[2] = (char*)t.q_out;
  a.scales[0] = t.codes.k_scale;
  a.scales[1] = t.codes.v_scale;
  a.table = t.table;
  a.table_batch = t.table_batch;
  a.cap_tokens = t.cap_tokens;
  a.dst_new = t.dst_new;
  a.pieces_turned = t.table ? t.rot_dim / 8 : 0;
  a.half = t.pairing == AMSKV_ROPE_HALF;
  a.inverse = t.inverse;
  a.batch = t.batch;
  a.heads = t.heads;
  a.tokens = t.tokens;
  a.blocks = (t.tokens + 15) / 16;
  a.row_shift = t.tokens > 8 ? 4 : t.tokens > 4 ? 3 : t.tokens > 2 ? 2 : t.tokens > 1 ? 1 : 0;
  const int together = 16 >> a.row_shift;
  const long long waves = (long long)t.batch * a.blocks * ((t.heads + together - 1) / together);
  a.heads_per_wave = together * (waves > 16384 ? 4 : 1);
  a.groups = (t.heads + a.heads_per_wave - 1) / a.heads_per_wave;
  const long long grid = ((long long)t.batch * a.blocks * a.groups + kWaves - 1) / kWaves;
  if (grid > 0xffffff) return hipErrorInvalidValue;  // 2^32 threads
  const dim3 g((unsigned)grid, n), block(64 * kWaves);
  if constexpr (sizeof(T) == 2) {
    if (t.eight_bits && t.moves != nullptr && t.moves->n > 0) {
      const BlockList list = block_list(*t.moves);
      if (slides_at_once(t.batch * t.heads, t.tokens, list.total, D)) {
        hipLaunchKernelGGL((slide_and_take_kernel<D>), dim3(t.batch * t.heads, n), dim3(64 * kOwners), 0, st, a, list);
        return hipGetLastError();
      }
      const hipError_t e = launch_move_codes(t.codes, t.batch * t.heads, t.head_dim, t.cap_tokens, *t.moves, st);
      if (e != hipSuccess) return e;
    }
    if (t.eight_bits) {
      hipLaunchKernelGGL((take_kernel<T, D, true>), g, block, 0, st, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((take_kernel<T, D, false>), g, block, 0, st, a);
  return hipGetLastError();
}

// Angles in 64 bits, one thread to a pair of a token; frequencies come with the arguments.  Bound: the vector pipe, on which sine and
// cosine of a double take some 200 instructions (300000 tokens of 64 pairs 83 us, 1.9 TB/s written; 4096 tokens 3.3 us, one 2.3).
struct Frequencies {
  double f[64];
};
__global__ __launch_bounds__(256) void rope_table_kernel(const double* __restrict__ positions, float2* __restrict__ table, int pairs, int axes,
                                                         double amplitude, long long total, Frequencies f) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const long long token = i / pairs;
  const int pair = (int)(i - token * pairs), per_axis = pairs / axes, axis = pair / per_axis;
  double s, c;
  sincos(positions[token * axes + axis] * f.f[pair - axis * per_axis], &s, &c);
  table[i] = make_float2((float)(amplitude * c), (float)(amplitude * s));
}

// The values of the resident segments, ascending and back to back, as bf16 [BH][T_kept][D]; a lane takes 16 channels of a row.
// Bound: HBM (960 (b,h), up to 640 tokens, head dim 64: 44 us, about 5 TB/s).
template <int D>
__global__ __launch_bounds__(256) void export_codes_kernel(Codes c, __bf16* __restrict__ k_out, __bf16* __restrict__ v_out, long long cap_tokens,
                                                           SegTable seg, ExtKV ext_kv, RowMap ext_map, int heads, int parts, int units,
                                                           int n_bh) {
  __bf16* out = blockIdx.y ? v_out : k_out;
  if (!out) return;
  constexpr int kPer = D / 16;
  const unsigned unit = blockIdx.x / (unsigned)parts, part = blockIdx.x - unit * parts;
  const long long bh = (long long)blockIdx.z * units + unit;
  if (bh >= n_bh) return;
  const long long i = (long long)part * 256 + threadIdx.x;
  const int j = (int)(i / kPer), piece = (int)(i % kPer);
  if (j >= seg.total) return;
  bool ext;
  const long long at = locate_row(seg, j, ext);
  u32x4 w[2];
  if (ext) {
    const char* row = (const char*)(blockIdx.y ? ext_kv.v : ext_kv.k) + unit_offset(ext_map, bh, heads) + at * ext_map.tok + piece * 32;
    w[0] = *reinterpret_cast<const u32x4*>(row);
    w[1] = *reinterpret_cast<const u32x4*>(row + 16);
  } else {
    const unsigned char* codes = (blockIdx.y ? c.v : c.k) + (bh * cap_tokens + at) * D + piece * 16;
    const u32x4 x = *reinterpret_cast<const u32x4*>(codes);
    const float scale = (blockIdx.y ? c.v_scale : c.k_scale)[(bh * cap_tokens + at) / AMSKV_KV8_BLOCK];
    w[0] = values8(u32x2{x[0], x[1]}, scale);
    w[1] = values8(u32x2{x[2], x[3]}, scale);
  }
  u32x4* to = reinterpret_cast<u32x4*>(out + (bh * seg.total + j) * D + piece * 16);
  to[0] = w[0];
  to[1] = w[1];
}

}  // namespace

hipError_t launch_take(const Take& t, hipStream_t st) {
  if (t.dtype == AMSKV_DTYPE_F32) return t.head_dim == 64 ? take<float, 64>(t, st) : take<float, 128>(t, st);
  return t.head_dim == 64 ? take<__bf16, 64>(t, st) : take<__bf16, 128>(t, st);
}

hipError_t launch_rope_table(const double* frequency, int pairs, int axes, double amplitude, const double* positions, int64_t n,
                             float* table, hipStream_t st) {
  Frequencies f{};
  for (int i = 0; i < pairs / axes; ++i) f.f[i] = frequency[i];
  const long long total = n * pairs;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, positions, (float2*)table, pairs, axes,
                     amplitude, total, f);
  return hipGetLastError();
}

hipError_t launch_move_codes(const Codes& c, int bh, int head_dim, int64_t cap_tokens, const MoveList& mv, hipStream_t st) {
  const BlockList list = block_list(mv);
  if (list.total == 0) return hipSuccess;
  const int threads = move_threads(list.total, head_dim, bh);
  auto kernel = head_dim == 64 ? move_codes_kernel<64> : move_codes_kernel<128>;
  hipLaunchKernelGGL(kernel, dim3(bh, 2), dim3(threads), 0, st, c, (long long)cap_tokens, list);
  return hipGetLastError();
}

hipError_t launch_export_codes(const Codes& c, void* k_out, void* v_out, int bh, int head_dim, int64_t cap_tokens, const SegTable& seg,
                               const ExtKV& ext, const RowMap& ext_map, int heads, hipStream_t st) {
  if (seg.total == 0) return hipSuccess;
  const ExportGrid g = export_grid(bh, seg.total, head_dim);
  if (g.layers > 65535) return hipErrorInvalidValue;
  auto kernel = head_dim == 64 ? export_codes_kernel<64> : export_codes_kernel<128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(g.parts * g.units), 2, (unsigned)g.layers), dim3(256), 0, st, c, (__bf16*)k_out, (__bf16*)v_out,
                     (long long)cap_tokens, seg, ext, ext_map, heads, (int)g.parts, (int)g.units, bh);
  return hipGetLastError();
}

}  // namespace amskv
