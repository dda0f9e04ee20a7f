// Attention of up to 32 * kTeamWaves query rows over keys in 4 bits, for teams of waves: attend_rows.hpp's formulation with K's codes as
// they are.
//
// The matrix cores take e2m1 numbers with a power of two to every 32 along the sum: S^T = K Q^T is formed by
// v_mfma_scale_f32_32x32x64_f8f6f4 from K's codes and powers straight out of LDS, a quarter of bf16's bytes there and no conversion.  Its
// other operand has 8 bits, and Q, whose numbers have 8 significant bits, is the sum of two e4m3 numbers (4 each), made once for a
// workgroup: 32 channels with largest element m, 2^a the least power with m <= 448 * 2^a, are hi * 2^a + lo * 2^(a - 4), hi the number
// nearest to q * 2^-a, lo what is left.  That is q itself: hi leaves at most half of its step, a sign and 4 bits.  (e4m3's own range ends it:
// elements below 2^-6 * 2^a, 2^-14 of m, may be off by 2^-14 * 2^a, 2^-21 of m.)  With 8 bits the products of 8 neighbouring channels are cut
// to units of 2^-13 of the power of two of their largest before they are added up in fp32 (as measured; products of 6 bits lie within that):
// a product, of 6 bits itself, loses something if it is 2^-8 of the largest and less.  Parts of 6 bits lose nothing there, but have the
// range of 4 bits and lose Q's small channels beside a large one.  Emulated, scores of standard deviation 9, outputs off by (rms of their size):
//                                                          Q itself  here    two e2m3  e4m3 + e3m2  three e2m3  bf16(Q * factor)
//   plain                                                  0.0015    0.0015  0.0026    0.0015       0.0015      0.0045
//   a channel of Q 30 times the others                     0.0015    0.0015  0.0071    0.0022       0.0015      0.0038
//   100 times                                              0.0019    0.0024  0.0097    0.0035       0.0019      0.0023
//   a channel of Q 30 times, K there as much smaller       0.0015    0.0015  0.014     0.0035       0.0016      0.0047
//   300 times                                              0.0016    0.0016  0.14      0.027        0.0074      0.0052
// and as measured (us; 64 units 4096 x 6421 and 2304 x 3925 at head dim 128, 3840 units 256 x 530 at 64): here 679, 263, 190; two e2m3 618, 242,
// 174; three 679, 269, 194; four, which lose nothing in either way, 728, 316, 198.  A product of both parts takes 57 ns of a SIMD for 64 channels, bf16's
// 74 (a part of 6 bits 15).  V becomes bf16 on its way to LDS, once for all waves: weights in 6 bits would have to be split in two for
// every block, which takes the vector ALUs more (a conversion of 32 numbers 38 ns, back 33) than the matrix cores save.
//
// Bound, and what it measured.  Head dim 128, 64 units: the matrix pipes (0.57 of a SIMD's cycles) and the power they take, 4096 x 6421 by teams
// of eight 671 to 712 us (1.21 to 1.29 PFLOP/s; codes of 8 bits through bf16 784), 2304 x 3925 by teams of four 258 to 269, 576 x 1076 33.
// Head dim 64, 3840 units: the vector ALUs (0.66 of a SIMD's cycles, the matrix pipe 0.24), 256 x 530 187 to 195 us (with 256 of the keys read in
// place as bf16, by attend_rows.hpp, 193 to 206), x 2066 554 (0.94 PFLOP/s).
//
// kExt: rows of bf16 may follow the codes (a scale that is read in place); they are walked as in attend_rows.hpp, with Q as it is.
#pragma once
#include "attend_rows.hpp"

#if defined(__HIPCC__)
namespace amskv {
namespace rows {

typedef unsigned u32x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Q of a lane's row in two parts, the larger first, where an operand of 8 bits has its channels: 64 c + 16 h .. + 15, then 64 c + 32 + 16 h
// .. + 15; and the bytes of their powers, of channels 64 c + 32 h .. + 31 (c's in bytes 2 c and 2 c + 1).
template <int D>
struct QueryParts {
  u32x8 high[D / 64], low[D / 64];
  unsigned powers;
};
// words of channels 32 h .. + 31 to where that is
__device__ __forceinline__ u32x8 across(u32x8 x) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const auto s = __builtin_amdgcn_permlane32_swap(x[w], x[4 + w], false, false);
    x[w] = s[0];
    x[4 + w] = s[1];
  }
  return x;
}
// (Q is asked for before anything that has to be waited for)
template <int D>
__device__ __forceinline__ void load_query(u32x4 (&raw)[D / 64][4], const char* row, int h) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[c][i] = *reinterpret_cast<const u32x4*>(row + 128 * c + 64 * h + 16 * i);
}
// two numbers of Q less what is held of them, which a bf16 number is
__device__ __forceinline__ bf16x2 left_of(unsigned two, const f32x2& held) {
  const float x = __builtin_bit_cast(float, two << 16) - held[0], y = __builtin_bit_cast(float, two & 0xffff0000u) - held[1];
  return __builtin_bit_cast(bf16x2, __builtin_bit_cast(unsigned, x) >> 16 | (__builtin_bit_cast(unsigned, y) & 0xffff0000u));
}
template <int D>
__device__ __forceinline__ void split_query(QueryParts<D>& q, const u32x4 (&raw)[D / 64][4]) {
  q.powers = 0;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, raw[c][i / 4][i % 4] & 0x7fff7fffu));
    const int m = max((int)most[0], (int)most[1]);  // the bits of the largest magnitude; 448 = 1.75 * 2^8
    const int byte = max((m >> 7) - 8 + ((m & 0x7f) > 0x60 ? 1 : 0), 5);
    const float by = power_of_byte(byte), by_low = power_of_byte(byte - 4);
    // (0xff: NaN, which is what all scores of the row become)
    q.powers |= (m < 0x7f80 ? (unsigned)byte | (unsigned)(byte - 4) << 8 : 0xffffu) << (16 * c);
    u32x8 high, low;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const unsigned x = raw[c][w / 2][2 * (w % 2)], y = raw[c][w / 2][2 * (w % 2) + 1];
      i16x2 code = {0, 0}, left = {0, 0};
      code = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(code, __builtin_bit_cast(bf16x2, x), by, false);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(code, __builtin_bit_cast(bf16x2, y), by, true);
      high[w] = __builtin_bit_cast(unsigned, code);
      left = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(left, left_of(x, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(high[w], by, false)), by_low, false);
      left = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(left, left_of(y, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(high[w], by, true)), by_low, true);
      low[w] = __builtin_bit_cast(unsigned, left);
    }
    q.high[c] = across(high);
    q.low[c] = across(low);
  }
}

template <int D, int kTeamWaves, bool kExt>
struct FourBitTeam : Unit<D, kTeamWaves, 1, 4> {
  typedef Unit<D, kTeamWaves, 1, 4> Base;
  typedef typename Base::Result Result;
  typedef typename Base::Staged Staged;
  typedef typename Base::Aim Aim;
  typedef typename Base::Behind Behind;
  static constexpr int RB = Base::RB, KS = Base::KS, kTile = Base::kTile, kThreads = Base::kThreads;
  static constexpr int kRowK = D / 2;                   // bytes of a row of codes
  static constexpr int kPowers = kTile * kRowK;         // where the powers of a tile's K begin: 32 bytes to a row
  static constexpr int kOfK = kExt ? Base::kTensor : kPowers + 32 * kTile;
  static constexpr int kStage = kOfK + Base::kTensor;
  static constexpr int kLds = 4 * kStage;
  typedef QueryParts<D> Query;
  static_assert(kPowers + 32 * kTile <= kOfK && kThreads == 8 * kTile, "eight threads bring a row of K and of V");

  __device__ static __forceinline__ int tiles(const Keys& k) { return kExt ? Base::tiles(k) : Base::tiles_of_codes(k); }
  __device__ static __forceinline__ int valid(const Keys& k, int it) {
    return kExt ? Base::valid(k, it) : min(kTile, k.n_codes - it * kTile);
  }

  // ---- from memory to LDS.  A thread has an eighth of a row of K and the same of V: D / 8 channels each, and their powers.
  // Where chunk c (16 bytes) of a row of K's codes sits: reads of 8 rows then spread over all banks
  __device__ static __forceinline__ unsigned chunk_of_k(unsigned row, unsigned c) { return D == 64 ? c ^ ((row >> 3) & 1) : c ^ ((row >> 2) & 3); }
  __device__ static __forceinline__ void aim_codes(Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    const int first = it * kTile, last = k.n_codes - 1;
    member = Base::fresh(member);
    if (first >= a.end)  // a handful of times: the segment that holds `first`
      for (int g = 0; g < seg.n; ++g)
        if (first >= seg.virt_start[g]) {
          a.end = seg.virt_start[g] + seg.len[g];
          a.delta = seg.phys_off[g] - seg.virt_start[g];
        }
    const int j = min(first + (int)((unsigned)member / 8), last);
    a.row[0] = j + a.delta;
    if (min(first + kTile - 1, last) >= a.end)  // rows of several segments
      for (int g = 0; g < seg.n; ++g)
        if (j >= seg.virt_start[g]) a.row[0] = j + seg.phys_off[g] - seg.virt_start[g];
  }
  // (x[0]: K's codes, V's; x[1]: the powers of K's row, of V's piece)
  __device__ static __forceinline__ void fetch_codes(Staged& s, const Aim& a, const Keys& k, int thread) {
    const unsigned member = Base::fresh(thread), piece = member % 8, at = a.row[0] * kRowK + piece * (D / 16), group = a.row[0] * (D / AMSKV_KV4_GROUP);
    if constexpr (D == 64) {
      s.x[0][0] = *reinterpret_cast<const unsigned*>(k.k_codes + at);
      s.x[0][2] = *reinterpret_cast<const unsigned*>(k.v_codes + at);
      s.x[1][0] = *reinterpret_cast<const unsigned short*>(k.k_group + group);
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(k.k_codes + at), y = *reinterpret_cast<const u32x2*>(k.v_codes + at);
      s.x[0] = u32x4{x[0], x[1], y[0], y[1]};
      s.x[1][0] = *reinterpret_cast<const unsigned*>(k.k_group + group);
    }
    s.x[1][1] = k.v_group[group + piece * (D / 8) / AMSKV_KV4_GROUP];
  }
  __device__ static __forceinline__ void store_codes(const Staged& s, char* lds_all, int lds, int thread) {
    const unsigned member = Base::fresh(thread), row = member / 8, piece = member % 8;
    char* tile = lds_all + lds;
    *reinterpret_cast<unsigned*>(tile + kPowers + 32 * row + 4 * piece) = s.x[1][0];  // (eight times: no lane stands aside)
    const float by = power_of_byte(s.x[1][1]);
    if constexpr (D == 64) {
      *reinterpret_cast<unsigned*>(tile + row * kRowK + 16 * chunk_of_k(row, piece / 4) + 4 * (piece % 4)) = s.x[0][0];
      *reinterpret_cast<u32x4*>(tile + kOfK + row * RB + 16 * (piece ^ (unsigned)swizzle<D>((int)row))) = values4(s.x[0][2], by);
    } else {
      *reinterpret_cast<u32x2*>(tile + row * kRowK + 16 * chunk_of_k(row, piece / 2) + 8 * (piece % 2)) = u32x2{s.x[0][0], s.x[0][1]};
      char* v = tile + kOfK + row * RB;
      const unsigned at = 16 * ((2 * piece) ^ (unsigned)swizzle<D>((int)row));
      *reinterpret_cast<u32x4*>(v + at) = values4(s.x[0][2], by);
      *reinterpret_cast<u32x4*>(v + (at ^ 16)) = values4(s.x[0][3], by);
    }
  }
  // of a tile of either kind (found out uniformly)
  __device__ static __forceinline__ void aim_any(Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      aim_codes(a, k, seg, it, member);
    else
      Base::template aim<Base::kRowsOnly>(a, k, seg, it, member);
  }
  __device__ static __forceinline__ void fetch_any(Staged& s, const Aim& a, const Keys& k, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      fetch_codes(s, a, k, member);
    else
      Base::template fetch<Base::kRowsOnly>(s, a, k, it, member);
  }
  __device__ static __forceinline__ void store_any(const Staged& s, char* lds_all, int lds, const Keys& k, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      store_codes(s, lds_all, lds, member);
    else
      Base::template store<Base::kRowsOnly>(s, lds_all, lds, k, it, member);
  }

  // ---- scores.  K of 32 keys: lane (r, h) has channels 64 c + 32 h .. + 31 of key r.
  struct KeyCodes {
    u32x4 code[D / 64];
    unsigned powers;  // c's in byte 2 c
  };
  __device__ static __forceinline__ int k_lane4(int lane) { return (lane & 31) * kRowK + 16 * chunk_of_k(lane & 31, lane >> 5); }
  // block: of 32 keys inside the tile at `slot`
  __device__ static __forceinline__ void load_codes(KeyCodes& kc, const char* lds_all, int slot, int block, int ka, int kp, int lane) {
    const char* at = lds_all + slot + block * 32 * kRowK;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) kc.code[c] = *reinterpret_cast<const u32x4*>(at + (ka ^ (32 * c)));
    kc.powers = *reinterpret_cast<const unsigned*>(lds_all + slot + 32 * 32 * block + kp) >> (8 * (lane >> 5));
  }
  template <int kChunk>
  __device__ static __forceinline__ f32x16 multiply(const KeyCodes& kc, const Query& q, f32x16 s) {
    const u32x4& k = kc.code[kChunk];
    const i32x8 codes = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
    // (4: e2m1, 0: e4m3; the bytes of the powers are picked by constants)
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes, __builtin_bit_cast(i32x8, q.high[kChunk]), s, 4, 0, 2 * kChunk, kc.powers,
                                                        2 * kChunk, q.powers);
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes, __builtin_bit_cast(i32x8, q.low[kChunk]), s, 4, 0, 2 * kChunk, kc.powers,
                                                           2 * kChunk + 1, q.powers);
  }
  // S^T of these keys.  The products start from 0: started from the references, a block would save 16 multiply-adds of some 106 vector
  // instructions, but scores come out rounded at the size of a reference that may lie far from them.
  __device__ static __forceinline__ f32x16 product(const KeyCodes& kc, const Query& q) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    s = multiply<0>(kc, q, s);
    if constexpr (D == 128) s = multiply<1>(kc, q, s);
    return s;
  }
  // Unit::step in one basic block (as its kOneBlock): the first block, which has none before it, takes weights of 0 for what lies in its slot.
  template <bool kFull, class Between>
  __device__ static __forceinline__ void step_codes(Result& x, Behind& w, const KeyCodes& kc, const Query& q, const char* lds_all, int va, int block,
                                                    int n_valid, float c, int lane, Between between) {
    f32x16 s = product(kc, q);
    between();
    if constexpr (!kFull) Base::mask(s, n_valid, lane);
    if constexpr (Base::kAlone) __builtin_amdgcn_s_setprio(1);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      Base::add_values(x, w.pf[u], lds_all, w.block + va, u);
      sum += Base::weights(s, w.pf[u], c, x.ref, u);
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kTripSum)) != 0, 0)) {
      const float full = Base::largest(s, c), ref = full - x.ref > kMaxLag ? full : x.ref, alpha = __builtin_amdgcn_exp2f(x.ref - ref);
      x.ref = ref;
      x.sum *= alpha;
      Base::scale_by(x, alpha);
      sum = Base::weights(s, w.pf[0], c, ref, 0);
      sum += Base::weights(s, w.pf[1], c, ref, 1);
    }
    if constexpr (Base::kAlone) __builtin_amdgcn_s_setprio(0);
    x.sum += sum;
    w.block = block;
  }

  // Tiles [from, to) of the keys, as Unit::walk.  q_row(): the lane's row of Q, for rows of bf16 (asked for when it comes to them).
  template <class QueryRow>
  __device__ static __forceinline__ void walk(Result& x, const Query& q, QueryRow q_row, char* lds_all, const Keys& k, const SegTable& seg,
                                              int from, int to, float c, bool active) {
    int lane = threadIdx.x & 63, member = threadIdx.x;
    asm volatile("" : "+v"(lane));  // (not kept for what follows)
    const int t8 = min(Base::tiles_of_codes(k), to);
    int it = from;
    const int ka = k_lane4(lane);
    int va = Base::v_lane(lane) - Base::kTensor + kOfK, kp = kPowers + 32 * (lane & 31) + 4 * ((lane & 31) >> 3);
    asm volatile("" : "+v"(va), "+v"(kp));  // (a register each)
    Staged s;
    Aim to_come;
    auto load = [&](Staged& y, int i) {
      aim_any(to_come, k, seg, i, member);
      fetch_any(y, to_come, k, i, member);
    };
    if (it < to) load(s, it);
    {
      Staged s2;
      if (it + 1 < to) load(s2, it + 1);
      if (it < to) store_any(s, lds_all, 0, k, it, member);
      if (it + 1 < to) store_any(s2, lds_all, kStage, k, it + 1, member);
    }
    if (it + 2 < to) load(s, it + 2);
    __syncthreads();
    int slot = 0, next = kStage, after = 2 * kStage, spare = 3 * kStage;
    auto turn_over = [&]() {
      __syncthreads();
      if (it + 2 < to) {
        store_any(s, lds_all, after, k, it + 2, member);
        if (it + 3 < to) fetch_any(s, to_come, k, it + 3, member);
      }
    };
    auto next_tile = [&]() {
      const int freed = slot;
      slot = next;
      next = after;
      after = spare;
      spare = freed;
      ++it;
    };
    if (!active) {  // a wave without rows only brings its part of the tiles
      while (it < to) {
        if (it + 3 < to) aim_any(to_come, k, seg, it + 3, member);
        turn_over();
        next_tile();
      }
      return;
    }
    if (it >= to) return;
    Behind w;  // (rescale and first: never so here)
    w.alpha = 1.f;
    w.rescale = w.first = false;
    w.block = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) w.pf[u][e] = (__bf16)0.f;
    KeyCodes kc;
    if (it < t8) load_codes(kc, lds_all, slot, 0, ka, kp, lane);
    // tiles of which everything is known have no branch between their instructions
    while (it + 3 < t8) {
      aim_codes(to_come, k, seg, it + 3, member);
      if constexpr (kTile == 64)
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, c, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, kp, lane); });
      step_codes<true>(x, w, kc, q, lds_all, va, slot + (kTile - 32) * RB, 32, c, lane, [&]() {
        if constexpr (kTile == 32) __syncthreads();
        store_codes(s, lds_all, after, member);
        fetch_codes(s, to_come, k, member);
        if constexpr (kTile == 64) __syncthreads();
        load_codes(kc, lds_all, next, 0, ka, kp, lane);
      });
      next_tile();
    }
    while (it < t8) {
      asm volatile("" : "+v"(lane), "+v"(member));  // (what is derived from them is not kept from tile to tile: 12 registers, a spill at head dim 128)
      if (it + 3 < to) aim_any(to_come, k, seg, it + 3, member);
      int left = valid(k, it), done = 0;
      if (kTile == 64 && left > 32) {
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, c, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, kp, lane); });
        done = 32;
      }
      step_codes<false>(x, w, kc, q, lds_all, va, slot + done * RB, left - done, c, lane, [&]() {
        turn_over();
        if (it + 1 < t8) load_codes(kc, lds_all, next, 0, ka, kp, lane);
      });
      next_tile();
    }
    if constexpr (kExt) {
      if (it < to) {
        bf16x8 qf[KS], kf[KS];
        const char* row = q_row();
#pragma unroll
        for (int t = 0; t < KS; ++t) qf[t] = *reinterpret_cast<const bf16x8*>(row + 32 * t + 16 * (lane >> 5));
        Base::settle(qf);
        const int kr = Base::k_lane(lane);
        constexpr bool kAhead = Base::kAhead;
        if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr);
        while (it < to) {
          while (it + 3 < to && (it - 1 >= t8 || it == from)) {  // (Unit::walk: behind a tile of two blocks)
            Base::template aim<Base::kRowsOnly>(to_come, k, seg, it + 3, member);
            if constexpr (kTile == 64)
              Base::template step<true>(x, w, kf, qf, lds_all, kr, va, slot, 32, c, lane, [&]() {
                if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr + 32 * RB);
              });
            Base::template step<true>(x, w, kf, qf, lds_all, kr, va, slot + (kTile - 32) * RB, 32, c, lane, [&]() {
              if constexpr (kTile == 32) __syncthreads();
              Base::template store<Base::kRowsOnly>(s, lds_all, after, k, it + 2, member);
              Base::template fetch<Base::kRowsOnly>(s, to_come, k, it + 3, member);
              if constexpr (kTile == 64) __syncthreads();
              if constexpr (kAhead) Base::load_k(kf, lds_all, next + kr);
            });
            next_tile();
          }
          if (it + 3 < to) Base::template aim<Base::kRowsOnly>(to_come, k, seg, it + 3, member);
          int left = valid(k, it), done = 0;
          if (kTile == 64 && left > 32) {
            Base::template step<false>(x, w, kf, qf, lds_all, kr, va, slot, 32, c, lane, [&]() {
              if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr + 32 * RB);
            });
            done = 32;
          }
          Base::template step<false>(x, w, kf, qf, lds_all, kr, va, slot + done * RB, left - done, c, lane, [&]() {
            __syncthreads();
            if (it + 2 < to) {
              Base::template store<Base::kRowsOnly>(s, lds_all, after, k, it + 2, member);
              if (it + 3 < to) Base::template fetch<Base::kRowsOnly>(s, to_come, k, it + 3, member);
            }
            if (kAhead && it + 1 < to) Base::load_k(kf, lds_all, next + kr);
          });
          next_tile();
        }
        Base::finish(x, w, lds_all, va);
        return;
      }
    }
    Base::finish(x, w, lds_all, va);
  }
};

}  // namespace rows
}  // namespace amskv
#endif
