// Attention of up to 32 * kTeamWaves query rows over keys in 4 bits, for teams of waves: attend_rows.hpp's formulation with K's codes as
// they are.
//
// The matrix cores take e2m1 numbers with a power of two to every 32 along the sum: S^T = K Q^T is formed by
// v_mfma_scale_f32_32x32x64_f8f6f4 from K's codes and powers straight out of LDS, a quarter of bf16's bytes there and no conversion.  Its
// other operand may have 6 bits without loss of speed (4 times bf16's rate; 8 bits: twice), so y = q times the factor of the scores is held
// as the sum of two e2m3 numbers (4 significant bits each), made once for a workgroup: 32 channels with largest element m, 2^a the least
// power with m <= 7.5 * 2^a, are hi * 2^a + lo * 2^(a - 5), hi the number nearest to y * 2^-a, lo nearest to what is left.  hi's step is
// 1/2 from 4 on, 1/4 from 2 on and 1/8 below, which leaves up to 8, 4 and 2 for lo: y is off by at most 2^(a - 8) from 2 * 2^a on and 2^(a
// - 9) below; from 4 * 2^a on by 2^(a - 7), and up to 2^(a - 6) where lo would be 7.75 to 8 and is 7.5 (one of 32; a bf16 number itself
// stands for what lies within 2^(a - 6) there).  lo at 2^(a - 4) has no such end, but steps twice as wide for all others: over normal
// values y is off by 0.0008 of its size (rms) as it is here, 0.0011 as it would be there, with gains from channel to channel of e^(0.5
// normal) 0.0009 and 0.0015.  Two products at 4 times the rate: half of the time of bf16's (15.4 ns of a SIMD each for 64 channels, bf16
// 73.6; e4m3 parts 28.6 each; a third part at head dim 128, 64 units 4096 x 6421, 584 -> 651 us).  V becomes bf16 on its way to LDS, once
// for all waves: weights in 6 bits would have to be split in two for every block, which takes the vector ALUs more (a conversion of 32
// numbers 38 ns, back 33) than the matrix cores save.
//
// Bound, and what it measured.  Head dim 128, 64 units: the matrix pipes and the power they take, 4096 x 6421 by teams of eight 576 to 601
// us (1.43 to 1.50 PFLOP/s; codes of 8 bits through bf16 784), 2304 x 3925 by teams of four 234 to 255, 576 x 1076 29.  Head dim 64, 3840
// units: the vector ALUs (0.66 of a SIMD's cycles, the matrix pipe 0.20), 256 x 530 174 to 181 us (with 256 of the keys read in place as
// bf16, by attend_rows.hpp, 195 to 201), x 2066 481 to 503 (1.03 to 1.08 PFLOP/s).
//
// kExt: rows of bf16 may follow the codes (a scale that is read in place); they are walked as in attend_rows.hpp, with Q as it is.
#pragma once
#include "attend_rows.hpp"

#if defined(__HIPCC__)
namespace amskv {
namespace rows {

typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Q of a lane times the factor of its scores: channels 64 c + 32 h .. + 31 of its row in two parts, the larger first, and the bytes of
// their powers.
constexpr int kParts = 2;
template <int D>
struct QueryParts {
  u32x6 part[D / 64][kParts];
  unsigned powers[D / 64];
};
// 32 numbers as e2m3 times a power of two, even and odd ones by turns, and back.  Written out: the conversions write their first results
// before they have read all operands, and the compiler's own may let the two overlap, which gave wrong parts of Q in some builds.  (The
// wait is for what reads the results: the compiler does not see into inline assembly.)
__device__ __forceinline__ u32x6 parts_of(const f32x16& even, const f32x16& odd, float by) {
  u32x6 r;
  asm("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 7" : "=&v"(r) : "v"(even), "v"(odd), "v"(by));
  return r;
}
__device__ __forceinline__ f32x32 values_of(const u32x6& x, float by) {
  f32x32 r;
  asm("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 7" : "=&v"(r) : "v"(x), "v"(by));
  return r;
}
// (Q is asked for before anything that has to be waited for)
template <int D>
__device__ __forceinline__ void load_query(u32x4 (&raw)[D / 64][4], const char* row, int h) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[c][i] = *reinterpret_cast<const u32x4*>(row + 128 * c + 64 * h + 16 * i);
}
template <int D>
__device__ __forceinline__ void split_query(QueryParts<D>& q, const u32x4 (&raw)[D / 64][4], float factor) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    f32x16 even, odd;
    u16x2 most = {0, 0};  // the bits of the largest magnitudes
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] = __builtin_bit_cast(float, raw[c][i / 4][i % 4] << 16) * factor;
      odd[i] = __builtin_bit_cast(float, raw[c][i / 4][i % 4] & 0xffff0000u) * factor;
      m = max3(m, __builtin_fabsf(even[i]), __builtin_fabsf(odd[i]));
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, raw[c][i / 4][i % 4] & 0x7fff7fffu));
    }
    const bool finite = max(most[0], most[1]) < 0x7f80;
    const int bits = __builtin_bit_cast(int, m);  // 7.5 = 1.875 * 2^2
    const int a = min(max((bits >> 23) - 127 - 2 + ((bits & 0x7fffff) > 0x700000 ? 1 : 0), -110), 126);
    q.powers[c] = 0;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
      const int byte = a - 5 * p + 127;
      const float by = power_of_byte(byte);
      q.powers[c] |= (unsigned)(finite ? byte : 255) << (8 * p);  // (255: NaN, which is what all scores of the row become)
      q.part[c][p] = parts_of(even, odd, by);
      if (p + 1 < kParts) {
        const f32x32 held = values_of(q.part[c][p], by);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          even[i] -= held[2 * i];
          odd[i] -= held[2 * i + 1];
        }
      }
    }
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
  // scores times the factor
  template <int kPart, int kChunk>
  __device__ static __forceinline__ f32x16 multiply(const KeyCodes& kc, const Query& q, const f32x16& add) {
    const u32x4& k = kc.code[kChunk];
    const u32x6& x = q.part[kChunk][kPart];
    // (4: e2m1, 2: e2m3; the bytes of the powers are picked by constants)
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(i32x8{(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0},
                                                           i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0}, add, 4, 2,
                                                           2 * kChunk, kc.powers, kPart, q.powers[kChunk]);
  }
  __device__ static __forceinline__ f32x16 product(const KeyCodes& kc, const Query& q) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    s = multiply<0, 0>(kc, q, s);
    s = multiply<1, 0>(kc, q, s);
    if constexpr (D == 128) {
      s = multiply<0, 1>(kc, q, s);
      s = multiply<1, 1>(kc, q, s);
    }
    return s;
  }
  // Unit::step in one basic block (as its kOneBlock): the first block, which has none before it, takes weights of 0 for what lies in its slot.
  // The products start from 0: started from the references, a block would save 16 multiply-adds of some 106 vector instructions, but
  // scores come out rounded at the size of a reference that may lie far from them.
  template <bool kFull, class Between>
  __device__ static __forceinline__ void step_codes(Result& x, Behind& w, const KeyCodes& kc, const Query& q, const char* lds_all, int va, int block,
                                                    int n_valid, int lane, Between between) {
    f32x16 s = product(kc, q);
    between();
    if constexpr (!kFull) Base::mask(s, n_valid, lane);
    if constexpr (Base::kAlone) __builtin_amdgcn_s_setprio(1);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      Base::add_values(x, w.pf[u], lds_all, w.block + va, u);
      sum += Base::weights(s, w.pf[u], 1.f, x.ref, u);
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kTripSum)) != 0, 0)) {
      const float full = Base::largest(s, 1.f), ref = full - x.ref > kMaxLag ? full : x.ref, alpha = __builtin_amdgcn_exp2f(x.ref - ref);
      x.ref = ref;
      x.sum *= alpha;
      Base::scale_by(x, alpha);
      sum = Base::weights(s, w.pf[0], 1.f, ref, 0);
      sum += Base::weights(s, w.pf[1], 1.f, ref, 1);
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
    const int ka = k_lane4(lane), va = Base::v_lane(lane) - Base::kTensor + kOfK;
    int kp = kPowers + 32 * (lane & 31) + 4 * ((lane & 31) >> 3);
    asm volatile("" : "+v"(kp));  // (one register)
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
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, kp, lane); });
      step_codes<true>(x, w, kc, q, lds_all, va, slot + (kTile - 32) * RB, 32, lane, [&]() {
        if constexpr (kTile == 32) __syncthreads();
        store_codes(s, lds_all, after, member);
        fetch_codes(s, to_come, k, member);
        if constexpr (kTile == 64) __syncthreads();
        load_codes(kc, lds_all, next, 0, ka, kp, lane);
      });
      next_tile();
    }
    while (it < t8) {
      if (it + 3 < to) aim_any(to_come, k, seg, it + 3, member);
      int left = valid(k, it), done = 0;
      if (kTile == 64 && left > 32) {
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, kp, lane); });
        done = 32;
      }
      step_codes<false>(x, w, kc, q, lds_all, va, slot + done * RB, left - done, lane, [&]() {
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
